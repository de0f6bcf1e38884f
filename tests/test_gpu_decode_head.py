"""The vocabulary projection's calls as the decoder runs them: a drafter fitted to its target
through the loss's gradients, then drafting with its head in 8-bit integers."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as H

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def mods():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_15371_amd import cmsd, decode, pipeline
    return cmsd, decode, pipeline


def _models(decode, V, d, seed, noise):
    target = decode.TinyLM(V, d=d, seed=seed).to(DEV)
    return target, target.perturbed(noise, seed + 1).to(DEV)


def test_fit_gradients_are_the_models(mods):
    # every parameter's gradient of one fitting step against autograd of the mean cross entropy
    # in float64 through the whole model.  Both are sums of up to 4e4 products and a chain of
    # some 20 operations in float32, whose roundings (2^-24 each) add up to under 1e-4 of the
    # largest entry where the conditioning is that of a layer norm over 48 values
    _, decode, _ = mods
    target, drafter = _models(decode, 700, 48, 51, 0.3)
    fit = decode.DrafterFit(drafter, target, B=3, T=9, seed=5)
    tok, labels = fit.batch()
    labels[4] = -1                                            # a position without a label
    loss = fit.gradients(tok, labels).clone()
    exact = decode.TinyLM(700, d=48, seed=0).to(DEV).double()
    exact.load_state_dict(drafter.state_dict())
    z = exact.scale * (exact.hidden(tok) @ exact.out)
    ref = torch.nn.functional.cross_entropy(z.view(-1, 700), torch.where(labels < 0, 0, labels).long(), reduction="none")
    ref = torch.where(labels < 0, 0.0, ref)
    (ref.sum() / len(labels)).backward()
    assert float((loss.double() - ref.detach()).abs().max()) < 1e-4 * float(ref.detach().abs().max())
    pairs = [("out", fit.weight.grad.t(), exact.out.grad)]
    pairs += [(n, p.grad, dict(exact.named_parameters())[n].grad) for n, p in drafter.named_parameters() if n != "out"]
    assert len(pairs) == 3 + 4 * len(drafter.layers)
    for name, got, want in pairs:
        far = float((got.double() - want).abs().max() / want.abs().max())
        assert far < 1e-4, (name, far)


@pytest.mark.parametrize("trunk", [True, False])
def test_fit_steps_run(mods, trunk):
    _, decode, _ = mods
    target, drafter = _models(decode, 900, 64, 61, 0.2)
    before = {n: p.detach().clone() for n, p in drafter.named_parameters()}
    fit = decode.DrafterFit(drafter, target, B=4, T=16, seed=6, trunk=trunk)
    for _ in range(3):
        loss = fit.step()
        assert loss.shape == (64,) and bool(torch.isfinite(loss).all())
    for n, p in drafter.named_parameters():
        assert bool(torch.isfinite(p).all())
        assert torch.equal(p, before[n]) == (not trunk and n != "out"), n
    assert torch.equal(drafter.out, fit.weight.t())


def test_head8_rows_are_the_oracles(mods):
    # the drafter's logit rows by the quantised head, written into the decoder's strided rows
    _, decode, _ = mods
    target, drafter = _models(decode, 1003, 64, 71, 0.2)
    drafter.use_head8(5)
    tok = torch.randint(0, 1003, (5, 12), generator=torch.Generator().manual_seed(1)).to(DEV)
    pos = torch.tensor([3, 11, 0, 7, 5], device=DEV)
    dl = torch.full((5, 4, 1003), -3.0, device=DEV)
    drafter.head_rows(tok, pos, dl[:, 2])
    with torch.no_grad():
        h = drafter.hidden(tok)[torch.arange(5, device=DEV), pos]
    c, s = H.quantize_rows(h.double().cpu().numpy())
    wc, ws = H.quantize_rows(drafter.out.detach().t().double().cpu().numpy())
    ref = H.head_logits(c, s, wc, ws, float(np.float32(drafter.scale)))
    got = dl[:, 2].double().cpu().numpy()
    assert (np.abs(got - ref) <= np.abs(ref) * 5 * 2.0 ** -24 * 1.0001).all()
    assert bool((dl[:, [0, 1, 3]] == -3.0).all())
    # near the head's own rows: a code stands for values half a step around it, so a product's
    # error is at most half a step of either side for each of the 64 terms, and their product
    with torch.no_grad():
        z = (drafter.scale * (h @ drafter.out)).double().cpu().numpy()
    hh, ww = np.abs(h.double().cpu().numpy()), np.abs(drafter.out.detach().t().double().cpu().numpy())
    sd, wd = s.astype(np.float64)[:, None], ws.astype(np.float64)[:, None]
    bound = drafter.scale * (0.5 * sd * ww.sum(1)[None, :] + 0.5 * hh.sum(1)[:, None] * wd.T + 16 * sd * wd.T)
    assert (np.abs(got - z) <= bound * 1.001 + 1e-4).all()


def test_fitted_head8_drafter_stays_lossless(mods):
    # fit, quantise, decode: exact-match verification still emits the target's greedy tokens,
    # whatever the drafter (positions whose two best logits are within 1e-4 may round
    # differently between forward shapes and end a sequence's comparison)
    cmsd, decode, pipeline = mods
    V, B, K, n_new = 5000, 6, 5, 24
    target, drafter = _models(decode, V, 128, 81, 0.1)
    fit = decode.DrafterFit(drafter, target, B=8, T=32, seed=8)
    for _ in range(2):
        fit.step()
    drafter.use_head8(B)
    prompt = torch.randint(0, V, (B, 10), generator=torch.Generator().manual_seed(9)).to(DEV)
    prm = pipeline.Params(mode=cmsd.CMSD_MODE_GREEDY, top_beta=0)
    out = decode.SpeculativeDecoder(target, drafter, B, K, prm, DEV).generate(prompt, n_new)
    ref, gaps = decode.greedy_reference(target, prompt, n_new)
    for b in range(B):
        for j in range(n_new):
            if gaps[j][b] < 1e-4:
                break
            assert out[b][j] == ref[b][j], (b, j)


@pytest.mark.parametrize("mode", [0, 1])
def test_head8_iterations_match_the_oracle(mods, mode):
    # the rows of the quantised head go on through the sampler, the confidences and the
    # verification: each checked against the oracle on the rows as they are
    from oracle import cmsd_oracle as O
    from tests import parity as Pa
    cmsd, decode, pipeline = mods
    V, B, K = 3000, 5, 4
    target, drafter = _models(decode, V, 64, 91 + mode, 0.15)
    drafter.use_head8(B)
    prm = pipeline.Params(mode=mode)
    dec = decode.SpeculativeDecoder(target, drafter, B, K, prm, DEV, seed=mode)
    tok = torch.zeros((B, 40), dtype=torch.long, device=DEV)
    tok[:, :8] = torch.randint(0, V, (B, 8), generator=torch.Generator().manual_seed(mode)).to(DEV)
    lens = torch.full((B,), 8, dtype=torch.long, device=DEV)
    P = {"lambdas": prm.lambdas, "beta_margin": prm.beta_margin, "k_min": prm.k_min, "alpha": prm.alpha,
         "top_beta": prm.top_beta, "tau_base": prm.tau_base, "gamma": prm.gamma}
    lam, bm = tuple(Pa.f32(x) for x in prm.lambdas), Pa.f32(prm.beta_margin)
    for _ in range(2):
        rec = []
        dec.step(tok, lens, record=rec)
        r, t = rec[0], Pa.Tally()
        gs = Pa.stats_fields(r["stats"].numpy(), r["stats"].view(torch.int32).numpy())
        ts = Pa.tstats_fields(r["tstats"].numpy(), r["tstats"].view(torch.int32).numpy())
        draft, rows = r["draft"].double().numpy(), r["target"].double().numpy()
        for b in range(B):
            C = []
            for i in range(K):
                rs = Pa.check_row_stats(t, gs, b * K + i, draft[b, i], V, lam, bm)
                C.append(O.confidence(rs, V, lam, bm))
                y, sl = O.draft_sample(draft[b, i], float(r["draft_u"][b, i]))
                t.decision(f"drafted[{b},{i}]", int(r["drafted"][b, i]), y, sl)
            kb, o = int(r["k"][b]), int(r["off"][b])
            unif = [float(x) for x in r["unif"][o:o + kb + 1]]
            Pa.check_sequence(t, b, [rows[o + i] for i in range(kb + 1)], [draft[b, i] for i in range(K)],
                              r["drafted"][b].numpy(), unif, C, kb, mode, P, ts, o, int(r["n_acc"][b]),
                              int(r["next"][b]))
        t.assert_ok()
