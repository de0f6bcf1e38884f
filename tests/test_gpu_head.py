"""The vocabulary projection's calls on the GPU against the float64 oracle, through the C ABI.

Every bound is what the roundings of the computation can add up to:
  - a sum of K products in single precision is off by at most K + 4 roundings (2^-23 each: the
    matrix cores may truncate) of the sum of the products' magnitudes;
  - storing a value rounds it by UNIT of its type;
  - exp2, log and a softmax's share each add a few roundings, counted at their place.
"""
import numpy as np
import pytest
import torch

from oracle import head_oracle as H

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
E = 2.0 ** -23
DEV = "cuda:0"


@pytest.fixture(scope="module")
def cm():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_15371_amd import cmsd
    return cmsd


def padded(n, w, pad, dtype, fill, offset=0):
    """A [n, w] view at row stride w + pad, `offset` elements into its memory, all `fill`."""
    flat = torch.full((offset + max(n, 1) * (w + pad),), fill, dtype=dtype, device=DEV)
    return flat[offset:].view(max(n, 1), w + pad)[:n, :w], flat


def gaps_left(flat, n, w, pad, fill, offset=0):
    """Whether nothing between the rows was written."""
    g = flat[offset:].view(-1, w + pad)[:, w:]
    return bool((g == fill).all()) and bool((flat[:offset] == fill).all())


def put(x, dtype, pad=0, offset=0):
    v, _ = padded(x.shape[0], x.shape[1], pad, dtype, 0, offset)
    v.copy_(torch.from_numpy(x).to(dtype))
    return v


def host(t):
    return t.detach().double().cpu().numpy()


def within(got, ref, bound, what):
    far = np.abs(got - ref)
    ok = far <= bound
    assert ok.all(), (what, int((~ok).sum()), float(np.nanmax(far / np.maximum(bound, 1e-300))), np.argwhere(~ok)[:3])


# ------------------------------------------------------------------------------- quantisation
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,w,pad,offset", [(1, 1, 0, 0), (3, 7, 0, 0), (2, 64, 0, 0), (5, 255, 9, 1), (4, 1000, 24, 0),
                                            (3, 2048, 0, 0), (2, 4097, 0, 3), (2, 8192, 8, 0), (2, 20000, 0, 0),
                                            (300, 256, 0, 0), (1, 131071, 0, 0)])
def test_quantize_rows(cm, dtype, n, w, pad, offset):
    g = np.random.default_rng(n * w + pad)
    x = put(g.normal(size=(n, w)) * np.exp(g.normal(size=(n, 1)) * 4), dtype, pad, offset)
    codes, flat = padded(n, w, pad, torch.int8, 77, offset)
    _, scales = cm.cmsd_quantize_rows(x, codes)
    want, want_scales = H.quantize_rows(host(x))
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    assert np.array_equal(codes.cpu().numpy(), want)
    assert gaps_left(flat, n, w, pad, 77, offset)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantize_special_rows(cm, dtype):
    w = 300
    x = np.zeros((8, w))
    x[1, 17] = 2.0 ** -133                   # / 127 rounds to zero in single precision? (2^-140: no)
    x[2, :3] = [1.0, np.inf, -2.0]
    x[3, 299] = np.nan
    x[4, :] = 127.0
    x[4, :6] = [0.5, 1.5, 2.5, -0.5, -1.5, -2.5]    # ties go to the even code
    x[5, 8] = -3.0e38
    x[6, 3] = -np.inf
    x[7, 0] = 2.0 ** -126
    t = put(x, dtype)
    codes, scales = cm.cmsd_quantize_rows(t)
    want, want_scales = H.quantize_rows(host(t))
    assert np.array_equal(scales.cpu().numpy(), want_scales, equal_nan=True)
    assert np.array_equal(codes.cpu().numpy(), want)
    assert list(codes.cpu().numpy()[4, :6]) == [0, 2, 2, 0, -2, -2]


# ------------------------------------------------------------------------------- the product
SHAPES = [  # rows, vocabulary, width
    (1, 2, 1), (1, 1000, 64), (2, 33, 16), (3, 65, 17), (5, 4000, 768), (16, 1024, 256), (17, 129, 100), (33, 300, 4096),
    (64, 512, 768), (70, 333, 1000), (130, 257, 64), (200, 1000, 320), (256, 256, 128), (260, 515, 2048), (513, 770, 144),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,w", SHAPES)
@pytest.mark.parametrize("pad,offset", [(0, 0), (16, 0), (5, 3)])
def test_head_logits(cm, dtype, n, v, w, pad, offset):
    g = np.random.default_rng(n + v + w)
    h, wt = g.integers(-128, 128, (n, w)).astype(np.int8), g.integers(-128, 128, (v, w)).astype(np.int8)
    sh, sw = (g.random(n) + 0.5).astype(np.float32), (g.random(v) + 0.5).astype(np.float32)
    out, flat = padded(n, v, pad, dtype, -7.0, offset)
    cm.cmsd_head_logits(put(h, torch.int8, pad, offset), torch.from_numpy(sh).to(DEV), put(wt, torch.int8, pad, offset),
                        torch.from_numpy(sw).to(DEV), out, scale=0.37)
    ref = H.head_logits(h, sh, wt, sw, float(np.float32(0.37)))
    # the whole sum to float, scale by scale, and two products: four roundings, then the store's
    within(host(out), ref, np.abs(ref) * (4 * 2.0 ** -24 + UNIT[dtype]) * 1.0001, (n, v, w))
    assert gaps_left(flat, n, v, pad, -7.0, offset)


def test_head_logits_reports_a_bad_row(cm):
    x = torch.randn(5, 64, device=DEV)
    x[2, 5] = float("nan")
    x[4, 0] = float("inf")
    c, s = cm.cmsd_quantize_rows(x)
    wc, ws = cm.cmsd_quantize_rows(torch.randn(100, 64, device=DEV))
    z = cm.cmsd_head_logits(c, s, wc, ws)
    assert torch.isnan(z).all(1).tolist() == [False, False, True, False, True]
    assert torch.isfinite(z[[0, 1, 3]]).all()


# ------------------------------------------------------------------------------- the loss
def problem(seed, n, v, w, dtype, pad=0, offset=0, scale=1.0, lean=6.0):
    """Hidden rows that lean towards their label, weight, labels (one in eight negative)."""
    g = np.random.default_rng(seed)
    wt = g.normal(size=(v, w)) / np.sqrt(w)
    y = g.integers(0, v, n).astype(np.int32)
    h = g.normal(size=(n, w)) + lean / max(1.0, abs(scale)) * g.random((n, 1)) * wt[y]
    if n > 1:
        y[g.random(n) < 0.125] = -1 - int(g.integers(0, 100))
    ht, wtt = put(h, dtype, pad, offset), put(wt, dtype, pad, offset)
    return ht, wtt, torch.from_numpy(y).to(DEV), host(ht), host(wtt), y, (g.random(n) * 2 - 0.5).astype(np.float32)


def loss_bounds(z, size, lse, w, scale):
    """How far a logit, and a row's lse, may be off."""
    at_z = size * ((w + 4) * E) + np.abs(z) * E
    # lse: its largest logit's error; exp2 of a rounded argument (2 roundings of up to the
    # row's spread, weighted by e^-x: under 2), exp2 itself, and sums in under 64 roundings;
    # the logarithm's and the last sum's
    at_lse = at_z.max(1) + 70 * E + 4 * E * np.abs(lse)
    return at_z, at_lse


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,w", SHAPES)
@pytest.mark.parametrize("pad,offset,scale", [(0, 0, 1.0), (8, 0, 5.0), (5, 3, -0.5)])
def test_head_loss(cm, dtype, n, v, w, pad, offset, scale):
    h, wt, y, hh, ww, yy, _ = problem(n + v + w, n, v, w, dtype, pad, offset, scale)
    loss, lse = cm.cmsd_head_loss(h, wt, y, scale=scale)
    ref, ref_lse, z, size = H.head_loss(hh, ww, yy, scale)
    at_z, at_lse = loss_bounds(z, size, ref_lse, w, scale)
    within(host(lse), ref_lse, at_lse, "lse")
    within(host(loss), ref, at_lse + at_z.max(1) + E * np.abs(ref), "loss")
    assert (host(loss)[yy < 0] == 0).all()


def test_head_loss_labels_and_extremes(cm):
    h, wt, y, hh, ww, yy, _ = problem(1, 40, 200, 96, F32)
    y[3], y[4], y[5] = 200, 2 ** 31 - 1, -2 ** 31
    loss, lse = cm.cmsd_head_loss(h, wt, y)
    assert torch.isnan(loss[3:5]).all() and loss[5] == 0 and torch.isfinite(lse).all()
    rest = [i for i in range(40) if i not in (3, 4)]
    assert torch.isfinite(loss[rest]).all()
    # logits of +-1e4: shares whose sums vanish beside the largest; a NaN and an overflowing row
    # (their own losses only); the first and the last entry as labels
    h = torch.zeros(5, 96, device=DEV)
    h[:, 0] = torch.tensor([1e4, -1e4, 0.0, float("nan"), 3e38])
    wt = torch.zeros(200, 96, device=DEV)
    wt[:, 0] = torch.linspace(-1, 1, 200, device=DEV)
    wt[199, 0] = 10.0
    y = torch.tensor([199, 0, 0, 1, 1], dtype=torch.int32, device=DEV)
    loss, lse = cm.cmsd_head_loss(h, wt, y)
    ref, ref_lse, _, _ = H.head_loss(host(h[:3]), host(wt), [199, 0, 0], 1.0)
    assert np.allclose(host(lse[:3]), ref_lse, rtol=1e-6) and np.allclose(host(loss[:3]), ref, rtol=1e-6, atol=2e-3)
    assert not torch.isfinite(loss[3:]).any()


# ------------------------------------------------------------------------------- the gradients
def grad_bounds(hh, ww, yy, gl, scale, dtype, w):
    """References and bounds of both gradients."""
    gh, _, gw, _, d, p = H.head_loss_grad(hh, ww, yy, gl, scale)
    _, lse, z, size = H.head_loss(hh, ww, yy, scale)
    at_z, at_lse = loss_bounds(z, size, lse, w, scale)
    # a probability: its exponent's error and exp2's own; times g * scale (2 roundings), and
    # the rounding to the products' type
    counts = ((yy >= 0) & (yy < ww.shape[0]))[:, None]
    g = np.abs(gl * scale)[:, None]
    at_p = p * (np.exp(at_z + at_lse[:, None] + 4 * E * (np.abs(z) + np.abs(lse)[:, None])) - 1 + 4 * E)
    at_d = np.where(counts, at_p * g * (1 + E) + np.abs(d) * (3 * E + UNIT[dtype]), 0) + 2.0 ** -133
    ad = np.abs(d) + at_d
    # sums of single precision (in up to 64 parts)
    at_gh = at_d @ np.abs(ww) + (ad @ np.abs(ww)) * (ww.shape[0] + 70) * E
    at_gw = at_d.T @ np.abs(hh) + (ad.T @ np.abs(hh)) * (len(hh) + 70) * E
    return (gh, at_gh + np.abs(gh) * UNIT[dtype] * 1.01 + 2.0 ** -133), (gw, at_gw + np.abs(gw) * UNIT[dtype] * 1.01 + 2.0 ** -133)


GRAD_SHAPES = SHAPES + [(1, 5000, 64), (3000, 40, 64), (2500, 300, 72), (9, 9000, 200), (1100, 1030, 257)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,w", GRAD_SHAPES)
@pytest.mark.parametrize("pad,offset,scale", [(0, 0, 1.0), (8, 0, 5.0), (5, 3, -0.5)])
def test_head_loss_grad(cm, dtype, n, v, w, pad, offset, scale):
    h, wt, y, hh, ww, yy, gl = problem(n + v + w, n, v, w, dtype, pad, offset, scale)
    glt = torch.from_numpy(gl).to(DEV)
    _, lse = cm.cmsd_head_loss(h, wt, y, scale=scale)
    gh, fh = padded(n, w, pad, dtype, -7.0, offset)
    gw, fw = padded(v, w, pad, dtype, -7.0, offset)
    cm.cmsd_head_loss_grad(h, wt, y, lse, glt, gh, gw, scale=scale)
    (rh, bh), (rw, bw) = grad_bounds(hh, ww, yy, gl.astype(np.float64), scale, dtype, w)
    within(host(gh), rh, bh, "grad_hidden")
    within(host(gw), rw, bw, "grad_weight")
    assert gaps_left(fh, n, w, pad, -7.0, offset) and gaps_left(fw, v, w, pad, -7.0, offset)
    assert (host(gh)[yy < 0] == 0).all()
    # each alone: the same values
    gh1, gw1 = torch.empty_like(gh), torch.empty_like(gw)
    cm.cmsd_head_loss_grad(h, wt, y, lse, glt, grad_hidden=gh1, scale=scale)
    cm.cmsd_head_loss_grad(h, wt, y, lse, glt, grad_weight=gw1, scale=scale)
    assert torch.equal(gh1, gh) and torch.equal(gw1, gw)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_grad_pieces_of_the_vocabulary(cm, dtype):
    # enough rows that the vocabulary takes several pieces, the last one ragged
    n, v, w = (33000, 9001, 16) if dtype == BF16 else (17000, 9001, 16)
    h, wt, y, hh, ww, yy, gl = problem(5, n, v, w, dtype)
    assert cm.cmsd_head_loss_grad_workspace_bytes(n, v, w, dtype) < n * v * h.element_size()
    _, lse = cm.cmsd_head_loss(h, wt, y)
    gh, gw = torch.empty_like(h), torch.empty_like(wt)
    cm.cmsd_head_loss_grad(h, wt, y, lse, torch.from_numpy(gl).to(DEV), gh, gw)
    hd, wd = h.double(), wt.double()
    p = torch.softmax(hd @ wd.t().contiguous(), 1)
    keep = y >= 0
    p[keep, y[keep].long()] -= 1
    p *= torch.where(keep, torch.from_numpy(gl).to(DEV).double(), 0.0)[:, None]
    u = UNIT[dtype]
    for got, ref, size, k in ((gh, p @ wd, p.abs() @ wd.abs(), v), (gw, p.t().contiguous() @ hd, p.t().abs().contiguous() @ hd.abs(), n)):
        # as in grad_bounds, with 2e-5 for a probability's exponent (|z| and lse under 30)
        bound = size * (u + 2e-5 + (k + 70) * E) + ref.abs() * u * 1.01 + 1e-30
        far = ((got.double() - ref).abs() / bound).max()
        assert far <= 1, float(far)


def _on_gpu(h, wt, y, gl, scale, dtype):
    """grad_bounds' references and bounds, and the loss's, formed on the GPU in float64."""
    hd, wd = h.double(), wt.double()
    keep = (y >= 0)[:, None]
    z = scale * (hd @ wd.t().contiguous())
    size = abs(scale) * (hd.abs() @ wd.abs().t().contiguous())
    lse = torch.logsumexp(z, 1, keepdim=True)
    at_z = size * ((h.shape[1] + 4) * E) + z.abs() * E
    at_lse = at_z.amax(1, keepdim=True) + 70 * E + 4 * E * lse.abs()
    loss = torch.where(keep, lse - torch.gather(z, 1, y.long().clamp(min=0)[:, None]), 0.0)
    p = torch.exp(z - lse)
    g = gl.double()[:, None] * scale
    at_p = p * (torch.expm1(at_z + at_lse + 4 * E * (z.abs() + lse.abs())) + 4 * E)
    d = p.scatter_add(1, y.long().clamp(min=0)[:, None], torch.full_like(lse, -1.0)) * g * keep
    at_d = (at_p * g.abs() * (1 + E) + d.abs() * (3 * E + UNIT[dtype])) * keep + 2.0 ** -133
    ad = d.abs() + at_d
    gh, gw = d @ wd, d.t().contiguous() @ hd
    at_gh = at_d @ wd.abs() + (ad @ wd.abs()) * ((len(wt) + 70) * E) + gh.abs() * UNIT[dtype] * 1.01 + 2.0 ** -133
    at_gw = at_d.t().contiguous() @ hd.abs() + (ad.t().contiguous() @ hd.abs()) * ((len(h) + 70) * E) \
        + gw.abs() * UNIT[dtype] * 1.01 + 2.0 ** -133
    return (loss[:, 0], (at_lse + at_z.amax(1, keepdim=True) + E * loss.abs())[:, 0]), (lse[:, 0], at_lse[:, 0]), \
        (gh, at_gh), (gw, at_gw)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,w,pad", [(700, 17000, 64, 0), (3300, 600, 4096, 0), (300, 13000, 1024, 8),
                                       (4100, 13001, 264, 0), (1024, 50257, 8, 0), (32, 50000, 136, 0),
                                       (50, 30001, 520, 8), (400, 2000, 1000, 0), (60, 4001, 320, 0),
                                       (90, 15000, 136, 3), (260, 9000, 129, 0)])
def test_every_tile_of_the_products(cm, dtype, n, v, w, pad):
    # extents that take the largest tiles in one product or another, and ragged ones in all
    h, wt, y, _, _, _, gl = problem(n, n, v, w, dtype, pad)
    gl = torch.from_numpy(gl).to(DEV)
    loss, lse = cm.cmsd_head_loss(h, wt, y, scale=1.5)
    gh, fh = padded(n, w, pad, dtype, -7.0)
    gw, fw = padded(v, w, pad, dtype, -7.0)
    cm.cmsd_head_loss_grad(h, wt, y, lse, gl, gh, gw, scale=1.5)
    for got, (ref, bound), what in zip((loss, lse, gh, gw), _on_gpu(h, wt, y, gl, 1.5, dtype),
                                       ("loss", "lse", "grad_hidden", "grad_weight")):
        far = float(((got.double() - ref).abs() / bound).max())
        assert far <= 1, (what, far)
    assert gaps_left(fh, n, w, pad, -7.0) and gaps_left(fw, v, w, pad, -7.0)
    c, s = cm.cmsd_quantize_rows(h)
    wc, ws = cm.cmsd_quantize_rows(wt)
    z = cm.cmsd_head_logits(c, s, wc, ws, dtype=dtype)
    ref = (c.double() @ wc.double().t().contiguous()) * s[:, None].double() * ws.double()
    assert bool(((z.double() - ref).abs() <= ref.abs() * (4 * 2.0 ** -24 + UNIT[dtype]) * 1.0001).all())


def test_gradient_against_differences_of_the_loss(cm):
    n, v, w, scale = 6, 500, 64, 2.0
    h, wt, y, _, _, yy, gl = problem(9, n, v, w, F32, scale=scale)
    y[:] = torch.arange(n, dtype=torch.int32, device=DEV) * 37
    glt = torch.from_numpy(np.abs(gl) + 0.5).to(DEV)
    _, lse = cm.cmsd_head_loss(h, wt, y, scale=scale)
    gh, gw = torch.empty_like(h), torch.empty_like(wt)
    cm.cmsd_head_loss_grad(h, wt, y, lse, glt, gh, gw, scale=scale)

    def total(h, wt):
        return float((cm.cmsd_head_loss(h, wt, y, scale=scale)[0].double() * glt.double()).sum())

    eps = 2.0 ** -5
    g = torch.Generator(device=DEV).manual_seed(3)
    for grad, x, f in ((gh, h, lambda x: total(x, wt)), (gw, wt, lambda x: total(h, x))):
        d = torch.randn(x.shape, generator=g, device=DEV)
        a, b = (x + eps * d), (x - eps * d)
        # the logits' change per unit step, and so the third derivative's bound: range^3
        dz = scale * ((d @ wt.t()) if x is h else (h @ d.t()))
        spread = (dz.max(1).values - dz.min(1).values).double()
        third = float((spread ** 3 * glt.double()).sum())
        # f: n losses, each off by at most 300 roundings of magnitudes up to 40
        noise = float(glt.sum()) * 300 * E * 40 / eps
        got = float((grad.double() * ((a - b) / (2 * eps)).double()).sum())
        diff = (f(a) - f(b)) / (2 * eps)
        assert abs(diff - got) <= eps ** 2 / 6 * third + noise, (diff, got, eps ** 2 / 6 * third, noise)


def test_no_rows(cm):
    for dtype in (F32, BF16):
        h, wt = torch.empty(0, 40, dtype=dtype, device=DEV), torch.randn(30, 40, device=DEV).to(dtype)
        y = torch.empty(0, dtype=torch.int32, device=DEV)
        loss, lse = cm.cmsd_head_loss(h, wt, y)
        assert loss.numel() == 0 and lse.numel() == 0
        gh, (gw, flat) = torch.empty_like(h), padded(30, 40, 8, dtype, 5.0)
        cm.cmsd_head_loss_grad(h, wt, y, lse, loss, gh, gw)
        assert not gw.any() and gaps_left(flat, 30, 40, 8, 5.0)
        c, s = cm.cmsd_quantize_rows(h)
        wc, ws = cm.cmsd_quantize_rows(wt)
        assert cm.cmsd_head_logits(c, s, wc, ws).shape == (0, 30)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_without_labels_and_zero_weights(cm, dtype):
    h, wt, y, _, _, _, gl = problem(11, 70, 300, 64, dtype)
    y[:] = -1
    loss, lse = cm.cmsd_head_loss(h, wt, y)
    gh, gw = torch.full_like(h, 3.0), torch.full_like(wt, 3.0)
    cm.cmsd_head_loss_grad(h, wt, y, lse, torch.from_numpy(gl).to(DEV), gh, gw)
    assert not loss.any() and not gh.any() and not gw.any()
    # a row that reports an error, or holds a NaN under a negative label, adds nothing
    h2 = h.clone()
    h2[5] = float("nan")
    y[7], y[8] = 300, 4
    _, lse = cm.cmsd_head_loss(h2, wt, y)
    cm.cmsd_head_loss_grad(h2, wt, y, lse, torch.ones(70, device=DEV), grad_hidden=gh)
    assert torch.isfinite(gh).all() and not gh[7].any() and gh[8].any() and not gh[5].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,w,pad,offset", [(70, 300, 64, 0, 0), (300, 1000, 257, 3, 1), (1000, 9000, 136, 0, 0),
                                              (5, 40, 7, 0, 0)])
def test_padding_that_is_not_finite(cm, dtype, n, v, w, pad, offset):
    # what rows without a loss hold reaches neither gradient: the same bits as zeros there
    h, wt, y, _, _, _, gl = problem(13, n, v, w, dtype, pad, offset)
    gl = torch.from_numpy(gl).to(DEV)
    y[1], y[2], y[n - 1], gl[3] = -1, v, -5, 0.0
    gone = (y < 0) | (y >= v) | (gl == 0)
    got = []
    for fill in ((0.0, 0.0), (float("nan"), float("inf"))):
        h[gone] = fill[0]
        h[n - 1] = fill[1]
        loss, lse = cm.cmsd_head_loss(h, wt, y)
        gh, gw = torch.empty_like(h), torch.empty_like(wt)
        cm.cmsd_head_loss_grad(h, wt, y, lse, gl, gh, gw)
        got.append((loss[~gone], gh, gw))
    for a, b in zip(*got):
        assert torch.isfinite(a).all() and torch.equal(a, b)
    assert not got[1][1][gone].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,w", [(900, 5000, 96), (200, 700, 65)])
def test_a_mean_over_the_rows_is_not_biased(cm, dtype, n, v, w):
    # one factor for all rows, 1 / n, and logits near zero: p = 1 / v, and a label's entry
    # 1 - p is off by half a step of [1/2, 1) (UNIT / 2) at most, or is 1; the others are a
    # 1 / v of it.  So a gradient's part along the exact one is off by UNIT / 2 + (its own
    # rounding, of mixed signs: under UNIT / 4 of it) and the sums' (70 + v) E
    h, wt, y, hh, ww, yy, _ = problem(17, n, v, w, dtype, scale=1e3, lean=0.0)
    gl = np.full(n, 1 / n, np.float32)
    _, lse = cm.cmsd_head_loss(h, wt, y, scale=1e-3)
    gh, gw = torch.empty_like(h), torch.empty_like(wt)
    cm.cmsd_head_loss_grad(h, wt, y, lse, torch.from_numpy(gl).to(DEV), gh, gw, scale=1e-3)
    rh, _, rw, _, _, _ = H.head_loss_grad(hh, ww, yy, gl.astype(np.float64), 1e-3)
    for got, ref in ((host(gh), rh), (host(gw), rw)):
        along = (got * ref).sum() / (ref * ref).sum() - 1
        assert abs(along) <= UNIT[dtype] * 0.75 + (70 + v) * E, along


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_factors_that_are_not_finite_stay_in_their_rows(cm, dtype):
    h, wt, y, hh, ww, yy, gl = problem(19, 40, 300, 64, dtype)
    y[:] = torch.arange(40, device=DEV) * 7
    gl[4], gl[9] = np.inf, np.nan
    _, lse = cm.cmsd_head_loss(h, wt, y)
    gh = torch.empty_like(h)
    cm.cmsd_head_loss_grad(h, wt, y, lse, torch.from_numpy(gl).to(DEV), grad_hidden=gh)
    rest = [i for i in range(40) if i not in (4, 9)]
    (rh, bh), _ = grad_bounds(hh[rest], ww, y.cpu().numpy()[rest], gl[rest].astype(np.float64), 1.0, dtype, 64)
    within(host(gh)[rest], rh, bh, "grad_hidden")
    assert not torch.isfinite(gh[[4, 9]]).any()
    # none at all: zeros
    gw = torch.empty_like(wt)
    cm.cmsd_head_loss_grad(h, wt, y, lse, torch.zeros(40, device=DEV), gh, gw)
    assert not gh.any() and not gw.any()


# ------------------------------------------------------------------------------- how they are called
def _all(cm, h, wt, y, gl, out, ws):
    cm.cmsd_quantize_rows(h, out["c"], out["s"])
    cm.cmsd_quantize_rows(wt, out["wc"], out["ws"])
    cm.cmsd_head_logits(out["c"], out["s"], out["wc"], out["ws"], out["z"])
    cm.cmsd_head_loss(h, wt, y, out["loss"], out["lse"], workspace=ws)
    cm.cmsd_head_loss_grad(h, wt, y, out["lse"], gl, out["gh"], out["gw"], workspace=ws)


def _outs(n, v, w, dtype):
    e = lambda *s, d=F32: torch.zeros(*s, dtype=d, device=DEV)  # noqa: E731
    return {"c": e(n, w, d=torch.int8), "s": e(n), "wc": e(v, w, d=torch.int8), "ws": e(v), "z": e(n, v, d=dtype),
            "loss": e(n), "lse": e(n), "gh": e(n, w, d=dtype), "gw": e(v, w, d=dtype)}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,w", [(7, 1000, 64), (300, 2000, 128)])
def test_captured_replayed_and_repeated(cm, dtype, n, v, w):
    h, wt, y, _, _, _, gl = problem(21, n, v, w, dtype)
    gl = torch.from_numpy(gl).to(DEV)
    ws = cm.head_workspace(n, v, w, dtype, DEV)
    out, want = _outs(n, v, w, dtype), _outs(n, v, w, dtype)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _all(cm, h, wt, y, gl, out, ws)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _all(cm, h, wt, y, gl, out, ws)
    for k in range(4):
        h2, _, _, _, _, _, _ = problem(30 + k, n, v, w, dtype)
        h.copy_(h2)
        for t in out.values():
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        _all(cm, h, wt, y, gl, want, cm.head_workspace(n, v, w, dtype, DEV))
        torch.cuda.synchronize()
        for f in out:
            assert torch.equal(out[f], want[f]), (k, f)


def test_native_marshalling_same_calls(cm):
    # the same calls through the native and the Python marshalling: equal outputs, every
    # well-formed call is the native one's case, and the same refusals
    from tests.test_binding import _Recorder
    h, wt, y, _, _, _, gl = problem(23, 40, 500, 64, F32)
    gl = torch.from_numpy(gl).to(DEV)
    ws = cm.head_workspace(40, 500, 64, F32, DEV)
    keep = cm._native
    assert keep is not None

    def calls():
        out = _outs(40, 500, 64, F32)
        _all(cm, h, wt, y, gl, out, ws)
        for which in ("grad_hidden", "grad_weight"):
            one = torch.zeros_like(h if which == "grad_hidden" else wt)
            cm.cmsd_head_loss_grad(h, wt, y, out["lse"], gl, workspace=ws, **{which: one})
            out[which] = one
        torch.cuda.synchronize()
        errs = []
        for call in (lambda: cm.cmsd_quantize_rows(h.t(), out["c"], out["s"]),
                     lambda: cm.cmsd_quantize_rows(h, out["c"][:39], out["s"]),
                     lambda: cm.cmsd_head_logits(out["c"], out["s"], out["wc"], out["ws"], out["z"], scale=float("nan")),
                     lambda: cm.cmsd_head_logits(out["c"], out["s"], out["wc"], out["ws"], out["z"].half()),
                     lambda: cm.cmsd_head_loss(h, wt, y.long(), out["loss"], out["lse"], workspace=ws),
                     lambda: cm.cmsd_head_loss(h, wt, y, out["loss"], out["lse"], workspace=ws[:1]),
                     lambda: cm.cmsd_head_loss_grad(h, wt, y, out["lse"], gl, workspace=ws),
                     lambda: cm.cmsd_head_loss_grad(h, wt, y, out["lse"], gl, out["gw"], workspace=ws)):
            with pytest.raises(Exception) as e:
                call()
            errs.append((type(e.value), str(e.value)))
        return out, errs

    try:
        cm._native = _Recorder(keep)
        native, native_errs = calls()
        answers = cm._native.answers
        cm._native = None
        plain, plain_errs = calls()
    finally:
        cm._native = keep
    assert {f: [s for s in answers[f] if s is not None][0] for f in answers} == dict.fromkeys(
        ("quantize_rows", "head_logits", "head_loss", "head_loss_grad"), cm.CMSD_OK)
    assert [s for s in answers["head_loss_grad"]][:3] == [cm.CMSD_OK] * 3
    for f in native:
        assert torch.equal(native[f], plain[f]), f
    # (a workspace that is too small is the library's own refusal in one, the binding's in the other)
    assert [e[0] for e in native_errs[:5]] == [e[0] for e in plain_errs[:5]]
    assert native_errs[:5] == plain_errs[:5] and native_errs[6:] == plain_errs[6:]


def test_on_another_stream(cm):
    h, wt, y, _, _, _, gl = problem(22, 64, 3000, 256, BF16)
    gl = torch.from_numpy(gl).to(DEV)
    want, got = _outs(64, 3000, 256, BF16), _outs(64, 3000, 256, BF16)
    ws = cm.head_workspace(64, 3000, 256, BF16, DEV)
    _all(cm, h, wt, y, gl, want, ws)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    cm.cmsd_quantize_rows(h, got["c"], got["s"], stream=s)
    cm.cmsd_quantize_rows(wt, got["wc"], got["ws"], stream=s)
    cm.cmsd_head_logits(got["c"], got["s"], got["wc"], got["ws"], got["z"], stream=s)
    cm.cmsd_head_loss(h, wt, y, got["loss"], got["lse"], workspace=ws, stream=s)
    cm.cmsd_head_loss_grad(h, wt, y, got["lse"], gl, got["gh"], got["gw"], workspace=ws, stream=s)
    s.synchronize()
    for f in want:
        assert torch.equal(got[f], want[f]), f


def test_own_workspace_on_another_stream(cm):
    # a workspace made for the call is not handed out again before its stream has passed it
    n, v, w = 512, 20000, 256
    h, wt, y, _, _, _, gl = problem(24, n, v, w, BF16)
    gl = torch.from_numpy(gl).to(DEV)
    want, want_lse = cm.cmsd_head_loss(h, wt, y)
    gh, gw = torch.empty_like(h), torch.empty_like(wt)
    cm.cmsd_head_loss_grad(h, wt, y, want_lse, gl, gh, gw)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    loss, lse, gh2, gw2 = torch.empty_like(want), torch.empty_like(want), torch.empty_like(h), torch.empty_like(wt)
    torch.cuda.synchronize()
    for stream in (s, s.cuda_stream):
        cm.cmsd_head_loss(h, wt, y, loss, lse, stream=stream)
        junk = [torch.full((cm.cmsd_head_loss_workspace_bytes(n, v) // 4,), float("nan"), device=DEV) for _ in range(3)]
        cm.cmsd_head_loss_grad(h, wt, y, want_lse, gl, gh2, gw2, stream=stream)
        size = cm.cmsd_head_loss_grad_workspace_bytes(n, v, w, BF16)
        junk += [torch.full((size // 4,), float("nan"), device=DEV) for _ in range(3)]
        torch.cuda.synchronize()
        del junk
        for a, b in ((loss, want), (lse, want_lse), (gh2, gh), (gw2, gw)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("far", [9_000_000, 40_000_000])
def test_rows_far_apart(cm, dtype, far):
    # the last position of long sequences: rows 18 to 160 MB apart
    n, v, w = 9, 1200, 64
    h, wt, y, _, _, _, gl = problem(25, n, v, w, dtype)
    gl = torch.from_numpy(gl).to(DEV)
    flat = torch.empty(n * far, dtype=dtype, device=DEV)
    hs = flat.as_strided((n, w), (far, 1))
    hs.copy_(h)
    loss, lse = cm.cmsd_head_loss(hs, wt, y)
    gh, gw = flat.as_strided((n, w), (far, 1), 128), torch.empty_like(wt)
    cm.cmsd_head_loss_grad(hs, wt, y, lse, gl, gh, gw)
    for got, (ref, bound), what in zip((loss, lse, gh, gw), _on_gpu(h, wt, y, gl, 1.0, dtype),
                                       ("loss", "lse", "grad_hidden", "grad_weight")):
        assert float(((got.double() - ref).abs() / bound).max()) <= 1, what
    c, s = cm.cmsd_quantize_rows(hs)
    wc, ws = cm.cmsd_quantize_rows(wt)
    cs = torch.empty(n * far, dtype=torch.int8, device=DEV).as_strided((n, w), (far, 1))
    cs.copy_(c)
    assert torch.equal(cm.cmsd_head_logits(cs, s, wc, ws), cm.cmsd_head_logits(c, s, wc, ws))


def test_more_entries_than_a_piece(cm):
    # few rows, more entries than a piece takes: the second piece is 300 entries
    n, v, w = 3, (1 << 20) + 300, 16
    for dtype in (F32, BF16):
        h, wt, y, _, _, _, gl = problem(26, n, v, w, dtype)
        y[1], y[2] = v - 1, (1 << 20) - 1
        gl = torch.from_numpy(np.abs(gl) + 0.1).to(DEV)
        loss, lse = cm.cmsd_head_loss(h, wt, y)
        gh, gw = torch.empty_like(h), torch.empty_like(wt)
        cm.cmsd_head_loss_grad(h, wt, y, lse, gl, gh, gw)
        for got, (ref, bound), what in zip((loss, lse, gh, gw), _on_gpu(h, wt, y, gl, 1.0, dtype),
                                           ("loss", "lse", "grad_hidden", "grad_weight")):
            assert float(((got.double() - ref).abs() / bound).max()) <= 1, (dtype, what)


def test_outputs_past_32_bit_offsets(cm):
    # 5.1 GB of logits and a weight of 2.6e9 elements: the last rows against a small call
    n, v, w = 20000, 128256, 16
    g = torch.Generator(device=DEV).manual_seed(1)
    c = torch.randint(-127, 128, (n, w), generator=g, device=DEV, dtype=torch.int8)
    wc = torch.randint(-127, 128, (v, w), generator=g, device=DEV, dtype=torch.int8)
    s, ws = torch.rand(n, generator=g, device=DEV), torch.rand(v, generator=g, device=DEV)
    z = cm.cmsd_head_logits(c, s, wc, ws)
    for a in (0, n // 2, n - 40):
        ref = (c[a:a + 40].double() @ wc.double().t().contiguous()) * s[a:a + 40, None].double() * ws.double()
        far = (z[a:a + 40].double() - ref).abs() <= ref.abs() * (2.0 ** -8 + 4 * 2.0 ** -24) * 1.0001
        assert bool(far.all())
    del z
    v, w, n = 640000, 4096, 3
    wt = torch.empty(v, w, dtype=BF16, device=DEV)
    wt.normal_(generator=g, std=1 / 64)
    h = torch.randn(n, w, generator=g, device=DEV).to(BF16)
    y = torch.tensor([v - 1, 0, v // 2], dtype=torch.int32, device=DEV)
    loss, lse = cm.cmsd_head_loss(h, wt, y)
    z = torch.empty(n, v, dtype=torch.float64, device=DEV)
    for a in range(0, v, 32768):
        z[:, a:a + 32768] = h.double() @ wt[a:a + 32768].double().t().contiguous()
    ref = torch.logsumexp(z, 1)
    assert float((lse.double() - ref).abs().max()) <= (w + 4) * E * 64 + 1e-4
    gw = torch.empty_like(wt)
    cm.cmsd_head_loss_grad(h, wt, y, lse, torch.ones(n, device=DEV), grad_weight=gw)
    p = torch.exp(z - ref[:, None])
    p[torch.arange(n), y.long()] -= 1
    for a in (0, v // 2, v - 1):
        r = p[:, a].view(1, n) @ h.double()
        size = p[:, a].abs().view(1, n) @ h.double().abs()
        assert bool(((gw[a].double() - r[0]).abs() <= size[0] * 2.0 ** -8 * 2.2 + 1e-30).all())
