"""The vocabulary projection's calls on the host: refusals before any HIP call, workspace
sizes, and the binding's checks of its buffers.  CPU only."""
import pytest
import torch

cm = pytest.importorskip("paper_2508_15371_amd.cmsd")

P = 0x10000          # a fake, aligned device address: never dereferenced on these paths
ARG, DTYPE, OK = cm.CMSD_ERR_ARG, cm.CMSD_ERR_DTYPE, cm.CMSD_OK
NAN, INF = float("nan"), float("inf")


def test_new_entry_points_are_declared():
    assert set(cm.header_symbols()) >= {"cmsd_quantize_rows", "cmsd_head_logits", "cmsd_head_loss",
                                        "cmsd_head_loss_workspace_bytes", "cmsd_head_loss_grad",
                                        "cmsd_head_loss_grad_workspace_bytes"}


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), DTYPE), (dict(n=-1), ARG), (dict(n=1 << 31), ARG), (dict(w=0), ARG), (dict(w=1 << 17), ARG),
    (dict(rs=63), ARG), (dict(cs=63), ARG), (dict(cs=1 << 40), ARG), (dict(x=None), ARG), (dict(c=None), ARG),
    (dict(s=None), ARG), (dict(x=P + 1), ARG), (dict(s=P + 2), ARG), (dict(n=0, x=None, c=None, s=None), OK),
])
def test_quantize_argument_errors(kw, want):
    a = dict(x=P, dtype=cm.CMSD_BF16, n=4, w=64, rs=64, c=P, cs=64, s=P)
    a.update(kw)
    assert cm.lib().cmsd_quantize_rows(a["x"], a["dtype"], a["n"], a["w"], a["rs"], a["c"], a["cs"], a["s"],
                                       None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), DTYPE), (dict(n=-1), ARG), (dict(n=1 << 24), ARG), (dict(v=1), ARG), (dict(v=1 << 31), ARG),
    (dict(w=0), ARG), (dict(w=1 << 17), ARG), (dict(hst=63), ARG), (dict(wst=63), ARG), (dict(lst=99), ARG),
    (dict(scale=NAN), ARG), (dict(scale=INF), ARG), (dict(h=None), ARG), (dict(hs=None), ARG), (dict(wt=None), ARG),
    (dict(ws=None), ARG), (dict(out=None), ARG), (dict(hs=P + 2), ARG), (dict(ws=P + 1), ARG), (dict(out=P + 1), ARG),
    # 2^24 - 1 rows of 2^31 - 1 entries: no grid holds the tiles
    (dict(n=(1 << 24) - 1, v=(1 << 31) - 1, lst=1 << 31), ARG),
    (dict(n=0, h=None, hs=None, wt=None, ws=None, out=None), OK),
])
def test_logits_argument_errors(kw, want):
    a = dict(h=P, hst=64, hs=P, wt=P, wst=64, ws=P, scale=1.0, n=4, v=100, w=64, out=P, dtype=cm.CMSD_BF16, lst=100)
    a.update(kw)
    assert cm.lib().cmsd_head_logits(a["h"], a["hst"], a["hs"], a["wt"], a["wst"], a["ws"], a["scale"], a["n"], a["v"],
                                     a["w"], a["out"], a["dtype"], a["lst"], None) == want


def _loss(**kw):
    a = dict(h=P, hst=64, wt=P, wst=64, dtype=cm.CMSD_BF16, y=P, scale=1.0, n=4, v=100, w=64, loss=P, lse=P, ws=P,
             wsb=1 << 40)
    a.update(kw)
    return cm.lib().cmsd_head_loss(a["h"], a["hst"], a["wt"], a["wst"], a["dtype"], a["y"], a["scale"], a["n"], a["v"],
                                   a["w"], a["loss"], a["lse"], a["ws"], a["wsb"], None)


def _grad(**kw):
    a = dict(h=P, hst=64, wt=P, wst=64, dtype=cm.CMSD_BF16, y=P, lse=P, gl=P, scale=1.0, n=4, v=100, w=64, gh=P,
             ghst=64, gw=P, gwst=64, ws=P, wsb=1 << 60)
    a.update(kw)
    return cm.lib().cmsd_head_loss_grad(a["h"], a["hst"], a["wt"], a["wst"], a["dtype"], a["y"], a["lse"], a["gl"],
                                        a["scale"], a["n"], a["v"], a["w"], a["gh"], a["ghst"], a["gw"], a["gwst"],
                                        a["ws"], a["wsb"], None)


SHARED = [
    (dict(dtype=2), DTYPE), (dict(n=-1), ARG), (dict(n=1 << 24), ARG), (dict(v=1), ARG), (dict(v=1 << 31), ARG),
    (dict(w=0), ARG), (dict(w=1 << 17), ARG), (dict(hst=63), ARG), (dict(wst=63), ARG), (dict(scale=NAN), ARG),
    (dict(h=None), ARG), (dict(wt=None), ARG), (dict(y=None), ARG), (dict(h=P + 1), ARG), (dict(wt=P + 1), ARG),
    (dict(y=P + 2), ARG), (dict(ws=None), ARG), (dict(ws=P + 4), ARG), (dict(wsb=16), ARG), (dict(lse=None), ARG),
    (dict(lse=P + 2), ARG),
]


@pytest.mark.parametrize("kw,want", SHARED + [
    (dict(loss=None), ARG), (dict(loss=P + 1), ARG),
    (dict(n=(1 << 24) - 1, v=(1 << 31) - 1, wsb=1 << 62), ARG),
    (dict(n=0, h=None, wt=None, y=None, loss=None, lse=None, ws=None, wsb=0), OK),
])
def test_loss_argument_errors(kw, want):
    assert _loss(**kw) == want


@pytest.mark.parametrize("kw,want", SHARED + [
    (dict(gl=None), ARG), (dict(gl=P + 1), ARG), (dict(gh=None, gw=None), ARG), (dict(gh=P + 1), ARG),
    (dict(gw=P + 1), ARG), (dict(ghst=63), ARG), (dict(gwst=63), ARG), (dict(ws=P + 8), ARG),
    (dict(n=0, gw=None, h=None, wt=None, y=None, lse=None, gl=None, ws=None, wsb=0), OK),
])
def test_grad_argument_errors(kw, want):
    assert _grad(**kw) == want


def test_workspace_sizes():
    f, g = cm.lib().cmsd_head_loss_workspace_bytes, cm.lib().cmsd_head_loss_grad_workspace_bytes
    assert f(0, 100) == 0 and f(-1, 100) == 0 and f(4, 1) == 0 and f(1 << 24, 100) == 0
    assert g(0, 100, 64, 1) == 0 and g(4, 100, 0, 1) == 0 and g(4, 100, 64, 2) == 0 and g(4, 1, 64, 0) == 0
    # exactly what is asked for is enough, a byte less is not (the launch itself is not reached
    # on the host: only the refusal is looked at)
    for n, v, w in ((1, 2, 1), (7, 1000, 65), (4096, 128256, 4096)):
        assert _loss(n=n, v=v, w=w, hst=w, wst=w, wsb=f(n, v) - 1) == ARG
        for dt in (cm.CMSD_F32, cm.CMSD_BF16):
            assert _grad(n=n, v=v, w=w, hst=w, wst=w, ghst=w, gwst=w, dtype=dt, wsb=g(n, v, w, dt) - 1) == ARG
    # no logits are kept: far less than their bytes at a training step's size
    assert g(8192, 128256, 4096, cm.CMSD_BF16) < 8192 * 128256 * 2 / 2
    assert f(8192, 128256) < 8192 * 128256 * 4 / 16


def _f(*s, dtype=torch.float32):
    return torch.zeros(*s, dtype=dtype)


I8, BF, I32 = torch.int8, torch.bfloat16, torch.int32


@pytest.mark.parametrize("call,match", [
    (lambda: cm.cmsd_quantize_rows(_f(3, 8)), "device"),
    (lambda: cm.cmsd_quantize_rows(_f(8)), "2-D"),
    (lambda: cm.cmsd_quantize_rows(_f(8, 3).t()), "inner stride"),
    (lambda: cm.cmsd_quantize_rows(_f(1, 8).expand(3, 8)), "overlap"),
    (lambda: cm.cmsd_quantize_rows(_f(3, 8), _f(3, 7, dtype=I8)), "shape"),
    (lambda: cm.cmsd_quantize_rows(_f(3, 8), _f(3, 8)), "codes"),
    (lambda: cm.cmsd_quantize_rows(_f(3, 8), None, _f(2)), "scales"),
    (lambda: cm.cmsd_head_logits(_f(3, 8, dtype=I8), _f(3), _f(5, 7, dtype=I8), _f(5)), "weight"),
    (lambda: cm.cmsd_head_logits(_f(3, 8), _f(3), _f(5, 8, dtype=I8), _f(5)), "hidden"),
    (lambda: cm.cmsd_head_logits(_f(3, 8, dtype=I8), _f(2), _f(5, 8, dtype=I8), _f(5)), "hidden_scales"),
    (lambda: cm.cmsd_head_logits(_f(3, 8, dtype=I8), _f(3), _f(5, 8, dtype=I8), _f(4)), "weight_scales"),
    (lambda: cm.cmsd_head_logits(_f(3, 8, dtype=I8), _f(3), _f(5, 8, dtype=I8), _f(5), _f(3, 4)), "logits"),
    (lambda: cm.cmsd_head_logits(_f(3, 8, dtype=I8), _f(3), _f(5, 8, dtype=I8), _f(5)), "device"),
    (lambda: cm.cmsd_head_loss(_f(3, 8), _f(5, 8, dtype=BF), _f(3, dtype=I32)), "weight"),
    (lambda: cm.cmsd_head_loss(_f(3, 8), _f(5, 8), _f(3, dtype=torch.int64)), "labels"),
    (lambda: cm.cmsd_head_loss(_f(3, 8), _f(5, 8), _f(2, dtype=I32)), "labels"),
    (lambda: cm.cmsd_head_loss(_f(3, 8), _f(5, 8), _f(3, dtype=I32), _f(2)), "loss"),
    (lambda: cm.cmsd_head_loss(_f(3, 8), _f(5, 8), _f(3, dtype=I32), workspace=_f(2)), "workspace"),
    (lambda: cm.cmsd_head_loss(_f(3, 8), _f(5, 8), _f(3, dtype=I32)), "device"),
    (lambda: cm.cmsd_head_loss_grad(_f(3, 8), _f(5, 8), _f(3, dtype=I32), _f(3), _f(3)), "one of"),
    (lambda: cm.cmsd_head_loss_grad(_f(3, 8), _f(5, 8), _f(3, dtype=I32), _f(3), _f(2), _f(3, 8)), "grad_loss"),
    (lambda: cm.cmsd_head_loss_grad(_f(3, 8), _f(5, 8), _f(3, dtype=I32), _f(3), _f(3), _f(3, 7)), "grad_hidden"),
    (lambda: cm.cmsd_head_loss_grad(_f(3, 8), _f(5, 8), _f(3, dtype=I32), _f(3), _f(3), None, _f(5, 8, dtype=BF)),
     "grad_weight"),
    (lambda: cm.cmsd_head_loss_grad(_f(3, 8), _f(5, 8), _f(3, dtype=I32), _f(3), _f(3), _f(3, 8)), "device"),
])
def test_binding_refuses(call, match):
    with pytest.raises(ValueError, match=match):
        call()


def test_binding_refuses_types():
    with pytest.raises(TypeError):
        cm.cmsd_quantize_rows(_f(3, 8, dtype=torch.float16))
    with pytest.raises(TypeError):
        cm.cmsd_head_loss(_f(3, 8, dtype=torch.float64), _f(5, 8, dtype=torch.float64), _f(3, dtype=I32))
    with pytest.raises(TypeError):
        cm.cmsd_head_logits(_f(3, 8, dtype=I8), _f(3), _f(5, 8, dtype=I8), _f(5), dtype=torch.float16)


def test_head8_refuses_more_rows_than_its_buffers():
    from paper_2508_15371_amd import pipeline
    h = object.__new__(pipeline.Head8)
    h.hidden_scales, h.hidden_codes = _f(4), _f(4, 8, dtype=I8)
    with pytest.raises(ValueError, match="5 rows"):
        h.logits(_f(5, 8))
