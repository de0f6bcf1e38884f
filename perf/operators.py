"""The vocabulary projection's operators, timed as a decoder and its training call them.

A case is one pass of one operator on buffers that the program keeps:

  logits  one head product in 8-bit integers: the hidden rows are quantised (one scale per
          token), then multiplied with the head's codes (one scale per vocabulary entry)
          into logit rows: cmsd_quantize_rows and cmsd_head_logits
  loss    the softmax cross entropy of hidden rows against token ids over the whole
          vocabulary, no logits kept: cmsd_head_loss
  grad    the loss and its gradients, to the hidden rows, the head's weight or both:
          cmsd_head_loss and cmsd_head_loss_grad

``run`` computes them with elementary torch operations in 32 bits unless ``own`` is true;
``exact`` gives them in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
MOST_WORK = 4.4e12       # rows * vocabulary * width of a drawn case in bfloat16 (f32: an eighth)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, kind, rows, vocab, width, dtype="bf16", scale=1.0, pad=0, ignored=0.0, hidden=True, weight=True):
    """``pad``: elements between the rows' ends and the next rows' starts; ``ignored``: the
    share of rows without a label; ``hidden``, ``weight``: which gradients."""
    return {"name": name, "kind": kind, "rows": rows, "vocab": vocab, "width": width, "dtype": dtype, "scale": scale,
            "pad": pad, "ignored": ignored, "hidden": hidden, "weight": weight}


def listed():
    return [
        # one token of one sequence through a small drafter's head: latency
        _case("logits_one_token", "logits", 1, 32000, 768),
        # a drafting position of the package's own decoder: 16 sequences, f32, its logit scale
        _case("logits_decoder_f32", "logits", 16, 32000, 256, "f32", scale=5.0),
        # a drafting position of a lightly loaded server with a large target's head
        _case("logits_small_batch", "logits", 8, 152064, 4096),
        # a drafting position of a full server
        _case("logits_draft_256", "logits", 256, 128256, 2048),
        # the verifier's rows of 64 sequences of 8 drafts, an odd vocabulary, padded rows
        _case("logits_verify_odd", "logits", 576, 50257, 768, pad=16),
        # the verifier's rows of a full server: 256 sequences of 16 drafts
        _case("logits_verify_large", "logits", 4352, 128256, 4096),
        # the smallest evaluation: one short sequence under a toy vocabulary
        _case("loss_tiny_f32", "loss", 16, 1024, 256, "f32", scale=5.0),
        # evaluating a batch of text, padding left out
        _case("loss_eval", "loss", 2048, 50257, 768, ignored=0.1),
        # fitting the package's own drafter's head: the weight's gradient only
        _case("grad_decoder_f32", "grad", 1024, 32000, 256, "f32", scale=5.0, hidden=False),
        # a drafter trained under its target's frozen head: the hidden rows' gradient only
        _case("grad_frozen_head", "grad", 4096, 32000, 1024, weight=False),
        # a micro-batch with an odd number of rows and an odd vocabulary, padding left out
        _case("grad_odd", "grad", 1000, 50257, 768, ignored=0.1),
        # a training step's head at full size
        _case("grad_large", "grad", 8192, 128256, 4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(("logits", "logits", "loss", "grad", "grad"))
        rows = _log_int(rng, 1, 4352 if kind == "logits" else 8192)
        vocab = _log_int(rng, 1000, 152064)
        width = _log_int(rng, 64, 4096)
        if rng.random() < 0.6:
            vocab -= vocab % 8           # most vocabularies are padded to a round size
        if rng.random() < 0.8:
            width -= width % 64          # most widths are heads times a power of two
        dtype = "f32" if rng.random() < 0.3 else "bf16"
        which = rng.choice(("both", "both", "hidden", "weight"))
        c = {"kind": kind, "rows": rows, "vocab": vocab, "width": width, "dtype": dtype,
             "scale": rng.choice((1.0, 1.0, 5.0, 0.25)), "pad": rng.choice((0, 0, 0, 16, rng.randint(1, 100))),
             "ignored": 0.0 if kind == "logits" else rng.choice((0.0, 0.1, 0.5)),
             "hidden": kind != "grad" or which != "weight", "weight": kind != "grad" or which != "hidden"}
        most = MOST_WORK if kind == "logits" or dtype == "bf16" else MOST_WORK / 8
        if rows * vocab * width <= most:
            return c


# ---------------------------------------------------------------------------- inputs
def _rows(c, n, width, dtype=None):
    """Zeroed rows of the case's padded stride."""
    dt = dtype or TYPES[c["dtype"]]
    return torch.zeros((n, width + c["pad"]), dtype=dt, device=DEV)[:, :width]


def _inputs(c, seed):
    """Hidden rows as a final norm leaves them, leaning towards their label's weight row by a
    logit of 0 to 12 over the scale; the weight; labels, -1 for an ignored row."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, v, w = c["rows"], c["vocab"], c["width"]
    weight = _rows(c, v, w)
    for a in range(0, v, 16384):
        m = min(v, a + 16384) - a
        weight[a:a + m] = torch.randn(m, w, generator=g, device=DEV) * w ** -0.5
    labels = torch.randint(0, v, (n,), generator=g, device=DEV)
    hidden = _rows(c, n, w)
    lean = torch.rand(n, 1, generator=g, device=DEV) * (12.0 / max(1.0, c["scale"]))
    hidden.copy_(torch.randn(n, w, generator=g, device=DEV) + lean * weight[labels].float())
    if c["ignored"]:
        gone = torch.rand(n, generator=g, device=DEV) < c["ignored"]
        labels = torch.where(gone, torch.full_like(labels, -1), labels)
    return hidden, weight, labels


def prepare(case, seed):
    c = case
    hidden, weight, labels = _inputs(c, seed)
    n, v, w = c["rows"], c["vocab"], c["width"]
    s = {"case": c, "hidden": hidden}
    if c["kind"] == "logits":
        # the head's codes, made once when the model is loaded
        codes = _rows(c, v, w, torch.int8)
        scales = torch.empty(v, dtype=torch.float32, device=DEV)
        for a in range(0, v, 16384):
            codes[a:a + 16384], scales[a:a + 16384] = _quantised(weight[a:a + 16384])
        s.update(weight_codes=codes, weight_scales=scales, codes=_rows(c, n, w, torch.int8),
                 scales=torch.zeros(n, dtype=torch.float32, device=DEV), logits=_rows(c, n, v))
        return s
    valid = labels >= 0
    s.update(weight=weight, labels=labels.int(),
             # the mean over the labelled rows
             grad_loss=valid.float() / valid.sum().clamp(min=1).float(),
             loss=torch.zeros(n, dtype=torch.float32, device=DEV), lse=torch.zeros(n, dtype=torch.float32, device=DEV))
    if c["kind"] == "grad":
        s["grad_hidden"] = _rows(c, n, w) if c["hidden"] else None
        s["grad_weight"] = _rows(c, v, w) if c["weight"] else None
    return s


# ---------------------------------------------------------------------------- the operators
def _quantised(x):
    """Codes and scales of rows: the largest magnitude stands at 127.  A code is the whole
    number next to the quotient.  Both quotients are formed in 64 bits: in 32 some codes
    would move over a border."""
    x = x.double()
    scale = (x.abs().amax(1) / 127.0).float()
    safe = torch.where(scale > 0, scale, torch.ones_like(scale)).double()
    return torch.round(x / safe[:, None]).clamp(-127, 127).to(torch.int8), scale


def _plain_logits(s):
    c = s["case"]
    codes, scales = _quantised(s["hidden"])
    z = codes.float() @ s["weight_codes"].float().t()
    z *= scales[:, None] * c["scale"]
    z *= s["weight_scales"]
    return {"logits": z.to(TYPES[c["dtype"]])}


def _plain_loss(s):
    """The loss, and what its gradient goes on from: 32-bit copies, logits, their lse."""
    c = s["case"]
    h, w = s["hidden"].float(), s["weight"].float()
    z = h @ w.t()
    z *= c["scale"]
    top = z.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    y = s["labels"].long()
    at = torch.gather(z, 1, y.clamp(min=0)[:, None])
    loss = torch.where(y[:, None] >= 0, lse - at, torch.zeros_like(lse))
    return loss[:, 0], h, w, z, lse, y


def _plain_grad(s):
    c = s["case"]
    loss, h, w, z, lse, y = _plain_loss(s)
    p = torch.exp(z.sub_(lse), out=z)
    p.scatter_add_(1, y.clamp(min=0)[:, None], -torch.ones_like(lse))
    p *= torch.where(y >= 0, s["grad_loss"] * c["scale"], torch.zeros_like(s["grad_loss"]))[:, None]
    out = {"loss": loss}
    if c["hidden"]:
        out["grad_hidden"] = (p @ w).to(TYPES[c["dtype"]])
    if c["weight"]:
        out["grad_weight"] = (p.t() @ h).to(TYPES[c["dtype"]])
    return out


def _own(s):
    from paper_2508_15371_amd import cmsd
    c = s["case"]
    if c["kind"] == "logits":
        cmsd.cmsd_quantize_rows(s["hidden"], s["codes"], s["scales"])
        cmsd.cmsd_head_logits(s["codes"], s["scales"], s["weight_codes"], s["weight_scales"], s["logits"],
                              scale=c["scale"])
        return {"logits": s["logits"]}
    if "workspace" not in s:             # allocated on the first pass and kept
        s["workspace"] = cmsd.head_workspace(c["rows"], c["vocab"], c["width"], TYPES[c["dtype"]], DEV,
                                             grad=c["kind"] == "grad")
    cmsd.cmsd_head_loss(s["hidden"], s["weight"], s["labels"], s["loss"], s["lse"], scale=c["scale"],
                        workspace=s["workspace"])
    if c["kind"] == "loss":
        return {"loss": s["loss"], "lse": s["lse"]}
    cmsd.cmsd_head_loss_grad(s["hidden"], s["weight"], s["labels"], s["lse"], s["grad_loss"], s["grad_hidden"],
                             s["grad_weight"], scale=c["scale"], workspace=s["workspace"])
    out = {"loss": s["loss"]}
    if c["hidden"]:
        out["grad_hidden"] = s["grad_hidden"]
    if c["weight"]:
        out["grad_weight"] = s["grad_weight"]
    return out


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "logits":
        return _plain_logits(state)
    if kind == "loss":
        loss, _, _, _, lse, _ = _plain_loss(state)
        return {"loss": loss, "lse": lse[:, 0]}
    return _plain_grad(state)


def work(case):
    c = case
    n, v, w, e = c["rows"], c["vocab"], c["width"], 4 if c["dtype"] == "f32" else 2
    product = 2.0 * n * v * w
    if c["kind"] == "logits":
        return {"bytes": n * w * e + v * w + 4 * v + n * v * e, "flops": product}
    read = (n + v) * w * e + 8 * n       # with the labels, and the loss written
    if c["kind"] == "loss":
        return {"bytes": read + 4 * n, "flops": product}
    both = c["hidden"] + c["weight"]
    return {"bytes": read + 4 * n + (n * c["hidden"] + v * c["weight"]) * w * e, "flops": product * (1 + both)}


# ---------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    n, v, step = c["rows"], c["vocab"], 1024
    h = s["hidden"].double()
    if c["kind"] == "logits":
        # the codes are the operator's own values: nearest multiples of a row's largest / 127
        unit = h.abs().max(dim=1).values.div(127).float().double()
        q = (h / unit.clamp(min=1e-300).unsqueeze(1)).round()
        out = torch.empty((n, v), dtype=torch.float64, device=DEV)
        for a in range(0, v, 16384):
            b = min(v, a + 16384)
            wq = s["weight_codes"][a:b].double().mul_(s["weight_scales"][a:b].double().unsqueeze(1))
            out[:, a:b] = torch.mm(q * (unit * c["scale"]).unsqueeze(1), wq.T.contiguous())
        return {"logits": out}
    w = s["weight"].double()
    wt = w.T.contiguous()
    y = s["labels"].long()
    out = {"loss": torch.zeros(n, dtype=torch.float64, device=DEV)}
    if c["kind"] == "loss":
        out["lse"] = torch.zeros(n, dtype=torch.float64, device=DEV)
    if c["kind"] == "grad" and c["hidden"]:
        out["grad_hidden"] = torch.zeros((n, c["width"]), dtype=torch.float64, device=DEV)
    if c["kind"] == "grad" and c["weight"]:
        out["grad_weight"] = torch.zeros((v, c["width"]), dtype=torch.float64, device=DEV)
    for a in range(0, n, step):
        ya, ha = y[a:a + step], h[a:a + step]
        at = torch.arange(len(ya), device=DEV)
        z = torch.mm(ha, wt) * c["scale"]
        if c["kind"] == "loss":
            out["lse"][a:a + step] = torch.logsumexp(z, dim=1)
        logp = torch.log_softmax(z, dim=1)
        keep = (ya >= 0).double()
        out["loss"][a:a + step] = -logp[at, ya.clamp(min=0)] * keep
        if c["kind"] == "loss":
            continue
        p = logp.exp_()
        p[at, ya.clamp(min=0)] -= 1.0
        p *= (s["grad_loss"][a:a + step].double() * keep * c["scale"]).unsqueeze(1)
        if c["hidden"]:
            out["grad_hidden"][a:a + step] = torch.mm(p, w)
        if c["weight"]:
            out["grad_weight"] += torch.mm(p.T.contiguous(), ha)
    return out
