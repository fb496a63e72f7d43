"""More operators of a learned proposer as measurable cases: layer norm with its
gradient, an AdamW step over all of a model's tensors, and beam search's selection
with the reordering of the beams' states.

`own` false computes every operator in its plain form, elementary torch operations in
32 bits (a beam's normaliser in 64: it decides which of two nearly equal beams goes
on); `own` true calls the library.  exact() computes the definitions in 64 bits with
numpy.
"""
import math

import numpy as np
import torch

own = False

FLT_MAX = 3.4028234663852886e38
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
MASK = 0xFFFFFFFF
BLOCK = 256  # elements that share the scale of their 8-bit moments


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # the norm of a block for one token of each of 64 sequences: latency
        dict(name="norm-step-64x1024", op="norm", rows=64, dim=1024, type="bf16", out="bf16", wtype="bf16",
             residual=True),
        # the same over a batch of prompts
        dict(name="norm-prompts-16384x4096", op="norm", rows=16384, dim=4096, type="bf16", out="bf16", wtype="bf16",
             residual=True),
        # one training batch
        dict(name="norm-grad-32768x2048", op="norm_grad", rows=32768, dim=2048, type="bf16", out="bf16", wtype="f32",
             residual=True),
        # training on decoded candidates: short odd rows, each weight's sum over a million of them
        dict(name="norm-grad-knobs-1048573x61", op="norm_grad", rows=1048573, dim=61, type="f32", out="f32",
             wtype="f32", residual=False),
        # a step of the small proposer over knob digits: latency
        dict(name="adamw-proposer-f32", op="adamw", layers=1, dim=64, inner=128, vocab=65, type="f32", grad="f32",
             copies="", bits=32, clip=False),
        # a step of a model trained in bf16 with fp32 parameters, moments in 32 bits
        dict(name="adamw-24x1024-32bit", op="adamw", layers=24, dim=1024, inner=1024, vocab=8021, type="f32",
             grad="bf16", copies="bf16", bits=32, clip=True),
        # the same with moments in 8 bits
        dict(name="adamw-24x1024-8bit", op="adamw", layers=24, dim=1024, inner=1024, vocab=8021, type="f32",
             grad="bf16", copies="bf16", bits=8, clip=True),
        # the 256 best configurations so far, each with 8 options for its next knob
        dict(name="beam-knobs-1x256x8", op="beam", batch=1, beams=256, n=8, m=256, type="f32", masked=0.0, eos=-1,
             start=False),
        # one request over a vocabulary
        dict(name="beam-one-1x4x50021", op="beam", batch=1, beams=4, n=50021, m=8, type="f32", masked=0.0, eos=2,
             start=False),
        # a served batch
        dict(name="beam-batch-64x8x50021", op="beam", batch=64, beams=8, n=50021, m=8, type="bf16", masked=0.1, eos=2,
             start=False),
        # the proposer's states after its beams were chosen
        dict(name="reorder-knobs-1x256", op="reorder", batch=1, beams=256, dim=128, states=16, taps=4, history=8,
             type="f32"),
        # the states of a served batch
        dict(name="reorder-batch-64x8x2048", op="reorder", batch=64, beams=8, dim=2048, states=16, taps=4, history=513,
             type="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm", "norm", "norm_grad", "norm_grad", "adamw", "adamw", "beam", "beam", "reorder"))
    kind = rng.choice(("f32", "bf16", "f16"))
    if op in ("norm", "norm_grad"):
        dim = _log_int(rng, 1, 65536)
        if rng.random() < 0.5:
            dim = max(1, dim // 8) * 8
        rows = _log_int(rng, 1, max(1, min(1048576, 67108864 // dim)))
        return dict(op=op, rows=rows, dim=dim, type=kind,
                    out=rng.choice(("f32", "bf16", "f16")) if kind == "f32" else kind,
                    wtype=rng.choice(("f32", kind, "")), residual=rng.random() < 0.5)
    if op == "adamw":
        dim, layers = _log_int(rng, 8, 1024), _log_int(rng, 1, 24)
        return dict(op=op, layers=layers, dim=dim, inner=_log_int(rng, 8, 1024), vocab=_log_int(rng, 9, 8021),
                    type=kind, grad=rng.choice(("f32", kind)),
                    copies=rng.choice(("", "bf16", "f16")) if kind == "f32" else "", bits=rng.choice((8, 32)),
                    clip=rng.random() < 0.5)
    if op == "beam":
        if rng.random() < 0.3:  # many beams over few options
            beams = _log_int(rng, 16, 1024)
            n = rng.randint(1, 8192 // beams if beams > 128 else 64)
            m = beams
        else:
            n, beams = _log_int(rng, 2, 262144), _log_int(rng, 1, 64)
            m = beams * rng.choice((1, 2))
        batch = _log_int(rng, 1, max(1, min(256, 25165824 // (n * beams))))
        return dict(op=op, batch=batch, beams=beams, n=n, m=m, type=kind, masked=rng.choice((0.0, 0.1, 0.9)),
                    eos=rng.choice((-1, min(2, n - 1))), start=rng.random() < 0.2)
    beams, dim, states = _log_int(rng, 1, 256), _log_int(rng, 1, 4096), rng.choice((1, 4, 8, 13, 16, 32))
    batch = _log_int(rng, 1, max(1, min(128, 16777216 // (beams * dim * states))))
    return dict(op=op, batch=batch, beams=beams, dim=dim, states=states, taps=rng.choice((2, 3, 4)),
                history=_log_int(rng, 1, 1024), type=kind)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 29)
    return g


def _shapes(case):
    """The tensors of a recurrent model: table, blocks, scores."""
    d, i, v = case["dim"], case["inner"], case["vocab"]
    block = [(d,), (d,), (d, 3 * i + 32), (i, 4), (i,), (i, 16), (i,), (i,), (i, d)]
    return [(v, d)] + block * case["layers"] + [(d, v)]


def _views(flat, shapes):
    """Tensors inside one buffer, each from a multiple of BLOCK elements on."""
    got, at = [], 0
    for s in shapes:
        n = math.prod(s)
        got.append(flat[at:at + n].view(s))
        at += -(-n // BLOCK) * BLOCK
    return got


def prepare(case, seed):
    g = _generator(seed)
    rnd = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    rand = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    st = dict(case)
    if case["op"] in ("norm", "norm_grad"):
        rows, d, dt, wt = case["rows"], case["dim"], TYPES[case["type"]], TYPES.get(case["wtype"])
        # channels of their own mean and size, as a residual stream has
        x = rnd(rows, d).mul_(0.5 + rand(d)).add_(rnd(d) * 0.3)
        st["weight"] = None if wt is None else (1 + 0.1 * rnd(d)).to(wt)
        st["bias"] = None if wt is None else (0.1 * rnd(d)).to(wt)
        st["x"], st["eps"] = x.to(dt), 1e-5
        if case["op"] == "norm":
            st["residual"] = rnd(rows, d).to(dt) if case["residual"] else None
            return st
        x = st["x"].float()
        mean = x.mean(1, keepdim=True)
        var = (x - mean).square_().mean(1, keepdim=True)
        st["stats"] = torch.cat([mean, 1.0 / torch.sqrt(var + st["eps"])], 1)
        del x
        st["gy"] = rnd(rows, d).to(TYPES[case["out"]])
        st["g_total"] = rnd(rows, d).to(dt) if case["residual"] else None
        return st
    if case["op"] == "adamw":
        shapes = _shapes(case)
        blocks = [-(-math.prod(s) // BLOCK) for s in shapes]
        total = sum(blocks) * BLOCK
        flat = torch.zeros(total, dtype=TYPES[case["type"]], device="cuda")
        m, v = torch.zeros(total, device="cuda"), torch.zeros(total, device="cuda")
        grads = []
        for p, a, b in zip(_views(flat, shapes), _views(m, shapes), _views(v, shapes)):
            size = 10.0 ** (-1 - 3 * rand(1))  # gradients of different tensors differ by decades
            p.copy_(rnd(*p.shape) * p.shape[-1] ** -0.5)
            row = size * torch.exp(0.7 * rnd(p.shape[0])).view(-1, *[1] * (p.dim() - 1))
            if p.dim() == 2 and p.shape[0] == case["vocab"]:
                row = row * (rand(p.shape[0], 1) < 0.7)  # tokens that never came
            a.copy_(0.3 * row * rnd(*p.shape))
            b.copy_((row * (0.5 + rand(*p.shape))) ** 2)
            grads.append((row * rnd(*p.shape)).to(TYPES[case["grad"]]))
        st.update(flat=flat, params=_views(flat, shapes), grads=grads, m=m, v=v, step=1001, lr=3e-4, betas=(0.9, 0.999),
                  eps=1e-8, seed=seed & MASK, m_scale=None, v_scale=None, flat_copy=None, copies=None, grad_scale=None)
        # matrices decay, vectors do not; rates and step sizes move slower
        st["decay"] = [0.1 if len(s) == 2 and s[1] > 16 else 0.0 for s in shapes]
        st["rate"] = [st["lr"] * (0.1 if len(s) == 2 and s[1] == 16 else 1.0) for s in shapes]
        per = torch.tensor([st["rate"], st["decay"]], dtype=torch.float64).repeat_interleave(torch.tensor(blocks), 1)
        st["block_rate"], st["block_decay"] = per.cuda()[:, :, None]
        if case["copies"]:
            st["flat_copy"] = flat.to(TYPES[case["copies"]])
            st["copies"] = _views(st["flat_copy"], shapes)
        if case["clip"]:
            st["grad_scale"] = 0.3 + 0.7 * rand(1)
        if case["bits"] == 8:
            key = torch.zeros((), dtype=torch.int64, device="cuda")
            st["m"], st["m_scale"], st["v"], st["v_scale"] = _to_8_bits(m, v, key)
        return st
    if case["op"] == "beam":
        b, w, n = case["batch"], case["beams"], case["n"]
        x = rnd(b, w, n) * 2.5
        if case["masked"]:
            x = torch.where(rand(b, w, n) < case["masked"], -math.inf, x)
        st["scores"] = x.to(TYPES[case["type"]])
        logp = -(3.0 * rnd(b, w)).abs() - 10.0
        st["logp"] = logp.sort(1, descending=True)[0].contiguous()
        if case["start"]:  # one beam so far
            st["logp"][:, 1:] = -math.inf
        st["done"] = None
        if case["eos"] >= 0:
            st["done"] = rand(b, w) < 0.15
            if case["start"]:
                st["done"][:] = False
        return st
    b, w, d, s = case["batch"], case["beams"], case["dim"], case["states"]
    dt = TYPES[case["type"]]
    st["tensors"] = [rnd(b * w, d, s), rnd(b * w, case["taps"] - 1, d).to(dt),
                     torch.randint(0, 50021, (b * w, case["history"]), generator=g, device="cuda")]
    # the better beams are continued more often; a beam that was not filled has no parent
    u = rand(b, w)
    st["parent"] = (u * u * w).long().clamp_(max=w - 1).masked_fill_(rand(b, w) < 0.01, -1)
    return st


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------

def _plain_norm(st):
    x = st["x"]
    out = {}
    if st["residual"] is not None:
        x = (x.float() + st["residual"].float()).to(x.dtype)
        out["total"] = x
    x = x.float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + st["eps"])
    y = x * rstd
    if st["weight"] is not None:
        y = y * st["weight"].float() + st["bias"].float()
    out.update(y=y.to(TYPES[st["out"]]), stats=torch.cat([mean, rstd], 1))
    return out


def _plain_norm_grad(st):
    x, gy, stats = st["x"].float(), st["gy"].float(), st["stats"]
    h = (x - stats[:, :1]) * stats[:, 1:]
    w = st["weight"]
    gw = gy if w is None else gy * w.float()
    gx = (gw - gw.mean(1, keepdim=True) - h * (gw * h).mean(1, keepdim=True)) * stats[:, 1:]
    if st["g_total"] is not None:
        gx = gx + st["g_total"].float()
    out = {"x": gx.to(st["x"].dtype)}
    if w is not None:
        out.update(weight=(gy * h).sum(0).to(w.dtype), bias=gy.sum(0).to(w.dtype))
    return out


def _mix(h):
    """A permutation of 32-bit numbers (held in int64)."""
    h = ((h ^ (h >> 16)) * 0x9E3779B1) & MASK
    h = ((h ^ (h >> 15)) * 0xB504F333) & MASK
    return h ^ (h >> 16)


def _to_8_bits(m, v, key):
    """Moments of whole blocks in 8 bits with one power of two a block: m as e4m3, its scale,
    v as e5m2, its scale.  Values between two codes go up or down by a hash of their place, in
    proportion to how near they are."""
    n = m.numel()
    block = torch.arange(n // BLOCK, device=m.device)
    lane = torch.arange(BLOCK, device=m.device)
    h = _mix((_mix((block + key) & MASK)[:, None] + lane * 0x9E3779B9) & MASK)
    got = []
    for x, low, drop, bias, kind in ((m, h & 0xFFFF, 20, 134, torch.float8_e4m3fn), (v, h >> 16, 21, 141, torch.float8_e5m2)):
        x = x.view(-1, BLOCK)
        bits = x.view(torch.int32) & 0x7FFFFFFF
        e = (bits.amax(1, keepdim=True) >> 23).clamp(min=16)
        up = ((127 + bias - e) << 23).view(torch.float32)
        small = x.abs() * up * 2.0 ** (14 - bias if kind == torch.float8_e4m3fn else 29 - bias)
        code = (small.view(torch.int32).long() + (low << (drop - 16))) >> drop
        if kind == torch.float8_e4m3fn:
            code = code + ((x.view(torch.int32) < 0).long() << 7)
        else:
            code = torch.where(bits > 0, code.clamp(min=1), code)
        code = torch.where(e == 255, 0x7F, code)
        got += [code.to(torch.uint8).view(kind).view(-1), ((127 - bias + e) << 23).view(torch.float32).view(-1)]
    return got


def _from_8_bits(code, scale):
    return (code.float().view(-1, BLOCK) * scale[:, None]).view(-1)


def _plain_adamw(st):
    (b1, b2), t = st["betas"], st["step"]
    pad = lambda g: torch.nn.functional.pad(g.reshape(-1), (0, -g.numel() % BLOCK))  # noqa: E731
    g = torch.cat([pad(q) for q in st["grads"]]).float()
    if st["grad_scale"] is not None:
        g = g * st["grad_scale"]
    m, v = st["m"], st["v"]
    if st["bits"] == 8:
        m, v = _from_8_bits(m, st["m_scale"]), _from_8_bits(v, st["v_scale"])
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    rate = (st["block_rate"] / (1 - b1 ** t)).float()
    keep = (1 - st["block_rate"] * st["block_decay"]).float()
    step = m / (torch.sqrt(v) * (1 / math.sqrt(1 - b2 ** t)) + st["eps"])
    p = st["flat"].float().view(-1, BLOCK) * keep - step.view(-1, BLOCK) * rate
    p = p.view(-1)
    st["flat"].copy_(p)
    out = {"params": st["flat"]}
    if st["flat_copy"] is not None:
        st["flat_copy"].copy_(p)
        out["copies"] = st["flat_copy"]
    if st["bits"] == 8:
        key = _mix((_mix(torch.tensor(st["seed"], device=p.device)) + t) & MASK)
        got = _to_8_bits(m, v, key)
        for name, q in zip(("m", "m_scale", "v", "v_scale"), got):
            st[name].copy_(q)
            out[name] = st[name]
        return out
    st["m"].copy_(m)
    st["v"].copy_(v)
    return dict(out, m=st["m"], v=st["v"])


def _plain_beam(st):
    x, logp, done, m = st["scores"], st["logp"], st["done"], st["m"]
    b, w, n = x.shape
    s = x.float()
    s = s.clamp(-FLT_MAX, FLT_MAX).masked_fill(torch.isnan(s) | (s == -math.inf), -math.inf) + 0.0
    top = s.amax(2, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top).double()
    lse = top + torch.log(torch.exp(s.double() - top).sum(2, keepdim=True))
    s, token = torch.sort(s, dim=2, descending=True, stable=True)
    s, token = s[..., :m], token[..., :m]
    total = torch.where(s == -math.inf, -math.inf, logp.double()[..., None] + (s.double() - lse))
    if done is not None:  # a finished beam goes on as it is
        first = torch.arange(s.shape[2], device=x.device) == 0
        total = torch.where(done[..., None], torch.where(first, logp.double()[..., None], -math.inf), total)
        token = torch.where(done[..., None], st["eos"], token)
    total, at = torch.sort(total.reshape(b, -1), dim=1, descending=True, stable=True)
    total, at = total[:, :m], at[:, :m]
    token = torch.gather(token.reshape(b, -1), 1, at)
    parent = at // s.shape[2]
    none = total == -math.inf
    ended = torch.zeros_like(none) if done is None else torch.gather(done, 1, parent) | (token == st["eos"])
    more = (0, m - total.shape[1])
    pad = torch.nn.functional.pad
    return {"parent": pad(parent.masked_fill(none, -1), more, value=-1),
            "token": pad(token.masked_fill(none, -1), more, value=-1),
            "logp": pad(total.float(), more, value=-math.inf), "done": pad(ended & ~none, more, value=False)}


def _plain_reorder(st):
    parent = st["parent"]
    b, w = parent.shape
    place = torch.arange(b * w, device=parent.device).view(b, w)
    source = torch.where(parent < 0, place, place[:, :1] + parent).view(-1)
    return [t.copy_(t[source]) for t in st["tensors"]]


# ---------------------------------------------------------------------------
# Passes
# ---------------------------------------------------------------------------

def run(state):
    op = state["op"]
    if not own:
        return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "adamw": _plain_adamw, "beam": _plain_beam,
                "reorder": _plain_reorder}[op](state)
    from paper_2411_10764_gb300 import mlt

    if op == "norm":
        y, total, stats = mlt.layer_norm(state["x"], state["weight"], state["bias"], state["eps"],
                                         residual=state["residual"], out_dtype=TYPES[state["out"]])
        out = {"y": y, "stats": stats}
        return out if state["residual"] is None else dict(out, total=total)
    if op == "norm_grad":
        g = mlt.layer_norm_grad(state["gy"], state["x"], state["stats"], state["weight"], state["bias"],
                                g_total=state["g_total"])
        return {k: t for k, t in g.items() if t is not None}
    if op == "adamw":
        moments = mlt.AdamWState(state["m"], state["v"], state["m_scale"], state["v_scale"])
        mlt.adamw(state["params"], state["grads"], moments, state["step"], lr=state["rate"], betas=state["betas"],
                  eps=state["eps"], weight_decay=state["decay"], copies=state["copies"],
                  grad_scale=state["grad_scale"], seed=state["seed"])
        out = {"params": state["flat"], "m": state["m"], "v": state["v"]}
        if state["flat_copy"] is not None:
            out["copies"] = state["flat_copy"]
        return out if state["bits"] == 32 else dict(out, m_scale=state["m_scale"], v_scale=state["v_scale"])
    if op == "beam":
        parent, token, logp, done = mlt.beam_step(state["scores"], state["logp"], state["m"], done=state["done"],
                                                  eos=state["eos"])
        return {"parent": parent, "token": token, "logp": logp, "done": done}
    mlt.beam_reorder(state["parent"], *state["tensors"])
    return state["tensors"]


def work(case):
    op = case["op"]
    if op in ("norm", "norm_grad"):
        e, o, w = SIZE[case["type"]], SIZE[case["out"]], SIZE.get(case["wtype"], 0)
        rows, d, more = case["rows"], case["dim"], case["residual"]
        if op == "norm":
            return {"bytes": rows * d * (e + o + 2 * more * e) + rows * 8 + 2 * d * w, "flops": 8.0 * rows * d}
        return {"bytes": rows * d * (2 * e + o + more * e) + rows * 8 + 3 * d * w, "flops": 14.0 * rows * d}
    if op == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        per = 2 * SIZE[case["type"]] + SIZE[case["grad"]] + SIZE.get(case["copies"], 0)
        per += 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * per, "flops": n * (15.0 if case["bits"] == 32 else 35.0)}
    if op == "beam":
        b, w, n, m = case["batch"], case["beams"], case["n"], case["m"]
        live = 1.0 / w if case["start"] else 0.85 if case["eos"] >= 0 else 1.0
        return {"bytes": b * (live * w * n * SIZE[case["type"]] + w * 5 + m * 21), "flops": 4.0 * live * b * w * n}
    b, w, d = case["batch"], case["beams"], case["dim"]
    row = d * case["states"] * 4 + (case["taps"] - 1) * d * SIZE[case["type"]] + case["history"] * 8
    # beam j is a parent with the probability of u * u * w in [j, j + 1)
    p = np.diff(np.sqrt(np.arange(w + 1) / w))
    read, written = (1 - (1 - p) ** w).sum() - (p * (1 - p) ** (w - 1)).sum(), 0.99 * (w - p.sum())
    return {"bytes": b * (row * (float(read) + written) + w * 8) if w > 1 else b * 8.0, "flops": 0.0}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def _np(t):
    return None if t is None else (t.float() if t.is_floating_point() else t).cpu().numpy()


def _exact_norm(st, backward):
    x, w, b = _np(st["x"]), _np(st["weight"]), _np(st["bias"])
    rows, d = x.shape
    wide = lambda a, i, j: a[i:j].astype(np.float64)  # noqa: E731
    w = np.ones(d) if w is None else w.astype(np.float64)
    b = np.zeros(d) if b is None else b.astype(np.float64)
    if not backward:
        out = {"y": np.empty((rows, d)), "stats": np.empty((rows, 2))}
        if st["residual"] is not None:  # rounded to the stream's type before the norm sees it
            x = _np((st["x"].double() + st["residual"].double()).to(st["x"].dtype))
            out["total"] = _np(st["x"]).astype(np.float64) + _np(st["residual"])
    else:
        gy, more = _np(st["gy"]), _np(st["g_total"])
        out = {"x": np.empty((rows, d)), "weight": np.zeros(d), "bias": np.zeros(d)}
        stats = _np(st["stats"]).astype(np.float64)
    step = max(1, 4194304 // d)
    for i in range(0, rows, step):
        j = min(rows, i + step)
        a = wide(x, i, j)
        if not backward:
            mean = a.sum(1, keepdims=True) / d
            a -= mean
            rstd = (np.einsum("ij,ij->i", a, a)[:, None] / d + st["eps"]) ** -0.5
            out["y"][i:j] = a * rstd * w + b
            out["stats"][i:j] = np.concatenate([mean, rstd], 1)
            continue
        a -= stats[i:j, :1]
        a *= stats[i:j, 1:]
        g = wide(gy, i, j)
        out["weight"] += np.einsum("ij,ij->j", g, a)
        out["bias"] += g.sum(0)
        g *= w
        along = np.einsum("ij,ij->i", g, a)[:, None] / d
        g -= g.sum(1, keepdims=True) / d
        g -= a * along
        g *= stats[i:j, 1:]
        out["x"][i:j] = g if more is None else g + more[i:j]
    if backward and st["weight"] is None:
        out = {"x": out["x"]}
    return out


def _exact_adamw(st):
    (b1, b2), t = st["betas"], st["step"]
    c = 1.0 if st["grad_scale"] is None else float(st["grad_scale"])
    m, v = _np(st["m"]).astype(np.float64), _np(st["v"]).astype(np.float64)
    if st["bits"] == 8:
        m = (m.reshape(-1, BLOCK) * _np(st["m_scale"])[:, None]).reshape(-1)
        v = (v.reshape(-1, BLOCK) * _np(st["v_scale"])[:, None]).reshape(-1)
    p = _np(st["flat"]).astype(np.float64)
    at = 0
    for grad, rate, decay in zip(st["grads"], st["rate"], st["decay"]):
        n = grad.numel()
        here = slice(at, at + n)
        g = _np(grad).reshape(-1).astype(np.float64) * c
        m[here] += (1 - b1) * (g - m[here])
        v[here] += (1 - b2) * (g * g - v[here])
        direction = (m[here] / (1 - b1 ** t)) / (np.sqrt(v[here] / (1 - b2 ** t)) + st["eps"])
        p[here] -= rate * (direction + decay * p[here])
        at += -(-n // BLOCK) * BLOCK
    out = {"params": p}
    if st["flat_copy"] is not None:
        out["copies"] = p
    if st["bits"] == 8:  # which neighbour a value goes to is no number to be near to
        return dict(out, m=None, m_scale=None, v=None, v_scale=None)
    return dict(out, m=m, v=v)


def _exact_beam(st):
    x, logp = _np(st["scores"]), _np(st["logp"]).astype(np.float64)
    b, w, n = x.shape
    m = st["m"]
    done = np.zeros((b, w), bool) if st["done"] is None else _np(st["done"])
    out = np.full((b, m), -np.inf)
    for i in range(b):
        got = []
        for j in range(w):
            if done[i, j]:
                got.append(logp[i, j:j + 1])
                continue
            row = x[i, j][x[i, j] > -np.inf].astype(np.float64)
            if row.size == 0 or logp[i, j] == -np.inf:
                continue
            best = np.partition(row, row.size - m)[-m:] if row.size > m else row
            top = best.max()
            got.append(logp[i, j] + best - (top + math.log(np.exp(row - top).sum())))
        got = -np.sort(-np.concatenate(got)) if got else np.empty(0)
        out[i, :min(m, got.size)] = got[:m]
    return {"parent": None, "token": None, "logp": out, "done": None}


def _exact_reorder(st):
    parent, out = _np(st["parent"]), [_np(t) for t in st["tensors"]]
    w = parent.shape[1]
    for t in out:
        for i, of in enumerate(parent):
            rows = t[i * w:(i + 1) * w]
            rows[of >= 0] = rows[of[of >= 0]].copy()
    return [t if t.dtype.kind != "f" else t.astype(np.float64) for t in out]


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "reorder":
        return _exact_reorder(st)
    if case["op"] in ("norm", "norm_grad"):
        return _exact_norm(st, case["op"] == "norm_grad")
    return _exact_adamw(st) if case["op"] == "adamw" else _exact_beam(st)
