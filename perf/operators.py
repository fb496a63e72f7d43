"""The sequence-model operators as measurable cases: drawing candidates or
tokens from scores, embedding lookup with its gradient, and the selective scan
with its short causal convolution (prompts, single tokens, gradients).

`own` false computes every operator in its plain form, elementary torch
operations in 32 bits; `own` true calls the library.  exact() computes the
definitions in 64 bits with numpy.
"""
import math

import numpy as np
import torch

own = False

FLT_MAX = 3.4028234663852886e38
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
# rule: "greedy", "plain" (temperature alone), "top_k", "top_p", "min_p", or
# "mixed" (every row has its own rule, all of these in turn, some combined)

def listed():
    return [
        # one knob of 8 options drawn for each of 256 search chains: latency
        dict(name="sample-chains-256x8", op="sample", rows=256, n=8, type="f32", rule="plain", k=0, m=1, masked=0.25),
        # next tokens of 64 sequences, every user with settings of their own
        dict(name="sample-tokens-64x50021", op="sample", rows=64, n=50021, type="bf16", rule="mixed", k=50, m=1,
             masked=0.0),
        # 512 different configurations out of each of 8 screened batches
        dict(name="sample-batches-8x1048576", op="sample", rows=8, n=1048576, type="f32", rule="top_k", k=8192, m=512,
             masked=0.6),
        # 1,024 different configurations out of the whole screened knob space
        dict(name="sample-space-1x16777216", op="sample", rows=1, n=16777216, type="f32", rule="min_p", k=0, m=1024,
             masked=0.5),
        # the tokens of one decoding step
        dict(name="embed-step-64x1024", op="embed", tokens=64, vocab=50021, dim=1024, type="bf16", skew=1.0),
        # the tokens of a prefilled batch
        dict(name="embed-prompt-32768x2048", op="embed", tokens=32768, vocab=32003, dim=2048, type="bf16", skew=1.0),
        # training on text-like tokens: many rare ones, few very frequent ones
        dict(name="embed-grad-32768x2048", op="embed_grad", tokens=32768, vocab=32003, dim=2048, type="bf16",
             skew=1.0),
        # training on decoded candidates: 8 knobs of 8 options, every row hit 16,384 times
        dict(name="embed-grad-knobs-1048573x128", op="embed_grad", tokens=1048573, vocab=64, dim=128, type="f32",
             skew=0.0),
        # one token for each of 512 chains
        dict(name="scan-step-512x2048", op="scan", batch=512, length=1, dim=2048, states=16, groups=1, taps=4,
             type="bf16", ragged=False),
        # prompts of different lengths
        dict(name="scan-prompts-8x2048x2048", op="scan", batch=8, length=2048, dim=2048, states=16, groups=1, taps=4,
             type="bf16", ragged=True),
        # one long tuning history
        dict(name="scan-history-1x16381x1024", op="scan", batch=1, length=16381, dim=1024, states=16, groups=2, taps=4,
             type="f32", ragged=False),
        # one training batch
        dict(name="scan-grad-4x1021x1024", op="scan_grad", batch=4, length=1021, dim=1024, states=16, groups=1, taps=4,
             type="bf16", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("sample", "sample", "embed", "embed_grad", "scan", "scan", "scan_grad"))
    kind = rng.choice(("f32", "bf16", "f16"))
    if op == "sample":
        n = _log_int(rng, 1, 16777216)
        rows = _log_int(rng, 1, max(1, min(65536, 8388608 // n)))
        rule = rng.choice(("greedy", "plain", "top_k", "top_p", "min_p", "mixed"))
        if rule in ("top_p", "mixed"):
            # a nucleus ends where a 32-bit sum says so: one draw a row, rows of a vocabulary's size
            n, m = min(n, 262144), 1
        else:
            m = _log_int(rng, 1, min(1024, n)) if rng.random() < 0.5 else 1
        return dict(op=op, rows=rows, n=n, type="f32" if m > 1 else kind, rule=rule, k=_log_int(rng, 1, min(n, 4096)),
                    m=m, masked=rng.choice((0.0, 0.1, 0.6, 0.99)))
    if op in ("embed", "embed_grad"):
        dim = _log_int(rng, 1, 4096)
        vocab = _log_int(rng, 2, min(131072, 67108864 // dim))
        tokens = _log_int(rng, 1, min(1048576, 67108864 // dim))
        return dict(op=op, tokens=tokens, vocab=vocab, dim=dim, type=kind, skew=rng.choice((0.0, 0.7, 1.0, 1.3)))
    states = rng.choice((1, 4, 8, 13, 16, 16, 32))
    groups = rng.choice((1, 1, 2, 4))
    most = 67108864 if op == "scan_grad" else 268435456  # state updates of the plain form
    length = 1 if op == "scan" and rng.random() < 0.4 else _log_int(rng, 1, 16384)
    dim = groups * _log_int(rng, 1, max(1, min(4096, most // (length * states)) // groups))
    batch = _log_int(rng, 1, max(1, min(512, most // (length * states * dim))))
    return dict(op=op, batch=batch, length=length, dim=dim, states=states, groups=groups, taps=rng.choice((0, 2, 3, 4, 4)),
                type=kind, ragged=rng.random() < 0.5)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 17)
    return g


def _rules(case, g):
    """int32 [rows][4]: the bits of temperature, top_k, top_p, min_p."""
    rows, k, rule = case["rows"], case["k"], case["rule"]
    u = torch.rand(rows, generator=g, device="cuda")
    t = 0.5 + u
    kk = torch.zeros(rows, dtype=torch.int32, device="cuda")
    p = torch.ones(rows, device="cuda")
    mp = torch.zeros(rows, device="cuda")
    j = torch.arange(rows, device="cuda") % 8 if rule == "mixed" else None

    def rows_of(name, places):
        if rule == name:
            return torch.ones(rows, dtype=torch.bool, device="cuda")
        return torch.isin(j, torch.tensor(places, device="cuda")) if rule == "mixed" else kk > 0

    t = torch.where(rows_of("greedy", [0]), 0.0, t)
    kk = torch.where(rows_of("top_k", [1, 5, 7]), k, kk)
    p = torch.where(rows_of("top_p", [2, 3, 5, 7]), 0.7 + 0.29 * torch.rand(rows, generator=g, device="cuda"), p)
    mp = torch.where(rows_of("min_p", [4, 6, 7]), 0.02 + 0.1 * torch.rand(rows, generator=g, device="cuda"), mp)
    return torch.stack([t.view(torch.int32), kk.to(torch.int32), p.view(torch.int32), mp.view(torch.int32)],
                       1).contiguous()


def prepare(case, seed):
    g = _generator(seed)
    dt = TYPES[case["type"]]
    rnd = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    if case["op"] == "sample":
        rows, n = case["rows"], case["n"]
        s = rnd(rows, n) * 2.5
        if case["masked"]:  # rejected candidates score -infinity; a row may have none left
            s = torch.where(torch.rand(rows, n, generator=g, device="cuda") < case["masked"], -math.inf, s)
        # Gumbel numbers, -log of a standard exponential one
        noise = -torch.empty(rows, n, device="cuda").exponential_(generator=g).log()
        return dict(case, scores=s.to(dt), noise=noise, rules=_rules(case, g))
    if case["op"] in ("embed", "embed_grad"):
        v, tokens, dim = case["vocab"], case["tokens"], case["dim"]
        w = torch.arange(1, v + 1, device="cuda", dtype=torch.float64) ** -case["skew"]
        c = w.cumsum(0)
        u = torch.rand(tokens, generator=g, device="cuda", dtype=torch.float64) * c[-1]
        place = torch.randperm(v, generator=g, device="cuda")
        ids = place[torch.searchsorted(c, u).clamp_(max=v - 1)]
        ids = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.02, -1, ids)  # padding
        st = dict(case, ids=ids, scale=math.sqrt(dim))
        if case["op"] == "embed":
            st["table"] = (rnd(v, dim) * dim ** -0.5).to(dt)
        else:
            st["grad"] = rnd(tokens, dim).to(dt)
        return st
    b, L, d, s, gr, k = (case[x] for x in ("batch", "length", "dim", "states", "groups", "taps"))
    st = dict(case)
    st["x"], st["z"] = rnd(b, L, d).to(dt), rnd(b, L, d).to(dt)
    # step sizes after softplus spread over about 0.001 .. 0.1
    st["dt"] = (rnd(b, L, d) * 0.5).to(dt)
    step = torch.exp(torch.rand(d, generator=g, device="cuda") * math.log(100.0) + math.log(0.001))
    st["dt_bias"] = torch.log(torch.expm1(step))
    st["B"], st["C"] = rnd(b, L, gr, s).to(dt), rnd(b, L, gr, s).to(dt)
    st["A"] = -torch.arange(1, s + 1, device="cuda", dtype=torch.float32).repeat(d, 1) * (1 + 0.1 * torch.rand(
        d, s, generator=g, device="cuda"))
    st["skip"] = 1 + 0.1 * rnd(d)
    st["conv_w"] = rnd(d, k) * 0.5 if k else None
    st["conv_b"] = rnd(d) * 0.1 if k else None
    st["state"] = rnd(b, d, s) * 0.3
    st["conv_state"] = rnd(b, k - 1, d).to(dt) if k > 1 else None
    st["lengths"] = None
    if case["ragged"]:
        st["lengths"] = torch.randint(0, L + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
        st["lengths"][0] = L
    if case["op"] == "scan_grad":
        st["gy"] = rnd(b, L, d).to(dt)
        st["g_state"] = rnd(b, d, s)
    return st


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------

def _plain_sample(st):
    x, noise, m = st["scores"], st["noise"], st["m"]
    rules = st["rules"]
    t, p, mp = (rules[:, j].contiguous().view(torch.float32)[:, None] for j in (0, 2, 3))
    k = rules[:, 1:2]
    n = x.shape[1]
    greedy = t == 0
    s = x.float() * (1.0 / torch.where(greedy, 1.0, t))
    out = torch.isnan(s) | (x == -math.inf)
    s = s.clamp(-FLT_MAX, FLT_MAX).masked_fill(out, -math.inf) + 0.0
    k = torch.where(greedy, 1, torch.where((k <= 0) | (k > n), n, k))
    ranked, order = torch.sort(s, dim=1, descending=True, stable=True)
    top = ranked[:, :1]
    top = torch.where(top == -math.inf, 0.0, top)
    w = torch.exp(ranked - top)
    total = w.sum(1, keepdim=True)
    first = torch.arange(n, device=x.device)[None] < k
    w = torch.where(first, w, 0.0)
    before = w.cumsum(1) - w
    keep = first & (ranked > -math.inf)
    keep &= (p >= 1) | greedy | (before < p * w.sum(1, keepdim=True))
    keep &= (mp <= 0) | greedy | (ranked - top >= torch.log(mp))
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    key = torch.where(greedy, s, s + noise)
    key = torch.nan_to_num(key, nan=-FLT_MAX, posinf=FLT_MAX, neginf=-FLT_MAX).masked_fill(~kept, -math.inf)
    best, index = torch.sort(key, dim=1, descending=True, stable=True)
    best, index = best[:, :m], index[:, :m]
    none = best == -math.inf
    logp = torch.gather(s, 1, index) - top - torch.log(total)
    logp = torch.where(greedy, 0.0, logp).masked_fill(none, -math.inf)
    return {"index": index.masked_fill(none, -1), "logprob": logp}


def _plain_embed(st):
    ids, table = st["ids"], st["table"]
    rows = table[ids.clamp(min=0)].float() * st["scale"]
    return torch.where(ids[:, None] >= 0, rows, 0.0).to(table.dtype)


def _plain_embed_grad(st):
    ids, grad = st["ids"], st["grad"]
    g = torch.zeros(st["vocab"], grad.shape[1], device=grad.device)
    g.index_add_(0, ids.clamp(min=0), torch.where(ids[:, None] >= 0, grad.float(), 0.0))
    return (g * st["scale"]).to(grad.dtype)


def _doubling(a, b):
    """h[t] = a[t] h[t-1] + b[t] along dimension 1 from h = 0, in log2(L) steps."""
    step = 1
    while step < a.shape[1]:
        b = torch.cat([b[:, :step], b[:, step:] + a[:, step:] * b[:, :-step]], 1)
        a = torch.cat([a[:, :step], a[:, step:] * a[:, :-step]], 1)
        step *= 2
    return b


def _plain_scan_parts(st):
    f = lambda name: None if st[name] is None else st[name].float()  # noqa: E731
    x, z, B, C, A = f("x"), f("z"), f("B"), f("C"), st["A"]
    b, L, d = x.shape
    taps = st["taps"]
    lengths = st["lengths"]
    live = torch.ones(b, L, 1, dtype=torch.bool, device=x.device) if lengths is None else (
        torch.arange(L, device=x.device)[None] < lengths[:, None])[..., None]
    q = {"live": live}
    x = torch.where(live, x, 0.0)
    past = x
    if taps:
        if taps > 1:
            past = torch.cat([f("conv_state"), x], 1)
        v = sum(past[:, j:j + L] * st["conv_w"][:, j] for j in range(taps)) + st["conv_b"]
        u = v * torch.sigmoid(v)
        q.update(v=v)
    else:
        u = x
    raw = f("dt") + st["dt_bias"]
    step = torch.where(live, raw.clamp(min=0) + torch.log1p(torch.exp(-raw.abs())), 0.0)
    u = torch.where(live, u, 0.0)
    Bd = torch.where(live[..., None], B, 0.0).repeat_interleave(d // B.shape[2], 2)
    Cd = torch.where(live[..., None], C, 0.0).repeat_interleave(d // C.shape[2], 2)
    a = torch.exp(step[..., None] * A)
    push = (step * u)[..., None] * Bd
    push[:, 0] += a[:, 0] * st["state"]
    h = _doubling(a, push)
    y = (h * Cd).sum(-1) + st["skip"] * u
    q.update(past=past, u=u, raw=raw, step=step, B=Bd, C=Cd, a=a, h=h, y=y, z=torch.where(live, z, 0.0))
    return q


def _last_inputs(past, lengths, taps):
    """The taps - 1 inputs before each sequence's end."""
    n = past.shape[1] - (taps - 1)
    end = torch.full((past.shape[0],), n, device=past.device) if lengths is None else lengths.long()
    at = end[:, None] + torch.arange(taps - 1, device=past.device)
    return torch.gather(past, 1, at[..., None].expand(-1, -1, past.shape[2]))


def _plain_scan(st):
    q = _plain_scan_parts(st)
    dt = st["x"].dtype
    out = {"y": (q["y"] * q["z"] * torch.sigmoid(q["z"])).to(dt), "state": q["h"][:, -1].contiguous()}
    if st["taps"] > 1:
        out["conv_state"] = _last_inputs(q["past"], st["lengths"], st["taps"]).to(dt)
    return out


def _plain_scan_grad(st):
    q = _plain_scan_parts(st)
    dt = st["x"].dtype
    live, z, a, h, taps = q["live"], q["z"], q["a"], q["h"], st["taps"]
    b, L, d = z.shape
    gr, n = st["B"].shape[2:]
    go = torch.where(live, st["gy"].float(), 0.0)
    sg = torch.sigmoid(z)
    gz = go * q["y"] * sg * (1 + z * (1 - sg))
    gy = go * z * sg
    push = gy[..., None] * q["C"]
    push[:, -1] += st["g_state"]
    after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    g = _doubling(after.flip(1), push.flip(1)).flip(1)
    prev = torch.cat([st["state"][:, None], h[:, :-1]], 1)
    ga = g * prev * a
    gB = (g * (q["step"] * q["u"])[..., None]).reshape(b, L, gr, d // gr, n).sum(3)
    gC = (gy[..., None] * h).reshape(b, L, gr, d // gr, n).sum(3)
    gp = (g * q["B"]).sum(-1)
    gu = torch.where(live, gp * q["step"] + gy * st["skip"], 0.0)
    gstep = gp * q["u"] + (ga * st["A"]).sum(-1)
    graw = torch.where(live, gstep * torch.sigmoid(q["raw"]), 0.0)
    out = {"z": gz.to(dt), "dt": graw.to(dt), "B": gB.to(dt), "C": gC.to(dt), "A": (ga * q["step"][..., None]).sum((0, 1)),
           "skip": (gy * q["u"]).sum((0, 1)), "dt_bias": graw.sum((0, 1)), "state": a[:, 0] * g[:, 0]}
    if taps:
        sv = torch.sigmoid(q["v"])
        gv = gu * sv * (1 + q["v"] * (1 - sv))
        gpast = torch.zeros_like(q["past"])
        cols = []
        for j in range(taps):
            gpast[:, j:j + L] += gv * st["conv_w"][:, j]
            cols.append((gv * q["past"][:, j:j + L]).sum((0, 1)))
        out.update(conv_w=torch.stack(cols, 1), conv_b=gv.sum((0, 1)))
        if taps > 1:
            out["conv_state"] = gpast[:, :taps - 1].to(dt)
        out["x"] = torch.where(live, gpast[:, taps - 1:], 0.0).to(dt)
    else:
        out["x"] = gu.to(dt)
    return out


# ---------------------------------------------------------------------------
# Passes
# ---------------------------------------------------------------------------

_SCAN = ("x", "dt", "B", "C", "A")
_SCAN_MORE = ("z", "skip", "dt_bias", "conv_w", "conv_b", "lengths", "state", "conv_state")


def run(state):
    op = state["op"]
    if not own:
        return {"sample": _plain_sample, "embed": _plain_embed, "embed_grad": _plain_embed_grad, "scan": _plain_scan,
                "scan_grad": _plain_scan_grad}[op](state)
    from paper_2411_10764_gb300 import mlt

    if op == "sample":
        index, logprob = mlt.sample(state["scores"], state["noise"], rules=state["rules"], m=state["m"])
        return {"index": index, "logprob": logprob}
    if op == "embed":
        return mlt.embed(state["ids"], state["table"], scale=state["scale"])
    if op == "embed_grad":
        return mlt.embed_grad(state["ids"], state["grad"], state["vocab"], scale=state["scale"])
    args = [state[k] for k in _SCAN]
    more = {k: state[k] for k in _SCAN_MORE}
    if op == "scan":
        y, h, c = mlt.scan(*args, **more)
        return {"y": y, "state": h} if c is None else {"y": y, "state": h, "conv_state": c}
    g = mlt.scan_grad(state["gy"], *args, g_state=state["g_state"], **more)
    return {k: v for k, v in g.items() if v is not None}


def work(case):
    e = SIZE[case["type"]]
    if case["op"] == "sample":
        rows, n, m, k = case["rows"], case["n"], case["m"], case["k"]
        # noise that has to be read: all of it where nothing is cut, the k best's under
        # top_k; how much a nucleus keeps depends on the scores and counts as nothing
        kinds = {"greedy": 0, "plain": n, "top_k": k, "top_p": 0, "min_p": 0, "mixed": 0}
        return {"bytes": rows * (n * e + kinds[case["rule"]] * 4 + 16 + m * 12), "flops": 4.0 * rows * n}
    if case["op"] == "embed":
        tokens, dim = case["tokens"], case["dim"]
        w = np.arange(1, case["vocab"] + 1) ** -case["skew"]
        rows = -np.expm1(0.98 * tokens * np.log1p(-w / w.sum())).sum()  # expected distinct ones
        return {"bytes": tokens * (8 + dim * e) + float(rows) * dim * e, "flops": tokens * dim}
    if case["op"] == "embed_grad":
        tokens, dim = case["tokens"], case["dim"]
        return {"bytes": tokens * (8 + dim * e) + case["vocab"] * dim * e, "flops": tokens * dim}
    b, L, d, s, g, k = (case[x] for x in ("batch", "length", "dim", "states", "groups", "taps"))
    # half of the positions of ragged batches lie past their sequence's end; outputs are written everywhere
    live = b * L * (0.5 + 0.5 / b if case["ragged"] else 1.0)
    state = b * d * s * 4 + b * max(0, k - 1) * d * e
    weights = d * (s + 2 + (k + 1 if k else 0)) * 4
    if case["op"] == "scan":
        return {"bytes": live * (3 * d + 2 * g * s) * e + b * L * d * e + 2 * state + weights,
                "flops": live * d * (7.0 * s + 20)}
    return {"bytes": (live + b * L) * (3 * d + 2 * g * s) * e + live * d * e + 2 * state + b * d * s * 4 + 2 * weights,
            "flops": live * d * (22.0 * s + 60)}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def _np(t):
    return None if t is None else (t.float() if t.is_floating_point() else t).cpu().numpy()


def _exact_sample(st):
    x, noise, m = _np(st["scores"]), _np(st["noise"]), st["m"]
    raw = st["rules"].cpu().numpy()
    rows, n = x.shape
    logp = np.full((rows, min(m, n)), -np.inf)
    fmax = np.float32(FLT_MAX)
    for r in range(rows):
        t, p, mp = (raw[r, [0, 2, 3]].view(np.float32)).astype(np.float64)
        k = int(raw[r, 1])
        with np.errstate(over="ignore", invalid="ignore"):
            # the scaled score is defined as a 32-bit product, its key as a 32-bit sum
            s = np.clip(x[r] * (np.float32(1) / np.float32(t if t > 0 else 1)), -fmax, fmax)
            key = np.clip(np.nan_to_num(s + noise[r], nan=-fmax, posinf=fmax, neginf=-fmax), -fmax, fmax)
        alive = np.flatnonzero(~np.isnan(x[r]) & (x[r] > -np.inf))
        if not alive.size:
            continue
        sd = s[alive].astype(np.float64)
        if t == 0:
            logp[r, 0] = 0.0
            continue
        w = np.exp(sd - sd.max())
        total = w.sum()
        order = np.argsort(-sd, kind="stable")
        if 0 < k < order.size:
            order = order[:k]
        ws = w[order]
        if p < 1:
            order = order[np.cumsum(ws) - ws < p * ws.sum()]
        if mp > 0:
            order = order[sd[order] - sd.max() >= math.log(mp)]
        kept = np.sort(alive[order])
        best = kept[np.argsort(-key[kept], kind="stable")[:m]]
        logp[r, :best.size] = s[best].astype(np.float64) - sd.max() - math.log(total)
    return {"index": None, "logprob": logp}


def _exact_embed(st):
    ids = _np(st["ids"])
    rows = _np(st["table"])[np.maximum(ids, 0)].astype(np.float64) * float(np.float32(st["scale"]))
    rows[ids < 0] = 0
    return rows


def _exact_embed_grad(st):
    ids, grad = _np(st["ids"]), _np(st["grad"])
    out = np.zeros((st["vocab"], grad.shape[1]))
    order = np.argsort(ids, kind="stable")
    order = order[ids[order] >= 0]
    if order.size:
        s = ids[order]
        starts = np.flatnonzero(np.r_[True, s[1:] != s[:-1]])
        ends = np.r_[starts[1:], s.size]
        for a, b in zip(starts, ends):
            out[s[a]] = grad[order[a:b]].sum(0, dtype=np.float64)
    return out * float(np.float32(st["scale"]))


def _sigmoid(v):
    return 0.5 * (1 + np.tanh(0.5 * v))


def _exact_scan(st, backward):
    """Sequence by sequence and step by step; the gradient by the chain rule on the recurrence."""
    w = {k: _np(v) if isinstance(v, torch.Tensor) else v for k, v in st.items()}
    w = {k: v.astype(np.float64) if isinstance(v, np.ndarray) and v.dtype == np.float32 else v for k, v in w.items()}
    nb, L, d = w["x"].shape
    gr, n = w["B"].shape[2:]
    k = w["taps"]
    group = np.arange(d) // (d // gr)
    y = np.zeros((nb, L, d))
    end_state, end_conv = w["state"].copy(), None if k < 2 else w["conv_state"].copy()
    if backward:
        G = {i: np.zeros_like(w[i]) for i in ("x", "z", "dt", "B", "C", "A", "skip", "dt_bias")}
        G["state"] = w["g_state"].copy()
        if k:
            G.update(conv_w=np.zeros((d, k)), conv_b=np.zeros(d))
        if k > 1:
            G["conv_state"] = np.zeros_like(w["conv_state"])
    for i in range(nb):
        T = L if w["lengths"] is None else int(w["lengths"][i])
        if T == 0:
            continue
        x = w["x"][i, :T]
        past = x if k < 2 else np.concatenate([w["conv_state"][i], x])
        if k:
            v = sum(past[j:j + T] * w["conv_w"][:, j] for j in range(k)) + w["conv_b"]
            u = v * _sigmoid(v)
        else:
            u = x
        raw = w["dt"][i, :T] + w["dt_bias"]
        step = np.logaddexp(0.0, raw)
        z = w["z"][i, :T]
        B, C = w["B"][i, :T], w["C"][i, :T]
        h = w["state"][i].copy()
        hs = np.empty((T + 1, d, n)) if backward else None
        core = np.empty((T, d))
        if backward:
            hs[0] = h
        for t in range(T):
            h = np.exp(step[t][:, None] * w["A"]) * h + (step[t] * u[t])[:, None] * B[t][group]
            core[t] = (h * C[t][group]).sum(1) + w["skip"] * u[t]
            if backward:
                hs[t + 1] = h
        y[i, :T] = core * z * _sigmoid(z)
        end_state[i] = h
        if k > 1:
            end_conv[i] = past[T:]
        if not backward:
            continue
        go, sz = w["gy"][i, :T], _sigmoid(z)
        G["z"][i, :T] = go * core * sz * (1 + z * (1 - sz))
        gc = go * z * sz
        g = w["g_state"][i].copy()
        gu, gs = np.empty((T, d)), np.empty((T, d))
        for t in range(T - 1, -1, -1):
            g += gc[t][:, None] * C[t][group]
            a = np.exp(step[t][:, None] * w["A"])
            G["C"][i, t] = (gc[t][:, None] * hs[t + 1]).reshape(gr, d // gr, n).sum(1)
            G["B"][i, t] = (g * (step[t] * u[t])[:, None]).reshape(gr, d // gr, n).sum(1)
            gp = (g * B[t][group]).sum(1)
            gu[t] = gp * step[t] + gc[t] * w["skip"]
            e = g * hs[t] * a
            gs[t] = gp * u[t] + (e * w["A"]).sum(1)
            G["A"] += e * step[t][:, None]
            g = g * a
        G["state"][i] = g
        G["skip"] += (gc * u).sum(0)
        graw = gs * _sigmoid(raw)
        G["dt"][i, :T] = graw
        G["dt_bias"] += graw.sum(0)
        if k:
            sv = _sigmoid(v)
            gv = gu * sv * (1 + v * (1 - sv))
            gpast = np.zeros_like(past)
            for j in range(k):
                gpast[j:j + T] += gv * w["conv_w"][:, j]
                G["conv_w"][:, j] += (gv * past[j:j + T]).sum(0)
            G["conv_b"] += gv.sum(0)
            if k > 1:
                G["conv_state"][i] = gpast[:k - 1]
            G["x"][i, :T] = gpast[max(0, k - 1):]
        else:
            G["x"][i, :T] = gu
    if backward:
        return G
    return {"y": y, "state": end_state} if end_conv is None else {"y": y, "state": end_state, "conv_state": end_conv}


def exact(case, seed):
    op = case["op"]
    if op in ("scan", "scan_grad"):
        cost = case["batch"] * case["length"] * (case["dim"] * case["states"] + 2000) * (3 if op == "scan_grad" else 1)
        if cost > 700e6:
            return None
    st = prepare(case, seed)
    if op == "sample":
        return _exact_sample(st)
    if op == "embed":
        return _exact_embed(st)
    if op == "embed_grad":
        return _exact_embed_grad(st)
    return _exact_scan(st, op == "scan_grad")
