"""A small learned proposer of candidate configurations.

The paper leaves the explorer's search open (ML^2Tuner Sec. 2, "Configuration
Explorer") and retrains its models every tuning iteration.  This one proposes:
a recurrent model reads a configuration's knob digits as tokens and gives, knob by
knob, scores for the next digit.  It puts the library's sequence operators
together as a user would:

    screen a part of the knob space         mlt.screen_decoded
    draw from its scores, not only the best mlt.sample (rejected ones score -inf)
    train the proposer on the draws         mlt.embed, mlt.scan and their gradients
    propose, digit by digit                 mlt.embed, mlt.scan in place, mlt.sample
    anneal from the proposals               mlt.sa_step

    python -m paper_2411_10764_gb300.proposer

Matrix products are torch's.  B, C and the step sizes are projected from the
embedded tokens, so that the short convolution stays inside mlt.scan.
"""
from __future__ import annotations

import math

import numpy as np

from . import mlt

TAPS = 4


class Proposer:
    """Embedding -> selective scan with gate -> residual -> scores of digits, in fp32.

    radices: options of each knob (knob 0 least significant).  Token of digit d of knob
    j: offset_j + d; the last token starts a sequence."""

    def __init__(self, radices, dim: int = 64, inner: int = 128, states: int = 16, seed: int = 0, device="cuda"):
        import torch

        self.radices = [int(r) for r in radices]
        self.offsets = np.concatenate([[0], np.cumsum(self.radices)]).astype(int).tolist()
        self.vocab = self.offsets[-1] + 1
        self.dim, self.inner, self.states = dim, inner, states
        g = torch.Generator(device="cpu")
        g.manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        step = torch.exp(torch.rand(inner, generator=g) * math.log(100.0) + math.log(0.001))
        p = dict(
            table=r(self.vocab, dim) / dim,
            w_in=r(dim, 3 * inner + 2 * states) / math.sqrt(dim),
            conv_w=r(inner, TAPS) / math.sqrt(TAPS),
            conv_b=torch.zeros(inner),
            A=-torch.arange(1, states + 1, dtype=torch.float32).repeat(inner, 1),
            skip=torch.ones(inner),
            dt_bias=torch.log(torch.expm1(step)),
            w_out=r(inner, dim) / math.sqrt(inner),
            head=r(dim, self.vocab - 1) / math.sqrt(dim),
        )
        self.params = {k: v.to(device).contiguous() for k, v in p.items()}

    # -- candidates and tokens ------------------------------------------------
    def tokens_of(self, index):
        """Start token and digits of candidates (int64 tensor [m]): [m][knobs + 1]."""
        import torch

        cols, rest = [torch.full_like(index, self.vocab - 1)], index
        for j, r in enumerate(self.radices):
            cols.append(rest % r + self.offsets[j])
            rest = rest // r
        return torch.stack(cols, 1)

    # -- the model ------------------------------------------------------------
    def _scan_inputs(self, e):
        """Views of one projection: x, z, dt, B, C."""
        p, i, n = e @ self.params["w_in"], self.inner, self.states
        return p, (p[..., :i], p[..., 2 * i:3 * i], p[..., 3 * i:3 * i + n], p[..., 3 * i + n:], p[..., i:2 * i])

    def forward(self, tokens, state=None, conv_state=None, in_place: bool = False):
        """Scores of the next digit [m][length][digits], the states, and what backward needs."""
        P = self.params
        e = mlt.embed(tokens, P["table"], scale=math.sqrt(self.dim))
        _, (x, dt, B, C, z) = self._scan_inputs(e)
        args = dict(z=z, skip=P["skip"], dt_bias=P["dt_bias"], conv_w=P["conv_w"], conv_b=P["conv_b"], state=state,
                    conv_state=conv_state)
        outs = dict(state_out=state, conv_state_out=conv_state) if in_place else {}
        y, state, conv_state = mlt.scan(x, dt, B, C, P["A"], **args, **outs)
        o = e + y @ P["w_out"]
        return o @ P["head"], state, conv_state, (tokens, e, x, dt, B, C, args, y, o)

    def loss_and_grads(self, index, weight=None):
        """Mean negative log-likelihood of candidates' digits (weighted) and its gradients."""
        import torch

        P = self.params
        tokens = self.tokens_of(index)
        scores, _, _, (_, e, x, dt, B, C, args, y, o) = self.forward(tokens[:, :-1].contiguous())
        # a position's digits are those of its knob
        at = torch.arange(self.vocab - 1, device=index.device)
        lo = torch.tensor(self.offsets[:-1], device=index.device)[:, None]
        hi = torch.tensor(self.offsets[1:], device=index.device)[:, None]
        logp = scores.masked_fill(~((at >= lo) & (at < hi)), -math.inf).log_softmax(-1)
        w = torch.ones(index.numel(), device=index.device) if weight is None else weight
        w = (w / (w.sum() * len(self.radices)))[:, None, None]
        want = torch.nn.functional.one_hot(tokens[:, 1:], self.vocab - 1)
        loss = -(torch.where(want > 0, logp, 0.0) * w).sum()
        gs = (logp.exp() - want) * w
        flat = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
        go = gs @ P["head"].t()
        grads = {"head": flat(o).t() @ flat(gs), "w_out": flat(y).t() @ flat(go)}
        s = mlt.scan_grad(go @ P["w_out"].t(), x, dt, B, C, P["A"], **args)
        for k in ("A", "skip", "dt_bias", "conv_w", "conv_b"):
            grads[k] = s[k]
        gp = torch.cat([s["x"], s["z"], s["dt"], s["B"], s["C"]], -1)
        grads["w_in"] = flat(e).t() @ flat(gp)
        ge = go + gp @ P["w_in"].t()
        grads["table"] = mlt.embed_grad(tokens[:, :-1].contiguous(), ge, self.vocab, scale=math.sqrt(self.dim))
        return loss, grads

    def train(self, index, weight=None, steps: int = 20, lr: float = 0.005):
        """Gradient steps scaled by each parameter's own root mean square; returns the losses."""
        losses = []
        mean = {k: v.new_zeros(v.shape) for k, v in self.params.items()}
        for t in range(steps):
            loss, grads = self.loss_and_grads(index, weight)
            losses.append(loss)
            for k, g in grads.items():
                mean[k].mul_(0.9).addcmul_(g, g, value=0.1)
                scale = (mean[k] / (1 - 0.9 ** (t + 1))).sqrt_().add_(1e-8)
                self.params[k].addcdiv_(g, scale, value=-lr * (0.1 if k in ("A", "dt_bias") else 1.0))
            self.params["A"].clamp_(max=-1e-3)
        return [float(v) for v in losses]

    def propose(self, m: int, generator=None, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0,
                min_p: float = 0.0):
        """m candidates drawn digit by digit: (indices int64 [m], log-probabilities [m])."""
        import torch

        P = self.params
        device = P["table"].device
        state = torch.zeros((m, self.inner, self.states), device=device)
        conv = torch.zeros((m, TAPS - 1, self.inner), device=device)
        token = torch.full((m, 1), self.vocab - 1, dtype=torch.int64, device=device)
        index = torch.zeros(m, dtype=torch.int64, device=device)
        logp, place = torch.zeros(m, device=device), 1
        for j, r in enumerate(self.radices):
            scores, _, _, _ = self.forward(token, state, conv, in_place=True)
            noise = -torch.empty((m, r), device=device).exponential_(generator=generator).log()
            digit, lp = mlt.sample(scores[:, 0, self.offsets[j]:self.offsets[j + 1]], noise, temperature, top_k, top_p,
                                   min_p)
            index += digit[:, 0] * place
            logp += lp[:, 0]
            place *= r
            token = digit + self.offsets[j]
        return index, logp


def explore(decoder, thr: float, first: int, n: int, keep: int = 256, chains: int = 1024, temperature: float = 0.05,
            seed: int = 0, steps: int = 20):
    """One round over a knob space whose V and P models are loaded: screen candidates first ..
    first + n - 1, draw `keep` of the valid ones by their scores, train a proposer on them, and
    anneal one step from its proposals.  Returns a dict of tensors and the losses."""
    import torch

    r, ov, prog = decoder.radices, decoder.option_values, decoder.program
    _, perf, topk = mlt.screen_decoded(r, ov, prog, first, n, thr, keep)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    noise = -torch.empty(n, device="cuda").exponential_(generator=g).log()
    drawn, logp = mlt.sample(perf, noise, temperature=temperature, m=keep)
    drawn = drawn[drawn >= 0]
    model = Proposer(r, seed=seed)
    losses = model.train(drawn + first, steps=steps) if drawn.numel() else []
    parent, _ = model.propose(chains, g, temperature=0.8, top_p=0.95)
    draw = lambda: torch.randint(0, 1 << 30, (chains,), dtype=torch.int32, device="cuda", generator=g)  # noqa: E731
    log_u = torch.rand(chains, device="cuda", generator=g).log()
    nxt, score, accepted = mlt.sa_step(r, ov, prog, parent, torch.full((chains,), -1e30, device="cuda"), draw(), draw(),
                                       log_u, 1.0, thr)
    mlt.sync_status()
    return dict(topk=topk, drawn=drawn, logprob=logp, proposed=parent, next=nxt, score=score, accepted=accepted,
                losses=losses, perf=perf)


def main() -> None:
    from . import workloads as W

    w = W.make_workload(4, seed=1, n=65536)
    mlt.load_workload_models(w)
    out = explore(w.decoder, w.thr, 0, 65536)
    ok, losses, screened = out["accepted"].bool(), out["losses"], float(out["perf"].max())
    print(f"screened 65536, drew {out['drawn'].numel()}"
          + (f", loss {losses[0]:.3f} -> {losses[-1]:.3f}" if losses else "")
          + f", {int(ok.sum())} of {ok.numel()} annealed proposals valid"
          + (f", best score {float(out['score'][ok].max()):.4f}" if bool(ok.any()) else "")
          + (f" (screened: {screened:.4f})" if math.isfinite(screened) else " (screened: none valid)"))


if __name__ == "__main__":
    main()
