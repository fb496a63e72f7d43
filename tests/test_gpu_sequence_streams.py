"""The sequence operators given a stream other than the current one, while work queued on the
current one still uses memory that is free again; and states updated in place."""
import pytest

from paper_2411_10764_gb300 import mlt
from test_gpu_scan import call, make

pytestmark = pytest.mark.gpu

ROWS = 1 << 24  # fp32 values of a block that the calls' memory may be taken from: 64 MB


def _calls():
    """Calls by name, each with memory of its own of some megabytes; the results as one tuple."""
    import torch

    gen = torch.Generator("cuda").manual_seed(3)
    ids = torch.randint(0, 1000, (1 << 20,), device="cuda", generator=gen)
    grad = torch.randn((1 << 20, 4), device="cuda", generator=gen)
    table = torch.randn((1000, 8), device="cuda", generator=gen)
    scores = torch.randn((8192, 100), device="cuda", generator=gen)
    noise = torch.randn((8192, 100), device="cuda", generator=gen)
    t = make(1, 3001, 512, 16, kind="f32")
    more = {k: v for k, v in t.items() if k not in ("x", "dt", "B", "C", "A")}
    five = [t[k] for k in ("x", "dt", "B", "C", "A")]

    def grads(**kw):
        g = mlt.scan_grad(t["x"], *five, **more, **kw)
        return tuple(v for v in g.values() if v is not None)

    return {"sample": lambda **kw: mlt.sample(scores, noise, m=64, **kw),
            "embed": lambda **kw: (mlt.embed(ids, table, **kw),),
            "embed_grad": lambda **kw: (mlt.embed_grad(ids, grad, 1000, **kw),),
            "embed_grad_copy": lambda **kw: (mlt.embed_grad(ids[:1 << 19].view(-1, 2), grad.view(2, -1, 4)
                                                            .transpose(0, 1)[:1 << 18], 1000, **kw),),
            "scan": lambda **kw: mlt.scan(*five, **more, **kw),
            "scan_grad": grads}


@pytest.mark.parametrize("name", ["sample", "embed", "embed_grad", "embed_grad_copy", "scan", "scan_grad"])
def test_another_stream_leaves_memory_in_use_alone(name):
    import torch

    run = _calls()[name]
    s = torch.cuda.Stream()
    want = tuple(w.clone() for w in run())
    run(stream=s)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    hold = torch.ones(ROWS, device="cuda")
    total = torch.empty((), device="cuda", dtype=torch.float64)
    hold.sum(dtype=torch.float64)  # so that the sum below allocates nothing new
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)  # about 10 ms
    torch.sum(hold, dtype=torch.float64, dim=0, out=total)
    hold.fill_(7.0)
    del hold
    got = run(stream=s)
    torch.cuda.synchronize()
    assert total.item() == ROWS
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_inputs_are_kept_until_the_stream_is_done():
    import torch

    ids = torch.arange(1 << 20, device="cuda")
    table = torch.ones((1 << 20, 16), device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
    got = mlt.embed(ids, table, stream=s)
    del table
    other = torch.zeros((1 << 20, 16), device="cuda")
    torch.cuda.synchronize()
    assert (got == 1).all() and (other == 0).all()


@pytest.mark.parametrize("b,L,d,taps", [(1, 700, 64, 4), (3, 2, 64, 4), (300, 40, 64, 3), (2, 0, 64, 4)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_states_in_place_at_every_length(b, L, d, taps, kind):
    import torch

    t = make(b, L, d, 16, 1, taps, kind, ragged=True)
    want = [w.clone() for w in call(t)]
    state, conv = t["state"].clone(), t["conv_state"].clone()
    got = call(dict(t, state=state, conv_state=conv), state_out=state, conv_state_out=conv)
    for a, w in zip(got, want):
        assert torch.equal(a, w)
