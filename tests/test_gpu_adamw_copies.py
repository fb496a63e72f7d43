"""mlt_adamw where only some parameters have a copy or a gradient, with few and with many tensors."""
import pytest

from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu


def _model(count, bits):
    import torch

    g = torch.Generator("cuda").manual_seed(count)
    sizes = [1 + (k * 37) % 600 for k in range(count)]
    params = [torch.randn(n, generator=g, device="cuda") for n in sizes]
    grads = [torch.randn(n, generator=g, device="cuda").bfloat16() for n in sizes]
    return params, grads, mlt.adamw_state(params, bits)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [1, 3, 32, 33, 40, 501])
def test_a_copy_for_some(count, bits):
    """Parameters without a copy or a gradient among others: what each has to get, as without copies."""
    import torch

    for every in (2, 3, count + 1):  # the last: the first tensor alone has none
        params, grads, state = _model(count, bits)
        copies = [None if k % every == 0 else torch.full((p.numel(),), 9.0, dtype=(torch.bfloat16, torch.float16)[k % 2],
                                                         device="cuda") for k, p in enumerate(params)]
        missing = [k for k in range(count) if k % 7 == 5]
        for k in missing:
            grads[k] = None
        alone, _, same = _model(count, bits)
        mlt.adamw(params, grads, state, 1, lr=0.01, copies=copies, seed=3)
        mlt.adamw(alone, grads, same, 1, lr=0.01, seed=3)
        assert all(torch.equal(a, b) for a, b in zip(params, alone))
        assert all(a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(state, same))
        for k, (p, c) in enumerate(zip(params, copies)):
            assert c is None or (c == 9.0).all() if k in missing else c is None or torch.equal(c, p.to(c.dtype))


@pytest.mark.parametrize("count", [3, 40])
def test_refused_alike(count):
    """A missing gradient excuses its parameter's place and layout, few tensors or many; a copy's faults are found."""
    import torch

    params, grads, state = _model(count, 32)
    copies = [None] * count
    for bad, kind in ((params[1].cpu(), ValueError), (params[1].double(), TypeError), (params[1][:5], ValueError),
                      (torch.zeros(2 * params[1].numel(), device="cuda")[::2], ValueError)):
        copies[1] = bad
        with pytest.raises(kind):
            mlt.adamw(params, grads, state, 1, copies=copies)
    copies[1] = None
    grads[1], n = None, params[1].numel()
    for p in (params[1].cpu(), params[1].double(), torch.zeros(2 * n, device="cuda")[::2]):
        params[1] = p
        old = p.clone()
        mlt.adamw(params, grads, state, 1, copies=copies)
        assert torch.equal(p, old)
