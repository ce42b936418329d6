"""Tensors that the calls allocate come from torch as any other: a profiler and a dispatch mode see them, and in deterministic mode
their memory is filled."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def mask():
    import paper_2407_16207_b200 as gsd
    ptr = torch.tensor([[0, 0, 1, 2]], dtype=torch.int32, device="cuda")
    idx = torch.tensor([[0, 0]], dtype=torch.int32, device="cuda")
    return lambda: gsd.gsd_build_mask(ptr, idx)


def rotary():
    import paper_2407_16207_b200 as gsd
    x = torch.randn((2, 3, 4, 64), device="cuda").to(torch.bfloat16)
    freqs, pos = torch.ones(32, device="cuda"), torch.arange(6, dtype=torch.int32, device="cuda").view(1, 2, 3)
    return lambda: gsd.gsd_rotary(x, None, freqs, pos)[0]


def attention():
    import paper_2407_16207_b200 as gsd
    q, kv = torch.randn((1, 2, 4, 64), device="cuda").to(torch.bfloat16), torch.randn((1, 40, 2, 64), device="cuda").to(torch.bfloat16)
    draft, see, lens = kv[:, :2].contiguous(), torch.full((1, 2, 1), 3, dtype=torch.int32, device="cuda"), torch.full((1,), 33, dtype=torch.int32, device="cuda")
    return lambda: gsd.gsd_verify_attn(q, kv, kv, draft, draft, see, lens)


CALLS = [mask, rotary, attention]


def operations(call):
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CPU]) as prof:
        out = call()
    return out, [e.name for e in prof.events()]


@pytest.mark.parametrize("make", CALLS)
def test_a_profiler_sees_the_allocation(make):
    out, names = operations(make())
    assert any(n.startswith("aten::empty") for n in names)


@pytest.mark.parametrize("make", CALLS)
def test_deterministic_mode_fills_new_memory(make):
    call = make()
    want = call()
    torch.use_deterministic_algorithms(True)
    try:
        out, names = operations(call)
    finally:
        torch.use_deterministic_algorithms(False)
    assert "aten::fill_" in names and torch.equal(out, want)


@pytest.mark.parametrize("make", CALLS)
def test_a_dispatch_mode_sees_the_allocation(make):
    from torch.utils._python_dispatch import TorchDispatchMode

    class Log(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            seen.append(str(func))
            return func(*args, **(kwargs or {}))

    seen, call = [], make()
    want = call()
    with Log():
        out = call()
    assert any("empty" in n for n in seen) and torch.equal(out, want)
