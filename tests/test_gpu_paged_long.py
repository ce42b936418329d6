"""gsd_verify_attn_paged over contexts in which a warp of the kernel for few rows has more tiles than it looks up the pages of at once:
32 tiles of 16 keys and 8 warps, 4096 keys of a range; a second look-up is used from 4097 keys on, a third from 8193 (tolerances:
paged_ref; up to 200 additions in a row in 32 bits are 2^-16 of a sum, within the 2^-15 of the scores)."""
import numpy as np
import pytest
import torch

from paged_ref import attn_check, attn_inputs, attn_tensors, bf16

pytestmark = pytest.mark.gpu


def inputs(seed, N, Hq, Hkv, D, lens, page, P=None):
    """Sequences over one pool, each in an order of its own (of P pages; None: as many as the longest needs)."""
    B, most = len(lens), -(-max(lens) // page)
    x = attn_inputs(seed, B, N, Hq, Hkv, D, [0] * B, page)
    rng = np.random.default_rng([seed, 1])
    P = P or most
    k, v = rng.standard_normal((2, P, page, Hkv, D), dtype=np.float32)
    x.update(k=bf16(k), v=bf16(v), lens=np.asarray(lens, np.int32), table=np.full((B, most + 2), -1, np.int32))
    for b, L in enumerate(lens):
        n = -(-L // page)
        x["table"][b, :n] = np.resize(rng.permutation(P), n)
    return x


def call(x, flag=0, **kw):
    import paper_2407_16207_b200 as gsd
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = gsd.gsd_verify_attn_paged(**attn_tensors(x), status=status, **kw)
    assert int(status.item()) == flag
    return out


@pytest.mark.parametrize("N,Hq,Hkv", [(1, 4, 1), (5, 4, 1), (8, 8, 2), (9, 3, 1)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 256])
def test_one_range(page, D, N, Hq, Hkv):
    x = inputs(1, N, Hq, Hkv, D, [4090, 4097, 8200, 12500], page)
    attn_check(x, call(x, kernel=1, num_splits=1))


@pytest.mark.parametrize("N", [1, 6])
@pytest.mark.parametrize("page", [16, 64])
def test_pages_that_the_table_does_not_name(page, N):
    # one among the second 32 tiles of a warp, one among the third, one at the end
    x = inputs(2, N, 4, 1, 128, [12500, 8300], page)
    at = [(0, 4096 // page + 3), (0, 8192 // page + 5), (0, 12499 // page), (1, 8192 // page)]
    for b, i in at:
        x["table"][b, i] = -1 - i
    got = call(x, 0x1000, kernel=1, num_splits=1)
    P = x["k"].shape[0]
    z = torch.zeros_like(x["k"][:1])
    x["k"], x["v"] = torch.cat((x["k"], z)), torch.cat((x["v"], z))
    for b, i in at:
        x["table"][b, i] = P
    attn_check(x, got)


@pytest.mark.parametrize("N", [1, 3])
def test_ranges_by_length(N):
    # nine sequences of eight kv heads, cut by length into ranges of more than 32 rounds
    lens = [9500, 9000, 9700, 9999, 9400, 9300, 9600, 9100, 9001]
    x = inputs(3, N, 8, 8, 128, lens, 32, P=200)
    out = call(x)
    attn_check(x, out)
    assert torch.equal(out, call(x))
    attn_check(x, call(x, kernel=1))


@pytest.mark.parametrize("N,Hq,Hkv", [(16, 8, 1), (40, 8, 2), (90, 4, 4)])
@pytest.mark.parametrize("page", [16, 32, 128, 256])
def test_the_padded_call_on_the_same_kernel(page, N, Hq, Hkv):
    # the tcgen05 kernel on units cut alike.  Whole numbers in Q and K: scores are exact in any order, so both calls have the same
    # weights, and differ in the order of 32-bit sums of at most `keys` products each (2^-23 an addition, for the sums of weights and
    # of weighted rows) and in the output's rounding, a step of bf16 at most
    import paper_2407_16207_b200 as gsd
    lens = [640, 0, 129, 77]
    x = attn_inputs(8, 4, N, Hq, Hkv, 128, lens, page, fill=0.0)
    rng = np.random.default_rng(9)
    for n in ("q", "k", "dk"):
        x[n] = bf16(rng.integers(-3, 4, tuple(x[n].shape)))
    t = attn_tensors(x)
    flat = [torch.zeros((4, 640, Hkv, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for b, L in enumerate(lens):
        for f, p in zip(flat, (t["k_pages"], t["v_pages"])):
            f[b, :L] = p[x["table"][b, :-(-L // page)].tolist()].flatten(0, 1)[:L] if L else 0
    other = gsd.gsd_verify_attn(t["q"], *flat, t["draft_k"], t["draft_v"], t["ancestor_mask"], t["seq_lens"], kernel=2, num_splits=1)
    got = call(x, kernel=2, num_splits=1, max_len=640)
    from paged_ref import attn_want
    _, spread, _ = attn_want(x)
    attn_check(x, got)
    a, b = got.double().cpu().numpy(), other.double().cpu().numpy()
    keys = max(lens) + N
    assert (np.abs(a - b) <= 2.0 ** -7 * np.abs(b) + 2 * keys * 2.0 ** -23 * spread).all()
