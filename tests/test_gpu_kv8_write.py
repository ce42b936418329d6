"""gsd_commit_kv_q8 and gsd_append_kv_q8: codes and exponents bit for bit against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import kv8_ref

pytestmark = pytest.mark.gpu
DT = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def rows_like(rng, *shape):
    """bf16 rows whose sizes differ from row to row, ties and exact powers among them."""
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-6, 5, shape[:-2] + (1, 1)))
    x[..., ::7] = np.round(x[..., ::7] * 4) / 4
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16)


def fresh(rng, B, Lmax, H, D, fmt, block, lens):
    """A cache with rows written by the definition; anything behind the ends."""
    c = rng.integers(0, 256, (2, B, Lmax, H, D)).astype(np.uint8)
    e = rng.integers(-128, 128, (2, B, -(-Lmax // block), H)).astype(np.int8)
    for kv in range(2):
        for b in range(B):
            x = rows_like(rng, lens[b], H, D).double().numpy()
            kv8_ref.append(c[kv, b], e[kv, b], x, 0, fmt, block)
    return c, e


def on_gpu(c, e, fmt):
    code = lambda a: torch.from_numpy(a.view(np.int8).copy()).cuda().view(DT[fmt])
    exp = lambda a: torch.from_numpy(a.copy()).cuda()
    return code(c[0]), code(c[1]), exp(e[0]), exp(e[1])


def same(got, c, e):
    for kv in range(2):
        assert np.array_equal(got[kv].view(torch.uint8).cpu().numpy(), c[kv])
        assert np.array_equal(got[2 + kv].cpu().numpy(), e[kv])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("H,T", [(1, 1), (3, 40), (5, 300)])
def test_append(fmt, D, block, H, T):
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng([1, D, block, T])
    lens = [0, 1, 15, 16, 100, 127, 250]
    B, Lmax = len(lens), 250 + T - min(T, 3)              # the last sequence does not have room for all
    counts = [T, T, 0, min(T, 1), T, max(T - 1, 0), T]
    c, e = fresh(rng, B, Lmax, H, D, fmt, block, lens)
    k, v = rows_like(rng, B, T, H, D), rows_like(rng, B, T, H, D)
    t = on_gpu(c, e, fmt)
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    gsd.gsd_append_kv_q8(*t, k.cuda(), v.cuda(), torch.tensor(counts, dtype=torch.int32, device="cuda"), sl, block=block, status=status)
    new = [max(kv8_ref.append(c[kv, b], e[kv, b], x[b, :counts[b]].double().numpy(), lens[b], fmt, block) for kv, x in enumerate((k, v)))
           for b in range(B)]
    assert sl.tolist() == new
    assert int(status.item()) == (0x20 if any(l + n > Lmax for l, n in zip(lens, counts)) else 0)
    same(t, c, e)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D,H,block,N,Tcap", [(128, 8, 64, 64, 64), (64, 3, 16, 40, 21), (128, 40, 32, 17, 9), (128, 1, 128, 512, 512), (128, 2, 16, 300, 600)])
def test_commit(fmt, D, H, block, N, Tcap):
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng([2, D, H, block])
    lens = [0, 5, 63, 64, 200]
    B, Lmax = len(lens), 520
    count = [1, min(Tcap, N), min(Tcap, 7), 0, min(Tcap, N, 330)]
    nodes = np.full((B, Tcap), -1, np.int32)
    for b in range(B):
        nodes[b, :count[b]] = np.sort(rng.permutation(N)[:count[b]])
    c, e = fresh(rng, B, Lmax, H, D, fmt, block, lens)
    dk, dv = rows_like(rng, B, N, H, D), rows_like(rng, B, N, H, D)
    t = on_gpu(c, e, fmt)
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    gsd.gsd_commit_kv_q8(*t, dk.cuda(), dv.cuda(), torch.from_numpy(nodes).cuda(), torch.tensor(count, dtype=torch.int32, device="cuda"),
                         sl, block=block, status=status)
    new = [max(kv8_ref.append(c[kv, b], e[kv, b], x[b, nodes[b, :count[b]]].double().numpy(), lens[b], fmt, block)
               for kv, x in enumerate((dk, dv))) for b in range(B)]
    assert sl.tolist() == new
    assert int(status.item()) == (0x20 if any(l + n > Lmax for l, n in zip(lens, count)) else 0)
    same(t, c, e)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_growing_row_by_row(fmt):
    # every row larger than the one before it: the block is rounded anew each time
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng(3)
    B, Lmax, H, D, block = 2, 40, 2, 128, 16
    c, e = fresh(rng, B, Lmax, H, D, fmt, block, [0, 0])
    t = on_gpu(c, e, fmt)
    sl = torch.zeros(B, dtype=torch.int32, device="cuda")
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    zero = torch.zeros((B, 1), dtype=torch.int32, device="cuda")
    for i in range(35):
        x = rows_like(rng, B, 1, H, D) * 2.0 ** (i * 0.7)
        x = x.to(torch.bfloat16)
        if i % 2:
            gsd.gsd_append_kv_q8(*t, x.cuda(), x.cuda(), one, sl, block=block)
        else:
            gsd.gsd_commit_kv_q8(*t, x.cuda(), x.cuda(), zero, one, sl, block=block)
        for kv in range(2):
            for b in range(B):
                kv8_ref.append(c[kv, b], e[kv, b], x[b].double().numpy(), i, fmt, block)
    assert sl.tolist() == [35, 35]
    same(t, c, e)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_largest_smallest_infinite_and_nan_values(fmt):
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng(4)
    B, Lmax, H, D, block = 1, 64, 1, 64, 16
    for special, flag in ((3.38e38, 0), (2.0 ** -126, 0), (1e-40, 0), (0.0, 0), (np.inf, 0x800), (np.nan, 0x800), (448.0, 0), (449.0, 0), (127.0, 0), (127.5, 0)):
        x = rows_like(rng, B, 5, H, D).float() * (0.0 if 0 < special < 1e-30 else 1.0)
        x[0, 2, 0, 7], x[0, 3, 0, 63] = special, -special
        x = x.to(torch.bfloat16)
        c, e = fresh(rng, B, Lmax, H, D, fmt, block, [13])
        t = on_gpu(c, e, fmt)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        sl = torch.tensor([13], dtype=torch.int32, device="cuda")
        gsd.gsd_append_kv_q8(*t, x.cuda(), x.cuda(), torch.tensor([5], dtype=torch.int32, device="cuda"), sl, block=block, status=status)
        for kv in range(2):
            kv8_ref.append(c[kv, 0], e[kv, 0], x[0].double().numpy(), 13, fmt, block)
        assert int(status.item()) == flag, special
        same(t, c, e)


def test_bad_nodes_counts_and_lengths_are_flagged():
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng(5)
    B, Lmax, H, D, block = 2, 64, 2, 64, 16
    c, e = fresh(rng, B, Lmax, H, D, "e4m3", block, [0, 10])
    dk = rows_like(rng, B, 6, H, D)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    t = on_gpu(c, e, "e4m3")
    status, sl = i32([0]), i32([-4, 10])
    nodes = [[0, 99, 3, -1], [0, 1, 1, 5]]
    gsd.gsd_commit_kv_q8(*t, dk.cuda(), dk.cuda(), i32(nodes), i32([4, 9]), sl, block=block, status=status)
    for kv in range(2):
        kv8_ref.append(c[kv, 0], e[kv, 0], dk[0, [0, 3]].double().numpy(), 0, "e4m3", block)
        kv8_ref.append(c[kv, 1], e[kv, 1], dk[1, nodes[1]].double().numpy(), 10, "e4m3", block)
    assert int(status.item()) == 0x1 | 0x10 and sl.tolist() == [2, 14]
    same(t, c, e)
    status, sl = i32([0]), i32([2, 70])
    gsd.gsd_append_kv_q8(*t, dk.cuda(), dk.cuda(), i32([7, 2]), sl, block=block, status=status)
    for kv in range(2):
        kv8_ref.append(c[kv, 0], e[kv, 0], dk[0].double().numpy(), 2, "e4m3", block)
    assert int(status.item()) == 0x10 | 0x20 and sl.tolist() == [8, 64]
    same(t, c, e)


def test_a_captured_commit_follows_its_buffers():
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng(6)
    B, Lmax, H, D, block, fmt = 3, 200, 4, 128, 32, "int8"
    lens = [0, 31, 40]
    c, e = fresh(rng, B, Lmax, H, D, fmt, block, lens)
    t = on_gpu(c, e, fmt)
    dk = rows_like(rng, B, 8, H, D).cuda()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    nodes, count, sl = i32([[0, 2, 5]] * B), i32([3, 2, 1]), i32(lens)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        gsd.gsd_commit_kv_q8(*t, dk, dk, nodes, count, sl, block=block)
        gsd.gsd_append_kv_q8(*t, dk, dk, count, sl, block=block)
    for r in range(6):
        dk.copy_(rows_like(rng, B, 8, H, D))
        g.replay()
        x = dk.double().cpu().numpy()
        for b, n in enumerate((3, 2, 1)):
            for kv in range(2):
                at = kv8_ref.append(c[kv, b], e[kv, b], x[b, [0, 2, 5][:n]], lens[b], fmt, block)
                kv8_ref.append(c[kv, b], e[kv, b], x[b, :n], at, fmt, block)
            lens[b] += 2 * n
    assert sl.tolist() == lens
    same(t, c, e)
