"""Seeded random shapes through the calls over a paged cache: group sizes 1-20, 1-5 kv heads, 1-140 nodes, prefixes of 0-900 rows with
NaN behind every end, arbitrary mask bits, every page size, kernels and numbers of key ranges; writers with paths, counts and
rotations of all kinds."""
import numpy as np
import pytest
import torch

from paged_ref import attn_check, attn_inputs, attn_tensors, bf16, i32, table_for, turn, turn_tol
from test_gpu_paged_write import check_pages, pools

pytestmark = pytest.mark.gpu


def attention(seed):
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng([77, seed])
    B, Hkv, G, D = int(rng.integers(1, 7)), int(rng.integers(1, 6)), int(rng.integers(1, 21)), int(rng.choice([64, 128]))
    N = 1 if rng.random() < 0.3 else int(rng.integers(2, 141))
    if B * N * Hkv * G > 4000:
        N = max(1, 4000 // (B * Hkv * G))
    page = int(rng.choice([16, 32, 64, 128, 256]))
    lens = [int(rng.integers(0, 900)) if rng.random() < 0.8 else int(rng.choice([0, 1, page - 1, page, page + 1, 128, 256])) for _ in range(B)]
    x = attn_inputs([78, seed], B, N, Hkv * G, Hkv, D, lens, page, mask=str(rng.choice(["random", "chain", "none"])), M=-(-max(lens) // page) + int(rng.integers(1, 60)))
    kernel = int(rng.choice([0, 0, 1, 2]))
    if kernel == 2 and (D != 128 or 128 % G):
        kernel = 0
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = gsd.gsd_verify_attn_paged(**attn_tensors(x), kernel=kernel, num_splits=int(rng.choice([0, 0, 0, 1, 2, 5])), status=status)
    assert int(status.item()) == 0
    attn_check(x, out)


def writing(seed):
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng([79, seed])
    B, H, D, page = int(rng.integers(1, 6)), int(rng.integers(1, 12)), int(rng.choice([64, 128])), int(rng.choice([16, 32, 64, 128, 256]))
    T = int(np.exp(rng.uniform(0, np.log(1200))))
    lens = rng.integers(0, 500, B).tolist()
    M = -(-(max(lens) + T) // page)
    table, P = table_for(rng, [M] * B, M)
    kp, vp = pools(rng, P, page, H, D)
    x = bf16(rng.standard_normal((B, T, 2 * H, D)))
    counts = rng.integers(0, T + 1, B).tolist()
    kd, vd, sl, status = kp.cuda(), vp.cuda(), i32(lens), torch.zeros(1, dtype=torch.int32, device="cuda")
    n, A = 8 * int(rng.integers(1, D // 16 + 1)), int(rng.integers(1, 5))
    freqs = (10000.0 ** (-np.arange(n) / n)).astype(np.float32)
    axes, pos, off, nb = rng.integers(0, A, n).tolist(), rng.integers(-9999, 9999, (A, B, T)).astype(np.int32), rng.integers(0, 9999, B).astype(np.int32), bool(rng.integers(2))
    xd, f = x.cuda(), torch.from_numpy(freqs).cuda()
    gsd.gsd_append_kv_paged(kd, vd, i32(table), xd[:, :, :H], xd[:, :, H:], i32(counts), sl, freqs=f, positions=i32(pos), offsets=i32(off), axes=axes, pairs=nb, status=status)
    assert sl.tolist() == [a + c for a, c in zip(lens, counts)] and int(status.item()) == 0
    check_pages(vd, vp, table, page, lens, [x[b, :counts[b], H:] for b in range(B)])
    raw = [x[b, :counts[b], :H].double().numpy() for b in range(B)]
    ref = [turn(r, (pos + off[:, None])[:, b, :counts[b]], freqs, axes, nb) for b, r in enumerate(raw)]
    check_pages(kd, kp, table, page, lens, ref, False, [turn_tol(r, w, n, nb) for r, w in zip(raw, ref)])
    # the same rows through gsd_rotary
    q, k = gsd.gsd_rotary(xd[:, :, H:], xd[:, :, :H], f, i32(pos), offsets=i32(off), axes=axes, pairs=nb)
    for b in range(B):
        j = np.arange(lens[b], lens[b] + counts[b])
        assert torch.equal(k[b, :counts[b]].cpu(), kd.cpu()[table[b, j // page], j % page])
    # a path behind it
    N, Tcap = min(T, 512), int(rng.integers(1, min(T, 512) + 1))
    lens = sl.tolist()
    room = [M * page - a for a in lens]
    nodes = rng.integers(0, N, (B, Tcap)).astype(np.int32)
    counts = [int(rng.integers(0, min(Tcap, r) + 1)) for r in room]
    kb, vb = kd.cpu(), vd.cpu()
    dk, dv = xd[:, :N, :H].contiguous(), xd[:, :N, H:].contiguous()
    gsd.gsd_commit_kv_paged(kd, vd, i32(table), dk, dv, i32(nodes), i32(counts), sl, status=status)
    assert sl.tolist() == [a + c for a, c in zip(lens, counts)] and int(status.item()) == 0
    for got, old, d in ((kd, kb, dk.cpu()), (vd, vb, dv.cpu())):
        check_pages(got, old, table, page, lens, [d[b, nodes[b, :counts[b]].tolist()] for b in range(B)])


@pytest.mark.parametrize("seed", range(60))
def test_attention(seed):
    attention(seed)


@pytest.mark.parametrize("seed", range(30))
def test_writing(seed):
    writing(seed)
