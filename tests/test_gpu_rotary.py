"""gsd_rotary against a 64-bit evaluation of its definition (tolerances: paged_ref)."""
import numpy as np
import pytest
import torch

from paged_ref import bf16, i32, turn, turn_tol

pytestmark = pytest.mark.gpu


def freqs_of(n, base=500000.0):
    return (base ** (-np.arange(n) / n)).astype(np.float32)


def check(got, x, pos, freqs, axes, neighbours):
    """got, x [B,T,H,D]; pos [axes,B,T]"""
    for b in range(x.shape[0]):
        y = x[b].double().numpy()
        ref = turn(y, pos[:, b], freqs, axes, neighbours)
        g = got[b].double().cpu().numpy()
        err, tol = np.abs(g - ref), turn_tol(y, ref, len(freqs), neighbours)
        assert (err <= tol).all(), float((err - tol).max())
        assert np.array_equal(g[..., 2 * len(freqs):], y[..., 2 * len(freqs):])


def inputs(seed, B, T, Hq, Hkv, D, n, A, top):
    rng = np.random.default_rng(seed)
    x = bf16(rng.standard_normal((B, T, Hq + 2 * Hkv, D)))
    pos = rng.integers(-top, top + 1, (A, B, T)).astype(np.int32)
    off = rng.integers(0, top + 1, B).astype(np.int32)
    return x, pos, off, freqs_of(n), rng.integers(0, A, n).tolist()


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("D,n", [(128, 64), (128, 32), (128, 8), (128, 56), (64, 32), (64, 16), (64, 8)])
@pytest.mark.parametrize("B,T,Hq,Hkv,A", [(1, 1, 1, 1, 1), (3, 1, 8, 2, 3), (2, 37, 4, 4, 1), (1, 130, 28, 4, 3), (5, 9, 5, 3, 4), (2, 3, 64, 8, 2)])
def test_rotary(B, T, Hq, Hkv, A, D, n, neighbours):
    import paper_2407_16207_b200 as gsd
    x, pos, off, freqs, axes = inputs([B, T, D, n], B, T, Hq, Hkv, D, n, A, 4000)
    q, k = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv]
    xd, f = x.cuda(), torch.from_numpy(freqs).cuda()
    qd, kd = xd[:, :, :Hq], xd[:, :, Hq:Hq + Hkv]
    # slices of the projection's output
    a, b = gsd.gsd_rotary(qd, kd, f, i32(pos), offsets=i32(off), axes=axes, pairs=neighbours)
    at = pos + off[:, None]
    check(a, q, at, freqs, axes, neighbours)
    check(b, k, at, freqs, axes, neighbours)
    assert torch.equal(xd.cpu(), x)
    # dense, in place, without offsets and through the Python path
    qc, kc = qd.contiguous().clone(), kd.contiguous().clone()      # (a slice of one head and token is dense already)
    r = gsd.gsd_rotary(qc, kc, f, i32(pos), axes=axes, pairs=neighbours, out=(qc, kc))
    assert r[0] is qc and r[1] is kc
    check(qc, q, pos, freqs, axes, neighbours)
    check(kc, k, pos, freqs, axes, neighbours)
    # q alone; one axis
    c, none = gsd.gsd_rotary(qd, None, f, i32(pos[:1]), pairs=neighbours)
    assert none is None
    check(c, q, pos[:1], freqs, [0] * n, neighbours)
    d, _ = gsd.gsd_rotary(qd, None, f, i32(pos[:1]), pairs=np.bool_(neighbours), axes=np.zeros(n, int))
    assert torch.equal(c, d)


@pytest.mark.parametrize("top", [0, 1, 100000, 2 ** 24 + 1, 2 ** 25])
def test_far_positions(top):
    # every position a fraction of a turn apart is told from the next, however far
    import paper_2407_16207_b200 as gsd
    x, _, _, freqs, _ = inputs(5, 1, 40, 2, 1, 128, 64, 1, 1)
    pos = (top - np.arange(40)).astype(np.int32)[None, None]
    q = x[:, :, :2].contiguous()
    got, _ = gsd.gsd_rotary(q.cuda(), None, torch.from_numpy(freqs).cuda(), i32(pos))
    check(got, q, pos, freqs, [0] * 64, False)


def test_positions_and_offsets_add_beyond_32_bits():
    import paper_2407_16207_b200 as gsd
    x = inputs(6, 1, 3, 2, 1, 64, 16, 1, 1)[0][:, :, :2].contiguous()
    freqs = (2.0 ** -np.arange(10, 26)).astype(np.float32)              # (angles below 2^22)
    pos, off = np.array([[[2 ** 31 - 1, 5, -2 ** 31]]], np.int32), np.array([2 ** 31 - 1], np.int32)
    got, _ = gsd.gsd_rotary(x.cuda(), None, torch.from_numpy(freqs).cuda(), i32(pos), offsets=i32(off))
    check(got, x, pos.astype(np.int64) + off[:, None], freqs, [0] * 16, False)


def test_a_turn_and_back_and_the_scores_of_a_shift():
    # the product of a rotated query and a rotated key depends on the distance alone: bf16 rows, |q| |k| of roundings
    import paper_2407_16207_b200 as gsd
    x, _, _, freqs, _ = inputs(7, 1, 1, 4, 4, 128, 64, 1, 1)
    q, k, f = x[:, :, :4].contiguous().cuda(), x[:, :, 4:8].contiguous().cuda(), torch.from_numpy(freqs).cuda()
    dots = []
    for start in (0, 7, 100003):
        a, _ = gsd.gsd_rotary(q, None, f, i32([[[start + 900]]]))
        b, _ = gsd.gsd_rotary(k, None, f, i32([[[start]]]))
        dots.append((a.double() * b.double()).sum(-1))
    room = 2 * (2 * 2.0 ** -8 + 2.0 ** -16) * q.double().norm(dim=-1) * k.double().norm(dim=-1)
    assert (dots[1] - dots[0]).abs().le(room).all() and (dots[2] - dots[0]).abs().le(room).all()


def test_nothing_outside_is_written_and_rows_of_nan_stay_by_themselves():
    import paper_2407_16207_b200 as gsd
    x, pos, off, freqs, axes = inputs(8, 3, 11, 7, 3, 64, 24, 3, 300)
    x[1, 4] = float("nan")
    x[2, 10] = float("inf")
    outs = []
    for H in (7, 3):
        flat = torch.full((3 * 11 * H * 64 * 2 + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
        outs.append((flat, flat[4096:-4096].view(torch.bfloat16).view(3, 11, H, 64)))
    xd = x.cuda()
    gsd.gsd_rotary(xd[:, :, :7], xd[:, :, 7:10], torch.from_numpy(freqs).cuda(), i32(pos), offsets=i32(off), axes=axes, out=(outs[0][1], outs[1][1]))
    for (flat, o), y in zip(outs, (x[:, :, :7], x[:, :, 7:10])):
        assert (flat[:4096] == 0xA5).all() and (flat[-4096:] == 0xA5).all()
        assert o[1, 4].isnan().all()
        keep = [(0, slice(None)), (1, slice(0, 4)), (1, slice(5, None)), (2, slice(0, 10))]
        for b, t in keep:
            check(o[b:b + 1, t], y[b:b + 1, t], (pos + off[:, None])[:, b:b + 1, t], freqs, axes, False)


def test_captured_with_moving_offsets():
    import paper_2407_16207_b200 as gsd
    x, pos, off, freqs, axes = inputs(9, 2, 5, 4, 2, 128, 64, 1, 100)
    q, k, f, p, o = x[:, :, :4].contiguous().cuda(), x[:, :, 4:6].contiguous().cuda(), torch.from_numpy(freqs).cuda(), i32(pos), i32(off)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        gsd.gsd_rotary(q, k, f, p, offsets=o)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            a, b = gsd.gsd_rotary(q, k, f, p, offsets=o)
        for step in range(3):
            o.fill_(1000 * step)
            g.replay()
            s.synchronize()
            check(a, x[:, :, :4], pos + 1000 * step, freqs, [0] * 64, False)
            check(b, x[:, :, 4:6], pos + 1000 * step, freqs, [0] * 64, False)
