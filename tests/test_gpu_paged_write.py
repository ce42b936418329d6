"""gsd_append_kv_paged and gsd_commit_kv_paged: rows that are copied bit for bit, rotated ones against 64 bits (tolerances:
paged_ref), and everything else as it was."""
import numpy as np
import pytest
import torch

from paged_ref import bf16, i32, table_for, turn, turn_tol

pytestmark = pytest.mark.gpu
PAGES = [16, 32, 64, 128, 256]


def pools(rng, P, page, H, D):
    """Random bits, NaN and infinities among them."""
    return [torch.from_numpy(rng.integers(-2 ** 15, 2 ** 15, (P, page, H, D)).astype(np.int16)).view(torch.bfloat16) for _ in range(2)]


def bits(t):
    return t.view(torch.int16).cpu().numpy()


def new_rows(table, page, L, n):
    j = np.arange(L, L + n)
    return table[j // page], j % page


def check_pages(got, old, table, page, lens, rows, exact=True, tol=None):
    """got against old with rows[b] [n,H,D] at lens[b]..., and nothing else changed."""
    want = bits(old).copy()
    have = bits(got).copy()
    for b, x in enumerate(rows):
        p, r = new_rows(table[b], page, lens[b], len(x))
        if exact:
            want[p, r] = bits(x)
        else:
            g = torch.from_numpy(have[p, r]).view(torch.bfloat16).double().numpy()
            err = np.abs(g - x)
            assert (err <= tol[b]).all(), float((err - tol[b]).max())
            have[p, r] = want[p, r]
    assert np.array_equal(have, want)


def freqs_of(n):
    return (10000.0 ** (-np.arange(n) / n)).astype(np.float32)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("H,T", [(1, 1), (3, 40), (5, 300), (8, 5), (2, 1500)])
@pytest.mark.parametrize("neighbours", [False, True])
def test_append(D, page, H, T, neighbours):
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng([1, D, page, T])
    lens = [0, 1, 15, 16, 100, 127, 250]
    counts = [T, T, 0, min(T, 1), T, max(T - 1, 0), T]
    B = len(lens)
    M = -(-(250 + T - min(T, 3)) // page)                         # the last sequence may not have room for all
    put = [min(n, M * page - L) for n, L in zip(counts, lens)]
    table, P = table_for(rng, [-(-(L + n) // page) for L, n in zip(lens, put)], M)
    kp, vp = pools(rng, P, page, H, D)
    x = bf16(rng.standard_normal((B, T, 2 * H + 1, D)))
    xd = x.cuda()
    n, A = {40: (D // 4, 1), 300: (D // 2, 3), 5: (D // 2, 1)}.get(T, (D // 2, 2))
    n = max(8, n // 8 * 8)
    freqs, axes = freqs_of(n), rng.integers(0, A, n).tolist()
    pos, off = rng.integers(0, 5000, (A, B, T)).astype(np.int32), rng.integers(0, 3000, B).astype(np.int32)
    for how in ("copy", "place", "positions"):
        kd, vd, sl = kp.cuda(), vp.cuda(), i32(lens)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        kw = {}
        if how == "place":
            kw = dict(freqs=torch.from_numpy(freqs).cuda(), axes=axes, pairs=neighbours)
            at = np.asarray([np.broadcast_to(L + np.arange(T), (A, T)) for L in lens])
        elif how == "positions":
            kw = dict(freqs=torch.from_numpy(freqs).cuda(), axes=axes, pairs=neighbours, positions=i32(pos), offsets=i32(off))
            at = (pos + off[:, None]).transpose(1, 0, 2)
        gsd.gsd_append_kv_paged(kd, vd, i32(table), xd[:, :, :H], xd[:, :, H + 1:], i32(counts), sl, status=status, **kw)
        assert sl.tolist() == [L + p for L, p in zip(lens, put)]
        assert int(status.item()) == (0x20 if put != counts else 0)
        check_pages(vd, vp, table, page, lens, [x[b, :put[b], H + 1:] for b in range(B)])
        rows = [x[b, :put[b], :H] for b in range(B)]
        if how == "copy":
            check_pages(kd, kp, table, page, lens, rows)
        else:
            y = [r.double().numpy() for r in rows]
            ref = [turn(r, at[b][:, :put[b]], freqs, axes, neighbours) for b, r in enumerate(y)]
            check_pages(kd, kp, table, page, lens, ref, False, [turn_tol(r, w, n, neighbours) for r, w in zip(y, ref)])


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("H,N,Tcap", [(1, 1, 1), (3, 20, 7), (8, 256, 17), (40, 57, 57), (2, 512, 512)])
def test_commit(D, page, H, N, Tcap):
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng([2, D, page, N])
    lens = [0, 15, 16, 250, 99]
    B = len(lens)
    M = -(-(250 + Tcap - min(Tcap, 2)) // page)
    count = rng.integers(0, Tcap + 1, B)
    count[3] = Tcap
    nodes = np.full((B, Tcap), -7, np.int32)
    for b in range(B):
        nodes[b, :count[b]] = np.sort(rng.permutation(N)[:count[b]])
    put = [min(int(n), M * page - L) for n, L in zip(count, lens)]
    table, P = table_for(rng, [-(-(L + n) // page) for L, n in zip(lens, put)], M)
    kp, vp = pools(rng, P, page, H, D)
    dk, dv = pools(rng, B, N, H, D)
    kd, vd, sl = kp.cuda(), vp.cuda(), i32(lens)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    gsd.gsd_commit_kv_paged(kd, vd, i32(table), dk.cuda(), dv.cuda(), i32(nodes), i32(count), sl, status=status)
    assert sl.tolist() == [L + p for L, p in zip(lens, put)]
    assert int(status.item()) == (0x20 if put != count.tolist() else 0)
    for got, old, d in ((kd, kp, dk), (vd, vp, dv)):
        check_pages(got, old, table, page, lens, [d[b, nodes[b, :put[b]].tolist()] for b in range(B)])


def test_bad_nodes_and_counts():
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng(3)
    table, P = table_for(rng, [2, 2, 2], 2)
    kp, vp = pools(rng, P, 16, 2, 64)
    dk, dv = pools(rng, 3, 9, 2, 64)
    nodes = np.array([[0, 9, 4, -1], [3, 3, 2, 1], [0, 1, 2, 3]], np.int32)
    kd, vd, sl, status = kp.cuda(), vp.cuda(), i32([5, 14, 3]), torch.zeros(1, dtype=torch.int32, device="cuda")
    gsd.gsd_commit_kv_paged(kd, vd, i32(table), dk.cuda(), dv.cuda(), i32(nodes), i32([3, 9, -2]), sl, status=status)
    assert sl.tolist() == [7, 18, 3] and int(status.item()) == 0x1
    for got, old, d in ((kd, kp, dk), (vd, vp, dv)):
        check_pages(got, old, table, 16, [5, 14, 3], [d[0, [0, 4]], d[1, [3, 3, 2, 1]], d[2, :0]])
    # an append with a count beyond T and one below 0, and lengths out of range
    kd, vd, sl, status = kp.cuda(), vp.cuda(), i32([-4, 2, 33]), torch.zeros(1, dtype=torch.int32, device="cuda")
    gsd.gsd_append_kv_paged(kd, vd, i32(table), dk.cuda(), dv.cuda(), i32([10, -1, 2]), sl, status=status)
    assert sl.tolist() == [9, 2, 32] and int(status.item()) == 0x30
    for got, old, d in ((kd, kp, dk), (vd, vp, dv)):
        check_pages(got, old, table, 16, [0, 2, 32], [d[0], d[1, :0], d[2, :0]])


@pytest.mark.parametrize("T", [3, 60, 3000])
@pytest.mark.parametrize("page", [16, 64])
def test_rows_without_a_page_are_dropped(T, page):
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng(4)
    lens = [page - 1, 0, 5 * page, 7]
    B, M = 4, -(-(5 * page + T) // page) + 1
    table, P = table_for(rng, [M] * B, M)
    kp, vp = pools(rng, P, page, 2, 128)
    k, v = pools(rng, B, T, 2, 128)
    # no page for the second entry, for the first, for one behind all rows, for one in the middle and a later one
    table[0, 1], table[1, 0], table[2, M - 1], table[3, min(2, M - 1)] = -1, P, -5, 2 ** 31 - 1
    if M > 12:
        table[3, 9] = -1
    last = {0: page, 1: 0, 2: (M - 1) * page, 3: min(2, M - 1) * page}
    put = [max(0, min(T, last[b] - lens[b])) for b in range(B)]
    flag = 0x1000 if any(p < T for p in put) else 0
    good = table.copy()
    good[(good < 0) | (good >= P)] = 0
    for call in ("append", "commit"):
        if call == "commit" and T > 512:
            continue
        kd, vd, sl, status = kp.cuda(), vp.cuda(), i32(lens), torch.zeros(1, dtype=torch.int32, device="cuda")
        if call == "append":
            gsd.gsd_append_kv_paged(kd, vd, i32(table), k.cuda(), v.cuda(), i32([T] * B), sl, status=status)
        else:
            gsd.gsd_commit_kv_paged(kd, vd, i32(table), k.cuda(), v.cuda(), i32(np.tile(np.arange(T), (B, 1))), i32([T] * B), sl, status=status)
        assert sl.tolist() == [L + p for L, p in zip(lens, put)]
        assert int(status.item()) == flag
        for got, old, d in ((kd, kp, k), (vd, vp, v)):
            check_pages(got, old, good, page, lens, [d[b, :put[b]] for b in range(B)])


def test_offsets_may_be_the_lengths_themselves():
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng(5)
    freqs = freqs_of(32)
    f = torch.from_numpy(freqs).cuda()
    for T in (4, 700):
        lens = [10, 33]
        table, P = table_for(rng, [50, 50], 50)
        kp, vp = pools(rng, P, 16, 2, 64)
        x = bf16(rng.standard_normal((2, T, 2, 64)))
        kd, vd, sl = kp.cuda(), vp.cuda(), i32(lens)
        pos = np.broadcast_to(np.arange(T), (1, 2, T))
        gsd.gsd_append_kv_paged(kd, vd, i32(table), x.cuda(), x.cuda(), i32([T, T]), sl, freqs=f, positions=i32(pos), offsets=sl)
        assert sl.tolist() == [10 + T, 33 + T]
        y = [r.double().numpy() for r in x]
        ref = [turn(r, pos[:, b] + lens[b], freqs, [0] * 32, False) for b, r in enumerate(y)]
        check_pages(kd, kp, table, 16, lens, ref, False, [turn_tol(r, w, 32, False) for r, w in zip(y, ref)])


def test_a_pool_beyond_4_gb():
    import paper_2407_16207_b200 as gsd
    P, page, H, D = 140000, 16, 8, 128
    k, v = (torch.zeros((P, page, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rng = np.random.default_rng(6)
    x = bf16(rng.standard_normal((2, 40, H, D))).cuda()
    where = i32([[P - 1, P - 2, 139000], [5, P - 9, 131072]])
    sl = i32([3, 8])
    gsd.gsd_append_kv_paged(k, v, where, x, x, i32([30, 40]), sl)
    gsd.gsd_commit_kv_paged(k, v, where, x, x, i32([[39, 2]] * 2), i32([2, 0]), sl)
    assert sl.tolist() == [35, 48]
    for pool in (k, v):
        a = pool[[P - 1, P - 2, 139000]].flatten(0, 1)
        b = pool[[5, P - 9, 131072]].flatten(0, 1)
        assert torch.equal(a[3:33], x[0, :30]) and torch.equal(a[33], x[0, 39]) and torch.equal(a[34], x[0, 2]) and torch.equal(b[8:48], x[1])
        assert int(pool.count_nonzero()) == int(a.count_nonzero() + b.count_nonzero())


@pytest.mark.parametrize("T", [2, 900])
def test_captured_and_replayed(T):
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng(7)
    table, P = table_for(rng, [60, 60], 60)
    kp, vp = pools(rng, P, 32, 2, 64)
    k, v = pools(rng, 2, T, 2, 64)
    kd, vd, tb, ks, vs = kp.cuda(), vp.cuda(), i32(table), k.cuda(), v.cuda()
    sl, cnt = i32([0, 5]), i32([T, T - 1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        gsd.gsd_append_kv_paged(kd, vd, tb, ks, vs, cnt, sl)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            gsd.gsd_append_kv_paged(kd, vd, tb, ks, vs, cnt, sl)
        g.replay()
        s.synchronize()
    assert sl.tolist() == [2 * T, 5 + 2 * (T - 1)]
    for got, old, d in ((kd, kp, k), (vd, vp, v)):
        check_pages(got, old, table, 32, [0, 5], [torch.cat((d[0], d[0])), torch.cat((d[1, :T - 1], d[1, :T - 1]))])
