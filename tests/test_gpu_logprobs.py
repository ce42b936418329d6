"""gsd_token_logprobs against 64 bits.

Tolerance: ln s is off by the relative error of s - 2^-22 for ex2, 2^-24 |y| (|y| < 60) for its argument, 2^-24 for each
of some 60 additions in a row - below 1e-5; the rest are a few roundings of the result, 2^-24 each.  The entropy
adds u / s, whose terms have the same relative errors: 1e-5 (1 + H)."""
import numpy as np
import pytest
import torch

import kv8_ref

pytestmark = pytest.mark.gpu


def run(x, nodes, tokens, lens, k, **kw):
    import paper_2407_16207_b200 as gsd
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    i32 = lambda v: torch.as_tensor(np.asarray(v, np.int32)).cuda()
    out = gsd.gsd_token_logprobs(x if isinstance(x, torch.Tensor) else torch.from_numpy(x).cuda(), i32(nodes), i32(tokens), i32(lens), k=k, status=status, **kw)
    return [o.cpu().numpy() for o in out], int(status.item())


def check(x, nodes, tokens, lens, k, got):
    lp, ent, top, val = got
    B, T = np.shape(nodes)
    assert lp.shape == ent.shape == (B, T) and top.shape == val.shape == (B, T, k)
    for b in range(B):
        for i in range(T):
            if i >= lens[b]:
                assert lp[b, i] == 0 and ent[b, i] == 0 and (top[b, i] == -1).all() and (val[b, i] == 0).all()
                continue
            w = kv8_ref.logprobs(x[b, nodes[b][i]], tokens[b][i], k)
            near = lambda a, r: np.array_equal(np.isfinite(a), np.isfinite(r)) and np.all((np.abs(a - r) <= 1e-5 + 2.0 ** -22 * np.abs(r))[np.isfinite(r)])
            with np.errstate(invalid="ignore"):
                assert near(lp[b, i], w[0]), (b, i, lp[b, i], w[0])
                assert near(val[b, i], w[3]), (b, i)
            assert abs(ent[b, i] - w[1]) <= 1e-5 * (1 + w[1]), (b, i, ent[b, i], w[1])
            assert np.array_equal(top[b, i], w[2]), (b, i, top[b, i], w[2])


@pytest.mark.parametrize("V", [1, 2, 3, 5, 31, 100, 1000, 1003, 8191, 8192, 8193, 32000, 50257, 128256])
@pytest.mark.parametrize("k", [0, 1, 5, 20, 32])
def test_vocabularies(V, k):
    k = min(k, V)
    rng = np.random.default_rng([V, k])
    B, N, T = 2, 5, 4
    x = (rng.standard_normal((B, N, V)) * 3).astype(np.float32)
    x[0, 2] = np.round(x[0, 2])                                # many equal entries
    x[1, 4, V // 2] = 30.0
    nodes, lens = rng.integers(0, N, (B, T)), [4, 3]
    tokens = rng.integers(0, V, (B, T))
    got, status = run(x, nodes, tokens, lens, k)
    assert status == 0
    check(x, nodes, tokens, lens, k, got)


@pytest.mark.parametrize("what", ["equal", "descending", "ascending", "filtered", "one", "lowest", "huge", "zeros of both signs", "a thread's share"])
@pytest.mark.parametrize("V", [37, 9001, 20000])
def test_rows_of_every_kind(what, V):
    rng = np.random.default_rng(V)
    x = rng.standard_normal((1, 2, V)).astype(np.float32)
    if what == "equal":
        x[:] = 0.25
    elif what == "descending":
        x[:] = -np.arange(V) * np.float32(0.01)
    elif what == "ascending":
        x[:] = np.arange(V) * np.float32(0.01)
    elif what == "filtered":                                   # fewer entries than alternatives
        keep = rng.permutation(V)[:7]
        y = np.full_like(x, -np.inf)
        y[..., keep] = x[..., keep]
        x = y
    elif what == "one":
        x[:] = -np.inf
        x[..., V // 3] = -2.0
    elif what == "lowest":                                     # masked with the type's lowest value
        x[..., rng.permutation(V)[:V - 9]] = np.finfo(np.float32).min
    elif what == "huge":
        x *= 1e30
    elif what == "zeros of both signs":
        x[:] = -1.0
        x[..., ::3] = 0.0
        x[..., 1::3] = -0.0
    else:                                                      # the best entries next to one another
        x[..., 4:36] += 50
    t = rng.integers(0, V, (1, 3))
    t[0, 0] = int(np.argmax(x[0, 0]))
    got, status = run(x, [[0, 1, 1]], t, [3], 32)
    assert status == 0
    check(x, [[0, 1, 1]], t, [3], 32, got)


def test_rows_without_a_distribution_and_indices_out_of_range():
    x = np.random.default_rng(1).standard_normal((1, 6, 5000)).astype(np.float32)
    x[0, 1] = -np.inf
    x[0, 2, 4999] = np.inf
    x[0, 3, 17] = np.nan
    (lp, ent, top, val), status = run(x, [[0, 1, 2, 3, 6, -1, 5]], [[5000, 1, 1, 1, 1, 1, -1]], [7], 3)
    assert status == 0x1 | 0x2 | 0x40
    assert np.isnan(lp).all()
    assert np.isfinite(ent[0, [0, 6]]).all() and np.isnan(ent[0, 1:6]).all()
    assert (top[0, 1:6] == -1).all() and (top[0, [0, 6]] >= 0).all() and np.isnan(val[0, 1:6]).all()
    for flag, i in ((0x40, 1), (0x40, 2), (0x40, 3), (0x1, 6)):
        assert run(x, [[i]], [[1]], [1], 0)[1] == flag
    assert run(x, [[0]], [[-1]], [1], 2)[1] == 0x2


@pytest.mark.parametrize("B,N,T,V", [(1, 1, 1, 200000), (1, 1, 1, 1 << 20), (40, 3, 3, 999), (300, 2, 2, 50), (4, 64, 64, 3001), (2, 512, 512, 77)])
def test_batches(B, N, T, V):
    rng = np.random.default_rng([B, V])
    x = (rng.standard_normal((B, N, V)) * 2).astype(np.float32)
    nodes, tokens = rng.integers(0, N, (B, T)), rng.integers(0, V, (B, T))
    lens = rng.integers(0, T + 1, B)
    lens[0] = T
    got, status = run(x, nodes, tokens, lens, 5)
    assert status == 0
    check(x, nodes, tokens, lens, 5, got)


@pytest.mark.parametrize("k", [0, 3, 32])
def test_rows_shared_out_between_warps_that_take_more_than_one(k):
    rng = np.random.default_rng(k)
    B, N, T, V = 4, 60, 300, 20483                             # 1.3 to 7 loads of a warp, from the middle of a row to another's
    x = (rng.standard_normal((B, N, V)) * 2).astype(np.float32)
    x[1, 7] = 1.5
    x[3, 5] = np.arange(V, dtype=np.float32) * np.float32(1e-3)
    nodes, tokens = rng.integers(0, N, (B, T)), rng.integers(0, V, (B, T))
    nodes[1, 20:25], nodes[3, 9] = 7, 5
    for lens in ([300, 0, 211, 300], [0, 0, 0, 77], [0, 260, 0, 0]):
        got, status = run(x, nodes, tokens, lens, k)
        assert status == 0
        seen = [min(n, 40) for n in lens]                      # (the oracle takes its time)
        check(x, nodes[:, :40], tokens[:, :40], seen, k, [g[:, :40] for g in got])
        for b in range(B):
            if lens[b] > 40:
                check(x[b:b + 1], nodes[b:b + 1, lens[b] - 9:lens[b]], tokens[b:b + 1, lens[b] - 9:lens[b]], [9], k, [g[b:b + 1, lens[b] - 9:lens[b]] for g in got])
            assert (got[0][b, lens[b]:] == 0).all()


@pytest.mark.parametrize("B", [1023, 1024, 1025, 2500])
def test_more_sequences_than_a_group(B):
    rng = np.random.default_rng(B)
    T, V = 3, 41
    x = rng.standard_normal((B, 2, V)).astype(np.float32)
    nodes, tokens, lens = rng.integers(0, 2, (B, T)), rng.integers(0, V, (B, T)), rng.integers(0, T + 1, B)
    lens[B // 2:B // 2 + 100] = 0
    got, status = run(x, nodes, tokens, lens, 4)
    assert status == 0
    check(x, nodes, tokens, lens, 4, got)


def test_lengths_are_clamped_and_outputs_may_be_given():
    x = np.random.default_rng(2).standard_normal((2, 3, 400)).astype(np.float32)
    out = (torch.full((2, 3), 7.0, device="cuda"), torch.full((2, 3), 7.0, device="cuda"),
           torch.full((2, 3, 4), 7, dtype=torch.int32, device="cuda"), torch.full((2, 3, 4), 7.0, device="cuda"))
    nodes, tokens = [[0, 1, 2]] * 2, [[3, 4, 5]] * 2
    got, _ = run(x, nodes, tokens, [-5, 99], 4, out=out)
    check(x, nodes, tokens, [0, 3], 4, got)


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_rows_that_start_anywhere(shift):
    rng = np.random.default_rng(shift)
    flat = torch.randn(2 * 3 * 10001 + 8, device="cuda")
    x = flat[shift:shift + 2 * 3 * 10001].view(2, 3, 10001)
    nodes, tokens = rng.integers(0, 3, (2, 3)), rng.integers(0, 10001, (2, 3))
    got, status = run(x, nodes, tokens, [3, 3], 8)
    assert status == 0
    check(x.cpu().numpy(), nodes, tokens, [3, 3], 8, got)


def test_captured_calls_that_share_scratch():
    import paper_2407_16207_b200 as gsd
    g0 = torch.Generator(device="cuda").manual_seed(1)
    xs = [torch.randn((3, 8, 9000), generator=g0, device="cuda") for _ in range(2)]
    nodes = torch.arange(8, device="cuda", dtype=torch.int32).expand(3, 8).contiguous()
    tokens = nodes * 1000
    lens = torch.tensor([8, 0, 5], device="cuda", dtype=torch.int32)
    ws = torch.empty(gsd.gsd_token_logprobs_workspace_bytes(3, 8, 9000, 8, 6), dtype=torch.uint8, device="cuda")
    plain = [gsd.gsd_token_logprobs(x, nodes, tokens, lens, k=6) for x in xs]
    got, graphs = [], []
    for x in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(gsd.gsd_token_logprobs(x, nodes, tokens, lens, k=6, workspace=ws))
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, plain):
            assert all(torch.equal(u, v) for u, v in zip(a, b))
