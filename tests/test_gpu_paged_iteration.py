"""The calls around the paged cache as a server makes them: prompts, then iterations of rotation, mask, attention, acceptance, log
probabilities and commit, without anything between the calls; also with the index-checking build, through captured graphs that
share a workspace, and with margins around every buffer."""
import numpy as np
import pytest
import torch

import kv8_ref
from paged_ref import attn_check, attn_inputs, attn_tensors, bf16, i32, rows_of, table_for, turn, turn_tol
from test_gpu_q8_iteration import chain_graph, checked_lib, margins  # noqa: F401

pytestmark = pytest.mark.gpu


def iterate(gsd, D, page, N, Hq, Hkv, steps=3, V=1003, kernel=0, neighbours=False, axes=None):
    rng = np.random.default_rng([D, N, Hq])
    B, T, most = 3, 50, 200
    M = -(-most // page)
    table, P = table_for(rng, [M] * B, M)
    kp, vp = (torch.full((P, page, Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    n, A = D // 2, 3 if axes else 1
    freqs = (10000.0 ** (-np.arange(n) / n)).astype(np.float32)
    axes = [i % 3 for i in range(n)] if axes else None
    rot = dict(axes=axes, pairs=neighbours)
    axes = axes or [0] * n
    counts = [T, 17, 1]
    tb, f, sl, cnt = i32(table), torch.from_numpy(freqs).cuda(), torch.zeros(B, dtype=torch.int32, device="cuda"), i32(counts)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    prompt = bf16(rng.standard_normal((B, T, Hq + 2 * Hkv, D)))
    ptr, idx, see = chain_graph(B, N)
    h = (N - 1) // 2
    depth = np.concatenate((np.arange(h + 1), np.arange(1, N - h)))
    pos = np.broadcast_to(depth, (A, B, N)).astype(np.int32)
    ins = []
    for _ in range(steps):
        tok = rng.integers(0, V, (B, N)).astype(np.int32)
        x = rng.standard_normal((B, N, V)).astype(np.float32)
        for b in range(B):                                # the model agrees with the first b + 1 nodes of a chain
            at = list(range(h + 1))
            for p, c in list(zip(at[:-1], at[1:]))[:b + 1]:
                x[b, p, tok[b, c]] = 9.0
        ins.append(dict(qkv=bf16(rng.standard_normal((B, N, Hq + 2 * Hkv, D))), tok=tok, x=x))
    dev = [dict(qkv=i["qkv"].cuda(), tok=i32(i["tok"]), x=torch.from_numpy(i["x"]).cuda()) for i in ins]
    pd, posd = prompt.cuda(), i32(pos)
    said = []
    torch.cuda.synchronize()
    gsd.gsd_append_kv_paged(kp, vp, tb, pd[:, :, Hq:Hq + Hkv], pd[:, :, Hq + Hkv:], cnt, sl, freqs=f, status=status, **rot)
    for i in dev:
        q, k = gsd.gsd_rotary(i["qkv"][:, :, :Hq], i["qkv"][:, :, Hq:Hq + Hkv], f, posd, offsets=sl, **rot)
        v = i["qkv"][:, :, Hq + Hkv:].contiguous()
        mask = gsd.gsd_build_mask(ptr, idx, status=status)
        out = gsd.gsd_verify_attn_paged(q, kp, vp, tb, k, v, mask, sl, status=status, kernel=kernel)
        toks, alen, nodes = gsd.gsd_accept(i["x"], i["tok"], ptr, idx, status=status)
        lp = gsd.gsd_token_logprobs(i["x"], nodes, toks, alen, k=4, status=status)
        gsd.gsd_commit_kv_paged(kp, vp, tb, k, v, nodes, alen, sl, status=status)
        said.append((q, k, v, out, alen, lp))
    torch.cuda.synchronize()
    assert int(status.item()) == 0

    double = lambda t: t.double().cpu().numpy()
    lens = list(counts)
    K, V_ = kp.cpu(), vp.cpu()
    for b in range(B):
        raw = double(prompt[b, :counts[b], Hq:Hq + Hkv])
        ref = turn(raw, np.broadcast_to(np.arange(counts[b]), (3, counts[b])), freqs, axes, neighbours)
        got = double(rows_of(K, table[b], counts[b]))
        assert (np.abs(got - ref) <= turn_tol(raw, ref, n, neighbours)).all()
        assert torch.equal(rows_of(V_, table[b], counts[b]), prompt[b, :counts[b], Hq + Hkv:])
    for i, (q, k, v, out, alen, lp) in zip(ins, said):
        for b in range(B):
            for got, lo, hi in ((q, 0, Hq), (k, Hq, Hq + Hkv)):
                raw = double(i["qkv"][b, :, lo:hi])
                ref = turn(raw, pos[:, b] + lens[b] if A == 3 else np.broadcast_to(pos[0, b] + lens[b], (3, N)), freqs, axes, neighbours)
                assert (np.abs(double(got[b]) - ref) <= turn_tol(raw, ref, n, neighbours)).all()
        x = dict(B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, lens=np.asarray(lens), page=page, table=table, k=K, v=V_, q=q.cpu(), dk=k.cpu(), dv=v.cpu(),
                 see=np.broadcast_to(see, (B, N, N)))
        attn_check(x, out)
        m = [min(b + 1, h) for b in range(B)]
        assert alen.tolist() == [s + 1 for s in m]
        lp = lp[0].cpu().numpy()
        for b in range(B):
            w = kv8_ref.logprobs(i["x"][b, 0], int(i["tok"][b, 1]) if m[b] else int(np.argmax(i["x"][b, 0])), 1)
            assert abs(lp[b, 0] - w[0]) < 1e-5
            path = list(range(m[b] + 1))
            for pool, rows in ((K, k), (V_, v)):
                assert torch.equal(rows_of(pool, table[b], lens[b] + m[b] + 1)[lens[b]:], rows[b, path].cpu())
            lens[b] += m[b] + 1
    assert sl.tolist() == lens
    for b in range(B):                                    # and nothing behind the ends
        j = np.arange(lens[b], M * page)
        assert K[table[b, j // page], j % page].isnan().all() and V_[table[b, j // page], j % page].isnan().all()


CASES = [(128, 64, 9, 8, 2), (64, 16, 5, 4, 4), (128, 32, 40, 16, 2), (64, 128, 33, 8, 1), (128, 16, 1, 8, 1), (128, 256, 70, 12, 4)]


@pytest.mark.parametrize("D,page,N,Hq,Hkv", CASES)
@pytest.mark.parametrize("kernel,neighbours,axes", [(0, False, None), (1, True, 3)])
def test_iterations(D, page, N, Hq, Hkv, kernel, neighbours, axes):
    import paper_2407_16207_b200 as gsd
    iterate(gsd, D, page, N, Hq, Hkv, kernel=kernel, neighbours=neighbours, axes=axes)


@pytest.mark.parametrize("D,page,N,Hq,Hkv", CASES)
def test_iterations_with_the_checking_build(checked_lib, D, page, N, Hq, Hkv):  # noqa: F811
    iterate(checked_lib, D, page, N, Hq, Hkv)


@pytest.mark.parametrize("D,N,Hq,Hkv,splits,kernel,page", [(128, 5, 8, 2, 3, 1, 16), (64, 21, 3, 1, 2, 0, 32), (128, 77, 8, 8, 0, 0, 64),
                                                           (128, 77, 16, 2, 5, 2, 128), (64, 50, 12, 4, 0, 0, 16), (128, 40, 12, 4, 0, 0, 256)])
def test_nothing_outside_the_buffers_is_written(D, N, Hq, Hkv, splits, kernel, page):
    import paper_2407_16207_b200 as gsd
    x = attn_inputs(21, 3, N, Hq, Hkv, D, [301, 100, 0], page, M=-(-301 // page) + 4)
    t = attn_tensors(x)
    out, ok_out = margins((3, N, Hq, D), torch.bfloat16)
    need = gsd.gsd_verify_attn_paged_workspace_bytes(3, N, Hq, Hkv, D, page, x["table"].shape[1], num_splits=splits, kernel=kernel)
    ws, ok_ws = margins((max(need, 256),), torch.uint8)
    gsd.gsd_verify_attn_paged(**t, out=out, num_splits=splits, kernel=kernel, workspace=ws)
    attn_check(x, out)
    assert ok_out() and ok_ws()
    # a pool that is full to its last row: the last pages are the sequences' own
    M = -(-(100 + N) // page) + 1
    table = np.arange(2 * M)[::-1].reshape(2, M).astype(np.int32)
    kv = {n: margins((2 * M, page, Hkv, D), torch.bfloat16) for n in "kv"}
    sl, ok_sl = margins((2,), torch.int32, torch.tensor([M * page - N - 1, 3], dtype=torch.int32))
    rows = torch.randn((2, N, Hkv, D), device="cuda").to(torch.bfloat16)
    gsd.gsd_append_kv_paged(kv["k"][0], kv["v"][0], i32(table), rows, rows, i32([N, N]), sl)
    gsd.gsd_commit_kv_paged(kv["k"][0], kv["v"][0], i32(table), rows, rows, i32([[0, 0]] * 2), i32([2, 1]), sl)
    assert sl.tolist() == [M * page, N + 4]
    assert ok_sl() and all(ok() for _, ok in kv.values())


def test_two_graphs_share_a_workspace_and_take_turns():
    import paper_2407_16207_b200 as gsd
    xs = [attn_inputs(31 + s, 3, n, 8, 2, 128, lens, 32, M=20) for s, (n, lens) in enumerate(((1, [600, 40, 333]), (4, [31, 640, 200]), (60, [640, 1, 500])))]
    ts = [attn_tensors(x) for x in xs]
    need = max(gsd.gsd_verify_attn_paged_workspace_bytes(3, x["N"], 8, 2, 128, 32, 20) for x in xs)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(t["q"]) for t in ts]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(s):
        for t, o in zip(ts, outs):
            gsd.gsd_verify_attn_paged(**t, out=o, workspace=ws)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                gsd.gsd_verify_attn_paged(**t, out=o, workspace=ws)
            graphs.append(g)
        for order in ((0, 1, 2), (2, 0, 1), (1, 1, 2, 0)):
            for o in outs:
                o.fill_(float("nan"))
            ws.fill_(0xFF)
            for i in order:
                graphs[i].replay()
            s.synchronize()
            for x, o in zip(xs, outs):
                attn_check(x, o)


def test_two_streams_with_workspaces_of_their_own():
    import paper_2407_16207_b200 as gsd
    xs = [attn_inputs(41 + s, 2, n, 8, 2, 128, [2000, 1500], 16) for s, n in enumerate((1, 40))]
    ts = [attn_tensors(x) for x in xs]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in ts], [None, None]
    for _ in range(5):
        for i, (s, t) in enumerate(zip(streams, ts)):
            with torch.cuda.stream(s):
                outs[i] = gsd.gsd_verify_attn_paged(**t)
    torch.cuda.synchronize()
    for x, o in zip(xs, outs):
        attn_check(x, o)


def test_repeated_calls_are_identical():
    import paper_2407_16207_b200 as gsd
    for N, kernel, D in ((1, 0, 128), (4, 1, 128), (90, 0, 128), (9, 0, 64)):
        x = attn_inputs(51, 4, N, 8, 2, D, [1999, 77, 1024, 500], 16)
        t = attn_tensors(x)
        first = gsd.gsd_verify_attn_paged(**t, kernel=kernel)
        for _ in range(5):
            assert torch.equal(first, gsd.gsd_verify_attn_paged(**t, kernel=kernel))
