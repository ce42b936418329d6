"""The calls around the 8-bit cache as a server makes them: prompts, then iterations of attention, acceptance, log
probabilities and commit, without anything between the calls; also with the index-checking build, and with margins
around every buffer."""
import numpy as np
import pytest
import torch

import kv8_ref
from test_gpu_attn_q8 import DT, check
from test_gpu_kv8_write import rows_like

pytestmark = pytest.mark.gpu


@pytest.fixture()
def checked_lib():
    from paper_2407_16207_b200 import binding, build
    path = build.build(checked=True)
    saved = (binding._lib, binding._LIB_PATH)
    binding._lib, binding._LIB_PATH = None, path
    try:
        import paper_2407_16207_b200 as gsd
        assert gsd.lib()._name == path
        yield gsd
    finally:
        binding._lib, binding._LIB_PATH = saved


def chain_graph(B, N):
    """Two chains from the root: parents of 1..h and h + 1..N - 1."""
    h = (N - 1) // 2
    par = [[]] + [[v - 1] for v in range(1, h + 1)] + [[0 if v == h + 1 else v - 1] for v in range(h + 1, N)]
    ptr = np.cumsum([0] + [len(p) for p in par])
    i32 = lambda a: torch.from_numpy(np.tile(np.asarray(a, np.int32), (B, 1))).cuda()
    see = np.eye(N, dtype=bool)
    for v in range(1, N):
        see[v] |= see[par[v][0]]
    return i32(ptr), i32([p[0] for p in par[1:]] or [-1]), see


def iterate(gsd, fmt, D, block, N, Hq, Hkv, steps=3, V=1003, kernel=0):
    rng = np.random.default_rng([D, N, Hq])
    B, T, Lmax = 3, 50, 200
    codes = rng.integers(0, 127, (2, B, Lmax, Hkv, D)).astype(np.uint8)
    exps = np.full((2, B, -(-Lmax // block), Hkv), 100, np.int8)
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    kc, vc = (cuda(codes[i].view(np.int8)).view(DT[fmt]) for i in range(2))
    ke, ve = cuda(exps[0]), cuda(exps[1])
    lens = [0] * B
    counts = [T, 17, 1]
    sl, cnt = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.tensor(counts, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = rows_like(rng, B, T, Hkv, D), rows_like(rng, B, T, Hkv, D)
    ptr, idx, see = chain_graph(B, N)
    said = []
    ins = []
    for _ in range(steps):
        tok = rng.integers(0, V, (B, N)).astype(np.int32)
        x = rng.standard_normal((B, N, V)).astype(np.float32)
        h = (N - 1) // 2
        for b in range(B):                                # the model agrees with the first b + 1 nodes of a chain
            at = [0] + list(range(1, h + 1))
            for p, c in list(zip(at[:-1], at[1:]))[:b + 1]:
                x[b, p, tok[b, c]] = 9.0
        ins.append(dict(q=rows_like(rng, B, N, Hq, D), dk=rows_like(rng, B, N, Hkv, D), dv=rows_like(rng, B, N, Hkv, D), tok=tok, x=x))
    dev = [{n: (a if isinstance(a, torch.Tensor) else torch.from_numpy(a)).cuda() for n, a in i.items()} for i in ins]
    kd, vd = k.cuda(), v.cuda()
    torch.cuda.synchronize()
    gsd.gsd_append_kv_q8(kc, vc, ke, ve, kd, vd, cnt, sl, block=block, status=status)
    for i in dev:
        mask = gsd.gsd_build_mask(ptr, idx, status=status)
        out = gsd.gsd_verify_attn_q8(i["q"], kc, vc, ke, ve, i["dk"], i["dv"], mask, sl, block=block, status=status, kernel=kernel)
        toks, alen, nodes = gsd.gsd_accept(i["x"], i["tok"], ptr, idx, status=status)
        lp = gsd.gsd_token_logprobs(i["x"], nodes, toks, alen, k=4, status=status)
        gsd.gsd_commit_kv_q8(kc, vc, ke, ve, i["dk"], i["dv"], nodes, alen, sl, block=block, status=status)
        said.append((out, toks, alen, nodes, lp))
    torch.cuda.synchronize()
    assert int(status.item()) == 0

    def append(rows_k, rows_v, n):
        for b in range(B):
            new = [kv8_ref.append(codes[kv, b], exps[kv, b], r[b][:n[b]], lens[b], fmt, block) for kv, r in enumerate((rows_k, rows_v))]
            lens[b] = new[0]
    f = lambda t: t.double().numpy()
    append(f(k), f(v), counts)
    for i, (out, toks, alen, nodes, lp) in zip(ins, said):
        x = dict(B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, lens=lens, fmt=fmt, block=block, k=codes[0], ke=exps[0], v=codes[1], ve=exps[1],
                 q=i["q"], dk=i["dk"], dv=i["dv"], see=np.broadcast_to(see, (B, N, N)))
        check(x, out)
        h = (N - 1) // 2
        m = [min(b + 1, h) for b in range(B)]
        assert alen.tolist() == [n + 1 for n in m]
        path = [list(range(n + 1)) for n in m]
        lp = [t.cpu().numpy() for t in lp]
        for b in range(B):
            for j, node in enumerate(path[b]):
                w = kv8_ref.logprobs(i["x"][b, node], int(toks[b, j]), 4)
                assert abs(lp[0][b, j] - w[0]) < 1e-5 and abs(lp[1][b, j] - w[1]) < 1e-5 * (1 + w[1])
                assert np.array_equal(lp[2][b, j], w[2]) and np.abs(lp[3][b, j] - w[3]).max() < 1e-5
            assert (lp[2][b, m[b] + 1:] == -1).all() and (lp[0][b, m[b] + 1:] == 0).all()
        append([f(i["dk"])[b, path[b]] for b in range(B)], [f(i["dv"])[b, path[b]] for b in range(B)], alen.tolist())
    assert sl.tolist() == lens
    for got, c, ex, e in ((kc, codes[0], ke, exps[0]), (vc, codes[1], ve, exps[1])):
        assert np.array_equal(got.view(torch.uint8).cpu().numpy(), c) and np.array_equal(ex.cpu().numpy(), e)


CASES = [("e4m3", 128, 64, 9, 8, 2), ("int8", 64, 16, 5, 4, 4), ("int8", 128, 32, 40, 16, 2), ("e4m3", 64, 128, 33, 8, 1), ("e4m3", 128, 16, 1, 8, 1)]


@pytest.mark.parametrize("fmt,D,block,N,Hq,Hkv", CASES)
@pytest.mark.parametrize("kernel", [0, 1])
def test_iterations(fmt, D, block, N, Hq, Hkv, kernel):
    import paper_2407_16207_b200 as gsd
    iterate(gsd, fmt, D, block, N, Hq, Hkv, kernel=kernel)


@pytest.mark.parametrize("fmt,D,block,N,Hq,Hkv", CASES)
def test_iterations_with_the_checking_build(checked_lib, fmt, D, block, N, Hq, Hkv):
    iterate(checked_lib, fmt, D, block, N, Hq, Hkv)


def margins(shape, dtype, fill=None):
    """A tensor between two margins of 4 KB, and a function that says whether they are as they were."""
    n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
    flat = torch.full((n + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    t = flat[4096:4096 + n].view(dtype).view(shape)
    if fill is not None:
        t.copy_(fill)
    return t, lambda: bool((flat[:4096] == 0xA5).all() and (flat[4096 + n:] == 0xA5).all())


@pytest.mark.parametrize("fmt,D,N,Hq,Hkv,splits,kernel", [("e4m3", 128, 5, 8, 2, 3, 1), ("int8", 64, 21, 3, 1, 2, 0), ("int8", 128, 77, 8, 8, 0, 0),
                                                          ("e4m3", 128, 77, 16, 2, 5, 2), ("e4m3", 64, 50, 12, 4, 0, 0), ("int8", 128, 40, 12, 4, 0, 0)])
def test_nothing_outside_the_buffers_is_written(fmt, D, N, Hq, Hkv, splits, kernel):
    import paper_2407_16207_b200 as gsd
    from test_gpu_attn_q8 import make, tensors
    x = make(21, 3, N, Hq, Hkv, D, 301, [301, 100, 0], fmt, 32)
    t = tensors(x)
    out, ok_out = margins((3, N, Hq, D), torch.bfloat16)
    need = gsd.gsd_verify_attn_q8_workspace_bytes(3, N, Hq, Hkv, D, 301, block=32, num_splits=splits, kernel=kernel)
    ws, ok_ws = margins((max(need, 256),), torch.uint8)
    gsd.gsd_verify_attn_q8(**t, out=out, block=32, num_splits=splits, kernel=kernel, workspace=ws)
    check(x, out)
    assert ok_out() and ok_ws()
    kv = {n: margins(tuple(t[n].shape), t[n].dtype, t[n]) for n in ("k_cache", "v_cache", "k_exp", "v_exp", "seq_lens")}
    c = [kv[n][0] for n in ("k_cache", "v_cache", "k_exp", "v_exp")]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    gsd.gsd_commit_kv_q8(*c, t["draft_k"], t["draft_v"], i32([[0, 1, 2]] * 3), i32([3, 2, 3]), kv["seq_lens"][0], block=32)
    gsd.gsd_append_kv_q8(*c, t["draft_k"], t["draft_v"], i32([N, N, N]), kv["seq_lens"][0], block=32)
    assert kv["seq_lens"][0].tolist() == [301, min(301, 102 + N), min(301, 3 + N)]
    assert all(ok() for _, ok in kv.values())
    V, T, k = 5003, 7, 9
    lg = torch.randn((3, N, V), device="cuda")
    outs = [margins((3, T), torch.float32), margins((3, T), torch.float32), margins((3, T, k), torch.int32), margins((3, T, k), torch.float32)]
    need = gsd.gsd_token_logprobs_workspace_bytes(3, N, V, T, k)
    ws, ok_ws = margins((need,), torch.uint8)
    gsd.gsd_token_logprobs(lg, torch.zeros((3, T), dtype=torch.int32, device="cuda"), torch.ones((3, T), dtype=torch.int32, device="cuda"),
                           i32([7, 0, 3]), k=k, workspace=ws, out=tuple(o for o, _ in outs))
    assert ok_ws() and all(ok() for _, ok in outs)
