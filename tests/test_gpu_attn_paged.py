"""gsd_verify_attn_paged against a 64-bit evaluation of its definition (tolerances: paged_ref)."""
import numpy as np
import pytest
import torch

from paged_ref import attn_check, attn_inputs, attn_tensors, i32

pytestmark = pytest.mark.gpu
PAGES = [16, 32, 64, 128, 256]


def call(x, **kw):
    import paper_2407_16207_b200 as gsd
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = gsd.gsd_verify_attn_paged(**attn_tensors(x), status=status, **kw)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return out


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("kernel", [0, 1])
def test_single_tokens(page, D, kernel):
    # lengths around tiles and pages, none and one among them; what lies behind the ends is NaN
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511]
    for Hq, Hkv in ((8, 1), (4, 4), (6, 2)):
        x = attn_inputs(1, len(lens), 1, Hq, Hkv, D, lens, page, mask="chain")
        attn_check(x, call(x, kernel=kernel))


@pytest.mark.parametrize("page", PAGES)
def test_single_tokens_on_the_tcgen05_kernel(page):
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511]
    x = attn_inputs(1, len(lens), 1, 8, 2, 128, lens, page, mask="chain")
    for splits in (0, 1, 3):
        attn_check(x, call(x, kernel=2, num_splits=splits))


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("N,Hq,Hkv", [(2, 8, 8), (9, 4, 2), (16, 3, 1), (33, 8, 2), (7, 28, 4), (64, 4, 4), (100, 6, 2), (130, 8, 1), (257, 2, 2), (512, 1, 1)])
def test_draft_graphs(page, D, N, Hq, Hkv):
    x = attn_inputs(2, 3, N, Hq, Hkv, D, [699, 130, 5], page)
    attn_check(x, call(x))


@pytest.mark.parametrize("kernel", [0, 1, 2])
@pytest.mark.parametrize("splits", [0, 1, 2, 3, 7, 64])
def test_key_ranges(kernel, splits):
    for page, N, Hq, Hkv in ((16, 5, 8, 2), (128, 40, 8, 1), (256, 90, 4, 2)):
        x = attn_inputs(3, 2, N, Hq, Hkv, 128, [1100, 333], page)
        attn_check(x, call(x, num_splits=splits, kernel=kernel))


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("B,Hkv,G,N", [(40, 8, 4, 33), (30, 16, 1, 130), (5, 8, 8, 40), (160, 1, 8, 16)])
def test_many_items(page, B, Hkv, G, N):
    # the plans made from the lengths: longest first, one wave, several units a CTA
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 700, B).tolist()
    x = attn_inputs(4, B, N, Hkv * G, Hkv, 128, lens, page)
    attn_check(x, call(x))


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("B,Hkv,G,N", [(1, 2, 4, 30), (3, 4, 4, 17), (5, 8, 4, 12), (12, 8, 1, 32), (10, 10, 3, 11), (33, 3, 5, 9), (40, 6, 4, 13)])
@pytest.mark.parametrize("longest", [250, 2600])
def test_items_of_every_size(B, Hkv, G, N, D, longest):
    # as the pairs grow in number, their rows are shared out among fewer items; left whole, cut alike and cut by length
    rng = np.random.default_rng([B, N])
    lens = rng.integers(0, 200, B)
    lens[B // 2] = longest
    x = attn_inputs(11, B, N, Hkv * G, Hkv, D, lens.tolist(), 32)
    out = call(x, kernel=1)
    attn_check(x, out)
    attn_check(x, call(x))
    assert torch.equal(out, call(x, kernel=1))


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("B,Hkv,G,N", [(2, 8, 4, 2), (3, 4, 7, 1), (4, 8, 1, 8), (8, 8, 8, 1), (5, 3, 3, 2), (9, 1, 5, 1), (30, 2, 2, 3), (20, 2, 4, 2), (13, 2, 8, 1)])
def test_ranges_of_a_cluster(B, Hkv, G, N, D):
    # a cluster of two to eight CTAs an item: no workspace; none of the keys, one, a range without any, a page that is not there
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng([B, Hkv, N])
    lens = rng.integers(0, 1800, B)
    lens[0], lens[1], lens[-1] = 0, 1, 1800
    x = attn_inputs(12, B, N, Hkv * G, Hkv, D, lens.tolist(), 32)
    assert gsd.gsd_verify_attn_paged_workspace_bytes(B, N, Hkv * G, Hkv, D, 32, x["table"].shape[1]) == 0
    out = call(x)
    attn_check(x, out)
    assert torch.equal(out, call(x))
    attn_check(x, call(x, num_splits=3))
    x["table"][-1, 20] = x["k"].shape[0]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = gsd.gsd_verify_attn_paged(**attn_tensors(x), status=status)
    assert int(status.item()) == 0x1000
    x["table"][-1, 20] = 0
    x["k"] = torch.cat([x["k"], torch.zeros_like(x["k"][:1])])
    x["v"] = torch.cat([x["v"], torch.zeros_like(x["v"][:1])])
    x["table"][-1, 20] = x["k"].shape[0] - 1
    attn_check(x, out)


@pytest.mark.parametrize("kernel", [1, 2])
def test_rows_that_see_nothing_are_zero(kernel):
    x = attn_inputs(5, 2, 11, 8, 2, 128, [0, 40], 16, mask="none")
    got = call(x, kernel=kernel)
    assert (got[0] == 0).all()
    attn_check(x, got)


@pytest.mark.parametrize("N,kernel", [(1, 0), (20, 1), (20, 2), (70, 0)])
def test_a_common_prompt(N, kernel):
    x = attn_inputs(6, 6, N, 8, 2, 128, [96, 97, 150, 96, 400, 111], 32, shared=3)
    attn_check(x, call(x, kernel=kernel))


@pytest.mark.parametrize("N,kernel", [(1, 0), (40, 1), (40, 2)])
def test_a_bound_on_the_lengths_below_the_room(N, kernel):
    x = attn_inputs(7, 3, N, 8, 2, 128, [300, 17, 200], 16, M=1000)
    attn_check(x, call(x, kernel=kernel, max_len=300))
    attn_check(x, call(x, kernel=kernel))


@pytest.mark.parametrize("N,Hq,Hkv,kernel", [(1, 8, 2, 0), (1, 8, 2, 1), (30, 4, 2, 1), (30, 8, 2, 2), (200, 8, 2, 0)])
@pytest.mark.parametrize("D", [128, 64])
def test_the_padded_call_gives_the_same(N, Hq, Hkv, kernel, D):
    # the same rows in one padded range per sequence, the same kernel: the same sums up to their order
    import paper_2407_16207_b200 as gsd
    if kernel == 2 and D == 64:
        kernel = 0
    lens = [640, 0, 129, 77]
    x = attn_inputs(8, 4, N, Hq, Hkv, D, lens, 32)
    t = attn_tensors(x)
    flat = [torch.zeros((4, 640, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for b, L in enumerate(lens):
        for f, p in zip(flat, (t["k_pages"], t["v_pages"])):
            f[b, :L] = p[x["table"][b, :-(-L // 32)].tolist()].flatten(0, 1)[:L] if L else 0
    other = gsd.gsd_verify_attn(t["q"], *flat, t["draft_k"], t["draft_v"], t["ancestor_mask"], t["seq_lens"], kernel=kernel)
    got = call(x, kernel=kernel, max_len=640)
    attn_check(x, got)
    attn_check(x, other)


@pytest.mark.parametrize("scale", [0.02, 1.5])
def test_scale(scale):
    for N, kernel in ((3, 1), (40, 2)):
        x = attn_inputs(9, 2, N, 4, 2, 128, [100, 35], 16)
        attn_check(x, call(x, softmax_scale=scale, kernel=kernel), scale)


@pytest.mark.parametrize("N,kernel,D", [(1, 0, 128), (6, 1, 128), (6, 1, 64), (40, 2, 128), (80, 0, 64), (300, 0, 128)])
@pytest.mark.parametrize("page", [16, 128, 256])
def test_pages_that_the_table_does_not_name(N, kernel, D, page):
    # their rows count as zeros, and the call says so; nothing else does
    import paper_2407_16207_b200 as gsd
    x = attn_inputs(10, 3, N, 8, 2, D, [600, 257, 300], page)
    x["table"][0, 1], x["table"][2, (300 - 1) // page] = -1, x["k"].shape[0]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = gsd.gsd_verify_attn_paged(**attn_tensors(x), status=status, kernel=kernel)
    assert int(status.item()) == 0x1000
    z = torch.zeros((2,) + tuple(x["k"].shape[1:]), dtype=torch.bfloat16)
    P = x["k"].shape[0]
    x["k"], x["v"] = torch.cat((x["k"], z)), torch.cat((x["v"], z))
    x["table"][0, 1], x["table"][2, (300 - 1) // page] = P, P + 1
    attn_check(x, got)
    gsd.gsd_verify_attn_paged(**attn_tensors(x), kernel=kernel)         # (no status word: fine too)


@pytest.mark.parametrize("N,kernel", [(2, 1), (40, 2)])
def test_lengths_out_of_range_are_clamped(N, kernel):
    import paper_2407_16207_b200 as gsd
    x = attn_inputs(11, 2, N, 4, 2, 128, [96, 0], 16, M=6)
    t = attn_tensors(x)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    t["seq_lens"] = i32([97, -5])
    got = gsd.gsd_verify_attn_paged(**t, status=status, kernel=kernel)
    assert int(status.item()) == 0x10
    attn_check(x, got)


@pytest.mark.parametrize("kernel", [1, 2])
def test_large_and_infinite_keys_in_masked_places(kernel):
    x = attn_inputs(12, 2, 40, 8, 2, 128, [300, 45], 16, fill=np.inf)
    x["see"][:, :, 39] = False                   # nobody sees this draft row
    W = x["mask"].shape[2]
    bits = np.zeros((2, 40, W * 32), bool)
    bits[:, :, :40] = x["see"]
    x["mask"] = np.packbits(bits, axis=2, bitorder="little").view(np.int32)
    x["dk"][:, 39] = 3e38
    attn_check(x, call(x, kernel=kernel))


def test_a_pool_beyond_4_gb():
    # pages far apart: offsets beyond 32 bits in elements
    import paper_2407_16207_b200 as gsd
    P, page, Hkv, D = 140000, 16, 8, 128
    k, v = (torch.zeros((P, page, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for N, kernel in ((1, 0), (1, 1), (40, 2)):
        x = attn_inputs(13, 2, N, 16, 8, D, [100, 61], page)
        t = attn_tensors(x)
        where = np.array([[P - 1 - i, i * 997 + 3] for i in range(7)]).T.astype(np.int32)
        for b, L in enumerate(x["lens"].tolist()):
            for i in range(-(-L // page)):
                for pool, own in ((k, "k_pages"), (v, "v_pages")):
                    pool[int(where[b, i])] = t[own][int(x["table"][b, i])]
        t.update(k_pages=k, v_pages=v, page_table=i32(where))
        attn_check(x, gsd.gsd_verify_attn_paged(**t, kernel=kernel))


@pytest.mark.parametrize("N", [1, 50])
def test_captured_and_replayed_on_another_stream(N):
    import paper_2407_16207_b200 as gsd
    x, y = attn_inputs(14, 3, N, 8, 2, 128, [500, 3, 130], 32, M=20), attn_inputs(15, 3, N, 8, 2, 128, [77, 512, 0], 32, M=20)
    for z in (x, y):                             # pools of one size
        pad = 40 - z["k"].shape[0]
        z["k"], z["v"] = (torch.cat((z[n], torch.zeros((pad,) + tuple(z[n].shape[1:]), dtype=torch.bfloat16))) for n in "kv")
    t, u = attn_tensors(x), attn_tensors(y)
    ws = torch.empty(gsd.gsd_verify_attn_paged_workspace_bytes(3, N, 8, 2, 128, 32, 20), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(t["q"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        gsd.gsd_verify_attn_paged(**t, out=out, workspace=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            gsd.gsd_verify_attn_paged(**t, out=out, workspace=ws)
        for _ in range(2):
            g.replay()
        s.synchronize()
        attn_check(x, out)
        for n in t:
            t[n].copy_(u[n])
        g.replay()
        first = out.clone()
        g.replay()
        s.synchronize()
    attn_check(y, out)
    assert torch.equal(first, out)


@pytest.mark.parametrize("N", [1, 33])
def test_out_is_used_and_the_workspace_is_checked(N):
    import paper_2407_16207_b200 as gsd
    x = attn_inputs(16, 1, N, 8, 2, 128, [3000], 64)
    t = attn_tensors(x)
    out = torch.empty_like(t["q"])
    assert gsd.gsd_verify_attn_paged(**t, out=out) is out
    attn_check(x, out)
    need = gsd.gsd_verify_attn_paged_workspace_bytes(1, N, 8, 2, 128, 64, x["table"].shape[1])
    assert need > 0
    with pytest.raises(gsd.GsdError):
        gsd.gsd_verify_attn_paged(**t, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    # the Python path gives what the extension gives
    same = gsd.gsd_verify_attn_paged(**t, num_splits=np.int64(0))
    assert torch.equal(same, out)


@pytest.mark.parametrize("B,Hkv,G,N,D", [(40, 1, 8, 2, 128), (33, 2, 4, 5, 64), (200, 2, 1, 1, 128), (32, 8, 8, 1, 128), (2, 1, 160, 2, 128), (3, 2, 136, 1, 64)])
@pytest.mark.parametrize("kernel", [0, 1])
def test_few_rows_in_many_sequences_and_large_groups(B, Hkv, G, N, D, kernel):
    # more sequences than the plan by length takes, more items than CTAs, groups that the tcgen05 kernel does not take
    rng = np.random.default_rng([B, G])
    x = attn_inputs(22, B, N, Hkv * G, Hkv, D, rng.integers(0, 900, B).tolist(), 32)
    attn_check(x, call(x, kernel=kernel))


@pytest.mark.parametrize("kernel", [1, 2])
def test_rows_of_nan_stay_by_themselves(kernel):
    x = attn_inputs(23, 2, 9, 8, 2, 128, [130, 40], 16)
    clean = call(x, kernel=kernel)
    x["q"][1, 4, 3] = float("nan")
    got = call(x, kernel=kernel)
    assert got[1, 4, 3].isnan().all()
    got[1, 4, 3] = clean[1, 4, 3]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("kernel", [1, 2])
def test_large_scores(kernel):
    # scores of thousands, of either sign: weights are taken off the row's own maximum
    x = attn_inputs(24, 2, 20, 8, 2, 128, [200, 33], 16)
    x["q"] = (x["q"].float() * 64).to(torch.bfloat16)
    attn_check(x, call(x, kernel=kernel))


@pytest.mark.parametrize("fill", [float("nan"), float("inf")])
@pytest.mark.parametrize("N,Hq,Hkv,D,kernel", [(3, 8, 2, 128, 1), (17, 8, 8, 64, 1), (40, 8, 2, 128, 2), (200, 4, 4, 128, 2), (300, 6, 2, 64, 0), (512, 2, 1, 128, 0), (70, 8, 8, 64, 0), (20, 4, 4, 128, 0)])
def test_draft_rows_that_no_node_sees(N, Hq, Hkv, D, kernel, fill):
    # padded nodes, whatever their rows hold; one in the middle and all of the last ones
    x = attn_inputs(25, 3, N, Hq, Hkv, D, [150, 0, 400], 32)
    pad = [min(1, N - 1)] + list(range(max(2, N - N // 3), N))
    x["see"] = x["see"].copy()
    x["see"][:, :, pad] = False
    W = x["mask"].shape[2]
    bits = np.zeros((3, N, W * 32), bool)
    bits[:, :, :N] = x["see"]
    if N % 32:
        bits[:, 0, N:] = True
    x["mask"] = np.packbits(bits, axis=2, bitorder="little").view(np.int32)
    clean = call(x, kernel=kernel)
    attn_check(x, clean)
    x["dk"][:, pad] = fill
    x["dv"][:, pad] = fill
    assert torch.equal(call(x, kernel=kernel), clean)


@pytest.mark.parametrize("name", ["tiny", "llama7b", "llama13b"])
@pytest.mark.parametrize("page", [16, 128])
def test_named_configurations_against_the_oracle(name, page):
    # generated graphs, the padded cache's rows dealt out over pages
    import gsd_inputs as gi
    import oracle
    import paper_2407_16207_b200 as gsd
    from gpu_util import attn_tensors as padded_tensors, out_to_f64
    cfg = gi.CONFIGS[name]
    inp = gi.make_inputs(cfg, accept=False, pad_fill="nan")
    t = padded_tensors(inp)
    B, Lmax, Hkv, D = t["k_cache"].shape
    M = -(-Lmax // page)
    table = torch.randperm(B * M, generator=torch.Generator().manual_seed(3)).to(torch.int32).view(B, M).cuda()
    pools = []
    for n in ("k_cache", "v_cache"):
        rows = torch.full((B, M * page, Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        rows[:, :Lmax] = t[n]
        pool = torch.empty((B * M, page, Hkv, D), dtype=torch.bfloat16, device="cuda")
        pool[table.long().flatten()] = rows.view(B * M, page, Hkv, D)
        pools.append(pool)
    out = gsd.gsd_verify_attn_paged(t["q"], *pools, table, t["draft_k"], t["draft_v"], t["ancestor_mask"], t["seq_lens"])
    want = oracle.attn(inp["q"], inp["k_cache"], inp["v_cache"], inp["draft_k"], inp["draft_v"], inp["ancestor_mask"], inp["seq_lens"])
    err = np.abs(out_to_f64(out) - want)
    assert err.max() <= 1e-2 and err.mean() <= 1e-3
