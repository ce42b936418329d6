"""gsd_verify_attn_q8 against a 64-bit evaluation of its definition.

Tolerance of an element: the output's rounding, 2^-8 of it; the weights' rounding to bf16, 2^-8 of sum p |v|; and what the
scores' errors do to the weights.  A score is an fp32 sum of D <= 128 products: off by at most 128 * 2^-23 of S = scale *
sum |q k|, i.e. 2^-16 S, which moves a weight by that much of itself and the sum it is divided by likewise: 2^-15 S, and
2^-20 for the exponential and the sums.  Over the codes weights are held in fp16 in units
of 2^-8 and of the largest scale 2^e of the head's V: the smallest ones are off by half of 2^-24 of the unit, 2^-33 2^e, and
there are L of them."""
import numpy as np
import pytest
import torch

import kv8_ref

pytestmark = pytest.mark.gpu
DT = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)


def make(seed, B, N, Hq, Hkv, D, rows, lens, fmt, block, mask="random", spread=3):
    """Numpy inputs: codes over all their values, exponents that differ by `spread`, rows past the end that would show."""
    rng = np.random.default_rng(seed)
    nb = -(-rows // block)
    codes = {}
    for n in "kv":
        c = kv8_ref.to_codes(rng.standard_normal((B, rows, Hkv, D)) * (40.0 if fmt == "int8" else 12.0), fmt)
        e = rng.integers(-spread - 5, -4, (B, nb, Hkv)).astype(np.int8) - (0 if fmt == "e4m3" else 2)
        for b in range(B):                      # what lies behind the end must never be looked at
            c[b, lens[b]:] = 0x7F
            e[b, -(-lens[b] // block):] = 127
        codes[n] = c, e
    x = dict(B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, rows=rows, lens=np.asarray(lens, np.int32), fmt=fmt, block=block,
             k=codes["k"][0], ke=codes["k"][1], v=codes["v"][0], ve=codes["v"][1],
             q=bf16(rng.standard_normal((B, N, Hq, D))), dk=bf16(rng.standard_normal((B, N, Hkv, D))),
             dv=bf16(rng.standard_normal((B, N, Hkv, D))))
    if mask == "none":
        see = np.zeros((B, N, N), bool)
    elif mask == "chain":
        see = np.broadcast_to(np.tril(np.ones((N, N), bool)), (B, N, N)).copy()
    else:
        see = rng.random((B, N, N)) < min(0.5, 12.0 / N)
        see[:, min(1, N - 1)] = False           # a node that sees no draft row
        see[:, range(0, N, 2), range(0, N, 2)] = True
    x["see"] = see
    W = (N + 31) // 32
    bits = np.zeros((B, N, W * 32), bool)
    bits[:, :, :N] = see
    if N % 32:
        bits[:, 0, N:] = True                   # bits at or past N are ignored
    x["mask"] = np.packbits(bits, axis=2, bitorder="little").view(np.int32)
    return x


def tensors(x):
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    code = lambda a: cuda(a.view(np.int8)).view(DT[x["fmt"]])
    return dict(q=x["q"].cuda(), k_cache=code(x["k"]), v_cache=code(x["v"]), k_exp=cuda(x["ke"]), v_exp=cuda(x["ve"]),
                draft_k=x["dk"].cuda(), draft_v=x["dv"].cuda(), ancestor_mask=cuda(x["mask"]), seq_lens=cuda(x["lens"]))


def want(x, scale=None):
    f = lambda t: t.double().numpy()
    out, spread, size, floor = [], [], [], []
    for b in range(x["B"]):
        L = int(x["lens"][b])
        blk = np.arange(L) // x["block"]
        val = lambda c, e: np.ldexp(kv8_ref.values(c[b, :L], x["fmt"]), e[b][blk][:, :, None].astype(int))
        o, a, s = kv8_ref.attention(f(x["q"][b]), val(x["k"], x["ke"]), val(x["v"], x["ve"]), L, f(x["dk"][b]), f(x["dv"][b]),
                                 x["see"][b], scale or x["D"] ** -0.5)
        out.append(o)
        spread.append(a)
        size.append(s)
        top = np.exp2(x["ve"][b][:-(-L // x["block"])].max(0, initial=-126).astype(float))              # [H]
        floor.append(np.repeat(L * 2.0 ** -33 * top * kv8_ref.QMAX[x["fmt"]], x["Hq"] // x["Hkv"])[None, :, None])
    return np.stack(out), np.stack(spread), np.stack(size), np.stack(floor)


def check(x, got, scale=None):
    ref, spread, size, floor = want(x, scale)
    err = np.abs(got.double().cpu().numpy() - ref)
    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -20 + 2.0 ** -15 * size) * spread + floor
    assert np.isfinite(err).all()
    assert (err <= tol).all(), (float((err - tol).max()), np.unravel_index(np.argmax(err - tol), err.shape))


def call(x, **kw):
    import paper_2407_16207_b200 as gsd
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = gsd.gsd_verify_attn_q8(**tensors(x), block=x["block"], status=status, **kw)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return out


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_single_tokens(fmt, D, block):
    # lengths around tiles and blocks, none and one among them
    lens = [0, 1, 15, 16, 17, 127, 128, 129, 300, 511]
    for Hq, Hkv in ((8, 1), (4, 4), (6, 2)):
        x = make(1, len(lens), 1, Hq, Hkv, D, 513, lens, fmt, block, mask="chain")
        check(x, call(x))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("N,Hq,Hkv", [(2, 8, 8), (9, 4, 2), (16, 3, 1), (33, 8, 2), (7, 28, 4), (64, 4, 4), (100, 6, 2), (130, 8, 1), (257, 2, 2)])
def test_draft_graphs(fmt, D, N, Hq, Hkv):
    x = make(2, 3, N, Hq, Hkv, D, 700, [699, 130, 5], fmt, 64)
    check(x, call(x))


@pytest.mark.parametrize("kernel", [0, 1, 2])
@pytest.mark.parametrize("splits", [0, 1, 2, 3, 7, 64])
def test_key_ranges(kernel, splits):
    for fmt, N, Hq, Hkv in (("e4m3", 5, 8, 2), ("int8", 40, 8, 1)):
        x = make(3, 2, N, Hq, Hkv, 128, 1100, [1100, 333], fmt, 32)
        check(x, call(x, num_splits=splits, kernel=kernel))


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("N,G", [(1, 17), (24, 1), (33, 1), (10, 4), (41, 1), (6, 8), (7, 7), (28, 2), (57, 1), (13, 5), (36, 2), (97, 1)])
def test_row_groups_of_few_rows(N, G, D, splits):
    x = make(11, 2, N, 2 * G, 2, D, 290, [289, 33], "int8" if N & 1 else "e4m3", 32)
    check(x, call(x, kernel=1, num_splits=splits))


@pytest.mark.parametrize("kernel", [1, 2])
def test_rows_that_see_nothing_are_zero(kernel):
    x = make(4, 2, 11, 8, 2, 128, 64, [0, 40], "e4m3", 16, mask="none")
    got = call(x, kernel=kernel)
    assert (got[0] == 0).all()
    check(x, got)


@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_exponents_far_apart(fmt, kernel):
    # blocks of zeros at the least exponent, blocks 2^12 larger than others, the largest block last and first
    for order in (1, -1):
        x = make(5, 2, 12, 4, 1, 128, 400, [400, 257], fmt, 16, spread=1)
        nb = x["ve"].shape[1]
        x["ve"][:, :, 0] = (np.arange(nb)[::order] * 12 // nb - 12).astype(np.int8)
        x["v"][:, 16:32] = 0
        x["ve"][:, 1] = -117
        x["k"][:, 48:64] = 0
        x["ke"][:, 3] = -117
        check(x, call(x, kernel=kernel))


@pytest.mark.parametrize("kernel", [1, 2])
def test_query_rows_of_any_size(kernel):
    # rows 2^40 apart, with a scale that brings their scores back; a row of zeros
    x = make(6, 1, 8, 4, 1, 128, 200, [200], "e4m3", 64)
    q = x["q"].float()
    q[:, 1] = 0
    q[:, 2] *= 2.0 ** -60
    x["q"] = q.to(torch.bfloat16)
    check(x, call(x, kernel=kernel))
    x["q"] = (x["q"].float() * 2.0 ** 20).to(torch.bfloat16)
    check(x, call(x, kernel=kernel, softmax_scale=128.0 ** -0.5 * 2.0 ** -20), 128.0 ** -0.5 * 2.0 ** -20)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_every_code(fmt):
    # one key a node: the output is that key's value, exactly
    import paper_2407_16207_b200 as gsd
    codes = np.array([c for c in range(256) if not (fmt == "e4m3" and c & 127 == 127)], np.uint8)
    for e in (-117, -20, 0, 7, 100):
        c = np.resize(codes, (1, 2, 1, 128))
        c[0, 1, 0] = np.resize(codes[128:], 128)
        t = torch.from_numpy(c.view(np.int8)).cuda()
        for b in range(2):
            kv = t[:, b:b + 1].contiguous().view(DT[fmt])
            ex = torch.full((1, 1, 1), e, dtype=torch.int8, device="cuda")
            zero = torch.zeros((1, 1, 1, 128), dtype=torch.bfloat16, device="cuda")
            i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
            for kernel in (1, 2):
                out = gsd.gsd_verify_attn_q8(zero, kv, kv, ex, ex, zero, zero, i32(0).view(1, 1, 1), i32(1), block=16, kernel=kernel)
                ref = np.ldexp(kv8_ref.values(c[0, b, 0], fmt), e)
                assert np.array_equal(out.double().cpu().numpy().ravel(), ref), (e, b, kernel)


def test_agrees_with_the_bf16_call():
    import paper_2407_16207_b200 as gsd
    x = make(7, 3, 64, 16, 4, 128, 900, [900, 64, 513], "int8", 32)
    t = tensors(x)
    blk = np.arange(900) // 32
    for b in range(3):
        x["k"][b, x["lens"][b]:] = 0
        x["v"][b, x["lens"][b]:] = 0
    val = lambda c, e: bf16(np.ldexp(kv8_ref.values(c, "int8"), np.minimum(e, 0)[:, blk][..., None].astype(int))).cuda()
    ref = gsd.gsd_verify_attn(t["q"], val(x["k"], x["ke"]), val(x["v"], x["ve"]), t["draft_k"], t["draft_v"], t["ancestor_mask"], t["seq_lens"])
    got = call(x)
    # both are within 2^-8 (weights) and 2^-8 (output) of the same values, which are below 8 here
    assert (got.float() - ref.float()).abs().max() <= 4 * 2.0 ** -8 * float(want(x)[1].max())


@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_draft_rows_that_nobody_sees_may_be_anything(kernel, bad):
    x = make(12, 2, 40, 4, 2, 128, 100, [100, 0], "e4m3", 64)
    x["see"][:, :, 5] = x["see"][:, :, 33] = x["see"][:, :, 39] = False
    bits = np.zeros((2, 40, 64), bool)
    bits[:, :, :40] = x["see"]
    x["mask"] = np.packbits(bits, axis=2, bitorder="little").view(np.int32)
    clean = {n: x[n].clone() for n in ("dk", "dv")}
    for n in ("dk", "dv"):
        x[n][:, [5, 33, 39]] = bad
    got = call(x, kernel=kernel)
    x.update(clean)
    check(x, got)


@pytest.mark.parametrize("kernel", [1, 2])
def test_draft_rows_of_any_size(kernel):
    x = make(13, 1, 70, 4, 2, 128, 150, [150], "int8", 32)
    for n in ("dk", "dv"):
        x[n][:, ::3] = (x[n][:, ::3].float() * 2.0 ** -9).to(torch.bfloat16)
    x["dv"][:, 1::7] = (x["dv"][:, 1::7].float() * 2.0 ** 12).to(torch.bfloat16)
    x["dk"][:, 40:] = 0
    check(x, call(x, kernel=kernel))


def test_lengths_out_of_range_are_clamped_and_flagged():
    import paper_2407_16207_b200 as gsd
    x = make(8, 2, 3, 4, 2, 128, 100, [100, 0], "e4m3", 64)
    t = tensors(x)
    t["seq_lens"] = torch.tensor([1000, -3], dtype=torch.int32, device="cuda")
    for kernel in (1, 2):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = gsd.gsd_verify_attn_q8(**t, block=64, status=status, kernel=kernel)
        assert int(status.item()) == 0x10
        check(x, out)


def test_repeated_and_captured_calls_are_identical_and_two_graphs_may_share_scratch():
    import paper_2407_16207_b200 as gsd
    xs = [make(9 + i, 2, 6, 8, 2, 128, 900, [900, 411], "int8", 64) for i in range(2)]
    ts = [tensors(x) for x in xs]
    need = gsd.gsd_verify_attn_q8_workspace_bytes(2, 6, 8, 2, 128, 900, block=64)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    plain = [gsd.gsd_verify_attn_q8(**t, block=64) for t in ts]
    outs = [torch.empty_like(o) for o in plain]
    graphs = []
    for t, o in zip(ts, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            gsd.gsd_verify_attn_q8(**t, out=o, block=64, workspace=ws)
        graphs.append(g)
    for r in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, plain):
            assert torch.equal(o, w)


def test_another_stream_and_unaligned_views():
    import paper_2407_16207_b200 as gsd
    x = make(11, 2, 5, 8, 2, 64, 130, [130, 77], "e4m3", 16)
    t = tensors(x)
    # exponents and mask that start on odd addresses
    pad = torch.zeros(1 + t["k_exp"].numel(), dtype=torch.int8, device="cuda")
    pad[1:] = t["k_exp"].flatten()
    t["k_exp"] = pad[1:].view(t["v_exp"].shape)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = gsd.gsd_verify_attn_q8(**t, block=16)
    s.synchronize()
    check(x, out)


def test_an_offset_past_32_bits():
    # the last sequence's rows lie more than 2^32 bytes into the cache
    import paper_2407_16207_b200 as gsd
    B, rows, H, D = 3, 1 << 18, 64, 128
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 26 GB")
    rng = torch.Generator(device="cuda").manual_seed(3)
    L = 100
    k = torch.zeros((B, rows, H, D), dtype=torch.int8, device="cuda")
    v = torch.zeros((B, rows, H, D), dtype=torch.int8, device="cuda")
    k[2, rows - L:] = torch.randint(-40, 40, (L, H, D), generator=rng, device="cuda", dtype=torch.int8)
    v[2, rows - L:] = torch.randint(-120, 120, (L, H, D), generator=rng, device="cuda", dtype=torch.int8)
    e = torch.full((B, rows // 128, H), -6, dtype=torch.int8, device="cuda")
    q = torch.randn((B, 1, H, D), generator=rng, device="cuda").to(torch.bfloat16)
    zero = torch.zeros((B, 1, H, D), dtype=torch.bfloat16, device="cuda")
    mask = torch.zeros((B, 1, 1), dtype=torch.int32, device="cuda")
    lens = torch.tensor([0, 0, rows], dtype=torch.int32, device="cuda")
    for kernel in (1, 2):
        out = gsd.gsd_verify_attn_q8(q, k, v, e, e, zero, zero, mask, lens, block=128, kernel=kernel)
        s = torch.einsum("hd,khd->hk", q[2, 0].double(), k[2, rows - L:].double() * 2.0 ** -6) * D ** -0.5
        p = torch.cat((s, torch.full((H, 1), float(np.log(rows - L)), device="cuda", dtype=torch.float64)), 1).softmax(1)[:, :L]
        V = v[2, rows - L:].double() * 2.0 ** -6
        ref, spread = torch.einsum("hk,khd->hd", p, V), torch.einsum("hk,khd->hd", p, V.abs())
        # (2^18 weights of keys with score 0 add up: 2^-24 of the sum for each addition of a lane's 2^11)
        assert ((out[2, 0].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -10) * spread).all()
        assert (out[:2] == 0).all()
