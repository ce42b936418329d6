"""gsd_verify_attn_q8 where the values of a call lie far apart, against a 64-bit evaluation.

Tolerance of an element: as in test_gpu_attn_q8 (the output's rounding, 2^-8 of it; the weights' rounding, 2^-8 of sum p |v|;
2^-15 S + 2^-20 of that for the scores' errors and the sums), and what the few-row kernel's weights in fp16 lose.  A warp has them
while the scales 2^e of V that it has met lie within 2^12, as p 2^(8 + e - top), top the largest e so far, p relative to
the largest so far or a larger one: the smallest are off by half of 2^-24, 2^(-33 + top - e) <= 2^-21 of the largest p of
a key whose scale lies within 2^12 of the key's own.  Over the keys: sum_j 2^-21 max_(|e_i - e_j| <= 12) p_i |v_j|."""
import numpy as np
import pytest
import torch

import kv8_ref
from test_gpu_attn_q8 import bf16, call, make, tensors, want

pytestmark = pytest.mark.gpu


def lost_in_fp16(x, b, scale):
    """The last term for sequence b: [N, Hq, D]."""
    L, G = int(x["lens"][b]), x["Hq"] // x["Hkv"]
    out = np.zeros((x["N"], x["Hq"], x["D"]))
    if L == 0:
        return out
    blk = np.arange(L) // x["block"]
    val = lambda n: np.ldexp(kv8_ref.values(x[n][b, :L], x["fmt"]), x[n + "e"][b][blk][:, :, None].astype(int))
    k, v = val("k"), np.abs(val("v"))
    q, dk = x["q"][b].double().numpy(), x["dk"][b].double().numpy()
    for h in range(x["Hq"]):
        c = h // G
        s = q[:, h] @ np.concatenate((k[:, c], dk[:, c])).T * scale
        s[:, L:][~x["see"][b]] = -np.inf
        p = np.exp(s - s.max(1, keepdims=True))
        p = (p / p.sum(1, keepdims=True))[:, :L]
        e = x["ve"][b][blk, c].astype(int)
        for one in np.unique(e):
            out[:, h] += 2.0 ** -21 * p[:, np.abs(e - one) <= 12].max(1)[:, None] * v[e == one, c].sum(0)
    return out


def check(x, got, scale=None):
    scale = scale or x["D"] ** -0.5
    ref, spread, size, _ = want(x, scale)
    floor = np.stack([lost_in_fp16(x, b, scale) for b in range(x["B"])])
    err = np.abs(got.double().cpu().numpy() - ref)
    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -20 + 2.0 ** -15 * size) * spread + floor
    assert np.isfinite(err).all()
    assert (err <= tol).all(), (float((err - tol).max()), np.unravel_index(np.argmax(err - tol), err.shape))


@pytest.mark.parametrize("splits", [0, 1, 3])
@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("N,Hq,Hkv", [(1, 8, 1), (70, 4, 2), (200, 2, 2)])
def test_large_draft_values(N, Hq, Hkv, kernel, splits):
    # warps without a prefix tile, all of them or some; nodes whose draft rows are small beside nodes with large ones
    for L, up in ((0, 16), (0, 100), (5, 20), (40, 24), (40, 100), (100, 60), (600, 30)):
        x = make(21, 2, N, Hq, Hkv, 128, 640, [L, 17], "int8" if L & 1 else "e4m3", 32, mask="chain" if N == 1 else "random")
        dv = x["dv"].double()
        dv[:, ::2] *= 2.0 ** up
        x["dv"] = dv.to(torch.bfloat16)
        check(x, call(x, kernel=kernel, num_splits=splits))


@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_large_draft_values_behind_a_prefix_of_zeros(fmt, kernel):
    # the writers give blocks of zeros the least exponent
    for N in (9, 200):
        x = make(22, 2, N, 4, 2, 128, 320, [320, 130], fmt, 64)
        x["v"][0], x["ve"][0] = 0, -117
        x["v"][1, :64], x["ve"][1, 0] = 0, -117
        x["dv"] = (x["dv"].double() * 2.0 ** 30).to(torch.bfloat16)
        check(x, call(x, kernel=kernel))


def constant(value, fmt, e):
    """The code nearest to value at exponent e."""
    return kv8_ref.to_codes(np.asarray(value * 2.0 ** -e), fmt)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("gap", [20, 28, 33, 60, 110])
def test_a_large_scale_that_no_row_looks_at(gap, kernel, fmt):
    # a block of keys that point away from every query, with values 2^gap above the others': first, in the middle, last
    for N, Hq, Hkv, at in ((1, 8, 1, 0), (1, 8, 1, 9), (12, 4, 1, 4), (7, 14, 2, 19), (7, 16, 2, 19), (40, 4, 2, 7)):
        if kernel == 2 and 128 % (Hq // Hkv):
            continue
        x = make(23, 2, N, Hq, Hkv, 128, 320, [320, 315], fmt, 16, spread=1)
        x["q"] = bf16(x["q"].float().numpy() * 0.3 + 2.0)
        x["k"][:, at * 16:at * 16 + 16] = constant(-40.0, fmt, 0)
        x["ke"][:, at] = 0
        x["ve"][:, at] += gap
        for splits in (0, 1, 3):
            check(x, call(x, kernel=kernel, num_splits=splits))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("gap", [12, 24, 40, 80])
def test_small_weights_of_large_values(gap, kernel, fmt):
    # weights of about 2^-gap of values 2^gap above the others': both count.  Half of the rows do not look at them.
    e = {12: 0, 24: 1, 40: 2, 80: 3}[gap] - (8 if fmt == "int8" else 7)
    for N, Hq, Hkv, at in ((1, 8, 1, 3), (12, 4, 1, 11), (40, 4, 2, 0)):
        x = make(24, 1, N, Hq, Hkv, 128, 256, [256], fmt, 16, spread=1)
        x["q"] = bf16(x["q"].float().numpy() * 0.01 + np.where(np.arange(Hq) % 2, 2.0, 1.0)[:, None])
        x["k"][:] = 0
        x["k"][:, at * 16:at * 16 + 16] = constant(-gap * np.log(2.0) / (2.0 * 128 ** 0.5), fmt, e)
        x["ke"][:, at] = e
        x["ve"][:, at] += gap
        check(x, call(x, kernel=kernel))


@pytest.mark.parametrize("T", [90, 300])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_an_infinity_in_the_cache_blanks_nothing_but_its_block(fmt, T):
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng(25)
    H, D, block = 2, 128, 16
    k, v = (bf16(rng.standard_normal((1, T, H, D))) for _ in range(2))
    k[0, 20] = -40.0
    v[0, 20, 1, 5] = float("inf")
    x = make(26, 1, 3, 8, H, D, T, [T], fmt, block)
    x["q"] = bf16(x["q"].float().numpy() * 0.3 + 2.0)
    t = tensors(x)
    t["seq_lens"].zero_()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    gsd.gsd_append_kv_q8(t["k_cache"], t["v_cache"], t["k_exp"], t["v_exp"], k.cuda(), v.cuda(),
                         torch.tensor([T], dtype=torch.int32, device="cuda"), t["seq_lens"], block=block, status=status)
    outs = [gsd.gsd_verify_attn_q8(**t, block=block, kernel=kernel) for kernel in (1, 2)]
    assert int(status.item()) == 0x800
    for n in "kv":
        x[n] = t[n + "_cache"].view(torch.int8).cpu().numpy().view(np.uint8)
        x[n + "e"] = t[n + "_exp"].cpu().numpy()
    assert x["ve"][0, 1, 1] == 119
    for got in outs:
        check(x, got)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [128, 64])
def test_scores_beyond_any_rounding(D, fmt):
    # few rows: the key that points with the query has the weight 1 exactly, whatever the size of its score, and what is
    # not rounded stays: its value
    for up in (10, 13, 14, 15, 16, 17, 18, 20, 26, 30, 40, 60):
        x = make(27, 1, 1, 4, 2, D, 64, [34], fmt, 32, mask="none")
        x["q"] = bf16(np.abs(x["q"].float().numpy()) * 2.0 ** up + 2.0 ** up)
        x["k"][:] = constant(-33.0, fmt, 0)
        x["k"][0, 5, 0] = x["k"][0, 33, 1] = constant(29.0, fmt, 0)
        x["ke"][:] = 0
        x["ve"][:] = -3
        got = call(x, kernel=1).double().cpu().numpy()[0, 0]
        v = np.ldexp(kv8_ref.values(x["v"][0], fmt), -3)
        ref = np.stack([v[5, 0], v[5, 0], v[33, 1], v[33, 1]])
        assert np.array_equal(got, ref), up


@pytest.mark.parametrize("kernel", [0, 1, 2])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_chunks_of_a_prompt(fmt, kernel):
    # a chain of as many nodes as there can be, over an empty cache and behind earlier chunks
    for D, Hq, Hkv in ((128, 4, 2), (64, 2, 1)):
        if kernel == 2 and D == 64:
            continue
        for N, lens in ((512, [0, 513]), (511, [130, 1])):
            x = make(28, 2, N, Hq, Hkv, D, 520, lens, fmt, 64, mask="chain")
            check(x, call(x, kernel=kernel))
