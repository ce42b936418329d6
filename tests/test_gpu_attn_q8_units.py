"""gsd_verify_attn_q8 where the values of a call lie far apart, against a 64-bit evaluation.

Tolerance of an element: as in test_gpu_attn_q8 (the output's rounding, 2^-8 of it; the weights' rounding, 2^-8 of sum p |v|;
2^-15 S + 2^-20 of that for the scores' errors and the sums), with what the fp16 weights of the few-row kernel lose as
include/gsd.h states it: a weight times the scale of its V is off by at most 2^-33 of the row's largest such product, which is
at most their sum.  Over L keys with codes of up to QMAX: L 2^-33 QMAX sum_j p_j 2^e_j."""
import numpy as np
import pytest
import torch

import kv8_ref
from test_gpu_attn_q8 import call, make, want

pytestmark = pytest.mark.gpu


def check(x, got, scale=None):
    ref, spread, size, _ = want(x, scale)
    floor = np.zeros(ref.shape)
    for b in range(x["B"]):
        L = int(x["lens"][b])
        if L == 0:
            continue
        blk = np.arange(L) // x["block"]
        unit = np.broadcast_to(np.exp2(x["ve"][b][blk].astype(float))[:, :, None], (L, x["Hkv"], x["D"]))
        key = np.ldexp(kv8_ref.values(x["k"][b, :L], x["fmt"]), x["ke"][b][blk][:, :, None].astype(int))
        dk = x["dk"][b].double().numpy()
        total, _, _ = kv8_ref.attention(x["q"][b].double().numpy(), key, unit, L, dk, np.zeros(dk.shape), x["see"][b],
                                        scale or x["D"] ** -0.5)
        floor[b] = L * 2.0 ** -33 * kv8_ref.QMAX[x["fmt"]] * total
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
