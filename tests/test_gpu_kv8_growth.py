"""gsd_commit_kv_q8 and gsd_append_kv_q8 where few new rows make the exponents of blocks grow that hold many earlier rows, bit for
bit; margins of every row that is not the call's stay as they were."""
import numpy as np
import pytest
import torch

from test_gpu_kv8_write import fresh, on_gpu, rows_like, same
import kv8_ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("block", [16, 128])
@pytest.mark.parametrize("T", [1, 5, 40])
def test_few_rows_into_blocks_that_hold_many(fmt, D, block, T):
    import paper_2407_16207_b200 as gsd
    rng = np.random.default_rng([7, D, block, T])
    lens = [1, 2, 15, 31, 32, 33, 63, 65, 100, 127, 129, 255]
    B, H, Lmax = len(lens), 3, 300
    c, e = fresh(rng, B, Lmax, H, D, fmt, block, lens)
    k, v = rows_like(rng, B, T, H, D), rows_like(rng, B, T, H, D)
    # a head that grows by much, one by a little, one by none
    up = torch.tensor([2.0 ** 9, 8.0, 2.0 ** -9])[:, None]
    k, v = (k.float() * up).to(torch.bfloat16), (v.float() * up.flip(0)).to(torch.bfloat16)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    for commit in (True, False):
        cc, ee = c.copy(), e.copy()
        t, sl, n = on_gpu(cc, ee, fmt), i32(lens), i32([T] * B)
        if commit:
            gsd.gsd_commit_kv_q8(*t, k.cuda(), v.cuda(), i32([list(range(T))] * B), n, sl, block=block)
        else:
            gsd.gsd_append_kv_q8(*t, k.cuda(), v.cuda(), n, sl, block=block)
        for b in range(B):
            for kv, x in enumerate((k, v)):
                kv8_ref.append(cc[kv, b], ee[kv, b], x[b].double().numpy(), lens[b], fmt, block)
        assert sl.tolist() == [min(l + T, Lmax) for l in lens]
        same(t, cc, ee)
