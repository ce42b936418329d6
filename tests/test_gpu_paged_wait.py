"""The bounded waits of the attention kernels over pages: a wait that runs out must end the launch cleanly with
GSD_DEV_WAIT_EXPIRED, and the next call must work as if nothing had happened.  As in test_gpu_attn_wait, the copy of a first key
tile is announced and not issued, and the limit is a few milliseconds; nothing else is broken."""
import pytest
import torch

from paged_ref import attn_check, attn_inputs, attn_tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,N,Hq,Hkv,D,lens,kernel", [(2, 3, 8, 2, 128, [700, 90], 1), (1, 20, 4, 4, 64, [0], 1), (1, 64, 8, 8, 128, [2000], 2),
                                                      (3, 200, 8, 1, 128, [600, 300, 77], 2), (2, 100, 4, 1, 64, [500, 40], 0)])
def test_expired_waits_are_reported_and_the_next_call_is_clean(B, N, Hq, Hkv, D, lens, kernel):
    import paper_2407_16207_b200 as gsd
    x = attn_inputs(21, B, N, Hq, Hkv, D, lens, 16)
    t = attn_tensors(x)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    gsd.gsd_debug_attn_wait(3_000_000, True)          # 3 ms instead of 2 s; first K tiles withheld
    try:
        gsd.gsd_verify_attn_paged(**t, kernel=kernel, status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0x8
    finally:
        gsd.gsd_debug_attn_wait(0, False)
    status.zero_()
    out = gsd.gsd_verify_attn_paged(**t, kernel=kernel, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    attn_check(x, out)
