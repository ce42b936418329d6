"""What the calls around the 8-bit cache and the log probabilities refuse, before anything touches a device."""
import ctypes

import pytest
import torch

import paper_2407_16207_b200 as gsd
from paper_2407_16207_b200.binding import AppendParams, AttnParams, CommitParams, Kv8Params, LogprobsParams

ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)
P = ctypes.byref


def attn(p, c, ptrs=None, ws=ONE, ws_bytes=1 << 40):
    return gsd.lib().gsd_verify_attn_q8(*(ptrs or [ONE] * 10), P(p) if p else None, P(c) if c else None, ws, ws_bytes, None, None)


def test_attention():
    good, c = AttnParams(1, 16, 4, 4, 64, 128, 0.0, 0, 0), Kv8Params(0, 64)
    assert attn(None, c) == -1 and attn(good, None) == -1
    for i in range(10):
        ptrs = [ONE] * 10
        ptrs[i] = None
        assert attn(good, c, ptrs) == -1, i
    for i in (0, 1, 2, 5, 6, 9):                     # q, codes, draft rows, out: 16 bytes
        ptrs = [ONE] * 10
        ptrs[i] = ODD
        assert attn(good, c, ptrs) == -3, i
    for i in (7, 8):                                 # mask words, lengths: 4 bytes
        ptrs = [ONE] * 10
        ptrs[i] = ctypes.c_void_p(258)
        assert attn(good, c, ptrs) == -3, i
    for bad in ((0, 48), (0, 8), (0, 256), (2, 64), (-1, 64)):
        assert attn(good, Kv8Params(*bad)) == -2, bad
        assert gsd.lib().gsd_verify_attn_q8_workspace_bytes(P(good), P(Kv8Params(*bad))) == 0
    for bad in ((0, 16, 4, 4, 64, 128), (1, 513, 4, 4, 64, 128), (1, 16, 4, 3, 64, 128), (1, 16, 4, 4, 96, 128), (1, 16, 4, 4, 64, 0)):
        assert attn(AttnParams(*bad, 0.0, 0, 0), c) == -2, bad
    assert attn(AttnParams(1, 16, 4, 4, 64, 128, 0.0, 65, 0), c) == -2
    assert attn(AttnParams(1, 16, 4, 4, 64, 128, 0.0, -3, 0), c) == -2
    assert attn(AttnParams(1, 16, 4, 4, 64, 128, 0.0, 0, 2), c) == -6      # the tcgen05 kernel by name: D = 128 only


def test_writers():
    L, c = gsd.lib(), Kv8Params(1, 16)
    good, ok = CommitParams(2, 8, 2, 64, 100, 8), AppendParams(2, 8, 2, 64, 100)
    for call, n, p in ((L.gsd_commit_kv_q8, 9, good), (L.gsd_append_kv_q8, 8, ok)):
        assert call(*[ONE] * n, None, P(c), None, None) == -1
        assert call(*[ONE] * n, P(p), None, None, None) == -1
        for i in range(n):
            ptrs = [ONE] * n
            ptrs[i] = None
            assert call(*ptrs, P(p), P(c), None, None) == -1, i
        for i in (0, 1, 4, 5):
            ptrs = [ONE] * n
            ptrs[i] = ODD
            assert call(*ptrs, P(p), P(c), None, None) == -3, i
        assert call(*[ONE] * n, P(p), P(Kv8Params(1, 20)), None, None) == -2
        assert call(*[ONE] * n, P(p), P(Kv8Params(7, 16)), None, None) == -2
    for bad in ((0, 8, 2, 64, 100, 8), (2, 513, 2, 64, 100, 8), (2, 8, 0, 64, 100, 8), (2, 8, 2, 72, 100, 8), (2, 8, 2, 64, 0, 8), (2, 8, 2, 64, 100, 0), (65536, 8, 2, 64, 100, 8)):
        assert L.gsd_commit_kv_q8(*[ONE] * 9, P(CommitParams(*bad)), P(c), None, None) == -2, bad
    for bad in ((0, 8, 2, 64, 100), (65536, 8, 2, 64, 100), (2, 0, 2, 64, 100), (2, 8, 0, 64, 100), (2, 8, 2, 72, 100), (2, 8, 2, 64, 0), (2, 1 << 30, 65535, 64, 100)):
        assert L.gsd_append_kv_q8(*[ONE] * 8, P(AppendParams(*bad)), P(c), None, None) == -2, bad


def test_logprobs():
    L = gsd.lib()
    call = lambda p, ptrs=None, ws=ONE, n=1 << 40: L.gsd_token_logprobs(*(ptrs or [ONE] * 8), P(p) if p else None, ws, n, None, None)
    good = LogprobsParams(2, 8, 100, 4, 5)
    assert call(None) == -1
    for i in (0, 1, 2, 3, 4, 6, 7):                  # (the entropy may be left out)
        ptrs = [ONE] * 8
        ptrs[i] = None
        assert call(good, ptrs) == -1, i
    assert call(good, [ctypes.c_void_p(258)] + [ONE] * 7) == -3
    for bad in ((0, 8, 100, 4, 5), (65536, 8, 100, 4, 5), (2, 0, 100, 4, 5), (2, 513, 100, 4, 5), (2, 8, 0, 4, 0), (2, 8, 100, 0, 5), (2, 8, 100, 513, 5), (2, 8, 100, 4, 33), (2, 8, 100, 4, -1), (2, 8, 4, 4, 5)):
        assert call(LogprobsParams(*bad)) == -2, bad
        assert L.gsd_token_logprobs_workspace_bytes(P(LogprobsParams(*bad))) == 0


def i32(*s):
    return torch.zeros(s, dtype=torch.int32)


def test_the_binding_refuses_what_it_cannot_hand_on():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    kv, ex = torch.zeros((1, 40, 2, 64), dtype=torch.int8), torch.zeros((1, 3, 2), dtype=torch.int8)
    a = dict(q=bf(1, 3, 4, 64), k_cache=kv, v_cache=kv, k_exp=ex, v_exp=ex, draft_k=bf(1, 3, 2, 64), draft_v=bf(1, 3, 2, 64),
             ancestor_mask=i32(1, 3, 1), seq_lens=i32(1))
    with pytest.raises(ValueError, match="k_cache: expected a CUDA tensor"):
        gsd.gsd_verify_attn_q8(**a, block=16)
    with pytest.raises(ValueError, match="block must be"):
        gsd.gsd_verify_attn_q8(**a, block=20)
    with pytest.raises(ValueError, match="k_cache: expected torch.float8_e4m3fn or torch.int8"):
        gsd.gsd_verify_attn_q8(**{**a, "k_cache": bf(1, 40, 2, 64)}, block=16)
    with pytest.raises(TypeError):
        gsd.gsd_verify_attn_q8(**a)
    with pytest.raises(ValueError, match="k_cache"):
        gsd.gsd_commit_kv_q8(kv, kv, ex, ex, bf(1, 3, 2, 64), bf(1, 3, 2, 64), i32(1, 3), i32(1), i32(1), block=16)
    with pytest.raises(ValueError, match="k_cache"):
        gsd.gsd_append_kv_q8(kv, kv, ex, ex, bf(1, 3, 2, 64), bf(1, 3, 2, 64), i32(1), i32(1), block=16)
    with pytest.raises(ValueError, match="logits: expected a CUDA tensor"):
        gsd.gsd_token_logprobs(torch.zeros(1, 3, 10), i32(1, 2), i32(1, 2), i32(1))
    with pytest.raises(ValueError, match="logits: expected contiguous torch.float32"):
        gsd.gsd_token_logprobs(torch.zeros(1, 3, 10).double(), i32(1, 2), i32(1, 2), i32(1))


@pytest.mark.gpu
def test_the_binding_refuses_mixed_shapes_types_and_strides():
    kv, ex = torch.zeros((1, 40, 2, 64), dtype=torch.int8, device="cuda"), torch.zeros((1, 3, 2), dtype=torch.int8, device="cuda")
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    c32 = lambda *s: i32(*s).cuda()
    a = dict(q=bf(1, 3, 4, 64), k_cache=kv, v_cache=kv, k_exp=ex, v_exp=ex, draft_k=bf(1, 3, 2, 64), draft_v=bf(1, 3, 2, 64),
             ancestor_mask=c32(1, 3, 1), seq_lens=c32(1))
    gsd.gsd_verify_attn_q8(**a, block=16)
    for change, name in ((dict(v_cache=kv.view(torch.float8_e4m3fn)), "v_cache"), (dict(k_exp=ex[:, :2].contiguous()), "k_exp"),
                         (dict(v_exp=ex.int()), "v_exp"), (dict(draft_k=bf(1, 3, 2, 128)[..., ::2]), "draft_k"),
                         (dict(seq_lens=c32(2)), "seq_lens"), (dict(ancestor_mask=c32(1, 3, 2)), "ancestor_mask"),
                         (dict(q=bf(1, 3, 4, 64).float()), "q"), (dict(draft_v=bf(1, 3, 2, 64).cpu()), "draft_v")):
        with pytest.raises(ValueError, match=name):
            gsd.gsd_verify_attn_q8(**{**a, **change}, block=16)
    with pytest.raises(gsd.GsdError):
        gsd.gsd_verify_attn_q8(**a, block=16, num_splits=65)
    with pytest.raises(gsd.GsdError):
        gsd.gsd_verify_attn_q8(**a, block=16, num_splits=4, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(gsd.GsdError):
        gsd.gsd_token_logprobs(torch.zeros((1, 3, 10), device="cuda"), c32(1, 2), c32(1, 2), c32(1), k=11)
    with pytest.raises(gsd.GsdError):
        gsd.gsd_token_logprobs(torch.zeros((1, 3, 10), device="cuda"), c32(1, 2), c32(1, 2), c32(1), k=2, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="accepted_nodes"):
        gsd.gsd_commit_kv_q8(kv, kv, ex, ex, a["draft_k"], a["draft_v"], c32(2, 3), c32(1), c32(1), block=16)
    with pytest.raises(ValueError, match="counts"):
        gsd.gsd_append_kv_q8(kv, kv, ex, ex, a["draft_k"], a["draft_v"], c32(2), c32(1), block=16)
