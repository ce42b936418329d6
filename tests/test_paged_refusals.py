"""What the calls around the paged cache and the rotary positions refuse, before anything touches a device."""
import ctypes

import pytest
import torch

import paper_2407_16207_b200 as gsd
from paper_2407_16207_b200.binding import AppendPagedParams, AttnParams, CommitParams, PageParams, RotaryParams, Rotation

ONE, ODD, HALF = ctypes.c_void_p(256), ctypes.c_void_p(264), ctypes.c_void_p(258)
P = ctypes.byref
BAD_PAGES = ((8, 4, 4), (24, 4, 4), (512, 4, 4), (0, 4, 4), (-16, 4, 4), (16, 0, 4), (16, -1, 4), (16, 4, 0), (16, 4, -3))


def axis(*a):
    return (ctypes.c_uint8 * 64)(*a)


def attn(p, c, ptrs=None, ws=ONE, ws_bytes=1 << 40):
    return gsd.lib().gsd_verify_attn_paged(*(ptrs or [ONE] * 9), P(p) if p else None, P(c) if c else None, ws, ws_bytes, None, None)


def test_attention():
    good, c = AttnParams(1, 16, 4, 4, 64, 128, 0.0, 0, 0), PageParams(64, 9, 2)
    assert attn(None, c) == -1 and attn(good, None) == -1
    for i in range(9):
        ptrs = [ONE] * 9
        ptrs[i] = None
        assert attn(good, c, ptrs) == -1, i
    for i in (0, 1, 2, 4, 5, 8):                     # q, pages, draft rows, out: 16 bytes
        ptrs = [ONE] * 9
        ptrs[i] = ODD
        assert attn(good, c, ptrs) == -3, i
    for i in (3, 6, 7):                              # table, mask words, lengths: 4 bytes
        ptrs = [ONE] * 9
        ptrs[i] = HALF
        assert attn(good, c, ptrs) == -3, i
    for bad in BAD_PAGES + ((64, 9, 1),):            # (the last: no room for 128 rows in one page)
        assert attn(good, PageParams(*bad)) == -2, bad
        assert gsd.lib().gsd_verify_attn_paged_workspace_bytes(P(good), P(PageParams(*bad))) == 0
    assert attn(AttnParams(1, 16, 4, 4, 64, (1 << 30) + 1, 0.0, 0, 0), PageParams(256, 9, 1 << 23)) == -2
    for bad in ((0, 16, 4, 4, 64, 128), (1, 513, 4, 4, 64, 128), (1, 16, 4, 3, 64, 128), (1, 16, 4, 4, 96, 128), (1, 16, 4, 4, 64, 0)):
        assert attn(AttnParams(*bad, 0.0, 0, 0), c) == -2, bad
    assert attn(AttnParams(1, 16, 4, 4, 64, 128, 0.0, 65, 0), c) == -2
    assert attn(AttnParams(1, 16, 4, 4, 64, 128, 0.0, -3, 0), c) == -2
    assert attn(AttnParams(1, 16, 4, 4, 64, 128, 0.0, 0, 2), c) == -6      # the tcgen05 kernel by name: D = 128 only
    assert attn(AttnParams(1, 16, 12, 4, 128, 128, 0.0, 0, 2), c) == -6    # and groups that divide 128


def test_commit():
    L, good, c = gsd.lib(), CommitParams(2, 8, 2, 64, 100, 8), PageParams(16, 20, 7)
    call = lambda p, c, ptrs=None: L.gsd_commit_kv_paged(*(ptrs or [ONE] * 8), P(p) if p else None, P(c) if c else None, None, None)
    assert call(None, c) == -1 and call(good, None) == -1
    for i in range(8):
        ptrs = [ONE] * 8
        ptrs[i] = None
        assert call(good, c, ptrs) == -1, i
    for i, p in [(i, ODD) for i in (0, 1, 3, 4)] + [(i, HALF) for i in (2, 5, 6, 7)]:
        ptrs = [ONE] * 8
        ptrs[i] = p
        assert call(good, c, ptrs) == -3, i
    for bad in BAD_PAGES + ((16, 20, 6),):
        assert call(good, PageParams(*bad)) == -2, bad
    for bad in ((0, 8, 2, 64, 100, 8), (2, 513, 2, 64, 100, 8), (2, 8, 0, 64, 100, 8), (2, 8, 2, 72, 100, 8), (2, 8, 2, 64, 0, 8),
                (2, 8, 2, 64, 100, 0), (65536, 8, 2, 64, 100, 8)):
        assert call(CommitParams(*bad), c) == -2, bad


BAD_ROTATIONS = [Rotation(*r) for r in ((0, 0, 1, axis()), (4, 0, 1, axis()), (12, 0, 1, axis()), (40, 0, 1, axis()), (16, 2, 1, axis()),
                                        (16, -1, 1, axis()), (16, 0, 0, axis()), (16, 0, 5, axis()), (16, 0, 3, axis(0, 1, 2, 3)), (16, 1, 1, axis(0, 1)))]


def test_append():
    L, c, r = gsd.lib(), PageParams(16, 20, 7), Rotation(32, 0, 3, axis(0, 1, 2))
    good = AppendPagedParams(2, 8, 2, 64, 100, 128, 512)

    def call(p, c, r, ptrs=None):
        return L.gsd_append_kv_paged(*(ptrs or [ONE] * 10), P(p) if p else None, P(c) if c else None, P(r) if r else None, None, None)
    assert call(None, c, r) == -1 and call(good, None, r) == -1
    assert call(good, c, None) == -1                 # freqs without a rotation
    for i in range(8):                               # (8, 9: positions and offsets may be left out)
        ptrs = [ONE] * 10
        ptrs[i] = None
        assert call(good, c, r, ptrs) == -1, i
    for i, p in [(i, ODD) for i in (0, 1, 3, 4)] + [(i, HALF) for i in (2, 5, 6, 7, 8, 9)]:
        ptrs = [ONE] * 10
        ptrs[i] = p
        assert call(good, c, r, ptrs) == -3, i
    for bad in BAD_PAGES + ((16, 20, 6),):
        assert call(good, PageParams(*bad), r) == -2, bad
    for bad in BAD_ROTATIONS:
        assert call(good, c, bad) == -2, (bad.pairs, bad.layout, bad.axes)
    for bad in ((0, 8, 2, 64, 100, 128, 128), (65536, 8, 2, 64, 100, 128, 128), (2, 0, 2, 64, 100, 128, 128), (2, 8, 0, 64, 100, 128, 128),
                (2, 8, 2, 72, 100, 144, 144), (2, 8, 2, 64, 0, 128, 128), (2, 1 << 30, 2, 64, 100, 128, 128),
                (2, 8, 2, 64, 100, 120, 128), (2, 8, 2, 64, 100, 128, 120)):
        assert call(AppendPagedParams(*bad), c, r) == -2, bad
    for bad in ((2, 8, 2, 64, 100, 132, 128), (2, 8, 2, 64, 100, 128, 130)):
        assert call(AppendPagedParams(*bad), c, r) == -3, bad


def test_rotary():
    L, good, r = gsd.lib(), RotaryParams(2, 8, 4, 2, 64, 256, 128), Rotation(32, 1, 1, axis())
    call = lambda p, r, ptrs=None: L.gsd_rotary(*(ptrs or [ONE] * 7), P(p) if p else None, P(r) if r else None, None)
    assert call(None, r) == -1 and call(good, None) == -1
    for i in (0, 1, 2, 3, 5, 6):                     # (k without its place and the other way round; offsets may be left out)
        ptrs = [ONE] * 7
        ptrs[i] = None
        assert call(good, r, ptrs) == -1, i
    for i, p in [(i, ODD) for i in (0, 1, 5, 6)] + [(i, HALF) for i in (2, 3, 4)]:
        ptrs = [ONE] * 7
        ptrs[i] = p
        assert call(good, r, ptrs) == -3, i
    for bad in BAD_ROTATIONS:
        assert call(good, bad) == -2, (bad.pairs, bad.layout, bad.axes)
    for bad in ((0, 8, 4, 2, 64, 256, 128), (2, 0, 4, 2, 64, 256, 128), (2, 8, 0, 2, 64, 256, 128), (2, 8, 4, 0, 64, 256, 128),
                (2, 8, 4, 2, 96, 512, 512), (2, 8, 4, 2, 64, 248, 128), (2, 8, 4, 2, 64, 256, 120), (1 << 16, 1 << 15, 4, 2, 64, 256, 128)):
        assert call(RotaryParams(*bad), r) == -2, bad
    assert call(RotaryParams(2, 8, 4, 2, 64, 260, 128), r) == -3 and call(RotaryParams(2, 8, 4, 2, 64, 256, 132), r) == -3


bf = lambda *s, dev="cpu": torch.zeros(s, dtype=torch.bfloat16, device=dev)
ints = lambda *s, dev="cpu": torch.zeros(s, dtype=torch.int32, device=dev)


def test_the_binding_refuses_what_it_cannot_hand_on():
    kv = bf(5, 16, 2, 64)
    a = dict(q=bf(1, 3, 4, 64), k_pages=kv, v_pages=kv, page_table=ints(1, 3), draft_k=bf(1, 3, 2, 64), draft_v=bf(1, 3, 2, 64),
             ancestor_mask=ints(1, 3, 1), seq_lens=ints(1))
    with pytest.raises(ValueError, match="k_pages: expected a CUDA tensor"):
        gsd.gsd_verify_attn_paged(**a)
    with pytest.raises(ValueError, match="pages must have"):
        gsd.gsd_verify_attn_paged(**{**a, "k_pages": bf(5, 20, 2, 64)})
    with pytest.raises(ValueError, match="page_table"):
        gsd.gsd_verify_attn_paged(**{**a, "page_table": ints(3)})
    with pytest.raises(ValueError, match="k_pages: expected a CUDA tensor"):
        gsd.gsd_commit_kv_paged(kv, kv, ints(1, 3), bf(1, 3, 2, 64), bf(1, 3, 2, 64), ints(1, 3), ints(1), ints(1))
    with pytest.raises(ValueError, match="k: expected a CUDA tensor"):
        gsd.gsd_append_kv_paged(kv, kv, ints(1, 3), bf(1, 3, 2, 64), bf(1, 3, 2, 64), ints(1), ints(1))
    with pytest.raises(ValueError, match="q: expected a CUDA tensor"):
        gsd.gsd_rotary(bf(1, 3, 4, 64), None, torch.zeros(32), ints(1, 1, 3))
    with pytest.raises(ValueError, match="q: expected bfloat16"):
        gsd.gsd_rotary(bf(1, 3, 4, 64).float(), None, torch.zeros(32), ints(1, 1, 3))


@pytest.mark.gpu
def test_the_binding_refuses_mixed_shapes_types_and_strides():
    d = dict(dev="cuda")
    kv = bf(5, 16, 2, 64, **d)
    a = dict(q=bf(1, 3, 4, 64, **d), k_pages=kv, v_pages=kv, page_table=ints(1, 3, **d), draft_k=bf(1, 3, 2, 64, **d),
             draft_v=bf(1, 3, 2, 64, **d), ancestor_mask=ints(1, 3, 1, **d), seq_lens=ints(1, **d))
    gsd.gsd_verify_attn_paged(**a)
    for change, name in ((dict(v_pages=kv[:4]), "v_pages"), (dict(page_table=ints(2, 3, **d)), "page_table"),
                         (dict(page_table=ints(1, 3, **d).long()), "page_table"), (dict(draft_k=bf(1, 3, 2, 128, **d)[..., ::2]), "draft_k"),
                         (dict(seq_lens=ints(2, **d)), "seq_lens"), (dict(ancestor_mask=ints(1, 3, 2, **d)), "ancestor_mask"),
                         (dict(q=bf(1, 3, 4, 64, **d).float()), "q"), (dict(draft_v=bf(1, 3, 2, 64)), "draft_v")):
        with pytest.raises(ValueError, match=name):
            gsd.gsd_verify_attn_paged(**{**a, **change})
    for kw in (dict(num_splits=65), dict(max_len=49), dict(max_len=-1), dict(num_splits=4, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(gsd.GsdError):
            gsd.gsd_verify_attn_paged(**a, **kw)
    w = dict(k_pages=kv, v_pages=kv, page_table=ints(1, 3, **d))
    k, f, n = bf(1, 3, 2, 64, **d), torch.zeros(32, device="cuda"), ints(1, **d)
    for change, name in ((dict(accepted_nodes=ints(2, 3, **d)), "accepted_nodes"), (dict(draft_v=bf(1, 4, 2, 64, **d)), "draft_v"),
                         (dict(accepted_len=n.long()), "accepted_len")):
        with pytest.raises(ValueError, match=name):
            gsd.gsd_commit_kv_paged(**{**w, **dict(draft_k=k, draft_v=k, accepted_nodes=ints(1, 3, **d), accepted_len=n, seq_lens=n), **change})
    for change, name in ((dict(counts=ints(2, **d)), "counts"), (dict(v=bf(1, 4, 2, 64, **d)), "v"), (dict(k=bf(1, 3, 2, 128, **d)[..., ::2]), "k"),
                         (dict(k=bf(1, 2, 3, 64, **d).transpose(1, 2)), "k"), (dict(freqs=f.double()), "freqs"),
                         (dict(freqs=f, positions=ints(1, 3, **d)), "positions"), (dict(freqs=f, positions=ints(1, 1, 4, **d)), "positions"),
                         (dict(freqs=f, offsets=ints(2, **d)), "offsets"), (dict(freqs=f, axes=[0] * 31), "axes"),
                         (dict(freqs=f, positions=ints(2, 1, 3, **d), axes=[2] * 32), "axes"), (dict(freqs=f, axes=[-1] * 32), "axes"),
                         (dict(positions=ints(1, 1, 3, **d)), "freqs"), (dict(axes=[0]), "freqs")):
        with pytest.raises(ValueError, match=name):
            gsd.gsd_append_kv_paged(**{**w, **dict(k=k, v=k, counts=n, seq_lens=n), **change})
    with pytest.raises(gsd.GsdError):
        gsd.gsd_append_kv_paged(**w, k=k, v=k, counts=n, seq_lens=n, freqs=f, axes=[4] * 32)
    with pytest.raises(gsd.GsdError):
        gsd.gsd_append_kv_paged(**w, k=bf(1, 3, 132, **d)[..., :128].unflatten(2, (2, 64)), v=k, counts=n, seq_lens=n)       # 264 bytes apart
    q, pos = bf(1, 3, 4, 64, **d), ints(1, 1, 3, **d)
    for args, kw, name in (((q, bf(1, 2, 2, 64, **d), f, pos), {}, "k"), ((q, k, f, None), {}, "positions"), ((q, k, f, pos), dict(out=(q, None)), "out"),
                           ((q, k, f, pos), dict(out=(k, k)), "q_out"), ((q, k, f.cpu(), pos), {}, "freqs")):
        with pytest.raises(ValueError, match=name):
            gsd.gsd_rotary(*args, **kw)
    with pytest.raises(gsd.GsdError):
        gsd.gsd_rotary(q, k, torch.zeros(12, device="cuda"), pos)
