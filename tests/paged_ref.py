"""A paged cache and rotary positions in 64 bits (numpy), row by row from their definitions, and inputs for the calls over them."""
import numpy as np
import torch

import kv8_ref


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()


def table_for(rng, need, M, spare=2, junk=(-1, 2 ** 31 - 1, -2 ** 31)):
    """(table [B, M], pages of the pool): need[b] pages for each sequence, out of order; the rest of a row names no page."""
    P = int(sum(need)) + spare
    ids = rng.permutation(P)
    table = np.empty((len(need), M), np.int32)
    table[:] = rng.choice(np.asarray(junk, np.int64), (len(need), M)).astype(np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, P


def rows_of(pages, table, L):
    """The first L rows of a sequence whose row of the table is given."""
    page = pages.shape[1]
    j = np.arange(L)
    return pages[table[j // page], j % page]


def turn(x, pos, freqs, axes, neighbours):
    """Rows x [T, H, D] (64 bits) rotated by pos [axes, T]."""
    n = len(freqs)
    out = x.copy()
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, n + i)
        ang = pos[axes[i]].astype(np.float64) * np.float64(freqs[i])
        c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return out


def turn_room(x, n, neighbours):
    """|x| + |y| of the pair of each rotated element, 0 for the others."""
    out = np.zeros_like(x)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, n + i)
        out[..., a] = out[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return out


# A rotated element: the rounding to bf16, 2^-8 of it; sine and cosine off by half of 2^-23 of an angle of up to pi and by 2 ulp of a
# value below 1, two products and a sum: below 2^-21 of |x| + |y| (angles here are below 2^22 turns, which adds 2^-28).
def turn_tol(x, ref, n, neighbours):
    return 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * turn_room(x, n, neighbours)


def attn_inputs(seed, B, N, Hq, Hkv, D, lens, page, mask="random", M=None, shared=0, fill=np.nan):
    """Inputs of the attention over pages; what no sequence may look at is `fill`."""
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lens]
    M = M or max(need) + 1
    table, P = table_for(rng, need, M)
    if shared:                                   # the first `shared` pages of all sequences in common
        table[:, :shared] = table[0, :shared]
    k, v = rng.standard_normal((2, P, page, Hkv, D)).astype(np.float32)
    used = np.zeros((P, page), bool)
    for b, L in enumerate(lens):
        j = np.arange(L)
        used[table[b, j // page], j % page] = True
    k[~used] = fill
    v[~used] = fill
    x = dict(B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, lens=np.asarray(lens, np.int32), page=page, table=table, k=bf16(k), v=bf16(v),
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


def attn_tensors(x):
    return dict(q=x["q"].cuda(), k_pages=x["k"].cuda(), v_pages=x["v"].cuda(), page_table=i32(x["table"]), draft_k=x["dk"].cuda(),
                draft_v=x["dv"].cuda(), ancestor_mask=i32(x["mask"]), seq_lens=i32(x["lens"]))


def attn_want(x, scale=None):
    """The definition's output, sum p |v|, and scale * sum |q k| of the visible keys."""
    f = lambda t: t.double().numpy()
    k, v = f(x["k"]), f(x["v"])
    got = [kv8_ref.attention(f(x["q"][b]), rows_of(k, x["table"][b], L), rows_of(v, x["table"][b], L), L, f(x["dk"][b]), f(x["dv"][b]),
                             x["see"][b], scale or x["D"] ** -0.5) for b, L in enumerate(x["lens"].tolist())]
    return [np.stack(a) for a in zip(*got)]


# The output's rounding, 2^-8 of it; the weights' rounding to bf16, 2^-8 of sum p |v|; a score is an fp32 sum of D <= 128 products, off
# by at most 2^-16 of S = scale * sum |q k|, which moves a weight by that much of itself and the sum it is divided by likewise; 2^-20
# for the exponentials and the sums.
def attn_check(x, got, scale=None):
    ref, spread, size = attn_want(x, scale)
    err = np.abs(got.double().cpu().numpy() - ref)
    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -20 + 2.0 ** -15 * size) * spread
    assert np.isfinite(err).all()
    assert (err <= tol).all(), (float((err - tol).max()), np.unravel_index(np.argmax(err - tol), err.shape))
