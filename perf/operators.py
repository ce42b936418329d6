"""The operators around an 8-bit KV cache and the log probabilities of a step, as cases that can be timed.

Kinds:

  attn      gsd_verify_attn_q8: DAG-masked attention of the draft nodes over a cache held in 8 bits, with a
            power-of-two scale for each block of tokens and head
  commit    gsd_commit_kv_q8: the accepted path's K/V rows rounded into that cache
  append    gsd_append_kv_q8: the K/V rows of a prompt, or of a chunk of one, rounded into that cache
  logprobs  gsd_token_logprobs: log probabilities of given tokens, entropy of their rows, best alternatives

`listed()` names twelve of them, `draw()` gives more of the same ranges.  `run` computes the plain form in
32-bit torch operations, or, where `own` is set, makes the library's calls.
"""
import math

import numpy as np
import torch

own = False

_DEV = "cuda"
_QMAX = {"e4m3": 448.0, "int8": 127.0}
_DTYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
_EXP_MIN, _EXP_MAX = -117, 119


def listed():
    return [
        # ordinary decoding, one token a sequence and no draft graph: a server's step without speculation
        dict(name="attn_single_token", kind="attn", B=8, Hq=64, Hkv=8, D=128, Lmin=500, Lmax=4000, rows=4096, N=1, depth=0, fmt="e4m3", block=64),
        # LLaMA-2-7B layer shape (one kv head per query head), one user, moderate context
        dict(name="attn_llama7b", kind="attn", B=1, Hq=32, Hkv=32, D=128, Lmin=2048, Lmax=2048, rows=2048, N=64, depth=8, fmt="e4m3", block=64),
        # LLaMA-2-70B layer shape, eight users, large draft graphs
        dict(name="attn_llama70b", kind="attn", B=8, Hq=64, Hkv=8, D=128, Lmin=4096, Lmax=4096, rows=4352, N=256, depth=16, fmt="e4m3", block=128),
        # one user with a long document and a small draft graph
        dict(name="attn_long_context", kind="attn", B=1, Hq=64, Hkv=8, D=128, Lmin=32768, Lmax=32768, rows=32768, N=32, depth=10, fmt="int8", block=64),
        # a busy server: many users, short and ragged contexts, graphs of an odd size
        dict(name="attn_busy_ragged", kind="attn", B=32, Hq=64, Hkv=8, D=128, Lmin=200, Lmax=2100, rows=2304, N=57, depth=9, fmt="int8", block=32),
        # the small head dimension, few nodes, ragged contexts, short blocks
        dict(name="attn_head64", kind="attn", B=4, Hq=32, Hkv=8, D=64, Lmin=1000, Lmax=4000, rows=4001, N=12, depth=5, fmt="e4m3", block=16),
        # the accepted paths of one iteration, 70B layer shape, blocks partly filled
        dict(name="commit_llama70b", kind="commit", B=8, Hkv=8, D=128, Lmin=4000, Lmax=4096, rows=4352, N=256, T=17, fmt="e4m3", block=128),
        # the same for many users and kv heads, short blocks
        dict(name="commit_busy", kind="commit", B=32, Hkv=40, D=128, Lmin=200, Lmax=2100, rows=2304, N=57, T=10, fmt="int8", block=32),
        # prompts of different lengths written into an empty cache
        dict(name="append_prompts", kind="append", B=8, Hkv=8, D=128, Lmin=0, Lmax=0, rows=4352, T=4096, Tmin=1000, fmt="e4m3", block=64),
        # a chunk of a long prompt behind an odd position
        dict(name="append_chunk", kind="append", B=1, Hkv=32, D=128, Lmin=5003, Lmax=5003, rows=8192, T=512, Tmin=512, fmt="int8", block=32),
        # what a server returns beside the accepted tokens: five alternatives a token, filtered rows among them
        dict(name="logprobs_path", kind="logprobs", B=8, N=64, V=32000, T=9, Tmin=2, k=5, filtered=True),
        # all nodes of large graphs scored, odd vocabulary, many alternatives
        dict(name="logprobs_graph", kind="logprobs", B=6, N=128, V=50257, T=128, Tmin=120, k=20, filtered=False),
    ]


_HEADS = [(32, 32, 128), (40, 40, 128), (64, 8, 128), (32, 8, 128), (24, 8, 128), (28, 4, 128), (8, 1, 128), (32, 8, 64), (12, 12, 64)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "commit", "append", "logprobs", "logprobs"])
    fmt, block = rng.choice(["e4m3", "int8"]), rng.choice([16, 32, 64, 128])
    if kind == "logprobs":
        while True:
            V = rng.choice([32000, 50257, 50272, 128256, _log_int(rng, 100, 130000)])
            B, N = _log_int(rng, 1, 32), _log_int(rng, 1, 512)
            T = _log_int(rng, 1, N)
            if B * N * V <= 1 << 28 and B * T * V <= 6 * 128 * 50257:
                return dict(kind=kind, B=B, N=N, V=V, T=T, Tmin=rng.randint(0, T), k=rng.choice([0, 1, 5, 8, 20, 32]), filtered=rng.random() < 0.4)
    while True:
        Hq, Hkv, D = rng.choice(_HEADS)
        B, L = _log_int(rng, 1, 32), _log_int(rng, 16, 32768)
        Lmin = L if rng.random() < 0.4 else max(1, int(L * rng.uniform(0.1, 0.9)))
        c = dict(kind=kind, B=B, Hkv=Hkv, D=D, Lmin=Lmin, Lmax=L, fmt=fmt, block=block)
        if kind == "attn":
            N = 1 if rng.random() < 0.25 else _log_int(rng, 2, 400)
            c.update(Hq=Hq, N=N, depth=max(1, min(N - 1, int(round(2 * math.log2(N))))) if N > 1 else 0,
                     rows=L + rng.choice([0, 1, 17, 128, L // 4]))
            if work(c)["flops"] > 2.5e11 or B * Hq * N * (c["rows"] + N) > 1.2e9:
                continue
        elif kind == "commit":
            N = _log_int(rng, 2, 512)
            c.update(N=N, T=max(1, min(N, _log_int(rng, 1, 40))))
            c["rows"] = L + c["T"] + rng.choice([0, 1, 100])
        else:
            T = _log_int(rng, 1, 8192)
            c.update(T=T, Tmin=T if rng.random() < 0.4 else rng.randint(1, T))
            if rng.random() < 0.5:
                c["Lmin"] = c["Lmax"] = 0
            c["rows"] = c["Lmax"] + T + rng.choice([0, 1, 100])
            if B * T * Hkv * D > 8 * 4096 * 8 * 128:
                continue
        if B * c["rows"] * Hkv * D <= 3e8:
            return c


# ------------------------------------------------------------------------------ inputs
def _least_exp(amax, fmt):
    """The least exponent e with amax <= QMAX * 2^e, in the range the cache has."""
    m, ex = torch.frexp(amax)
    qm, qe = math.frexp(_QMAX[fmt])
    e = ex.to(torch.int32) - qe + (m > qm).to(torch.int32)
    return torch.where(amax > 0, e, torch.full_like(e, _EXP_MIN)).clamp(_EXP_MIN, _EXP_MAX)


def _two(e):
    """2^e, exactly."""
    return ((e.to(torch.int32).clamp(-126, 127) + 127) << 23).view(torch.float32)


def _codes(x, fmt):
    """x (already divided by its scale) rounded to what 8 bits hold, half to even."""
    q = _QMAX[fmt]
    if fmt == "int8":
        return torch.round(x).clamp(-q, q).to(torch.int8)
    return x.clamp(-q, q).to(torch.float8_e4m3fn)


def _round_cache(x, fmt, block):
    """Codes and exponents of rows [B, rows, H, D], a scale for each block of rows and head."""
    B, rows, H, D = x.shape
    nb = -(-rows // block)
    pad = torch.zeros((B, nb * block, H, D), device=x.device)
    pad[:, :rows] = x
    e = _least_exp(pad.view(B, nb, block, H, D).abs().amax((2, 4)), fmt)
    y = pad.view(B, nb, block, H, D) * _two(-e)[:, :, None, :, None]
    return _codes(y, fmt).view(B, nb * block, H, D)[:, :rows].contiguous(), e.to(torch.int8)


def _kv(gen, B, rows, H, D):
    """bf16 rows as attention layers have them: a few channels of a head stand out, heads differ in size."""
    x = torch.randn((B, rows, H, D), generator=gen, device=_DEV)
    loud = torch.where(torch.rand((H, D), generator=gen, device=_DEV) < 0.03, 4.0, 1.0)
    size = 0.5 + torch.rand((H, 1), generator=gen, device=_DEV)
    return x.mul_(loud * size / (1.0 + 3.0 * (loud.sum(1, keepdim=True) / D - 1.0))).to(torch.bfloat16)


def _masks(B, N, depth, rng):
    """Ancestor bitmask words of random level-structured graphs (a node's parents lie in the level above)."""
    W = (N + 31) // 32
    words = np.zeros((B, N, W * 32), bool)
    level = np.zeros(N, int)
    if N > 1:
        level[1:] = 1 + np.arange(N - 1) * max(depth, 1) // (N - 1)
    for b in range(B):
        see = words[b]
        for v in range(N):
            see[v, v] = True
            if v:
                above = np.flatnonzero(level == level[v] - 1)
                for p in rng.choice(above, min(len(above), int(rng.integers(1, 3))), replace=False):
                    see[v] |= see[p]
    packed = np.packbits(words, axis=2, bitorder="little").view(np.int32)
    return torch.from_numpy(np.ascontiguousarray(packed)).to(_DEV)


def prepare(case, seed):
    c, kind = case, case["kind"]
    rng = np.random.default_rng([seed, 3])
    gen = torch.Generator(device=_DEV).manual_seed(seed)
    B = c["B"]
    s = dict(kind=kind)
    if kind == "logprobs":
        N, V, T, k = c["N"], c["V"], c["T"], c["k"]
        k = min(k, V)
        x = torch.randn((B, N, V), generator=gen, device=_DEV).mul_(2.0)
        # most rows are fairly sure of a few tokens
        at = torch.randint(0, V, (B, N, 3), generator=gen, device=_DEV)
        x.scatter_(2, at, (torch.tensor([14.0, 13.0, 11.0], device=_DEV) + torch.randn((B, N, 3), generator=gen, device=_DEV)).expand(B, N, 3).contiguous())
        if c["filtered"]:               # what top-p or top-k sampling leaves of every second row
            x[:, ::2] = x[:, ::2].masked_fill(x[:, ::2] < 3.0, -math.inf)
        s["k"] = k
        s["logits"] = x
        s["nodes"] = torch.from_numpy(np.sort(rng.permuted(np.tile(np.arange(N), (B, 1)), axis=1)[:, :T], axis=1).astype(np.int32)).to(_DEV)
        s["lens"] = torch.from_numpy(rng.integers(c["Tmin"], T + 1, B).astype(np.int32)).to(_DEV)
        # the emitted token is mostly one that the row is sure of
        sure = at.gather(1, s["nodes"].long()[:, :, None].expand(B, T, 3))[:, :, 0]
        other = torch.randint(0, V, (B, T), generator=gen, device=_DEV)
        s["tokens"] = torch.where(torch.rand((B, T), generator=gen, device=_DEV) < 0.8, sure, other).to(torch.int32)
        return s
    H, D, fmt, block = c["Hkv"], c["D"], c["fmt"], c["block"]
    s["fmt"], s["block"] = fmt, block
    s["k_cache"], s["k_exp"] = _round_cache(_kv(gen, B, c["rows"], H, D), fmt, block)
    s["v_cache"], s["v_exp"] = _round_cache(_kv(gen, B, c["rows"], H, D), fmt, block)
    s["seq_lens"] = torch.from_numpy(rng.integers(c["Lmin"], c["Lmax"] + 1, B, dtype=np.int32)).to(_DEV)
    if kind == "attn":
        N, Hq = c["N"], c["Hq"]
        s["q"] = torch.randn((B, N, Hq, D), generator=gen, device=_DEV, dtype=torch.bfloat16)
        s["draft_k"], s["draft_v"] = _kv(gen, B, N, H, D), _kv(gen, B, N, H, D)
        s["mask"] = _masks(B, N, c["depth"], rng)
        return s
    s["lens0"] = s["seq_lens"].clone()
    T = c["T"]
    if kind == "commit":
        N = c["N"]
        s["draft_k"], s["draft_v"] = _kv(gen, B, N, H, D), _kv(gen, B, N, H, D)
        n = rng.integers(1, T + 1, B).astype(np.int32)
        nodes = np.full((B, T), -1, np.int32)
        for b in range(B):
            nodes[b, :n[b]] = np.concatenate(([0], np.sort(rng.permutation(np.arange(1, N))[:n[b] - 1])))
        s["nodes"], s["count"] = torch.from_numpy(nodes).to(_DEV), torch.from_numpy(n).to(_DEV)
    else:
        s["k"], s["v"] = _kv(gen, B, T, H, D), _kv(gen, B, T, H, D)
        s["count"] = torch.from_numpy(rng.integers(c["Tmin"], T + 1, B).astype(np.int32)).to(_DEV)
    return s


# -------------------------------------------------------------------------------- plain forms
def _attn_plain(s):
    q, (B, N, Hq, D) = s["q"], s["q"].shape
    rows, H = s["k_cache"].shape[1:3]
    G = Hq // H
    qs = q.float().view(B, N, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, N * G, D)

    def values(codes, exp, draft):
        scale = _two(exp).repeat_interleave(s["block"], 1)[:, :rows]
        return torch.cat((codes.float() * scale[..., None], draft.float()), 1).permute(0, 2, 1, 3)     # [B, H, keys, D]
    K, V = values(s["k_cache"], s["k_exp"], s["draft_k"]), values(s["v_cache"], s["v_exp"], s["draft_v"])
    j = torch.arange(N, device=q.device)
    bits = (s["mask"][:, :, j // 32] >> (j % 32).to(torch.int32)) & 1                                   # [B, N, N]
    seen = torch.arange(rows, device=q.device)[None, :] < s["seq_lens"][:, None]
    seen = torch.cat((seen[:, None, :].expand(B, N, rows), bits.bool()), 2)                             # [B, N, keys]
    seen = seen[:, None, :, None, :].expand(B, 1, N, G, rows + N).reshape(B, 1, N * G, rows + N)
    x = torch.matmul(qs, K.transpose(2, 3)).mul_(D ** -0.5)
    x.masked_fill_(~seen, -math.inf)
    x.sub_(x.amax(3, keepdim=True)).exp_()
    V = V.masked_fill(~seen.any(2)[..., None], 0.0)
    out = torch.matmul(x, V) / x.sum(3, keepdim=True)
    return out.view(B, H, N, G, D).permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D).to(torch.bfloat16)


def _write_plain(s, codes, exp, x, L, n):
    """Rows x [B, M, H, D] (the first n of each sequence) into positions L, L + 1, ... of codes / exp, in place."""
    fmt, block = s["fmt"], s["block"]
    B, M, H, D = x.shape
    rows, nb = codes.shape[1], exp.shape[1]
    wb = -(-M // block) + 1
    first = L.long() // block
    blk = first[:, None] + torch.arange(wb, device=x.device)
    pos = first[:, None] * block + torch.arange(wb * block, device=x.device)                            # [B, W]
    inside = pos < rows
    at = pos.clamp(max=rows - 1)
    b = torch.arange(B, device=x.device)[:, None]
    src = pos - L[:, None]
    new = (src >= 0) & (src < n[:, None]) & inside
    rowsx = torch.where(new[..., None, None], x[b, src.clamp(0, M - 1)].float(), 0.0)
    top = rowsx.view(B, wb, block, H, D).abs().amax((2, 4))
    e_old = exp[b, blk.clamp(max=nb - 1)].to(torch.int32)
    held = (blk * block < L[:, None])[..., None]
    e = torch.maximum(torch.where(held, e_old, torch.full_like(e_old, _EXP_MIN)), _least_exp(top, fmt))
    e = torch.where(new.view(B, wb, block).any(2)[..., None], e, e_old)
    per_row = e.repeat_interleave(block, 1)[..., None]
    old = codes[b, at].float() * _two(e_old.repeat_interleave(block, 1)[..., None] - per_row)
    keep = (pos < L[:, None])[..., None, None]
    got = _codes(torch.where(keep, old, rowsx * _two(-per_row)), fmt)
    put = (new | (pos < L[:, None])) & inside
    bb = b.expand_as(pos)[put]
    codes.view(torch.int8)[bb, pos[put]] = got.view(torch.int8)[put]
    fits = blk < nb
    exp[b.expand_as(blk)[fits], blk[fits]] = e.to(torch.int8)[fits]
    return torch.minimum(n, rows - L)


def _logprobs_plain(s):
    B, T = s["nodes"].shape
    b = torch.arange(B, device=_DEV)[:, None]
    x = s["logits"][b, s["nodes"].long()]                                                               # [B, T, V]
    used = torch.arange(T, device=_DEV)[None, :] < s["lens"][:, None]
    m = x.amax(2, keepdim=True)
    d = x - m
    e = torch.exp(d)
    total = e.sum(2)
    lse = torch.log(total)
    lp = d.gather(2, s["tokens"].long()[..., None])[..., 0] - lse
    ent = lse - torch.where(e > 0, e * d, 0.0).sum(2) / total
    val, idx = torch.sort(x, dim=2, descending=True, stable=True)
    val, idx = val[..., :s["k"]], idx[..., :s["k"]]
    return dict(logprobs=torch.where(used, lp, 0.0), entropy=torch.where(used, ent, 0.0),
                top_tokens=torch.where(used[..., None], idx, -1).to(torch.int32),
                top_logprobs=torch.where(used[..., None], val - m - lse[..., None], 0.0))


# -------------------------------------------------------------------------------- calls
def _run_own(s):
    import paper_2407_16207_b200 as gsd
    kind = s["kind"]
    if kind == "attn":
        return gsd.gsd_verify_attn_q8(s["q"], s["k_cache"], s["v_cache"], s["k_exp"], s["v_exp"], s["draft_k"], s["draft_v"],
                                      s["mask"], s["seq_lens"], block=s["block"])
    if kind == "logprobs":
        lp, ent, tok, val = gsd.gsd_token_logprobs(s["logits"], s["nodes"], s["tokens"], s["lens"], k=s["k"])
        return dict(logprobs=lp, entropy=ent, top_tokens=tok, top_logprobs=val)
    s["seq_lens"].copy_(s["lens0"])             # a pass starts from the same committed lengths again
    if kind == "commit":
        gsd.gsd_commit_kv_q8(s["k_cache"], s["v_cache"], s["k_exp"], s["v_exp"], s["draft_k"], s["draft_v"],
                             s["nodes"], s["count"], s["seq_lens"], block=s["block"])
    else:
        gsd.gsd_append_kv_q8(s["k_cache"], s["v_cache"], s["k_exp"], s["v_exp"], s["k"], s["v"], s["count"], s["seq_lens"],
                             block=s["block"])
    return _cache(s)


def _cache(s):
    return dict(k_cache=s["k_cache"], v_cache=s["v_cache"], k_exp=s["k_exp"], v_exp=s["v_exp"], seq_lens=s["seq_lens"])


def run(state):
    s, kind = state, state["kind"]
    if own:
        return _run_own(s)
    if kind == "attn":
        return _attn_plain(s)
    if kind == "logprobs":
        return _logprobs_plain(s)
    L, n = s["lens0"], s["count"]
    if kind == "commit":
        b, at = torch.arange(L.shape[0], device=_DEV)[:, None], s["nodes"].long().clamp(min=0)
        k, v = s["draft_k"][b, at], s["draft_v"][b, at]
    else:
        k, v = s["k"], s["v"]
    _write_plain(s, s["k_cache"], s["k_exp"], k, L, n)
    s["seq_lens"].copy_(L + _write_plain(s, s["v_cache"], s["v_exp"], v, L, n))
    return _cache(s)


# ------------------------------------------------------------------------- 64-bit answer
def _exact_attn(s):
    q, B, N = s["q"], s["q"].shape[0], s["q"].shape[1]
    Hq, D, H = q.shape[2], q.shape[3], s["draft_k"].shape[2]
    G, lens = Hq // H, s["seq_lens"].cpu().numpy()
    words = s["mask"].cpu().numpy().view(np.uint8).reshape(B, N, -1)
    see = torch.from_numpy(np.unpackbits(words, axis=2, bitorder="little")[:, :, :N].astype(bool)).to(_DEV)
    out = torch.empty(q.shape, dtype=torch.float64, device=_DEV)
    for b in range(B):
        L = int(lens[b])
        step = torch.arange(L, device=_DEV) // s["block"]
        hide = ~see[b].repeat_interleave(G, 0)
        for c in range(H):
            k = torch.cat((s["k_cache"][b, :L, c].double() * _pow2(s["k_exp"][b, step, c])[:, None], s["draft_k"][b, :, c].double()))
            v = torch.cat((s["v_cache"][b, :L, c].double() * _pow2(s["v_exp"][b, step, c])[:, None], s["draft_v"][b, :, c].double()))
            x = q[b, :, c * G:(c + 1) * G].reshape(N * G, D).double() @ k.T
            x *= D ** -0.5
            x[:, L:].masked_fill_(hide, -math.inf)
            out[b, :, c * G:(c + 1) * G] = (torch.softmax(x, 1) @ v).view(N, G, D)
    return out


def _pow2(k):
    """2^k for whole k, exactly (a library's power may be an ulp off, and ties would fall the other way)."""
    return ((k.double().clamp(min=-1000).long() + 1023) << 52).view(torch.float64)


def _exact_round(y, fmt):
    """y (64 bits, in units of the scale) to the nearest value of the format, ties to the even one."""
    q = _QMAX[fmt]
    if fmt == "int8":
        step = torch.ones_like(y)
    else:                               # three bits behind the leading one, down to 2^-9
        step = _pow2(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return (torch.round(y / step) * step).clamp(-q, q)


def _exact_write(s, name, x):
    """The cache `name` with rows x [B, M, H, D] behind the old ends, block by block."""
    codes, exp, fmt, block = s[name + "_cache"].double(), s[name + "_exp"].double(), s["fmt"], s["block"]
    rows, lens, count = codes.shape[1], s["lens0"].tolist(), s["count"].tolist()
    for b in range(codes.shape[0]):
        L, end = lens[b], min(lens[b] + count[b], rows)
        at = L
        while at < end:
            blk = at // block
            lo, hi = blk * block, min(end, (blk + 1) * block)
            new = x[b, at - L:hi - L].double()                                                          # [rows, H, D]
            top = new.abs().amax((0, 2))
            e = torch.ceil(torch.log2(top / _QMAX[fmt]))
            e = torch.where(top > _QMAX[fmt] * _pow2(e), e + 1, e)                                      # (what a rounded logarithm leaves)
            e = torch.where(top <= _QMAX[fmt] * _pow2(e - 1), e - 1, e).clamp(_EXP_MIN, _EXP_MAX)
            if lo < at:
                e = torch.maximum(e, exp[b, blk])
                codes[b, lo:at] = _exact_round(codes[b, lo:at] * _pow2(exp[b, blk] - e)[None, :, None], fmt)
            codes[b, at:hi] = _exact_round(new * _pow2(-e)[None, :, None], fmt)
            exp[b, blk] = e
            at = hi
    return codes


def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    if kind == "attn":
        return _exact_attn(s)
    if kind == "logprobs":
        B, T = s["nodes"].shape
        out = dict(logprobs=torch.zeros((B, T), dtype=torch.float64), entropy=torch.zeros((B, T), dtype=torch.float64),
                   top_tokens=None, top_logprobs=torch.zeros((B, T, s["k"]), dtype=torch.float64))
        for b in range(B):
            n = int(s["lens"][b])
            lp = torch.log_softmax(s["logits"][b, s["nodes"][b, :n].long()].double(), 1)
            out["logprobs"][b, :n] = lp.gather(1, s["tokens"][b, :n].long()[:, None])[:, 0]
            out["entropy"][b, :n] = -torch.special.xlogy(lp.exp(), lp.exp()).sum(1)
            out["top_logprobs"][b, :n] = lp.topk(s["k"], 1).values
        return out
    if case["fmt"] == "int8":
        return None                     # whole numbers only
    if kind == "commit":
        rows = [s[n][torch.arange(case["B"], device=_DEV)[:, None], s["nodes"].long().clamp(min=0)] for n in ("draft_k", "draft_v")]
    else:
        rows = [s["k"], s["v"]]
    return dict(k_cache=_exact_write(s, "k", rows[0]), v_cache=_exact_write(s, "v", rows[1]), k_exp=None, v_exp=None, seq_lens=None)


def work(case):
    c, kind, B = case, case["kind"], case["B"]
    if kind == "logprobs":
        n = B * (c["Tmin"] + c["T"]) / 2
        return {"bytes": n * (c["V"] * 4.0 + 12 + 8 * c["k"] + 8), "flops": 6.0 * n * c["V"]}
    row = c["Hkv"] * c["D"]
    if kind == "attn":
        L, N = (c["Lmin"] + c["Lmax"]) / 2, c["N"]
        nbytes = 2 * B * N * c["Hq"] * c["D"] * 2 + 2 * B * L * (row + c["Hkv"] / c["block"]) + 2 * B * N * row * 2 + B * N * ((N + 31) // 32) * 4
        return {"bytes": nbytes, "flops": 4.0 * B * N * c["Hq"] * c["D"] * (L + max(c["depth"], 1))}
    n = B * ((1 if kind == "commit" else c["Tmin"]) + c["T"]) / 2
    return {"bytes": 2 * n * row * 3.0 + 8.0 * B, "flops": 4.0 * n * row}
