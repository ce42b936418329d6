"""The operators around a paged KV cache, as cases that can be timed.

Kinds:

  attn    gsd_verify_attn_paged: DAG-masked attention of the draft nodes over a cache held in pages
  append  gsd_append_kv_paged: the K/V rows of a prompt, or of a chunk of one, into the pages, K rotated by position
  commit  gsd_commit_kv_paged: the accepted path's K/V rows into the pages
  rotary  gsd_rotary: the draft nodes' Q and K rotated by position, with one axis (text) or three (images, video)

`listed()` names twelve of them, `draw()` gives more of the same ranges.  `run` computes the plain form in 32-bit torch
operations (angles in 64), or, where `own` is set, makes the library's calls.
"""
import math

import numpy as np
import torch

own = False

_DEV = "cuda"


def listed():
    return [
        # ordinary decoding, one token a sequence and no draft graph, short pages as servers use them
        dict(name="attn_single_token", kind="attn", B=8, Hq=64, Hkv=8, D=128, Lmin=500, Lmax=4000, page=16, shared=0, N=1, depth=0),
        # LLaMA-2-7B layer shape (one kv head per query head), one user, moderate context
        dict(name="attn_llama7b", kind="attn", B=1, Hq=32, Hkv=32, D=128, Lmin=2048, Lmax=2048, page=16, shared=0, N=64, depth=8),
        # LLaMA-2-70B layer shape, eight users, large draft graphs
        dict(name="attn_llama70b", kind="attn", B=8, Hq=64, Hkv=8, D=128, Lmin=4096, Lmax=4096, page=64, shared=0, N=256, depth=16),
        # one user with a long document and a small draft graph, long pages
        dict(name="attn_long_context", kind="attn", B=1, Hq=64, Hkv=8, D=128, Lmin=32768, Lmax=32768, page=256, shared=0, N=32, depth=10),
        # a busy server: many users behind one system prompt whose pages they share, ragged contexts, graphs of an odd size
        dict(name="attn_busy_shared", kind="attn", B=32, Hq=64, Hkv=8, D=128, Lmin=500, Lmax=2100, page=32, shared=448, N=57, depth=9),
        # the small head dimension, few nodes, ragged contexts
        dict(name="attn_head64", kind="attn", B=4, Hq=32, Hkv=8, D=64, Lmin=1000, Lmax=4000, page=128, shared=0, N=12, depth=5),
        # prompts of different lengths written into fresh pages
        dict(name="append_prompts", kind="append", B=8, Hq=64, Hkv=8, D=128, Lmin=0, Lmax=0, page=64, T=4096, Tmin=1000, R=128, pairs=False, axes="text"),
        # a chunk of a prompt with images in it, behind an odd position, short pages
        dict(name="append_images", kind="append", B=1, Hq=28, Hkv=4, D=128, Lmin=5003, Lmax=5003, page=16, T=1031, Tmin=1031, R=128, pairs=False, axes="blocks"),
        # the accepted paths of one iteration, 70B layer shape
        dict(name="commit_llama70b", kind="commit", B=8, Hkv=8, D=128, Lmin=4000, Lmax=4096, page=64, N=256, T=17),
        # the same for many users and kv heads, short pages
        dict(name="commit_busy", kind="commit", B=32, Hkv=40, D=128, Lmin=200, Lmax=2100, page=16, N=57, T=10),
        # Q and K of the draft graphs of one iteration, 70B layer shape, out of the fused projection
        dict(name="rotary_llama70b", kind="rotary", B=8, Hq=64, Hkv=8, D=128, N=256, depth=16, L=4096, R=128, pairs=False, axes="text"),
        # single tokens behind images: three axes in turn, half of the columns rotated, neighbours as pairs
        dict(name="rotary_single_token", kind="rotary", B=32, Hq=32, Hkv=8, D=128, N=1, depth=0, L=30000, R=64, pairs=True, axes="turns"),
    ]


_HEADS = [(32, 32, 128), (40, 40, 128), (64, 8, 128), (32, 8, 128), (28, 4, 128), (8, 1, 128), (16, 4, 64), (12, 12, 64)]
_ATTN_HEADS = _HEADS + [(32, 8, 64)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "append", "append", "commit", "rotary", "rotary"])
    while True:
        B, page = _log_int(rng, 1, 32), rng.choice([16, 32, 64, 128, 256])
        Hq, Hkv, D = rng.choice(_ATTN_HEADS if kind in ("attn", "commit") else _HEADS)
        L = _log_int(rng, 16, 32768)
        Lmin = L if rng.random() < 0.4 else max(1, int(L * rng.uniform(0.1, 0.9)))
        N = 1 if rng.random() < 0.25 else _log_int(rng, 2, 400)
        depth = max(1, min(N - 1, int(round(2 * math.log2(N))))) if N > 1 else 0
        turned = dict(R=rng.choice([D, D, D // 2, D // 4]), pairs=rng.random() < 0.4, axes=rng.choice(["text", "blocks", "turns"]))
        if kind == "rotary":
            c = dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, D=D, N=N, depth=depth, L=_log_int(rng, 1, 1000000), **turned)
            if B * N * (Hq + Hkv) * D <= 8 * 256 * 72 * 128:
                return c
            continue
        c = dict(kind=kind, B=B, Hkv=Hkv, D=D, Lmin=Lmin, Lmax=L, page=page)
        if kind == "attn":
            c.update(Hq=Hq, N=N, depth=depth, shared=rng.choice([0, 0, Lmin // 2]) // page * page)
            if work(c)["flops"] > 2.5e11 or B * Hq * N * (L + N) > 1.2e9:
                continue
        elif kind == "commit":
            N = _log_int(rng, 2, 512)
            c.update(N=N, T=max(1, min(N, _log_int(rng, 1, 40))))
        else:
            T = _log_int(rng, 1, 8192)
            c.update(Hq=Hq, T=T, Tmin=T if rng.random() < 0.4 else rng.randint(1, T), **turned)
            if rng.random() < 0.5:
                c["Lmin"] = c["Lmax"] = 0
            if B * T * Hkv * D > 8 * 4096 * 8 * 128 or B * T * (Hq + 2 * Hkv) * D > 1 << 29:
                continue
        if B * (c["Lmax"] + c.get("T", 0) + page) * Hkv * D <= 3e8:
            return c


# ------------------------------------------------------------------------------ inputs
def _kv(gen, shape):
    """bf16 rows [..., H, D] as attention layers have them: a few channels of a head stand out, heads differ in size."""
    H, D = shape[-2:]
    x = torch.randn(shape, generator=gen, device=_DEV)
    loud = torch.where(torch.rand((H, D), generator=gen, device=_DEV) < 0.03, 4.0, 1.0)
    size = 0.5 + torch.rand((H, 1), generator=gen, device=_DEV)
    return x.mul_(loud * size / (1.0 + 3.0 * (loud.sum(1, keepdim=True) / D - 1.0))).to(torch.bfloat16)


def _levels(N, depth):
    level = np.zeros(N, np.int32)
    if N > 1:
        level[1:] = 1 + np.arange(N - 1) * max(depth, 1) // (N - 1)
    return level


def _masks(B, N, depth, rng):
    """Ancestor bitmask words of random level-structured graphs (a node's parents lie in the level above)."""
    W = (N + 31) // 32
    words = np.zeros((B, N, W * 32), bool)
    level = _levels(N, depth)
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


def _table(c, lens, room, rng):
    """Page table [B, M] and pool size: every sequence has pages for `room` tokens, out of order in the pool, the first
    `shared` tokens' pages in common; the rest of a row is -1, and some pages of the pool belong to nobody."""
    B, page = c["B"], c["page"]
    M = -(-(c["Lmax"] + c.get("T", 0)) // page) + 1
    common = c.get("shared", 0) // page
    need = [max(-(-int(n) // page), common) for n in lens + room]
    P = common + B * (M - 1 - common) + 3               # what the longest sequences would need
    ids = rng.permutation(P).astype(np.int32)
    table = np.full((B, M), -1, np.int32)
    at = common
    for b in range(B):
        table[b, :common] = ids[:common]
        table[b, common:need[b]] = ids[at:at + need[b] - common]
        at += need[b] - common
    return torch.from_numpy(table).to(_DEV), P


def _axes(c):
    """The position axis of each pair of columns: one axis, three in blocks of a quarter and twice three eighths, or in turns."""
    n = c["R"] // 2
    if c["axes"] == "text":
        return [0] * n
    if c["axes"] == "turns":
        return [i % 3 for i in range(n)]
    return [0 if i < n // 4 else 1 if i < n // 4 + 3 * n // 8 else 2 for i in range(n)]


def _image_positions(T, rng):
    """Positions (time, height, width) of T tokens: text, where all three go on together, and images in raster order."""
    out, at, start = np.zeros((3, T), np.int32), 0, 0
    while at < T:
        n = min(T - at, int(rng.integers(5, 120)))
        out[:, at:at + n] = start + np.arange(n)
        at, start = at + n, start + n
        h, w = int(rng.integers(4, 24)), int(rng.integers(4, 24))
        n = min(T - at, h * w)
        i = np.arange(n)
        out[0, at:at + n], out[1, at:at + n], out[2, at:at + n] = start, start + i // w, start + i % w
        at, start = at + n, start + max(h, w)
    return out


def _rotation(c, s, gen):
    n = c["R"] // 2
    s["pairs"], s["axes"] = c["pairs"], _axes(c)
    s["freqs"] = torch.from_numpy((500000.0 ** (-np.arange(n) / n)).astype(np.float32)).to(_DEV)


def prepare(case, seed):
    c, kind = case, case["kind"]
    rng = np.random.default_rng([seed, 5])
    gen = torch.Generator(device=_DEV).manual_seed(seed)
    B, Hkv, D = c["B"], c["Hkv"], c["D"]
    s = dict(kind=kind)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(_DEV)
    if kind == "rotary":
        # the projection's output: the heads of Q, of K and of V of a token side by side
        N, Hq = c["N"], c["Hq"]
        qkv = _kv(gen, (B, N, Hq + 2 * Hkv, D))
        s["q"], s["k"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
        _rotation(c, s, gen)
        lens = rng.integers(max(c["L"] // 2, 1), c["L"] + 1, B).astype(np.int32)
        s["offsets"] = put(lens)
        level = _levels(N, c["depth"])
        # behind an image the three axes of text go on together: a draft node lies its level behind the sequence
        s["positions"] = put(np.broadcast_to(level, (1 if c["axes"] == "text" else 3, B, N)).astype(np.int32))
        return s
    lens = rng.integers(c["Lmin"], c["Lmax"] + 1, B).astype(np.int32)
    s["seq_lens"], s["page"] = put(lens), c["page"]
    if kind == "append":
        count = rng.integers(c["Tmin"], c["T"] + 1, B).astype(np.int32)
    elif kind == "commit":
        count = rng.integers(1, c["T"] + 1, B).astype(np.int32)
    else:
        count = np.zeros(B, np.int32)
    s["table"], P = _table(c, lens, count, rng)
    s["k_pages"], s["v_pages"] = _kv(gen, (P, c["page"], Hkv, D)), _kv(gen, (P, c["page"], Hkv, D))
    if kind == "attn":
        N, Hq = c["N"], c["Hq"]
        s["q"] = torch.randn((B, N, Hq, D), generator=gen, device=_DEV, dtype=torch.bfloat16)
        s["draft_k"], s["draft_v"] = _kv(gen, (B, N, Hkv, D)), _kv(gen, (B, N, Hkv, D))
        s["mask"] = _masks(B, N, c["depth"], rng)
        return s
    s["lens0"], s["count"] = s["seq_lens"].clone(), put(count)
    T = c["T"]
    if kind == "commit":
        N = c["N"]
        s["draft_k"], s["draft_v"] = _kv(gen, (B, N, Hkv, D)), _kv(gen, (B, N, Hkv, D))
        nodes = np.full((B, T), -1, np.int32)
        for b in range(B):
            nodes[b, :count[b]] = np.concatenate(([0], np.sort(rng.permutation(np.arange(1, N))[:count[b] - 1])))
        s["nodes"] = put(nodes)
        return s
    Hq = c["Hq"]
    qkv = _kv(gen, (B, T, Hq + 2 * Hkv, D))
    s["k"], s["v"] = qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    _rotation(c, s, gen)
    s["positions"] = s["offsets"] = None                # text: the token's place in the sequence
    if c["axes"] != "text":
        s["positions"] = put(np.stack([_image_positions(T, rng) for _ in range(B)], 1))
        s["offsets"] = put((lens * 0.7).astype(np.int32))
    return s


# -------------------------------------------------------------------------------- plain forms
def _rows(s, pages):
    """The pages' rows in the order of the sequences: [B, M * page, H, D]."""
    B, M = s["table"].shape
    return pages[s["table"].clamp(min=0).long()].reshape(B, M * s["page"], *pages.shape[2:])


def _attn_plain(s):
    q, (B, N, Hq, D) = s["q"], s["q"].shape
    H = s["k_pages"].shape[2]
    G = Hq // H
    qs = q.float().view(B, N, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, N * G, D)
    K = torch.cat((_rows(s, s["k_pages"]).float(), s["draft_k"].float()), 1).permute(0, 2, 1, 3)         # [B, H, keys, D]
    V = torch.cat((_rows(s, s["v_pages"]).float(), s["draft_v"].float()), 1).permute(0, 2, 1, 3)
    rows = K.shape[2] - N
    j = torch.arange(N, device=q.device)
    bits = (s["mask"][:, :, j // 32] >> (j % 32).to(torch.int32)) & 1                                   # [B, N, N]
    seen = torch.arange(rows, device=q.device)[None, :] < s["seq_lens"][:, None]
    seen = torch.cat((seen[:, None, :].expand(B, N, rows), bits.bool()), 2)                             # [B, N, keys]
    seen = seen[:, None, :, None, :].expand(B, 1, N, G, rows + N).reshape(B, 1, N * G, rows + N)
    x = torch.matmul(qs, K.transpose(2, 3)).mul_(D ** -0.5)
    x.masked_fill_(~seen, -math.inf)
    x.sub_(x.amax(3, keepdim=True)).exp_()
    out = torch.matmul(x, V) / x.sum(3, keepdim=True)
    return out.view(B, H, N, G, D).permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D).to(torch.bfloat16)


def _turn_plain(s, x, pos):
    """Rows x [B, T, H, D] rotated by the positions pos [axes, B, T] (64-bit whole numbers)."""
    n = s["freqs"].shape[0]
    at = pos[torch.tensor(s["axes"], device=x.device)].permute(1, 2, 0)                                  # [B, T, pairs]
    angle = at.double() * s["freqs"].double()
    c, d = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    y = x.float()
    out = y.clone()
    one, two = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if s["pairs"] else (slice(0, n), slice(n, 2 * n))
    out[..., one] = y[..., one] * c - y[..., two] * d
    out[..., two] = y[..., one] * d + y[..., two] * c
    return out.to(torch.bfloat16)


def _positions(s, T, start):
    """Positions [axes, B, T] in 64 bits."""
    if s["positions"] is None:
        return (start.long()[:, None] + torch.arange(T, device=_DEV))[None]
    return s["positions"].long() + s["offsets"].long()[None, :, None]


def _put_plain(s, k, v):
    """Rows k, v [B, T, H, D], the first count of each sequence, into the pages behind the old ends."""
    B, T = k.shape[:2]
    t = torch.arange(T, device=_DEV)
    at = s["lens0"].long()[:, None] + t
    M, page = s["table"].shape[1], s["page"]
    new = (t < s["count"][:, None]) & (at < M * page)
    row = s["table"].gather(1, (at // page).clamp(max=M - 1)).long() * page + at % page
    s["k_pages"].flatten(0, 1)[row[new]] = k[new]
    s["v_pages"].flatten(0, 1)[row[new]] = v[new]
    s["seq_lens"].copy_(s["lens0"] + s["count"])


# -------------------------------------------------------------------------------- calls
def _cache(s):
    return dict(k_pages=s["k_pages"], v_pages=s["v_pages"], seq_lens=s["seq_lens"])


def _run_own(s):
    import paper_2407_16207_b200 as gsd
    kind = s["kind"]
    if kind == "attn":
        return gsd.gsd_verify_attn_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["draft_k"], s["draft_v"], s["mask"],
                                         s["seq_lens"])
    if kind == "rotary":
        return gsd.gsd_rotary(s["q"], s["k"], s["freqs"], s["positions"], offsets=s["offsets"], axes=s["axes"], pairs=s["pairs"])
    s["seq_lens"].copy_(s["lens0"])             # a pass starts from the same committed lengths again
    if kind == "commit":
        gsd.gsd_commit_kv_paged(s["k_pages"], s["v_pages"], s["table"], s["draft_k"], s["draft_v"], s["nodes"], s["count"],
                                s["seq_lens"])
    else:
        gsd.gsd_append_kv_paged(s["k_pages"], s["v_pages"], s["table"], s["k"], s["v"], s["count"], s["seq_lens"],
                                freqs=s["freqs"], positions=s["positions"], offsets=s["offsets"], axes=s["axes"], pairs=s["pairs"])
    return _cache(s)


def run(state):
    s, kind = state, state["kind"]
    if own:
        return _run_own(s)
    if kind == "attn":
        return _attn_plain(s)
    if kind == "rotary":
        pos = _positions(s, s["q"].shape[1], None)
        return _turn_plain(s, s["q"], pos), _turn_plain(s, s["k"], pos)
    if kind == "commit":
        b, at = torch.arange(s["lens0"].shape[0], device=_DEV)[:, None], s["nodes"].long().clamp(min=0)
        _put_plain(s, s["draft_k"][b, at], s["draft_v"][b, at])
    else:
        _put_plain(s, _turn_plain(s, s["k"], _positions(s, s["k"].shape[1], s["lens0"])), s["v"])
    return _cache(s)


# ------------------------------------------------------------------------- 64-bit answer
def _exact_attn(s):
    q, B, N = s["q"], s["q"].shape[0], s["q"].shape[1]
    Hq, D, H = q.shape[2], q.shape[3], s["draft_k"].shape[2]
    G, lens, page, table = Hq // H, s["seq_lens"].tolist(), s["page"], s["table"].tolist()
    words = s["mask"].cpu().numpy().view(np.uint8).reshape(B, N, -1)
    see = torch.from_numpy(np.unpackbits(words, axis=2, bitorder="little")[:, :, :N].astype(bool)).to(_DEV)
    out = torch.empty(q.shape, dtype=torch.float64, device=_DEV)
    for b in range(B):
        L = lens[b]
        used = table[b][:-(-L // page)]
        hide = ~see[b].repeat_interleave(G, 0)
        for c in range(H):
            k = torch.cat([s["k_pages"][used, :, c].reshape(-1, D)[:L].double(), s["draft_k"][b, :, c].double()])
            v = torch.cat([s["v_pages"][used, :, c].reshape(-1, D)[:L].double(), s["draft_v"][b, :, c].double()])
            x = q[b, :, c * G:(c + 1) * G].reshape(N * G, D).double() @ k.T
            x *= D ** -0.5
            x[:, L:].masked_fill_(hide, -math.inf)
            out[b, :, c * G:(c + 1) * G] = (torch.softmax(x, 1) @ v).view(N, G, D)
    return out


def _exact_turn(s, x, pos):
    """Each pair of columns as a complex number times exp(i angle)."""
    n = s["freqs"].shape[0]
    out = x.double()
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if s["pairs"] else (i, i + n)
        z = torch.complex(out[..., a], out[..., b])
        z *= torch.polar(torch.ones(1, dtype=torch.float64, device=_DEV), pos[s["axes"][i]].double() * float(s["freqs"][i]))[:, :, None]
        out[..., a], out[..., b] = z.real, z.imag
    return out


def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    if kind == "attn":
        return _exact_attn(s)
    if kind == "rotary":
        pos = s["positions"].long() + s["offsets"].long()[:, None]
        return _exact_turn(s, s["q"], pos), _exact_turn(s, s["k"], pos)
    lens, count, page, table = s["lens0"].tolist(), s["count"].tolist(), s["page"], s["table"].tolist()
    if kind == "commit":
        k, v = s["draft_k"].double(), s["draft_v"].double()
        rows = [s["nodes"][b, :count[b]].tolist() for b in range(case["B"])]
    else:
        if s["positions"] is None:
            pos = torch.tensor([[n + t for t in range(case["T"])] for n in lens], device=_DEV)[None]
        else:
            pos = s["positions"].long() + s["offsets"].long()[:, None]
        k, v = _exact_turn(s, s["k"], pos), s["v"].double()
        rows = [list(range(n)) for n in count]
    K, V = s["k_pages"].double(), s["v_pages"].double()
    for b, src in enumerate(rows):
        at = 0
        while at < len(src):                    # page by page
            j = lens[b] + at
            n = min(len(src) - at, page - j % page)
            p = table[b][j // page]
            K[p, j % page:j % page + n] = k[b, src[at:at + n]]
            V[p, j % page:j % page + n] = v[b, src[at:at + n]]
            at += n
    return dict(k_pages=K, v_pages=V, seq_lens=None)


def work(case):
    c, kind, B = case, case["kind"], case["B"]
    if kind == "rotary":
        n = B * c["N"] * (c["Hq"] + c["Hkv"]) * float(c["D"])
        return {"bytes": 4.0 * n + 4.0 * B * c["N"], "flops": 3.0 * n * c["R"] / c["D"]}
    row = c["Hkv"] * c["D"]
    if kind == "attn":
        L, N = (c["Lmin"] + c["Lmax"]) / 2, c["N"]
        rows = B * (L - c["shared"]) + c["shared"]
        nbytes = 2 * B * N * c["Hq"] * c["D"] * 2 + 4 * rows * row + 2 * B * N * row * 2 + B * N * ((N + 31) // 32) * 4
        return {"bytes": float(nbytes), "flops": 4.0 * B * N * c["Hq"] * c["D"] * (L + max(c["depth"], 1))}
    n = B * ((1 if kind == "commit" else c["Tmin"]) + c["T"]) / 2
    return {"bytes": 8.0 * n * row + 8.0 * B, "flops": 0.0 if kind == "commit" else 3.0 * n * c["Hkv"] * c["R"]}
