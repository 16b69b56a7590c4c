"""The operators of a cached attention layer, as timed cases.

A video transformer that makes its frames in chunks keeps the keys and values
of the frames it has made.  Per layer and chunk it rotates the new queries and
keys by their (time, height, width) position, writes the new keys and values
into the cache (8-bit codes, one scale per block of tokens and head) and
attends from the new queries to what the cache holds, over all blocks or over
lists of kept blocks.  The same calls serve single tokens.

Kinds of a case:
  rope    rotation of one tensor of a layer, forward ("bwd": false) or the
          gradient with respect to its input, between the projection's
          token-major layout and the attention's head-major one
  write   quantisation of new keys and values into the cache
  read    what a stretch of the cache stands for, in bf16
  attn    attention of new queries over the cache
"""
import math

import torch

own = False   # False: plain torch operations; True: the framework's calls

DEVICE = "cuda"
E4M3, INT8 = "e4m3", "int8"


def _rope(B, H, L, d, dims, grid, theta, halves=False, bwd=False, text=0, first=0, ragged=False, name=None):
    """L tokens, the last `text` of them text, from position `first` of a video
    of grid = (frames, height, width); ragged: another start per sequence."""
    return _named(dict(kind="rope", B=B, H=H, L=L, d=d, d_t=dims[0], d_h=dims[1], d_w=dims[2], frames=grid[0],
                       height=grid[1], width=grid[2], theta=float(theta), halves=halves, bwd=bwd, text=text,
                       first=first, ragged=ragged), name)


def _store(kind, fmt, B, H, L, d, block, capacity, first, ragged=False, name=None):
    """write/read of L tokens from position `first` (ragged: other starts and
    fewer tokens in the later sequences)."""
    return _named(dict(kind=kind, fmt=fmt, B=B, H=H, L=L, d=d, block=block, capacity=capacity, first=first,
                       ragged=ragged), name)


def _attn(fmt, B, Hq, H, Lq, length, d, block, density=1.0, lists=False, ragged=False, name=None):
    """Lq queries of Hq heads over `length` cached tokens of H heads; lists:
    every query block keeps ceil(density * n) of the n blocks."""
    return _named(dict(kind="attn", fmt=fmt, B=B, Hq=Hq, H=H, Lq=Lq, length=length, d=d, block=block,
                       density=density, lists=lists, ragged=ragged), name)


def _named(c, name):
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # One new token of a toy layer, far into the video: latency alone.
        _rope(1, 2, 1, 64, (16, 24, 24), (64, 16, 16), 10000, first=15 * 1000 + 7, name="rope-token"),
        # The gradient of a training step's keys: 64-wide heads, two sequences
        # with a text segment (30 heads, 23 frames of 32 x 40, 226 text tokens).
        _rope(2, 30, 23 * 1280 + 226, 64, (16, 24, 24), (23, 32, 40), 10000, halves=True, bwd=True, text=226,
              name="rope-text-bwd"),
        # All queries of a Wan-shaped 720p layer (40 heads, 21 frames of
        # 45 x 80), axis widths that no 16-byte chunk divides.
        _rope(1, 40, 21 * 3600, 128, (44, 42, 42), (21, 45, 80), 10000, name="rope-720p"),
        # One new token for each of eight sequences of different lengths.
        _store("write", INT8, 8, 24, 1, 128, 128, 8192, 5000, ragged=True, name="write-token"),
        # One latent frame behind seventeen others, HunyuanVideo-shaped (24
        # heads): it starts and ends inside a block.
        _store("write", E4M3, 1, 24, 3600, 128, 128, 33 * 3600, 17 * 3600, name="write-frame"),
        # A whole 720p sequence at once (33 frames).
        _store("write", INT8, 1, 24, 33 * 3600, 128, 128, 33 * 3600, 0, name="write-720p"),
        # A stretch of odd length of two sequences, 64-wide heads and blocks.
        _store("read", INT8, 2, 8, 1537, 64, 64, 4096, 701, ragged=True, name="read-window"),
        # A whole Wan-shaped sequence (40 heads, 75,600 tokens).
        _store("read", E4M3, 1, 40, 21 * 3600, 128, 128, 21 * 3600, 0, name="read-720p"),
        # One query over a thousand tokens of a toy layer: latency alone.
        _attn(E4M3, 1, 2, 2, 1, 1000, 64, 64, name="attn-token-small"),
        # One query per sequence over long caches of different lengths, four
        # query heads to a key/value head.
        _attn(INT8, 4, 32, 8, 1, 32768, 128, 128, ragged=True, name="attn-token-long"),
        # One latent frame against 33 frames over lists that keep a quarter of
        # the blocks (24 heads).
        _attn(E4M3, 1, 24, 24, 3600, 33 * 3600, 128, 128, 0.25, lists=True, name="attn-frame-lists"),
        # A chunk of three latent frames against all 33 frames.
        _attn(INT8, 1, 24, 24, 3 * 3600, 33 * 3600, 128, 128, name="attn-chunk-dense"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case of these ranges: both head widths, block sizes and
    formats, one token to whole 720p sequences, aligned or not; no dearer than
    the dearest listed case of its kind."""
    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"]] = [max(a, b) for a, b in zip(most.get(c["kind"], (0, 0)), (w["bytes"], w["flops"]))]
    while True:
        kind = rng.choice(["rope", "write", "read", "attn", "attn", "attn"])
        d, block, fmt = rng.choice([64, 128, 128]), rng.choice([64, 128, 128]), rng.choice([E4M3, INT8])
        B, H = rng.choice([1, 1, 2, rng.randint(3, 8)]), _log(rng, 1, 40)
        ragged = B > 1 and rng.random() < 0.7
        if kind == "rope":
            dims = [2 * rng.randint(2, d // 6) for _ in range(2)]
            dims.append(d - sum(dims) - 2 * rng.choice([0, 0, rng.randint(0, 4)]))
            grid = (rng.randint(1, 64), rng.randint(4, 64), rng.randint(4, 80))
            total = grid[0] * grid[1] * grid[2]
            if total < 8:
                continue
            Lv = _log(rng, 1, total)
            text = rng.choice([0, 0, rng.randint(1, 512)])
            c = _rope(B, H, Lv + text, d, dims, grid, rng.choice([256, 10000, 1000000]), rng.random() < 0.5,
                      rng.random() < 0.5, text, rng.randint(0, total - Lv), ragged)
        elif kind in ("write", "read"):
            capacity = _log(rng, 64, 33 * 3600)
            L = _log(rng, 1, capacity)
            c = _store(kind, fmt, B, H, L, d, block, capacity, rng.randint(0, capacity - L), ragged)
        else:
            group = rng.choice([1, 1, 2, 4, 8])
            length, Lq = _log(rng, 1, 33 * 3600), rng.choice([1, _log(rng, 1, 64), _log(rng, 64, 3 * 3600)])
            lists = rng.random() < 0.5
            c = _attn(fmt, B, H * group, H, Lq, length, d, block, round(rng.uniform(0.05, 0.6), 3) if lists else 1.0,
                      lists, ragged)
            if B * H * group > 128:
                continue
        w = work(c)
        if w["bytes"] <= most[kind][0] and w["flops"] <= most[kind][1]:
            return c


# ---------------------------------------------------------------- sizes of a case

def _offsets(c):
    """Per sequence its start less `first`, and its number of tokens."""
    B, L = c["B"], c["L"]
    if not c["ragged"]:
        return [0] * B, [L] * B
    room = c["frames"] * c["height"] * c["width"] if c["kind"] == "rope" else c["capacity"]
    room -= c["first"] + L - c.get("text", 0)
    starts = [min(room, 37 * b) for b in range(B)]
    counts = [L if c["kind"] == "rope" else L - (L * b) // (2 * B) for b in range(B)]
    return starts, counts


def _lengths(c):
    """Cached tokens per sequence."""
    return [max(1, c["length"] - c["length"] * b // (2 * c["B"])) if c["ragged"] else c["length"]
            for b in range(c["B"])]


def _kept(c):
    n = -(-c["length"] // c["block"])
    return max(1, min(n, math.ceil(c["density"] * n))) if c["lists"] else n


def work(case):
    c, d = case, case["d"]
    if c["kind"] == "rope":
        values = c["B"] * c["H"] * c["L"] * d
        tables = 4 * (c["frames"] * c["d_t"] + c["height"] * c["d_h"] + c["width"] * c["d_w"])
        return {"bytes": 4 * values + min(tables, 4 * c["B"] * c["L"] * d), "flops": 3 * values}
    if c["kind"] in ("write", "read"):
        tokens = sum(_offsets(c)[1])
        return {"bytes": c["H"] * (tokens * 2 * d * 3 + (tokens / c["block"] + c["B"]) * 8),
                "flops": 2 * c["H"] * tokens * d * (2 if c["kind"] == "write" else 1)}
    n, nq, block = -(-c["length"] // c["block"]), -(-c["Lq"] // c["block"]), c["block"]
    share = _kept(c) / n                                    # of a row's keys
    # blocks that some row of a head reads
    touched = min(1.0, share * nq * (c["Hq"] // c["H"]))
    keys = sum(_lengths(c))
    lists = 4 * c["B"] * c["Hq"] * nq * (_kept(c) + 1) if c["lists"] else 0
    return {"bytes": c["H"] * touched * keys * (2 * d + 8 / block) + c["B"] * c["Hq"] * c["Lq"] * (4 * d + 4) + lists,
            "flops": 4 * d * c["Hq"] * c["Lq"] * share * keys}


# ---------------------------------------------------------------- inputs

def _values(shape, gen, spread=True):
    """Activations of a head: unit noise with a few channels that are much
    larger, as keys and values have them."""
    x = torch.randn(shape, device=DEVICE, generator=gen)
    if spread:
        wide = 1.0 + 5.0 * (torch.rand(shape[-1], device=DEVICE, generator=gen) < 0.04)
        x *= wide
    return x.bfloat16()


def _codes(shape, fmt, gen):
    """Codes of a filled cache and the scales of its blocks."""
    x = torch.randn(shape, device=DEVICE, generator=gen)
    if fmt == INT8:
        return (x * 28).round_().clamp_(-127, 127).to(torch.int8).view(torch.uint8)
    return (x * 100).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _scales(shape, fmt, gen):
    e = torch.randint(-9 if fmt == E4M3 else -7, -6 if fmt == E4M3 else -4, shape, device=DEVICE, generator=gen)
    s = torch.exp2(e.float())
    return s if fmt == E4M3 else s * (1 + torch.rand(shape, device=DEVICE, generator=gen))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    c, kind, d, B, H = case, case["kind"], case["d"], case["B"], case["H"]
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    st = {"c": c}
    if kind == "rope":
        L = c["L"]
        tokens = _values((B, L, H, d), gen, False).transpose(1, 2)        # as a projection leaves it
        heads = torch.empty((B, H, L, d), dtype=torch.bfloat16, device=DEVICE)
        if c["bwd"]:   # the gradient comes in the attention's layout and leaves in the projection's
            st["x"], st["y"] = heads.copy_(tokens), torch.empty_like(tokens)
        else:
            st["x"], st["y"] = tokens, heads
        st["starts"] = _ints(_offsets(c)[0]) if c["ragged"] else None
        if own:
            import paper_2601_11641_amd as M
            st["shape"] = M.make_shape(B, H, L, d, 128, c["height"] * c["width"], c["text"])
            st["rope"] = M.Rope(M.make_rope_params(d, (c["d_t"], c["d_h"], c["d_w"]),
                                                   (c["frames"], c["height"], c["width"]), c["theta"],
                                                   "halves" if c["halves"] else "adjacent"))
        return st
    capacity = c["capacity"] if kind != "attn" else c["length"]
    n = -(-capacity // c["block"])
    for name in ("k", "v"):
        st[name + "8"] = _codes((B, H, capacity, d), c["fmt"], gen)
        st[name + "s"] = _scales((B, H, n), c["fmt"], gen)
    if own:
        import paper_2601_11641_amd as M
        st["shape"] = M.make_cache_shape(B, H, capacity, d, c["block"], c["fmt"])
        st["cache"] = M.make_cache(st["k8"], st["v8"], st["ks"], st["vs"])
    if kind == "attn":
        Lq, Hq, nq = c["Lq"], c["Hq"], -(-c["Lq"] // c["block"])
        # queries lean towards the last keys, their own
        st["q"] = torch.randn((B, Hq, Lq, d), device=DEVICE, generator=gen).bfloat16()
        at = torch.arange(Lq, device=DEVICE) % capacity
        at = capacity - 1 - at.flip(0)
        lean = _decode(st["k8"], c["fmt"])[:, :, at] * st["ks"][:, :, at // c["block"], None]
        st["q"] += 0.25 * lean.repeat_interleave(Hq // H, 1).bfloat16()
        del lean
        st["o"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty((B, Hq, Lq), dtype=torch.float32, device=DEVICE)
        st["len"] = _ints(_lengths(c)) if c["ragged"] else None
        st["idx"] = st["cnt"] = None
        if c["lists"]:
            keep = _kept(c)
            order = torch.rand((B, Hq, nq, n), device=DEVICE, generator=gen).argsort(-1)[..., :keep]
            st["idx"] = torch.full((B, Hq, nq, n), -1, dtype=torch.int32, device=DEVICE)
            st["idx"][..., :keep] = order.sort(-1)[0].int()
            st["cnt"] = torch.full((B, Hq, nq), keep, dtype=torch.int32, device=DEVICE)
        if own:
            st["ws_bytes"] = M.mod_cache_attn_workspace_bytes(st["shape"], Hq, Lq, c["length"])
            st["ws"] = torch.empty(max(1, st["ws_bytes"]), dtype=torch.uint8, device=DEVICE)
        return st
    L = c["L"]
    starts, counts = _offsets(c)
    st["starts"], st["counts"] = (_ints(starts), _ints(counts)) if c["ragged"] else (None, None)
    if kind == "write":
        st["k"] = _values((B, H, L, d), gen)                               # rotated: head-major
        st["v"] = _values((B, L, H, d), gen).transpose(1, 2)               # from the projection: token-major
    else:
        st["k"] = torch.zeros((B, H, L, d), dtype=torch.bfloat16, device=DEVICE)
        st["v"] = torch.zeros_like(st["k"])
    return st


# ---------------------------------------------------------------- one pass

def _as_values(codes, fmt):
    """The codes as the numbers they are."""
    return codes.view(torch.int8 if fmt == INT8 else torch.float8_e4m3fn)


def run(st):
    c, kind = st["c"], st["c"]["kind"]
    if kind == "rope":
        if own:
            import paper_2601_11641_amd as M
            call = M.mod_rope_bwd if c["bwd"] else M.mod_rope_fwd
            call(st["rope"].handle, st["shape"], st["x"], st["y"], c["first"], st["starts"])
        else:
            _plain_rope(st)
        return st["y"]
    if kind == "attn":
        if own:
            import paper_2601_11641_amd as M
            M.mod_cache_attn_fwd(st["shape"], st["cache"], st["q"], c["length"], st["len"], st["idx"], st["cnt"], 0.0,
                                 st["o"], st["lse"], st["ws"], st["ws_bytes"])
            return {"o": st["o"], "lse": st["lse"]}
        return _plain_attn(st)
    if own:
        import paper_2601_11641_amd as M
        call = M.mod_cache_write if kind == "write" else M.mod_cache_read
        call(st["shape"], st["cache"], st["k"], st["v"], c["first"], st["starts"], st["counts"])
    elif kind == "write":
        _plain_write(st, "k")
        _plain_write(st, "v")
    else:
        _plain_read(st, "k")
        _plain_read(st, "v")
    if kind == "read":
        return {"k": st["k"], "v": st["v"]}
    return {"k": _as_values(st["k8"], c["fmt"]), "v": _as_values(st["v8"], c["fmt"]), "ks": st["ks"], "vs": st["vs"]}


# ---------------------------------------------------------------- plain forms

def _angles(c, starts):
    """[B, video tokens, rotated pairs] in 64 bits: position along each axis
    times theta^(-2j / axis width)."""
    Lv = c["L"] - c["text"]
    pos = c["first"] + torch.arange(Lv, device=DEVICE)[None]
    if starts is not None:
        pos = pos + starts.long()[:, None]
    hw = c["height"] * c["width"]
    axes = (pos // hw, pos % hw // c["width"], pos % c["width"])
    out = []
    for p, w in zip(axes, (c["d_t"], c["d_h"], c["d_w"])):
        j = torch.arange(w // 2, device=DEVICE, dtype=torch.float64)
        out.append(p[..., None] * c["theta"] ** (-2 * j / w))
    return torch.cat(out, -1)


def _pairs(c):
    """Channels of the first and second member of every rotated pair."""
    first, second, at = [], [], 0
    for w in (c["d_t"], c["d_h"], c["d_w"]):
        j = torch.arange(w // 2, device=DEVICE)
        first.append(at + (j if c["halves"] else 2 * j))
        second.append(at + (j + w // 2 if c["halves"] else 2 * j + 1))
        at += w
    return torch.cat(first), torch.cat(second)


def _plain_rope(st):
    c, x, y = st["c"], st["x"], st["y"]
    Lv = c["L"] - c["text"]
    ang = _angles(c, st["starts"])[:, None]
    cos, sin = ang.cos().float(), ang.sin().float()
    if c["bwd"]:
        sin = -sin
    a, b = _pairs(c)
    x0, x1 = x[:, :, :Lv, a].float(), x[:, :, :Lv, b].float()
    y.copy_(x)
    y[:, :, :Lv, a] = (x0 * cos - x1 * sin).bfloat16()
    y[:, :, :Lv, b] = (x0 * sin + x1 * cos).bfloat16()


def _decode(codes, fmt):
    return _as_values(codes, fmt).float()


def _scale_of(amax, fmt):
    """The scale that a block's largest magnitude asks for (fp32); 0 for a
    block of zeros, NaN where a value is not finite."""
    if fmt == INT8:
        s = (amax.double() / 127).float()
    else:
        f, e = torch.frexp(amax)
        s = torch.exp2((e - 8 - (f <= 0.875).int()).float().clamp(min=-126))   # 448 = 0.875 * 2^9
    s = torch.where(amax > 0, s.clamp(min=2.0 ** -126), torch.zeros_like(s))
    return torch.where(amax.isfinite(), s, torch.full_like(s, math.nan))


def _encode(x, s, fmt):
    """RNE of x / s, the quotient in 64 bits (values next to a border)."""
    z = torch.where(s > 0, x.double() / s, torch.zeros((), dtype=torch.float64, device=DEVICE))
    if fmt == INT8:
        return z.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return z.float().to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_write(st, name):
    c, x, codes, scales = st["c"], st[name], st[name + "8"], st[name + "s"]
    B, H, L, d = x.shape
    block, fmt, n = c["block"], c["fmt"], scales.shape[2]
    start = torch.full((B,), c["first"], device=DEVICE)
    count = torch.full((B,), L, device=DEVICE)
    if c["ragged"]:
        start, count = start + st["starts"], st["counts"].long()
    live = torch.arange(L, device=DEVICE) < count[:, None]                                   # [B, L]
    pos = start[:, None] + torch.arange(L, device=DEVICE)
    blk = (pos // block)[:, None].expand(B, H, L)
    # the largest magnitude that each block receives; -1: none
    top = torch.where(live[:, None], x.abs().amax(-1).float(), torch.full((), -1.0, device=DEVICE))
    amax = torch.full((B, H, n), -1.0, device=DEVICE).scatter_reduce_(2, blk, top, "amax")
    block0 = torch.arange(n, device=DEVICE) * block
    goes_on = ((block0 < start[:, None]) & (block0 + block > start[:, None]))[:, None]       # holds earlier tokens
    s_new = torch.where(goes_on, torch.maximum(scales, _scale_of(amax, fmt)), _scale_of(amax, fmt))
    s_new = torch.where(amax >= 0, s_new, scales)
    # earlier tokens of a block that is continued, under its new scale
    b, r = torch.arange(B, device=DEVICE)[:, None], torch.arange(block, device=DEVICE)
    back = (start // block * block)[:, None] + r
    mine = (back < start[:, None]) & (count > 0)[:, None]
    back = back.clamp(max=codes.shape[2] - 1)
    held = codes[b, :, back]                                                                # [B, block, H, d]
    old, new = (t[b, :, back // block][..., None] for t in (scales, s_new))
    again = _encode(_decode(held, fmt).double() * old, new, fmt)
    codes[b, :, back] = torch.where((mine[..., None, None]) & (old != new), again, held)
    bi, li = live.nonzero(as_tuple=True)
    codes[bi, :, pos[bi, li]] = _encode(x[bi, :, li], s_new[bi, :, pos[bi, li] // block][..., None], fmt)
    scales.copy_(s_new)


def _plain_read(st, name):
    c, out, codes, scales = st["c"], st[name], st[name + "8"], st[name + "s"]
    B, H, L, d = out.shape
    pos = c["first"] + torch.arange(L, device=DEVICE)[None].expand(B, L)
    live = torch.ones((B, L), dtype=torch.bool, device=DEVICE)
    if c["ragged"]:
        pos, live = pos + st["starts"][:, None], torch.arange(L, device=DEVICE) < st["counts"][:, None]
    b = torch.arange(B, device=DEVICE)[:, None]
    held = _decode(codes[b, :, pos], c["fmt"]) * scales[b, :, pos // c["block"]][..., None]   # [B, L, H, d]
    out.copy_(torch.where(live[:, None, :, None], held.bfloat16().transpose(1, 2), out))


def _plain_attn(st):
    c, q = st["c"], st["q"]
    B, Hq, Lq, d = q.shape
    H, block, length, fmt = c["H"], c["block"], c["length"], c["fmt"]
    n, nq, keep = -(-length // block), -(-Lq // block), _kept(c)
    pad, padq = n * block - length, nq * block - Lq
    o, lse = st["o"].view(B * Hq, Lq, d), st["lse"].view(B * Hq, Lq)
    # as many heads at once as 3e9 scores allow
    width = keep * block if c["lists"] else length
    step = max(1, int(3e9 // (width * nq * block)))
    for h0 in range(0, B * Hq, step):
        h = torch.arange(h0, min(B * Hq, h0 + step), device=DEVICE)
        kv, b = h // Hq * H + h % Hq // (Hq // H), h // Hq
        k, v = (_decode(st[t + "8"].view(B * H, length, d)[kv], fmt) for t in ("k", "v"))
        ks, vs = (st[t].view(B * H, n)[kv].repeat_interleave(block, 1)[:, :length, None] for t in ("ks", "vs"))
        k, v = k.mul_(ks), v.mul_(vs)
        x = q.view(B * Hq, Lq, d)[h].float() / math.sqrt(d)
        m = h.numel()
        if c["lists"]:
            k, v = (torch.nn.functional.pad(t, (0, 0, 0, pad)).view(m, n, block, d) for t in (k, v))
            at = st["idx"].view(B * Hq, nq, n)[h, :, :keep].long()                           # [m, nq, keep]
            k, v = (t[torch.arange(m, device=DEVICE)[:, None, None], at].view(m * nq, keep * block, d) for t in (k, v))
            x = torch.nn.functional.pad(x, (0, 0, 0, padq)).view(m * nq, block, d)
            pos = (at[..., None] * block + torch.arange(block, device=DEVICE)).view(m, nq, 1, width)
        else:
            pos = torch.arange(length, device=DEVICE).view(1, 1, 1, -1)
        s = torch.bmm(x, k.transpose(1, 2).contiguous())
        if st["len"] is not None or c["lists"]:
            end = st["len"][b].view(m, 1, 1, 1) if st["len"] is not None else length
            s.view(m, nq if c["lists"] else 1, -1, width).masked_fill_(pos >= end, -math.inf)
        top = s.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = s.sub_(top).exp_()
        l = p.sum(-1, keepdim=True)
        y = torch.bmm(p, v) / torch.where(l > 0, l, torch.ones_like(l))
        o[h] = y.view(m, -1, d)[:, :Lq].bfloat16()
        lse[h] = (top + l.log()).view(m, -1)[:, :Lq]
    return {"o": st["o"], "lse": st["lse"]}


# ---------------------------------------------------------------- 64-bit values

def exact(case, seed):
    """What run() returns, from the definitions in 64 bits, sequence by
    sequence; codes of 8-bit integers are whole numbers and have to be equal."""
    st = prepare(case, seed)
    return {"rope": _rope64, "write": _write64, "read": _read64, "attn": _attn64}[case["kind"]](case, st)


def _number(codes, fmt):
    """The number that each code is: an 8-bit integer, or sign, 4 bits of
    exponent (bias 7) and 3 of fraction."""
    i = codes.long()
    if fmt == INT8:
        return (i - 256 * (i > 127)).double()
    e, f = (i >> 3) & 15, (i & 7).double()
    size = torch.where(e > 0, (1 + f / 8) * torch.exp2(e.double() - 7), f / 512)
    return torch.where(i > 127, -size, size)


def _rope64(c, st):
    x = st["x"]
    out = x.double()
    starts = _offsets(c)[0]
    for b in range(c["B"]):
        pos = starts[b] + c["first"] + torch.arange(c["L"] - c["text"], device=DEVICE)
        y = torch.div(pos, c["width"], rounding_mode="floor")
        place = {"d_t": y // c["height"], "d_h": y % c["height"], "d_w": pos - y * c["width"]}
        at = 0
        for axis in ("d_t", "d_h", "d_w"):
            for j in range(c[axis] // 2):
                i0, i1 = (at + j, at + j + c[axis] // 2) if c["halves"] else (at + 2 * j, at + 2 * j + 1)
                turn = torch.polar(torch.ones(len(pos), device=DEVICE, dtype=torch.float64),
                                   place[axis].double() * math.exp(-2 * j / c[axis] * math.log(c["theta"])))
                z = torch.complex(x[b, :, :len(pos), i0].double(), x[b, :, :len(pos), i1].double())
                z = z * (turn.conj() if c["bwd"] else turn)
                out[b, :, :len(pos), i0], out[b, :, :len(pos), i1] = z.real, z.imag
            at += c[axis]
    return out


def _write64(c, st):
    starts, counts = _offsets(c)
    block, fmt, res = c["block"], c["fmt"], {}
    for name in ("k", "v"):
        value, scale = _number(st[name + "8"], fmt), st[name + "s"].double()
        for b in range(c["B"]):
            p0 = c["first"] + starts[b]
            p1 = p0 + counts[b]
            for j in range(p0 // block, -(-p1 // block)) if p1 > p0 else ():
                lo, hi = max(p0, j * block), min(p1, (j + 1) * block)
                x = st[name][b, :, lo - p0:hi - p0].double()
                amax = x.abs().amax((1, 2))
                if fmt == INT8:
                    s = (amax / 127).float().double()
                else:
                    s = torch.exp2(torch.ceil(torch.log2(amax / 448)))
                s = torch.where(amax > 0, s.clamp(min=2.0 ** -126), 0 * s)
                if lo > j * block:
                    was = scale[b, :, j].clone()
                    s = torch.maximum(s, was)
                    held = value[b, :, j * block:lo]
                    value[b, :, j * block:lo] = torch.where((s != was)[:, None, None],
                                                            _nearest(held * was[:, None, None], s, fmt), held)
                scale[b, :, j] = s
                value[b, :, lo:hi] = _nearest(x, s, fmt)
        res[name] = value if fmt == E4M3 else value.long()
        res[name + "s"] = scale
    return res


def _nearest(x, s, fmt):
    """The number of the format nearest to x / s, ties to the even one."""
    z = x / torch.where(s > 0, s, torch.ones_like(s))[:, None, None]
    if fmt == INT8:
        return torch.round(z).clamp(-127, 127)
    # spacing of the numbers around |z|: 2^(floor(log2 |z|) - 3), 2^-9 below 2^-6
    gap = torch.exp2((torch.frexp(z)[1] - 1).clamp(min=-6).double() - 3)
    return (torch.round(z / gap) * gap).clamp(-448, 448)


def _read64(c, st):
    starts, counts = _offsets(c)
    res = {}
    for name in ("k", "v"):
        out = st[name].double()
        for b in range(c["B"]):
            p = c["first"] + starts[b] + torch.arange(counts[b], device=DEVICE)
            out[b, :, :counts[b]] = (_number(st[name + "8"][b, :, p], c["fmt"]) *
                                     st[name + "s"][b].double()[:, p // c["block"], None])
        res[name] = out
    return res


def _attn64(c, st):
    B, Hq, H, Lq, block, d = c["B"], c["Hq"], c["H"], c["Lq"], c["block"], c["d"]
    o = torch.zeros((B, Hq, Lq, d), dtype=torch.float64, device=DEVICE)
    lse = torch.full((B, Hq, Lq), -math.inf, dtype=torch.float64, device=DEVICE)
    lengths = _lengths(c)
    for b in range(B):
        place = torch.arange(lengths[b], device=DEVICE)
        for h in range(Hq):
            g = h * H // Hq
            if h * H % Hq == 0:
                k = _number(st["k8"][b, g, :lengths[b]], c["fmt"]) * st["ks"][b, g].double()[place // block, None]
                v = _number(st["v8"][b, g, :lengths[b]], c["fmt"]) * st["vs"][b, g].double()[place // block, None]
                kt = k.t().contiguous()
            for i in range(0, Lq, block) if c["lists"] else range(0, Lq, 3600):
                q = st["q"][b, h, i:i + (block if c["lists"] else 3600)].double()
                keys, kk, vv = q.shape[0], kt, v
                if c["lists"]:
                    js = st["idx"][b, h, i // block, :_kept(c)].long()
                    at = (js[:, None] * block + torch.arange(block, device=DEVICE)).reshape(-1)
                    at = at[at < lengths[b]]
                    kk, vv = k[at].t().contiguous(), v[at]
                    if not at.numel():
                        continue
                z = (q @ kk) * d ** -0.5
                total = torch.logsumexp(z, 1)
                o[b, h, i:i + keys] = torch.exp_(z.sub_(total[:, None])) @ vv
                lse[b, h, i:i + keys] = total
    return {"o": o, "lse": lse}
