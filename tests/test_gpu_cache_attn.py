"""Attention over the 8-bit cache against the definition in 64 bits."""
import math

import pytest
import torch

import cached_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import paper_2601_11641_amd as m
    return m


class Filled:
    """A cache with arbitrary codes and scales; nothing behind a sequence's
    end or in blocks past it is a number."""

    def __init__(self, M, B, H, cap, d, block, fmt, lens, seed=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.M, self.B, self.H, self.cap, self.d, self.block, self.fmt, self.lens = M, B, H, cap, d, block, fmt, lens
        self.shape = M.make_cache_shape(B, H, cap, d, block, fmt)
        n = -(-cap // block)
        self.codes, self.scales = [], []
        for t in range(2):
            x = torch.randn((B, H, cap, d), generator=g)
            if fmt == R.INT8:
                c = (x * 40).round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
                s = (0.5 + torch.rand((B, H, n), generator=g)) * (spread if t == 0 else 1.0) / 40
            else:
                c = (x * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                s = torch.exp2(torch.randint(-8, -5, (B, H, n), generator=g).float()) * (spread if t == 0 else 1.0)
            for b in range(B):
                c[b, :, lens[b]:] = 0x7f                       # e4m3: NaN; int8: the largest
                s[b, :, -(-lens[b] // block):] = math.nan
            self.codes.append(c)
            self.scales.append(s)
        self.dev = [t.cuda() for t in self.codes + self.scales]
        self.ref = M.make_cache(*self.dev)
        k, v = (R.dequant_by(c, s, fmt, block) for c, s in zip(self.codes, self.scales))
        self.kv = (k, v)

    def lists(self, Hq, nq, max_len, seed, keep=0.5):
        """Kept blocks per row, some rows empty, in any order, with entries
        that have to be skipped among them."""
        g = torch.Generator().manual_seed(seed)
        n = -(-max_len // self.block)
        idx = torch.randint(-2 ** 31, 2 ** 31 - 1, (self.B, Hq, nq, n), generator=g).int()
        cnt = torch.zeros((self.B, Hq, nq), dtype=torch.int32)
        kept = []
        for b in range(self.B):
            kept.append([])
            for h in range(Hq):
                kept[-1].append([])
                for i in range(nq):
                    js = torch.randperm(n, generator=g)
                    js = js[torch.rand(n, generator=g) < (0.0 if (h + i) % 5 == 4 else keep)].tolist()
                    row = list(js)
                    if len(row) < n and (h + i) % 3 == 0:
                        row.insert(len(row) // 2, [-1, n, 2 ** 31 - 1][i % 3])
                    idx[b, h, i, :len(row)] = torch.tensor(row, dtype=torch.int32)
                    cnt[b, h, i] = len(row)
                    kept[-1][-1].append(js)
        return idx, cnt, kept

    def run(self, q, max_len, kv_len=None, idx=None, cnt=None, scale=0.0, stream=None, workspace=None):
        B, Hq, Lq, d = q.shape
        o = torch.full(q.shape, 7.0, dtype=torch.bfloat16).cuda()
        lse = torch.full((B, Hq, Lq), 7.0).cuda()
        args = [None if t is None else t.cuda() for t in (kv_len, idx, cnt)]
        self.M.mod_cache_attn_fwd(self.shape, self.ref, q.cuda(), max_len, *args, scale, o, lse, workspace,
                                  0 if workspace is None else workspace.numel(), stream)
        return o, lse


def check(f, q, o, lse, lens, scale, kept=None, lost=None):
    """lost: what fp32 does not hold of an output."""
    want, wl, eo, el = R.attention(q, *f.kv, lens, f.block, scale, kept)
    eo = eo if lost is None else eo + lost
    o, lse = o.cpu().double(), lse.cpu().double()
    assert torch.equal(lse == -math.inf, wl == -math.inf)
    none = wl == -math.inf
    assert torch.all(o[none] == 0)
    assert torch.all(((lse - wl).abs() <= el)[~none]), ((lse - wl).abs() / el)[~none].max()
    assert torch.all(((o - want).abs() <= eo)[~none]), ((o - want).abs() / eo.clamp(min=1e-30))[~none].max()


def queries(B, Hq, Lq, d, seed, amp=1.0):
    return (amp * torch.randn((B, Hq, Lq, d), generator=torch.Generator().manual_seed(seed))).bfloat16()


FORMS = [(d, block, fmt) for d in (64, 128) for block in (64, 128) for fmt in (R.E4M3, R.INT8)]


@pytest.mark.parametrize("d,block,fmt", FORMS)
@pytest.mark.parametrize("Lq", [1, 3, 16, 17, 40, 65, 130])
def test_all_blocks(M, d, block, fmt, Lq):
    """Grouped heads, sequences of different lengths: none, one token, inside
    and at the ends of steps and blocks."""
    lens = [0, 1, 31, 32, 33, 128, 200, 300]
    f = Filled(M, 8, 2, 300, d, block, fmt, lens, seed=Lq)
    q = queries(8, 4, Lq, d, Lq)
    o, lse = f.run(q, 300, torch.tensor(lens, dtype=torch.int32))
    check(f, q, o, lse, lens, d ** -0.5)


@pytest.mark.parametrize("d,block,fmt", FORMS)
@pytest.mark.parametrize("Lq", [1, 20, 64, 129, 300])
def test_lists(M, d, block, fmt, Lq):
    lens = [500, 333, 7]
    f = Filled(M, 3, 2, 500, d, block, fmt, lens, seed=Lq)
    q = queries(3, 4, Lq, d, Lq + 1)
    idx, cnt, kept = f.lists(4, -(-Lq // block), 500, Lq)
    o, lse = f.run(q, 500, torch.tensor(lens, dtype=torch.int32), idx, cnt, 0.3)
    check(f, q, o, lse, lens, 0.3, kept)


@pytest.mark.parametrize("Lq,Hq,lists", [(1, 2, False), (1, 16, False), (5, 2, True), (40, 8, False), (200, 2, False),
                                         (200, 2, True), (700, 2, True)])
@pytest.mark.parametrize("d,fmt", [(128, R.INT8), (64, R.E4M3)])
def test_long_walks_are_split(M, Lq, Hq, lists, d, fmt):
    """Few rows over a long cache: parts of a walk, joined; keys whose scores
    grow along it, so that the running maximum moves."""
    cap, block = 9001, 128
    f = Filled(M, 1, 2, cap, d, block, fmt, [cap], seed=3, spread=2.0)
    q = queries(1, Hq, Lq, d, 5, 2.0)
    idx = cnt = kept = None
    if lists:
        idx, cnt, kept = f.lists(Hq, -(-Lq // block), cap, 9, 0.6)
    assert M.mod_cache_attn_workspace_bytes(f.shape, Hq, Lq, cap) > 0
    o, lse = f.run(q, cap, None, idx, cnt)
    check(f, q, o, lse, [cap], d ** -0.5, kept)
    again = f.run(q, cap, None, idx, cnt)
    assert torch.equal(again[0], o) and torch.equal(again[1], lse)


@pytest.mark.parametrize("Lq", [1, 70, 200])
def test_large_scores_and_empty_parts(M, Lq):
    """Scores up to a few hundred, and sequences much shorter than the cut-up
    length, which leave parts without a token."""
    lens, d, block = [40, 4000, 1, 0], 128, 64
    f = Filled(M, 4, 1, 4000, d, block, R.INT8, lens, seed=3, spread=12.0)
    q = queries(4, 2, Lq, d, 5, 3.0)
    o, lse = f.run(q, 4000, torch.tensor(lens, dtype=torch.int32))
    check(f, q, o, lse, lens, d ** -0.5)


def test_empty_cache_and_shorter_length(M):
    f = Filled(M, 2, 2, 200, 64, 64, R.E4M3, [150, 150])
    q = queries(2, 2, 5, 64, 1)
    o, lse = f.run(q, 0)
    assert torch.all(o == 0) and torch.all(lse == -math.inf)
    o, lse = f.run(q, 150)
    check(f, q, o, lse, [150, 150], 0.125)
    # lengths of the device past max_len and below zero
    o, lse = f.run(q, 100, torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32))
    check(f, q, o, lse, [100, 0], 0.125)


@pytest.mark.parametrize("Lq", [1, 150])
@pytest.mark.parametrize("lists", [False, True])
def test_infinities_and_nan(M, Lq, lists):
    """A NaN scale reaches the rows that read its block and no others; an
    infinite query gives NaN in its own row alone."""
    d, block, n = 128, 64, 6
    f = Filled(M, 1, 2, n * block, d, block, R.INT8, [n * block])
    q = queries(1, 2, Lq, d, 1)
    nq = -(-Lq // block)
    if not lists:
        o0, lse0 = f.run(q, n * block)
        q[0, 1, 0, 3] = math.inf
        o, lse = f.run(q, n * block)
        assert not o[0, 1, 0].isfinite().any() and lse[0, 1, 0].isnan()
        o[0, 1, 0], lse[0, 1, 0] = o0[0, 1, 0], lse0[0, 1, 0]
        assert torch.equal(o, o0) and torch.equal(lse, lse0)
        return
    for t in (2, 3):
        idx = torch.zeros((1, 2, nq, n), dtype=torch.int32)
        idx[0, 0] = torch.arange(n)
        idx[0, 1] = torch.tensor([0, 1, 3, 4, 5, 2])
        cnt = torch.tensor([6, 5], dtype=torch.int32).view(1, 2, 1).expand(1, 2, nq).contiguous()
        f.dev[t][0, :, 2] = math.nan           # block 2: head 0 reads it, head 1 does not
        o, lse = f.run(q, n * block, None, idx, cnt)
        assert o[0, 0].isnan().all() and o[0, 1].isfinite().all() and lse[0, 1].isfinite().all()
        assert lse[0, 0].isnan().all() == (t == 2)
        f.dev[t][0, :, 2] = 1.0


def test_offsets_past_32_bits(M):
    """A cache of 5 GB per tensor: its last head's last tokens, written, read
    and attended to over lists and over a long walk."""
    B, H, cap, d, block, L = 1, 5, 1 << 23, 128, 128, 300
    shape = M.make_cache_shape(B, H, cap, d, block, R.E4M3)
    c = M.Cache(shape)
    c.k.zero_()
    c.v.zero_()
    c.k_scale.zero_()
    c.v_scale.zero_()
    k, v = queries(B, H, L, d, 1), queries(B, H, L, d, 2)
    M.mod_cache_write(shape, c.ref, k.cuda(), v.cuda(), cap - L)
    kb, vb = torch.empty_like(k, device="cuda"), torch.empty_like(v, device="cuda")
    M.mod_cache_read(shape, c.ref, kb, vb, cap - L)
    kd, vd = kb.cpu().double(), vb.cpu().double()
    assert torch.all((kd - k.double()).abs() <= 2.0 ** -4 * k.double().abs() + 2.0 ** -9 * 2.0 ** -6)
    assert torch.all((vd - v.double()).abs() <= 2.0 ** -4 * v.double().abs() + 2.0 ** -9 * 2.0 ** -6)
    n, first = cap // block, (cap - L) // block
    q = queries(B, H, 2, d, 3)
    idx = torch.full((B, H, 1, n), -1, dtype=torch.int32)
    idx[..., :3] = torch.arange(first, first + 3)
    cnt = torch.full((B, H, 1), 3, dtype=torch.int32)
    o, lse = torch.empty_like(q, device="cuda"), torch.empty((B, H, 2)).cuda()
    M.mod_cache_attn_fwd(shape, c.ref, q.cuda(), cap, None, idx.cuda(), cnt.cuda(), 0.0, o, lse)
    at = 3 * block - L     # zero rows of the first listed block
    pad = torch.zeros((B, H, at, d), dtype=torch.float64)
    class F:
        kv = (torch.cat([pad, kd], 2), torch.cat([pad, vd], 2))
    F.block = block
    check(F, q, o, lse, [3 * block], d ** -0.5)
    # every token: the zeros in front have score 0
    M.mod_cache_attn_fwd(shape, c.ref, q.cuda(), cap, None, None, None, 0.0, o, lse)
    s = q.double() @ kd.transpose(2, 3) * d ** -0.5
    w = torch.exp(s)
    total = w.sum(-1) + (cap - L)
    want = (w @ vd) / total[..., None]
    assert torch.all((lse.cpu().double() - total.log()).abs() <= 1e-4)   # sums of 2^23 ones in parts: 2^-24 each step
    err = (o.cpu().double() - want).abs()
    assert torch.all(err <= 2 * R.BF16 * (want.abs() + (w @ vd.abs()) / total[..., None]) + 1e-4 * want.abs())


def test_other_stream_and_no_lse(M):
    f = Filled(M, 2, 2, 5000, 128, 128, R.INT8, [5000, 5000], seed=4)
    q = queries(2, 2, 1, 128, 2)
    o0, _ = f.run(q, 5000)
    qd, o = q.cuda(), torch.empty_like(q, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    M.mod_cache_attn_fwd(f.shape, f.ref, qd, 5000, None, None, None, 0.0, o, None, stream=side)
    trash = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")   # would take the workspace's place
    side.synchronize()
    assert torch.equal(o, o0) and trash[0] == 255
    # nor does it take memory that work of the current stream still writes
    need = M.mod_cache_attn_workspace_bytes(f.shape, 2, 1, 5000)
    assert need > 0
    for _ in range(3):
        big = torch.ones(4096, 4096, dtype=torch.bfloat16, device="cuda")
        held = torch.empty(need, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        for _ in range(8):
            big = big @ big
        held.fill_(255)
        del held
        M.mod_cache_attn_fwd(f.shape, f.ref, qd, 5000, None, None, None, 0.0, o, None, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(o, o0)


def test_captured_and_replayed(M):
    """A captured step over lengths of the device, in two graphs with a
    workspace each."""
    B, H, Hq, cap, d = 2, 2, 8, 4096, 128
    f = Filled(M, B, H, cap, d, 128, R.E4M3, [cap, cap], seed=5)
    need = M.mod_cache_attn_workspace_bytes(f.shape, Hq, 1, cap)
    assert need > 0
    states = []
    for s in range(2):
        q = queries(B, Hq, 1, d, s).cuda()
        st = dict(q=q, o=torch.empty_like(q), lse=torch.empty((B, Hq, 1)).cuda(),
                  len=torch.tensor([5, 7], dtype=torch.int32).cuda(),
                  ws=torch.full((need,), 255, dtype=torch.uint8).cuda(), g=torch.cuda.CUDAGraph())
        def call(st=st):
            M.mod_cache_attn_fwd(f.shape, f.ref, st["q"], cap, st["len"], None, None, 0.0, st["o"], st["lse"], st["ws"],
                                 need)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.synchronize()
        with torch.cuda.graph(st["g"]):
            call()
        states.append(st)
    for t in range(4):
        lens = [[5, 7], [4096, 1], [0, 3000], [129, 4000]][t]
        for s, st in enumerate(states):
            q = queries(B, Hq, 1, d, 10 * t + s)
            st["q"].copy_(q)
            st["len"].copy_(torch.tensor(lens, dtype=torch.int32))
            st["ref"] = f.run(q, cap, torch.tensor(lens, dtype=torch.int32))
        torch.cuda.synchronize()
        for st in states:
            st["g"].replay()
        torch.cuda.synchronize()
        for st in states:
            assert torch.equal(st["o"], st["ref"][0]) and torch.equal(st["lse"], st["ref"][1])


@pytest.mark.parametrize("fmt", [R.E4M3, R.INT8])
def test_layer_of_a_stream_of_frames(M, fmt):
    """The layer as a streamed video runs it: every chunk of frames is rotated,
    written and attended from, over all blocks and over predicted lists, with
    the layer's own predictor; each stage against 64 bits on its inputs."""
    H, d, block, grid, chunk = 2, 64, 64, (6, 9, 12), 2
    hw = grid[1] * grid[2]
    total, Lc = grid[0] * hw, chunk * hw
    g = torch.Generator().manual_seed(7)
    qkv = torch.randn((1, total, 3, H, d), generator=g).bfloat16()
    q, k, v = (qkv[:, :, t].transpose(1, 2) for t in range(3))
    dims, pos = (16, 24, 24), torch.arange(total)[None]
    qr, kr = (R.rope(x, dims, grid, 1e4, False, pos) for x in (q, k))
    dev = qkv.cuda()
    rope = M.Rope(M.make_rope_params(d, dims, grid))
    cs = M.make_cache_shape(1, H, total, d, block, fmt)
    c = M.Cache(cs)
    codes = [torch.zeros((1, H, total, d), dtype=torch.uint8) for _ in range(2)]
    scales = [torch.zeros((1, H, c.n)) for _ in range(2)]
    allq, allk = (torch.empty((1, H, total, d), dtype=torch.bfloat16).cuda() for _ in range(2))
    for at in range(0, total, Lc):
        shape = M.make_shape(1, H, Lc, d, block, hw)
        part = [dev[:, at:at + Lc, t].transpose(1, 2) for t in range(3)]
        qd, kd = (torch.empty((1, H, Lc, d), dtype=torch.bfloat16).cuda() for _ in range(2))
        M.mod_rope_fwd(rope.handle, shape, part[0], qd, at)
        M.mod_rope_fwd(rope.handle, shape, part[1], kd, at)
        for got, want, x in ((qd, qr, q), (kd, kr, k)):
            w = want[:, :, at:at + Lc]
            top = x[:, :, at:at + Lc].double().abs().amax(-1, keepdim=True)
            assert torch.all((got.cpu().double() - w).abs() <= R.BF16 * w.abs() + 8.1 * R.F32 * top)
        M.mod_cache_write(cs, c.ref, kd, part[2], at)
        R.write(codes[0], scales[0], kd.cpu(), block, fmt, [at], [Lc])
        R.write(codes[1], scales[1], part[2].cpu(), block, fmt, [at], [Lc])
        o, lse = torch.empty_like(qd), torch.empty((1, H, Lc)).cuda()
        M.mod_cache_attn_fwd(cs, c.ref, qd, at + Lc, None, None, None, 0.0, o, lse)
        class F:
            kv = tuple(R.dequant_by(a, b, fmt, block) for a, b in zip(codes, scales))
        F.block = block
        check(F, qd.cpu(), o, lse, [at + Lc], d ** -0.5)
        allq[:, :, at:at + Lc], allk[:, :, at:at + Lc] = qd, kd
    # the whole sequence over the predictor's lists, as the bf16 attention has them
    shape = M.make_shape(1, H, total, d, block, hw)
    stats = M.Stats(shape, M.make_params(warmup_m=1))
    n = stats.n
    idx = torch.full((1, H, n, n), -1, dtype=torch.int32).cuda()
    cnt = torch.zeros((1, H, n), dtype=torch.int32).cuda()
    M.mod_collect_stats(stats.handle, allq, allk, 1)
    M.mod_predict_block_mask(stats.handle, allq, allk, 2, M.make_budget("topk", density=0.4), idx, cnt)
    o, lse = torch.empty_like(allq), torch.empty((1, H, total)).cuda()
    M.mod_cache_attn_fwd(cs, c.ref, allq, total, None, idx, cnt, 0.0, o, lse)
    ic, cc = idx.cpu(), cnt.cpu()
    kept = [[[ic[0, h, i, :cc[0, h, i]].tolist() for i in range(n)] for h in range(H)]]
    check(F, allq.cpu(), o, lse, [total], d ** -0.5, kept)
    # and next to the bf16 attention over what the cache stands for: the same sums
    kb, vb, o2 = (torch.empty_like(allq) for _ in range(3))
    M.mod_cache_read(cs, c.ref, kb, vb)
    lse2 = torch.empty_like(lse)
    M.mod_block_sparse_attn_fwd(shape, allq, kb, vb, idx, cnt, 0.0, o2, lse2)
    if fmt == R.E4M3:      # code * scale is a bf16 number: the same K and V
        w, wl, eo, el = R.attention(allq.cpu(), *F.kv, [total], block, d ** -0.5, kept)
        assert torch.all((o.double() - o2.double()).cpu().abs() <= 2 * eo)
        assert torch.all((lse.double() - lse2.double()).cpu().abs() <= 2 * el)


@pytest.mark.parametrize("fmt", [R.E4M3, R.INT8])
@pytest.mark.parametrize("Lq,lists", [(1, False), (150, False), (600, False), (150, True)])
def test_scales_of_any_size(M, fmt, Lq, lists):
    """Value scales from 2^-100 to 2^100 (side by side in a walk) and zero, key
    scales of zero."""
    d, block, n = 128, 128, 9
    f = Filled(M, 1, 2, n * block, d, block, fmt, [n * block], seed=8)
    for t, vals in ((1, [2.0 ** -100, 1.0, 0.0, 2.0 ** 66, 2.0 ** -66, 3.0, 2.0 ** 100, 0.0, 2.0 ** -3]), (0, [None] * 4 + [0.0] * 2)):
        for j, x in enumerate(vals):
            if x is not None:
                f.scales[t][:, :, j] = x
    f.dev[2].copy_(f.scales[0])
    f.dev[3].copy_(f.scales[1])
    f.kv = tuple(R.dequant_by(c, s, fmt, block) for c, s in zip(f.codes, f.scales))
    q = queries(1, 2, Lq, d, 3)
    idx = cnt = kept = None
    if lists:   # the rows of every query block end with another of the scales
        nq = -(-Lq // block)
        kept = [[[[j for j in range(n) if j != 6 and (j + h + i) % 3] for i in range(nq)] for h in range(2)]]
        idx = torch.zeros((1, 2, nq, n), dtype=torch.int32)
        cnt = torch.zeros((1, 2, nq), dtype=torch.int32)
        for h in range(2):
            for i in range(nq):
                js = kept[0][h][i]
                idx[0, h, i, :len(js)] = torch.tensor(js, dtype=torch.int32)
                cnt[0, h, i] = len(js)
    o, lse = f.run(q, n * block, None, idx, cnt)
    check(f, q, o, lse, [n * block], d ** -0.5, kept)


@pytest.mark.parametrize("t", [2, 3])
def test_nan_scale_in_tiles(M, t):
    """A NaN scale of a listed block in the kernel for many rows: NaN in the
    rows that list it, in no others, and a NaN value scale leaves the lse."""
    d, block, n, Lq = 128, 128, 5, 300
    f = Filled(M, 1, 2, n * block, d, block, R.INT8, [n * block])
    q = queries(1, 2, Lq, d, 1)
    idx = torch.zeros((1, 2, 3, n), dtype=torch.int32)
    idx[0, 0] = torch.arange(n)
    idx[0, 1] = torch.tensor([0, 1, 3, 4, 2])
    cnt = torch.tensor([5, 4], dtype=torch.int32).view(1, 2, 1).expand(1, 2, 3).contiguous()
    o0, lse0 = f.run(q, n * block, None, idx, cnt)
    f.dev[t][0, :, 2] = math.nan
    o, lse = f.run(q, n * block, None, idx, cnt)
    assert o[0, 0].isnan().all() and torch.equal(o[0, 1], o0[0, 1]) and torch.equal(lse[0, 1], lse0[0, 1])
    assert lse[0, 0].isnan().all() if t == 2 else torch.all((lse[0, 0] - lse0[0, 0]).abs() <= 1e-5)
    # and without lists, where every row reads it
    o, lse = f.run(q, n * block)
    assert o.isnan().all()


def test_strided_views_and_shared_tensors(M):
    """Two calls at once on two streams with a workspace each, and the same
    call on both formats' caches, leave each other alone; q, o and lists that
    are not contiguous are refused."""
    f = Filled(M, 2, 2, 5000, 128, 128, R.E4M3, [5000, 4000], seed=4)
    lens = torch.tensor([5000, 4000], dtype=torch.int32)
    qs = [queries(2, 4, 3, 128, s) for s in (1, 2)]
    want = [f.run(q, 5000, lens) for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    qd, ld = [q.cuda() for q in qs], lens.cuda()
    outs = [torch.empty_like(q) for q in qd]
    need = M.mod_cache_attn_workspace_bytes(f.shape, 4, 3, 5000)
    wss = [torch.full((need,), 255, dtype=torch.uint8).cuda() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, q, o, ws in zip(streams, qd, outs, wss):
            M.mod_cache_attn_fwd(f.shape, f.ref, q, 5000, ld, None, None, 0.0, o, None, ws, need, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w[0])
    bad = torch.empty((2, 3, 4, 128), dtype=torch.bfloat16).cuda().transpose(1, 2)
    for q, o in ((bad, outs[0]), (qd[0], bad)):
        with pytest.raises(ValueError):
            M.mod_cache_attn_fwd(f.shape, f.ref, q, 5000, ld, None, None, 0.0, o)


# Calls that take tiles of 256 (d = 128 without lists), 128, 64, 32 and 16 rows, each
# whole and in parts where it is chosen so: d, block, B, H, query heads per
# head, Lq, tokens, lists
MANY_ROWS = [
    (128, 128, 2, 16, 1, 129, 5000, False), (128, 64, 3, 24, 1, 700, 500, False),      # 256
    (128, 128, 3, 24, 1, 100, 70, False), (128, 64, 2, 16, 1, 70, 5000, False),        # 128
    (64, 64, 2, 16, 2, 129, 70, False), (64, 128, 3, 16, 1, 70, 9000, False),
    (128, 128, 3, 12, 1, 129, 70, True), (128, 128, 3, 16, 2, 70, 5000, True),
    (64, 128, 3, 12, 1, 129, 70, True), (64, 128, 3, 16, 2, 70, 9000, True),
    (128, 128, 3, 16, 2, 17, 9000, False), (64, 64, 3, 24, 1, 33, 9000, False),        # 64
    (128, 64, 3, 12, 2, 70, 70, True), (128, 64, 3, 12, 2, 70, 5000, True),
    (64, 64, 3, 12, 2, 70, 70, True), (64, 64, 3, 12, 2, 70, 9000, True),
    (128, 64, 2, 8, 2, 129, 300, False), (128, 128, 3, 16, 1, 17, 3000, False),        # 32
    (64, 64, 2, 8, 2, 129, 300, False), (64, 128, 3, 12, 1, 17, 5000, False),
    (128, 64, 3, 12, 2, 17, 9000, True), (64, 64, 3, 12, 1, 70, 70, True), (64, 128, 3, 16, 2, 40, 70, True),
    (128, 64, 2, 1, 1, 17, 1000, False), (64, 128, 2, 1, 1, 17, 9000, True),           # 16, two tiles
]


def flushed(f, group):
    """What fp32 does not hold of an output: a probability p (of a row's largest)
    and its product with the value scale s are 0 under 2^-126, so a token of code
    c may lose p |c s| <= 2^-126 |c| max(1, s)."""
    codes, scales = R.numbers(f.codes[1], f.fmt).abs(), f.scales[1].double()
    lost = torch.zeros(f.B, f.H, 1, f.d, dtype=torch.float64)
    for b in range(f.B):
        at = torch.arange(f.lens[b])
        lost[b, :, 0] = (codes[b, :, at] * scales[b, :, at // f.block, None].clamp(min=1.0)).sum(1)
    return 2.0 ** -126 * lost.repeat_interleave(group, 1)


@pytest.mark.parametrize("fmt", [R.E4M3, R.INT8])
@pytest.mark.parametrize("case", MANY_ROWS)
def test_many_rows(M, case, fmt):
    """Scores that make the running maximum move, sequences of different lengths
    (none among them), and in head 0 value scales from 2^-100 to 2^100 and zero
    side by side, and a key scale of zero."""
    d, block, B, H, group, Lq, L, lists = case
    lens = [L, max(1, L // 3 - 5), 0][:B]
    f = Filled(M, B, H, L, d, block, fmt, lens, seed=Lq + L, spread=3.0)
    for t, vals in ((1, [2.0 ** -100, 1.0, 0.0, 2.0 ** 66, 2.0 ** -66, 3.0, 2.0 ** 100, 0.0, 2.0 ** -3]),
                    (0, [None] * 4 + [0.0] * 2)):
        for b in range(B):
            for j, x in enumerate(vals[:-(-lens[b] // block)]):
                if x is not None:
                    f.scales[t][b, 0, j] = x
    f.dev[2].copy_(f.scales[0])
    f.dev[3].copy_(f.scales[1])
    f.kv = tuple(R.dequant_by(c, s, fmt, block) for c, s in zip(f.codes, f.scales))
    q = queries(B, H * group, Lq, d, Lq, 2.0)
    idx = cnt = kept = None
    if lists:
        idx, cnt, kept = f.lists(H * group, -(-Lq // block), L, L, 0.6)
    args = (q, L, torch.tensor(lens, dtype=torch.int32), idx, cnt)
    o, lse = f.run(*args)
    check(f, q, o, lse, lens, d ** -0.5, kept, flushed(f, group))
    again = f.run(*args)
    assert torch.equal(again[0], o) and torch.equal(again[1], lse)


@pytest.mark.parametrize("case", [c for c in MANY_ROWS if c[2] > 1])
def test_many_rows_with_large_scores_and_short_sequences(M, case):
    """Scores up to a few hundred, and sequences much shorter than the cut-up
    length, which leave parts without a token."""
    d, block, B, H, group, Lq, L, lists = case
    lens = [min(L, 40), L, 1][:B]
    f = Filled(M, B, H, L, d, block, R.INT8, lens, seed=3, spread=12.0)
    q = queries(B, H * group, Lq, d, 5, 3.0)
    idx = cnt = kept = None
    if lists:
        idx, cnt, kept = f.lists(H * group, -(-Lq // block), L, L, 0.6)
    o, lse = f.run(q, L, torch.tensor(lens, dtype=torch.int32), idx, cnt)
    check(f, q, o, lse, lens, d ** -0.5, kept, flushed(f, group))


@pytest.mark.parametrize("case", MANY_ROWS)
def test_many_rows_with_infinities_and_nan(M, case):
    """An infinite query gives NaN in its own row alone; a NaN scale in the rows
    of the head that read its block and in no others."""
    d, block, B, H, group, Lq, L, lists = case
    f = Filled(M, B, H, L, d, block, R.E4M3, [L] * B)
    q = queries(B, H * group, Lq, d, 1)
    n, nq = -(-L // block), -(-Lq // block)
    idx = cnt = None
    if lists:      # every query block but the first lists all blocks, that one all but block 0
        idx = torch.arange(n, dtype=torch.int32).expand(B, H * group, nq, n).contiguous()
        cnt = torch.full((B, H * group, nq), n, dtype=torch.int32)
        idx[:, :, 0] = idx[:, :, 0].flip(-1)
        cnt[:, :, 0] = n - 1
    o0, lse0 = f.run(q, L, None, idx, cnt)
    row = Lq - 1
    q2 = q.clone()
    q2[B - 1, 0, row, 3] = math.inf
    o, lse = f.run(q2, L, None, idx, cnt)
    some = cnt is None or cnt[0, 0, row // block] > 0
    if some:
        assert not o[B - 1, 0, row].isfinite().any() and not lse[B - 1, 0, row].isfinite()
    o[B - 1, 0, row], lse[B - 1, 0, row] = o0[B - 1, 0, row], lse0[B - 1, 0, row]
    assert torch.equal(o, o0) and torch.equal(lse, lse0)
    for t in (2, 3):
        f.dev[t].copy_(f.scales[t - 2])
        f.dev[t][B - 1, H - 1, 0] = math.nan
        o, lse = f.run(q, L, None, idx, cnt)
        hit = torch.zeros(B, H * group, Lq, dtype=torch.bool)
        hit[B - 1, (H - 1) * group:] = True
        if lists:
            hit[:, :, :block] = False
        hit = hit.cuda()
        assert o[hit].isnan().all() and torch.equal(o[~hit], o0[~hit]) and torch.equal(lse[~hit], lse0[~hit])
        assert lse[hit].isnan().all() if t == 2 else torch.all((lse[hit] - lse0[hit]).abs() <= 1e-5)
        f.dev[t].copy_(f.scales[t - 2])


# value scales from the smallest that a write gives on, past 2^-64 and 2^64 on
# either side
FAR = [2.0 ** -126, 1.37 * 2.0 ** -126, 1.9 * 2.0 ** -125, 1.37 * 2.0 ** -100, 1.9 * 2.0 ** -65, 1.37 * 2.0 ** 66,
       1.37 * 2.0 ** 110]


@pytest.mark.parametrize("fmt", [R.E4M3, R.INT8])
@pytest.mark.parametrize("sv", FAR)
@pytest.mark.parametrize("Lq,lists", [(1, False), (20, False), (150, False), (2000, False), (20, True), (150, True)])
def test_value_scales_of_the_whole_range(M, fmt, sv, Lq, lists):
    """Probabilities below one times the smallest scales: nothing is lost but
    what fp32 sums (at most four roundings a token, 2^-150 each) and the bf16
    output (half a step of 2^-133) do not hold."""
    if fmt == R.E4M3:
        sv = 2.0 ** math.floor(math.log2(sv))
    d, block, n, H = 128, 128, 5, 16
    f = Filled(M, 1, H, n * block, d, block, fmt, [n * block], seed=8)
    f.scales[1].fill_(sv)
    f.dev[3].copy_(f.scales[1])
    f.kv = tuple(R.dequant_by(c, s, fmt, block) for c, s in zip(f.codes, f.scales))
    q = queries(1, H, Lq, d, 3)
    idx = cnt = kept = None
    if lists:
        idx, cnt, kept = f.lists(H, -(-Lq // block), n * block, Lq, 0.7)
    o, lse = f.run(q, n * block, None, idx, cnt)
    check(f, q, o, lse, [n * block], d ** -0.5, kept, 2.0 ** -134 + 4 * n * block * 2.0 ** -150)


@pytest.mark.parametrize("sv", FAR)
@pytest.mark.parametrize("case", MANY_ROWS)
def test_codes_stay_exact_under_any_scale(M, case, sv):
    """Equal scores give every token of a sequence the same rounded probability,
    a common factor of the output, so values that nearly cancel leave errors of
    the small sum and not of its terms: two half steps of bf16 of the output and
    the roundings of fp32 sums (at most four per token of the sum of magnitudes;
    2^-150 each where that is subnormal)."""
    d, block, B, H, group, Lq, L, lists = case
    f = Filled(M, B, H, L, d, block, R.INT8, [L] * B)
    c = 60 + torch.arange(d) % 64
    codes = torch.where((torch.arange(L) % 2 == 0)[:, None], c, 1 - c).to(torch.int8)
    f.dev[1].copy_(codes.view(torch.uint8).expand(B, H, L, d))
    f.dev[3].fill_(sv)
    sv = float(f.dev[3][0, 0, 0])
    idx = cnt = None
    n, nq = -(-L // block), -(-Lq // block)
    if lists:
        idx = torch.arange(n, dtype=torch.int32).expand(B, H * group, nq, n).contiguous()
        cnt = torch.full((B, H * group, nq), n, dtype=torch.int32)
    o, lse = f.run(torch.zeros((B, H * group, Lq, d), dtype=torch.bfloat16), L, None, idx, cnt)
    want, size = codes.double().mean(0) * sv, codes.double().abs().mean(0) * sv
    bound = 2.01 * R.BF16 * want.abs() + 4 * L * (R.F32 * size + 2.0 ** -150) + 2.0 ** -134
    off = (o.cpu().double() - want).abs()
    assert torch.all(off <= bound), (off / bound).max()
    assert torch.all((lse.cpu().double() - math.log(L)).abs() <= 4 * L * R.F32 + 2.0 ** -20)


@pytest.mark.parametrize("how", ["current", "side", "side address", "default", "default address"])
def test_workspace_belongs_to_the_stream_that_uses_it(M, monkeypatch, how):
    """While another stream is the current one, also for the default stream,
    whose address is 0."""
    f = Filled(M, 2, 2, 5000, 128, 128, R.INT8, [5000, 5000], seed=4)
    q = queries(2, 2, 1, 128, 2)
    o0, _ = f.run(q, 5000)
    qd, o = q.cuda(), torch.empty_like(q, device="cuda")
    assert M.mod_cache_attn_workspace_bytes(f.shape, 2, 1, 5000) > 0
    side, current = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    want, stream = {"current": (current.cuda_stream, None), "side": (side.cuda_stream, side),
                    "side address": (side.cuda_stream, side.cuda_stream), "default": (0, torch.cuda.default_stream()),
                    "default address": (0, 0)}[how]
    seen, empty = [], torch.empty
    def spy(*args, **kw):
        seen.append(torch.cuda.current_stream().cuda_stream)
        return empty(*args, **kw)
    with torch.cuda.stream(current):
        monkeypatch.setattr(torch, "empty", spy)
        M.mod_cache_attn_fwd(f.shape, f.ref, qd, 5000, None, None, None, 0.0, o, None, stream=stream)
        monkeypatch.undo()
    torch.cuda.synchronize()
    assert seen == [want]
    assert torch.equal(o, o0)
