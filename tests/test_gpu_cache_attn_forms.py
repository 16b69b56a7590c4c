"""Attention over the cache in the kernel for many rows, at sizes for which the
library is asked first that it takes it."""
import math

import pytest
import torch

import cached_ref as R
from test_gpu_cache_attn import Filled, check, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import paper_2601_11641_amd as m
    return m


def test_many_parts_of_the_largest_tile(M):
    """256 rows, joined in eight slices: 256 queries over a long cache."""
    H, Lq, L, d = 4, 256, 40000, 128
    f = Filled(M, 1, H, L, d, 128, R.INT8, [L - 77], seed=2, spread=2.0)
    rows, parts = M.mod_cache_attn_plan(f.shape, H, Lq, L)
    assert rows == 256 and parts > 8
    q = queries(1, H, Lq, d, 3, 2.0)
    lens = torch.tensor([L - 77], dtype=torch.int32)
    o, lse = f.run(q, L, lens)
    check(f, q, o, lse, [L - 77], d ** -0.5)
    again = f.run(q, L, lens)
    assert torch.equal(again[0], o) and torch.equal(again[1], lse)


@pytest.mark.parametrize("Lq", [200, 1100])
def test_many_rows_past_32_bits(M, Lq):
    """A cache of 5 GB per tensor: its last heads' last tokens, over lists and
    over the whole cache."""
    B, H, cap, d, block, L = 1, 5, 1 << 23, 128, 128, 300
    shape = M.make_cache_shape(B, H, cap, d, block, R.E4M3)
    for lists in (False, True):
        assert M.mod_cache_attn_plan(shape, H, Lq, cap, lists)[0] >= 64
    c = M.Cache(shape)
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        t.zero_()
    k, v = queries(B, H, L, d, 1), queries(B, H, L, d, 2)
    M.mod_cache_write(shape, c.ref, k.cuda(), v.cuda(), cap - L)
    kb, vb = torch.empty_like(k, device="cuda"), torch.empty_like(v, device="cuda")
    M.mod_cache_read(shape, c.ref, kb, vb, cap - L)
    kd, vd = kb.cpu().double(), vb.cpu().double()
    n, first, nq = cap // block, (cap - L) // block, -(-Lq // block)
    q = queries(B, H, Lq, d, 3)
    idx = torch.full((B, H, nq, n), -1, dtype=torch.int32)
    idx[..., :3] = torch.arange(first, first + 3)
    cnt = torch.full((B, H, nq), 3, dtype=torch.int32)
    o, lse = torch.empty_like(q, device="cuda"), torch.empty((B, H, Lq)).cuda()
    M.mod_cache_attn_fwd(shape, c.ref, q.cuda(), cap, None, idx.cuda(), cnt.cuda(), 0.0, o, lse)
    pad = torch.zeros((B, H, 3 * block - L, d), dtype=torch.float64)     # zero rows of the first listed block
    class F:
        kv = (torch.cat([pad, kd], 2), torch.cat([pad, vd], 2))
    F.block = block
    check(F, q, o, lse, [3 * block], d ** -0.5)
    # every token: the zeros in front have score 0
    M.mod_cache_attn_fwd(shape, c.ref, q.cuda(), cap, None, None, None, 0.0, o, lse)
    w = torch.exp(q.double() @ kd.transpose(2, 3) * d ** -0.5)
    total = w.sum(-1) + (cap - L)
    want = (w @ vd) / total[..., None]
    # sums of up to 2^23 / 2 ones per lane: at most 2^-24 each step of a part
    assert torch.all((lse.cpu().double() - total.log()).abs() <= 1e-4)
    err = (o.cpu().double() - want).abs()
    assert torch.all(err <= 2 * R.BF16 * (want.abs() + (w @ vd.abs()) / total[..., None]) + 1e-4 * want.abs())


@pytest.mark.parametrize("fmt,d", [(R.E4M3, 128), (R.INT8, 64)])
def test_layer_of_a_stream_in_large_chunks(M, fmt, d):
    """The streamed layer at sizes that the kernel for many rows takes: every
    chunk rotated, written and attended from, then the whole sequence over the
    predictor's lists, each stage against 64 bits on its inputs."""
    H, block, grid, chunk = 12, 128, (4, 16, 24), 2
    hw = grid[1] * grid[2]
    total, Lc = grid[0] * hw, chunk * hw
    g = torch.Generator().manual_seed(7)
    qkv = torch.randn((1, total, 3, H, d), generator=g).bfloat16()
    dims = (16, 24, 24) if d == 64 else (44, 42, 42)
    dev = qkv.cuda()
    rope = M.Rope(M.make_rope_params(d, dims, grid))
    cs = M.make_cache_shape(1, H, total, d, block, fmt)
    c = M.Cache(cs)
    codes = [torch.zeros((1, H, total, d), dtype=torch.uint8) for _ in range(2)]
    scales = [torch.zeros((1, H, c.n)) for _ in range(2)]
    allq, allk = (torch.empty((1, H, total, d), dtype=torch.bfloat16).cuda() for _ in range(2))
    for at in range(0, total, Lc):
        assert M.mod_cache_attn_plan(cs, H, Lc, at + Lc)[0] >= 64
        shape = M.make_shape(1, H, Lc, d, block, hw)
        part = [dev[:, at:at + Lc, t].transpose(1, 2) for t in range(3)]
        qd, kd = (torch.empty((1, H, Lc, d), dtype=torch.bfloat16).cuda() for _ in range(2))
        M.mod_rope_fwd(rope.handle, shape, part[0], qd, at)
        M.mod_rope_fwd(rope.handle, shape, part[1], kd, at)
        pos = torch.arange(at, at + Lc)[None]
        for got, t in ((qd, 0), (kd, 1)):
            x = part[t].cpu()
            w = R.rope(x, dims, grid, 1e4, False, pos)
            top = x.double().abs().amax(-1, keepdim=True)
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
    shape = M.make_shape(1, H, total, d, block, hw)
    stats = M.Stats(shape, M.make_params(warmup_m=1))
    n = stats.n
    idx = torch.full((1, H, n, n), -1, dtype=torch.int32).cuda()
    cnt = torch.zeros((1, H, n), dtype=torch.int32).cuda()
    M.mod_collect_stats(stats.handle, allq, allk, 1)
    M.mod_predict_block_mask(stats.handle, allq, allk, 2, M.make_budget("topk", density=0.4), idx, cnt)
    assert M.mod_cache_attn_plan(cs, H, total, total, True)[0] >= 64
    o, lse = torch.empty_like(allq), torch.empty((1, H, total)).cuda()
    M.mod_cache_attn_fwd(cs, c.ref, allq, total, None, idx, cnt, 0.0, o, lse)
    ic, cc = idx.cpu(), cnt.cpu()
    kept = [[[ic[0, h, i, :cc[0, h, i]].tolist() for i in range(n)] for h in range(H)]]
    check(F, allq.cpu(), o, lse, [total], d ** -0.5, kept)
    # a chunk that starts at a block's start takes its rows of the lists
    first = Lc // block
    assert Lc % block == 0
    o1, lse1 = torch.empty((1, H, Lc, d), dtype=torch.bfloat16).cuda(), torch.empty((1, H, Lc)).cuda()
    M.mod_cache_attn_fwd(cs, c.ref, allq[:, :, Lc:2 * Lc].contiguous(), total, None, idx[:, :, first:first + Lc // block]
                         .contiguous(), cnt[:, :, first:first + Lc // block].contiguous(), 0.0, o1, lse1)
    kept = [[rows[first:first + Lc // block] for rows in kept[0]]]
    check(F, allq[:, :, Lc:2 * Lc].cpu(), o1, lse1, [total], d ** -0.5, kept)


@pytest.mark.parametrize("lists", [False, True])
@pytest.mark.parametrize("fmt", [R.E4M3, R.INT8])
def test_scales_of_any_size_in_large_tiles(M, fmt, lists):
    """Value scales from 2^-126 to 2^100 and zero side by side in a walk, key
    scales of zero, then a NaN scale of one block."""
    d, block, n, H, Lq = 128, 128, 9, 24, 700
    f = Filled(M, 1, H, n * block, d, block, fmt, [n * block], seed=8)
    assert M.mod_cache_attn_plan(f.shape, H, Lq, n * block, lists)[0] >= 64
    for t, vals in ((1, [2.0 ** -126, 1.0, 0.0, 2.0 ** 66, 2.0 ** -66, 3.0, 2.0 ** 100, 0.0, 2.0 ** -3]), (0, [None] * 4 + [0.0] * 2)):
        for j, x in enumerate(vals):
            if x is not None:
                f.scales[t][:, :, j] = x
    f.dev[2].copy_(f.scales[0])
    f.dev[3].copy_(f.scales[1])
    f.kv = tuple(R.dequant_by(c, s, fmt, block) for c, s in zip(f.codes, f.scales))
    q = queries(1, H, Lq, d, 3)
    idx = cnt = kept = None
    if lists:
        idx, cnt, kept = f.lists(H, -(-Lq // block), n * block, 5, 0.6)
    o, lse = f.run(q, n * block, None, idx, cnt)
    check(f, q, o, lse, [n * block], d ** -0.5, kept, 2.0 ** -134 + 4 * n * block * 2.0 ** -150)
    for t in (2, 3):
        f.dev[t][0, 0, 3] = math.nan
        o1, lse1 = f.run(q, n * block, None, idx, cnt)
        hit = torch.zeros(1, H, Lq, dtype=torch.bool)
        for i in range(-(-Lq // block)):
            hit[0, 0, i * block:(i + 1) * block] = not lists or 3 in kept[0][0][i]
        hit = hit.cuda()
        assert hit.any() and o1[hit].isnan().all()
        assert torch.equal(o1[~hit], o[~hit]) and torch.equal(lse1[~hit], lse[~hit])
        f.dev[t].copy_(f.scales[t - 2])
