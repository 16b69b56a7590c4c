"""Where at most 16 rows share a key/value head, probabilities are two bf16 each:
a value's rounding must not show.  Two tokens whose values nearly cancel leave an
output small next to its terms, so that its own rounding hides nothing."""
import pytest
import torch

import cached_ref as R

# the first bf16 is off by at most 2^-8 of a probability, the second by 2^-8 of that
TWO = 2.0 ** -16


@pytest.fixture(scope="module")
def M():
    import paper_2601_11641_amd as m
    return m


def nearest(x, fmt):
    if fmt == R.INT8:
        return x.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return x.float().to(torch.float8_e4m3fn).view(torch.uint8)


def case(d, fmt, L, rows, seed):
    """8 heads of L tokens: q [1, 8 rows, 1, d], codes of k and v, the scale and
    the block; all but two tokens have the value 0."""
    g = torch.Generator().manual_seed(seed)
    H, block, scale = 8, 64, 0.25 * d ** -0.5
    q = torch.randn((1, H, 1, d), generator=g).bfloat16().repeat_interleave(rows, 1)   # a head's rows are alike
    k = nearest(torch.randn((1, H, L, d), generator=g) * 40, fmt)
    s = torch.full((1, H, -(-L // block)), 2.0 ** -5)
    kd = R.dequant_by(k, s, fmt, block)
    at = (0, 1) if L == 2 else (7, L - 100)
    score = (q[:, ::rows].double() * kd[:, :, at]).sum(-1) * scale
    ratio = torch.exp(score[..., 1] - score[..., 0])                  # of the second token to the first
    a = 64 + torch.arange(d, dtype=torch.float64) % 63
    a = torch.where(ratio[..., None] > 1, a / ratio[..., None], a)    # the larger value within the codes
    v = torch.zeros((1, H, L, d), dtype=torch.uint8)
    v[:, :, at[1]] = nearest(-a, fmt)
    second = R.numbers(v[:, :, at[1]], fmt)
    v[:, :, at[0]] = nearest(-second * ratio[..., None], fmt)
    return q, k, v, s, scale, block


def wanted(q, k, v, s, scale, block, fmt):
    """The output and its bound with `TWO` in the place of a bf16 rounding."""
    kd, vd = (R.dequant_by(x, s, fmt, block) for x in (k, v))
    L = k.shape[2]
    want, lse, bound, _ = R.attention(q, kd, vd, [L], block, scale)
    rows = q.shape[1] // k.shape[1]
    p = torch.exp((q.double() @ kd.repeat_interleave(rows, 1).transpose(2, 3)) * scale - lse[..., None])
    spread = p @ vd.abs().repeat_interleave(rows, 1)
    return want, bound - (R.BF16 - TWO) * 1.01 * spread


CASES = [(d, fmt, L, rows) for d in (64, 128) for fmt in (R.E4M3, R.INT8) for L, rows in ((2, 1), (2, 16), (3000, 1), (3000, 4))]


@pytest.mark.parametrize("d,fmt,L,rows", CASES)
def test_the_bound_tells_one_bf16_from_two(d, fmt, L, rows):
    """A model of either rounding: one bf16 fails in every head's channels that
    cancel, two pass."""
    q, k, v, s, scale, block = case(d, fmt, L, rows, L + rows)
    want, bound = wanted(q, k, v, s, scale, block, fmt)
    kd, vd = (R.dequant_by(x, s, fmt, block).repeat_interleave(rows, 1) for x in (k, v))
    x = (q.double() @ kd.transpose(2, 3)) * scale
    p = torch.exp(x - x.amax(-1, keepdim=True))
    once = p.bfloat16().double()
    twice = once + (p - once).bfloat16().double()
    off = [((r @ vd / p.sum(-1, keepdim=True)).bfloat16().double() - want).abs() for r in (once, twice)]
    assert torch.all(off[1] <= bound)
    assert (off[0] > bound).any(-1).double().mean() > 0.5


@pytest.mark.gpu
@pytest.mark.parametrize("d,fmt,L,rows", CASES)
def test_probabilities_are_two_bf16(M, d, fmt, L, rows):
    q, k, v, s, scale, block = case(d, fmt, L, rows, L + rows)
    want, bound = wanted(q, k, v, s, scale, block, fmt)
    shape = M.make_cache_shape(1, 8, L, d, block, fmt)
    assert M.mod_cache_attn_plan(shape, 8 * rows, 1, L)[0] == 16
    if L > 2:
        assert M.mod_cache_attn_plan(shape, 8 * rows, 1, L)[1] > 1
    dev = [t.cuda() for t in (k, v, s, s.clone())]
    o = torch.empty_like(q, device="cuda")
    M.mod_cache_attn_fwd(shape, M.make_cache(*dev), q.cuda(), L, None, None, None, scale, o)
    off = (o.cpu().double() - want).abs()
    assert torch.all(off <= bound), (off / bound).max()
    # the same rows as queries of one head, over a list of every block
    n = -(-L // block)
    idx = torch.arange(n, dtype=torch.int32).expand(1, 8, 1, n).contiguous().cuda()
    cnt = torch.full((1, 8, 1), n, dtype=torch.int32).cuda()
    q2 = q.view(1, 8, rows, d).contiguous()
    o2 = torch.empty_like(q2, device="cuda")
    M.mod_cache_attn_fwd(shape, M.make_cache(*dev), q2.cuda(), L, None, idx, cnt, scale, o2)
    off = (o2.cpu().double().view(want.shape) - want).abs()
    assert torch.all(off <= bound), (off / bound).max()
