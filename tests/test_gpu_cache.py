"""The 8-bit cache: codes and scales bit by bit against the definition in 64
bits, and reading back."""
import math

import pytest
import torch

import cached_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import paper_2601_11641_amd as m
    return m


def fresh(B, H, cap, d, block, seed=0):
    """Memory with arbitrary contents: codes, scales."""
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (B, H, cap, d), generator=g).to(torch.uint8)
    return codes, torch.full((B, H, -(-cap // block)), math.nan)


def values(B, H, L, d, seed, magnitude=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, L, H, d), generator=g) * magnitude
    x *= torch.exp2(torch.randint(-3, 4, (B, L, H, 1), generator=g).float())
    return x.bfloat16().transpose(1, 2)


class Pair:
    """A cache on the device and its model on the host."""

    def __init__(self, M, B, H, cap, d, block, fmt):
        self.M, self.dims, self.fmt, self.block = M, (B, H, cap, d), fmt, block
        self.shape = M.make_cache_shape(B, H, cap, d, block, fmt)
        self.k, self.ks = fresh(B, H, cap, d, block, 1)
        self.v, self.vs = fresh(B, H, cap, d, block, 2)
        self.dev = [t.cuda() for t in (self.k, self.v, self.ks, self.vs)]
        self.ref = M.make_cache(*self.dev)

    def write(self, k, v, first=0, starts=None, counts=None):
        B, L = k.shape[0], k.shape[2]
        kd, vd = k.cuda(), v.cuda()
        ints = [None if t is None else torch.tensor(t, dtype=torch.int32).cuda() for t in (starts, counts)]
        self.M.mod_cache_write(self.shape, self.ref, kd, vd, first, *ints)
        st = [first + s for s in (starts or [0] * B)]
        for x, codes, scales in ((k, self.k, self.ks), (v, self.v, self.vs)):
            R.write(codes, scales, x, self.block, self.fmt, st, counts or [L] * B)

    def check(self):
        for want, got in zip((self.k, self.v), self.dev[:2]):
            if self.fmt == R.E4M3:   # a zero may have either sign, and a NaN any
                a, b = R.numbers(want, R.E4M3), R.numbers(got.cpu(), R.E4M3)
                assert torch.equal(a.nan_to_num(nan=1e9), b.nan_to_num(nan=1e9))
            else:
                assert torch.equal(want, got.cpu())
        for want, got in zip((self.ks, self.vs), self.dev[2:]):
            got = got.cpu()
            assert torch.equal(want.isnan(), got.isnan())
            assert torch.equal(want.nan_to_num(nan=-1.0), got.nan_to_num(nan=-1.0))


FORMS = [(d, block, fmt) for d in (64, 128) for block in (64, 128) for fmt in (R.E4M3, R.INT8)]


@pytest.mark.parametrize("d,block,fmt", FORMS)
def test_write_whole_and_continued(M, d, block, fmt):
    """A write from the start, continuations inside blocks with smaller and
    larger values, single tokens, a rewrite from a block's start, the end of
    the capacity."""
    p = Pair(M, 2, 3, 300, d, block, fmt)
    seed = 10
    for first, L, mag in ((0, 130, 1.0), (130, 1, 0.01), (131, 1, 40.0), (132, 70, 1.0), (202, 98, 300.0),
                          (128, 40, 0.1), (37, 1, 1e4), (299, 1, 1e-3)):
        seed += 1
        p.write(values(2, 3, L, d, seed, mag), values(2, 3, L, d, seed + 50, mag), first)
        p.check()


@pytest.mark.parametrize("d,block,fmt", [(64, 64, R.INT8), (128, 128, R.E4M3), (128, 64, R.INT8)])
def test_write_ragged(M, d, block, fmt):
    """Starts and counts of the device, some of them out of range: nothing of
    such a sequence, nor a token past the capacity, is written."""
    B, cap, L = 8, 200, 70
    p = Pair(M, B, 2, cap, d, block, fmt)
    p.write(values(B, 2, 64, d, 1), values(B, 2, 64, d, 2))
    for starts, counts in (([64, 60, 0, 199, -1, 200, 130, 64], [70, 1, 0, 70, 70, 70, 70, -5]),
                           ([0, 1, 127, 128, 129, 190, 2 ** 31 - 1 - 9, -2 ** 31], [71, 70, 69, 3, 2, 1000, 1, 1])):
        p.write(values(B, 2, L, d, 3), values(B, 2, L, d, 4), 0, starts, counts)
        p.check()
    p.write(values(B, 2, L, d, 5), values(B, 2, L, d, 6), 9, [0] * 7 + [2 ** 31 - 1], None)   # first + start past 2^31
    p.check()


@pytest.mark.parametrize("fmt", [R.E4M3, R.INT8])
def test_write_special_values(M, fmt):
    """Zeros, subnormals, the largest numbers, borders between codes, and
    blocks that receive infinities and NaN."""
    d, block, cap = 64, 64, 64 * 12
    p = Pair(M, 1, 1, cap, d, block, fmt)
    x = torch.zeros(1, 1, cap, d)
    g = torch.Generator().manual_seed(1)
    x[0, 0, 64:128] = torch.randn(64, d, generator=g) * 1e-39          # subnormal
    x[0, 0, 128:192] = torch.randn(64, d, generator=g) * 1e-36
    x[0, 0, 192:256] = torch.rand(64, d, generator=g) * 3.3e38
    x[0, 0, 256:320] = torch.arange(64 * d).view(64, d) % 255 - 127.0  # s = 1: codes, exactly
    x[0, 0, 320:384] = (torch.arange(64 * d).view(64, d) % 255 - 127) * 0.5   # s = 1/2 ...
    x[0, 0, 320, 0] = 127.0                                            # ... and halves are borders
    x[0, 0, 384:448] = 448 * torch.exp2(-(torch.arange(64 * d).view(64, d) % 24).float()) * 0.97
    x[0, 0, 448:512] = torch.randn(64, d, generator=g)
    x[0, 0, 460, 7] = math.inf
    x[0, 0, 512:576] = torch.randn(64, d, generator=g)
    x[0, 0, 520, 9] = math.nan
    x[0, 0, 576:640] = -0.0
    x[0, 0, 640:704] = 3.3895e38
    x[0, 0, 704] = 2.0 ** -133                                         # one smallest number
    x = x.bfloat16()
    p.write(x, x)
    p.check()
    # continued: a NaN stays, a scale of zero grows, then the block is begun anew
    for first in (450, 530, 60, 600):
        p.write(x[:, :, 256:260], x[:, :, 260:264], first)
        p.check()
    p.write(x[:, :, :128], x[:, :, 448:576], 448)
    p.check()
    assert p.ks[0, 0, 7] == 0 and p.vs[0, 0, 7].isnan()


@pytest.mark.parametrize("fmt", [R.E4M3, R.INT8])
def test_write_all_borders(M, fmt):
    """Every bf16 number of eight binades under scales whose last bits vary:
    the rounding is that of the real quotient."""
    d, block = 64, 64
    mant = torch.arange(128) / 128 + 1
    x = torch.cat([mant * 2.0 ** e for e in range(-8, 0)])               # 1024 numbers
    x = torch.cat([x, -x]).view(32, d)
    n = 300
    rows = torch.zeros(1, n, block, d)
    for i in range(n):
        rows[0, i, :32] = x
        rows[0, i, 32, 0] = 1 + i % 128 / 128 + (i // 128)               # the largest: another scale per block
    k = rows.view(1, 1, n * block, d).bfloat16()
    p = Pair(M, 1, 1, n * block, d, block, fmt)
    p.write(k, -k)
    p.check()


@pytest.mark.parametrize("d,block,fmt", FORMS)
def test_read(M, d, block, fmt):
    B, H, cap, L = 3, 2, 150, 60
    p = Pair(M, B, H, cap, d, block, fmt)
    p.write(values(B, H, cap, d, 1), values(B, H, cap, d, 2))
    p.dev[2][1, 1, 1] = p.ks[1, 1, 1] = math.nan
    for first, starts, counts in ((0, None, None), (cap - L, None, None),
                                  (3, [80, 0, 140], [60, 31, 60]), (0, [-1, 150, 149], [60, 60, 60])):
        k = torch.full((B, L, H, d), 7.0, dtype=torch.bfloat16).cuda().transpose(1, 2)
        v = torch.full((B, H, L, d), 7.0, dtype=torch.bfloat16).cuda()
        ints = [None if t is None else torch.tensor(t, dtype=torch.int32).cuda() for t in (starts, counts)]
        p.M.mod_cache_read(p.shape, p.ref, k, v, first, *ints)
        only = torch.full_like(v, 7.0)
        p.M.mod_cache_read(p.shape, p.ref, None, only, first, *ints)
        assert torch.equal(only, v)
        for got, codes, scales in ((k, p.k, p.ks), (v, p.v, p.vs)):
            all_ = R.dequant_by(codes, scales, fmt, block)
            got = got.cpu().double()
            for b in range(B):
                s = first + (starts[b] if starts else 0)
                c = counts[b] if counts else L
                e = min(cap, s + c) if 0 <= s < cap else s
                want = torch.full((H, L, d), 7.0, dtype=torch.float64)
                if e > s:
                    want[:, :e - s] = all_[b, :, s:e]
                assert torch.equal(want.isnan(), got[b].isnan())
                off = (got[b] - want).abs().nan_to_num()
                assert torch.all(off <= 1.001 * R.BF16 * want.abs().nan_to_num())


def test_write_is_captured_and_replayed(M):
    """A captured append advances through device positions; each replay equals
    the eager result."""
    B, H, cap, d, block = 2, 2, 256, 128, 128
    p = Pair(M, B, H, cap, d, block, R.INT8)
    p.write(values(B, H, 100, d, 1), values(B, H, 100, d, 2))
    k, v = (torch.zeros(B, H, 1, d, dtype=torch.bfloat16).cuda() for _ in range(2))
    at = torch.zeros(B, dtype=torch.int32).cuda()
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        M.mod_cache_write(p.shape, p.ref, k, v, 100, at)
    torch.cuda.synchronize()
    R.write(p.k, p.ks, k.cpu(), block, R.INT8, [100] * B, [1] * B)
    R.write(p.v, p.vs, v.cpu(), block, R.INT8, [100] * B, [1] * B)
    with torch.cuda.graph(g):
        M.mod_cache_write(p.shape, p.ref, k, v, 100, at)
    for t in range(40):
        a, b = values(B, H, 1, d, 100 + t, 1.5 ** (t % 7)), values(B, H, 1, d, 200 + t)
        k.copy_(a)
        v.copy_(b)
        at.copy_(torch.tensor([t, t + 5], dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        for x, codes, scales in ((a, p.k, p.ks), (b, p.v, p.vs)):
            R.write(codes, scales, x, block, R.INT8, [100 + t, 105 + t], [1, 1])
    p.check()
