"""Rotary positions over several axes against the plain form in 64 bits."""
import pytest
import torch

import cached_ref as R

pytestmark = pytest.mark.gpu
A = 1 << 20   # an aligned address that is never used


@pytest.fixture(scope="module")
def M():
    import paper_2601_11641_amd as m
    return m


def make(B, H, L, d, seed, token_major=True):
    x = torch.randn((B, L, H, d) if token_major else (B, H, L, d), generator=torch.Generator().manual_seed(seed))
    x = x.bfloat16()
    return x.transpose(1, 2) if token_major else x


def bound(x, y):
    """Half a bf16 step of the result, and of the two products and their sum
    four fp32 roundings (the table's among them) of the pair's magnitudes, at
    most the token's largest channel twice."""
    return R.BF16 * y.abs() + 1.01 * 8 * R.F32 * x.double().abs().amax(-1, keepdim=True)


CASES = [
    # B, H, L, d, dims, grid, theta, halves, text, first, starts
    (1, 1, 1, 64, (16, 24, 24), (4, 8, 8), 1e4, False, 0, 0, None),
    (1, 2, 1, 128, (44, 42, 42), (3000, 30, 40), 1e4, False, 0, 3000 * 1200 - 1, None),   # far position
    (1, 3, 7, 128, (44, 42, 42), (5, 3, 7), 256.0, True, 0, 93, None),                     # partial frames, odd halves
    (2, 5, 130, 64, (16, 24, 24), (9, 5, 7), 1e4, True, 17, 4, [0, 150]),
    (2, 5, 130, 128, (16, 56, 56), (9, 5, 7), 256.0, False, 17, 4, [150, 0]),
    (1, 9, 33, 64, (0, 32, 30), (1, 6, 8), 1e6, False, 3, 2, None),                        # an image; channels left over
    (1, 9, 33, 64, (2, 0, 0), (64, 1, 1), 1e4, True, 0, 30, None),                         # time alone, one pair
    (3, 41, 300, 128, (40, 40, 40), (20, 4, 5), 1e4, True, 12, 0, [1, 0, 100]),            # heads past a group of four
    (1, 2, 40, 64, (16, 24, 24), (4, 8, 8), 1e4, False, 40, 0, None),                      # text alone
]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("token_major", [True, False])
def test_rope_matches_the_formula(M, case, backward, token_major):
    B, H, L, d, dims, grid, theta, halves, text, first, starts = case
    x = make(B, H, L, d, 1, token_major)
    pos = first + torch.arange(L - text)[None] + torch.tensor(starts or [0] * B)[:, None]
    y = R.rope(x, dims, grid, theta, halves, pos, text, transpose=backward)
    rope = M.Rope(M.make_rope_params(d, dims, grid, theta, "halves" if halves else "adjacent"))
    xd = x.cuda()
    assert xd.stride() == x.stride()
    out = make(B, H, L, d, 2, not token_major).cuda()      # the other layout
    st = torch.tensor(starts, dtype=torch.int32).cuda() if starts else None
    shape = M.make_shape(B, H, L, d, 128, grid[1] * grid[2], text)
    (M.mod_rope_bwd if backward else M.mod_rope_fwd)(rope.handle, shape, xd, out, first, st)
    got = out.cpu().double()
    assert torch.all((got - y).abs() <= bound(x, y))
    # text tokens and channels past the axes are copies
    assert torch.equal(got[:, :, L - text:], x[:, :, L - text:].double())
    assert torch.equal(got[..., sum(dims):], x[..., sum(dims):].double())
    # in place
    (M.mod_rope_bwd if backward else M.mod_rope_fwd)(rope.handle, shape, xd, xd, first, st)
    assert torch.equal(xd.cpu().double(), got)
    rope.close()


def test_rope_gradient_is_the_transpose(M):
    """<R x, g> = <x, R^T g> over random x and g, each side within the sums of
    its roundings, and backward after forward returns x."""
    B, H, L, d, grid = 2, 3, 77, 128, (6, 5, 4)
    x, g = (make(B, H, L, d, s).cuda() for s in (3, 4))
    rope = M.Rope(M.make_rope_params(d, (44, 42, 42), grid))
    shape = M.make_shape(B, H, L, d, 64)
    y, dx, back = (torch.empty_like(x) for _ in range(3))
    M.mod_rope_fwd(rope.handle, shape, x, y, 5)
    M.mod_rope_bwd(rope.handle, shape, g, dx, 5)
    a, b = (y.double() * g.double()), (x.double() * dx.double())
    assert abs(a.sum() - b.sum()) <= 1.1 * R.BF16 * (a.abs().sum() + b.abs().sum())
    M.mod_rope_bwd(rope.handle, shape, y, back, 5)
    # two roundings of values no larger than the pair, which the largest channel bounds
    top = x.double().abs().amax(-1, keepdim=True)
    assert torch.all((back.double() - x.double()).abs() <= 1.1 * R.BF16 * 4 * top)
    # differences: R is linear, so (R (x + e) - R x) is R e for channels that bf16 holds exactly
    e = torch.zeros_like(x)
    e[:, :, :, 10] = 1.0
    ye, dxe = torch.empty_like(x), torch.empty_like(x)
    M.mod_rope_fwd(rope.handle, shape, e, ye, 5)
    M.mod_rope_bwd(rope.handle, shape, g, dxe, 5)
    want = (ye.double() * g.double()).sum(-1)                 # d<R x, g> / d x[10]
    assert torch.all((dxe[..., 10].double() - want).abs() <= 3 * R.BF16 * g.double().abs().amax(-1))


def test_rope_positions_outside_and_special_values(M):
    d, grid = 64, (2, 3, 4)
    rope = M.Rope(M.make_rope_params(d, (16, 24, 20), grid))
    x = torch.randn(3, 2, 6, d).bfloat16().cuda()
    x[1, 0, 2, 63] = float("inf")       # not rotated: a copy, and its neighbour too
    x[1, 0, 3, 4] = float("inf")        # rotated: its pair alone
    y = torch.empty_like(x)
    starts = torch.tensor([-2, 0, 20], dtype=torch.int32).cuda()
    shape = M.make_shape(3, 2, 6, d, 64)
    M.mod_rope_fwd(rope.handle, shape, x, y, 0, starts)
    y = y.cpu()
    assert y[0, :, :2, :60].isnan().all() and y[2, :, 4:, :60].isnan().all()
    assert torch.equal(y[..., 60:], x.cpu()[..., 60:])
    y[0, :, :2] = y[2, :, 4:] = 0
    assert not y[1, 0, 3, 4:6].isfinite().all()
    y[1, 0, 3, 4:6] = 0
    y[1, 0, 2, 63] = 0
    assert y.isfinite().all()


def test_rope_refusals_on_the_device(M):
    rope = M.Rope(M.make_rope_params(64, (16, 24, 24), (2, 3, 4)))
    x = torch.zeros(1, 2, 25, 64, dtype=torch.bfloat16).cuda()
    def status(shape, a=x, b=x, first=0):
        with pytest.raises(M.ModError) as e:
            M.mod_rope_fwd(rope.handle, shape, a, b, first)
        return e.value.status
    assert status(M.make_shape(1, 2, 25, 64, 64)) == 1                       # past the last position
    M.mod_rope_fwd(rope.handle, M.make_shape(1, 2, 25, 64, 64, 12, 1), x, x)  # 24 and one of text
    assert status(M.make_shape(1, 2, 25, 64, 64, 12, 1), first=1) == 1
    assert status(M.make_shape(1, 2, 25, 64, 64, 13, 1)) == 1                # another frame size
    assert status(M.make_shape(1, 2, 25, 64, 64, 12, 26)) == 1
    assert status(M.make_shape(1, 2, 25, 64, 64, 12, 1), first=-1) == 1
    y = torch.zeros(1, 2, 25, 128, dtype=torch.bfloat16).cuda()
    assert status(M.make_shape(1, 2, 25, 128, 64, 12, 1), y, y) == 1         # another head dimension
    odd = torch.zeros(1, 2, 25, 65, dtype=torch.bfloat16).cuda()[..., 1:]
    assert status(M.make_shape(1, 2, 25, 64, 64, 12, 1), odd) == 1           # alignment
    with pytest.raises(ValueError):
        M.mod_rope_fwd(rope.handle, M.make_shape(1, 2, 25, 64, 64, 12, 1), x, x, 0,
                       torch.zeros(2, dtype=torch.int32).cuda())
    # a result whose rows lie on each other; in place under other strides
    s = M.make_shape(1, 2, 24, 64, 64, 12)
    a = torch.zeros(1, 2, 24, 64, dtype=torch.bfloat16).cuda()
    assert status(s, a, a[:, :1].expand(1, 2, 24, 64)) == 1
    assert status(s, a, a.view(-1).as_strided((1, 2, 24, 64), (0, 24 * 64, 32, 1))) == 1
    assert status(s, a, a.view(1, 24, 2, 64).transpose(1, 2)) == 1
    assert status(M.make_shape(1 << 12, 1 << 12, 1, 64, 64), A, A) == 2      # B*H


def test_rope_of_a_broadcast_input(M):
    d, grid = 128, (3, 4, 5)
    rope = M.Rope(M.make_rope_params(d, (44, 42, 42), grid, pairing="halves"))
    x = torch.randn(2, 1, 60, d).bfloat16().cuda().expand(2, 6, 60, d)
    y, want = (torch.empty(2, 6, 60, d, dtype=torch.bfloat16).cuda() for _ in range(2))
    shape = M.make_shape(2, 6, 60, d, 64)
    M.mod_rope_fwd(rope.handle, shape, x, y)
    M.mod_rope_fwd(rope.handle, shape, x.contiguous(), want)
    assert torch.equal(y, want)
