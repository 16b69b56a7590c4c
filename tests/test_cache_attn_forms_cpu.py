"""Which kernel the attention tests reach: the rows of a tile and the parts of a
walk that the library chooses for their sizes (no GPU needed)."""
import ctypes

import pytest

import test_gpu_cache_attn as T

# rows of a tile per case of MANY_ROWS
ROWS = [256] * 2 + [128] * 8 + [64] * 6 + [32] * 7 + [16] * 2


@pytest.fixture(scope="module")
def M():
    import paper_2601_11641_amd as m
    return m


def plan(M, d, block, B, H, group, Lq, L, lists):
    return M.mod_cache_attn_plan(M.make_cache_shape(B, H, L, d, block, "int8"), H * group, Lq, L, lists)


def test_many_rows_take_every_tile(M):
    forms = [plan(M, *c) for c in T.MANY_ROWS]
    assert [r for r, _ in forms] == ROWS
    whole, parts = {r for r, c in forms if c == 1}, {r for r, c in forms if c > 1}
    assert whole == parts == {16, 32, 64, 128, 256}
    # more than eight parts are joined in slices; with lists and without
    assert {r for r, c in forms if c > 8} >= {64, 128}
    for lists in (False, True):
        assert {r for (r, _), c in zip(forms, T.MANY_ROWS) if c[-1] == lists} == ({16, 32, 64, 128} if lists else
                                                                                  {16, 32, 64, 128, 256})


def test_single_tokens_take_the_smallest_tile(M):
    """Up to 16 rows that share a key/value head, whatever the sizes (the
    probabilities there are two bf16 each)."""
    for d in (64, 128):
        for rows in (1, 2, 15, 16):
            for L in (1, 100, 9000, 118800):
                for B, H in ((1, 1), (1, 24), (8, 40)):
                    for lists in (False, True):
                        assert plan(M, d, 128, B, H, 1, rows, L, lists)[0] == 16
                    assert plan(M, d, 128, B, H, rows, 1, L, False)[0] == 16


def test_plan_refusals(M):
    s = M.make_cache_shape(1, 2, 100, 64, 64, "int8")
    for bad in ((3, 1, 100), (2, 0, 100), (2, 1, 101), (2, 1, -1)):
        with pytest.raises(M.ModError):
            M.mod_cache_attn_plan(s, *bad)
    lib, n = M.raw_lib(), ctypes.c_int()
    for rows, parts in ((None, n), (n, None)):
        assert lib.mod_cache_attn_plan(ctypes.byref(s), 2, 1, 100, 0, rows and ctypes.byref(rows),
                                       parts and ctypes.byref(parts)) == 1
    assert M.mod_cache_attn_plan(s, 2, 1, 0) == (16, 1)


def call_bytes(B, H, Hq, Lq, L, d):
    """Codes of the call's tokens, q and o; 256 MB at least."""
    return max(256e6, B * d * (2 * H * L + 4 * Hq * Lq))


@pytest.mark.parametrize("B,H,Hq,Lq,L,d,most", [
    (1, 24, 24, 10800, 118800, 128, 600e6),      # a chunk of three frames: under its cache's 730 MB
    (1, 24, 24, 10800, 118800, 64, 300e6),
    (1, 24, 24, 3600, 118800, 128, 340e6),
    (7, 2, 16, 7447, 127292, 128, 1300e6),
    (7, 2, 16, 3000, 60000, 128, 600e6),
])
def test_workspace_of_many_rows_is_worth_it(M, B, H, Hq, Lq, L, d, most):
    s = M.make_cache_shape(B, H, L, d, 128, "int8")
    assert M.mod_cache_attn_workspace_bytes(s, Hq, Lq, L) <= most


def test_workspace_is_bounded(M):
    """By three times the bytes of the call's own tensors, and 2.2 GB."""
    for B in (1, 3, 16):
        for H, Hq in ((1, 1), (1, 16), (5, 40), (24, 24), (46, 92)):
            for Lq in (1, 17, 300, 2444, 9621):
                for L in (100, 9241, 34672, 90719, 250000):
                    for d, block in ((64, 64), (128, 128)):
                        s = M.make_cache_shape(B, H, L, d, block, "int8")
                        need = M.mod_cache_attn_workspace_bytes(s, Hq, Lq, L)
                        assert need <= min(2.2e9, 3 * call_bytes(B, H, Hq, Lq, L, d)), (B, H, Hq, Lq, L, d)
