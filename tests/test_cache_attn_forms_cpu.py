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
