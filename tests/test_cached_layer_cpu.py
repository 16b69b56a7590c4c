"""The cached layer's entry points reject bad arguments on the host, before
the device is touched (no GPU needed)."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20   # an aligned address that is never used


@pytest.fixture(scope="module")
def M():
    import paper_2601_11641_amd as m
    return m


def refused(M, call, *args):
    with pytest.raises(M.ModError) as e:
        call(*args)
    assert M.mod_last_error()
    return e.value.status


@pytest.mark.parametrize("change,status", [
    (dict(d=96), 2),
    (dict(dims=(15, 24, 24)), 1),        # odd width
    (dict(dims=(-2, 24, 24)), 1),
    (dict(dims=(0, 0, 0)), 1),           # nothing to rotate
    (dict(dims=(32, 24, 24)), 1),        # more channels than the head has
    (dict(grid=(0, 4, 4)), 1),
    (dict(grid=(1 << 15, 1 << 10, 1 << 10)), 2),
    (dict(grid=(1 << 30, 1, 1)), 2),     # tables too large
    (dict(theta=1.0), 1),
    (dict(theta=float("nan")), 1),
    (dict(theta=float("inf")), 1),
    (dict(pairing=2), 1),
])
def test_rope_create_refuses(M, change, status):
    p = dict(d=64, dims=(16, 24, 24), grid=(4, 8, 8), theta=10000.0, pairing="adjacent")
    p.update(change)
    assert refused(M, M.mod_rope_create, M.make_rope_params(**p)) == status
    assert M.raw_lib().mod_rope_create(None, ctypes.byref(ctypes.c_void_p())) == 1
    assert M.raw_lib().mod_rope_create(None, None) == 1


def test_rope_calls_refuse_null(M):
    s = M.make_shape(1, 2, 4, 64, 64)
    for f in (M.mod_rope_fwd, M.mod_rope_bwd):
        assert refused(M, f, None, s, A, A, 0, None, 0) == 1
    M.mod_rope_destroy(None)


@pytest.mark.parametrize("shape,status", [
    ((0, 2, 100, 64, 64), 1), ((1, 0, 100, 64, 64), 1), ((1, 2, 0, 64, 64), 1),
    ((1, 2, 100, 96, 64), 2), ((1, 2, 100, 64, 32), 2), ((1, 2, (1 << 24) + 1, 64, 64), 2),
    ((1 << 12, 1 << 12, 100, 64, 64), 2), ((1, 2, 100, 64, 64, 2), 1),
])
def test_cache_shapes_refused(M, shape, status):
    s = M.make_cache_shape(*shape)
    c = M.mod_cache(A, A, A, A)
    assert M.mod_cache_blocks(s) == 0 and M.mod_cache_attn_workspace_bytes(s, 2, 1, 1) == 0
    assert refused(M, M.mod_cache_write, s, c, A, A, 0, None, None, 1, 0) == status
    assert refused(M, M.mod_cache_read, s, c, A, A, 0, None, None, 1, 0) == status
    assert refused(M, M.mod_cache_attn_fwd, s, c, A, 1, None, None, None, 0.0, A, None, None, 0, 0, 2, 1) == status


def test_cache_blocks(M):
    assert M.mod_cache_blocks(M.make_cache_shape(1, 2, 129, 64, 128)) == 2
    assert M.mod_cache_blocks(M.make_cache_shape(1, 2, 128, 64, 64)) == 2
    assert M.mod_cache_blocks(None) == 0


@pytest.mark.parametrize("L,first,starts,k,v", [
    (0, 0, None, A, A), (-1, 0, None, A, A), (1, -1, None, A, A), (101, 0, None, A, A), (60, 41, None, A, A),
    (2 ** 31 - 1, 2 ** 31 - 1, None, A, A), (101, 0, A, A, A), (1, 0, None, A + 8, A), (1, 0, None, A, A + 2),
])
def test_cache_ranges_refused(M, L, first, starts, k, v):
    s, c = M.make_cache_shape(2, 2, 100, 64, 64), M.mod_cache(A, A, A, A)
    for f in (M.mod_cache_write, M.mod_cache_read):
        assert refused(M, f, s, c, k, v, first, starts, None, L, 0) == 1


def test_cache_pointers_and_strides_refused(M):
    lib, s = M.raw_lib(), M.make_cache_shape(1, 2, 100, 64, 64)
    good = M.mod_cache(A, A, A, A)
    def write(cache, k, v, ks=None, vs=None):
        return lib.mod_cache_write(ctypes.byref(s), cache and ctypes.byref(cache), k, ks and ctypes.byref(ks), v,
                                   vs and ctypes.byref(vs), 1, 0, None, None, None)
    assert write(None, A, A) == 1
    assert write(good, None, A) == 1 and write(good, A, None) == 1
    for bad in ((0, A, A, A), (A, 0, A, A), (A, A, 0, A), (A, A, A, 0), (A + 8, A, A, A), (A, A + 1, A, A)):
        assert write(M.mod_cache(*bad), A, A) == 1
    for st in ((1, 0, 0), (0, 4, 0), (0, 0, 12)):
        assert write(good, A, A, M.mod_strides(*st)) == 1 and write(good, A, A, None, M.mod_strides(*st)) == 1
    assert lib.mod_cache_read(ctypes.byref(s), ctypes.byref(good), None, None, None, None, 1, 0, None, None,
                              None) == 1


@pytest.mark.parametrize("change,status", [
    (dict(Hq=3), 1), (dict(Hq=0), 1), (dict(Lq=0), 1), (dict(max_len=-1), 1), (dict(max_len=101), 1),
    (dict(q=None), 1), (dict(o=None), 1), (dict(q=A + 2), 1), (dict(o=A + 8), 1), (dict(kv_idx=A), 1),
    (dict(kv_cnt=A), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(Lq=(1 << 24) + 1), 2), (dict(Lq=1 << 24, Hq=16), 2),
])
def test_attention_refused(M, change, status):
    s, c = M.make_cache_shape(1, 2, 100, 64, 64), M.mod_cache(A, A, A, A)
    p = dict(q=A, max_len=100, kv_len=None, kv_idx=None, kv_cnt=None, scale=0.0, o=A, lse=None, workspace=A,
             ws_bytes=1 << 40, stream=0, Hq=4, Lq=1)
    p.update(change)
    assert refused(M, lambda: M.mod_cache_attn_fwd(s, c, **p)) == status


@pytest.mark.parametrize("strides", [(0, 1024, 64), (1024, 0, 64), (2048, 1024, 0), (2048, 1024, 32),
                                     (2048, -56, 64), (-8, 1024, 64)])
def test_read_into_overlapping_rows_refused(M, strides):
    lib, s = M.raw_lib(), M.make_cache_shape(2, 2, 100, 64, 64)
    c, st = M.mod_cache(A, A, A, A), ctypes.byref(M.mod_strides(*strides))
    for ks, vs in ((st, None), (None, st)):
        assert lib.mod_cache_read(ctypes.byref(s), ctypes.byref(c), A, ks, A, vs, 16, 0, None, None, None) == 1


def test_attention_workspace(M):
    s, c = M.make_cache_shape(1, 2, 100000, 128, 128), M.mod_cache(A, A, A, A)
    need = M.mod_cache_attn_workspace_bytes(s, 2, 1, 100000)
    assert 0 < need < 256 << 20
    args = dict(q=A, max_len=100000, kv_len=None, kv_idx=None, kv_cnt=None, scale=0.0, o=A, stream=0, Hq=2, Lq=1)
    assert refused(M, lambda: M.mod_cache_attn_fwd(s, c, workspace=A, ws_bytes=need - 1, **args)) == 1
    assert refused(M, lambda: M.mod_cache_attn_fwd(s, c, workspace=None, ws_bytes=need, **args)) == 1
    assert refused(M, lambda: M.mod_cache_attn_fwd(s, c, workspace=A + 4, ws_bytes=need, **args)) == 1
    # a short cache needs none
    assert M.mod_cache_attn_workspace_bytes(s, 2, 1, 10) == 0
    assert M.mod_cache_attn_workspace_bytes(s, 3, 1, 100) == 0 and M.mod_last_error()


def test_binding_checks_tensors(M):
    torch = pytest.importorskip("torch")
    s = M.make_cache_shape(1, 2, 100, 64, 64)
    x = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16)
    c = M.mod_cache(A, A, A, A)
    for bad in (x, x.float(), x[:, :, :, :32], x.transpose(2, 3)):
        with pytest.raises(ValueError):
            M.mod_cache_write(s, c, bad, bad, stream=0)
    with pytest.raises(ValueError):
        M.make_cache(x, x, x, x)
    with pytest.raises(ValueError):
        M.mod_cache_attn_fwd(s, c, x, 100, None, None, None, 0.0, x[:, :1], stream=0)
    with pytest.raises(ValueError):   # a workspace smaller than its stated size
        M.mod_cache_attn_fwd(s, c, A, 100, None, None, None, 0.0, A, None, x, x.nbytes + 1, stream=0, Hq=2, Lq=1)
    # addresses need their sizes
    with pytest.raises(TypeError):
        M.mod_cache_attn_fwd(s, c, A, 100, None, None, None, 0.0, A, stream=0)
    with pytest.raises(TypeError):
        M.mod_cache_write(s, c, A, A, stream=0)
    assert refused(M, lambda: M.mod_cache_read(s, c, None, None, stream=0)) == 1


def test_struct_layouts_match_the_header(M, tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    names = {"mod_strides": "bhl", "mod_rope_params": ("d", "dims", "frames", "height", "width", "theta", "pairing"),
             "mod_cache_shape": ("B", "H", "capacity", "d", "block", "format"),
             "mod_cache": ("k", "v", "k_scale", "v_scale")}
    lines = "".join(f'printf("%zu\\n", sizeof({t}));' + "".join(f'printf("%zu\\n", offsetof({t}, {f}));' for f in fs)
                    for t, fs in names.items())
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "moddit.h"\nint main(void) {' + lines +
                   ' return 0; }\n')
    exe = tmp_path / "layout"
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for t, fs in names.items():
        cls = getattr(M, t)
        want += [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f in fs]
    assert got == want


@pytest.fixture
def anywhere(M, monkeypatch):
    """Tensors of the host stand for tensors of the current device."""
    monkeypatch.setattr(M._capi, "_device", lambda x, what: None)
    monkeypatch.setattr(M._capi, "_current_device", lambda: -1)
    return monkeypatch


def calls(M, s, c):
    """Calls with that cache that get past the binding's checks and no further:
    a length, then a query head count that the library refuses."""
    return [lambda: M.mod_cache_write(s, c, A, A, 0, None, None, 0, 0), lambda: M.mod_cache_read(s, c, A, A, 0, None, None, 0, 0),
            lambda: M.mod_cache_attn_fwd(s, c, A, 1, None, None, None, 0.0, A, None, None, 0, 0, 0, 1)]


@pytest.mark.parametrize("shape", [
    (1, 2, 201, 64, 64), (1, 2, 200, 128, 64), (1, 2, 200, 64, 128), (2, 2, 200, 64, 64), (1, 3, 200, 64, 64),
    (1, 2, 1 << 24, 64, 64), (1, 2, 199, 64, 64), (2, 1, 200, 64, 64), (1, 2, 100, 128, 64),
])
def test_cache_of_another_shape_refused(M, anywhere, shape):
    """The tensors that a cache was made of are those of the call's shape: larger
    ones would be read and written past their end, others in the wrong places."""
    torch = pytest.importorskip("torch")
    codes = lambda *n: torch.zeros(n, dtype=torch.uint8)   # noqa: E731
    c = M.make_cache(codes(1, 2, 200, 64), codes(1, 2, 200, 64), torch.zeros(1, 2, 4), torch.zeros(1, 2, 4))
    for call in calls(M, M.make_cache_shape(1, 2, 200, 64, 64), c):
        assert refused(M, call) == 1
    for call in calls(M, M.make_cache_shape(*shape), c):
        with pytest.raises(ValueError):
            call()


def test_cache_of_one_dimension_and_of_addresses(M, anywhere):
    torch = pytest.importorskip("torch")
    s, f32 = M.make_cache_shape(1, 2, 200, 64, 64), torch.float32
    flat = lambda n, t: torch.zeros(n, dtype=t)            # noqa: E731
    for kn, vn, ksn, vsn, fits in ((25600, 25600, 8, 8, True), (30000, 25600, 9, 8, True), (25599, 25600, 8, 8, False),
                                   (25600, 25599, 8, 8, False), (25600, 25600, 7, 8, False), (25600, 25600, 8, 7, False)):
        c = M.make_cache(flat(kn, torch.uint8), flat(vn, torch.uint8), flat(ksn, f32), flat(vsn, f32))
        for call in calls(M, s, c):
            if fits:
                assert refused(M, call) == 1
            else:
                with pytest.raises(ValueError):
                    call()
    # addresses are taken as they are, also where one is put into the struct later
    for call in calls(M, s, M.make_cache(A, A, A, A)):
        assert refused(M, call) == 1
    c = M.make_cache(flat(25599, torch.uint8), flat(25600, torch.uint8), flat(8, f32), flat(8, f32))
    c.k = A
    for call in calls(M, s, c):
        assert refused(M, call) == 1


def test_cache_of_another_device_refused(M, anywhere):
    torch = pytest.importorskip("torch")
    codes = torch.zeros(1, 2, 200, 64, dtype=torch.uint8)
    c = M.make_cache(codes, codes.clone(), torch.zeros(1, 2, 4), torch.zeros(1, 2, 4))
    anywhere.setattr(M._capi, "_current_device", lambda: 1)
    for call in calls(M, M.make_cache_shape(1, 2, 200, 64, 64), c):
        with pytest.raises(ValueError):
            call()


def test_shapes_without_a_block_refused(M):
    s, c = M.make_cache_shape(1, 2, 200, 64, 0), M.mod_cache(A, A, A, A)
    for call in calls(M, s, c):
        assert refused(M, call) == 2


def test_cache_of_merged_axes(M, anywhere):
    """[B * H, capacity, d] and [B * H, n] hold the same in the same order."""
    torch = pytest.importorskip("torch")
    s = M.make_cache_shape(2, 3, 200, 64, 64)
    for codes, scales, fits in (((6, 200, 64), (6, 4), True), ((1200, 64), (24,), True), ((6, 201, 64), (6, 4), False),
                                ((6, 199, 64), (6, 4), False), ((6, 200, 64), (6, 5), False), ((6, 200, 64), (6, 3), False),
                                ((3, 2, 200, 64), (6, 4), False), ((6, 200, 64), (3, 2, 4), False)):
        c = M.make_cache(*(torch.zeros(codes, dtype=torch.uint8) for _ in range(2)), *(torch.zeros(scales) for _ in range(2)))
        for call in calls(M, s, c):
            if fits:
                assert refused(M, call) == 1
            else:
                with pytest.raises(ValueError):
                    call()
