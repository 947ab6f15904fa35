"""What the paged cache refuses before anything is enqueued, through the C ABI and the binding, without a GPU."""
import ctypes

import pytest
import torch

import __graft_entry__ as entry
from paper_2607_27744_b200 import binding

INVALID, ALIGN, UNSUPPORTED, WORKSPACE = -1, -2, -3, -5
P = ctypes.c_void_p(1 << 20)          # stands for device memory: nothing here is read through


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(binding.LIB_PATH):
        entry.build()
    L = ctypes.CDLL(binding.LIB_PATH)
    i32, i64, vp, sz, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
    L.rocs_cache_create.argtypes = [ctypes.POINTER(vp), ctypes.c_int, i32, i32, i32, i32, i32, vp, vp, i64, i64, i64, i64, i32, i32,
                                    vp, vp, vp]
    L.rocs_cache_destroy.argtypes = [vp]
    L.rocs_cache_workspace.restype = sz
    L.rocs_cache_workspace.argtypes = [vp, i32]
    L.rocs_cache_fork.argtypes = [vp, i32, vp, vp, vp, vp, sz, vp]
    L.rocs_cache_truncate.argtypes = [vp, i32, vp, vp, vp, vp, sz, vp]
    L.rocs_cache_compact.argtypes = [vp, vp, vp, vp, vp, sz, vp]
    L.rocs_cache_extend.argtypes = [vp, vp, vp, vp, vp, vp, sz, vp]
    L.rocs_cache_append.argtypes = [vp, i32, vp, vp, vp, vp, vp, i64, i64, vp]
    L.rocs_cache_attention_workspace.restype = sz
    L.rocs_cache_attention_workspace.argtypes = [vp, vp, i32]
    L.rocs_cache_attention.argtypes = [vp, i32, vp, vp, i32, vp, i64, i64, i32, f32, f32, vp, vp, vp, vp, i64, i64, vp, sz, vp]
    return L


def create(L, **change):
    a = dict(dtype=0, layers=2, n_pages=10, page=16, H=4, dh=64, K=P, V=P, ld_layer=10 * 16 * 256, ld_page=16 * 256, ld_token=256,
             ld_head=64, n_slots=5, width=7, table=P, lens=P, refs=P)
    a.update(change)
    out = ctypes.c_void_p()
    return L.rocs_cache_create(ctypes.byref(out), *a.values()), out


@pytest.mark.parametrize("change,code", [
    ({}, 0), ({"refs": None}, 0), ({"dtype": 1}, 0), ({"dtype": 2}, INVALID), ({"layers": 0}, INVALID), ({"n_pages": 0}, INVALID),
    ({"page": 0}, INVALID), ({"H": 0}, INVALID), ({"dh": 0}, INVALID), ({"n_slots": 0}, INVALID), ({"width": 0}, INVALID),
    ({"K": None}, INVALID), ({"V": None}, INVALID), ({"table": None}, INVALID), ({"lens": None}, INVALID),
    ({"K": ctypes.c_void_p(1048584)}, ALIGN), ({"lens": ctypes.c_void_p(1048580)}, ALIGN), ({"refs": ctypes.c_void_p(1048580)}, ALIGN),
    ({"dh": 60}, ALIGN), ({"dh": 264, "ld_head": 264, "ld_token": 1056, "ld_page": 16896, "ld_layer": 168960}, UNSUPPORTED),
    ({"ld_token": 252}, ALIGN), ({"ld_token": 248}, INVALID),                       # rows that overlap
    ({"ld_head": 0}, INVALID), ({"ld_page": 16 * 256 - 8}, INVALID), ({"ld_layer": -4096}, INVALID),
    ({"ld_head": 16 * 64, "ld_token": 64}, 0),                                       # heads in front of rows
    ({"ld_layer": 16 * 256, "ld_page": 2 * 16 * 256}, 0),                            # layers inside a page
    ({"width": (1 << 20) + 1, "page": 1}, UNSUPPORTED), ({"width": 1 << 20, "page": 2048, "ld_page": 2048 * 256, "ld_layer": 10 * 2048 * 256}, UNSUPPORTED),
])
def test_what_a_cache_may_be(lib, change, code):
    got, handle = create(lib, **change)
    assert got == code
    assert bool(handle) == (code == 0)
    lib.rocs_cache_destroy(handle)


@pytest.mark.parametrize("page,width,code", [(1 << 10, 1 << 20, 0), ((1 << 10) + 1, 1 << 20, UNSUPPORTED), (65537, 16383, 0), (65537, 16384, UNSUPPORTED),
                                             (65537, 32767, UNSUPPORTED)])
def test_how_long_a_slot_may_be(lib, page, width, code):
    """Positions stay far enough below 2^31 that the end of their last page or block does too."""
    got, handle = create(lib, page=page, width=width, H=1, ld_head=0, ld_token=64, ld_page=64 * page, ld_layer=640 * page)
    assert got == code
    lib.rocs_cache_destroy(handle)


def test_calls_on_a_cache(lib):
    _, c = create(lib)
    _, bare = create(lib, refs=None)
    need = lib.rocs_cache_workspace(c, 4)
    assert need > 0 and need % 256 == 0 and lib.rocs_cache_workspace(c, -1) == 0 and lib.rocs_cache_workspace(None, 4) == 0
    assert lib.rocs_cache_fork(c, -1, P, P, None, P, need, None) == INVALID
    assert lib.rocs_cache_fork(c, 4, None, P, None, P, need, None) == INVALID
    assert lib.rocs_cache_fork(c, 4, P, None, None, P, need, None) == INVALID
    assert lib.rocs_cache_fork(c, 4, P, P, None, None, need, None) == WORKSPACE
    assert lib.rocs_cache_fork(c, 4, P, P, None, P, need - 1, None) == WORKSPACE
    assert lib.rocs_cache_fork(c, 4, P, P, None, ctypes.c_void_p((1 << 20) + 16), need, None) == WORKSPACE
    assert lib.rocs_cache_fork(bare, 4, P, P, None, P, need, None) == INVALID       # nobody counts the holders
    assert lib.rocs_cache_truncate(c, 4, None, None, None, P, need, None) == INVALID
    assert lib.rocs_cache_truncate(None, 4, P, None, None, P, need, None) == INVALID
    assert lib.rocs_cache_compact(c, ctypes.c_void_p((1 << 20) + 4), None, None, P, need, None) == ALIGN
    assert lib.rocs_cache_compact(bare, None, None, None, P, need, None) == INVALID
    assert lib.rocs_cache_extend(c, None, None, P, None, P, need, None) == INVALID
    assert lib.rocs_cache_append(c, 0, None, None, P, P, P, 256, 64, None) == INVALID
    assert lib.rocs_cache_attention(c, 0, None, None, 4, P, 256, 64, 1, 0.0, 0.0, None, None, None, P, 256, 64, P, 1 << 30, None) == INVALID
    assert lib.rocs_cache_attention_workspace(c, None, 4) == 0
    lib.rocs_cache_destroy(c)
    lib.rocs_cache_destroy(bare)
    lib.rocs_cache_destroy(None)


def test_the_binding_takes_tensors_of_the_gpu_only():
    K, t, n = torch.zeros(3, 16, 1, 64), torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises((AssertionError, RuntimeError)):
        binding.cache_create(K, K, t, n)
    with pytest.raises(TypeError):
        binding.cache_create(K.half(), K.half(), t, n)
    with pytest.raises(AssertionError):
        binding.cache_create(K, K.bfloat16(), t, n)
    with pytest.raises(AssertionError):
        binding.cache_create(K, K.transpose(0, 1).contiguous().transpose(0, 1), t, n)
    with pytest.raises(ValueError):
        binding.cache_create(K[0], K[0], t, n)
    closed = type("C", (), {"spec": None})
    plan = type("P", (), {"handle": None, "R": 1, "N": 4})
    for call in (lambda: binding.cache_attention(closed, plan, K), lambda: binding.cache_fork(closed, n, n),
                 lambda: binding.cache_truncate(closed, n), lambda: binding.cache_compact(closed),
                 lambda: binding.cache_extend(closed, plan), lambda: binding.cache_append(closed, plan, n, K, K)):
        with pytest.raises(ValueError, match="closed"):
            call()


def test_how_many_pages_and_slots_are_counted(lib):
    """Kernels go over pages and slots some thousands at a time, in 32 bits."""
    most = (1 << 31) - (1 << 13) - 1
    for name in ("n_pages", "n_slots"):
        small = dict(page=1, H=1, layers=1, dh=8, ld_head=0, ld_token=0, ld_page=8, ld_layer=0)
        got, handle = create(lib, **small, **{name: most})
        assert got == 0
        lib.rocs_cache_destroy(handle)
        got, handle = create(lib, **small, **{name: most + 1})
        assert got == UNSUPPORTED and not handle
    _, c = create(lib)
    for n in (most + 1, (1 << 31) - 1):
        assert lib.rocs_cache_fork(c, n, P, P, None, P, 1 << 40, None) == UNSUPPORTED
        assert lib.rocs_cache_truncate(c, n, P, None, None, P, 1 << 40, None) == UNSUPPORTED
    lib.rocs_cache_destroy(c)
