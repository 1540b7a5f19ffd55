"""Host-side checks of the paged cache's entry points: every bad argument is
refused before anything is launched, and the workspace query (no GPU needed:
the addresses are never dereferenced)."""

import ctypes

import pytest
import torch

from paper_2602_07160_amd import binding

OK, NULLPTR, SHAPE, UNSUPPORTED, ALIGN, HIPERR, WORKSPACE = range(7)
A = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def cache(**over):
    x = dict(k=A, v=A, k_scale=A, v_scale=A, pages=4, page=16, heads=2, d_qk=64, d_v=64, type=1)
    x.update(over)
    return binding._Cache(*x.values())


def batch(**over):
    x = dict(q_start=A, lens=A, table=A, n_seq=3, table_len=5, n_tok=7, max_q=7)
    x.update(over)
    return binding._Batch(*x.values())


def fwd(lib, c=None, s=None, q=A, ld=4 * 64, beta=A, out=A, H=4, flags=0, ws=None, n=0):
    c, s = c or cache(), s or batch()
    return lib.fem_paged_fwd(ctypes.byref(c), ctypes.byref(s), q, ld, beta, out, H, flags, ws, n, None)


def append(lib, c=None, s=None, k=A, kld=128, v=A, vld=128):
    c, s = c or cache(), s or batch()
    return lib.fem_cache_append(ctypes.byref(c), ctypes.byref(s), k, kld, v, vld, None)


def gather(lib, c=None, s=None, k=A, v=A, L=9):
    c, s = c or cache(), s or batch()
    return lib.fem_cache_gather(ctypes.byref(c), ctypes.byref(s), k, v, L, None)


CALLS = [fwd, append, gather]


@pytest.mark.parametrize("call", CALLS)
def test_cache_is_checked(lib, call):
    for name in ("k", "v", "k_scale", "v_scale"):
        assert call(lib, cache(**{name: None})) == NULLPTR, name
    for name in ("pages", "page", "heads", "d_qk", "d_v"):
        assert call(lib, cache(**{name: 0})) == SHAPE, name
        assert call(lib, cache(**{name: -1})) == SHAPE, name
    for page in (1, 8, 24, 48, 2048):
        assert call(lib, cache(page=page)) == UNSUPPORTED, page
    for t in (-1, 3):
        assert call(lib, cache(type=t)) == UNSUPPORTED
    for d, dv in ((16, 16), (64, 128), (128, 32), (96, 96), (256, 256)):
        assert call(lib, cache(d_qk=d, d_v=dv)) == UNSUPPORTED, (d, dv)
    assert call(lib, cache(heads=70000)) == SHAPE
    assert call(lib, cache(pages=1 << 30, heads=1 << 10)) == SHAPE
    assert call(lib, cache(k=A + 8)) == ALIGN
    assert call(lib, cache(v=A + 4)) == ALIGN
    assert call(lib, cache(k_scale=A + 4)) == ALIGN
    assert call(lib, cache(v_scale=A + 8)) == ALIGN


@pytest.mark.parametrize("call", CALLS)
def test_batch_is_checked(lib, call):
    for name in ("lens", "table"):
        assert call(lib, s=batch(**{name: None})) == NULLPTR, name
    for name in ("n_seq", "table_len"):
        assert call(lib, s=batch(**{name: 0})) == SHAPE, name
    assert call(lib, s=batch(n_seq=65536)) == SHAPE
    assert call(lib, s=batch(table_len=(1 << 22) + 1)) == SHAPE  # more than 2^26 tokens
    if call is not gather:
        assert call(lib, s=batch(q_start=None)) == NULLPTR
        for name in ("n_tok", "max_q"):
            assert call(lib, s=batch(**{name: 0})) == SHAPE, name


def test_null_structs(lib):
    c, s = ctypes.byref(cache()), ctypes.byref(batch())
    assert lib.fem_cache_append(None, s, A, 128, A, 128, None) == NULLPTR
    assert lib.fem_cache_gather(c, None, A, A, 9, None) == NULLPTR
    assert lib.fem_paged_fwd(None, s, A, 256, A, A, 4, 0, None, 0, None) == NULLPTR
    assert lib.fem_paged_workspace_bytes(None, s, 4) == 0
    assert lib.fem_paged_workspace_bytes(c, None, 4) == 0


def test_append_arguments(lib):
    assert append(lib, k=None) == NULLPTR
    assert append(lib, v=None) == NULLPTR
    assert append(lib, kld=120) == SHAPE   # shorter than a token
    assert append(lib, vld=132) == SHAPE   # not a multiple of 8
    assert append(lib, k=A + 8) == ALIGN
    assert append(lib, v=A + 2) == ALIGN


def test_gather_arguments(lib):
    assert gather(lib, k=None, v=None) == NULLPTR
    assert gather(lib, L=0) == SHAPE
    assert gather(lib, L=-5) == SHAPE
    assert gather(lib, v=A + 8) == ALIGN


def test_read_arguments(lib):
    assert fwd(lib, q=None) == NULLPTR
    assert fwd(lib, beta=None) == NULLPTR
    assert fwd(lib, out=None) == NULLPTR
    assert fwd(lib, H=0) == SHAPE
    assert fwd(lib, H=3) == SHAPE          # not a multiple of the cached heads
    assert fwd(lib, ld=4 * 64 - 8) == SHAPE
    assert fwd(lib, ld=4 * 64 + 4) == SHAPE
    assert fwd(lib, flags=4) == UNSUPPORTED
    assert fwd(lib, q=A + 8) == ALIGN
    assert fwd(lib, out=A + 8) == ALIGN
    need = lib.fem_paged_workspace_bytes(ctypes.byref(cache(page=256)), ctypes.byref(batch()), 4)
    assert need > 0
    c = cache(page=256)
    assert fwd(lib, c) == WORKSPACE
    assert fwd(lib, c, ws=A, n=need - 1) == WORKSPACE
    assert fwd(lib, c, ws=A + 16, n=need) == ALIGN


def test_too_many_workgroups(lib):
    c, s = cache(heads=65535, pages=1), batch(n_seq=65535, n_tok=1 << 14, max_q=1 << 14)
    assert fwd(lib, c, s, H=65535, ld=65535 * 64, ws=A, n=1 << 60) == SHAPE


def test_workspace_is_a_function_of_the_sizes(lib):
    def need(H=4, **over):
        return lib.fem_paged_workspace_bytes(ctypes.byref(cache(page=1024)),
                                             ctypes.byref(batch(**over)), H)

    assert need() == need(lens=A + 4, table=A + 8)
    assert need(H=3) == 0 and need(H=-4) == 0 and need(n_tok=0) == 0
    assert need(n_seq=64, n_tok=64, max_q=1) <= 64 << 20


def test_binding_refuses():
    with pytest.raises(ValueError):
        binding.PagedCache(torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16),
                           torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16))  # not on a GPU
    with pytest.raises(ValueError):
        binding.PagedCache(torch.zeros(2, 2, 16, 64), torch.zeros(2, 2, 16, 64))
    with pytest.raises(ValueError):
        binding.PagedBatch(None, torch.zeros(2, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError):
        binding.fem_paged_fwd(None, None, None, None)
