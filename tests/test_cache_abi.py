"""The cache's entry points without a GPU: sizes, and everything they refuse before a launch."""
import ctypes
import os

import pytest
import torch


@pytest.fixture(scope="module")
def P():
    import paper_2604_12219_amd as P
    if not os.path.exists(P.lib_path()):
        from paper_2604_12219_amd.build import build
        build()
    P.load_library()
    return P


EINVAL, EUNSUPPORTED, EWORKSPACE, EALIGN = -1, -2, -3, -4
A, B_, BIG = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), ctypes.c_size_t(1 << 62)  # never dereferenced


def _cache(P, **kw):
    return P.Cache(**{**dict(H_kv=2, d=128, n_pages=9, max_pages=4, group=32, page=64), **kw})


def _shape(P, **kw):
    base = dict(B=1, H=2, n=100, d=128, block=64, group=32, stride_n=128)
    base.update(kw)
    base.setdefault("stride_h", max(base["n"], 1) * base["stride_n"])
    base.setdefault("stride_b", base["H"] * base["stride_h"])
    return P.Shape(**base)


@pytest.mark.parametrize("d, group, token", [(64, 32, 80), (64, 64, 72), (128, 32, 160), (128, 64, 144), (128, 128, 136)])
def test_sizes(P, d, group, token):
    assert P.cache_bytes(_cache(P, d=d, group=group, page=16)) == 9 * 2 * 16 * token
    assert P.cache_bytes(_cache(P, d=d, group=group, n_pages=1 << 20, H_kv=40)) == (1 << 20) * 40 * 64 * token  # beyond 32 bits


BAD_CACHES = [(dict(H_kv=0), EINVAL), (dict(n_pages=0), EINVAL), (dict(max_pages=0), EINVAL), (dict(d=96), EUNSUPPORTED), (dict(group=16), EUNSUPPORTED),
              (dict(group=48), EUNSUPPORTED), (dict(d=64, group=128), EUNSUPPORTED), (dict(page=8), EUNSUPPORTED), (dict(page=48), EUNSUPPORTED),
              (dict(page=1 << 17), EUNSUPPORTED), (dict(page=-64), EUNSUPPORTED), (dict(page=64, max_pages=1 << 25), EUNSUPPORTED),
              (dict(H_kv=1 << 17), EUNSUPPORTED), (dict(H_kv=65535, n_pages=2**31 - 1), EUNSUPPORTED)]


@pytest.mark.parametrize("bad, status", BAD_CACHES)
def test_bad_descriptions(P, bad, status):
    L, c, s = P.load_library(), _cache(P, **bad), _shape(P, d=bad.get("d", 128))
    cr, sr = ctypes.byref(c.c()), ctypes.byref(s.c())
    assert L.pasa_cache_bytes(cr) == 0 and L.pasa_cache_attn_workspace_bytes(sr, cr, 0) == 0
    with pytest.raises(ValueError):
        P.cache_bytes(c)
    if bad.get("d") != 96:
        assert L.pasa_cache_write(A, B_, sr, cr, A, BIG, A, A, None, None) == status
        assert L.pasa_cache_read(sr, cr, A, BIG, A, A, None, A, B_, None) == status
        assert L.pasa_cache_attn(A, sr, cr, A, BIG, A, A, None, 0, 0, B_, None, A, BIG, None) == status


def test_arguments_are_checked_before_any_launch(P):
    L = P.load_library()
    odd4, odd16 = ctypes.c_void_p(0x1002), ctypes.c_void_p(0x1008)

    def all_three(status, shape=None, cache=None, attn_shape=None, **kw):
        c = ctypes.byref((cache or _cache(P)).c())
        s = ctypes.byref((shape or _shape(P)).c())
        a = dict(pool=A, nbytes=BIG, pages=A, length=A, n_new=None)
        a.update(kw)
        tail = (a["pool"], a["nbytes"], a["pages"], a["length"], a["n_new"])
        assert L.pasa_cache_write(A, B_, s, c, *tail, None) == status
        assert L.pasa_cache_read(s, c, *tail, A, B_, None) == status
        assert L.pasa_cache_attn(A, s, c, *tail, 0, 0, B_, None, A, BIG, None) == status

    all_three(EINVAL, pool=None)
    all_three(EINVAL, pages=None)
    all_three(EINVAL, length=None)
    all_three(EALIGN, pool=odd16)
    all_three(EALIGN, pages=odd4)
    all_three(EALIGN, length=odd4)
    all_three(EALIGN, n_new=odd4)
    all_three(EWORKSPACE, nbytes=ctypes.c_size_t(P.cache_bytes(_cache(P)) - 1))
    all_three(EINVAL, shape=_shape(P, n=0))
    all_three(EINVAL, shape=_shape(P, d=64, stride_n=128))  # the cache's d is another
    all_three(EUNSUPPORTED, shape=_shape(P, d=96))
    all_three(EALIGN, shape=_shape(P, stride_n=132))
    all_three(EINVAL, shape=_shape(P, scale=float("nan")))
    all_three(EUNSUPPORTED, shape=_shape(P, n=1 << 24, stride_n=256))
    all_three(EINVAL, shape=_shape(P, H=3))  # neither H_kv nor a multiple of it
    c, s = ctypes.byref(_cache(P).c()), ctypes.byref(_shape(P).c())
    two = ctypes.byref(_shape(P, H=4).c())
    mid = (A, BIG, A, A, None)
    assert L.pasa_cache_write(A, B_, None, c, *mid, None) == EINVAL and L.pasa_cache_write(A, B_, s, None, *mid, None) == EINVAL
    # write and read take the key/value heads themselves
    assert L.pasa_cache_write(A, B_, two, c, *mid, None) == EINVAL and L.pasa_cache_read(two, c, *mid, A, B_, None) == EINVAL
    assert L.pasa_cache_write(None, B_, s, c, *mid, None) == EINVAL and L.pasa_cache_write(A, None, s, c, *mid, None) == EINVAL
    assert L.pasa_cache_write(odd16, B_, s, c, *mid, None) == EALIGN and L.pasa_cache_write(A, odd16, s, c, *mid, None) == EALIGN
    assert L.pasa_cache_read(s, c, *mid, None, B_, None) == EINVAL and L.pasa_cache_read(s, c, *mid, A, A, None) == EINVAL
    assert L.pasa_cache_read(s, c, *mid, odd16, B_, None) == EALIGN

    def attn(status, q=A, out=B_, lse=None, ws=A, nbytes=BIG, n_max=0):
        assert L.pasa_cache_attn(q, s, c, *mid, 1, n_max, out, lse, ws, nbytes, None) == status

    attn(EINVAL, q=None)
    attn(EINVAL, out=None)
    attn(EINVAL, out=A)  # aliases q
    attn(EINVAL, ws=None)
    attn(EINVAL, n_max=-1)
    attn(EALIGN, q=odd16)
    attn(EALIGN, out=odd16)
    attn(EALIGN, ws=odd16)
    attn(EALIGN, lse=odd4)
    attn(EWORKSPACE, nbytes=ctypes.c_size_t(0))


def test_rows_that_cannot_be_numbered_are_refused(P):
    """2^31 (row, head) pairs of one key/value head"""
    L = P.load_library()
    c, s = ctypes.byref(_cache(P, H_kv=1).c()), ctypes.byref(_shape(P, H=65535, n=1 << 15, stride_h=128, stride_n=128).c())
    assert L.pasa_cache_attn_workspace_bytes(s, c, 0) == 0
    assert L.pasa_cache_attn(A, s, c, A, BIG, A, A, None, 0, 0, B_, None, A, BIG, None) == EUNSUPPORTED


@pytest.mark.parametrize("B, H, H_kv, n", [(1, 1, 1, 1), (65535, 1, 1, 1), (1, 65535, 65535, 9), (1, 65535, 1, 1), (1, 8, 8, 1 << 23), (255, 257, 1, 16), (4095, 16, 2, 100)])
@pytest.mark.parametrize("n_max", [0, 1, 1000, 2 ** 31 - 1])
def test_workspaces_at_the_ends_of_the_ranges(P, B, H, H_kv, n, n_max):
    """at most 64 parts of every row, or two parts of 256 rows of 256 workgroups"""
    for d, group in ((64, 32), (128, 32), (128, 128)):
        c = _cache(P, H_kv=H_kv, d=d, group=group, page=1024, max_pages=1 << 20)
        s = _shape(P, B=B, H=H, n=n, d=d, stride_n=d)
        got = P.cache_attn_workspace_bytes(s, c, n_max)
        most = max(64 * B * H * n, 2 * 256 * 256) * (d + 2) * 4 + 16384
        assert 0 < got <= most
        if B * H * n > 1 << 22:  # far more rows than there is anything to divide for
            assert got < 1 << 28


def test_the_binding_refuses_what_the_library_cannot_see(P):
    cache, shape = _cache(P), _shape(P, n=5)
    rows = torch.zeros(1, 2, 5, 128, dtype=torch.bfloat16)
    pool = torch.zeros(P.cache_bytes(cache), dtype=torch.uint8)
    pages, length = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)

    def refused(match, k=rows, v=rows.clone(), pool=pool, pages=pages, length=length, n_new=None):
        for call in (lambda: P.cache_write(k, v, shape, cache, pool, pages, length, n_new),
                     lambda: P.cache_read(shape, cache, pool, pages, length, n_new, k=k, v=v),
                     lambda: P.cache_attn(k, shape, cache, pool, pages, length, n_new, out=v)):
            with pytest.raises(ValueError, match=match):
                call()

    refused("current GPU")  # all on the CPU
    refused("bf16", k=rows.float())
    refused("as the shape says", k=rows[:, :1])
    refused("as the shape says", v=rows[:, :, :4])
    refused("strides", v=torch.zeros(1, 5, 2, 128, dtype=torch.bfloat16).transpose(1, 2))
    refused("uint8", pool=pool.view(torch.int32))
    refused("uint8", pool=pool[::2])
    refused("pages", pages=pages.long())
    refused("pages", pages=pages[:, :3])
    refused("pages", pages=torch.zeros(1, 8, dtype=torch.int32)[:, ::2])
    refused("length", length=length.float())
    refused("length", length=torch.zeros(2, dtype=torch.int32))
    refused("n_new", n_new=torch.zeros(2, dtype=torch.int32))


def test_generated_sequences_are_up_to_date():
    """pasa_cache_pipes.hpp is written by gen_cache_pipes.py; the committed header must be what the generator emits"""
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    csrc = os.path.join(root, "paper_2604_12219_amd", "csrc")
    got = subprocess.run([sys.executable, "-c", "import gen_cache_pipes; print(gen_cache_pipes.gen(), end='')"], cwd=csrc, capture_output=True,
                         text=True, check=True).stdout
    with open(os.path.join(csrc, "pasa_cache_pipes.hpp")) as f:
        assert f.read() == got
