"""Paged 8-bit cache, host side: sizes, and what its entry points refuse before any device work."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2507_19823_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    binding.lib()
    return binding


BASE = dict(n_seqs=3, n_q_heads=32, n_kv_heads=8, page=64, n_pages=100, max_pages=40)


def test_buffer_sizes_follow_the_layout(B):
    s = B.make_paged_shape(**BASE)
    assert B.hca_paged_cache_bytes(s) == 100 * 8 * 2 * 64 * 128
    assert B.hca_paged_scale_bytes(s) == 100 * 8 * 2 * 4
    assert B.hca_paged_open_bytes(s) == 3 * 8 * 2 * 64 * 128 * 2
    assert B.hca_paged_workspace_bytes(s, 3, 1) > 0
    assert B.hca_paged_workspace_bytes(s, -1, 1) == 0
    big = B.make_paged_shape(**dict(BASE, n_pages=(2 ** 31 - 1) // 64))
    assert B.hca_paged_cache_bytes(big) == ((2 ** 31 - 1) // 64) * 8 * 2 * 64 * 128       # beyond 32 bits


BAD = [(dict(n_seqs=0), -1), (dict(n_q_heads=30), -1), (dict(n_pages=0), -1), (dict(max_pages=0), -1), (dict(n_kv_heads=0), -1),
       (dict(n_seqs=1025), -2), (dict(page=48), -2), (dict(page=8), -2), (dict(page=256), -2), (dict(head_dim=96), -2),
       (dict(head_dim=256), -2), (dict(n_q_heads=136), -2), (dict(n_pages=2 ** 25), -2), (dict(max_pages=2 ** 24 + 1), -2),
       (dict(n_seqs=1024, max_pages=2 ** 21 + 1), -2)]


@pytest.mark.parametrize("kw,code", BAD)
def test_shapes_outside_the_supported_set(B, kw, code):
    s = B.make_paged_shape(**dict(BASE, **kw))
    assert B.hca_paged_cache_bytes(s) == 0 and B.hca_paged_workspace_bytes(s, 8, 1) == 0
    one = C.c_void_p(256)
    L, p = B.lib(), C.byref(s)
    assert L.hca_paged_map(p, one, one, one, one, one, one, one, 8, one, one, None, None, None, None) == code
    assert L.hca_paged_store(p, one, 4096, one, 4096, 8, one, one, one, one, one, one, None) == code
    assert L.hca_paged_attend(p, one, 65536, one, 8, 1, one, 100, one, one, one, one, 0.1, 1, one, None, one, None) == code


@pytest.mark.parametrize("field,value", [("elem", 2), ("elem", -1), ("code", 2), ("code", -1)])
def test_unknown_types(B, field, value):
    s = B.make_paged_shape(**BASE)
    setattr(s, field, value)
    assert B.hca_paged_cache_bytes(s) == 0


def test_map_refuses(B):
    L, s, one = B.lib(), B.make_paged_shape(**BASE), C.c_void_p(256)
    good = [one] * 7 + [8] + [one] * 2
    for i in (0, 1, 2, 3, 4, 5, 6, 8, 9):
        args = list(good)
        args[i] = None
        assert L.hca_paged_map(C.byref(s), *args, None, None, None, None) == -1, i
    assert L.hca_paged_map(C.byref(s), *good[:7], -1, one, one, None, None, None, None) == -1
    assert L.hca_paged_map(C.byref(s), *good[:7], 2 ** 30 + 1, one, one, None, None, None, None) == -2
    assert L.hca_paged_map(None, *good, None, None, None, None) == -1


def test_store_refuses(B):
    L, s, one, odd = B.lib(), B.make_paged_shape(**BASE), C.c_void_p(256), C.c_void_p(264)
    good = [one, 1024, one, 1024, 8, one, one, one, one, one, one]

    def rc(**kw):
        names = ["k", "ks", "v", "vs", "total", "start", "cu", "tables", "kv", "scale", "open"]
        return L.hca_paged_store(C.byref(s), *[kw.get(n, g) for n, g in zip(names, good)], None)

    for n in ("k", "v", "start", "cu", "tables", "kv", "scale", "open"):
        assert rc(**{n: None}) == -1, n
    for n in ("k", "v", "kv", "open"):
        assert rc(**{n: odd}) == -1, n
    for n in ("ks", "vs"):
        assert rc(**{n: 1016}) == -1 and rc(**{n: 1028}) == -1, n      # shorter than a row; no multiple of 8
    assert rc(total=-1) == -1 and rc(total=2 ** 27 + 1) == -2
    assert rc(total=0, k=None, v=None) == 0                            # nothing to do, nothing launched


def test_attend_refuses(B):
    L, s, one, odd = B.lib(), B.make_paged_shape(**BASE), C.c_void_p(256), C.c_void_p(264)
    names = ["q", "qs", "cu", "total", "max_q", "lens", "max_len", "tables", "kv", "scale", "open", "sm", "causal", "y", "lse", "ws"]
    good = [one, 4096, one, 8, 1, one, 100, one, one, one, one, 0.1, 1, one, None, one]

    def rc(**kw):
        return L.hca_paged_attend(C.byref(s), *[kw.get(n, g) for n, g in zip(names, good)], None)

    for n in ("q", "cu", "lens", "tables", "kv", "scale", "open", "y", "ws"):
        assert rc(**{n: None}) == -1, n
    for n in ("q", "y", "kv", "open", "ws"):
        assert rc(**{n: odd}) == -1, n
    assert rc(qs=4088) == -1 and rc(qs=4100) == -1
    assert rc(sm=0.0) == -1 and rc(sm=-1.0) == -1 and rc(sm=float("nan")) == -1
    assert rc(total=-1) == -1 and rc(max_q=-1) == -1 and rc(max_len=-1) == -1
    assert rc(total=2 ** 26 + 1) == -2 and rc(total=2 ** 22 + 1) == -2
    assert rc(scale=C.c_void_p(260)) == -1
    assert rc(total=0, q=None, y=None) == 0 and rc(max_q=0) == 0


def test_paged_cache_checks_what_calls_take_by_address(B):
    """Types, sizes, strides, devices and the rows that the workspace was made for, before anything is launched."""
    import torch
    from paper_2507_19823_amd.session import PagedCache
    c = PagedCache(1, 3, 4, 2, 16, 10, 5, 64, "f16", "int8", max_tokens=8, device="cpu")
    h = dict(dtype=torch.float16)
    k, q, y, lse = torch.zeros(4, 2, 64, **h), torch.zeros(4, 4, 64, **h), torch.zeros(4, 4, 64, **h), torch.zeros(4, 4)
    add = torch.ones(3, dtype=torch.int32)
    for bad in (add.long(), add[:2], torch.ones(3, 2, dtype=torch.int32)[:, 0], add.to("meta")):
        with pytest.raises(ValueError, match="add"):
            c.step(bad, 3)
    with pytest.raises(ValueError, match="max_tokens"):
        c.step(add, 9)
    wide = torch.zeros(4, 64, 2, **h)
    for bad in (k.bfloat16(), k[:3], torch.zeros(4, 2, 128, **h), wide.transpose(1, 2), torch.zeros(4, 4, 64, **h)[:, ::2]):
        with pytest.raises(ValueError, match="v:"):
            c.store(0, k, bad)
    with pytest.raises(ValueError, match="k:"):
        c.store(0, wide.transpose(1, 2), k)
    with pytest.raises(ValueError, match="max_tokens"):             # a workspace of single queries' size would be overrun
        c.attend(0, torch.zeros(9, 4, 64, **h), 9, torch.zeros(9, 4, 64, **h))
    with pytest.raises(ValueError, match="y:"):
        c.attend(0, q, 1, torch.zeros(4, 8, 64, **h)[:, :4], lse)
    with pytest.raises(ValueError, match="lse:"):
        c.attend(0, q, 1, y, lse.double())
    with pytest.raises(ValueError, match="cu:"):
        c.attend(0, q, 1, y, lse, cu=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="q:"):
        c.attend(0, q[:, :2], 1, y, lse)
    with pytest.raises(B.HcaError):
        PagedCache(1, 3, 4, 2, 16, 10, 5, 80, device="cpu")
