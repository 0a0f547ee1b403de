"""The paged cache's C ABI on the host: symbols, argument checks, workspace sizes, and the
page arithmetic (no GPU work: every invalid call is refused before any HIP call)."""
import ctypes
import re

import pytest

from paper_2606_03928_amd import pages, vase

FAKE, ODD = 1 << 20, (1 << 20) + 4


@pytest.fixture(scope="module")
def lib():
    return pages.load()


def cache(**kw):
    a = dict(k=FAKE, v=FAKE, ref=FAKE, table=FAKE, len=FAKE, page_stride=8 * 64 * 128, dtype=0,
             n_pages=100, H=8, page=64, d=128, S=4, M=16)
    a.update(kw)
    return pages._Pages(*[a[n] for n, _ in pages._Pages._fields_])


def test_header_declares_what_the_library_exports(lib):
    with open(vase.HEADER_PATH.replace("vase.h", "vase_page.h")) as f:
        text = f.read()
    names = set(re.findall(r"^\s*(?:int|size_t)\s+(vase_page_\w+)\s*\(", text, re.M))
    assert names == {"vase_page_workspace_bytes", "vase_page_attn", "vase_page_write", "vase_page_resize",
                     "vase_page_fork", "vase_page_compact"}
    assert all(hasattr(lib, n) for n in names)
    value = dict(re.findall(r"#define (VASE_\w+)\s+(\d+)", text))
    assert int(value["VASE_STATUS_PAGE_FULL"]) == pages.STATUS_PAGE_FULL
    assert int(value["VASE_STATUS_PAGE_BAD"]) == pages.STATUS_PAGE_BAD
    assert [int(value["VASE_OP_PAGE_" + n]) for n in ("ATTN", "RESIZE", "COMPACT")] == [
        pages.OP_PAGE_ATTN, pages.OP_PAGE_RESIZE, pages.OP_PAGE_COMPACT]


def attn(lib, c, **kw):
    a = dict(q=FAKE, stride=8 * 4 * 128, cu=FAKE, T=9, G=4, max_new=3, max_len=1000, causal=1, out=FAKE,
             lse=None, ws=FAKE, wsb=1 << 40, st=None)
    a.update(kw)
    return lib.vase_page_attn(None if c is None else ctypes.byref(c), a["q"], a["stride"], a["cu"], a["T"],
                              a["G"], a["max_new"], a["max_len"], a["causal"], a["out"], a["lse"], a["ws"],
                              a["wsb"], a["st"], None)


def calls(lib, c):
    """Each call with the cache c and arguments that are valid otherwise."""
    r = ctypes.byref(c)
    return [lambda: attn(lib, c),
            lambda: lib.vase_page_write(r, FAKE, FAKE, 8 * 128, FAKE, 9, None, None),
            lambda: lib.vase_page_resize(r, FAKE, FAKE, 1 << 40, None, None),
            lambda: lib.vase_page_fork(r, FAKE, None, None),
            lambda: lib.vase_page_compact(r, FAKE, FAKE, 2, 100, FAKE, 1 << 40, None, None)]


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), vase.ERR_INVALID_ARG), (dict(v=ODD), vase.ERR_INVALID_ARG),
    (dict(ref=None), vase.ERR_INVALID_ARG), (dict(table=FAKE + 2), vase.ERR_INVALID_ARG),
    (dict(len=None), vase.ERR_INVALID_ARG), (dict(dtype=2), vase.ERR_DTYPE),
    (dict(n_pages=0), vase.ERR_INVALID_ARG), (dict(H=0), vase.ERR_INVALID_ARG),
    (dict(H=9), vase.ERR_INVALID_ARG),                       # a page would overlap the next
    (dict(page=24), vase.ERR_INVALID_ARG), (dict(page=0), vase.ERR_INVALID_ARG),
    (dict(page=8), vase.ERR_INVALID_ARG), (dict(d=96), vase.ERR_INVALID_ARG),
    (dict(S=0), vase.ERR_INVALID_ARG), (dict(S=65537), vase.ERR_INVALID_ARG),
    (dict(M=0), vase.ERR_INVALID_ARG), (dict(M=(1 << 23) + 1), vase.ERR_INVALID_ARG),
    (dict(page_stride=8 * 64 * 128 + 4), vase.ERR_INVALID_ARG),
    (dict(page_stride=1 << 59), vase.ERR_INVALID_ARG),
])
def test_caches_refused(lib, kw, code):
    for call in calls(lib, cache(**kw)):
        assert call() == code


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), vase.ERR_INVALID_ARG), (dict(q=ODD), vase.ERR_INVALID_ARG),
    (dict(cu=None), vase.ERR_INVALID_ARG), (dict(out=None), vase.ERR_INVALID_ARG),
    (dict(out=ODD), vase.ERR_INVALID_ARG), (dict(lse=FAKE + 2), vase.ERR_INVALID_ARG),
    (dict(st=FAKE + 2), vase.ERR_INVALID_ARG), (dict(T=-1), vase.ERR_INVALID_ARG),
    (dict(T=(1 << 24) + 1), vase.ERR_INVALID_ARG), (dict(G=0), vase.ERR_INVALID_ARG),
    (dict(G=17), vase.ERR_INVALID_ARG), (dict(max_new=0), vase.ERR_INVALID_ARG),
    (dict(max_new=10), vase.ERR_INVALID_ARG), (dict(max_len=0), vase.ERR_INVALID_ARG),
    (dict(max_len=1025), vase.ERR_INVALID_ARG), (dict(stride=8 * 4 * 128 - 8), vase.ERR_INVALID_ARG),
    (dict(stride=8 * 4 * 128 + 4), vase.ERR_INVALID_ARG), (dict(stride=1 << 60), vase.ERR_INVALID_ARG),
    (dict(ws=None), vase.ERR_WORKSPACE), (dict(wsb=64), vase.ERR_WORKSPACE), (dict(ws=ODD), vase.ERR_WORKSPACE),
    (dict(T=0), vase.OK),
])
def test_attn_refuses(lib, kw, code):
    assert attn(lib, cache(), **kw) == code
    if code == vase.ERR_INVALID_ARG:
        assert attn(lib, None, **kw) == code


def test_attn_refuses_more_workgroups_than_a_launch_takes(lib):
    # a workgroup of 256 threads to each slot and head: 2^24 of them would be 2^32 threads
    T, H = 1 << 16, 256
    c = cache(S=T, H=H, page_stride=H * 64 * 128)
    assert attn(lib, c, T=T, G=1, max_new=1, stride=H * 128, wsb=1 << 62) == vase.ERR_UNSUPPORTED
    # 2^31 query rows
    c = cache(S=128, H=1 << 12, page_stride=(1 << 12) * 64 * 128)
    assert attn(lib, c, T=1 << 15, G=16, max_new=1 << 15, stride=(1 << 16) * 128, wsb=1 << 62) == vase.ERR_UNSUPPORTED


def test_the_others_refuse(lib):
    c = cache()
    r = ctypes.byref(c)
    E, W = vase.ERR_INVALID_ARG, vase.ERR_WORKSPACE
    write, resize, fork, compact = (lib.vase_page_write, lib.vase_page_resize, lib.vase_page_fork,
                                    lib.vase_page_compact)
    for a in ((None, FAKE, 1024, FAKE, 9), (FAKE, ODD, 1024, FAKE, 9), (FAKE, FAKE, 1016, FAKE, 9),
              (FAKE, FAKE, 1028, FAKE, 9), (FAKE, FAKE, 1024, None, 9), (FAKE, FAKE, 1024, FAKE, -1),
              (FAKE, FAKE, 1024, FAKE, (1 << 24) + 1)):
        assert write(r, *a, None, None) == E
    assert write(r, FAKE, FAKE, 1024, FAKE, 9, FAKE + 1, None) == E
    assert write(r, FAKE, FAKE, 1024, FAKE, 0, None, None) == vase.OK
    need = lib.vase_page_workspace_bytes(pages.OP_PAGE_RESIZE, r, 0, 0, 0, 0)
    assert need > 0
    assert resize(r, None, FAKE, need, None, None) == E
    assert resize(r, FAKE, FAKE, need, FAKE + 2, None) == E
    for ws, n in ((None, need), (FAKE, need - 1), (ODD, need)):
        assert resize(r, FAKE, ws, n, None, None) == W
    assert fork(r, None, None, None) == E
    assert fork(r, FAKE, FAKE + 3, None) == E
    need = lib.vase_page_workspace_bytes(pages.OP_PAGE_COMPACT, r, 0, 0, 0, 0)
    for m, s, n, K in ((None, FAKE, 1, 9), (FAKE, None, 1, 9), (FAKE, FAKE, 0, 9), (FAKE, FAKE, 1, 0),
                       (FAKE, FAKE, 1, 1025)):
        assert compact(r, m, s, n, K, FAKE, need, None, None) == E
    for ws, n in ((None, need), (FAKE, need - 1), (ODD, need)):
        assert compact(r, FAKE, FAKE, 1, 9, ws, n, None, None) == W


def test_workspace_sizes(lib):
    def need(op, c, *a):
        return lib.vase_page_workspace_bytes(op, ctypes.byref(c), *(a or (0, 0, 0, 0)))

    # one token: what the ranges of its 8 heads' 4 rows take, at most 64 of them
    one = need(pages.OP_PAGE_ATTN, cache(), 1, 4, 1, 1000)
    assert 0 < one <= 64 * 32 * (128 + 2) * 4
    # many rows fill the chip as they are
    assert need(pages.OP_PAGE_ATTN, cache(S=64), 1 << 16, 4, 1024, 1024) == 0
    for op in (0, 1, 2):
        assert need(op, cache(d=80), 1, 4, 1, 1000) == 0
    assert need(7, cache()) == 0
    assert need(pages.OP_PAGE_ATTN, cache(), 1, 17, 1, 1000) == 0
    # the largest cache does not overflow
    big = cache(S=65536, M=1 << 13, page=65536, H=1, page_stride=65536 * 128, n_pages=1 << 20)
    assert need(pages.OP_PAGE_COMPACT, big) > 2 * 4 * 65536 * (1 << 13)


def test_page_of_a_group():
    # n // D for every page size, as a product and a shift (page_internal.hpp): exact
    # where a quotient changes, over all groups that a slot may have
    for D in range(1, 4097):
        b = (D - 1).bit_length()
        m = ((1 << (26 + b)) + D - 1) // D
        assert m < 1 << 32
        top = (1 << 25) + 4096
        for q in {0, 1, 2, 3, 1000, top // D - 1, top // D}:
            for n in (q * D - 1, q * D, q * D + 1):
                if 0 <= n <= top:
                    assert (n * m) >> (26 + b) == n // D


def test_binding_refuses_host_tensors():
    import torch
    k = torch.zeros(4, 2, 16, 64)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        pages.PageCache(k, k, i, i.view(2, 2), i[:2])
