"""The paged cache on the GPU, against a plain host model (tests/page_model.py): attention in 64
bits within its derived bound, and every row, page number, count and length bit for bit."""
import math
import random

import numpy as np
import pytest
import torch

from paper_2606_03928_amd import pages, synth, vase
from tests import page_model as pm

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF16, F32 = torch.bfloat16, torch.float32


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def make(lengths, H=2, page=16, d=128, dtype=BF16, M=None, extra=6, seed=0, garbage=float("nan"), gap=0):
    """A cache whose slots hold `lengths` rows of N(0, 1) on shuffled pages; every other row of
    the pools holds `garbage`.  gap: elements between pages."""
    g = torch.Generator().manual_seed(seed)
    used = [pm.pages_for(n, page) for n in lengths]
    M = M or max(used) + 2
    P = sum(used) + extra
    order = random.Random(seed).sample(range(P), P)
    table, ref = -np.ones((len(lengths), M), np.int32), np.zeros(P, np.int32)
    pools = []
    for _ in range(2):
        flat = torch.full((P, H * page * d + gap), garbage, dtype=dtype)
        pools.append(flat[:, :H * page * d].view(P, H, page, d))
    for s, n in enumerate(lengths):
        for j in range(used[s]):
            p = table[s, j] = order.pop()
            ref[p] = 1
            r = min(page, n - j * page)
            for x in pools:
                x[p, :, :r] = torch.randn((H, r, d), generator=g).to(dtype)
    k, v = (torch.full((P, H * page * d + gap), garbage, dtype=dtype, device=DEV)[:, :H * page * d]
            .view(P, H, page, d).copy_(x) for x in pools)
    return pages.PageCache(k, v, ints(ref), ints(table), ints(lengths),
                           status=torch.zeros(1, dtype=torch.int32, device=DEV))


def model(c):
    return pm.Model(pm.raw(c.k), pm.raw(c.v), *(x.cpu().numpy() for x in (c.ref, c.table, c.length)))


def same(c, m, status=0):
    torch.cuda.synchronize()
    for n in ("ref", "table", "length"):
        np.testing.assert_array_equal(getattr(c, n).cpu().numpy(), getattr(m, n), n)
    np.testing.assert_array_equal(pm.raw(c.k), m.k)
    np.testing.assert_array_equal(pm.raw(c.v), m.v)
    assert int(c.status) == status


def cumulative(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


def queries(T, heads, d, dtype, seed, wide=0):
    """[T, heads, d] N(0, 1), in a wider tensor with `wide` more heads."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, heads + wide, d), generator=g).to(dtype).to(DEV)
    return x[:, :heads]


def check_attn(c, q, new, out, lse=None, causal=True, slots=None):
    """out (and lse) of the batch against 64 bits; returns the largest share of the bound."""
    G, bf16, worst = q.shape[1] // c.H, c.dtype == BF16, 0.0
    table, length, cu = c.table.cpu().numpy(), c.length.cpu().numpy(), cumulative(new)
    k, v = c.k.cpu(), c.v.cpu()
    for s in range(c.S) if slots is None else slots:
        n, L = int(new[s]), int(length[s])
        if n == 0:
            continue
        at = np.arange(L)
        rows = [x[table[s, at // c.page].astype(np.int64), :, at % c.page].double().numpy().transpose(1, 0, 2)
                if L else np.zeros((c.H, 0, c.d)) for x in (k, v)]
        qs = q[cu[s]:cu[s + 1]].cpu().double().numpy().reshape(n, c.H, G, c.d)
        ref, ref_lse, b = pm.attend(qs, *rows, L, causal)
        got = out[cu[s]:cu[s + 1]].cpu().double().numpy().reshape(ref.shape)
        bound = pm.out_bound(ref, b, L, bf16)
        assert np.isfinite(got).all(), "slot %d" % s
        err = np.abs(got - ref) / bound
        assert err.max() <= 1, "slot %d: %g of the bound at %s" % (s, err.max(), np.unravel_index(err.argmax(), err.shape))
        worst = max(worst, err.max())
        if lse is not None:
            got = lse[cu[s]:cu[s + 1]].cpu().double().numpy().reshape(ref_lse.shape)
            np.testing.assert_array_equal(np.isneginf(got), np.isneginf(ref_lse))
            fine = np.isfinite(ref_lse)
            assert (np.abs(got[fine] - ref_lse[fine]) <= pm.lse_bound(ref_lse, b, L)[fine]).all(), "lse of slot %d" % s
    return worst


# --- attention ----------------------------------------------------------------------------

SHAPES = [  # page, d, H, G, lengths, new
    (16, 128, 2, 4, [1, 17, 300, 64], [1, 1, 1, 1]),
    (16, 64, 1, 1, [1, 2, 15, 16, 33], [1, 2, 15, 3, 33]),
    (32, 128, 2, 8, [130, 95], [2, 2]),
    (48, 64, 2, 3, [200, 7, 129], [77, 7, 1]),
    (64, 128, 1, 5, [257, 64, 500], [130, 64, 0]),
    (176, 128, 3, 2, [400, 176, 352], [70, 1, 176]),
    (128, 64, 2, 16, [300, 128], [1, 40]),
    (16, 128, 1, 7, [90, 1, 31, 16, 47, 64, 5], [64, 1, 2, 16, 1, 0, 5]),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "page%d-d%d-H%d-G%d" % s[:4])
def test_attn(gpu_lib, shape, causal, dtype):
    page, d, H, G, lengths, new = shape
    c = make(lengths, H, page, d, dtype, seed=1, gap=32)
    T = sum(new)
    q = queries(T + 3, H * G, d, dtype, 2, wide=2 * H)
    out = torch.full((T + 3, H * G, d), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((T + 3, H * G), 7.0, device=DEV)
    c.attn(q, ints(cumulative(new)), max(new), causal=causal, out=out, lse=lse)
    torch.cuda.synchronize()
    check_attn(c, q, new, out, lse, causal)
    assert (out[T:] == 7).all() and (lse[T:] == 7).all()      # tokens of no slot
    assert int(c.status) == 0
    again = torch.empty_like(out)
    c.attn(q, ints(cumulative(new)), max(new), causal=causal, out=again)
    assert torch.equal(again[:T], out[:T])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [[1, 1, 1], [3, 1, 0], [130, 70, 1]])
@pytest.mark.parametrize("max_len", [1, 700, 2900, None])
def test_attn_over_ranges_of_a_long_cache(gpu_lib, new, max_len, dtype):
    # few rows over long slots: the keys are split, whatever max_len says of the longest
    c = make([2900, 1025, 70], 2, 64, 128, dtype, M=50, seed=3)
    T = sum(new)
    q = queries(T, 8, 128, dtype, 4)
    lse = torch.empty((T, 8), device=DEV)
    out = c.attn(q, ints(cumulative(new)), max(new), max_len=max_len, lse=lse)
    check_attn(c, q, new, out, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attn_of_tokens_that_see_nothing(gpu_lib, dtype):
    # slots of no rows, and of fewer rows than new tokens
    new = [2, 3, 40, 1]
    c = make([0, 1, 20, 5], 2, 16, 64, dtype, seed=5)
    q = queries(sum(new), 4, 64, dtype, 6)
    for causal in (True, False):
        lse = torch.empty((sum(new), 4), device=DEV)
        out = c.attn(q, ints(cumulative(new)), 40, lse=lse, causal=causal)
        check_attn(c, q, new, out, lse, causal)
        assert (out[:2] == 0).all() and torch.isneginf(lse[:2]).all()
        if causal:
            assert (out[2:4] == 0).all() and (out[5:25] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [3, 4, 90])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_attn_keeps_unseen_rows_out(gpu_lib, value, n, dtype):
    # the last token's K and V rows hold values that a product with 0 does not keep out
    c = make([150], 2, 16, 128, dtype, seed=7)
    last = int(c.table[0, 149 // 16])
    clean = [x.clone() for x in (c.k, c.v)]
    q = queries(n, 4, 128, dtype, 8)
    cu = ints([0, n])
    want = c.attn(q, cu, n)
    c.v[last, :, 149 % 16] = value
    got = c.attn(q, cu, n)
    assert torch.equal(got[:-1], want[:-1])
    assert not torch.isfinite(got[-1]).any()
    c.v.copy_(clean[1])
    c.k[last, :, 149 % 16] = value
    got = c.attn(q, cu, n)
    assert torch.equal(got[:-1], want[:-1])
    c.k.copy_(clean[0])
    # one column of one head: the others stand
    c.v[last, 1, 149 % 16, 77] = value
    got = c.attn(q, cu, n)
    assert torch.equal(got[:-1], want[:-1]) and torch.equal(got[-1, :2], want[-1, :2])
    assert not torch.isfinite(got[-1, 2:, 77]).any()
    keep = torch.arange(128, device=DEV) != 77
    assert torch.equal(got[-1][:, keep], want[-1][:, keep])


WIDE_TABLE = 1 << 20    # rows of a slot that a table may have: with it even a small batch is not a small call
TILES = [  # page, d, H, G, lengths, new, rows of a slot at most
    (16, 128, 2, 4, [1, 17, 300, 64], [1, 1, 40, 3], WIDE_TABLE),
    (48, 64, 2, 3, [200, 7, 129], [77, 7, 1], WIDE_TABLE),
    (64, 128, 1, 5, [257, 64, 500, 0], [130, 64, 0, 2], WIDE_TABLE),
    (176, 128, 3, 2, [2500, 176, 1352], [170, 1, 176], WIDE_TABLE),
    (128, 64, 2, 16, [2300, 128, 0], [1, 40, 0], WIDE_TABLE),
    (16, 128, 1, 7, [90, 1, 31, 16, 47, 64, 5], [64, 1, 2, 16, 1, 0, 5], WIDE_TABLE),
    (32, 64, 4, 1, [3000], [300], 0),                                     # workgroups with a part of a tile
    (16, 128, 8, 4, [40 + 7 * i for i in range(40)], [1 + i for i in range(40)], WIDE_TABLE),   # with many tiles
    (16, 64, 3, 2, [i % 19 for i in range(150)], [1 + i % 60 for i in range(150)], WIDE_TABLE),
    (16, 64, 1, 2, [9 + i % 7 for i in range(1100)], [40] + [i % 3 for i in range(1099)], WIDE_TABLE),
    (16, 64, 2, 4, [3 + i % 50 for i in range(900)], [0] * 300 + [100] + [0] * 598 + [17], WIDE_TABLE),
    (16, 64, 3, 4, [3 + i % 50 for i in range(900)], [0] * 7 + [1] + [0] * 700 + [4] + [0] * 190 + [2], 0),
    (16, 128, 40, 4, [150, 1, 33], [130, 1, 33], 0),                      # a workgroup to each tile
    (64, 64, 72, 3, [170, 64, 0, 200], [100, 9, 2, 200], 0),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", TILES, ids=lambda s: "d%d-H%d-G%d-S%d" % (s[1:4] + (len(s[4]),)))
def test_attn_of_many_rows(gpu_lib, shape, causal, dtype):
    page, d, H, G, lengths, new, most = shape
    c = make(lengths, H, page, d, dtype, M=most // page or None, seed=20, gap=64)
    T = sum(new)
    q = queries(T + 3, H * G, d, dtype, 21, wide=H)
    out = torch.full((T + 3, H * G, d), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((T + 3, H * G), 7.0, device=DEV)
    ws = torch.full((c.attn_workspace_bytes(T + 3, G, max(new)) + 64,), 255, dtype=torch.uint8, device=DEV)
    c.attn(q, ints(cumulative(new)), max(new), causal=causal, out=out, lse=lse, ws=ws)
    torch.cuda.synchronize()
    check_attn(c, q, new, out, lse, causal)
    assert (out[T:] == 7).all() and (lse[T:] == 7).all()      # tokens of no slot
    assert (ws[-64:] == 255).all() and int(c.status) == 0
    again = torch.empty_like(out)
    c.attn(q, ints(cumulative(new)), max(new), causal=causal, out=again, ws=ws.zero_())
    assert torch.equal(again[:T], out[:T])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,M", [(2, WIDE_TABLE // 16), (40, 64)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_attn_of_many_rows_keeps_unseen_rows_out(gpu_lib, value, H, M, dtype):
    n, L = 150, 330
    c = make([L], H, 16, 128, dtype, M=M, seed=22)
    q = queries(n, 2 * H, 128, dtype, 23)
    cu = ints([0, n])
    want = c.attn(q, cu, n)
    keep = torch.arange(128, device=DEV) != 77
    for x in (c.k, c.v):
        for back in (1, 70):             # the last token's row; one of a tile that many rows see in part
            at = (int(c.table[0, (L - back) // 16]), 1, (L - back) % 16, 77)
            old = x[at].clone()
            x[at] = value
            got = c.attn(q, cu, n)
            x[at] = old
            assert torch.equal(got[:n - back], want[:n - back])           # rows that do not see it
            assert torch.equal(got[:, :2], want[:, :2]) and torch.equal(got[:, 4:], want[:, 4:])
            if x is c.v:
                assert not torch.isfinite(got[n - back:, 2:4, 77]).any()
                assert torch.equal(got[:, 2:4][..., keep], want[:, 2:4][..., keep])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attn_of_many_rows_at_the_edges(gpu_lib, dtype):
    # scores of +-10^4, and a slot that has fewer rows than tokens
    c = make([1700, 5], 1, 32, 64, dtype, M=WIDE_TABLE // 32, seed=24)
    c.k.mul_(100)
    q = queries(400, 2, 64, dtype, 25) * 10
    lse = torch.empty((400, 2), device=DEV)
    out = c.attn(q, ints([0, 340, 400]), 340, lse=lse)
    check_attn(c, q, [340, 60], out, lse)
    assert (out[340:395] == 0).all() and torch.isneginf(lse[340:395]).all()
    # offsets that fall or leave the batch, and bad pages, read and write nothing outside
    for cu in ([0, 400, 20], [390, 10, 400], [-5, 99, 9999], [400, 400, 400], [300, 300, 400]):
        c.attn(q, ints(cu), 400, out=out)
    small = make([1700, 5], 1, 32, 64, dtype, seed=24)
    small.k.mul_(100)
    for cu in ([0, 400, 20], [390, 10, 400], [-5, 99, 9999], [400, 400, 400], [300, 300, 400]):
        small.attn(q, ints(cu), 400, max_len=64, out=out)
    torch.cuda.synchronize()
    assert int(c.status) == 0
    c.table[0, 3], c.table[0, 40] = -1, c.n_pages
    got = c.attn(q, ints([0, 340, 400]), 340)
    assert int(c.status) == pages.STATUS_PAGE_BAD
    check_attn(c, q, [340, 60], got, slots=[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attn_extreme_scores(gpu_lib, dtype):
    # scores of +-10^4: only the largest counts, and nothing overflows
    c = make([700], 1, 32, 64, dtype, seed=9)
    c.k.mul_(100)
    q = queries(40, 2, 64, dtype, 10) * 10
    out = c.attn(q, ints([0, 40]), 40)
    check_attn(c, q, [40], out)


def test_attn_behind_32_bit_offsets(gpu_lib):
    # pages whose first element lies behind 2^32 elements of the pools
    H, page, d, P = 64, 64, 128, 8400
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    k = torch.empty((P, H, page, d), dtype=BF16, device=DEV)
    v = torch.empty_like(k)
    assert (P - 3) * H * page * d > 1 << 32
    table = ints([[P - 1, P - 2], [P - 3, 0]])
    for x in (k, v):
        for p in (P - 1, P - 2, P - 3, 0):
            x[p].normal_()
    ref = torch.zeros(P, dtype=torch.int32, device=DEV)
    ref[[P - 1, P - 2, P - 3, 0]] = 1
    c = pages.PageCache(k, v, ref, table, ints([100, 128]), status=ints([0]))
    new = [1, 30]
    q = queries(31, 2, d, BF16, 11)
    view = c.heads(63, 1)
    view.write(queries(31, 1, d, BF16, 12), queries(31, 1, d, BF16, 13), ints([0, 1, 31]))
    small = pages.PageCache(k[[0, P - 3, P - 2, P - 1]][:, 63:].contiguous(),
                            v[[0, P - 3, P - 2, P - 1]][:, 63:].contiguous(), ints([1, 1, 1, 1]),
                            ints([[3, 2], [1, 0]]), ints([100, 128]))
    assert torch.equal(small.k[3, 0, 36:64], k[P - 1, 63, 36:64])
    assert torch.equal(small.k[2, 0, 99 - 64], queries(31, 1, d, BF16, 12)[0, 0])
    out = view.attn(q, ints([0, 1, 31]), 30)
    check_attn(small, q, new, out)
    # compacted in place: a map that drops every third row
    src = torch.arange(0, 96, device=DEV)[torch.arange(96, device=DEV) % 3 != 1].int()
    want = torch.cat([k[P - 1], k[P - 2]], 1)[:, src.long()]
    c.compact(ints([0, -1]), src.expand(1, H, -1).contiguous())
    assert torch.equal(k[P - 1], want)
    assert c.table.tolist() == [[P - 1, -1], [P - 3, 0]] and int(c.status) == 0


def test_attn_flags_bad_pages_and_stays_inside(gpu_lib):
    c = make([40, 40, 40], 1, 16, 64, seed=13, garbage=0.0)
    q = queries(3, 1, 64, BF16, 14)
    want = c.attn(q, ints([0, 1, 2, 3]), 1)
    for bad in (-1, c.n_pages, 2 ** 31 - 1):
        keep = c.table[1, 1].clone()
        c.table[1, 1] = bad
        got = c.attn(q, ints([0, 1, 2, 3]), 1)
        assert torch.equal(got[[0, 2]], want[[0, 2]])
        assert int(c.status) == pages.STATUS_PAGE_BAD
        c.status.zero_()
        c.table[1, 1] = keep
    # a slot with more tokens than max_new said
    q = queries(40, 1, 64, BF16, 15)
    out = torch.full_like(q, 3.0).contiguous()
    c.attn(q, ints([0, 20, 20, 21]), 1, out=out)
    assert int(c.status) == pages.STATUS_PAGE_BAD
    check_attn(c, q, [20, 0, 1], out, slots=[2])
    c.status.zero_()
    # offsets out of order or out of range read and write nothing outside
    for cu in ([0, 50, 20, 30], [0, -5, 3, 99], [5, 5, 5, 5], [0, 0, 0, 0]):
        c.attn(q, ints(cu), 20, out=out)
        c.write(q, q, ints(cu))
    torch.cuda.synchronize()


@pytest.mark.parametrize("n", [1, 17])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attn_over_a_million_rows(gpu_lib, dtype, n):
    L = 1_050_037
    c = make([70, L], 1, 1024, 64, dtype, seed=29, garbage=0.0, extra=1)
    q = queries(n + 1, 4, 64, dtype, 30)
    lse = torch.empty((n + 1, 4), device=DEV)
    out = c.attn(q, ints([0, 1, n + 1]), n, lse=lse)
    check_attn(c, q, [1, n], out, lse)
    assert int(c.status) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,H", [(WIDE_TABLE // 16, 2), (40, 40)])
def test_attn_of_many_rows_captured(gpu_lib, M, H, dtype):
    """A chunk's attention captured once and replayed over other lengths, offsets and queries,
    with eager calls between: what the host said at capture are upper bounds alone."""
    T, G = 200, 2
    c = make([600, 333, 90], H, 16, 128, dtype, M=M, seed=31, garbage=0.0)
    q = queries(T, H * G, 128, dtype, 32)
    cu = ints([0, 120, 121, 200])
    out, lse = torch.zeros((T, H * G, 128), dtype=dtype, device=DEV), torch.zeros((T, H * G), device=DEV)
    ws = torch.empty(max(c.attn_workspace_bytes(T, G, 150), 16), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.attn(q, cu, 150, out=out, lse=lse, ws=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            c.attn(q, cu, 150, out=out, lse=lse, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    for new, length in (([120, 1, 79], [600, 333, 90]), ([50, 150, 0], [599, 150, 0]), ([1, 1, 1], [17, 333, 1]),
                        ([0, 130, 70], [600, 140, 64]), ([120, 1, 79], [600, 333, 90])):
        cu.copy_(ints(cumulative(new)))
        c.length.copy_(ints(length))
        q.normal_()
        out.fill_(7), lse.fill_(7)
        g.replay()
        check_attn(c, q, new, out, lse)
        n = sum(new)
        assert (out[n:] == 7).all() and (lse[n:] == 7).all()
        eager = c.attn(q, cu, 150, ws=ws)
        assert torch.equal(eager[:n], out[:n])
    assert int(c.status) == 0


@pytest.mark.parametrize("M,n", [(8, 1), (8, 30), (WIDE_TABLE // 16, 50)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attn_flags_lengths_out_of_range(gpu_lib, dtype, M, n):
    c = make([60, 60, 60], 1, 16, 64, dtype, M=M, seed=26, garbage=0.0)
    q = queries(3 * n, 2, 64, dtype, 27)
    cu = ints([0, n, 2 * n, 3 * n])
    want = c.attn(q, cu, n)
    assert int(c.status) == 0
    for bad in (-1, -2 ** 31, M * 16 + 1, 2 ** 31 - 1):
        if bad > 0 and M > 8:
            continue                                 # 2^20 rows of page 0: nothing to learn
        c.length[1] = bad
        got = c.attn(q, cu, n)
        assert torch.equal(got[:n], want[:n]) and torch.equal(got[2 * n:], want[2 * n:])
        assert int(c.status) == pages.STATUS_PAGE_BAD
        if bad < 0:
            assert (got[n:2 * n] == 0).all()
        c.status.zero_()


def test_state_workspace_on_other_streams(gpu_lib):
    """A cache's own workspace is made on one stream and used on others, by name or as the
    current one; what is allocated where it lay must not run ahead of them."""
    want = None
    for by_name in (None, False, True):
        c = make([100, 37, 5], 2, 16, 64, F32, M=20, extra=40, seed=28)
        c.resize(ints([90, 37, 5]))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        more = ints([200, 60, 5])
        torch.cuda.synchronize()
        if by_name is None:
            c.resize(more)
        elif by_name:
            c.resize(more, stream=side)
        else:
            with torch.cuda.stream(side):
                c.resize(more)
        state = (c.table, c.length, c.ref)
        size = c.state_workspace_bytes()
        del c
        torch.full((size,), 255, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        got = [x.tolist() for x in state]
        assert want is None or got == want
        want = got


def test_workspaces_belong_to_the_stream_that_uses_them(gpu_lib, monkeypatch):
    # memory that another stream's pending work has just given up must not be taken for it
    c = make([3000, 900], 1, 16, 64, F32, M=200, extra=20, seed=33)
    q, cu = queries(2, 2, 64, F32, 34), ints([0, 1, 2])
    assert c.attn_workspace_bytes(2, 2, 1) > 0
    out, want = torch.empty_like(q).contiguous(), c.attn(q, cu, 1)
    side, made, empty = torch.cuda.Stream(), [], torch.empty

    def noted(*args, **kw):
        made.append(torch.cuda.current_stream())
        return empty(*args, **kw)

    torch.cuda.synchronize()
    monkeypatch.setattr(torch, "empty", noted)
    c.attn(q, cu, 1, out=out, stream=side)
    c.resize(ints([3010, 0]), stream=side)
    monkeypatch.undo()
    side.synchronize()
    assert made == [side, side]
    assert torch.equal(out, want) and c.length.tolist() == [3010, 0]


# --- state --------------------------------------------------------------------------------


def new_rows(T, H, d, dtype, seed, wide=0):
    x = queries(T, H * (2 + wide), d, dtype, seed)
    return x[:, :H], x[:, H:2 * H]


def model_write(m, kn, vn, cu):
    return m.write(pm.raw(kn), pm.raw(vn), np.asarray(cu))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page,d,H,lengths,new", [
    (16, 128, 2, [1, 40, 16, 100], [1, 1, 1, 1]),
    (16, 64, 1, [5, 0, 33, 70], [5, 0, 20, 1]),
    (48, 64, 40, [100, 49, 96], [60, 2, 48]),
    (32, 128, 20, [130], [77]),
])
def test_write(gpu_lib, page, d, H, lengths, new, dtype):
    c = make(lengths, H, page, d, dtype, seed=20, gap=16)
    m = model(c)
    kn, vn = new_rows(sum(new) + 2, H, d, dtype, 21, wide=1)
    c.write(kn, vn, ints(cumulative(new)))
    model_write(m, kn, vn, cumulative(new))
    same(c, m)


def test_write_flags_rows_without_a_page(gpu_lib):
    c = make([20, 8, 33], 2, 16, 64, seed=22)
    m = model(c)
    kn, vn = new_rows(30, 2, 64, BF16, 23)
    c.table[0, 1] = m.table[0, 1] = c.n_pages
    cu = [0, 7, 17, 30]            # slot 0 reaches the bad page, slot 1 has more than its rows
    c.write(kn, vn, ints(cu))
    assert model_write(m, kn, vn, cu) == pm.BAD
    same(c, m, pages.STATUS_PAGE_BAD)


@pytest.mark.parametrize("S", [1, 5, 300, 1500])
def test_resize(gpu_lib, S):
    rng = random.Random(S)
    lengths = [rng.choice([0, 1, 15, 16, 17, 40]) for _ in range(S)]
    c = make(lengths, 2, 16, 64, M=6, extra=2 * S + 6, seed=24)
    m = model(c)
    for step in range(4):
        new = [rng.choice([-1, 0, 1, 16, 31, 48, 33]) for _ in range(S)]
        status = m.resize(new)
        c.resize(ints(new))
        same(c, m, status)
        c.status.zero_()


def test_resize_refuses_all_or_nothing(gpu_lib):
    c = make([20, 30, 0], 2, 16, 64, M=4, extra=3, seed=25)
    for new, bit in (([64, 64, 0], pages.STATUS_PAGE_FULL), ([0, 0, 65], pages.STATUS_PAGE_BAD),
                     ([64, 0, 64], pages.STATUS_PAGE_FULL)):      # what a call frees is not its to take
        m = model(c)
        assert m.resize(new) == bit
        c.resize(ints(new))
        same(c, m, bit)
        c.status.zero_()
    c.length[1] = -3
    m = model(c)
    assert m.resize([5, 10, 0]) == pm.BAD
    c.resize(ints([5, 10, 0]))
    same(c, m, pages.STATUS_PAGE_BAD)
    c.status.zero_()
    c.resize(ints([5, -1, 7]))     # the slot left alone is not looked at
    m.resize([5, -1, 7])
    same(c, m)
    # an entry given up that names no page
    c.table[0, 0] = m.table[0, 0] = 99
    c.resize(ints([0, -1, 0]))
    assert m.resize([0, -1, 0]) == pm.BAD
    same(c, m, pages.STATUS_PAGE_BAD)


def test_resize_takes_pages_in_order_from_a_large_pool(gpu_lib):
    # more pages than one pass of the search looks at, the free ones far apart
    P, S, M = 30000, 40, 32
    g = torch.Generator().manual_seed(26)
    ref = (torch.rand(P, generator=g) < 0.97).int()
    k = torch.zeros((P, 1, 16, 64), dtype=BF16, device=DEV)
    c = pages.PageCache(k, k.clone(), ref.to(DEV), ints(-np.ones((S, M))), ints(np.zeros(S)), status=ints([0]))
    new = [(37 * i) % (M * 16) for i in range(S)]
    need = sum(pm.pages_for(n, 16) for n in new)
    free = torch.nonzero(ref == 0)[:, 0].tolist()
    assert 600 < need < len(free)
    c.resize(ints(new))
    table, at = c.table.cpu(), 0
    for s in range(S):
        n = pm.pages_for(new[s], 16)
        assert table[s, :n].tolist() == free[at:at + n]
        at += n
    assert int(c.status) == 0 and int((c.ref > 0).sum()) == int(ref.sum()) + need


def test_fork(gpu_lib):
    c = make([40, 17, 0, 0, 0, 64, 0], 2, 16, 64, M=6, seed=27)
    m = model(c)
    for parent in ([-1, -1, 0, 0, 1, -1, 2],           # slot 6's parent is forked itself
                   [1, -1, -1, -1, -1, -1, 99],        # not free; no such slot
                   [-1, -1, -1, -1, -1, -1, 5],
                   [-1] * 7):
        status = m.fork(parent)
        c.fork(ints(parent))
        same(c, m, status)
        c.status.zero_()
    # forks that grow within a shared page copy it, all but none of them at its end
    for new in ([41, -1, 42, -1, -1, -1, 65], [-1, 18, -1, 60, 16, 63, -1], [0, 0, -1, -1, -1, 64, 0]):
        status = m.resize(new)
        c.resize(ints(new))
        same(c, m, status)
        c.status.zero_()
    c.table[5, 1] = m.table[5, 1] = -7
    c.fork(ints([5, -1, -1, -1, -1, -1, -1]))
    assert m.fork([5, -1, -1, -1, -1, -1, -1]) == pm.BAD
    same(c, m, pages.STATUS_PAGE_BAD)


def survivors(n_map, H, K, L, seed):
    """Strictly increasing maps of K rows of L, the last one kept."""
    r = np.random.default_rng(seed).random((n_map, H, L - 1))
    kept = np.sort(np.argsort(r, -1)[..., :K - 1], -1)
    return np.concatenate([kept, np.full((n_map, H, 1), L - 1)], -1).astype(np.int32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page,d,H,K,L", [(16, 128, 2, 100, 130), (48, 64, 3, 96, 97), (64, 128, 1, 500, 900),
                                          (16, 64, 2, 1, 40), (32, 128, 2, 64, 64), (176, 64, 1, 400, 1000)])
def test_compact_in_place(gpu_lib, page, d, H, K, L, dtype):
    c = make([L, 3, L + 5, L], H, page, d, dtype, seed=28, gap=8)
    m = model(c)
    src = survivors(2, H, K, L, 29)
    where = [1, -1, 0, 0]
    c.compact(ints(where), ints(src))
    assert m.compact(where, src) == 0
    same(c, m)


def test_compact_with_shared_pages(gpu_lib):
    K, L = 70, 100
    c = make([L, 0, 0, 50, 0], 2, 16, 64, extra=20, seed=30)
    m = model(c)
    for x in (m.fork, lambda p: c.fork(ints(p))):
        x([-1, 0, 0, -1, 3])
    src = survivors(3, 2, K, L, 31)
    for where in ([-1, 0, -1, -1, -1], [2, -1, 1, -1, -1]):     # one sharer; then all that are left
        assert m.compact(where, src) == 0
        c.compact(ints(where), ints(src))
        same(c, m)
    # slots that share only some pages: 4 grew away from 3
    new = [-1, -1, -1, 80, 90]
    m.resize(new), c.resize(ints(new))
    same(c, m)
    src = survivors(1, 2, 40, 80, 32)
    assert m.compact([-1, -1, -1, 0, 0], src) == 0
    c.compact(ints([-1, -1, -1, 0, 0]), ints(src))
    same(c, m)


def test_compact_refuses_all_or_nothing(gpu_lib):
    c = make([100, 0, 60, 0], 2, 16, 64, extra=2, seed=33)
    c.fork(ints([-1, 0, -1, 2]))
    src = survivors(1, 2, 40, 60, 34)
    for where, bit in (([0, 0, -1, -1], pages.STATUS_PAGE_FULL), ([1, -1, -1, -1], pages.STATUS_PAGE_BAD),
                       ([-1, -1, 0, 2 ** 30], pages.STATUS_PAGE_BAD)):
        m = model(c)
        assert m.compact(where, src) == bit
        c.compact(ints(where), ints(src))
        same(c, m, bit)
        c.status.zero_()
    m = model(c)
    src = survivors(1, 2, 61, 62, 34)
    assert m.compact([-1, -1, 0, -1], src) == pm.BAD      # K above the slot's rows
    c.compact(ints([-1, -1, 0, -1]), ints(src))
    same(c, m, pages.STATUS_PAGE_BAD)
    c.status.zero_()
    c.table[2, 3] = -1
    m = model(c)
    src = survivors(1, 2, 10, 60, 34)
    assert m.compact([-1, -1, 0, -1], src) == pm.BAD
    c.compact(ints([-1, -1, 0, -1]), ints(src))
    same(c, m, pages.STATUS_PAGE_BAD)
    # maps that break their contract stay inside the slot
    c = make([60], 1, 16, 64, seed=35)
    wild = np.array([[[-5, 2 ** 31 - 1, 70, 3, 3, 59]]], np.int32)
    c.compact(ints([0]), ints(wild))
    torch.cuda.synchronize()
    assert c.length.tolist() == [6]


# --- together -----------------------------------------------------------------------------


@pytest.mark.parametrize("seed", range(4))
def test_a_run_of_serving(gpu_lib, seed):
    """Requests come, are forked, decoded, evicted and leave, every state as the model's and
    every step's attention within its bound."""
    rng = random.Random(seed)
    H, G, d, page, S = 4, 2, 64, 16, 6
    dtype = F32 if seed % 2 else BF16
    c = make([0] * S, H, page, d, dtype, M=20, extra=70, seed=40 + seed)
    m = model(c)
    for step in range(14):
        length = m.length.copy()
        target, new = [-1] * S, [0] * S
        parent = [-1] * S
        for s in range(S):
            if length[s] == 0:
                others = [p for p in range(S) if length[p] > 0 and parent[p] < 0]
                if others and rng.random() < 0.4:
                    parent[s] = rng.choice(others)
                else:
                    new[s] = rng.choice([1, 5, 37, 90])
            elif rng.random() < 0.1:
                target[s] = 0
            else:
                new[s] = rng.choice([0, 1, 1, 1, 3, 20])
            if new[s]:
                target[s] = length[s] + new[s]
        status = m.fork(parent)
        c.fork(ints(parent))
        status |= m.resize(target)
        c.resize(ints(target))
        same(c, m, status)
        if status:                      # the pool is full: the largest slot leaves
            c.status.zero_()
            out = [-1] * S
            out[int(m.length.argmax())] = 0
            m.resize(out), c.resize(ints(out))
            continue
        cu = cumulative(new)
        if cu[-1] == 0:
            continue
        for layer in range(2):          # two layers of two heads
            view = c.heads(2 * layer, 2)
            kn, vn = new_rows(int(cu[-1]), 2, d, dtype, 1000 * seed + 10 * step + layer)
            view.write(kn, vn, ints(cu))
            q = queries(int(cu[-1]), 2 * G, d, dtype, 5000 + 10 * step + layer)
            lse = torch.empty((int(cu[-1]), 2 * G), device=DEV)
            out = view.attn(q, ints(cu), max(new), lse=lse)
            check_attn(view, q, new, out, lse)
            for x, rows in ((m.k, kn), (m.v, vn)):
                part = pm.Model(x[:, 2 * layer:2 * layer + 2], x[:, 2 * layer:2 * layer + 2], m.ref, m.table, m.length)
                model_write(part, rows, rows, cu)
                x[:, 2 * layer:2 * layer + 2] = part.k
        same(c, m)
        if step % 4 == 3:
            where = [0 if m.length[s] >= 40 else -1 for s in range(S)]
            src = survivors(1, H, 25, 40, step)
            assert m.compact(where, src) == 0
            c.compact(ints(where), ints(src))
            same(c, m)


@pytest.mark.parametrize("name", ["tiny", "qwen3-1.7b"])
def test_rounds_on_pages_that_are_a_static_cache(gpu_lib, name):
    """A prompt goes in by chunks, then one page per slot is the static cache of vase.score,
    vase.select and vase.decode_attn: their round and the paged one leave the same rows."""
    cfg = synth.CONFIGS[name].with_(K=128, B=32, w=8, Nv=8)
    H, G, d, N, S = cfg.h_kv, cfg.G, cfg.d, cfg.N, 3
    dt = cfg.torch_dtype
    c = pages.PageCache.new(S, H, N, d, S, 1, dtype=dt, device=DEV)
    c.k.zero_(), c.v.zero_()
    done = np.zeros(S, np.int64)
    for chunk in ([100, 7, 60], [0, 93, 60], [60, 60, 40]):
        done += chunk
        cu = ints(cumulative(chunk))
        c.resize(ints(done))
        kn, vn = new_rows(sum(chunk), H, d, dt, int(done.sum()))
        c.write(kn, vn, cu)
        q = queries(sum(chunk), H * G, d, dt, 7 + int(done.sum()))
        out = c.attn(q, cu, max(chunk))
        check_attn(c, q, chunk, out)
    assert done.tolist() == [N] * S and int(c.status) == 0
    n = S * H
    order = c.table[:, 0].long()
    k, v = (x[order].reshape(n, N, d).clone() for x in (c.k, c.v))
    q_win = queries(n * G, cfg.w, d, dt, 50).reshape(n, G, cfg.w, d).contiguous()
    attn, vr = vase.score(k, v, q_win, cfg.K, cfg.B, cfg.pool)
    src = vase.select(attn, vr, cfg.K, cfg.B, cfg.Nv, seed=1, round=0)
    vase.compact(k, v, src, cfg.K, cfg.B)
    c.compact(ints(range(S)), src.view(S, H, cfg.K))
    for x, y in ((c.k, k), (c.v, v)):
        assert torch.equal(x[order].reshape(n, N, d)[:, :cfg.K], y[:, :cfg.K])
    # a token of decoding over the compacted rows
    q = queries(S, H * G, d, dt, 51)
    out = c.attn(q, ints(range(S + 1)), 1)
    check_attn(c, q, [1] * S, out)
    ref = vase.decode_attn(k, v, q.reshape(n, G, d).contiguous(), cfg.K, cfg.B, cfg.K)
    torch.testing.assert_close(out.reshape(n, G, d).float(), ref.float(), rtol=2 ** -7, atol=2e-2)


def test_streams_and_graphs(gpu_lib):
    """A step on a stream of its own, and captured once and replayed on other data, with the
    program's own work between; two graphs with workspaces of their own."""
    H, G, d, page, S = 2, 4, 128, 16, 4
    c = make([60, 33, 200, 1], H, page, d, M=40, extra=100, seed=60)
    kn, vn = new_rows(S, H, d, BF16, 61)
    q = queries(S, H * G, d, BF16, 62)
    cu = ints(range(S + 1))
    more = torch.empty(S, dtype=torch.int32, device=DEV)
    out = torch.empty((S, H * G, d), dtype=BF16, device=DEV)
    need = c.attn_workspace_bytes(S, G, 1)
    spaces = [(torch.empty(max(need, 16), dtype=torch.uint8, device=DEV),
               torch.empty(c.state_workspace_bytes(), dtype=torch.uint8, device=DEV)) for _ in range(2)]

    def step(ws):
        torch.add(c.length, 1, out=more)
        c.resize(more, ws=ws[1])
        c.write(kn, vn, cu)
        c.attn(q, cu, 1, out=out, ws=ws[0])

    m = model(c)

    def model_step():
        m.resize(m.length + 1)
        model_write(m, kn, vn, list(range(S + 1)))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(spaces[0])
        graphs = []
        for ws in spaces:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                step(ws)
            graphs.append(g)
    torch.cuda.current_stream().wait_stream(side)
    model_step()
    same(c, m)
    check_attn(c, q, [1] * S, out)
    for i in range(6):
        kn.normal_(), vn.normal_(), q.normal_()
        graphs[i % 2].replay()
        model_step()
        same(c, m)
        check_attn(c, q, [1] * S, out)
        if i == 2:                       # eager work of the same cache between replays
            step(spaces[1])
            model_step()
            same(c, m)
    # the stream given by name, with the buffers made by the call
    torch.cuda.synchronize()
    got = c.attn(q, cu, 1, stream=side)
    side.synchronize()
    assert torch.equal(got, out)


def test_binding_refuses(gpu_lib):
    c = make([20, 8], 2, 16, 64, seed=70)
    q, cu = queries(3, 4, 64, BF16, 71), ints([0, 2, 3])
    for call in (lambda: c.attn(q[:, :3], cu, 2), lambda: c.attn(q.float(), cu, 2),
                 lambda: c.attn(q, cu[:2], 2), lambda: c.attn(q, cu.long(), 2),
                 lambda: c.attn(q.transpose(0, 1), cu, 2), lambda: c.attn(q, cu, 2, out=q.float()),
                 lambda: c.attn(q, cu, 2, lse=torch.empty(3, 3, device=DEV)),
                 lambda: c.attn(q.cpu(), cu, 2), lambda: c.write(q[:, :2], q[:, :1], cu),
                 lambda: c.write(q[:, :2], q[:, 2:].contiguous(), cu), lambda: c.resize(ints([1])),
                 lambda: c.fork(ints([1, 2]).long()), lambda: c.compact(ints([0, 1]), ints([[[1]]])),
                 lambda: c.heads(1, 2), lambda: c.heads(0, 1).resize(ints([1, 1])),
                 lambda: c.heads(0, 1).compact(ints([0, 0]), ints([[[1]]])),
                 lambda: c.resize(ints([1, 1]), ws=torch.empty(8, device=DEV)),
                 lambda: pages.PageCache(c.k.transpose(1, 2), c.v.transpose(1, 2), c.ref, c.table, c.length),
                 lambda: pages.PageCache(c.k, c.v, c.ref, c.table, c.length[:1]),
                 lambda: pages.PageCache(c.k, c.v.float(), c.ref, c.table, c.length)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(vase.VaseError) as e:
        c.attn(q, cu, 4)
    assert e.value.status == vase.ERR_INVALID_ARG
    assert int(c.status) == 0
    assert c.attn(q[:0], cu, 1).shape == (0, 4, 64)
    assert math.isfinite(float(c.attn(q, cu, 2).float().sum()))
