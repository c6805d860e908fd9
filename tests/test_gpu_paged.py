"""The paged K/V cache on the GPU against its fp64 oracle: block tables and slots bit for bit, rows and codes bit for bit,
attention of one new token within tolerances counted from the number formats, and the operators together."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from oracle import pafu_oracle as orc
from paper_2601_21896_amd import binding as B
from tests.gpu_util import DEV, bits

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def bf16_values(rng, *shape):
    """N(0,1) rounded to bf16, as a host tensor."""
    return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(BF)


# ------------------------------------------------------------------------------------------------ tables and slots
def _tables(kv, new, n_free, page, columns, max_slots, start, extra_ld=0, seed=0):
    rng = np.random.default_rng(seed)
    n = len(kv)
    pages = rng.permutation(max(100000, n * columns + n_free))[:n * columns + n_free]
    free, table = pages[:n_free], pages[n_free:].reshape(n, columns)
    wide = np.full((n, columns + extra_ld), -77)
    wide[:, :columns] = table
    d_table = ints(wide)[:, :columns]
    slots, row_start = torch.full((max_slots + 8,), 99, dtype=torch.int32, device=DEV), ints(np.full(n + 1, 99))
    kv_out, end = ints(np.full(n, 99)), ints([99])
    want = po.paged_tables(kv, new, free, page, table, max_slots, start or 0)
    B.pafu_paged_tables(ints(kv), ints(new), ints(free), page, d_table, slots[:max_slots], row_start, kv_out, end,
                        free_start=None if start is None else ints([start]))
    torch.cuda.synchronize()
    got = [x.cpu().numpy() for x in (d_table, slots, row_start, kv_out, end)]
    for g, w, what in zip(got, (want[0], np.append(want[1], [99] * 8), want[2], want[3], [want[4]]),
                          ("table", "slots", "row_start", "kv_len_out", "free_end")):
        assert np.array_equal(g, w), (what, g, w)


@pytest.mark.parametrize("n,page,new_high,max_extra,start,short", [
    (1, 16, 1, 0, None, 0), (1, 8, 3000, 5, 0, 0), (3, 64, 1, 3, 2, 0), (64, 16, 1, 0, 1, 0), (65, 16, 40, 7, 4, 0),
    (257, 32, 300, 1, 9, 0), (300, 8, 100, -400, 0, 60), (1000, 256, 3, 2000, 3, 10), (2, 4096, 9000, 0, 1, 1),
    (1025, 16, 65, 0, 0, 0), (8192, 8, 20, 3, 5, 100)])
def test_tables_are_the_oracles(n, page, new_high, max_extra, start, short):
    rng = np.random.default_rng(n * 1000 + page)
    kv = rng.integers(0, 700, n) * (rng.random(n) < 0.8)
    new = rng.integers(0, new_high + 1, n)
    new[0] = new_high
    need = sum(-(-(a + b) // page) - -(-a // page) for a, b in zip(kv, new))
    columns = max(-(-(a + b) // page) for a, b in zip(kv, new))
    _tables(kv, new, max(need + (start or 0) - short, 0), page, columns, max(int(new.sum()) + max_extra, 0), start,
            extra_ld=n % 3)


def test_tables_with_narrow_tables_and_out_of_range_lengths():
    # columns end before the tokens do; negative lengths count as 0; a negative start as 0; no free page at all
    _tables([5, 40, 0, 7], [60, 3, 100, 1], 40, 8, 3, 170, 0)
    _tables([-5, 9, 3], [4, -7, 2], 10, 8, 2, 9, -4)
    _tables([0, 16], [3, 1], 0, 16, 4, 6, None)
    _tables([0, 0, 0], [0, 0, 0], 4, 16, 1, 3, 2)
    _tables([10], [5], 3, 16, 1, 0, None)


def test_tables_saturate_and_leave_tokens_past_the_limit_without_a_slot():
    big = 2 ** 31 - 1
    kv, new = ints([big - 3, 5]), ints([10, 2])
    table, slots = ints(np.full((2, 2), 7)), ints(np.full(16, 99))
    row_start, out, end = ints([9] * 3), ints([9] * 2), ints([9])
    B.pafu_paged_tables(kv, new, ints([1, 2, 3]), 16, table, slots, row_start, out, end)
    torch.cuda.synchronize()
    assert out.tolist() == [big, 7] and row_start.tolist() == [0, 10, 12] and end.tolist() == [0]
    assert slots.tolist() == [-1] * 10 + [7 * 16 + 5, 7 * 16 + 6] + [-1] * 4
    B.pafu_paged_tables(ints([0, 0]), ints([big, big]), ints([1, 2, 3]), 16, table, slots, row_start, out, end)
    torch.cuda.synchronize()
    assert row_start.tolist() == [0, big, big] and out.tolist() == [big, big] and end.tolist() == [2 ** 28]
    assert table.tolist() == [[1, 2], [-1, -1]]
    assert slots.tolist() == list(range(16, 32))


@pytest.mark.parametrize("n,page,columns,extra", [(1, 16, 1, 0), (1, 64, 512, 3), (7, 8, 9, 100), (300, 16, 40, 0),
                                                  (1500, 32, 5, -333), (8192, 8, 3, 1)])
def test_slots_are_the_oracles(n, page, columns, extra):
    rng = np.random.default_rng(n + columns)
    table = rng.permutation(n * columns).reshape(n, columns)
    table[rng.random((n, columns)) < 0.05] = -1
    table[rng.random((n, columns)) < 0.02] = 2 ** 31 // page      # its slots would pass 2^31
    start = rng.integers(-2, columns * page, n)
    count = rng.integers(-3, page * columns, n) * (rng.random(n) < 0.7)   # some run over the table's end
    total = int(np.maximum(count, 0).sum())
    max_slots = max(total + extra, 0)
    want, want_start = po.paged_slots(table, start, count, page, max_slots)
    slots, row_start = ints(np.full(max_slots + 4, 99)), ints(np.full(n + 1, 99))
    B.pafu_paged_slots(ints(table), ints(start), ints(count), page, slots[:max_slots], row_start)
    torch.cuda.synchronize()
    assert np.array_equal(slots.cpu().numpy(), np.append(want, [99] * 4))
    assert np.array_equal(row_start.cpu().numpy(), want_start)


# ------------------------------------------------------------------------------------------------ rows into pages
def _pool(n_pages, page, heads, D, dtype, layout, fill=0x7F):
    """K and V page tensors over one filled slab (0x7f7f is a large bf16 number, 0x7f a NaN code)."""
    shape = {"token": (2, n_pages, page, heads, D), "head": (2, n_pages, heads, page, D), "pages alternate": (n_pages, 2, page, heads, D),
             "rows alternate": (n_pages, page, 2, heads, D), "gaps": (2, n_pages, page + 1, heads + 2, D)}[layout]
    width = 2 if dtype == BF else 1
    slab = torch.full((int(np.prod(shape)) * width,), fill, dtype=torch.uint8, device=DEV).view(dtype).view(shape)
    if layout == "token":
        return slab, slab[0], slab[1]
    if layout == "head":
        return slab, slab[0].permute(0, 2, 1, 3), slab[1].permute(0, 2, 1, 3)
    if layout == "pages alternate":
        return slab, slab[:, 0], slab[:, 1]
    if layout == "rows alternate":
        return slab, slab[:, :, 0], slab[:, :, 1]
    return slab, slab[0, :, :page, 1:heads + 1], slab[1, :, :page, 1:heads + 1]


LAYOUTS = ("token", "head", "pages alternate", "rows alternate", "gaps")


def _raw(t):
    return t.contiguous().view(torch.int16 if t.dtype == BF else torch.uint8).cpu().numpy()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("rows,heads,D,page,kv", [(1, 1, 128, 16, "bf16"), (37, 3, 64, 8, "bf16"), (700, 8, 128, 64, "bf16"),
                                                  (1, 1, 64, 16, "e4m3"), (333, 5, 128, 16, "e4m3"), (90, 12, 64, 32, "e4m3")])
def test_append_writes_its_rows_and_nothing_else(layout, rows, heads, D, page, kv):
    rng = np.random.default_rng(rows)
    dtype = BF if kv == "bf16" else torch.uint8
    n_pages = -(-rows // page) + 2
    slab, Kp, Vp = _pool(n_pages, page, heads, D, dtype, layout)
    slots = rng.permutation(n_pages * page)[:rows]
    if rows > 4:
        slots[1], slots[2], slots[3], slots[rows - 1] = -1, n_pages * page, 2 ** 31 - 1, -2 ** 31
    K, V = (bf16_values(rng, rows, heads + 1, D).to(DEV)[:, :heads] for _ in range(2))   # rows with a gap behind them
    K[0, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, -0.0], dtype=BF)
    before = slab.clone()
    ks, vs = (-5, -6) if kv == "e4m3" else (0, 0)
    B.pafu_paged_append(K, V, ints(slots), Kp, Vp, ks, vs)
    torch.cuda.synchronize()
    new = []
    for x, s in ((K, ks), (V, vs)):
        new.append(_raw(x) if kv == "bf16" else orc.quantise_e4m3(x.double().cpu().numpy(), s))
    # the same rows on the host into a copy of the slab, through the same views
    want = before.cpu().view(torch.int16 if dtype == BF else torch.uint8).clone()
    on_host = _views(want, layout, page, heads)
    got = slab.cpu().view(want.dtype)
    for t, rows_new in zip(on_host, new):
        t.copy_(torch.from_numpy(po.paged_append(t.numpy(), rows_new, slots)))
    assert torch.equal(got, want)


def _views(slab, layout, page, heads):
    if layout == "head":
        return slab[0].permute(0, 2, 1, 3), slab[1].permute(0, 2, 1, 3)
    if layout == "pages alternate":
        return slab[:, 0], slab[:, 1]
    if layout == "rows alternate":
        return slab[:, :, 0], slab[:, :, 1]
    if layout == "gaps":
        return slab[0, :, :page, 1:heads + 1], slab[1, :, :page, 1:heads + 1]
    return slab[0], slab[1]


# ------------------------------------------------------------------------------------------------ attention
def _tolerance(Q, K, V, out, n_tokens, D, scale):
    """Bound on |O - O_exact| for one request: see below.  K, V [tokens, heads, D] in float64."""
    if n_tokens == 0:
        return 0.0
    G = Q.shape[0] // K.shape[1]
    S = max(float((np.abs(K[:, h // G]) @ np.abs(Q[h])).max()) for h in range(Q.shape[0])) * scale
    # scores: D exact products summed in fp32 and scaled (each step half a unit, 2^-24, of at most S) -> D + 4 steps;
    # a weight is off by that relatively, and so is the sum of weights: twice.  The sums over tokens: n + 16 steps each.
    # A weight in [1, 2) enters the second product as its upper half and a bf16 number for the rest, which is less than 2^-7
    # and has steps of 2^-15 at most: half a step is 2^-16.  exp2 and the division: 8 steps.
    rel = 2 * (D + 4) * 2.0 ** -24 * S + 2 * (n_tokens + 16) * 2.0 ** -24 + 2.0 ** -16 + 8 * 2.0 ** -24
    return rel * float(np.abs(V).max()) + (2.0 ** -8 * float(np.abs(V).max()) if out == BF else 0.0)


def _attend(lens, heads, kv_heads, D, page, kv="bf16", layout="token", out=BF, pinned=0, window=0, ws=True, seed=0,
            scale=0.0, q_gain=1.0, spoil=None, columns=None, extra_ld=0):
    """Runs one call over a pool whose unused rows are NaN, checks every row of O, returns O."""
    rng = np.random.default_rng(seed)
    n = len(lens)
    columns = columns or max(1, max(-(-x // page) for x in lens))
    need = [min(-(-x // page), columns) for x in lens]
    n_pages = sum(need) + 3
    dtype = BF if kv == "bf16" else torch.uint8
    slab, Kp, Vp = _pool(n_pages, page, kv_heads, D, dtype, layout, fill=0xFF)   # 0xffff, 0xff: NaN
    order = rng.permutation(n_pages)
    table = np.full((n, columns + extra_ld), 2 ** 31 - 1)                        # pages that are not there
    at = 0
    for b in range(n):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    if spoil is not None:
        spoil(table)
    rows = [(b, j) for b in range(n) for j in range(min(lens[b], columns * page))]
    host_K, host_V = np.full((n_pages, page, kv_heads, D), np.nan), np.full((n_pages, page, kv_heads, D), np.nan)
    ks, vs = (-5, -6) if kv == "e4m3" else (0, 0)
    if rows:
        K, V = bf16_values(rng, len(rows), kv_heads, D), bf16_values(rng, len(rows), kv_heads, D)
        page_of = np.array([table[b, j // page] for b, j in rows])
        off = np.array([j % page for _, j in rows])
        ok = (page_of >= 0) & (page_of < n_pages)
        # rows that no query may see stay NaN
        seen = np.array([window <= 0 or j < pinned or j >= lens[b] - window for b, j in rows])
        ok &= seen
        for t, host, x, s in ((Kp, host_K, K, ks), (Vp, host_V, V, vs)):
            if kv == "bf16":
                stored, values = x, x.double().numpy()
            else:
                codes = orc.quantise_e4m3(x.double().numpy(), s)
                stored, values = torch.from_numpy(codes), orc.dequantise_e4m3(codes, s)
            p, o = torch.from_numpy(page_of[ok]).to(DEV), torch.from_numpy(off[ok]).to(DEV)
            t[p, o] = stored[torch.from_numpy(ok)].to(DEV)
            host[page_of[ok], off[ok]] = values[ok]
    Qw = (bf16_values(rng, n, heads + 1, D).float() * q_gain).to(BF)
    Q = Qw.to(DEV)[:, :heads]
    O = torch.full((n + 2, heads + 1, D), 55.0, dtype=out, device=DEV)
    workspace = None
    if ws:
        size = B.pafu_paged_attention_workspace_bytes(n, heads, kv_heads, D)
        workspace = torch.full((size + 64,), 0xFF, dtype=torch.uint8, device=DEV)
    d_table = ints(table)[:, :columns]
    B.pafu_paged_attention(Q, Kp, Vp, d_table, ints(lens), O[1:n + 1, :heads], n_pinned=pinned, window=window,
                           softmax_scale=scale, k_scale_log2=ks, v_scale_log2=vs,
                           workspace=workspace[:size] if ws else None)
    torch.cuda.synchronize()
    if ws:
        assert bool((workspace[size:] == 0xFF).all())
    assert bool((O[0] == 55).all() and (O[n + 1] == 55).all() and (O[:, heads] == 55).all())
    s = scale if scale > 0 else D ** -0.5
    q64 = Qw[:, :heads].double().numpy()
    want = po.paged_attention(q64, host_K, host_V, table[:, :columns], lens, s, pinned, window)
    got = O[1:n + 1, :heads].double().cpu().numpy()
    for b in range(n):
        at = [(int(table[b, j // page]), j % page) for j in po.visible_tokens(lens[b], pinned, window, columns * page)]
        at = [x for x in at if 0 <= x[0] < n_pages]
        p, o = (np.array(at).T if at else (np.zeros(0, int), np.zeros(0, int)))
        tol = _tolerance(q64[b], host_K[p, o], host_V[p, o], out, len(at), D, s)
        err = np.abs(got[b] - want[b]).max()
        assert err <= tol, (b, lens[b], err, tol)
    return O


@pytest.mark.parametrize("out", [BF, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 1), (12, 12), (32, 8), (35, 5), (48, 2), (17, 1), (64, 1)])
@pytest.mark.parametrize("columns", [None, 64], ids=["narrow table", "wide table"])   # (a wide one lets requests be cut)
def test_attention_head_layouts(heads, kv_heads, D, kv, out, columns):
    _attend([0, 1, 33, 300, 77], heads, kv_heads, D, 16, kv=kv, out=out, seed=heads * D, columns=columns)


@pytest.mark.parametrize("ws", [True, False], ids=["cut", "whole"])
@pytest.mark.parametrize("page", [8, 16, 128, 4096])
@pytest.mark.parametrize("lens", [[1], [0, 0], [31, 32, 33, 15, 16, 17, 7, 8, 9], [127, 128, 129, 255, 256, 257, 0, 511, 513],
                                  [4097, 0, 3, 1023], [6000], [0, 0, 0, 1700]], ids=str)
def test_attention_lengths_and_page_sizes(lens, page, ws):
    _attend(lens, 8, 2, 128, page, ws=ws, out=torch.float32, seed=page)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_attention_pool_layouts(layout, kv):
    for columns in (None, 100):
        _attend([70, 5, 0, 450], 6, 3, 128, 16, kv=kv, layout=layout, out=torch.float32, extra_ld=3, columns=columns)
        _attend([70, 5, 0, 450], 20, 5, 128, 16, kv=kv, layout=layout, out=torch.float32, columns=columns)
        _attend([70, 5, 0, 450], 6, 1, 64, 32, kv=kv, layout=layout, out=torch.float32, columns=columns)


@pytest.mark.parametrize("window,pinned", [(1, 0), (1, 1), (5, 0), (64, 3), (100, 33), (33, 100), (1000, 7), (5000, 0),
                                           (2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 31 - 1), (31, 31), (257, 640)])
@pytest.mark.parametrize("kv,D", [("bf16", 128), ("e4m3", 64)])
def test_attention_sliding_window_behind_a_sink(window, pinned, kv, D):
    _attend([1, 40, 0, 1300, 101, 640, 33], 8, 2, D, 16, kv=kv, out=torch.float32, window=window, pinned=pinned)


def test_attention_pages_outside_the_pool_take_no_part():
    def spoil(table):
        table[0, 2], table[0, 5], table[0, 6] = -1, 10 ** 9, -2 ** 31
        table[1, :] = -1                                   # nothing left of this one
        table[2, 0] = 2 ** 31 - 1
        table[3, 0:4] = -5
    for kv in ("bf16", "e4m3"):
        _attend([200, 50, 17, 65], 8, 4, 128, 16, kv=kv, out=torch.float32, spoil=spoil)
        _attend([200, 50, 17, 65], 8, 4, 128, 16, kv=kv, out=torch.float32, spoil=spoil, columns=80)
        _attend([2000, 50, 17, 650], 8, 4, 64, 16, kv=kv, out=torch.float32, spoil=spoil)


def test_attention_lengths_beyond_the_table_and_below_zero():
    _attend([500, 64, 65, -3, 2 ** 31 - 1], 4, 2, 128, 16, out=torch.float32, columns=4)
    _attend([500, 64, 65, -3, 200], 4, 2, 128, 16, out=torch.float32, columns=4, window=450, pinned=5)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_attention_scores_far_apart(kv):
    # scores of some hundreds: one weight takes all, and the running maximum moves again and again
    _attend([900, 64, 3, 130], 8, 2, 128, 16, kv=kv, out=torch.float32, q_gain=64.0)
    _attend([900, 64, 3, 130], 8, 2, 128, 16, kv=kv, out=torch.float32, scale=1e-30)


def test_attention_many_short_requests_and_few_long_ones():
    rng = np.random.default_rng(5)
    _attend(list(rng.integers(0, 40, 700)), 8, 2, 64, 16, out=torch.float32)
    _attend(list(rng.integers(0, 40, 700)), 8, 2, 64, 16, out=torch.float32, columns=40)
    _attend(list(rng.integers(0, 40, 300)), 16, 8, 128, 16, out=torch.float32, columns=40)
    _attend(list(rng.integers(300, 512, 130)), 8, 8, 64, 16, out=torch.float32)
    _attend(list(rng.integers(1, 300, 257)), 4, 4, 128, 8, out=BF)
    _attend([3, 20000, 1, 9, 0, 7000], 4, 1, 64, 64, out=torch.float32)


def test_attention_of_the_largest_batch():
    rng = np.random.default_rng(9)
    lens = rng.integers(0, 30, 8192)
    lens[4000:4090], lens[5000] = 0, 3000        # many without a token, one long
    _attend(list(lens), 2, 2, 64, 8, out=torch.float32)
    lens[5000] = 30
    _attend(list(lens), 2, 2, 64, 8, out=torch.float32)


def _plain_pool(rng, n_pages, page, kv_heads, D):
    return (bf16_values(rng, n_pages, page, kv_heads, D).to(DEV) for _ in range(2))


def _ws(n, heads, kv_heads, D):
    return torch.empty(B.pafu_paged_attention_workspace_bytes(n, heads, kv_heads, D), dtype=torch.uint8, device=DEV)


def test_attention_infinities_and_nan_in_sight():
    rng = np.random.default_rng(3)
    D = 64
    Kp, Vp = _plain_pool(rng, 40, 16, 1, D)
    table, lens = ints(np.arange(40).reshape(4, 10)), ints([150, 150, 150, 150])
    Q = bf16_values(rng, 4, 2, D).abs().to(DEV)
    Vp[3, 2, 0, 5] = math.inf                # request 0: a value
    Vp[13, 2, 0, 5], Vp[13, 4, 0, 6] = math.nan, -math.inf
    Kp[25, 1, 0, 7] = math.nan               # request 2: a score, so the whole row
    Kp[30:40, :, :, 3] = -math.inf           # request 3: every score is -infinity
    O = torch.empty(4, 2, D, dtype=torch.float32, device=DEV)
    for ws in (None, _ws(4, 2, 1, D)):
        O.fill_(9)
        B.pafu_paged_attention(Q, Kp, Vp, table, lens, O, workspace=ws)
        got = O.cpu()
        assert bool((got[0, :, 5] == math.inf).all()) and bool(torch.isfinite(got[0, :, [x for x in range(D) if x != 5]]).all())
        assert bool(torch.isnan(got[1, :, 5]).all()) and bool((got[1, :, 6] == -math.inf).all())
        assert bool(torch.isnan(got[2]).all())
        assert bool((got[3] == 0).all())
    # one token, whose weight is 1 to the last bit
    Vp[7, 0, 0, 9], Vp[7, 0, 0, 10] = math.inf, -math.inf
    for ws in (None, _ws(1, 2, 1, D)):
        B.pafu_paged_attention(Q[:1], Kp, Vp, ints([[7, 7]]), ints([1]), O[:1], workspace=ws)
        assert bool((O[0, :, 9] == math.inf).all()) and bool((O[0, :, 10] == -math.inf).all())
        assert bool(torch.isfinite(O[0, :, :9]).all())


def test_attention_on_a_side_stream_and_twice_with_one_result():
    rng = np.random.default_rng(4)
    Kp, Vp = _plain_pool(rng, 300, 16, 2, 128)
    table, lens = ints(rng.permutation(300).reshape(3, 100)), ints([1600, 900, 31])
    Q, ws = bf16_values(rng, 3, 8, 128).to(DEV), _ws(3, 8, 2, 128)
    first = torch.empty(3, 8, 128, dtype=torch.float32, device=DEV)
    B.pafu_paged_attention(Q, Kp, Vp, table, lens, first, workspace=ws)
    torch.cuda.synchronize()
    side, again = torch.cuda.Stream(), torch.empty_like(first)
    B.pafu_paged_attention(Q, Kp, Vp, table, lens, again, workspace=ws, stream=side)
    side.synchronize()
    assert np.array_equal(bits(first), bits(again))
    with torch.cuda.stream(side):
        again.zero_()
        ws.fill_(255)
        B.pafu_paged_attention(Q, Kp, Vp, table, lens, again, workspace=ws)
    side.synchronize()
    assert np.array_equal(bits(first), bits(again))


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_pools_beyond_32_bit_offsets(kv):
    # 4.5 GiB each of K and V: slots beyond 2^22 rows of 1 KiB, byte offsets beyond 2^32
    heads, D, page = 4, 128, 64
    dtype, width = (BF, 2) if kv == "bf16" else (torch.uint8, 1)
    n_pages = int(4.5 * 2 ** 30) // (page * heads * D * width)
    Kp, Vp = (torch.empty(n_pages, page, heads, D, dtype=dtype, device=DEV) for _ in range(2))
    rng = np.random.default_rng(6)
    n = 200
    pages = np.array([n_pages - 1, 3, n_pages - 2, n_pages // 2 + 1])
    slots = (pages[np.arange(n) // page] * page + np.arange(n) % page)
    K, V = bf16_values(rng, n, heads, D), bf16_values(rng, n, heads, D)
    ks, vs = (-5, -6) if kv == "e4m3" else (0, 0)
    B.pafu_paged_append(K.to(DEV), V.to(DEV), ints(slots), Kp, Vp, ks, vs)
    Q = bf16_values(rng, 1, 8, D)
    O = torch.empty(1, 8, D, dtype=torch.float32, device=DEV)
    B.pafu_paged_attention(Q.to(DEV), Kp, Vp, ints(pages[None]), ints([n]), O, k_scale_log2=ks, v_scale_log2=vs,
                           workspace=_ws(1, 8, heads, D))
    torch.cuda.synchronize()
    values = [x.double().numpy() if kv == "bf16" else orc.dequantise_e4m3(orc.quantise_e4m3(x.double().numpy(), s), s)
              for x, s in ((K, ks), (V, vs))]
    padded = [np.zeros((4, page, heads, D)) for _ in range(2)]
    for p, v in zip(padded, values):
        p.reshape(-1, heads, D)[:n] = v
    want = po.paged_attention(Q.double().numpy(), *padded, np.arange(4)[None], [n])
    tol = _tolerance(Q.double().numpy()[0], values[0], values[1], torch.float32, n, D, D ** -0.5)
    assert np.abs(O.double().cpu().numpy() - want).max() <= tol


# ------------------------------------------------------------------------------------------------ together
class _Decode:
    """A decode loop of a padded batch: pages and slots, rows into the cache, attention; lengths ping-pong."""

    def __init__(self, n, heads, kv_heads, D, page, columns, kv, seed=0):
        rng = np.random.default_rng(seed)
        self.n, self.heads, self.kv_heads, self.D, self.page, self.kv = n, heads, kv_heads, D, page, kv
        self.n_pages = n * columns
        dtype = BF if kv == "bf16" else torch.uint8
        self.Kp, self.Vp = (torch.full((self.n_pages, page, kv_heads, D), 255 if kv != "bf16" else math.nan, dtype=dtype,
                                       device=DEV) for _ in range(2))
        self.scales = (-5, -6) if kv == "e4m3" else (0, 0)
        self.free = rng.permutation(self.n_pages)
        self.d_free = ints(self.free)
        self.table = ints(np.full((n, columns), -1))
        self.lens = [ints(np.zeros(n)), ints(np.zeros(n))]
        self.ends = [ints([0]), ints([0])]
        self.row_start = ints(np.zeros(n + 1))
        self.ws = _ws(n, heads, kv_heads, D)

    def step(self, i, new, K, V, Q, slots, O):
        old, out = i & 1, 1 - (i & 1)
        B.pafu_paged_tables(self.lens[old], new, self.d_free, self.page, self.table, slots, self.row_start, self.lens[out],
                            self.ends[out], free_start=self.ends[old])
        B.pafu_paged_append(K, V, slots, self.Kp, self.Vp, *self.scales)
        B.pafu_paged_attention(Q, self.Kp, self.Vp, self.table, self.lens[out], O, k_scale_log2=self.scales[0],
                               v_scale_log2=self.scales[1], workspace=self.ws)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_prompts_then_decode_steps_follow_dense_caches(kv):
    n, heads, kv_heads, D, page = 5, 8, 2, 128, 16
    rng = np.random.default_rng(11)
    d = _Decode(n, heads, kv_heads, D, page, 12, kv)
    dense = [[[], []] for _ in range(n)]
    for i in range(6):
        # two ragged launches of prompts (one request empty), then one token each but for an idle place
        new = [np.array([40, 0, 7, 100, 16]), np.array([3, 20, 0, 1, 33])][i] if i < 2 else np.array([1, 1, 1, 0, 1])
        rows = int(new.sum()) + 4                                   # a padded launch
        K, V, Q = bf16_values(rng, rows, kv_heads, D), bf16_values(rng, rows, kv_heads, D), bf16_values(rng, n, heads, D)
        slots = ints(np.full(rows, 5))
        O = torch.full((n, heads, D), 9.0, dtype=torch.float32, device=DEV)
        d.step(i, ints(new), K.to(DEV), V.to(DEV), Q.to(DEV), slots, O)
        torch.cuda.synchronize()
        at = 0
        for b in range(n):
            for x, s, kept in ((K, d.scales[0], dense[b][0]), (V, d.scales[1], dense[b][1])):
                v = x[at:at + new[b]].double().numpy()
                kept.extend(v if kv == "bf16" else orc.dequantise_e4m3(orc.quantise_e4m3(v, s), s))
            at += new[b]
        got = O.double().cpu().numpy()
        for b in range(n):
            if not dense[b][0]:
                assert np.all(got[b] == 0)
                continue
            k, v, q = np.array(dense[b][0]), np.array(dense[b][1]), Q[b].double().numpy()
            g = np.repeat(np.arange(kv_heads), heads // kv_heads)
            want = orc.chunk_attention(q[None], k[:-1][:, g], v[:-1][:, g], k[-1:][:, g], v[-1:][:, g], 1)[0]
            tol = _tolerance(q, k, v, torch.float32, len(k), D, D ** -0.5)
            assert np.abs(got[b] - want).max() <= tol, (i, b)


def test_captured_decode_steps_follow_the_lengths_on_the_device():
    n, heads, kv_heads, D, page = 4, 8, 2, 64, 8
    runs = []
    for captured in (False, True):
        rng = np.random.default_rng(12)
        d = _Decode(n, heads, kv_heads, D, page, 20, "bf16", seed=1)
        d.Kp.zero_(); d.Vp.zero_()
        bufs = [(torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n + 60, kv_heads, D, dtype=BF, device=DEV),
                 torch.zeros(n + 60, kv_heads, D, dtype=BF, device=DEV), torch.zeros(n, heads, D, dtype=BF, device=DEV),
                 torch.zeros(n + 60, dtype=torch.int32, device=DEV), torch.zeros(n, heads, D, dtype=BF, device=DEV))
                for _ in range(2)]
        graphs = []
        if captured:  # one graph for each direction of the ping-pong; both use the one workspace
            warm = torch.cuda.Stream()
            with torch.cuda.stream(warm):
                d.step(0, *bufs[0])
                d.step(1, *bufs[1])
            torch.cuda.synchronize()
            for x in d.lens + d.ends:
                x.zero_()
            d.table.fill_(-1)
            for i in range(2):
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g):
                    d.step(i, *bufs[i])
                graphs.append(g)
            torch.cuda.synchronize()
        outs = []
        for i in range(8):
            new = rng.integers(0, 16, n) if i < 3 else (rng.random(n) < 0.8).astype(int)
            new_d, K, V, Q, slots, O = bufs[i & 1]
            new_d.copy_(ints(new))
            for x in (K, V, Q):
                x.copy_(bf16_values(rng, *x.shape).to(DEV))
            O.fill_(3)
            torch.cuda.synchronize()
            if captured:
                graphs[i & 1].replay()
            else:
                d.step(i, *bufs[i & 1])
            torch.cuda.synchronize()
            outs.append([bits(O).copy(), slots.cpu().numpy(), d.table.cpu().numpy(), d.lens[1 - (i & 1)].cpu().numpy(),
                         bits(d.Kp).copy(), bits(d.Vp).copy()])
        runs.append(outs)
    for i, (eager, replayed) in enumerate(zip(*runs)):
        for a, b in zip(eager, replayed):
            assert np.array_equal(a, b), i


def test_slots_are_row_ids_for_the_gather_attention_and_the_compaction():
    # a chunk of queries over a paged cache through the slots, and a selection compacted out of the pages
    n, heads, D, page = 333, 4, 128, 16
    rng = np.random.default_rng(13)
    Kp, Vp = _plain_pool(rng, 30, page, heads, D)
    table = ints(rng.permutation(30)[:21][None])
    slots, row_start = ints(np.full(336, 7)), ints([0, 0])
    B.pafu_paged_slots(table, ints([0]), ints([n]), page, slots, row_start)
    Krows, Vrows = Kp.view(-1, heads, D), Vp.view(-1, heads, D)
    Q, Kn, Vn = (bf16_values(rng, 70, heads, D).to(DEV) for _ in range(3))
    O, want = (torch.empty(70, heads, D, dtype=torch.float32, device=DEV) for _ in range(2))
    B.pafu_chunk_attention_gather(Q, Krows, Vrows, slots, n, Kn, Vn, 70, O)
    dense_K, dense_V = Krows[slots[:n].long()].contiguous(), Vrows[slots[:n].long()].contiguous()
    B.pafu_chunk_attention_gather(Q, dense_K, dense_V, ints(np.arange(n)), n, Kn, Vn, 70, want)
    assert np.array_equal(bits(O), bits(want))
    # keep the 100 most salient tokens of the request, dense, then on fresh pages
    scores = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).to(DEV)
    ids = ints(np.zeros(100))
    B.pafu_select_topk(scores, 100, ids)
    rows = slots[ids.long()].contiguous()
    K2, V2 = (torch.empty(100, heads, D, dtype=BF, device=DEV) for _ in range(2))
    B.pafu_compact_kv(Krows, Vrows, None, rows, 100, K2, V2, None)
    kept = orc.select_topk(scores.cpu().numpy(), 100)
    assert np.array_equal(bits(K2), bits(dense_K)[kept]) and np.array_equal(bits(V2), bits(dense_V)[kept])
