"""The paged calls in every way their launches are planned: whole and cut requests (partial results in the workspace and their
join), small and large calls, all counts of query heads, layouts and masks together, appends past the caches."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from oracle import pafu_oracle as orc
from paper_2601_21896_amd import binding as B
from tests import test_gpu_paged as t
from tests.gpu_util import DEV, bits

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture
def cut(monkeypatch):
    """Whether the calls of a test left something in their workspaces, which hold one byte's value over and over before."""
    seen, call = [], B.pafu_paged_attention

    def spy(*a, **kw):
        ws = kw.get("workspace")
        before = None if ws is None else int(ws[0]) if ws.numel() else 0
        if ws is not None:
            assert bool((ws == before).all())
        out = call(*a, **kw)
        seen.append(ws is not None and bool((ws != before).any()))
        return out
    monkeypatch.setattr(B, "pafu_paged_attention", spy)
    return seen


# 704 tokens of room a request: cut where there is a workspace, and read through the caches; 65536: past them where they may be
ROOM = {"small": 44, "large": 4096}
LENS = [0, 1, 33, 700, 77]


@pytest.mark.parametrize("room", ROOM)
@pytest.mark.parametrize("plan", ["cut", "whole"])
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,kv_heads,D", [
    (4, 4, 128), (12, 3, 128), (24, 1, 128), (32, 1, 128), (68, 4, 128), (48, 1, 128), (130, 2, 128),
    (4, 4, 64), (12, 3, 64), (17, 1, 64), (128, 4, 64), (33, 1, 64), (48, 1, 64), (160, 4, 64), (64, 1, 64), (100, 1, 64)])
def test_attention_of_every_kernel(cut, heads, kv_heads, D, kv, plan, room):
    _attend = t._attend
    for layout in ("token", "head", "gaps"):
        _attend(LENS, heads, kv_heads, D, 16, kv=kv, layout=layout, out=torch.float32, columns=ROOM[room], ws=plan == "cut", seed=D)
    _attend(LENS, heads, kv_heads, D, 16, kv=kv, out=BF, columns=ROOM[room], ws=plan == "cut", window=300, pinned=40)
    _attend(LENS, heads, kv_heads, D, 16, kv=kv, layout="head", out=torch.float32, columns=ROOM[room], ws=plan == "cut", window=90,
            pinned=500)
    assert cut == [plan == "cut"] * 5


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,kv_heads,D", [(4, 1, 128), (24, 1, 128), (8, 8, 64), (17, 1, 64), (40, 1, 64), (96, 2, 64)])
def test_attention_of_many_short_requests(cut, heads, kv_heads, D, kv):
    # room for at most 256 tokens: whole, a wave each where there are more than 512 of them
    rng = np.random.default_rng(heads)
    for n, page, layout in ((600 // kv_heads + 7, 16, "token"), (600 // kv_heads + 7, 32, "head"), (50, 16, "gaps")):
        lens = rng.integers(0, 60, n)
        lens[n // 2] = 250
        t._attend(list(lens), heads, kv_heads, D, page, kv=kv, layout=layout, out=torch.float32, columns=256 // page)
        t._attend(list(lens), heads, kv_heads, D, page, kv=kv, layout=layout, out=torch.float32, columns=256 // page, window=50,
                  pinned=9)
    assert not any(cut)


@pytest.mark.parametrize("heads,kv_heads,D,cuts", [(16, 4, 128, True), (64, 4, 64, True), (68, 4, 128, False), (96, 4, 64, False),
                                                   (128, 4, 64, False)])
def test_attention_of_up_to_512_tokens_is_cut_for_few_query_heads_to_a_key_head(cut, heads, kv_heads, D, cuts):
    # 560 waves and more: two workgroups to a unit, not four
    rng = np.random.default_rng(heads)
    t._attend(list(rng.integers(1, 401, 140)), heads, kv_heads, D, 16, out=torch.float32, columns=25)
    assert cut == [cuts]


@pytest.mark.parametrize("n,kv", [(63, "bf16"), (64, "e4m3"), (65, "bf16"), (130, "e4m3"), (300, "bf16"), (700, "bf16")])
@pytest.mark.parametrize("window,pinned", [(0, 0), (100, 20), (31, 700), (600, 1)])
def test_attention_of_cut_batches_with_windows(cut, n, kv, window, pinned):
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 120, n)
    lens[n // 3], lens[n - 1], lens[1] = 1200, 640, 0
    t._attend(list(lens), 8, 4, 64, 16, kv=kv, out=torch.float32, columns=80, window=window, pinned=pinned)
    t._attend(list(lens), 4, 2, 128, 32, kv=kv, layout="head", out=torch.float32, columns=40, window=window, pinned=pinned)
    assert all(cut)


@pytest.mark.parametrize("layout", ["token", "head"])
def test_attention_of_runs_of_several_tiles_and_requests(cut, layout):
    # 128 (head dim 64: as many) runs of several tiles: requests within a run, over two and over many
    t._attend([5000, 40, 3000, 70, 0, 1, 4100, 33, 33], 16, 16, 64, 64, layout=layout, out=torch.float32)
    t._attend([5000, 40, 3000, 70, 0, 1, 4100, 33, 33], 16, 16, 128, 64, kv="e4m3", layout=layout, out=torch.float32, window=4096,
              pinned=64)
    assert all(cut)


def test_attention_of_infinities_and_nan_in_cut_requests(cut):
    rng = np.random.default_rng(3)
    D, n, page, columns = 64, 4, 16, 64
    Kp, Vp = t._plain_pool(rng, n * columns, page, 1, D)
    table, lens = t.ints(np.arange(n * columns).reshape(n, columns)), t.ints([900] * n)
    Q = t.bf16_values(rng, n, 2, D).abs().to(DEV)
    Vp[3, 2, 0, 5] = Vp[40, 2, 0, 5] = math.inf                        # request 0: values, in two runs
    Vp[30, 1, 0, 6], Vp[50, 1, 0, 6] = math.inf, -math.inf             # and two whose sum is none
    Vp[64 + 3, 2, 0, 5], Vp[64 + 40, 4, 0, 6] = math.nan, -math.inf    # request 1
    Kp[2 * 64 + 25, 1, 0, 7] = math.nan                                # request 2: a score, so the whole row
    Kp[3 * 64:] *= 0
    Kp[3 * 64:, :, :, 3] = -math.inf                                   # request 3: every score is -infinity
    Vp[3 * 64 + 20, 1] = math.nan
    O = torch.empty(n, 2, D, dtype=torch.float32, device=DEV)
    for ws in (None, t._ws(n, 2, 1, D)):
        O.fill_(9)
        if ws is not None:
            ws.fill_(0xFF)                                             # NaN
        B.pafu_paged_attention(Q, Kp, Vp, table, lens, O, workspace=ws)
        got = O.cpu()
        rest = [x for x in range(D) if x not in (5, 6)]
        assert bool((got[0, :, 5] == math.inf).all()) and bool(torch.isnan(got[0, :, 6]).all())
        assert bool(torch.isfinite(got[0][:, rest]).all()) and bool(torch.isfinite(got[1][:, rest]).all())
        assert bool(torch.isnan(got[1, :, 5]).all()) and bool((got[1, :, 6] == -math.inf).all())
        assert bool(torch.isnan(got[2]).all())
        assert bool((got[3] == 0).all())
    assert cut == [False, True]


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("layout", ["token", "head"])
def test_cut_requests_in_pools_beyond_32_bit_offsets(cut, kv, layout):
    # 4.5 GiB each of K and V, a request's pages at both ends
    heads, D, page, n, columns = 4, 128, 64, 700, 16
    dtype, width = (BF, 2) if kv == "bf16" else (torch.uint8, 1)
    n_pages = int(4.5 * 2 ** 30) // (page * heads * D * width)
    shape = (n_pages, page, heads, D) if layout == "token" else (n_pages, heads, page, D)
    Kp, Vp = (torch.empty(shape, dtype=dtype, device=DEV) for _ in range(2))
    if layout == "head":
        Kp, Vp = Kp.permute(0, 2, 1, 3), Vp.permute(0, 2, 1, 3)
    rng = np.random.default_rng(6)
    pages = np.concatenate([n_pages - 1 - np.arange(0, 12, 2), [3, n_pages // 2, n_pages - 2, 0, n_pages - 4, 1, 5, 7, 9, 11]])
    slots = pages[np.arange(n) // page] * page + np.arange(n) % page
    K, V = t.bf16_values(rng, n, heads, D), t.bf16_values(rng, n, heads, D)
    ks, vs = (-5, -6) if kv == "e4m3" else (0, 0)
    B.pafu_paged_append(K.to(DEV), V.to(DEV), t.ints(slots), Kp, Vp, ks, vs)
    Q = t.bf16_values(rng, 1, 8, D)
    O = torch.empty(1, 8, D, dtype=torch.float32, device=DEV)
    B.pafu_paged_attention(Q.to(DEV), Kp, Vp, t.ints(pages[None]), t.ints([n]), O, k_scale_log2=ks, v_scale_log2=vs,
                           workspace=t._ws(1, 8, heads, D).fill_(0xA5))
    values = [x.double().numpy() if kv == "bf16" else orc.dequantise_e4m3(orc.quantise_e4m3(x.double().numpy(), s), s)
              for x, s in ((K, ks), (V, vs))]
    padded = [np.zeros((columns, page, heads, D)) for _ in range(2)]
    for p, v in zip(padded, values):
        p.reshape(-1, heads, D)[:n] = v
    want = po.paged_attention(Q.double().numpy(), *padded, np.arange(columns)[None], [n])
    tol = t._tolerance(Q.double().numpy()[0], values[0], values[1], torch.float32, n, D, D ** -0.5)
    assert np.abs(O.double().cpu().numpy() - want).max() <= tol
    assert cut == [True]


def test_attention_where_the_strides_of_one_head_differ():
    rng = np.random.default_rng(8)
    K, V = t._plain_pool(rng, 50, 16, 1, 64)
    V2 = V.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    by_heads = torch.empty(50, 1, 16, 64, dtype=BF, device=DEV).copy_(V.permute(0, 2, 1, 3)).permute(0, 2, 1, 3)
    Q, table, lens = t.bf16_values(rng, 2, 4, 64).to(DEV), t.ints(rng.permutation(50).reshape(2, 25)), t.ints([400, 31])
    want, got = (torch.empty(2, 4, 64, dtype=BF, device=DEV) for _ in range(2))
    B.pafu_paged_attention(Q, K, V, table, lens, want)
    for other in (V2, by_heads):
        B.pafu_paged_attention(Q, K, other, table, lens, got)
        assert np.array_equal(bits(want), bits(got))


# ------------------------------------------------------------------------------------------------ together, with cut requests
@pytest.mark.parametrize("kv,heads,kv_heads,D", [("bf16", 8, 2, 128), ("e4m3", 8, 8, 64), ("bf16", 40, 1, 64)])
def test_long_prompts_then_decode_steps_follow_dense_caches(cut, kv, heads, kv_heads, D):
    n, page = 5, 16
    rng = np.random.default_rng(11)
    d = t._Decode(n, heads, kv_heads, D, page, 60, kv)
    dense = [[[], []] for _ in range(n)]
    for i in range(5):
        new = [np.array([400, 0, 7, 500, 160]), np.array([300, 200, 0, 1, 33])][i] if i < 2 else np.array([1, 1, 1, 0, 1])
        rows = int(new.sum()) + 4                                   # a padded launch
        K, V, Q = t.bf16_values(rng, rows, kv_heads, D), t.bf16_values(rng, rows, kv_heads, D), t.bf16_values(rng, n, heads, D)
        slots = t.ints(np.full(rows, 5))
        O = torch.full((n, heads, D), 9.0, dtype=torch.float32, device=DEV)
        d.ws.fill_(0xFF)
        d.step(i, t.ints(new), K.to(DEV), V.to(DEV), Q.to(DEV), slots, O)
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
            assert np.abs(got[b] - want).max() <= t._tolerance(q, k, v, torch.float32, len(k), D, D ** -0.5), (i, b)
    assert all(cut) and len(cut) == 5


def test_captured_steps_of_cut_requests_follow_the_lengths_and_share_a_workspace():
    n, heads, kv_heads, D, page, most = 4, 8, 2, 64, 8, 4 * 150 + 40
    runs = []
    for captured in (False, True):
        rng = np.random.default_rng(12)
        d = t._Decode(n, heads, kv_heads, D, page, 90, "bf16", seed=1)
        d.Kp.zero_(); d.Vp.zero_()
        bufs = [(torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(most, kv_heads, D, dtype=BF, device=DEV),
                 torch.zeros(most, kv_heads, D, dtype=BF, device=DEV), torch.zeros(n, heads, D, dtype=BF, device=DEV),
                 torch.zeros(most, dtype=torch.int32, device=DEV), torch.zeros(n, heads, D, dtype=torch.float32, device=DEV))
                for _ in range(2)]
        graphs = []
        if captured:
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
        for i in range(9):
            new = rng.integers(0, 150, n) if i < 4 else (rng.random(n) < 0.8).astype(int)
            new_d, K, V, Q, slots, O = bufs[i & 1]
            new_d.copy_(t.ints(new))
            for x in (K, V, Q):
                x.copy_(t.bf16_values(rng, *x.shape).to(DEV))
            O.fill_(3)
            d.ws.fill_(0xFF)                                        # nothing is kept in it from one replay to the next
            torch.cuda.synchronize()
            if captured:
                graphs[i & 1].replay()
            else:
                d.step(i, *bufs[i & 1])
            torch.cuda.synchronize()
            assert bool((d.ws != 0xFF).any())
            outs.append([bits(O).copy(), slots.cpu().numpy(), d.table.cpu().numpy(), d.lens[1 - (i & 1)].cpu().numpy(),
                         bits(d.Kp).copy(), bits(d.Vp).copy()])
        runs.append(outs)
    for i, (eager, replayed) in enumerate(zip(*runs)):
        for a, b in zip(eager, replayed):
            assert np.array_equal(a, b), i


# ------------------------------------------------------------------------------------------------ appends past the caches
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows,heads,D,page,layout", [
    (16384, 8, 128, 16, "token"),       # 64 MiB of K and V, where they begin to pass the caches
    (16385, 8, 128, 16, "head"), (33000, 16, 64, 8, "token"),
    (212000, 5, 128, 64, "token"),      # more rows than the launch has threads for at once: a second turn each, at another column
    (190000, 12, 64, 64, "head")])
def test_large_appends_are_bit_exact(rows, heads, D, page, layout, kv):
    assert rows * heads * D * 4 >= 64 << 20
    g = torch.Generator(device=DEV)
    g.manual_seed(rows)
    n_pages = -(-rows // page) + 3
    dtype = BF if kv == "bf16" else torch.uint8
    shape = (n_pages, page, heads, D) if layout == "token" else (n_pages, heads, page, D)
    pages = [torch.full(shape, 3, dtype=dtype, device=DEV) for _ in range(2)]
    if layout == "head":
        pages = [x.permute(0, 2, 1, 3) for x in pages]
    want = [x.clone() for x in pages]
    K, V = (torch.randn(rows, heads, D, device=DEV, generator=g).to(BF) for _ in range(2))
    slots = torch.randperm(n_pages * page, device=DEV, generator=g)[:rows]
    left_out = torch.rand(rows, device=DEV, generator=g) < 0.02
    left_out[rows // 2] = left_out[rows - 1] = True
    slots = torch.where(left_out, torch.where(slots % 2 == 0, -1, n_pages * page + slots), slots)
    ks, vs = (-5, -6) if kv == "e4m3" else (0, 0)
    B.pafu_paged_append(K, V, slots.to(torch.int32), *pages, ks, vs)
    stored = [K, V]
    if kv == "e4m3":
        stored = [torch.empty(rows, heads, D, dtype=torch.uint8, device=DEV) for _ in range(2)]
        B.pafu_quantize_kv(K, V, ks, vs, *stored)
    used = slots[~left_out]
    for w, x, got in zip(want, stored, pages):
        w[used // page, used % page] = x[~left_out]
        assert torch.equal(w.view(torch.int16) if dtype == BF else w, got.view(torch.int16) if dtype == BF else got)
