"""The paged K/V cache at the limits of its numbers: sums of pages that saturate, the bits of the attention's weights, infinities,
rows that see nothing."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from oracle import pafu_oracle as orc
from paper_2601_21896_amd import binding as B
from tests.gpu_util import DEV
from tests.test_gpu_paged import _tables, bf16_values

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _codes(x):
    """Pages as they are stored: bf16 values, or the E4M3 codes of x (scale 1)."""
    return torch.from_numpy(orc.quantise_e4m3(x.double().numpy(), 0)).to(DEV)


def _workspace(n, heads, kv_heads, D):
    """The bytes of a call's workspace, filled with 0xa5."""
    size = B.pafu_paged_attention_workspace_bytes(n, heads, kv_heads, D)
    return torch.full((size,), 0xA5, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("columns", [8, 80], ids=["whole", "cut"])   # (room for more than 512 tokens: cut)
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,kv_heads,D", [(16, 1, 128), (8, 4, 128), (32, 1, 128), (16, 4, 64), (48, 1, 64)])
def test_attention_weights_keep_their_24_bits(heads, kv_heads, D, kv, columns):
    # Values are rows of the identity, token j's is 1 at element j: the result is the softmax itself.  Scores are one exact
    # product each, q0 * k0, of at most 4 in steps that bf16 and E4M3 hold.
    n, tokens, page = 6, 64, 16
    rng = np.random.default_rng(heads + D)
    K, V = torch.zeros(n, columns * page, kv_heads, D), torch.zeros(n, columns * page, kv_heads, D)
    k0 = rng.integers(-8, 9, (n, tokens, kv_heads)) / 8.0               # 4 bits: E4M3 numbers
    q0 = rng.integers(-255, 256, (n, heads)) / 64.0                     # 8 bits: bf16 numbers
    K[:, :tokens, :, 0] = torch.from_numpy(k0).float()
    V[:, torch.arange(tokens), :, torch.arange(tokens)] = 1.0
    store = (lambda x: x.to(BF).to(DEV)) if kv == "bf16" else _codes
    Kp, Vp = (store(x.view(n * columns, page, kv_heads, D)) for x in (K, V))
    Q = torch.zeros(n, heads, D)
    Q[:, :, 0] = torch.from_numpy(q0).float()
    O = torch.empty(n, heads, D, dtype=torch.float32, device=DEV)
    ws = _workspace(n, heads, kv_heads, D)
    B.pafu_paged_attention(Q.to(BF).to(DEV), Kp, Vp, ints(np.arange(n * columns).reshape(n, columns)), ints([tokens] * n), O,
                           softmax_scale=1.0, workspace=ws)
    assert bool((ws != 0xA5).any()) == (columns > 32)                   # cut or not: as named
    s = q0[:, :, None] * np.repeat(k0.transpose(0, 2, 1), heads // kv_heads, axis=1)
    w = np.exp(s - s.max(-1, keepdims=True))
    w /= w.sum(-1, keepdims=True)
    got = O.double().cpu().numpy()
    # In units u = 2^-24.  A score in the exponent of 2 is at most 5.8, the distance to the reference at most 11.6 (and 8 more
    # where the reference lags).  Scale times log2(e): three roundings, 3 * 11.6 of the distance; the reference's own rounding 5.8,
    # the distance's 20: 61, times ln 2: 42.  exp2: 2.  That holds for the weight and for the normaliser: 88.  Sums and rescalings of
    # 64 weights: 24; of a result 8; the division and the product by it: 4.  Weights off by 2^-16 would be off by 256.
    err = np.abs(got[:, :, :tokens] - w) / w
    assert err.max() <= 124 * 2.0 ** -24, err.max() * 2.0 ** 24
    assert bool((O[:, :, tokens:] == 0).all())


@pytest.mark.parametrize("columns", [8, 80], ids=["whole", "cut"])
@pytest.mark.parametrize("heads,kv_heads,D", [(4, 1, 128), (32, 1, 128), (48, 1, 64)])
def test_attention_infinite_values_under_small_weights(heads, kv_heads, D, columns):
    # a weight of 2^-x is not 0 as long as fp32 has it: times an infinite value it is infinite
    page = 16
    for x in (8, 60, 100, 112, 120, 125):
        K, V = (torch.zeros(columns, page, 1, D) for _ in range(2))
        K[:, :, 0, 0] = -1.0
        K[1, 3, 0, 0] = 0.0                                             # the highest score
        V[0, 5, 0, 7], V[2, 1, 0, 9], V[1, 3, 0, 2] = math.inf, -math.inf, 1.0
        Q = torch.zeros(1, heads, D)
        Q[:, :, 0] = 1.0
        O = torch.empty(1, heads, D, dtype=torch.float32, device=DEV)
        B.pafu_paged_attention(Q.to(BF).to(DEV), K.to(BF).to(DEV), V.to(BF).to(DEV), ints(np.arange(columns)[None]), ints([100]), O,
                               softmax_scale=x * math.log(2.0), workspace=_workspace(1, heads, kv_heads, D))
        got = O[0].cpu()
        assert bool((got[:, 7] == math.inf).all() and (got[:, 9] == -math.inf).all()), x
        rest = [d for d in range(D) if d not in (7, 9)]
        assert bool(torch.isfinite(got[:, rest]).all()), x


@pytest.mark.parametrize("kv,new,page,start", [
    ([0, 0], [8, 8], 8, 2 ** 31 - 2),
    ([3, 5, 0, 100, 7], [40, 600, 0, 30, 1], 8, 2 ** 31 - 3),
    ([0, 0, 3], [5000, 2500, 900], 16, 2 ** 31 - 200),
    ([16] * 300, [33] * 300, 16, 2 ** 31 - 100),
    ([0, 9], [20, 20], 8, 2 ** 31 - 1)],
                         ids=["one page each", "within a request", "many pages", "300 requests", "from the start"])
def test_tables_enter_pages_behind_a_saturated_sum_as_missing(kv, new, page, start):
    _tables(kv, new, 5, page, max(-(-(a + b) // page) for a, b in zip(kv, new)), sum(new) + 3, start, extra_ld=1)


@pytest.mark.parametrize("columns", [8, 80], ids=["whole", "cut"])
@pytest.mark.parametrize("heads,kv_heads,D", [(4, 1, 128), (8, 8, 64), (48, 1, 64)])
def test_attention_of_scores_that_are_all_minus_infinity_is_0_whatever_the_values(heads, kv_heads, D, columns):
    page = 16
    K, V = (torch.ones(2 * columns, page, kv_heads, D, dtype=BF, device=DEV) for _ in range(2))
    K[:columns] = -math.inf
    V[0, 0], V[0, 1], V[1, 1] = math.inf, math.nan, -math.inf
    for tokens in (1, 20, 100):
        O = torch.full((2, heads, D), 9.0, dtype=torch.float32, device=DEV)
        B.pafu_paged_attention(torch.ones(2, heads, D, dtype=BF, device=DEV), K, V, ints(np.arange(2 * columns).reshape(2, columns)),
                               ints([tokens, tokens]), O, workspace=_workspace(2, heads, kv_heads, D))
        assert bool((O[0] == 0).all()), tokens
        assert bool((O[1] == 1).all()), tokens


def _side_by_side(layout, n_pages, page, heads, D, dtype):
    """A slab of numbers, and how K and V lie in it."""
    shape, views = {
        "rows alternate": ((n_pages, page, 2, heads, D), lambda s: (s[:, :, 0], s[:, :, 1])),
        "rows alternate, gaps": ((n_pages, page + 3, 2, heads + 1, D), lambda s: (s[:, :page, 1, :heads], s[:, 1:page + 1, 0, 1:])),
        "heads alternate": ((n_pages, heads, 2, page, D), lambda s: (s[:, :, 1].permute(0, 2, 1, 3), s[:, :, 0].permute(0, 2, 1, 3))),
        "pages alternate": ((n_pages, 2, page, heads, D), lambda s: (s[:, 1], s[:, 0])),
        "pages and heads alternate": ((n_pages, 2, heads, page, D), lambda s: (s[:, 0].permute(0, 2, 1, 3), s[:, 1].permute(0, 2, 1, 3))),
    }[layout]
    count = int(np.prod(shape))
    numbers = torch.arange(count, dtype=torch.int32) * 7919 % 251
    return (numbers.to(BF) if dtype == BF else numbers.to(torch.uint8)).view(shape), views


@pytest.mark.parametrize("n_pages", [1, 3])
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,D", [(1, 64), (3, 128)])
@pytest.mark.parametrize("layout", ["rows alternate", "rows alternate, gaps", "heads alternate", "pages alternate",
                                    "pages and heads alternate"])
def test_append_to_pools_that_lie_side_by_side(layout, heads, D, kv, n_pages):
    page, dtype = 16, BF if kv == "bf16" else torch.uint8
    rng = np.random.default_rng(heads + n_pages)
    slab, views = _side_by_side(layout, n_pages, page, heads, D, dtype)
    slots = rng.permutation(n_pages * page)[:13]
    rows = [bf16_values(rng, 13, heads, D) for _ in range(2)]
    on_gpu = slab.to(DEV)
    B.pafu_paged_append(*(x.to(DEV) for x in rows), ints(slots), *views(on_gpu))
    want = slab.clone().view(torch.int16 if dtype == BF else torch.uint8)
    for t, x in zip(views(want), rows):
        new = x.view(torch.int16).numpy() if dtype == BF else orc.quantise_e4m3(x.double().numpy(), 0)
        t.copy_(torch.from_numpy(po.paged_append(t.numpy(), new, slots)))
    assert torch.equal(on_gpu.cpu().view(want.dtype), want)


@pytest.mark.parametrize("columns", [8, 80], ids=["whole", "cut"])
@pytest.mark.parametrize("heads,kv_heads,D", [(16, 1, 128), (8, 4, 128), (32, 1, 128), (16, 4, 64), (48, 1, 64)])
def test_attention_of_scores_far_beyond_the_range_of_weights(heads, kv_heads, D, columns):
    # scores of 2^20 .. 2^80, each one exact product: the tokens of the highest share the weight equally, the others have none
    n, tokens, page = 3, 64, 16
    rng = np.random.default_rng(heads + D)
    V = torch.zeros(n, columns * page, kv_heads, D)
    V[:, torch.arange(tokens), :, torch.arange(tokens)] = 1.0
    Vp = V.view(n * columns, page, kv_heads, D).to(BF).to(DEV)
    for gain in (2.0 ** 20, 2.0 ** 31, 2.0 ** 40, 2.0 ** 80):
        K, Q = torch.zeros(n, columns * page, kv_heads, D), torch.zeros(n, heads, D)
        k0 = rng.integers(-127, 128, (n, tokens, kv_heads)) / 128.0
        k0[:, 40:] = k0[:, 10:34]                                       # pairs, in one tile and in two
        q0 = rng.integers(129, 256, (n, heads)) * rng.choice([-1, 1], (n, heads)) / 128.0 * gain
        K[:, :tokens, :, 0], Q[:, :, 0] = torch.from_numpy(k0).float(), torch.from_numpy(q0).float()
        Kp = K.view(n * columns, page, kv_heads, D).to(BF).to(DEV)
        O = torch.empty(n, heads, D, dtype=torch.float32, device=DEV)
        B.pafu_paged_attention(Q.to(BF).to(DEV), Kp, Vp, ints(np.arange(n * columns).reshape(n, columns)), ints([tokens] * n), O,
                               softmax_scale=0.3, workspace=_workspace(n, heads, kv_heads, D))
        s = q0[:, :, None] * np.repeat(k0.transpose(0, 2, 1), heads // kv_heads, axis=1)
        best = s == s.max(-1, keepdims=True)
        want = best / best.sum(-1, keepdims=True)                       # (the next one is gain / 2^14 * 0.3 below, 2^4 at least ...
        w = np.exp(0.3 * (s - s.max(-1, keepdims=True)))
        w /= w.sum(-1, keepdims=True)
        assert np.abs(w - want).max() <= 2.0 ** -24                     # ... so this holds)
        # weights 2^0 of exact differences, sums of at most 64 of them, a division and a product: as above without the scores' part
        got = O.double().cpu().numpy()[:, :, :tokens]
        assert np.abs(got - want).max() <= 40 * 2.0 ** -24, gain
