"""The paged calls at the limits of what they accept, on the host (no GPU needed).  Calls that are to be accepted pass NULL for
Q, which is told after the shapes: nothing is launched."""
import pytest
import torch

from paper_2601_21896_amd import binding as B

A = 0x10000  # a fake, 16-byte aligned "device address"
MB = 0x100000


def _attention(**kw):
    a = dict(Q=None, ldq=1024, Kp=A + 0x10000000, Vp=A + 0x20000000, np=10, ps=32, ldp=32 * 256, ldt=256, ldh=128, dt=0, ks=0, vs=0,
             table=A + MB, mp=8, ld=8, kv=A + 2 * MB, B=4, N=8, Nkv=2, D=128, pin=0, win=0, sc=0.0, O=A + 3 * MB, ldo=1024, od=0,
             ws=None, wsb=0)
    a.update(kw)
    return B.library().pafu_paged_attention(None, *a.values())


def _tiles(length, window, pinned):
    """32-token tiles that hold a request's visible tokens, those of the sink and those of the window in tiles of their own."""
    lo = length - window if 0 < window < length else 0
    pin = min(pinned, length) if lo > min(pinned, length) else 0
    lo = lo if pin or lo > pinned else 0
    return -(-pin // 32) + (-(-(length - lo // 32 * 32) // 32))


def test_attention_refuses_more_tiles_than_32_bits_count_with_a_sink_too():
    columns = (2 ** 31 - 1) // 8192                     # of 32 tokens: a tile each
    assert 8192 * columns < 2 ** 31 <= 8192 * (columns + 1)
    # a sink and a window that begins inside a tile: one tile more than the table has room for
    assert _tiles(columns * 32, columns * 32 - 17, 1) == columns + 1
    assert _tiles(columns * 32, columns * 32 - 17, 0) == _tiles(columns * 32, 0, 1) == columns
    big = dict(B=8192, mp=columns, ld=columns)
    assert _attention(**big) == _attention(**big, win=columns * 32 - 17) == _attention(**big, pin=1) == -1
    assert _attention(**big, win=columns * 32 - 17, pin=1) == -2
    assert _attention(**dict(big, mp=columns - 1), win=columns * 32 - 17, pin=1) == -1
    assert _attention(**dict(big, mp=columns + 1, ld=columns + 1)) == -2


def _append(**kw):
    a = dict(K=A, V=A + MB, ld=256, rows=20, slots=A + 2 * MB, N=2, D=128, Kp=A + 0x10000000, Vp=A + 0x20000000, np=10, ps=16,
             ldp=16 * 256, ldt=256, ldh=128, dt=0, ks=0, vs=0)
    a.update(kw)
    return B.library().pafu_paged_append(None, *a.values())


def test_append_refuses_pools_that_share_a_byte_on_one_page_too():
    K = A + 0x10000000
    for pages in (1, 2, 10):
        # rows of 256 elements at a stride of 512, V's shifted: by less than a row, by so much that they reach the next of K's
        for shift in (0, 8, 248, 264, 504, 512, 512 * 3 + 248):
            for sign in (1, -1):
                assert _append(Vp=K + sign * shift * 2, np=pages, ldt=512, ldp=16 * 512) == -6, (pages, shift, sign)
                assert _append(Vp=K + sign * shift * 2, np=pages, ldt=512, ldp=17 * 512) == -6, (pages, shift, sign)
        # tokens inside heads: 16 * 128 elements at a stride of 4096
        for shift in (0, 8, 2040, 2056, 4088, 4096):
            assert _append(Vp=K + shift * 2, np=pages, ldt=128, ldh=4096, ldp=2 * 4096) == -6, (pages, shift)
    assert _append(Kp=A - 0x1000, Vp=K, np=1) == _append(Kp=K, Vp=A + 2 * MB - 64, np=1) == -6    # over rows, over slots


def test_binding_does_not_read_the_strides_of_axes_of_length_one():
    # one head or one page: K by tokens, V by heads is the same memory.  On the host such a pool gets as far as the check of its place.
    i, table = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 1, dtype=torch.int32)
    one_head = torch.zeros(3, 16, 1, 64, dtype=torch.bfloat16), torch.zeros(3, 1, 16, 64, dtype=torch.bfloat16).permute(0, 2, 1, 3)
    wide = torch.zeros(2, 40, 2, 64, dtype=torch.bfloat16)
    one_page = torch.zeros(1, 16, 2, 64, dtype=torch.bfloat16), wide[1:, :16]
    for K, V in (one_head, one_page):
        assert K.shape == V.shape and K.stride() != V.stride()
        rows = torch.zeros(4, K.shape[2], 64, dtype=torch.bfloat16)
        for pages in ((K, V), (V, K)):
            with pytest.raises(ValueError, match="GPU"):
                B.pafu_paged_append(rows, rows, i, *pages)
            with pytest.raises(ValueError, match="GPU"):
                B.pafu_paged_attention(rows, *pages, table, i, rows)
    K, V = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16).permute(0, 2, 1, 3)
    with pytest.raises(ValueError, match="one shape and stride"):
        B.pafu_paged_append(torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 64, dtype=torch.bfloat16), i, K, V)
