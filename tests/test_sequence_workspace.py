"""How the workspace of linear attention is laid out, by its size and without a device: the order of packed sequences' segments, pairs of ints that the
kernels read as one, lies behind the segments' states and needs 8 bytes, whatever the states' sizes come to."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def la():
    import __graft_entry__ as ge
    ge.build()
    from paper_2002_03629_b200 import linear_attention
    return linear_attention


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("dtype", [0, 1], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,N,H,Dk,Dv", [(4096, 1, 1, 33, 33), (2048, 1, 3, 47, 33), (9000, 3, 1, 7, 9), (2176, 2, 5, 1, 1), (4096, 1, 1, 65, 127), (5000, 4, 3, 32, 33)])
def test_the_order_of_packed_segments_lies_on_8_bytes(la, T, N, H, Dk, Dv, dtype, backward):
    """Odd widths and heads: an odd number of slots and jobs times Dk Dv states of four bytes leaves a place at 4 mod 8.  What stands behind the states
    is whole pairs (8 bytes each), so the size is a multiple of 8 if and only if they begin on one."""
    lib = la._lib()
    packed = la._Shape(type=dtype, B=1, N=N, T=T, H=H, Dk=Dk, Dv=Dv, cu_seqlens=1 << 20, log_decay=1 << 20, scale=1.0)
    size = lib.la_workspace(C.byref(packed), backward)
    assert size > 4 * H * Dk * Dv                            # (it is cut: the states of more than one segment)
    assert size % 8 == 0


def test_the_longest_sequences(la):
    """Steps are counted in 32 bits, by chunks of 32 and of 128, up to a chunk beyond the last step: 2^31 - 128 of them at most."""
    lib, most = la._lib(), 2 ** 31 - 128
    t = la._Tensor(1 << 20, 0, 1, 0)
    r = C.byref(t)
    for packed in (False, True):
        def shape(T):
            return la._Shape(type=1, B=1, N=1 if packed else 0, T=T, H=1, Dk=1, Dv=1, cu_seqlens=1 << 20 if packed else None, log_decay=1 << 20, scale=1.0)
        assert lib.la_workspace(C.byref(shape(most)), 0) > 0 and lib.la_workspace(C.byref(shape(most)), 1) > 0
        for T in (most + 1, 2 ** 31 - 32, 2 ** 31 - 1):
            s = shape(T)
            p = C.byref(s)
            assert lib.la_workspace(p, 0) == 0 and lib.la_workspace(p, 1) == 0
            assert lib.la_forward(p, r, r, r, None, r, None, 1 << 20, 1 << 30, None) == la.LA_ERR_INVALID
            assert lib.la_backward(p, r, r, r, None, r, None, r, r, r, None, 1 << 20, 1 << 30, None) == la.LA_ERR_INVALID
