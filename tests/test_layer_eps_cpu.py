"""eps of the q/k head norms: what is too small for the arithmetic is refused on the host."""
import ctypes as C

import pytest

import paper_2607_03229_amd as mp
from paper_2607_03229_amd import _binding as B


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("eps", [1.1754942e-38, 1e-40, 1.4e-45, 1e-46])
def test_subnormal_eps_refused(bwd, eps):
    """Of a head of zeros the mean is eps, whose reciprocal root is not taken below 2^-126."""
    L, cfg, mb = B.load(), mp.RopeCfg(64, [32]), 1 << 20
    h = lambda i: B._HEADS.pack(i * mb, 128, 64, 2, 0)
    common = (h(1), None, 3 * mb, None, eps, 4 * mb, 4, h(5), None)
    if bwd:
        st = L.mpipe_op_qk_norm_rope_bwd(0, C.byref(cfg), 4, h(6), None, *common, 7 * mb, None, 1, 8 * mb,
                                         mb, None)
    else:
        st = L.mpipe_op_qk_norm_rope_fwd(0, C.byref(cfg), 4, *common, None)
    assert st == -1 and "eps" in B.last_error()
