"""Sizes that the token operators' 32-bit indexes do not reach are refused on the host (no GPU)."""
import pytest

from paper_2509_26092_gb300 import build_lib

P = 4096  # an aligned address that no refused call touches
TOP = 2 ** 31 - 1


@pytest.fixture(scope="module")
def D():
    build_lib.build()
    from paper_2509_26092_gb300 import dbl
    return dbl


def refused(D, f, *args):
    with pytest.raises(D.DblError) as e:
        f(*args, stream=0)
    assert e.value.code == D.DBL_ERR_UNSUPPORTED and "2^30" in str(e.value)


@pytest.mark.parametrize("prec", ["bf16", "f16"])
@pytest.mark.parametrize("c", [1 << 30, TOP - 255, TOP])
@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_of_2_to_the_30_are_refused(D, prec, c, dtype):
    with D.precision(prec):
        ln = D.ln_shape(1, c, 1e-5, dtype)
        refused(D, D.dbl_layer_norm_fwd, ln, P, None, P, P, None, P, P, P)
        refused(D, D.dbl_layer_norm_bwd, ln, P, None, P, P, P, P, P, P, P, P, 1 << 60)
        assert D.dbl_layer_norm_workspace_bytes(ln) == 0
        for t in (1, 100):
            scan = D.scan_shape(1, t, c, dtype)
            refused(D, D.dbl_gated_scan_fwd, scan, P, P, None, None, P, None, None)
            refused(D, D.dbl_gated_scan_bwd, scan, P, None, P, P, P, None, P, P, None)
            assert D.dbl_gated_scan_states_bytes(scan) == 0
        refused(D, D.dbl_distill_fwd_bwd, D.distill_shape(1, c, 1, dtype=dtype), P, P, P, None, None, None, P, None, P)


def test_the_largest_sizes_have_sizes(D):
    c = (1 << 30) - 1
    assert D.dbl_layer_norm_workspace_bytes(D.ln_shape(1, c)) == 8 * c
    assert D.dbl_gated_scan_states_bytes(D.scan_shape(1, 65, c)) == 2 * 4 * c
    refused(D, D.dbl_gated_scan_fwd, D.scan_shape(1, (1 << 30) + 1, 8), P, P, None, None, P, None, None)
