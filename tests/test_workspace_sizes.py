"""Workspace sizes of calls that are refused are 0, up to the ends of the 32-bit range, where sums of rows and blocks would wrap."""
import pytest

from paper_2603_06626_b200 import binding as B

MOST = 2 ** 31 - 1
ROWS = MOST - (1 << 20)            # the most rows a norm takes
COLS = 1 << 27                     # the longest row in 8 bits


@pytest.fixture(scope="module")
def size():
    lib = B.load_library()
    return lambda name, *sizes: getattr(lib, f"grouter_{name}_workspace_bytes")(*sizes)


@pytest.mark.parametrize("name,rows_kept", [("rmsnorm_bwd", 1), ("layernorm_bwd", 2)])
def test_norms(size, name, rows_kept):
    for rows in (MOST, MOST - 1, ROWS + 1, -1):
        assert size(name, rows, 128) == size(name, rows, 16384) == 0
    for rows in (0, 1, ROWS):
        for d in (1, 128, 16384):
            got = size(name, rows, d)
            assert got >= rows_kept * 4 * d and got % (rows_kept * 4 * d) == 0, (rows, d, got)
    assert size(name, 4, 0) == size(name, 4, 16385) == 0


def test_products_in_8_bits(size):
    assert size("linear_fp8_fwd", MOST, 64) == size("linear_fp8_fwd", 4, COLS + 1) == size("linear_fp8_fwd", 4, 0) == 0
    assert size("linear_fp8_fwd", MOST - 256, 64) >= (MOST - 256) * 64
    assert size("linear_fp8_bwd", COLS + 1, 64, 64) == size("linear_fp8_bwd", 4, 12, 64) == size("linear_fp8_bwd", 4, 64, 12) == 0
    assert size("gated_ffn_fp8_fwd", MOST, 64, 64) == size("gated_ffn_fp8_fwd", 4, 12, 64) == size("gated_ffn_fp8_fwd", 4, 64, 12) == 0
    assert size("gated_ffn_fp8_fwd", 4, COLS + 8, 64) == size("gated_ffn_fp8_fwd", 4, 64, 2 ** 30) == 0
    assert size("gated_ffn_fp8_fwd", 4, 64, 128) >= 4 * 192 + 1024
    assert size("gated_ffn_bwd", MOST, 64, 64) == size("gated_ffn_bwd", 4, 64, 2 ** 30) == 0


def test_the_size_is_0_where_the_call_says_so(size):
    """Sizes around the limits: the call's own answer (before it touches an address) beside its size function's."""
    lib, A = B.load_library(), 1 << 20
    for rows, d in ((MOST, 64), (ROWS + 1, 64), (4, 16385)):
        assert lib.grouter_rmsnorm_bwd(A, A, d, None, A, A, rows, d, 0, 0, A, A, A, None) == -3 and size("rmsnorm_bwd", rows, d) == 0
    for T, K in ((MOST, 64), (4, COLS + 1)):
        assert lib.grouter_linear_fp8_fwd(A, None, K, A, A, None, None, T, K, 64, A, A, A, None) == -3 and size("linear_fp8_fwd", T, K) == 0
    for T, d, H in ((MOST, 64, 64), (4, 12, 64), (4, 64, 12), (4, COLS + 8, 64)):
        assert lib.grouter_gated_ffn_fp8_fwd(A, None, d, A, A, A, A, A, A, None, T, d, H, 2, A, A, A, None) == -3
        assert size("gated_ffn_fp8_fwd", T, d, H) == 0
