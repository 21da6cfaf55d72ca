"""Launches of the 8-bit contraction have less than 2^32 threads, chosen or forced (host code: no GPU needed)."""
import pytest

from paper_2605_17633_amd import binding as B
from test_linear_i8_forms import FORMS, TILES, form

MOST = 1 << 38                # M * N
SIZES = [((MOST - 1) // 136, 136), ((MOST - 1) // 264, 264), (2 ** 31 - 65536, 8), (2 ** 31 - 65536, 120), (192 * 8388480, 168), (256 * 8388352 - 5, 8), (8, 2 ** 31 - 65536)]


def workgroups(f, M, N):
    """As they are launched: of tiles, those past whole rounds of 256 in two pieces where that is a round at most (12 to 14), dealt to eight XCDs."""
    rows, columns = {32: (16, 16), 33: (32, 16)}.get(f) or TILES[f]
    n = -(-M // rows) * -(-N // columns)
    if f >= 32:
        return n
    cut = n % 256 if f >= 12 and n % 256 <= 128 else 0
    return 8 * (-(-(n - cut) // 8) + -(-2 * cut // 8))


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("K", [16, 1040])
def test_chosen(M, N, K):
    for epilogue in range(4):
        assert workgroups(form(M, N, K, epilogue), M, N) * 512 < 2 ** 32


def _forced(f, M, N, epilogue):
    # (addresses that are never followed: only forms that have to be refused come here)
    return B.lib().ssam_linear_i8_as(4096, 16, 4096, 4096, 16, 4096, 4096, 4096, -(-N // 8) * 8, M, N, 16, epilogue, None, 1, 0, 1, f, None)


@pytest.mark.parametrize("M,N", SIZES)
def test_forced(M, N):
    refused = [f for f in FORMS if workgroups(f, M, N) * 512 >= 2 ** 32]
    assert refused or (M, N) == (8, 2 ** 31 - 65536)
    for f in refused:
        for epilogue in (B.EPI_BIAS, B.EPI_BIAS_GELU):
            assert _forced(f, M, N, epilogue) == B.EUNSUPPORTED, f
