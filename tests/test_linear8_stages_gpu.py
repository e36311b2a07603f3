"""8-bit products of rows at any address, by their number of stages of 128 k:
4 m + 1 of them end on a word of scales of their own."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from test_linear8_gpu import BF16, F32, check  # noqa: E402


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [513, 577, 639, 767, 1025, 1089, 1151, 1537, 2049])
def test_rows_at_any_address(k, dtype):
    """5, 9, 13 and 17 stages, and 6; scales differ from block to block."""
    check((None, 200, k, 131), dtype, "none", False, False, False, 3, seed=k)
    check(([70, 0, 1, 129], 0, k, 66), dtype, "swiglu", True, False, True, 3, seed=k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [4609, 5121, 8833])
def test_splits_of_a_long_sum(k, dtype):
    """Few tiles: shares of whole words, the last with what is left, one stage or more."""
    check((None, 70, k, 66), dtype, "none", False, False, False, 3, seed=k)
