"""Sizes at the ends of what the serving entry points take; nothing is launched."""
import pytest

from paper_2012_01114_b200 import binding, build

P = 1 << 20                                     # an address; nothing is read there


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


@pytest.mark.parametrize("q_rows,k_rows", [(1, 0x7fffffff), (1, 0x7ffffe01), (0x7fffffff, 1), (0x7ffffe01, 0x7ffffe01)])
def test_prompts_of_almost_2_31_rows(lib, q_rows, k_rows):
    """Tiles are counted in 32 bits, so that the last 511 numbers of rows are refused."""
    assert lib.psa_prompt_attention(P, P, P, 8, 8, 8, P, P, 1, q_rows, k_rows, 1, 1, 8, 0.1, binding.BF16, P, None, None) == binding.ERR_SHAPE
