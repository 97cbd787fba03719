"""A top_k of any size reaches the library as what it means: beyond the vocabulary, or not above zero, no limit.  The library
is not called."""
import pytest

import paper_1810_08061_amd as ld
from tests.test_ops_devices_cpu import _tensor, no_library  # noqa: F401  (a fixture)

N, V = 3, 70


@pytest.mark.parametrize("top_k", [1, 3, V - 1, V, V + 1, 2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 32 + 3, 2 ** 64 + 2, 0, -1, -2 ** 31,
                                   2 - 2 ** 32])
def test_top_k_is_not_cut_to_32_bits(top_k, no_library):  # noqa: F811
    m = ld.TokenSample(N, V, "f32")
    m.sample(_tensor((N, V)), _tensor((N,)), top_k=top_k)
    no_limit = top_k <= 0 or top_k >= V
    got = m._filter.top_k
    assert (got <= 0 or got >= V) if no_limit else got == top_k


@pytest.mark.parametrize("top_k", [2.0, 1e12, "3"])
def test_top_k_is_a_whole_number(top_k, no_library):  # noqa: F811
    m = ld.TokenSample(N, V, "f32")
    with pytest.raises(TypeError):
        m.sample(_tensor((N, V)), _tensor((N,)), top_k=top_k)
    assert not [n for n in no_library if n.endswith("step")]
