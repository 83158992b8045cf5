"""The attention's scale: what its kernels cannot hold is refused (no GPU needed)."""
import pytest

from test_abi_generation import attend, lib, paged  # noqa: F401


@pytest.mark.parametrize("scale,status", [
    (0.0, 0), (-0.5, 0), (1e38, 0), (-2.0 ** 127, 0), (2.358e38, 0), (1e-45, 0),
    # finite, but times log2 e infinite: a score of 0 would have become NaN
    (2.36e38, 1), (-2.36e38, 1), (3e38, 1), (-3.4e38, 1), (float("inf"), 1), (float("-inf"), 1), (float("nan"), 1),
])
def test_scales(lib, scale, status):  # noqa: F811
    assert attend(lib, paged(seqs=0), scale=scale) == status  # (of no sequences, which launches nothing)
