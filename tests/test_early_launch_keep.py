"""The kernels of a round's end are placed early too, and read by ordinary loads (see test_early_launch)."""
import pytest

from test_early_launch import NON_COHERENT, _code


@pytest.mark.parametrize("name", ["verify.cu", "key_weights.cu", "evict.cu"])
def test_no_non_coherent_loads(name):
    src = _code(name)
    assert "grid_dep_launch()" in src and "grid_dep_wait()" in src
    assert not NON_COHERENT.search(src)
