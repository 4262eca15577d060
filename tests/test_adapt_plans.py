"""What the library's plans of the stored layer in use ask of a caller (CPU
only; sizes alone)."""
import pytest

from paper_2608_28113_amd import _lib, build


@pytest.fixture(scope="module")
def L():
    if not _lib.LIB_PATH.exists():
        build.build()
    _lib.load()
    return _lib


@pytest.mark.parametrize("T", [1, 16, 33, 64, 65, 512])
def test_few_tokens_without_adapters_write_their_result_in_one_pass(L, T):
    """Nothing is split in a row of up to 512 and no adapter's part is added:
    there is nothing to keep in between."""
    assert all(L.hscale_adapted_linear_workspace_bytes(T, n, m, 0, 0) == 0 for n in (16, 512) for m in (1, 24, 14336))
