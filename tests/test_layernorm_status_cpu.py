"""Layer norm's status entry on a machine without a GPU: refused like every other call."""

import pytest


def test_no_device_is_refused(lib):
    from conftest import cuda_available
    if cuda_available():
        pytest.skip("a GPU is visible")
    assert lib.LIB.zo_layernorm_sync_status(None) == lib.ZO_ERR_CUDA
    with pytest.raises(lib.ZoError) as e:
        lib.zo_layernorm_sync_status()
    assert e.value.status == lib.ZO_ERR_CUDA
