"""The Muon handles refuse sets that they cannot run, before anything is launched (no GPU
needed)."""

import types

import pytest
import torch


@pytest.fixture
def fo(lib, monkeypatch):
    """With the check that a matrix is on a GPU out of the way of the set's."""
    from paper_2608_15665_gb300 import firstorder
    monkeypatch.setattr(lib, "make_muon_matrix", lambda W, G, M: object())
    return firstorder


def _made(fo, which, mats, stream=None):
    return fo.Muon(mats, stream=stream) if which == "Muon" else fo.Orthogonalizer(mats, stream=stream)


@pytest.mark.parametrize("which", ["Muon", "Orthogonalizer"])
def test_an_empty_set_is_refused(lib, fo, which):
    with pytest.raises(lib.ZoError, match="at least one matrix") as e:
        _made(fo, which, [])
    assert e.value.status == lib.ZO_ERR_INVALID_ARG


@pytest.mark.parametrize("which", ["Muon", "Orthogonalizer"])
def test_matrices_on_several_devices_are_refused(lib, fo, which):
    mats = [torch.zeros(4, 4), torch.zeros(4, 4, device="meta")]
    with pytest.raises(lib.ZoError, match="one CUDA device") as e:
        _made(fo, which, mats)
    assert e.value.status == lib.ZO_ERR_INVALID_ARG


@pytest.mark.parametrize("which", ["Muon", "Orthogonalizer"])
def test_a_stream_of_another_device_is_refused(lib, fo, which):
    stream = types.SimpleNamespace(device=torch.device("meta"), cuda_stream=0)
    with pytest.raises(lib.ZoError, match="one CUDA device") as e:
        _made(fo, which, [torch.zeros(4, 4)], stream)
    assert e.value.status == lib.ZO_ERR_INVALID_ARG
