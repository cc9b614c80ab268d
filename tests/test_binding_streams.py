"""Where the Python calls take their stream and device from when none is given.  No GPU: torch's answers are stand-ins."""
from types import SimpleNamespace

import pytest
import torch

from paper_2409_19134_b200 import binding as spd


@pytest.fixture
def public_only(monkeypatch):
    """A torch that has its documented functions alone."""
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: SimpleNamespace(cuda_stream=0x77))


def test_a_given_stream_is_taken():
    assert spd._stream_ptr(SimpleNamespace(cuda_stream=0x55)) == 0x55


def test_the_current_stream_without_torchs_private_functions(public_only):
    assert spd._stream_ptr(None) == 0x77


def test_the_current_device_without_torchs_private_functions(public_only):
    on = lambda dev: SimpleNamespace(is_cuda=True, get_device=lambda: dev, device=f"cuda:{dev}")  # noqa: E731
    assert spd._here(on(1)) == 1
    with pytest.raises(ValueError):
        spd._here(on(0))
