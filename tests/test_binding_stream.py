"""The binding finds the caller's stream through the public API of torch where the short way is not there."""
import types

import pytest


@pytest.fixture
def torch_parts(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2406_04984_amd import binding
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=0x1234))
    return torch, binding, monkeypatch


def test_without_the_short_way(torch_parts):
    torch, binding, monkeypatch = torch_parts
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert binding._stream(None) == 0x1234


def test_the_short_way(torch_parts):
    torch, binding, monkeypatch = torch_parts
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x5600 + device, raising=False)
    assert binding._stream(None) == 0x5603


def test_a_given_stream(torch_parts):
    _, binding, _ = torch_parts
    assert binding._stream(77) == 77 and binding._stream(types.SimpleNamespace(cuda_stream=78)) == 78
