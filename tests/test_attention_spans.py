"""Windows and sinks that no int64 holds reach the library as ones that pass every length
(on the host, with a stand-in for the library)."""

import importlib

import pytest
import torch

from paper_2609_02846_amd import rotary

attention = importlib.import_module("paper_2609_02846_amd.attention")
HUGE = [2 ** 62, 2 ** 63, 2 ** 64, 2 ** 64 + 5, 10 ** 30]


class Library:
    """Keeps what paged attention is called with."""

    def ue5m3_paged_attention_scratch(self, *args):
        self.sizes = args
        return 0

    def ue5m3_paged_attention(self, args, scratch, stream):
        self.args = args
        return 0


@pytest.fixture
def host(monkeypatch):
    for module in (rotary, attention):
        monkeypatch.setattr(module, "_on_device", lambda t, name: t)
    lib = Library()
    monkeypatch.setattr(attention, "load_library", lambda: lib)
    monkeypatch.setattr(attention, "_stream", lambda: None)
    return lib


@pytest.mark.parametrize("n", HUGE)
def test_attention(host, n):
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    args, _ = attention._arguments(x, x, x, None, None, None, True, n, n)
    assert args.window >= 2 ** 40 and args.sinks >= 2 ** 40
    for bad in (dict(window=-n), dict(sinks=-n)):
        with pytest.raises(ValueError, match="negative"):
            attention.attention_forward(x, x, x, **bad)


@pytest.mark.parametrize("n", HUGE)
def test_paged_attention(host, n):
    x, c = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    attention.paged_attention(x, c, c, torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), window=n, sinks=n)
    assert host.args.window >= 2 ** 40 and host.args.sinks >= 2 ** 40 and host.sizes[-2:] == (host.args.window, host.args.sinks)
