"""What the binding checks of the tensors of a call on a fused q/k/v layer before it hands their addresses to the library (a stand-in for it here)."""
import pytest
import torch

from paper_2605_16732_b200 import binding as dq

M, K, HQ, HK, D = 5, 128, 4, 2, 64
N = (HQ + 2 * HK) * D


class Recorder:
    """In the library's place: every call succeeds and is noted."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or 0


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(dq, "_lib", r)
    monkeypatch.setattr(dq, "_stream", lambda stream=None: 0)
    return r


def _call(x=None, y=None, qk=None, layer_k=K, layer_n=N):
    layer = dq.Layer(None, torch.empty(1024, dtype=torch.uint8), layer_k, layer_n, 16, 64)
    x = torch.zeros((M, K), dtype=torch.bfloat16) if x is None else x
    y = torch.zeros((M, N), dtype=torch.bfloat16) if y is None else y
    dq.dirotq_linear_qkv(x, layer, y, torch.zeros(4096, dtype=torch.uint8), qk or dq.QkNorm(HQ, HK, D))


def test_a_call_that_fits(recorder):
    _call()
    assert recorder.calls == ["dirotq_linear_qkv"]


BF16 = dict(dtype=torch.bfloat16)


@pytest.mark.parametrize("change", [
    dict(y=torch.zeros((M, N - 64), **BF16)),                    # narrower than the layer: its rows would be written past their end
    dict(y=torch.zeros((M - 1, N), **BF16)), dict(y=torch.zeros((M * N,), **BF16)),
    dict(y=torch.zeros((M, N), dtype=torch.float32)), dict(y=torch.zeros((M, N), dtype=torch.float16)),
    dict(y=torch.zeros((M, N + 8), **BF16)[:, :N]), dict(y=torch.zeros((N, M), **BF16).T),
    dict(x=torch.zeros((M, K - 64), **BF16)), dict(x=torch.zeros((M, K + 64), **BF16)), dict(x=torch.zeros((M, K), dtype=torch.float32)),
    dict(x=torch.zeros((M, K), dtype=torch.float16)), dict(x=torch.zeros((M, K + 8), **BF16)[:, :K]), dict(x=torch.zeros((K, M), **BF16).T),
    dict(layer_k=K + 64), dict(layer_n=N + 64)])
def test_calls_that_do_not(recorder, change):
    with pytest.raises(AssertionError):
        _call(**change)
    assert recorder.calls == []


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 1


@pytest.mark.parametrize("name,width", [("x", K), ("y", N)])
def test_tensors_on_another_device(recorder, name, width):
    with pytest.raises(AssertionError):
        _call(**{name: torch.zeros((M, width), **BF16).as_subclass(Elsewhere)})
    assert recorder.calls == []
