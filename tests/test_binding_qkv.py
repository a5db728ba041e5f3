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


# ------------------------------------------------------------------ the description's own tensors

class OnCuda(torch.Tensor):
    """A tensor of the host's that says it is on GPU `where`."""
    is_cuda = True

    def get_device(self):
        return self.where


def _on(where, *shape, dtype=torch.float32):
    t = torch.zeros(shape, dtype=dtype).as_subclass(OnCuda)
    t.where = where
    return t


def _description(w_q=0, w_k=0, cos=0, sin=0, positions=0):
    return dq.QkNorm(HQ, HK, D, q_weight=_on(w_q, D, **BF16), k_weight=_on(w_k, D, **BF16), rope="pairs", cos=_on(cos, 9, D // 2), sin=_on(sin, 9, D // 2),
                     positions=_on(positions, M, dtype=torch.int32))


@pytest.mark.parametrize("name", ["w_q", "w_k", "cos", "sin", "positions"])
def test_a_description_on_two_devices(name):
    _description()
    with pytest.raises(AssertionError):
        _description(**{name: 1})


def _norm_rope(where, qk):
    rows = lambda n: _on(where, M, n * D, **BF16)
    dq.dirotq_qk_norm_rope(rows(HQ + 2 * HK), qk, rows(HQ), rows(HK), rows(HK))


def _mxfp4_qkv(where, qk):
    w = dq.Mxfp4(None, _on(where, 4096, dtype=torch.uint8), N, K)
    dq.dirotq_mxfp4_qkv(_on(where, M, K, **BF16), w, _on(where, M, N, **BF16), _on(where, 4096, dtype=torch.uint8), qk)


def _linear_qkv(where, qk):
    layer = dq.Layer(None, _on(where, 1024, dtype=torch.uint8), K, N, 16, 64)
    dq.dirotq_linear_qkv(_on(where, M, K, **BF16), layer, _on(where, M, N, **BF16), _on(where, 4096, dtype=torch.uint8), qk)


@pytest.mark.parametrize("call", [_norm_rope, _mxfp4_qkv, _linear_qkv])
@pytest.mark.parametrize("where", [0, 1])
def test_a_description_on_another_device_than_the_call(recorder, monkeypatch, call, where):
    monkeypatch.setattr(dq, "_current_device", lambda: where)
    call(where, dq.QkNorm(HQ, HK, D))  # (no tensors: right anywhere)
    kw = dict.fromkeys(("w_q", "w_k", "cos", "sin", "positions"), where)
    call(where, _description(**kw))
    assert len(recorder.calls) == 2
    with pytest.raises(AssertionError):
        call(where, _description(**dict.fromkeys(kw, 1 - where)))
    assert len(recorder.calls) == 2
