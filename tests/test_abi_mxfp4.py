"""Host-side checks of the MXFP4 and q/k entry points that need no GPU: sizes, and refusals before anything touches CUDA."""
import ctypes

import pytest

from paper_2605_16732_b200 import binding

OK, INVALID, SHAPE, SMALL = 0, 1, 2, 3
PTR = 0x10000  # never dereferenced: every call below is refused


@pytest.fixture(scope="module")
def L():
    from paper_2605_16732_b200 import build
    build.build()
    return binding.lib()


def test_operand_bytes(L):
    n = ctypes.c_size_t(0)
    for rows, K in [(1, 1), (1, 32), (333, 4600), (4608, 12288), (257, 257)]:
        assert L.dirotq_mxfp4_bytes(rows, K, ctypes.byref(n)) == OK
        codes, scales = rows * -(-K // 32) * 16, -(-rows // 256) * 256 * -(-K // 256) * 8
        assert codes + scales <= n.value <= codes + scales + 2 * 1024
        w = ctypes.c_size_t(0)
        assert L.dirotq_mxfp4_workspace_bytes(rows, K, ctypes.byref(w)) == OK and w.value == n.value + 1024
    for rows, K, want in [(0, 32, INVALID), (32, 0, INVALID), (-1, 32, INVALID), (1, (1 << 20) + 1, SHAPE), ((1 << 24) + 1, 1, SHAPE), (1 << 24, 1 << 20, SHAPE)]:
        assert L.dirotq_mxfp4_bytes(rows, K, ctypes.byref(n)) == want
        assert L.dirotq_mxfp4_workspace_bytes(rows, K, ctypes.byref(n)) == want
    assert L.dirotq_mxfp4_bytes(1, 1, None) == INVALID


def test_workspace_of_more_rows_serves_fewer(L):
    n, m = ctypes.c_size_t(0), ctypes.c_size_t(0)
    last = 0
    for rows in (1, 7, 128, 129, 256, 257, 1000):
        assert L.dirotq_mxfp4_workspace_bytes(rows, 777, ctypes.byref(n)) == OK and n.value >= last
        last = n.value


def test_create_refuses(L):
    h = ctypes.c_void_p(0)
    assert L.dirotq_mxfp4_create(4, 64, None, 1 << 20, ctypes.byref(h)) == INVALID
    assert L.dirotq_mxfp4_create(4, 64, PTR + 16, 1 << 20, ctypes.byref(h)) == INVALID
    assert L.dirotq_mxfp4_create(4, 64, PTR, 1 << 20, None) == INVALID
    assert L.dirotq_mxfp4_create(0, 64, PTR, 1 << 20, ctypes.byref(h)) == INVALID
    assert L.dirotq_mxfp4_create(4, 64, PTR, 64, ctypes.byref(h)) == SMALL


def test_calls_refuse_null_and_foreign_handles(L):
    fake = ctypes.create_string_buffer(4096)
    for t in (None, ctypes.addressof(fake)):
        assert L.dirotq_mxfp4_destroy(t) == INVALID
        assert L.dirotq_mxfp4_info(t, None, None) == INVALID
        assert L.dirotq_mxfp4_quantize(PTR, 1, 1, 64, 0, t, None) == INVALID
        assert L.dirotq_mxfp4_dequantize(t, PTR, 1, 64, None) == INVALID
        assert L.dirotq_mxfp4_import(PTR, PTR, t, None) == INVALID
        assert L.dirotq_mxfp4_export(t, PTR, PTR, None) == INVALID
        assert L.dirotq_mxfp4_gemm(t, t, None, PTR, 1, 64, PTR, 256, None) == INVALID
        assert L.dirotq_mxfp4_linear(PTR, 1, 64, 1, 0, t, None, PTR, 1, 64, PTR, 1 << 20, None) == INVALID


def _qk(**change):
    s = binding._QkStruct(4, 2, 64, 1, 1e-6, 0, PTR, PTR, 1, 64, PTR, PTR, 32, 100, PTR)
    for k, v in change.items():
        setattr(s, k, v)
    return s


def _norm(L, s, x=PTR, dtype=1, M=8, ldx=512, q=1 << 24, ldq=256, k=2 << 24, ldk=128, v=3 << 24, ldv=128, slots=None, num_slots=0):
    return L.dirotq_qk_norm_rope(x, dtype, M, ldx, None if s is None else ctypes.byref(s), q, ldq, k, ldk, v, ldv, slots, num_slots, None)


@pytest.mark.parametrize("change,want", [
    ({"heads_q": 0}, INVALID), ({"heads_kv": 0}, INVALID), ({"head_dim": 0}, INVALID), ({"head_dim": 60}, SHAPE), ({"head_dim": 264}, SHAPE),
    ({"norm": 2}, INVALID), ({"eps": -1.0}, INVALID), ({"eps": float("nan")}, INVALID), ({"weight_dtype": 2}, INVALID), ({"q_weight": PTR + 1}, INVALID),
    ({"rope": 3}, INVALID), ({"rope": 0}, INVALID), ({"rot_dim": 0}, INVALID), ({"rot_dim": 33}, INVALID), ({"rot_dim": 66}, INVALID),
    ({"cos_table": None}, INVALID), ({"sin_table": PTR + 2}, INVALID), ({"ld_table": 31}, INVALID), ({"num_positions": 0}, INVALID),
    ({"positions": None, "num_positions": 7}, INVALID), ({"positions": PTR + 1}, INVALID)])
def test_qk_refuses_descriptions(L, change, want):
    assert _norm(L, _qk(**change)) == want


@pytest.mark.parametrize("change", [
    {"x": None}, {"q": None}, {"k": None}, {"M": 0}, {"dtype": 2}, {"x": PTR + 8}, {"q": (1 << 24) + 2}, {"ldx": 504}, {"ldx": 516}, {"ldq": 248},
    {"ldk": 120}, {"ldv": 120}, {"ldk": 132}, {"slots": PTR, "num_slots": 0}, {"slots": PTR + 2, "num_slots": 10},
    {"q": PTR, "ldq": 256},                       # over x with another stride
    {"q": PTR + 512, "ldq": 512},                 # over x's k
    {"k": PTR + 512, "ldk": 512, "slots": PTR, "num_slots": 8},  # in place and by slots
    {"k": 1 << 24}, {"v": 2 << 24}, {"v": (1 << 24) + 1024}])   # outputs over one another
def test_qk_refuses_tensors(L, change):
    assert _norm(L, _qk(), **change) == INVALID


def test_qk_null_description(L):
    assert _norm(L, None) == INVALID
    assert L.dirotq_linear_qkv(PTR, 4, None, None, PTR, PTR, 1 << 20, None) == INVALID
    s = _qk()
    assert L.dirotq_linear_qkv(PTR, 4, None, ctypes.byref(s), PTR, PTR, 1 << 20, None) == INVALID
    assert L.dirotq_mxfp4_qkv(PTR, 1, 64, 1, 0, None, None, None, PTR, 1, 64, PTR, 1 << 20, None) == INVALID


def test_qk_accepts_before_it_looks_for_a_device(L):
    """Arguments that are all right get as far as the device: an error of CUDA's here, not of the arguments."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("would launch")
    assert _norm(L, _qk()) == 5
    assert _norm(L, _qk(), q=PTR, ldq=512, k=PTR + 512, ldk=512, v=PTR + 768, ldv=512) == 5  # all in place
    assert _norm(L, _qk(), q=PTR, ldq=512, k=PTR + 512, ldk=512, v=None, ldv=0) == 5
    assert _norm(L, _qk(), q=PTR, ldq=512, k=PTR + 512, ldk=512, v=None, ldv=0, M=1, ldx=1024) == 5  # one row has no stride
    assert _norm(L, _qk(q_weight=None, k_weight=None, rope=0, rot_dim=0, cos_table=None, sin_table=None)) == 5
