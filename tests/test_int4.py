"""The 4-bit formats and the refusals of the 4-bit calls (CPU: no kernel is launched)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_13076_gb300 as spade
from oracle import int4_oracle as O
from paper_2608_13076_gb300 import int4


@pytest.fixture(scope="module")
def lib():
    spade.build()
    return spade.load()


def test_word_layout():
    """Number i of eight codes sits where the header says, worked by hand: codes 0 .. 7 make 0x75316420."""
    packed = int4.pack_codes(torch.arange(8))
    assert packed.numpy().view("<u4")[0] == 0x75316420
    assert int4.unpack_codes(packed).tolist() == list(range(8))


def test_worked_group():
    """lo = -3, hi = 12: scale 1, zero 3; 0 is held exactly, 2.5 goes to the even neighbour."""
    x = torch.zeros(64)
    x[0], x[1], x[2], x[3] = -3.0, 12.0, 2.5, 3.5
    codes, params = int4.quantize(x, 64)
    assert params.tolist() == [[1.0, 3.0]]
    assert int4.dequantize(codes, params)[:6].tolist() == [-3.0, 12.0, 2.0, 4.0, 0.0, 0.0]


@pytest.mark.parametrize("lo,hi,scale,zero", [
    (0.0, 0.0, 0.0, 0.0),            # nothing but zeros
    (0.0, 1e-8, 0.0, 0.0),           # a span below float16's smallest step
    (1.0, 15.0, 1.0, 0.0),           # 0 joins a positive span
    (-15.0, -1.0, 1.0, 15.0),        # and a negative one
    (-1e30, 1e30, 4364.0, 15.0),     # cut to what float16 holds
])
def test_group_edges(lo, hi, scale, zero):
    x = torch.full((64,), lo)
    x[1::2] = hi
    codes, params = int4.quantize(x, 64)
    assert params.tolist() == [[scale, zero]]
    v = int4.dequantize(codes, params)
    assert v.half().isfinite().all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_group_not_finite(bad):
    x = torch.ones(2, 128)
    x[0, 70] = bad
    codes, params = int4.quantize(x, 64)
    assert params[0, 0].isfinite().all() and params[1].isfinite().all()
    assert params[0, 1, 0].isnan() and int4.dequantize(codes, params)[0, 64:].isnan().all()


def test_quantize_is_a_rounding():
    g = torch.Generator().manual_seed(4)
    x = torch.randn((37, 128), generator=g) * torch.exp(3 * torch.randn((37, 1), generator=g))
    codes, params = int4.quantize(x, 64)
    assert O.check_quantised(x.double().numpy(), np.zeros(x.shape), codes.numpy(), params.float().numpy()) == 0
    assert np.array_equal(O.values(codes.numpy(), params.numpy()), int4.dequantize(codes, params).double().numpy())


def test_a_wrong_rounding_is_seen():
    """The comparison of cached numbers catches a code, a zero or a scale that is one step off."""
    x = torch.randn((8, 64), generator=torch.Generator().manual_seed(5))
    codes, params = int4.quantize(x, 64)
    xd, e = x.double().numpy(), np.zeros(x.shape)
    c = int4.unpack_codes(codes)
    c[3, 9] += 1 if c[3, 9] < 8 else -1
    assert O.check_quantised(xd, e, int4.pack_codes(c).numpy(), params.float().numpy()) > 0
    for j, step in ((0, 1.01), (1, None)):
        p = params.float().clone()
        p[2, 0, j] = p[2, 0, j] * step if step else p[2, 0, j] + 1
        assert O.check_quantised(xd, e, codes.numpy(), p.numpy()) > 0


def test_rope_table_turns():
    """theta = (2 / pi)^2 makes the second of two frequencies pi / 2."""
    t = int4.rope_table((2 / np.pi) ** 2, 4, 3, device="cpu")
    assert torch.allclose(t[1, 1], torch.tensor([0.0, 1.0]), atol=1e-7)
    assert torch.allclose(t[2, 0], torch.tensor([np.cos(2.0), np.sin(2.0)], dtype=torch.float32))


# ---- refusals --------------------------------------------------------------------------------------
P = ctypes.c_void_p(256)
ODD = ctypes.c_void_p(264)  # not 16-byte aligned


def linear(lib, ptrs=None, R=1, N=8, K=128, group=64, status=P):
    ptrs = [P] * 5 if ptrs is None else ptrs
    return lib.spade_linear_w4(*ptrs, R, N, K, group, status, None)


def norm_rope(lib, null=None, B=1, R=2, Hq=4, Hkv=2, D=128, page=64, pages=4, max_pages=2, max_pos=64, max_k=1, eps=1e-6,
              status=P):
    ptrs = [P] * 13
    if null is not None:
        ptrs[null] = None
    return lib.spade_verify_qk_norm_rope_kv4(*ptrs, B, R, Hq, Hkv, D, page, pages, max_pages, max_pos, max_k,
                                             ctypes.c_float(eps), status, None)


def attention(lib, null=None, B=1, Hq=4, Hkv=2, D=128, page=64, pages=4, max_pages=2, max_k=1, R=2, ws=P, status=P):
    ptrs = [P] * 11
    if null is not None:
        ptrs[null] = None
    return lib.spade_verify_attention_kv4(*ptrs, B, Hq, Hkv, D, page, pages, max_pages, max_k, R, ws, 1 << 30, status, None)


def commit(lib, null=None, B=1, Hkv=2, D=128, page=64, pages=4, max_pages=2, status=P):
    ptrs = [P] * 9
    if null is not None:
        ptrs[null] = None
    return lib.spade_kv_commit_kv4(*ptrs, B, Hkv, D, page, pages, max_pages, status, None)


def read(lib, null=None, B=1, R=2, Hkv=2, D=128, page=64, pages=4, max_pages=2, status=P):
    ptrs = [P] * 9
    if null is not None:
        ptrs[null] = None
    return lib.spade_kv_read_kv4(*ptrs, B, R, Hkv, D, page, pages, max_pages, status, None)


def test_exports_and_types(lib):
    for name in ("spade_linear_w4", "spade_verify_qk_norm_rope_kv4", "spade_verify_attention_kv4", "spade_kv_commit_kv4",
                 "spade_kv_read_kv4"):
        assert hasattr(lib, name) and name in spade.__all__


def test_null_pointers(lib):
    for i in (0, 1, 2, 4):
        ptrs = [P] * 5
        ptrs[i] = None
        assert linear(lib, ptrs) == 1
    assert linear(lib, status=None) == 1
    for i in range(13):
        if i not in (1, 2):  # the norm weights may be missing
            assert norm_rope(lib, null=i) == 1, i
    for i in range(10):  # (the lse may be missing)
        assert attention(lib, null=i) == 1, i
    for i in range(9):
        assert commit(lib, null=i) == 1 and read(lib, null=i) == 1, i
    for f in (norm_rope, attention, commit, read):
        assert f(lib, status=None) == 1


@pytest.mark.parametrize("size", ["R", "N", "K"])
def test_linear_sizes(lib, size):
    assert linear(lib, **{size: 0}) == 1


def test_linear_shapes(lib):
    assert linear(lib, group=16) == 2
    assert linear(lib, K=96, group=64) == 2
    for i in range(5):
        ptrs = [P] * 5
        ptrs[i] = ODD
        assert linear(lib, ptrs) == 1


@pytest.mark.parametrize("f", [norm_rope, attention, commit, read])
def test_cache_shapes(lib, f):
    assert f(lib, D=96) == 2 and f(lib, D=256) == 2
    assert f(lib, page=32) == 2 and f(lib, page=96) == 2
    for name in ("B", "Hkv", "page", "pages", "max_pages"):
        assert f(lib, **{name: 0}) == 1, name
    assert f(lib, page=1 << 20, max_pages=1 << 11) == 3  # positions past 31 bits


def test_other_sizes(lib):
    assert norm_rope(lib, Hq=5) == 2 and attention(lib, Hq=5) == 2
    assert norm_rope(lib, R=0) == 1 and attention(lib, R=0) == 1 and read(lib, R=0) == 1
    assert norm_rope(lib, max_k=-1) == 1 and attention(lib, max_k=-1) == 1
    assert norm_rope(lib, B=3) == 1 and attention(lib, B=3) == 1  # fewer rows than sequences
    assert norm_rope(lib, max_pos=0) == 1
    for eps in (-1e-6, float("nan"), float("inf")):
        assert norm_rope(lib, eps=eps) == 1
    assert attention(lib, B=513, R=513) == 2
    assert attention(lib, page=1 << 16, pages=1 << 15, Hkv=2) == 3  # pool rows past 31 bits
    assert norm_rope(lib, B=65536, R=65536) == 2 and commit(lib, B=65536) == 2 and read(lib, B=65536) == 2


def _tensors():
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16)
    return u8, f16


def test_python_checks():
    """Tensors on the wrong device or of the wrong type are refused before any call."""
    u8, f16 = _tensors()
    x = torch.zeros((1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="x must be a CUDA tensor"):
        spade.spade_linear_w4(x, u8(8, 32), f16(8, 1, 2), torch.zeros(1, 8), status=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(TypeError, match="x must be torch.bfloat16"):
        spade.spade_linear_w4(x.float(), u8(8, 32), f16(8, 1, 2), torch.zeros(1, 8),
                              status=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(TypeError, match="k_codes must be torch.uint8"):
        spade.spade_kv_commit_kv4(f16(1, 1, 64, 32), *[None] * 8, status=None)
