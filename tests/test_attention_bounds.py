"""Bounds of the attention calls that leave 32-bit row and unit numbers are refused before any device work
(CPU: no kernel is launched)."""
import ctypes

import pytest

import paper_2608_13076_gb300 as spade

P = ctypes.c_void_p(256)
CAPACITY = 3


@pytest.fixture(scope="module")
def lib():
    spade.build()
    return spade.load()


def kv4(lib, B, Hq, Hkv, max_k):
    return lib.spade_verify_attention_kv4(*[P] * 11, B, Hq, Hkv, 128, 64, 4, 2, max_k, 600, P, 1 << 62, P, None)


def paged(lib, B, Hq, Hkv, max_k):
    return lib.spade_verify_attention_paged(*[P] * 9, B, Hq, Hkv, 128, 64, 4, 2, max_k, 600, P, 1 << 62, P, None)


def dense(lib, B, Hq, Hkv, max_k):
    return lib.spade_verify_attention(*[P] * 8, B, Hq, Hkv, 128, 256, max_k, 600, P, 1 << 62, P, None)


def noalloc(lib, B, Hq, Hkv, max_k):
    return lib.spade_verify_attention_noalloc(*[P] * 8, B, Hq, Hkv, 128, 256, max_k, 600, P, None)


# Rows of a KV head G (max_k + 1) that wrap to 4, to 0 and past 2^31; max_k + 1 itself past it; units B Hkv (rows / 64)
# that wrap though the rows do not.
SIZES = [(1, 8, 2, 1 << 30), (1, 64, 1, (1 << 26) - 1), (1, 8, 8, 2**31 - 1), (1, 4, 1, (1 << 29) - 1),
         (512, 64, 64, (1 << 23) - 1), (512, 512, 64, 1 << 20)]


@pytest.mark.parametrize("call", [kv4, paged, dense, noalloc])
@pytest.mark.parametrize("sizes", SIZES)
def test_refused(lib, call, sizes):
    assert call(lib, *sizes) == CAPACITY
    assert b"max_k" in lib.spade_last_error()


@pytest.mark.parametrize("sizes", SIZES)
def test_no_workspace_size(lib, sizes):
    B, Hq, Hkv, max_k = sizes
    assert lib.spade_attn_workspace_size(B, Hq, Hkv, 128, 256, max_k) == 0
    assert b"max_k" in lib.spade_last_error()


@pytest.mark.parametrize("call", [kv4, paged, dense])
def test_others_are_not(lib, call):
    """A loose bound that 32 bits hold is not refused for its size."""
    assert call(lib, 1, 8, 2, 5000) != CAPACITY


# A prompt of a million rows behind a million slots: a KV head's 131072 row blocks of up to 32768 slices each; and
# the longest cache under 64 blocks.
LONG = [(1, 64, 8, (1 << 20) - 1, 1 << 21), (1, 8, 1, 511, (1 << 31) - 64)]


@pytest.mark.parametrize("sizes", LONG)
def test_schedules_past_32_bits_are_refused(lib, sizes):
    B, Hq, Hkv, max_k, cap = sizes
    rows = (B, Hq, Hkv, 64)
    pages = (64, (2**31 - 64) // 64 // Hkv, cap // 64)
    assert lib.spade_verify_attention_kv4(*[P] * 11, *rows, *pages, max_k, 1 << 20, P, 1 << 62, P, None) == CAPACITY
    assert b"max_k" in lib.spade_last_error()
    assert lib.spade_verify_attention_paged(*[P] * 9, *rows, *pages, max_k, 1 << 20, P, 1 << 62, P, None) == CAPACITY
    assert b"max_k" in lib.spade_last_error()
    assert lib.spade_attn_workspace_size(*rows, cap, max_k) == 0
    assert b"max_k" in lib.spade_last_error()


def test_long_prompts_are_not(lib):
    """128 thousand rows of eight heads a KV head behind four million slots."""
    assert lib.spade_verify_attention_kv4(*[P] * 11, 1, 64, 8, 64, 64, 1 << 20, 1 << 16, (1 << 17) - 1, 1 << 17, P, 1 << 62, P,
                                          None) != CAPACITY
