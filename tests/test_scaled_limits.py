"""The calls over pages of codes, rotations and appends: limits and alignments that are refused, none of which reaches a GPU."""
import ctypes

import pytest

import paper_2311_08252_b200 as rest

OK, INVALID, UNSUPPORTED, SMALL = 0, 1, 2, 3


def strides(*s):
    return (ctypes.c_int64 * len(s))(*s)


def attend(page, k_scales, v_scales):
    st = strides(4096, 1024, 128, 2 * page * 128, page * 128, 128, 4096, 1024, 128)
    return rest.lib().rest_paged_attention_scaled(256, 256, 256, st, k_scales, v_scales, 0, 4, page, 256, 3, 3, 256, None, 256, 1, 8,
                                                  2, 4, 128, 0, 0, 1.0, 256, None, 256, 0, None)


@pytest.mark.parametrize("page,bytes_", [(16, 4), (32, 8), (64, 16), (256, 16)])
def test_scales_are_aligned_to_what_is_copied_of_them(page, bytes_):
    """Scales of 64 rows, or of a page, at once.  (No scratch: what is right gets as far as that.)"""
    assert attend(page, 256, 256) == SMALL and attend(page, 256 + bytes_, 256 + 3 * bytes_) == SMALL
    assert attend(page, 256 + bytes_ // 2, 256) == INVALID and attend(page, 256, 256 + bytes_ // 2) == INVALID


def rotary(N=4, H=2):
    return rest.lib().rest_rotary(256, strides(1 << 40, 1 << 24, 64), 0, 256, 256, 32, 0, 1.0, None, 1, H, N, 64, 256,
                                  strides(1 << 40, 1 << 24, 64), None)


def append(scaled, N=4, H=0, H_kv=2):
    name = "rest_paged_kv_append_scaled" if scaled else "rest_paged_kv_append"
    st = strides(16 * 128 * H_kv, 16 * 128, 128)
    return getattr(rest.lib(), name)(256, 256, st, *([256, 256] if scaled else []), 4, 16, 256, 3, 3, 256, 256, 256,
                                     strides(1 << 40, 1 << 24, 128), None, 0, 256, 256, 64, 0, 1.0, None, None, None, None, H, 1,
                                     H_kv, N, 128, None)


def test_sizes_whose_sums_would_not_fit_are_refused():
    assert rotary(H=65537) == UNSUPPORTED and rotary(N=(1 << 30) + 1) == UNSUPPORTED and rotary(N=(1 << 31) - 1) == UNSUPPORTED
    for scaled in (False, True):
        assert append(scaled, H=65537) == UNSUPPORTED and append(scaled, N=(1 << 31) - 1) == UNSUPPORTED
        assert append(scaled, H_kv=65537) == UNSUPPORTED and append(scaled, N=0) == OK
