"""The form that window attention takes, seen by the workspace it asks for: none where
blocks join their waves' parts themselves, parts of rows where a second launch does."""
import ctypes

from paper_2608_26806_amd import avtp as A


def size(Hq, Hkv, d, dtype, B, N, bound, window, sinks):
    pages = A._Pages(256, 256, dtype, 1 << 20, 16, Hkv, d)   # (addresses that are only looked at)
    return A.lib().avtp_page_attention_window_workspace_size(ctypes.byref(pages), Hq, B, N, bound, window, sinks)


def test_borders_do_not_follow_one_number_of_sinks():
    # fp32 chunks of 257 to 512 tiles: up to 320 keys in one launch, however they are made up of window and sinks
    for B, N in ((1, 600), (1, 1000), (1, 1150), (3, 990), (10, 1000)):
        for window, sinks in ((256, 0), (256, 4), (256, 5), (256, 64), (200, 100), (320, 0), (16, 300)):
            assert size(14, 2, 64, A.FP32, B, N, 3500, window, sinks) == 0, (B, N, window, sinks)
        for window, sinks in ((340, 4), (512, 4), (257, 100)):
            assert size(14, 2, 64, A.FP32, B, N, 3500, window, sinks) > 0, (B, N, window, sinks)


def test_workspaces_of_the_largest_sizes():
    big = 2 ** 31 - 1
    # more blocks than a launch has: refused
    assert size(256, 256, 128, A.BF16, 1 << 16, big // 256, 2 ** 62, big, big) == 0
    # as many workers as four on a CU, two parts of 16 rows and their log2 sums each, and whose they are
    assert size(16, 2, 128, A.BF16, 1 << 15, 1 << 15, 2 ** 62, big, big) == 2 * 1024 * 16 * (128 + 1) * 4 + 1024 * 32
