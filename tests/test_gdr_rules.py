"""The rules by which a scan of the gated delta rule takes 16 or 32 columns a workgroup and the forward brings later chunks' lines into the L2
(csrc/mdn_scan_rules.h), compiled for the host."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_05838_amd", "csrc")


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("rules")
    (tmp / "rules.cpp").write_text("""
#include "mdn_scan_rules.h"
extern "C" bool sixteen(size_t sequences, size_t chunks, size_t longest, size_t heads, int dv) {
    return mdn::sixteen_columns(sequences, chunks, longest, heads, dv, 256);
}
extern "C" bool touch(bool f32, bool sixteen, size_t blocks, int dk, int dv, bool kept) {
    return mdn::gdr_forward_touch(f32, sixteen, dv, kept, mdn::gdr_bytes(blocks, dk, dv, 2, kept ? 3 : 2, kept));
}
""")
    so = str(tmp / "rules.so")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, "-o", so, str(tmp / "rules.cpp")], check=True)
    lib = ctypes.CDLL(so)
    lib.sixteen.restype = ctypes.c_bool
    lib.sixteen.argtypes = 4 * [ctypes.c_size_t] + [ctypes.c_int]
    lib.touch.restype = ctypes.c_bool
    lib.touch.argtypes = [ctypes.c_bool, ctypes.c_bool, ctypes.c_size_t, ctypes.c_int, ctypes.c_int, ctypes.c_bool]
    return lib


@pytest.fixture
def sixteen(rules):
    return rules.sixteen


@pytest.mark.parametrize("B,T,H,dv,columns", [(1, 777, 16, 128, 16), (2, 2048, 16, 128, 16), (3, 2048, 16, 128, 32), (8, 2048, 16, 128, 32),
                                              (8, 2048, 16, 64, 32), (1, 1, 4096, 64, 32), (1, 32768, 33, 128, 32), (1, 1, 32, 128, 16)])
def test_equal_lengths(sixteen, B, T, H, dv, columns):
    assert sixteen(B, 0, (T + 63) // 64, H, dv) is (columns == 16)


@pytest.mark.parametrize("lens,columns", [([16384] + [64] * 20, 16), ([4096] + [64] * 20, 16), ([4096] + [512] * 20, 32),
                                          ([4096, 2048, 1024] + [300] * 10, 32), ([8192] * 2 + [32] * 40, 32), ([777] * 3, 32), ([777], 16),
                                          ([1] * 300, 32), ([16384] + [1] * 60, 16), ([16384] + [1] * 150, 32), ([32768] + [1] * 500, 32),
                                          ([4096] + [1] * 20, 16), ([4096] + [1] * 40, 32), ([8192] + [1000] * 4, 16),
                                          ([2048, 1500] + [20] * 8, 32), ([2048] + [64] * 10, 16)])
def test_packed_where_it_was_faster(sixteen, lens, columns):
    """16 heads of 128: sequences beside one long one count by what there is to do beside it."""
    chunks = [(n + 63) // 64 for n in lens]
    assert sixteen(len(lens), sum(chunks), max(chunks), 16, 128) is (columns == 16)


# B, tokens, heads, dk, dv, whether states are kept, whether it was faster with (16 heads a sequence or few: 16 columns)
@pytest.mark.parametrize("B,T,H,dk,dv,kept,faster", [
    (1, 8192, 16, 128, 128, False, False), (1, 16384, 16, 128, 128, False, False), (1, 24576, 16, 128, 128, False, True), (1, 32768, 16, 128, 128, False, True),
    (1, 16384, 16, 128, 128, True, True), (1, 24576, 16, 128, 128, True, True), (4, 8192, 16, 128, 128, True, True), (4, 8192, 16, 128, 128, False, False),
    (8, 4096, 16, 64, 128, True, True), (8, 4096, 16, 128, 64, True, False), (8, 8192, 16, 64, 64, True, False), (8, 8192, 16, 64, 64, False, False),
    (4, 2048, 16, 128, 128, True, False)])
def test_lines_into_the_l2(rules, B, T, H, dk, dv, kept, faster):
    chunks = (T + 63) // 64
    assert rules.touch(False, rules.sixteen(B, 0, chunks, H, dv), B * H * chunks, dk, dv, kept) is faster
    assert rules.touch(True, rules.sixteen(B, 0, chunks, H, dv), B * H * chunks, dk, dv, kept) # fp32: always


def test_packed_sequences_of_equal_lengths_are_a_batch(sixteen):
    for B in (1, 2, 3, 5, 40):
        for n in (1, 2, 13, 512):
            for H in (1, 7, 16, 100):
                assert sixteen(B, B * n, n, H, 128) == sixteen(B, 0, n, H, 128)
