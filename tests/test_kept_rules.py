"""The rule by which the checkpoints' parameter gradients are summed in one launch or in two (csrc/mdn_kept_rules.h), compiled for the host."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_05838_amd", "csrc")


@pytest.fixture(scope="module")
def slabs(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("rules")
    (tmp / "rules.cpp").write_text('#include "mdn_kept_rules.h"\nextern "C" int slabs(unsigned rows, int heads) { return mdn::kept_slabs(rows, heads); }\n')
    so = str(tmp / "rules.so")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, "-o", so, str(tmp / "rules.cpp")], check=True)
    lib = ctypes.CDLL(so)
    lib.slabs.argtypes = [ctypes.c_uint, ctypes.c_int]
    return lib.slabs


@pytest.mark.parametrize("heads,rows,two", [(16, 12432, False), (16, 24576, False), (16, 32768, True), (16, 262144, True), (4, 24576, False),
                                            (4, 65536, True), (512, 24576, False), (512, 32768, True), (1, 32768, False), (1, 65536, False),
                                            (1, 131072, True), (2, 32768, False), (2, 65536, True), (4096, 16384, False), (4096, 65536, True)])
def test_the_side_that_was_faster(slabs, heads, rows, two):
    assert (slabs(rows, heads) > 1) is two


def test_neither_launch_has_much_more_to_do_than_the_other(slabs):
    """In rows: the longest slab and all the slabs' sums; and no more slabs than the workspace has room for, or than there are tokens."""
    for heads in (1, 2, 3, 16, 100, 1000, 4096):
        for tokens in (1, 2, 7, 8, 40, 200, 1000, 4097, 16384, 16385):
            n = slabs(tokens * heads, heads)
            assert 1 <= n <= min(128, tokens)
            if n > 1:
                per = -(-tokens // n)
                assert n <= 2 * per and (per <= 4 * n + 1 or n == 128)
    assert slabs(0x7fffffff, 1) == 128


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H", [(16, 4096), (71, 1000), (2003, 16), (90113, 1), (90112, 1)])
def test_gradients_on_either_side(dtype, T, H):
    """dd: T d terms of both signs, each off by 1e-6 (row sums) and the sum by sqrt(T d) 2^-24 of a term."""
    import numpy as np
    import torch
    from gpu_util import host
    from oracle import layer_ops_oracle as lo
    from paper_2605_05838_amd import binding
    r = torch.Generator(device="cuda").manual_seed(T)
    n = lambda: torch.randn(1, T, H, 64, generator=r, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    d = torch.rand(H, generator=r, device="cuda") - 0.5
    kept, grads = [binding.mdn_keep(n()) for _ in range(3)], [n() for _ in range(3)]
    dd = binding.mdn_frontend_bwd_kept(*kept, d, *grads)["dd"]
    want = lo.frontend_backward(*[host(binding.mdn_kept_values(k, torch.float32)) for k in kept], host(d), *map(host, grads))["dd"]
    assert np.abs(host(dd) - want).max() <= 1e-5 * max(np.abs(want).max(), np.sqrt(T) * 0.1)
    assert torch.equal(dd, binding.mdn_frontend_bwd_kept(*kept, d, *grads)["dd"])
