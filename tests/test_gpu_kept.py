"""8-bit checkpoints and the front end and back end from them, on the GPU, against the fp64 oracles."""
import numpy as np
import pytest
import torch

from gpu_util import host
from oracle import kept_oracle
from oracle import layer_ops_oracle as lo
from paper_2605_05838_amd import binding

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# Elements are off by one rounding of the output (2^-8 of 16 bits) or by the sums of a row (128 terms off by 2^-24 each and the chain behind
# them: 1e-5 of the largest element); parameter gradients by the sums of all rows, in 32 bits either way.
TOL = {"f32": 1e-5, "bf16": 2.0 ** -8}


def rel(x, ref):
    assert x.shape == ref.shape
    return float(np.abs(x - ref).max() / max(np.abs(ref).max(), 1e-30))


def tensors(dtype, B, T, H, d, seed=0):
    r = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=r)
    x = {k: n(B, T, H, d).to(DT[dtype]).cuda() for k in ("x_q", "x_k", "x_v", "o", "g", "dq", "dk", "dv", "dy")}
    x["d"], x["w"] = (torch.rand(H, generator=r) - 0.5).cuda(), (torch.rand(d, generator=r) + 0.5).cuda()
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,d", [(1, 1, 1, 64), (1, 1, 1, 128), (2, 13, 3, 64), (3, 70, 5, 128), (1, 9000, 4, 64)])
def test_values(dtype, B, T, H, d):
    x = tensors(dtype, B, T, H, d)["x_q"] * torch.exp2(torch.randint(-20, 20, (B, T, H, 1), device="cuda").float()).to(DT[dtype])
    codes, exponents = kept = binding.mdn_keep(x)
    assert codes.dtype == torch.int8 and codes.shape == x.shape and exponents.dtype == torch.uint8 and exponents.shape == (B, T, H, d // 32)
    y = binding.mdn_kept_values(kept, DT[dtype])
    want = kept_oracle.values(host(x))
    assert y.dtype == DT[dtype] and np.array_equal(host(y), want)
    # (exact in either type)
    assert np.array_equal(host(binding.mdn_kept_values(kept, torch.float32)), want)
    assert np.array_equal(host(binding.mdn_kept_values(kept, torch.bfloat16)), want)
    top = np.abs(host(x)).reshape(B, T, H, -1, 32).max(-1, keepdims=True)
    assert (np.abs(want - host(x)).reshape(B, T, H, -1, 32) <= top / 64).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_at_the_ends_of_the_range(dtype):
    x = torch.zeros(1, 12, 1, 64, dtype=DT[dtype], device="cuda")
    big = torch.finfo(DT[dtype]).max
    x[0, 0, 0, :4] = torch.tensor([1.0, -1.0, 127.5 / 64, -127.5 / 64])    # the last code is limited
    x[0, 1, 0, :3] = torch.tensor([big, -big, 1.0])
    x[0, 2, 0, :3] = torch.tensor([2.0 ** -126, -2.0 ** -126, 2.0 ** -120])
    x[0, 3, 0, :2] = torch.tensor([2.0 ** -130, 2.0 ** -133])              # below the smallest step
    x[0, 4, 0, 5], x[0, 5, 0, 5], x[0, 6, 0, 40] = float("inf"), float("nan"), -float("inf")
    x[0, 7, 0, :] = -0.0
    x[0, 8, 0, :4] = torch.tensor([64.0, 0.5, 1.5, 2.5])                    # halves go to the even code
    y = host(binding.mdn_kept_values(binding.mdn_keep(x), DT[dtype]))
    want = kept_oracle.values(host(x))
    assert np.array_equal(np.isnan(y), np.isnan(want)) and np.isnan(y[0, 4, 0, :32]).all() and not np.isnan(y[0, 4, 0, 32:]).any()
    assert np.isnan(y[0, 6, 0, 32:]).all() and np.isnan(y[0, 5, 0, :32]).all()
    ok = ~np.isnan(want)
    assert np.array_equal(y[ok], want[ok])


def check(x, dtype):
    f = binding.mdn_frontend_fwd_keep(x["x_q"], x["x_k"], x["x_v"], x["d"])
    plain = binding.mdn_frontend_fwd(x["x_q"], x["x_k"], x["x_v"], x["d"])
    kept = [f["kept_" + n] for n in "qkv"]
    a = {k: host(v) for k, v in x.items()}
    vals = {n: kept_oracle.values(a["x_" + n]) for n in "qkv"}
    for n in "qkv":
        assert np.array_equal(host(binding.mdn_kept_values(f["kept_" + n], torch.float32)), vals[n])
    want = lo.frontend_forward(a["x_q"], a["x_k"], a["x_v"], a["d"])
    again = lo.frontend_forward(vals["q"], vals["k"], vals["v"], a["d"])
    r = binding.mdn_frontend_fwd_kept(*kept, x["d"], DT[dtype])
    for n in "qkv":
        assert rel(host(f[n]), want[n]) <= TOL[dtype] and rel(host(r[n]), again[n]) <= TOL[dtype], n
        assert rel(host(f[n]), host(plain[n])) <= TOL[dtype]
    b = binding.mdn_frontend_bwd_kept(*kept, x["d"], x["dq"], x["dk"], x["dv"])
    want = lo.frontend_backward(vals["q"], vals["k"], vals["v"], a["d"], a["dq"], a["dk"], a["dv"])
    for n in ("dx_q", "dx_k", "dx_v"):
        assert rel(host(b[n]), want[n]) <= TOL[dtype], n
    # dd: n = B T d terms of both signs; each is off by 1e-6 (row sums) and the sum by sqrt(n) 2^-24 of a term: against the sum of squares
    n = a["dq"][:, :, 0].size
    assert np.abs(host(b["dd"]) - want["dd"]).max() <= 1e-5 * max(np.abs(want["dd"]).max(), np.sqrt(n / a["dq"].shape[-1]) * 0.1)
    e = binding.mdn_epilogue_fwd_keep(x["o"], x["g"], x["w"])
    assert rel(host(e["y"]), lo.epilogue_forward(a["o"], a["g"], a["w"])) <= TOL[dtype]
    vo, vg = kept_oracle.values(a["o"]), kept_oracle.values(a["g"])
    be = binding.mdn_epilogue_bwd_kept(e["kept_o"], e["kept_g"], x["w"], x["dy"])
    want = lo.epilogue_backward(vo, vg, a["w"], a["dy"])
    assert rel(host(be["do"]), want["do"]) <= TOL[dtype] and rel(host(be["dg"]), want["dg"]) <= TOL[dtype]
    assert np.abs(host(be["dw"]) - want["dw"]).max() <= 1e-5 * np.abs(want["dw"]).max()
    # in a fixed order
    assert torch.equal(b["dd"], binding.mdn_frontend_bwd_kept(*kept, x["d"], x["dq"], x["dk"], x["dv"])["dd"])
    assert torch.equal(be["dw"], binding.mdn_epilogue_bwd_kept(e["kept_o"], e["kept_g"], x["w"], x["dy"])["dw"])
    # without parameter gradients
    b2 = binding.mdn_frontend_bwd_kept(*kept, x["d"], x["dq"], x["dk"], x["dv"], want_dd=False)
    be2 = binding.mdn_epilogue_bwd_kept(e["kept_o"], e["kept_g"], x["w"], x["dy"], want_dw=False)
    assert b2["dd"] is None and be2["dw"] is None and torch.equal(b2["dx_q"], b["dx_q"]) and torch.equal(be2["do"], be["do"])


# one row; a few; rows enough for several trips of the largest launches; heads that divide the step from trip to trip and heads that do
# not; one slab of tokens and several; more heads than a workgroup has threads
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,d", [(1, 1, 1, 64), (1, 1, 1, 128), (2, 13, 3, 128), (1, 5, 300, 64), (1, 3000, 5, 64), (2, 1151, 16, 128),
                                     (1, 7, 4096, 64)])
def test_front_end_and_back_end(dtype, B, T, H, d):
    check(tensors(dtype, B, T, H, d, seed=T), dtype)


def test_many_rows():
    check(tensors("bf16", 1, 9001, 5, 64, seed=3), "bf16")


def test_tensors_need_no_more_than_the_alignment_of_their_elements():
    flat = torch.randn(1 + 2 * 3 * 64, device="cuda").bfloat16()
    x = flat[1:].view(1, 2, 3, 64)
    codes, exponents = torch.empty(1 + 384, dtype=torch.int8, device="cuda"), torch.empty(1 + 12, dtype=torch.uint8, device="cuda")
    kept = (codes[1:].view(1, 2, 3, 64), exponents[1:].view(1, 2, 3, 2))
    a, b = binding.mdn_keep(x)
    kept[0].copy_(a)
    kept[1].copy_(b)
    assert np.array_equal(host(binding.mdn_kept_values(kept, torch.bfloat16)), kept_oracle.values(host(x)))
