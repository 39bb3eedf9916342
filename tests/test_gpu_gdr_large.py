"""Gated delta rule on calls larger than the last-level cache, which bring later chunks' operands into the L2: bit for bit what calls on
parts of the same tensors give, which do not."""
import pytest
import torch

from paper_2605_05838_amd import binding

pytestmark = pytest.mark.gpu


def tensors(B, T, H, Hk, d, seed):
    r = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=r, device="cuda")
    unit = lambda *s: torch.nn.functional.normalize(n(*s), dim=-1).bfloat16()
    return dict(q=unit(B, T, Hk, d), k=unit(B, T, Hk, d), v=n(B, T, H, d).bfloat16(), g=-0.1 * torch.nn.functional.softplus(n(B, T, H)),
                beta=torch.sigmoid(n(B, T, H)))


def call(x, **kw):
    return binding.mdn_gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], output_final_state=False, **kw)


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("cu", [None, [0, 9001, 9002, 25003]])
def test_few_heads(keep, cu):
    """16 columns a workgroup: 16 value heads on 8, and two value heads by themselves."""
    x = tensors(1, 25003, 16, 8, 128, 1)
    got = call(x, save_e=keep, save_states=keep, cu_seqlens=cu)
    for h in range(0, 16, 6):
        part = {n: t[:, :, h // 2:h // 2 + 1] if n in "qk" else t[:, :, h:h + 2] for n, t in x.items()}
        want = call({n: t.contiguous() for n, t in part.items()}, save_e=keep, save_states=keep, cu_seqlens=cu)
        assert torch.equal(got["o"][:, :, h:h + 2], want["o"]), h
        if keep:
            assert torch.equal(got["e"][:, :, h:h + 2], want["e"]), h
            if cu is None: # [heads][chunks][d][d]
                a, b = (t["states"].view(torch.int16).view(-1, (25003 + 63) // 64, 128 * 128) for t in (got, want))
                assert torch.equal(a[h:h + 2], b), h


@pytest.mark.parametrize("keep", [False, True])
def test_many_heads(keep):
    """32 columns a workgroup: two sequences of 34 heads, and each by itself."""
    x = tensors(2, 6394, 34, 34, 128, 2) # (an even number: gates of 16-byte alignment in either sequence)
    got = call(x, save_e=keep, save_states=keep)
    for b in range(2):
        want = call({n: t[b:b + 1] for n, t in x.items()}, save_e=keep, save_states=keep)
        assert torch.equal(got["o"][b:b + 1], want["o"]), b
        if keep:
            assert torch.equal(got["e"][b:b + 1], want["e"]), b
            assert torch.equal(got["states"].view(2, -1)[b], want["states"]), b
