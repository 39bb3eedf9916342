"""The gated delta rule's calls from several host threads at once, each on a stream of its own, some split over the library's second stream:
bit for bit what they give one after the other."""
import os
import sys
import threading

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from gdr_util import inputs, run
from paper_2605_05838_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("segments", [0, 3])
def test_four_threads(segments):
    xs = [inputs(dtype, B=B, T=T, H=4, Hk=2, dk=64, dv=128, seed=i) for i, (dtype, B, T) in enumerate((("bf16", 1, 1500), ("f32", 2, 700), ("bf16", 2, 999),
                                                                                                      ("f32", 1, 1300)))]
    old = binding.set_segments(segments)
    try:
        want = [run(x, keep=(False, False)) for x in xs]
        torch.cuda.synchronize()
        got, errors = [[] for _ in xs], []

        def work(i):
            try:
                with torch.cuda.stream(torch.cuda.Stream()):
                    for _ in range(6):
                        got[i].append(run(xs[i], keep=(False, False)))
                    torch.cuda.current_stream().synchronize()
            except Exception as e: # (a thread's own exception would be lost)
                errors.append(e)
        threads = [threading.Thread(target=work, args=(i,)) for i in range(len(xs))]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not errors, errors
        for w, g in zip(want, got):
            assert len(g) == 6 and all(torch.equal(r[n], w[n]) for r in g for n in w)
    finally:
        binding.set_segments(old)
