"""The reverse scan's loading waves (csrc/mdn_gdr_ring.h), compiled for the host, against a queue that answers in order: what a step works on
is there, nothing is overwritten while it is worked on, and the ring of three has two steps' requests on their way."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_05838_amd", "csrc")
WRAPPER = """
#include "mdn_gdr_ring.h"
template <int T> int run(int N, int *out) {
    int *p = out;
    auto put = [&](int kind, int n) { *p++ = kind; *p++ = n; };
    mdn::reverse_ring<T>(N, [&](int n) { put('q', n); }, [&](int n) { put('k', n); }, [&](int n) { put('t', n); },
                         [&](bool all) { put('w', all); }, [&] { put('b', 0); });
    return (int)(p - out) / 2;
}
extern "C" {
int ring(bool precise, int N, int *out) { return precise ? run<mdn::reverse_t(true)>(N, out) : run<mdn::reverse_t(false)>(N, out); }
int depth(int kind, bool precise) { return kind == 'k' ? mdn::kReverseK : kind == 't' ? mdn::reverse_t(precise) : mdn::kReverseQ; }
int coefficients() { return mdn::kReverseCoef; }
}
"""


@pytest.fixture(scope="module")
def ring(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("ring")
    (tmp / "ring.cpp").write_text(WRAPPER)
    so = str(tmp / "ring.so")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, "-o", so, str(tmp / "ring.cpp")], check=True)
    lib = ctypes.CDLL(so)
    lib.ring.argtypes = [ctypes.c_bool, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
    lib.depth.argtypes = [ctypes.c_int, ctypes.c_bool]

    def events(precise, N):
        out = (ctypes.c_int * (16 * (N + 4)))()
        n = lib.ring(precise, N, out)
        return [(chr(out[2 * i]), out[2 * i + 1]) for i in range(n)]
    return lib, events


# Barrier b: 0 and 1 in front, 2 + 2 n at the start of step n, 3 + 2 n in its middle.
# What of step n is worked on between which barriers (the second one: when it is done with)
USE = {"k": lambda n: (2 + 2 * n, 4 + 2 * n), "t": lambda n: (2 + 2 * n, 4 + 2 * n), "q": lambda n: (1 + 2 * n if n else 0, 2 + 2 * n)}
COEFFICIENTS = lambda n: (USE["q"](n)[0], 4 + 2 * n)  # by the waves beside the chain, then by the chain


@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 6, 7, 12, 13, 40])
def test_every_request(ring, precise, N):
    lib, events = ring
    depth = {kind: lib.depth(ord(kind), precise) for kind in "ktq"}
    kept = 2 if depth["t"] == 3 else 1
    queue, asked, there, ahead, b = [], {}, {}, {}, -1
    for kind, n in events(precise, N):
        if kind == "b":
            b += 1
            if b >= 2 and b % 2 == 0:
                ahead[(b - 2) // 2] = list(queue)
        elif kind == "w":
            for x in queue if n else queue[:len(queue) - kept]:
                there[x] = b
            queue = [] if n else queue[len(queue) - kept:]
        else:
            assert (kind, n) not in asked and 0 <= n < N
            asked[kind, n] = b
            queue.append((kind, n))
    assert b == 3 + 2 * N and not queue and sorted(asked) == sorted((kind, n) for kind in "ktq" for n in range(N))
    for (kind, n), at in asked.items():
        assert there[kind, n] < USE[kind](n)[0], ("not there", kind, n)
        if n >= depth[kind]:
            assert at >= USE[kind](n - depth[kind])[1], ("overwritten", kind, n)
        if kind == "q" and n >= lib.coefficients():
            assert at >= COEFFICIENTS(n - lib.coefficients())[1], ("coefficients overwritten", n)
    for n in range(1, N):  # at the start of step n, what step n + 1 will work on is still on its way
        assert ahead[n] == ([("k", n + 1)] + ([("t", n + 1)] if depth["t"] == 3 else []) if n + 1 < N else []), n
