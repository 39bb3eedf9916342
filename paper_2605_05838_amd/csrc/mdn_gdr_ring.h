// The order in which a loading wave of the reverse scan asks for chunks and waits for them.  (Plain C++: what asks and waits is passed in.)
#pragma once

namespace mdn {

// Rings of the reverse scan: K, T^T (two with remainders: LDS), q and dO, coefficients
constexpr int kReverseK = 3, kReverseQ = 2, kReverseCoef = 4;
constexpr int reverse_t(bool precise) { return precise ? 2 : 3; }

// Two barriers in front of step 0, then two in every step n = 0 .. N: at its start and in its middle.  The chain works on K and T^T of step n from
// the start of step n to that of step n + 1; the waves beside it on q and dO of step n + 1 from the middle of step n (of step 0 from the first
// barrier on).  So what step n asks for behind its first barrier overwrites nothing that is in use: K and T^T of step n + 2 (T^T of step n + 1 in a
// ring of two) and q, dO of step n + 2.
// q(n), k(n), t(n) ask for step n's; wait(false) waits for everything but the last k and, in a ring of three, t asked for; wait(true) for
// everything.  Requests arrive in order: at the end of step n all that the next one works on is there, and K and T^T of step n + 2 have
// that one's time as well.  (Most of what a step needs is there early, out of the L2: waiting for everything at the end of every step takes 932 us for 926,
// the backward call of 32 768 tokens of 16 heads of 128, 236 for 235 of 8 192, 1 371 for 1 369 with remainders, 67.5 for 67.8 in fp32 ([2, 1 024]
// tokens, 4 heads, d = 64).)
template <int T, class Q, class K, class Tt, class Wait, class Barrier>
__attribute__((always_inline)) constexpr void reverse_ring(int N, Q &&q, K &&k, Tt &&t, Wait &&wait, Barrier &&barrier) {
    q(0);
    wait(true);
    barrier();
    k(0);
    t(0);
    if (N > 1) {
        q(1);
        k(1);
        if (T == 3) t(1);
    }
    wait(true);
    barrier();
    for (int n = 0; n <= N; ++n) {
        barrier();
        if (T == 2 && n + 1 < N) t(n + 1);
        if (n + 2 < N) {
            q(n + 2);
            k(n + 2);
            if (T == 3) t(n + 2);
        }
        barrier();
        wait(n + 2 >= N);
    }
}

} // namespace mdn
