// The rows that a workgroup takes where a launch has fewer workgroups than rows.  A plain function, so that the walk can
// also be replayed on the host.
#pragma once

// f(t) for t = first, first + step, ... below T.  Counted without a sign: the step past the last row may reach 2^31.
template <class F>
constexpr __attribute__((always_inline)) inline void each_row(unsigned first, unsigned step, int T, F f) {
    for (unsigned t = first; t < (unsigned)T; t += step) f((int)t);
}
