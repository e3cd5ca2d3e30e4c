// Places and rows of a paged cache, arithmetic that host and device share (no CUDA
// needed: host code can ask too).
#pragma once

#include <cstdint>

#include "paged_scores.h"

namespace prism {

constexpr int kAttendUnit = 64;          // keys per unit of the attention's work split

// Division of 0 <= n < 2^31 by a divisor 1 <= d < 2^31 that the launch knows: with
// s = ceil(log2 d) and m = floor(2^32 (2^s - d) / d) + 1, floor(n / d) =
// (floor(n m / 2^32) + n) / 2^s.
struct Divisor {
    uint32_t d, m, s;
    Divisor() = default;
    explicit Divisor(uint32_t by) : d(by), m(0), s(0) {
        while ((1u << s) < d) ++s;
        m = (uint32_t)((((1ull << s) - d) << 32) / d + 1);
    }
    PRISM_HD int of(int n) const { return (int)(((uint32_t)((uint64_t)(uint32_t)n * m >> 32) + (uint32_t)n) >> s); }
};

// The rows j of `len` that are seen, j < sinks or j >= len - window, as places side by
// side: `count` of them from 0 on, in whole blocks of kAttendUnit; place r is row
// key(r) and counts where sees(key(r)).  Whole blocks of the sinks, then, `shift` rows
// on, those of the window.
struct SeenRows {
    int len, sinks, start, split, shift;
    PRISM_HD void set(int n, int window, int n_sinks) {
        len = n;
        sinks = n_sinks;
        start = n - (n < window ? n : window);
        split = shift = 0;
        if (start <= sinks) {
            start = 0;
        } else {
            const int sink_blocks = (sinks + kAttendUnit - 1) / kAttendUnit, first = start / kAttendUnit;
            split = sink_blocks * kAttendUnit;
            shift = (first > sink_blocks ? first : sink_blocks) * kAttendUnit - split;
        }
    }
    PRISM_HD int count() const { return len - shift; }
    PRISM_HD int key(int r) const { return r < split ? r : r + shift; }
    PRISM_HD bool sees(int key) const { return key < len && (key < sinks || key >= start); }
    // all, any of the n rows from `key` on
    PRISM_HD bool sees_all(int key, int n) const { return key + n <= len && (key + n <= sinks || key >= start); }
    PRISM_HD bool sees_any(int key, int n) const { return key < len && (key < sinks || (key + n > start && start < len)); }
};

}  // namespace prism
