// checks.hpp — argument checks that the forward pass's entry points share
// (forward.cpp, generation.cpp): alignment, storage types and memory ranges.
#pragma once

#include <stdint.h>

#include "../../include/mezo.h"

namespace mezo {

inline uint64_t address(const void* p) { return reinterpret_cast<uint64_t>(p); }

inline bool aligned(const void* p, uint64_t bytes) { return (address(p) & (bytes - 1)) == 0; }

inline bool dense(uint32_t dtype) { return dtype == MEZO_F32 || dtype == MEZO_BF16; }

inline uint64_t element_bytes(uint32_t dtype) { return dtype == MEZO_F32 ? 4 : 2; }

// The bytes of rows rows of cols elements, ld apart (false: past 64 bits).
inline bool matrix_bytes(uint64_t rows, uint64_t cols, uint64_t ld, uint64_t element, uint64_t& bytes)
{
    return !__builtin_mul_overflow(rows - 1, ld, &bytes) && !__builtin_add_overflow(bytes, cols, &bytes) &&
           !__builtin_mul_overflow(bytes, element, &bytes);
}

struct Range {
    uint64_t at, bytes;
};

// Whether a buffer ends within the address space.
inline bool whole(Range r) { return r.bytes <= ~r.at; }

// (an empty one shares memory with nothing)
inline bool overlap(Range a, Range b)
{
    return a.bytes && b.bytes && a.at < b.at + b.bytes && b.at < a.at + a.bytes;
}

// Whether a buffer that is written shares memory with one of n others.
inline bool clashes(Range out, const Range* others, int n)
{
    for (int i = 0; i < n; ++i)
        if (overlap(out, others[i])) return true;
    return false;
}

}  // namespace mezo
