// n bytes from any address by whole 32-bit words: which words hold one of them, and how a word of the run is put together.  Device code;
// it compiles as plain C++ too.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define VP_ODD __host__ __device__ __forceinline__
#else
#define VP_ODD inline
#endif

// Whether word i, counted from the border `off` bytes (0 to 3) in front of the first byte, holds one of the n bytes.  Only such a word may be
// read: it lies in the same memory as that byte.  Without a byte (n = 0) none does, the one around the address neither.
VP_ODD bool odd_word_holds(int i, int off, int n) { return n > 0 && 4 * i - off < n; }

// Word i of the run itself, from words i and i + 1 of those; bytes from the n-th on are those of `fill`.
VP_ODD uint32_t odd_word(uint32_t lo, uint32_t hi, int i, int off, int n, uint32_t fill) {
    const uint32_t x = off ? lo >> (8 * off) | hi << (32 - 8 * off) : lo;
    const int left = n - 4 * i;
    const uint32_t keep = left >= 4 ? ~0u : (left <= 0 ? 0u : (1u << (8 * left)) - 1);
    return (x & keep) | (fill & ~keep);
}
