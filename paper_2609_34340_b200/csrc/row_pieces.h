// Rows dealt to threads in pieces: the row of a piece that begins `down` rows below the first row of its CTA.  Device code; it compiles as plain
// C++ too.
#pragma once

#ifdef __CUDACC__
#define VP_PIECE __host__ __device__ __forceinline__
#else
#define VP_PIECE inline
#endif

// Whether that row is one of `rows` (above 0, below 2^31); `row` is the last of them where it is not.
VP_PIECE bool row_below(int first, int down, int rows, int& row) {
    const unsigned r = (unsigned)first + (unsigned)down;          // (may pass 2^31)
    const bool in = r < (unsigned)rows;
    row = in ? (int)r : rows - 1;
    return in;
}
