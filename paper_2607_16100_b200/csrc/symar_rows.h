// Rows on no 16-byte boundary: which of the aligned 16-byte pieces that cover them are read.  Plain arithmetic on addresses, the
// same on the device and on a host that replays it.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define SYMAR_ROWS_FN __host__ __device__ __forceinline__
#else
#define SYMAR_ROWS_FN inline
#endif

namespace symar {

constexpr int kSlice = 64;                 // elements of two bytes of a row's slice: eight pieces

struct Span {
    uintptr_t lo, hi;                      // an operand's bytes: nothing outside is read
};

// What is known of a row: its first byte's place in a piece, + 16 where the row exists, + 32 where all that piece_wanted() names
// lies in the operand: the pieces begin at most 14 bytes before the row and end at most 31 bytes behind it.
SYMAR_ROWS_FN int row_kind(uintptr_t row, bool exists, int k, Span s)
{
    return (int)(row & 15) | (exists ? 16 : 0) | (row >= s.lo + 16 && row + 2 * (uintptr_t)k + 32 <= s.hi ? 32 : 0);
}

// Whether piece c of a slice holds elements of a row of k: the row begins up to seven elements into its first piece, so a piece
// may hold what the slice before it ends with.
SYMAR_ROWS_FN bool piece_wanted(int k, int slice, int c)
{
    return (int)((uint32_t)k - (uint32_t)slice * kSlice) - c * 8 + 8 > 0;       // (slice * kSlice may pass 2^31 where k is near it)
}

// Whether the piece at `at` is read in one load.  One that is wanted and not, lies in the operand in part.
SYMAR_ROWS_FN bool piece_whole(uintptr_t at, int kind, Span s) { return (kind & 32) || (at >= s.lo && at + 16 <= s.hi); }

}  // namespace symar
