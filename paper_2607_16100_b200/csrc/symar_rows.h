// Arithmetic on rows and their addresses, the same in the library and in a host program that replays it.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define SYMAR_ROWS_FN __host__ __device__ __forceinline__
#else
#define SYMAR_ROWS_FN inline
#endif

namespace symar {

// ---- rows on no 16-byte boundary: which of the aligned 16-byte pieces that cover them are read ----
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

// ---- rows that a call writes ----
// Whether rows of `len` elements at i * a + j * b, i < na, j < nb, have an element in common, which a call would write twice.
inline bool rows_meet(int64_t na, int64_t a, int64_t nb, int64_t b, int64_t len)
{
    if ((na > 1 && a < len) || (nb > 1 && b < len)) return true;
    if (na < 2 || nb < 2) return false;
    if (a > b) {
        const int64_t x = a, n = na;
        a = b, b = x, na = nb, nb = n;
    }
    const __int128 reach = (__int128)a * (na - 1) + len;
    for (int64_t j = 1; j < nb && (__int128)j * b < reach; ++j) {           // (b is at least a: not more often than the smaller number of rows)
        const __int128 i = (__int128)j * b / a;
        const int64_t over = (int64_t)((__int128)j * b - i * a);
        if (over < len || (i + 1 < na && a - over < len)) return true;
    }
    return false;
}

}  // namespace symar
