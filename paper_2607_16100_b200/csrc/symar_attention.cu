// Attention of new tokens over the paged 4-bit cache (formulas in include/symar.h).
#include <cmath>

#include "symar_attention.cuh"

namespace symar {
namespace {

constexpr int kStages   = 3;           // copies in flight per warp: two chunks ahead of the one in use (three ahead: 51.7 us against 49.3 for one long sequence)
constexpr int kMinChunks = 1;          // a warp's share of the work is at least this many chunks of 16 tokens
constexpr int kItemCost  = 3;          // what an item costs a warp besides its chunks, in chunks

__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// c[16][8] += a[16][16] b[16][8]
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// the upper halves of a f and b f, and what is left of each, rounded
__device__ __forceinline__ uint32_t high_and_rest(float a, float b, float f, uint32_t &rest)
{
    uint32_t x, y;
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %4};\n\tmul.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}"
        : "=r"(x), "=r"(y) : "f"(a), "f"(b), "f"(f));
    rest = pack_bf16(__uint_as_float(x) - __uint_as_float(x & 0xffff0000u), __uint_as_float(y) - __uint_as_float(y & 0xffff0000u));
    return __byte_perm(x, y, 0x7632);
}

template <int R>
__device__ __forceinline__ int64_t places_of(const AttnArgs &a, const Seq &s)
{
    const int blocks = (s.fresh * a.share + R - 1) / R;
    int64_t n = 0;
#pragma unroll 1
    for (int i = 0; i < blocks; ++i) n += item_of<R>(a, s, i).chunks + kItemCost;
    return n * a.c.kv_heads;
}

// S^T = K Q^T and O^T = V^T P^T: the cache's tokens (then its channels) are the sixteen rows of the matrix
// instruction and eight query rows its columns, so that the eight heads of a share fill it with one token.  A chunk's 16
// tokens are one warp's own: it copies them to its shared memory two chunks ahead, turns codes into exact bf16
// whole numbers (n - z) in registers, multiplies, and keeps its own running maximum and sum; warps meet once per
// piece of work.  The scale of a token's group multiplies the group's partial score (K) and the probability (V), which
// goes into the product as two bf16 numbers, its upper eight bits and what they leave: sixteen bits of it count.  (With the first alone, rounded, the
// result's error is that of a second rounding of the output, 0.0024 instead of 0.0017 of its size, up to 0.0025 where it is small;
// the second product costs 8%: 48.3 -> 52.2 us for the batch below when it came.)
// The maximum in use may lie up to 2^8 below the true one: rescaling the output costs more than it is worth for less.
// Work is split over the cache as evenly as chunks allow, whatever the lengths: all chunks of all items lie in one order, every warp takes an
// equal stretch of it, pieces of an item meet in the block and, where it crosses blocks, at the last block to come (in order, so that
// results do not depend on which that is).
// Bound: instructions, not bytes.  64 sequences of about 4096 tokens, 64 heads, 8 key/value heads of 128: 155 MB in 52.9 us, 2.9 TB/s of the
// 6.5 measured for a copy (14 us of it are start, joins and end; 256 such sequences ran at 4.7 TB/s before the second product); one
// sequence of 131072: 151 MB in 49.4 us.  Issue slots are 56% used, the pipe of integer and bit
// operations (which turns codes into operands) 48%, tensor cores 21%, DRAM half its rate.  One token after 511 with one key/value head: 9.4 us, a chain of
// lengths, page table, page and join, each a trip to memory.  D = 64: 35.6 us, D = 256 (lengths of 2048): 60.2 us.
// Spills (bytes stored, loaded): D = 128 with eight rows 24, 76, its 16 warps having 128 registers each; D = 256 with sixteen 412, 364; others none.
template <int D, int NB>
struct Shape {
    static constexpr int R = 8 * NB, NG = D / 64, kRow = D / 2;
    // one block per multiprocessor, of as many warps as its registers let it have: blocks that share one have an older and a
    // younger, which starves while the older runs (measured: 34 and 47 us for equal shares)
    static constexpr int kWarps = NB == 1 && D <= 128 ? 16 : (D == 256 && NB == 2 ? 4 : 8);
    static constexpr int kOut    = D + 4;                                // floats from row to row of a partial result: rows start in different banks
    static constexpr int kPart   = (R * kOut + 2 * R) * 4;               // output, maxima, sums
    static constexpr int kStage  = 2 * 16 * (kRow + NG * 4);
    static constexpr int kRing   = kStages * kStage > kPart ? kStages * kStage : kPart;
    static constexpr int kBytes  = kWarps * (kRing + kPart);
};
// A piece of an item that does not make it whole: chunks [begin, end) of `chunks`.
struct Piece {
    int64_t at;                  // the item's place in the order of all work
    int     block, head, begin, end, chunks;
    Seq     s;
};

template <int D, int NB>
__device__ __forceinline__ void attention_block(const AttnArgs &a)
{
    using S = Shape<D, NB>;
    constexpr int R = S::R, NG = S::NG, kRow = S::kRow, kUnits = D / 32, kWarps = S::kWarps, kThreads = 32 * kWarps;
    constexpr int kCodes = 16 * kRow, kStage = S::kStage, kOut = S::kOut;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int64_t warp_sum[kWarps], before[kThreads];
    __shared__ int     is_last[2];
    __shared__ Piece   piece[2 * kWarps];        // of each warp: the end of an item that began before, the beginning of one that goes on
    __shared__ float   row_sum[R];
    __shared__ uint32_t odd_rows[kWarps][R];     // of a warp's item, bit gr: the row sees a value of group gr that is NaN, in a chunk that hides something

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    // this warp's ring; its unfinished first piece has a place of its own, its unfinished last piece that of the ring
    unsigned char *mine = smem + warp * S::kRing;
    auto result_of = [&](int i) { return reinterpret_cast<float *>(i & 1 ? smem + (i >> 1) * S::kRing : smem + kWarps * S::kRing + (i >> 1) * S::kPart); };
    const uint32_t mine_addr = smem_addr(mine);

    wait_for_stream();
    // ---- shares: places [begin, end) of all items in order, kItemCost places and one per chunk each ----
    const int each = (a.b.seqs + kThreads - 1) / kThreads;
    const int s0 = min(tid * each, a.b.seqs), s1 = min(s0 + each, a.b.seqs);
    int64_t own = 0;
#pragma unroll 1
    for (int b = s0; b < s1; ++b) own += places_of<R>(a, sequence(a, b));
    int64_t incl = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 31) warp_sum[warp] = incl;
    if (tid < 2 * kWarps) piece[tid].chunks = 0;
    if (tid < kWarps * R) odd_rows[tid / R][tid % R] = 0;
    __syncthreads();
    int64_t total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w == warp) incl += total;
        total += warp_sum[w];
    }
    const int64_t per_warp = max(quotient(total + (int64_t)gridDim.x * kWarps - 1, (int64_t)gridDim.x * kWarps), (int64_t)(kMinChunks + kItemCost));
    // (little work goes to many multiprocessors, four warps each at least, rather than to all warps of a few; what one block can do by
    // itself spares the joining of blocks)
    const int used = total <= per_warp * kWarps ? kWarps
                                                : (int)min((int64_t)kWarps, max(quotient(total + per_warp * gridDim.x - 1, per_warp * gridDim.x), (int64_t)4));
    const int64_t per = per_warp * used, block_begin = per * blockIdx.x;
    if (block_begin >= total) return;
    before[tid] = incl - own;
    __syncthreads();
    const int64_t begin = block_begin + warp * per_warp, end = warp < used ? min(begin + per_warp, total) : begin;
    const int ps = 1 << a.c.page_shift;

    if (begin < end) {
    // the last thread whose sequences begin no later than this warp's share, then the sequence among them
    int owner = -1;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) owner += __popc(__ballot_sync(0xffffffffu, before[i * 32 + lane] <= begin));
    int seq = owner * each, block = 0, head = 0;
    int64_t item_at = before[owner];                 // place of the current item
    Seq  s    = sequence(a, seq);
    if (each > 1) {
#pragma unroll 1
        for (int64_t n; item_at + (n = places_of<R>(a, s)) <= begin; item_at += n) s = sequence(a, ++seq);
    }
    Item item = item_of<R>(a, s, 0);
#pragma unroll 1
    while (item_at + (int64_t)(item.chunks + kItemCost) * a.c.kv_heads <= begin) {
        item_at += (int64_t)(item.chunks + kItemCost) * a.c.kv_heads;
        item = item_of<R>(a, s, ++block);
    }
    head = (int)quotient(begin - item_at, item.chunks + kItemCost);
    item_at += (int64_t)head * (item.chunks + kItemCost);

    for (;;) {
        // (an item's own places come before those of its chunks)
        const int c_begin = (int)max(begin - item_at - kItemCost, (int64_t)0), c_end = (int)min((int64_t)item.chunks, end - item_at - kItemCost);
        const int rows = s.fresh * a.share;
        if (c_begin < c_end) {
        if (lane == 0 && s.len > (a.b.table_ld << a.c.page_shift)) kv_record(a.status, seq, (int)(a.b.table_ld << a.c.page_shift));
        float o[NB][NG * 4][4], m[NB][2], l[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int i = 0; i < NG * 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[nb][i][j] = 0.0f;
            m[nb][0] = m[nb][1] = kNothing;
            l[nb][0] = l[nb][1] = 0.0f;
        }

        // ---- the chunks ----
        const int n = c_end - c_begin;
        int pages = -1;                                       // lane i: the page of chunk (k & ~31) + i
        bool torn = false;                                    // a chunk without a page was met: every chunk is looked at again
        const int first_tok = item.lo + c_begin * 16;
        const unsigned char *head_base = a.c.pages + head * a.c.head_bytes + lane * 16;
        const int side_bytes = ps * kRow;
        const int word_side = lane / (4 * NG);                // lanes below 8 NG copy words: 4 NG pieces of each side
        const int word_src = 2 * side_bytes + word_side * (ps * NG * 4 - 4 * NG * 16);
        int f_tok = first_tok, f_at = 0;                      // next fetch: its first token, its stage's offset
        uint4 q_in[R * D / 256];                              // the queries: asked for before the pages are waited for
#pragma unroll
        for (int i = 0; i < R * D / 256; ++i) {
            const int row = block * R + (i * 32 + lane) / (D / 8), d = (i * 32 + lane) % (D / 8) * 8;
            q_in[i] = make_uint4(0, 0, 0, 0);
            if (row < rows) {
                const int tok = by_share(a, row), hh = row - tok * a.share;
                const __nv_bfloat16 *p = a.q + (int64_t)(s.start + tok) * a.q_ld + (int64_t)(head * a.share + hh) * a.q_head + d;
                if (a.q_vec) {
                    q_in[i] = *reinterpret_cast<const uint4 *>(p);
                } else {
                    const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
                    q_in[i] = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
                }
            }
        }
        auto fetch = [&](int k) {
            if (k < n) {
                if ((k & 31) == 0) {
                    const int tok = f_tok + lane * 16;
                    pages = k + lane < n && tok < s.len ? kv_page_of(a.c, a.b, a.status, seq, tok) : -1;
                }
                const int page = __shfl_sync(0xffffffffu, pages, k & 31), slot = f_tok & (ps - 1);
                const bool on = page >= 0;
                const unsigned char *base = head_base + (int64_t)(on ? page : 0) * a.c.page_bytes;
                const unsigned char *src = base + slot * kRow;
                const uint32_t dst = mine_addr + f_at;
#pragma unroll
                for (int u0 = 0; u0 < 16 * kUnits; u0 += 32) {
                    const int tok = (u0 + lane) / kUnits, c = lane % kUnits;
                    const int turn = D == 64 ? tok >> 2 & 1 : (D == 128 ? tok >> 1 & 3 : tok & 7);
                    const uint32_t to = dst + tok * kRow + ((c ^ turn) << 4);
                    copy16(to, src + u0 * 16, on);
                    copy16(to + kCodes, src + side_bytes + u0 * 16, on);
                }
                if (lane < 8 * NG) copy16(dst + 2 * kCodes + lane * 16, base + word_src + slot * (NG * 4), on);
                torn |= !on;
                f_tok += 16;
                f_at = f_at == (kStages - 1) * kStage ? 0 : f_at + kStage;
            }
            copies_commit();
        };
#pragma unroll 1
        for (int k = 0; k < kStages - NB; ++k) fetch(k);
        // ---- query rows, by way of the ring's stages that are still free: fragments of Q^T, and what each of this thread's two
        // columns sees ----
        static_assert(NB * kStage >= R * D * 2, "the queries fit the last NB stages");
        uint32_t qf[NB][NG * 4][2];
        float qs[NB][NG][2];                    // the sum of a group's channels in this thread's two columns
        int hi[NB][2], lo[NB][2];
        uint4 *q_at = reinterpret_cast<uint4 *>(mine + (kStages - NB) * kStage);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < R * D / 256; ++i) q_at[i * 32 + lane] = q_in[i];
        __syncwarp();
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int gr = 0; gr < NG; ++gr)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint4 v = q_at[(nb * 8 + g) * (D / 8) + gr * 8 + half * 4 + t];
                    qf[nb][gr * 4 + 0][half] = __byte_perm(v.x, v.z, 0x5410);       // channels i and i + 4 of eight
                    qf[nb][gr * 4 + 1][half] = __byte_perm(v.x, v.z, 0x7632);
                    qf[nb][gr * 4 + 2][half] = __byte_perm(v.y, v.w, 0x5410);
                    qf[nb][gr * 4 + 3][half] = __byte_perm(v.y, v.w, 0x7632);
                }
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t v = qf[nb][gr * 4 + i / 2][i & 1];
                    sum += __uint_as_float(v << 16) + __uint_as_float(v & 0xffff0000u);
                }
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                qs[nb][gr][0] = __shfl_sync(0xffffffffu, sum, 8 * t);
                qs[nb][gr][1] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);
            }
#pragma unroll
            for (int i = 0; i < NG * 4; ++i)
#pragma unroll
                for (int half = 0; half < 2; ++half) qf[nb][i][half] = mul2(qf[nb][i][half], i & 1 ? kTwo60 : kTwo64);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = block * R + nb * 8 + 2 * t + j;
                hi[nb][j] = 0x7fffffff;                                             // a row of padding masks nothing
                lo[nb][j] = 0;
                if (r < rows) {
                    hi[nb][j] = s.len - s.fresh + by_share(a, r) + 1;
                    lo[nb][j] = a.window > 0 ? max(hi[nb][j] - a.window, 0) : 0;
                }
            }
        }
        const int least_hi = s.len - s.fresh + by_share(a, block * R) + 1;
        const int most_lo  = a.window > 0 ? s.len - s.fresh + min(by_share(a, block * R + R - 1), s.fresh - 1) + 1 - a.window : 0;
        __syncwarp();                           // (q has been read: the stages are free)
#pragma unroll
        for (int k = kStages - NB; k < kStages - 1; ++k) fetch(k);
        int tok0 = first_tok, at = 0;
#pragma unroll 1
        for (int k = 0; k < n; ++k, tok0 += 16, at = at == (kStages - 1) * kStage ? 0 : at + kStage) {
            copies_wait<kStages - 2>();
            __syncwarp();
            fetch(k + kStages - 1);
            const uint32_t base = mine_addr + at;
            const unsigned char *stage = mine + at;
            // lane i names row i % 8 of matrix i / 8: tokens 0-7 and 8-15, first and second 32 channels of the group
            const int mt = (lane >> 4) * 8 + (lane & 7), mc = lane >> 3 & 1;
            const int turn = D == 64 ? mt >> 2 & 1 : (D == 128 ? mt >> 1 & 3 : mt & 7);
            const uint32_t *kw = reinterpret_cast<const uint32_t *>(stage + 2 * kCodes), *vw = kw + 16 * NG;

            // score = s (sum of q n - z sum of q): the zero points are taken off the sums, not off every code
            float sc[NB][4];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int j = 0; j < 4; ++j) sc[nb][j] = 0.0f;
            uint32_t w0[NG], w1[NG];
            load_words<NG>(w0, kw + g * NG);
            load_words<NG>(w1, kw + (g + 8) * NG);
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                uint32_t r[4];
                matrices(r, base + mt * kRow + (((2 * gr + mc) ^ turn) << 4));
                float acc[NB][4];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[nb][j] = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t a0 = codes(r[0], i), a1 = codes(r[2], i), a2 = codes(r[1], i), a3 = codes(r[3], i);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma(acc[nb], a0, a1, a2, a3, qf[nb][gr * 4 + i][0], qf[nb][gr * 4 + i][1]);
                }
                // (a word as a number is the scale but for the zero point's bits, less than 2^-19 of it)
                const float s0 = __uint_as_float(w0[gr]), s1 = __uint_as_float(w1[gr]), f0 = s0 * a.scale_code, f1 = s1 * a.scale_code;
                const float h0 = -(s0 * a.scale_log2) * (float)(w0[gr] & 15u), h1 = -(s1 * a.scale_log2) * (float)(w1[gr] & 15u);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    sc[nb][0] = __fmaf_rn(qs[nb][gr][0], h0, __fmaf_rn(acc[nb][0], f0, sc[nb][0]));
                    sc[nb][1] = __fmaf_rn(qs[nb][gr][1], h0, __fmaf_rn(acc[nb][1], f0, sc[nb][1]));
                    sc[nb][2] = __fmaf_rn(qs[nb][gr][0], h1, __fmaf_rn(acc[nb][2], f1, sc[nb][2]));
                    sc[nb][3] = __fmaf_rn(qs[nb][gr][1], h1, __fmaf_rn(acc[nb][3], f1, sc[nb][3]));
                }
            }
            // rows of the fragment: tokens tok0 + g (0, 1) and tok0 + g + 8 (2, 3); columns 2t and 2t + 1
            const bool whole = tok0 + 16 <= least_hi && tok0 >= most_lo && !torn;
            if (!whole) {
                const bool paged = !torn || (tok0 < s.len && kv_page_of(a.c, a.b, a.status, seq, tok0) >= 0);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int tok = tok0 + g + (j >> 1) * 8;
                        if (!paged || tok >= hi[nb][j & 1] || tok < lo[nb][j & 1] || tok >= s.len) sc[nb][j] = -INFINITY;
                    }
                // What is hidden, or lies beyond the sequence's end, may be stored as anything: no scale that is NaN may meet its probability
                // of 0.  Such a scale becomes 0, and the rows that see the value are noted.
#pragma unroll 1
                for (int x = lane; x < 16 * NG; x += 32) {
                    uint32_t *w = reinterpret_cast<uint32_t *>(mine + at + 2 * kCodes) + 16 * NG + x;
                    const bool bad = !(fabsf(__uint_as_float(*w)) < INFINITY);
                    if (bad) *w = 0u;
#pragma unroll 1
                    for (uint32_t rest = __ballot_sync(NG == 1 ? 0xffffu : 0xffffffffu, bad); rest; rest &= rest - 1) {
                        const int i = (x & ~31) + __ffs(rest) - 1, tok = tok0 + i / NG, r = block * R + lane;
                        const int place = s.len - s.fresh + by_share(a, r);              // of this lane's row
                        if (lane < R && r < rows && tok <= place && tok < s.len && (a.window == 0 || tok > place - a.window)) odd_rows[warp][lane] |= 1u << i % NG;
                    }
                }
                __syncwarp();
            }
            bool rise = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int j = 0; j < 2; ++j) rise |= fmaxf(sc[nb][j], sc[nb][j + 2]) > m[nb][j] + 8.0f;
            if (__any_sync(0xffffffffu, rise)) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float top = fmaxf(sc[nb][j], sc[nb][j + 2]);
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                        top = fmaxf(top, m[nb][j]);
                        const float keep = power2(m[nb][j] - top);
                        m[nb][j] = top;
                        l[nb][j] *= keep;
#pragma unroll
                        for (int i = 0; i < NG * 4; ++i) {
                            o[nb][i][j] *= keep;
                            o[nb][i][j + 2] *= keep;
                        }
                    }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                for (int j = 0; j < 4; ++j) sc[nb][j] = power2(sc[nb][j] - m[nb][j & 1]);
                l[nb][0] += sc[nb][0] + sc[nb][2];
                l[nb][1] += sc[nb][1] + sc[nb][3];
            }
            uint32_t z2[4][NG];                              // words of the tokens 2t, 2t + 1, 2t + 8, 2t + 9
            load_words<NG>(w0, vw + g * NG);
            load_words<NG>(w1, vw + (g + 8) * NG);
#pragma unroll
            for (int j = 0; j < 4; ++j) load_words<NG>(z2[j], vw + (2 * t + (j >> 1) * 8 + (j & 1)) * NG);
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                uint32_t r[4], pf[NB][2], pr[NB][2];
                matrices_t(r, base + kCodes + mt * kRow + (((2 * gr + mc) ^ turn) << 4));
                const float f0 = __uint_as_float(w0[gr]), f1 = __uint_as_float(w1[gr]);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    pf[nb][0] = transposed(high_and_rest(sc[nb][0], sc[nb][1], f0, pr[nb][0]));
                    pf[nb][1] = transposed(high_and_rest(sc[nb][2], sc[nb][3], f1, pr[nb][1]));
                    pr[nb][0] = transposed(pr[nb][0]);
                    pr[nb][1] = transposed(pr[nb][1]);
                }
                const uint32_t z0 = zeros_of(z2[0][gr], z2[1][gr]), z1 = zeros_of(z2[2][gr], z2[3][gr]);
                const uint32_t y0 = mul2(z0, kSixteen), y1 = mul2(z1, kSixteen);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t a0 = fma2(codes(r[0], i), kTwo127, i & 1 ? y0 : z0), a1 = fma2(codes(r[1], i), kTwo127, i & 1 ? y0 : z0);
                    const uint32_t a2 = fma2(codes(r[2], i), kTwo127, i & 1 ? y1 : z1), a3 = fma2(codes(r[3], i), kTwo127, i & 1 ? y1 : z1);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        mma(o[nb][gr * 4 + i], a0, a1, a2, a3, pf[nb][0], pf[nb][1]);
                        mma(o[nb][gr * 4 + i], a0, a1, a2, a3, pr[nb][0], pr[nb][1]);
                    }
                }
            }
        }
        copies_wait<0>();

        __syncwarp();
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                l[nb][j] += __shfl_xor_sync(0xffffffffu, l[nb][j], 4);
                l[nb][j] += __shfl_xor_sync(0xffffffffu, l[nb][j], 8);
                l[nb][j] += __shfl_xor_sync(0xffffffffu, l[nb][j], 16);
            }
        const bool all = c_begin == 0 && c_end == item.chunks;
        const int which = 2 * warp + (c_begin == 0 ? 1 : 0);
        float *to = result_of(which);
        if (!all && lane == 0) piece[which] = Piece{item_at, block, head, c_begin, c_end, item.chunks, s};
        // fragment i of a group: channels 4 g + i (0, 1) and 32 + 4 g + i (2, 3) of it
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = nb * 8 + 2 * t + j;
                if (g == 0) {
                    to[R * kOut + row]     = m[nb][j];
                    to[R * kOut + R + row] = l[nb][j];
                }
#pragma unroll
                for (int gr = 0; gr < NG; ++gr)
#pragma unroll
                    for (int half = 0; half < 2; ++half)
                        *reinterpret_cast<float4 *>(to + row * kOut + gr * 64 + half * 32 + 4 * g) =
                            make_float4(64.0f * o[nb][gr * 4 + 0][j + 2 * half], 4.0f * o[nb][gr * 4 + 1][j + 2 * half],
                                        64.0f * o[nb][gr * 4 + 2][j + 2 * half], 4.0f * o[nb][gr * 4 + 3][j + 2 * half]);
            }
        __syncwarp();
        if (__any_sync(0xffffffffu, lane < R && odd_rows[warp][lane & (R - 1)])) {
#pragma unroll 1
            for (int e = lane; e < R * D; e += 32)
                if (odd_rows[warp][e / D] >> (e % D / 64) & 1u) to[e / D * kOut + e % D] = __uint_as_float(0x7fc00000u);
            __syncwarp();
            if (lane < R) odd_rows[warp][lane] = 0;
            __syncwarp();
        }
        if (all) {
#pragma unroll 1
            for (int e = lane; e < R * D / 4; e += 32) {
                const int row = e / (D / 4), d = e % (D / 4) * 4;
                store4(a, s, rows, block * R + row, head, d, *reinterpret_cast<const float4 *>(to + row * kOut + d), to[R * kOut + R + row]);
            }
            __syncwarp();
        }
        }
        // ---- next ----
        item_at += kItemCost + item.chunks;
        if (item_at >= end) break;
        if (++head == a.c.kv_heads) {
            head = 0;
            if (++block >= (rows + R - 1) / R) {
                block = 0;
#pragma unroll 1
                do s = sequence(a, ++seq);
                while (s.fresh == 0);
            }
            item = item_of<R>(a, s, block);
        }
    }
    }

    // ---- pieces become items: a warp takes a row of an item at a time ----
    __syncthreads();
    static_assert(2 * kWarps <= 32, "a lane per piece");
    const int64_t my_at = lane < 2 * kWarps ? piece[lane].at : 0;
    const uint32_t there = __ballot_sync(0xffffffffu, lane < 2 * kWarps && piece[lane].chunks > 0);
    const uint32_t below = there & ((1u << lane) - 1u);
    const int64_t before_at = __shfl_sync(0xffffffffu, my_at, below ? 31 - __clz(below) : lane);
    const uint32_t firsts = __ballot_sync(0xffffffffu, (there >> lane & 1u) && (below == 0 || before_at != my_at));
    const int items = __popc(firsts);
    if (items == 0) return;
    uint32_t rest = firsts;
#pragma unroll 1
    for (int j = 0; j < lane && rest; ++j) rest &= rest - 1;
    const int nth = rest ? __ffs(rest) - 1 : 32;              // lane i: the first piece of the i-th item
    auto item_pieces = [&](int i, uint32_t &mask) {           // first piece of the i-th item; all of its pieces
        const int from = __shfl_sync(0xffffffffu, nth, i), to = __shfl_sync(0xffffffffu, nth, i + 1);
        mask = there & ~((1u << from) - 1u) & (to < 32 ? (1u << to) - 1u : 0xffffffffu);
        return from;
    };
#pragma unroll 1
    for (int u = warp; u < items * R; u += kWarps) {
        const int i = u / R, row = u - i * R;
        uint32_t mask;
        const Piece &p = piece[item_pieces(i, mask)];
        const bool all = p.begin == 0 && piece[31 - __clz(mask)].end == p.chunks;
        float *slot = a.partials + (size_t)(2 * blockIdx.x + (p.begin == 0 ? 1 : 0)) * (R * (D + 2));
        const float *r0 = result_of(min(lane, 2 * kWarps - 1));            // lane i: the i-th piece's maximum and sum
        const float m0 = mask >> lane & 1u ? r0[R * kOut + row] : kNothing;
        float top = m0;
#pragma unroll
        for (int d = 1; d < 2 * kWarps; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        top = __shfl_sync(0xffffffffu, top, 0);
        const float f0 = mask >> lane & 1u ? power2(m0 - top) : 0.0f;
        float sum = mask >> lane & 1u ? r0[R * kOut + R + row] * f0 : 0.0f;
#pragma unroll
        for (int d = 1; d < 2 * kWarps; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        sum = __shfl_sync(0xffffffffu, sum, 0);
        float4 v[(D + 127) / 128];
#pragma unroll
        for (int j = 0; j < (D + 127) / 128; ++j) v[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
        for (uint32_t x = mask; x;) {                                     // four pieces at a time
            float f[4];
            float4 y[4][(D + 127) / 128];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = x ? __ffs(x) - 1 : 0;
                const float w = __shfl_sync(0xffffffffu, f0, at);
                f[i] = x ? w : 0.0f;
#pragma unroll
                for (int j = 0; j < (D + 127) / 128; ++j)
                    if (x && (D >= 128 || lane < D / 4)) y[i][j] = *reinterpret_cast<const float4 *>(result_of(at) + row * kOut + j * 128 + lane * 4);
                    else y[i][j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                x &= x - 1;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < (D + 127) / 128; ++j) {
                    v[j].x = __fmaf_rn(y[i][j].x, f[i], v[j].x); v[j].y = __fmaf_rn(y[i][j].y, f[i], v[j].y);
                    v[j].z = __fmaf_rn(y[i][j].z, f[i], v[j].z); v[j].w = __fmaf_rn(y[i][j].w, f[i], v[j].w);
                }
        }
#pragma unroll
        for (int j = 0; j < (D + 127) / 128; ++j) {
            if (D >= 128 || lane < D / 4) {
                if (all) store4(a, p.s, p.s.fresh * a.share, p.block * R + row, p.head, j * 128 + lane * 4, v[j], sum);
                else *reinterpret_cast<float4 *>(slot + 2 * R + row * D + j * 128 + lane * 4) = v[j];
            }
        }
        if (!all && lane == 0) {
            slot[row]     = top;
            slot[R + row] = sum;
        }
    }
    // ---- items that this block shares with others, at most its first and its last: the last block to come joins their
    // results, in the blocks' order ----
    uint32_t mask0, mask1;
    const int at0 = item_pieces(0, mask0), at1 = item_pieces(items - 1, mask1);
    const bool goes_on = piece[31 - __clz(mask1)].end < piece[at1].chunks, came = piece[at0].begin > 0;
    if (!goes_on && !came) return;
    __syncthreads();
    if (tid < 2) {
        // (one thread's fence is enough: the barrier orders what the others wrote before it)
        is_last[tid] = 0;
        if (tid == 0 ? came : goes_on && (items > 1 || !came)) {
            const Piece &p = piece[tid ? at1 : at0];
            const int64_t first = quotient(p.at + kItemCost, per), last = quotient(p.at + kItemCost + p.chunks - 1, per);
            __threadfence();
            const unsigned arrived = atomicAdd(&a.counters[first], 1u);
            if (arrived == (unsigned)(last - first)) {
                a.counters[first] = 0;
                is_last[tid] = 1;
            }
            __threadfence();
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
        if (is_last[i]) {
            const Piece &p = piece[i ? at1 : at0];
            const Seq &s = p.s;
            const int rows = s.fresh * a.share;
            const int64_t first = quotient(p.at + kItemCost, per), last = quotient(p.at + kItemCost + p.chunks - 1, per);
            // weights first, a warp per row, then every thread its part of the output, many loads at a time
            const int joined = (int)(last - first) + 1;
            float *weight = reinterpret_cast<float *>(smem);          // [part][R]; the pieces' results are not needed any more
            auto part = [&](int x) { return a.partials + (size_t)(2 * (first + x) + (x == 0 ? 1 : 0)) * (R * (D + 2)); };
#pragma unroll 1
            for (int row = warp; row < R; row += kWarps) {
                float top = kNothing, sum = 0.0f;
#pragma unroll 1
                for (int x = lane; x < joined; x += 32) top = fmaxf(top, __ldcg(part(x) + row));
#pragma unroll
                for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
#pragma unroll 1
                for (int x = lane; x < joined; x += 32) {
                    const float f = power2(__ldcg(part(x) + row) - top);
                    weight[x * R + row] = f;
                    sum = __fmaf_rn(__ldcg(part(x) + R + row), f, sum);
                }
#pragma unroll
                for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                if (lane == 0) row_sum[row] = sum;
            }
            __syncthreads();
#pragma unroll 1
            for (int e = tid; e < R * D / 4; e += kThreads) {
                const int row = e / (D / 4), d = e % (D / 4) * 4;
                float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
                for (int x0 = 0; x0 < joined; x0 += 8) {
                    float4 y[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (x0 + j < joined) y[j] = __ldcg(reinterpret_cast<const float4 *>(part(x0 + j) + 2 * R + row * D + d));
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (x0 + j < joined) {
                            const float f = weight[(x0 + j) * R + row];
                            v.x = __fmaf_rn(y[j].x, f, v.x); v.y = __fmaf_rn(y[j].y, f, v.y);
                            v.z = __fmaf_rn(y[j].z, f, v.z); v.w = __fmaf_rn(y[j].w, f, v.w);
                        }
                }
                store4(a, s, rows, p.block * R + row, p.head, d, v, row_sum[row]);
            }
            __syncthreads();
        }
    }
}

template <int D, int NB>
__global__ void __launch_bounds__(32 * Shape<D, NB>::kWarps, 1) attention_kernel(const AttnArgs a)
{
    attention_block<D, NB>(a);
    zero_other_rows(a, blockIdx.x, gridDim.x, 32 * Shape<D, NB>::kWarps);
}

template <int D, int NB>
cudaError_t launch(const AttnArgs &a, int num_sms, int device, cudaStream_t stream)
{
    using S = Shape<D, NB>;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_shared((const void *)attention_kernel<D, NB>, S::kBytes, device, allowed);
    if (e != cudaSuccess) return e;
    return launch_early(attention_kernel<D, NB>, dim3(num_sms < kAttnMaxBlocks ? num_sms : kAttnMaxBlocks), 32 * S::kWarps, S::kBytes, stream, a);
}

}  // namespace
}  // namespace symar

using namespace symar;

extern "C" int symar_kv_attention(symar_kv_t *kv, const symar_kv_cache_t *cache, const symar_kv_batch_t *batch,
                                  const symar_kv_attention_t *args, void *cuda_stream)
{
    AttnArgs a;
    const int rc = kv_check(kv, cache, batch, &a.c, &a.b);
    if (rc != SYMAR_OK) return rc;
    if (!args || (args->dtype != SYMAR_F32 && args->dtype != SYMAR_BF16)) return SYMAR_ERR_INVAL;
    if (args->dtype != SYMAR_BF16) return SYMAR_ERR_UNSUPPORTED;
    if (args->q_heads > 4096) return SYMAR_ERR_UNSUPPORTED;
    if (args->q_heads < 1 || args->q_heads % cache->kv_heads || args->window < 0) return SYMAR_ERR_INVAL;
    if (!(args->scale >= 0.0f) || std::isinf(args->scale)) return SYMAR_ERR_INVAL;
    if (batch->tokens == 0) return SYMAR_OK;
    if (!args->q || !args->out || ((uintptr_t)args->q | (uintptr_t)args->out) % 2) return SYMAR_ERR_INVAL;
    if (args->q_ld < 0 || args->q_head < 0 || args->out_ld < 0 || args->out_head < 0 ||
        rows_meet(batch->tokens, args->out_ld, args->q_heads, args->out_head, a.c.dim))
        return SYMAR_ERR_INVAL;
    a.q          = (const __nv_bfloat16 *)args->q;
    a.out        = (__nv_bfloat16 *)args->out;
    a.q_ld       = args->q_ld;
    a.q_head     = args->q_head;
    a.out_ld     = args->out_ld;
    a.out_head   = args->out_head;
    const double scale = args->scale == 0.0f ? 1.0 / std::sqrt((double)cache->head_dim) : (double)args->scale;
    a.scale_log2 = (float)(scale * 1.4426950408889634);
    a.scale_code = std::ldexp(a.scale_log2, 69);
    a.q_heads    = args->q_heads;
    // (a window that no sequence in the table is longer than hides nothing, and differences of positions and smaller ones stay in 32 bits)
    a.window     = args->window < (batch->table_ld << a.c.page_shift) ? args->window : 0;
    a.status     = kv->status;
    a.share      = args->q_heads / cache->kv_heads;
    a.q_vec      = (uintptr_t)args->q % 16 == 0 && args->q_ld % 8 == 0 && args->q_head % 8 == 0;
    a.out_vec    = (uintptr_t)args->out % 8 == 0 && args->out_ld % 4 == 0 && args->out_head % 4 == 0;
    int bits = 0;
    while ((1 << bits) < a.share) ++bits;
    a.share_shift = 31 + bits;
    a.share_mul   = (uint32_t)((((uint64_t)1 << a.share_shift) + a.share - 1) / a.share);
    a.counters   = kv->counters;
    a.partials   = kv->partials;
    if ((int64_t)a.b.tokens * a.share > 0x7fff0000) return SYMAR_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    if (prompt_attention_takes(a, kv->num_sms, kv->device)) {
        e = launch_prompt_attention(a, kv->device, st);
        return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_kv_attention");
    }
    // eight rows where no sequence is likely to have more: a row block of sixteen halves the work per cached token
    const bool wide = (int64_t)a.b.tokens * a.share > 8ll * a.b.seqs;
    if (a.c.dim == 64) e = wide ? launch<64, 2>(a, kv->num_sms, kv->device, st) : launch<64, 1>(a, kv->num_sms, kv->device, st);
    else if (a.c.dim == 128) e = wide ? launch<128, 2>(a, kv->num_sms, kv->device, st) : launch<128, 1>(a, kv->num_sms, kv->device, st);
    else e = wide ? launch<256, 2>(a, kv->num_sms, kv->device, st) : launch<256, 1>(a, kv->num_sms, kv->device, st);
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_kv_attention");
}
