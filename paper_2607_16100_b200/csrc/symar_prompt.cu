// Attention of many query rows (prompts, pieces of prompts) over the paged 4-bit cache, on the fifth generation's tensor cores.
//
// A block has 256 query rows (tokens and the heads of one key/value head's share), two groups of 128, and walks over the cached tokens 64 at
// a time.  Eight warps bring the codes in and write them out again as what a tensor-core operand is: whole numbers n - z in bf16, exact, keys
// as rows of channels, values transposed.  The scales stay apart, so that nothing is rounded that the definition does not round but the
// probabilities: every group of 64 channels has a product of its own, S_g = Q_g N_g^T, whose columns the softmax multiplies by the keys'
// scales and adds; and a set of probabilities of its own, P_g = P s_g, for O_g = P_g N_g.  A channel's place in an operand is the one that its
// code comes out of the register at: the queries are permuted alike, the output back.
// Tensor memory: 64 columns of scores, two sets of 32 of probabilities (the products' first operand) and 128 of output per group, all 512.
// Scores are therefore made for 32 keys at a time: with 64 the probabilities had to take the scores' place, and the next scores waited for
// the product (569 us against 517 for the call below).  Sixteen warps have sixteen rows each, a thread two rows and every fourth pair of
// columns (a row per thread loads every scale once per row: 746 us with the probabilities in shared memory; four rows, eight warps: 485).
// Each group has a warp that issues scores and one that issues outputs (one thread for both: 527 us).  Registers are shared out between the
// roles.
// (Values scaled and probabilities in f16 would halve the products' and the softmax's traffic, but f16 has nothing below 2^-24: a row
// whose likeliest token has a value of 0 loses what the others give it.)
// Bound: a tile of 64 keys takes 3700 cycles, of which 2400 issue instructions (9500 on four schedulers), 2050 move softmax and codes
// through shared memory, 1500 feed the products from there, and 1024 take exponentials; taking any one of them out gains 3% or less.
// Two pieces of 1024 tokens over 4099 with a window of 4096, 64 heads, 8 key/value heads of 128: 459 us, 600 TFLOP/s; a prompt of 4096 tokens:
// 445 us, 617 TFLOP/s (of 1640 measured for a plain product); the same with heads of 64 channels 338 us, 407 TFLOP/s: the softmax, the scales and the
// waits of a tile are what they are at 128, its products half.  (These times follow the compiler's order of instructions: edits outside
// the loops moved them by 2%, at D = 64 once by 10%.)  D = 256 has no form here: its output alone, 256 columns for each of two groups, is all of tensor memory.
#include <cfloat>

#include "symar_attention.cuh"

namespace symar {
namespace {

constexpr int kRows = 128, kBlockRows = 2 * kRows, kKeys = 64, kSub = 32, kStages = 4, kRaw = 3;
constexpr int kWorkers = 8;                            // warps that expand codes: a chunk of 16 keys or values of every tile each
constexpr int kSoftmax = 16;                           // warps of the softmax: eight to a group of 128 rows, sixteen rows each
constexpr int kThreads = 32 * (kSoftmax + kWorkers + 4);       // ... the workers, two warps for each group's products
constexpr int kRegsSoftmax = 88, kRegsWorker = 56, kRegsRest = 40, kRegsLaunch = 72;
static_assert(4 * kRegsSoftmax + 2 * kRegsWorker + kRegsRest <= 7 * kRegsLaunch, "the warpgroups' shares must not be above what a block is launched with");

template <int D>
struct Shape {
    static constexpr int NG = D / 64, kRow = D / 2;
    static constexpr int kSlabQ = kRows * 128, kSlabK = kKeys * 128;      // 64 channels (or keys) of every row: 128 bytes, swizzled
    static constexpr int kStage = 2 * NG * kSlabK;
    static constexpr int kScales = 2 * NG * kKeys * 4;
    static constexpr int kRawChunk = 16 * (kRow + NG * 4);
    static constexpr int kQ = 0, kKV = kQ + 2 * NG * kSlabQ, kSc = kKV + kStages * kStage, kRawAt = kSc + kStages * kScales;
    static constexpr int kBytes = kRawAt + kWorkers * kRaw * kRawChunk + 1024;
};

__device__ __forceinline__ void matrices_out(uint32_t addr, const uint32_t (&r)[4])
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
// Sixteen lanes and 32 columns, as the result of a matrix instruction lies in a warp: a thread has columns 8 j + 2 t and the next one of
// lanes lane / 4 (v[4 j], v[4 j + 1]) and lane / 4 + 8 (v[4 j + 2], v[4 j + 3]), t = lane % 4.  Waited for later (acc_loaded).
__device__ __forceinline__ void acc_ask_rows(uint32_t addr, uint32_t *r)
{
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
__device__ __forceinline__ void acc_store_rows(uint32_t addr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
// The same lanes, sixteen columns of pairs of bf16: a thread's pairs 4 j + t of lanes lane / 4 (v[2 j]) and lane / 4 + 8 (v[2 j + 1]).
__device__ __forceinline__ void pairs_store(uint32_t addr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
// Products and commits of the one lane that `on` names: the warp stays together, what it addresses stays in uniform registers.
__device__ __forceinline__ void product_if(uint32_t acc, uint64_t a, uint64_t b, uint32_t how, uint32_t add, uint32_t on)
{
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(acc),
                 "l"(a), "l"(b), "r"(how), "r"(add), "r"(on) : "memory");
}
// (the first operand in tensor memory)
__device__ __forceinline__ void product_if(uint32_t acc, uint32_t a, uint64_t b, uint32_t how, uint32_t add, uint32_t on)
{
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(acc),
                 "r"(a), "l"(b), "r"(how), "r"(add), "r"(on) : "memory");
}
__device__ __forceinline__ void commit_if(uint32_t bar, uint32_t on)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
                 "r"(on) : "memory");
}
template <int N> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void acc_loaded(uint32_t (&r)[N])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));         // not used before the wait
}
// two binary32 numbers at a time
__device__ __forceinline__ uint64_t two(float a, float b)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ void apart(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t mul_two(uint64_t a, uint64_t b)
{
    uint64_t v;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}
__device__ __forceinline__ uint64_t add_two(uint64_t a, uint64_t b)
{
    uint64_t v;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}
__device__ __forceinline__ uint64_t fma_two(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t v;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
    return v;
}
__device__ __forceinline__ uint32_t pack_two(uint64_t v)
{
    float a, b;
    apart(v, a, b);
    return pack_bf16(a, b);
}
__device__ __forceinline__ void acc_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void to_engine() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <int D>
__global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const AttnArgs a)
{
    using S = Shape<D>;
    constexpr int NG = S::NG, kRow = S::kRow, kUnits = D / 32;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[4 * kStages + 14];
    __shared__ int64_t warp_sum[kThreads / 32];
    __shared__ __align__(4) unsigned char bad[kStages][4];          // chunks of a stage without a page
    __shared__ uint32_t tmem_at, odd_rows[kBlockRows];              // bit gr: the row sees a value of group gr that is NaN
    __shared__ int failed, at_seq, at_item;
    unsigned char *smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
    const uint32_t base = smem_addr(smem);
    const uint32_t k_full = smem_addr(bars), v_full = k_full + 8 * kStages, v_empty = v_full + 8 * kStages, k_read = v_empty + 8 * kStages, s_full = k_read + 8 * kStages, p_full = s_full + 16, o_done = p_full + 32, s_read = o_done + 32, q_full = s_read + 16;
    // (p_full and o_done of a group: one for even, one for odd tiles.  A warp may be a tile ahead of the others' probabilities, and not every
    // product's end is waited for.)
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // ---- this block's item ----
    wait_for_stream();
    const int each = (a.b.seqs + kThreads - 1) / kThreads;
    const int s0 = min(tid * each, a.b.seqs), s1 = min(s0 + each, a.b.seqs);
    auto items_of = [&](const Seq &s) { return (int64_t)((s.fresh * a.share + kBlockRows - 1) / kBlockRows) * a.c.kv_heads; };
    int64_t own = 0;
#pragma unroll 1
    for (int b = s0; b < s1; ++b) own += items_of(sequence(a, b));
    int64_t incl = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 31) warp_sum[warp] = incl;
    if (tid < kBlockRows) odd_rows[tid] = 0;
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            bar_init(k_full + 8 * i, kWorkers / 2);
            bar_init(v_full + 8 * i, kWorkers / 2);
            bar_init(v_empty + 8 * i, 2);
            bar_init(k_read + 8 * i, 2);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(s_full + 8 * i, 1);
            bar_init(p_full + 16 * i, kSoftmax / 2);
            bar_init(p_full + 16 * i + 8, kSoftmax / 2);
            bar_init(o_done + 16 * i, 1);
            bar_init(o_done + 16 * i + 8, 1);
            bar_init(s_read + 8 * i, kSoftmax / 2);
            bar_init(q_full + 8 * i, kSoftmax / 2);
        }
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    int64_t total = 0;
#pragma unroll 1
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w == warp) incl += total;
        total += warp_sum[w];
    }
    if ((int64_t)blockIdx.x >= total) {                 // (there is one such block at least)
        zero_other_rows(a, (int)((int64_t)blockIdx.x - total), (int)((int64_t)gridDim.x - total), kThreads);
        return;
    }
    if ((int64_t)blockIdx.x >= incl - own && (int64_t)blockIdx.x < incl) {
        int64_t flat = incl - own;
#pragma unroll 1
        for (int b = s0; b < s1; ++b) {
            const int64_t n = items_of(sequence(a, b));
            if ((int64_t)blockIdx.x < flat + n) {
                at_seq  = b;
                at_item = (int)((int64_t)blockIdx.x - flat);
                break;
            }
            flat += n;
        }
    }
    if (warp == kSoftmax + kWorkers) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = tmem_at;
    const int  seq = at_seq;
    const Seq  s   = sequence(a, seq);
    const int  rows = s.fresh * a.share, blocks = (rows + kBlockRows - 1) / kBlockRows;
    const int  block = blocks - 1 - at_item / a.c.kv_heads, head = at_item % a.c.kv_heads;      // (the longest first)
    const int64_t most = a.b.table_ld << a.c.page_shift;
    const int  first_tok = by_share(a, block * kBlockRows), last_tok = min(by_share(a, block * kBlockRows + kBlockRows - 1), s.fresh - 1);
    const int  end = (int)min((int64_t)(s.len - s.fresh + last_tok + 1), most);
    const int  lo  = a.window > 0 ? max(s.len - s.fresh + first_tok + 1 - a.window, 0) & ~15 : 0;
    const int  subs = end > lo ? (end - lo + kSub - 1) / kSub : 0, n = (subs + 1) / 2;
    if (tid == 0 && s.len > most) kv_record(a.status, seq, (int)most);

    if (warp >= kSoftmax && warp < kSoftmax + kWorkers) {
        registers_down<kRegsWorker>();
        // ---- codes to operands ----
        const int dw = warp - kSoftmax, c = dw & 3, side = dw >> 2, ps = 1 << a.c.page_shift, g = lane >> 2, t = lane & 3;
        unsigned char *raw = smem + S::kRawAt + dw * kRaw * S::kRawChunk;
        const uint32_t raw_addr = smem_addr(raw);
        int pages = -1;
        uint32_t have = 0;                              // bit i: the chunk fetched i fetches ago has a page
        auto fetch = [&](int j) {
            if (j < n) {
                if ((j & 31) == 0) {
                    const int tok = lo + (j + lane) * kKeys + c * 16;
                    pages = j + lane < n && tok < end ? kv_page_of(a.c, a.b, a.status, seq, tok) : -1;
                }
                const int page = __shfl_sync(0xffffffffu, pages, j & 31), slot = (lo + j * kKeys + c * 16) & (ps - 1);
                const bool on = page >= 0;
                const unsigned char *head_at = a.c.pages + (int64_t)(on ? page : 0) * a.c.page_bytes + (int64_t)head * a.c.head_bytes;
                const unsigned char *src = head_at + (side * ps + slot) * kRow + lane * 16;
                const uint32_t dst = raw_addr + (j % kRaw) * S::kRawChunk;
#pragma unroll
                for (int u0 = 0; u0 < 16 * kUnits; u0 += 32) {
                    const int tok = (u0 + lane) / kUnits, u = lane % kUnits, turn = D == 64 ? tok >> 2 & 1 : tok >> 1 & 3;
                    copy16(dst + tok * kRow + ((u ^ turn) << 4), src + u0 * 16, on);
                }
                if (lane < 4 * NG) copy16(dst + 16 * kRow + lane * 16, head_at + ps * D + (side * ps + slot) * NG * 4 + lane * 16, on);
                have = have << 1 | (uint32_t)on;
            }
            copies_commit();
        };
#pragma unroll 1
        for (int j = 0; j < kRaw - 1; ++j) fetch(j);
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
            copies_wait<kRaw - 2>();
            __syncwarp();
            fetch(j + kRaw - 1);
            const bool on = have >> min(kRaw - 1, n - 1 - j) & 1;
            const int st = j % kStages, tok0 = lo + j * kKeys + c * 16;
            // a stage's keys are free once both softmax groups have taken the scores (and the scales) of the tile before it there, its
            // values once that tile's products with them are over (a barrier of its own for every stage: nobody can be two phases behind)
            if (j >= kStages && !warp_wait((side ? v_empty : k_read) + 8 * st, (j / kStages - 1) & 1, &failed)) goto done;
            const uint32_t from = raw_addr + (j % kRaw) * S::kRawChunk;
            const uint32_t *words = reinterpret_cast<const uint32_t *>(raw + (j % kRaw) * S::kRawChunk + 16 * kRow);
            const uint32_t to = base + S::kKV + st * S::kStage + side * NG * S::kSlabK;
            const int mt = (lane >> 4) * 8 + (lane & 7), mc = lane >> 3 & 1, turn = D == 64 ? mt >> 2 & 1 : mt >> 1 & 3;
            // what is hidden, or lies beyond the sequence's end, may be stored as anything, and a probability of 0 times a scale that is NaN would
            // count: such a value's scale is 0 here, and the rows that see it are noted
            uint32_t odd = 0;                           // bit gr: this lane's token
            if (lane < 16) {
                float *scales = reinterpret_cast<float *>(smem + S::kSc + st * S::kScales) + side * NG * kKeys + (c * 8 + (lane >> 1)) * 2 * NG + (lane & 1);
#pragma unroll
                for (int gr = 0; gr < NG; ++gr) {
                    const float f = __uint_as_float(words[lane * NG + gr]);
                    const bool fine = side == 0 || fabsf(f) < INFINITY;
                    scales[gr * 2] = side ? (fine ? f : 0.0f) : f * a.scale_log2;
                    if (!fine) odd |= 1u << gr;
                }
            }
            if (side && __any_sync(0xffffffffu, odd != 0)) {
#pragma unroll 1
                for (uint32_t rest = __ballot_sync(0xffffffffu, odd != 0); rest; rest &= rest - 1) {
                    const int of = __ffs(rest) - 1, tok = tok0 + of;
                    const uint32_t groups = __shfl_sync(0xffffffffu, odd, of);
#pragma unroll 1
                    for (int row = lane; row < kBlockRows && block * kBlockRows + row < rows; row += 32) {
                        const int at = s.len - s.fresh + by_share(a, block * kBlockRows + row);
                        if (tok <= at && (a.window == 0 || tok > at - a.window)) atomicOr(&odd_rows[row], groups);
                    }
                }
            }
            if (side == 0 && lane == 0) bad[st][c] = !on && tok0 < end;
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                uint32_t r[4], z0, z1, y0, y1;
                if (side == 0) {
                    matrices(r, from + mt * kRow + (((2 * gr + mc) ^ turn) << 4));
                    const uint32_t w0 = words[g * NG + gr], w1 = words[(g + 8) * NG + gr];
                    z0 = zeros_of(w0, w0), z1 = zeros_of(w1, w1);
                } else {
                    matrices_t(r, from + mt * kRow + (((2 * gr + mc) ^ turn) << 4));
                    z0 = zeros_of(words[2 * t * NG + gr], words[(2 * t + 1) * NG + gr]);
                    z1 = zeros_of(words[(2 * t + 8) * NG + gr], words[(2 * t + 9) * NG + gr]);
                }
                y0 = mul2(z0, kSixteen), y1 = mul2(z1, kSixteen);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t v[4] = {fma2(codes(r[0], i), kTwo127, i & 1 ? y0 : z0), fma2(codes(r[1], i), kTwo127, i & 1 ? y0 : z0),
                                           fma2(codes(r[2], i), kTwo127, i & 1 ? y1 : z1), fma2(codes(r[3], i), kTwo127, i & 1 ? y1 : z1)};
                    // four 8 x 8 matrices: keys' rows are tokens, their sixteen bytes channels; values' rows are channels 32 c + 4 g + i (at row
                    // 32 c + 8 i + g), their sixteen bytes eight tokens
                    const int row = side == 0 ? c * 16 + mt : mc * 32 + i * 8 + (lane & 7);
                    const int piece = side == 0 ? 4 * mc + i : c * 2 + (lane >> 4);
                    matrices_out(to + gr * S::kSlabK + row * 128 + ((piece ^ (row & 7)) << 4), v);
                }
            }
            to_engine();
            __syncwarp();
            bar_arrive_if((side ? v_full : k_full) + 8 * st, lane == 0);
        }
        copies_wait<0>();
    } else if (warp >= kSoftmax + kWorkers) {
        registers_down<kRegsRest>();
        // ---- products, 32 keys at a time: a warp for a group's scores, one for its outputs.  The next scores follow as soon as the softmax has
        // read the ones before; there are two sets of probabilities.  (The softmax takes a set's place, and the scales of the values, without a
        // wait of its own: when scores are there, the values are, and the product with the probabilities of two times before is over.) ----
        constexpr uint32_t kHow = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kRows / 16) << 24);
        constexpr uint32_t kHowScores = kHow | ((uint32_t)(kSub / 8) << 17), kHowOut = kHow | (8u << 17);
        const int which = __shfl_sync(0xffffffffu, warp - (kSoftmax + kWorkers), 0), w = which & 1;
        const uint32_t sc_at = __shfl_sync(0xffffffffu, tmem, 0) + w * 256, out_at = sc_at + 128, at = __shfl_sync(0xffffffffu, base, 0);
        const uint32_t on = elected();
        if (which < 2) {
            if (subs > 0 && !warp_wait(q_full + 8 * w, 0, &failed)) goto done;
#pragma unroll 1
            for (int i = 0; i < subs; ++i) {
                const int st = (i >> 1) % kStages;
                if (!(i & 1)) {
                    const uint32_t round = ((i >> 1) / kStages) & 1;
                    if (!warp_wait(k_full + 8 * st, round, &failed) || !warp_wait(v_full + 8 * st, round, &failed)) goto done;
                }
                if (i > 1 && !warp_wait(o_done + 16 * w + 8 * (i & 1), (i >> 1) - 1 & 1, &failed)) goto done;
                if (i > 0) {
                    if (!warp_wait(s_read + 8 * w, (i - 1) & 1, &failed)) goto done;
                    if (!(i & 1)) bar_arrive_if(k_read + 8 * (((i >> 1) - 1) % kStages), on);       // the stage before is read
                }
                tc_after();
#pragma unroll
                for (int gr = 0; gr < NG; ++gr) {
                    const uint64_t q = operand(at + S::kQ + (w * NG + gr) * S::kSlabQ);
                    const uint64_t k = operand(at + S::kKV + st * S::kStage + gr * S::kSlabK + (i & 1) * kSub * 128);
#pragma unroll
                    for (int x = 0; x < 4; ++x) product_if(sc_at + gr * kSub, q + 2 * x, k + 2 * x, kHowScores, x > 0, on);
                }
                commit_if(s_full + 8 * w, on);
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < subs; ++i) {
                const int st = (i >> 1) % kStages;
                if (!(i & 1) && !warp_wait(v_full + 8 * st, ((i >> 1) / kStages) & 1, &failed)) goto done;
                if (!warp_wait(p_full + 16 * w + 8 * (i & 1), i >> 1 & 1, &failed)) goto done;
                tc_after();
#pragma unroll
                for (int gr = 0; gr < NG; ++gr) {
                    const uint64_t v = operand(at + S::kKV + st * S::kStage + (NG + gr) * S::kSlabK) + 4 * (i & 1);
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        product_if(out_at + gr * 64, sc_at + 64 + (i & 1) * 32 + gr * 16 + x * 8, v + 2 * x, kHowOut, i > 0 || x > 0, on);
                }
                commit_if(o_done + 16 * w + 8 * (i & 1), on);
                if ((i & 1) || i + 1 == subs) commit_if(v_empty + 8 * st, on);
            }
        }
    } else {
        // ---- softmax: a warp has sixteen rows of its quarter of tensor memory, a thread two of them (8 b + lane / 4) and every fourth pair of
        // columns, so that a scale that it loads serves two rows ----
        registers_up<kRegsSoftmax>();
        const int w = warp >> 3, half = warp >> 2 & 1, row0 = block * kBlockRows + w * kRows, t2 = (lane & 3) * 2;
        const int mine = row0 + (warp & 3) * 32 + half * 16 + (lane >> 2);
        const uint32_t sc_at = tmem + ((uint32_t)(2 * (warp & 3) + half) << 20) + w * 256, out_at = sc_at + 128;
        const int least_hi = row0 < rows ? s.len - s.fresh + by_share(a, row0) + 1 : 0x7fffffff, most_lo = a.window > 0 ? s.len - s.fresh + last_tok + 1 - a.window : 0;
        // ---- the queries: half a row per thread; times 64 or 4, which the codes lack ----
        {
            const int r = (tid & 255) >> 1, side = tid & 1, row = row0 + r, tok = by_share(a, min(row, rows - 1)), hh = min(row, rows - 1) - tok * a.share;
            const __nv_bfloat16 *src = a.q + (int64_t)(s.start + tok) * a.q_ld + (int64_t)(head * a.share + hh) * a.q_head + side * (D / 2);
            uint4 v[NG * 4];
#pragma unroll
            for (int t = 0; t < NG * 4; ++t) {
                v[t] = make_uint4(0, 0, 0, 0);
                if (row < rows) {
                    if (a.q_vec) {
                        v[t] = *reinterpret_cast<const uint4 *>(src + t * 8);
                    } else {
                        const uint16_t *h = reinterpret_cast<const uint16_t *>(src + t * 8);
                        v[t] = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
                    }
                }
            }
#pragma unroll
            for (int cc = 0; cc < NG; ++cc) {
                const int gr = NG == 2 ? side : 0, c = NG == 2 ? cc : side;
#pragma unroll
                for (int i = 0; i < 4; ++i) {              // sixteen bytes: channels 8 t + i and 8 t + i + 4
                    uint32_t x[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const uint4 &y = v[cc * 4 + t];
                        x[t] = mul2(__byte_perm(i < 2 ? y.x : y.y, i < 2 ? y.z : y.w, i & 1 ? 0x7632 : 0x5410), i & 1 ? 0x40804080u : 0x42804280u);
                    }
                    *reinterpret_cast<uint4 *>(smem + S::kQ + (w * NG + gr) * S::kSlabQ + r * 128 + (((4 * c + i) ^ (r & 7)) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
                }
            }
            to_engine();
            __syncwarp();
            bar_arrive_if(q_full + 8 * w, lane == 0);
        }
        // scores are taken relative to m at once; `limit`: what they may come to before m is moved (a row that has seen nothing: any)
        float m[2] = {0.0f, 0.0f}, limit[2] = {-FLT_MAX, -FLT_MAX};
        uint64_t less[2] = {0, 0}, l[2] = {0, 0};       // -m twice; the sums of the thread's even and odd columns
        const int clean = min(least_hi, end) - kSub;    // tiles that start at most here, and at least at most_lo, hide nothing
#pragma unroll 1
        for (int i = 0; i < subs; ++i) {
            const int st = (i >> 1) % kStages, tok0 = lo + i * kSub;
            const float *ks = reinterpret_cast<const float *>(smem + S::kSc + st * S::kScales) + ((i & 1) * kSub + t2) * NG, *vs = ks + NG * kKeys;
            if (!warp_wait(s_full + 8 * w, i & 1, &failed)) goto done;
            tc_after();
            uint64_t sc[2][4];                          // rows 8 b + lane / 4, columns 8 j + t2 and the next
            {
                uint32_t x[16 * NG];
                acc_ask_rows(sc_at, x);
                if (NG == 2) acc_ask_rows(sc_at + kSub, x + 16 * (NG - 1));
                acc_loaded(x);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    ulonglong2 k;
                    if (NG == 2) k = *reinterpret_cast<const ulonglong2 *>(ks + j * 8 * NG);
                    else k.x = *reinterpret_cast<const uint64_t *>(ks + j * 8 * NG), k.y = 0;
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const uint32_t *y = x + 4 * j + 2 * b;
                        uint64_t v = fma_two(two(__uint_as_float(y[0]), __uint_as_float(y[1])), k.x, less[b]);
                        if (NG == 2) v = fma_two(two(__uint_as_float(y[16 * (NG - 1)]), __uint_as_float(y[16 * (NG - 1) + 1])), k.y, v);
                        sc[b][j] = v;
                    }
                }
            }
            const uint32_t gone = *reinterpret_cast<const volatile uint16_t *>(bad[st] + 2 * (i & 1));
            tc_before();
            __syncwarp();
            bar_arrive_if(s_read + 8 * w, lane == 0);         // scores, scales and `bad` are in registers
            if (tok0 > clean || tok0 < most_lo || gone != 0) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    int hi = 0x7fffffff, low = 0;       // a row of padding masks nothing
                    if (mine + 8 * b < rows) {
                        hi  = s.len - s.fresh + by_share(a, mine + 8 * b) + 1;
                        low = a.window > 0 ? max(hi - a.window, 0) : 0;
                    }
                    hi = min(hi, end);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float u, v;
                        apart(sc[b][j], u, v);
                        const int tok = tok0 + 8 * j + t2;
                        const bool lost = gone >> 8 * (j >> 1) & 1u;
                        if (tok >= hi || tok < low || lost) u = -INFINITY;
                        if (tok + 1 >= hi || tok + 1 < low || lost) v = -INFINITY;
                        sc[b][j] = two(u, v);
                    }
                }
            }
            float top[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                top[b] = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float u, v;
                    apart(sc[b][j], u, v);
                    top[b] = fmaxf(fmaxf(top[b], u), v);
                }
            }
            // (the maximum in use may lie up to 2^8 below the true one)
            if (__any_sync(0xffffffffu, top[0] > limit[0] || top[1] > limit[1])) {
                float keep[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    top[b] = fmaxf(top[b], __shfl_xor_sync(0xffffffffu, top[b], 1));
                    top[b] = fmaxf(top[b], __shfl_xor_sync(0xffffffffu, top[b], 2));
                    const bool first = limit[b] < 0.0f, up = top[b] > (first ? limit[b] : 0.0f);
                    const float now = up ? m[b] + top[b] : m[b], by = now - m[b];
                    keep[b] = first ? 0.0f : power2(-by);
                    if (up) limit[b] = 8.0f;
                    m[b]    = now;
                    less[b] = two(-now, -now);
                    l[b]    = mul_two(l[b], two(keep[b], keep[b]));
#pragma unroll
                    for (int j = 0; j < 4; ++j) sc[b][j] = add_two(sc[b][j], two(-by, -by));
                }
                if (i > 0) {
                    if (!warp_wait(o_done + 16 * w + 8 * ((i - 1) & 1), (i - 1) >> 1 & 1, &failed)) goto done;
                    tc_after();
#pragma unroll 1
                    for (int c0 = 0; c0 < D; c0 += 32) {
                        uint32_t v[16];
                        acc_ask_rows(out_at + c0, v);
                        acc_loaded(v);
#pragma unroll
                        for (int x = 0; x < 16; ++x) v[x] = __float_as_uint(__uint_as_float(v[x]) * keep[x >> 1 & 1]);
                        acc_store_rows(out_at + c0, v);
                    }
                }
            }
            uint32_t p[NG][8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                ulonglong2 f;
                if (NG == 2) f = *reinterpret_cast<const ulonglong2 *>(vs + j * 8 * NG);
                else f.x = *reinterpret_cast<const uint64_t *>(vs + j * 8 * NG), f.y = 0;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    float u, v;
                    apart(sc[b][j], u, v);
                    const uint64_t e = two(power2(u), power2(v));
                    l[b] = add_two(l[b], e);
                    p[0][2 * j + b] = pack_two(mul_two(e, f.x));
                    if (NG == 2) p[NG - 1][2 * j + b] = pack_two(mul_two(e, f.y));
                }
            }
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) pairs_store(sc_at + 64 + (i & 1) * 32 + gr * 16, p[gr]);
            acc_stored();
            tc_before();
            __syncwarp();
            bar_arrive_if(p_full + 16 * w + 8 * (i & 1), lane == 0);
        }
        // ---- the output: what is left in tensor memory, divided by the row's sum.  Column 8 j + g of 32 is channel 4 g + j: a thread has eight
        // neighbouring channels of each of its rows ----
        if (subs > 0 && !warp_wait(o_done + 16 * w + 8 * ((subs - 1) & 1), (subs - 1) >> 1 & 1, &failed)) goto done;
        tc_after();
        float inv[2];
        __nv_bfloat16 *out[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            float u, v;
            apart(l[b], u, v);
            u += v;
            u += __shfl_xor_sync(0xffffffffu, u, 1);
            u += __shfl_xor_sync(0xffffffffu, u, 2);
            inv[b] = u > 0.0f ? 1.0f / u : (u == 0.0f ? 0.0f : u);
            const int row = min(mine + 8 * b, rows - 1), tok = by_share(a, row);
            out[b] = a.out + (int64_t)(s.start + tok) * a.out_ld + (int64_t)(head * a.share + row - tok * a.share) * a.out_head + t2 * 4;
        }
#pragma unroll 1
        for (int at = 0; at < D; at += 32) {
            uint32_t v[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) v[x] = 0;
            if (subs > 0) {
                acc_ask_rows(out_at + at, v);
                acc_loaded(v);
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (mine + 8 * b < rows) {
                    const float f = odd_rows[mine - block * kBlockRows + 8 * b] >> (at / 64) & 1u ? __uint_as_float(0x7fc00000u) : inv[b];
                    auto of = [&](int j, int g) { return (j & 1 ? 4.0f : 64.0f) * __uint_as_float(v[4 * j + 2 * b + g]) * f; };
                    const uint4 x = make_uint4(pack_bf16(of(0, 0), of(1, 0)), pack_bf16(of(2, 0), of(3, 0)), pack_bf16(of(0, 1), of(1, 1)), pack_bf16(of(2, 1), of(3, 1)));
                    __nv_bfloat16 *to = out[b] + at;
                    if (a.out_vec) {
                        *reinterpret_cast<uint2 *>(to) = make_uint2(x.x, x.y);
                        *reinterpret_cast<uint2 *>(to + 4) = make_uint2(x.z, x.w);
                    } else {
                        uint16_t *h = reinterpret_cast<uint16_t *>(to);
                        const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int z = 0; z < 4; ++z) h[2 * z] = (uint16_t)y[z], h[2 * z + 1] = (uint16_t)(y[z] >> 16);
                    }
                }
            }
        }
    }
done:
    __syncwarp();
    tc_before();
    __syncthreads();
    tc_after();
    if (failed) {
        // copies and products may still be in flight: give them time to end before the memory is let go
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        if (tid == 0 && atomicCAS(a.status + 3, 0, 1) == 0) atomicExch(a.status, SYMAR_ERR_TIMEOUT);
    }
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == kSoftmax + kWorkers) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// items that the call has at most: a block each (blocks beyond the last item have only rows of no sequence to look at)
int64_t items_at_most(const AttnArgs &a)
{
    return ((int64_t)a.b.tokens * a.share / kBlockRows + (a.b.seqs < a.b.tokens ? a.b.seqs : a.b.tokens)) * a.c.kv_heads;
}

// The warpgroups share out what a block is launched with; with less than that they would wait for ever.
template <int D>
bool registers_suffice(int device)
{
    static std::atomic<uint64_t> known{0};
    const uint64_t bit = device >= 0 && device < 64 ? 1ull << device : 0;
    if (known.load(std::memory_order_relaxed) & bit) return true;
    cudaFuncAttributes at;
    if (cudaFuncGetAttributes(&at, (const void *)prompt_kernel<D>) != cudaSuccess || at.numRegs < kRegsLaunch) return false;
    known.fetch_or(bit, std::memory_order_relaxed);
    return true;
}
template <int D>
cudaError_t launch(const AttnArgs &a, unsigned blocks, int device, cudaStream_t stream)
{
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_shared((const void *)prompt_kernel<D>, Shape<D>::kBytes, device, allowed);
    if (e != cudaSuccess) return e;
    return launch_early(prompt_kernel<D>, dim3(blocks), kThreads, Shape<D>::kBytes, stream, a);
}
}  // namespace

bool prompt_attention_takes(const AttnArgs &a, int num_sms, int device)
{
    if (a.c.dim > 128 || items_at_most(a) > 0x3fffffff) return false;
    // Blocks that are half full at least, and for a quarter of the multiprocessors.  (64 heads, 8 key/value heads of 128 unless said; this kernel
    // against the one that shares a sequence's tokens between blocks, us: 512 new tokens over 8192, 128 blocks: 230, 867; 256: 217, 438; 128,
    // 32 blocks: 214, 226; 64: 214, 121.  512 over 32768 with 8 heads of one, 16 blocks: 817, 441.  8 x 16 over 2048, half-full blocks: 63, 73;
    // 64 x 8 over 1024, a quarter full: 140, 134; 32 x 32 over 1024 with 8 heads of 8, an eighth: 70, 48.  Heads of 64: 512 over 8192: 185, 553; 128: 174, 149.)
    // Lengths are on the device, so the rule knows averages alone: a batch of long pieces and single tokens goes to one kernel as a whole.
    const int64_t rows = (int64_t)a.b.tokens * a.share;                // of one key/value head
    const int64_t blocks = rows / kBlockRows > a.b.seqs ? rows / kBlockRows : a.b.seqs;
    if (rows < (int64_t)kRows * a.b.seqs || blocks * a.c.kv_heads < num_sms / 4) return false;
    return a.c.dim == 64 ? registers_suffice<64>(device) : registers_suffice<128>(device);
}

cudaError_t launch_prompt_attention(const AttnArgs &a, int device, cudaStream_t stream)
{
    const unsigned blocks = (unsigned)items_at_most(a) + 1;
    return a.c.dim == 64 ? launch<64>(a, blocks, device, stream) : launch<128>(a, blocks, device, stream);
}

}  // namespace symar
