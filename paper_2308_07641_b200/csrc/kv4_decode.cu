// Attention over the 4-bit cache for few query rows (single tokens, short pieces): bound by streaming the cache.
//
//     out = sum_j p_j v_j / sum_j p_j,   p_j = exp2(c q.k_j - ref),   c = scale log2(e)
//
// Work.  An item is (sequence, key/value head, group of 8 NT query rows: the heads that share the key/value head, of one
// or several tokens); its unit is a block of 16 cached positions.  All units of the call, item after item, are cut into
// equal runs, one for each block of a persistent grid, so ragged batches and single long sequences spread alike.  A block's
// eight warps take the run's units in turn; each warp has its own ring of units in shared memory, filled by bulk copies
// that run ahead across item borders.  At an item's end the warps' sums meet in shared memory; an item that spans blocks
// leaves its parts in scratch, and the block that finishes last adds them in their order (so results do not depend on it).
//
// Arithmetic.  mma.sync m16n8k16 in fp16 with fp32 sums, the cached side as the 16-row operand, the query rows as the
// 8-column one.  Scores use the codes as they are: a mask and an or make fp16 pairs 1024 + code, or 1024 + 16 code for the
// odd nibbles, whose q is divided by 16 beforehand; 1024 sum q comes off through the accumulator's start value, and step and
// base of the group are applied to the fp32 sum: s (q.code) + b (sum q).  So scores carry no rounding of k at all.  q enters
// as fp16 after division by a power of two per row (exact up to 2^-24 of the row's largest).  Values become fp16 numbers
// code * step + base (one rounding); probabilities fp16, at most 2^8 above the reference, which moves only when a score
// passes it by more than 8 (in units of log2): no exchange between lanes otherwise.
#include <algorithm>

#include "serving.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace ptx;

constexpr int DEC_WARPS = 7;             // warps that compute; one more feeds their rings
constexpr int DEC_THREADS = (DEC_WARPS + 1) * 32;
constexpr int DEC_QUEUE = 4;             // items that the feeding warp may be ahead
constexpr float kSlack = 8.0f;           // how far (log2) a score may pass the reference before it moves
constexpr float kNone = -1e30f;          // the reference before the first score

struct DecParams {
    Kv4Geom g;
    Kv4Batch b;
    const __nv_bfloat16* q;
    long long ldq;
    __nv_bfloat16* out;
    long long ldo;
    int group;           // query heads of one key/value head
    int max_q;
    float c;             // scale * log2(e)
    int window, causal;
    int min_share;       // units of a run at least
    float* parts;        // [grid][2][rows][D + 2]
    unsigned* tickets;   // [grid]
    int* status;
};

__device__ __forceinline__ uint32_t lop_or(uint32_t x, uint32_t mask) { return (x & mask) | 0x64006400u; }
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t h2(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t hfma(uint32_t a, uint32_t b, uint32_t c)
{
    const __half2 v = __hfma2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b), *reinterpret_cast<__half2*>(&c));
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 halves(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

__device__ __forceinline__ void warps_sync() { asm volatile("bar.sync 1, %0;" ::"n"(DEC_WARPS * 32) : "memory"); }
__device__ __forceinline__ bool any_of_the_warps(bool x)
{
    uint32_t y;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.red.or.pred q, 1, %2, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(y)
        : "r"((uint32_t)x), "n"(DEC_WARPS * 32)
        : "memory");
    return y != 0;
}

template <int WORDS>
struct alignas(4 * WORDS) Words { uint32_t w[WORDS]; };

// What one sequence brings (the lanes of the feeding warp hold 32 sequences, one each).
struct Seq {
    int rows, len, first, items, blk0, units;   // units of one item; blk0: its first block
    int all;                                    // its rows, those beyond max_q (which are not computed) included
};

template <int ROWS>
__device__ __forceinline__ Seq load_seq(const DecParams& p, int s)
{
    Seq q{0, 0, 0, 0, 0, 0, 0};
    if (s >= p.b.n_seq) return q;
    q.first = kv4_first_row(p.b, s);
    q.all = kv4_first_row(p.b, s + 1) - q.first;
    q.rows = min(q.all, p.max_q);
    if (q.rows <= 0) { q.rows = 0; return q; }
    q.len = p.b.seq_len[s];
    const long long room = (long long)p.b.max_pages * p.g.page_tokens;
    const long long seen = q.len < 0 ? 0 : min((long long)q.len, room);
    if (q.len > room) atomicOr(p.status, KV4_DEV_INDEX);
    long long lo = 0, hi = seen;
    const long long pos0 = (long long)q.len - q.all;          // of the first row
    if (p.window) lo = max(0LL, pos0 - p.window + 1);
    if (p.causal) hi = min(hi, pos0 + q.rows);
    q.items = p.g.heads * ((q.rows * p.group + ROWS - 1) / ROWS);
    q.blk0 = (int)(lo / KV4_BLOCK);
    q.units = hi > lo ? (int)((hi + KV4_BLOCK - 1) / KV4_BLOCK) - q.blk0 : 1;   // an item that sees nothing still writes zeros
    return q;
}

// An item as the computing warps get it.
struct Item {
    int first_row, n_rows;     // of the call; (row, head) pairs of the item's sequence and head in all
    int head, row0;            // the pairs row0 .. are this item's
    int len, pos0;             // positions that can be seen at all; position of the sequence's first row
    int blk0, unit0, unit1, units;
    int b_first, b_last;       // the blocks of the grid that share it
};

template <int D, int NT, int STAGES>
__global__ void __launch_bounds__(DEC_THREADS, NT == 1 ? 2 : 1)
kv4_decode_kernel(const DecParams p)
{
    constexpr int ROWS = 8 * NT, W = D / KV4_GROUP, UNIT = 20 * D, VW = D / 64;   // VW: words of value codes per thread and key
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 127) & ~(uintptr_t)127);
    float* meet = reinterpret_cast<float*>(ring + DEC_WARPS * STAGES * UNIT);       // [warps][ROWS][D]
    __shared__ uint64_t full[DEC_WARPS][STAGES], empty[DEC_WARPS][STAGES], item_full[DEC_QUEUE], item_empty[DEC_QUEUE];
    __shared__ uint8_t there[DEC_WARPS][STAGES];
    __shared__ Item queue[DEC_QUEUE];
    __shared__ float ref_2[2][DEC_WARPS][ROWS], sum_2[2][DEC_WARPS][ROWS];   // one pair is read while the next item's is written
    __shared__ int ctl_[2];
    __shared__ unsigned last_s;
    volatile int* ctl = ctl_;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        ctl[0] = 0;
        ctl[1] = kWaitLimitDefault;
        for (int w = 0; w < DEC_WARPS; ++w)
            for (int i = 0; i < STAGES; ++i) { mbar_init(&full[w][i], 1); mbar_init(&empty[w][i], 1); }
        for (int i = 0; i < DEC_QUEUE; ++i) { mbar_init(&item_full[i], 1); mbar_init(&item_empty[i], DEC_WARPS); }
        fence_mbar_init();
    }
    __syncthreads();
    pdl_launch_dependents();
    pdl_wait();

    if (warp == DEC_WARPS) {
        // ================= the feeding warp: the block's run of units, item by item =================
        long long total = 0;
        for (int s0 = 0; s0 < p.b.n_seq; s0 += 32) {
            const Seq q = load_seq<ROWS>(p, s0 + lane);
            total += (long long)q.items * q.units;
        }
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        const long long share = max((total + gridDim.x - 1) / gridDim.x, (long long)p.min_share);
        const long long u0 = share * blockIdx.x, u1 = min(u0 + share, total);
        int q_at = 0;
        uint32_t q_phase = 0;
        if (u0 < u1) {
            int base = 0, s = 0, item = 0, unit = 0;     // base: the sequences that the lanes hold
            long long item_u0 = 0;                       // where the item begins in the call's list of units
            Seq mine = load_seq<ROWS>(p, lane);
            for (long long before = 0;;) {
                const long long n = (long long)mine.items * mine.units;
                long long scan = n;
                for (int o = 1; o < 32; o <<= 1) {
                    const long long v = __shfl_up_sync(0xffffffffu, scan, o);
                    if (lane >= o) scan += v;
                }
                const unsigned holds = __ballot_sync(0xffffffffu, before + scan > u0);
                if (holds) {
                    const int l = __ffs(holds) - 1;
                    const long long start = before + __shfl_sync(0xffffffffu, scan - n, l);
                    const int units = __shfl_sync(0xffffffffu, mine.units, l);
                    s = base + l;
                    item = (int)((u0 - start) / units);
                    unit = (int)((u0 - start) % units);
                    item_u0 = u0 - unit;
                    break;
                }
                before += __shfl_sync(0xffffffffu, scan, 31);
                base += 32;
                mine = load_seq<ROWS>(p, base + lane);
            }
            const int per_page = p.g.page_tokens / KV4_BLOCK;
            int stage = 0;                               // of the ring that this lane feeds
            uint32_t phase = 0;
            bool ok = true;
            while (ok) {
                const int who = s - base;
                const int units = __shfl_sync(0xffffffffu, mine.units, who), items = __shfl_sync(0xffffffffu, mine.items, who);
                const int blk0 = __shfl_sync(0xffffffffu, mine.blk0, who), len = __shfl_sync(0xffffffffu, mine.len, who);
                const int rows = __shfl_sync(0xffffffffu, mine.rows, who), first = __shfl_sync(0xffffffffu, mine.first, who);
                const int all = __shfl_sync(0xffffffffu, mine.all, who);
                const int unit1 = (int)min((long long)units, u1 - item_u0), head = item % p.g.heads;
                if (lane == 0) {
                    ok = mbar_wait(&item_empty[q_at], q_phase ^ 1, ctl);
                    if (ok) {
                        Item it;
                        it.first_row = first;
                        it.n_rows = rows * p.group;
                        it.head = head;
                        it.row0 = item / p.g.heads * ROWS;
                        it.len = (int)max(0LL, min((long long)len, (long long)p.b.max_pages * p.g.page_tokens));
                        it.pos0 = len - all;
                        it.blk0 = blk0;
                        it.unit0 = unit;
                        it.unit1 = unit1;
                        it.units = units;
                        it.b_first = (int)(item_u0 / share);
                        it.b_last = (int)((item_u0 + units - 1) / share);
                        queue[q_at] = it;
                        mbar_arrive(&item_full[q_at]);
                    }
                }
                if (!__shfl_sync(0xffffffffu, ok, 0)) break;
                if (++q_at == DEC_QUEUE) { q_at = 0; q_phase ^= 1; }
                // lane w: units unit + w, + DEC_WARPS, ... into the ring of warp w; a page number is asked for one turn ahead
                auto page_of = [&](int u) {
                    const int blk = blk0 + u;
                    if (u >= unit1 || (long long)blk * KV4_BLOCK >= len || blk / per_page >= p.b.max_pages) return -2;   // no such position
                    return p.b.table[(long long)s * p.b.max_pages + blk / per_page];
                };
                if (lane < DEC_WARPS) {
                    int page = page_of(unit + lane);
                    for (int u = unit + lane; u < unit1; u += DEC_WARPS) {
                        const int next = page_of(u + DEC_WARPS);
                        if (!mbar_wait(&empty[lane][stage], phase ^ 1, ctl)) { ok = false; break; }
                        const bool in = page >= 0 && page < p.g.n_pages;
                        there[lane][stage] = in;
                        if (in) {
                            mbar_arrive_expect_tx(&full[lane][stage], UNIT);
                            bulk_g2s(ring + (lane * STAGES + stage) * UNIT, p.g.block(page, head, (blk0 + u) % per_page * KV4_BLOCK), UNIT,
                                     &full[lane][stage]);
                        } else {
                            if (page != -2) atomicOr(p.status, KV4_DEV_INDEX);
                            mbar_arrive(&full[lane][stage]);
                        }
                        page = next;
                        if (++stage == STAGES) { stage = 0; phase ^= 1; }
                    }
                }
                ok = __all_sync(0xffffffffu, ok);
                // the next item
                item_u0 += units;
                if (item_u0 >= u1) break;
                unit = 0;
                if (++item == items) {
                    item = 0;
                    int more = 0;
                    do {
                        if (++s == base + 32) { base += 32; mine = load_seq<ROWS>(p, base + lane); }
                        more = __shfl_sync(0xffffffffu, mine.items, s - base);
                    } while (more == 0 && s < p.b.n_seq);
                    if (more == 0) break;                // only if the lengths changed meanwhile
                }
            }
            // where a wait gave up, copies in flight are waited for (with a limit)
            if (ctl[0] && lane < DEC_WARPS)
                for (int i = 0; i < STAGES; ++i)
                    for (int n = 0; n < 4096 && !mbar_try_wait_64(&full[lane][i], i < stage ? phase : phase ^ 1); ++n) { }
        }
        __syncwarp();
        if (lane == 0 && mbar_wait(&item_empty[q_at], q_phase ^ 1, ctl)) {
            queue[q_at].units = 0;                       // the end
            mbar_arrive(&item_full[q_at]);
        }
        return;
    }

    // ================= the computing warps =================
    const int r = lane >> 2, j = lane & 3;
    int stage = 0, q_at = 0;
    uint32_t phase = 0, q_phase = 0;
    bool ok = true;
    for (int turn = 0;; turn ^= 1) {
        float (*ref_s)[ROWS] = ref_2[turn], (*sum_s)[ROWS] = sum_2[turn];
        if (!mbar_wait(&item_full[q_at], q_phase, ctl)) ok = false;
        if (any_of_the_warps(!ok)) break;          // a wait gave up: all leave together
        if (queue[q_at].units == 0) break;
        const Item it = queue[q_at];

        // ---- the item's query rows ----
        uint32_t qf[NT][2 * W][2];           // [..][MMA step][word]: column r
        float off[NT][W][2], qsum[NT][W][2], cmul[NT][2];   // columns 2 j, 2 j + 1
        int lo[NT][2], hi[NT][2];            // positions [lo, hi) that those columns see
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int row = it.row0 + 8 * t + r;
            const __nv_bfloat16* src = nullptr;
            if (row < it.n_rows) src = p.q + (long long)(it.first_row + row / p.group) * p.ldq + (long long)(it.head * p.group + row % p.group) * D;
            float v[W][8];
            float top = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                uint4 x = src ? *reinterpret_cast<const uint4*>(src + 32 * w + 8 * j) : make_uint4(0, 0, 0, 0);
                const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[w][2 * i] = __uint_as_float(xs[i] << 16);
                    v[w][2 * i + 1] = __uint_as_float(xs[i] & 0xffff0000u);
                    top = fmaxf(top, fmaxf(fabsf(v[w][2 * i]), fabsf(v[w][2 * i + 1])));
                }
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // divide by the power of two at or below the row's largest (2^-60 at least)
            const int e = min(max((int)(__float_as_uint(top) >> 23), 67), 253) - 127;
            const float down = __uint_as_float((uint32_t)(127 - e) << 23);
            float so[W], ss[W];
#pragma unroll
            for (int w = 0; w < W; ++w) {
                so[w] = ss[w] = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {      // pairs (2 i, 2 i + 1): odd i hold q / 16
                    const float f = (i & 1) ? down * 0.0625f : down, back = (i & 1) ? 16.0f : 1.0f;
                    const uint32_t pr = h2(v[w][2 * i] * f, v[w][2 * i + 1] * f);
                    qf[t][2 * w + (i >> 1)][i & 1] = pr;
                    const float2 as = halves(pr);
                    so[w] += 1024.0f * (as.x + as.y);
                    ss[w] += back * (as.x + as.y);
                }
                so[w] += __shfl_xor_sync(0xffffffffu, so[w], 1);
                so[w] += __shfl_xor_sync(0xffffffffu, so[w], 2);
                ss[w] += __shfl_xor_sync(0xffffffffu, ss[w], 1);
                ss[w] += __shfl_xor_sync(0xffffffffu, ss[w], 2);
            }
            const float up = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int from = 4 * (2 * j + k);
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    off[t][w][k] = -__shfl_sync(0xffffffffu, so[w], from);
                    qsum[t][w][k] = __shfl_sync(0xffffffffu, ss[w], from);
                }
                cmul[t][k] = p.c * __shfl_sync(0xffffffffu, up, from);
                const int col = it.row0 + 8 * t + 2 * j + k;
                const int pos = it.pos0 + col / p.group;
                // (a column without a row: its q is 0, nothing is hidden and nothing written)
                hi[t][k] = col >= it.n_rows ? 0x7fffffff : p.causal ? max(0, min(pos + 1, it.len)) : it.len;
                lo[t][k] = p.window && col < it.n_rows ? max(0, pos - p.window + 1) : 0;
            }
        }

        float o[NT][D / 16][4], ref[NT][2], sum[NT][2];
        int all_lo = 0, all_hi = 0x7fffffff;      // positions that every column sees
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[t][i][k] = 0.0f;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                ref[t][k] = kNone;
                sum[t][k] = 0.0f;
                all_lo = max(all_lo, lo[t][k]);
                all_hi = min(all_hi, hi[t][k]);
            }
        }
        all_lo = __reduce_max_sync(0xffffffffu, all_lo);
        all_hi = __reduce_min_sync(0xffffffffu, all_hi);

        // ---- its units ----
        for (int u = it.unit0 + warp; u < it.unit1; u += DEC_WARPS) {
            if (!mbar_wait(&full[warp][stage], phase, ctl)) { ok = false; break; }
            const uint8_t* blk = ring + (warp * STAGES + stage) * UNIT;
            if (there[warp][stage]) {
                const int pos_blk = (it.blk0 + u) * KV4_BLOCK;
                // rows r and r + 8 of the score tile are the block's positions kr and kr + 8
                const int kr = (r >> 1) + 4 * (r & 1);
                Words<W> kw[2], ks[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    kw[h] = *reinterpret_cast<const Words<W>*>(blk + (kr + 8 * h) * (D / 2) + j * 4 * W);
                    ks[h] = *reinterpret_cast<const Words<W>*>(blk + 8 * D + (kr + 8 * h) * (D / 8));
                }
                float sc[NT][4];
#pragma unroll
                for (int t = 0; t < NT; ++t) sc[t][0] = sc[t][1] = sc[t][2] = sc[t][3] = 0.0f;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const uint32_t x0 = kw[0].w[w], x1 = kw[1].w[w], y0 = x0 >> 8, y1 = x1 >> 8;
                    const uint32_t a[8] = {lop_or(x0, 0x000f000fu), lop_or(x1, 0x000f000fu), lop_or(x0, 0x00f000f0u), lop_or(x1, 0x00f000f0u),
                                           lop_or(y0, 0x000f000fu), lop_or(y1, 0x000f000fu), lop_or(y0, 0x00f000f0u), lop_or(y1, 0x00f000f0u)};
                    const float2 s0 = halves(ks[0].w[w]), s1 = halves(ks[1].w[w]);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        float d[4] = {off[t][w][0], off[t][w][1], off[t][w][0], off[t][w][1]};
                        mma_f16(d, a[0], a[1], a[2], a[3], qf[t][2 * w][0], qf[t][2 * w][1]);
                        mma_f16(d, a[4], a[5], a[6], a[7], qf[t][2 * w + 1][0], qf[t][2 * w + 1][1]);
                        sc[t][0] = fmaf(s0.y, qsum[t][w][0], fmaf(s0.x, d[0], sc[t][0]));
                        sc[t][1] = fmaf(s0.y, qsum[t][w][1], fmaf(s0.x, d[1], sc[t][1]));
                        sc[t][2] = fmaf(s1.y, qsum[t][w][0], fmaf(s1.x, d[2], sc[t][2]));
                        sc[t][3] = fmaf(s1.y, qsum[t][w][1], fmaf(s1.x, d[3], sc[t][3]));
                    }
                }
                if (pos_blk < all_lo || pos_blk + KV4_BLOCK > all_hi) {
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int pos = pos_blk + kr + (k & 2 ? 8 : 0);
                            // hidden whatever the scale's sign: the product below has to be -inf
                            if (pos < lo[t][k & 1] || pos >= hi[t][k & 1]) sc[t][k] = cmul[t][k & 1] < 0.0f ? INFINITY : -INFINITY;
                        }
                }
                float e[NT][4];
                bool over = false;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        e[t][k] = fmaf(sc[t][k], cmul[t][k & 1], -ref[t][k & 1]);
                        over |= e[t][k] > kSlack;
                    }
                if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float x = sc[t][k] * cmul[t][k], y = sc[t][k + 2] * cmul[t][k];
                            float m = fmaxf(ref[t][k], fmaxf(x, y));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                            const float keep = ex2(ref[t][k] - m);       // 0 before the first score
                            ref[t][k] = m;
                            sum[t][k] *= keep;
#pragma unroll
                            for (int i = 0; i < D / 16; ++i) { o[t][i][k] *= keep; o[t][i][k + 2] *= keep; }
                            e[t][k] = x - m;
                            e[t][k + 2] = y - m;
                        }
                }
                uint32_t pb[NT][2];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) e[t][k] = ex2(e[t][k]);
                    sum[t][0] += e[t][0] + e[t][2];
                    sum[t][1] += e[t][1] + e[t][3];
                    pb[t][0] = transpose8(h2(e[t][0], e[t][1]));
                    pb[t][1] = transpose8(h2(e[t][2], e[t][3]));
                }
                // values: this thread's key pairs (j, j + 4) and (j + 8, j + 12), numbers D/8 r .. of each
                const uint8_t* vb = blk + 10 * D;
                Words<VW> vw[4];
                uint32_t vs[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    vw[h] = *reinterpret_cast<const Words<VW>*>(vb + (j + 4 * h) * (D / 2) + r * 4 * VW);
                    vs[h] = *reinterpret_cast<const uint32_t*>(blk + 18 * D + (j + 4 * h) * (D / 8) + (r * W / 8) * 4);
                }
                const uint32_t st0 = __byte_perm(vs[0], vs[1], 0x5410), bs0 = __byte_perm(vs[0], vs[1], 0x7632);
                const uint32_t st1 = __byte_perm(vs[2], vs[3], 0x5410), bs1 = __byte_perm(vs[2], vs[3], 0x7632);
                constexpr uint32_t kOne = 0x3c003c00u, kMinus1024 = 0xe400e400u, kSixteenth = 0x2c002c00u, kMinus64 = 0xd400d400u;
#pragma unroll
                for (int x = 0; x < VW; ++x) {
                    uint32_t lo0 = __byte_perm(vw[0].w[x], vw[1].w[x], 0x5410), hi0 = __byte_perm(vw[0].w[x], vw[1].w[x], 0x7632);
                    uint32_t lo1 = __byte_perm(vw[2].w[x], vw[3].w[x], 0x5410), hi1 = __byte_perm(vw[2].w[x], vw[3].w[x], 0x7632);
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const uint32_t mask = (n & 1) ? 0x00f000f0u : 0x000f000fu;
                        const uint32_t mul = (n & 1) ? kSixteenth : kOne, add = (n & 1) ? kMinus64 : kMinus1024;
                        const uint32_t a0 = hfma(hfma(lop_or(lo0, mask), mul, add), st0, bs0), a1 = hfma(hfma(lop_or(hi0, mask), mul, add), st0, bs0);
                        const uint32_t a2 = hfma(hfma(lop_or(lo1, mask), mul, add), st1, bs1), a3 = hfma(hfma(lop_or(hi1, mask), mul, add), st1, bs1);
#pragma unroll
                        for (int t = 0; t < NT; ++t) mma_f16(o[t][4 * x + n], a0, a1, a2, a3, pb[t][0], pb[t][1]);
                        if (n == 1) { lo0 >>= 8; hi0 >>= 8; lo1 >>= 8; hi1 >>= 8; }
                    }
                }
            }
            __syncwarp();                      // every lane has read the slot
            if (lane == 0) mbar_arrive(&empty[warp][stage]);
            if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }

        // ---- the warps' sums ----
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float v = sum[t][k];
                v += __shfl_xor_sync(0xffffffffu, v, 4);
                v += __shfl_xor_sync(0xffffffffu, v, 8);
                v += __shfl_xor_sync(0xffffffffu, v, 16);
                if (r == 0) {
                    ref_s[warp][8 * t + 2 * j + k] = ref[t][k];
                    sum_s[warp][8 * t + 2 * j + k] = v;
                }
            }
        warps_sync();
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int col = 8 * t + 2 * j + k;
                float top = kNone;
#pragma unroll
                for (int w = 0; w < DEC_WARPS; ++w) top = fmaxf(top, ref_s[w][col]);
                const float f = ex2(ref[t][k] - top);
                float* to = meet + (warp * ROWS + col) * D + (D / 8) * r;
#pragma unroll
                for (int i = 0; i < D / 16; ++i)       // tile 4 x + n: numbers 8 x + 2 n and the next
                    *reinterpret_cast<float2*>(to + 2 * i) = make_float2(o[t][i][k] * f, o[t][i][k + 2] * f);
            }
        warps_sync();
        const int cols = min(ROWS, it.n_rows - it.row0);
        const bool starts = it.unit0 == 0, whole = starts && it.unit1 == it.units;
        auto write = [&](int col, int d, float4 v, float l) {
            const int row = it.row0 + col;
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            __nv_bfloat162 a = __floats2bfloat162_rn(v.x * inv, v.y * inv), b = __floats2bfloat162_rn(v.z * inv, v.w * inv);
            *reinterpret_cast<uint2*>(p.out + (long long)(it.first_row + row / p.group) * p.ldo +
                                      (long long)(it.head * p.group + row % p.group) * D + d) =
                make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
        };
        constexpr int PART = ROWS * (D + 2);
        float* part = p.parts + ((size_t)blockIdx.x * 2 + (starts ? 1 : 0)) * PART;
        for (int i = threadIdx.x; i < cols * (D / 4); i += DEC_WARPS * 32) {
            const int col = i / (D / 4), d = i % (D / 4) * 4;
            float top = kNone, l = 0.0f;
#pragma unroll
            for (int w = 0; w < DEC_WARPS; ++w) top = fmaxf(top, ref_s[w][col]);
            float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
            for (int w = 0; w < DEC_WARPS; ++w) {
                const float4 x = *reinterpret_cast<const float4*>(meet + (w * ROWS + col) * D + d);
                v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
                l += ex2(ref_s[w][col] - top) * sum_s[w][col];
            }
            if (whole) {
                write(col, d, v, l);
            } else {
                __stcg(reinterpret_cast<float4*>(part + col * D + d), v);
                if (d == 0) { __stcg(part + ROWS * D + col, top); __stcg(part + ROWS * (D + 1) + col, l); }
            }
        }
        if (!whole) {
            // ---- the parts of an item that spans blocks ----
            __threadfence();
            warps_sync();
            if (threadIdx.x == 0) {
                const unsigned n = (unsigned)(it.b_last - it.b_first + 1);
                const unsigned seen = atomicAdd(&p.tickets[it.b_first], 1u);
                last_s = seen + 1 == n;
                if (seen + 1 == n) p.tickets[it.b_first] = 0;
                __threadfence();
            }
            warps_sync();
            if (last_s) {
                for (int i = threadIdx.x; i < cols * (D / 4); i += DEC_WARPS * 32) {
                    const int col = i / (D / 4), d = i % (D / 4) * 4;
                    float top = kNone, l = 0.0f;
                    float4 v = make_float4(0, 0, 0, 0);
#pragma unroll 8
                    for (int b = it.b_first; b <= it.b_last; ++b) {
                        const float* src = p.parts + ((size_t)b * 2 + (b == it.b_first ? 1 : 0)) * PART;
                        const float t = __ldcg(src + ROWS * D + col), ls = __ldcg(src + ROWS * (D + 1) + col);
                        const float4 x = __ldcg(reinterpret_cast<const float4*>(src + col * D + d));
                        const float nt = fmaxf(top, t);
                        const float fa = ex2(top - nt), fb = ex2(t - nt);
                        v.x = v.x * fa + x.x * fb; v.y = v.y * fa + x.y * fb;
                        v.z = v.z * fa + x.z * fb; v.w = v.w * fa + x.w * fb;
                        l = l * fa + ls * fb;
                        top = nt;
                    }
                    write(col, d, v, l);
                }
            }
        }
        if (lane == 0) mbar_arrive(&item_empty[q_at]);
        if (++q_at == DEC_QUEUE) { q_at = 0; q_phase ^= 1; }
    }
    if (!ok && lane == 0) atomicOr(p.status, KV4_DEV_TIMEOUT);
}

template <int D, int NT, int STAGES>
constexpr size_t smem_bytes() { return 128 + (size_t)DEC_WARPS * STAGES * 20 * D + sizeof(float) * DEC_WARPS * 8 * NT * D; }

template <int D, int NT, int STAGES>
tsvd_status_t launch(const DecParams& p, int blocks, cudaStream_t st)
{
    PdlLaunch l((unsigned)blocks, DEC_THREADS, smem_bytes<D, NT, STAGES>(), st);
    TSVD_CUDA_OK(cudaLaunchKernelEx(&l.cfg, kv4_decode_kernel<D, NT, STAGES>, p));
    tsvd_count_launch();
    return TSVD_OK;
}

template <int D, int NT, int STAGES>
cudaError_t prepare()
{
    return cudaFuncSetAttribute(kv4_decode_kernel<D, NT, STAGES>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D, NT, STAGES>());
}

constexpr int kRowsMost = 16;      // rows of an item: 8 or 16

}  // namespace

size_t kv4_decode_parts_bytes(int sms, int dim) { return sizeof(float) * (size_t)(2 * sms) * 2 * kRowsMost * (dim + 2); }
size_t kv4_decode_tickets(int sms) { return (size_t)(2 * sms); }

tsvd_status_t kv4_decode_prepare()
{
    TSVD_CUDA_OK((prepare<128, 1, 4>()));
    TSVD_CUDA_OK((prepare<64, 1, 8>()));
    TSVD_CUDA_OK((prepare<128, 2, 8>()));
    TSVD_CUDA_OK((prepare<64, 2, 8>()));
    return TSVD_OK;
}

tsvd_status_t kv4_attend_decode(const AttendArgs& a)
{
    DecParams p{};
    p.g = a.h->g;
    p.b = a.b;
    p.q = (const __nv_bfloat16*)a.q;
    p.ldq = a.ldq;
    p.out = (__nv_bfloat16*)a.out;
    p.ldo = a.ldo;
    p.group = a.n_heads / a.h->g.heads;
    p.max_q = a.max_q;
    // (a scale of 0 is a tiny one: hidden positions become -inf through the product with it)
    p.c = fabsf(a.scale) < 1e-18f ? 1e-18f : a.scale * 1.4426950408889634f;
    p.window = a.window;
    p.causal = a.causal;
    p.min_share = 16;
    p.parts = a.h->parts;
    p.tickets = a.h->tickets;
    p.status = a.h->dev_status;
    const long long rows = (long long)a.max_q * p.group;
    const bool two = rows > 8;
    const long long items = (long long)a.b.n_seq * p.g.heads * ((rows + (two ? 15 : 7)) / (two ? 16 : 8));
    const long long most = items * (((long long)a.max_kv + KV4_BLOCK - 1) / KV4_BLOCK + 1);
    const long long blocks = std::min((long long)a.h->sms * (two ? 1 : 2), (most + p.min_share - 1) / p.min_share);
    if (p.g.dim == 128)
        return two ? launch<128, 2, 8>(p, (int)blocks, a.stream) : launch<128, 1, 4>(p, (int)blocks, a.stream);
    return two ? launch<64, 2, 8>(p, (int)blocks, a.stream) : launch<64, 1, 8>(p, (int)blocks, a.stream);
}
