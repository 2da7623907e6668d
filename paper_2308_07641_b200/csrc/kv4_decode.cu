// Attention over the 4-bit cache for few query rows (single tokens, short pieces): bound by streaming the cache.
//
//     out = sum_j p_j v_j / sum_j p_j,   p_j = exp2(c q.k_j - ref),   c = scale log2(e)
//
// Work.  An item is (sequence, key/value head, group of 8 NT query rows: the heads that share the key/value head, of one
// or several tokens); its unit is two blocks of 16 cached positions.  All units of the call, item after item, are cut into
// equal runs, one for each warp of a persistent grid, so ragged batches and single long sequences spread alike, and no warp
// waits for another until its run is done.  Each warp keeps a ring of units in shared memory that it fills by bulk copies,
// ahead across item borders.  A warp writes the items that lie in its run; of one that reaches beyond it, at either end, it
// keeps its part.  At the end the block adds its warps' parts; what still lacks other blocks' parts goes to scratch, and the
// block that finishes last adds those in their order (so results do not depend on it).  Few short items get a block each
// instead, which saves that last step.
//
// Arithmetic.  mma.sync m16n8k16 in fp16 with fp32 sums, the cached side as the 16-row operand, the query rows as the
// 8-column one.  Scores use the codes as they are: two masks leave pairs of them in the low bits of a word, which is what fp16
// calls code * 2^-24, or 16 code * 2^-24 for the odd nibbles, whose q is divided by 16 beforehand; the group's step is applied
// to the fp32 sum.  The bases' part, sum over groups of base * (sum of q), is one more small product with the sums of q in
// two fp16 terms.  So scores carry no rounding of k at all.  q enters as fp16 after division by a power of two per row (a bf16
// number is exact down to 2^-23 of the row's largest, and off by at most 2^-31 of it below).  Values become fp16 numbers
// code * step + base (one rounding); probabilities fp16, relative to a reference that moves only when a score passes the one
// it was set by by more than 5 (in units of log2): no exchange between lanes otherwise.  Both roundings are what the fp16
// operands of the second product cost: 2^-11 of a term at most, up or down, where the result's own to bf16 is 2^-8; the
// sum of probabilities is taken before their rounding.  Error against 64 bits 0.0017 of the results' size, 0.0016 to 0.0017
// for fp32 throughout with the same last rounding.
//
// Measured: 32 sequences of 32 heads on 8, 174 MB of cache, 56 us = 3.1 TB/s (floor 27); one sequence of 100003 positions, 128 MB,
// 40 us = 3.2 TB/s (floor 20); one short sequence of 12 heads 8.8 us.  What bounds the long ones is instructions and their
// latency, not the copies: issue slots 48% busy with three warps a scheduler, 1057 clocks a unit and scheduler, of which turning the
// values' codes into fp16 is the largest share; some 4 us pass before the first unit and 4 to 8 after the last (the parts'
// exchange).  Warps that only convert, feeding others, were slower (they were the bottleneck), as were 16 warps (80 us).
//
// A window beside first positions that stay visible (SINKS: kernels of their own, so that the others keep their code) makes an
// item's units those of the first positions and then the window's, counted as one run, with one step of the copies over what lies
// between; pages of hidden positions are not looked at.  32 sequences of 32 heads on 8 behind up to 20000 positions, window 4096 and 4 first
// ones, 50 us (floor 23.5), bound as above.
#include <algorithm>

#include "serving.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace ptx;

constexpr int DEC_MAX_STAGES = 6;
constexpr int DEC_QUEUE = 8;             // items that the copies may be ahead: more than DEC_MAX_STAGES
// Units a warp up to which items get a block each: a step over scratch costs as much.  8 sequences of 8 heads: 600 positions 11.1
// us apart, 15.5 in equal runs; 1500 positions 15.9 and 17.7; 3000 25.5 and 22.1; 2 sequences, 4000: 32 and 16.
constexpr int DEC_APART = 6;
constexpr int DEC_STATIC = 13 * 1024;    // room for what the kernel declares
// Warps of a block: 12 of up to 168 registers a thread for eight rows (8 of 255: 46 -> 42 us for 100003 positions), 8 for sixteen
// rows, whose sums need more.
template <int NT> constexpr int kWarps = NT == 1 ? 12 : 8;
constexpr int DEC_UNIT = 2 * KV4_BLOCK;  // positions of a unit

// Probabilities are 2^(score - reference): 2^10 where the reference was set, up to 2^15 before it moves, so that fp16
// reaches down to 2^-35 of it.
constexpr float kSet = 10.0f, kMove = 15.0f;
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
    int sinks;           // (with SINKS) first positions that the window does not hide
    int test_stall;      // test hook: no unit is ever copied, so the waits must give up
    int stages;          // units of a warp's ring
    int keep_cols;       // query rows of an item that can hold anything: what is kept of a part
    float* parts;        // [grid][2][rows][D + 2]
    unsigned* tickets;   // [grid]
    int* status;
    int sms;
};

// (x & mask) | 0x64006400 in one instruction
__device__ __forceinline__ uint32_t lop_or(uint32_t x, uint32_t mask)
{
    uint32_t y;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(y) : "r"(x), "r"(mask), "r"(0x64006400u));
    return y;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_k8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0)
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(b0));
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

template <int WORDS>
struct alignas(4 * WORDS) Words { uint32_t w[WORDS]; };

// What one sequence brings.
struct Seq {
    int rows, len, first, items, unit0, units;  // units of one item; unit0: its first, counted from position 0
    int all;                                    // its rows, those beyond max_q (which are not computed) included
    int front;                                  // (SINKS) units 0 .. front-1 are the cache's first; unit u >= front is its unit0 + u
    int lo;                                     // (SINKS) positions from `sinks` up to it are seen by no row
};

template <int ROWS, bool SINKS>
__device__ __forceinline__ Seq load_seq(const DecParams& p, int s)
{
    Seq q{0, 0, 0, 0, 0, 0, 0, 0, 0};
    if (s >= p.b.n_seq) return q;
    q.first = kv4_first_row(p.b, s);
    q.all = kv4_first_row(p.b, s + 1) - q.first;
    q.len = p.b.seq_len[s];
    q.rows = min(min(q.all, p.max_q), p.b.n_rows - q.first);
    if (q.rows <= 0 || q.first < 0) { q.rows = q.units = 0; return q; }
    const long long room = (long long)p.b.max_pages * p.g.page_tokens;
    const long long seen = q.len < 0 ? 0 : min((long long)q.len, room);
    if (q.len > room) atomicOr(p.status, KV4_DEV_INDEX);
    long long lo = 0, hi = seen;
    const long long pos0 = (long long)q.len - q.all;          // of the first row
    if (p.window) lo = max(0LL, pos0 - p.window + 1);
    if (p.causal) hi = min(hi, pos0 + q.rows);
    q.items = p.g.heads * ((q.rows * p.group + ROWS - 1) / ROWS);
    if constexpr (SINKS) {
        // what lies between the first positions and the window is left out, where that is a unit or more
        const long long front = (min((long long)p.sinks, hi) + DEC_UNIT - 1) / DEC_UNIT, ends = (hi + DEC_UNIT - 1) / DEC_UNIT;
        const long long from = min(lo / DEC_UNIT, ends);
        if (front < from) {
            q.front = (int)front;
            q.unit0 = (int)(from - front);
        }
        q.units = max(1, (int)ends - q.unit0);
        q.lo = (int)lo;
        return q;
    }
    q.unit0 = (int)(lo / DEC_UNIT);
    q.units = hi > lo ? (int)((hi + DEC_UNIT - 1) / DEC_UNIT) - q.unit0 : 1;   // an item that sees nothing still writes zeros
    return q;
}

// A warp's share of an item.
struct Item {
    int first_row, n_rows;     // of the call; (row, head) pairs of the item's sequence and head in all
    int head, row0;            // the pairs row0 .. are this item's
    int len, pos0;             // positions that can be seen at all; position of the sequence's first row
    int at0, unit0, unit1, units;    // position of its unit 0; units [unit0, unit1) of `units` are the warp's
    int front;                 // (SINKS) units below it count from position 0
    long long u0;              // where the item begins in the call's list of units
};

// How the call's units are shared out to the blocks.
struct Runs {
    long long total;
    int blocks, share;         // share: of a block, where items lie apart
    __device__ __forceinline__ long long first_of(int b) const
    {
        if (share) return (long long)share * b;
        if (b >= blocks) return total;
        return total < (1LL << 31) / 1024 ? (long long)((unsigned)total * (unsigned)b / (unsigned)blocks) : total * b / blocks;   // (blocks <= 1024)
    }
    __device__ __forceinline__ int block_of(long long u) const
    {
        return share ? (int)(u / share) : (int)(((u + 1) * blocks - 1) / total);
    }
};

// The run behind a warp's copies (what changes with every unit is in registers).
struct Feed {
    int s, item, page_at;
    Seq q;
    long long item_u0, run_u0, u1;
};

template <int D, int NT, bool SINKS>
__global__ void __launch_bounds__(kWarps<NT> * 32, 1)
kv4_decode_kernel(const DecParams p)
{
    constexpr int WARPS = kWarps<NT>;
    constexpr int ROWS = 8 * NT, W = D / KV4_GROUP, BLOCK = 20 * D, UNIT = 2 * BLOCK;
    constexpr int VW = D / 64;   // words of value codes per thread and key
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 127) & ~(uintptr_t)127);
    float* heads_kept = reinterpret_cast<float*>(ring + (size_t)WARPS * p.stages * UNIT);   // [warps][keep_cols][D]
    __shared__ uint64_t full[WARPS][DEC_MAX_STAGES];
    __shared__ Item queue[WARPS][DEC_QUEUE];
    __shared__ Feed feeds[WARPS];
    // What a warp keeps of an item that began before its run (0; the numbers in heads_kept) or ends after it (1; the numbers
    // in the warp's own ring, which is then idle).
    __shared__ float kept_ref[2][WARPS][ROWS], kept_sum[2][WARPS][ROWS];
    __shared__ Item kept[2][WARPS];
    __shared__ int ctl_[2];
    volatile int* ctl = ctl_;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, j = lane & 3;

    if (threadIdx.x == 0) { ctl[0] = 0; ctl[1] = p.test_stall ? kWaitLimitStall : kWaitLimitDefault; }
    if (threadIdx.x < WARPS) {
        for (int i = 0; i < p.stages; ++i) mbar_init(&full[threadIdx.x][i], 1);
        kept[0][threadIdx.x].units = kept[1][threadIdx.x].units = 0;
        fence_mbar_init();
    }
    __syncthreads();
    pdl_launch_dependents();
    pdl_wait();

    // ---- the warp's run of units ----
    long long total = 0;
    int total_items = 0, most = 0;
    Seq mine = load_seq<ROWS, SINKS>(p, lane);
    for (int s0 = 0;; mine = load_seq<ROWS, SINKS>(p, s0 + lane)) {
        total += (long long)mine.items * mine.units;
        total_items += mine.items;
        most = max(most, mine.units);
        s0 += 32;
        if (s0 >= p.b.n_seq) break;
    }
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    total_items = __reduce_add_sync(0xffffffffu, total_items);
    most = __reduce_max_sync(0xffffffffu, most);
    // Block b has the units from share * b on where items lie apart, else from total * b / blocks on; warps likewise in it.
    const bool apart = total_items <= (int)gridDim.x && most <= DEC_APART * WARPS;
    const int share = apart ? (most + WARPS - 1) / WARPS * WARPS : 0;
    if (apart) total = (long long)share * total_items;         // a block's share for each item, whatever its length
    // (no more blocks than have units for all their warps: a block without units would be waited for)
    const Runs runs{total, apart ? (int)gridDim.x : (int)min((long long)gridDim.x, max(1LL, total / WARPS)), share};
    Feed& f = feeds[warp];
    {
        const long long c0 = runs.first_of(blockIdx.x), c1 = min(runs.first_of(blockIdx.x + 1), total);
        const unsigned n = c1 > c0 ? (unsigned)(c1 - c0) : 0;
        // the first n % WARPS warps have one more: where there are fewer units than warps, the last ones have none
        const unsigned each = n / WARPS, over = n % WARPS;
        const long long u0 = c0 + each * (unsigned)warp + min((unsigned)warp, over), u1 = u0 + each + ((unsigned)warp < over);
        long long before = 0;
        if (p.b.n_seq > 32) mine = load_seq<ROWS, SINKS>(p, lane);
        if (u0 < u1)
            for (int s0 = 0; s0 < p.b.n_seq; mine = load_seq<ROWS, SINKS>(p, s0 + lane)) {
                const int span = apart ? share : mine.units;
                const long long have = (long long)mine.items * span;
                long long scan = have;
                for (int o = 1; o < 32; o <<= 1) {
                    const long long v = __shfl_up_sync(0xffffffffu, scan, o);
                    if (lane >= o) scan += v;
                }
                const unsigned holds = __ballot_sync(0xffffffffu, before + scan > u0);
                if (holds) {
                    if (lane == __ffs(holds) - 1) {
                        const unsigned in = (unsigned)(u0 - before - (scan - have));
                        f.s = s0 + lane;
                        f.item = (int)(in / (unsigned)span) - 1;          // the step to the first item adds one
                        f.q = mine;
                        f.item_u0 = u0 - in % (unsigned)span - span;
                    }
                    break;
                }
                before += __shfl_sync(0xffffffffu, scan, 31);
                s0 += 32;
            }
        __syncwarp();
        if (lane == 0) {
            f.u1 = u1;
            f.run_u0 = u0;
            if (u0 >= u1) { f.u1 = f.item_u0 = 0; f.q.units = 0; }   // nothing to do
        }
        __syncwarp();
    }
    const int per_page = p.g.page_tokens / KV4_BLOCK;
    // The whole warp moves along the run together; one lane writes and copies.
    const uint8_t* ptr = nullptr;        // the next block, null where its page number is out of range
    int in_page = 0, in_item = 0;        // blocks left in the page, units left in the warp's share of the item
    int next_page = 0, pushed = 0;       // a page number is asked for one page ahead
    int to_front = -1;                   // (SINKS) units left before the step over what the window hides
    uint32_t there = 0;                  // two bits a slot: which of its blocks are in range
    auto ask_page = [&](int at) {        // -2: no such position, or (SINKS) none that is seen
        if (SINKS && (long long)at * p.g.page_tokens >= p.sinks && (long long)(at + 1) * p.g.page_tokens <= f.q.lo) return -2;
        return at < p.b.max_pages && (long long)at * p.g.page_tokens < f.q.len ? p.b.table[(long long)f.s * p.b.max_pages + at] : -2;
    };
    auto open_page = [&](int page, int in) {
        ptr = nullptr;
        if (page >= 0 && page < p.g.n_pages) ptr = p.g.block(page, f.item % p.g.heads, in * KV4_BLOCK);
        else if (page != -2 && lane == 0) atomicOr(p.status, KV4_DEV_INDEX);
        in_page = per_page - in;
        next_page = ask_page(f.page_at + 1);
    };
    auto turn_page = [&]() {
        __syncwarp();
        if (lane == 0) ++f.page_at;
        __syncwarp();
        open_page(next_page, 0);
    };
    auto next_item = [&]() -> bool {     // false: the run is done
        __syncwarp();
        if (lane == 0) {
            const int span = apart ? share : f.q.units;
            f.item_u0 += span;
            if (f.item_u0 < f.u1 && ++f.item == f.q.items) {
                f.item = 0;
                do f.q = load_seq<ROWS, SINKS>(p, ++f.s); while (f.q.items == 0 && f.s < p.b.n_seq);
                if (f.q.items == 0) f.u1 = 0;                  // only if the lengths changed meanwhile
            }
        }
        __syncwarp();
        const long long run_u0 = f.run_u0, item_u0 = f.item_u0, u1 = f.u1;
        const int unit0 = (int)max(0LL, run_u0 - item_u0), unit1 = (int)min((long long)f.q.units, u1 - item_u0);
        if (item_u0 >= u1 || unit0 >= unit1) return false;     // (unit0 >= unit1: an item apart, shorter than the block's share)
        const int blk = (SINKS && unit0 < f.q.front ? unit0 : f.q.unit0 + unit0) * 2;
        if (lane == 0) {
            Item& it = queue[warp][pushed % DEC_QUEUE];
            it.first_row = f.q.first;
            it.n_rows = f.q.rows * p.group;
            it.head = f.item % p.g.heads;
            it.row0 = f.item / p.g.heads * ROWS;
            it.len = (int)max(0LL, min((long long)f.q.len, (long long)p.b.max_pages * p.g.page_tokens));
            it.pos0 = f.q.len - f.q.all;
            it.at0 = f.q.unit0 * DEC_UNIT;
            it.unit0 = unit0;
            it.unit1 = unit1;
            it.units = f.q.units;
            if constexpr (SINKS) it.front = f.q.front;
            it.u0 = item_u0;
            f.page_at = blk / per_page;
        }
        __syncwarp();
        ++pushed;
        in_item = unit1 - unit0;
        if constexpr (SINKS) to_front = unit0 < f.q.front ? f.q.front - unit0 : -1;
        open_page(ask_page(blk / per_page), blk % per_page);
        return true;
    };
    bool more = true;
    // The next unit of the run into slot `st`.  What is out of range is replaced by the pool's first block (its numbers are
    // finite) and hidden.
    auto feed = [&](int st) {
        if (!more || (in_item == 0 && !(more = next_item()))) return;
        if (SINKS && to_front-- == 0) {
            const int blk = (f.q.unit0 + f.q.front) * 2;
            __syncwarp();
            if (lane == 0) f.page_at = blk / per_page;
            __syncwarp();
            open_page(ask_page(blk / per_page), blk % per_page);
        }
        if (in_page == 0) turn_page();
        const uint8_t *a = ptr, *b;
        const bool joined = in_page >= 2;
        if (joined) {
            b = ptr ? ptr + BLOCK : nullptr;
            in_page -= 2;
        } else {
            turn_page();
            b = ptr;
            --in_page;
        }
        ptr = b ? b + BLOCK : nullptr;
        --in_item;
        there = (there & ~(3u << (2 * st))) | (uint32_t)((a ? 1 : 0) | (b ? 2 : 0)) << (2 * st);
        if (lane == 0 && !p.test_stall) {
            uint8_t* to = ring + (size_t)(warp * p.stages + st) * UNIT;
            mbar_arrive_expect_tx(&full[warp][st], UNIT);
            if (joined && a) {
                bulk_g2s(to, a, UNIT, &full[warp][st]);
            } else {
                bulk_g2s(to, a ? a : p.g.pool, BLOCK, &full[warp][st]);
                bulk_g2s(to + BLOCK, b ? b : p.g.pool, BLOCK, &full[warp][st]);
            }
        }
    };
    // An item's query rows: column r of each group of eight, numbers 32 w + 8 j .. + 7.
    auto ask_q = [&](const Item& it, uint4 (&x)[NT][W]) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int row = it.row0 + 8 * t + r;
            const __nv_bfloat16* src = nullptr;
            if (row < it.n_rows) src = p.q + (long long)(it.first_row + row / p.group) * p.ldq + (long long)(it.head * p.group + row % p.group) * D;
#pragma unroll
            for (int w = 0; w < W; ++w) x[t][w] = src ? *reinterpret_cast<const uint4*>(src + 32 * w + 8 * j) : make_uint4(0, 0, 0, 0);
        }
    };
    // (the first item's before any copy: behind the copies of all warps they took 3 us)
    uint4 qx[NT][W];
    more = next_item();
    if (more) ask_q(queue[warp][0], qx);
    for (int i = 0; i < p.stages; ++i) feed(i);
    __syncwarp();

    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int popped = 0; popped < pushed; ++popped) {
        const Item it = queue[warp][popped % DEC_QUEUE];

        // ---- the item's query rows ----
        if (popped > 0) ask_q(it, qx);
        uint32_t qf[NT][2 * W][2];           // [..][MMA step][word]: column r
        uint32_t qs[NT];                     // column r: the sum of q over group j, in two fp16 terms
        float cmul[NT][2];                   // columns 2 j, 2 j + 1
        int lo[NT][2], hi[NT][2];            // positions [lo, hi) that those columns see
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float v[W][8];
            float top = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const uint4 x = qx[t][w];
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
            // divide by the power of two at or below the row's largest (2^-60 at least), times 2^10
            const int e = min(max((int)(__float_as_uint(top) >> 23), 67), 253) - 127;
            const float down = __uint_as_float((uint32_t)(137 - e) << 23);
            float ss[W];
#pragma unroll
            for (int w = 0; w < W; ++w) {
                ss[w] = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {      // pairs (2 i, 2 i + 1): odd i hold q / 16
                    const float f = (i & 1) ? down * 0.0625f : down, back = (i & 1) ? 0x1p-6f : 0x1p-10f;
                    const uint32_t pr = h2(v[w][2 * i] * f, v[w][2 * i + 1] * f);
                    qf[t][2 * w + (i >> 1)][i & 1] = pr;
                    const float2 as = halves(pr);
                    ss[w] = fmaf(back, as.x + as.y, ss[w]);
                }
                ss[w] += __shfl_xor_sync(0xffffffffu, ss[w], 1);
                ss[w] += __shfl_xor_sync(0xffffffffu, ss[w], 2);
            }
            float mine_s = 0.0f;                   // group j's
#pragma unroll
            for (int w = 0; w < W; ++w) mine_s = j == w ? ss[w] : mine_s;
            const float hi_s = __half2float(__float2half_rn(mine_s));
            qs[t] = h2(hi_s, mine_s - hi_s);
            const float up = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                cmul[t][k] = p.c * __shfl_sync(0xffffffffu, up, 4 * (2 * j + k));
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
        for (int u = it.unit0; u < it.unit1; ++u) {
            if (!(ok = mbar_wait_warp(&full[warp][stage], phase, ctl))) break;
            const uint8_t* unit = ring + (size_t)(warp * p.stages + stage) * UNIT;
            const int at = (SINKS && u < it.front ? 0 : it.at0) + u * DEC_UNIT, here = (int)(there >> (2 * stage) & 3u);
            // rows r and r + 8 of a block's score tile are its positions kr and kr + 8
            const int kr = (r >> 1) + 4 * (r & 1);
            float sc[2][NT][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint8_t* blk = unit + h * BLOCK;
                Words<W> kw[2], ks[2];
                uint32_t kb[2];                    // (step, base) of group j
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    kw[x] = *reinterpret_cast<const Words<W>*>(blk + (kr + 8 * x) * (D / 2) + j * 4 * W);
                    ks[x] = *reinterpret_cast<const Words<W>*>(blk + 8 * D + (kr + 8 * x) * (D / 8));
                    kb[x] = *reinterpret_cast<const uint32_t*>(blk + 8 * D + (kr + 8 * x) * (D / 8) + (j & (W - 1)) * 4);
                }
                float part[NT][4];
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const uint32_t x0 = kw[0].w[w], x1 = kw[1].w[w], y0 = x0 >> 8, y1 = x1 >> 8;
                    const uint32_t a[8] = {x0 & 0x000f000fu, x1 & 0x000f000fu, x0 & 0x00f000f0u, x1 & 0x00f000f0u,
                                           y0 & 0x000f000fu, y1 & 0x000f000fu, y0 & 0x00f000f0u, y1 & 0x00f000f0u};
                    const float s0 = halves(ks[0].w[w]).x, s1 = halves(ks[1].w[w]).x;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        mma_f16(d, a[0], a[1], a[2], a[3], qf[t][2 * w][0], qf[t][2 * w][1]);
                        mma_f16(d, a[4], a[5], a[6], a[7], qf[t][2 * w + 1][0], qf[t][2 * w + 1][1]);
#pragma unroll
                        for (int k = 0; k < 4; ++k) part[t][k] = w ? fmaf(k < 2 ? s0 : s1, d[k], part[t][k]) : (k < 2 ? s0 : s1) * d[k];
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    mma_f16_k8(d, __byte_perm(kb[0], 0, 0x3232), __byte_perm(kb[1], 0, 0x3232), qs[t]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) sc[h][t][k] = fmaf(part[t][k], 16384.0f, d[k]);      // 2^(24 - 10)
                }
            }
            if ((at < all_lo && (!SINKS || at + DEC_UNIT > p.sinks)) || at + DEC_UNIT > all_hi || here != 3) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int pos = at + h * KV4_BLOCK + kr + (k & 2 ? 8 : 0);
                            // hidden whatever the scale's sign: the product below has to be -inf
                            if ((pos < lo[t][k & 1] && (!SINKS || pos >= p.sinks)) || pos >= hi[t][k & 1] || !(here >> h & 1)) sc[h][t][k] = cmul[t][k & 1] < 0.0f ? INFINITY : -INFINITY;
                        }
            }
            float e[2][NT][4];
            bool over = false;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        e[h][t][k] = fmaf(sc[h][t][k], cmul[t][k & 1], -ref[t][k & 1]);
                        over |= e[h][t][k] > kMove;
                    }
            if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float x[4] = {sc[0][t][k] * cmul[t][k], sc[0][t][k + 2] * cmul[t][k], sc[1][t][k] * cmul[t][k], sc[1][t][k + 2] * cmul[t][k]};
                        float m = fmaxf(fmaxf(ref[t][k] + kSet, fmaxf(x[0], x[1])), fmaxf(x[2], x[3]));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16)) - kSet;
                        const float keep = ex2(ref[t][k] - m);       // 0 before the first score
                        ref[t][k] = m;
                        sum[t][k] *= keep;
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) { o[t][i][k] *= keep; o[t][i][k + 2] *= keep; }
                        e[0][t][k] = x[0] - m;
                        e[0][t][k + 2] = x[1] - m;
                        e[1][t][k] = x[2] - m;
                        e[1][t][k + 2] = x[3] - m;
                    }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint8_t* blk = unit + h * BLOCK;
                uint32_t pb[NT][2];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) e[h][t][k] = ex2(e[h][t][k]);
                    sum[t][0] += e[h][t][0] + e[h][t][2];
                    sum[t][1] += e[h][t][1] + e[h][t][3];
                    pb[t][0] = transpose8(h2(e[h][t][0], e[h][t][1]));
                    pb[t][1] = transpose8(h2(e[h][t][2], e[h][t][3]));
                }
                // values: this thread's key pairs (j, j + 4) and (j + 8, j + 12), numbers D/8 r .. of each
                const uint8_t* vb = blk + 10 * D;
                Words<VW> vw[4];
                uint32_t vs[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    vw[x] = *reinterpret_cast<const Words<VW>*>(vb + (j + 4 * x) * (D / 2) + r * 4 * VW);
                    vs[x] = *reinterpret_cast<const uint32_t*>(blk + 18 * D + (j + 4 * x) * (D / 8) + (r * W / 8) * 4);
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
            feed(stage);
            __syncwarp();
            if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;

        // ---- write it, or keep it ----
        const int which = it.unit0 > 0 ? 0 : 1;                // began before the run: 0
        const bool whole = it.unit0 == 0 && it.unit1 == it.units;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float l = sum[t][k];
                l += __shfl_xor_sync(0xffffffffu, l, 4);
                l += __shfl_xor_sync(0xffffffffu, l, 8);
                l += __shfl_xor_sync(0xffffffffu, l, 16);
                const int col = 8 * t + 2 * j + k, row = it.row0 + col;
                if (row >= it.n_rows) continue;
                if (whole) {
                    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                    __nv_bfloat16* to = p.out + (long long)(it.first_row + row / p.group) * p.ldo +
                                        (long long)(it.head * p.group + row % p.group) * D + (D / 8) * r;
#pragma unroll
                    for (int i = 0; i < D / 16; i += 4) {
                        uint32_t w[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) {          // tile i: numbers 2 i and the next
                            const __nv_bfloat162 b = __floats2bfloat162_rn(o[t][i + x][k] * inv, o[t][i + x][k + 2] * inv);
                            w[x] = *reinterpret_cast<const uint32_t*>(&b);
                        }
                        *reinterpret_cast<uint4*>(to + 2 * i) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                } else {
                    float* to = which ? reinterpret_cast<float*>(ring + (size_t)warp * p.stages * UNIT) : heads_kept + (size_t)warp * p.keep_cols * D;
                    to += col * D + (D / 8) * r;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) *reinterpret_cast<float2*>(to + 2 * i) = make_float2(o[t][i][k], o[t][i][k + 2]);
                    if (r == 0) { kept_ref[which][warp][col] = ref[t][k]; kept_sum[which][warp][col] = l; }
                }
            }
        if (!whole && lane == 0) kept[which][warp] = it;
    }
    if (!ok) {
        // a wait gave up: the warp's copies in flight are waited for (with a limit)
        if (lane == 0) atomicOr(p.status, KV4_DEV_TIMEOUT);
        for (int i = 0; i < p.stages; ++i) mbar_drain(&full[warp][i], i < stage ? phase ^ 1 : phase);
    }

    // ================= the block's parts: chains of warps that share an item =================
    __syncthreads();
    constexpr int THREADS = WARPS * 32, PART = ROWS * (D + 2);
    // In the order of the units: warp 0's part of an item from before (-1), then each warp's item that ends after it (its
    // number), with the parts of the warps that follow.  At most two of them lack other blocks' parts: the first and the last.
    struct Open { int chain, b_first, b_last; };
    __shared__ Open open_s[2];
    __shared__ unsigned last_s[2];
    const unsigned chains = __ballot_sync(0xffffffffu, lane <= WARPS && kept[lane ? 1 : 0][lane ? min(lane, WARPS) - 1 : 0].units != 0);
    if (chains == 0) return;
    auto write = [&](const Item& it, int col, int d, float4 v, float l) {
        const int row = it.row0 + col;
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        __nv_bfloat162 x = __floats2bfloat162_rn(v.x * inv, v.y * inv), y = __floats2bfloat162_rn(v.z * inv, v.w * inv);
        *reinterpret_cast<uint2*>(p.out + (long long)(it.first_row + row / p.group) * p.ldo + (long long)(it.head * p.group + row % p.group) * D + d) =
            make_uint2(*reinterpret_cast<uint32_t*>(&x), *reinterpret_cast<uint32_t*>(&y));
    };
    int open = 0;
    for (unsigned rest = chains; rest; rest &= rest - 1) {
        const int a = __ffs(rest) - 2, from = max(a, 0);
        const bool starts = a >= 0;
        const Item& it = kept[starts][from];
        int to = from;                                         // the last warp of the chain
        bool ends = it.unit1 == it.units;
        while (!ends && to + 1 < WARPS && kept[0][to + 1].units != 0) {
            ++to;
            ends = kept[0][to].unit1 == kept[0][to].units;
        }
        const int cols = min(ROWS, it.n_rows - it.row0);
        const bool whole = starts && ends;
        float* part = p.parts + ((size_t)blockIdx.x * 2 + (starts ? 1 : 0)) * PART;
        for (int i = threadIdx.x; i < cols * (D / 4); i += THREADS) {
            const int col = i / (D / 4), d = i % (D / 4) * 4;
            float top = kNone, l = 0.0f;
            float4 v = make_float4(0, 0, 0, 0);
            for (int w = from; w <= to; ++w) top = fmaxf(top, kept_ref[starts && w == from][w][col]);
            for (int w = from; w <= to; ++w) {
                const bool own = starts && w == from;
                const float* src = own ? reinterpret_cast<const float*>(ring + (size_t)w * p.stages * UNIT) : heads_kept + (size_t)w * p.keep_cols * D;
                const float4 x = *reinterpret_cast<const float4*>(src + col * D + d);
                const float f = ex2(kept_ref[own][w][col] - top);
                v.x = fmaf(x.x, f, v.x); v.y = fmaf(x.y, f, v.y); v.z = fmaf(x.z, f, v.z); v.w = fmaf(x.w, f, v.w);
                l = fmaf(kept_sum[own][w][col], f, l);
            }
            if (whole) {
                write(it, col, d, v, l);
            } else {
                __stcg(reinterpret_cast<float4*>(part + col * D + d), v);
                if (d == 0) { __stcg(part + ROWS * D + col, top); __stcg(part + ROWS * (D + 1) + col, l); }
            }
        }
        if (!whole) {
            if (threadIdx.x == 0) open_s[open] = Open{a, runs.block_of(it.u0), runs.block_of(it.u0 + it.units - 1)};
            ++open;
        }
    }
    if (open == 0) return;
    __threadfence();
    __syncthreads();
    if ((int)threadIdx.x < open) {
        const Open o = open_s[threadIdx.x];
        const unsigned seen = atomicAdd(&p.tickets[o.b_first], 1u) + 1, n = (unsigned)(o.b_last - o.b_first + 1);
        last_s[threadIdx.x] = seen == n;
        if (seen == n) p.tickets[o.b_first] = 0;
        __threadfence();
    }
    __syncthreads();
    for (int k = 0; k < open; ++k) {
        if (!last_s[k]) continue;
        // this block's part was the last
        const Open o = open_s[k];
        const Item& it = kept[o.chain >= 0][max(o.chain, 0)];
        const int cols = min(ROWS, it.n_rows - it.row0), parts = o.b_last - o.b_first + 1;
        // Each number's parts are dealt to `deal` threads, which load eight at a time, references and sums beside them, and meet
        // in the (idle) ring: what counts here is how many loads follow one another, 1 to 2 us each.
        const int numbers = cols * (D / 4), deal = max(1, THREADS / numbers);
        float4* met = reinterpret_cast<float4*>(ring);
        float2* met_tl = reinterpret_cast<float2*>(met + deal * numbers);
        if (k) __syncthreads();
        for (int i = threadIdx.x; i < deal * numbers; i += THREADS) {
            const int g = i / numbers, n = i - g * numbers, col = n / (D / 4), d = n % (D / 4) * 4;
            float top = kNone, l = 0.0f;
            float4 v = make_float4(0, 0, 0, 0);
            const float* src = p.parts + (size_t)o.b_first * 2 * PART;
            for (int b0 = g; b0 < parts; b0 += 8 * deal) {
                float4 x[8];
                float t[8], ls[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int b = b0 + e * deal;
                    const float* at = src + (size_t)(2 * b + (b == 0 ? 1 : 0)) * PART;
                    x[e] = make_float4(0, 0, 0, 0);
                    t[e] = kNone;
                    ls[e] = 0.0f;
                    if (b < parts) {
                        x[e] = __ldcg(reinterpret_cast<const float4*>(at + col * D + d));
                        t[e] = __ldcg(at + ROWS * D + col);
                        ls[e] = __ldcg(at + ROWS * (D + 1) + col);
                    }
                }
                float high = top;
#pragma unroll
                for (int e = 0; e < 8; ++e) high = fmaxf(high, t[e]);
                const float keep = ex2(top - high);
                top = high;
                v.x *= keep; v.y *= keep; v.z *= keep; v.w *= keep;
                l *= keep;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float f = ex2(t[e] - top);
                    v.x = fmaf(x[e].x, f, v.x); v.y = fmaf(x[e].y, f, v.y); v.z = fmaf(x[e].z, f, v.z); v.w = fmaf(x[e].w, f, v.w);
                    l = fmaf(ls[e], f, l);
                }
            }
            met[i] = v;
            met_tl[i] = make_float2(top, l);
        }
        __syncthreads();
        for (int n = threadIdx.x; n < numbers; n += THREADS) {
            float top = kNone, l = 0.0f;
            for (int g = 0; g < deal; ++g) top = fmaxf(top, met_tl[g * numbers + n].x);
            float4 v = make_float4(0, 0, 0, 0);
            for (int g = 0; g < deal; ++g) {
                const float4 x = met[g * numbers + n];
                const float2 tl = met_tl[g * numbers + n];
                const float f = ex2(tl.x - top);
                v.x = fmaf(x.x, f, v.x); v.y = fmaf(x.y, f, v.y); v.z = fmaf(x.z, f, v.z); v.w = fmaf(x.w, f, v.w);
                l = fmaf(tl.y, f, l);
            }
            write(it, n / (D / 4), n % (D / 4) * 4, v, l);
        }
    }
}

template <int D, int NT, bool SINKS>
tsvd_status_t launch(DecParams p, long long items, long long units_most, cudaStream_t st)
{
    constexpr size_t kRoom = 227 * 1024 - DEC_STATIC;          // beside what the kernel declares itself
    const size_t kept = sizeof(float) * kWarps<NT> * p.keep_cols * D;
    const size_t unit = (size_t)kWarps<NT> * 40 * D;
    p.stages = (int)std::min<size_t>(DEC_MAX_STAGES, (kRoom - 128 - kept) / unit);
    const long long blocks = std::min((long long)p.sms, std::max(items, (units_most + kWarps<NT> - 1) / kWarps<NT>));
    PdlLaunch l((unsigned)blocks, kWarps<NT> * 32, 128 + kept + p.stages * unit, st);
    TSVD_CUDA_OK(cudaLaunchKernelEx(&l.cfg, kv4_decode_kernel<D, NT, SINKS>, p));
    tsvd_count_launch();
    return TSVD_OK;
}

template <bool SINKS>
tsvd_status_t launch_dim(const DecParams& p, bool two, long long items, long long most, cudaStream_t st)
{
    if (p.g.dim == 128) return two ? launch<128, 2, SINKS>(p, items, most, st) : launch<128, 1, SINKS>(p, items, most, st);
    return two ? launch<64, 2, SINKS>(p, items, most, st) : launch<64, 1, SINKS>(p, items, most, st);
}

constexpr int kRowsMost = 16;      // rows of an item: 8 or 16

}  // namespace

size_t kv4_decode_parts_bytes(int sms, int dim) { return sizeof(float) * (size_t)sms * 2 * kRowsMost * (dim + 2); }
size_t kv4_decode_tickets(int sms) { return (size_t)sms; }

tsvd_status_t kv4_decode_prepare()
{
    const int most = 227 * 1024 - DEC_STATIC;
    for (const void* kernel : {(const void*)kv4_decode_kernel<128, 1, false>, (const void*)kv4_decode_kernel<64, 1, false>,
                               (const void*)kv4_decode_kernel<128, 2, false>, (const void*)kv4_decode_kernel<64, 2, false>,
                               (const void*)kv4_decode_kernel<128, 1, true>, (const void*)kv4_decode_kernel<64, 1, true>,
                               (const void*)kv4_decode_kernel<128, 2, true>, (const void*)kv4_decode_kernel<64, 2, true>})
        TSVD_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
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
    p.sinks = a.sinks;
    p.causal = a.causal;
    p.test_stall = a.test_stall;
    p.parts = a.h->parts;
    p.tickets = a.h->tickets;
    p.status = a.h->dev_status;
    p.sms = a.h->sms;
    const long long rows = (long long)a.max_q * p.group;
    const bool two = rows > 8;
    p.keep_cols = (int)std::min<long long>(rows, two ? 16 : 8);
    const long long items = (long long)a.b.n_seq * p.g.heads * ((rows + (two ? 15 : 7)) / (two ? 16 : 8));
    const long long most = items * (((long long)a.max_kv + DEC_UNIT - 1) / DEC_UNIT + 1);
    return a.sinks ? launch_dim<true>(p, two, items, most, a.stream) : launch_dim<false>(p, two, items, most, a.stream);
}
