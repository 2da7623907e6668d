// Attention over the 4-bit cache for many query rows (prompts, and pieces of prompts behind earlier context): bound by the
// tensor cores and the exponentials.
//
//     out = sum_j p_j v_j / sum_j p_j,   p_j = exp2(c q.k_j - ref),   c = scale log2(e)
//
// A block takes up to two tiles of 128 query rows of one sequence and key/value head -- (token, head) pairs of the heads
// that share it -- and walks over tiles of 128 cached positions:
//   warp 13     copies the packed positions into shared memory, keys and values in turn
//   warps 8-11  turn codes into fp16 numbers, code * step + base, in the order the tensor cores read (keys with head_dim
//               contiguous, values likewise: the second product takes them as an MN-major operand, so nothing is transposed)
//   warp 12     issues tcgen05.mma: scores S = Q K^T into tensor memory, then O += P V with P from tensor memory
//   warps 0-3 and 4-7, one row a thread: running maximum, exponentials, P as fp16 over S's own columns, the sum
// A step is 64 positions.  Each row tile has two score buffers: the scores of the next step are formed while a step's
// exponentials run, so a row never waits for a product.  A row's reference moves
// only when a score passes the one it was set by by more than 5 (log2), so that O, which stays in tensor memory, is seldom rescaled.
//
// Measured: a prompt of 2048 tokens, 32 heads of 128: 52 us, 34.4 GFLOP (floor 20.6 us), tensor pipe 33% of the active cycles; seven
// pieces of 16 heads of 64 on 4, 27 us.  A step of 64 positions and 256 rows takes some 1900 clocks, of which the products
// need 1024 (4096 multiplications a clock) and the exponentials 1024 (16 a clock an SM), with two row warps a scheduler to hide
// each other's latency; a block starts for 3.8 us (64 KB of q at what an SM takes in, its conversion, the first scores) and
// ends for 2.  Of the prompt's 91 K active clocks an SM, 31 steps take 59 K (30 K of them with the tensor pipe busy), the starts
// and ends of two blocks 22 K, and the rest is blocks of unlike length in two rounds.  Tried and slower:
// fetching the next step's scores into a second register set (67 us), a cubic for a quarter of the exponentials (59 -> 65),
// persistent blocks whose copies run ahead into the next pair (57: the row loop needs more registers and a step takes 2300).
// With one row tile alone the codes bound it, 2 us per 128 positions: both groups of row warps on one tile gained nothing.
//
// With first positions beside a window (SINKS, kernels of their own) a block walks over the tiles of both as one run, and each row tile
// leaves out the steps that only the other one's window holds: a prompt of 4096 tokens, 32 heads of 128, window 1024 and 16 first ones
// 118 us (floor 39; 512 blocks on 148 SMs are 3.5 rounds of 3.8 us of start and 2 of end); seven pieces of 16 heads of 64 on 4, 32 us.
//
// Arithmetic: q as fp16 times a power of two for each row that brings its largest number to 2^15 (a bf16 number is then exact
// down to 2^-32 of it; the power goes into the row's factor c), keys and values as fp16 (one rounding), probabilities as fp16,
// sums in fp32 (that of the probabilities before their rounding).  The roundings, 2^-11 of a term at most, are what fp16
// operands of the tensor cores cost; the result's own to bf16 is 2^-8.  Error against 64 bits 0.0017 of the results' size,
// 0.0016 to 0.0017 for fp32 throughout with the same last rounding.
#include <algorithm>

#include "serving.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace ptx;

constexpr int PRE_THREADS = 14 * 32;
constexpr int PRE_ROWS = 128;            // rows of a tile
constexpr int PRE_KEYS = 128;            // positions of a tile
constexpr int PRE_STEP = 64;             // positions of a step: half a tile
constexpr int PRE_HIDE = 8;              // tiles whose hidden blocks are remembered: more than any copy can be ahead
// Probabilities are 2^(score - reference): 2^10 where the reference was set, up to 2^15 before it moves, so that fp16
// reaches down to 2^-35 of it.
constexpr float kSet = 10.0f, kMove = 15.0f;
constexpr float kNone = -1e30f;

struct PreParams {
    Kv4Geom g;
    Kv4Batch b;
    const __nv_bfloat16* q;
    long long ldq;
    __nv_bfloat16* out;
    long long ldo;
    int group, max_q;
    int tiles;               // pairs of row tiles of a sequence and head
    float c;
    float sign;              // of the scale: goes into q
    int window, causal;
    int sinks;               // (with SINKS) first positions that the window does not hide
    int test_stall;          // test hook: no position is ever copied, so the waits must give up
    int splits;              // blocks that share a pair's positions; above 1 they leave their parts in `parts`
    float* parts;            // [block][2 * PRE_ROWS][D] sums, [2 * PRE_ROWS] (reference, sum)
    int* status;
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t lop_or(uint32_t x, uint32_t mask)
{
    uint32_t y;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(y) : "r"(x), "r"(mask), "r"(0x64006400u));
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
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
// two at once: (a, b) * m + c, and a sum
__device__ __forceinline__ float2 fma2(float2 a, float2 m, float2 c)
{
    float2 y;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<unsigned long long&>(y))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(m)), "l"(reinterpret_cast<unsigned long long&>(c)));
    return y;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 y;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long&>(y))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return y;
}
// Eight numbers of a group from their codes: pairs in order, step and base in both halves.
__device__ __forceinline__ uint4 numbers(uint32_t x, uint32_t step, uint32_t base)
{
    constexpr uint32_t kOne = 0x3c003c00u, kMinus1024 = 0xe400e400u, kSixteenth = 0x2c002c00u, kMinus64 = 0xd400d400u;
    const uint32_t y = x >> 8;
    uint4 v;
    v.x = hfma(hfma(lop_or(x, 0x000f000fu), kOne, kMinus1024), step, base);
    v.y = hfma(hfma(lop_or(x, 0x00f000f0u), kSixteenth, kMinus64), step, base);
    v.z = hfma(hfma(lop_or(y, 0x000f000fu), kOne, kMinus1024), step, base);
    v.w = hfma(hfma(lop_or(y, 0x00f000f0u), kSixteenth, kMinus64), step, base);
    return v;
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
          "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
          "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// kind::f16, both operands fp16, fp32 sums; B_MN: the N x K operand has N contiguous.
__host__ __device__ constexpr uint32_t idesc_f16(int m, int n, bool b_mn)
{
    return (1u << 4) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// MN-major operand, 128-byte swizzle: rows of 64 numbers (one k each), eight rows a 1 KiB group, 64 numbers to the next
// `apart` bytes later.
__device__ __forceinline__ uint64_t umma_desc_mn_sw128(uint32_t smem_addr, uint32_t apart)
{
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(apart >> 4) << 16;
    d |= (uint64_t)(1024u >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
__device__ __forceinline__ void umma_f16_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
__device__ __forceinline__ void umma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}

// Sixteen bytes, or zeros.  Volatile: a row's loads go out together, one behind the other (left to the compiler, the prompt took
// 58 us in place of 53).
__device__ __forceinline__ uint4 ld_or_zero(const void* at, bool there)
{
    uint4 v;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.u32 p, %5, 0;\n\t"
        "mov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\tmov.u32 %2, 0;\n\tmov.u32 %3, 0;\n\t"
        "@p ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
        : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
        : "l"(at), "r"((uint32_t)there)
        : "memory");
    return v;
}
template <int WORDS>
struct alignas(4 * WORDS) Words { uint32_t w[WORDS]; };

// Shared memory (1024-aligned): Q [2 tiles][D/64][128 rows][128 B] | K [2][D/64][128][128 B] | V [2][D/64][128][128 B] |
// packed halves [STAGES][8 blocks][10 D bytes]
template <int D>
struct Layout {
    static constexpr int kHalves = D / 64;
    static constexpr int kTile = kHalves * 16384;
    static constexpr int kPacked = 8 * 10 * D;              // keys or values of a tile of positions
    static constexpr int kStages = D == 128 ? 3 : 6;
    static constexpr int kQ = 0, kK = 2 * kTile, kV = 4 * kTile, kStg = 6 * kTile;
    static constexpr int kBytes = kStg + kStages * kPacked;
};

template <int D, bool SINKS>
__global__ void __launch_bounds__(PRE_THREADS, 1)
kv4_prefill_kernel(const PreParams p)
{
    using L = Layout<D>;
    constexpr int W = D / KV4_GROUP;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    __shared__ uint64_t stg_full[L::kStages], stg_empty[L::kStages], k_full[2], k_empty[2], v_full[2], v_empty[2], q_full, s_full[2][2], p_full[2][2],
        o_done[2][2], drained;
    __shared__ uint32_t tmem_slot;
    __shared__ uint8_t hidden[PRE_HIDE];
    __shared__ int2 row_at[2][PRE_ROWS];      // its row of the call and first number there; -1: none
    __shared__ int ctl_[2];
    volatile int* ctl = ctl_;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kStages; ++i) { mbar_init(&stg_full[i], 8); mbar_init(&stg_empty[i], 4); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&k_full[i], 4);
            mbar_init(&k_empty[i], 1);
            mbar_init(&v_full[i], 4);
            mbar_init(&v_empty[i], 1);
            for (int h = 0; h < 2; ++h) { mbar_init(&s_full[i][h], 1); mbar_init(&p_full[i][h], 4); mbar_init(&o_done[i][h], 1); }
        }
        mbar_init(&q_full, 8);
        mbar_init(&drained, 1);
        ctl[0] = 0;
        ctl[1] = p.test_stall ? kWaitLimitStall : kWaitLimitDefault;
        fence_mbar_init();
    }
    // Tensor memory before the kernel after this one may start (see PdlLaunch).
    if (warp == 12) { tmem_alloc(&tmem_slot, 512); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;                        // S or P of tile x, buffer h: column 128 x + 64 h; O: column 256 + 128 x
    // ---- which rows: pairs of tiles with the most positions first ----
    pdl_launch_dependents();
    pdl_wait();
    const int per = p.g.heads * p.b.n_seq;
    const int job = (int)blockIdx.x / p.splits, split = (int)blockIdx.x - job * p.splits;
    const int pair = p.tiles - 1 - job / per, rest = job % per;
    const int head = rest % p.g.heads, s = rest / p.g.heads;
    const int first = kv4_first_row(p.b, s), all = kv4_first_row(p.b, s + 1) - first;
    const int n_rows = max(0, first < 0 ? 0 : min(min(all, p.max_q), p.b.n_rows - first)) * p.group;
    const int row_base = pair * 2 * PRE_ROWS;
    const int len = p.b.seq_len[s];
    if (row_base >= n_rows) {
        if (warp == 12) tmem_dealloc(tmem, 512);
        return;
    }
    const long long room = (long long)p.b.max_pages * p.g.page_tokens;
    if (len > room && threadIdx.x == 0) atomicOr(p.status, KV4_DEV_INDEX);
    const int len_in = (int)max(0LL, min((long long)len, room));
    const int pos0 = len - all;                             // position of the sequence's first row
    auto token_hi = [&](int token) { return p.causal ? max(0, min(pos0 + token + 1, len_in)) : len_in; };
    auto token_lo = [&](int token) { return p.window ? max(0, pos0 + token - p.window + 1) : 0; };
    int t_lo[2], t_hi[2];                                   // steps [t_lo, t_hi) that each row tile sees
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int r0 = row_base + x * PRE_ROWS, r1 = min(r0 + PRE_ROWS, n_rows) - 1;
        t_lo[x] = t_hi[x] = 0;
        const int lo = token_lo(r0 / p.group), hi = token_hi(r1 / p.group);
        if (r1 >= r0 && hi > (SINKS ? 0 : lo)) {
            t_lo[x] = lo / PRE_STEP;
            t_hi[x] = (hi + PRE_STEP - 1) / PRE_STEP;
        }
    }
    // With first positions that stay visible, the pair's tiles [0, front) and those from its window's first on are counted as one
    // run: what is left out between them, `gap` tiles, is added where a tile becomes positions.  Steps from 2 front up to skip[x] of
    // that run are hidden from row tile x (the other one's window begins earlier): it leaves them out, an even number of them, so
    // that its steps go on taking turns at the two score buffers.
    int front = 0, gap = 0, skip[2] = {0, 0};
    if constexpr (SINKS) {
        const int ends = max(t_hi[0], t_hi[1]);
        int from = ends;
#pragma unroll
        for (int x = 0; x < 2; ++x)
            if (t_hi[x] > 0) from = min(from, t_lo[x]);
        front = (int)((min((long long)p.sinks, (long long)ends * PRE_STEP) + PRE_KEYS - 1) / PRE_KEYS);
        gap = max(0, from / 2 - front);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            skip[x] = t_hi[x] > 0 ? max(2 * front, min((t_lo[x] & ~1) - 2 * gap, t_hi[x] - 2 * gap & ~1)) : 2 * front;
            t_lo[x] = 0;
            t_hi[x] = min(t_hi[x], max(2 * front, t_hi[x] - 2 * gap));
        }
    }
    auto left_out = [&](int x, int k) { return SINKS && k >= 2 * front && k < (x ? skip[1] : skip[0]); };
    const bool one = t_hi[1] == t_lo[1], none = t_hi[0] == t_lo[0];
    const int j_lo = none ? t_lo[1] : one ? t_lo[0] : min(t_lo[0], t_lo[1]);
    int j_hi = none ? t_hi[1] : one ? t_hi[0] : max(t_hi[0], t_hi[1]);
    int k_lo = j_lo / 2, k_hi = (j_hi + 1) / 2;             // tiles
    if (p.splits > 1) {
        const int n = k_hi - k_lo, k0 = k_lo;
        k_lo = k0 + (int)((long long)n * split / p.splits);
        k_hi = k0 + (int)((long long)n * (split + 1) / p.splits);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            t_lo[x] = min(max(t_lo[x], 2 * k_lo), 2 * k_hi);
            t_hi[x] = max(min(t_hi[x], 2 * k_hi), t_lo[x]);
        }
        j_hi = max(t_hi[0], t_hi[1]);
        if (t_hi[0] == t_lo[0] && t_hi[1] == t_lo[1]) k_hi = k_lo;
    }
    if constexpr (SINKS) {
        // a share's steps neither begin nor end with ones that are left out
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (left_out(x, t_lo[x])) t_lo[x] = min(skip[x], t_hi[x]);
            if (t_hi[x] > t_lo[x] && left_out(x, t_hi[x] - 1)) t_hi[x] = max(2 * front, t_lo[x]);
        }
    }

    if (warp < 8) {
        // ================= rows: one a thread =================
        const int x = warp >> 2, r = threadIdx.x & 127, row = row_base + x * PRE_ROWS + r;
        const bool live = row < n_rows;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const int wrow = r & ~31;                           // the warp's first row of the tile
        const int token = row / p.group;
        row_at[x][r] = make_int2(live ? first + token : -1, (head * p.group + row - token * p.group) * D);
        __syncwarp();
        uint8_t* own = smem + L::kQ + x * L::kTile;
        float cm;
        {   // Q: the warp's 32 rows, read by D / 8 lanes a row; then each thread has its own row, and scales it by the power of two
            // that brings its largest number (2^-60 at least) to 2^15.
            constexpr int LANES = D / 8, ROWS = 32 / LANES;
            const int u = lane % LANES;
            uint4 v[LANES];
#pragma unroll
            for (int i = 0; i < LANES; ++i) {
                const int2 from = row_at[x][wrow + i * ROWS + lane / LANES];
                v[i] = ld_or_zero(p.q + max(from.x, 0) * p.ldq + from.y + 8 * u, from.x >= 0);
            }
#pragma unroll
            for (int i = 0; i < LANES; ++i) {
                const int rr = wrow + i * ROWS + lane / LANES;
                *reinterpret_cast<uint4*>(own + (u >> 3) * 16384 + rr * 128 + (((u & 7) ^ (rr & 7)) << 4)) = v[i];
            }
            __syncwarp();
            uint32_t top = 0;                               // magnitudes compared as 16-bit integers, two at a time
#pragma unroll
            for (int i = 0; i < LANES; ++i) {
                v[i] = *reinterpret_cast<const uint4*>(own + (i >> 3) * 16384 + r * 128 + (((i & 7) ^ (r & 7)) << 4));
                top = __vmaxu2(__vmaxu2(top, __vmaxu2(v[i].x & 0x7fff7fffu, v[i].y & 0x7fff7fffu)), __vmaxu2(v[i].z & 0x7fff7fffu, v[i].w & 0x7fff7fffu));
            }
            const int e = min(max((int)(max(top & 0xffffu, top >> 16) >> 7), 67), 254) - 127;
            const float by = p.sign * __uint_as_float((uint32_t)(127 + 15 - e) << 23);
            cm = p.c * __uint_as_float((uint32_t)(127 - 15 + e) << 23);
#pragma unroll
            for (int i = 0; i < LANES; ++i) {
                const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                uint32_t h[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) h[k] = h2(__uint_as_float(w[k] << 16) * by, __uint_as_float(w[k] & 0xffff0000u) * by);
                *reinterpret_cast<uint4*>(own + (i >> 3) * 16384 + r * 128 + (((i & 7) ^ (r & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&q_full);
        }
        const int lo = live ? token_lo(token) : 0, hi = live ? token_hi(token) : 0x7fffffff;
        const int all_lo = __reduce_max_sync(0xffffffffu, lo), all_hi = __reduce_min_sync(0xffffffffu, hi);
        const uint32_t t_o = t_lane + 256u + 128u * x;
        float ref = kNone, sum = 0.0f;
        uint32_t pho = 0, phs = 0;                          // of o_done and of s_full (bit h: odd steps have barriers of their own)
        bool ok = true;
        const int a = x ? t_lo[1] : t_lo[0], b = x ? t_hi[1] : t_hi[0];
        for (int k = a; k < b; ++k) {
            if (SINKS && left_out(x, k)) k = x ? skip[1] : skip[0];
            const int h = k & 1, at = (SINKS && k >= 2 * front ? k + 2 * gap : k) * PRE_STEP;
            ok = mbar_wait(&s_full[x][h], phs >> h & 1, ctl);   // (the warp agrees on it where it looks at `over`)
            phs ^= 1u << h;
            tc_fence_after_sync();
            const uint32_t t_s = t_lane + 128u * x + 64u * h;
            uint32_t v[2][32];
            tmem_ld32(t_s, v[0]);
            tmem_ld32(t_s + 32, v[1]);
            const uint32_t hide = hidden[(k >> 1) % PRE_HIDE] >> (4 * h) & 15;
            const bool edge = (at < all_lo && (!SINKS || at + PRE_STEP > p.sinks)) || at + PRE_STEP > all_hi || hide;
            tmem_ld_wait();
            if (edge) {
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int pos = at + 32 * c + i;
                        if ((pos < lo && (!SINKS || pos >= p.sinks)) || pos >= hi || (hide >> (2 * c + (i >> 4)) & 1)) v[c][i] = 0xff800000u;
                    }
            }
            float m[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t* w = v[c >> 1] + 16 * (c & 1);
                m[c] = fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
#pragma unroll
                for (int i = 2; i < 16; i += 2) m[c] = max3(m[c], __uint_as_float(w[i]), __uint_as_float(w[i + 1]));
            }
            const float top = fmaxf(max3(m[0], m[1], m[2]), m[3]) * cm;
            const bool over = top > ref + kMove;
            if (__any_sync(0xffffffffu, over || !ok)) {
                if (!(ok = __all_sync(0xffffffffu, ok))) break;
                const float to = over ? top - kSet : ref, keep = ex2(ref - to);    // 0 before the first score
                ref = to;
                sum *= keep;
                if (k > a) {
                    if (!(ok = mbar_wait_warp(&o_done[x][h ^ 1], (pho >> (h ^ 1) & 1) ^ 1, ctl))) break;   // the product of the step before
                    tc_fence_after_sync();
#pragma unroll 1
                    for (int c0 = 0; c0 < D; c0 += 16) {
                        uint32_t u[16];
                        tmem_ld16(t_o + c0, u);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(__uint_as_float(u[i]) * keep);
                        tmem_st16(t_o + c0, u);
                    }
                }
            }
            const float2 cm2 = make_float2(cm, cm), ref2 = make_float2(-ref, -ref);
            float2 s2[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float2 e = fma2(make_float2(__uint_as_float(v[c][2 * i]), __uint_as_float(v[c][2 * i + 1])), cm2, ref2);
                    e.x = ex2(e.x);
                    e.y = ex2(e.y);
                    s2[i & 1] = add2(s2[i & 1], e);
                    w[i] = h2(e.x, e.y);
                }
                tmem_st16(t_s + 16 * c, w);                  // over the scores, which have all been read
            }
            sum += (s2[0].x + s2[0].y) + (s2[1].x + s2[1].y);
            tmem_st_wait();
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full[x][h]);
            pho ^= 1u << h;
        }
        if (ok && b > a) ok = mbar_wait_warp(&o_done[x][(b - 1) & 1], (pho >> ((b - 1) & 1) & 1) ^ 1, ctl);
        tc_fence_after_sync();
        if (ok && p.splits > 1) {
            // Its part, unnormalised, through the tile's own Q as below, half of the numbers at a time.
            constexpr int LANES = D / 8, ROWS = 32 / LANES;
            uint8_t* mine = own + wrow * (2 * D);
            float* part = p.parts + (size_t)blockIdx.x * (2 * PRE_ROWS * (D + 2)) + (size_t)(x * PRE_ROWS + wrow) * D;
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int c0 = 0; c0 < D / 2; c0 += 32) {
                    uint32_t v[32] = {};
                    if (b > a) {
                        tmem_ld32(t_o + (uint32_t)(half * (D / 2) + c0), v);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        *reinterpret_cast<uint4*>(mine + lane * (2 * D) + ((((c0 + i) >> 2) ^ (lane & (LANES - 1))) << 4)) =
                            make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                }
                __syncwarp();
#pragma unroll
                for (int i = 0; i < LANES; ++i) {
                    const int rl = i * ROWS + lane / LANES, u = lane % LANES;
                    *reinterpret_cast<uint4*>(part + rl * D + half * (D / 2) + 4 * u) =
                        *reinterpret_cast<const uint4*>(mine + rl * (2 * D) + ((u ^ (rl & (LANES - 1))) << 4));
                }
                __syncwarp();
            }
            reinterpret_cast<float2*>(p.parts + (size_t)blockIdx.x * (2 * PRE_ROWS * (D + 2)) + 2 * PRE_ROWS * D)[x * PRE_ROWS + r] =
                make_float2(b > a ? ref : kNone, sum);
        } else if (ok) {
            const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
            // Through the tile's own Q, which the products are done with: the warp's 32 rows, 16 bytes of a row at unit
            // u ^ row, then D / 8 lanes a row.
            constexpr int LANES = D / 8, ROWS = 32 / LANES;
            uint8_t* mine = own + wrow * (2 * D);
#pragma unroll
            for (int c0 = 0; c0 < D; c0 += 32) {
                uint32_t v[32] = {};
                if (b > a) {
                    tmem_ld32(t_o + c0, v);
                    tmem_ld_wait();
                }
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    uint32_t w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const __nv_bfloat162 y = __floats2bfloat162_rn(__uint_as_float(v[i + 2 * k]) * inv, __uint_as_float(v[i + 2 * k + 1]) * inv);
                        w[k] = *reinterpret_cast<const uint32_t*>(&y);
                    }
                    *reinterpret_cast<uint4*>(mine + lane * (2 * D) + ((((c0 + i) >> 3) ^ (lane & (LANES - 1))) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < LANES; ++i) {
                const int rl = i * ROWS + lane / LANES, u = lane % LANES;
                const int2 at = row_at[x][wrow + rl];
                if (at.x >= 0)
                    *reinterpret_cast<uint4*>(p.out + at.x * p.ldo + at.y + 8 * u) =
                        *reinterpret_cast<const uint4*>(mine + rl * (2 * D) + ((u ^ (rl & (LANES - 1))) << 4));
            }
        }
        tc_fence_before_sync();
    } else if (warp < 12) {
        // ================= numbers from codes =================
        const int w4 = warp - 8, j = lane & 3, idx = lane >> 2;
        int st = 0;
        uint32_t sph = 0, ph[2] = {0, 0};                   // phases of the two stages
        bool ok = true;
        for (int k = k_lo; k < k_hi && ok; ++k) {
            const int buf = (k - k_lo) & 1;
            // keys: lane (position, j) has one word of every group; positions in the order 0 4 1 5 ... keep the stores apart
            if (!(ok = mbar_wait_warp(&stg_full[st], sph, ctl) && mbar_wait_warp(&k_empty[buf], ph[buf] ^ 1, ctl))) break;
            const uint8_t* src = smem + L::kStg + st * L::kPacked;
            uint8_t* dst = smem + L::kK + buf * L::kTile;
            const int kr = (idx >> 1) + 4 * (idx & 1);
            Words<W> code[4], sb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = i * 32 + w4 * 8 + kr, pos = key & 15;
                const uint8_t* blk = src + (key >> 4) * (10 * D);
                code[i] = *reinterpret_cast<const Words<W>*>(blk + pos * (D / 2) + j * 4 * W);
                sb[i] = *reinterpret_cast<const Words<W>*>(blk + 8 * D + pos * (D / 8));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = i * 32 + w4 * 8 + kr;
#pragma unroll
                for (int w = 0; w < W; ++w)
                    *reinterpret_cast<uint4*>(dst + (w >> 1) * 16384 + key * 128 + (((4 * (w & 1) + j) ^ (key & 7)) << 4)) =
                        numbers(code[i].w[w], __byte_perm(sb[i].w[w], 0, 0x1010), __byte_perm(sb[i].w[w], 0, 0x3232));
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) { mbar_arrive(&k_full[buf]); mbar_arrive(&stg_empty[st]); }
            if (++st == L::kStages) { st = 0; sph ^= 1; }
            // values: lane (position, j) has D / 4 consecutive numbers; the upper two quarters start elsewhere
            if (!(ok = mbar_wait_warp(&stg_full[st], sph, ctl) && mbar_wait_warp(&v_empty[buf], ph[buf] ^ 1, ctl))) break;
            src = smem + L::kStg + st * L::kPacked;
            dst = smem + L::kV + buf * L::kTile;
            const int turn = W == 4 ? j & 2 : 0;             // the words of a lane in the order n ^ turn
            uint32_t sv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = i * 32 + w4 * 8 + idx, pos = key & 15;
                const uint8_t* blk = src + (key >> 4) * (10 * D);
                code[i] = *reinterpret_cast<const Words<W>*>(blk + pos * (D / 2) + j * 4 * W);
                sv[i] = *reinterpret_cast<const uint32_t*>(blk + 8 * D + pos * (D / 8) + j * W / 4 * 4);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = i * 32 + w4 * 8 + idx;
                const uint32_t step = __byte_perm(sv[i], 0, 0x1010), base = __byte_perm(sv[i], 0, 0x3232);
                if constexpr (W == 4) {
                    if (turn) {
                        const uint32_t a0 = code[i].w[0], a1 = code[i].w[1];
                        code[i].w[0] = code[i].w[2]; code[i].w[1] = code[i].w[3];
                        code[i].w[2] = a0; code[i].w[3] = a1;
                    }
                }
#pragma unroll
                for (int n = 0; n < W; ++n) {                // numbers 8 W j + 8 (n ^ turn) ..
                    const int unit = W * j + (n ^ turn);
                    *reinterpret_cast<uint4*>(dst + (unit >> 3) * 16384 + key * 128 + (((unit & 7) ^ (key & 7)) << 4)) = numbers(code[i].w[n], step, base);
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) { mbar_arrive(&v_full[buf]); mbar_arrive(&stg_empty[st]); }
            if (++st == L::kStages) { st = 0; sph ^= 1; }
            ph[buf] ^= 1;
        }
    } else {
      if (warp == 12) {
        // ================= products =================
        if (elect_one() && k_hi > k_lo) {
            constexpr uint32_t kQk = idesc_f16(PRE_ROWS, PRE_STEP, false), kPv = idesc_f16(PRE_ROWS, D, true);
            const uint32_t base = smem_u32(smem);
            // Descriptors count addresses in 16 bytes, so that a step is one addition.
            const uint64_t desc_q = umma_desc_k_sw128(base + L::kQ), desc_k = umma_desc_k_sw128(base + L::kK), desc_v = umma_desc_mn_sw128(base + L::kV, 16384u);
            // step j of row tile x: half j & 1 of the tile of positions in stage (j / 2 - k_lo) & 1
            auto scores = [&](int x, int j) {
                const uint64_t q = desc_q + (uint32_t)(x * (L::kTile >> 4));
                const uint64_t keys = desc_k + (uint32_t)((((j >> 1) - k_lo) & 1) * (L::kTile >> 4) + (j & 1) * (PRE_STEP * 128 >> 4));
                const uint32_t to = tmem + 128u * x + 64u * (j & 1);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {           // 16 numbers at a time: 32 bytes of a 128-byte row
                    const uint32_t at = (uint32_t)((i >> 2) * (16384 >> 4) + (i & 3) * 2);
                    umma_f16_ss(to, q + at, keys + at, kQk, i > 0);
                }
                umma_commit(&s_full[x][j & 1]);
            };
            auto values = [&](int x, int j, bool more) {
                const uint64_t vals = desc_v + (uint32_t)((((j >> 1) - k_lo) & 1) * (L::kTile >> 4) + (j & 1) * (PRE_STEP * 128 >> 4));
                const uint32_t to = tmem + 256u + 128u * x, probs = tmem + 128u * x + 64u * (j & 1);
#pragma unroll
                for (int i = 0; i < PRE_STEP / 16; ++i)      // 16 positions at a time: 16 rows of values, 8 columns of P
                    umma_f16_ts(to, probs + 8u * i, vals + (uint32_t)(i * (2048 >> 4)), kPv, more || i > 0);
                umma_commit(&o_done[x][j & 1]);
            };
            bool ok = mbar_wait(&q_full, 0, ctl);
            uint32_t pph[2] = {0, 0};                        // phases of p_full (bit h)
            for (int j = 2 * k_lo - 1; j < j_hi && ok; ++j) {
                // the scores of the next step, then the values of this one
                const int n = j + 1;
                if (n < j_hi) {
                    if (!(n & 1) && !(ok = mbar_wait(&k_full[((n >> 1) - k_lo) & 1], (uint32_t)((n >> 1) - k_lo) >> 1 & 1, ctl))) break;
                    tc_fence_after_sync();
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (n >= t_lo[x] && n < t_hi[x] && !left_out(x, n)) scores(x, n);
                    if (n & 1) umma_commit(&k_empty[((n >> 1) - k_lo) & 1]);
                }
                if (j < 2 * k_lo) continue;
                if (!(j & 1) && !(ok = mbar_wait(&v_full[((j >> 1) - k_lo) & 1], (uint32_t)((j >> 1) - k_lo) >> 1 & 1, ctl))) break;
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (j >= t_lo[x] && j < t_hi[x] && !left_out(x, j)) {
                        if (!(ok = mbar_wait(&p_full[x][j & 1], pph[x] >> (j & 1) & 1, ctl))) break;
                        pph[x] ^= 1u << (j & 1);
                        tc_fence_after_sync();
                        values(x, j, j > t_lo[x]);
                    }
                if (!ok) break;
                if (j & 1) umma_commit(&v_empty[((j >> 1) - k_lo) & 1]);
            }
            // every product has ended before the block does
            umma_commit(&drained);
            mbar_drain(&drained, 0);
        }
        __syncwarp();
      } else if (warp == 13) {
        // ================= packed positions: lane i copies block i of a tile, keys and values in turn =================
        const int per_page = p.g.page_tokens / KV4_BLOCK;
        int st = 0;
        uint32_t ph = 0;
        bool ok = !p.test_stall;
        for (int k = k_lo; k < k_hi && ok; ++k) {
            const int blk = (SINKS && k >= front ? k + gap : k) * (PRE_KEYS / KV4_BLOCK) + (lane & 7);
            const uint8_t* src = nullptr;
            // (with SINKS, blocks that no row of the pair sees may lie in pages that are gone)
            const bool seen = !SINKS || (long long)blk * KV4_BLOCK < p.sinks || (long long)(blk + 1) * KV4_BLOCK > token_lo(row_base / p.group);
            if (seen && (long long)blk * KV4_BLOCK < len_in) {
                const int page = p.b.table[(long long)s * p.b.max_pages + blk / per_page];
                if (page >= 0 && page < p.g.n_pages) src = p.g.block(page, head, blk % per_page * KV4_BLOCK);
                else if (lane < 8) atomicOr(p.status, KV4_DEV_INDEX);
            }
            // what is out of range is replaced by the pool's first block (its numbers are finite) and hidden
            const uint32_t gone = __ballot_sync(0xffffffffu, src == nullptr) & 0xffu;
            if (!src) src = p.g.pool;
            for (int half = 0; half < 2 && ok; ++half) {
                ok = mbar_wait_warp(&stg_empty[st], ph ^ 1, ctl);
                if (ok && half == 0 && lane == 0) hidden[k % PRE_HIDE] = (uint8_t)gone;
                __syncwarp();
                if (ok && lane < 8) {
                    mbar_arrive_expect_tx(&stg_full[st], 10 * D);
                    bulk_g2s(smem + L::kStg + st * L::kPacked + lane * (10 * D), src + half * (10 * D), 10 * D, &stg_full[st]);
                }
                if (ok && ++st == L::kStages) { st = 0; ph ^= 1; }
            }
        }
        // where a wait gave up, copies in flight are waited for (with a limit)
        if (ctl[0])
            for (int i = 0; i < L::kStages; ++i) mbar_drain(&stg_full[i], i < st ? ph : ph ^ 1);
        __syncwarp();
      }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (threadIdx.x == 0 && ctl[0]) atomicOr(p.status, KV4_DEV_TIMEOUT);
    if (warp == 12) tmem_dealloc(tmem, 512);
}

// The parts of a pair's rows, in their order: D / 4 lanes a row, eight parts' loads side by side.
constexpr int JOIN_ROWS = 32;            // rows of a block
template <int D>
__global__ void __launch_bounds__(256)
kv4_join_kernel(const PreParams p)
{
    constexpr int LANES = D / 4, PART = 2 * PRE_ROWS * (D + 2);
    pdl_launch_dependents();
    pdl_wait();
    const int per = p.g.heads * p.b.n_seq, blocks_per_job = 2 * PRE_ROWS / JOIN_ROWS;
    const int job = (int)blockIdx.x / blocks_per_job, row_in0 = ((int)blockIdx.x - job * blocks_per_job) * JOIN_ROWS;
    const int pair = p.tiles - 1 - job / per, rest = job % per, head = rest % p.g.heads, s = rest / p.g.heads;
    const int first = kv4_first_row(p.b, s), all = kv4_first_row(p.b, s + 1) - first;
    const int n_rows = max(0, first < 0 ? 0 : min(min(all, p.max_q), p.b.n_rows - first)) * p.group;
    const int d = (int)(threadIdx.x % LANES) * 4;
    for (int r = (int)(threadIdx.x / LANES); r < JOIN_ROWS; r += 256 / LANES) {
        const int row_in = row_in0 + r, row = pair * 2 * PRE_ROWS + row_in;
        if (row >= n_rows) return;
        const float* src = p.parts + (size_t)job * p.splits * PART;
        float top = kNone, l = 0.0f;
        float4 v = make_float4(0, 0, 0, 0);
        for (int b0 = 0; b0 < p.splits; b0 += 8) {
            float4 y[8];
            float2 tl[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = make_float4(0, 0, 0, 0);
                tl[e] = make_float2(kNone, 0.0f);
                if (b0 + e < p.splits) {
                    const float* at = src + (size_t)(b0 + e) * PART;
                    y[e] = __ldcg(reinterpret_cast<const float4*>(at + row_in * D + d));
                    tl[e] = __ldcg(reinterpret_cast<const float2*>(at + 2 * PRE_ROWS * D) + row_in);
                }
            }
            float high = top;
#pragma unroll
            for (int e = 0; e < 8; ++e) high = fmaxf(high, tl[e].x);
            const float keep = ex2(top - high);
            top = high;
            v.x *= keep; v.y *= keep; v.z *= keep; v.w *= keep;
            l *= keep;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float f = ex2(tl[e].x - top);
                v.x = fmaf(y[e].x, f, v.x); v.y = fmaf(y[e].y, f, v.y); v.z = fmaf(y[e].z, f, v.z); v.w = fmaf(y[e].w, f, v.w);
                l = fmaf(tl[e].y, f, l);
            }
        }
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        const __nv_bfloat162 y0 = __floats2bfloat162_rn(v.x * inv, v.y * inv), y1 = __floats2bfloat162_rn(v.z * inv, v.w * inv);
        const int token = row / p.group;
        *reinterpret_cast<uint2*>(p.out + (long long)(first + token) * p.ldo + (long long)(head * p.group + row - token * p.group) * D + d) =
            make_uint2(*reinterpret_cast<const uint32_t*>(&y0), *reinterpret_cast<const uint32_t*>(&y1));
    }
}

template <int D, bool SINKS>
tsvd_status_t launch(const PreParams& p, cudaStream_t st)
{
    const long long blocks = (long long)p.tiles * p.g.heads * p.b.n_seq * p.splits;
    if (blocks > 0x7fffffffLL) return TSVD_E_TOOBIG;
    PdlLaunch l((unsigned)blocks, PRE_THREADS, Layout<D>::kBytes + 1024, st);
    TSVD_CUDA_OK(cudaLaunchKernelEx(&l.cfg, kv4_prefill_kernel<D, SINKS>, p));
    tsvd_count_launch();
    if (p.splits > 1) {
        PdlLaunch j((unsigned)(blocks / p.splits * (2 * PRE_ROWS / JOIN_ROWS)), 256, 0, st);
        TSVD_CUDA_OK(cudaLaunchKernelEx(&j.cfg, kv4_join_kernel<D>, p));
        tsvd_count_launch();
    }
    return TSVD_OK;
}

}  // namespace

size_t kv4_prefill_parts_bytes(int sms, int dim) { return sizeof(float) * (size_t)sms * 2 * PRE_ROWS * (dim + 2); }

tsvd_status_t kv4_prefill_prepare()
{
    for (const void* kernel : {(const void*)kv4_prefill_kernel<128, false>, (const void*)kv4_prefill_kernel<128, true>})
        TSVD_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<128>::kBytes + 1024));
    for (const void* kernel : {(const void*)kv4_prefill_kernel<64, false>, (const void*)kv4_prefill_kernel<64, true>})
        TSVD_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<64>::kBytes + 1024));
    return TSVD_OK;
}

tsvd_status_t kv4_attend_prefill(const AttendArgs& a)
{
    PreParams p{};
    p.g = a.h->g;
    p.b = a.b;
    p.q = (const __nv_bfloat16*)a.q;
    p.ldq = a.ldq;
    p.out = (__nv_bfloat16*)a.out;
    p.ldo = a.ldo;
    p.group = a.n_heads / a.h->g.heads;
    p.max_q = a.max_q;
    p.tiles = (int)(((long long)a.max_q * p.group + 2 * PRE_ROWS - 1) / (2 * PRE_ROWS));
    // (a scale of 0 is a tiny one: hidden positions become -inf through the product with it)
    p.c = std::max(fabsf(a.scale) * 1.4426950408889634f, 1e-18f);
    p.sign = a.scale < 0.0f ? -1.0f : 1.0f;
    p.window = a.window;
    p.sinks = a.sinks;
    p.causal = a.causal;
    p.test_stall = a.test_stall;
    p.status = a.h->dev_status;
    p.parts = a.h->parts;
    // Fewer pairs than half the SMs: blocks share a pair's positions, at least four tiles each (a tile takes about 2 us, the
    // step over scratch about 4).  64 rows of 8 heads after 32000 positions: 519 us in one block each, 58 shared; 40 rows of 32
    // heads after 1000 (two blocks): 22.1 and 22.2.
    const long long jobs = (long long)p.tiles * p.g.heads * p.b.n_seq;
    long long seen = a.max_kv;
    if (a.window) seen = std::min<long long>(seen, (long long)a.window + 2 * PRE_ROWS / p.group + 1 + a.sinks);
    p.splits = (int)std::max(1LL, std::min(a.h->sms / jobs, seen / (4 * PRE_KEYS)));
    if (a.sinks) return p.g.dim == 128 ? launch<128, true>(p, a.stream) : launch<64, true>(p, a.stream);
    return p.g.dim == 128 ? launch<128, false>(p, a.stream) : launch<64, false>(p, a.stream);
}
