// Low-rank adapters of many requests beside a shared projection:  out_i = base_i + c_s B_s (A_s x_i),  s the adapter of row i's
// sequence (A_s [rank, N], B_s [M, rank] in bf16).
//
// Two launches, the second a programmatic dependent of the first: z_i = A_s x_i (down), then out_i = base_i + c_s B_s z_i (up).
// Both walk over tiles of consecutive rows, whatever sequences they belong to, and inside a tile over the adapters that its
// rows ask for, each once; so one kernel serves single tokens with an adapter each, prompts of one adapter, and anything
// between.  A row's result depends on its own numbers and adapter only: what the products of an adapter give for rows of
// another one is dropped, never added.
//
// The weights lie in the order in which the lanes of a warp hand them to mma.sync m16n8k16, 16 bytes a lane, so that a lane
// copies (cp.async, some stages ahead) just what it will read, and nothing is exchanged between lanes.  What bounds both
// kernels is bytes: the adapters' for single tokens, x and base and out for prompts; the products are small beside them.
//
// Arithmetic: bf16 operands, fp32 sums.  8-bit x is exact in bf16.  fp32 x is cut into three bf16 terms that add up to it
// exactly.  z stays fp32 between the kernels, and enters the second product as two bf16 terms (2^-17 of it is lost, the result's
// own rounding being 2^-9) for bf16 results, as three (exactly) for fp32.  The parts of a contraction that blocks share are
// added in their order.
#include <new>
#include <vector>

#include "serving.cuh"

struct tsvd_adapters_s {
    int device = 0;
    int sms = 0;
    int N = 0, M = 0, max_rank = 0, n_slots = 0;
    int groups = 0;                  // of 16 ranks, of the largest rank
    int chunks = 0, blocks = 0;      // of 32 columns of A, of 64 channels of B
    size_t a_slot = 0, b_slot = 0;   // bytes of a slot
    uint8_t* A = nullptr;            // [slot][chunk][its groups][2][32 lanes][16]
    uint8_t* B = nullptr;            // [slot][block][its groups][4][32 lanes][16]
    int* ranks = nullptr;            // [slot], 0: empty
    float* scales = nullptr;         // [slot]
    float* z = nullptr;              // scratch: [split][row][16 * groups]
    size_t z_bytes = 0;
    std::vector<void*>* outgrown = nullptr;   // scratch that captured graphs may still use
    int* dev_status = nullptr;
};

namespace {

constexpr int GROUP = 16;        // ranks
constexpr int CHUNK = 32;        // columns of A that a lane's 32 bytes of a group reach over
constexpr int BLOCK = 64;        // channels of B that a warp takes at a time
constexpr int MAX_RANK = 128;
constexpr int DOWN_WARPS = 8, UP_WARPS = 4;
constexpr int UP_ROWS = 64;      // rows of a tile of the second kernel at most
constexpr int MAX_SPLITS = 32;

struct Rows {                    // which adapter a row has
    const int* slots;            // [n_seq]
    const int* q_start;          // [n_seq + 1] or null
    int n_seq, n_rows, n_slots;
    const int* ranks;
    int* status;
};

constexpr int kNoAdapter = -1, kNoRow = -2;

// The adapters of the rows row0 .. row0 + COUNT - 1, into shared memory: a slot, kNoAdapter or kNoRow.  The whole block.
template <int COUNT, int WARPS>
__device__ __forceinline__ void find_slots(const Rows& r, int row0, int* slot_s)
{
    constexpr int PER = (COUNT + WARPS - 1) / WARPS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = row0 + warp * PER;
    const int row = first + lane;
    int seq = row;
    if (r.q_start) {
        seq = 0;                 // sequences that end at or before the row
        if (warp * PER < COUNT) {
#pragma unroll 4
            for (int s0 = 0; s0 < r.n_seq; s0 += 32) {
                const int end = s0 + lane < r.n_seq ? r.q_start[s0 + lane + 1] : 0x7fffffff;
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int n = __popc(__ballot_sync(0xffffffffu, end <= first + i));
                    if (lane == i) seq += n;
                }
            }
        }
    }
    if (lane < PER && warp * PER + lane < COUNT) {
        int slot = kNoRow;
        if (row < r.n_rows && seq < r.n_seq && (!r.q_start || row >= r.q_start[0])) {
            slot = r.slots[seq];
            if (slot < -1 || slot >= r.n_slots) {
                atomicOr(r.status, KV4_DEV_INDEX);
                slot = kNoAdapter;
            }
            if (slot >= 0 && r.ranks[slot] == 0) slot = kNoAdapter;
        }
        slot_s[warp * PER + lane] = slot;
    }
    __syncthreads();
}

__device__ __forceinline__ void copy16(void* to, const void* from, int bytes = 16)      // what lacks to 16 becomes zeros
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy8(void* to, const void* from, int bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint4& a, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}

// The leading bf16 of two numbers, cut off (not rounded), as a pair; what remains of them is exact in fp32.
__device__ __forceinline__ uint32_t cut(float& lo, float& hi)
{
    const uint32_t a = __float_as_uint(lo), b = __float_as_uint(hi);
    lo -= __uint_as_float(a & 0xffff0000u);
    hi -= __uint_as_float(b & 0xffff0000u);
    return __byte_perm(a, b, 0x7632);
}
__device__ __forceinline__ uint32_t rounded(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// ---- weights ----------------------------------------------------------------------------------------------------------

template <typename T>
__device__ __forceinline__ uint32_t pair_of(const T* m, long long ld, int r, int c, int rows, int cols)      // (r, c), (r, c + 1)
{
    return rounded(r < rows && c < cols ? to_f32(m[r * ld + c]) : 0.0f, r < rows && c + 1 < cols ? to_f32(m[r * ld + c + 1]) : 0.0f);
}

// A slot's matrices into the order above; a thread writes 16 bytes.  Setup: bound by nothing that matters.
template <typename T>
__global__ void adapter_set_kernel(const T* A, long long lda, const T* B, long long ldb, int rank, int N, int M, int chunks, int blocks,
                                   uint4* a_out, uint4* b_out, int* rank_out, float* scale_out, float scale)
{
    const int groups = (rank + GROUP - 1) / GROUP;
    const long long na = (long long)chunks * groups * 64, nb = (long long)blocks * groups * 128;
    const long long step = (long long)gridDim.x * blockDim.x, first = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (first == 0) { *rank_out = rank; *scale_out = scale; }
    for (long long i = first; i < na + nb; i += step) {
        if (i < na) {
            const int lane = (int)(i & 31), half = (int)(i >> 5 & 1), g = lane >> 2, t = lane & 3;
            const long long piece = i >> 6;
            const int group = (int)(piece % groups), chunk = (int)(piece / groups);
            const int r = group * GROUP + g, c = chunk * CHUNK + 8 * t + 4 * half;
            a_out[i] = make_uint4(pair_of(A, lda, r, c, rank, N), pair_of(A, lda, r + 8, c, rank, N),
                                  pair_of(A, lda, r, c + 2, rank, N), pair_of(A, lda, r + 8, c + 2, rank, N));
        } else {
            const long long k = i - na;
            const int lane = (int)(k & 31), quarter = (int)(k >> 5 & 3), n = lane >> 2, t = lane & 3;
            const long long piece = k >> 7;
            const int group = (int)(piece % groups), block = (int)(piece / groups);
            // column n of product j is channel 16 (n / 2) + 2 j + n % 2: a lane's results are 16 channels in a row
            const int ch = block * BLOCK + 16 * (n >> 1) + 4 * quarter + (n & 1), r = group * GROUP + 4 * t;
            b_out[k] = make_uint4(pair_of(B, ldb, ch, r, M, rank), pair_of(B, ldb, ch, r + 2, M, rank),
                                  pair_of(B, ldb, ch + 2, r, M, rank), pair_of(B, ldb, ch + 2, r + 2, M, rank));
        }
    }
}

// ---- z = A x ------------------------------------------------------------------------------------------------------------

struct DownParams {
    Rows rows;
    const void* x;
    long long ldx;
    int aligned;             // rows may be copied 16 (8-bit: 8) bytes at a time
    int N, chunks, splits, groups;
    const uint8_t* A;
    size_t a_slot;
    float* z;
};

template <typename T> constexpr int kXBytes = 8 * (int)sizeof(T);    // of a lane: eight columns of a row
template <typename T, int NT, int RG> constexpr int kDownStage = RG * 1024 + NT * 32 * kXBytes<T>;
template <typename T, int NT, int RG> constexpr int kDownStages = 12 * 1024 / kDownStage<T, NT, RG> < 3 ? 3 : 12 * 1024 / kDownStage<T, NT, RG> > 8 ? 8 : 12 * 1024 / kDownStage<T, NT, RG>;

// Eight columns of a row as bf16 pairs: the terms of fp32 numbers one after another.
template <typename T> struct Terms;
template <> struct Terms<__nv_bfloat16> {
    static constexpr int n = 1;
    uint32_t w[1][4];
    __device__ __forceinline__ void read(const uint8_t* at)
    {
        const uint4 u = *reinterpret_cast<const uint4*>(at);
        w[0][0] = u.x; w[0][1] = u.y; w[0][2] = u.z; w[0][3] = u.w;
    }
};
template <> struct Terms<int8_t> {
    static constexpr int n = 1;
    uint32_t w[1][4];
    __device__ __forceinline__ void read(const uint8_t* at)
    {
        const uint2 u = *reinterpret_cast<const uint2*>(at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = (i < 2 ? u.x : u.y) >> (16 * (i & 1));
            w[0][i] = rounded((float)(int8_t)(v & 0xff), (float)(int8_t)(v >> 8 & 0xff));       // exact
        }
    }
};
template <> struct Terms<float> {
    static constexpr int n = 3;
    uint32_t w[3][4];
    __device__ __forceinline__ void read(const uint8_t* at)
    {
        // (the halves of a row's eight columns lie 512 bytes apart)
        const float4 a = *reinterpret_cast<const float4*>(at), b = *reinterpret_cast<const float4*>(at + 512);
        float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[0][i] = cut(v[2 * i], v[2 * i + 1]);
            w[1][i] = cut(v[2 * i], v[2 * i + 1]);
            w[2][i] = rounded(v[2 * i], v[2 * i + 1]);
        }
    }
};

// A block: 8 NT rows, a share of the columns; a warp every eighth chunk of 32 of them.  RG: groups of ranks at a time.
template <typename T, int NT, int RG>
__global__ void __launch_bounds__(DOWN_WARPS * 32)
adapter_down_kernel(const DownParams p)
{
    constexpr int ROWS = 8 * NT, STAGE = kDownStage<T, NT, RG>, STAGES = kDownStages<T, NT, RG>;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int slot_s[ROWS], entry_slot[ROWS], entry_groups[ROWS], entries_s;
    __shared__ unsigned entry_mask[ROWS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    // What the kernel ahead has written is there before the next kernel starts: that one reads it ahead of its own wait.
    pdl_wait();
    pdl_launch_dependents();
    const int row0 = blockIdx.x * ROWS, rank_pad = p.groups * GROUP;
    find_slots<ROWS, DOWN_WARPS>(p.rows, row0, slot_s);
    if (warp == 0) {
        const int slot = lane < ROWS ? slot_s[lane] : kNoRow;
        const unsigned same = __match_any_sync(0xffffffffu, slot);
        const bool leads = slot >= 0 && lane == __ffs(same) - 1;
        const unsigned leaders = __ballot_sync(0xffffffffu, leads);
        if (leads) {
            const int e = __popc(leaders & ((1u << lane) - 1));
            entry_slot[e] = slot;
            entry_mask[e] = same;
            entry_groups[e] = (p.rows.ranks[slot] + GROUP - 1) / GROUP;
        }
        if (lane == 0) entries_s = __popc(leaders);
    }
    __syncthreads();
    const int entries = entries_s;
    const int c0 = (int)((long long)p.chunks * blockIdx.y / p.splits), c1 = (int)((long long)p.chunks * (blockIdx.y + 1) / p.splits);
    uint8_t* ring = smem + (size_t)warp * STAGES * STAGE;
    float* parts = reinterpret_cast<float*>(smem + (size_t)DOWN_WARPS * STAGES * STAGE);     // [warp][row][rank_pad]

    // ---- the next item (adapter, groups, chunk) into a stage ----
    int fe = 0, fg = 0, fc = c0 + warp, fs = 0;
    auto fetch = [&]() {
        if (fe < entries && fc < c1) {
            uint8_t* to = ring + fs * STAGE;
            const int groups = entry_groups[fe], here = min(RG, groups - fg);
            const uint8_t* a = p.A + (size_t)entry_slot[fe] * p.a_slot + ((size_t)fc * groups + fg) * 1024 + lane * 16;
#pragma unroll
            for (int i = 0; i < 2 * RG; ++i)
                if (i < 2 * here) copy16(to + i * 512 + lane * 16, a + i * 512);
            const unsigned mask = entry_mask[fe];
            const int col = fc * CHUNK + 8 * t, left = p.N - col;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (!(mask >> (8 * n) & 0xffu)) continue;
                const int row = row0 + 8 * n + g;
                const bool there = row < p.rows.n_rows && left > 0;
                const T* x = (const T*)p.x + (there ? (long long)row * p.ldx + col : 0);
                uint8_t* dst = to + RG * 1024 + n * 32 * kXBytes<T>;
                const int have = there ? min(left, 8) * (int)sizeof(T) : 0;
                if (p.aligned) {
                    if constexpr (sizeof(T) == 1) {
                        copy8(dst + lane * 8, x, have);
                    } else {
#pragma unroll
                        for (int i = 0; i < kXBytes<T> / 16; ++i)
                            copy16(dst + i * 512 + lane * 16, have > 16 * i ? x + i * (16 / (int)sizeof(T)) : (const T*)p.x, max(0, min(16, have - 16 * i)));
                    }
                } else {
                    alignas(16) T v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = i * (int)sizeof(T) < have ? x[i] : T(0.0f);
                    if constexpr (sizeof(T) == 1) {
                        *reinterpret_cast<uint2*>(dst + lane * 8) = *reinterpret_cast<uint2*>(v);
                    } else {
#pragma unroll
                        for (int i = 0; i < kXBytes<T> / 16; ++i) *reinterpret_cast<uint4*>(dst + i * 512 + lane * 16) = reinterpret_cast<uint4*>(v)[i];
                    }
                }
            }
            fc += DOWN_WARPS;
            if (fc >= c1) {
                fc = c0 + warp;
                fg += RG;
                if (fg >= groups) { fg = 0; ++fe; }
            }
        }
        copies_commit();
        if (++fs == STAGES) fs = 0;
    };
    for (int i = 0; i < STAGES - 1; ++i) fetch();

    int stage = 0;
    if (c0 + warp < c1)
        for (int e = 0; e < entries; ++e) {
            const int groups = entry_groups[e];
            const unsigned mask = entry_mask[e];
            for (int g0 = 0; g0 < groups; g0 += RG) {
                const int here = min(RG, groups - g0);
                float acc[RG][NT][4];
#pragma unroll
                for (int i = 0; i < RG; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[i][n][k] = 0.0f;
                for (int c = c0 + warp; c < c1; c += DOWN_WARPS) {
                    copies_wait<STAGES - 2>();
                    const uint8_t* from = ring + stage * STAGE;
                    uint4 a[RG][2];
#pragma unroll
                    for (int i = 0; i < RG; ++i)
                        if (i < here) {
                            a[i][0] = *reinterpret_cast<const uint4*>(from + i * 1024 + lane * 16);
                            a[i][1] = *reinterpret_cast<const uint4*>(from + i * 1024 + 512 + lane * 16);
                        }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if (!(mask >> (8 * n) & 0xffu)) continue;
                        Terms<T> x;
                        x.read(from + RG * 1024 + n * 32 * kXBytes<T> + lane * (sizeof(T) == 1 ? 8 : 16));
#pragma unroll
                        for (int i = 0; i < RG; ++i)
                            if (i < here) {
#pragma unroll
                                for (int k = Terms<T>::n - 1; k >= 0; --k) {
                                    mma_bf16(acc[i][n], a[i][0], x.w[k][0], x.w[k][1]);
                                    mma_bf16(acc[i][n], a[i][1], x.w[k][2], x.w[k][3]);
                                }
                            }
                    }
                    fetch();
                    if (++stage == STAGES) stage = 0;
                }
                // rank g (+ 8) of rows 2 t and 2 t + 1 of each eight
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int row = 8 * n + 2 * t + (k & 1);
                        if (mask >> row & 1)
#pragma unroll
                            for (int i = 0; i < RG; ++i)
                                if (i < here) parts[(warp * ROWS + row) * rank_pad + (g0 + i) * GROUP + g + (k & 2 ? 8 : 0)] = acc[i][n][k];
                    }
            }
        }
    copies_wait<0>();
    __syncthreads();
    const int warps = min(DOWN_WARPS, c1 - c0);
    for (int i = threadIdx.x; i < ROWS * rank_pad; i += DOWN_WARPS * 32) {
        const int row = i / rank_pad, r = i - row * rank_pad, slot = slot_s[row];
        if (slot < 0 || r >= p.rows.ranks[slot]) continue;
        float sum = 0.0f;
        for (int w = 0; w < warps; ++w) sum += parts[w * ROWS * rank_pad + i];
        p.z[((size_t)blockIdx.y * p.rows.n_rows + row0 + row) * rank_pad + r] = sum;
    }
}

// ---- out = base + c B z ---------------------------------------------------------------------------------------------------

struct UpParams {
    Rows rows;
    const float* z;
    int splits, groups;
    const float* scales;     // [slot]
    const float* x_scale;    // [row] or null
    const void* base;        // null: zeros
    long long ldb;
    void* out;
    long long ldo;
    int vec;                 // rows of base and out on 16-byte boundaries
    int in_place;            // out is base: rows without an adapter are as they should be
    int M, blocks, per_warp; // per_warp: blocks of 64 channels that a warp takes
    int tile_rows;           // rows of a block of threads: at most UP_ROWS
    int stages;
    const uint8_t* B;
    size_t b_slot;
};

template <typename T> constexpr int kTerms = sizeof(T) == 2 ? 2 : 3;

// Sixteen channels of a row, in the row's type.
template <typename T> struct Piece {
    static constexpr int U = (int)sizeof(T);         // 16-byte units
    uint4 u[U];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < U; ++i) u[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void load(const T* at, int left, bool vec)
    {
        if (vec && left >= 16) {
#pragma unroll
            for (int i = 0; i < U; ++i) u[i] = reinterpret_cast<const uint4*>(at)[i];
        } else {
            alignas(16) T v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = i < left ? at[i] : T(0.0f);
#pragma unroll
            for (int i = 0; i < U; ++i) u[i] = reinterpret_cast<uint4*>(v)[i];
        }
    }
    __device__ __forceinline__ void store(T* at, int left, bool vec) const
    {
        if (vec && left >= 16) {
#pragma unroll
            for (int i = 0; i < U; ++i) reinterpret_cast<uint4*>(at)[i] = u[i];
        } else {
            alignas(16) T v[16];
#pragma unroll
            for (int i = 0; i < U; ++i) reinterpret_cast<uint4*>(v)[i] = u[i];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < left) at[i] = v[i];
        }
    }
    // channels 2 j and 2 j + 1
    __device__ __forceinline__ void add(int j, float a, float b)
    {
        if constexpr (sizeof(T) == 2) {
            uint32_t& w = reinterpret_cast<uint32_t*>(u)[j];
            w = rounded(__uint_as_float(w << 16) + a, __uint_as_float(w & 0xffff0000u) + b);
        } else {
            float* f = reinterpret_cast<float*>(u);
            f[2 * j] += a;
            f[2 * j + 1] += b;
        }
    }
};

// A warp: tiles of 16 rows by 64 channels, the rows of the block's tile for each of its channel blocks in turn.
template <typename T>
__global__ void __launch_bounds__(UP_WARPS * 32)
adapter_up_kernel(const UpParams p)
{
    constexpr int TERMS = kTerms<T>;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int slot_s[UP_ROWS];
    // what a channel block does: for each 16 rows the adapters they ask for, those that differ from the one before being fetched
    __shared__ int use_slot[UP_ROWS], use_groups[UP_ROWS], use_first[UP_ROWS / 16 + 1], fetches_s;
    __shared__ unsigned short use_mask[UP_ROWS];
    __shared__ int fetch_slot[UP_ROWS], fetch_groups[UP_ROWS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int row0 = blockIdx.x * p.tile_rows, tiles = (p.tile_rows + 15) / 16;
    // Adapters, slots and base are there: the first kernel let this one start after its own wait.  z is behind this one's wait.
    {
        Rows mine = p.rows;
        mine.n_rows = min(mine.n_rows, row0 + p.tile_rows);
        find_slots<UP_ROWS, UP_WARPS>(mine, row0, slot_s);
    }
    if (warp == 0) {
        int uses = 0, fetches = 0, last = kNoAdapter;
        for (int m = 0; m < tiles; ++m) {
            const int slot = lane < 16 ? slot_s[16 * m + lane] : kNoRow;
            const unsigned same = __match_any_sync(0xffffffffu, slot);
            const bool leads = slot >= 0 && lane == __ffs(same) - 1;
            const unsigned leaders = __ballot_sync(0xffffffffu, leads);
            const int n = __popc(leaders), e = __popc(leaders & ((1u << lane) - 1));
            const int first_slot = __shfl_sync(0xffffffffu, slot, n ? __ffs(leaders) - 1 : 0);
            const int kept = n && first_slot == last;        // the first of them is there already
            if (leads) {
                const int groups = (p.rows.ranks[slot] + GROUP - 1) / GROUP;
                use_slot[uses + e] = slot;
                use_groups[uses + e] = groups;
                use_mask[uses + e] = (unsigned short)same;
                if (e >= kept) {
                    fetch_slot[fetches + e - kept] = slot;
                    fetch_groups[fetches + e - kept] = groups;
                }
            }
            if (n) last = __shfl_sync(0xffffffffu, slot, 31 - __clz(leaders));
            if (lane == 0) use_first[m] = uses;
            uses += n;
            fetches += n - kept;
        }
        if (lane == 0) { use_first[tiles] = uses; fetches_s = fetches; }
    }
    __syncthreads();
    const int fetches = fetches_s;
    const int b0 = (blockIdx.y * UP_WARPS + warp) * p.per_warp, b1 = min(b0 + p.per_warp, p.blocks);
    const int stage_bytes = p.groups * 2048;
    uint8_t* ring = smem + (size_t)warp * p.stages * stage_bytes;
    uint4* zs = reinterpret_cast<uint4*>(smem + (size_t)UP_WARPS * p.stages * stage_bytes);     // [tile][group][term][lane]

    int fb = b0, ff = 0, fs = 0;
    auto fetch = [&]() {
        if (fb < b1 && ff < fetches) {
            const int groups = fetch_groups[ff];
            const uint8_t* from = p.B + (size_t)fetch_slot[ff] * p.b_slot + (size_t)fb * groups * 2048 + lane * 16;
            uint8_t* to = ring + fs * stage_bytes + lane * 16;
            for (int i = 0; i < groups; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) copy16(to + i * 2048 + k * 512, from + i * 2048 + k * 512);
            if (++ff == fetches) { ff = 0; ++fb; }
        }
        copies_commit();
        if (++fs == p.stages) fs = 0;
    };
    for (int i = 0; i < p.stages - 1; ++i) fetch();

    // base of 16 rows, this lane's two rows and 16 channels
    Piece<T> base[2];
    auto ask = [&](int b, int m) {
        const int ch = b * BLOCK + 16 * t;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 16 * m + g + 8 * h;
            base[h].zero();
            if (p.base && slot_s[r] != kNoRow && ch < p.M)
                base[h].load((const T*)p.base + (long long)(row0 + r) * p.ldb + ch, p.M - ch, p.vec);
        }
    };
    if (b0 < b1) ask(b0, 0);

    // ---- z: the splits' sum, scaled, as bf16 terms in the order of the product's first operand ----
    pdl_wait();
    pdl_launch_dependents();
    const int rank_pad = p.groups * GROUP;
    for (int i = threadIdx.x; i < tiles * p.groups * 32; i += UP_WARPS * 32) {
        const int ln = i & 31, group = (i >> 5) % p.groups, m = (i >> 5) / p.groups;
        float v[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 16 * m + (ln >> 2) + 8 * h, slot = slot_s[r], first = group * GROUP + 4 * (ln & 3);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[h][k] = 0.0f;
            const int have = slot >= 0 ? p.rows.ranks[slot] - first : 0;     // z is written for the adapter's own ranks only
            if (have > 0) {
                const float* z = p.z + (size_t)(row0 + r) * rank_pad + first;
#pragma unroll 8
                for (int s = 0; s < p.splits; ++s) {
                    const float4 u = __ldcg(reinterpret_cast<const float4*>(z + (size_t)s * p.rows.n_rows * rank_pad));
                    v[h][0] += u.x; v[h][1] += u.y; v[h][2] += u.z; v[h][3] += u.w;
                }
                const float c = p.scales[slot] * (p.x_scale ? p.x_scale[row0 + r] : 1.0f);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[h][k] = k < have ? v[h][k] * c : 0.0f;
            }
        }
        uint4* to = zs + (size_t)((i >> 5) * TERMS) * 32 + ln;
#pragma unroll
        for (int k = 0; k < TERMS; ++k) {
            uint4 w;
            if (k + 1 < TERMS) {
                w.x = cut(v[0][0], v[0][1]); w.y = cut(v[1][0], v[1][1]);
                w.z = cut(v[0][2], v[0][3]); w.w = cut(v[1][2], v[1][3]);
            } else {
                w.x = rounded(v[0][0], v[0][1]); w.y = rounded(v[1][0], v[1][1]);
                w.z = rounded(v[0][2], v[0][3]); w.w = rounded(v[1][2], v[1][3]);
            }
            to[k * 32] = w;
        }
    }
    __syncthreads();

    int stage = -1;
    for (int b = b0; b < b1; ++b) {
        int last = kNoAdapter;
        for (int m = 0; m < tiles; ++m) {
            for (int e = use_first[m]; e < use_first[m + 1]; ++e) {
                const int groups = use_groups[e];
                if (use_slot[e] != last) {           // its weights: the stage before is free
                    last = use_slot[e];
                    if (stage >= 0) fetch();
                    if (++stage == p.stages) stage = 0;
                    // (a stage's copies are one group, and stages - 2 groups may follow the one that is needed)
                    if (p.stages == 2) copies_wait<0>();
                    else if (p.stages == 3) copies_wait<1>();
                    else if (p.stages == 4) copies_wait<2>();
                    else copies_wait<6>();
                }
                const uint8_t* from = ring + stage * stage_bytes + lane * 16;
                float acc[8][4];
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[j][k] = 0.0f;
                for (int i = 0; i < groups; ++i) {
                    uint4 z[TERMS];
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) z[k] = zs[(size_t)((m * p.groups + i) * TERMS + k) * 32 + lane];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint4 w = *reinterpret_cast<const uint4*>(from + i * 2048 + q * 512);
#pragma unroll
                        for (int k = TERMS - 1; k >= 0; --k) {
                            mma_bf16(acc[2 * q], z[k], w.x, w.y);
                            mma_bf16(acc[2 * q + 1], z[k], w.z, w.w);
                        }
                    }
                }
                const unsigned mask = use_mask[e];
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (mask >> (g + 8 * h) & 1)
#pragma unroll
                        for (int j = 0; j < 8; ++j) base[h].add(j, acc[j][2 * h], acc[j][2 * h + 1]);
            }
            const int ch = b * BLOCK + 16 * t;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = 16 * m + g + 8 * h, slot = slot_s[r];
                if (slot != kNoRow && ch < p.M && !(p.in_place && slot == kNoAdapter))
                    base[h].store((T*)p.out + (long long)(row0 + r) * p.ldo + ch, p.M - ch, p.vec);
            }
            if (m + 1 < tiles) ask(b, m + 1);
            else if (b + 1 < b1) ask(b + 1, 0);
        }
    }
    copies_wait<0>();
}

// ---- launches ---------------------------------------------------------------------------------------------------------------

bool off(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) != 0; }

template <typename T, int NT, int RG>
size_t down_smem(int groups)
{
    return (size_t)DOWN_WARPS * (kDownStages<T, NT, RG> * kDownStage<T, NT, RG> + 8 * NT * groups * GROUP * sizeof(float));
}

template <typename T, int NT, int RG>
cudaError_t prepare_down()
{
    return cudaFuncSetAttribute(adapter_down_kernel<T, NT, RG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)down_smem<T, NT, RG>(MAX_RANK / GROUP));
}
template <typename T>
cudaError_t prepare_type()
{
    cudaError_t e = prepare_down<T, 1, 1>();
    if (e == cudaSuccess) e = prepare_down<T, 1, 2>();
    if (e == cudaSuccess) e = prepare_down<T, 1, 4>();
    if (e == cudaSuccess) e = prepare_down<T, 2, 1>();
    if (e == cudaSuccess) e = prepare_down<T, 2, 2>();
    if (e == cudaSuccess) e = prepare_down<T, 2, 4>();
    return e;
}
cudaError_t prepare()
{
    cudaError_t e = prepare_type<float>();
    if (e == cudaSuccess) e = prepare_type<__nv_bfloat16>();
    if (e == cudaSuccess) e = prepare_type<int8_t>();
    if (e == cudaSuccess) e = cudaFuncSetAttribute(adapter_up_kernel<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(adapter_up_kernel<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
    return e;
}

template <typename T, int NT, int RG>
cudaError_t down(const DownParams& p, cudaStream_t st)
{
    PdlLaunch l((unsigned)((p.rows.n_rows + 8 * NT - 1) / (8 * NT)), DOWN_WARPS * 32, down_smem<T, NT, RG>(p.groups), st);
    l.cfg.gridDim.y = (unsigned)p.splits;
    return cudaLaunchKernelEx(&l.cfg, adapter_down_kernel<T, NT, RG>, p);
}

template <typename T>
cudaError_t down_type(const DownParams& p, bool wide, cudaStream_t st)
{
    const int rg = p.groups == 1 ? 1 : p.groups == 2 ? 2 : 4;
    if (wide) return rg == 1 ? down<T, 2, 1>(p, st) : rg == 2 ? down<T, 2, 2>(p, st) : down<T, 2, 4>(p, st);
    return rg == 1 ? down<T, 1, 1>(p, st) : rg == 2 ? down<T, 1, 2>(p, st) : down<T, 1, 4>(p, st);
}

struct Shape {
    bool wide;           // the first kernel's tiles have 16 rows, else 8
    int splits;          // blocks that share a contraction
};
Shape shape_of(const tsvd_adapters_s* h, int rows)
{
    Shape s;
    s.wide = rows >= 1024;
    const int tiles = (rows + (s.wide ? 15 : 7)) / (s.wide ? 16 : 8);
    // two blocks an SM, a chunk for every warp
    const int want = (2 * h->sms + tiles - 1) / tiles, most = (h->chunks + DOWN_WARPS - 1) / DOWN_WARPS;
    s.splits = want < most ? want : most;
    if (s.splits > MAX_SPLITS) s.splits = MAX_SPLITS;
    return s;
}
size_t z_bytes(const tsvd_adapters_s* h, int rows) { return (size_t)shape_of(h, rows).splits * rows * h->groups * GROUP * sizeof(float); }

tsvd_status_t grow(tsvd_adapters_s* h, size_t need)
{
    if (need <= h->z_bytes) return TSVD_OK;
    float* z = nullptr;
    if (need < 2 * h->z_bytes) need = 2 * h->z_bytes;
    TSVD_CUDA_OK(cudaMalloc(&z, need));
    if (h->z) {
        try {
            h->outgrown->push_back(h->z);        // a captured graph may hold it: freed with the handle
        } catch (...) {
            cudaFree(z);
            return TSVD_E_NOMEM;
        }
    }
    h->z = z;
    h->z_bytes = need;
    return TSVD_OK;
}

void release(tsvd_adapters_s* h)
{
    if (h->A) cudaFree(h->A);
    if (h->B) cudaFree(h->B);
    if (h->ranks) cudaFree(h->ranks);
    if (h->scales) cudaFree(h->scales);
    if (h->z) cudaFree(h->z);
    if (h->outgrown)
        for (void* p : *h->outgrown) cudaFree(p);
    if (h->dev_status) cudaFree(h->dev_status);
    (void)cudaGetLastError();
    delete h->outgrown;
    delete h;
}

}  // namespace

extern "C" tsvd_status_t tsvd_adapters_create(int N, int M, int max_rank, int n_slots, tsvd_adapters_t* out)
{
    if (!out) return TSVD_E_NULL;
    *out = nullptr;
    if (N < 1 || M < 1 || max_rank < 1 || n_slots < 1) return TSVD_E_SHAPE;
    if (max_rank > MAX_RANK || N > (1 << 24) || M > (1 << 21)) return TSVD_E_TOOBIG;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return TSVD_E_CUDA; }
    tsvd_adapters_s* h = new (std::nothrow) tsvd_adapters_s();
    if (!h) return TSVD_E_NOMEM;
    h->outgrown = new (std::nothrow) std::vector<void*>();
    if (!h->outgrown) { delete h; return TSVD_E_NOMEM; }
    h->device = dev;
    h->N = N;
    h->M = M;
    h->max_rank = max_rank;
    h->n_slots = n_slots;
    h->groups = (max_rank + GROUP - 1) / GROUP;
    h->chunks = (N + CHUNK - 1) / CHUNK;
    h->blocks = (M + BLOCK - 1) / BLOCK;
    h->a_slot = (size_t)h->chunks * h->groups * 1024;
    h->b_slot = (size_t)h->blocks * h->groups * 2048;
    cudaError_t e = cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaMalloc(&h->A, h->a_slot * n_slots);
    if (e == cudaSuccess) e = cudaMalloc(&h->B, h->b_slot * n_slots);
    if (e == cudaSuccess) e = cudaMalloc(&h->ranks, sizeof(int) * n_slots);
    if (e == cudaSuccess) e = cudaMemset(h->ranks, 0, sizeof(int) * n_slots);
    if (e == cudaSuccess) e = cudaMalloc(&h->scales, sizeof(float) * n_slots);
    if (e == cudaSuccess) e = cudaMalloc(&h->dev_status, sizeof(int));
    if (e == cudaSuccess) e = cudaMemset(h->dev_status, 0, sizeof(int));
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
    if (e == cudaSuccess) e = prepare();
    if (e != cudaSuccess) {
        release(h);
        return e == cudaErrorMemoryAllocation ? TSVD_E_NOMEM : TSVD_E_CUDA;
    }
    *out = h;
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_adapters_set(tsvd_adapters_t h, int slot, const void* A, long long lda, const void* B, long long ldb,
                                           tsvd_dtype_t dtype, int rank, float scale, void* stream)
{
    if (!h) return TSVD_E_NULL;
    if (slot < 0 || slot >= h->n_slots) return TSVD_E_INDEX;
    if (rank < 0 || rank > h->max_rank || (rank && (lda < h->N || ldb < rank))) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (rank && (!A || !B)) return TSVD_E_NULL;
    const size_t size = dtype == TSVD_F32 ? 4 : 2;
    if (rank && (off(A, size) || off(B, size))) return TSVD_E_ALIGN;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    // (not a programmatic dependent: it begins when all work ahead has ended, and what follows begins when it has)
    uint4 *a = reinterpret_cast<uint4*>(h->A + h->a_slot * slot), *b = reinterpret_cast<uint4*>(h->B + h->b_slot * slot);
    const unsigned grid = (unsigned)h->sms * 4;
    if (dtype == TSVD_F32)
        adapter_set_kernel<<<grid, 256, 0, (cudaStream_t)stream>>>((const float*)A, lda, (const float*)B, ldb, rank, h->N, h->M, h->chunks, h->blocks,
                                                                   a, b, h->ranks + slot, h->scales + slot, scale);
    else
        adapter_set_kernel<<<grid, 256, 0, (cudaStream_t)stream>>>((const __nv_bfloat16*)A, lda, (const __nv_bfloat16*)B, ldb, rank, h->N, h->M,
                                                                   h->chunks, h->blocks, a, b, h->ranks + slot, h->scales + slot, scale);
    TSVD_CUDA_OK(cudaGetLastError());
    tsvd_count_launch();
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_adapters_reserve(tsvd_adapters_t h, int rows_max)
{
    if (!h) return TSVD_E_NULL;
    if (rows_max < 1) return TSVD_E_SHAPE;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    // (fewer rows may be cut into more splits: the most that any number of rows up to rows_max takes)
    size_t need = z_bytes(h, rows_max);
    for (int rows = 8; rows < rows_max; rows += 8) {
        const size_t n = z_bytes(h, rows);
        if (n > need) need = n;
        if (shape_of(h, rows).splits == 1 && rows >= 1024) break;
    }
    return grow(h, need);
}

extern "C" tsvd_status_t tsvd_adapters_forward(tsvd_adapters_t h, const void* x, long long ldx, const float* x_scale, tsvd_dtype_t dtype,
                                               const void* base, long long ldb, void* out, long long ldo, tsvd_dtype_t out_dtype,
                                               const int* slots, const int* q_start, int n_seq, int n_rows, void* stream)
{
    if (!h) return TSVD_E_NULL;
    if (n_rows < 0 || n_seq < 1 || (!q_start && n_rows != n_seq) || ldx < h->N || (base && ldb < h->M) || ldo < h->M) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16 && dtype != TSVD_I8) return TSVD_E_DTYPE;
    if (out_dtype != TSVD_F32 && out_dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (x_scale && dtype != TSVD_I8) return TSVD_E_DTYPE;
    if (n_rows == 0) return TSVD_OK;
    if (!x || !out || !slots) return TSVD_E_NULL;
    const size_t size = dtype == TSVD_F32 ? 4 : dtype == TSVD_BF16 ? 2 : 1, out_size = out_dtype == TSVD_F32 ? 4 : 2;
    if (off(x, size) || off(base, out_size) || off(out, out_size) || off(x_scale, 4) || off(slots, 4) || off(q_start, 4)) return TSVD_E_ALIGN;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    const tsvd_status_t grown = grow(h, z_bytes(h, n_rows));
    if (grown != TSVD_OK) return grown;
    cudaStream_t st = (cudaStream_t)stream;
    const Rows rows{slots, q_start, n_seq, n_rows, h->n_slots, h->ranks, h->dev_status};
    const Shape s = shape_of(h, n_rows);
    const size_t step = dtype == TSVD_I8 ? 8 : 16;
    const DownParams d{rows, x, ldx, !off(x, step) && (n_rows == 1 || ldx * (long long)size % (long long)step == 0), h->N, h->chunks, s.splits, h->groups,
                       h->A, h->a_slot, h->z};
    if (dtype == TSVD_F32) TSVD_CUDA_OK(down_type<float>(d, s.wide, st));
    else if (dtype == TSVD_BF16) TSVD_CUDA_OK(down_type<__nv_bfloat16>(d, s.wide, st));
    else TSVD_CUDA_OK(down_type<int8_t>(d, s.wide, st));
    tsvd_count_launch();

    auto even = [&](const void* p, long long ld) { return !p || (!off(p, 16) && (n_rows == 1 || ld * (long long)out_size % 16 == 0)); };
    UpParams u{};
    u.rows = rows;
    u.z = h->z;
    u.splits = s.splits;
    u.groups = h->groups;
    u.scales = h->scales;
    u.x_scale = x_scale;
    u.base = base;
    u.ldb = ldb;
    u.out = out;
    u.ldo = ldo;
    u.vec = even(base, ldb) && even(out, ldo);
    u.in_place = base == out && ldb == ldo;
    u.M = h->M;
    u.blocks = h->blocks;
    u.B = h->B;
    u.b_slot = h->b_slot;
    u.tile_rows = n_rows >= 1024 ? UP_ROWS : n_rows > 256 ? 16 : 8;
    const long long tiles = (n_rows + u.tile_rows - 1) / u.tile_rows;
    // channel blocks a warp, so that there are about three blocks of threads an SM
    u.per_warp = 1;
    while (tiles * ((h->blocks + UP_WARPS * u.per_warp - 1) / (UP_WARPS * u.per_warp)) > 4LL * h->sms && u.per_warp < h->blocks) ++u.per_warp;
    u.stages = h->groups == 1 ? (u.tile_rows == UP_ROWS ? 4 : 8) : h->groups == 2 ? 4 : 2;
    const size_t smem = (size_t)UP_WARPS * u.stages * h->groups * 2048 + (size_t)((u.tile_rows + 15) / 16) * h->groups * (out_size == 2 ? 2 : 3) * 512;
    PdlLaunch l((unsigned)tiles, UP_WARPS * 32, smem, st);
    l.cfg.gridDim.y = (unsigned)((h->blocks + UP_WARPS * u.per_warp - 1) / (UP_WARPS * u.per_warp));
    if (out_dtype == TSVD_F32) TSVD_CUDA_OK(cudaLaunchKernelEx(&l.cfg, adapter_up_kernel<float>, u));
    else TSVD_CUDA_OK(cudaLaunchKernelEx(&l.cfg, adapter_up_kernel<__nv_bfloat16>, u));
    tsvd_count_launch();
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_adapters_info(tsvd_adapters_t h, int* N, int* M, int* max_rank, int* n_slots, size_t* bytes)
{
    if (!h) return TSVD_E_NULL;
    if (N) *N = h->N;
    if (M) *M = h->M;
    if (max_rank) *max_rank = h->max_rank;
    if (n_slots) *n_slots = h->n_slots;
    if (bytes) *bytes = (h->a_slot + h->b_slot + sizeof(int) + sizeof(float)) * h->n_slots;
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_adapters_last_status(tsvd_adapters_t h)
{
    if (!h) return TSVD_E_NULL;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    int word = 0;
    TSVD_CUDA_OK(cudaMemcpy(&word, h->dev_status, sizeof(int), cudaMemcpyDeviceToHost));
    if (word) TSVD_CUDA_OK(cudaMemset(h->dev_status, 0, sizeof(int)));
    if (word) TSVD_CUDA_OK(cudaStreamSynchronize(nullptr));      // other streams do not wait for the memset
    return word ? TSVD_E_INDEX : TSVD_OK;
}

extern "C" void tsvd_adapters_destroy(tsvd_adapters_t h)
{
    if (!h) return;
    const int dev = h->device;
    int prev = dev;
    if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) cudaSetDevice(dev);
    cudaDeviceSynchronize();
    release(h);
    if (prev != dev) cudaSetDevice(prev);
}
