// Low-rank adapters of many requests beside a shared projection:  out_i = base_i + c_s B_s (A_s x_i),  s the adapter of row i's
// sequence (A_s [rank, N], B_s [M, rank] in bf16).
//
// z_i = A_s x_i (down), then out_i = base_i + c_s B_s z_i (up).  Three forms, chosen in tsvd_adapters_forward:
//   few rows      one launch; a cluster of blocks takes up to eight rows through both products (adapter_few_kernel)
//   more          two launches, the second a programmatic dependent of the first, on mma.sync: tiles of consecutive rows, whatever
//                 sequences they belong to, and inside a tile the adapters that its rows ask for, each once (adapter_down_kernel,
//                 adapter_up_kernel).  What the products of an adapter give for rows of another one is dropped, never added
//   many rows of  two launches on tcgen05: tiles of up to 128 rows of one sequence, so of one adapter (adapter_down_many_kernel,
//   a sequence    adapter_many_kernel)
// In all of them a row's result is made of its own numbers and adapter only.  How its sums are cut, and with that their last bits, goes
// by the call: its rows and sequences choose the form, and a cluster of the first form shares its work out by the adapters of all its rows.
// The same call gives the same bits.
//
// The weights lie as tcgen05 takes them: eight rows of 16 bytes one after another, and are brought by bulk copies for it; the lanes
// of a warp that uses mma.sync copy the 16 bytes that they will read (cp.async, some stages ahead), and nothing is exchanged.
//
// What bounds them, in time of the device alone (the bytes' at 6.55 TB/s in brackets): 64 tokens with 48 adapters of rank 16, 4096 to
// 12288, 13.9 us (4.4; one token 5.9 us, so launch, two chains of loads and a cluster's exchange are most of it; of rank 64 26.2 (15.9): bytes);
// 2046 rows of five sequences, all of rank 64, 38.5 us (19.5), base and out being 15 of the bytes' 19.5; of unlike ranks, 64 and below, 36 to
// 38.  Under ncu, each alone, the second product takes 30 and the first one 16, with 64 KB of x on their way to an SM.
//
// Arithmetic: bf16 operands, fp32 sums.  8-bit x is exact in bf16.  fp32 x is cut into three bf16 terms that add up to it
// exactly.  z stays fp32 between the kernels, and enters the second product as two bf16 terms (off by 2^-16 of it at most, the
// result's own rounding by 2^-8) for bf16 results, as three (exactly) for fp32.  The parts of a contraction that blocks share are
// added in their order.
#include <algorithm>
#include <new>
#include <vector>

#include "serving.cuh"
#include "sm100_ptx.cuh"

struct tsvd_adapters_s {
    int device = 0;
    int sms = 0;
    int N = 0, M = 0, max_rank = 0, n_slots = 0;
    int groups = 0;                  // of 16 ranks, of the largest rank
    int chunks = 0, blocks = 0;      // of 32 columns of A, of 64 channels of B
    size_t a_slot = 0, b_slot = 0;   // bytes of a slot
    uint8_t* A = nullptr;            // [slot][chunk][its groups][2][4][8 ranks][16]: see adapter_set_kernel
    uint8_t* B = nullptr;            // [slot][block][its groups][2][64 rows][16]: see adapter_set_kernel
    int* ranks = nullptr;            // [slot], 0: empty
    float* scales = nullptr;         // [slot]
    int few[9] = {};                 // [1, 2, 4, 8]: clusters of so many blocks of the kernel for few rows that run at a time
    float* z = nullptr;              // scratch: [row][16 * groups]
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
constexpr int MAX_SPLITS = 8;      // a cluster
constexpr int MOST_ROWS = 1 << 30; // and sequences: their numbers are added in 32 bits

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
// (shared addresses of 32 bits, and sixteen bytes for certain: the offsets of a run of copies go into the instructions)
__device__ __forceinline__ void copy16(uint32_t to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t to, const void* from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
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

// 16 ranks by the 32 columns of a chunk: eight columns of rank g (lo) and of rank g + 8 (hi) a lane.
__device__ __forceinline__ void mma_a(float (&d)[4], const uint4& lo, const uint4& hi, const uint32_t (&x)[4])
{
    mma_bf16(d, make_uint4(lo.x, hi.x, lo.y, hi.y), x[0], x[1]);
    mma_bf16(d, make_uint4(lo.z, hi.z, lo.w, hi.w), x[2], x[3]);
}
// Where the 16 bytes at columns 8 t and rank g of a group's half lie in shared memory: copied in their order (lane 8 t + g) and read by
// lane 4 g + t, both without a bank met twice.
__device__ __forceinline__ int a_place(int g, int t) { return (8 * t + (g ^ 2 * t)) * 16; }

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
            // Eight columns of a row are 16 bytes, eight rows in a row one matrix, four of them (the chunk's columns) before the next
            // eight ranks.
            const int g = (int)(i & 7), t = (int)(i >> 3 & 3), half = (int)(i >> 5 & 1);
            const long long piece = i >> 6;
            const int group = (int)(piece % groups), chunk = (int)(piece / groups);
            const int r = group * GROUP + 8 * half + g, c = chunk * CHUNK + 8 * t;
            a_out[i] = make_uint4(pair_of(A, lda, r, c, rank, N), pair_of(A, lda, r, c + 2, rank, N), pair_of(A, lda, r, c + 4, rank, N),
                                  pair_of(A, lda, r, c + 6, rank, N));
        } else {
            const long long k = i - na;
            const int row = (int)(k & 63), half = (int)(k >> 6 & 1);
            const long long piece = k >> 7;
            const int group = (int)(piece % groups), block = (int)(piece / groups);
            // Eight ranks of a row are 16 bytes, eight rows in a row what the tensor cores take as one matrix.  Row 8 j + n is channel
            // 8 n + j: a lane (or a thread) gets its results as eight channels in a row.
            const int ch = block * BLOCK + 8 * (row & 7) + (row >> 3), r = group * GROUP + 8 * half;
            b_out[k] = make_uint4(pair_of(B, ldb, ch, r, M, rank), pair_of(B, ldb, ch, r + 2, M, rank), pair_of(B, ldb, ch, r + 4, M, rank),
                                  pair_of(B, ldb, ch, r + 6, M, rank));
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
    int test_stall;          // test hook (tcgen05): the weights are never copied, so the waits must give up
};

template <typename T> constexpr int kXBytes = 8 * (int)sizeof(T);    // of a lane: eight columns of a row
template <typename T, int NT, int RG> constexpr int kDownStage = RG * 1024 + NT * 32 * kXBytes<T>;
// (as many as 16 KB a warp hold, 12 for few rows; with four groups and 32 rows the warps' parts take the rest)
template <typename T, int NT, int RG> constexpr int kDownRoom = (NT == 1 ? 12 : RG == 4 ? 20 : 16) * 1024 / kDownStage<T, NT, RG>;
template <typename T, int NT, int RG> constexpr int kDownStages = kDownRoom<T, NT, RG> < 2 ? 2 : kDownRoom<T, NT, RG> > 8 ? 8 : kDownRoom<T, NT, RG>;

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
        make({u.x, u.y});
    }
    __device__ __forceinline__ void make(const uint32_t (&u)[2])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = u[i >> 1] >> (16 * (i & 1));
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
        const uint4 a = *reinterpret_cast<const uint4*>(at), b = *reinterpret_cast<const uint4*>(at + 512);
        make({a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w});
    }
    __device__ __forceinline__ void make(const uint32_t (&u)[8])
    {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(u[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[0][i] = cut(v[2 * i], v[2 * i + 1]);
            w[1][i] = cut(v[2 * i], v[2 * i + 1]);
            w[2][i] = rounded(v[2 * i], v[2 * i + 1]);
        }
    }
};

// A lane's eight columns of a row into its place; zeros where the row or the columns end.
template <typename T>
__device__ __forceinline__ void copy_x(uint8_t* dst, const void* m, long long ldx, int row, int n_rows, int col, int left, int aligned, int lane)
{
    const bool there = row < n_rows && left > 0;
    const T* x = (const T*)m + (there ? (long long)row * ldx + col : 0);
    const int have = there ? min(left, 8) * (int)sizeof(T) : 0;
    if (aligned) {
        if constexpr (sizeof(T) == 1) {
            copy8(dst + lane * 8, x, have);
        } else {
#pragma unroll
            for (int i = 0; i < kXBytes<T> / 16; ++i)
                copy16(dst + i * 512 + lane * 16, have > 16 * i ? x + i * (16 / (int)sizeof(T)) : (const T*)m, max(0, min(16, have - 16 * i)));
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

constexpr int DOWN_GROUPS = 4;   // groups of ranks of a block at most (more are dealt to blocks of their own: the parts' place)

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
    const int row0 = blockIdx.x * ROWS, rank_pad = p.groups * GROUP, first_group = (int)blockIdx.z * DOWN_GROUPS;
    const int here_pad = min(DOWN_GROUPS, p.groups - first_group) * GROUP;
    find_slots<ROWS, DOWN_WARPS>(p.rows, row0, slot_s);
    if (warp == 0) {
        const int slot = lane < ROWS ? slot_s[lane] : kNoRow;
        const unsigned same = __match_any_sync(0xffffffffu, slot);
        const int groups = slot >= 0 ? (p.rows.ranks[slot] + GROUP - 1) / GROUP : 0;
        const bool leads = groups > first_group && lane == __ffs(same) - 1;
        const unsigned leaders = __ballot_sync(0xffffffffu, leads);
        if (leads) {
            const int e = __popc(leaders & ((1u << lane) - 1));
            entry_slot[e] = slot;
            entry_mask[e] = same;
            entry_groups[e] = groups;
        }
        if (lane == 0) entries_s = __popc(leaders);
    }
    __syncthreads();
    const int entries = entries_s;
    const int c0 = (int)((long long)p.chunks * blockIdx.y / p.splits), c1 = (int)((long long)p.chunks * (blockIdx.y + 1) / p.splits);
    uint8_t* ring = smem + (size_t)warp * STAGES * STAGE;
    float* parts = reinterpret_cast<float*>(smem + (size_t)DOWN_WARPS * STAGES * STAGE);     // [warp][row][here_pad]

    const uint32_t a_put = (uint32_t)a_place(lane & 7, lane >> 3);
    // ---- the next item (adapter, groups, chunk) into a stage ----
    int fe = 0, fg = first_group, fc = c0 + warp, fs = 0, f_here = 0;
    const uint8_t* fa = nullptr;
    size_t f_step = 0;
    unsigned f_mask = 0;
    auto aim = [&]() {                       // at the first chunk of (adapter fe, groups from fg on)
        const int groups = entry_groups[fe];
        f_here = min(RG, min(groups, first_group + DOWN_GROUPS) - fg);
        f_step = (size_t)groups * (DOWN_WARPS * 1024);
        f_mask = entry_mask[fe];
        fa = p.A + (size_t)entry_slot[fe] * p.a_slot + ((size_t)fc * groups + fg) * 1024 + lane * 16;
    };
    const T* xp = (const T*)p.x + (long long)(row0 + g) * p.ldx + 8 * t;
    const long long ldx8 = 8 * p.ldx;
    auto fetch = [&]() {
        if (fe < entries && fc < c1) {
            uint8_t* to = ring + fs * STAGE;
            const uint32_t to32 = ptx::smem_u32(to) + lane * 16;
#pragma unroll
            for (int i = 0; i < 2 * RG; ++i)
                if (i < 2 * f_here) copy16(ptx::smem_u32(to) + a_put + i * 512, fa + i * 512);
            const bool whole = p.aligned && (fc + 1) * CHUNK <= p.N && row0 + ROWS <= p.rows.n_rows;
            const T* x = xp + fc * CHUNK;
#pragma unroll
            for (int n = 0; n < NT; ++n, x += ldx8) {
                if (NT > 1 && !(f_mask >> (8 * n) & 0xffu)) continue;
                uint8_t* dst = to + RG * 1024 + n * 32 * kXBytes<T>;
                if (whole) {
                    if constexpr (sizeof(T) == 1) {
                        copy8(to32 - lane * 8 + RG * 1024 + n * 32 * kXBytes<T>, x);
                    } else {
#pragma unroll
                        for (int i = 0; i < kXBytes<T> / 16; ++i) copy16(to32 + RG * 1024 + n * 32 * kXBytes<T> + i * 512, x + i * (16 / (int)sizeof(T)));
                    }
                } else {
                    copy_x<T>(dst, p.x, p.ldx, row0 + 8 * n + g, p.rows.n_rows, fc * CHUNK + 8 * t, p.N - fc * CHUNK - 8 * t, p.aligned, lane);
                }
            }
            fc += DOWN_WARPS;
            fa += f_step;
            if (fc >= c1) {
                fc = c0 + warp;
                fg += RG;
                if (fg >= min(entry_groups[fe], first_group + DOWN_GROUPS)) { fg = first_group; ++fe; }
                if (fe < entries) aim();
            }
        }
        copies_commit();
        if (++fs == STAGES) fs = 0;
    };
    if (entries > 0) aim();
    for (int i = 0; i < STAGES - 1; ++i) fetch();

    int stage = 0;
    if (c0 + warp < c1)
        for (int e = 0; e < entries; ++e) {
            const int groups = min(entry_groups[e], first_group + DOWN_GROUPS);
            const unsigned mask = entry_mask[e];
            for (int g0 = first_group; g0 < groups; g0 += RG) {
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
                    __syncwarp();                    // (weights are the other lanes' copies too; and the place that fetch fills has been read)
                    const uint8_t* from = ring + stage * STAGE;
                    uint4 a[RG][2];
#pragma unroll
                    for (int i = 0; i < RG; ++i)
                        if (i < here) {
                            a[i][0] = *reinterpret_cast<const uint4*>(from + i * 1024 + a_place(g, t));
                            a[i][1] = *reinterpret_cast<const uint4*>(from + i * 1024 + 512 + a_place(g, t));
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
                                for (int k = Terms<T>::n - 1; k >= 0; --k) mma_a(acc[i][n], a[i][0], a[i][1], x.w[k]);
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
                                if (i < here) parts[(warp * ROWS + row) * here_pad + (g0 - first_group + i) * GROUP + g + (k & 2 ? 8 : 0)] = acc[i][n][k];
                    }
            }
        }
    copies_wait<0>();
    __syncthreads();
    // The blocks that share the contraction are a cluster: each adds its warps' parts, the first one gets them all (over its own
    // warps' parts, which are read by then) and adds them in their order.
    const int warps = min(DOWN_WARPS, c1 - c0), numbers = ROWS * here_pad;
    float sums[(ROWS * DOWN_GROUPS * GROUP + DOWN_WARPS * 32 - 1) / (DOWN_WARPS * 32)];
#pragma unroll
    for (int j = 0; j < (int)(sizeof(sums) / sizeof(float)); ++j) {
        const int i = (int)threadIdx.x + j * DOWN_WARPS * 32;
        sums[j] = 0.0f;
        if (i < numbers && slot_s[i / here_pad] >= 0)
            for (int w = 0; w < warps; ++w) sums[j] += parts[w * numbers + i];
    }
    if (p.splits > 1) {
        ptx::cluster_sync_all();
        const uint32_t first = ptx::cluster_map_u32(ptx::smem_u32(parts + blockIdx.y * numbers), 0);
#pragma unroll
        for (int j = 0; j < (int)(sizeof(sums) / sizeof(float)); ++j) {
            const int i = (int)threadIdx.x + j * DOWN_WARPS * 32;
            if (i < numbers) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(first + 4u * (unsigned)i), "f"(sums[j]) : "memory");
        }
        ptx::cluster_sync_all();
        if (blockIdx.y > 0) return;
    }
#pragma unroll
    for (int j = 0; j < (int)(sizeof(sums) / sizeof(float)); ++j) {
        const int i = (int)threadIdx.x + j * DOWN_WARPS * 32, row = i / here_pad, r = first_group * GROUP + i - row * here_pad;
        if (i >= numbers) break;
        const int slot = slot_s[row];
        if (slot < 0 || r >= p.rows.ranks[slot]) continue;
        if (p.splits > 1) {
            sums[j] = 0.0f;
            for (int k = 0; k < p.splits; ++k) sums[j] += parts[k * numbers + i];
        }
        p.z[(size_t)(row0 + row) * rank_pad + r] = sums[j];
    }
}

// ---- the same for many rows, on tcgen05 -----------------------------------------------------------------------------------
// A block: up to 128 rows of one sequence, a share of the columns, 64 of them a stage.  D = X A^T, 128 x the ranks, in tensor memory:
//   warps 0-7  x as bf16 (its terms one after another), rows of 128 bytes swizzled; bf16 is copied as it is, the other types are turned
//              in registers, the next stage's on their way meanwhile.  Warp 0 also asks for the weights (one bulk copy: their order)
//   warp 8     issues the products
// The blocks that share a tile's columns are a cluster; each adds the parts of its share of the rows, in their order.  Four stages, two
// blocks an SM: with six or eight of ranks of 64 one block fits, and clusters of eight find no place for each of sixteen tiles at once (2048
// rows of four sequences, 4096 to 4096, both products 25.0 us against 34.4 and 34.3).  Parts sent to the block that adds them, instead of
// fetched by it, need a place of their own, for a stage less: 36.4 against 36.1 us for five prompts.

constexpr int MANY_ROWS = 128, MANY_THREADS = 9 * 32;

// 32 lanes x 4 consecutive 32-bit columns.
__device__ __forceinline__ void tmem_ld4(uint32_t taddr, uint32_t (&r)[4])  // whole warp
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void umma_bf16_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// kind::f16, both operands bf16 and K-major, fp32 sums
__host__ __device__ constexpr uint32_t idesc_bf16(int m, int n)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// K-major without swizzle: eight rows of 16 bytes a matrix, the next eight rows `rows` bytes on, the next 16 bytes of a row `along`.
__device__ __forceinline__ uint64_t umma_desc_k_plain(uint32_t smem_addr, uint32_t along, uint32_t rows)
{
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(along >> 4) << 16;
    d |= (uint64_t)(rows >> 4) << 32;
    d |= (uint64_t)1 << 46;
    return d;
}

// The rows of a tile: a sequence is cut evenly into as few tiles of up to MANY_ROWS rows as it takes, and they are counted sequence by
// sequence.  A warp.  (What a sequence's adapter is comes with its ends: a load's time less.)
struct SeqTile { int row0, rows, slot, rank; };
__device__ __forceinline__ SeqTile find_tile(const Rows& r, int tile)
{
    const int lane = threadIdx.x & 31;
    SeqTile found{0, 0, kNoRow, 0};
    for (int s0 = 0, before = 0; s0 < r.n_seq; s0 += 32) {
        const int s = s0 + lane;
        const int begin = s < r.n_seq ? min(max(0, r.q_start[s]), r.n_rows) : 0, end = s < r.n_seq ? min(max(0, r.q_start[s + 1]), r.n_rows) : 0;
        const int mine = max(0, end - begin + MANY_ROWS - 1) / MANY_ROWS, its = s < r.n_seq ? r.slots[s] : kNoAdapter;
        int scan = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += v;
        }
        const unsigned holds = __ballot_sync(0xffffffffu, before + scan > tile);
        if (holds) {
            const int in = __ffs(holds) - 1, each = mine ? (end - begin + mine - 1) / mine : 0, at = begin + (tile - before - (scan - mine)) * each;
            found.row0 = __shfl_sync(0xffffffffu, at, in);
            found.rows = __shfl_sync(0xffffffffu, min(each, end - at), in);
            int slot = __shfl_sync(0xffffffffu, its, in);
            if (slot < -1 || slot >= r.n_slots) {
                if (lane == 0) atomicOr(r.status, KV4_DEV_INDEX);
                slot = kNoAdapter;
            }
            found.rank = slot >= 0 ? r.ranks[slot] : 0;
            found.slot = found.rank ? slot : kNoAdapter;
            return found;
        }
        before += __shfl_sync(0xffffffffu, scan, 31);
    }
    return found;
}

template <typename T>
struct DownMany {
    static constexpr int kStages = sizeof(T) == 4 ? 3 : 4, kX = Terms<T>::n * MANY_ROWS * 128;
    __host__ __device__ static constexpr int stage(int groups) { return kX + groups * 2048; }
    // (the parts lie over the stages; 16 bytes more a row, so that rows beside each other meet no bank twice)
    __host__ __device__ static constexpr int pitch(int groups) { return groups * GROUP * 4 + 16; }
    __host__ __device__ static constexpr size_t smem(int groups) { return (size_t)kStages * stage(groups) + 1024; }
};

template <typename T>
__global__ void __launch_bounds__(MANY_THREADS, sizeof(T) == 4 ? 1 : 2)
adapter_down_many_kernel(const DownParams p)
{
    using namespace ptx;
    using L = DownMany<T>;
    constexpr int TERMS = Terms<T>::n, STAGES = L::kStages;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    __shared__ uint64_t x_full[STAGES], w_full[STAGES], freed[STAGES], drained;
    __shared__ uint32_t tmem_slot;
    __shared__ int ctl_[2];
    volatile int* ctl = ctl_;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) { mbar_init(&x_full[i], 8); mbar_init(&w_full[i], 1); mbar_init(&freed[i], 1); }
        mbar_init(&drained, 1);
        ctl[0] = 0;
        ctl[1] = p.test_stall ? kWaitLimitStall : kWaitLimitDefault;
        fence_mbar_init();
    }
    // Tensor memory before the kernel after this one may start (see PdlLaunch).
    const uint32_t columns = p.groups <= 2 ? 32u : p.groups <= 4 ? 64u : 128u;
    if (warp == 8) { tmem_alloc(&tmem_slot, columns); tmem_relinquish(); }
    pdl_wait();
    const SeqTile tile = find_tile(p.rows, (int)blockIdx.x);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    // (behind the wait as well: what the kernel ahead has written is there before the next kernel, which reads it ahead of its own)
    pdl_launch_dependents();
    if (tile.slot < 0 || tile.rows == 0) {           // (all blocks of the cluster)
        if (warp == 8) tmem_dealloc(tmem, columns);
        return;
    }
    const int groups = (tile.rank + GROUP - 1) / GROUP, stage_bytes = L::stage(groups), all = (p.chunks + 1) / 2;
    // Stage i of block y is the i splits + y-th of the row: what the cluster reads at a time lies side by side.
    const int n = (all - (int)blockIdx.y + p.splits - 1) / p.splits, apart = 64 * p.splits, col0 = 64 * (int)blockIdx.y;
    auto chunks_of = [&](int i) { return min(2, p.chunks - 2 * (i * p.splits + (int)blockIdx.y)); };
    bool ok = true;
    int asked = 0;                                   // stages whose weights were asked for
    if (warp < 8) {
        // ================= x and the weights =================
        const int r0 = 16 * warp + (lane >> 3), u = lane & 7;            // its rows: r0 + 4 i
        const T* from = (const T*)p.x + (long long)(tile.row0 + r0) * p.ldx + col0 + 8 * u;
        const uint8_t* weights = p.A + (size_t)tile.slot * p.a_slot + (size_t)blockIdx.y * 2 * groups * 1024;
        const long long ldx4 = 4 * p.ldx;
        auto place = [&](int i, int k) { return (uint32_t)((i % STAGES) * stage_bytes + (r0 + 4 * k) * 128 + ((u ^ ((r0 + 4 * k) & 7)) << 4)); };
        auto room = [&](int i) {                     // the stage's place is free again, and its weights are on their way
            const int at = i % STAGES;
            if (i >= STAGES && !(ok = mbar_wait_warp(&freed[at], (uint32_t)(i / STAGES & 1) ^ 1, ctl))) return false;
            if (threadIdx.x == 0 && !p.test_stall) {
                const uint32_t bytes = (uint32_t)(chunks_of(i) * groups * 1024);
                mbar_arrive_expect_tx(&w_full[at], bytes);
                bulk_g2s(smem + at * stage_bytes + L::kX, weights + (size_t)i * p.splits * 2 * groups * 1024, bytes, &w_full[at]);
            }
            return true;
        };
        auto filled = [&](int i) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&x_full[i % STAGES]);
        };
        if constexpr (sizeof(T) == 2) {
            const uint32_t base = smem_u32(smem);
            for (int i = 0; i < n + STAGES - 1; ++i) {
                if (i < n) {
                    if (!room(i)) break;
                    ++asked;
                    const int left = p.N - i * apart - col0 - 8 * u;
                    const T* x = from + i * apart;
#pragma unroll
                    for (int k = 0; k < 4; ++k, x += ldx4)
                        if (r0 + 4 * k < tile.rows) {
                            if (left >= 8) copy16(base + place(i, k), x);
                            else copy16(smem + place(i, k), left > 0 ? x : (const T*)p.x, max(0, left) * 2);
                        }
                }
                copies_commit();
                copies_wait<STAGES - 1>();
                if (i >= STAGES - 1) filled(i - (STAGES - 1));
            }
            copies_wait<0>();
        } else {
            constexpr int RAW = 2 * (int)sizeof(T);              // words of eight columns
            uint32_t raw[4][RAW];
            auto load = [&](int i) {
                const int left = p.N - i * apart - col0 - 8 * u;
                const T* x = from + i * apart;
#pragma unroll
                for (int k = 0; k < 4; ++k, x += ldx4) {
                    const int have = r0 + 4 * k < tile.rows ? left : 0;
                    if (have >= 8) {
                        if constexpr (sizeof(T) == 1) {
                            const uint2 v = *reinterpret_cast<const uint2*>(x);
                            raw[k][0] = v.x; raw[k][1] = v.y;
                        } else {
                            const uint4 a = reinterpret_cast<const uint4*>(x)[0], b = reinterpret_cast<const uint4*>(x)[1];
                            raw[k][0] = a.x; raw[k][1] = a.y; raw[k][2] = a.z; raw[k][3] = a.w;
                            raw[k][4] = b.x; raw[k][5] = b.y; raw[k][6] = b.z; raw[k][7] = b.w;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < RAW; ++e) raw[k][e] = 0;
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (e < have) {
                                if constexpr (sizeof(T) == 1) raw[k][e / 4] |= (uint32_t)(uint8_t)x[e] << (8 * (e & 3));
                                else raw[k][e] = __float_as_uint(x[e]);
                            }
                    }
                }
            };
            load(0);
            for (int i = 0; i < n; ++i) {
                if (!room(i)) break;
                ++asked;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    Terms<T> x;
                    x.make(raw[k]);
#pragma unroll
                    for (int j = 0; j < TERMS; ++j)
                        *reinterpret_cast<uint4*>(smem + place(i, k) + j * (MANY_ROWS * 128)) = make_uint4(x.w[j][0], x.w[j][1], x.w[j][2], x.w[j][3]);
                }
                if (i + 1 < n) load(i + 1);
                filled(i);
            }
        }
    } else if (lane == 0) {
        // ================= products =================
        const uint64_t desc_x = umma_desc_k_sw128(smem_u32(smem)), desc_a = umma_desc_k_plain(smem_u32(smem + L::kX), 128, 512);
        const uint32_t kDesc = idesc_bf16(MANY_ROWS, groups * GROUP);
        for (int i = 0; i < n; ++i) {
            const int at = i % STAGES;
            if (!(ok = mbar_wait(&w_full[at], (uint32_t)(i / STAGES & 1), ctl))) break;
            if (!(ok = mbar_wait(&x_full[at], (uint32_t)(i / STAGES & 1), ctl))) break;
            tc_fence_after_sync();
            const uint32_t here = (uint32_t)(at * (stage_bytes >> 4));
            const int steps = 2 * chunks_of(i);                          // of 16 columns
            for (int k = TERMS - 1; k >= 0; --k)                         // (the smallest terms first)
                for (int j = 0; j < steps; ++j)
                    umma_bf16_ss(tmem, desc_x + here + (uint32_t)(k * (MANY_ROWS * 128 >> 4) + 2 * j), desc_a + here + (uint32_t)((j >> 1) * groups * (1024 >> 4) + (j & 1) * (256 >> 4)),
                                 kDesc, i > 0 || k < TERMS - 1 || j > 0);
            umma_commit(&freed[at]);
        }
        // every product has ended before its place is used again
        umma_commit(&drained);
        mbar_drain(&drained, 0);
    }
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    // Whoever gave up a wait, weights may still be on their way: they land before the parts lie over the stages, and the block ends.
    if (ctl[0]) {
        if (threadIdx.x == 0)
            for (int i = max(0, asked - STAGES); i < asked; ++i) mbar_drain(&w_full[i % STAGES], (uint32_t)(i / STAGES & 1));
        __syncthreads();
    }
    // ---- the parts: one row and half of the ranks a thread ----
    const int pitch = L::pitch(groups);
    if (warp < 8) {
        const int quarter = warp & 3, half = warp >> 2, row = 32 * quarter + lane;
        for (int j = half * groups; j < (half + 1) * groups; ++j) {      // of eight ranks
            uint32_t v[8];
            tmem_ld8(tmem + ((uint32_t)(quarter * 32) << 16) + 8u * j, v);
            tmem_ld_wait();
            if (row < tile.rows) {
                uint4* to = reinterpret_cast<uint4*>(smem + row * pitch + j * 32);
                to[0] = make_uint4(v[0], v[1], v[2], v[3]);
                to[1] = make_uint4(v[4], v[5], v[6], v[7]);
            }
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    // The tensor memory goes back before the cluster meets: its blocks share SMs with others that may wait for it (see PdlLaunch).
    if (warp == 8) tmem_dealloc(tmem, columns);
    if (p.splits > 1) cluster_sync_all();
    const int first = tile.rows * (int)blockIdx.y / p.splits, rows = tile.rows * (int)(blockIdx.y + 1) / p.splits - first, quads = groups * (GROUP / 4);
    for (int i = threadIdx.x; i < rows * quads; i += MANY_THREADS) {
        const int row = first + i / quads, quad = i % quads;
        const uint32_t at = smem_u32(smem + row * pitch + quad * 16);
        float4 v[MAX_SPLITS], sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < MAX_SPLITS; ++k)
            if (k < p.splits)
                asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
                             : "=f"(v[k].x), "=f"(v[k].y), "=f"(v[k].z), "=f"(v[k].w) : "r"(cluster_map_u32(at, (uint32_t)k)) : "memory");
#pragma unroll
        for (int k = 0; k < MAX_SPLITS; ++k)
            if (k < p.splits) { sum.x += v[k].x; sum.y += v[k].y; sum.z += v[k].z; sum.w += v[k].w; }
        *reinterpret_cast<float4*>(p.z + (size_t)(tile.row0 + row) * (p.groups * GROUP) + quad * 4) = sum;
    }
    if (p.splits > 1) cluster_sync_all();            // (a block's parts stay until the others have read them)
    if (threadIdx.x == 0 && ctl[0]) atomicOr(p.rows.status, KV4_DEV_TIMEOUT);
}

// ---- out = base + c B z ---------------------------------------------------------------------------------------------------

struct UpParams {
    Rows rows;
    const float* z;
    int groups;
    const float* scales;     // [slot]
    const float* x_scale;    // [row] or null
    const void* base;        // null: zeros
    long long ldb;
    void* out;
    long long ldo;
    int vec;                 // rows of base and out on 16-byte boundaries
    int in_place;            // out is base: rows without an adapter are as they should be
    int M, blocks, per_warp; // per_warp: blocks of 64 channels that a warp takes
    int columns;             // the kernel for many rows: blocks of threads that share a tile of rows
    int tile_rows;           // rows of a block of threads: at most UP_ROWS
    const uint8_t* B;
    size_t b_slot;
    int test_stall;          // test hook (tcgen05): the weights are never copied, so the waits must give up
};

template <typename T> constexpr int kTerms = sizeof(T) == 2 ? 2 : 3;

// Eight channels of a row, in the row's type.
template <typename T> struct Piece {
    static constexpr int U = (int)sizeof(T) / 2;     // 16-byte units
    uint4 u[U];
    __device__ __forceinline__ void load(const T* at, int left)                // number by number; zeros behind the row's end
    {
        alignas(16) T v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? at[i] : T(0.0f);
#pragma unroll
        for (int i = 0; i < U; ++i) u[i] = reinterpret_cast<uint4*>(v)[i];
    }
    __device__ __forceinline__ void store(T* at, int left) const
    {
        alignas(16) T v[8];
#pragma unroll
        for (int i = 0; i < U; ++i) reinterpret_cast<uint4*>(v)[i] = u[i];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) at[i] = v[i];
    }
};
template <typename T> constexpr int kBaseBytes = 32 * 2 * 8 * (int)sizeof(T);    // base of eight rows and 64 channels

// Base of rows 2 t and 2 t + 1 of eight and this lane's eight channels, into a stage: of the rows in `mask` (bits 0, 1).  at: the
// first row's place; left: channels there; full (of the whole warp): all 64 channels, and rows on 16-byte boundaries.
template <typename T>
__device__ __forceinline__ void copy_base(uint8_t* dst, const T* at, long long ld, unsigned mask, int left, bool full, int lane)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t to32 = ptx::smem_u32(dst) + lane * 16;
        const T* src = at + h * ld;
        uint8_t* to = dst + h * (Piece<T>::U * 512) + lane * 16;
        if (full) {
            if (mask >> h & 1)
#pragma unroll
                for (int i = 0; i < Piece<T>::U; ++i) copy16(to32 + (h * Piece<T>::U + i) * 512, src + i * (16 / (int)sizeof(T)));
        } else if ((mask >> h & 1) && left > 0) {
            Piece<T> v;
            v.load(src, left);
#pragma unroll
            for (int i = 0; i < Piece<T>::U; ++i) *reinterpret_cast<uint4*>(to + i * 512) = v.u[i];
        }
    }
}

// The sums of a product of 64 channels and eight rows: acc[q] holds channels 2 q, 2 q + 1 (elements 0 and 2, 1 and 3) of this lane's
// eight, of rows 2 t, 2 t + 1.  bf16: the tensor core adds to base; fp32, where its sums' last bits count, base is added afterwards.
template <typename T>
struct Sums {
    float acc[4][4];
    uint4 base[sizeof(T) == 4 ? 4 : 1];
    __device__ __forceinline__ void begin(const uint8_t* from, int lane)
    {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 u = *reinterpret_cast<const uint4*>(from + h * 512 + lane * 16);
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) { acc[q][h] = __uint_as_float(w[q] << 16); acc[q][2 + h] = __uint_as_float(w[q] & 0xffff0000u); }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) base[i] = *reinterpret_cast<const uint4*>(from + i * 512 + lane * 16);
            zero();
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[q][k] = 0.0f;
    }
    __device__ __forceinline__ void store(T* at, long long ld, unsigned mask, int left, bool full) const
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Piece<T> v;
            if constexpr (sizeof(T) == 2) {
                v.u[0] = make_uint4(rounded(acc[0][h], acc[0][2 + h]), rounded(acc[1][h], acc[1][2 + h]), rounded(acc[2][h], acc[2][2 + h]),
                                    rounded(acc[3][h], acc[3][2 + h]));
            } else {
                const float* f = reinterpret_cast<const float*>(base + 2 * h);
                float* y = reinterpret_cast<float*>(v.u);
#pragma unroll
                for (int q = 0; q < 4; ++q) { y[2 * q] = f[2 * q] + acc[q][h]; y[2 * q + 1] = f[2 * q + 1] + acc[q][2 + h]; }
            }
            T* to = at + h * ld;
            if (full) {
                if (mask >> h & 1)
#pragma unroll
                    for (int i = 0; i < Piece<T>::U; ++i) reinterpret_cast<uint4*>(to)[i] = v.u[i];
            } else if (mask >> h & 1) {
                v.store(to, left);
            }
        }
    }
};

// z of eight rows and sixteen ranks as the product's second operand, a lane's rank quadruple of its row: TERMS pairs of words.
template <int TERMS>
struct ZTerms {
    uint32_t w[TERMS][2];
    __device__ __forceinline__ void make(float (&v)[4])
    {
#pragma unroll
        for (int k = 0; k < TERMS; ++k) {
            const bool last = k + 1 == TERMS;
            w[k][0] = last ? rounded(v[0], v[1]) : cut(v[0], v[1]);
            w[k][1] = last ? rounded(v[2], v[3]) : cut(v[2], v[3]);
        }
    }
    __device__ __forceinline__ void put(uint8_t* at, int lane) const           // at: 32 * 8 * TERMS bytes
    {
        *reinterpret_cast<uint4*>(at + lane * 16) = make_uint4(w[0][0], w[0][1], w[1][0], w[1][1]);
        if constexpr (TERMS == 3) *reinterpret_cast<uint2*>(at + 512 + lane * 8) = make_uint2(w[2][0], w[2][1]);
    }
    __device__ __forceinline__ void get(const uint8_t* at, int lane)
    {
        const uint4 u = *reinterpret_cast<const uint4*>(at + lane * 16);
        w[0][0] = u.x; w[0][1] = u.y; w[1][0] = u.z; w[1][1] = u.w;
        if constexpr (TERMS == 3) {
            const uint2 v = *reinterpret_cast<const uint2*>(at + 512 + lane * 8);
            w[2][0] = v.x; w[2][1] = v.y;
        }
    }
};

// Product q's first operand out of 16 ranks' weights of 64 channels: rows 16 q + g and + 8, this lane's rank quadruple.
__device__ __forceinline__ uint4 b_rows(const uint8_t* at, int q, int lane)
{
    const uint8_t* from = at + (lane >> 1 & 1) * 1024 + (16 * q + (lane >> 2)) * 16 + (lane & 1) * 8;
    const uint2 lo = *reinterpret_cast<const uint2*>(from), hi = *reinterpret_cast<const uint2*>(from + 128);
    return make_uint4(lo.x, hi.x, lo.y, hi.y);
}

constexpr int UP_STAGES = 3;
// Blocks of threads an SM: 102, 128, 168 or 255 registers a thread.
template <typename T, int G> constexpr int kUpBlocks = G == 8 ? 2 : sizeof(T) == 2 ? (G == 4 ? 4 : 5) : G == 4 ? 3 : 4;

// A warp: 64 channels, whose weights (of one adapter) it holds in registers, sixteen rows after another of the block's tile; then the
// tile's next adapter; then its next 64 channels.  Weights and base are copied ahead into the warp's own shared memory.  G: groups
// of ranks at most.
template <typename T, int G>
__global__ void __launch_bounds__(UP_WARPS * 32, kUpBlocks<T, G>)
adapter_up_kernel(const UpParams p)
{
    constexpr int TERMS = kTerms<T>, Z = 256 * TERMS;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int slot_s[UP_ROWS], entry_slot[UP_ROWS + 1], entry_groups[UP_ROWS + 1], steps_s;
    // what is done for each 64 channels: (adapter, sixteen rows); behind the adapters the rows without one, whose base is copied
    __shared__ unsigned step_s[2 * UP_ROWS];                                   // adapter | tile << 8 | rows << 16
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int row0 = blockIdx.x * p.tile_rows, tiles = (p.tile_rows + 15) / 16;
    // Adapters, slots and base are there: the first kernel let this one start after its own wait.  z is behind this one's wait.
    {
        Rows mine = p.rows;
        mine.n_rows = min(mine.n_rows, row0 + p.tile_rows);
        find_slots<UP_ROWS, UP_WARPS>(mine, row0, slot_s);
    }
    if (warp == 0) {
        int a = slot_s[lane], b = slot_s[32 + lane], entries = 0, steps = 0;
        auto add = [&](int slot, unsigned in_a, unsigned in_b) {               // one adapter's rows
            const unsigned in = lane < 2 ? in_a >> (16 * lane) & 0xffffu : lane < 4 ? in_b >> (16 * (lane - 2)) & 0xffffu : 0u;
            const unsigned there = __ballot_sync(0xffffffffu, in != 0);
            if (in) {
                const int k = steps + __popc(there & ((1u << lane) - 1));
                step_s[k] = (unsigned)entries | (unsigned)lane << 8 | in << 16;
            }
            if (lane == 0) {
                entry_slot[entries] = slot;
                entry_groups[entries] = slot < 0 ? 0 : (p.rows.ranks[slot] + GROUP - 1) / GROUP;
            }
            steps += __popc(there);
            ++entries;
        };
        unsigned rest_a = __ballot_sync(0xffffffffu, a >= 0), rest_b = __ballot_sync(0xffffffffu, b >= 0);
        while (rest_a | rest_b) {
            const int slot = rest_a ? __shfl_sync(0xffffffffu, a, __ffs(rest_a) - 1) : __shfl_sync(0xffffffffu, b, __ffs(rest_b) - 1);
            const unsigned in_a = __ballot_sync(0xffffffffu, a == slot), in_b = __ballot_sync(0xffffffffu, b == slot);
            add(slot, in_a, in_b);
            rest_a &= ~in_a;
            rest_b &= ~in_b;
        }
        const unsigned none_a = __ballot_sync(0xffffffffu, a == kNoAdapter), none_b = __ballot_sync(0xffffffffu, b == kNoAdapter);
        if ((none_a | none_b) && !p.in_place) add(kNoAdapter, none_a, none_b);
        if (lane == 0) steps_s = steps;
    }
    __syncthreads();
    const int steps = steps_s, b0 = (blockIdx.y * UP_WARPS + warp) * p.per_warp, b1 = min(b0 + p.per_warp, p.blocks);
    uint8_t* zs = smem;                                                        // [eight rows][group][Z]
    uint8_t* weights = smem + 2 * tiles * p.groups * Z + warp * (p.groups * 2048 + 2 * UP_STAGES * kBaseBytes<T>);
    uint8_t* ring = weights + p.groups * 2048;

    // ---- copies: base of the next (block, step); weights of the next (block, adapter) ----
    const long long ldb8 = 8 * p.ldb, ldo8 = 8 * p.ldo;
    auto rows16 = [](unsigned step, long long ld8) { return (step >> 8 & 1u ? 2 * ld8 : 0) + (step >> 9 & 1u ? 4 * ld8 : 0); };   // (tile 0 .. 3)
    int fb = b0, fk = 0, fs = 0;
    const T* fbase = (const T*)p.base + (long long)(row0 + 2 * t) * p.ldb + b0 * BLOCK + 8 * g;
    auto left_of = [&](int b) { return p.M - b * BLOCK - 8 * g; };
    auto full_of = [&](int b) { return p.vec && (b + 1) * BLOCK <= p.M; };
    auto fetch = [&]() {
        if (fb < b1 && steps > 0) {
            const unsigned step = step_s[fk];
            if (p.base) {
                uint8_t* to = ring + fs * (2 * kBaseBytes<T>);
                const T* from = fbase + rows16(step, ldb8);
                copy_base<T>(to, from, p.ldb, step >> (16 + 2 * t), left_of(fb), full_of(fb), lane);
                copy_base<T>(to + kBaseBytes<T>, from + ldb8, p.ldb, step >> (24 + 2 * t), left_of(fb), full_of(fb), lane);
            }
            if (++fk == steps) { fk = 0; ++fb; fbase += BLOCK; }
        }
        copies_commit();
        if (++fs == UP_STAGES) fs = 0;
    };
    int wb = b0, wk = 0;                                                       // the step at which the weights on their way are needed
    auto fetch_weights = [&]() {                                               // (in the next group that is committed)
        if (wb >= b1 || steps == 0) return;
        const int e = (int)(step_s[wk] & 0xffu), groups = entry_groups[e];
        if (groups) {
            const uint8_t* from = p.B + (size_t)entry_slot[e] * p.b_slot + (size_t)wb * groups * 2048 + lane * 16;
#pragma unroll
            for (int i = 0; i < 4 * G; ++i)
                if (i < 4 * groups) copy16(ptx::smem_u32(weights) + lane * 16 + i * 512, from + i * 512);
        }
    };
    auto next_weights = [&]() {                                                // behind the adapter at (wb, wk)
        const unsigned e = step_s[wk] & 0xffu;
        while (wk < steps && (step_s[wk] & 0xffu) == e) ++wk;
        if (wk == steps) { wk = 0; ++wb; }
    };
    fetch_weights();
    for (int i = 0; i < UP_STAGES - 1; ++i) fetch();

    // ---- z, scaled, as bf16 terms in the order of the product's second operand ----
    pdl_wait();
    pdl_launch_dependents();
    const int rank_pad = p.groups * GROUP;
    for (int i = threadIdx.x; i < 2 * tiles * p.groups * 32; i += UP_WARPS * 32) {
        const int ln = i & 31, group = (i >> 5) % p.groups, tile = (i >> 5) / p.groups;
        const int r = 8 * tile + (ln >> 2), slot = slot_s[r], first = group * GROUP + 4 * (ln & 3);
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        const int have = slot >= 0 ? p.rows.ranks[slot] - first : 0;           // z is written for the adapter's own ranks only
        if (have > 0) {
            const float4 u = __ldcg(reinterpret_cast<const float4*>(p.z + (size_t)(row0 + r) * rank_pad + first));
            v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
            const float c = p.scales[slot] * (p.x_scale ? p.x_scale[row0 + r] : 1.0f);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = k < have ? v[k] * c : 0.0f;
        }
        ZTerms<TERMS> z;
        z.make(v);
        z.put(zs + (i >> 5) * Z, ln);
    }
    __syncthreads();

    int stage = 0, since = UP_STAGES;                                          // since: groups committed after the weights'
    uint4 w[4 * G];
    T* out = (T*)p.out + (long long)(row0 + 2 * t) * p.ldo + b0 * BLOCK + 8 * g;
    for (int b = b0; b < b1; ++b, out += BLOCK) {
        int last = -1, groups = 0;
        const int left = left_of(b);
        const bool full = full_of(b);
        for (int k = 0; k < steps; ++k) {
            const unsigned step = step_s[k];
            // (a step's copies are one group, and UP_STAGES - 2 groups may follow the one that is needed)
            copies_wait<UP_STAGES - 2>();
            if ((int)(step & 0xffu) != last) {
                last = (int)(step & 0xffu);
                groups = entry_groups[last];
                if (since < UP_STAGES - 1) copies_wait<0>();
                __syncwarp();                                                  // (the other lanes' copies)
#pragma unroll
                for (int i = 0; i < 4 * G; ++i)
                    w[i] = i < 4 * groups ? b_rows(weights + (i >> 2) * 2048, i & 3, lane) : make_uint4(0, 0, 0, 0);
                __syncwarp();                                                  // (all have read)
                next_weights();
                fetch_weights();
                since = 0;
            }
            Sums<T> sums[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                if (p.base) sums[n].begin(ring + (2 * stage + n) * kBaseBytes<T>, lane);
                else sums[n] = Sums<T>{};
            }
            const uint8_t* z_at = zs + 2 * (int)(step >> 8 & 0xffu) * p.groups * Z;
            auto product = [&](int i) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    ZTerms<TERMS> z;
                    z.get(z_at + (n * p.groups + i) * Z, lane);
#pragma unroll
                    for (int j = TERMS - 1; j >= 0; --j)
#pragma unroll
                        for (int q = 0; q < 4; ++q) mma_bf16(sums[n].acc[q], w[4 * i + q], z.w[j][0], z.w[j][1]);
                }
            };
            if (groups == G) {
#pragma unroll
                for (int i = 0; i < G; ++i) product(i);
            } else {
#pragma unroll
                for (int i = 0; i < G; ++i)
                    if (i < groups) product(i);
            }
            T* to = out + rows16(step, ldo8);
            sums[0].store(to, p.ldo, step >> (16 + 2 * t), left, full);
            sums[1].store(to + ldo8, p.ldo, step >> (24 + 2 * t), left, full);
            fetch();
            ++since;
            if (++stage == UP_STAGES) stage = 0;
        }
    }
    copies_wait<0>();
}

// ---- the same for many rows, on tcgen05 --------------------------------------------------------------------------------------
// A block: up to 128 rows of one sequence, blocks of 64 channels one after another.  D = Z B^T, 128 x 64, in tensor memory, with the
// terms of z side by side along the contraction and the same weights against each:
//   warp 8     brings the weights into shared memory (in the order they lie in: one bulk copy), and issues the products
//   warps 0-7  one row and 32 channels a thread: base, copied ahead into the warp's own place, plus D, by way of that place to out

constexpr int MANY_D = 4, MANY_B = 3;   // accumulators of 64 columns; blocks of channels whose weights are there or on their way

// Shared memory (1024-aligned): Z [eight ranks of a term][128 rows][16 B] | B [MANY_B][groups][2 KB] | base [8 warps][stages][32 rows][32 channels],
// the 16-byte unit u of row r turned by r (see unit_at)
template <typename T>
struct Many {
    static constexpr int kPitch = BLOCK / 2 * (int)sizeof(T), kStage = 32 * kPitch, kStages = sizeof(T) == 2 ? 3 : 2;
    // a row of 64 or 128 bytes: threads on neighbouring rows and the same unit, or on neighbouring units, meet no bank twice
    __device__ static __forceinline__ int unit_at(int r, int u) { return r * kPitch + ((sizeof(T) == 2 ? u ^ (r >> 1 & 3) : u ^ (r & 7)) << 4); }
    int groups;
    __host__ __device__ int z_bytes() const { return kTerms<T> * groups * 2 * 2048; }
    __host__ __device__ int b_bytes() const { return groups * 2048; }
    __host__ __device__ int base() const { return z_bytes() + MANY_B * b_bytes(); }
    __host__ __device__ size_t smem() const { return (size_t)base() + 8 * kStages * kStage + 1024; }
};

template <typename T>
__global__ void __launch_bounds__(MANY_THREADS, 2)
adapter_many_kernel(const UpParams p)
{
    using namespace ptx;
    using L = Many<T>;
    constexpr int TERMS = kTerms<T>, E = 16 / (int)sizeof(T), LANES = 32 / E, PER = 32 / LANES;    // lanes of a row's 32 channels, rows at a time
    const L lay{p.groups};
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    __shared__ uint64_t d_full[MANY_D], d_free[MANY_D], b_full[MANY_B], b_done[MANY_B], drained;
    __shared__ uint32_t tmem_slot;
    __shared__ int ctl_[2];
    volatile int* ctl = ctl_;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < MANY_D; ++i) { mbar_init(&d_full[i], 1); mbar_init(&d_free[i], 8); }
        for (int i = 0; i < MANY_B; ++i) { mbar_init(&b_full[i], 1); mbar_init(&b_done[i], 1); }
        mbar_init(&drained, 1);
        ctl[0] = 0;
        ctl[1] = p.test_stall ? kWaitLimitStall : kWaitLimitDefault;
        fence_mbar_init();
    }
    // Tensor memory before the kernel after this one may start (see PdlLaunch).
    if (warp == 8) { tmem_alloc(&tmem_slot, MANY_D * 64); tmem_relinquish(); }
    // Adapters, slots and base are there: the first kernel let this one start after its own wait.  z is behind this one's wait.
    const SeqTile tile = find_tile(p.rows, (int)blockIdx.x / p.columns);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    pdl_launch_dependents();
    const bool real = tile.slot >= 0;
    if (tile.rows == 0 || (!real && p.in_place)) {
        pdl_wait();              // (whoever waits for this kernel waits for those before it)
        if (warp == 8) tmem_dealloc(tmem, MANY_D * 64);
        return;
    }
    const int row0 = tile.row0, b0 = (int)blockIdx.x % p.columns * p.per_warp, b1 = min(b0 + p.per_warp, p.blocks);
    const int rank = tile.rank, groups = (rank + GROUP - 1) / GROUP, eights = 2 * groups;

    // ---- base of the next 64 channels into the warp's next stage: its rows, 32 channels of each by LANES lanes ----
    const int quarter = warp & 3, half = warp >> 2 & 1, mine0 = row0 + 32 * quarter;         // its rows (the tensor memory's lanes) and channels
    const int mine = max(0, min(32, tile.rows - 32 * quarter));
    uint8_t* place = smem + lay.base() + (warp & 7) * (L::kStages * L::kStage);
    const int sub = lane / LANES, u = lane % LANES, ch_in = 32 * half + u * E;
    int fb = b0, fs = 0;
    auto fetch = [&]() {
        if (fb < b1 && p.base) {
            const int ch = fb * BLOCK + ch_in, left = p.M - ch;
            const T* from = (const T*)p.base + (long long)(mine0 + sub) * p.ldb + ch;
            uint8_t* to = place + fs * L::kStage;
            if (p.vec && (fb + 1) * BLOCK <= p.M) {
#pragma unroll
                for (int i = 0; i < 32; i += PER, from += PER * p.ldb)
                    if (i + sub < mine) copy16(smem_u32(to) + L::unit_at(i + sub, u), from);
            } else {
                for (int i = sub; i < mine; i += PER, from += PER * p.ldb) {
                    T* unit = reinterpret_cast<T*>(to + L::unit_at(i, u));
                    for (int e = 0; e < E; ++e) unit[e] = e < left ? from[e] : T(0.0f);
                }
            }
        }
        ++fb;
        copies_commit();
        if (++fs == L::kStages) fs = 0;
    };
    if (warp < 8)
        for (int i = 0; i < L::kStages - 1; ++i) fetch();
    // ---- weights of the next 64 channels: one thread ----
    int wb = b0;
    auto ask = [&]() {
        if (wb < b1 && !p.test_stall) {
            const int buf = (wb - b0) % MANY_B;
            mbar_arrive_expect_tx(&b_full[buf], (uint32_t)groups * 2048);
            bulk_g2s(smem + lay.z_bytes() + buf * lay.b_bytes(), p.B + (size_t)tile.slot * p.b_slot + (size_t)wb * groups * 2048, (uint32_t)groups * 2048, &b_full[buf]);
            ++wb;
        }
    };
    if (real && threadIdx.x == 8 * 32)
        for (int i = 0; i < MANY_B - 1; ++i) ask();

    // ---- z, scaled, as bf16 terms, each at its ranks behind those of the term before ----
    pdl_wait();
    if (real) {
        // (four lanes take 32 ranks of a row, two its 16: between loads of whole lines and stores without conflicts)
        const int rank_pad = p.groups * GROUP, wide = groups == 1 ? 2 : 4, across = (eights + wide - 1) / wide;
        const float factor = p.scales[tile.slot];
#pragma unroll 2
        for (int i = threadIdx.x; i < MANY_ROWS * across * wide; i += MANY_THREADS) {
            const int piece = i / (MANY_ROWS * wide), rest = i - piece * (MANY_ROWS * wide), r = rest / wide, eight = piece * wide + rest % wide;
            if (eight >= eights) continue;
            const int first = 8 * eight, have = r < tile.rows ? rank - first : 0;              // z is written for the adapter's own ranks only
            float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
            if (have > 0) {
                const float4* at = reinterpret_cast<const float4*>(p.z + (size_t)(row0 + r) * rank_pad + first);
                const float4 lo = __ldcg(at), hi = __ldcg(at + 1);
                const float c = factor * (p.x_scale ? p.x_scale[row0 + r] : 1.0f);
                v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w; v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = k < have ? v[k] * c : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < TERMS; ++k) {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = k + 1 == TERMS ? rounded(v[2 * j], v[2 * j + 1]) : cut(v[2 * j], v[2 * j + 1]);
                *reinterpret_cast<uint4*>(smem + (k * eights + eight) * 2048 + r * 16) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
    fence_proxy_async_smem();
    __syncthreads();

    bool ok = true;
    if (warp == 8) {
        // ================= products =================
        if (real && lane == 0) {
            const uint64_t desc_z = umma_desc_k_plain(smem_u32(smem), 2048, 128), desc_b = umma_desc_k_plain(smem_u32(smem + lay.z_bytes()), 1024, 128);
            constexpr uint32_t kDesc = idesc_bf16(MANY_ROWS, BLOCK);
            for (int job = 0; job < b1 - b0; ++job) {
                const int buf = job % MANY_B, d = job % MANY_D;
                // (the place of the weights after next was the last one's)
                if (job > 0 && !(ok = mbar_wait(&b_done[(job - 1) % MANY_B], (uint32_t)((job - 1) / MANY_B & 1), ctl))) break;
                ask();
                if (!(ok = mbar_wait(&b_full[buf], (uint32_t)(job / MANY_B & 1), ctl))) break;
                if (!(ok = mbar_wait(&d_free[d], (uint32_t)(job / MANY_D & 1) ^ 1, ctl))) break;
                tc_fence_after_sync();
                const uint64_t weights = desc_b + (uint32_t)(buf * (lay.b_bytes() >> 4));
                for (int k = TERMS - 1; k >= 0; --k)
                    for (int i = 0; i < groups; ++i)
                        umma_bf16_ss(tmem + 64u * d, desc_z + (uint32_t)((k * groups + i) * (4096 >> 4)), weights + (uint32_t)(i * (2048 >> 4)), kDesc,
                                     k != TERMS - 1 || i > 0);
                umma_commit(&b_done[buf]);
                umma_commit(&d_full[d]);
            }
            // every copy has landed and every product ended before the block does
            if (!ok)
                for (int i = 0; i < MANY_B; ++i)
                    if (wb - b0 > i) mbar_drain(&b_full[i], (uint32_t)((wb - b0 - 1 - i) / MANY_B & 1));
            umma_commit(&drained);
            mbar_drain(&drained, 0);
        }
        __syncwarp();
    } else {
        // ================= rows: one a thread =================
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + 4u * half;
        int stage = 0;
        for (int b = b0; b < b1; ++b) {
            const int job = b - b0, d = job % MANY_D;
            uint32_t v[8][4] = {};                           // channel 8 n + j is column 8 j + n: [j][n % 4] of the half's n
            if (real) {
                if (!(ok = mbar_wait_warp(&d_full[d], (uint32_t)(job / MANY_D & 1), ctl))) break;
                tc_fence_after_sync();
#pragma unroll
                for (int j = 0; j < 8; ++j) tmem_ld4(lanes + 64u * d + 8u * j, v[j]);
                tmem_ld_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&d_free[d]);
            }
            uint8_t* here = place + stage * L::kStage;
            copies_wait<L::kStages - 2>();
            __syncwarp();
            if (lane < mine) {
#pragma unroll
                for (int n = 0; n < 4; ++n) {
#pragma unroll
                    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
                        uint4* unit = reinterpret_cast<uint4*>(here + L::unit_at(lane, n * ((int)sizeof(T) / 2) + h));
                        uint4 x = p.base ? *unit : make_uint4(0, 0, 0, 0);
                        uint32_t* w = reinterpret_cast<uint32_t*>(&x);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            if constexpr (sizeof(T) == 2)
                                w[k] = rounded(__uint_as_float(w[k] << 16) + __uint_as_float(v[2 * k][n]),
                                               __uint_as_float(w[k] & 0xffff0000u) + __uint_as_float(v[2 * k + 1][n]));
                            else
                                w[k] = __float_as_uint(__uint_as_float(w[k]) + __uint_as_float(v[4 * h + k][n]));
                        }
                        *unit = x;
                    }
                }
            }
            __syncwarp();
            const int ch = b * BLOCK + ch_in, left = p.M - ch;
            T* to = (T*)p.out + (long long)(mine0 + sub) * p.ldo + ch;
            if (p.vec && (b + 1) * BLOCK <= p.M) {
                uint4 x[32 / PER];
#pragma unroll
                for (int i = 0; i < 32; i += PER) x[i / PER] = *reinterpret_cast<const uint4*>(here + L::unit_at(i + sub, u));
#pragma unroll
                for (int i = 0; i < 32; i += PER, to += PER * p.ldo)
                    if (i + sub < mine) *reinterpret_cast<uint4*>(to) = x[i / PER];
            } else {
                for (int i = sub; i < mine; i += PER, to += PER * p.ldo)
                    for (int e = 0; e < E; ++e)
                        if (e < left) to[e] = reinterpret_cast<const T*>(here + L::unit_at(i, u))[e];
            }
            __syncwarp();
            fetch();
            if (++stage == L::kStages) stage = 0;
        }
        copies_wait<0>();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (threadIdx.x == 0 && ctl[0]) atomicOr(p.rows.status, KV4_DEV_TIMEOUT);
    if (warp == 8) tmem_dealloc(tmem, MANY_D * 64);
}

// ---- both in one launch, for few rows ---------------------------------------------------------------------------------------
// A cluster of blocks takes up to eight rows.  The adapters that they ask for, one after another, are cut into equal runs of
// chunks of columns for its warps, and then into runs of blocks of channels: a warp reads a few long pieces.  Its copies run through
// both products, so that while the parts of z are added up and exchanged (each block writes its part to every block's shared
// memory: one cluster barrier), the first weights of the second product are on their way.  Against two launches this saves a
// launch, the way of z through memory, and the second search for the rows' adapters.

constexpr int FEW_WARPS = 12, FEW_ROWS = 8, FEW_GROUPS = 4;      // (of more than 64 ranks shared memory holds too few stages)

struct FewParams {
    DownParams d;
    UpParams u;
    int cluster, rows;       // blocks; rows of a cluster
};

// A stage of a warp's ring: weights (of one adapter; chunks as a whole, blocks in groups of ranks), then x of the chunks, or base of
// the block whose last groups they are.  G: groups of ranks at most.
template <typename T, typename O, int G>
struct FewStage {
    static constexpr int chunks = G == 1 ? 2 : 1, units = G == 4 ? 2 : 1, weights = G == 1 ? 2048 : G * 1024;
    static constexpr int bytes = weights + (chunks * 32 * kXBytes<T> > kBaseBytes<O> ? chunks * 32 * kXBytes<T> : kBaseBytes<O>);
    static constexpr int stages = G <= 2 ? 4 : sizeof(O) == 4 ? 2 : 3, ring = FEW_WARPS * stages * bytes;
    static size_t smem(int cluster) { return (size_t)ring + (size_t)(FEW_WARPS + cluster) * FEW_ROWS * G * GROUP * sizeof(float); }
};

template <typename T, typename O, int G>
__global__ void __launch_bounds__(FEW_WARPS * 32, 1)
adapter_few_kernel(const FewParams p)
{
    constexpr int TERMS = kTerms<O>, Z = 256 * TERMS, MOST = FEW_ROWS + 1;
    extern __shared__ __align__(16) uint8_t smem[];
    // the adapters asked for, and behind them (slot kNoAdapter) the rows without one, whose base is copied
    __shared__ int slot_s[FEW_ROWS], entry_slot[MOST], entry_groups[MOST], entries_s, all_s;
    __shared__ unsigned entry_mask[MOST];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int rank = p.cluster > 1 ? (int)ptx::cluster_ctarank() : 0, row0 = (int)(blockIdx.x / (unsigned)p.cluster) * p.rows;
    using St = FewStage<T, O, G>;
    constexpr int rank_pad = G * GROUP, numbers = FEW_ROWS * rank_pad;
    uint8_t* ring = smem + warp * St::stages * St::bytes;
    float* parts = reinterpret_cast<float*>(smem + St::ring);           // [warp][row][rank_pad]
    float* z_all = parts + FEW_WARPS * numbers;                          // [block of the cluster][row][rank_pad]
    uint8_t* zs = reinterpret_cast<uint8_t*>(parts);                     // over the parts, once they are added up: [group][Z]
    pdl_wait();
    pdl_launch_dependents();
    if (p.cluster > 1) asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");               // (its blocks have all begun)
    {
        Rows mine = p.d.rows;
        mine.n_rows = min(mine.n_rows, row0 + p.rows);
        find_slots<FEW_ROWS, FEW_WARPS>(mine, row0, slot_s);
    }
    if (warp == 0) {
        const int slot = lane < FEW_ROWS ? slot_s[lane] : kNoRow;
        const unsigned same = __match_any_sync(0xffffffffu, slot);
        const bool leads = slot >= 0 && lane == __ffs(same) - 1;
        const unsigned leaders = __ballot_sync(0xffffffffu, leads), none = __ballot_sync(0xffffffffu, slot == kNoAdapter);
        const int n = __popc(leaders);
        if (leads) {
            const int e = __popc(leaders & ((1u << lane) - 1));
            entry_slot[e] = slot;
            entry_mask[e] = same;
            entry_groups[e] = (p.d.rows.ranks[slot] + GROUP - 1) / GROUP;
        }
        if (lane == 0) {
            entries_s = n;
            all_s = n + (none && !p.u.in_place);
            entry_slot[n] = kNoAdapter;
            entry_groups[n] = 0;
            entry_mask[n] = none;
        }
    }
    __syncthreads();
    const int entries = entries_s, all = all_s, of = p.cluster * FEW_WARPS, me = rank * FEW_WARPS + warp;

    // A warp's run of (adapter, chunk) or (adapter, block), by weight: from (e, at) on, of `left` weight.
    struct Run { int e, at, end, stop; };          // at, end: in adapter e; stop: weight where the run ends
    auto weight_of = [&](int e, bool up) { return up ? entry_groups[e] + 1 : entry_groups[e]; };
    auto enter = [&](Run& r, int before, bool up) {          // the run's part of adapter r.e, which begins at weight `before`
        const int count = up ? p.u.blocks : p.d.chunks, w = weight_of(r.e, up);
        r.end = min(count, (r.stop - before + w - 1) / w);
    };
    auto begin = [&](bool up) {
        const int n = up ? all : entries, count = up ? p.u.blocks : p.d.chunks;
        unsigned total = 0;                                  // (below 2^24, and `of` below 2^7)
        for (int e = 0; e < n; ++e) total += (unsigned)(weight_of(e, up) * count);
        const int start = (int)(total * (unsigned)me / (unsigned)of);
        Run r{0, 0, 0, (int)(total * (unsigned)(me + 1) / (unsigned)of)};
        int before = 0;
        for (; r.e < n; ++r.e) {
            const int w = weight_of(r.e, up);
            r.at = max(0, (start - before + w - 1) / w);
            enter(r, before, up);
            if (r.at < r.end || before >= r.stop) break;
            before += w * count;
        }
        if (r.e >= n || r.at >= r.end) r.e = n;
        r.stop -= before;                                    // from here on counted from adapter e's begin
        return r;
    };
    auto advance = [&](Run& r, bool up) {                    // behind r.end: the next adapter's part, or e = n
        const int n = up ? all : entries, count = up ? p.u.blocks : p.d.chunks;
        r.stop -= weight_of(r.e, up) * count;
        ++r.e;
        r.at = 0;
        if (r.e >= n || r.stop <= 0) { r.e = n; return; }
        enter(r, 0, up);
    };

    // ---- the copies ----
    const Run first_up = begin(true);
    Run run = begin(false);
    bool up = run.e == entries;
    if (up) run = first_up;
    Run mine = run, mine_up = first_up;
    const bool has_down = !up;
    int unit = 0, fs = 0;                                    // up: the groups of the block that are on their way
    // of the run's adapter: its groups, whether this lane's row is its (up: bits of its two rows), its weights, and x or base
    int f_groups = 0;
    unsigned f_rows = 0;
    const uint8_t* f_weights = nullptr;
    const T* f_x = nullptr;
    const O* f_base = nullptr;
    const uint32_t a_put = (uint32_t)a_place(lane & 7, lane >> 3);
    auto aim = [&]() {
        if (run.e >= (up ? all : entries)) return;
        f_groups = entry_groups[run.e];
        f_rows = entry_mask[run.e] >> (up ? 2 * t : g);
        if (up) {
            f_weights = p.u.B + (size_t)entry_slot[run.e] * p.u.b_slot + (size_t)run.at * f_groups * 2048 + lane * 16;
            f_base = (const O*)p.u.base + (long long)(row0 + 2 * t) * p.u.ldb + run.at * BLOCK + 8 * g;
        } else {
            f_weights = p.d.A + (size_t)entry_slot[run.e] * p.d.a_slot + (size_t)run.at * f_groups * 1024 + lane * 16;
            f_x = (const T*)p.d.x + (long long)(row0 + g) * p.d.ldx + run.at * CHUNK + 8 * t;
        }
    };
    auto fetch = [&]() {
        uint8_t* to = ring + fs * St::bytes;
        const uint32_t to32 = ptx::smem_u32(to) + lane * 16;
        if (!up) {
            const int n = min(St::chunks, run.end - run.at);
#pragma unroll
            for (int i = 0; i < St::weights / 512; ++i)
                if (i < 2 * n * f_groups) copy16(ptx::smem_u32(to) + a_put + i * 512, f_weights + i * 512);
            f_weights += n * f_groups * 1024;
            const bool whole = p.d.aligned && (run.at + n) * CHUNK <= p.d.N;
            for (int c = 0; c < n; ++c, f_x += CHUNK) {
                uint8_t* dst = to + St::weights + c * 32 * kXBytes<T>;
                if (whole) {
                    if (f_rows & 1) {
                        if constexpr (sizeof(T) == 1) {
                            copy8(to32 - lane * 8 + (uint32_t)(St::weights + c * 32 * kXBytes<T>), f_x);
                        } else {
#pragma unroll
                            for (int i = 0; i < kXBytes<T> / 16; ++i) copy16(to32 + (uint32_t)(St::weights + c * 32 * kXBytes<T>) + i * 512, f_x + i * (16 / (int)sizeof(T)));
                        }
                    }
                } else if (f_rows & 1) {
                    const int col = (run.at + c) * CHUNK + 8 * t;
                    copy_x<T>(dst, p.d.x, p.d.ldx, row0 + g, p.d.rows.n_rows, col, p.d.N - col, p.d.aligned, lane);
                }
            }
            if ((run.at += n) >= run.end) {
                advance(run, false);
                if (run.e == entries) { up = true; run = first_up; }
                aim();
            }
        } else if (run.e < all) {
            const int n = min(St::units, f_groups - unit);
#pragma unroll
            for (int i = 0; i < 4 * St::units; ++i)
                if (i < 4 * n) copy16(to32 + i * 512, f_weights + i * 512);
            f_weights += n * 2048;
            unit += n;
            if (unit >= f_groups) {                          // with the block's last ones, base
                if (p.u.base)
                    copy_base<O>(to + St::weights, f_base, p.u.ldb, f_rows, p.u.M - run.at * BLOCK - 8 * g, p.u.vec && (run.at + 1) * BLOCK <= p.u.M, lane);
                f_base += BLOCK;
                unit = 0;
                if (++run.at >= run.end) { advance(run, true); aim(); }
            }
        }
        copies_commit();
        if (++fs == St::stages) fs = 0;
    };
    aim();
    // (a stage's copies are one group, and stages - 2 groups may follow the one that is needed)
    auto arrived = [&]() { copies_wait<St::stages - 2>(); };
    int stage = 0;
    auto done = [&]() {
        fetch();
        if (++stage == St::stages) stage = 0;
    };
    for (int i = 0; i < St::stages - 1; ++i) fetch();
    for (int i = lane; i < numbers; i += 32) parts[warp * numbers + i] = 0.0f;
    __syncwarp();

    // ---- parts of z ----
    if (has_down)
        while (mine.e < entries) {
            const int groups = entry_groups[mine.e];
            const unsigned mask = entry_mask[mine.e];
            float acc[G][4];
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[i][k] = 0.0f;
            while (mine.at < mine.end) {
                const int n = min(St::chunks, mine.end - mine.at);
                arrived();
                __syncwarp();                                    // (weights are the other lanes' copies too)
                const uint8_t* from = ring + stage * St::bytes;
                for (int c = 0; c < n; ++c) {
                    Terms<T> x{};
                    if (mask >> g & 1) x.read(from + St::weights + c * 32 * kXBytes<T> + lane * (sizeof(T) == 1 ? 8 : 16));
#pragma unroll
                    for (int i = 0; i < G; ++i)
                        if (i < groups) {
                            const uint8_t* w = from + (c * groups + i) * 1024 + a_place(g, t);
                            const uint4 a0 = *reinterpret_cast<const uint4*>(w), a1 = *reinterpret_cast<const uint4*>(w + 512);
#pragma unroll
                            for (int k = Terms<T>::n - 1; k >= 0; --k) mma_a(acc[i], a0, a1, x.w[k]);
                        }
                }
                mine.at += n;
                done();
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int row = 2 * t + (k & 1);
                if (mask >> row & 1)
#pragma unroll
                    for (int i = 0; i < G; ++i)
                        if (i < groups) parts[warp * numbers + row * rank_pad + i * GROUP + g + (k & 2 ? 8 : 0)] = acc[i][k];
            }
            advance(mine, false);
        }
    __syncwarp();
    if (p.cluster > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    __syncthreads();
    for (int i = threadIdx.x; i < numbers; i += FEW_WARPS * 32) {
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) sum += parts[w * numbers + i];
        if (p.cluster > 1) {
            const uint32_t at = ptx::smem_u32(z_all + rank * numbers + i);
            for (int c = 0; c < p.cluster; ++c)
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(ptx::cluster_map_u32(at, (uint32_t)c)), "f"(sum) : "memory");
        } else {
            z_all[i] = sum;
        }
    }
    if (p.cluster > 1) ptx::cluster_sync_all();
    else __syncthreads();

    // ---- z, scaled, as bf16 terms in the order of the product's second operand ----
    for (int i = threadIdx.x; i < G * 32; i += FEW_WARPS * 32) {
        const int ln = i & 31, group = i >> 5, row = ln >> 2, slot = slot_s[row];
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (slot >= 0) {
            for (int c = 0; c < p.cluster; ++c) {
                const float4 u = *reinterpret_cast<const float4*>(z_all + c * numbers + row * rank_pad + group * GROUP + 4 * (ln & 3));
                v[0] += u.x; v[1] += u.y; v[2] += u.z; v[3] += u.w;
            }
            const float c = p.u.scales[slot] * (p.u.x_scale ? p.u.x_scale[row0 + row] : 1.0f);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] *= c;
        }
        ZTerms<TERMS> z;
        z.make(v);
        z.put(zs + group * Z, ln);
    }
    __syncthreads();

    while (mine_up.e < all) {
        const int groups = entry_groups[mine_up.e];
        const unsigned rows = entry_mask[mine_up.e] >> (2 * t);
        O* out = (O*)p.u.out + (long long)(row0 + 2 * t) * p.u.ldo + mine_up.at * BLOCK + 8 * g;
        for (; mine_up.at < mine_up.end; ++mine_up.at, out += BLOCK) {
            Sums<O> sums;
            int i = 0;
            do {
                arrived();
                __syncwarp();                                    // (weights are the other lanes' copies too)
                const uint8_t* from = ring + stage * St::bytes;
                const int n = G == 1 ? min(1, groups) : min(St::units, groups - i);
                if (p.u.base && i + n >= groups && (i == 0 || sizeof(O) == 4)) {
                    // the block's last stage brings base
                    float kept[4][4];
                    if (i > 0) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
#pragma unroll
                            for (int k = 0; k < 4; ++k) kept[q][k] = sums.acc[q][k];
                    }
                    sums.begin(from + St::weights, lane);
                    if (i > 0) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
#pragma unroll
                            for (int k = 0; k < 4; ++k) sums.acc[q][k] = kept[q][k];
                    }
                } else if (i == 0) {
                    sums = Sums<O>{};
                } else if (p.u.base && i + n >= groups) {
                    Sums<O> b;
                    b.begin(from + St::weights, lane);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int k = 0; k < 4; ++k) sums.acc[q][k] += b.acc[q][k];
                }
                for (int c = 0; c < n; ++c, ++i) {
                    ZTerms<TERMS> z;
                    z.get(zs + i * Z, lane);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint4 w = b_rows(from + c * 2048, q, lane);
#pragma unroll
                        for (int k = TERMS - 1; k >= 0; --k) mma_bf16(sums.acc[q], w, z.w[k][0], z.w[k][1]);
                    }
                }
                if (i >= groups) sums.store(out, p.u.ldo, rows, p.u.M - mine_up.at * BLOCK - 8 * g, p.u.vec && (mine_up.at + 1) * BLOCK <= p.u.M);
                done();
            } while (i < groups);
        }
        advance(mine_up, true);
    }
    copies_wait<0>();
}

// ---- launches ---------------------------------------------------------------------------------------------------------------

bool off(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) != 0; }

template <typename T, int NT, int RG>
size_t down_smem(int groups)
{
    return (size_t)DOWN_WARPS * (kDownStages<T, NT, RG> * kDownStage<T, NT, RG> + 8 * NT * (groups < DOWN_GROUPS ? groups : DOWN_GROUPS) * GROUP * sizeof(float));
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
    if (e == cudaSuccess) e = prepare_down<T, 4, 1>();
    if (e == cudaSuccess) e = prepare_down<T, 4, 2>();
    if (e == cudaSuccess) e = prepare_down<T, 4, 4>();
    return e;
}
template <typename T, int NT, int RG>
cudaError_t down(const DownParams& p, cudaStream_t st)
{
    PdlLaunch l((unsigned)((p.rows.n_rows + 8 * NT - 1) / (8 * NT)), DOWN_WARPS * 32, down_smem<T, NT, RG>(p.groups), st);
    cudaLaunchAttribute attr[2] = {l.attr[0], {}};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = attr[1].val.clusterDim.z = 1;
    attr[1].val.clusterDim.y = (unsigned)p.splits;
    l.cfg.attrs = attr;
    l.cfg.numAttrs = p.splits > 1 ? 2 : 1;
    l.cfg.gridDim.y = (unsigned)p.splits;
    l.cfg.gridDim.z = (unsigned)(p.groups + DOWN_GROUPS - 1) / DOWN_GROUPS;
    return cudaLaunchKernelEx(&l.cfg, adapter_down_kernel<T, NT, RG>, p);
}

// Sequences cut into tiles: as many as there are if all have the same length, and how many there are at most.
struct Tiles { int about, most; };
Tiles tiles_of(const Rows& r)
{
    const int each = (r.n_rows + r.n_seq - 1) / r.n_seq;
    return {r.n_seq * ((each + MANY_ROWS - 1) / MANY_ROWS), r.n_rows / MANY_ROWS + r.n_seq};
}

template <typename T>
cudaError_t down_many(DownParams& p, int sms, cudaStream_t st)
{
    // Blocks that share a contraction: as many as run in one round with the other tiles', and as there are stages for.
    const size_t smem = DownMany<T>::smem(p.groups);
    const Tiles tiles = tiles_of(p.rows);
    const int at_once = (smem <= 109 * 1024 ? 2 : 1) * sms, stages = (p.chunks + 1) / 2;
    p.splits = 1;
    while (p.splits < MAX_SPLITS && 2 * p.splits <= stages && (long long)tiles.about * p.splits * 2 <= at_once) p.splits *= 2;
    PdlLaunch l((unsigned)tiles.most, MANY_THREADS, smem, st);                       // (those of tiles that are not there come last)
    cudaLaunchAttribute attr[2] = {l.attr[0], {}};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = attr[1].val.clusterDim.z = 1;
    attr[1].val.clusterDim.y = (unsigned)p.splits;
    l.cfg.attrs = attr;
    l.cfg.numAttrs = p.splits > 1 ? 2 : 1;
    l.cfg.gridDim.y = (unsigned)p.splits;
    return cudaLaunchKernelEx(&l.cfg, adapter_down_many_kernel<T>, p);
}

template <typename T>
cudaError_t down_type(const DownParams& p, bool wide, cudaStream_t st)
{
    const int rg = p.groups == 1 ? 1 : p.groups == 2 ? 2 : 4;
    if (wide) return rg == 1 ? down<T, 4, 1>(p, st) : rg == 2 ? down<T, 4, 2>(p, st) : down<T, 4, 4>(p, st);
    return rg == 1 ? down<T, 1, 1>(p, st) : rg == 2 ? down<T, 1, 2>(p, st) : down<T, 1, 4>(p, st);
}

template <typename T, typename O>
cudaError_t prepare_few()
{
    for (const void* kernel : {(const void*)adapter_few_kernel<T, O, 1>, (const void*)adapter_few_kernel<T, O, 2>, (const void*)adapter_few_kernel<T, O, 4>})
        if (const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024); e != cudaSuccess) return e;
    return cudaSuccess;
}

struct FewLaunch {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    FewLaunch(unsigned tiles, int cluster, size_t smem, cudaStream_t st)
    {
        cfg.gridDim = dim3(tiles * (unsigned)cluster);
        cfg.blockDim = dim3(FEW_WARPS * 32);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)cluster;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = cluster > 1 ? 2 : 1;
    }
};

template <typename T, typename O, int G>
cudaError_t few_as(const FewParams& p, unsigned tiles, cudaStream_t st)
{
    FewLaunch l(tiles, p.cluster, FewStage<T, O, G>::smem(p.cluster), st);
    return cudaLaunchKernelEx(&l.cfg, adapter_few_kernel<T, O, G>, p);
}
template <typename T, typename O>
cudaError_t few_ranks(const FewParams& p, unsigned tiles, cudaStream_t st)
{
    return p.d.groups == 1 ? few_as<T, O, 1>(p, tiles, st) : p.d.groups == 2 ? few_as<T, O, 2>(p, tiles, st) : few_as<T, O, 4>(p, tiles, st);
}
template <typename T>
cudaError_t few(const FewParams& p, unsigned tiles, bool out_f32, cudaStream_t st)
{
    return out_f32 ? few_ranks<T, float>(p, tiles, st) : few_ranks<T, __nv_bfloat16>(p, tiles, st);
}

cudaError_t prepare()
{
    cudaError_t e = prepare_type<float>();
    if (e == cudaSuccess) e = prepare_type<__nv_bfloat16>();
    if (e == cudaSuccess) e = prepare_type<int8_t>();
    if (e == cudaSuccess) e = prepare_few<float, float>();
    if (e == cudaSuccess) e = prepare_few<float, __nv_bfloat16>();
    if (e == cudaSuccess) e = prepare_few<__nv_bfloat16, float>();
    if (e == cudaSuccess) e = prepare_few<__nv_bfloat16, __nv_bfloat16>();
    if (e == cudaSuccess) e = prepare_few<int8_t, float>();
    if (e == cudaSuccess) e = prepare_few<int8_t, __nv_bfloat16>();
    for (const void* kernel : {(const void*)adapter_up_kernel<float, 1>, (const void*)adapter_up_kernel<float, 2>, (const void*)adapter_up_kernel<float, 4>,
                               (const void*)adapter_up_kernel<float, 8>, (const void*)adapter_up_kernel<__nv_bfloat16, 1>,
                               (const void*)adapter_up_kernel<__nv_bfloat16, 2>, (const void*)adapter_up_kernel<__nv_bfloat16, 4>,
                               (const void*)adapter_up_kernel<__nv_bfloat16, 8>, (const void*)adapter_many_kernel<float>,
                               (const void*)adapter_many_kernel<__nv_bfloat16>, (const void*)adapter_down_many_kernel<float>,
                               (const void*)adapter_down_many_kernel<__nv_bfloat16>, (const void*)adapter_down_many_kernel<int8_t>})
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024);
    return e;
}

constexpr int kUpStatic = 2560;      // shared memory that the second kernel declares, and what the system keeps of a block's
template <typename T, int G>
cudaError_t up(UpParams& p, int sms, cudaStream_t st)
{
    // Channel blocks a warp: so many that the blocks run in one round (they read z again each), as many an SM as registers and shared memory
    // leave, and four or three where those leave more.  With four or three whatever they leave, fp32 results and ranks above 64 took rounds
    // more: 4096 to 4096, 4000 rows by 20, ranks of 128, 262 us in place of 224 (fp32 383 and 344); 700 single rows of rank 64 in fp32 280 and
    // 239; 300 by 10, ranks of 128, whose second round was eight blocks, 50.4 in place of 53.3.
    const size_t smem = (size_t)(p.tile_rows + 15) / 16 * 2 * p.groups * 256 * kTerms<T> + (size_t)UP_WARPS * (p.groups * 2048 + 2 * UP_STAGES * kBaseBytes<T>);
    const int fit = (int)(TSVD_SM_SMEM / (smem + kUpStatic)), most = p.groups <= 2 ? 4 : 3;
    const int at_once = sms * std::max(1, std::min({fit, kUpBlocks<T, G>, most}));
    const int tiles = (p.rows.n_rows + p.tile_rows - 1) / p.tile_rows;
    auto columns = [&] { return (p.blocks + UP_WARPS * p.per_warp - 1) / (UP_WARPS * p.per_warp); };
    p.per_warp = 1;
    while ((long long)tiles * columns() > at_once && p.per_warp < p.blocks) ++p.per_warp;
    PdlLaunch l((unsigned)tiles, UP_WARPS * 32, smem, st);
    l.cfg.gridDim.y = (unsigned)columns();
    return cudaLaunchKernelEx(&l.cfg, adapter_up_kernel<T, G>, p);
}

template <typename T>
cudaError_t up_type(UpParams& p, int sms, cudaStream_t st)
{
    return p.groups == 1 ? up<T, 1>(p, sms, st) : p.groups == 2 ? up<T, 2>(p, sms, st) : p.groups <= 4 ? up<T, 4>(p, sms, st) : up<T, 8>(p, sms, st);
}

template <typename T>
cudaError_t up_many(UpParams& p, int sms, cudaStream_t st)
{
    // Blocks of channels of a block of threads: so many that all run in one round.
    const Many<T> lay{p.groups};
    const Tiles tiles = tiles_of(p.rows);
    const int at_once = (lay.smem() <= 109 * 1024 ? 2 : 1) * sms;
    p.per_warp = (int)(((long long)p.blocks * tiles.about + at_once - 1) / at_once);
    while ((long long)tiles.about * ((p.blocks + p.per_warp - 1) / p.per_warp) > at_once && p.per_warp < p.blocks) ++p.per_warp;
    p.columns = (p.blocks + p.per_warp - 1) / p.per_warp;
    PdlLaunch l((unsigned)(tiles.most * p.columns), MANY_THREADS, lay.smem(), st);         // (those of tiles that are not there come last)
    return cudaLaunchKernelEx(&l.cfg, adapter_many_kernel<T>, p);
}

struct Shape {
    bool wide;           // the first kernel's tiles have 32 rows, else 8
    int splits;          // blocks that share a contraction
};
// Tiles of 32 rows where sequences fill them, or where there are many: a tile goes over the columns once for each of its adapters, and with
// tiles of 8 the weights are read four times as often.  Both products, 4096 to 4096, tiles of 8 and of 32: 900 rows by 20 for each sequence,
// ranks of 32, 32.9 and 41.5 us; 300 by 10, ranks of 128, 53.3 and 62.4; 200 by 50, ranks of 128, 28.5 and 26.5; 4000 by 30, ranks of 16, 53.2
// and 50.6.
Shape shape_of(const tsvd_adapters_s* h, int rows, int n_seq)
{
    Shape s;
    s.wide = rows >= 4000 || (rows >= 192 && rows / n_seq >= 32);
    const int tiles = (rows + (s.wide ? 31 : 7)) / (s.wide ? 32 : 8);
    // wide: one block an SM, in one round; else two; a chunk for every warp
    const int want = s.wide ? (h->sms > tiles ? h->sms / tiles : 1) : (2 * h->sms + tiles - 1) / tiles, most = (h->chunks + DOWN_WARPS - 1) / DOWN_WARPS;
    s.splits = want < most ? want : most;
    if (s.splits > MAX_SPLITS) s.splits = MAX_SPLITS;
    return s;
}
// How the kernel for few rows serves a call of so many, if it does (else cluster = 0): clusters of as many blocks as have a chunk
// or a block of channels for each of their warps, eight at most, or half or a quarter of that where this lets more blocks run; as few
// rows each as are served by the clusters that run at a time (a second round would cost what the other kernels' second launch does).
struct Few { int cluster, rows; };
Few few_of(const tsvd_adapters_s* h, int rows)
{
    if (h->groups > FEW_GROUPS) return {0, 0};
    const int work = h->chunks > h->blocks ? h->chunks : h->blocks;
    int most = 1;
    while (most < 8 && most * FEW_WARPS < work) most *= 2;
    Few best{0, 0};
    int blocks = 0;
    for (int c = most; c >= 1 && 4 * c >= most; c /= 2)
        for (int r = 1; r <= FEW_ROWS; r *= 2) {
            const int clusters = (rows + r - 1) / r;
            if (clusters > h->few[c]) continue;
            if (clusters * c > blocks) { best = {c, r}; blocks = clusters * c; }
            break;
        }
    return best;
}
// The kernels on tcgen05 where sequences have rows for a tile of 128, as far as their number tells: half of one, a quarter where ranks above
// 48 make the warps' products long.  2048 rows by 64 and 32 for each sequence, 2048 to 8192, ranks of 16: 30 and 48 us against 32 and 34; 4096 to
// 4096, ranks of 32, 1024 rows by 32 26.0 against 26.7; ranks of 64, 4000 rows by 50 and 20 63 and 135 against 96 and 117; of 128, 300 rows by 40 22
// against 44.
constexpr int MANY_FROM = 192;
bool many_rows(const tsvd_adapters_s* h, int rows, int n_seq) { return rows >= MANY_FROM && rows / n_seq >= (h->groups >= 4 ? 32 : 64); }
// What both could serve is the kernel's for few rows (512 rows of four sequences, 4096 to 4096, ranks of 16 10.8 us against 16.5, of 64 17.1
// against 19.4), but for adapters of half a megabyte and more where its clusters, each of which reads them, leave a third of the device idle
// (300 rows of three sequences: 4096 to 4096, ranks of 16 and 32 13.2 and 17.6 against 14.1 and 15.4; 4096 to 12288, ranks of 16, 32 and 64 21.8,
// 30.8 and 40.6 against 17.4, 18.4 and 20.2).
bool large(const tsvd_adapters_s* h) { return h->a_slot + h->b_slot >= 512 * 1024; }
bool prefers_many(const tsvd_adapters_s* h, const Few& how, int rows, int n_seq)
{
    return large(h) && many_rows(h, rows, n_seq) && 3 * ((rows + how.rows - 1) / how.rows) * how.cluster < 2 * h->sms;
}
size_t z_bytes(const tsvd_adapters_s* h, int rows) { return (size_t)rows * h->groups * GROUP * sizeof(float); }

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
    if (h->groups <= FEW_GROUPS)
        for (int c = 1; c <= 8 && e == cudaSuccess; c *= 2) {
            // (one block an SM, whatever the types)
            const size_t smem = h->groups == 1 ? FewStage<float, float, 1>::smem(c) : h->groups == 2 ? FewStage<float, float, 2>::smem(c) : FewStage<float, float, 4>::smem(c);
            FewLaunch l((unsigned)(h->sms / 8 * 8), c, smem, nullptr);
            l.cfg.numAttrs = 0;
            if (c > 1) { l.attr[0] = l.attr[1]; l.cfg.numAttrs = 1; }
            h->few[c] = h->sms;
            const void* kernel = h->groups == 1 ? (const void*)adapter_few_kernel<float, float, 1> : h->groups == 2 ? (const void*)adapter_few_kernel<float, float, 2>
                                                                                                       : (const void*)adapter_few_kernel<float, float, 4>;
            if (c > 1) e = cudaOccupancyMaxActiveClusters(&h->few[c], kernel, &l.cfg);
        }
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
    if (rows_max > MOST_ROWS) return TSVD_E_TOOBIG;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    const bool none = few_of(h, rows_max).cluster && (!large(h) || rows_max < MANY_FROM);          // no call of so many rows or fewer needs it
    return none ? TSVD_OK : grow(h, z_bytes(h, rows_max));
}

extern "C" tsvd_status_t tsvd_adapters_forward(tsvd_adapters_t h, const void* x, long long ldx, const float* x_scale, tsvd_dtype_t dtype,
                                               const void* base, long long ldb, void* out, long long ldo, tsvd_dtype_t out_dtype,
                                               const int* slots, const int* q_start, int n_seq, int n_rows, void* stream)
{
    return tsvd_adapters_forward_ex(h, x, ldx, x_scale, dtype, base, ldb, out, ldo, out_dtype, slots, q_start, n_seq, n_rows, 0, stream);
}

extern "C" tsvd_status_t tsvd_adapters_forward_ex(tsvd_adapters_t h, const void* x, long long ldx, const float* x_scale, tsvd_dtype_t dtype,
                                                  const void* base, long long ldb, void* out, long long ldo, tsvd_dtype_t out_dtype,
                                                  const int* slots, const int* q_start, int n_seq, int n_rows, unsigned flags, void* stream)
{
    if (!h) return TSVD_E_NULL;
    if (n_rows < 0 || n_seq < 1 || (!q_start && n_rows != n_seq) || ldx < h->N || (base && ldb < h->M) || ldo < h->M) return TSVD_E_SHAPE;
    if (n_rows > MOST_ROWS || n_seq > MOST_ROWS) return TSVD_E_TOOBIG;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16 && dtype != TSVD_I8) return TSVD_E_DTYPE;
    if (out_dtype != TSVD_F32 && out_dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (x_scale && dtype != TSVD_I8) return TSVD_E_DTYPE;
    if (flags & ~TSVD_FLAG_TEST_STALL) return TSVD_E_DTYPE;
    if (n_rows == 0) return TSVD_OK;
    if (!x || !out || !slots) return TSVD_E_NULL;
    const size_t size = dtype == TSVD_F32 ? 4 : dtype == TSVD_BF16 ? 2 : 1, out_size = out_dtype == TSVD_F32 ? 4 : 2;
    if (off(x, size) || off(base, out_size) || off(out, out_size) || off(x_scale, 4) || off(slots, 4) || off(q_start, 4)) return TSVD_E_ALIGN;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    cudaStream_t st = (cudaStream_t)stream;
    const Rows rows{slots, q_start, n_seq, n_rows, h->n_slots, h->ranks, h->dev_status};
    const size_t step = dtype == TSVD_I8 ? 8 : 16;
    DownParams d{rows, x, ldx, !off(x, step) && (n_rows == 1 || ldx * (long long)size % (long long)step == 0), h->N, h->chunks, 0, h->groups,
                 h->A, h->a_slot, nullptr, (flags & TSVD_FLAG_TEST_STALL) != 0};
    auto even = [&](const void* p, long long ld) { return !p || (!off(p, 16) && (n_rows == 1 || ld * (long long)out_size % 16 == 0)); };
    UpParams u{};
    u.rows = rows;
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
    u.test_stall = d.test_stall;
    if (const Few how = few_of(h, n_rows); how.cluster && !prefers_many(h, how, n_rows, n_seq)) {
        const FewParams f{d, u, how.cluster, how.rows};
        const unsigned tiles = (unsigned)((n_rows + how.rows - 1) / how.rows);
        if (dtype == TSVD_F32) TSVD_CUDA_OK(few<float>(f, tiles, out_dtype == TSVD_F32, st));
        else if (dtype == TSVD_BF16) TSVD_CUDA_OK(few<__nv_bfloat16>(f, tiles, out_dtype == TSVD_F32, st));
        else TSVD_CUDA_OK(few<int8_t>(f, tiles, out_dtype == TSVD_F32, st));
        tsvd_count_launch();
        return TSVD_OK;
    }
    const tsvd_status_t grown = grow(h, z_bytes(h, n_rows));
    if (grown != TSVD_OK) return grown;
    d.z = h->z;
    u.z = h->z;
    const bool many = many_rows(h, n_rows, n_seq);
    const Shape s = shape_of(h, n_rows, n_seq);
    d.splits = s.splits;
    // The first product there too: its time hardly grows with the rank, and a tile has one adapter (2048 rows of four sequences, 4096
    // columns, both products: ranks of 16, 32, 48 in 21.9, 21.9, 23.7 us against 20.5, 25.5, 31.2; five of 120 rows, 16 ranks, 13.0 against 18.0;
    // 8192 rows 47.6 against 55.3).  fp32 is turned into terms in registers, with fewer loads under way: ranks of 16 from 4096 rows
    // on (2048 rows 44 against 34, 8192 95 against 108).
    if (many && d.aligned && (dtype != TSVD_F32 || h->groups > 1 || n_rows >= 4096)) {
        if (dtype == TSVD_F32) TSVD_CUDA_OK(down_many<float>(d, h->sms, st));
        else if (dtype == TSVD_BF16) TSVD_CUDA_OK(down_many<__nv_bfloat16>(d, h->sms, st));
        else TSVD_CUDA_OK(down_many<int8_t>(d, h->sms, st));
    } else if (dtype == TSVD_F32) TSVD_CUDA_OK(down_type<float>(d, s.wide, st));
    else if (dtype == TSVD_BF16) TSVD_CUDA_OK(down_type<__nv_bfloat16>(d, s.wide, st));
    else TSVD_CUDA_OK(down_type<int8_t>(d, s.wide, st));
    tsvd_count_launch();

    // Rows of a tile: a warp's weights serve all of them, but with many sequences a tile holds many adapters, one after another, and
    // with few rows there are few tiles (8, 16, 64 rows: 32 single tokens with ranks of 128, 4096 to 4096, 45.9, 67.6, 109 us; 200 rows by 50
    // for each sequence 32.3, 26.4, 33.1; 900 by 20, ranks of 32, 40.1, 32.7, 36.9; 4000 by 30, ranks of 16, 80, 58, 51, fp32 318, 117, 88).
    u.tile_rows = n_rows >= 1024 ? UP_ROWS : n_rows >= 192 ? 16 : 8;
    if (many) {
        if (out_dtype == TSVD_F32) TSVD_CUDA_OK(up_many<float>(u, h->sms, st));
        else TSVD_CUDA_OK(up_many<__nv_bfloat16>(u, h->sms, st));
    } else if (out_dtype == TSVD_F32) TSVD_CUDA_OK(up_type<float>(u, h->sms, st));
    else TSVD_CUDA_OK(up_type<__nv_bfloat16>(u, h->sms, st));
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
    return (word & KV4_DEV_TIMEOUT) ? TSVD_E_TIMEOUT : word ? TSVD_E_INDEX : TSVD_OK;
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
