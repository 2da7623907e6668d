// Root-mean-square norm of rows, with the residual's addition ahead of it and, on request, a result in 8-bit rows.
//
//     h = round(x + r) to x's type,   rho = 1 / sqrt(mean h^2 + eps),   y = h rho w
//     in 8 bits:  t = h w,  a = max |t|,  q = rint(t ((1 / a) 127)),  scale = (a / 127) rho
//
// rho is one number a row, so it belongs into the scale: q is a function of t alone, elementwise in fp32, and the order in
// which the squares are summed cannot move a value to the next step.  A row is read once; its numbers stay in registers until
// its sum and its largest product, for which its threads meet once, are known.
//
// Bound by memory where rows are aligned and many: 8192 x 4096 bf16 with residual, 8 bits 39.7 us (copy bandwidth: 35.9), as numbers
// 42.6 (41.0); 2048 x 4096 11.1 (9.0) and 10.2 (10.2), fp32 17.1 (16.7).  A block goes on to further rows with its weights in
// registers and the next row's numbers on their way: with a block for each row, weights loaded behind the sum and two
// meetings, 2048 x 4096 took 16.9.  Rows off the boundaries are bound by the instructions that move single numbers (2048 x 4097 30 us, 9.0); few rows by the
// launch and two round trips to memory (one row of 4096 2.2 us).
#include <float.h>

#include <algorithm>

#include "rows8.cuh"
#include "serving.cuh"

namespace {

struct NormArgs {
    const void* x;
    const void* r;       // residual, or null
    void* h;             // x + r; null without a residual
    const void* w;
    void* y;             // the result as numbers; null: in 8 bits
    int8_t* q;
    float* scale;
    long long ldx, ldr, ldh, ldy, ldq;
    int rows, cols;
    int w_bf16;
    float eps;
};

// How the rows lie.  ALIGNED: on 16-byte boundaries, all of them and w; a thread's unit is 16 bytes.  PAIRS (bf16), SINGLES: on
// boundaries of two numbers, or anyhow; a unit is as many numbers, spread over the row two or one at a time, neighbouring
// threads on neighbouring ones.  (Cutting units out of aligned words, through registers or shared memory, gains on wide rows what it loses
// on narrow ones: 2048 x 1001 bf16 with residual to 8 bits 12.3 us in place of 9.0, 2048 x 4097 26 in place of 30.  Single numbers serve both.)
enum Mode { ALIGNED, PAIRS, SINGLES };

// The numbers of a unit, and back (rounded).
template <typename T, int E>
__device__ __forceinline__ void numbers(const uint4& u, float (&v)[E])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = __uint_as_float(E == 4 ? w[e] : e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
}
template <typename T, int E>
__device__ __forceinline__ uint4 unit_of(const float (&v)[E])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (E == 4) {
            w[i] = __float_as_uint(v[i]);
        } else {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A thread's unit: E numbers, of `threads` that share a row.
template <typename T, Mode MODE>
struct Place {
    static constexpr int E = 16 / (int)sizeof(T), S = MODE == ALIGNED ? E : MODE == PAIRS ? 2 : 1;    // S: in one piece
    int t, threads;
    __device__ __forceinline__ int col(int i, int e) const { return ((i * (E / S) + e / S) * threads + t) * S + e % S; }
    __device__ __forceinline__ uint4 load(const T* row, int i, int cols) const
    {
        if (MODE == ALIGNED && col(i, E - 1) < cols) return *reinterpret_cast<const uint4*>(row + col(i, 0));
        alignas(16) T u[E];
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            if (MODE == PAIRS && col(i, e + 1) < cols) {
                *reinterpret_cast<uint32_t*>(u + e) = *reinterpret_cast<const uint32_t*>(row + col(i, e));
            } else {
                u[e] = col(i, e) < cols ? row[col(i, e)] : T(0.0f);
                u[e + 1] = col(i, e + 1) < cols ? row[col(i, e + 1)] : T(0.0f);
            }
        }
        return *reinterpret_cast<uint4*>(u);
    }
    __device__ __forceinline__ void store(T* row, int i, int cols, uint4 v) const
    {
        if (MODE == ALIGNED && col(i, E - 1) < cols) { *reinterpret_cast<uint4*>(row + col(i, 0)) = v; return; }
        alignas(16) T u[E];
        *reinterpret_cast<uint4*>(u) = v;
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            if (MODE == PAIRS && col(i, e + 1) < cols) {
                *reinterpret_cast<uint32_t*>(row + col(i, e)) = *reinterpret_cast<uint32_t*>(u + e);
            } else {
                if (col(i, e) < cols) row[col(i, e)] = u[e];
                if (col(i, e + 1) < cols) row[col(i, e + 1)] = u[e + 1];
            }
        }
    }
    __device__ __forceinline__ void load_weight(const NormArgs& a, int i, float (&v)[E]) const
    {
        if (MODE == ALIGNED && col(i, E - 1) < a.cols) {
            if (a.w_bf16) {
                alignas(16) __nv_bfloat16 u[E];
                if constexpr (E == 8) *reinterpret_cast<uint4*>(u) = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)a.w + col(i, 0));
                else *reinterpret_cast<uint2*>(u) = *reinterpret_cast<const uint2*>((const __nv_bfloat16*)a.w + col(i, 0));
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = to_f32(u[e]);
            } else {
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const float4 u = *reinterpret_cast<const float4*>((const float*)a.w + col(i, e));
                    v[e] = u.x; v[e + 1] = u.y; v[e + 2] = u.z; v[e + 3] = u.w;
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                v[e] = col(i, e) >= a.cols ? 0.0f : a.w_bf16 ? to_f32(((const __nv_bfloat16*)a.w)[col(i, e)]) : ((const float*)a.w)[col(i, e)];
        }
    }
    // E 8-bit results, as rows8::quantised rounds them: 1.5 * 2^23 added to a small number rounds it to an integer (to even),
    // which is then in the low bits
    __device__ __forceinline__ void store8(int8_t* row, int i, int cols, const float (&v)[E], float inv) const
    {
        uint32_t b[E];
#pragma unroll
        for (int e = 0; e < E; ++e) b[e] = __float_as_uint(__fadd_rn(__fmul_rn(v[e], inv), 12582912.0f));
        if (MODE == ALIGNED && col(i, E - 1) < cols) {
            uint32_t w[E / 4];
#pragma unroll
            for (int j = 0; j < E / 4; ++j)
                w[j] = __byte_perm(__byte_perm(b[4 * j], b[4 * j + 1], 0x0040), __byte_perm(b[4 * j + 2], b[4 * j + 3], 0x0040), 0x5410);
            if constexpr (E == 8) *reinterpret_cast<uint2*>(row + col(i, 0)) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t*>(row + col(i, 0)) = w[0];
        } else {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                if (MODE == PAIRS && col(i, e + 1) < cols) {
                    *reinterpret_cast<uint16_t*>(row + col(i, e)) = (uint16_t)__byte_perm(b[e], b[e + 1], 0x0040);
                } else {
                    if (col(i, e) < cols) row[col(i, e)] = (int8_t)b[e];
                    if (col(i, e + 1) < cols) row[col(i, e + 1)] = (int8_t)b[e + 1];
                }
            }
        }
    }
};

__device__ __forceinline__ float max_or_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// Sum over the threads of a row, and the largest of `top` (not below 0; a NaN wins), the same in all of them.  One meeting of
// the block.
template <bool WARP, typename S>
__device__ __forceinline__ S row_sum(S v, float& top, S* sums, uint32_t* tops)
{
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(top) & 0x7fffffffu);
    if constexpr (!WARP) {
        const unsigned lane = threadIdx.x & 31;
        if (lane == 0) { sums[threadIdx.x >> 5] = v; tops[threadIdx.x >> 5] = m; }
        __syncthreads();
        v = lane < blockDim.x / 32 ? sums[lane] : S(0);
        m = __reduce_max_sync(0xffffffffu, lane < blockDim.x / 32 ? tops[lane] : 0u);
        for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        v = __shfl_sync(0xffffffffu, v, 0);
    }
    top = __uint_as_float(m);
    return v;
}

// Blocks of an SM, by the most threads that a block has (128: four rows of a warp each).  ALIGNED: 80 registers a thread, 64 for
// fp32, of which 16 bytes hold half as many numbers.
template <typename T, Mode MODE, int MOST, int NU>
constexpr int kBlocks = NU != 2 ? 512 / MOST : (MODE != ALIGNED || sizeof(T) == 4 ? 1024 : MOST == 512 ? 512 : 768) / MOST;

// A block takes a row, or (MOST = 128) each of its warps one; a thread NU units of it, held in registers.  ALIGNED: weights are
// held too, and the block goes on to the row a grid further on, whose numbers are asked for before this one's are summed up.
// NU = 0: rows of any length, read twice.
template <typename T, Mode MODE, int MOST, int NU, bool OUT8>
__global__ void __launch_bounds__(MOST, kBlocks<T, MODE, MOST, NU>)
rms_norm_kernel(const NormArgs a)
{
    using P = Place<T, MODE>;
    constexpr bool WARP = MOST == 128;
    constexpr int E = P::E, KEEP = NU ? NU : 1, WARPS = WARP ? 1 : MOST / 32;
    __shared__ float sums[2][WARPS];
    __shared__ double wide_sums[WARPS];
    __shared__ uint32_t tops[2][WARPS], no_tops[WARPS];
    pdl_launch_dependents();
    const P p{WARP ? (int)(threadIdx.x & 31) : (int)threadIdx.x, WARP ? 32 : (int)blockDim.x};
    const unsigned step = WARP ? gridDim.x * (blockDim.x >> 5) : gridDim.x;
    unsigned at = WARP ? blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    pdl_wait();
    float w[KEEP][E];
    uint4 x[KEEP], r[KEEP];
    auto ask = [&](long long row) {
#pragma unroll
        for (int i = 0; i < NU; ++i) x[i] = p.load((const T*)a.x + row * a.ldx, i, a.cols);
        if (a.r) {
#pragma unroll
            for (int i = 0; i < NU; ++i) r[i] = p.load((const T*)a.r + row * a.ldr, i, a.cols);
        }
    };
    if (at < (unsigned)a.rows) ask(at);
    if constexpr (NU > 0) {
#pragma unroll
        for (int i = 0; i < NU; ++i) p.load_weight(a, i, w[i]);
    }
    for (int turn = 0; at < (unsigned)a.rows; turn ^= 1, at += step) {
        const long long row = at;
        T* h = a.h ? (T*)a.h + row * a.ldh : nullptr;
        float v[KEEP][E];           // h; for 8 bits then t = h w
        float sum = 0.0f, top = 0.0f;
        auto take = [&](int i, float (&v)[E], const uint4& x, const uint4& r, const float (&w)[E]) {
            numbers<T>(x, v);
            if (a.r) {
                float u[E];
                numbers<T>(r, u);
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = __fadd_rn(v[e], u[e]);
                const uint4 sum16 = unit_of<T>(v);
                p.store(h, i, a.cols, sum16);
                numbers<T>(sum16, v);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                sum = fmaf(v[e], v[e], sum);
                if constexpr (OUT8) {
                    v[e] = __fmul_rn(v[e], w[e]);
                    top = max_or_nan(top, fabsf(v[e]));
                }
            }
        };
        // h once more (its own stores, where it wrote h)
        auto again = [&](int i, float (&v)[E]) { numbers<T>(p.load(a.r ? h : (const T*)a.x + row * a.ldx, i, a.cols), v); };
        const int units = NU ? NU : (a.cols + E * p.threads - 1) / (E * p.threads);
        if constexpr (NU > 0) {
#pragma unroll
            for (int i = 0; i < NU; ++i) take(i, v[i], x[i], r[i], w[i]);
            if (MODE == ALIGNED && at + step < (unsigned)a.rows) ask((long long)at + step);
        } else {
            for (int i = 0; i < units; ++i) {
                const uint4 x0 = p.load((const T*)a.x + row * a.ldx, i, a.cols);
                uint4 r0 = make_uint4(0, 0, 0, 0);
                if (a.r) r0 = p.load((const T*)a.r + row * a.ldr, i, a.cols);
                p.load_weight(a, i, w[0]);
                take(i, v[0], x0, r0, w[0]);
            }
        }
        sum = row_sum<WARP>(sum, top, sums[turn], tops[turn]);
        float rho = 1.0f / sqrtf(sum / (float)a.cols + a.eps);
        if (!(sum <= FLT_MAX)) {                 // the squares left fp32's range (or the row is not finite): once more in 64 bits
            double wide = 0.0;
            for (int i = 0; i < units; ++i) {
                float u[E];
                again(i, u);
#pragma unroll
                for (int e = 0; e < E; ++e) wide += (double)u[e] * u[e];
            }
            float none = 0.0f;
            wide = row_sum<WARP>(wide, none, wide_sums, no_tops);
            rho = wide <= DBL_MAX ? (float)(1.0 / sqrt(wide / a.cols + a.eps)) : __int_as_float(0x7fc00000);
            if constexpr (!WARP) __syncthreads();            // (the sums are used again)
        }
        const float inv = rows8::inverse_step(top);
        if (OUT8 && p.t == 0) a.scale[row] = __fmul_rn(__fmul_rn(top, rows8::kPart), rho);
        auto put = [&](int i, float (&v)[E], const float (&w)[E]) {
            if constexpr (OUT8) {
                p.store8(a.q + row * a.ldq, i, a.cols, v, inv);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = v[e] * rho * w[e];
                p.store((T*)a.y + row * a.ldy, i, a.cols, unit_of<T>(v));
            }
        };
        if constexpr (NU > 0) {
#pragma unroll
            for (int i = 0; i < NU; ++i) put(i, v[i], w[i]);
            if constexpr (MODE != ALIGNED) return;
        } else {
            for (int i = 0; i < units; ++i) {
                again(i, v[0]);
                p.load_weight(a, i, w[0]);
                if constexpr (OUT8) {
#pragma unroll
                    for (int e = 0; e < E; ++e) v[0][e] = __fmul_rn(v[0][e], w[0][e]);
                }
                put(i, v[0], w[0]);
            }
        }
    }
}

template <typename T, Mode MODE, int MOST, int NU>
cudaError_t launch(const NormArgs& a, unsigned threads, cudaStream_t st)
{
    // As many blocks as run at a time, where they go on to further rows, each with as many rows as the others or one less.
    // 148: the SMs of the one GPU that this is built for.
    const unsigned most = 148u * std::min(32u, (unsigned)(kBlocks<T, MODE, MOST, NU> * MOST) / threads);
    unsigned blocks = (unsigned)a.rows;
    if (MOST == 128 && blocks > most) {                      // (few rows: a warp a block spreads them over the SMs)
        threads = 128;
        blocks = (blocks + 3) / 4;
    }
    if (MODE == ALIGNED || NU == 0) {
        const unsigned at_once = 148u * std::min(32u, (unsigned)(kBlocks<T, MODE, MOST, NU> * MOST) / threads), turns = (blocks + at_once - 1) / at_once;
        blocks = (blocks + turns - 1) / turns;
    }
    PdlLaunch l(blocks, threads, 0, st);
    return a.q ? cudaLaunchKernelEx(&l.cfg, rms_norm_kernel<T, MODE, MOST, NU, true>, a) : cudaLaunchKernelEx(&l.cfg, rms_norm_kernel<T, MODE, MOST, NU, false>, a);
}

template <typename T, Mode MODE>
cudaError_t by_width(const NormArgs& a, cudaStream_t st)
{
    // A warp a row while two units a thread hold it, then a block of as few warps as do; four units for the widest.
    const unsigned units = ((unsigned)a.cols + 16 / sizeof(T) - 1) / (16 / sizeof(T));
    if (units <= 64) return launch<T, MODE, 128, 2>(a, 32, st);
    if (units <= 512) return launch<T, MODE, 256, 2>(a, (units + 63) / 64 * 32, st);
    if (units <= 1024) return launch<T, MODE, 512, 2>(a, (units + 63) / 64 * 32, st);
    if (units <= 2048) return launch<T, MODE, 512, 4>(a, (units + 127) / 128 * 32, st);
    return launch<T, MODE, 512, 0>(a, 512, st);
}

bool off(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) != 0; }

}  // namespace

extern "C" tsvd_status_t tsvd_rms_norm(const void* x, tsvd_dtype_t dtype, long long rows, int cols, long long ldx, const void* residual,
                                       long long ldr, void* h, long long ldh, const void* weight, tsvd_dtype_t weight_dtype, float eps,
                                       void* y, long long ldy, int8_t* q, long long ldq, float* scale, void* stream)
{
    if (rows < 0 || rows > 0x7fffffffLL || cols < 1 || ldx < cols || (residual && (ldr < cols || ldh < cols)) || (y && ldy < cols) || (q && ldq < cols))
        return TSVD_E_SHAPE;
    if (cols > TSVD_COUNT_MOST) return TSVD_E_TOOBIG;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (weight_dtype != TSVD_F32 && weight_dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (!(eps >= 1e-12f && eps <= FLT_MAX)) return TSVD_E_VALUE;
    if (rows == 0) return TSVD_OK;
    if (!x || !weight || (residual != nullptr) != (h != nullptr) || (y != nullptr) == (q != nullptr) || (q != nullptr) != (scale != nullptr))
        return TSVD_E_NULL;
    const size_t size = dtype == TSVD_F32 ? 4 : 2, wsize = weight_dtype == TSVD_F32 ? 4 : 2;
    if (off(x, size) || off(residual, size) || off(h, size) || off(y, size) || off(weight, wsize) || off(scale, 4)) return TSVD_E_ALIGN;
    const NormArgs a{x, residual, h, weight, y, q, scale, ldx, ldr, ldh, ldy, ldq, (int)rows, cols, weight_dtype == TSVD_BF16, eps};
    // numbers and 8-bit results in pieces of so many bytes
    auto even = [&](int piece, int piece8) {
        auto on = [&](const void* p, long long ld, long long bytes) { return ((uintptr_t)p | (rows > 1 ? (uintptr_t)(ld * bytes) : 0)) % piece == 0; };
        return on(x, ldx, size) && (!residual || (on(residual, ldr, size) && on(h, ldh, size))) && (!y || on(y, ldy, size)) &&
               (!q || ((uintptr_t)q | (rows > 1 ? (uintptr_t)ldq : 0)) % piece8 == 0);
    };
    const bool vec = even(16, 16) && !off(weight, 16);
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == TSVD_F32) TSVD_CUDA_OK((vec ? by_width<float, ALIGNED>(a, st) : by_width<float, SINGLES>(a, st)));
    else if (vec) TSVD_CUDA_OK((by_width<__nv_bfloat16, ALIGNED>(a, st)));
    else TSVD_CUDA_OK((even(4, 2) ? by_width<__nv_bfloat16, PAIRS>(a, st) : by_width<__nv_bfloat16, SINGLES>(a, st)));
    tsvd_count_launch();
    return TSVD_OK;
}
