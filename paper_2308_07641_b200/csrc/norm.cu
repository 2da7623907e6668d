// Root-mean-square norm of rows, with the residual's addition ahead of it and, on request, a result in 8-bit rows.
//
//     h = round(x + r) to x's type,   rho = 1 / sqrt(mean h^2 + eps),   y = h rho w
//     in 8 bits:  t = h w,  a = max |t|,  q = rint(t ((1 / a) 127)),  scale = (a / 127) rho
//
// rho is one number a row, so it belongs into the scale: q is a function of t alone, elementwise in fp32, and the order in
// which the squares are summed cannot move a value to the next step.  A row is read once; its numbers stay in registers until
// its sum and its largest magnitude are known.
#include <float.h>

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

// A thread's unit: 16 bytes of x, E numbers.  VEC: consecutive ones, every row and w on 16-byte boundaries (a unit that the row
// ends inside is taken number by number).  Otherwise the unit is spread over the row, neighbouring threads on
// neighbouring numbers.
template <typename T, bool VEC, int TPR>
struct Place {
    static constexpr int E = 16 / (int)sizeof(T);
    int t;
    __device__ __forceinline__ int col(int i, int e) const { return VEC ? (i * TPR + t) * E + e : (i * E + e) * TPR + t; }
    __device__ __forceinline__ void load(const T* row, int i, int cols, float (&v)[E]) const
    {
        if (VEC && col(i, E - 1) < cols) {
            alignas(16) T u[E];
            *reinterpret_cast<uint4*>(u) = *reinterpret_cast<const uint4*>(row + col(i, 0));
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = to_f32(u[e]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = col(i, e) < cols ? to_f32(row[col(i, e)]) : 0.0f;
        }
    }
    __device__ __forceinline__ void store(T* row, int i, int cols, const float (&v)[E]) const
    {
        if (VEC && col(i, E - 1) < cols) {
            alignas(16) T u[E];
#pragma unroll
            for (int e = 0; e < E; ++e) u[e] = from_f32<T>(v[e]);
            *reinterpret_cast<uint4*>(row + col(i, 0)) = *reinterpret_cast<uint4*>(u);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (col(i, e) < cols) row[col(i, e)] = from_f32<T>(v[e]);
        }
    }
    __device__ __forceinline__ void load_weight(const NormArgs& a, int i, float (&v)[E]) const
    {
        if (VEC && col(i, E - 1) < a.cols) {
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
    // eight or four 8-bit results
    __device__ __forceinline__ void store8(int8_t* row, int i, int cols, const float (&v)[E], float inv) const
    {
        if (VEC && col(i, E - 1) < cols) {
            uint32_t w[E / 4];
#pragma unroll
            for (int j = 0; j < E / 4; ++j)
                w[j] = ((uint32_t)rows8::quantised(v[4 * j], inv) & 0xff) | ((uint32_t)rows8::quantised(v[4 * j + 1], inv) & 0xff) << 8 |
                       ((uint32_t)rows8::quantised(v[4 * j + 2], inv) & 0xff) << 16 | (uint32_t)rows8::quantised(v[4 * j + 3], inv) << 24;
            if constexpr (E == 8) *reinterpret_cast<uint2*>(row + col(i, 0)) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t*>(row + col(i, 0)) = w[0];
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (col(i, e) < cols) row[col(i, e)] = (int8_t)rows8::quantised(v[e], inv);
        }
    }
};

// Sum over the threads of a row, the same in all of them.
template <int TPR, typename S>
__device__ __forceinline__ S row_sum(S v, S* slots)
{
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
        __syncthreads();
        v = (threadIdx.x & 31) < TPR / 32 ? slots[threadIdx.x & 31] : S(0);
        for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    }
    return v;
}

// TPR threads take a row (32: a warp each, several rows a block; else the whole block), each up to NU units held in registers;
// NU = 0: rows of any length, read twice.
template <typename T, bool VEC, int TPR, int NU>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR)
rms_norm_kernel(const NormArgs a)
{
    constexpr int E = Place<T, VEC, TPR>::E, KEEP = NU ? NU : 1;
    __shared__ float sums[TPR == 32 ? 1 : TPR / 32];
    __shared__ double wide_sums[TPR == 32 ? 1 : TPR / 32];
    __shared__ uint32_t tops[TPR == 32 ? 1 : TPR / 32];
    pdl_launch_dependents();
    pdl_wait();
    const unsigned at = TPR == 32 ? blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    if (at >= (unsigned)a.rows) return;
    const long long row = at;
    const Place<T, VEC, TPR> p{TPR == 32 ? (int)(threadIdx.x & 31) : (int)threadIdx.x};
    const T* x = (const T*)a.x + row * a.ldx;
    const T* r = a.r ? (const T*)a.r + row * a.ldr : nullptr;
    T* h = a.h ? (T*)a.h + row * a.ldh : nullptr;
    float v[KEEP][E];
    float sum = 0.0f;
    uint32_t top = 0;
    // h of a unit, written where there is a residual
    auto add = [&](int i, float (&v)[E], const float (&u)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = to_f32(from_f32<T>(__fadd_rn(v[e], u[e])));
        p.store(h, i, a.cols, v);
    };
    auto weigh = [&](int i, float (&v)[E]) {
        float w[E];
        p.load_weight(a, i, w);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = __fmul_rn(v[e], w[e]);
    };
    auto look = [&](const float (&v)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e) sum = fmaf(v[e], v[e], sum);
    };
    const int units = NU ? NU : (a.cols + E * TPR - 1) / (E * TPR);
    if constexpr (NU > 0) {
#pragma unroll
        for (int i = 0; i < NU; ++i) p.load(x, i, a.cols, v[i]);
        if (r) {
            // (all loads before the first store: h may be x or the residual, so the compiler keeps their order)
            float u[NU][E];
#pragma unroll
            for (int i = 0; i < NU; ++i) p.load(r, i, a.cols, u[i]);
#pragma unroll
            for (int i = 0; i < NU; ++i) add(i, v[i], u[i]);
        }
#pragma unroll
        for (int i = 0; i < NU; ++i) look(v[i]);
    } else {
        for (int i = 0; i < units; ++i) {
            p.load(x, i, a.cols, v[0]);
            if (r) {
                float u[E];
                p.load(r, i, a.cols, u);
                add(i, v[0], u);
            }
            look(v[0]);
        }
    }
    auto again = [&](int i) { p.load(r ? h : x, i, a.cols, v[0]); };     // its own stores, where it wrote h
    sum = row_sum<TPR>(sum, sums);
    float rho = 1.0f / sqrtf(sum / (float)a.cols + a.eps);
    if (!(sum <= FLT_MAX)) {                     // the squares left fp32's range (or the row is not finite): once more in 64 bits
        double wide = 0.0;
        for (int i = 0; i < units; ++i) {
            if constexpr (NU == 0) again(i);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float f = 0.0f;
                if constexpr (NU > 0) {
#pragma unroll
                    for (int k = 0; k < NU; ++k) f = k == i ? v[k][e] : f;
                } else {
                    f = v[0][e];
                }
                wide += (double)f * f;
            }
        }
        rho = (float)(1.0 / sqrt(row_sum<TPR>(wide, wide_sums) / a.cols + a.eps));
    }
    if (a.y) {
        T* y = (T*)a.y + row * a.ldy;
        auto put = [&](int i, float (&v)[E]) {
            float w[E];
            p.load_weight(a, i, w);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = v[e] * rho * w[e];
            p.store(y, i, a.cols, v);
        };
        if constexpr (NU > 0) {
#pragma unroll
            for (int i = 0; i < NU; ++i) put(i, v[i]);
        } else {
            for (int i = 0; i < units; ++i) { again(i); put(i, v[0]); }
        }
        return;
    }
    auto largest = [&](const float (&v)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e) top = rows8::max_magnitude(top, v[e]);
    };
    if constexpr (NU > 0) {
#pragma unroll
        for (int i = 0; i < NU; ++i) { weigh(i, v[i]); largest(v[i]); }
    } else {
        for (int i = 0; i < units; ++i) { again(i); weigh(i, v[0]); largest(v[0]); }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
        __syncthreads();
        top = __reduce_max_sync(0xffffffffu, (threadIdx.x & 31) < TPR / 32 ? tops[threadIdx.x & 31] : 0u);
    }
    const float most = __uint_as_float(top), inv = rows8::inverse_step(most);
    if (p.t == 0) a.scale[row] = __fmul_rn(__fmul_rn(most, rows8::kPart), rho);
    int8_t* q = a.q + row * a.ldq;
    if constexpr (NU > 0) {
#pragma unroll
        for (int i = 0; i < NU; ++i) p.store8(q, i, a.cols, v[i], inv);
    } else {
        for (int i = 0; i < units; ++i) { again(i); weigh(i, v[0]); p.store8(q, i, a.cols, v[0], inv); }
    }
}

template <typename T, bool VEC, int TPR, int NU>
cudaError_t launch(const NormArgs& a, cudaStream_t st)
{
    // (a warp a row: one warp a block spreads few rows over the SMs, eight where there are enough of them)
    const unsigned warps = a.rows >= 148 * 16 ? 8 : 1;
    PdlLaunch l(TPR == 32 ? ((unsigned)a.rows + warps - 1) / warps : (unsigned)a.rows, TPR == 32 ? warps * 32 : TPR, 0, st);
    return cudaLaunchKernelEx(&l.cfg, rms_norm_kernel<T, VEC, TPR, NU>, a);
}

template <typename T, bool VEC>
cudaError_t by_width(const NormArgs& a, cudaStream_t st)
{
    // Threads a row by its width: the fewest that hold it in two or four units of 16 bytes each.
    const int units = (a.cols + 16 / (int)sizeof(T) - 1) / (16 / (int)sizeof(T));
    if (units <= 64) return launch<T, VEC, 32, 2>(a, st);
    if (units <= 128) return launch<T, VEC, 32, 4>(a, st);
    if (units <= 256) return launch<T, VEC, 128, 2>(a, st);
    if (units <= 512) return launch<T, VEC, 256, 2>(a, st);
    if (units <= 1024) return launch<T, VEC, 256, 4>(a, st);
    if (units <= 2048) return launch<T, VEC, 512, 4>(a, st);
    return launch<T, VEC, 512, 0>(a, st);
}

bool off(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) != 0; }

}  // namespace

extern "C" tsvd_status_t tsvd_rms_norm(const void* x, tsvd_dtype_t dtype, long long rows, int cols, long long ldx, const void* residual,
                                       long long ldr, void* h, long long ldh, const void* weight, tsvd_dtype_t weight_dtype, float eps,
                                       void* y, long long ldy, int8_t* q, long long ldq, float* scale, void* stream)
{
    if (rows < 0 || rows > 0x7fffffffLL || cols < 1 || ldx < cols || (residual && (ldr < cols || ldh < cols)) || (y && ldy < cols) || (q && ldq < cols))
        return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (weight_dtype != TSVD_F32 && weight_dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (!(eps >= 1e-12f && eps <= FLT_MAX)) return TSVD_E_VALUE;
    if (rows == 0) return TSVD_OK;
    if (!x || !weight || (residual != nullptr) != (h != nullptr) || (y != nullptr) == (q != nullptr) || (q != nullptr) != (scale != nullptr))
        return TSVD_E_NULL;
    const size_t size = dtype == TSVD_F32 ? 4 : 2, wsize = weight_dtype == TSVD_F32 ? 4 : 2;
    if (off(x, size) || off(residual, size) || off(h, size) || off(y, size) || off(weight, wsize) || off(scale, 4)) return TSVD_E_ALIGN;
    const NormArgs a{x, residual, h, weight, y, q, scale, ldx, ldr, ldh, ldy, ldq, (int)rows, cols, weight_dtype == TSVD_BF16, eps};
    auto even = [&](const void* p, long long ld, size_t s) { return !p || (!off(p, 16) && (rows == 1 || ld * (long long)s % 16 == 0)); };
    const bool vec = even(x, ldx, size) && even(residual, ldr, size) && even(h, ldh, size) && even(y, ldy, size) && even(q, ldq, 1) && !off(weight, 16);
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == TSVD_F32) TSVD_CUDA_OK((vec ? by_width<float, true>(a, st) : by_width<float, false>(a, st)));
    else TSVD_CUDA_OK((vec ? by_width<__nv_bfloat16, true>(a, st) : by_width<__nv_bfloat16, false>(a, st)));
    tsvd_count_launch();
    return TSVD_OK;
}
