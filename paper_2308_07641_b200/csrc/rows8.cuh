// Rows into 8-bit integers, shared by tsvd_quantize (row-major result) and the 8-bit layer (tensor-core order).
//
//     a = max |x|,  scale = a * (1 / 127),  q = rint(x * ((1 / a) * 127))     each reciprocal and product rounded to fp32
//
// The largest magnitude of a row is needed before its first result, so a row's values stay in registers between the two
// steps: a thread holds units of 16 columns (one 16-byte store of results).
//
// Bound by memory where there is much of it: 2048 x 4096 bf16, 25 MB, 5.7 us a call over inputs larger than L2 (the copy
// bandwidth of 6.46 TB/s would take 3.9; the rest is a round trip and the ends); 8192 x 4096 17.3 (15.6).  By the launch
// otherwise: 333 x 1001 fp32 2.3 us.  Rows off the 16-byte boundaries are read number by number: 8192 x 1001 bf16 12 us (3.8).
#pragma once

#include "serving.cuh"

namespace rows8 {

constexpr float kSmallest = 7.888609e-31f;   // 2^-100: below it 127 / a is no longer safely finite
constexpr float kPart = 1.0f / 127.0f;

// 0 for a row without values of any size; where a is not finite the scale says so
__device__ __forceinline__ float inverse_step(float a) { return a >= kSmallest ? __fmul_rn(__frcp_rn(a), 127.0f) : 0.0f; }
__device__ __forceinline__ int quantised(float x, float inv) { return __float2int_rn(__fmul_rn(x, inv)); }

// Magnitudes compared as integers: a NaN (its bits exceed infinity's) wins over everything.
__device__ __forceinline__ uint32_t max_magnitude(uint32_t m, float v) { return max(m, __float_as_uint(v) & 0x7fffffffu); }

// Sixteen consecutive columns c .. c+15 of a row, zeros from `cols` on.  VEC: the row starts on a 16-byte boundary and may
// be read 16 bytes at a time wherever those lie inside it.
template <typename T, bool VEC>
struct Unit {
    float v[16];
    __device__ __forceinline__ void load(const T* row, int c, int cols)
    {
        if (VEC && c + 16 <= cols) {
            alignas(16) T t[16];
#pragma unroll
            for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<uint4*>(t)[i] = reinterpret_cast<const uint4*>(row + c)[i];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = to_f32(t[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = c + i < cols ? to_f32(row[c + i]) : 0.0f;
        }
    }
    __device__ __forceinline__ uint32_t magnitude(uint32_t m) const
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max_magnitude(m, v[i]);
        return m;
    }
    __device__ __forceinline__ uint4 pack(float inv) const
    {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = ((uint32_t)quantised(v[4 * j], inv) & 0xff) | ((uint32_t)quantised(v[4 * j + 1], inv) & 0xff) << 8 |
                   ((uint32_t)quantised(v[4 * j + 2], inv) & 0xff) << 16 | (uint32_t)quantised(v[4 * j + 3], inv) << 24;
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

template <>
struct Unit<int8_t, true> {
    uint4 u;
    __device__ __forceinline__ void load(const int8_t* row, int c, int cols)
    {
        if (c + 16 <= cols) { u = *reinterpret_cast<const uint4*>(row + c); return; }
        alignas(16) int8_t t[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) t[i] = c + i < cols ? row[c + i] : (int8_t)0;
        u = *reinterpret_cast<uint4*>(t);
    }
    __device__ __forceinline__ uint32_t magnitude(uint32_t m) const { return m; }
    __device__ __forceinline__ uint4 pack(float) const { return u; }
};
template <>
struct Unit<int8_t, false> : Unit<int8_t, true> {
    __device__ __forceinline__ void load(const int8_t* row, int c, int cols)
    {
        alignas(16) int8_t t[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) t[i] = c + i < cols ? row[c + i] : (int8_t)0;
        u = *reinterpret_cast<uint4*>(t);
    }
};

// Where a unit goes: row-major rows of ldq bytes (16 bytes at once where `wide`), or tensor-core order, where the columns
// up to the next multiple of 128 are written as zeros.
struct RowMajor {
    int8_t* q;
    long long ldq;
    bool wide;
    __device__ __forceinline__ int width(int cols) const { return cols; }
    __device__ __forceinline__ void store(int row, int c, int cols, uint4 u) const
    {
        int8_t* p = q + (long long)row * ldq + c;
        if (wide && c + 16 <= cols) { *reinterpret_cast<uint4*>(p) = u; return; }
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (c + i < cols) p[i] = (int8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
};
struct Tiles {
    uint8_t* tiles;
    int groups;      // of 8 tokens
    __device__ __forceinline__ int width(int cols) const { return (cols + 127) & ~127; }
    __device__ __forceinline__ void store(int row, int c, int, uint4 u) const
    {
        *reinterpret_cast<uint4*>(tiles + ((size_t)(c >> 7) * groups + (row >> 3)) * 1024 + i8_group_offset(row & 7, c & 127)) = u;
    }
};

// TPR threads take a row (32: a warp each, several rows a block; else the whole block), each up to NU units held in
// registers; NU = 0: rows of any length, read twice.
template <typename T, bool VEC, int TPR, int NU, typename OUT>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR)
quantize_kernel(const T* x, int rows, int cols, long long ldx, const float* given, OUT out, float* scale)
{
    __shared__ uint32_t slots[TPR == 32 ? 1 : TPR / 32];
    pdl_launch_dependents();
    pdl_wait();
    const unsigned at = TPR == 32 ? blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    const int t = TPR == 32 ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
    if (at >= (unsigned)rows) return;
    const int row = (int)at;
    const T* src = x + (long long)row * ldx;
    const int width = out.width(cols);
    constexpr bool kInt = sizeof(T) == 1;
    Unit<T, VEC> u[NU ? NU : 1];
    uint32_t m = 0;
    if constexpr (NU > 0) {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            u[i].load(src, (t + i * TPR) * 16, cols);   // reads nothing from `cols` on
            m = u[i].magnitude(m);
        }
    } else {
        if (!kInt)
            for (int c = t * 16; c < cols; c += TPR * 16) { u[0].load(src, c, cols); m = u[0].magnitude(m); }
    }
    float a = 0.0f, inv = 1.0f;
    if constexpr (!kInt) {
        m = __reduce_max_sync(0xffffffffu, m);
        if constexpr (TPR > 32) {
            if ((t & 31) == 0) slots[t >> 5] = m;
            __syncthreads();
            m = __reduce_max_sync(0xffffffffu, (t & 31) < TPR / 32 ? slots[t & 31] : 0u);
        }
        a = __uint_as_float(m);
        inv = inverse_step(a);
    }
    if (t == 0) scale[row] = kInt ? (given ? given[row] : 1.0f) : __fmul_rn(a, kPart);
    if constexpr (NU > 0) {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int c = (t + i * TPR) * 16;
            if (c < width) out.store(row, c, cols, u[i].pack(inv));
        }
    } else {
        for (int c = t * 16; c < width; c += TPR * 16) { u[0].load(src, c, cols); out.store(row, c, cols, u[0].pack(inv)); }
    }
}

template <typename T, bool VEC, int TPR, int NU, typename OUT>
cudaError_t launch(const void* x, int rows, int cols, long long ldx, const float* given, const OUT& out, float* scale, cudaStream_t st)
{
    // A warp a row: blocks of one warp spread few rows over the SMs (333 x 1001 fp32 2.5 us, with eight 3.9; 1500 x 512 2.0 and
    // 2.3), but at most 32 of them fit an SM (8192 x 512 9.1 us, with eight 4.5).  148: the SMs of the one GPU that this is built for.
    const unsigned warps = rows >= 148 * 16 ? 8 : 1;
    PdlLaunch l(TPR == 32 ? ((unsigned)rows + warps - 1) / warps : (unsigned)rows, TPR == 32 ? warps * 32 : TPR, 0, st);
    return cudaLaunchKernelEx(&l.cfg, quantize_kernel<T, VEC, TPR, NU, OUT>, (const T*)x, rows, cols, ldx, given, out, scale);
}

template <typename T, bool VEC, typename OUT>
cudaError_t by_width(const void* x, int rows, int cols, long long ldx, const float* given, const OUT& out, float* scale, cudaStream_t st)
{
    // Threads a row by its width: a warp (several rows a block, no barrier) while two units a thread hold the row, then the
    // smallest block that does with one (2048 x 4096 fp32: 256 threads of one 7.1 us, 128 of two 7.4).
    const int units = (cols + 127) / 128 * 8;
    if (units <= 32) return launch<T, VEC, 32, 1>(x, rows, cols, ldx, given, out, scale, st);
    if (units <= 64) return launch<T, VEC, 32, 2>(x, rows, cols, ldx, given, out, scale, st);
    if (units <= 128) return launch<T, VEC, 128, 1>(x, rows, cols, ldx, given, out, scale, st);
    if (units <= 256) return launch<T, VEC, 256, 1>(x, rows, cols, ldx, given, out, scale, st);
    if (units <= 512) return launch<T, VEC, 256, 2>(x, rows, cols, ldx, given, out, scale, st);
    if (units <= 1024) return launch<T, VEC, 256, 4>(x, rows, cols, ldx, given, out, scale, st);
    return launch<T, VEC, 256, 0>(x, rows, cols, ldx, given, out, scale, st);
}

template <typename OUT>
cudaError_t quantize(const void* x, tsvd_dtype_t dtype, int rows, int cols, long long ldx, const float* given, const OUT& out, float* scale,
                     cudaStream_t st)
{
    const long long size = dtype == TSVD_F32 ? 4 : dtype == TSVD_BF16 ? 2 : 1;
    const bool vec = (((uintptr_t)x) & 15) == 0 && (rows == 1 || (ldx * size) % 16 == 0);
    if (dtype == TSVD_F32) return vec ? by_width<float, true>(x, rows, cols, ldx, given, out, scale, st) : by_width<float, false>(x, rows, cols, ldx, given, out, scale, st);
    if (dtype == TSVD_BF16)
        return vec ? by_width<__nv_bfloat16, true>(x, rows, cols, ldx, given, out, scale, st) : by_width<__nv_bfloat16, false>(x, rows, cols, ldx, given, out, scale, st);
    if constexpr (sizeof(OUT) != sizeof(RowMajor))
        return vec ? by_width<int8_t, true>(x, rows, cols, ldx, given, out, scale, st) : by_width<int8_t, false>(x, rows, cols, ldx, given, out, scale, st);
    return cudaErrorInvalidValue;
}

}  // namespace rows8
