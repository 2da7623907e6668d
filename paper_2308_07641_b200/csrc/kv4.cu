// Keys and values in 4 bits: the pool of pages, append, read, and the entry point of the attention.
//
// Per position, head and group of 32 numbers: step = fp16((hi - lo) * (1 / 15)), base = fp16(lo),
// code = clamp(rint((x - base) * (1 / step)), 0, 15).
#include <new>
#include <type_traits>

#include "serving.cuh"

namespace {

constexpr float kMost = 65000.0f;   // the largest magnitude kept: 15 steps above -kMost still are an fp16 number

// Where row `row` of the batch lives: its page and place, or page = -1 (with the status bit) when that is out of range.
struct Place { int page, at; };
__device__ __forceinline__ Place place_of_row(const Kv4Geom& g, const Kv4Batch& b, int row, int* status)
{
    Place p{-1, 0};
    const int s = kv4_seq_of_row(b, row);
    if (s >= b.n_seq || row < kv4_first_row(b, s)) return p;   // behind the last sequence or before the first: not a row
    const int end = b.q_start ? b.q_start[s + 1] : row + 1;
    const long long pos = (long long)b.seq_len[s] - (end - row);
    if (pos >= 0 && pos < (long long)b.max_pages * g.page_tokens) {
        const unsigned at = (unsigned)pos, n = at / (unsigned)g.page_tokens;
        const int page = b.table[(long long)s * b.max_pages + n];
        if (page >= 0 && page < g.n_pages) {
            p.page = page;
            p.at = (int)(at - n * (unsigned)g.page_tokens);
        }
    }
    if (p.page < 0 && threadIdx.x == 0) atomicOr(status, KV4_DEV_INDEX);
    return p;
}

// Eight consecutive numbers; VEC: the address is a multiple of 16 bytes.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, float (&v)[8])
{
    if constexpr (VEC) {
        alignas(16) T t[8];
#pragma unroll
        for (int i = 0; i < (int)(8 * sizeof(T) / 16); ++i) reinterpret_cast<uint4*>(t)[i] = reinterpret_cast<const uint4*>(p)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32(p[i]);
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, const float (&v)[8])
{
    alignas(16) T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = from_f32<T>(v[i]);
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < (int)(8 * sizeof(T) / 16); ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<uint4*>(t)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = t[i];
    }
}

// What one thread holds: eight numbers, a quarter of a group.  Item `u` of a row: key or value, head, word of eight.
template <int D>
struct Item {
    int is_v, head, word;
    __device__ __forceinline__ Item(int u, int heads)
    {
        word = u & (D / 8 - 1);
        head = u / (D / 8);
        is_v = head >= heads;
        if (is_v) head -= heads;
    }
    // byte offsets inside a 16-position block
    __device__ __forceinline__ int codes(int at) const
    {
        const int w = word >> 2, j = word & 3;           // group, quarter
        const int place = is_v ? word : j * (D / KV4_GROUP) + w;
        return (is_v ? 10 * D : 0) + at * (D / 2) + place * 4;
    }
    __device__ __forceinline__ int scales(int at) const { return (is_v ? 18 * D : 8 * D) + at * (D / 8) + (word >> 2) * 4; }
};

// Smallest and largest of three.
__device__ __forceinline__ float min3(float a, float b, float c)
{
    float y;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}

// A block takes a row; the rows of a call go into different positions, so no two blocks write the same bytes.  A thread takes
// sixteen numbers, half a group.  The kernel is bound by its instructions, the half-rate integer and comparison ones above
// all, so the codes are put together as floats: four codes are an exact fp32 integer below 2^16.  Issue slots 64% busy; three
// prompts of 4095 rows together, 32 heads of 128, 67 MB in and 21 out: 33 us from DRAM (copy bandwidth: 13.6).  64 rows of 8 heads:
// 2.1 us, a launch.
template <typename T, bool VEC, int D>
__global__ void __launch_bounds__(512)
kv4_append_kernel(Kv4Geom g, Kv4Batch b, const T* k, long long ldk, const T* v, long long ldv, int* status)
{
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x;
    __shared__ Place place_s;
    if (threadIdx.x < 32) {
        const Place p = place_of_row(g, b, row, status);
        if (threadIdx.x == 0) place_s = p;
    }
    __syncthreads();
    const Place at = place_s;
    if (at.page < 0) return;
    const int items = g.heads * (D / 8), pos = at.at & (KV4_BLOCK - 1);
    for (int u0 = threadIdx.x & ~31; u0 < items; u0 += blockDim.x) {
        const bool in = u0 + (int)(threadIdx.x & 31) < items;  // (whole warps take part in the exchange)
        const int u = in ? u0 + (int)(threadIdx.x & 31) : items - 1;
        const Item<D> t(2 * u, g.heads), t1(2 * u + 1, g.heads);
        const T* src = (t.is_v ? v + row * ldv : k + row * ldk) + t.head * D + t.word * 8;
        float x[16];
        load8<T, VEC>(src, reinterpret_cast<float (&)[8]>(x[0]));
        load8<T, VEC>(src + 8, reinterpret_cast<float (&)[8]>(x[8]));
        float lo = fminf(x[0], x[1]), hi = fmaxf(x[0], x[1]);
#pragma unroll
        for (int i = 2; i < 16; i += 2) { lo = min3(lo, x[i], x[i + 1]); hi = max3(hi, x[i], x[i + 1]); }
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, 1));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, 1));
        lo = fminf(fmaxf(lo, -kMost), kMost);
        hi = fmaxf(fminf(hi, kMost), -kMost);
        const __half step = __float2half_rn(__fmul_rn(hi - lo, 1.0f / 15.0f)), base = __float2half_rn(lo);
        const float s = __half2float(step), m = __half2float(base);
        const float inv = s > 0.0f ? __frcp_rn(s) : 0.0f;
        uint32_t word[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            // nibble (e >> 1) + 4 (e & 1) holds number e: the even numbers are the lower half of the word
            float half[2] = {0.0f, 0.0f};
#pragma unroll
            for (int e = 7; e >= 0; --e) {
                const float c = fminf(fmaxf(__fmul_rn(__fsub_rn(x[8 * w + e], m), inv), 0.0f), 15.0f);
                const float n = __fsub_rn(__fadd_rn(c, 12582912.0f), 12582912.0f);      // rounded to even
                half[e & 1] = fmaf(half[e & 1], 16.0f, n);
            }
            // 2^23 + integer: the integer is in the low bits
            word[w] = __byte_perm(__float_as_uint(half[0] + 8388608.0f), __float_as_uint(half[1] + 8388608.0f), 0x5410);
        }
        uint8_t* blk = g.block(at.page, t.head, at.at);
        if (in) {
            *reinterpret_cast<uint32_t*>(blk + t.codes(pos)) = word[0];
            *reinterpret_cast<uint32_t*>(blk + t1.codes(pos)) = word[1];
            if ((t.word & 3) == 0) *reinterpret_cast<__half2*>(blk + t.scales(pos)) = __halves2half2(step, base);
        }
    }
}

// The way back, a thread eight numbers at a time.  Bound by its stores: 4095 rows of 32 heads of 128 to fp32, 21 MB in and 134
// out, 37.5 us (copy bandwidth: 24.0); several rows a block gained nothing.
template <typename T, bool VEC, int D>
__global__ void __launch_bounds__(512)
kv4_read_kernel(Kv4Geom g, Kv4Batch b, T* __restrict__ k, long long ldk, T* __restrict__ v, long long ldv, int* status)
{
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x;
    __shared__ Place place_s;
    if (threadIdx.x < 32) {
        const Place p = place_of_row(g, b, row, status);
        if (threadIdx.x == 0) place_s = p;
    }
    __syncthreads();
    const Place at = place_s;
    const int items = 2 * g.heads * (D / 8);
    const int pos = at.at & (KV4_BLOCK - 1);
#pragma unroll 2
    for (int u = threadIdx.x; u < items; u += blockDim.x) {
        const Item<D> t(u, g.heads);
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (at.page >= 0) {
            const uint8_t* blk = g.block(at.page, t.head, at.at);
            const uint32_t word = *reinterpret_cast<const uint32_t*>(blk + t.codes(pos));
            const float2 sm = __half22float2(*reinterpret_cast<const __half2*>(blk + t.scales(pos)));
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = fmaf((float)((word >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15u), sm.x, sm.y);
        }
        store8<T, VEC>((t.is_v ? v + row * ldv : k + row * ldk) + t.head * D + t.word * 8, x);
    }
}

unsigned row_threads(const Kv4Geom& g, int numbers)   // a thread
{
    const int items = 2 * g.heads * (g.dim / numbers);
    return (unsigned)(items >= 512 ? 512 : (items + 31) / 32 * 32);
}

bool aligned16(const void* p, long long ld, size_t size) { return (((uintptr_t)p) & 15) == 0 && (ld * (long long)size) % 16 == 0; }

tsvd_status_t check_batch(const tsvd_kv4_s* h, const int* page_table, int max_pages, const int* seq_len, int n_seq, int n_rows,
                          const int* q_start)
{
    if (!h || !page_table || !seq_len) return TSVD_E_NULL;
    if (max_pages < 1 || n_seq < 1 || n_rows < 0 || (!q_start && n_rows != n_seq)) return TSVD_E_SHAPE;
    if (((uintptr_t)page_table | (uintptr_t)seq_len | (uintptr_t)q_start) & 3) return TSVD_E_ALIGN;
    return TSVD_OK;
}

}  // namespace

extern "C" tsvd_status_t tsvd_kv4_create(int n_kv_heads, int head_dim, int page_tokens, long long n_pages, tsvd_kv4_t* out)
{
    if (!out) return TSVD_E_NULL;
    *out = nullptr;
    if (n_kv_heads < 1 || (head_dim != 64 && head_dim != 128) || page_tokens < 1 || page_tokens % KV4_BLOCK || n_pages < 1)
        return TSVD_E_SHAPE;
    if (n_pages > 0x7fffffffLL / page_tokens || page_tokens > (1 << 24) || n_kv_heads > 65535) return TSVD_E_TOOBIG;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return TSVD_E_CUDA; }
    tsvd_kv4_s* h = new (std::nothrow) tsvd_kv4_s();
    if (!h) return TSVD_E_NOMEM;
    h->device = dev;
    h->g.heads = n_kv_heads;
    h->g.dim = head_dim;
    h->g.page_tokens = page_tokens;
    h->g.n_pages = (int)n_pages;
    h->g.block_bytes = 20u * (unsigned)head_dim;
    h->g.head_bytes = (unsigned)page_tokens / KV4_BLOCK * h->g.block_bytes;
    h->g.page_bytes = (size_t)n_kv_heads * h->g.head_bytes;
    h->pool_bytes = (size_t)n_pages * h->g.page_bytes;
    cudaError_t e = cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaMalloc(&h->g.pool, h->pool_bytes);
    if (e == cudaSuccess) e = cudaMemset(h->g.pool, 0, h->pool_bytes);
    if (e == cudaSuccess) e = cudaMalloc(&h->dev_status, sizeof(int));
    if (e == cudaSuccess) e = cudaMemset(h->dev_status, 0, sizeof(int));
    const size_t tickets = kv4_decode_tickets(h->sms) * sizeof(unsigned);
    const size_t parts = kv4_decode_parts_bytes(h->sms, head_dim), parts2 = kv4_prefill_parts_bytes(h->sms, head_dim);
    if (e == cudaSuccess) e = cudaMalloc(&h->parts, parts > parts2 ? parts : parts2);
    if (e == cudaSuccess) e = cudaMalloc(&h->tickets, tickets);
    if (e == cudaSuccess) e = cudaMemset(h->tickets, 0, tickets);
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);   // (a memset returns before its end, and other streams do not wait for it)
    if (e == cudaSuccess && (kv4_decode_prepare() != TSVD_OK || kv4_prefill_prepare() != TSVD_OK)) e = cudaErrorUnknown;
    if (e != cudaSuccess) {
        tsvd_kv4_destroy(h);
        (void)cudaGetLastError();
        return e == cudaErrorMemoryAllocation ? TSVD_E_NOMEM : TSVD_E_CUDA;
    }
    *out = h;
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_kv4_append(tsvd_kv4_t h, const void* k, long long ldk, const void* v, long long ldv, tsvd_dtype_t dtype,
                                         const int* page_table, int max_pages, const int* seq_len, const int* q_start, int n_seq,
                                         int n_rows, void* stream)
{
    const tsvd_status_t ok = check_batch(h, page_table, max_pages, seq_len, n_seq, n_rows, q_start);
    if (ok != TSVD_OK) return ok;
    const long long width = (long long)h->g.heads * h->g.dim;
    if (ldk < width || ldv < width) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (n_rows == 0) return TSVD_OK;
    if (!k || !v) return TSVD_E_NULL;
    const size_t size = dtype == TSVD_F32 ? 4 : 2;
    if (((uintptr_t)k | (uintptr_t)v) & (size - 1)) return TSVD_E_ALIGN;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    const Kv4Batch b{page_table, max_pages, seq_len, q_start, n_seq, n_rows};
    const bool vec = aligned16(k, ldk, size) && aligned16(v, ldv, size);
    cudaStream_t st = (cudaStream_t)stream;
    const unsigned t = row_threads(h->g, 16);
    cudaError_t e = cudaSuccess;
    auto go = [&](auto kernel, auto* kp, auto* vp) {
        PdlLaunch l((unsigned)n_rows, t, 0, st);
        e = cudaLaunchKernelEx(&l.cfg, kernel, h->g, b, kp, ldk, vp, ldv, h->dev_status);
    };
    auto by_type = [&](auto* kp, auto* vp) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(kp)>>;
        if (h->g.dim == 128) {
            if (vec) go(kv4_append_kernel<T, true, 128>, kp, vp);
            else go(kv4_append_kernel<T, false, 128>, kp, vp);
        } else {
            if (vec) go(kv4_append_kernel<T, true, 64>, kp, vp);
            else go(kv4_append_kernel<T, false, 64>, kp, vp);
        }
    };
    if (dtype == TSVD_F32) by_type((const float*)k, (const float*)v);
    else by_type((const __nv_bfloat16*)k, (const __nv_bfloat16*)v);
    TSVD_CUDA_OK(e);
    tsvd_count_launch();
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_kv4_read(tsvd_kv4_t h, void* k, long long ldk, void* v, long long ldv, tsvd_dtype_t dtype,
                                       const int* page_table, int max_pages, const int* seq_len, const int* q_start, int n_seq,
                                       int n_rows, void* stream)
{
    const tsvd_status_t ok = check_batch(h, page_table, max_pages, seq_len, n_seq, n_rows, q_start);
    if (ok != TSVD_OK) return ok;
    const long long width = (long long)h->g.heads * h->g.dim;
    if (ldk < width || ldv < width) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (n_rows == 0) return TSVD_OK;
    if (!k || !v) return TSVD_E_NULL;
    const size_t size = dtype == TSVD_F32 ? 4 : 2;
    if (((uintptr_t)k | (uintptr_t)v) & (size - 1)) return TSVD_E_ALIGN;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    const Kv4Batch b{page_table, max_pages, seq_len, q_start, n_seq, n_rows};
    const bool vec = aligned16(k, ldk, size) && aligned16(v, ldv, size);
    cudaStream_t st = (cudaStream_t)stream;
    const unsigned t = row_threads(h->g, 8);
    cudaError_t e = cudaSuccess;
    auto go = [&](auto kernel, auto* kp, auto* vp) {
        PdlLaunch l((unsigned)n_rows, t, 0, st);
        e = cudaLaunchKernelEx(&l.cfg, kernel, h->g, b, kp, ldk, vp, ldv, h->dev_status);
    };
    auto by_type = [&](auto* kp, auto* vp) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(kp)>>;
        if (h->g.dim == 128) {
            if (vec) go(kv4_read_kernel<T, true, 128>, kp, vp);
            else go(kv4_read_kernel<T, false, 128>, kp, vp);
        } else {
            if (vec) go(kv4_read_kernel<T, true, 64>, kp, vp);
            else go(kv4_read_kernel<T, false, 64>, kp, vp);
        }
    };
    if (dtype == TSVD_F32) by_type((float*)k, (float*)v);
    else by_type((__nv_bfloat16*)k, (__nv_bfloat16*)v);
    TSVD_CUDA_OK(e);
    tsvd_count_launch();
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_kv4_attend(tsvd_kv4_t h, const void* q, long long ldq, void* out, long long ldo, int n_heads,
                                         tsvd_dtype_t dtype, const int* page_table, int max_pages, const int* seq_len,
                                         const int* q_start, int n_seq, int n_rows, int max_q, int max_kv, float scale, int window,
                                         unsigned flags, void* stream)
{
    const tsvd_status_t ok = check_batch(h, page_table, max_pages, seq_len, n_seq, n_rows, q_start);
    if (ok != TSVD_OK) return ok;
    if (n_heads < 1 || n_heads % h->g.heads || n_heads > 65535) return TSVD_E_SHAPE;
    const long long width = (long long)n_heads * h->g.dim;
    if (ldq < width || ldo < width || max_q < 1 || max_kv < 0 || window < 0 || !(scale == scale)) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (flags & ~(TSVD_FLAG_CAUSAL | TSVD_FLAG_PATH_SIMPLE | TSVD_FLAG_TEST_STALL)) return TSVD_E_DTYPE;
    if (n_rows == 0) return TSVD_OK;
    if (!q || !out) return TSVD_E_NULL;
    if ((((uintptr_t)q | (uintptr_t)out) & 15) || ldq % 8 || ldo % 8) return TSVD_E_ALIGN;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    AttendArgs a{};
    a.h = h;
    a.b = Kv4Batch{page_table, max_pages, seq_len, q_start, n_seq, n_rows};
    a.q = q;
    a.ldq = ldq;
    a.out = out;
    a.ldo = ldo;
    a.n_heads = n_heads;
    a.dtype = dtype;
    a.max_q = max_q < n_rows ? max_q : n_rows;
    const long long room = (long long)max_pages * h->g.page_tokens;
    a.max_kv = (int)(max_kv && max_kv < room ? max_kv : room < 0x7fffffffLL ? room : 0x7fffffffLL);
    a.scale = scale;
    a.window = window;
    a.causal = flags & TSVD_FLAG_CAUSAL;
    a.test_stall = flags & TSVD_FLAG_TEST_STALL;
    a.stream = (cudaStream_t)stream;
    if (dtype == TSVD_F32 || (flags & TSVD_FLAG_PATH_SIMPLE)) return kv4_attend_simple(a);
    // Up to 16 rows a key/value head are one item of the kernel for few rows: 34 us against 40 (16 rows, 32 heads) and 60 against
    // 94 (32 sequences of 8 heads) behind 8000 and 3000 positions.  At 17 to 32 rows it reads the cache twice, 45 against 42
    // and 100 against 94; but with more than four heads and sequences an SM the other one's start and end, of about 9 us a
    // block, weigh more: 42 against 74 us for 32 sequences of 32 heads and 88 positions, 142 against 165 for 1024 positions.
    // Beyond 32 rows: 60 against 42 at 48 rows, 32 heads and 8000 positions.
    const long long rows = (long long)a.max_q * (n_heads / h->g.heads);
    const bool few = rows <= 16 || (rows <= 32 && (long long)n_seq * h->g.heads > 4LL * h->sms);
    return few ? kv4_attend_decode(a) : kv4_attend_prefill(a);
}

extern "C" tsvd_status_t tsvd_kv4_info(tsvd_kv4_t h, int* n_kv_heads, int* head_dim, int* page_tokens, long long* n_pages, size_t* pool_bytes)
{
    if (!h) return TSVD_E_NULL;
    if (n_kv_heads) *n_kv_heads = h->g.heads;
    if (head_dim) *head_dim = h->g.dim;
    if (page_tokens) *page_tokens = h->g.page_tokens;
    if (n_pages) *n_pages = h->g.n_pages;
    if (pool_bytes) *pool_bytes = h->pool_bytes;
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_kv4_last_status(tsvd_kv4_t h)
{
    if (!h) return TSVD_E_NULL;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    int word = 0;
    TSVD_CUDA_OK(cudaMemcpy(&word, h->dev_status, sizeof(int), cudaMemcpyDeviceToHost));
    if (word) TSVD_CUDA_OK(cudaMemset(h->dev_status, 0, sizeof(int)));
    if (word & KV4_DEV_TIMEOUT) TSVD_CUDA_OK(cudaMemset(h->tickets, 0, kv4_decode_tickets(h->sms) * sizeof(unsigned)));
    if (word) TSVD_CUDA_OK(cudaStreamSynchronize(nullptr));
    return (word & KV4_DEV_TIMEOUT) ? TSVD_E_TIMEOUT : (word & KV4_DEV_INDEX) ? TSVD_E_INDEX : TSVD_OK;
}

extern "C" void tsvd_kv4_destroy(tsvd_kv4_t h)
{
    if (!h) return;
    const int dev = h->device;
    int prev = dev;
    if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) cudaSetDevice(dev);
    cudaDeviceSynchronize();
    if (h->g.pool) cudaFree(h->g.pool);
    if (h->dev_status) cudaFree(h->dev_status);
    if (h->parts) cudaFree(h->parts);
    if (h->tickets) cudaFree(h->tickets);
    (void)cudaGetLastError();
    delete h;
    if (prev != dev) cudaSetDevice(prev);
}
