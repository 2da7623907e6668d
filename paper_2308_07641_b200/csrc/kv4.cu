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
struct Place {
    int page, at;
    int pos;             // its position in the sequence: below 0 if that is before its start
    bool row;            // it belongs to a sequence
};
__device__ __forceinline__ Place place_of_row(const Kv4Geom& g, const Kv4Batch& b, int row, int* status)
{
    Place p{-1, 0, 0, false};
    const int s = kv4_seq_of_row(b, row);
    if (s >= b.n_seq || row < kv4_first_row(b, s)) return p;   // behind the last sequence or before the first: not a row
    const int end = b.q_start ? b.q_start[s + 1] : row + 1;
    const long long pos = (long long)b.seq_len[s] - (end - row);
    p.row = true;
    p.pos = (int)max(pos, -1LL);
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

// Sixteen numbers, half a group, into the cache; the lane beside holds the other half.  Whole warps; `in`: the lane has numbers.
template <int D>
__device__ __forceinline__ void keep16(const Kv4Geom& g, const Place& at, const Item<D>& t, const Item<D>& t1, const float (&x)[16], bool in)
{
    const int pos = at.at & (KV4_BLOCK - 1);
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
    const int items = g.heads * (D / 8);
    for (int u0 = threadIdx.x & ~31; u0 < items; u0 += blockDim.x) {
        const bool in = u0 + (int)(threadIdx.x & 31) < items;  // (whole warps take part in the exchange)
        const int u = in ? u0 + (int)(threadIdx.x & 31) : items - 1;
        const Item<D> t(2 * u, g.heads), t1(2 * u + 1, g.heads);
        const T* src = (t.is_v ? v + row * ldv : k + row * ldk) + t.head * D + t.word * 8;
        float x[16];
        load8<T, VEC>(src, reinterpret_cast<float (&)[8]>(x[0]));
        load8<T, VEC>(src + 8, reinterpret_cast<float (&)[8]>(x[8]));
        keep16<D>(g, at, t, t1, x, in);
    }
}

// ---- append with the rotation ---------------------------------------------------------------------------------------------
// Pairs (u, v) of a head's first `turned` numbers become (u cos - v sin, v cos + u sin), every product and sum rounded to fp32,
// and go on in fp32: keys into the cache's codes, queries rounded once to their type.  The table holds, for each position, the
// cosines of its turned / 2 angles and then their sines, so nothing here knows how the angles were chosen, and far positions
// are as exact as near ones.  A row's cosines and sines are one line of the table, which its heads share from the caches.
//
// Bound by loads that start late, behind the search for the row's place, and by instructions: 4095 rows of 32 heads of 128, keys,
// values and queries, 49 us (floor 24; the append alone 33), 3.1 stalls an issue on loads, issue slots 54% busy.  Read twice, once for
// either half of a pair, it took 64.  One token of 64 sequences, 32 heads on 8, and the read of it 6.1 us: two launches, each two round
// trips to memory.
struct Turn {
    const float* table;      // [positions][turned]
    int turned, positions;
    int interleaved;         // pairs (2 i, 2 i + 1); else (i, i + turned / 2)
};

// Numbers d0 .. d0 + 15 of a head that begins at `head`, turned.  FAST: sixteen numbers are turned all or none, have their
// partners in one piece, and cosines and sines may be read 16 bytes at a time.
template <typename T, bool VEC, bool FAST>
__device__ __forceinline__ void turn16(const T* head, int d0, const Turn& t, const float* cosines, float (&x)[16])
{
    load8<T, VEC>(head + d0, reinterpret_cast<float (&)[8]>(x[0]));
    load8<T, VEC>(head + d0 + 8, reinterpret_cast<float (&)[8]>(x[8]));
    if (d0 >= t.turned) return;
    const int half = t.turned >> 1;
    const float* sines = cosines + half;
    if (t.interleaved) {
        float c[8], s[8];
        if constexpr (FAST) {
            load8<float, true>(cosines + (d0 >> 1), c);
            load8<float, true>(sines + (d0 >> 1), s);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = (d0 >> 1) + i < half;
                c[i] = in ? cosines[(d0 >> 1) + i] : 1.0f;
                s[i] = in ? sines[(d0 >> 1) + i] : 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float u = x[2 * i], v = x[2 * i + 1];
            if (FAST || (d0 >> 1) + i < half) {
                x[2 * i] = __fsub_rn(__fmul_rn(u, c[i]), __fmul_rn(v, s[i]));
                x[2 * i + 1] = __fadd_rn(__fmul_rn(v, c[i]), __fmul_rn(u, s[i]));
            }
        }
        return;
    }
    if constexpr (FAST) {
        const bool lower = d0 < half;
        const int at = lower ? d0 : d0 - half;
        const float sign = lower ? -1.0f : 1.0f;
#pragma unroll
        for (int h = 0; h < 16; h += 8) {
            float o[8], c[8], s[8];
            load8<T, VEC>(head + (lower ? d0 + half : at) + h, o);
            load8<float, true>(cosines + at + h, c);
            load8<float, true>(sines + at + h, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[h + i] = __fadd_rn(__fmul_rn(x[h + i], c[i]), sign * __fmul_rn(o[i], s[i]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int d = d0 + i;
            if (d < t.turned) {
                const bool lower = d < half;
                const int at = lower ? d : d - half;
                const float o = to_f32(head[lower ? d + half : at]);
                const float p = __fmul_rn(o, sines[at]);
                x[i] = __fadd_rn(__fmul_rn(x[i], cosines[at]), lower ? -p : p);
            }
        }
    }
}

// Numbers d0 .. d0 + 15 and their partners half a rotation on, turned: one reading of either, of cosines and of sines.
template <typename T, bool VEC>
__device__ __forceinline__ void turn_both(const T* head, int d0, int half, const float* cosines, float (&x)[16], float (&y)[16])
{
#pragma unroll
    for (int h = 0; h < 16; h += 8) {
        float u[8], v[8], c[8], s[8];
        load8<T, VEC>(head + d0 + h, u);
        load8<T, VEC>(head + d0 + half + h, v);
        load8<float, true>(cosines + d0 + h, c);
        load8<float, true>(cosines + half + d0 + h, s);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[h + i] = __fsub_rn(__fmul_rn(u[i], c[i]), __fmul_rn(v[i], s[i]));
            y[h + i] = __fadd_rn(__fmul_rn(v[i], c[i]), __fmul_rn(u[i], s[i]));
        }
    }
}

// A block takes a row, a warp 32 items of its keys, values or queries.  FAST: see turn16.  WHOLE: as FAST, and all of a head is turned,
// half against half: a thread takes sixteen numbers of either half, so that nothing is read twice.
template <typename T, bool VEC, int D, bool FAST, bool WHOLE>
__global__ void __launch_bounds__(512)
kv4_append_rotated_kernel(Kv4Geom g, Kv4Batch b, Turn turn, const T* q, long long ldq, T* q_out, long long ldqo, int n_heads, const T* k,
                          long long ldk, const T* v, long long ldv, int* status)
{
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x;
    __shared__ Place place_s;
    if (threadIdx.x < 32) {
        Place p = place_of_row(g, b, row, status);
        if (p.page >= 0 && p.pos >= turn.positions) {
            p.page = -1;
            if (threadIdx.x == 0) atomicOr(status, KV4_DEV_INDEX);
        }
        if (threadIdx.x == 0) place_s = p;
    }
    __syncthreads();
    const Place at = place_s;
    if (!at.row) return;
    const int lane = threadIdx.x & 31;
    const bool known = at.pos >= 0 && at.pos < turn.positions;
    const float* cosines = turn.table + (size_t)(known ? at.pos : 0) * turn.turned;
    constexpr int BOTH = WHOLE ? 32 : 16;                      // numbers of an item of keys or queries
    const int k_items = g.heads * (D / BOTH), v_items = g.heads * (D / 16), q_items = n_heads * (D / BOTH);
    const int k_warps = (k_items + 31) / 32, v_warps = (v_items + 31) / 32, warps = k_warps + v_warps + (q_items + 31) / 32;
    for (int w = threadIdx.x >> 5; w < warps; w += blockDim.x >> 5) {
        float x[16], y[16];
        if (w < k_warps + v_warps) {
            if (at.page < 0) continue;
            const bool is_v = w >= k_warps;
            const int u0 = (is_v ? w - k_warps : w) * 32 + lane, items = is_v ? v_items : k_items;
            const bool in = u0 < items;                        // (whole warps take part in the exchange)
            const int u = in ? u0 : items - 1;
            if (is_v) {
                const Item<D> t(2 * (v_items + u), g.heads), t1(2 * (v_items + u) + 1, g.heads);
                const T* src = v + row * ldv + u * 16;
                load8<T, VEC>(src, reinterpret_cast<float (&)[8]>(x[0]));
                load8<T, VEC>(src + 8, reinterpret_cast<float (&)[8]>(x[8]));
                keep16<D>(g, at, t, t1, x, in);
            } else {
                const int head = u / (D / BOTH), d0 = u % (D / BOTH) * 16, first = head * (D / 8) + d0 / 8;
                if constexpr (WHOLE) turn_both<T, VEC>(k + row * ldk + head * D, d0, D / 2, cosines, x, y);
                else turn16<T, VEC, FAST>(k + row * ldk + head * D, d0, turn, cosines, x);
                keep16<D>(g, at, Item<D>(first, g.heads), Item<D>(first + 1, g.heads), x, in);
                if constexpr (WHOLE) keep16<D>(g, at, Item<D>(first + D / 16, g.heads), Item<D>(first + D / 16 + 1, g.heads), y, in);
            }
        } else {
            const int u = (w - k_warps - v_warps) * 32 + lane;
            if (u >= q_items) continue;
            const int head = u / (D / BOTH), d0 = u % (D / BOTH) * 16;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = y[i] = 0.0f;
            if (known) {
                if constexpr (WHOLE) turn_both<T, VEC>(q + row * ldq + head * D, d0, D / 2, cosines, x, y);
                else turn16<T, VEC, FAST>(q + row * ldq + head * D, d0, turn, cosines, x);
            }
            T* to = q_out + row * ldqo + head * D + d0;
            store8<T, VEC>(to, reinterpret_cast<float (&)[8]>(x[0]));
            store8<T, VEC>(to + 8, reinterpret_cast<float (&)[8]>(x[8]));
            if constexpr (WHOLE) {
                store8<T, VEC>(to + D / 2, reinterpret_cast<float (&)[8]>(y[0]));
                store8<T, VEC>(to + D / 2 + 8, reinterpret_cast<float (&)[8]>(y[8]));
            }
        }
    }
}

// cos and sin of position * rate, in 64 bits, kept in fp32.
__global__ void rotary_table_kernel(float* table, int positions, int half, const double* rates, float amplitude)
{
    const long long n = (long long)positions * half;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const long long pos = i / half;
        const int at = (int)(i - pos * half);
        double s, c;
        sincos((double)pos * rates[at], &s, &c);
        table[pos * 2 * half + at] = (float)(c * amplitude);
        table[pos * 2 * half + half + at] = (float)(s * amplitude);
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
    if (n_seq > TSVD_COUNT_MOST || n_rows > TSVD_COUNT_MOST) return TSVD_E_TOOBIG;
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

extern "C" tsvd_status_t tsvd_kv4_append_rotated(tsvd_kv4_t h, const void* q, long long ldq, void* q_out, long long ldqo, int n_heads,
                                                 const void* k, long long ldk, const void* v, long long ldv, tsvd_dtype_t dtype,
                                                 const float* table, int positions, int turned, int interleaved, const int* page_table,
                                                 int max_pages, const int* seq_len, const int* q_start, int n_seq, int n_rows, void* stream)
{
    const tsvd_status_t ok = check_batch(h, page_table, max_pages, seq_len, n_seq, n_rows, q_start);
    if (ok != TSVD_OK) return ok;
    const long long width = (long long)h->g.heads * h->g.dim, q_width = (long long)n_heads * h->g.dim;
    if (n_heads < 0 || n_heads > 65535 || ldk < width || ldv < width || (n_heads && (ldq < q_width || ldqo < q_width))) return TSVD_E_SHAPE;
    if (positions < 1 || turned < 2 || turned % 2 || turned > h->g.dim) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (n_rows == 0) return TSVD_OK;
    if (!k || !v || !table || (n_heads && (!q || !q_out))) return TSVD_E_NULL;
    if (n_heads && q == q_out) return TSVD_E_VALUE;
    const size_t size = dtype == TSVD_F32 ? 4 : 2;
    if (((uintptr_t)k | (uintptr_t)v | (n_heads ? (uintptr_t)q | (uintptr_t)q_out : 0)) & (size - 1)) return TSVD_E_ALIGN;
    if ((uintptr_t)table & 3) return TSVD_E_ALIGN;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    const Kv4Batch b{page_table, max_pages, seq_len, q_start, n_seq, n_rows};
    const Turn turn{table, turned, positions, interleaved != 0};
    const bool vec = aligned16(k, ldk, size) && aligned16(v, ldv, size) && (!n_heads || (aligned16(q, ldq, size) && aligned16(q_out, ldqo, size)));
    // (neighbours: eight angles of an item; halves: sixteen)
    const bool fast = ((uintptr_t)table & 15) == 0 && turned % (interleaved ? 16 : 32) == 0;
    cudaStream_t st = (cudaStream_t)stream;
    const bool whole = vec && fast && !interleaved && turned == h->g.dim;
    const int both = whole ? 32 : 16;
    const long long items = (h->g.heads * (h->g.dim / both) + 31) / 32 + (h->g.heads * (h->g.dim / 16) + 31) / 32 + (n_heads * (h->g.dim / both) + 31) / 32;
    cudaError_t e = cudaSuccess;
    auto go = [&](auto kernel, auto* kp) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(kp)>>;
        PdlLaunch l((unsigned)n_rows, (unsigned)(items > 16 ? 16 : items) * 32, 0, st);
        e = cudaLaunchKernelEx(&l.cfg, kernel, h->g, b, turn, (const T*)q, ldq, (T*)q_out, ldqo, n_heads, kp, ldk, (const T*)v, ldv, h->dev_status);
    };
    auto by_type = [&](auto* kp) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(kp)>>;
        if (h->g.dim == 128) {
            if (whole) go(kv4_append_rotated_kernel<T, true, 128, true, true>, kp);
            else if (vec && fast) go(kv4_append_rotated_kernel<T, true, 128, true, false>, kp);
            else if (vec) go(kv4_append_rotated_kernel<T, true, 128, false, false>, kp);
            else if (fast) go(kv4_append_rotated_kernel<T, false, 128, true, false>, kp);
            else go(kv4_append_rotated_kernel<T, false, 128, false, false>, kp);
        } else {
            if (whole) go(kv4_append_rotated_kernel<T, true, 64, true, true>, kp);
            else if (vec && fast) go(kv4_append_rotated_kernel<T, true, 64, true, false>, kp);
            else if (vec) go(kv4_append_rotated_kernel<T, true, 64, false, false>, kp);
            else if (fast) go(kv4_append_rotated_kernel<T, false, 64, true, false>, kp);
            else go(kv4_append_rotated_kernel<T, false, 64, false, false>, kp);
        }
    };
    if (dtype == TSVD_F32) by_type((const float*)k);
    else by_type((const __nv_bfloat16*)k);
    TSVD_CUDA_OK(e);
    tsvd_count_launch();
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_rotary_table(float* table, int positions, int turned, const double* rates, float amplitude, void* stream)
{
    if (positions < 1 || turned < 2 || turned % 2) return TSVD_E_SHAPE;
    if (!table || !rates) return TSVD_E_NULL;
    if (((uintptr_t)table & 3) || ((uintptr_t)rates & 7)) return TSVD_E_ALIGN;
    const long long n = (long long)positions * (turned / 2), blocks = (n + 255) / 256;
    rotary_table_kernel<<<(unsigned)(blocks > 148 * 8 ? 148 * 8 : blocks), 256, 0, (cudaStream_t)stream>>>(table, positions, turned / 2, rates, amplitude);
    TSVD_CUDA_OK(cudaGetLastError());
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
    return tsvd_kv4_attend_sinks(h, q, ldq, out, ldo, n_heads, dtype, page_table, max_pages, seq_len, q_start, n_seq, n_rows, max_q, max_kv,
                                 scale, window, 0, flags, stream);
}

extern "C" tsvd_status_t tsvd_kv4_attend_sinks(tsvd_kv4_t h, const void* q, long long ldq, void* out, long long ldo, int n_heads,
                                               tsvd_dtype_t dtype, const int* page_table, int max_pages, const int* seq_len,
                                               const int* q_start, int n_seq, int n_rows, int max_q, int max_kv, float scale, int window,
                                               int sinks, unsigned flags, void* stream)
{
    const tsvd_status_t ok = check_batch(h, page_table, max_pages, seq_len, n_seq, n_rows, q_start);
    if (ok != TSVD_OK) return ok;
    if (n_heads < 1 || n_heads % h->g.heads || n_heads > 65535) return TSVD_E_SHAPE;
    const long long width = (long long)n_heads * h->g.dim;
    if (ldq < width || ldo < width || max_q < 1 || max_kv < 0 || window < 0 || sinks < 0 || !(scale == scale)) return TSVD_E_SHAPE;
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
    a.sinks = window ? sinks : 0;
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
