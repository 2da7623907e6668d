// Attention over the 4-bit cache on the CUDA cores, fp32 throughout: the kernel for fp32 queries, and for any with
// TSVD_FLAG_PATH_SIMPLE.
//
// out = sum_j p_j v_j with p = softmax(scale q.k_j), one pass with a running maximum and sum.  A block takes one row and
// head; its warps take 32 positions at a time.  For the scores a lane owns a position (its whole code row: no exchange);
// for the sum over values a lane owns head_dim / 32 numbers.
//
// Bound by fp32 instructions, some 40 a number: every row and head reads and decodes its positions again.  One token of 12 heads,
// 500 positions: 37 us; 32 tokens of 32 heads, 136000 positions together 0.9 ms; a prompt of 2048 tokens, 32 heads 5.7 ms.  It is the exact form
// (no fp16 anywhere), not the fast one.
#include "serving.cuh"

namespace {

constexpr int SIMPLE_WARPS = 4;

template <int D>
__device__ __forceinline__ float code_dot(const uint8_t* blk, int pos, const float* __restrict__ q)
{
    // sum_w step_w (q . code)_w + base_w (sum q)_w, the groups w of a position
    const uint32_t* row = reinterpret_cast<const uint32_t*>(blk + pos * (D / 2));
    const __half2* sm = reinterpret_cast<const __half2*>(blk + 8 * D + pos * (D / 8));
    float total = 0.0f;
#pragma unroll
    for (int w = 0; w < D / KV4_GROUP; ++w) {
        const float2 s = __half22float2(sm[w]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t word = row[j * (D / KV4_GROUP) + w];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                total = fmaf(fmaf((float)((word >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15u), s.x, s.y), q[32 * w + 8 * j + e], total);
        }
    }
    return total;
}

template <typename T, int D>
__global__ void __launch_bounds__(SIMPLE_WARPS * 32)
kv4_attend_simple_kernel(Kv4Geom g, Kv4Batch b, const T* __restrict__ q, long long ldq, T* __restrict__ out, long long ldo, int group,
                         int max_q, float scale, int window, int sinks, int causal, int* status)
{
    constexpr int PER = D / 32;               // numbers of the head that a lane sums
    __shared__ float qs[D];
    __shared__ float acc_s[SIMPLE_WARPS][D];
    __shared__ float top_s[SIMPLE_WARPS], sum_s[SIMPLE_WARPS];
    const int row = blockIdx.x, head = blockIdx.y, kvh = head / group;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int s = kv4_seq_of_row(b, row);
    if (s >= b.n_seq) return;                 // behind the last sequence: not a row
    const int first = kv4_first_row(b, s), last = b.q_start ? b.q_start[s + 1] : row + 1;
    if (row < first || row - first >= max_q) return;
    const long long room = (long long)b.max_pages * g.page_tokens;
    const int len = b.seq_len[s];
    const long long len_in = len < room ? (len < 0 ? 0 : len) : room;
    if (len > room && threadIdx.x == 0) atomicOr(status, KV4_DEV_INDEX);
    const long long pos = (long long)len - (last - row);
    const long long hi = causal ? (pos + 1 < len_in ? pos + 1 : len_in) : len_in;   // sees [lo, hi)
    const long long lo = window && pos - window + 1 > 0 ? pos - window + 1 : 0;   // and [0, sinks) below hi
    // runs of 32 positions: those of the first positions, then from the window's on
    const long long runs = (hi + 31) / 32, first_runs = ((sinks < hi ? sinks : hi) + 31) / 32;
    const long long gap = lo / 32 > first_runs ? lo / 32 - first_runs : 0;
    for (int d = threadIdx.x; d < D; d += blockDim.x) qs[d] = to_f32(q[row * ldq + (long long)head * D + d]) * scale;
    __syncthreads();

    float top = -INFINITY, sum = 0.0f, acc[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] = 0.0f;
    for (long long run = warp; run < first_runs || run + gap < runs; run += SIMPLE_WARPS) {
        const long long j0 = (run < first_runs ? run : run + gap) * 32, j = j0 + lane;
        float score = -INFINITY;
        const uint8_t* blk = nullptr;
        if ((j >= lo || j < sinks) && j < hi) {
            const int page = b.table[(long long)s * b.max_pages + j / g.page_tokens];
            if (page >= 0 && page < g.n_pages) {
                blk = g.block(page, kvh, (int)(j % g.page_tokens));
                score = code_dot<D>(blk, (int)(j & 15), qs);
            } else {
                atomicOr(status, KV4_DEV_INDEX);
            }
        }
        float new_top = score;
        for (int o = 16; o; o >>= 1) new_top = fmaxf(new_top, __shfl_xor_sync(0xffffffffu, new_top, o));
        new_top = fmaxf(new_top, top);
        if (new_top == -INFINITY) continue;   // nothing seen so far
        const float p = blk ? expf(score - new_top) : 0.0f, keep = expf(top - new_top);
        top = new_top;
        sum *= keep;
#pragma unroll
        for (int i = 0; i < PER; ++i) acc[i] *= keep;
        float psum = p;
        for (int o = 16; o; o >>= 1) psum += __shfl_xor_sync(0xffffffffu, psum, o);
        sum += psum;
        for (int jj = 0; jj < 32; ++jj) {
            const float pj = __shfl_sync(0xffffffffu, p, jj);
            const uint8_t* bj = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, (unsigned long long)blk, jj));
            if (!bj) continue;
            const int at = (int)((j0 + jj) & 15);
            // numbers PER*lane .. : eight of them lie in one word
            const uint32_t word = reinterpret_cast<const uint32_t*>(bj + 10 * D + at * (D / 2))[PER * lane / 8];
            const float2 sm = __half22float2(reinterpret_cast<const __half2*>(bj + 18 * D + at * (D / 8))[PER * lane / KV4_GROUP]);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = (PER * lane + i) & 7;
                acc[i] = fmaf(pj, fmaf((float)((word >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15u), sm.x, sm.y), acc[i]);
            }
        }
    }
    // the warps' parts
#pragma unroll
    for (int i = 0; i < PER; ++i) acc_s[warp][PER * lane + i] = acc[i];
    if (lane == 0) { top_s[warp] = top; sum_s[warp] = sum; }
    __syncthreads();
    float all = -INFINITY, total = 0.0f;
#pragma unroll
    for (int w = 0; w < SIMPLE_WARPS; ++w) all = fmaxf(all, top_s[w]);
#pragma unroll
    for (int w = 0; w < SIMPLE_WARPS; ++w) total += all == -INFINITY ? 0.0f : expf(top_s[w] - all) * sum_s[w];
    for (int d = threadIdx.x; d < D; d += blockDim.x) {
        float v = 0.0f;
        if (all != -INFINITY) {
#pragma unroll
            for (int w = 0; w < SIMPLE_WARPS; ++w) v += expf(top_s[w] - all) * acc_s[w][d];
            v /= total;
        }
        out[row * ldo + (long long)head * D + d] = from_f32<T>(v);
    }
}

template <typename T, int D>
void launch(const AttendArgs& a)
{
    kv4_attend_simple_kernel<T, D><<<dim3((unsigned)a.b.n_rows, (unsigned)a.n_heads), SIMPLE_WARPS * 32, 0, a.stream>>>(
        a.h->g, a.b, (const T*)a.q, a.ldq, (T*)a.out, a.ldo, a.n_heads / a.h->g.heads, a.max_q, a.scale, a.window, a.sinks, a.causal, a.h->dev_status);
}

}  // namespace

tsvd_status_t kv4_attend_simple(const AttendArgs& a)
{
    if (a.h->g.dim == 128) {
        if (a.dtype == TSVD_F32) launch<float, 128>(a);
        else launch<__nv_bfloat16, 128>(a);
    } else {
        if (a.dtype == TSVD_F32) launch<float, 64>(a);
        else launch<__nv_bfloat16, 64>(a);
    }
    TSVD_CUDA_OK(cudaGetLastError());
    tsvd_count_launch();
    return TSVD_OK;
}
