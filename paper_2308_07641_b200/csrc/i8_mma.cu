// The 8-bit product on tcgen05:  y_bm = (sum_n q_bn W_mn) * scale_b * wscale_m + bias_m.
//
// tcgen05.mma.kind::i8 with int32 accumulators in tensor memory: M = 128 channels (the weights' rows, one accumulator lane
// each), N = a tile of up to 256 tokens (one accumulator column each), K = 32 bytes.  Both operands lie in global memory in
// the order the instruction reads (serving.cuh), so a stage of 128 contraction bytes is two contiguous bulk copies.
//
// Many tokens: a persistent grid, one tile of 128 channels by up to 256 tokens an SM at a time, two accumulators, so that a
// tile's results leave (through shared memory, a token's 128 channels together) while the next one's products run.
// 12288 x 4096 weights, 2048 tokens: tiles of 240 tokens (six rounds of 864 tiles, as 256 would take), the call 87 us with the
// 6 to 9 of the quantisation, product some 80 = 2.6 POP/s (0.78 of twice the measured bf16 rate); 101 us when run for seconds,
// the power limit then holds the SMs at 1582 MHz.  Tensor pipe 71% of the active cycles: a stage of 46 KB feeds 480 clocks of
// products, and the 1.26 GB that the SMs take in come at 15.7 TB/s.  Two row tiles a block for one token tile take in a quarter
// less and were slower (88 -> 93 us: no second pair of accumulators to overlap the results with); pairs of SMs on one tile
// (cta_group::2) would take in a third less and were not built.
// Few tokens: bound by streaming the weights, and by the latency of a launch, a round trip and the results; the contraction is
// split over a cluster whose blocks add their parts through distributed shared memory.  One token, 4096 x 4096: 5.8 us with
// the quantisation before it and the weights in L2, 7.2 with the weights from DRAM, where the 16.8 MB take 2.6 at the copy
// bandwidth.
#include <algorithm>

#include "serving.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace ptx;

constexpr int I8_THREADS = 192;          // warps 0-3: epilogue; 4: copies; 5: tensor memory and MMA issue
constexpr int I8_MAX_STAGES = 12;
constexpr int I8_SMEM_LIMIT = 227 * 1024;
constexpr int I8_OUT_BYTES = 2 * 16 * 128 * 4;   // results on their way out: 16 tokens of 128 channels, twice

struct I8Params {
    const int8_t* W;
    const uint8_t* x;        // tokens in tensor-core order
    const float* x_scale;    // [B]
    const float* w_scale;    // [row_tiles * 128]
    const float* bias;       // the same, or null
    void* y;
    long long ldy;
    int y_bf16, y_wide;      // y_wide: rows start on 16-byte boundaries
    int M, B;
    int KB;                  // blocks of 128 columns
    int groups;              // groups of 8 tokens in x
    int row_tiles, tok_tiles, NT;
    int band;                // row tiles of a band: a band's tiles are walked token tile by token tile
    int stages;
    int test_stall;          // test hook: the tokens are never copied, so the waits must give up
    int columns;             // of tensor memory: one accumulator for a cluster's block, two for the others
    int* status;
};

__device__ __forceinline__ void st_cluster_u32(uint32_t addr, uint32_t v)
{
    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

__device__ __forceinline__ float scaled(const I8Params&, int sum, float xs, float ws, float bias)
{
    return __fadd_rn(__fmul_rn(__fmul_rn((float)sum, xs), ws), bias);
}
__device__ __forceinline__ void store_y(const I8Params& p, int b, int m, int sum, float xs, float ws, float bias)
{
    const float v = scaled(p, sum, xs, ws, bias);
    if (p.y_bf16) reinterpret_cast<__nv_bfloat16*>(p.y)[(long long)b * p.ldy + m] = __float2bfloat16_rn(v);
    else reinterpret_cast<float*>(p.y)[(long long)b * p.ldy + m] = v;
}

// Tile `i` of the call: bands of row tiles one after another, so that the blocks that run at the same time share both the
// weights and the tokens that they read.
__device__ __forceinline__ void tile_at(const I8Params& p, int i, int& rt, int& tt)
{
    const int per_band = p.band * p.tok_tiles, b = i / per_band, in = i - b * per_band;
    const int rows = min(p.band, p.row_tiles - b * p.band);
    tt = in / rows;
    rt = b * p.band + in - tt * rows;
}

// The 128 threads of the results agree whether any of them gave up (a wait that runs out is not seen by all at the same time).
__device__ __forceinline__ bool any_of_128(bool x)
{
    uint32_t y;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.red.or.pred q, 1, 128, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(y)
        : "r"((uint32_t)x)
        : "memory");
    return y != 0;
}

// CL = 1: persistent, a block walks over tiles (row tile fastest), two accumulators.
// CL > 1: one tile for each cluster of CL blocks, which share its contraction and meet through distributed shared memory;
// one block an SM (TSVD_ALONE_SMEM), because they hold tensor memory while they wait for one another.
template <int CL>
__global__ void __launch_bounds__(I8_THREADS, 1)
i8_mma_kernel(const I8Params p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    __shared__ uint64_t full[I8_MAX_STAGES], empty[I8_MAX_STAGES], acc_full[2], acc_empty[2];
    __shared__ uint32_t tmem_slot;
    __shared__ int ctl_[2];
    volatile int* ctl = ctl_;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t stage_bytes = 16384u + (uint32_t)p.NT * 128u;
    const int tiles = p.row_tiles * p.tok_tiles;
    const int first = (int)blockIdx.x / CL, step = (int)gridDim.x / CL;
    const int c = CL > 1 ? (int)cluster_ctarank() : 0;
    const int kb0 = c * p.KB / CL, kb1 = (c + 1) * p.KB / CL;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&acc_full[a], 1); mbar_init(&acc_empty[a], 4); }
        ctl[0] = 0;
        ctl[1] = p.test_stall ? kWaitLimitStall : kWaitLimitDefault;
        fence_mbar_init();
    }
    if (warp == 5) { tmem_alloc(&tmem_slot, (uint32_t)p.columns); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    pdl_launch_dependents();

    if (warp == 4) {
        if (elect_one()) {
            // The weights of the first stages are requested before the kernel that writes the tokens has ended.
            int s = 0, ahead = 0;
            uint32_t ph = 0;
            int rt0 = 0, tt0 = 0;
            tile_at(p, min(first, tiles - 1), rt0, tt0);
            if (first < tiles)
                for (int kb = kb0; kb < kb1 && ahead < p.stages; ++kb, ++ahead) {
                    const uint32_t tok = (uint32_t)min(p.NT, p.groups * 8 - tt0 * p.NT);
                    mbar_arrive_expect_tx(&full[ahead], 16384u + tok * 128u);
                    bulk_g2s(smem + (size_t)ahead * stage_bytes, p.W + ((size_t)rt0 * p.KB + kb) * 16384, 16384u, &full[ahead]);
                }
            pdl_wait();
            bool ok = !p.test_stall;
            for (int tile = first; tile < tiles && ok; tile += step) {
                int rt, t0;
                tile_at(p, tile, rt, t0);
                t0 *= p.NT;
                const uint32_t tok = (uint32_t)min(p.NT, p.groups * 8 - t0);   // groups behind the last token are not copied
                for (int kb = kb0; kb < kb1; ++kb) {
                    uint8_t* at = smem + (size_t)s * stage_bytes;
                    if (ahead > 0) {
                        --ahead;
                    } else {
                        if (!(ok = mbar_wait(&empty[s], ph ^ 1, ctl))) break;
                        mbar_arrive_expect_tx(&full[s], 16384u + tok * 128u);
                        bulk_g2s(at, p.W + ((size_t)rt * p.KB + kb) * 16384, 16384u, &full[s]);
                    }
                    bulk_g2s(at + 16384, p.x + ((size_t)kb * p.groups + (t0 >> 3)) * 1024, tok * 128u, &full[s]);
                    if (++s == p.stages) { s = 0; ph ^= 1; }
                }
            }
            // No copy may be in flight when the block ends.  The contraction waits for every stage; where a wait gave up,
            // the copies of each stage's last use are waited for here (again with a limit).
            if (ctl[0])
                for (int i = 0; i < p.stages; ++i) mbar_drain(&full[i], i < s ? ph : ph ^ 1);
        }
    } else if (warp == 5) {
        if (elect_one()) {
            const uint32_t idesc = umma_idesc_s8(128, p.NT);
            int s = 0, a = 0;
            uint32_t ph = 0, aph = 0;
            bool ok = true;
            for (int tile = first; tile < tiles && ok; tile += step) {
                if (!(ok = mbar_wait(&acc_empty[a], aph ^ 1, ctl))) break;
                tc_fence_after_sync();
                const uint32_t d = tmem + (uint32_t)a * 256u;
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!(ok = mbar_wait(&full[s], ph, ctl))) break;
                    const uint32_t at = smem_u32(smem + (size_t)s * stage_bytes);
                    const uint64_t da = umma_desc_k_sw128(at), db = umma_desc_k_sw128(at + 16384u);
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_s8_ss(d, da + 2 * k, db + 2 * k, idesc, kb > kb0 || k > 0);
                    umma_commit(&empty[s]);
                    if (++s == p.stages) { s = 0; ph ^= 1; }
                }
                if (!ok) break;
                umma_commit(&acc_full[a]);
                if (++a == 2) { a = 0; aph ^= 1; }
            }
        }
    } else {
        pdl_wait();
        int a = 0, flip = 0;
        uint32_t aph = 0;
        uint8_t* out_stage = smem + (size_t)p.stages * stage_bytes;
        for (int tile = first; tile < tiles; tile += step) {
            int rt, t0;
            tile_at(p, tile, rt, t0);
            t0 *= p.NT;
            const int n = min(p.NT, p.B - t0);
            const int m = rt * 128 + warp * 32 + lane;
            const float ws = p.w_scale[m], bias = p.bias ? p.bias[m] : 0.0f;
            bool ok = kb1 == kb0 || mbar_wait(&acc_full[a], aph, ctl);
            tc_fence_after_sync();
            const uint32_t src = tmem + ((uint32_t)(warp * 32) << 16) + (uint32_t)a * 256u;
            if constexpr (CL == 1) {
                if (any_of_128(!ok)) break;
                // Through shared memory, 16 tokens at a time: a lane has one channel of them, the output wants a token's
                // channels together.
                const int c = warp * 32 + lane, width = min(128, p.M - rt * 128);
                for (int j0 = 0; j0 < n; j0 += 16, flip ^= 1) {
                    uint32_t r[16];
                    tmem_ld16(src + (uint32_t)j0, r);
                    float xs[16];
#pragma unroll
                    for (int j = 0; j < 4; ++j) *reinterpret_cast<float4*>(xs + 4 * j) = reinterpret_cast<const float4*>(p.x_scale + t0 + j0)[j];
                    tmem_ld_wait();
                    uint8_t* chunk = out_stage + flip * 16 * 128 * 4;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float v = scaled(p, (int)r[j], xs[j], ws, bias);
                        if (p.y_bf16) reinterpret_cast<__nv_bfloat16*>(chunk)[j * 128 + c] = __float2bfloat16_rn(v);
                        else reinterpret_cast<float*>(chunk)[j * 128 + c] = v;
                    }
                    asm volatile("bar.sync 1, 128;" ::: "memory");   // one barrier a chunk: the other buffer's readers are through before it
                    const int rows = min(16, n - j0), size = p.y_bf16 ? 2 : 4;
                    uint8_t* to = reinterpret_cast<uint8_t*>(p.y) + ((long long)(t0 + j0) * p.ldy + (long long)rt * 128) * size;
                    if (p.y_wide) {
                        const int units = 128 * size / 16;            // of a token
                        for (int i = threadIdx.x; i < rows * units; i += 128) {
                            const int j = i / units, u = i - j * units;
                            const uint4 w = *reinterpret_cast<const uint4*>(chunk + i * 16);
                            uint8_t* at = to + (long long)j * p.ldy * size + u * 16;
                            if ((u + 1) * 16 <= width * size) {
                                *reinterpret_cast<uint4*>(at) = w;
                            } else {                                  // the ragged end of a row, 2 or 4 bytes at a time
                                const uint32_t part[4] = {w.x, w.y, w.z, w.w};
                                for (int e = 0; e < 16 / size; ++e)
                                    if (u * 16 + (e + 1) * size <= width * size) {
                                        if (size == 4) reinterpret_cast<uint32_t*>(at)[e] = part[e];
                                        else reinterpret_cast<uint16_t*>(at)[e] = (uint16_t)(part[e >> 1] >> (16 * (e & 1)));
                                    }
                            }
                        }
                    } else if (c < width) {
                        for (int j = 0; j < rows; ++j) {
                            if (p.y_bf16) reinterpret_cast<__nv_bfloat16*>(to)[(long long)j * p.ldy + c] = reinterpret_cast<__nv_bfloat16*>(chunk)[j * 128 + c];
                            else reinterpret_cast<float*>(to)[(long long)j * p.ldy + c] = reinterpret_cast<float*>(chunk)[j * 128 + c];
                        }
                    }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&acc_empty[a]);
                if (++a == 2) { a = 0; aph ^= 1; }
            }
        }
    }
    __syncwarp();
    if constexpr (CL > 1) {
        // Every block's contraction is done and its ring is free: the parts go to the block that owns the channel (rows
        // 128/CL of the tile each), slot [source][token][row], in the ring's memory.
        constexpr int OWN = 128 / CL;
        const bool works = first < tiles;
        int rt, t0;
        tile_at(p, min(first, tiles - 1), rt, t0);
        t0 *= p.NT;
        const int n = works ? min(p.NT, p.B - t0) : 0;
        cluster_sync_all();
        const bool ok = ctl[0] == 0;
        if (works && warp < 4) {
            const uint32_t src = tmem + ((uint32_t)(warp * 32) << 16);
            const int row = warp * 32 + lane;
            const uint32_t to = cluster_map_u32(smem_u32(smem), (uint32_t)(row / OWN)) + 4u * (uint32_t)(c * p.NT * OWN + row % OWN);
            for (int j0 = 0; j0 < n; j0 += 16) {
                uint32_t r[16] = {};
                if (kb1 > kb0 && ok) { tmem_ld16(src + (uint32_t)j0, r); tmem_ld_wait(); }
#pragma unroll
                for (int j = 0; j < 16; ++j) st_cluster_u32(to + 4u * (uint32_t)((j0 + j) * OWN), r[j]);
            }
            tc_fence_before_sync();
        }
        cluster_sync_all();
        if (works) {
            const int* slots = reinterpret_cast<const int*>(smem);
            for (int i = threadIdx.x; i < n * OWN; i += I8_THREADS) {
                const int r = i % OWN, j = i / OWN, m = rt * 128 + c * OWN + r;
                int sum = 0;
#pragma unroll
                for (int k = 0; k < CL; ++k) sum += slots[k * p.NT * OWN + i];
                if (m < p.M) store_y(p, t0 + j, m, sum, p.x_scale[t0 + j], p.w_scale[m], p.bias ? p.bias[m] : 0.0f);
            }
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (threadIdx.x == 0 && ctl[0]) atomicOr(p.status, TSVD_DEV_TIMEOUT);
    if (warp == 5) tmem_dealloc(tmem, (uint32_t)p.columns);
}

template <int CL>
tsvd_status_t launch(I8Params p, int blocks, cudaStream_t st)
{
    const size_t stage = 16384 + (size_t)p.NT * 128;
    const size_t out = CL == 1 ? I8_OUT_BYTES : 0;
    p.stages = (int)std::min<size_t>(I8_MAX_STAGES, (I8_SMEM_LIMIT - 2048 - out) / stage);
    size_t ring = p.stages * stage + out;
    if (CL > 1) {
        const int longest = (p.KB + CL - 1) / CL;
        p.stages = std::min(p.stages, std::max(longest, 1));
        ring = std::max(p.stages * stage, (size_t)p.NT * 512);
    }
    p.columns = 512;
    if (CL > 1)
        for (p.columns = 32; p.columns < p.NT; p.columns *= 2) { }
    const size_t smem = CL > 1 ? std::max(ring + 1024, TSVD_ALONE_SMEM) : ring + 1024;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(I8_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CL;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CL > 1 ? 2 : 1;
    TSVD_CUDA_OK(cudaLaunchKernelEx(&cfg, i8_mma_kernel<CL>, p));
    tsvd_count_launch();
    return TSVD_OK;
}

}  // namespace

tsvd_status_t i8_product(const tsvd_i8_s* h, const uint8_t* x, const float* x_scale, int B, void* y, long long ldy, bool y_bf16, bool test_stall, cudaStream_t st)
{
    I8Params p{};
    p.test_stall = test_stall;
    p.W = h->W;
    p.x = x;
    p.x_scale = x_scale;
    p.w_scale = h->w_scale;
    p.bias = h->bias;
    p.y = y;
    p.ldy = ldy;
    p.y_bf16 = y_bf16;
    p.y_wide = ((uintptr_t)y & 15) == 0 && (B == 1 || ldy * (y_bf16 ? 2 : 4) % 16 == 0);
    p.M = h->M;
    p.B = B;
    p.KB = h->col_blocks;
    p.groups = (B + 7) / 8;
    p.row_tiles = h->row_tiles;
    p.status = h->dev_status;
    // Token tile and split of the contraction, by an estimate in SM clocks: a block of 128 columns costs its MMAs (2 clocks
    // a token) or its copies (about 56 bytes a clock), whichever is longer; a tile's end about 8 clocks a token; a cluster's
    // two barriers and exchange about 2500.  No more clusters than run at a time: eighteen of eight for 2304 channels, one token,
    // took 9.0 us in two rounds where eighteen of four take 5.6.  One token, 4096 x 4096: 5.8 us, without clusters 9.7, with tiles of 256
    // tokens 6.8; 197 tokens, 1001 x 770: 7.0, without clusters the same, with tiles of 256 tokens 11.7.
    const int sms = h->sms;
    long long best = -1;
    int cl = 1;
    for (int nt = 16; nt <= 256; nt += 16) {
        const long long tok = (B + nt - 1) / nt, tiles = tok * p.row_tiles;
        const long long block = std::max(2 * nt, (16384 + 128 * nt) / 56);
        for (int c = 1; c <= 8; c *= 2) {
            if (c > 1 && (tiles > h->clusters[c] || p.KB < c)) break;
            const long long cost = ((tiles * c + sms - 1) / sms) * ((p.KB + c - 1) / c) * block + 8 * nt + (c > 1 ? 2500 : 0);
            if (best < 0 || cost < best) { best = cost; p.NT = nt; p.tok_tiles = (int)tok; cl = c; }
        }
    }
    p.band = std::min(p.row_tiles, (sms + p.tok_tiles - 1) / p.tok_tiles);
    const int tiles = p.row_tiles * p.tok_tiles;
    switch (cl) {
        case 8: return launch<8>(p, tiles * 8, st);
        case 4: return launch<4>(p, tiles * 4, st);
        case 2: return launch<2>(p, tiles * 2, st);
        default: return launch<1>(p, std::min(tiles, sms), st);
    }
}

// How many clusters of CL blocks, one block an SM, the device runs at a time.
template <int CL>
static cudaError_t most_clusters(int* most)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(CL);
    cfg.blockDim = dim3(I8_THREADS);
    cfg.dynamicSmemBytes = I8_SMEM_LIMIT - 1024;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CL;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaOccupancyMaxActiveClusters(most, i8_mma_kernel<CL>, &cfg);
}

tsvd_status_t i8_product_prepare(tsvd_i8_s* h)
{
    const int most = I8_SMEM_LIMIT - 1024;
    TSVD_CUDA_OK(cudaFuncSetAttribute(i8_mma_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    TSVD_CUDA_OK(cudaFuncSetAttribute(i8_mma_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    TSVD_CUDA_OK(cudaFuncSetAttribute(i8_mma_kernel<4>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    TSVD_CUDA_OK(cudaFuncSetAttribute(i8_mma_kernel<8>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    TSVD_CUDA_OK(most_clusters<2>(&h->clusters[2]));
    TSVD_CUDA_OK(most_clusters<4>(&h->clusters[4]));
    TSVD_CUDA_OK(most_clusters<8>(&h->clusters[8]));
    return TSVD_OK;
}
