// Ternary linear layer for few rows (decoding): out = act(affine(S_xw) + bias) + residual, S_xw by Eq. 9 (AND / XOR / popcount
// on the packed planes).
//
// Bound: DRAM, the packed weights read once (K/4 bytes per column against 2 POPC per 32 codes and row; from about four rows on
// the POPC rate binds).  A group of GL lanes (a power of two, at most a warp) owns CPG weight rows at a time: lane i takes
// the 128-code blocks i, i + GL, ... of each (32 adjacent bytes, so a group reads whole lines), keeps a
// counter pair per activation row and column, and one shuffle tree joins the group.  CPG columns at once keep that many loads in flight.
// 1 x 4096 x 4096 (4.3 MB of planes): 2.9 us in a graph, 0.2 of a plain copy's rate: the latency of a launch and of two loads one after
// the other; 48 x 1000 x 512: 5.0 us.
#include "rtn_internal.cuh"
#include "rtn_epilogue.cuh"
#include "rtn_tcgen05.cuh"

namespace rtn {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 8;             // activation rows of a pass

template <int MT, int CPG>
__global__ void __launch_bounds__(kThreads)
linear_rows_kernel(const GemmArgs g, const LinearArgs p, int GL)
{
    constexpr int kOut = MT * CPG;
    const int gl = threadIdx.x & (GL - 1);
    const int64_t group = (int64_t)blockIdx.x * (kThreads / GL) + threadIdx.x / GL;
    const int64_t n0 = group * CPG;
    const int64_t m0 = (int64_t)blockIdx.y * MT;
    const int64_t nblk = (g.K + kBlockCodes - 1) / kBlockCodes;
    const uint4* __restrict__ A = reinterpret_cast<const uint4*>(g.a_packed);
    const uint4* __restrict__ W = reinterpret_cast<const uint4*>(g.w_packed);
    int cnt[kOut];
    #pragma unroll
    for (int i = 0; i < kOut; ++i) cnt[i] = 0;
    // Lane o of the group finishes outputs o, o + GL, ... of its MT x CPG; the operands of the first are on their way during the loop
    // (fetched after it, one output after the other, they were most of the time of a small call).
    struct Params { float as, ao, ws, wo, bias, res; int sx, sw; bool ok; };
    auto fetch = [&](int o) {
        Params q;
        const int64_t m = m0 + o / CPG, n = n0 + o % CPG;
        q.ok = o < kOut && m < g.M && n < g.N;
        q.as = q.ao = q.ws = q.wo = q.bias = q.res = 0.f;
        q.sx = q.sw = 0;
        if (q.ok) {
            const EpilogueParams& ep = g.ep;
            const int64_t ia = ep.n_aparam == 1 ? 0 : m, iw = ep.n_wparam == 1 ? 0 : n;
            q.as = ep.a_scale[ia]; q.ao = ep.a_offset[ia]; q.ws = ep.w_scale[iw]; q.wo = ep.w_offset[iw];
            q.sx = g.a_sum[m]; q.sw = g.w_sum[n];
            if (p.bias != nullptr) q.bias = p.bias[n];
            if (p.residual != nullptr) q.res = load_as_f32(p.residual, m * p.res_stride + n, p.dtype);
        }
        return q;
    };
    Params first = fetch(gl);
    for (int64_t kb = gl; kb < nblk; kb += GL) {
        uint4 w1[CPG], w2[CPG];
        #pragma unroll
        for (int j = 0; j < CPG; ++j) {
            const bool ok = n0 + j < g.N;
            const uint4* src = W + ((ok ? n0 + j : 0) * nblk + kb) * 2;
            w1[j] = ok ? __ldg(src) : make_uint4(0, 0, 0, 0);
            w2[j] = ok ? __ldg(src + 1) : make_uint4(0, 0, 0, 0);
        }
        #pragma unroll
        for (int i = 0; i < MT; ++i) {
            const bool ok = m0 + i < g.M;
            const uint4* src = A + ((ok ? m0 + i : 0) * nblk + kb) * 2;
            const uint4 a1 = ok ? __ldg(src) : make_uint4(0, 0, 0, 0), a2 = __ldg(src + 1);
            #pragma unroll
            for (int j = 0; j < CPG; ++j) {
                const uint32_t c0 = a1.x & w1[j].x, c1 = a1.y & w1[j].y, c2 = a1.z & w1[j].z, c3 = a1.w & w1[j].w;
                cnt[i * CPG + j] += (__popc(c0) + __popc(c1)) + (__popc(c2) + __popc(c3))
                                  - 2 * ((__popc((a2.x ^ w2[j].x) & c0) + __popc((a2.y ^ w2[j].y) & c1)) +
                                         (__popc((a2.z ^ w2[j].z) & c2) + __popc((a2.w ^ w2[j].w) & c3)));
            }
        }
    }
    for (int d = GL / 2; d > 0; d >>= 1) {
        #pragma unroll
        for (int i = 0; i < kOut; ++i) cnt[i] += __shfl_xor_sync(0xffffffffu, cnt[i], d);
    }
    for (int o = gl; o < kOut; o += GL) {
        const Params q = o == gl ? first : fetch(o);
        int s = 0;
        #pragma unroll
        for (int i = 0; i < kOut; ++i) s = o == i ? cnt[i] : s;
        if (!q.ok) continue;
        // the arithmetic of the tensor-core forms, so that a row's result does not depend on how many rows it comes with
        const float p3 = (float)((double)q.ws * (double)q.sw + (double)g.K * (double)q.wo);
        const float y = activate(fmaf(q.as, fmaf(q.ws, (float)s, q.wo * (float)q.sx), q.ao * p3) + q.bias, p.act) + q.res;
        store_from_f32(p.out, (m0 + o / CPG) * p.out_stride + n0 + o % CPG, p.dtype, y);
    }
}

// ------------------------------------------------------------------------------------------------ some to many rows, small products

// linear_tiles_kernel: 128 weight rows (the MMA's M, lanes of tensor memory) by BT <= 64 tokens (its N), tcgen05.mma kind::i8.  Sixteen
// warps expand the bit planes of both operands into a ring of eight stages, a team of two warps to a stage and a whole
// K = 128 block at a time (three rows per lane in flight, and no team waits for another); a seventeenth issues the MMAs; then the
// sixteen write out.  A lane is one output column: its scale, offset, code sum and bias live in registers, and a warp's
// store is 32 adjacent columns of a token, with no staging.
// Bound: the expansion (280 warp instructions per 32 rows and block, epilogue included, with 0.42 of the issue slots used: the planes' loads are
// waited for) while the weights stream by; the epilogue for short K.  48 x 16384 x 4096 with bias and GELU: 17.2 us in a graph, of which the
// MMAs are 3 us (46 clocks each up to 48 columns, 48 at 64, by the probe; four to a block of K, 32 blocks); 777 x 1000 x 512 with bias and SiLU: 8.8 us.
// Few tiles and a long K: the K blocks are dealt to the CTAs of a cluster, which leave their int32 sums in shared memory and
// each finish a share of the tokens from all of them (exact whatever the order).
constexpr int kTileWarps = 16;
constexpr int kTileThreads = (kTileWarps + 1) * 32;
constexpr int kTileStages = 8;                  // 18 to 24 KB each
constexpr int kTeamWarps = kTileWarps / kTileStages;
constexpr int kTileMaxTokens = 64;
constexpr int kLaneRows = (4 + kTileMaxTokens / 32) / kTeamWarps;      // 32-row groups of a block to a warp
constexpr uint32_t kTileTries = 1u << 20;

struct TilePlan {
    int BT;                 // tokens of a tile, a multiple of 16
    int tiles_n, tiles_m;
    int slices;             // CTAs of a cluster, along K
    uint32_t tmem_cols;
    uint32_t smem_bytes;
};

struct TileBars {
    uint64_t full[kTileStages], empty[kTileStages], acc;
    uint32_t tmem_slot;
    int dead;
};

// One packed 128-code block of a row, expanded to eight 16-byte chunks `ld` rows apart.
__device__ __forceinline__ void expand_block(const uint4& nz, const uint4& sg, uint4* dst, int ld)
{
    uint32_t o[8];
    tc::unpack32(nz.x, sg.x, o);
    dst[0 * ld] = make_uint4(o[0], o[1], o[2], o[3]); dst[1 * ld] = make_uint4(o[4], o[5], o[6], o[7]);
    tc::unpack32(nz.y, sg.y, o);
    dst[2 * ld] = make_uint4(o[0], o[1], o[2], o[3]); dst[3 * ld] = make_uint4(o[4], o[5], o[6], o[7]);
    tc::unpack32(nz.z, sg.z, o);
    dst[4 * ld] = make_uint4(o[0], o[1], o[2], o[3]); dst[5 * ld] = make_uint4(o[4], o[5], o[6], o[7]);
    tc::unpack32(nz.w, sg.w, o);
    dst[6 * ld] = make_uint4(o[0], o[1], o[2], o[3]); dst[7 * ld] = make_uint4(o[4], o[5], o[6], o[7]);
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <typename T>
__global__ void __launch_bounds__(kTileThreads, 1)
linear_tiles_kernel(const GemmArgs g, const LinearArgs l, const TilePlan p)
{
    extern __shared__ __align__(128) uint8_t smem[];
    TileBars& bar = *reinterpret_cast<TileBars*>(smem);
    float4* token = reinterpret_cast<float4*>(smem + 512);                  // {a_s, a_o, S_x, -} of the tile's tokens
    uint8_t* ring = smem + 512 + kTileMaxTokens * 16;
    static_assert(sizeof(TileBars) <= 512, "barriers");
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x % p.slices);
    const int tile = (int)(blockIdx.x / p.slices);
    const int64_t n0 = (int64_t)(tile / p.tiles_m) * 128, m0 = (int64_t)(tile % p.tiles_m) * p.BT;
    const int nblk = (int)((g.K + kBlockCodes - 1) / kBlockCodes);
    const int kb0 = (int)((int64_t)nblk * rank / p.slices), kb1 = (int)((int64_t)nblk * (rank + 1) / p.slices);
    const uint32_t stage_bytes = (uint32_t)(128 + p.BT) * 128u;
    volatile int* dead = &bar.dead;

    if (warp == kTileWarps) tc::tmem_alloc(&bar.tmem_slot, p.tmem_cols);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kTileStages; ++i) { tc::mbar_init(&bar.full[i], kTeamWarps); tc::mbar_init(&bar.empty[i], 1); }
        tc::mbar_init(&bar.acc, 1);
        tc::mbar_init_fence();
        bar.dead = 0;
    }
    // the epilogue's operands, asked for now and looked at after the loop: a token's (one per thread), a column's
    const int quad = warp & 3;
    const int64_t n = n0 + quad * 32 + lane;
    const bool col_ok = n < g.N && warp < kTileWarps;
    float t_s = 0.f, t_o = 0.f, w_s = 0.f, w_o = 0.f, bias = 0.f;
    int t_x = 0, w_x = 0;
    if (threadIdx.x < p.BT && m0 + threadIdx.x < g.M) {
        const int64_t m = m0 + threadIdx.x;
        t_s = g.ep.a_scale[g.ep.n_aparam == 1 ? 0 : m]; t_o = g.ep.a_offset[g.ep.n_aparam == 1 ? 0 : m]; t_x = g.a_sum[m];
    }
    if (col_ok) {
        w_s = g.ep.w_scale[g.ep.n_wparam == 1 ? 0 : n]; w_o = g.ep.w_offset[g.ep.n_wparam == 1 ? 0 : n]; w_x = g.w_sum[n];
        if (l.bias != nullptr) bias = l.bias[n];
    }
    const uint4* __restrict__ W = reinterpret_cast<const uint4*>(g.w_packed);
    const uint4* __restrict__ X = reinterpret_cast<const uint4*>(g.a_packed);
    const int s = (warp < kTileWarps ? warp : 0) / kTeamWarps, member = warp % kTeamWarps;
    const int row_groups = 4 + (p.BT + 31) / 32;
    uint4* dst = reinterpret_cast<uint4*>(ring + s * stage_bytes);
    // A warp's 32-row groups of a block: member, member + 2, member + 4.  The planes of its next block are on their way while this one's
    // are expanded.
    uint4 nz[kLaneRows], sg[kLaneRows];
    auto load = [&](int i) {
        #pragma unroll
        for (int k = 0; k < kLaneRows; ++k) {
            const int rg = member + k * kTeamWarps;
            const bool isW = rg < 4;
            const int r = (isW ? rg : rg - 4) * 32 + lane;
            const int64_t row = (isW ? n0 : m0) + r;
            const bool ok = i < kb1 - kb0 && rg < row_groups && (isW || r < p.BT) && row < (isW ? g.N : g.M);
            nz[k] = sg[k] = make_uint4(0, 0, 0, 0);
            if (ok) { const uint4* q = (isW ? W : X) + (row * nblk + kb0 + i) * 2; nz[k] = __ldg(q); sg[k] = __ldg(q + 1); }
        }
    };
    if (warp < kTileWarps) load(s);
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    const uint32_t tmem = bar.tmem_slot;
    auto warp_wait = [&](uint64_t* m, uint32_t parity) {
        const bool ok = __all_sync(0xffffffffu, tc::mbar_wait_tries(m, parity & 1u, kTileTries)) != 0;
        if (!ok) *dead = 1;
        return ok;
    };

    if (warp < kTileWarps) {
        // ------------------------------------------------------------ expand: the warps of a team own one stage, so that a stage's
        // phases follow each other in one program order
        for (int i = s; i < kb1 - kb0; i += kTileStages) {
            if (!warp_wait(&bar.empty[s], (uint32_t)(i / kTileStages) + 1)) break;
            uint4 cnz[kLaneRows], csg[kLaneRows];
            #pragma unroll
            for (int k = 0; k < kLaneRows; ++k) { cnz[k] = nz[k]; csg[k] = sg[k]; }
            load(i + kTileStages);
            #pragma unroll
            for (int k = 0; k < kLaneRows; ++k) {
                const int rg = member + k * kTeamWarps;
                if (rg < 4) expand_block(cnz[k], csg[k], dst + rg * 32 + lane, 128);
                else if (rg < row_groups && (rg - 4) * 32 + lane < p.BT) expand_block(cnz[k], csg[k], dst + 128 * 8 + (rg - 4) * 32 + lane, p.BT);
            }
            tc::fence_smem_to_async_proxy();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bar.full[s]);
        }
        if (threadIdx.x < p.BT) token[threadIdx.x] = make_float4(t_s, t_o, (float)t_x, 0.f);
        asm volatile("bar.sync 1, %0;" ::"n"(kTileWarps * 32) : "memory");
    } else {
        // ------------------------------------------------------------ MMA
        const uint32_t elected = tc::elect_one();
        const uint32_t idesc = tc::idesc_i8(128, (uint32_t)p.BT);
        const uint32_t at = tc::smem_addr(ring);
        const uint64_t desc_w = tc::smem_desc_kmajor(at, 2048, 128), desc_x = tc::smem_desc_kmajor(at + 128u * 128u, (uint32_t)p.BT * 16u, 128);
        bool alive = true;
        for (int i = 0; i < kb1 - kb0; ++i) {
            const int s = i % kTileStages;
            if (!(alive = warp_wait(&bar.full[s], (uint32_t)(i / kTileStages)))) break;
            tc::tc_fence_after_sync();
            const uint64_t step = (uint64_t)(s * (stage_bytes >> 4));          // descriptors count 16 bytes
            #pragma unroll
            for (int j = 0; j < 4; ++j)                             // K = 32: chunks 2j and 2j + 1
                tc::mma_i8_ss(elected, tmem, desc_w + step + (uint64_t)(j * 256), desc_x + step + (uint64_t)(j * 2 * p.BT), idesc, i > 0 || j > 0);
            if (elected) tc::mma_commit(&bar.empty[s]);
            __syncwarp();
        }
        if (elected && alive) tc::mma_commit(&bar.acc);
        __syncwarp();
    }

    // ---------------------------------------------------------------- write out: column n0 + 32 (warp mod 4) + lane, every fourth
    // group of 4 tokens of the CTA's share
    const bool done = warp_wait(&bar.acc, 0);
    tc::tc_fence_after_sync();
    const int groups = p.BT / 4;
    int* part = reinterpret_cast<int*>(ring);                        // [token][128]
    if (p.slices > 1) {
        if (warp < kTileWarps && done) {
            for (int q = warp >> 2; q < groups; q += kTileWarps / 4) {
                uint32_t v[4];
                tc::tmem_ld4(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(q * 4), v);
                tc::tmem_ld_wait();
                #pragma unroll
                for (int x = 0; x < 4; ++x) part[(q * 4 + x) * 128 + quad * 32 + lane] = (int)v[x];
            }
        }
        cluster_sync();
    }
    if (warp < kTileWarps && done && !(p.slices > 1 && *dead)) {
        const float p3 = (float)((double)w_s * (double)w_x + (double)g.K * (double)w_o);
        const T* res = static_cast<const T*>(l.residual);
        T* out = static_cast<T*>(l.out);
        for (int q = (warp >> 2) * p.slices + rank; q < groups; q += kTileWarps / 4 * p.slices) {
            uint32_t v[4];
            if (p.slices == 1) {
                tc::tmem_ld4(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(q * 4), v);
            } else {
                #pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = 0;
                const uint32_t mine = tc::smem_addr(part + q * 4 * 128 + quad * 32 + lane);
                for (int r = 0; r < p.slices; ++r) {
                    uint32_t at;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(mine), "r"(r));
                    #pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        uint32_t y;
                        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(y) : "r"(at + (uint32_t)x * 512u) : "memory");
                        v[x] += y;
                    }
                }
            }
            const int64_t m = m0 + q * 4;
            const int rows = !col_ok || m >= g.M ? 0 : g.M - m < 4 ? (int)(g.M - m) : 4;
            float add[4] = {0.f, 0.f, 0.f, 0.f};
            if (res != nullptr) {
                const T* r = res + m * l.res_stride + n;
                #pragma unroll
                for (int x = 0; x < 4; ++x) { if (x < rows) add[x] = to_f32(*r); r += l.res_stride; }
            }
            if (p.slices == 1) tc::tmem_ld_wait();
            float y[4];
            #pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float4 t = token[q * 4 + x];
                y[x] = fmaf(t.x, fmaf(w_s, (float)(int)v[x], w_o * t.z), t.y * p3) + bias;
            }
            if (l.act != RTN_ACT_NONE) {
                const float4 a = activation4(make_float4(y[0], y[1], y[2], y[3]), l.act);
                y[0] = a.x; y[1] = a.y; y[2] = a.z; y[3] = a.w;
            }
            T* o = out + m * l.out_stride + n;
            #pragma unroll
            for (int x = 0; x < 4; ++x) { if (x < rows) *o = from_f32<T>(y[x] + add[x]); o += l.out_stride; }
        }
    }
    if (p.slices > 1) cluster_sync();            // nobody leaves while its sums are read
    if (threadIdx.x == 0 && *dead) atomicOr(g.status, kStatusWaitTimeout);
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    if (warp == kTileWarps) tc::tmem_dealloc(tmem, p.tmem_cols);
}

// False where gemm_i8_kernel does better.
bool make_tile_plan(int64_t M, int64_t N, int64_t K, TilePlan& p)
{
    const int sms = device_sm_count();
    const int nblk = (int)((K + kBlockCodes - 1) / kBlockCodes);
    p = TilePlan{};
    p.tiles_n = (int)((N + 127) / 128);
    if (p.tiles_n > sms) return false;
    // Tokens of a tile, and CTAs of a cluster that share its K (while one keeps at least four blocks and the machine has the SMs): what
    // makes rounds of CTAs times a tile's time least.  Per block the slower of expanding 128 + BT rows (1.6 clocks each) and the MMAs (2 BT);
    // 30 clocks per token for the epilogue, shared by a cluster, which takes 2000 to meet; 4000 to start and end.  Clusters of eight fill
    // three quarters of the machine at most (more of them wait for a place: 64 x 1024 x 16384 26 us, in clusters of four 16).  Where more than 64
    // tokens to a tile would do better, or one round of tiles is not enough, gemm_i8_kernel's larger tiles are ahead.
    double best = 0.0;
    const int most = M >= 256 ? 256 : (int)((M + 15) / 16 * 16);
    for (int bt = 16; bt <= most; bt += 16) {
        if (bt > 128 && bt % 32 != 0 && bt != most) continue;
        const int64_t tiles_m = (M + bt - 1) / bt, tiles = (int64_t)p.tiles_n * tiles_m;
        int slices = 1;
        while (slices < 8 && bt <= kTileMaxTokens && tiles * slices * 2 <= (slices < 4 ? sms : sms * 3 / 4) && nblk >= slices * 8) slices *= 2;
        const double block = 1.6 * (128 + bt) > 2.0 * bt ? 1.6 * (128 + bt) : 2.0 * bt;
        const double cost = (double)((tiles + sms - 1) / sms) * (4000.0 + (nblk + slices - 1) / slices * block + 30.0 * bt / slices + (slices > 1 ? 2000.0 : 0.0));
        if (p.BT == 0 || cost < best) { best = cost; p.BT = bt; p.slices = slices; p.tiles_m = (int)tiles_m; }
    }
    if (p.BT > kTileMaxTokens || (int64_t)p.tiles_n * p.tiles_m > sms) return false;
    p.tmem_cols = p.BT <= 32 ? 32 : 64;
    p.smem_bytes = 512 + kTileMaxTokens * 16 + (uint32_t)(kTileStages * (128 + p.BT) * 128);
    return true;
}

cudaError_t launch_tiles(const GemmArgs& g, const LinearArgs& l, const TilePlan& p, cudaStream_t s)
{
    return with_dtype(l.dtype, [&](auto t) {
        auto kernel = linear_tiles_kernel<decltype(t)>;
        cudaError_t e = allow_shared_memory(kernel);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t cfg;
        memset(&cfg, 0, sizeof(cfg));
        cfg.gridDim = dim3((unsigned)(p.tiles_n * p.tiles_m * p.slices));
        cfg.blockDim = dim3(kTileThreads);
        cfg.dynamicSmemBytes = p.smem_bytes;
        cfg.stream = s;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)p.slices;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, kernel, g, l, p);
    });
}

template <int MT, int CPG>
cudaError_t launch_rows(const GemmArgs& g, const LinearArgs& l, cudaStream_t s)
{
    const int64_t nblk = (g.K + kBlockCodes - 1) / kBlockCodes;
    int GL = 1;
    while (GL < nblk && GL < 32) GL *= 2;
    const int64_t groups = (g.N + CPG - 1) / CPG, per_cta = kThreads / GL;
    const dim3 grid((unsigned)((groups + per_cta - 1) / per_cta), (unsigned)((g.M + MT - 1) / MT));
    linear_rows_kernel<MT, CPG><<<grid, kThreads, 0, s>>>(g, l, GL);
    return cudaGetLastError();
}

}  // namespace

// Which of the three forms a shape takes; times in a graph on one B200 (bf16 out, us):
//                      M   N     K      rows   tiles  two launches
//   rows               1  4096  4096     2.7    8.3               5  4096  4096   5.5   8.4
//                      8  4096  4096     5.7    8.6               8 11008  4096  11.4  14.6
//                      8 16384  4096    15.3   14.8               4 16384 16384  27.0  41.1
//                     64  2048   512     4.6    5.6    8.6     1000   100   300   4.6   5.2  11.5
//   tiles             16  4096  4096     9.3    8.6   25.4       24  4096  4096  13.0   8.9  25.5
//                     16  4096 16384    23.7   16.0   83.5      643   809   247  10.3   5.1  10.2
//                    256  4096  4096           17.8   22.3      100  1000   128   7.9   4.5   6.5
//   two launches     512  4096  4096           34.0   22.4      256 16384  4096        66.9  33.4
// rows: the weights are streamed once per eight rows and the POPC rate binds, 2.9 us per million rows x columns x blocks, on top of 4 (with
// one or two blocks of K the lanes of a group are too few for the outputs); tiles start at 5.3 and take 0.11 us and more per block of K.
// Up to eight rows the weights are streamed once, and rows are within 4 % of tiles or ahead from three blocks of K on.
bool linear_rows_path(int64_t M, int64_t N, int64_t K)
{
    const double nblk = (double)((K + kBlockCodes - 1) / kBlockCodes);
    const bool rows_win = nblk > 2 && 2.9e-6 * (double)((M + 7) / 8 * 8) * (double)N * nblk <= 1.3 + 0.11 * nblk;
    return M <= kMaxRows || rows_win || !gemm_i8_supported(M, N, K);
}

cudaError_t launch_linear(const GemmArgs& g, const LinearArgs& l, cudaStream_t s)
{
    if (!linear_rows_path(g.M, g.N, g.K)) {
        TilePlan p;
        return make_tile_plan(g.M, g.N, g.K, p) ? launch_tiles(g, l, p, s) : launch_gemm_i8_linear(g, l, s);
    }
    if (g.M == 1) return launch_rows<1, 4>(g, l, s);
    if (g.M == 2) return launch_rows<2, 4>(g, l, s);
    if (g.M <= 4) return launch_rows<4, 4>(g, l, s);
    return launch_rows<8, 2>(g, l, s);
}

}  // namespace rtn
