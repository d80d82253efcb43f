// The experts' ternary products on the tensor cores: codes as 4-bit floating point.
#include "rtn_experts.cuh"
#include "rtn_tcgen05.cuh"
#include "rtn_tensormap.cuh"

namespace rtn {

namespace {

constexpr int kExpandWarps = 8, kEpilogueWarps = 8;             // two of each for every quarter of the lanes
constexpr int kLoadWarp = kExpandWarps + kEpilogueWarps, kMmaWarp = kLoadWarp + 1;
constexpr int kThreads = (kMmaWarp + 1) * 32;
constexpr int kStageCodes = 256;                                // codes of K in a stage: a 128-byte row of 4-bit values, 32 columns
constexpr int kMaxRows = 192;                                   // of a tile
constexpr int kMaxStages = 6;
constexpr int kBoxRows = 16;                                    // of a copy
constexpr uint32_t kTries = 1u << 20;
constexpr uint32_t kScaleCols = 16;

struct TilesPlan {
    int max_rows;               // of a tile, a multiple of 16
    int stages;
    int col_tiles;
    int k_stages;
    uint32_t ring;              // offset of the ring in shared memory
    uint32_t stage_bytes;
    uint32_t smem;
};

struct Bars {
    uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2];
    uint32_t most[3][2];        // the largest |a_s S_x| and |a_o| of a tile, the next and the one after it, as bit patterns
    uint32_t tmem_slot;
    int dead;
};

// What the epilogue of a tile needs: a_s, a_s S_x, a_o and input row (-1: out of range) of its tokens, w_s, w_o, p3 and bias of its weight rows by
// TMEM lane; the votes of each 16 tokens and quarter of the lanes.
struct TileParams {
    float as[kMaxRows], asx[kMaxRows], ao[kMaxRows];
    int token[kMaxRows];
    float4 col[128];
    uint4 votes[4][kMaxRows / 4][2];
};

struct Tile { int e, row, rows, height; };

// 32 codes (a word of each plane) as four words of 4-bit values; nibble i of word r is code 4 i + r.  The magnitude of a nonzero weight is
// 1/2, 1, 2, 1 by r, so that the plane's bits are used where they are, and an input's its reciprocal: their product is 1.
__device__ __forceinline__ uint4 expand_weight(uint32_t nz, uint32_t pos)
{
    const uint32_t neg = ~pos;
    return make_uint4((nz & 0x11111111u) | (neg << 3 & 0x88888888u), (nz & 0x22222222u) | (neg << 2 & 0x88888888u),
                      (nz & 0x44444444u) | (neg << 1 & 0x88888888u), (nz >> 2 & 0x22222222u) | (neg & 0x88888888u));
}
__device__ __forceinline__ uint4 expand_input(uint32_t nz, uint32_t pos)
{
    const uint32_t neg = ~pos;
    return make_uint4((nz << 2 & 0x44444444u) | (neg << 3 & 0x88888888u), (nz & 0x22222222u) | (neg << 2 & 0x88888888u),
                      (nz >> 2 & 0x11111111u) | (neg << 1 & 0x88888888u), (nz >> 2 & 0x22222222u) | (neg & 0x88888888u));
}

// Instruction descriptor of kind::mxf4: e2m1 operands, both K-major, ue8m0 scales, fp32 accumulator.
__device__ __forceinline__ uint32_t idesc_mxf4(uint32_t M, uint32_t N)
{
    return (1u << 7) | (1u << 10) | ((N >> 3) << 17) | (1u << 23) | ((M >> 7) << 27);
}
// D[tmem] (+)= A[tmem] * B[smem]^T, one K = 64 slice; every scale is read at `scales`.
__device__ __forceinline__ void mma_mxf4(uint32_t elected, uint32_t d, uint32_t a, uint64_t b_desc, uint32_t idesc, uint32_t scales, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 e, %6, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], [%1], %2, %3, [%4], [%4], p;\n\t}"
        ::"r"(d), "r"(a), "l"(b_desc), "r"(idesc), "r"(scales), "r"((uint32_t)accumulate), "r"(elected) : "memory");
}

// kBoxRows rows of a [rows][pitch bytes] tensor from row r on, 128 bytes of each from byte x on, under the 128-byte swizzle.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int r, uint64_t* bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(r), "r"(tc::smem_addr(bar)) : "memory");
}

// The experts' rows one after the other as 4-bit values, `pitch` bytes each (a row's end is zeros); and the sums of their codes begin at 0.
__global__ void __launch_bounds__(256)
expand_inputs_kernel(const __grid_constant__ ExpertsArgs g, int nblk, int chunks, uint4* __restrict__ out)
{
    tc::pdl_trigger();
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    const uint32_t row = i / (uint32_t)chunks, c = i % (uint32_t)chunks;
    if (row >= g.R || row < (uint32_t)g.start[0] || row >= (uint32_t)g.start[g.E]) return;
    if (c == 0 && g.out_sum != nullptr) g.out_sum[row] = 0;
    const int64_t m = g.tokens != nullptr ? g.tokens[row] : row;
    uint32_t nz = 0, pos = 0;
    if ((int)(c / 4) < nblk && m >= 0 && m < g.T) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(g.a_packed) + (m * nblk + c / 4) * 8 + c % 4;
        nz = p[0]; pos = p[4];
    }
    out[(int64_t)row * chunks + c] = expand_input(nz, pos);
}

template <typename T, bool kGated, bool kCodes>
__global__ void __launch_bounds__(kThreads, 1)
experts_tiles_kernel(const __grid_constant__ ExpertsArgs g, const __grid_constant__ CUtensorMap map, const __grid_constant__ TilesPlan p)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    Bars& bar = *reinterpret_cast<Bars*>(smem);
    TileParams* params = reinterpret_cast<TileParams*>(smem + 256);              // [2]
    int* before = reinterpret_cast<int*>(params + 2);                            // [E + 1] tiles before an expert's
    int* first = before + g.E + 1;                                               // [E] its first row
    int* count = first + g.E;                                                    // [E] its rows
    int* height = count + g.E;                                                   // [E] rows of its tiles
    static_assert(sizeof(Bars) <= 256, "barriers");
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    volatile int* dead = &bar.dead;
    const uint32_t ring = tc::smem_addr(smem) + p.ring;

    if (warp == kMmaWarp) tc::tmem_alloc(&bar.tmem_slot, 512);
    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) { tc::mbar_init(&bar.full[i], 5); tc::mbar_init(&bar.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { tc::mbar_init(&bar.acc_full[i], 1); tc::mbar_init(&bar.acc_empty[i], kEpilogueWarps); }
        tc::mbar_init_fence();
        bar.dead = 0;
    }
    // Tiles of each expert: as few as hold its rows, and of about the same height, so that little of the last one is empty.
    if (warp == 0) {
        int sum = 0;
        for (int e0 = 0; e0 < g.E; e0 += 32) {
            const int e = e0 + lane;
            int s = 0, n = 0;
            if (e < g.E) {
                s = g.start[e];
                const int64_t len = (int64_t)g.start[e + 1] - s;
                if (s >= 0 && len >= 0 && s + len <= g.R) n = (int)len;
                else if (blockIdx.x == 0) atomicOr(g.status, kStatusBadIndex);
            }
            const int tiles = (n + p.max_rows - 1) / p.max_rows;
            int x = tiles;
            #pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, d);
                if (lane >= d) x += y;
            }
            if (e < g.E) {
                before[e] = sum + x - tiles; first[e] = s; count[e] = n;
                height[e] = tiles > 0 ? ((n + tiles - 1) / tiles + 15) / 16 * 16 : 0;
            }
            sum += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0) before[g.E] = sum;
    }
    if (threadIdx.x < 6) bar.most[threadIdx.x / 2][threadIdx.x % 2] = 0;
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    const uint32_t tmem = bar.tmem_slot;
    const uint32_t acc_cols = (uint32_t)p.max_rows, scales = tmem + 2 * acc_cols, a_tmem = scales + kScaleCols;
    if (warp >= kExpandWarps && warp < kExpandWarps + 4) {                        // every scale is 1
        uint32_t one[16];
        #pragma unroll
        for (int i = 0; i < 16; ++i) one[i] = 0x7f7f7f7fu;
        tc::tmem_st16(scales + ((uint32_t)((warp & 3) * 32) << 16), one);
        tc::tmem_st_wait();
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();

    // Tiles go round the CTAs with the columns fastest: those at work at a time share their rows.
    const uint32_t cols = (uint32_t)p.col_tiles, total = (uint32_t)before[g.E] * cols;
    auto find = [&](uint32_t t) {                                                 // whole warp
        const int rt = (int)(t / cols);
        Tile r{0, 0, 0, 16};
        for (int e0 = 0; e0 < g.E; e0 += 32) {
            const int e = e0 + lane;
            const uint32_t who = __ballot_sync(0xffffffffu, e < g.E && before[e] <= rt && rt < before[e + 1]);
            if (who != 0) {
                r.e = e0 + __ffs(who) - 1;
                r.height = height[r.e];
                const int at = (rt - before[r.e]) * r.height, left = count[r.e] - at;
                r.row = first[r.e] + at;
                r.rows = left < r.height ? left : r.height;
                break;
            }
        }
        return r;
    };
    auto warp_wait = [&](uint64_t* m, uint32_t parity) {
        const bool ok = __all_sync(0xffffffffu, tc::mbar_wait_tries(m, parity & 1u, kTries)) != 0;
        if (!ok) *dead = 1;
        return ok;
    };
    const int quad = warp & 3;
    const int64_t nblk = (g.K + kBlockCodes - 1) / kBlockCodes;
    constexpr int kTileOuts = kGated ? 64 : 128;
    // The output that TMEM lane 32 q + l belongs to, so that the lanes r, r + 8, ... which one thread of the epilogue reads are adjacent outputs; gated,
    // lanes l >= 16 are the rows that those of l - 16 are multiplied with.
    auto output_at = [&](uint32_t t, int q, int l) {
        return (int64_t)(t % cols) * kTileOuts + (kGated ? q * 16 + 2 * (l & 7) + (l >> 3 & 1) : q * 32 + 4 * (l & 7) + (l >> 3));
    };
    bool alive = true;

    if (warp < kExpandWarps) {
        // ------------------------------------------------------------ weights: a team of four warps has every other stage
        const uint4* __restrict__ W = reinterpret_cast<const uint4*>(g.w_packed);
        uint4 next[4];
        uint32_t t = blockIdx.x;                                                  // the stage that `next` is of
        int k = warp >> 2, left = 0;                                              // blocks of the row from this stage on
        const uint4* src = nullptr;
        auto enter = [&]() {                                                      // stage k of tile t, or k - k_stages of the next, ...
            bool moved = src == nullptr;
            while (k >= p.k_stages && t < total) { k -= p.k_stages; t += gridDim.x; moved = true; }
            if (moved && t < total) {
                const int64_t f = output_at(t, quad, lane), e = find(t).e;
                src = W;
                left = 0;
                if (f < g.F) {
                    src = W + ((e * g.N + (kGated && lane >= 16 ? g.F + f : f)) * nblk + 2 * k) * 2;
                    left = (int)nblk - 2 * k;
                }
            }
        };
        auto fetch = [&]() {
            #pragma unroll
            for (int i = 0; i < 2; ++i) {
                next[2 * i] = next[2 * i + 1] = make_uint4(0, 0, 0, 0);
                if (i < left) { next[2 * i] = __ldg(src + 2 * i); next[2 * i + 1] = __ldg(src + 2 * i + 1); }
            }
        };
        enter();
        if (t < total) fetch();
        int s = warp >> 2;
        uint32_t phase = 0;
        while (t < total) {
            // expanded before the slot is free: what follows the wait is the store alone
            uint32_t o[2][16];
            #pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 c0 = expand_weight(next[2 * i].x, next[2 * i + 1].x), c1 = expand_weight(next[2 * i].y, next[2 * i + 1].y);
                const uint4 c2 = expand_weight(next[2 * i].z, next[2 * i + 1].z), c3 = expand_weight(next[2 * i].w, next[2 * i + 1].w);
                o[i][0] = c0.x; o[i][1] = c0.y; o[i][2] = c0.z; o[i][3] = c0.w; o[i][4] = c1.x; o[i][5] = c1.y; o[i][6] = c1.z; o[i][7] = c1.w;
                o[i][8] = c2.x; o[i][9] = c2.y; o[i][10] = c2.z; o[i][11] = c2.w; o[i][12] = c3.x; o[i][13] = c3.y; o[i][14] = c3.z; o[i][15] = c3.w;
            }
            k += 2; src += 8; left -= 4;
            enter();
            if (t < total) fetch();
            if (!warp_wait(&bar.empty[s], phase + 1)) break;
            const uint32_t at = a_tmem + (uint32_t)(s * 32) + ((uint32_t)(quad * 32) << 16);
            tc::tmem_st16(at, o[0]);
            tc::tmem_st16(at + 16u, o[1]);
            tc::tmem_st_wait();
            tc::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bar.full[s]);
            s += 2;
            if (s >= p.stages) { s -= p.stages; phase ^= 1; }
        }
    } else if (warp == kLoadWarp) {
        // ------------------------------------------------------------ input rows: a lane has 16 of them
        tc::pdl_wait();
        int s = 0;
        uint32_t phase = 0;
        for (uint32_t t = blockIdx.x; t < total && alive; t += gridDim.x) {
            const Tile tile = find(t);
            for (int k = 0; k < p.k_stages; ++k) {
                if (!(alive = warp_wait(&bar.empty[s], phase + 1))) break;
                if (lane == 0) tc::mbar_arrive_expect_tx(&bar.full[s], (uint32_t)tile.height * 128u);
                __syncwarp();
                if (lane * kBoxRows < tile.height)
                    load_box(ring + (uint32_t)s * p.stage_bytes + (uint32_t)lane * (kBoxRows * 128u), &map, k * 128, tile.row + lane * kBoxRows, &bar.full[s]);
                if (++s == p.stages) { s = 0; phase ^= 1; }
            }
        }
        // nobody leaves while copies are on their way: the last of each stage
        for (int i = 0; i < p.stages; ++i) {
            const uint32_t uses = i < s ? phase + 1 : phase;                      // parity of the number of copies to this stage
            tc::mbar_wait_tries(&bar.full[i], (uses + 1) & 1u, kTries);
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------ products
        const uint32_t elected = tc::elect_one();
        const uint64_t desc = tc::smem_desc_sw128(ring, 0);
        int s = 0;
        uint32_t phase = 0, ti = 0;
        for (uint32_t t = blockIdx.x; t < total && alive; t += gridDim.x, ++ti) {
            const uint32_t idesc = idesc_mxf4(128, (uint32_t)__shfl_sync(0xffffffffu, find(t).height, 0)), d = tmem + (ti & 1) * acc_cols;
            if (!(alive = warp_wait(&bar.acc_empty[ti & 1], (ti >> 1) + 1))) break;
            for (int k = 0; k < p.k_stages; ++k) {
                if (!(alive = warp_wait(&bar.full[s], phase))) break;
                tc::tc_fence_after_sync();
                const uint64_t b = desc + (uint64_t)((uint32_t)s * (p.stage_bytes >> 4));
                const uint32_t a = a_tmem + (uint32_t)(s * 32);
                #pragma unroll
                for (int j = 0; j < 4; ++j)                                       // K = 64: 32 bytes, eight columns
                    mma_mxf4(elected, d, a + (uint32_t)(j * 8), b + (uint64_t)(j * 2), idesc, scales, k > 0 || j > 0);
                if (elected) tc::mma_commit(&bar.empty[s]);
                __syncwarp();
                if (++s == p.stages) { s = 0; phase ^= 1; }
            }
            if (elected && alive) tc::mma_commit(&bar.acc_full[ti & 1]);
            __syncwarp();
        }
    } else {
        // ------------------------------------------------------------ write out: a warp has a quarter of the lanes and every other 16 tokens; a thread
        // kOwn adjacent outputs of two tokens in each 8.
        constexpr int kOwn = kGated ? 2 : 4;
        const int mine = threadIdx.x - kExpandWarps * 32, half = (warp - kExpandWarps) >> 2, r8 = lane >> 2, q4 = lane & 3;
        // Parameters of the tile after this one, asked for as they are and looked at when this one is done: of token `mine`, of TMEM lane `mine`.
        struct Raw { int token; float as, ao, ws, wo, bias; int sx, sw; bool col; };
        Raw raw{};
        int token_ahead = -1;
        Tile tile_ahead{};
        auto ask_token = [&](uint32_t t) {                                        // input row of token `mine` of tile t, a tile ahead of its parameters
            token_ahead = -1;
            if (t >= total) return;
            tile_ahead = find(t);
            if (mine < tile_ahead.rows) token_ahead = g.tokens != nullptr ? g.tokens[tile_ahead.row + mine] : tile_ahead.row + mine;
        };
        auto ask_params = [&](uint32_t t) {                                       // after ask_token(t)
            raw.token = -1; raw.col = false;
            if (t >= total) return;
            if (mine < tile_ahead.rows) {
                const int64_t m = token_ahead;
                if (m >= 0 && m < g.T) {
                    const int64_t i = g.ep.n_aparam == 1 ? 0 : m;
                    raw.token = (int)m; raw.as = g.ep.a_scale[i]; raw.ao = g.ep.a_offset[i]; raw.sx = g.a_sum[m];
                } else if (t % cols == 0) atomicOr(g.status, kStatusBadIndex);
            }
            if (mine < 128) {
                const int64_t f = output_at(t, mine >> 5, mine & 31);
                if (f < g.F) {
                    const int64_t at = (int64_t)tile_ahead.e * g.N + (kGated && (mine & 16) ? g.F + f : f), i = g.ep.n_wparam == 1 ? 0 : at;
                    raw.col = true; raw.ws = g.ep.w_scale[i]; raw.wo = g.ep.w_offset[i]; raw.sw = g.w_sum[at];
                    raw.bias = g.bias != nullptr ? g.bias[at] : 0.f;
                }
            }
        };
        auto keep = [&](TileParams& q, uint32_t (&most)[2], int rows) {
            if (mine < kMaxRows) {
                const float nan = __int_as_float(0x7fffffff);
                float as = 0.f, asx = 0.f, ao = 0.f;
                if (mine < rows) {
                    as = raw.token >= 0 ? raw.as : nan; ao = raw.token >= 0 ? raw.ao : nan;
                    asx = raw.token >= 0 ? raw.as * (float)raw.sx : nan;
                }
                q.as[mine] = as; q.asx[mine] = asx; q.ao[mine] = ao; q.token[mine] = raw.token;
                if constexpr (kCodes) {
                    const uint32_t a = __reduce_max_sync(0xffffffffu, __float_as_uint(fabsf(asx))), b = __reduce_max_sync(0xffffffffu, __float_as_uint(fabsf(ao)));
                    if (lane == 0) { atomicMax(&most[0], a); atomicMax(&most[1], b); }
                }
            }
            if (mine < 128) {
                ColParams c{0.f, 0.f, 0.f, 0.f};
                if (raw.col) c = ColParams{raw.ws, raw.wo, (float)((double)raw.ws * (double)raw.sw + (double)g.K * (double)raw.wo), raw.bias};
                q.col[mine] = make_float4(c.ws, c.wo, c.p3, c.bias);
            }
        };
        ask_token(blockIdx.x);
        ask_params(blockIdx.x);
        Tile tile = tile_ahead;
        keep(params[0], bar.most[0], tile.rows);
        ask_token(blockIdx.x + gridDim.x);
        asm volatile("bar.sync 1, %0;" ::"n"(kEpilogueWarps * 32) : "memory");
        tc::pdl_wait();
        const int64_t width = (g.F + kBlockCodes - 1) / kBlockCodes * kBlockCodes;
        const bool vec = kCodes || ((reinterpret_cast<uintptr_t>(g.out) % (kOwn * sizeof(T))) == 0 && g.out_stride % kOwn == 0);
        uint32_t ti = 0, m3 = 0;
        for (uint32_t t = blockIdx.x; t < total; t += gridDim.x, ++ti) {
            const uint32_t(&most)[2] = bar.most[m3];
            TileParams& here = params[ti & 1];
            const Tile next_tile = tile_ahead;
            if (mine < 2) bar.most[m3 == 0 ? 2 : m3 - 1][mine] = 0;                 // the last tile's, for the one after the next
            ask_params(t + gridDim.x);
            ask_token(t + 2 * gridDim.x);
            // this thread's weight rows: kOwn outputs, or kOwn and the kOwn that they are multiplied with
            pair_t ws[4], wo[4], p3[4], bias[4];
            float off = 0.f, lo = 0.f, hi = 0.f;
            #pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 c = here.col[quad * 32 + r8 + 8 * j];
                ws[j] = make_pair(c.x, c.x); wo[j] = make_pair(c.y, c.y); p3[j] = make_pair(c.z, c.z); bias[j] = make_pair(c.w, c.w);
                // what the terms of the affine form other than the product add up to at most, twice (they may cancel)
                if constexpr (kCodes) {
                    const float x = __uint_as_float(most[0]) * fabsf(c.y) + __uint_as_float(most[1]) * fabsf(c.z) + fabsf(c.w);
                    off = !(x <= off) ? x : off;                                   // (a NaN stays)
                }
            }
            if constexpr (kCodes) { lo = g.t_lo[g.n_thr == 1 ? 0 : tile.e]; hi = g.t_hi[g.n_thr == 1 ? 0 : tile.e]; off *= 2.f; }
            const int64_t f = output_at(t, quad, r8);                              // the first of this thread's outputs
            alive = warp_wait(&bar.acc_full[ti & 1], ti >> 1);
            tc::tc_fence_after_sync();
            const uint32_t acc = tmem + (ti & 1) * acc_cols + ((uint32_t)(quad * 32) << 16);
            #pragma unroll 1
            for (int c = half * 16; alive && c < tile.rows; c += 32) {
                uint32_t v[2][8];                                                  // TMEM lanes r8, r8 + 8 and r8 + 16, r8 + 24
                tc::tmem_ld_16x16(acc + (uint32_t)c, v[0]);
                tc::tmem_ld_16x16(acc + (uint32_t)c + (16u << 16), v[1]);
                tc::tmem_ld_wait();
                bool near = false;
                #pragma unroll
                for (int a = 0; a < 2; ++a) {
                    const int at = c + 8 * a + 2 * q4;                             // tokens at and at + 1
                    const float2 as = *reinterpret_cast<const float2*>(&here.as[at]), sx = *reinterpret_cast<const float2*>(&here.asx[at]);
                    const float2 ao = *reinterpret_cast<const float2*>(&here.ao[at]);
                    const pair_t as2 = make_pair(as.x, as.y), sx2 = make_pair(sx.x, sx.y), ao2 = make_pair(ao.x, ao.y);
                    float y[4][2];                                                 // by weight row and token
                    #pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t* S = &v[j >> 1][4 * a + 2 * (j & 1)];
                        take_pair(fma_pair(ws[j], mul_pair(as2, make_pair(__uint_as_float(S[0]), __uint_as_float(S[1]))),
                                           fma_pair(wo[j], sx2, fma_pair(p3[j], ao2, bias[j]))), y[j][0], y[j][1]);
                    }
                    float o[kOwn][2];
                    if (g.act == RTN_ACT_SILU) {
                        #pragma unroll
                        for (int j = 0; j < kOwn; ++j) { o[j][0] = fast_silu(y[j][0]); o[j][1] = fast_silu(y[j][1]); }
                    } else if (g.act == RTN_ACT_NONE) {
                        #pragma unroll
                        for (int j = 0; j < kOwn; ++j) { o[j][0] = y[j][0]; o[j][1] = y[j][1]; }
                    } else {
                        #pragma unroll
                        for (int j = 0; j < kOwn; j += 2) {
                            const float4 x = activation4(make_float4(y[j][0], y[j][1], y[j + 1][0], y[j + 1][1]), g.act);
                            o[j][0] = x.x; o[j][1] = x.y; o[j + 1][0] = x.z; o[j + 1][1] = x.w;
                        }
                    }
                    if constexpr (kGated) {
                        #pragma unroll
                        for (int j = 0; j < kOwn; ++j) { o[j][0] *= y[kOwn + j][0]; o[j][1] *= y[kOwn + j][1]; }
                    }
                    if constexpr (kCodes) {
                        uint32_t nz[2][kOwn], up[2][kOwn];
                        #pragma unroll
                        for (int i = 0; i < 2; ++i)
                            #pragma unroll
                            for (int j = 0; j < kOwn; ++j) {
                                // (the bound of output_of: |y| and the other terms for what the terms add up to; gated,
                                // |y2| (25 |y1| + 6.8 off) + |y1| (7 |y2| + 6 off) <= (32 |y1| + 6.8 off)(|y2| + off))
                                constexpr float u = 1.25f * kUnit;
                                const float e = fmaf(32.f * u, fabsf(y[j][i]), 6.8f * u * off), x = o[j][i];
                                const float err = kGated ? e * (fabsf(y[kGated ? kOwn + j : j][i]) + off) : e;
                                const bool p = x > hi, n = p || x < lo;
                                near = near || !(fminf(fabsf(x - lo), fabsf(x - hi)) > err);
                                nz[i][j] = __ballot_sync(0xffffffffu, n);
                                up[i][j] = __ballot_sync(0xffffffffu, p);
                            }
                        if (lane == 0) {
                            #pragma unroll
                            for (int i = 0; i < 2; ++i)
                                #pragma unroll
                                for (int j = 0; j < kOwn; j += 2) here.votes[quad][c / 4 + 2 * a + i][j / 2] = make_uint4(nz[i][j], up[i][j], nz[i][j + 1], up[i][j + 1]);
                        }
                    }
                    if (!kCodes || g.out != nullptr) {
                        #pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            if (at + i >= tile.rows) continue;
                            T* out = static_cast<T*>(g.out) + (int64_t)(tile.row + at + i) * g.out_stride + f;
                            if (!kCodes && vec && f + kOwn <= g.F) {
                                if constexpr (sizeof(T) == 2) {
                                    if constexpr (kOwn == 4) *reinterpret_cast<uint2*>(out) = make_uint2(pack2<T>(o[0][i], o[1][i]), pack2<T>(o[2][i], o[3][i]));
                                    else *reinterpret_cast<uint32_t*>(out) = pack2<T>(o[0][i], o[1][i]);
                                } else {
                                    if constexpr (kOwn == 4) *reinterpret_cast<float4*>(out) = make_float4(o[0][i], o[1][i], o[2][i], o[3][i]);
                                    else *reinterpret_cast<float2*>(out) = make_float2(o[0][i], o[1][i]);
                                }
                            } else {
                                #pragma unroll
                                for (int j = 0; j < kOwn; ++j) if (f + j < g.F) out[j] = from_f32<T>(o[j][i]);
                            }
                        }
                    }
                }
                if constexpr (kCodes) {
                    if (__any_sync(0xffffffffu, near)) {                           // the 16 tokens again, in double
                        #pragma unroll 1
                        for (int a = 0; a < 2; ++a) {
                            uint32_t w[2][4];
                            tc::tmem_ld_16x8(acc + (uint32_t)(c + 8 * a), w[0]);
                            tc::tmem_ld_16x8(acc + (uint32_t)(c + 8 * a) + (16u << 16), w[1]);
                            tc::tmem_ld_wait();
                            #pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const int at = c + 8 * a + 2 * q4 + i, m = at < tile.rows ? here.token[at] : -1;
                                uint32_t nz[kOwn], up[kOwn];
                                #pragma unroll
                                for (int j = 0; j < kOwn; ++j) {
                                    bool p = false, n = false;
                                    if (m >= 0 && f + j < g.F) {
                                        const double x = exact_value(g, m, tile.e, f + j, __uint_as_float(w[j >> 1][2 * (j & 1) + i]),
                                                                     __uint_as_float(w[1][2 * (j & 1) + i]));
                                        p = x > (double)hi;
                                        n = p || x < (double)lo;
                                    }
                                    __syncwarp();
                                    nz[j] = __ballot_sync(0xffffffffu, n);
                                    up[j] = __ballot_sync(0xffffffffu, p);
                                }
                                if (lane == 0) {
                                    #pragma unroll
                                    for (int j = 0; j < kOwn; j += 2) here.votes[quad][c / 4 + 2 * a + i][j / 2] = make_uint4(nz[j], up[j], nz[j + 1], up[j + 1]);
                                }
                            }
                        }
                    }
                }
            }
            tc::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bar.acc_empty[ti & 1]);
            m3 = m3 == 2 ? 0 : m3 + 1;
            keep(params[(ti + 1) & 1], bar.most[m3], next_tile.rows);
            asm volatile("bar.sync 1, %0;" ::"n"(kEpilogueWarps * 32) : "memory");
            if (*dead) break;                                                     // (all of them, whichever gave up)
            if constexpr (kCodes) {
                // a token's codes of this tile, from the votes: bit 4 r + q of vote j is output kOwn r + j of a quarter, for token 2 q + i
                if (mine < tile.rows) {
                    const int q = mine >> 1 & 3, slot = mine / 16 * 4 + (mine >> 3 & 1) * 2 + (mine & 1);
                    const int64_t f0 = (int64_t)(t % cols) * kTileOuts;
                    uint32_t nz[4], up[4];
                    #pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint4 b0 = here.votes[w][slot][0];
                        nz[w] = (b0.x >> q & 0x11111111u) | (b0.z >> q & 0x11111111u) << 1;
                        up[w] = (b0.y >> q & 0x11111111u) | (b0.w >> q & 0x11111111u) << 1;
                        if constexpr (kGated) {
                            auto squeeze = [](uint32_t x) {                        // two bits of every four
                                x = (x | x >> 2) & 0x0f0f0f0fu;
                                x = (x | x >> 4) & 0x00ff00ffu;
                                return (x | x >> 8) & 0x0000ffffu;
                            };
                            nz[w] = squeeze(nz[w]); up[w] = squeeze(up[w]);
                        } else {
                            const uint4 b1 = here.votes[w][slot][1];
                            nz[w] |= (b1.x >> q & 0x11111111u) << 2 | (b1.z >> q & 0x11111111u) << 3;
                            up[w] |= (b1.y >> q & 0x11111111u) << 2 | (b1.w >> q & 0x11111111u) << 3;
                        }
                        constexpr int kBits = kGated ? 16 : 32;                    // (padding: zeros)
                        const int64_t n = g.F - f0 - w * kBits;
                        if (n < kBits) { const uint32_t real = n <= 0 ? 0u : (1u << (uint32_t)n) - 1u; nz[w] &= real; up[w] &= real; }
                    }
                    uint8_t* to = g.out_packed + (int64_t)(tile.row + mine) * (width / 4) + f0 / kBlockCodes * kBlockBytes + f0 % kBlockCodes / 8;
                    if constexpr (kGated) {
                        *reinterpret_cast<uint2*>(to) = make_uint2(nz[0] | nz[1] << 16, nz[2] | nz[3] << 16);
                        *reinterpret_cast<uint2*>(to + 16) = make_uint2(up[0] | up[1] << 16, up[2] | up[3] << 16);
                    } else {
                        *reinterpret_cast<uint4*>(to) = make_uint4(nz[0], nz[1], nz[2], nz[3]);
                        *reinterpret_cast<uint4*>(to + 16) = make_uint4(up[0], up[1], up[2], up[3]);
                    }
                    const int sum = 2 * (__popc(up[0]) + __popc(up[1]) + __popc(up[2]) + __popc(up[3])) - (__popc(nz[0]) + __popc(nz[1]) + __popc(nz[2]) + __popc(nz[3]));
                    if (sum != 0) atomicAdd(&g.out_sum[tile.row + mine], sum);     // (whole numbers: any order gives the same)
                }
            }
            tile = next_tile;
        }
    }

    if (!alive) *dead = 1;
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    if (threadIdx.x == 0 && *dead) atomicOr(g.status, kStatusWaitTimeout);
    if (warp == kMmaWarp) tc::tmem_dealloc(tmem, 512);
}

// Rows of a tile at most, from the rows that an expert has on average: what makes rounds of tiles times a tile's time least.
TilesPlan make_plan(const ExpertsArgs& g)
{
    TilesPlan p{};
    const int outs = g.gated ? 64 : 128;
    const int64_t width = g.out_packed != nullptr ? (g.F + kBlockCodes - 1) / kBlockCodes * kBlockCodes : g.F;
    p.col_tiles = (int)((width + outs - 1) / outs);
    p.k_stages = (int)((g.K + kStageCodes - 1) / kStageCodes);
    const double used = (double)(g.R < g.E ? g.R : g.E), each = (double)g.R / used, sms = device_sm_count();
    double best = 0.0;
    for (int h = 16; h <= 160; h += 16) {
        const double per = (double)(int64_t)((each + h - 1) / h), tiles = used * per * p.col_tiles, height = each / per < 16 ? 16 : each / per;
        const double stage = 2.6 * height > 350.0 ? 2.6 * height : 350.0, loop = stage * p.k_stages, out = 20.0 * height + 500.0;
        const double rounds = tiles / sms < 1.0 ? 1.0 : (double)(int64_t)((tiles + sms - 1) / sms);
        const double cost = rounds * (loop > out ? loop : out) + (loop > out ? out : loop);
        if (p.max_rows == 0 || cost < best) { best = cost; p.max_rows = h; }
    }
    p.stage_bytes = (uint32_t)p.max_rows * 128u;
    p.ring = (uint32_t)((256 + 2 * sizeof(TileParams) + (4 * g.E + 1) * 4 + 1023) / 1024 * 1024);
    const int by_smem = (int)((227u * 1024u - p.ring) / p.stage_bytes), by_tmem = (512 - 2 * p.max_rows - (int)kScaleCols) / 32;
    p.stages = by_smem < by_tmem ? by_smem : by_tmem;
    if (p.stages > kMaxStages) p.stages = kMaxStages;
    p.smem = p.ring + (uint32_t)p.stages * p.stage_bytes;
    return p;
}

}  // namespace

cudaError_t launch_experts_tiles(const ExpertsArgs& g, cudaStream_t s)
{
    const TilesPlan p = make_plan(g);
    const EncodeTiledFn encode = encode_tiled_fn();
    if (encode == nullptr) return cudaErrorNotSupported;
    const int nblk = (int)((g.K + kBlockCodes - 1) / kBlockCodes), pitch = p.k_stages * 128;
    void* scratch = nullptr;
    cudaError_t e = scratch_alloc(&scratch, (size_t)g.R * pitch, s);
    if (e != cudaSuccess) return e;
    CUtensorMap map;
    const cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)g.R}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {128, kBoxRows}, unit[2] = {1, 1};
    if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, scratch, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) e = cudaErrorInvalidValue;
    if (e == cudaSuccess) {
        const int64_t threads = g.R * (pitch / 16);
        expand_inputs_kernel<<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(g, nblk, pitch / 16, static_cast<uint4*>(scratch));
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) {
        e = with_dtype(g.dtype, [&](auto t) {
            using T = decltype(t);
            auto run = [&](auto kernel) {
                cudaError_t x = allow_shared_memory(kernel);
                if (x != cudaSuccess) return x;
                return launch_pdl(kernel, dim3((unsigned)device_sm_count()), dim3(kThreads), p.smem, s, g, map, p);
            };
            if (g.out_packed != nullptr) return g.gated ? run(experts_tiles_kernel<T, true, true>) : run(experts_tiles_kernel<T, false, true>);
            return g.gated ? run(experts_tiles_kernel<T, true, false>) : run(experts_tiles_kernel<T, false, false>);
        });
    }
    const cudaError_t e2 = cudaFreeAsync(scratch, s);
    return e == cudaSuccess ? e2 : e;
}

// What the tensor-core form counts in 32 bits.
bool experts_tiles_supported(const ExpertsArgs& g)
{
    const int64_t pitch = (g.K + kStageCodes - 1) / kStageCodes * 8, cols = (g.F + 191) / 64 + 1;
    return g.R * pitch < (int64_t(1) << 32) - 256 && (g.R / 16 + g.E) * cols < (int64_t(1) << 31);
}

}  // namespace rtn
