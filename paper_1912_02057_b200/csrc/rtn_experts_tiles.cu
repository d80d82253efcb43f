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
    uint32_t tmem_slot;
    int dead;
};

struct TokenParams { float as[kMaxRows], asx[kMaxRows], ao[kMaxRows]; int token[kMaxRows]; };     // a_s, a_s S_x, a_o, input row (-1: out of range)

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
    TokenParams* token = reinterpret_cast<TokenParams*>(smem + 256);             // [2]
    int* sums = reinterpret_cast<int*>(token + 2);                               // [2][kMaxRows]
    int* before = sums + 2 * kMaxRows;                                           // [E + 1] tiles before an expert's
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
    if (threadIdx.x < 2 * kMaxRows) sums[threadIdx.x] = 0;
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
    // The weight row of a lane: 32 adjacent ones to a warp; gated, 16 and the 16 that they are multiplied with.
    auto output_at = [&](uint32_t t) { return (int64_t)(t % cols) * kTileOuts + (kGated ? quad * 16 + (lane & 15) : quad * 32 + lane); };
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
                const int64_t f = output_at(t), e = find(t).e;
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
            uint4 w[4];
            #pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = next[i];
            k += 2; src += 8; left -= 4;
            enter();
            if (t < total) fetch();
            if (!warp_wait(&bar.empty[s], phase + 1)) break;
            const uint32_t at = a_tmem + (uint32_t)(s * 32) + ((uint32_t)(quad * 32) << 16);
            #pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 c0 = expand_weight(w[2 * i].x, w[2 * i + 1].x), c1 = expand_weight(w[2 * i].y, w[2 * i + 1].y);
                const uint4 c2 = expand_weight(w[2 * i].z, w[2 * i + 1].z), c3 = expand_weight(w[2 * i].w, w[2 * i + 1].w);
                const uint32_t o[16] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w, c2.x, c2.y, c2.z, c2.w, c3.x, c3.y, c3.z, c3.w};
                tc::tmem_st16(at + (uint32_t)(i * 16), o);
            }
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
        // ------------------------------------------------------------ write out: a warp has 32 lanes (weight rows) of every other 32 tokens
        const int mine = threadIdx.x - kExpandWarps * 32, half = (warp - kExpandWarps) >> 2;
        struct Own { Tile tile; float as, asx, ao; int token; ColParams col; };
        auto fetch = [&](uint32_t t) {
            Own o{};
            o.token = -1;
            if (t >= total) return o;
            o.tile = find(t);
            if (mine < o.tile.rows) {
                const RowParams r = row_params(g, o.tile.row + mine);
                o.as = r.as; o.asx = r.as * r.sx; o.ao = r.ao; o.token = r.token;
                if (r.token < 0 && t % cols == 0) atomicOr(g.status, kStatusBadIndex);
            }
            const int64_t f = output_at(t);
            if (f < g.F) o.col = col_params(g, o.tile.e, kGated && lane >= 16 ? g.F + f : f);
            return o;
        };
        auto keep = [&](const Own& o, uint32_t at) {
            if (mine < kMaxRows) { token[at].as[mine] = o.as; token[at].asx[mine] = o.asx; token[at].ao[mine] = o.ao; token[at].token[mine] = o.token; }
        };
        Own next = fetch(blockIdx.x);
        keep(next, 0);
        asm volatile("bar.sync 1, %0;" ::"n"(kEpilogueWarps * 32) : "memory");
        tc::pdl_wait();
        const int64_t width = (g.F + kBlockCodes - 1) / kBlockCodes * kBlockCodes;
        uint32_t ti = 0;
        for (uint32_t t = blockIdx.x; t < total; t += gridDim.x, ++ti) {
            const Tile tile = next.tile;
            const ColParams col = next.col;
            const int64_t f = output_at(t);
            const TokenParams& rows = token[ti & 1];
            int* sum = sums + (ti & 1) * kMaxRows;
            next = fetch(t + gridDim.x);
            const pair_t ws = make_pair(col.ws, col.ws), wo = make_pair(col.wo, col.wo), p3 = make_pair(col.p3, col.p3), bias = make_pair(col.bias, col.bias);
            float lo = 0.f, hi = 0.f, off = 0.f, off2 = 0.f;
            if constexpr (kCodes) {
                lo = g.t_lo[g.n_thr == 1 ? 0 : tile.e]; hi = g.t_hi[g.n_thr == 1 ? 0 : tile.e];
                // what the terms of the affine form other than the product add up to at most, twice (they may cancel)
                float asx = 0.f, ao = 0.f;
                for (int r = lane; r < tile.rows; r += 32) { asx = fmaxf(asx, fabsf(rows.asx[r])); ao = fmaxf(ao, fabsf(rows.ao[r])); }
                #pragma unroll
                for (int d = 16; d > 0; d >>= 1) { asx = fmaxf(asx, __shfl_xor_sync(0xffffffffu, asx, d)); ao = fmaxf(ao, __shfl_xor_sync(0xffffffffu, ao, d)); }
                off = 2.f * (asx * fabsf(col.wo) + ao * fabsf(col.p3) + fabsf(col.bias));
                if constexpr (kGated) {
                    off2 = __shfl_xor_sync(0xffffffffu, off, 16);
                    if (lane >= 16) { const float x = off; off = off2; off2 = x; }
                }
                off *= 6.8f * 1.25f * kUnit;
                off2 *= 6.f * 1.25f * kUnit;
            }
            alive = warp_wait(&bar.acc_full[ti & 1], ti >> 1);
            tc::tc_fence_after_sync();
            const uint32_t acc = tmem + (ti & 1) * acc_cols + ((uint32_t)(quad * 32) << 16);
            for (int c0 = half * 32; alive && c0 < tile.rows; c0 += 64) {
                constexpr int kOwn = kGated ? 8 : 16;                             // outputs of a lane in 16 tokens
                uint32_t my_nz = 0, my_up = 0;                                    // lane x: the warp's bits of output x
                T* out = static_cast<T*>(g.out) + (int64_t)(tile.row + c0 + (kGated ? lane >> 4 : 0)) * g.out_stride + f;
                #pragma unroll 1
                for (int part = 0; part < 2; ++part) {
                    const int c = c0 + part * 16;
                    if (c >= tile.rows) break;
                    uint32_t v[16];
                    tc::tmem_ld16(acc + (uint32_t)c, v);
                    tc::tmem_ld_wait();
                    bool near = false;
                    #pragma unroll
                    for (int x0 = 0; x0 < kOwn; x0 += 4) {
                        float y1[4], y2[4];
                        auto two = [&](int i, float& a, float& b) {               // tokens c + i and c + i + 1 (i even)
                            const float2 as = *reinterpret_cast<const float2*>(&rows.as[c + i]), sx = *reinterpret_cast<const float2*>(&rows.asx[c + i]);
                            const float2 ao = *reinterpret_cast<const float2*>(&rows.ao[c + i]);
                            const pair_t S = mul_pair(make_pair(as.x, as.y), make_pair(__uint_as_float(v[i]), __uint_as_float(v[i + 1])));
                            take_pair(fma_pair(ws, S, fma_pair(wo, make_pair(sx.x, sx.y), fma_pair(p3, make_pair(ao.x, ao.y), bias))), a, b);
                        };
                        if constexpr (kGated) {
                            #pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                float a, b;
                                two(2 * (x0 + x), a, b);
                                // lanes 0-15 take the first token of the two, 16-31 the second
                                const float own = lane < 16 ? a : b, other = __shfl_xor_sync(0xffffffffu, lane < 16 ? b : a, 16);
                                y1[x] = lane < 16 ? own : other;
                                y2[x] = lane < 16 ? other : own;
                            }
                        } else {
                            two(x0, y1[0], y1[1]);
                            two(x0 + 2, y1[2], y1[3]);
                        }
                        float o[4] = {y1[0], y1[1], y1[2], y1[3]};
                        if (g.act == RTN_ACT_SILU) {
                            #pragma unroll
                            for (int x = 0; x < 4; ++x) o[x] = fast_silu(o[x]);
                        } else if (g.act != RTN_ACT_NONE) {
                            const float4 a = activation4(make_float4(o[0], o[1], o[2], o[3]), g.act);
                            o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w;
                        }
                        #pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            if constexpr (kGated) o[x] *= y2[x];
                            if constexpr (kCodes) {
                                // (the bound of output_of, with |y| and the other terms for what the terms add up to)
                                constexpr float u = 1.25f * kUnit;
                                float err = fmaf(25.f * u, fabsf(y1[x]), off);
                                if constexpr (kGated) err = fmaf(fabsf(y2[x]), fmaf(32.f * u, fabsf(y1[x]), off), off2 * fabsf(y1[x]));
                                const bool up = o[x] > hi, nz = up || o[x] < lo;
                                near = near || !(fminf(fabsf(o[x] - lo), fabsf(o[x] - hi)) > err);
                                const uint32_t a = __ballot_sync(0xffffffffu, nz), b = __ballot_sync(0xffffffffu, up);
                                if (lane == part * kOwn + x0 + x) { my_nz = a; my_up = b; }
                            }
                            if (!kCodes || g.out != nullptr) {
                                const int r = kGated ? c + 2 * (x0 + x) + (lane >> 4) : c + x0 + x;
                                if (r < tile.rows && f < g.F) *out = from_f32<T>(o[x]);
                                out += kGated ? 2 * g.out_stride : g.out_stride;
                            }
                        }
                    }
                    if constexpr (kCodes) {
                        if (__any_sync(0xffffffffu, near && f < g.F)) {           // all of them again, in double
                            #pragma unroll 1
                            for (int x = 0; x < kOwn; ++x) {
                                float S, S2 = 0.f;
                                uint32_t q[4];
                                tc::tmem_ld4(acc + (uint32_t)(c + (kGated ? (x & ~1) * 2 : x & ~3)), q);
                                tc::tmem_ld_wait();
                                int r;
                                if constexpr (kGated) {
                                    const float a = __uint_as_float(x & 1 ? q[2] : q[0]), b = __uint_as_float(x & 1 ? q[3] : q[1]);
                                    const float own = lane < 16 ? a : b, other = __shfl_xor_sync(0xffffffffu, lane < 16 ? b : a, 16);
                                    S = lane < 16 ? own : other;
                                    S2 = lane < 16 ? other : own;
                                    r = c + 2 * x + (lane >> 4);
                                } else {
                                    S = __uint_as_float(x & 2 ? (x & 1 ? q[3] : q[2]) : (x & 1 ? q[1] : q[0]));
                                    r = c + x;
                                }
                                bool up = false, down = false;
                                const int m = r < tile.rows ? rows.token[r] : -1;
                                if (m >= 0 && f < g.F) {
                                    const double e = exact_value(g, m, tile.e, f, S, S2);
                                    up = e > (double)hi;
                                    down = !up && e < (double)lo;
                                }
                                __syncwarp();
                                const uint32_t a = __ballot_sync(0xffffffffu, up || down), b = __ballot_sync(0xffffffffu, up);
                                if (lane == part * kOwn + x) { my_nz = a; my_up = b; }
                            }
                        }
                    }
                }
                if constexpr (kCodes) {
                    const int64_t f0 = (int64_t)(t % cols) * kTileOuts + quad * (kGated ? 16 : 32);
                    const uint32_t real = g.F - f0 >= (kGated ? 16 : 32) ? 0xffffffffu : g.F <= f0 ? 0u : (1u << (uint32_t)(g.F - f0)) - 1u;     // (padding: zeros)
                    if (lane < 2 * kOwn && f0 < width) {
                        uint8_t* at = g.out_packed + (int64_t)(tile.row + c0) * (width / 4) + f0 / kBlockCodes * kBlockBytes + f0 % kBlockCodes / 8;
                        #pragma unroll
                        for (int x = 0; x < (kGated ? 2 : 1); ++x) {
                            const int r = kGated ? 2 * lane + x : lane;
                            if (c0 + r >= tile.rows) continue;
                            uint8_t* w = at + (int64_t)r * (width / 4);
                            uint32_t nz = my_nz, up = my_up;
                            if constexpr (kGated) {
                                nz = nz >> (16 * x) & 0xffffu & real; up = up >> (16 * x) & 0xffffu & real;
                                *reinterpret_cast<uint16_t*>(w) = (uint16_t)nz;
                                *reinterpret_cast<uint16_t*>(w + 16) = (uint16_t)up;
                            } else {
                                nz &= real; up &= real;
                                *reinterpret_cast<uint32_t*>(w) = nz;
                                *reinterpret_cast<uint32_t*>(w + 16) = up;
                            }
                            atomicAdd(&sum[c0 + r], 2 * __popc(up) - __popc(nz));
                        }
                    }
                }
            }
            tc::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bar.acc_empty[ti & 1]);
            keep(next, (ti + 1) & 1);
            asm volatile("bar.sync 1, %0;" ::"n"(kEpilogueWarps * 32) : "memory");
            if (*dead) break;                                                     // (all of them, whichever gave up)
            if constexpr (kCodes) {
                if (mine < tile.rows) {
                    if (sum[mine] != 0) atomicAdd(&g.out_sum[tile.row + mine], sum[mine]);          // (whole numbers: any order gives the same)
                    sum[mine] = 0;
                }
            }
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
    for (int h = 16; h <= kMaxRows; h += 16) {
        const double per = (double)(int64_t)((each + h - 1) / h), tiles = used * per * p.col_tiles, height = each / per < 16 ? 16 : each / per;
        const double stage = 2.6 * height > 350.0 ? 2.6 * height : 350.0, loop = stage * p.k_stages, out = 20.0 * height + 500.0;
        const double rounds = tiles / sms < 1.0 ? 1.0 : (double)(int64_t)((tiles + sms - 1) / sms);
        const double cost = rounds * (loop > out ? loop : out) + (loop > out ? out : loop);
        if (p.max_rows == 0 || cost < best) { best = cost; p.max_rows = h; }
    }
    p.stage_bytes = (uint32_t)p.max_rows * 128u;
    p.ring = (uint32_t)((256 + 2 * sizeof(TokenParams) + 2 * kMaxRows * 4 + (4 * g.E + 1) * 4 + 1023) / 1024 * 1024);
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
