// The experts' ternary products on the tensor cores: codes as 4-bit floating point.
#include "rtn_experts.cuh"
#include "rtn_tcgen05.cuh"
#include "rtn_tensormap.cuh"

namespace rtn {

namespace {

#ifndef RTN_X_TMEM_A
#define RTN_X_TMEM_A 1
#endif
constexpr bool kTmemA = RTN_X_TMEM_A;

constexpr int kExpandWarps = 8, kEpilogueWarps = 8;             // two of each for every quarter of the lanes
constexpr int kLoadWarp = kExpandWarps + kEpilogueWarps, kMmaWarp = kLoadWarp + 1;
constexpr int kThreads = (kMmaWarp + 1) * 32;
constexpr int kStageCodes = 256;                                // codes of K in a stage: a 128-byte row of 4-bit values
constexpr int kMaxRows = 192;                                   // of a tile
constexpr int kMaxStages = kTmemA ? 3 : 6;
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
    uint64_t a_full[kMaxStages], b_full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2];
    uint32_t tmem_slot;
    int dead;
    int total;
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
// D[tmem] (+)= A * B^T, one K = 64 slice, A in tensor memory or shared memory.
__device__ __forceinline__ void mma_mxf4(uint32_t elected, uint32_t d, uint32_t a_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t scales, bool accumulate)
{
    if constexpr (kTmemA)
        asm volatile(
            "{\n\t.reg .pred p, e;\n\t"
            "setp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 e, %6, 0;\n\t"
            "@e tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], [%1], %2, %3, [%4], [%4], p;\n\t}"
            ::"r"(d), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(scales), "r"((uint32_t)accumulate), "r"(elected) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p, e;\n\t"
            "setp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 e, %6, 0;\n\t"
            "@e tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%4], p;\n\t}"
            ::"r"(d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(scales), "r"((uint32_t)accumulate), "r"(elected) : "memory");
}

// Four rows of a [rows][pitch bytes] tensor, 128 bytes of each from byte x on, to 512 bytes of shared memory under the 128-byte swizzle;
// a row out of range is read as zeros.
__device__ __forceinline__ void gather4(uint32_t dst, const CUtensorMap* map, int x, const int (&r)[4], uint64_t* bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(tc::smem_addr(bar)) : "memory");
}

// Input rows as 4-bit values, `pitch` bytes each (the end of a row is zeros); and the sums of the codes begin at 0.
__global__ void __launch_bounds__(256)
expand_inputs_kernel(const uint32_t* __restrict__ planes, int64_t rows, int nblk, int pitch, uint4* __restrict__ out, const int32_t* __restrict__ start,
                     int E, int32_t* sums, int64_t R)
{
    const int chunks = pitch / 16;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (sums != nullptr && i < R && i >= start[0] && i < start[E]) sums[i] = 0;
    if (i >= rows * chunks) return;
    const int64_t row = i / chunks;
    const int c = (int)(i % chunks);
    uint32_t nz = 0, pos = 0;
    if (c / 4 < nblk) {
        const uint32_t* p = planes + (row * nblk + c / 4) * 8 + c % 4;
        nz = p[0]; pos = p[4];
    }
    out[i] = expand_input(nz, pos);
}

template <typename T, bool kGated, bool kCodes>
__global__ void __launch_bounds__(kThreads, 1)
experts_tiles_kernel(const __grid_constant__ ExpertsArgs g, const __grid_constant__ CUtensorMap map, const __grid_constant__ TilesPlan p)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    Bars& bar = *reinterpret_cast<Bars*>(smem);
    float4* token = reinterpret_cast<float4*>(smem + 256);                       // [2][kMaxRows] {a_s, a_o, S_x, token}
    int* sums = reinterpret_cast<int*>(smem + 256 + 2 * kMaxRows * 16);          // [2][kMaxRows]
    int* before = sums + 2 * kMaxRows;                                           // [E + 1] tiles before an expert's
    int* first = before + g.E + 1;                                               // [E] its first row
    int* count = first + g.E;                                                    // [E] its rows
    static_assert(sizeof(Bars) <= 256, "barriers");
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    volatile int* dead = &bar.dead;
    const uint32_t ring = tc::smem_addr(smem) + p.ring;

    if (warp == kMmaWarp) tc::tmem_alloc(&bar.tmem_slot, 512);
    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) { tc::mbar_init(&bar.a_full[i], 4); tc::mbar_init(&bar.b_full[i], 1); tc::mbar_init(&bar.empty[i], 1); }
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
            if (e < g.E) { before[e] = sum + x - tiles; first[e] = s; count[e] = n; }
            sum += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0) { before[g.E] = sum; bar.total = sum; }
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

    const int64_t total = (int64_t)bar.total * p.col_tiles;
    auto find = [&](int64_t t) {                                                  // whole warp
        const int rt = (int)(t / p.col_tiles);
        Tile r{0, 0, 0, 16};
        for (int e0 = 0; e0 < g.E; e0 += 32) {
            const int e = e0 + lane;
            const uint32_t who = __ballot_sync(0xffffffffu, e < g.E && before[e] <= rt && rt < before[e + 1]);
            if (who != 0) {
                r.e = e0 + __ffs(who) - 1;
                const int tiles = before[r.e + 1] - before[r.e], n = count[r.e];
                r.height = ((n + tiles - 1) / tiles + 15) / 16 * 16;
                const int at = (rt - before[r.e]) * r.height;
                r.row = first[r.e] + at;
                r.rows = n - at < r.height ? n - at : r.height;                   // (0 or less: the rounding left nothing for the last)
                if (r.rows < 0) r.rows = 0;
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
    auto output_at = [&](int64_t t) { return (t % p.col_tiles) * kTileOuts + (kGated ? quad * 16 + (lane & 15) : quad * 32 + lane); };
    bool alive = true;

    if (warp < kExpandWarps) {
        // ------------------------------------------------------------ weights: a team of four warps has every other stage
        const uint4* __restrict__ W = reinterpret_cast<const uint4*>(g.w_packed);
        uint4 next[4];
        int64_t t = blockIdx.x;                                                   // the stage that `next` is of
        int k = warp >> 2;
        const uint4* src = nullptr;
        auto enter = [&]() {                                                      // (t, k) is a tile's stage
            bool moved = src == nullptr;
            while (k >= p.k_stages && t < total) { k -= p.k_stages; t += gridDim.x; moved = true; }
            if (moved && t < total) {
                const int64_t f = output_at(t), e = find(t).e;
                src = f < g.F ? W + (e * g.N + (kGated && lane >= 16 ? g.F + f : f)) * nblk * 2 : W;
            }
        };
        auto fetch = [&]() {
            const bool ok = t < total && output_at(t) < g.F;
            #pragma unroll
            for (int i = 0; i < 2; ++i) {
                next[2 * i] = next[2 * i + 1] = make_uint4(0, 0, 0, 0);
                if (ok && 2 * k + i < nblk) { next[2 * i] = __ldg(src + (2 * k + i) * 2); next[2 * i + 1] = __ldg(src + (2 * k + i) * 2 + 1); }
            }
        };
        enter();
        fetch();
        int s = warp >> 2;
        uint32_t phase = 0;
        while (t < total) {
            uint4 w[4];
            #pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = next[i];
            k += 2;
            enter();
            if (!warp_wait(&bar.empty[s], phase + 1)) break;
            fetch();
            if constexpr (kTmemA) {
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
            } else {
                const int row = quad * 32 + lane;
                uint4* dst = reinterpret_cast<uint4*>(smem + p.ring + (uint32_t)s * p.stage_bytes + (uint32_t)p.max_rows * 128u + row * 128);
                #pragma unroll
                for (int i = 0; i < 2; ++i) {
                    dst[(4 * i + 0) ^ (row & 7)] = expand_weight(w[2 * i].x, w[2 * i + 1].x);
                    dst[(4 * i + 1) ^ (row & 7)] = expand_weight(w[2 * i].y, w[2 * i + 1].y);
                    dst[(4 * i + 2) ^ (row & 7)] = expand_weight(w[2 * i].z, w[2 * i + 1].z);
                    dst[(4 * i + 3) ^ (row & 7)] = expand_weight(w[2 * i].w, w[2 * i + 1].w);
                }
                tc::fence_smem_to_async_proxy();
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bar.a_full[s]);
            s += 2;
            if (s >= p.stages) { s -= p.stages; phase ^= 1; }
        }
    } else if (warp == kLoadWarp) {
        // ------------------------------------------------------------ input rows, gathered four at a time
        int row[8], next_row[8];
        auto fetch = [&](int64_t t) {
            if (t >= total) return;
            const Tile tile = find(t);
            #pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = (i >> 2) * 128 + lane * 4 + (i & 3);
                int64_t m = g.T;                                                  // (out of range: zeros)
                if (r < tile.rows) m = g.tokens != nullptr ? g.tokens[tile.row + r] : tile.row + r;
                next_row[i] = m >= 0 && m < g.T ? (int)m : (int)g.T;
            }
        };
        fetch(blockIdx.x);
        int s = 0;
        uint32_t phase = 0;
        for (int64_t t = blockIdx.x; t < total && alive; t += gridDim.x) {
            const int height = find(t).height;
            #pragma unroll
            for (int i = 0; i < 8; ++i) row[i] = next_row[i];
            fetch(t + gridDim.x);
            const int a[4] = {row[0], row[1], row[2], row[3]}, b[4] = {row[4], row[5], row[6], row[7]};
            for (int k = 0; k < p.k_stages; ++k) {
                if (!(alive = warp_wait(&bar.empty[s], phase + 1))) break;
                if (lane == 0) tc::mbar_arrive_expect_tx(&bar.b_full[s], (uint32_t)height * 128u);
                __syncwarp();
                const uint32_t dst = ring + (uint32_t)s * p.stage_bytes + (uint32_t)lane * 512u;
                if (lane * 4 < height) gather4(dst, &map, k * 128, a, &bar.b_full[s]);
                if (128 + lane * 4 < height) gather4(dst + 128u * 128u, &map, k * 128, b, &bar.b_full[s]);
                if (++s == p.stages) { s = 0; phase ^= 1; }
            }
        }
        // nobody leaves while copies are on their way: the last of each stage
        for (int i = 0; i < p.stages; ++i) {
            const uint32_t uses = i < s ? phase + 1 : phase;                      // parity of the number of copies to this stage
            tc::mbar_wait_tries(&bar.b_full[i], (uses + 1) & 1u, kTries);
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------ products
        const uint32_t elected = tc::elect_one();
        const uint64_t desc_b = tc::smem_desc_sw128(ring, 0), desc_a = tc::smem_desc_sw128(ring + (uint32_t)p.max_rows * 128u, 0);
        int s = 0, ti = 0;
        uint32_t phase = 0;
        for (int64_t t = blockIdx.x; t < total && alive; t += gridDim.x, ++ti) {
            const uint32_t idesc = idesc_mxf4(128, (uint32_t)find(t).height), d = tmem + (uint32_t)(ti & 1) * acc_cols;
            if (!(alive = warp_wait(&bar.acc_empty[ti & 1], (uint32_t)(ti >> 1) + 1))) break;
            for (int k = 0; k < p.k_stages; ++k) {
                if (!(alive = warp_wait(&bar.a_full[s], phase) && warp_wait(&bar.b_full[s], phase))) break;
                tc::tc_fence_after_sync();
                const uint64_t step = (uint64_t)((uint32_t)s * (p.stage_bytes >> 4));
                #pragma unroll
                for (int j = 0; j < 4; ++j)                                       // K = 64: 32 bytes, eight columns
                    mma_mxf4(elected, d, a_tmem + (uint32_t)(s * 32 + j * 8), desc_a + step + (uint64_t)(j * 2), desc_b + step + (uint64_t)(j * 2), idesc, scales, k > 0 || j > 0);
                if (elected) tc::mma_commit(&bar.empty[s]);
                __syncwarp();
                if (++s == p.stages) { s = 0; phase ^= 1; }
            }
            if (elected && alive) tc::mma_commit(&bar.acc_full[ti & 1]);
            __syncwarp();
        }
    } else {
        // ------------------------------------------------------------ write out: a warp has 32 lanes (weight rows) of every other 16 tokens
        const int mine = threadIdx.x - kExpandWarps * 32, half = (warp - kExpandWarps) >> 2;
        struct Own { Tile tile; float4 row; ColParams col; };
        auto fetch = [&](int64_t t) {
            Own o{};
            if (t >= total) return o;
            o.tile = find(t);
            if (mine < o.tile.rows) {
                const RowParams r = row_params(g, o.tile.row + mine);
                o.row = make_float4(r.as, r.ao, r.sx, __int_as_float(r.token));
                if (r.token < 0 && t % p.col_tiles == 0) atomicOr(g.status, kStatusBadIndex);
            }
            const int64_t f = output_at(t);
            if (f < g.F) o.col = col_params(g, o.tile.e, kGated && lane >= 16 ? g.F + f : f);
            return o;
        };
        Own next = fetch(blockIdx.x);
        if (mine < kMaxRows) token[mine] = next.row;
        asm volatile("bar.sync 1, %0;" ::"n"(kEpilogueWarps * 32) : "memory");
        int ti = 0;
        for (int64_t t = blockIdx.x; t < total; t += gridDim.x, ++ti) {
            const Tile tile = next.tile;
            const ColParams col = next.col;
            const int64_t f = output_at(t);
            const float4* rows = token + (ti & 1) * kMaxRows;
            int* sum = sums + (ti & 1) * kMaxRows;
            next = fetch(t + gridDim.x);
            float lo = 0.f, hi = 0.f, off = 0.f, off2 = 0.f;
            if constexpr (kCodes) {
                lo = g.t_lo[g.n_thr == 1 ? 0 : tile.e]; hi = g.t_hi[g.n_thr == 1 ? 0 : tile.e];
                // what the terms of the affine form other than the product add up to at most, twice (they may cancel)
                float as = 0.f, ao = 0.f, sx = 0.f;
                for (int r = lane; r < tile.rows; r += 32) { as = fmaxf(as, fabsf(rows[r].x)); ao = fmaxf(ao, fabsf(rows[r].y)); sx = fmaxf(sx, fabsf(rows[r].z)); }
                #pragma unroll
                for (int d = 16; d > 0; d >>= 1) {
                    as = fmaxf(as, __shfl_xor_sync(0xffffffffu, as, d)); ao = fmaxf(ao, __shfl_xor_sync(0xffffffffu, ao, d));
                    sx = fmaxf(sx, __shfl_xor_sync(0xffffffffu, sx, d));
                }
                off = 2.f * (as * sx * fabsf(col.wo) + ao * fabsf(col.p3) + fabsf(col.bias));
                if constexpr (kGated) {
                    off2 = __shfl_xor_sync(0xffffffffu, off, 16);
                    if (lane >= 16) { const float x = off; off = off2; off2 = x; }
                }
            }
            alive = warp_wait(&bar.acc_full[ti & 1], (uint32_t)(ti >> 1));
            tc::tc_fence_after_sync();
            const uint32_t acc = tmem + (uint32_t)(ti & 1) * acc_cols + ((uint32_t)(quad * 32) << 16);
            for (int c = half * 16; alive && c < tile.rows; c += 32) {
                uint32_t v[16];
                tc::tmem_ld16(acc + (uint32_t)c, v);
                tc::tmem_ld_wait();
                constexpr int kOwn = kGated ? 8 : 16;                             // outputs of a lane
                uint32_t up = 0, down = 0, near = 0;
                #pragma unroll
                for (int x0 = 0; x0 < kOwn; x0 += 4) {
                    float y1[4], y2[4];
                    #pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        if constexpr (kGated) {
                            const float4 ra = rows[c + 2 * (x0 + x)], rb = rows[c + 2 * (x0 + x) + 1];
                            const float ya = affine(RowParams{ra.x, ra.y, ra.z, 0}, col, __uint_as_float(v[2 * (x0 + x)]));
                            const float yb = affine(RowParams{rb.x, rb.y, rb.z, 0}, col, __uint_as_float(v[2 * (x0 + x) + 1]));
                            // lanes 0-15 take the first token of the two, 16-31 the second
                            const float other = __shfl_xor_sync(0xffffffffu, lane < 16 ? yb : ya, 16);
                            y1[x] = lane < 16 ? ya : other;
                            y2[x] = lane < 16 ? other : yb;
                        } else {
                            const float4 ra = rows[c + x0 + x];
                            y1[x] = affine(RowParams{ra.x, ra.y, ra.z, 0}, col, __uint_as_float(v[x0 + x]));
                        }
                    }
                    float o[4] = {y1[0], y1[1], y1[2], y1[3]};
                    if (g.act != RTN_ACT_NONE) {
                        const float4 a = activation4(make_float4(o[0], o[1], o[2], o[3]), g.act);
                        o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w;
                    }
                    #pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        if constexpr (kGated) o[x] *= y2[x];
                        const int r = kGated ? c + 2 * (x0 + x) + (lane >> 4) : c + x0 + x;
                        if (g.out != nullptr && r < tile.rows && f < g.F) static_cast<T*>(g.out)[(int64_t)(tile.row + r) * g.out_stride + f] = from_f32<T>(o[x]);
                        if constexpr (kCodes) {
                            // (the bound of output_of, with |y| and the other terms for what the terms add up to)
                            float err = fmaf(25.f, fabsf(y1[x]), 6.8f * off);
                            if constexpr (kGated) err = fmaf(fabsf(y2[x]), fmaf(32.f, fabsf(y1[x]), 6.8f * off), 6.f * off2 * fabsf(y1[x]));
                            const bool a = o[x] > hi, b = !a && o[x] < lo;
                            const float d = fminf(fabsf(o[x] - lo), fabsf(o[x] - hi));
                            up |= (uint32_t)a << (x0 + x);
                            down |= (uint32_t)b << (x0 + x);
                            near |= (uint32_t)(!(d > 1.25f * kUnit * err) || !(fabsf(o[x]) < 1e37f)) << (x0 + x);
                        }
                    }
                }
                if constexpr (kCodes) {
                    if (f >= g.F) up = down = near = 0;
                    for (uint32_t todo = __reduce_or_sync(0xffffffffu, near); todo != 0; todo &= todo - 1) {
                        const int x = __ffs(todo) - 1;
                        float S, S2 = 0.f;
                        int r;
                        if constexpr (kGated) {
                            uint32_t two[4];
                            tc::tmem_ld4(acc + (uint32_t)(c + (x & ~1) * 2), two);
                            tc::tmem_ld_wait();
                            const float sa = __uint_as_float(x & 1 ? two[2] : two[0]), sb = __uint_as_float(x & 1 ? two[3] : two[1]);
                            const float other = __shfl_xor_sync(0xffffffffu, lane < 16 ? sb : sa, 16);
                            S = lane < 16 ? sa : other;
                            S2 = lane < 16 ? other : sb;
                            r = c + 2 * x + (lane >> 4);
                        } else {
                            uint32_t four[4];
                            tc::tmem_ld4(acc + (uint32_t)(c + (x & ~3)), four);
                            tc::tmem_ld_wait();
                            S = __uint_as_float(x & 2 ? (x & 1 ? four[3] : four[2]) : (x & 1 ? four[1] : four[0]));
                            r = c + x;
                        }
                        if (near >> x & 1) {
                            bool a = false, b = false;
                            const int m = r < tile.rows ? __float_as_int(rows[r].w) : -1;
                            if (m >= 0) {
                                const double e = exact_value(g, m, tile.e, f, S, S2);
                                a = e > (double)hi;
                                b = !a && e < (double)lo;
                            }
                            up = (up & ~(1u << x)) | (uint32_t)a << x;
                            down = (down & ~(1u << x)) | (uint32_t)b << x;
                        }
                        __syncwarp();
                    }
                    const uint32_t nz = up | down;
                    uint32_t my_nz = 0, my_up = 0;
                    #pragma unroll
                    for (int x = 0; x < kOwn; ++x) {                              // lane x keeps the warp's bits of output x
                        const uint32_t a = __ballot_sync(0xffffffffu, nz >> x & 1), b = __ballot_sync(0xffffffffu, up >> x & 1);
                        if (lane == x) { my_nz = a; my_up = b; }
                    }
                    const int64_t f0 = (t % p.col_tiles) * kTileOuts + quad * (kGated ? 16 : 32);
                    const int64_t width = (g.F + kBlockCodes - 1) / kBlockCodes * kBlockCodes;
                    if (lane < kOwn && f0 < width) {
                        uint8_t* at = g.out_packed + (int64_t)tile.row * (width / 4) + f0 / kBlockCodes * kBlockBytes + f0 % kBlockCodes / 8;
                        #pragma unroll
                        for (int x = 0; x < (kGated ? 2 : 1); ++x) {
                            const int r = kGated ? c + 2 * lane + x : c + lane;
                            if (r >= tile.rows) continue;
                            uint8_t* w = at + (int64_t)r * (width / 4);
                            if constexpr (kGated) {
                                const uint32_t n16 = my_nz >> (16 * x) & 0xffffu, u16 = my_up >> (16 * x) & 0xffffu;
                                *reinterpret_cast<uint16_t*>(w) = (uint16_t)n16;
                                *reinterpret_cast<uint16_t*>(w + 16) = (uint16_t)u16;
                                atomicAdd(&sum[r], 2 * __popc(u16) - __popc(n16));
                            } else {
                                *reinterpret_cast<uint32_t*>(w) = my_nz;
                                *reinterpret_cast<uint32_t*>(w + 16) = my_up;
                                atomicAdd(&sum[r], 2 * __popc(my_up) - __popc(my_nz));
                            }
                        }
                    }
                }
            }
            tc::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bar.acc_empty[ti & 1]);
            if (mine < kMaxRows) token[((ti + 1) & 1) * kMaxRows + mine] = next.row;
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
    p.stage_bytes = (uint32_t)(p.max_rows + (kTmemA ? 0 : 128)) * 128u;
    p.ring = (uint32_t)((256 + 2 * kMaxRows * 20 + (3 * g.E + 1) * 4 + 1023) / 1024 * 1024);
    const int by_smem = (int)((227u * 1024u - p.ring) / p.stage_bytes), by_tmem = kTmemA ? (512 - 2 * p.max_rows - (int)kScaleCols) / 32 : kMaxStages;
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
    const int64_t rows = g.tokens != nullptr ? g.T : g.R;
    void* scratch = nullptr;
    cudaError_t e = scratch_alloc(&scratch, (size_t)rows * pitch, s);
    if (e != cudaSuccess) return e;
    CUtensorMap map;
    const cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {128, 1}, unit[2] = {1, 1};
    if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, scratch, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) e = cudaErrorInvalidValue;
    if (e == cudaSuccess) {
        const int64_t chunks = rows * (pitch / 16), threads = chunks > g.R ? chunks : g.R;
        expand_inputs_kernel<<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(reinterpret_cast<const uint32_t*>(g.a_packed), rows, nblk, pitch,
                                                                              static_cast<uint4*>(scratch), g.start, g.E, g.out_sum, g.R);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) {
        e = with_dtype(g.dtype, [&](auto t) {
            using T = decltype(t);
            auto run = [&](auto kernel) {
                cudaError_t x = allow_shared_memory(kernel);
                if (x != cudaSuccess) return x;
                kernel<<<(unsigned)device_sm_count(), kThreads, p.smem, s>>>(g, map, p);
                return cudaGetLastError();
            };
            if (g.out_packed != nullptr) return g.gated ? run(experts_tiles_kernel<T, true, true>) : run(experts_tiles_kernel<T, false, true>);
            return g.gated ? run(experts_tiles_kernel<T, true, false>) : run(experts_tiles_kernel<T, false, false>);
        });
    }
    const cudaError_t e2 = cudaFreeAsync(scratch, s);
    return e == cudaSuccess ? e2 : e;
}

}  // namespace rtn
