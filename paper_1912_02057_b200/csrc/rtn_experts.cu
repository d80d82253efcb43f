// The experts' ternary products for few rows (decoding): bit planes, AND / XOR / popcount (Eq. 9), act, gate and codes in the epilogue.
//
// experts_rows_kernel: a CTA has a tile of MT rows of one expert and a block of output columns.  A group of GL lanes owns CPG outputs at a time, that
// is CPG weight rows or, gated, CPG pairs of them; lane i takes the 128-code blocks i, i + GL, ... of each (32 adjacent bytes), and one
// shuffle tree joins the group.
// Bound: latency for a token (a launch, one trip to DRAM for the planes, the epilogue), then DRAM, the packed weights of the experts that have rows,
// read once; from about two rows of an expert on the POPC rate.
// Measured (one B200): a token's 4 of 64 experts of 2048 x 2048, gated, codes 5.8 us in a graph (4.2 MB of planes: 0.7 us at the copy rate).
#include "rtn_experts.cuh"
#include "rtn_tcgen05.cuh"

#include <math.h>

namespace rtn {

namespace {

constexpr int kThreads = 256;
constexpr int kOutputs = 4;             // of a group at a time: columns of a CTA = 256 / GL * 4, a multiple of 32

template <int MT, bool kGated, bool kCodes>
__global__ void __launch_bounds__(kThreads)
experts_rows_kernel(const __grid_constant__ ExpertsArgs g, int GL, int col_blocks)
{
    constexpr int NR = kGated ? 2 * kOutputs : kOutputs;       // weight rows of a group
    __shared__ uint32_t bits[kCodes ? MT : 1][2][kCodes ? kThreads * kOutputs / 32 : 1];
    const int gl = threadIdx.x & (GL - 1), per_cta = kThreads / GL * kOutputs;
    const int col = (int)(blockIdx.x % (unsigned)col_blocks);
    const int64_t f0 = (int64_t)col * per_cta, n0 = f0 + threadIdx.x / GL * kOutputs;
    const RowTile tile = find_tile(g.start, g.E, g.R, MT, (int)(blockIdx.x / (unsigned)col_blocks), g.status);
    if (tile.e < 0) {
        if constexpr (kCodes) tc::pdl_wait();                  // (nobody ends before the kernel that this one overlaps)
        return;
    }
    const int64_t nblk = (g.K + kBlockCodes - 1) / kBlockCodes;
    if constexpr (kCodes) {
        for (int i = threadIdx.x; i < MT * 2 * per_cta / 32; i += kThreads)
            bits[i / (2 * (per_cta / 32))][i / (per_cta / 32) % 2][i % (per_cta / 32)] = 0;
        __syncthreads();
    }
    const uint4* __restrict__ W = reinterpret_cast<const uint4*>(g.w_packed) + (int64_t)tile.e * g.N * nblk * 2;
    const uint4* A[MT];
    #pragma unroll
    for (int i = 0; i < MT; ++i) {
        A[i] = nullptr;
        if (i < tile.rows) {
            const int64_t m = g.tokens != nullptr ? g.tokens[tile.row + i] : tile.row + i;
            if (m >= 0 && m < g.T) A[i] = reinterpret_cast<const uint4*>(g.a_packed) + m * nblk * 2;
            else if (col == 0 && threadIdx.x == 0) atomicOr(g.status, kStatusBadIndex);
        }
    }
    int cnt[MT][NR];
    #pragma unroll
    for (int i = 0; i < MT; ++i)
        #pragma unroll
        for (int j = 0; j < NR; ++j) cnt[i][j] = 0;
    for (int64_t kb = gl; kb < nblk; kb += GL) {
        uint4 w1[NR], w2[NR];
        #pragma unroll
        for (int j = 0; j < NR; ++j) {
            const int64_t n = n0 + j % kOutputs;
            const bool ok = n < g.F;
            const uint4* src = W + ((ok ? n + (j >= kOutputs ? g.F : 0) : 0) * nblk + kb) * 2;
            w1[j] = ok ? __ldg(src) : make_uint4(0, 0, 0, 0);
            w2[j] = ok ? __ldg(src + 1) : make_uint4(0, 0, 0, 0);
        }
        #pragma unroll
        for (int i = 0; i < MT; ++i) {
            if (A[i] == nullptr) continue;
            const uint4 a1 = __ldg(A[i] + kb * 2), a2 = __ldg(A[i] + kb * 2 + 1);
            #pragma unroll
            for (int j = 0; j < NR; ++j) {
                const uint32_t c0 = a1.x & w1[j].x, c1 = a1.y & w1[j].y, c2 = a1.z & w1[j].z, c3 = a1.w & w1[j].w;
                cnt[i][j] += (__popc(c0) + __popc(c1)) + (__popc(c2) + __popc(c3))
                           - 2 * ((__popc((a2.x ^ w2[j].x) & c0) + __popc((a2.y ^ w2[j].y) & c1)) +
                                  (__popc((a2.z ^ w2[j].z) & c2) + __popc((a2.w ^ w2[j].w) & c3)));
            }
        }
    }
    for (int d = GL / 2; d > 0; d >>= 1) {
        #pragma unroll
        for (int i = 0; i < MT; ++i)
            #pragma unroll
            for (int j = 0; j < NR; ++j) cnt[i][j] += __shfl_xor_sync(0xffffffffu, cnt[i][j], d);
    }
    float lo = 0.f, hi = 0.f;
    if constexpr (kCodes) { lo = g.t_lo[g.n_thr == 1 ? 0 : tile.e]; hi = g.t_hi[g.n_thr == 1 ? 0 : tile.e]; }
    for (int o = gl; o < MT * kOutputs; o += GL) {              // lane o of the group finishes outputs o, o + GL, ...
        const int i = o / kOutputs, j = o % kOutputs;
        int s = 0, s2 = 0;
        #pragma unroll
        for (int a = 0; a < MT; ++a)
            #pragma unroll
            for (int b = 0; b < kOutputs; ++b)
                if (a * kOutputs + b == o) { s = cnt[a][b]; if constexpr (kGated) s2 = cnt[a][kOutputs + b]; }
        const int64_t n = n0 + j;
        if (i >= tile.rows || n >= g.F) continue;
        const RowParams r = row_params(g, tile.row + i);
        const ColParams c = col_params(g, tile.e, n), c2 = kGated ? col_params(g, tile.e, g.F + n) : c;
        bool up = false, down = false;
        const float v = output_of<kCodes>(g, r, tile.e, n, c, (float)s, c2, (float)s2, lo, hi, up, down);
        if (g.out != nullptr) store_from_f32(g.out, (tile.row + i) * g.out_stride + n, g.dtype, v);
        if constexpr (kCodes) {
            const int at = (int)(n - f0);
            if (up || down) atomicOr(&bits[i][0][at / 32], 1u << (at & 31));
            if (up) atomicOr(&bits[i][1][at / 32], 1u << (at & 31));
        }
    }
    if constexpr (kCodes) {
        __syncthreads();
        tc::pdl_wait();                                         // (the sums begin at 0)
        const int words = per_cta / 32;
        const int64_t width = (g.F + kBlockCodes - 1) / kBlockCodes * kBlockCodes;     // (a packed row's padding is written too)
        for (int x = threadIdx.x; x < tile.rows * words; x += kThreads) {
            const int i = x / words, w = x % words;
            const int64_t c = f0 + w * 32;
            if (c >= width) continue;
            uint32_t* at = reinterpret_cast<uint32_t*>(g.out_packed + (tile.row + i) * (width / kBlockCodes * kBlockBytes) +
                                                       c / kBlockCodes * kBlockBytes + c % kBlockCodes / 8);
            const uint32_t nz = bits[i][0][w], pos = bits[i][1][w];
            at[0] = nz;
            at[4] = pos;
            const int sum = 2 * __popc(pos) - __popc(nz);
            if (sum != 0) atomicAdd(&g.out_sum[tile.row + i], sum);                     // (whole numbers: any order gives the same)
        }
    }
}

__global__ void __launch_bounds__(256)
zero_sums_kernel(const ExpertsArgs g)
{
    tc::pdl_wait();
    tc::pdl_trigger();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < g.R && i >= g.start[0] && i < g.start[g.E]) g.out_sum[i] = 0;
}

template <int MT>
cudaError_t launch_rows(const ExpertsArgs& g, cudaStream_t s)
{
    const int64_t nblk = (g.K + kBlockCodes - 1) / kBlockCodes;
    int GL = 1;
    while (GL < nblk && GL < 32) GL *= 2;
    const int per_cta = kThreads / GL * kOutputs;
    const int64_t tiles = g.R / MT + (g.E < g.R ? g.E : g.R);           // at most: an expert has one tile that is not full
    const int64_t width = g.out_packed != nullptr ? (g.F + kBlockCodes - 1) / kBlockCodes * kBlockCodes : g.F;
    const int64_t cols = (width + per_cta - 1) / per_cta;
    if (cols * tiles > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const unsigned grid = (unsigned)(cols * tiles);
    if (g.out_packed != nullptr) {
        const cudaError_t e = launch_pdl(zero_sums_kernel, dim3((unsigned)((g.R + 255) / 256)), dim3(256), 0, s, g);
        if (e != cudaSuccess) return e;
        return launch_pdl(g.gated ? experts_rows_kernel<MT, true, true> : experts_rows_kernel<MT, false, true>, dim3(grid), dim3(kThreads), 0, s, g, GL, (int)cols);
    } else {
        if (g.gated) experts_rows_kernel<MT, true, false><<<grid, kThreads, 0, s>>>(g, GL, (int)cols);
        else experts_rows_kernel<MT, false, false><<<grid, kThreads, 0, s>>>(g, GL, (int)cols);
    }
    return cudaGetLastError();
}

}  // namespace

// Which form: rows cost 6.2 us per million rows x columns x blocks of K (two rows to a tile: the POPC rate) on top of 4; tiles 8 us and, a round of one to every SM,
// 0.45 us per 512 codes of K or 1.4, whichever is more (of R rows dealt at random).  In a graph on one B200 (us, rows of an expert on average in brackets):
//                                                    rows  tiles                                             rows  tiles
//   4 rows (0.1), 64 x 2048 x 2048, gated, codes      5.8    9.7     320 (5.3), 60 x 1006 x 429              11.1   13.1
//   32 (0.5), 64 x 2048 x 2048, gated, codes         11.3   14.0     80 (1.3), 60 x 4096 x 300               12.0   23.1
//   64 (1), 64 x 2048 x 2048, gated, codes           17.3   16.1     512 (32), 16 x 512 x 512                 9.5    9.4
//   128 (2), 64 x 2048 x 2048, gated, codes          27.5   19.8     1554 (194), 8 x 1000 x 520              57.4   13.7
// One row to a tile where an expert has hardly more (16 rows (0.25): 6.7 us, two to a tile 7.2; 32: 11.3 and 12.5); four or eight were nowhere ahead.
cudaError_t launch_ternary_experts(const ExpertsArgs& g, cudaStream_t s)
{
    const double nblk = (double)((g.K + kBlockCodes - 1) / kBlockCodes), used = g.E * (1.0 - exp(-(double)g.R / g.E)), sms = device_sm_count();
    const double high = (double)g.R / used / 160.0, rounds = used * (high > 1.0 ? high : 1.0) * (double)((g.N + 127) / 128) / sms, each = 0.1125 * nblk;
    const double rows_us = 4.0 + 6.2e-6 * (double)g.R * (double)g.N * nblk, tiles_us = 8.0 + (rounds > 1.0 ? rounds : 1.0) * (each > 1.4 ? each : 1.4);
    if (rows_us > tiles_us && experts_tiles_supported(g)) return launch_experts_tiles(g, s);
    return 2 * g.R <= g.E ? launch_rows<1>(g, s) : launch_rows<2>(g, s);
}

}  // namespace rtn
