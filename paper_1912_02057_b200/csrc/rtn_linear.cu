// Ternary linear layer for few rows (decoding): out = act(affine(S_xw) + bias) + residual, S_xw by Eq. 9 (AND / XOR / popcount
// on the packed planes).
//
// Bound: DRAM, the packed weights read once (K/4 bytes per column against 2 POPC per 32 codes and row; from about four rows on
// the POPC rate binds).  A group of GL lanes (a power of two, at most a warp) owns CPG weight rows at a time: lane i takes
// the 128-code blocks i, i + GL, ... of each (32 adjacent bytes, so a group reads whole lines), keeps a
// counter pair per activation row and column, and one shuffle tree joins the group.  CPG columns at once keep that many loads in flight.
#include "rtn_internal.cuh"
#include "rtn_epilogue.cuh"

namespace rtn {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 8;             // activation rows of a pass

template <int MT, int CPG>
__global__ void __launch_bounds__(kThreads)
linear_rows_kernel(const GemmArgs g, const LinearArgs p, int GL)
{
    const int gl = threadIdx.x & (GL - 1);
    const int64_t group = (int64_t)blockIdx.x * (kThreads / GL) + threadIdx.x / GL;
    const int64_t n0 = group * CPG;
    const int64_t m0 = (int64_t)blockIdx.y * MT;
    const int64_t nblk = (g.K + kBlockCodes - 1) / kBlockCodes;
    const uint4* __restrict__ A = reinterpret_cast<const uint4*>(g.a_packed);
    const uint4* __restrict__ W = reinterpret_cast<const uint4*>(g.w_packed);
    int cnt[MT][CPG];
    #pragma unroll
    for (int i = 0; i < MT; ++i)
        #pragma unroll
        for (int j = 0; j < CPG; ++j) cnt[i][j] = 0;
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
            for (int j = 0; j < CPG; ++j) cnt[i][j] += __shfl_xor_sync(0xffffffffu, cnt[i][j], d);
    }
    // lane j of the group finishes outputs j, j + GL, ... of its MT x CPG
    #pragma unroll
    for (int i = 0; i < MT; ++i)
        #pragma unroll
        for (int j = 0; j < CPG; ++j) {
            const int64_t m = m0 + i, n = n0 + j;
            if (((i * CPG + j) & (GL - 1)) != gl || m >= g.M || n >= g.N) continue;
            const EpilogueParams& ep = g.ep;
            const int64_t ia = ep.n_aparam == 1 ? 0 : m, iw = ep.n_wparam == 1 ? 0 : n;
            float y = epilogue_f64(cnt[i][j], g.a_sum[m], g.w_sum[n], (double)g.K, ep.a_scale[ia], ep.a_offset[ia],
                                   ep.w_scale[iw], ep.w_offset[iw]);
            if (p.bias != nullptr) y += p.bias[n];
            y = activate(y, p.act);
            if (p.residual != nullptr) y += load_as_f32(p.residual, m * p.res_stride + n, p.dtype);
            store_from_f32(p.out, m * p.out_stride + n, p.dtype, y);
        }
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

// Few rows: the weights are streamed once through the bit-plane kernel.
bool linear_rows_path(int64_t M, int64_t N, int64_t K)
{
    return M <= kMaxRows || !gemm_i8_supported(M, N, K);
}

cudaError_t launch_linear(const GemmArgs& g, const LinearArgs& l, cudaStream_t s)
{
    if (!linear_rows_path(g.M, g.N, g.K)) return launch_gemm_i8_linear(g, l, s);
    if (g.M == 1) return launch_rows<1, 4>(g, l, s);
    if (g.M == 2) return launch_rows<2, 4>(g, l, s);
    if (g.M <= 4) return launch_rows<4, 4>(g, l, s);
    return launch_rows<8, 2>(g, l, s);
}

}  // namespace rtn
