// Linear attention with a decay l per head over whole prompts, chunked on the tensor cores (bf16, head dimension D = 64 or 128).
// For a chunk of C = 128 tokens with the state S before it (g = log2 l, i and j count within the chunk):
//
//   scores = Q K^T                                   P_ij = l^(i-j) scores_ij for j <= i, else 0
//   O      = diag(l^(i+1)) Q S + P V                 out = scale O
//   S^T   <- l^C S^T + (diag(l^(C-1-j)) V)^T K
//
// Every product is a tcgen05.mma of kind::f16 with M = 128 and fp32 accumulators in tensor memory.  Operands that come
// from memory (Q, K, V) are exact in bf16.  What the kernel computes on the way to a product is split into bf16 terms that
// are multiplied one after the other into the same accumulator: P and S into two (2^-17 relative, far below the bf16
// output's own rounding), the decayed V into three (2^-25), because the state it enters is kept and returned in fp32.
//
// A CTA walks the chunks of one (sequence, query head, segment).  Warp roles, coupled by mbarriers:
//   P   (4 warps)  scores -> P terms, in place in tensor memory (A operand of P V); scales Q S by l^(i+1) before P V adds to it
//   S   (4 warps)  S^T -> bf16 terms in shared memory (B operand of Q S); scales S^T by l^C; initial and final state
//   V   (4 warps)  V tile -> decayed, transposed V terms in tensor memory (A operand of the state update), 32 tokens at a time
//   O   (4 warps)  O -> output rows
//   one thread loads the K, Q and V tiles by TMA into a ring, one issues every MMA in the order Q S, state, P V, next Q K^T:
//   the scores' conversion then runs beside Q S and the state update, the state's beside P V and the next scores.
// Tensor memory (512 columns): S^T | scores, then P | O | two entries of V terms.
//
// Rows past a sequence's end belong to its neighbour: K and V rows are zeroed in shared memory before a product reads
// them (0 * NaN), scores are masked by selection.  Inside a sequence a non-finite value can reach the outputs of up to 127
// tokens before it (0 * NaN in P V).
//
// Few heads and long prompts: the sequence is cut into segments; a first launch computes what each segment adds to the state
// (V and MMA roles only), and the second starts each segment from the decayed sum of what came before.
#include "rtn_internal.cuh"
#include "rtn_types.cuh"
#include "rtn_decay.cuh"
#include "rtn_tcgen05.cuh"
#include "rtn_tensormap.cuh"
#include "rtn_timeline.cuh"

RTN_TL_DEFINE(decay_chunk)
#include "rtn_conv_i8_common.cuh"

namespace rtn {

namespace {

using conv_detail::wait_or_die;

constexpr int kC = 128;                     // tokens of a chunk
constexpr int kEntry = 32;                  // tokens of an entry of V terms
constexpr int kThreads = 18 * 32;
constexpr int kWarpS = 4, kWarpV = 8, kWarpO = 12, kWarpLoad = 16, kWarpMma = 17;
constexpr uint32_t kColS = 0, kColP = 128, kColO = 256, kColV = 384, kTmemCols = 512;
constexpr int kMaxSlots = 9;

template <int D> struct Layout {
    static constexpr int kSlots = D == 128 ? 5 : 9;             // ring of K, Q, V tiles
    static constexpr uint32_t kTile = kC * D * 2;
    static constexpr uint32_t kHalf = kC * 128;                 // 64 columns of a tile
    static constexpr uint32_t kState = D * D * 2;               // one bf16 term of S^T
    static constexpr uint32_t off_state = kSlots * kTile;
    static constexpr uint32_t off_table = off_state + 2 * kState;
    static constexpr uint32_t off_bar = off_table + kC * 4;
    static constexpr uint32_t kBytes = off_bar + 512 + 1024;    // and room to start on a 1024-byte boundary
};

struct Bars {
    uint64_t full[kMaxSlots], empty[kMaxSlots];     // tiles: load -> users, MMA -> load
    uint64_t sc_full, p_full, qs_done;              // scores ready; P ready and Q S scaled; Q S in the accumulator
    uint64_t s_full, kv_done;                       // state terms ready and S^T scaled; state updated
    uint64_t vt_full[2], vt_empty[2];               // V terms
    uint64_t o_full, o_empty;                       // O complete; O read
    uint64_t fixed;                                 // rows past the end zeroed
    uint32_t tmem_slot;
    int dead;
};
static_assert(sizeof(Bars) <= 512, "barriers");

struct ChunkPlan {
    int64_t seg_len;        // tokens of a segment, a multiple of kC
    int segments;           // of the longest sequence
    float* local;           // [B][H][segments - 1][D][D]: what a segment adds to the state
};

// l^n from log2 l; n = 0 gives 1 for every l (log2 l may be -inf).
__device__ __forceinline__ float decay_pow(float g2, float n) { return n == 0.f ? 1.f : exp2f(n * g2); }

__device__ __forceinline__ float bf16_low(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_high(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

__device__ __forceinline__ void tma_load_tile(uint32_t dst, const CUtensorMap* map, int c, int head, int token, uint64_t* bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c), "r"(head), "r"(token), "r"(tc::smem_addr(bar)) : "memory");
}

template <int D, bool kStates>
__global__ void __launch_bounds__(kThreads, 1)
decay_chunk_kernel(const DecayArgs g, const ChunkPlan p, const __grid_constant__ CUtensorMap map_q,
                   const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    using L = Layout<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float* table = reinterpret_cast<float*>(smem + L::off_table);            // l^(C-1-j)
    Bars& bar = *reinterpret_cast<Bars*>(smem + L::off_bar);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = warp & 3;

    // ---- what this CTA works on
    const int segs = kStates ? p.segments - 1 : p.segments;
    const int h = (int)(blockIdx.x % g.H), hk = h / (g.H / g.Hk);
    const int64_t rest = blockIdx.x / g.H;
    const int seg = (int)(rest % segs);
    const int64_t b = rest / segs;
    int64_t first, len, slot;
    if (!sequence_bounds(g, b, first, len, slot)) {
        if (!kStates && seg == 0 && threadIdx.x == 0) atomicOr(g.status, kStatusBadIndex);
        return;
    }
    const int64_t s0 = (int64_t)seg * p.seg_len;
    if (seg > 0 && s0 >= len) return;
    const bool last_seg = s0 + p.seg_len >= len;
    if (kStates && (last_seg || slot < 0)) return;
    const int n_tok = (int)(last_seg ? len - s0 : p.seg_len);
    const int64_t row0 = first + s0;                                           // first token's row
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(g.out) + row0 * g.o_token + h * g.o_head;
    if (!kStates && slot < 0) {
        for (int64_t i = threadIdx.x; i < (int64_t)n_tok * D; i += kThreads) out[(i / D) * g.o_token + i % D] = __float2bfloat16_rn(0.f);
        return;
    }
    const int chunks = (n_tok + kC - 1) / kC;
    const int tail = n_tok - (chunks - 1) * kC;                                // tokens of the last chunk
    const float g2 = g.log_decay[h] * 1.4426950408889634f;

    // ---- set-up
    if (warp == kWarpMma) tc::tmem_alloc(&bar.tmem_slot, kTmemCols);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kMaxSlots; ++i) { tc::mbar_init(&bar.full[i], 1); tc::mbar_init(&bar.empty[i], 1); }
        tc::mbar_init(&bar.sc_full, 1); tc::mbar_init(&bar.p_full, 128); tc::mbar_init(&bar.qs_done, 1);
        tc::mbar_init(&bar.s_full, D); tc::mbar_init(&bar.kv_done, 1);
        for (int i = 0; i < 2; ++i) { tc::mbar_init(&bar.vt_full[i], D); tc::mbar_init(&bar.vt_empty[i], 1); }
        tc::mbar_init(&bar.o_full, 1); tc::mbar_init(&bar.o_empty, 128); tc::mbar_init(&bar.fixed, D);
        tc::mbar_init_fence();
        bar.dead = 0;
    }
    if (threadIdx.x < kC) table[threadIdx.x] = decay_pow(g2, (float)(kC - 1 - threadIdx.x));
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    const uint32_t tmem = bar.tmem_slot;
    const uint32_t base = tc::smem_addr(smem);
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    volatile int* dead = &bar.dead;
    auto wait = [&](uint64_t* m, int phase) { return wait_or_die(m, (uint32_t)phase & 1u, g.status, dead); };
    // whole warps wait together and give up together: what follows is warp-collective
    auto warp_wait = [&](uint64_t* m, int phase) { return __all_sync(0xffffffffu, wait(m, phase)) != 0; };
    // tiles in the order K, Q, V of each chunk (K, V where only states are wanted)
    constexpr int kPer = kStates ? 2 : 3;
    auto tile_slot = [&](int c, int which) { return (c * kPer + which) % L::kSlots; };
    auto tile_phase = [&](int c, int which) { return (c * kPer + which) / L::kSlots; };
    constexpr int kTileK = 0, kTileQ = 1, kTileV = kStates ? 1 : 2;

    if (warp == kWarpLoad) {
        // ------------------------------------------------------------ tiles (one thread)
        if (lane == 0) {
            int t = 0;
            for (; t < chunks * kPer; ++t) {
                const int s = t % L::kSlots, c = t / kPer, which = t % kPer;
                if (!wait(&bar.empty[s], t / L::kSlots + 1)) break;
                const CUtensorMap* map = which == kTileK ? &map_k : which == kTileV ? &map_v : &map_q;
                tc::mbar_arrive_expect_tx(&bar.full[s], L::kTile);
                for (int half = 0; half < D / 64; ++half)
                    tma_load_tile(base + s * L::kTile + half * L::kHalf, map, half * 64, !kStates && which == kTileQ ? h : hk,
                                  (int)row0 + c * kC, &bar.full[s]);
            }
            // every copy has landed before the CTA ends, also when a wait gave up
            for (int u = t > L::kSlots ? t - L::kSlots : 0; u < t; ++u) tc::mbar_wait(&bar.full[u % L::kSlots], (uint32_t)(u / L::kSlots) & 1u, g.status);
        }
    } else if (warp == kWarpMma) {
        // ------------------------------------------------------------ every MMA (one thread)
        if (lane == 0) {
            constexpr uint32_t id_kk = tc::idesc_bf16(128, kC, false);           // scores
            constexpr uint32_t id_s = tc::idesc_bf16(128, D, false), id_mn = tc::idesc_bf16(128, D, true);
            auto kmajor = [&](uint32_t tile, uint32_t half_bytes, int step) {
                return tc::smem_desc_sw128(tile + (uint32_t)(step >> 2) * half_bytes + (uint32_t)(step & 3) * 32u, 16);
            };
            auto mnmajor = [&](uint32_t tile, int step) { return tc::smem_desc_sw128(tile + (uint32_t)step * 2048u, L::kHalf); };
            auto scores = [&](int c) {
                const int sk = tile_slot(c, kTileK), sq = tile_slot(c, kTileQ);
                if (!wait(&bar.full[sk], tile_phase(c, kTileK)) || !wait(&bar.full[sq], tile_phase(c, kTileQ))) return false;
                tc::tc_fence_after_sync();
                #pragma unroll
                for (int s = 0; s < D / 16; ++s)
                    tc::mma_f16_ss(tmem + kColP, kmajor(base + sq * L::kTile, L::kHalf, s), kmajor(base + sk * L::kTile, L::kHalf, s), id_kk, s > 0);
                tc::mma_commit(&bar.sc_full);
                return true;
            };
            bool alive = chunks == 0 || kStates || scores(0);
            for (int c = 0; c < chunks && alive; ++c) {
                const int sk = tile_slot(c, kTileK), sq = tile_slot(c, kTileQ), sv = tile_slot(c, kTileV);
                if constexpr (!kStates) {
                    alive = wait(&bar.s_full, c) && (c == 0 || wait(&bar.o_empty, c - 1));
                    if (!alive) break;
                    tc::tc_fence_after_sync();
                    #pragma unroll
                    for (int term = 0; term < 2; ++term)
                        #pragma unroll
                        for (int s = 0; s < D / 16; ++s)
                            tc::mma_f16_ss(tmem + kColO, kmajor(base + sq * L::kTile, L::kHalf, s),
                                           kmajor(base + L::off_state + term * L::kState, D * 128, s), id_s, term + s > 0);
                    tc::mma_commit(&bar.qs_done);
                    tc::mma_commit(&bar.empty[sq]);
                } else {
                    alive = wait(&bar.full[sk], tile_phase(c, kTileK));
                    if (!alive) break;
                }
                // the last chunk's rows past the end are zero before a product reads them
                if (c == chunks - 1 && tail < kC && !(alive = wait(&bar.fixed, 0))) break;
                for (int e = 0; e < kC / kEntry && alive; ++e) {
                    const int ve = c * (kC / kEntry) + e;
                    if (!(alive = wait(&bar.vt_full[ve & 1], ve >> 1))) break;
                    tc::tc_fence_after_sync();
                    #pragma unroll
                    for (int term = 0; term < 3; ++term)
                        #pragma unroll
                        for (int s = 0; s < kEntry / 16; ++s)
                            tc::mma_f16_ts(tmem + kColS, tmem + kColV + (uint32_t)((ve & 1) * 64 + term * 16 + s * 8),
                                           mnmajor(base + sk * L::kTile, e * (kEntry / 16) + s), id_mn, !kStates || ve + term + s > 0);
                    tc::mma_commit(&bar.vt_empty[ve & 1]);
                }
                if (!alive) break;
                if (!kStates || c == chunks - 1) tc::mma_commit(&bar.kv_done);       // states only: nobody follows the chunks
                tc::mma_commit(&bar.empty[sk]);
                if constexpr (!kStates) {
                    if (!(alive = wait(&bar.p_full, c))) break;
                    tc::tc_fence_after_sync();
                    #pragma unroll
                    for (int term = 0; term < 2; ++term)
                        #pragma unroll
                        for (int s = 0; s < kC / 16; ++s)
                            tc::mma_f16_ts(tmem + kColO, tmem + kColP + (uint32_t)((s >> 1) * 32 + term * 16 + (s & 1) * 8),
                                           mnmajor(base + sv * L::kTile, s), id_mn, true);
                    tc::mma_commit(&bar.o_full);
                }
                tc::mma_commit(&bar.empty[sv]);
                if constexpr (!kStates) {
                    if (c + 1 < chunks) alive = scores(c + 1);
                }
            }
        }
    } else if (warp < kWarpS) {
        // ------------------------------------------------------------ P: row i of the chunk per thread
        if constexpr (!kStates) {
            const int i = quad * 32 + lane;
            float near[16];                                                   // l^(15 - jj)
            #pragma unroll
            for (int jj = 0; jj < 16; ++jj) near[jj] = decay_pow(g2, (float)(15 - jj));
            const float own = decay_pow(g2, (float)(i + 1));
            for (int c = 0; c < chunks; ++c) {
                if (!warp_wait(&bar.sc_full, c)) break;
                tc::tc_fence_after_sync();
                #pragma unroll 1
                for (int kb = 0; kb < kC / 32; ++kb) {
                    const uint32_t at = tmem + lanes + kColP + (uint32_t)(kb * 32);
                    uint32_t v[32], t[32];                                    // t: sixteen words of high terms, sixteen of low
                    if (kb > quad) {                                          // keys after every row of the warp
                        #pragma unroll
                        for (int x = 0; x < 32; ++x) t[x] = 0;
                    } else {
                        tc::tmem_ld32(at, v);
                        float f0 = 0.f, f1 = 0.f;
                        if (kb < quad) { f0 = decay_pow(g2, (float)(i - kb * 32 - 15)); f1 = decay_pow(g2, (float)(i - kb * 32 - 31)); }
                        tc::tmem_ld_wait();
                        #pragma unroll
                        for (int x = 0; x < 32; x += 2) {
                            float y0, y1;
                            if (kb < quad) {
                                const float f = x < 16 ? f0 : f1;
                                y0 = __uint_as_float(v[x]) * (f * near[x & 15]);
                                y1 = __uint_as_float(v[x + 1]) * (f * near[(x & 15) + 1]);
                            } else {                                          // the diagonal block: row lane, key x
                                y0 = x <= lane ? __uint_as_float(v[x]) * decay_pow(g2, (float)(lane - x)) : 0.f;
                                y1 = x + 1 <= lane ? __uint_as_float(v[x + 1]) * decay_pow(g2, (float)(lane - x - 1)) : 0.f;
                            }
                            const uint32_t hi = pack2<__nv_bfloat16>(y0, y1);
                            t[x >> 1] = hi;
                            t[16 + (x >> 1)] = pack2<__nv_bfloat16>(y0 - bf16_low(hi), y1 - bf16_high(hi));
                        }
                    }
                    tc::tmem_st32(at, t);
                }
                tc::tmem_st_wait();
                if (!warp_wait(&bar.qs_done, c)) break;
                tc::tc_fence_after_sync();
                #pragma unroll 1
                for (int x0 = 0; x0 < D; x0 += 32) {
                    uint32_t v[32];
                    tc::tmem_ld32(tmem + lanes + kColO + (uint32_t)x0, v);
                    tc::tmem_ld_wait();
                    #pragma unroll
                    for (int x = 0; x < 32; ++x) v[x] = __float_as_uint(__uint_as_float(v[x]) * own);
                    tc::tmem_st32(tmem + lanes + kColO + (uint32_t)x0, v);
                }
                tc::tmem_st_wait();
                tc::tc_fence_before_sync();
                tc::mbar_arrive(&bar.p_full);
            }
        }
    } else if (warp < kWarpV) {
        // ------------------------------------------------------------ S: state column (row of S^T) d per thread
        const int d = quad * 32 + lane;
        if (d < D) {
            const int64_t at = (slot * g.H + h) * (int64_t)D * D + d;
            const float* local = p.local + ((b * g.H + h) * (int64_t)(p.segments - 1)) * D * D + d;
            // 32 rows of the state before the segment: the given one and what the segments before this one added
            auto initial = [&](int r0, float (&v)[32]) {
                const float w0 = decay_pow(g2, (float)s0);
                #pragma unroll
                for (int x = 0; x < 32; ++x) v[x] = g.state != nullptr && w0 != 0.f ? w0 * g.state[at + (int64_t)(r0 + x) * D] : 0.f;
                for (int s = 0; s < seg; ++s) {
                    const float w = decay_pow(g2, (float)((int64_t)(seg - 1 - s) * p.seg_len));
                    if (w == 0.f) continue;
                    #pragma unroll
                    for (int x = 0; x < 32; ++x) v[x] = fmaf(w, local[((int64_t)s * D + r0 + x) * D], v[x]);
                }
            };
            bool alive = true;
            if constexpr (!kStates) {
                for (int c = 0; c < chunks; ++c) {
                    if (c > 0 && !(alive = warp_wait(&bar.kv_done, c - 1))) break;
                    tc::tc_fence_after_sync();
                    const float keep = decay_pow(g2, (float)(c == chunks - 1 ? tail : kC));
                    uint8_t* terms = smem + L::off_state + d * 128;
                    #pragma unroll 1
                    for (int r0 = 0; r0 < D; r0 += 32) {
                        const uint32_t col = tmem + lanes + kColS + (uint32_t)r0;
                        uint32_t u[32];
                        if (c == 0) {
                            float v[32];
                            initial(r0, v);
                            #pragma unroll
                            for (int x = 0; x < 32; ++x) u[x] = __float_as_uint(v[x]);
                            __syncwarp();
                        } else {
                            tc::tmem_ld32(col, u);
                            tc::tmem_ld_wait();
                        }
                        #pragma unroll
                        for (int x = 0; x < 32; x += 8) {
                            uint32_t hi[4], lo[4];
                            #pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                const float a = __uint_as_float(u[x + 2 * y]), bb = __uint_as_float(u[x + 2 * y + 1]);
                                hi[y] = pack2<__nv_bfloat16>(a, bb);
                                lo[y] = pack2<__nv_bfloat16>(a - bf16_low(hi[y]), bb - bf16_high(hi[y]));
                            }
                            const int r = r0 + x;
                            const uint32_t o = (uint32_t)(r >> 6) * (D * 128) + ((uint32_t)(((r & 63) >> 3) ^ (d & 7)) << 4);
                            *reinterpret_cast<uint4*>(terms + o) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                            *reinterpret_cast<uint4*>(terms + L::kState + o) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                        }
                        #pragma unroll
                        for (int x = 0; x < 32; ++x) u[x] = __float_as_uint(__uint_as_float(u[x]) * keep);
                        tc::tmem_st32(col, u);
                    }
                    tc::tmem_st_wait();
                    tc::fence_smem_to_async_proxy();
                    tc::tc_fence_before_sync();
                    tc::mbar_arrive(&bar.s_full);
                }
            }
            // the state after the segment
            if ((kStates || last_seg) && alive && (chunks == 0 || warp_wait(&bar.kv_done, kStates ? 0 : chunks - 1))) {
                tc::tc_fence_after_sync();
                float* dst = kStates ? p.local + (((b * g.H + h) * (int64_t)(p.segments - 1)) + seg) * D * D + d : g.state_out + at;
                #pragma unroll 1
                for (int r0 = 0; r0 < D; r0 += 32) {
                    uint32_t u[32];
                    if (chunks > 0) {
                        tc::tmem_ld32(tmem + lanes + kColS + (uint32_t)r0, u);
                        tc::tmem_ld_wait();
                    } else {
                        float v[32];
                        initial(r0, v);
                        #pragma unroll
                        for (int x = 0; x < 32; ++x) u[x] = __float_as_uint(v[x]);
                    }
                    #pragma unroll
                    for (int x = 0; x < 32; ++x) dst[(int64_t)(r0 + x) * D] = __uint_as_float(u[x]);
                }
            }
        }
    } else if (warp < kWarpO) {
        // ------------------------------------------------------------ V: column d of the V tile per thread
        const int d = quad * 32 + lane;
        if (d < D) {
            const uint32_t v_col = (uint32_t)(d >> 6) * L::kHalf + (uint32_t)(d & 7) * 2u;
            const uint32_t chunk16 = (uint32_t)((d & 63) >> 3);
            for (int c = 0; c < chunks; ++c) {
                const int sv = tile_slot(c, kTileV);
                if (!warp_wait(&bar.full[sv], tile_phase(c, kTileV))) break;
                const int n = c == chunks - 1 ? tail : kC;
                uint8_t* tile = smem + sv * L::kTile;
                if (n < kC) {
                    const int sk = tile_slot(c, kTileK);
                    if (!warp_wait(&bar.full[sk], tile_phase(c, kTileK))) break;
                    // 16-byte pieces of the rows n .. C-1 of both tiles (every half)
                    const int pieces = (kC - n) * 8;
                    for (int x = d; x < pieces * (D / 64); x += D) {
                        const uint32_t o = (uint32_t)(x / pieces) * L::kHalf + (uint32_t)n * 128u + (uint32_t)(x % pieces) * 16u;
                        *reinterpret_cast<uint4*>(tile + o) = make_uint4(0, 0, 0, 0);
                        *reinterpret_cast<uint4*>(smem + sk * L::kTile + o) = make_uint4(0, 0, 0, 0);
                    }
                    tc::fence_smem_to_async_proxy();
                    tc::mbar_arrive(&bar.fixed);
                }
                // only states: the weight runs on to the end of the segment
                const float run = kStates ? decay_pow(g2, (float)(n_tok - (c * kC + n))) : 1.f;
                bool alive = true;
                #pragma unroll 1
                for (int e = 0; e < kC / kEntry; ++e) {
                    const int ve = c * (kC / kEntry) + e;
                    uint32_t hi[16], mid[16], lo[16];
                    #pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        float y[2];
                        #pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int j = e * kEntry + 2 * x + k;
                            const uint32_t o = v_col + (uint32_t)j * 128u + ((chunk16 ^ (uint32_t)(j & 7)) << 4);
                            const float v = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(tile + o) << 16);
                            const float w = table[j + kC - n < kC ? j + kC - n : 0];
                            y[k] = j < n ? v * (kStates ? w * run : w) : 0.f;
                        }
                        hi[x] = pack2<__nv_bfloat16>(y[0], y[1]);
                        y[0] -= bf16_low(hi[x]); y[1] -= bf16_high(hi[x]);
                        mid[x] = pack2<__nv_bfloat16>(y[0], y[1]);
                        lo[x] = pack2<__nv_bfloat16>(y[0] - bf16_low(mid[x]), y[1] - bf16_high(mid[x]));
                    }
                    if (!(alive = warp_wait(&bar.vt_empty[ve & 1], (ve >> 1) + 1))) break;
                    tc::tc_fence_after_sync();
                    const uint32_t col = tmem + lanes + kColV + (uint32_t)((ve & 1) * 64);
                    tc::tmem_st16(col, hi);
                    tc::tmem_st16(col + 16, mid);
                    tc::tmem_st16(col + 32, lo);
                    tc::tmem_st_wait();
                    tc::tc_fence_before_sync();
                    tc::mbar_arrive(&bar.vt_full[ve & 1]);
                }
                if (!alive) break;
            }
        }
    } else {
        // ------------------------------------------------------------ O: row i of the chunk per thread
        if constexpr (!kStates) {
            const int i = quad * 32 + lane;
            for (int c = 0; c < chunks; ++c) {
                if (!warp_wait(&bar.o_full, c)) break;
                tc::tc_fence_after_sync();
                uint32_t w[D / 2];
                #pragma unroll
                for (int x0 = 0; x0 < D; x0 += 32) {
                    uint32_t v[32];
                    tc::tmem_ld32(tmem + lanes + kColO + (uint32_t)x0, v);
                    tc::tmem_ld_wait();
                    #pragma unroll
                    for (int x = 0; x < 32; x += 2)
                        w[(x0 + x) / 2] = pack2<__nv_bfloat16>(g.scale * __uint_as_float(v[x]), g.scale * __uint_as_float(v[x + 1]));
                }
                tc::tc_fence_before_sync();
                tc::mbar_arrive(&bar.o_empty);
                if (c * kC + i < n_tok) {
                    uint4* dst = reinterpret_cast<uint4*>(out + (int64_t)(c * kC + i) * g.o_token);
                    #pragma unroll
                    for (int x = 0; x < D / 8; ++x) dst[x] = make_uint4(w[4 * x], w[4 * x + 1], w[4 * x + 2], w[4 * x + 3]);
                }
            }
        }
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    if (warp == kWarpMma) tc::tmem_dealloc(tmem, kTmemCols);
}

// [tokens][heads][D] bf16 tensor in boxes of 128 tokens x 64 elements of one head, rows under the 128-byte swizzle.
bool encode_heads(CUtensorMap* map, const void* ptr, int64_t tokens, int heads, int D, int64_t token, int64_t head)
{
    if ((reinterpret_cast<uintptr_t>(ptr) & 15) != 0 || ((token | head) & 7) != 0) return false;
    if (heads == 1) head = 8;                       // never stepped over, but the map wants a stride
    if (token < 8) { if (tokens > 1) return false; token = 8; }
    if (head < 8) return false;
    EncodeTiledFn enc = encode_tiled_fn();
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)head * 2, (cuuint64_t)token * 2};
    const cuuint32_t box[3] = {64, 1, (cuuint32_t)kC};
    const cuuint32_t estr[3] = {1, 1, 1};
    return enc != nullptr && enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr,
                                 CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

ChunkPlan make_plan(const DecayArgs& g)
{
    ChunkPlan p{};
    const int64_t chunks = (g.max_len + kC - 1) / kC, ctas = g.B * g.H, sms = device_sm_count();
    int64_t segs = 1;
    if (ctas < sms) segs = sms / ctas;
    if (segs > chunks / 4) segs = chunks / 4;
    if (segs > 16) segs = 16;
    if (segs < 1) segs = 1;
    p.seg_len = (chunks + segs - 1) / segs * kC;
    if (p.seg_len < kC) p.seg_len = kC;
    p.segments = (int)((chunks * kC + p.seg_len - 1) / p.seg_len);
    if (p.segments < 1) p.segments = 1;
    return p;
}

template <int D>
cudaError_t launch_typed(const DecayArgs& g, cudaStream_t s, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v)
{
    constexpr int bytes = (int)Layout<D>::kBytes;
    ChunkPlan p = make_plan(g);
    cudaError_t e = cudaFuncSetAttribute(decay_chunk_kernel<D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    void* scratch = nullptr;
    if (p.segments > 1) {
        e = cudaFuncSetAttribute(decay_chunk_kernel<D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != cudaSuccess) return e;
        e = cudaMallocAsync(&scratch, (size_t)g.B * g.H * (p.segments - 1) * D * D * sizeof(float), s);
        if (e != cudaSuccess) return e;
        p.local = static_cast<float*>(scratch);
        decay_chunk_kernel<D, true><<<(unsigned)(g.B * g.H * (p.segments - 1)), kThreads, bytes, s>>>(g, p, q, k, v);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) {
        decay_chunk_kernel<D, false><<<(unsigned)(g.B * g.H * p.segments), kThreads, bytes, s>>>(g, p, q, k, v);
        e = cudaGetLastError();
    }
    if (scratch != nullptr) {
        const cudaError_t e2 = cudaFreeAsync(scratch, s);
        if (e == cudaSuccess) e = e2;
    }
    return e;
}

}  // namespace

bool decay_chunk_supported(const DecayArgs& g)
{
    return g.dtype == RTN_BF16 && g.Dk == g.Dv && (g.Dk == 64 || g.Dk == 128) && g.max_len > 16 && g.total > 0 &&
           (reinterpret_cast<uintptr_t>(g.out) & 15) == 0 && ((g.o_token | g.o_head) & 7) == 0 && g.B * g.H * 16 < 0x7fffffff;
}

cudaError_t launch_decay_chunk(const DecayArgs& g, cudaStream_t s, bool& taken)
{
    CUtensorMap q, k, v;
    taken = encode_heads(&q, g.q, g.total, g.H, g.Dk, g.q_token, g.q_head) && encode_heads(&k, g.k, g.total, g.Hk, g.Dk, g.k_token, g.k_head) &&
            encode_heads(&v, g.v, g.total, g.Hk, g.Dv, g.v_token, g.v_head);
    if (!taken) return cudaSuccess;
    return g.Dk == 64 ? launch_typed<64>(g, s, q, k, v) : launch_typed<128>(g, s, q, k, v);
}

}  // namespace rtn
