// Linear attention with a decay l per head over whole prompts, chunked on the tensor cores (bf16, head dimension D = 64 or 128).
// For a chunk of C = 128 tokens with the state S before it (g = log2 l, i and j count within the chunk):
//
//   scores = Q K^T                                   P_ij = l^(i-j) scores_ij for j <= i, else 0
//   O      = diag(l^(i+1)) Q S + P V                 out = scale O
//   S^T   <- l^C S^T + (diag(l^(C-1-j)) V)^T K
//
// Every product is a tcgen05.mma of kind::f16 with M = 128 and fp32 accumulators in tensor memory.  Operands that come
// from memory (Q, K, V) are exact in bf16.  What the kernel computes on the way to a product is split into bf16 terms that
// are multiplied one after the other into the same accumulator: P and S into two (2^-17 relative, against 2^-9 of the bf16
// output: 0.24 % of the outputs are not the bf16 value nearest to the definition's in double, 0.05 % of the token-by-token kernel's; the
// error in norm is the same 1.66e-3), the decayed V into three (2^-25), because the state it enters is kept and returned in fp32.
// The tensor core's accumulation rounds towards zero, so what a chunk adds to the state gets an accumulator of its own and is
// added in registers: accumulated onto the state itself, its 24 products a chunk bent the state by 1.3e-6.
//
// A CTA walks the chunks of one (sequence, query head, segment).  Warp roles, coupled by mbarriers:
//   P   (8 warps)  scores -> P terms, in place in tensor memory (A operand of P V); scales Q S by l^(i+1) before P V adds to it;
//                  O -> bf16 rows, staged in the K tile's slot and stored by TMA
//   S   (8 warps)  the state, in registers (a row of S^T per pair of threads): decays it, adds the chunk's part, writes its terms
//                  to shared memory (B operand of Q S); initial and final state
//   V   (8 warps)  V tile -> decayed, transposed V terms in tensor memory (A operand of the state update), 32 tokens at a time
//   three threads load the Q, K and V tiles by TMA into a ring each, one warp issues every MMA in the order Q S, state, P V, next Q K^T:
//   the scores' conversion then runs beside Q S and the state update, the state's beside P V and the next scores.
// The conversions are what the kernel spends its issue slots on, with a chain of dependent instructions per value: two warps per
// role and scheduler hide what one could not.  The state's 64 registers a thread come from the other roles' shares (setmaxnreg).
// Bound: at D = 128 a chunk's products are 4100 clocks of the tensor pipe (terms counted), the hand-overs between them and the
// conversions make them 5900; the conversions use 0.59 of the issue slots.  148 heads of 2048 tokens: D = 128 73 us, 0.67 of a plain copy
// of the same bytes, D = 64 44 us, 0.54.
// Tensor memory (512 columns): state update | scores, then P | O | two entries of V terms (what is left of each 128 columns, too).
//
// Rows past a sequence's end belong to its neighbour: K and V rows are zeroed in shared memory before a product reads
// them (0 * NaN), scores are masked by selection.  A non-finite v of a later token in the chunk would reach a row through the
// zeros of P: the V warps see every value, and one whose third term is not finite is zeroed in the tile P V reads; the rows from
// its token on get a NaN in that column when they are written.
//
// Few heads and long prompts: the sequence is cut into segments; a first launch computes what each segment adds to the state
// (V and MMA roles only), and the second starts each segment from the decayed sum of what came before.
#include "rtn_internal.cuh"
#include "rtn_types.cuh"
#include "rtn_decay.cuh"
#include "rtn_tcgen05.cuh"
#include "rtn_tensormap.cuh"
#include "rtn_timeline.cuh"

// Timeline slots (instrumented build only): 0 kernel entry, 1 set-up done, 4 kernel end; chunk c in 4 .. 7 of a CTA, from
// slot 8 + 20 (c - 4): 0 state update begins, 1 / 2 Q S begins / issued, 3 state update issued, 4 P ready, 5 P V issued,
// 6 next scores issued (MMA thread); 7 scores ready, 8 P written, 9 Q S ready, 10 Q S scaled; 11 state updated, 12 state
// terms written; 13 V tile landed, 14 V terms written; 15 O complete, 16 O read and staged.
RTN_TL_DEFINE(decay_chunk)
#define CHUNK_TL(k) RTN_TL(decay_chunk, c >= 4 && c < 8 ? 8 + 20 * (c - 4) + (k) : -1)

namespace rtn {

namespace {

constexpr int kC = 128;                     // tokens of a chunk
constexpr int kThreads = 28 * 32;
// (the MMA warp on the scheduler with the fewest conversions: heads of 64 have 64 rows of states and values, in the lanes of warps 0 and 1
// modulo 4; on that of warp 1 a prompt of 32768 tokens of 16 such heads takes 127 us instead of 119)
constexpr int kWarpLoadQ = 0, kWarpMma = 2, kWarpLoadK = 1 /* V: 3 */, kWarpS = 4, kWarpP = 12, kWarpV = 20;
// registers a thread: 72 at launch (V keeps them); 40 + 2 x (96 + 64 + 72) = 504 = 7 x 72 per warp group of 128
constexpr int kRegsRest = 40, kRegsS = 96, kRegsP = 64;

constexpr uint32_t kColS = 0, kColP = 128, kColO = 256, kTmemCols = 512;

template <int D, bool kStates> struct Layout {
    // Slots of the three rings.  A Q tile lives from its scores to Q S, a V tile from its conversion to P V, a K tile from its scores to the
    // store of the rows that are staged in its slot after the state update.  Where only states are wanted the slots of Q and the
    // state's terms go to K and V.
    static constexpr int kSlotsQ = kStates ? 0 : D == 128 ? 1 : 3;
    static constexpr int kSlotsK = kStates ? (D == 128 ? 3 : 4) : D == 128 ? 2 : 3;
    static constexpr int kSlotsV = kStates ? (D == 128 ? 4 : 5) : D == 128 ? 2 : 3;
    static constexpr int kSlots = kSlotsQ + kSlotsK + kSlotsV;
    static constexpr uint32_t kTile = kC * D * 2;
    // Tokens of an entry of V terms (the MMA warp waits and commits once per entry); two entries in tensor memory, a column to two tokens
    // of each of the three terms, where S^T, scores and O leave room.
    static constexpr int kEntry = D == 64 ? 64 : 32;
    static constexpr int kEntries = kC / kEntry;                // of a chunk
    static __host__ __device__ constexpr uint32_t term_col(int place, int term)
    {
        return D == 64 ? (place == 0 ? 384 + 32 * term : term == 0 ? 480 : 32 + 32 * term) : 384 + 64 * place + 16 * term;
    }
    static constexpr uint32_t kHalf = kC * 128;                 // 64 columns of a tile
    static constexpr uint32_t kState = D * D * 2;               // one bf16 term of S^T
    static constexpr uint32_t off_state = kSlots * kTile;
    static constexpr uint32_t off_table = off_state + (kStates ? 0 : 2 * kState);
    static constexpr uint32_t off_bad = off_table + (kC + 32 + kC) * 4;    // first token with a non-finite v, by column
    static constexpr uint32_t off_bar = off_bad + D * 4;
    static constexpr uint32_t kBytes = off_bar + 288 + 1024;    // and room to start on a 1024-byte boundary
};

struct Bars {
    uint64_t full[9], empty[9];                     // tiles: load -> users, last user -> load
    uint64_t sc_full, p_full, qs_done;              // scores ready; P ready and Q S scaled; Q S in the accumulator
    uint64_t s_full, kv_done, d_free;               // state terms ready; a chunk's addition to the state complete; read
    uint64_t vt_full[2], vt_empty[2];               // V terms
    uint64_t o_full, o_empty, o_staged;             // O complete; O read; rows staged
    uint64_t fixed;                                 // rows past the end zeroed
    uint32_t tmem_slot;
    int dead;
    int any_bad;                                    // some column has a non-finite v
};
static_assert(sizeof(Bars) <= 288, "barriers");

struct ChunkPlan {
    int64_t seg_len;        // tokens of a segment, a multiple of kC
    int segments;           // of the longest sequence
    float* local;           // [B][H][segments][D][D]: the state before the first segment, then what each but the last adds to it
};

constexpr uint32_t kTries = 1u << 22;       // of a wait before it gives up

// l^n from log2 l; n = 0 gives 1 for every l (log2 l may be -inf).
__device__ __forceinline__ float decay_pow(float g2, float n) { return n == 0.f ? 1.f : exp2f(n * g2); }

__device__ __forceinline__ float bf16_low(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_high(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

__device__ __forceinline__ void tma_load_tile(uint32_t dst, const CUtensorMap* map, int c, int head, int token, uint64_t* bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c), "r"(head), "r"(token), "r"(tc::smem_addr(bar)) : "memory");
}

__device__ __forceinline__ void tma_store_tile(const CUtensorMap* map, uint32_t src, int c, int head, int token)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c), "r"(head), "r"(token), "r"(src) : "memory");
}

// The pair rounded to bf16 (packed low / high) and what is left of it.
__device__ __forceinline__ pair_t split_term(pair_t y, uint32_t& term)
{
    float a, b;
    take_pair(y, a, b);
    term = pack2<__nv_bfloat16>(a, b);
    return fma_pair(make_pair(bf16_low(term), bf16_high(term)), make_pair(-1.f, -1.f), y);
}
__device__ __forceinline__ uint32_t round_pair(pair_t y)
{
    float a, b;
    take_pair(y, a, b);
    return pack2<__nv_bfloat16>(a, b);
}
// Two bf16 terms of each (16 bits), three (24 bits).
__device__ __forceinline__ void split2(pair_t y, uint32_t& hi, uint32_t& lo) { lo = round_pair(split_term(y, hi)); }
__device__ __forceinline__ void split3(pair_t y, uint32_t& hi, uint32_t& mid, uint32_t& lo)
{
    lo = round_pair(split_term(split_term(y, hi), mid));
}
__device__ __forceinline__ float value(const uint8_t* p) { return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16); }
__device__ __forceinline__ pair_t as_pair(uint32_t a, uint32_t b) { return make_pair(__uint_as_float(a), __uint_as_float(b)); }

template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

template <int D, bool kStates>
__global__ void __launch_bounds__(kThreads, 1)
decay_chunk_kernel(const DecayArgs g, const ChunkPlan p, const __grid_constant__ CUtensorMap map_q,
                   const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const __grid_constant__ CUtensorMap map_o)
{
    using L = Layout<D, kStates>;
    extern __shared__ uint8_t smem_raw[];
    // (an offset, not a rounded address: through an integer the compiler loses that it is shared memory, and every access becomes generic)
    uint8_t* smem = smem_raw + ((1024u - (tc::smem_addr(smem_raw) & 1023u)) & 1023u);
    float* table = reinterpret_cast<float*>(smem + L::off_table);            // l^(C-1-j), then 32 zeros, then the last chunk's
    int* bad_from = reinterpret_cast<int*>(smem + L::off_bad);
    Bars& bar = *reinterpret_cast<Bars*>(smem + L::off_bar);
    // the warp's number by a shuffle: the branches on it are then known to be uniform, and what the MMA warp computes for its
    // instructions stays in uniform registers
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, quad = warp & 3;

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
    RTN_TL_INIT(decay_chunk)
    if (threadIdx.x == 0) RTN_TL(decay_chunk, 0);
    if (warp == kWarpMma) tc::tmem_alloc(&bar.tmem_slot, kTmemCols);
    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kSlots; ++i) { tc::mbar_init(&bar.full[i], 1); tc::mbar_init(&bar.empty[i], 1); }
        tc::mbar_init(&bar.sc_full, 1); tc::mbar_init(&bar.p_full, 256); tc::mbar_init(&bar.qs_done, 1);
        tc::mbar_init(&bar.s_full, 2 * D); tc::mbar_init(&bar.kv_done, 1); tc::mbar_init(&bar.d_free, 2 * D);
        for (int i = 0; i < 2; ++i) { tc::mbar_init(&bar.vt_full[i], D); tc::mbar_init(&bar.vt_empty[i], 1); }
        tc::mbar_init(&bar.o_full, 1); tc::mbar_init(&bar.o_empty, 256); tc::mbar_init(&bar.o_staged, 256); tc::mbar_init(&bar.fixed, 2 * D);
        tc::mbar_init_fence();
        bar.dead = bar.any_bad = 0;
    }
    if (threadIdx.x < D) bad_from[threadIdx.x] = 0x7fffffff;
    if (threadIdx.x < kC) table[kC - 1 - threadIdx.x] = decay_pow(g2, (float)threadIdx.x);
    else if (threadIdx.x < kC + 32) table[threadIdx.x] = 0.f;
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    constexpr uint32_t tmem = 0;                // all 512 columns are this CTA's: they begin at 0
    if (bar.tmem_slot != tmem && threadIdx.x == 0) bar.dead = 1;
    if (threadIdx.x == 0) RTN_TL(decay_chunk, 1);
    const uint32_t base = tc::smem_addr(smem);
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    volatile int *dead = &bar.dead, *any_bad = &bar.any_bad;
    // Bounded waits: one that runs out marks the CTA, which reports it at its end.  Whole warps wait together and give up together
    // (what follows is warp-collective).
    auto wait = [&](uint64_t* m, int phase) {
        const bool ok = tc::mbar_wait_tries(m, (uint32_t)phase & 1u, kTries);
        if (!ok) *dead = 1;
        return ok;
    };
    auto warp_wait = [&](uint64_t* m, int phase) {
        const bool ok = __all_sync(0xffffffffu, tc::mbar_wait_tries(m, (uint32_t)phase & 1u, kTries)) != 0;
        if (!ok) *dead = 1;
        return ok;
    };
    // rings: Q, then K, then V slots
    enum { kTileQ, kTileK, kTileV };
    auto slots_of = [](int which) { return which == kTileQ ? L::kSlotsQ : which == kTileK ? L::kSlotsK : L::kSlotsV; };
    auto tile_slot = [&](int c, int which) {
        return (which == kTileQ ? 0 : which == kTileK ? L::kSlotsQ : L::kSlotsQ + L::kSlotsK) + c % slots_of(which);
    };
    auto tile_phase = [&](int c, int which) { return c / slots_of(which); };

    if (warp < kWarpS) {
      regs_down<kRegsRest>();
      if (warp == kWarpLoadK && lane == 1) {
        // ------------------------------------------------------------ rows out (one thread)
        if constexpr (!kStates) {
            const int stores = tail == kC ? chunks : chunks - 1;              // the last rows of a sequence are stored by their threads
            for (int c = 0; c < stores; ++c) {
                const int sk = tile_slot(c, kTileK);
                if (!wait(&bar.o_staged, c)) break;
                for (int x = 0; x < D / 64; ++x) tma_store_tile(&map_o, base + sk * L::kTile + x * L::kHalf, x * 64, h, (int)row0 + c * kC);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                tc::mbar_arrive(&bar.empty[sk]);
            }
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        }
      } else if (warp != kWarpMma) {
        // ------------------------------------------------------------ tiles (one thread per ring)
        const int which = warp == kWarpLoadQ ? kTileQ : warp == kWarpLoadK ? kTileK : kTileV;
        if (lane == 0 && !(kStates && which == kTileQ)) {
            const CUtensorMap* map = which == kTileK ? &map_k : which == kTileV ? &map_v : &map_q;
            int c = 0;
            for (; c < chunks; ++c) {
                const int s = tile_slot(c, which);
                if (!wait(&bar.empty[s], tile_phase(c, which) + 1)) break;
                tc::mbar_arrive_expect_tx(&bar.full[s], L::kTile);
                for (int half = 0; half < D / 64; ++half)
                    tma_load_tile(base + s * L::kTile + half * L::kHalf, map, half * 64, which == kTileQ ? h : hk,
                                  (int)row0 + c * kC, &bar.full[s]);
            }
            // every copy has landed before the CTA ends, also when a wait gave up
            for (int u = c > slots_of(which) ? c - slots_of(which) : 0; u < c; ++u)
                tc::mbar_wait(&bar.full[tile_slot(u, which)], (uint32_t)tile_phase(u, which) & 1u, g.status);
        }
      } else {
        // ------------------------------------------------------------ every MMA
        {
            const uint32_t elected = tc::elect_one();
            auto commit = [&](uint64_t* m) { if (elected) tc::mma_commit(m); __syncwarp(); };
            constexpr uint32_t id_kk = tc::idesc_bf16(128, kC, false);           // scores
            constexpr uint32_t id_s = tc::idesc_bf16(128, D, false), id_mn = tc::idesc_bf16(128, D, true);
            // descriptors: a tile's own, and constant steps along k on top (addresses count 16 bytes, and stay below 2^14)
            auto tile_desc = [&](int slot_) { return tc::smem_desc_sw128(base + (uint32_t)slot_ * L::kTile, L::kHalf); };
            auto kmajor = [](uint64_t desc, uint32_t half_bytes, int step) {
                return desc + (((uint32_t)(step >> 2) * half_bytes + (uint32_t)(step & 3) * 32u) >> 4);
            };
            auto mnmajor = [](uint64_t desc, int step) { return desc + (((uint32_t)step * 2048u) >> 4); };
            const uint64_t state_desc = tc::smem_desc_sw128(base + L::off_state, 16);
            auto scores = [&](int c) {
                const int sk = tile_slot(c, kTileK), sq = tile_slot(c, kTileQ);
                if (!warp_wait(&bar.full[sk], tile_phase(c, kTileK)) || !warp_wait(&bar.full[sq], tile_phase(c, kTileQ))) return false;
                tc::tc_fence_after_sync();
                const uint64_t dq = tile_desc(sq), dk = tile_desc(sk);
                #pragma unroll
                for (int s = 0; s < D / 16; ++s)
                    tc::mma_f16_ss(elected, tmem + kColP, kmajor(dq, L::kHalf, s), kmajor(dk, L::kHalf, s), id_kk, s > 0);
                commit(&bar.sc_full);
                return true;
            };
            bool alive = true;
            if constexpr (!kStates) alive = chunks == 0 || scores(0);
            for (int c = 0; c < chunks && alive; ++c) {
                const int sk = tile_slot(c, kTileK), sq = kStates ? 0 : tile_slot(c, kTileQ), sv = tile_slot(c, kTileV);
                const uint64_t dq = tile_desc(sq), dk = tile_desc(sk), dv = tile_desc(sv);
                if constexpr (kStates) { if (!(alive = warp_wait(&bar.full[sk], tile_phase(c, kTileK)))) break; }
                if (c > 0 && !(alive = warp_wait(&bar.d_free, c - 1))) break;
                // the last chunk's rows past the end are zero before a product reads them
                if (c == chunks - 1 && tail < kC && !(alive = warp_wait(&bar.fixed, 0))) break;
                CHUNK_TL(0);
                // state update by entries; Q S between the second and the third: its own terms may come late, and the V warps
                // are two entries ahead at most
                #pragma unroll 1
                for (int e = 0; e < L::kEntries && alive; ++e) {
                    if constexpr (!kStates) {
                        if (e == L::kEntries / 2) {
                            alive = warp_wait(&bar.s_full, c) && (c == 0 || warp_wait(&bar.o_empty, c - 1));
                            if (!alive) break;
                            tc::tc_fence_after_sync();
                            CHUNK_TL(1);
                            #pragma unroll 1
                            for (int term = 0; term < 2; ++term)
                                #pragma unroll
                                for (int s = 0; s < D / 16; ++s)
                                    tc::mma_f16_ss(elected, tmem + kColO, kmajor(dq, L::kHalf, s),
                                                   kmajor(state_desc + (term * L::kState >> 4), D * 128, s), id_s, term + s > 0);
                            commit(&bar.qs_done);
                            CHUNK_TL(2);
                        }
                    }
                    const int ve = c * L::kEntries + e;
                    if (!(alive = warp_wait(&bar.vt_full[ve & 1], ve >> 1))) break;
                    tc::tc_fence_after_sync();
                    #pragma unroll
                    for (int term = 0; term < 3; ++term)
                        #pragma unroll
                        for (int s = 0; s < L::kEntry / 16; ++s)
                            tc::mma_f16_ts(elected, tmem + kColS, tmem + ((e & 1) ? L::term_col(1, term) : L::term_col(0, term)) + (uint32_t)(s * 8),
                                           mnmajor(dk, e * (L::kEntry / 16) + s), id_mn, e + term + s > 0);
                    commit(&bar.vt_empty[ve & 1]);
                }
                if (!alive) break;
                CHUNK_TL(3);
                commit(&bar.kv_done);
                if constexpr (!kStates) {
                    if (!(alive = warp_wait(&bar.p_full, c))) break;
                    CHUNK_TL(4);
                    tc::tc_fence_after_sync();
                    #pragma unroll 1
                    for (int term = 0; term < 2; ++term)
                        #pragma unroll
                        for (int s = 0; s < kC / 16; ++s)
                            tc::mma_f16_ts(elected, tmem + kColO, tmem + kColP + (uint32_t)(s * 16 + term * 8),
                                           mnmajor(dv, s), id_mn, true);
                    commit(&bar.o_full);
                    CHUNK_TL(5);
                }
                if constexpr (!kStates) {
                    if (c + 1 < chunks) alive = scores(c + 1);
                    CHUNK_TL(6);
                }
            }
        }
      }
    } else if (warp >= kWarpP && warp < kWarpV) {
        // ------------------------------------------------------------ P: row i of the chunk, every other 16 keys, per thread
        // (each of the two warps of 32 rows then has one of the two blocks on the diagonal, which take twice as long as the others)
        regs_down<kRegsP>();
        if constexpr (!kStates) {
            const int i = quad * 32 + lane, half = (warp >> 2) & 1;
            pair_t near[8];                                                   // l^(15 - x), by pairs
            #pragma unroll
            for (int x = 0; x < 8; ++x) near[x] = make_pair(table[kC - 16 + 2 * x], table[kC - 15 + 2 * x]);
            const float own = decay_pow(g2, (float)(i + 1));
            for (int c = 0; c < chunks; ++c) {
                if (!warp_wait(&bar.sc_full, c)) break;
                if (threadIdx.x == (kWarpP + 3) * 32) CHUNK_TL(7);
                tc::tc_fence_after_sync();
                #pragma unroll 1
                for (int kb = half; kb < 8; kb += 2) {                        // 16 keys: eight words of high terms, eight of low
                    const uint32_t at = tmem + lanes + kColP + (uint32_t)(kb * 16);
                    const float* w = table + (kC - 1 - i + kb * 16);          // l^(i - key), zero past the diagonal
                    uint32_t t[16];
                    if (kb * 16 >= quad * 32 + 32) {                          // keys after every row of the warp
                        #pragma unroll
                        for (int x = 0; x < 16; ++x) t[x] = 0;
                    } else {
                        uint32_t v[16];
                        tc::tmem_ld16(at, v);
                        if (kb * 16 + 16 <= quad * 32) {                      // keys before every row of the warp
                            const pair_t f = make_pair(w[15], w[15]);
                            tc::tmem_ld_wait();
                            #pragma unroll
                            for (int x = 0; x < 16; x += 2)
                                split2(mul_pair(as_pair(v[x], v[x + 1]), mul_pair(f, near[x >> 1])), t[x >> 1], t[8 + (x >> 1)]);
                        } else {                                              // masked by selection: scores there may be anything
                            const int n = i - kb * 16;
                            tc::tmem_ld_wait();
                            #pragma unroll
                            for (int x = 0; x < 16; x += 2) {
                                const float y0 = x > n ? 0.f : __uint_as_float(v[x]), y1 = x + 1 > n ? 0.f : __uint_as_float(v[x + 1]);
                                split2(mul_pair(make_pair(y0, y1), make_pair(w[x], w[x + 1])), t[x >> 1], t[8 + (x >> 1)]);
                            }
                        }
                    }
                    tc::tmem_st16(at, t);
                }
                tc::tmem_st_wait();
                if (threadIdx.x == (kWarpP + 3) * 32) CHUNK_TL(8);
                if (!warp_wait(&bar.qs_done, c)) break;
                if (threadIdx.x == kWarpP * 32) tc::mbar_arrive(&bar.empty[tile_slot(c, kTileQ)]);       // Q S was the tile's last use
                if (threadIdx.x == (kWarpP + 3) * 32) CHUNK_TL(9);
                __syncwarp();
                tc::tc_fence_after_sync();
                #pragma unroll 1
                for (int x0 = half * (D / 2); x0 < (half + 1) * (D / 2); x0 += 16) {
                    uint32_t v[16];
                    tc::tmem_ld16(tmem + lanes + kColO + (uint32_t)x0, v);
                    tc::tmem_ld_wait();
                    #pragma unroll
                    for (int x = 0; x < 16; x += 2) {
                        float a, b2;
                        take_pair(mul_pair(as_pair(v[x], v[x + 1]), make_pair(own, own)), a, b2);
                        v[x] = __float_as_uint(a); v[x + 1] = __float_as_uint(b2);
                    }
                    tc::tmem_st16(tmem + lanes + kColO + (uint32_t)x0, v);
                }
                tc::tmem_st_wait();
                tc::tc_fence_before_sync();
                tc::mbar_arrive(&bar.p_full);
                if (threadIdx.x == (kWarpP + 3) * 32) CHUNK_TL(10);

                // the chunk's rows
                if (!warp_wait(&bar.o_full, c)) break;
                if (threadIdx.x == (kWarpP + 3) * 32) CHUNK_TL(15);
                tc::tc_fence_after_sync();
                if (threadIdx.x == kWarpP * 32) tc::mbar_arrive(&bar.empty[tile_slot(c, kTileV)]);       // P V was the V tile's last use
                __syncwarp();
                const bool whole = c < chunks - 1 || tail == kC;              // a store of 128 rows stays inside the sequence
                uint8_t* row = smem + tile_slot(c, kTileK) * L::kTile + i * 128;        // the state update has read the slot's K tile
                __nv_bfloat16* orow = out + (int64_t)(c * kC + i) * g.o_token;
                const bool mine = c * kC + i < n_tok;
                #pragma unroll 1
                for (int x0 = half * (D / 2); x0 < (half + 1) * (D / 2); x0 += 16) {
                    uint32_t v[16];
                    tc::tmem_ld16(tmem + lanes + kColO + (uint32_t)x0, v);
                    tc::tmem_ld_wait();
                    uint8_t* dst = row + (x0 >> 6) * L::kHalf;
                    #pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        uint32_t w[4];
                        #pragma unroll
                        for (int x = 0; x < 4; ++x)
                            w[x] = round_pair(mul_pair(as_pair(v[y * 8 + 2 * x], v[y * 8 + 2 * x + 1]), make_pair(g.scale, g.scale)));
                        const uint4 u = make_uint4(w[0], w[1], w[2], w[3]);
                        if (whole) *reinterpret_cast<uint4*>(dst + (((((x0 & 63) >> 3) + y) ^ (i & 7)) << 4)) = u;
                        else if (mine) *reinterpret_cast<uint4*>(orow + x0 + y * 8) = u;
                    }
                }
                if (*any_bad) {
                    #pragma unroll 1
                    for (int x = half * (D / 2); x < (half + 1) * (D / 2); ++x)
                        if (c * kC + i >= bad_from[x]) {
                            if (whole) *reinterpret_cast<uint16_t*>(row + (x >> 6) * L::kHalf + ((((x & 63) >> 3) ^ (i & 7)) << 4) + (x & 7) * 2) = 0x7fff;
                            else if (mine) orow[x] = __ushort_as_bfloat16(0x7fff);
                        }
                }
                tc::tc_fence_before_sync();
                tc::mbar_arrive(&bar.o_empty);
                if (threadIdx.x == (kWarpP + 3) * 32) CHUNK_TL(16);
                if (whole) {
                    tc::fence_smem_to_async_proxy();
                    tc::mbar_arrive(&bar.o_staged);
                }
            }
        }
    } else if (warp >= kWarpS && warp < kWarpP) {
        // ------------------------------------------------------------ S: row d of S^T, half of its columns, per thread
        regs_up<kRegsS>();
        const int d = quad * 32 + lane, half = (warp >> 2) & 1;
        if (d < D) {
            constexpr int N = D / 2;
            const int r0 = half * N;
            const int64_t at = ((slot * g.H + h) * (int64_t)D + r0) * D + d;
            pair_t S[N / 2];                                // S^T row d, columns r0 .. r0 + N - 1
            float* local = p.local + ((b * g.H + h) * (int64_t)p.segments * D + r0) * D + d;
            {
                float v[N];
                if constexpr (kStates) {
                    // The last segment's CTA writes state_out, which may be the state itself, while other segments may not have begun:
                    // they take the given state from here.
                    if (seg == 0 && g.state != nullptr) {
                        #pragma unroll
                        for (int x = 0; x < N; ++x) v[x] = g.state[at + (int64_t)x * D];
                        #pragma unroll
                        for (int x = 0; x < N; ++x) local[(int64_t)x * D] = v[x];
                    }
                    #pragma unroll
                    for (int x = 0; x < N; ++x) v[x] = 0.f;
                } else {
                    // the given state (a sequence of one segment: read and written by this CTA alone), and what the segments before added
                    const float w0 = decay_pow(g2, (float)s0);
                    const float* given = seg == 0 && last_seg ? g.state + at : local;
                    const bool any = g.state != nullptr;        // (also where w0 is 0: a non-finite state stays one)
                    #pragma unroll
                    for (int x = 0; x < N; ++x) v[x] = any ? w0 * given[(int64_t)x * D] : 0.f;
                    for (int s = 0; s < seg; ++s) {
                        const float w = decay_pow(g2, (float)((int64_t)(seg - 1 - s) * p.seg_len));
                        #pragma unroll
                        for (int x = 0; x < N; ++x) v[x] = fmaf(w, local[((int64_t)(s + 1) * D + x) * D], v[x]);
                    }
                }
                #pragma unroll
                for (int x = 0; x < N; x += 2) S[x >> 1] = make_pair(v[x], v[x + 1]);
                __syncwarp();
            }
            const float keep = decay_pow(g2, (float)kC);
            const uint32_t col = tmem + lanes + kColS + (uint32_t)r0;
            auto add = [&](float l) {                       // S <- l S + the chunk's part
                #pragma unroll
                for (int x0 = 0; x0 < N; x0 += 32) {
                    uint32_t u[2][16];
                    tc::tmem_ld16(col + (uint32_t)x0, u[0]);
                    tc::tmem_ld16(col + (uint32_t)(x0 + 16), u[1]);
                    tc::tmem_ld_wait();
                    #pragma unroll
                    for (int x = 0; x < 32; x += 2)
                        S[(x0 + x) >> 1] = fma_pair(make_pair(l, l), S[(x0 + x) >> 1], as_pair(u[x >> 4][x & 15], u[x >> 4][(x & 15) + 1]));
                }
                tc::tc_fence_before_sync();
            };
            bool alive = true;
            for (int c = 0; c < chunks; ++c) {
                if (c > 0) {
                    if (!(alive = warp_wait(&bar.kv_done, c - 1))) break;
                    if constexpr (kStates) {                                  // the update was both tiles' last use
                        if (threadIdx.x == kWarpS * 32) {
                            tc::mbar_arrive(&bar.empty[tile_slot(c - 1, kTileK)]);
                            tc::mbar_arrive(&bar.empty[tile_slot(c - 1, kTileV)]);
                        }
                        __syncwarp();
                    }
                    if (threadIdx.x == (kWarpS + (D / 32 - 1)) * 32) CHUNK_TL(11);
                    tc::tc_fence_after_sync();
                    add(keep);
                    tc::mbar_arrive(&bar.d_free);
                }
                if constexpr (!kStates) {
                    if (c > 0 && !(alive = warp_wait(&bar.qs_done, c - 1))) break;      // the terms of the chunk before have been read
                    uint8_t* terms = smem + L::off_state + d * 128;
                    #pragma unroll
                    for (int x = 0; x < N; x += 8) {
                        uint32_t hi[4], lo[4];
                        #pragma unroll
                        for (int y = 0; y < 4; ++y) split2(S[(x >> 1) + y], hi[y], lo[y]);
                        const int r = r0 + x;
                        const uint32_t o = (uint32_t)(r >> 6) * (D * 128) + ((uint32_t)(((r & 63) >> 3) ^ (d & 7)) << 4);
                        *reinterpret_cast<uint4*>(terms + o) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                        *reinterpret_cast<uint4*>(terms + L::kState + o) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                    }
                    tc::fence_smem_to_async_proxy();
                    tc::mbar_arrive(&bar.s_full);
                    if (threadIdx.x == (kWarpS + (D / 32 - 1)) * 32) CHUNK_TL(12);
                }
            }
            // the state after the segment
            if ((kStates || last_seg) && alive && (chunks == 0 || warp_wait(&bar.kv_done, chunks - 1))) {
                tc::tc_fence_after_sync();
                if (chunks > 0) add(decay_pow(g2, (float)tail));
                float* dst = kStates ? local + (int64_t)(seg + 1) * D * D : g.state_out + at;
                #pragma unroll
                for (int x = 0; x < N; x += 2) {
                    float a, b2;
                    take_pair(S[x >> 1], a, b2);
                    dst[(int64_t)x * D] = a; dst[(int64_t)(x + 1) * D] = b2;
                }
            }
        }
    } else {
        // ------------------------------------------------------------ V: column d of the V tile, every other entry, per thread
        const int d = quad * 32 + lane, half = (warp >> 2) & 1;
        if (d < D) {
            uint32_t v_at[8];                               // where column d of token row j lies, for j & 7 (1024 bytes to the next 8)
            #pragma unroll
            for (int j = 0; j < 8; ++j)
                v_at[j] = (uint32_t)(d >> 6) * L::kHalf + (uint32_t)(d & 7) * 2u + (uint32_t)j * 128u + ((uint32_t)(((d & 63) >> 3) ^ j) << 4);
            const uint32_t col_hi = tmem + lanes + (half ? L::term_col(1, 0) : L::term_col(0, 0));
            const uint32_t col_mid = tmem + lanes + (half ? L::term_col(1, 1) : L::term_col(0, 1));
            const uint32_t col_lo = tmem + lanes + (half ? L::term_col(1, 2) : L::term_col(0, 2));
            for (int c = 0; c < chunks; ++c) {
                const int sv = tile_slot(c, kTileV);
                if (!warp_wait(&bar.full[sv], tile_phase(c, kTileV))) break;
                if (threadIdx.x == (kWarpV + (D / 32 - 1)) * 32) CHUNK_TL(13);
                const int n = c == chunks - 1 ? tail : kC;
                uint8_t* tile = smem + sv * L::kTile;
                if (n < kC) {
                    const int sk = tile_slot(c, kTileK);
                    if (!warp_wait(&bar.full[sk], tile_phase(c, kTileK))) break;
                    // 16-byte pieces of the rows n .. C-1 of both tiles (every 64 columns)
                    const int pieces = (kC - n) * 8;
                    for (int x = half * D + d; x < pieces * (D / 64); x += 2 * D) {
                        const uint32_t o = (uint32_t)(x / pieces) * L::kHalf + (uint32_t)n * 128u + (uint32_t)(x % pieces) * 16u;
                        *reinterpret_cast<uint4*>(tile + o) = make_uint4(0, 0, 0, 0);
                        *reinterpret_cast<uint4*>(smem + sk * L::kTile + o) = make_uint4(0, 0, 0, 0);
                    }
                    for (int j = half * D + d; j < kC; j += 2 * D) table[kC + 32 + j] = j < n ? table[j + kC - n] : 0.f;
                    tc::fence_smem_to_async_proxy();
                    tc::mbar_arrive(&bar.fixed);
                    if (!warp_wait(&bar.fixed, 0)) break;
                }
                const float* weight = n < kC ? table + kC + 32 : table;       // l^(n - 1 - j)
                bool alive = true;
                #pragma unroll 1
                for (int e = half; e < L::kEntries; e += 2) {
                    uint32_t seen = 0;                  // every low term: NaN where a value is not finite, under 2 where it is under 2^17
                    #pragma unroll 2                    // (two register sets: a store to tensor memory is slow to let go of its own)
                    for (int sub = 0; sub < L::kEntry / 16; ++sub) {
                        uint32_t hi[8], mid[8], lo[8];
                        const int j0 = e * L::kEntry + sub * 16;
                        const uint8_t* rows = tile + j0 * 128;
                        float v[16];
                        #pragma unroll
                        for (int x = 0; x < 16; ++x) v[x] = value(rows + v_at[x & 7] + (x >> 3) * 1024);
                        #pragma unroll
                        for (int x = 0; x < 16; x += 4) {
                            const float4 w = *reinterpret_cast<const float4*>(weight + j0 + x);
                            const int k = x >> 1;
                            split3(mul_pair(make_pair(v[x], v[x + 1]), make_pair(w.x, w.y)), hi[k], mid[k], lo[k]);
                            split3(mul_pair(make_pair(v[x + 2], v[x + 3]), make_pair(w.z, w.w)), hi[k + 1], mid[k + 1], lo[k + 1]);
                        }
                        if constexpr (!kStates) {
                            #pragma unroll
                            for (int x = 0; x < 8; ++x) seen |= lo[x];
                        }
                        if (sub == 0) {
                            if (!(alive = warp_wait(&bar.vt_empty[half], ((c * L::kEntries + e) >> 1) + 1))) break;
                            tc::tc_fence_after_sync();
                        }
                        tc::tmem_st8(col_hi + (uint32_t)(sub * 8), hi);
                        tc::tmem_st8(col_mid + (uint32_t)(sub * 8), mid);
                        tc::tmem_st8(col_lo + (uint32_t)(sub * 8), lo);
                    }
                    if (!alive) break;
                    if (!kStates && (seen & 0x40004000u)) {
                        #pragma unroll 1
                        for (int j = e * L::kEntry; j < (e + 1) * L::kEntry; ++j) {
                            uint16_t* x = reinterpret_cast<uint16_t*>(tile + j * 128 + (d >> 6) * L::kHalf + ((((d & 63) >> 3) ^ (j & 7)) << 4) + (d & 7) * 2);
                            if ((*x & 0x7f80) != 0x7f80) continue;
                            *x = 0;
                            atomicMin(&bad_from[d], c * kC + j);
                            *any_bad = 1;
                        }
                        tc::fence_smem_to_async_proxy();
                    }
                    __syncwarp();
                    tc::tmem_st_wait();
                    tc::tc_fence_before_sync();
                    tc::mbar_arrive(&bar.vt_full[half]);
                }
                if (!alive) break;
                if (threadIdx.x == (kWarpV + (D / 32 - 1)) * 32) CHUNK_TL(14);
            }
        }
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    if (warp == kWarpMma) tc::tmem_dealloc(tmem, kTmemCols);
    if (threadIdx.x == 0 && *dead) atomicOr(g.status, kStatusWaitTimeout);
    if (threadIdx.x == 0) RTN_TL(decay_chunk, 4);
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
    // Times in chunks of the main pass: a segment's chunks in both passes (0.4 in the first), four for another launch, and a sixth for each
    // segment's part that the last one adds up.  16 heads of 128: 512 tokens 21 us in one segment, 28 in two; 1024 tokens 34 in one, 31 in
    // four; 2048 tokens 58 in one, 42 in four, 36 in eight.
    int64_t segs = 1;
    double best = (double)chunks;
    for (int64_t n = 2; n * ctas <= sms && 2 * n <= chunks; ++n) {
        const double cost = 1.4 * (double)((chunks + n - 1) / n) + 4.0 + (double)n / 6.0;
        if (cost < best) { best = cost; segs = n; }
    }
    p.seg_len = (chunks + segs - 1) / segs * kC;
    if (p.seg_len < kC) p.seg_len = kC;
    p.segments = (int)((chunks * kC + p.seg_len - 1) / p.seg_len);
    if (p.segments < 1) p.segments = 1;
    return p;
}

template <int D>
cudaError_t launch_typed(const DecayArgs& g, cudaStream_t s, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v,
                         const CUtensorMap& o)
{
    constexpr int bytes = (int)Layout<D, false>::kBytes, bytes_states = (int)Layout<D, true>::kBytes;
    ChunkPlan p = make_plan(g);
    cudaError_t e = allow_shared_memory(decay_chunk_kernel<D, false>);
    if (e != cudaSuccess) return e;
    void* scratch = nullptr;
    if (p.segments > 1) {
        e = allow_shared_memory(decay_chunk_kernel<D, true>);
        if (e != cudaSuccess) return e;
        e = scratch_alloc(&scratch, (size_t)g.B * g.H * p.segments * D * D * sizeof(float), s);
        if (e != cudaSuccess) return e;
        p.local = static_cast<float*>(scratch);
        decay_chunk_kernel<D, true><<<(unsigned)(g.B * g.H * (p.segments - 1)), kThreads, bytes_states, s>>>(g, p, q, k, v, o);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) {
        decay_chunk_kernel<D, false><<<(unsigned)(g.B * g.H * p.segments), kThreads, bytes, s>>>(g, p, q, k, v, o);
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
    CUtensorMap q, k, v, o;
    taken = encode_heads(&q, g.q, g.total, g.H, g.Dk, g.q_token, g.q_head) && encode_heads(&k, g.k, g.total, g.Hk, g.Dk, g.k_token, g.k_head) &&
            encode_heads(&v, g.v, g.total, g.Hk, g.Dv, g.v_token, g.v_head) && encode_heads(&o, g.out, g.total, g.H, g.Dv, g.o_token, g.o_head);
    if (!taken) return cudaSuccess;
    return g.Dk == 64 ? launch_typed<64>(g, s, q, k, v, o) : launch_typed<128>(g, s, q, k, v, o);
}

}  // namespace rtn
