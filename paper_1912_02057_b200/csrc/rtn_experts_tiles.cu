// The experts' ternary products on the tensor cores: codes as 4-bit floating point.
//
// A product of codes is -1, 0 or 1, and so is one of e2m1 values of reciprocal magnitudes; with every block scale 1 the fp32 accumulators hold
// S = sum_k x_k w_k exactly (|S| <= K <= 2^24).  kind::mxf4 runs at four times the bf16 rate (8.8 PFLOP/s measured; int8 twice).
//   y = w_s (a_s S) + w_o a_s S_x + (w_s S_w + K w_o) a_o + bias, then act, gate, codes, all in the epilogue.
// A tile: 128 weight rows (gated: 64 outputs' two rows each) times 16 .. 160 rows of one expert.  The weights are the operand of 128 rows, out of tensor
// memory: planes come by TMA, warps expand them in registers straight into it (no shared memory in between, whose bandwidth both operands
// would share), and a product of 32 inputs runs at the full rate (of 16 at two thirds).  Inputs are expanded once, ahead, into the experts' order
// (K / 2 bytes a row of scratch): a row meets every column tile.  A persistent CTA per SM; two accumulators, so that a tile's outputs are written during the
// next one's products; parameters are fetched two tiles ahead by warps of their own, which also put a token's codes together from the votes.
// Codes are those of the exact output: a value nearer to a threshold than its error bound is worked out again in double, of 16 tokens at a time.  One that equals
// it always is: an upper threshold of 0 behind a ReLU, or one of 0 behind a gated one, whose outputs are 0 half of the time, sends nearly everything there (65536
// rows, 64 experts of 2048 x 2048, gated ReLU 1800 us in place of 273, of 2048 x 1024, ReLU 1440 in place of 208), and so do a last tile's padding columns
// (zeros) with a threshold of 0, though not on to double.
// Bound: for long prompts the instructions of the epilogue (50 to 65 per output) and of the expansion (some 200 per 32 rows x 256 codes), the tensor
// pipe idles three quarters of the time; for few rows of an expert its start (2.6 us) and the first planes' way (2.6 us).
// Measured (one B200, in a graph): 65536 rows, 64 experts of 2048 x 2048, gated, codes 242 us (2.3 PFLOP/s; the matrix instructions alone 63); of 2048 x 1024,
// bf16 values 133 us (268 MB written); 384 rows, 64 experts of 2048 x 2048, gated, codes 22.4 us (67 MB of planes at 3.0 TB/s).
#include "rtn_experts.cuh"
#include "rtn_tcgen05.cuh"
#include "rtn_tensormap.cuh"

#include <float.h>

namespace rtn {

namespace {

// Warps: two groups of four expand weights, two write out (a warp of each for every quarter of the lanes), the fifth copies and issues the products, the
// sixth has what a tile begins and ends with.  Registers a thread by group; what they add up to is what the block is launched with.
constexpr int kExpandWarps = 8, kEpilogueWarps = 8, kEdgeWarps = 4;
constexpr int kLoadWarp = kExpandWarps + kEpilogueWarps, kPlanesWarp = kLoadWarp + 1, kMmaWarp = kLoadWarp + 2, kEdgeWarp = kLoadWarp + 4;
constexpr int kThreads = (kEdgeWarp + kEdgeWarps) * 32;
constexpr int kLaunchRegs = 80, kExpandRegs = 80, kEpilogueRegs = 104, kIssueRegs = 40, kEdgeRegs = 72;
static_assert(kThreads == 768 && 2 * kExpandRegs + 2 * kEpilogueRegs + kIssueRegs + kEdgeRegs <= 6 * kLaunchRegs, "registers");
template <int kRegs> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs)); }
template <int kRegs> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs)); }
// A slot holds a span of K, 512 codes (or the last 256): two 128-byte rows of 4-bit values to an input, 64 columns of tensor memory to a weight row.
// (Slots of 256 codes: twice the barriers, which a small tile's time is made of.)
constexpr int kMaxRows = 160;                                   // of a tile (with what tells them apart: make_plan)
constexpr int kMaxStages = 6, kMaxSpans = 8;                    // slots of the rings
constexpr uint32_t kSpanBytes = 128 * 128;                       // 512 codes of 128 weight rows, as planes
constexpr uint32_t kTries = 1u << 20;
constexpr uint32_t kSmemBytes = 227 * 1024;
constexpr uint32_t kScaleCols = 16;

struct TilesPlan {
    int max_rows;               // of a tile, a multiple of 16
    int stages, spans;          // slots of the two rings
    int col_tiles;
    int k_halves;               // 256 codes each
    int box_rows;               // of a copy
    uint32_t ring, planes;      // offsets of the rings in shared memory
    uint32_t half_bytes;        // of a slot: the inputs' rows of 256 codes
    uint32_t smem;
};

struct Bars {
    uint64_t full[kMaxStages], empty[kMaxStages], planes_full[kMaxSpans], planes_empty[kMaxSpans], acc_full[2], acc_empty[2], params_full[2], votes_full[2];
    uint32_t tmem_slot;
    int dead;
};

// What the epilogue of a tile needs (looking the tile up itself, it lost 700 of a tile's 4000 clocks): a_s, a_s S_x, a_o and input row (-1: out of range) of its tokens, w_s, w_o, p3 and bias of its weight rows by
// TMEM lane; the votes of each 16 tokens and quarter of the lanes.
struct Tile { int e, row, rows, height; };

struct TileParams {
    float as[kMaxRows], asx[kMaxRows], ao[kMaxRows];
    int token[kMaxRows];
    float4 col[128];
    uint4 most_asx, most_ao;                                    // the largest |a_s S_x| and |a_o|, in four parts, as bit patterns (a NaN is the largest)
    uint4 votes[4][kMaxRows / 4][2];
    Tile tile[kEdgeWarps];                                      // the same place four times: each edge warp writes and reads its own
};

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

// box_rows rows of a [rows][pitch bytes] tensor from row r on, 128 bytes of each from byte x on, under the 128-byte swizzle.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int r, uint64_t* bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(r), "r"(tc::smem_addr(bar)) : "memory");
}

// Order of a row's codes in K, the same for both operands: what lets four lanes that read a row's planes side by side (16 bytes of each plane
// to a lane) hold whole fragments of a store to tensor memory.  A span is four blocks of 128 codes, or the last two; it is expanded in stages of 32 words (256 codes).
// A lane q has 8 words w of a stage, and word w is at 8 (w / 2) + 2 q + w % 2.
//   four blocks: lane q has block q; words 0-3 and 4-7 of stage h come from the block's plane words 2 h and 2 h + 1
//   two blocks:  lane q has plane words 2 (q % 2) and the next of block q / 2
__host__ __device__ __forceinline__ int halves_of(int nblk) { return nblk / 4 * 2 + (nblk % 4 + 1) / 2; }

// The experts' rows one after the other as 4-bit values, `pitch` bytes each (a row's end is zeros); and the sums of their codes begin at 0.
__global__ void __launch_bounds__(256)
expand_inputs_kernel(const __grid_constant__ ExpertsArgs g, int nblk, int chunks, uint2* __restrict__ out)
{
    tc::pdl_wait();
    tc::pdl_trigger();                                          // (now that what the products read ahead of their own wait is there)
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    const uint32_t row = i / (uint32_t)chunks, c = i % (uint32_t)chunks;          // a chunk: 32 codes, four words
    if (row >= g.R || row < (uint32_t)g.start[0] || row >= (uint32_t)g.start[g.E]) return;
    if (c == 0 && g.out_sum != nullptr) g.out_sum[row] = 0;
    const int64_t m = g.tokens != nullptr ? g.tokens[row] : row;
    const int stage = (int)(c / 8), q = (int)(c % 4), part = (int)(c % 8) / 4;    // this lane's words 4 part .. 4 part + 3 of the stage
    const bool four = stage / 2 * 4 + 2 < nblk;
    const int block = stage / 2 * 4 + (four ? q : q / 2), word = four ? stage % 2 * 2 + part : q % 2 * 2 + part;
    uint32_t nz = 0, pos = 0;
    if (block < nblk && m >= 0 && m < g.T) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(g.a_packed) + (m * nblk + block) * 8 + word;
        nz = p[0]; pos = p[4];
    }
    const uint4 w = expand_input(nz, pos);
    uint2* to = out + ((int64_t)row * chunks + stage * 8) * 2 + part * 8 + q;
    to[0] = make_uint2(w.x, w.y);
    to[4] = make_uint2(w.z, w.w);
}

template <typename T, bool kGated, bool kCodes>
__global__ void __launch_bounds__(kThreads, 1)
experts_tiles_kernel(const __grid_constant__ ExpertsArgs g, const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap weight_map,
                     const __grid_constant__ TilesPlan p)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    Bars& bar = *reinterpret_cast<Bars*>(smem);
    TileParams* params = reinterpret_cast<TileParams*>(smem + 512);              // [2]
    int* before = reinterpret_cast<int*>(params + 2);                            // [E + 1] tiles before an expert's
    int* first = before + g.E + 1;                                               // [E] its first row
    int* count = first + g.E;                                                    // [E] its rows
    int* height = count + g.E;                                                   // [E] rows of its tiles
    static_assert(sizeof(Bars) <= 512, "barriers");
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    volatile int* dead = &bar.dead;
    const uint32_t ring = tc::smem_addr(smem) + p.ring;

    if (warp == kMmaWarp) tc::tmem_alloc(&bar.tmem_slot, 512);
    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) { tc::mbar_init(&bar.full[i], 5); tc::mbar_init(&bar.empty[i], 1); }
        for (int i = 0; i < p.spans; ++i) { tc::mbar_init(&bar.planes_full[i], 1); tc::mbar_init(&bar.planes_empty[i], 4); }
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&bar.acc_full[i], 1); tc::mbar_init(&bar.acc_empty[i], kEpilogueWarps);
            tc::mbar_init(&bar.params_full[i], kEdgeWarps); tc::mbar_init(&bar.votes_full[i], kEpilogueWarps);
        }
        tc::mbar_init_fence();
        bar.dead = 0;
    }
    // Tiles of each expert: as few as hold its rows, and of about the same height, so that little of the last one is empty.
    if (warp == 0) {
        const uint32_t most = 0x7fffffffu / (uint32_t)p.col_tiles;               // (bounds that overlap can add up to any number of tiles)
        uint32_t sum = 0;
        constexpr int kTogether = 4;                                              // bounds of 32 experts on their way
        #pragma unroll 1
        for (int e0 = 0; e0 < g.E; e0 += 32 * kTogether) {
            int from[kTogether], to[kTogether];
            #pragma unroll
            for (int i = 0; i < kTogether; ++i) {
                const int e = e0 + 32 * i + lane < g.E ? e0 + 32 * i + lane : 0;
                from[i] = g.start[e]; to[i] = g.start[e + 1];
            }
            #pragma unroll
            for (int i = 0; i < kTogether; ++i) {
                const int e = e0 + 32 * i + lane;
                if (e0 + 32 * i >= g.E) break;
                int n = 0;
                const int64_t len = (int64_t)to[i] - from[i];
                if (from[i] >= 0 && len >= 0 && from[i] + len <= g.R) n = e < g.E ? (int)len : 0;
                else if (e < g.E && blockIdx.x == 0) atomicOr(g.status, kStatusBadIndex);
                const uint32_t tiles = ((uint32_t)n + (uint32_t)p.max_rows - 1) / (uint32_t)p.max_rows;
                uint32_t x = min(tiles, most);
                #pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
                    if (lane >= d) x = min(x + y, most);
                }
                if (e < g.E) {
                    before[e + 1] = (int)min(sum + x, most); first[e] = from[i]; count[e] = n;
                    height[e] = tiles > 0 ? ((n + (int)tiles - 1) / (int)tiles + 15) / 16 * 16 : 0;
                }
                sum = min(sum + __shfl_sync(0xffffffffu, x, 31), most);
            }
        }
        if (lane == 0) before[0] = 0;
    }
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
    int seen = 0;                                                                 // this warp's last expert: tiles only go up
    auto find = [&](uint32_t t) {                                                 // whole warp
        const int rt = (int)(t / cols);
        Tile r{0, 0, 0, 16};
        for (; seen < g.E; seen += 32) {
            const int e = seen + lane;
            const uint32_t who = __ballot_sync(0xffffffffu, e < g.E && rt < before[e + 1]);
            if (who != 0) { seen += __ffs(who) - 1; break; }
        }
        if (seen >= g.E) return r;
        r.e = seen;
        r.height = height[seen];
        const int at = (rt - before[seen]) * r.height, left = count[seen] - at;
        r.row = first[seen] + at;
        r.rows = left < r.height ? left : r.height;
        return r;
    };
    auto warp_wait = [&](uint64_t* m, uint32_t parity) {
        const bool ok = __all_sync(0xffffffffu, tc::mbar_wait_tries(m, parity & 1u, kTries)) != 0;
        if (!ok) *dead = 1;
        return ok;
    };
    const int quad = warp & 3;
    const int nblk = (int)((g.K + kBlockCodes - 1) / kBlockCodes), spans = (nblk + 3) / 4;
    const bool short_last = nblk % 4 == 1 || nblk % 4 == 2;
    auto halves_in = [&](int span) { return span == spans - 1 && short_last ? 1 : 2; };
    constexpr int kTileOuts = kGated ? 64 : 128;
    // The output that TMEM lane 32 q + l belongs to, so that the lanes r, r + 8, ... which one thread of the epilogue reads are adjacent outputs; gated,
    // lanes l >= 16 are the rows that those of l - 16 are multiplied with.
    auto output_at = [&](uint32_t t, int q, int l) {
        return (int64_t)(t % cols) * kTileOuts + (kGated ? q * 16 + 2 * (l & 7) + (l >> 3 & 1) : q * 32 + 4 * (l & 7) + (l >> 3));
    };
    bool alive = true;

    if (warp < kExpandWarps) {
        // ------------------------------------------------------------ weights: two teams of four warps have the spans in turn
        const int row4 = lane >> 2, q4 = lane & 3;
        const uint32_t mine = blockIdx.x < total ? (total - 1 - blockIdx.x) / gridDim.x + 1 : 0, n_spans = mine * (uint32_t)spans;
        int k = warp >> 2, sp = k;                                                // span of a tile, its slot
        while (k >= spans) k -= spans;
        if (sp >= p.spans) sp -= p.spans;
        uint32_t planes_phase = 0, phase = 0;
        int s = warp >> 2;                                                        // slot of the expanded codes
        if (s >= p.stages) s -= p.stages;
        for (uint32_t n = (uint32_t)warp >> 2; n < n_spans && alive; n += 2) {
            const int halves = halves_in(k);
            if (!(alive = warp_wait(&bar.planes_full[sp], planes_phase))) break;
            uint4 nz[4], pos[4];                                                  // TMEM lanes row4 + 8 j of the quarter, this lane's part of the span
            const uint8_t* from = smem + p.planes + (uint32_t)sp * kSpanBytes;
            const int block = 4 * k + 2 < nblk ? q4 : q4 >> 1;
            #pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = kGated ? (j >> 1) * 64 + quad * 16 + 2 * row4 + (j & 1) : quad * 32 + 4 * row4 + j;
                nz[j] = *reinterpret_cast<const uint4*>(from + row * 128 + (((2 * block) ^ (row & 7)) << 4));
                pos[j] = *reinterpret_cast<const uint4*>(from + row * 128 + (((2 * block + 1) ^ (row & 7)) << 4));
            }
            if (halves == 1) {                                                    // the last two blocks: this lane's half of one
                #pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (q4 & 1) { nz[j].x = nz[j].z; nz[j].y = nz[j].w; pos[j].x = pos[j].z; pos[j].y = pos[j].w; }
            }
            const uint32_t at = a_tmem + (uint32_t)(s * 64) + ((uint32_t)(quad * 32) << 16);
            #pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h >= halves) break;
                uint32_t o[2][16];
                #pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint4 a = h == 0 ? expand_weight(nz[j].x, pos[j].x) : expand_weight(nz[j].z, pos[j].z);
                    const uint4 b = h == 0 ? expand_weight(nz[j].y, pos[j].y) : expand_weight(nz[j].w, pos[j].w);
                    uint32_t* to = o[j >> 1] + 2 * (j & 1);
                    to[0] = a.x; to[1] = a.y; to[4] = a.z; to[5] = a.w; to[8] = b.x; to[9] = b.y; to[12] = b.z; to[13] = b.w;
                }
                if (h == 0 && !(alive = warp_wait(&bar.empty[s], phase + 1))) break;
                if (h == 0) tc::tc_fence_after_sync();
                tc::tmem_st_16x32(at + (uint32_t)(h * 32), o[0]);
                tc::tmem_st_16x32(at + (uint32_t)(h * 32) + (16u << 16), o[1]);
            }
            tc::tmem_st_wait();
            tc::tc_fence_before_sync();
            __syncwarp();
            // (The planes' slot is given back here and not behind the loads: an arrival that nothing waits for data with went ahead of loads under way, and the
            // next planes came into what they were still to read.)
            if (lane == 0) { tc::mbar_arrive(&bar.planes_empty[sp]); tc::mbar_arrive(&bar.full[s]); }
            s += 2;
            while (s >= p.stages) { s -= p.stages; phase ^= 1; }
            k += 2;
            while (k >= spans) k -= spans;
            sp += 2;
            if (sp >= p.spans) { sp -= p.spans; planes_phase ^= 1; }
        }
    } else if (warp >= kLoadWarp && warp < kEdgeWarp) {
      fewer_registers<kIssueRegs>();
      // (Tiles are looked up by whole warps: one thread that went on expert by expert took 2000 clocks where tiles are few to an expert.)
      if (warp == kLoadWarp) {
        // ------------------------------------------------------------ copies of input rows (one takes some 60 clocks to issue: few and large)
        tc::pdl_wait();
        const uint32_t elected = tc::elect_one(), box_bytes = (uint32_t)p.box_rows * 128u;
        int s = 0;
        uint32_t phase = 0;
        for (uint32_t t = blockIdx.x; t < total && alive; t += gridDim.x) {
            const Tile tile = find(t);
            const int boxes = (tile.height + p.box_rows - 1) / p.box_rows;        // (what lies behind the tile's rows belongs to no output)
            for (int k = 0; k < spans; ++k) {
                if (!(alive = warp_wait(&bar.empty[s], phase + 1))) break;
                const int halves = halves_in(k);
                if (elected) {
                    tc::mbar_arrive_expect_tx(&bar.full[s], (uint32_t)(halves * boxes) * box_bytes);
                    uint32_t dst = ring + (uint32_t)s * 2 * p.half_bytes;
                    for (int h = 0; h < halves; ++h, dst += p.half_bytes) {
                        load_box(dst, &map, k * 256 + h * 128, tile.row, &bar.full[s]);
                        if (boxes > 1) load_box(dst + box_bytes, &map, k * 256 + h * 128, tile.row + p.box_rows, &bar.full[s]);
                    }
                }
                __syncwarp();
                if (++s == p.stages) { s = 0; phase ^= 1; }
            }
        }
        // nobody leaves while copies are on their way: the last of each slot
        for (int i = 0; i < p.stages; ++i) {
            const uint32_t uses = i < s ? phase + 1 : phase;                      // parity of the number of copies to this slot
            tc::mbar_wait_tries(&bar.full[i], (uses + 1) & 1u, kTries);
        }
      } else if (warp == kPlanesWarp) {
        // ------------------------------------------------------------ copies of planes
        const uint32_t elected = tc::elect_one();
        int s = 0;
        uint32_t phase = 0;
        for (uint32_t t = blockIdx.x; t < total && alive; t += gridDim.x) {
            const int row = (int)((int64_t)find(t).e * g.N + (int64_t)(t % cols) * kTileOuts);
            for (int k = 0; k < spans; ++k) {
                if (!(alive = warp_wait(&bar.planes_empty[s], phase + 1))) break;
                if (elected) {
                    tc::mbar_arrive_expect_tx(&bar.planes_full[s], kSpanBytes);
                    const uint32_t dst = ring - p.ring + p.planes + (uint32_t)s * kSpanBytes;
                    load_box(dst, &weight_map, k * 128, row, &bar.planes_full[s]);                          // (rows of other outputs behind the last,
                    if (kGated) load_box(dst + kSpanBytes / 2, &weight_map, k * 128, row + (int)g.F, &bar.planes_full[s]);          // zeros behind the last row)
                }
                __syncwarp();
                if (++s == p.spans) { s = 0; phase ^= 1; }
            }
        }
        for (int i = 0; i < p.spans; ++i) {
            const uint32_t uses = i < s ? phase + 1 : phase;
            tc::mbar_wait_tries(&bar.planes_full[i], (uses + 1) & 1u, kTries);
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
            for (int k = 0; k < spans; ++k) {
                if (!(alive = warp_wait(&bar.full[s], phase))) break;
                tc::tc_fence_after_sync();
                uint64_t b = desc + (uint64_t)((uint32_t)s * (p.half_bytes >> 3));
                uint32_t a = a_tmem + (uint32_t)(s * 64);
                for (int h = halves_in(k); h > 0; --h, a += 32u, b += (uint64_t)(p.half_bytes >> 4)) {
                    #pragma unroll
                    for (int j = 0; j < 4; ++j)                                   // K = 64: 32 bytes, eight columns
                        mma_mxf4(elected, d, a + (uint32_t)(j * 8), b + (uint64_t)(j * 2), idesc, scales, k > 0 || j > 0 || h == 1 && halves_in(k) == 2);
                }
                if (elected) tc::mma_commit(&bar.empty[s]);
                __syncwarp();
                if (++s == p.stages) { s = 0; phase ^= 1; }
            }
            if (elected && alive) tc::mma_commit(&bar.acc_full[ti & 1]);
            __syncwarp();
        }
      }
      __syncwarp();
    } else if (warp >= kEdgeWarp) {
        // ------------------------------------------------------------ what a tile begins with, parameters of its tokens and weight rows, and ends with, its
        // codes put together from the votes: a quarter of each to a warp.  Parameters are asked for a tile ahead, input rows two ahead (with
        // both asked for and waited for in a tile's turn, that took 4000 clocks, longer than its products).
        fewer_registers<kEdgeRegs>();
        constexpr int kEach = (kMaxRows + 127) / 128;
        const int part = warp - kEdgeWarp;
        int m[kEach], m_next[kEach];                                              // -1: out of range, -2: no such row
        float ws = 0.f, wo = 0.f, bias = 0.f, as[kEach], ao[kEach];
        int sw = 0, sx[kEach];
        Tile asked{}, tile{};                                                     // whose rows, and whose parameters, have been asked for last
        auto row_of = [&](int i) { return lane + 32 * (part + 4 * i); };
        auto ask_rows = [&](uint32_t t) {
            #pragma unroll
            for (int i = 0; i < kEach; ++i) m_next[i] = -2;
            if (t >= total) return;
            asked = find(t);
            #pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (row_of(i) < asked.rows) m_next[i] = g.tokens != nullptr ? __ldg(g.tokens + asked.row + row_of(i)) : asked.row + row_of(i);
        };
        auto ask_params = [&](uint32_t t) {
            if (t >= total) return;
            tile = asked;
            const int64_t first_row = (int64_t)tile.e * g.N;
            #pragma unroll
            for (int i = 0; i < kEach; ++i) {
                m[i] = m_next[i];
                as[i] = ao[i] = 0.f; sx[i] = 0;
                if (m[i] != -2) {
                    const bool ok = m[i] >= 0 && m[i] < g.T;
                    const int64_t in = ok ? m[i] : 0, at = g.ep.n_aparam == 1 ? 0 : in;
                    as[i] = __ldg(g.ep.a_scale + at); ao[i] = __ldg(g.ep.a_offset + at); sx[i] = __ldg(g.a_sum + in);
                    if (!ok) m[i] = -1;
                }
            }
            const int64_t f = output_at(t, part, lane), at = first_row + (kGated && lane >= 16 ? g.F + f : f), w = g.ep.n_wparam == 1 ? 0 : at;
            ws = wo = bias = 0.f; sw = 0;
            if (f < g.F) { ws = __ldg(g.ep.w_scale + w); wo = __ldg(g.ep.w_offset + w); sw = __ldg(g.w_sum + at); if (g.bias != nullptr) bias = __ldg(g.bias + at); }
        };
        auto tell = [&](uint32_t t, uint32_t at) {                                // the parameters of tile t, and asks for those of the next
            if (t >= total) return;
            TileParams& here = params[at];
            uint32_t most_asx = 0, most_ao = 0;
            bool bad = false;
            #pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int r = row_of(i);
                if (m[i] == -1) { as[i] = ao[i] = __int_as_float(0x7fffffff); bad = true; }
                const float asx = as[i] * (float)sx[i];
                if (r < kMaxRows) { here.as[r] = as[i]; here.asx[r] = asx; here.ao[r] = ao[i]; here.token[r] = m[i]; }
                most_asx = max(most_asx, __float_as_uint(fabsf(asx))); most_ao = max(most_ao, __float_as_uint(fabsf(ao[i])));
            }
            here.col[part * 32 + lane] = make_float4(ws, wo, (float)((double)ws * (double)sw + (double)g.K * (double)wo), bias);
            most_asx = __reduce_max_sync(0xffffffffu, most_asx); most_ao = __reduce_max_sync(0xffffffffu, most_ao);
            if (lane == 0) { (&here.most_asx.x)[part] = most_asx; (&here.most_ao.x)[part] = most_ao; here.tile[part] = tile; }
            if (bad && t % cols == 0) atomicOr(g.status, kStatusBadIndex);
            __threadfence_block();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bar.params_full[at]);
            ask_params(t + gridDim.x);
            ask_rows(t + 2 * gridDim.x);
        };
        ask_rows(blockIdx.x);
        ask_params(blockIdx.x);
        ask_rows(blockIdx.x + gridDim.x);
        tell(blockIdx.x, 0);
        tell(blockIdx.x + gridDim.x, 1);
        tc::pdl_wait();
        uint32_t ti = 0;
        for (uint32_t t = blockIdx.x; t < total; t += gridDim.x, ++ti) {
            if (!(alive = warp_wait(&bar.votes_full[ti & 1], ti >> 1))) break;
            if constexpr (kCodes) {
                const TileParams& here = params[ti & 1];
                // (A place of this warp's own: nothing orders the edge warps among each other, so the first of them may be a tile ahead and have put the
                // place of the one two rounds on where the others are still to read.)
                const Tile tile = here.tile[part];
                const int64_t f0 = (int64_t)(t % cols) * kTileOuts, width = (g.F + kBlockCodes - 1) / kBlockCodes * kBlockCodes;
                #pragma unroll 1
                for (int r = lane + 32 * part; r < tile.rows; r += 32 * kEdgeWarps) {
                    // bit 4 i + q of vote j is output kOwn i + j of a quarter, for token 2 q or the one after it
                    const int q = r >> 1 & 3, slot = r / 16 * 4 + (r >> 3 & 1) * 2 + (r & 1);
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
                    uint8_t* to = g.out_packed + (int64_t)(tile.row + r) * (width / 4) + f0 / kBlockCodes * kBlockBytes + f0 % kBlockCodes / 8;
                    if constexpr (kGated) {
                        *reinterpret_cast<uint2*>(to) = make_uint2(nz[0] | nz[1] << 16, nz[2] | nz[3] << 16);
                        *reinterpret_cast<uint2*>(to + 16) = make_uint2(up[0] | up[1] << 16, up[2] | up[3] << 16);
                    } else {
                        *reinterpret_cast<uint4*>(to) = make_uint4(nz[0], nz[1], nz[2], nz[3]);
                        *reinterpret_cast<uint4*>(to + 16) = make_uint4(up[0], up[1], up[2], up[3]);
                    }
                    const int sum = 2 * (__popc(up[0]) + __popc(up[1]) + __popc(up[2]) + __popc(up[3])) - (__popc(nz[0]) + __popc(nz[1]) + __popc(nz[2]) + __popc(nz[3]));
                    if (sum != 0) atomicAdd(&g.out_sum[tile.row + r], sum);        // (whole numbers: any order gives the same)
                }
                __syncwarp();
            }
            tell(t + 2 * gridDim.x, ti & 1);                                      // (the votes have been read, and so have the parameters, before they were cast)
        }
    } else {
        // ------------------------------------------------------------ write out: a warp has a quarter of the lanes and every other 16 tokens; a thread
        // kOwn adjacent outputs of two tokens in each 8.
        more_registers<kEpilogueRegs>();
        constexpr int kOwn = kGated ? 2 : 4;
        const int half = (warp - kExpandWarps) >> 2, r8 = lane >> 2, q4 = lane & 3;
        tc::pdl_wait();
        const bool whole = kCodes || ((reinterpret_cast<uintptr_t>(g.out) % (kOwn * sizeof(T))) == 0 && g.out_stride % kOwn == 0);
        // Units of an output's error for its value before the activation: the affine form's own (below), passed on with a slope of at most
        // 1.13, and the activation's.
        const float units = g.act == RTN_ACT_SILU ? 8.3f : g.act == RTN_ACT_NONE || g.act == RTN_ACT_RELU ? 2.f : 18.3f;
        const float c1 = (units + (kGated ? 3.f : 0.f)) * 1.1f * kUnit;
        uint32_t ti = 0;
        for (uint32_t t = blockIdx.x; t < total; t += gridDim.x, ++ti) {
            TileParams& here = params[ti & 1];
            if (!(alive = warp_wait(&bar.params_full[ti & 1], ti >> 1))) break;
            const Tile tile = here.tile[0];
            // this thread's weight rows: kOwn outputs, or kOwn and the kOwn that they are multiplied with
            pair_t ws[4], wo[4], p3[4], bias[4];
            float off = 0.f, lo = 0.f, hi = 0.f, most_asx = 0.f, most_ao = 0.f;
            if constexpr (kCodes) {
                const uint4 a = here.most_asx, b = here.most_ao;
                most_asx = __uint_as_float(max(max(a.x, a.y), max(a.z, a.w)));
                most_ao = __uint_as_float(max(max(b.x, b.y), max(b.z, b.w)));
            }
            #pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 c = here.col[quad * 32 + r8 + 8 * j];
                ws[j] = make_pair(c.x, c.x); wo[j] = make_pair(c.y, c.y); p3[j] = make_pair(c.z, c.z); bias[j] = make_pair(c.w, c.w);
                // what the terms of the affine form other than the product add up to at most
                if constexpr (kCodes) {
                    const float x = most_asx * fabsf(c.y) + most_ao * fabsf(c.z) + fabsf(c.w);
                    off = !(x <= off) ? x : off;                                   // (a NaN stays)
                }
            }
            // y = w_s (a_s S) + P with P = w_o a_s S_x + (p3 a_o + bias): u (2 |y| + 4 off) covers its roundings (those of a_s S, a_s S_x and p3, and
            // three sums).  Gated, with |activation| <= |y1|:
            //   |y2| (units |y1| + 4.6 off) + |y1| (2 |y2| + 4 off) + |y1 y2| <= ((units + 3) |y1| + 4.6 off) (|y2| + 0.8 off)
            float c0 = 0.f, c2 = 0.f;
            if constexpr (kCodes) { lo = g.t_lo[g.n_thr == 1 ? 0 : tile.e]; hi = g.t_hi[g.n_thr == 1 ? 0 : tile.e]; c0 = 4.6f * 1.1f * kUnit * off; c2 = 0.8f * off; }
            if (!kGated && g.act == RTN_ACT_RELU && lo <= 0.f) lo = -FLT_MAX;        // (never below it: a threshold of 0 is not near)
            const int64_t f = output_at(t, quad, r8);                              // the first of this thread's outputs
            if (!(alive = warp_wait(&bar.acc_full[ti & 1], ti >> 1))) break;
            tc::tc_fence_after_sync();
            const uint32_t acc = tmem + (ti & 1) * acc_cols + ((uint32_t)(quad * 32) << 16);
            T* out = static_cast<T*>(g.out) + (int64_t)(tile.row + half * 16 + 2 * q4) * g.out_stride + f;
            const bool vec = whole && f + kOwn <= g.F;
            #pragma unroll 1
            for (int c = half * 16; c < tile.rows; c += 32, out += 32 * g.out_stride) {
                uint32_t v[2][8];                                                  // TMEM lanes r8, r8 + 8 and r8 + 16, r8 + 24
                tc::tmem_ld_16x16(acc + (uint32_t)c, v[0]);
                tc::tmem_ld_16x16(acc + (uint32_t)c + (16u << 16), v[1]);
                tc::tmem_ld_wait();
                // the 16 tokens in steps of their own, so that each has many independent values: affine forms, activations, codes
                bool near = false;
                float y[2][4][2], err[2][kOwn][2];                                 // by group of 8 tokens, weight row and token
                #pragma unroll
                for (int a = 0; a < 2; ++a) {
                    const int at = c + 8 * a + 2 * q4;                             // tokens at and at + 1
                    const float2 as = *reinterpret_cast<const float2*>(&here.as[at]), sx = *reinterpret_cast<const float2*>(&here.asx[at]);
                    const float2 ao = *reinterpret_cast<const float2*>(&here.ao[at]);
                    const pair_t as2 = make_pair(as.x, as.y), sx2 = make_pair(sx.x, sx.y), ao2 = make_pair(ao.x, ao.y);
                    #pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t* S = &v[j >> 1][4 * a + 2 * (j & 1)];
                        take_pair(fma_pair(ws[j], mul_pair(as2, make_pair(__uint_as_float(S[0]), __uint_as_float(S[1]))),
                                           fma_pair(wo[j], sx2, fma_pair(p3[j], ao2, bias[j]))), y[a][j][0], y[a][j][1]);
                    }
                    if constexpr (kCodes) {
                        #pragma unroll
                        for (int j = 0; j < kOwn; ++j)
                            #pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                err[a][j][i] = fmaf(c1, fabsf(y[a][j][i]), c0);
                                if constexpr (kGated) err[a][j][i] *= fabsf(y[a][kGated ? kOwn + j : j][i]) + c2;
                            }
                    }
                }
                if (g.act == RTN_ACT_SILU) {
                    #pragma unroll
                    for (int a = 0; a < 2; ++a)
                        #pragma unroll
                        for (int j = 0; j < kOwn; ++j) { y[a][j][0] = fast_silu(y[a][j][0]); y[a][j][1] = fast_silu(y[a][j][1]); }
                } else if (g.act != RTN_ACT_NONE) {
                    #pragma unroll
                    for (int a = 0; a < 2; ++a)
                        #pragma unroll
                        for (int j = 0; j < kOwn; j += 2) {
                            const float4 x = activation4(make_float4(y[a][j][0], y[a][j][1], y[a][j + 1][0], y[a][j + 1][1]), g.act);
                            y[a][j][0] = x.x; y[a][j][1] = x.y; y[a][j + 1][0] = x.z; y[a][j + 1][1] = x.w;
                        }
                }
                #pragma unroll
                for (int a = 0; a < 2; ++a) {
                    if constexpr (kGated) {
                        #pragma unroll
                        for (int j = 0; j < kOwn; ++j) { y[a][j][0] *= y[a][kOwn + j][0]; y[a][j][1] *= y[a][kOwn + j][1]; }
                    }
                    if constexpr (kCodes) {
                        #pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            uint32_t nz[kOwn], up[kOwn];
                            #pragma unroll
                            for (int j = 0; j < kOwn; ++j) {
                                const float x = y[a][j][i];
                                const bool p = x > hi, n = p || x < lo;
                                near = near || !(fminf(fabsf(x - lo), fabsf(x - hi)) > err[a][j][i]);
                                nz[j] = __ballot_sync(0xffffffffu, n);
                                up[j] = __ballot_sync(0xffffffffu, p);
                            }
                            if (lane == 0) {
                                #pragma unroll
                                for (int j = 0; j < kOwn; j += 2) here.votes[quad][c / 4 + 2 * a + i][j / 2] = make_uint4(nz[j], up[j], nz[j + 1], up[j + 1]);
                            }
                        }
                    }
                    if (!kCodes || g.out != nullptr) {
                        #pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            if (c + 8 * a + 2 * q4 + i >= tile.rows) continue;
                            T* to = out + (8 * a + i) * g.out_stride;
                            const auto& w = y[a];
                            if (!kCodes && vec) {
                                if constexpr (sizeof(T) == 2) {
                                    if constexpr (kOwn == 4) *reinterpret_cast<uint2*>(to) = make_uint2(pack2<T>(w[0][i], w[1][i]), pack2<T>(w[2][i], w[3][i]));
                                    else *reinterpret_cast<uint32_t*>(to) = pack2<T>(w[0][i], w[1][i]);
                                } else {
                                    if constexpr (kOwn == 4) *reinterpret_cast<float4*>(to) = make_float4(w[0][i], w[1][i], w[2][i], w[3][i]);
                                    else *reinterpret_cast<float2*>(to) = make_float2(w[0][i], w[1][i]);
                                }
                            } else {
                                #pragma unroll
                                for (int j = 0; j < kOwn; ++j) if (f + j < g.F) to[j] = from_f32<T>(w[j][i]);
                            }
                        }
                    }
                }
                if constexpr (kCodes) {
                    if (__any_sync(0xffffffffu, near)) {                           // the 16 tokens again, those too near in double
                        #pragma unroll 1
                        for (int a = 0; a < 2; ++a) {
                            uint32_t w[2][4];
                            tc::tmem_ld_16x8(acc + (uint32_t)(c + 8 * a), w[0]);
                            tc::tmem_ld_16x8(acc + (uint32_t)(c + 8 * a) + (16u << 16), w[1]);
                            tc::tmem_ld_wait();
                            #pragma unroll 1
                            for (int i = 0; i < 2; ++i) {
                                const int at = c + 8 * a + 2 * q4 + i, m = at < tile.rows ? here.token[at] : -1;
                                const RowParams row{here.as[at], here.ao[at], 0.f, m};
                                uint32_t nz[kOwn], up[kOwn];
                                #pragma unroll
                                for (int j = 0; j < kOwn; ++j) {
                                    const float S = __uint_as_float(i ? w[j >> 1][2 * (j & 1) + 1] : w[j >> 1][2 * (j & 1)]);
                                    const float S2 = __uint_as_float(i ? w[1][2 * (j & 1) + 1] : w[1][2 * (j & 1)]);
                                    const float asx = here.asx[at];
                                    auto value = [&](int k, float sum) {
                                        const float4 q = here.col[quad * 32 + r8 + 8 * k];
                                        return fmaf(q.x, row.as * sum, fmaf(q.y, asx, fmaf(q.z, row.ao, q.w)));
                                    };
                                    const float y1 = value(j, S), y2 = kGated ? value(kGated ? kOwn + j : j, S2) : 1.f;
                                    const float act = g.act == RTN_ACT_SILU ? fast_silu(y1) : g.act == RTN_ACT_NONE ? y1 : activation(y1, g.act);
                                    const float x = kGated ? act * y2 : act, e = fmaf(c1, fabsf(y1), c0), err = kGated ? e * (fabsf(y2) + c2) : e;
                                    bool p = x > hi, n = p || x < lo;
                                    if (!(fminf(fabsf(x - lo), fabsf(x - hi)) > err)) {
                                        p = n = false;
                                        if (m >= 0 && f + j < g.F) {
                                            const double d = exact_value(g, m, tile.e, f + j, S, S2);
                                            p = d > (double)hi;
                                            n = p || d < (double)lo;
                                        }
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
            __threadfence_block();
            __syncwarp();
            if (lane == 0) { tc::mbar_arrive(&bar.acc_empty[ti & 1]); tc::mbar_arrive(&bar.votes_full[ti & 1]); }
        }
    }

    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    if (threadIdx.x == 0 && *dead) atomicOr(g.status, kStatusWaitTimeout);
    if (warp == kMmaWarp) tc::tmem_dealloc(tmem, 512);
}

// Rows of a tile at most, from the rows that an expert has on average: what makes rounds of tiles times a tile's time least.  A tile's time in clocks is the
// longer of its expansion and products (350 for 256 codes, from 135 rows on 2.6 a row) and its outputs (500 and 20 a row; fitted to
// measured times), and the shorter once more at the end.  65536 rows of 64 experts, 2048 x 2048 gated with codes, and 2048 x 1024 to bf16 (before later
// steps took 26 and 20 us off): 160 rows 271 and 153 us, 144 280 and 162, 128 279 and 164, 112 304 and 179.  (512 - 16 - 2 h) / 64 slots of weights fit
// tensor memory beside two accumulators of h rows: two from 160 on, three from 144 down.  Above kMaxRows nothing was measured; 176 would have two slots, too.
TilesPlan make_plan(const ExpertsArgs& g)
{
    TilesPlan p{};
    const int outs = g.gated ? 64 : 128;
    const int64_t width = g.out_packed != nullptr ? (g.F + kBlockCodes - 1) / kBlockCodes * kBlockCodes : g.F;
    p.col_tiles = (int)((width + outs - 1) / outs);
    p.k_halves = halves_of((int)((g.K + kBlockCodes - 1) / kBlockCodes));
    const double used = (double)(g.R < g.E ? g.R : g.E), each = (double)g.R / used, sms = device_sm_count();
    double best = 0.0;
    for (int h = 16; h <= kMaxRows; h += 16) {
        const double per = (double)(int64_t)((each + h - 1) / h), tiles = used * per * p.col_tiles, height = each / per < 16 ? 16 : each / per;
        const double stage = 2.6 * height > 350.0 ? 2.6 * height : 350.0, loop = stage * p.k_halves, out = 20.0 * height + 500.0;
        const double rounds = tiles / sms < 1.0 ? 1.0 : (double)(int64_t)((tiles + sms - 1) / sms);
        const double cost = rounds * (loop > out ? loop : out) + (loop > out ? out : loop);
        if (p.max_rows == 0 || cost < best) { best = cost; p.max_rows = h; }
    }
    p.box_rows = p.max_rows > 64 ? (p.max_rows + 31) / 32 * 16 : p.max_rows;          // two to a tile, or one
    p.half_bytes = (uint32_t)((p.max_rows + p.box_rows - 1) / p.box_rows * p.box_rows) * 128u;
    p.ring = (uint32_t)((512 + 2 * sizeof(TileParams) + (4 * g.E + 1) * 4 + 1023) / 1024 * 1024);
    const int by_tmem = (512 - 2 * p.max_rows - (int)kScaleCols) / 64;
    p.stages = by_tmem < kMaxStages ? by_tmem : kMaxStages;
    while (p.stages > 2 && p.ring + (uint32_t)p.stages * 2 * p.half_bytes + 4 * kSpanBytes > kSmemBytes) --p.stages;
    p.planes = p.ring + (uint32_t)p.stages * 2 * p.half_bytes;                   // (a multiple of 1024: halves are multiples of 2048 bytes)
    p.spans = (int)((kSmemBytes - p.planes) / kSpanBytes);
    if (p.spans > kMaxSpans) p.spans = kMaxSpans;
    p.smem = p.planes + (uint32_t)p.spans * kSpanBytes;
    return p;
}

}  // namespace

cudaError_t launch_experts_tiles(const ExpertsArgs& g, cudaStream_t s)
{
    const TilesPlan p = make_plan(g);
    const EncodeTiledFn encode = encode_tiled_fn();
    if (encode == nullptr) return cudaErrorNotSupported;
    const int nblk = (int)((g.K + kBlockCodes - 1) / kBlockCodes), pitch = p.k_halves * 128;
    void* scratch = nullptr;
    cudaError_t e = scratch_alloc(&scratch, (size_t)g.R * pitch, s);
    if (e != cudaSuccess) return e;
    CUtensorMap map, weight_map;
    const cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)g.R}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {128, (cuuint32_t)p.box_rows}, unit[2] = {1, 1};
    if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, scratch, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) e = cudaErrorInvalidValue;
    const cuuint64_t wdims[2] = {(cuuint64_t)nblk * kBlockBytes, (cuuint64_t)g.E * (cuuint64_t)g.N}, wstrides[1] = {(cuuint64_t)nblk * kBlockBytes};
    const cuuint32_t wbox[2] = {128, g.gated ? 64u : 128u};
    if (encode(&weight_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(g.w_packed), wdims, wstrides, wbox, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) e = cudaErrorInvalidValue;
    if (e == cudaSuccess) {
        const int64_t threads = g.R * (pitch / 16);
        // (its launch under the end of what ran before, too: calls one after the other 24.6 -> 21.6 us for 384 rows of 2048 x 2048)
        e = launch_pdl(expand_inputs_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, g, nblk, pitch / 16, static_cast<uint2*>(scratch));
    }
    if (e == cudaSuccess) {
        e = with_dtype(g.dtype, [&](auto t) {
            using T = decltype(t);
            auto run = [&](auto kernel) {
                cudaError_t x = allow_shared_memory(kernel);
                if (x != cudaSuccess) return x;
                return launch_pdl(kernel, dim3((unsigned)device_sm_count()), dim3(kThreads), p.smem, s, g, map, weight_map, p);
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
    const int64_t pitch = (g.K + 255) / 256 * 8, cols = (g.F + 191) / 64 + 1;
    return g.R * pitch < (int64_t(1) << 32) - 256 && (g.R / 16 + g.E) * cols < (int64_t(1) << 31);
}

}  // namespace rtn
