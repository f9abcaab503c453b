// Split-KV single-token decode of Eq. 5 over paged levels whose keys and values are 8-bit codes with one exponent per block of rows and
// KV head (code8.cuh), grouped-query heads:
//     s_j = tau 2^ek(j) (q . ck_j),   p_j = lambda exp(s_j - m),   O = sum_j p_j 2^ev(j) cv_j / sum_j p_j
// What bounds it are the codes' bytes, 2 d per row and KV head: half of what the bf16 cache takes, for the same products.  The work is dealt as in
// the bf16 form (tile_deal.cuh): one share of the tiles (8 KB: 32 rows at d = 128, 64 at d = 64) for each of two CTAs per SM, two producing warps that have the
// copy engine bring the pages' rows into a ring, and computing warps that take the tiles in turn, whole: with a tile split between
// four warps, 16 rows to each, what a step costs besides the products (waits, the walk, the running maximum) took 470 instructions per 16 rows at d = 128.
// Four sequences at up to 128K rows, 28 heads on 4 of 128 (413 MB): 82 us with the combine kernel where the inputs change from call to call, 5.0 TB/s (0.77 of a copy), 76 to 78 back to
// back on the same ones, 72 so without any computing; 64 sequences of up to 6500 rows, 32 heads on 8 of 64, integer codes (371 MB): 83 us (0.68), 80.5 and 74 so.  About 10 us of each
// are the start, the merges and the combine; one sequence of 10,000 rows takes 12.6 us.
//
// The products are turned over: S^T = K Q^T and O^T = V^T P^T, m16n8k16, with 16 keys or 16 columns as the rows of the left operand and eight query heads as
// the columns of the right one.  A group of up to eight heads then fills the products (as the rows of the left operand it would fill half of them), and
// accumulators, scores and weights take half of the registers and instructions; wider groups take two such products.
// Codes become f16 in registers, exactly, straight out of ldmatrix: a 16-byte piece of a key row is 16 codes, of which a lane gets four
// neighbouring ones.  The sum over the columns does not care for their order, so the lane's four serve as its two pairs of a
// product's k-step, and the query fragments are loaded in the same order.  Value rows come through ldmatrix.trans as pairs of neighbouring columns; one
// byte permutation pairs up the rows, and rows g and g + 8 of the left operand are the columns 2 g and 2 g + 1.  The weights change sides through movmatrix.
//
// Ranges: f16 has the precision for codes (exact), queries (8 bits) and weights (11 bits), but not the range.  Every query row is scaled by the power of two
// that brings its largest element to 2^14 .. 2^15; what falls below f16's smallest number then is 2^-39 of that.  The keys' exponent and the row's
// factor are applied to the scores in fp32.  Weights enter the second product as p 2^ev / 2^mv with mv the running maximum of (group maximum of
// log2 p) + ev over the row groups, at 2^14 the largest.  An f16 below 2^-14 is off by up to 2^-25, which is 2^-39 of 2^mv; mv lies less than 5 above the largest real product
// (4 where a tile's exponents lie up to 4 apart, 1 as it is a whole number): 2^-34 of that.  p itself, and a warp's or a share's whole state, counts as 0 below 2^-125 of the
// largest weight: at exponents D apart, 2^(D - 125) of the largest product, which is more only from D = 92 on (2^-29 at D = 96).  Maximum, sum of the weights and accumulators are fp32, each row's accumulator in units of 2^(mv - 14).
#include <cuda_fp16.h>

#include <type_traits>

#include "code8.cuh"
#include "tile_deal.cuh"

namespace mka {
namespace {


__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {               // of an 8 x 8 matrix of f16, a pair to a lane
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float bf_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.f;                          // (NaN too)
}
// A partial's maximum and sum.  A score of NaN (a NaN among the row's keys or queries, or an infinite score) leaves NaN in the sum and in every
// column; the combine kernel takes partials by "sum > 0", so such a one is made the largest, with an infinite sum: O is NaN, LSE infinite.  (Of several
// tokens it ends as 0 and -infinity, as the tensor-core forward ends it.)
__device__ __forceinline__ void put_max_sum(float* out, float m, float z) {
    const bool nan = !(z == z);
    out[0] = nan ? 1e38f : m;
    out[1] = nan ? INFINITY : z;
}

struct Maps8 {
    CUtensorMap k[3], v[3];
};

// Computing warps of a CTA; two more produce.  Six of them (four warps to a scheduler) were no faster: 83.6 us to 82.1 on a mixed batch to 128K rows, 88.9 to 86.0
// at d = 64.  Spills to memory (bytes stored): NB = 2 at d = 128 40 to 64, of several tokens 164 to 220, and 76 to 84 at d = 64; combine8 with four warps to a CTA 40.
constexpr int C = 4, kThreads = (C + 2) * 32;
template <int DH> struct Ring {
    static constexpr int kRows = tile_rows8(DH), kGroups = kRows / 16;
    static constexpr int kTileBytes = kRows * DH;           // codes of K or of V
    // 64 or 96 KB in flight per CTA, two CTAs per SM, beside the warps' states (d = 64 with two products, NB = 2: 121 KB with the states, one CTA to an SM: 64 heads on 4 at up to 128K rows
    // 89 us, 32 on 4 50, for 31.5 of bytes).  A multiple of the computing warps: a stage belongs to one warp, so nobody
    // waits for a phase of a barrier without having seen the phase before (which a wait by parity could not tell from the one before that).
    static constexpr int kStages = DH == 128 ? 8 : 12;
    static_assert(kStages % C == 0, "a stage belongs to one warp");
};

// NB: eights of query heads to a KV head, 1 or 2.  kChunk: the rows are heads x T tokens, each token with its gate and its place; see launch_chunk_paged8.
template <int DH, bool kS8, int NB, bool kChunk>
__global__ void __launch_bounds__(kThreads, 2) decode_paged8_kernel(const __grid_constant__ Maps8 maps, const DecodePaged8Params p8) {
    const DecodePagedParams& p = p8.base;
    constexpr int kTileBytes = Ring<DH>::kTileBytes, kStages = Ring<DH>::kStages, kTileRows = Ring<DH>::kRows, kGroups = Ring<DH>::kGroups;
    constexpr int KS = DH / 16;                             // 16-byte pieces of a row, k-steps of Q K^T
    constexpr int kAcc = NB * KS * 4, kState = kAcc + NB * 4;            // one thread's accumulators; with its maxima and sums
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    float* states = reinterpret_cast<float*>(smem + kStages * 2 * kTileBytes);       // [C][kState][32]: the computing warps' at the end of a list
    int* before = reinterpret_cast<int*>(states + C * kState * 32);                  // [blocks + 1]
    __shared__ uint64_t full[kStages], empty[kStages];
    __shared__ __align__(16) float k_scale[kStages][kGroups], v_exp[kStages][kGroups];       // 2^ek, and ev, of every 16 rows of a tile
    __shared__ WaitCtl ctl;
    using Lists = std::conditional_t<kChunk, ChunkLists, GatedLists>;
    using Walk = TileWalk<kTileRows, Lists>;
    __shared__ typename Walk::Place place;

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int blocks = kChunk ? p8.blocks : 1, GT = p.H / (p.H_kv / blocks);          // lists to a KV head; its rows
    const long long slot_floats = DH + 2, list_floats = p.total_chunks * slot_floats;   // entry 0 of a head: how many partials follow
    if (tid == 0) {
        ctl.abort = 0;
        ctl.limit_ns = p.wait_limit_ns;
        for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 2); mbar_init(&empty[i], 1); }      // (two producers; one warp)
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    chain_enter();
    if (blockIdx.x == 0 && tid == 0 && p.status) atomicExch(p.status, (unsigned int)MKA_OK);
    volatile WaitCtl* ctlp = &ctl;
    Walk walk(p);
    int share;
    if (!deal_share<kTileRows, kThreads, Lists>(p, walk, share, before, place, list_floats, tid, warp, lane)) return;

    if (warp >= C) {
        // ------------------------------------------------------------ producers, of keys and of values
        // Each takes up to kBatch consecutive tiles of a list at a time, a lane to 16 rows of one of them, whose page is looked up two batches ahead and
        // whose exponent is fetched one batch ahead.  Tile by tile every look-up's way to memory and back showed (1600 cycles to a tile); one warp for keys
        // and values issued its copies in 1060 cycles a tile (mixed batch to 128K rows: 82 us without any computing, 100 with it).
        constexpr int kBatch = 32 / kGroups, kFirst = 4;    // (the first batch is short: its copies leave sooner)
        static_assert(kFirst < kStages && kFirst <= kBatch, "the first batch goes into an empty ring and leaves it unfilled");
        const bool values = warp > C;
        struct Batch { int count, b, kvh, lvl, page, in_row; unsigned int e; };
        int seg_left = walk.segment(), t = walk.at;
        bool more = true;
        auto next = [&](Batch& x, int most) {
            x.count = 0;
            if (!more) return;
            x.count = min(most, seg_left);
            x.b = walk.b; x.kvh = walk.kvh / blocks;
            int row0, rows;
            walk.locate(t + min(lane / kGroups, x.count - 1), x.lvl, row0, rows);
            const PagedLevelDev& L = p.L[x.lvl];
            int r = row0 + (lane % kGroups) * 16;
            if (r >= rows) r = row0;                        // (rows behind the last one: the tile's first again)
            if (kChunk) r += p.skip[x.lvl];
            x.page = L.table[(long long)x.b * L.table_stride + (long long)x.kvh * L.table_head_stride + (r >> L.page_shift)];
            x.in_row = r & ((1 << L.page_shift) - 1);
            t += x.count;
            seg_left -= x.count;
            if (seg_left == 0) {
                more = walk.advance(walk.segment());
                if (more) { seg_left = walk.segment(); t = walk.at; }
            }
        };
        // (a page outside the pool reads as zeros: the copy engine fills them in, and no exponent is asked for)
        auto fetch = [&](Batch& x) {
            x.e = 127u;
            if (x.count > 0 && (unsigned int)x.page < (unsigned int)p.L[x.lvl].pool_pages)
                x.e = (values ? p8.v_exp : p8.k_exp)[x.lvl][x.page * p8.esp[x.lvl] + x.kvh * p8.esh[x.lvl] + (x.in_row >> p8.block_shift[x.lvl])];
        };
        uint8_t* const ring = smem + (values ? kTileBytes : 0) + lane % kGroups * 16 * DH;
        float* const exps = values ? v_exp[0] : k_scale[0];
        auto copy = [&](const Batch& x, int u, int st) {
            if (lane / kGroups == u && (lane % kGroups * 16 & ((1 << p.L[x.lvl].page_shift) - 1)) == 0)
                tma_load_4d(ring + (size_t)st * 2 * kTileBytes, (values ? maps.v : maps.k) + x.lvl, 0, x.in_row >> p8.pairs, x.kvh, x.page, &full[st]);
        };
        // (the arrival that tells the barrier of the copy's bytes; the copy itself may be ahead of it)
        auto hand_over = [&](const Batch& x, int u, int st) {
            const int e = block_exponent(x.e);
            if (lane / kGroups == u) exps[st * kGroups + lane % kGroups] = values ? (float)e : pow2i(e);
            __syncwarp();
            if (lane == 0) mbar_expect_tx(&full[st], kTileBytes);
        };
        Batch cur, nxt, far;
        next(cur, kFirst);
        next(nxt, kBatch);
        fetch(cur);
        int issued = 0, st = 0;
        uint32_t parity = 1;
        // test hook: the last tile of the share never arrives
        auto tiles_of = [&](const Batch& x, bool last) { return p.test_stall && last ? x.count - 1 : x.count; };
        const int head = tiles_of(cur, nxt.count == 0);
        for (int u = 0; u < head; ++u) copy(cur, u, u);     // (the ring is empty)
        next(far, kBatch);
        fetch(nxt);
        for (; issued < head; ++issued) hand_over(cur, issued, issued);
        st = issued;
        for (bool ok = true; ok && nxt.count > 0;) {
            cur = nxt; nxt = far;
            next(far, kBatch);
            fetch(nxt);
            const int count = tiles_of(cur, nxt.count == 0);
            for (int u = 0; u < count; ++u) {
                ok = mbar_wait_warp(&empty[st], parity, ctlp);
                if (!ok) break;
                copy(cur, u, st);
                hand_over(cur, u, st);
                ++issued;
                if (++st == kStages) { st = 0; parity ^= 1u; }
            }
        }
        // the shared memory must not be given up with a copy in flight, whoever gave up: wait (bounded) for the stages still out
        const unsigned long long t0 = gtimer();
        for (int i = issued > kStages ? issued - kStages : 0; i < issued; ++i)
            mbar_drain(&full[i % kStages], (uint32_t)(i / kStages) & 1u, ctlp, t0);
        return;
    }

    // ---------------------------------------------------------------- computing warps
    const int g = lane >> 2, t4 = lane & 3;
    const float c2 = p.scale * kLog2e;
    const int mi = lane >> 3, l7 = lane & 7;
    // Where the copy engine puts piece c (16 bytes) of row r of a tile: it swizzles the pieces over 128 bytes.  d = 128: place c ^ r % 8 of the row; d = 64: c ^ r / 2 % 4 of
    // the row, or, with two rows taken as one of 128 bytes (pairs), place (4 (r & 1) + c) ^ r / 2 % 8 of the pair.
    const bool pairs = DH == 64 && p8.pairs;
    auto piece_at = [&](int r, int c) { return pairs ? (r >> 1) * 128 + ((((r & 1) * 4 + c) ^ (r >> 1 & 7)) << 4) : r * DH + ((c ^ (DH == 128 ? r & 7 : r >> 1 & 3)) << 4); };
    // ldmatrix: a lane's row of matrices 0 .. 3, rows 0-7 and 8-15 of a piece, then of the next; pieces are (c + side) ^ swz
    const int lane_row = (mi & 1) * 8 + l7;
    const uint32_t k_row = pairs ? (lane_row >> 1) * 128 : lane_row * DH;
    const int swz = pairs ? lane_row >> 1 : (DH == 128 ? l7 : l7 >> 1), side = (mi >> 1) + (pairs ? (l7 & 1) * 4 : 0);
    int turn = warp;                                        // this warp's next tile, from the start of the list (tiles go round)
    int st = warp;                                          // ... and its stage and that barrier's parity
    uint32_t parity = 0;
    bool more = true;
    while (more) {
        const int b = walk.b, kvh = walk.kvh, first = walk.at, count = walk.segment();
        const int row_first = kChunk ? kvh % blocks * (8 * NB) : 0, G = kChunk ? min(8 * NB, GT - row_first) : GT;       // this list's rows of the KV head's
        const long long rows0 = (long long)b * p.H + (long long)(kChunk ? kvh / blocks : kvh) * GT + row_first;
        uint32_t qb[NB][KS][2];
        float row_scale[NB][2];                             // of heads 2 t4 and 2 t4 + 1: tau log2(e) over the power of two that the row's elements carry
        {
            const __nv_bfloat16* q0 = static_cast<const __nv_bfloat16*>(p.q) + rows0 * DH;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int row = nb * 8 + g;
                uint2 x[KS];
                float top = 0.f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    x[ks] = row < G ? *reinterpret_cast<const uint2*>(q0 + (long long)row * DH + 16 * ks + 4 * t4) : make_uint2(0u, 0u);
                    top = fmaxf(fmaxf(top, fmaxf(finite_abs(bf_lo(x[ks].x)), finite_abs(bf_hi(x[ks].x)))),
                                fmaxf(finite_abs(bf_lo(x[ks].y)), finite_abs(bf_hi(x[ks].y))));
                }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const int a = min(14 + 127 - (int)(__float_as_uint(top) >> 23), 120);      // (top = 0: any factor does)
                const float up = pow2i(a), own = c2 * pow2i(-a);
                row_scale[nb][0] = __shfl_sync(0xffffffffu, own, t4 * 8);
                row_scale[nb][1] = __shfl_sync(0xffffffffu, own, t4 * 8 + 4);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    qb[nb][ks][0] = pack_f16(bf_lo(x[ks].x) * up, bf_hi(x[ks].x) * up);
                    qb[nb][ks][1] = pack_f16(bf_lo(x[ks].y) * up, bf_hi(x[ks].y) * up);
                }
            }
        }
        // log2 of the gate, of the rows 2 t4 and 2 t4 + 1 where they are several tokens' (a closed level of a single token has no tiles); their places
        constexpr int kOwn = kChunk ? NB * 2 : 1;
        float bias[kOwn][3];
        int place_of[kOwn];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int token = kChunk ? (row_first + i / 2 * 8 + 2 * t4 + i % 2) % p8.T : 0;
            place_of[i] = p8.q_offset + token;
#pragma unroll
            for (int l = 0; l < 3; ++l) {
                const float gate = p.gate[((long long)b * (kChunk ? p8.T : 1) + token) * 3 + l];
                bias[i][l] = log2f(kChunk ? fmaxf(gate, 0.f) : gate);          // (negative ones and NaN close a level too, as in the tensor-core forward)
            }
        }
        // of heads 2 t4 and 2 t4 + 1.  m, mv: whole numbers not below the maxima, so that they move only when a maximum passes one
        float m[NB][2], mv[NB][2];
        uint64_t z[NB];                                     // this lane's keys
        float o[NB][KS][4];                                 // o[nb][c]: columns 16 c + 2 g, heads 2 t4 and 2 t4 + 1; then column 16 c + 2 g + 1
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m[nb][0] = m[nb][1] = mv[nb][0] = mv[nb][1] = -INFINITY;
            z[nb] = 0;
#pragma unroll
            for (int c = 0; c < KS; ++c) o[nb][c][0] = o[nb][c][1] = o[nb][c][2] = o[nb][c][3] = 0.f;
        }
        bool ok = true;
#pragma unroll 1
        for (; turn < count; turn += C) {
            ok = mbar_wait_warp(&full[st], parity, ctlp);
            if (!ok) break;
            int lvl, tile_base, rows;
            walk.locate(first + turn, lvl, tile_base, rows);
            float bl[NB][2];
#pragma unroll
            for (int i = 0; i < NB * 2; ++i) bl[i / 2][i % 2] = pick3(bias[kChunk ? i : 0], lvl);
            const int valid = rows - tile_base;             // rows of the tile that are the level's
            const int row0 = tile_base + (kChunk ? p.skip[lvl] : 0);
            // keys that some of the tokens do not see: behind the first one's place, or in front of the last one's window
            const bool partly = kChunk && lvl < 2 && (row0 + kTileRows - 1 > p8.q_offset || (lvl == 0 && row0 <= p8.q_offset + p8.T - 1 - p8.window));
            uint8_t* sK = smem + (size_t)st * 2 * kTileBytes;
            uint8_t* sV = sK + kTileBytes;
            if (valid < kTileRows) {                        // clear the value rows past the level's last row
                for (int idx = lane; idx < (kTileRows - valid) * KS; idx += 32) *reinterpret_cast<uint4*>(sV + piece_at(valid + idx / KS, idx % KS)) = make_uint4(0u, 0u, 0u, 0u);
                // (the copy engine writes the same bytes again once the stage is free, which the mbarrier alone does not order behind these stores)
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            if (kChunk && lvl == 0 && row0 < p8.from) {     // ... and those in front of every window: their weights are 0, but 0 x NaN is not
                for (int idx = lane; idx < min(p8.from - row0, kTileRows) * KS; idx += 32) *reinterpret_cast<uint4*>(sV + piece_at(idx / KS, idx % KS)) = make_uint4(0u, 0u, 0u, 0u);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            float s[kGroups][NB][4];                        // keys 16 r16 + g, heads 2 t4 and 2 t4 + 1; then keys 16 r16 + g + 8
#pragma unroll
            for (int r16 = 0; r16 < kGroups; ++r16)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) s[r16][nb][0] = s[r16][nb][1] = s[r16][nb][2] = s[r16][nb][3] = 0.f;
            {
                const uint32_t a0 = smem_u32(sK) + k_row;
#pragma unroll
                for (int ks = 0; ks < KS; ks += 2) {
#pragma unroll
                    for (int r16 = 0; r16 < kGroups; ++r16) {
                        uint32_t r[4], a[4];
                        ldmatrix_x4(a0 + r16 * 16 * DH + ((uint32_t)((ks + side) ^ swz) << 4), r);
#pragma unroll
                        for (int k1 = 0; k1 < 2; ++k1) {
                            decode4<kS8, 0>(r[2 * k1], a[0], a[2]);
                            decode4<kS8, 0>(r[2 * k1 + 1], a[1], a[3]);
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb) mma_f16(s[r16][nb], a, qb[nb][ks + k1][0], qb[nb][ks + k1][1]);
                        }
                    }
                }
            }
            float ksc[kGroups], ev[kGroups], ev_top = -INFINITY, ev_low = INFINITY;
#pragma unroll
            for (int r16 = 0; r16 < kGroups; ++r16) {
                ksc[r16] = k_scale[st][r16]; ev[r16] = v_exp[st][r16];
                ev_top = fmaxf(ev_top, ev[r16]); ev_low = fminf(ev_low, ev[r16]);
            }
            uint32_t pb[kGroups][NB][2];
            uint64_t resc[NB];
            bool moved = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                // scores without the gate, the keys' exponents and the rows' factors applied (a factor is above 0: a masked key's -inf stays)
                uint64_t x[kGroups][2];
                float top[2] = {-INFINITY, -INFINITY}, top_v[2];
#pragma unroll
                for (int r16 = 0; r16 < kGroups; ++r16) {
                    const uint64_t f = pack2(fminf(fmaxf(row_scale[nb][0] * ksc[r16], 1.2e-38f), 3.4e38f), fminf(fmaxf(row_scale[nb][1] * ksc[r16], 1.2e-38f), 3.4e38f));
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float y0 = s[r16][nb][2 * half], y1 = s[r16][nb][2 * half + 1];
                        const int key = 16 * r16 + 8 * half + g;
                        if (valid < kTileRows && key >= valid) y0 = y1 = -INFINITY;
                        if (kChunk && partly) {
                            const int p0 = place_of[nb * 2 * kChunk], p1 = place_of[nb * 2 * kChunk + kChunk];
                            if (row0 + key > p0 || (lvl == 0 && row0 + key <= p0 - p8.window)) y0 = -INFINITY;
                            if (row0 + key > p1 || (lvl == 0 && row0 + key <= p1 - p8.window)) y1 = -INFINITY;
                        }
                        x[r16][half] = mul2(pack2(y0, y1), f);
                        unpack2(x[r16][half], y0, y1);
                        top[0] = fmaxf(top[0], y0); top[1] = fmaxf(top[1], y1);
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], d));
                    top_v[h] = top[h] + ev_top;             // (no less than the largest score + ev)
                }
                if (ev_top - ev_low > 4.f) {                // far apart: exactly
                    top_v[0] = top_v[1] = -INFINITY;
#pragma unroll
                    for (int r16 = 0; r16 < kGroups; ++r16)
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            float y0, y1;
                            unpack2(x[r16][half], y0, y1);
                            top_v[0] = fmaxf(top_v[0], y0 + ev[r16]); top_v[1] = fmaxf(top_v[1], y1 + ev[r16]);
                        }
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top_v[h] = fmaxf(top_v[h], __shfl_xor_sync(0xffffffffu, top_v[h], d));
                }
                float less[2], fall[2], rs[2], to_unit[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float m_new = fmaxf(m[nb][h], ceilf(top[h] + bl[nb][h])), mv_new = fmaxf(mv[nb][h], ceilf(top_v[h] + bl[nb][h]));
                    const float sub = m_new > -INFINITY ? m_new : 0.f;
                    less[h] = bl[nb][h] - sub;
                    fall[h] = ex2(m[nb][h] - sub);          // (m = -inf: z is 0)
                    rs[h] = mv_new > -INFINITY ? ex2(mv[nb][h] - mv_new) : 1.f;
                    moved |= mv_new != mv[nb][h];
                    to_unit[h] = mv_new > -INFINITY ? sub - mv_new + 14.f : -INFINITY;
                    m[nb][h] = m_new; mv[nb][h] = mv_new;
                }
                resc[nb] = pack2(rs[0], rs[1]);
                z[nb] = mul2(z[nb], pack2(fall[0], fall[1]));
#pragma unroll
                for (int r16 = 0; r16 < kGroups; ++r16) {
                    // p 2^ev in units of 2^(mv - 14): at most 2^14, as score + ev <= mv.  The unit is at most 2^111: mv is no less than m - 49, and ev no more than 48
                    const uint64_t unit = pack2(ex2(to_unit[0] + ev[r16]), ex2(to_unit[1] + ev[r16]));
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float y0, y1;
                        unpack2(add2(x[r16][half], pack2(less[0], less[1])), y0, y1);
                        const uint64_t w = pack2(ex2(y0), ex2(y1));
                        z[nb] = add2(z[nb], w);
                        unpack2(mul2(w, unit), y0, y1);
                        pb[r16][nb][half] = transposed(pack_f16(y0, y1));
                    }
                }
            }
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int c = 0; c < KS; ++c)
#pragma unroll
                        for (int j = 0; j < 4; j += 2) unpack2(mul2(pack2(o[nb][c][j], o[nb][c][j + 1]), resc[nb]), o[nb][c][j], o[nb][c][j + 1]);
            }
            {
                const uint32_t a0 = smem_u32(sV) + k_row;
#pragma unroll
                for (int c = 0; c < KS; c += 2) {
#pragma unroll
                    for (int r16 = 0; r16 < kGroups; ++r16) {
                        uint32_t r[4], a[4];
                        ldmatrix_x4_trans(a0 + r16 * 16 * DH + ((uint32_t)((c + side) ^ swz) << 4), r);
#pragma unroll
                        for (int c1 = 0; c1 < 2; ++c1) {
                            decode4<kS8, 1>(r[2 * c1], a[0], a[1]);
                            decode4<kS8, 1>(r[2 * c1 + 1], a[2], a[3]);
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb) mma_f16(o[nb][c + c1], a, pb[r16][nb][0], pb[r16][nb][1]);
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[st]);         // the warp has read the stage
            if ((st += C) >= kStages) { st -= kStages; parity ^= 1u; }
        }
        turn -= count;
        // accumulators in units of 2^m, as the partials are; sums of all lanes' keys
        float zsum[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            unpack2(z[nb], zsum[nb][0], zsum[nb][1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float f = m[nb][h] > -INFINITY ? ex2(mv[nb][h] - m[nb][h] - 14.f) : 0.f;
#pragma unroll
                for (int c = 0; c < KS; ++c) { o[nb][c][h] *= f; o[nb][c][2 + h] *= f; }
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) zsum[nb][h] += __shfl_xor_sync(0xffffffffu, zsum[nb][h], d);
            }
        }
        // The computing warps meet at a named barrier that also carries their "no wait ran out" flags.
        {
            uint32_t out;
            asm volatile("{\n.reg .pred pi, po;\nsetp.ne.u32 pi, %1, 0;\nbar.red.and.pred po, 1, %2, pi;\nselp.u32 %0, 1, 0, po;\n}"
                         : "=r"(out) : "r"((uint32_t)ok), "n"(C * 32) : "memory");
            if (!out) {
                if (tid == 0 && p.status) atomicExch(p.status, (unsigned int)MKA_ERR_TIMEOUT);
                return;
            }
        }
        // this share is the list's partial number slot; the share with the list's first tile also says how many there are
        const long long list0 = (long long)walk.ahead * p.H_kv + (long long)kvh * walk.tiles;
        const int first_share = (int)(list0 / share), slot = (int)blockIdx.x - first_share;
        const int n_slots = (int)((list0 + walk.tiles - 1) / share) - first_share + 1;
        float* const head0 = p.partial + rows0 * list_floats;
        // The warps' states side by side; each adds up some of the columns.  (The barrier above also says that the states before have been read.)
        {
            float* const at = states + warp * kState * 32 + lane;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                for (int c = 0; c < KS; ++c)
#pragma unroll
                    for (int j = 0; j < 4; ++j) at[((nb * KS + c) * 4 + j) * 32] = o[nb][c][j];
#pragma unroll
                for (int h = 0; h < 2; ++h) { at[(kAcc + nb * 4 + h) * 32] = m[nb][h]; at[(kAcc + nb * 4 + 2 + h) * 32] = zsum[nb][h]; }
            }
        }
        asm volatile("bar.sync 1, %0;" ::"n"(C * 32) : "memory");
        const float* const at = states + lane;
#pragma unroll 1                                            // (unrolled, the loads of all heads at once spilled 500 bytes)
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const int row = nb * 8 + 2 * t4 + h;
                if (row >= G) continue;
                float f[C], mx = -INFINITY, zs = 0.f;
#pragma unroll
                for (int w = 0; w < C; ++w) { f[w] = at[(w * kState + kAcc + nb * 4 + h) * 32]; mx = fmaxf(mx, f[w]); }
#pragma unroll
                for (int w = 0; w < C; ++w) {
                    f[w] = mx > -INFINITY ? ex2(f[w] - mx) : 0.f;
                    zs = fmaf(at[(w * kState + kAcc + nb * 4 + 2 + h) * 32], f[w], zs);
                }
                float* const head = head0 + row * list_floats;
                float* const out = head + (1 + slot) * slot_floats;
                if (warp == 0 && g == 0) {
                    if (slot == 0) head[0] = (float)n_slots;
                    put_max_sum(out, mx, zs);
                }
#pragma unroll
                for (int i = 0; i < KS / C; ++i) {
                    const int c = warp * (KS / C) + i;
                    float v[2] = {0.f, 0.f};                // columns 16 c + 2 g and 16 c + 2 g + 1
#pragma unroll
                    for (int w = 0; w < C; ++w)
#pragma unroll
                        for (int j = 0; j < 2; ++j) v[j] = fmaf(at[(w * kState + (nb * KS + c) * 4 + 2 * j + h) * 32], f[w], v[j]);
                    out[2 + 16 * c + 2 * g] = v[0];         // (4 bytes each: the workspace may lie at any multiple of 4)
                    out[3 + 16 * c + 2 * g] = v[1];
                }
            }
        more = walk.advance(count);
    }
}

template <int DH, bool kS8, int NB, bool kChunk>
cudaError_t launch_t(DecodePaged8Params p8, cudaStream_t st) {
    constexpr int kTileRows = Ring<DH>::kRows;
    DecodePagedParams& p = p8.base;
    long long rows = 0;
    for (int l = 0; l < 3; ++l) rows += p.L[l].n;
    p.few = p.B <= 32 && (rows / kTileRows + 3) * p.B * p.H_kv < (1LL << 30);
    p.deal_shift = 0;
    while (((p.B - 1) >> p.deal_shift) >= kDealBlocks) ++p.deal_shift;
    // d = 64 with dense rows: two rows as one of 128 bytes.  The copy engine takes as long for a row of 64 bytes as for one of 128: 64 sequences, 32 heads on 8,
    // integer codes: 80.2 us in rows of 64 bytes.
    p8.pairs = DH == 64;
    for (int l = 0; l < 3; ++l) p8.pairs &= p.L[l].n == 0 || p.L[l].sn == DH;
    const int H_kv = p.H_kv / (kChunk ? p8.blocks : 1);
    Maps8 maps;
    int real = -1;
    for (int l = 0; l < 3; ++l) {
        const PagedLevelDev& L = p.L[l];
        if (L.n == 0) continue;
        real = l;
        const int page_rows = 1 << L.page_shift, box = page_rows < kTileRows ? page_rows : kTileRows, two = p8.pairs;
        if (!make_code_map(&maps.k[l], L.k, DH << two, page_rows >> two, H_kv, L.pool_pages, L.sn << two, L.sh, L.sp, box >> two) ||
            !make_code_map(&maps.v[l], L.v, DH << two, page_rows >> two, H_kv, L.pool_pages, L.sn << two, L.sh, L.sp, box >> two))
            return cudaErrorNotSupported;
    }
    if (real < 0) return cudaSuccess;
    for (int l = 0; l < 3; ++l) if (p.L[l].n == 0) { maps.k[l] = maps.k[real]; maps.v[l] = maps.v[real]; }     // (never asked for anything)
    const size_t smem = (size_t)Ring<DH>::kStages * 2 * Ring<DH>::kTileBytes + 1024 + C * NB * (DH / 4 + 4) * 32 * sizeof(float) + (kDealBlocks + 1) * sizeof(int);
    cudaError_t e = cudaFuncSetAttribute(decode_paged8_kernel<DH, kS8, NB, kChunk>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch_chained(decode_paged8_kernel<DH, kS8, NB, kChunk>, dim3(kDealCtas), dim3(kThreads), smem, st, 0, maps, p8);
}

// Adds up the partials where they are few and the rows many, R rows to a warp (the dense decode's combine kernel takes a CTA to a row, and asks for 32 partials
// ahead).  The counts and the first kAhead partials of all R rows are asked for together.
template <int DH, int R, int W>
__global__ void __launch_bounds__(W * 32, W == 4 ? 12 : 0) combine8_kernel(const DecodePaged8Params p8) {
    chain_enter();
    const DecodePagedParams& p = p8.base;
    const int lane = threadIdx.x & 31;
    const long long rows = (long long)p.B * p.H, row0 = ((long long)blockIdx.x * W + (threadIdx.x >> 5)) * R;
    constexpr int kSlot = DH + 2, kCols = DH / 32, kAhead = R == 1 ? 4 : 2;
    const long long list_floats = p.total_chunks * kSlot;
    const int room = (int)p.total_chunks - 1;
    float count[R], m[R], z[R], x[R][kAhead][kCols];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool real = row0 + r < rows;
        const float* const head = p.partial + (real ? row0 + r : 0) * list_floats;
        count[r] = real ? head[0] : 0.f;
        m[r] = -INFINITY; z[r] = 0.f;
        if (lane < room) { m[r] = head[(1 + lane) * kSlot]; z[r] = head[(1 + lane) * kSlot + 1]; }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int i = 0; i < kCols; ++i) x[r][u][i] = u < room ? head[(1 + u) * kSlot + 2 + lane + 32 * i] : 0.f;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const long long row = row0 + r;
        if (row >= rows) return;
        const float* const part = p.partial + row * list_floats + kSlot;
        const int total = count[r] > 0.f ? (int)fminf(count[r], (float)room) : 0;         // (a call whose waits ran out may not have written it)
        float M = -INFINITY, Z = 0.f, A[kCols] = {};
        for (int c = lane; c < total; c += 32) {
            const float mc = c == lane ? m[r] : part[c * kSlot], zc = c == lane ? z[r] : part[c * kSlot + 1];
            if (zc > 0.f) M = fmaxf(M, mc);
        }
        M = warp_max(M);
        for (int c0 = 0; M > -INFINITY && c0 < total; c0 += 32) {
            const int c = c0 + lane;
            float w = 0.f;
            if (c < total) {
                if (c0) { m[r] = part[c * kSlot]; z[r] = part[c * kSlot + 1]; }
                if (z[r] > 0.f) { w = exp2f(m[r] - M); Z = fmaf(w, z[r], Z); }
            }
            int j = 0;
            if (c0 == 0)
#pragma unroll
                for (; j < kAhead; ++j) {
                    const float wj = __shfl_sync(0xffffffffu, w, j);
#pragma unroll
                    for (int i = 0; i < kCols; ++i) A[i] = j < total ? fmaf(wj, x[r][j][i], A[i]) : A[i];
                }
            for (; j < min(32, total - c0); ++j) {
                const float wj = __shfl_sync(0xffffffffu, w, j);
#pragma unroll
                for (int i = 0; i < kCols; ++i) A[i] = fmaf(wj, part[(c0 + j) * kSlot + 2 + lane + 32 * i], A[i]);
            }
        }
        Z = warp_sum(Z);
        const bool some = Z > 0.f && !(p8.T > 0 && Z == INFINITY);                        // (several tokens: see DecodeParams::nan_is_none)
        __nv_bfloat16* const O = static_cast<__nv_bfloat16*>(p8.O) + row * DH;
#pragma unroll
        for (int i = 0; i < kCols; ++i) O[lane + 32 * i] = __float2bfloat16_rn(some ? A[i] / Z : 0.f);
        if (p8.LSE && lane == 0) p8.LSE[row] = some ? (M + log2f(Z)) * kLn2 : -INFINITY;
    }
}
template <int DH, int R, int W>
static cudaError_t launch_combine_t(const DecodePaged8Params& p, cudaStream_t st) {
    const long long rows = (long long)p.base.B * p.base.H;
    return launch_chained(combine8_kernel<DH, R, W>, dim3((unsigned)((rows + W * R - 1) / (W * R))), dim3(W * 32), 0, st, 0, p);
}
}  // namespace

template <int DH, bool kS8, bool kChunk>
static cudaError_t launch_rows(const DecodePaged8Params& p, int rows, cudaStream_t st) {
    return block_rows8(rows) == 8 ? launch_t<DH, kS8, 1, kChunk>(p, st) : launch_t<DH, kS8, 2, kChunk>(p, st);
}
template <bool kChunk>
static cudaError_t launch_d(const DecodePaged8Params& p, int rows, cudaStream_t st) {
    if (p.base.d == 128) return p.s8 ? launch_rows<128, true, kChunk>(p, rows, st) : launch_rows<128, false, kChunk>(p, rows, st);
    return p.s8 ? launch_rows<64, true, kChunk>(p, rows, st) : launch_rows<64, false, kChunk>(p, rows, st);
}

cudaError_t launch_decode_paged8(const DecodePaged8Params& p, cudaStream_t st) { return launch_d<false>(p, p.base.H / p.base.H_kv, st); }
// A few tokens at once (a verified draft): the rows of a KV head, heads x tokens, in blocks of up to sixteen, each of which walks the keys.
cudaError_t launch_chunk_paged8(const DecodePaged8Params& p, cudaStream_t st) { return launch_d<true>(p, p.base.H / (p.base.H_kv / p.blocks), st); }

// What counts is how many rows' warps find registers beside two of the decode's CTAs.  At d = 64 eight warps to an SM do: up to two rows to a warp then let all of them start
// there (one row / two, 32 heads on 8: 1216 rows 43.8 / 44.5 us, 1536 54.8 / 51.8, 2048 66.7 / 63.2, 2336 73.9 / 70.6, 2368 70.7 / 70.1; 8 on 2: 1216 25.2 / 25.8, 1536 30.9 / 28.9,
// 2048 39.3 / 37.4, 2368 41.1 / 40.2; four rows to a warp lost 3 to 10).  At d = 128 four warps of 40 registers do: 288 rows 35.5 -> 33.8 us, 512 36.3 -> 35.9, but 1120 39.2 -> 40.5
// and 14,336 58.1 -> 60.4, where the warps without that limit are faster.
cudaError_t launch_combine8(const DecodePaged8Params& p, cudaStream_t st) {
    const long long rows = (long long)p.base.B * p.base.H;
    if (p.base.d == 128) return rows <= 148 * 4 ? launch_combine_t<128, 1, 4>(p, st) : launch_combine_t<128, 1, 8>(p, st);
    return rows > 148 * 8 && rows <= 148 * 16 ? launch_combine_t<64, 2, 8>(p, st) : launch_combine_t<64, 1, 8>(p, st);
}

}  // namespace mka
