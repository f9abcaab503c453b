// C-ABI entry points of the 8-bit paged cache and of the page tables: host-side validation, workspace layout, dispatch.  See include/mka.h.
#include <string.h>

#include "common.cuh"
#include "tc_ptx.cuh"

using namespace mka;

namespace {

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool power_of_two(int x) { return x > 0 && (x & (x - 1)) == 0; }
inline int log2_of(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

// What attention and append ask of a level alike.
mka_status check_level8(const mka_paged_level8& L, int d, int H_kv) {
    if (!L.k || !L.v || !L.k_exp || !L.v_exp || !L.page_table) return MKA_ERR_ARG;
    if (L.code != MKA_CODE_E4M3 && L.code != MKA_CODE_S8) return MKA_ERR_ARG;
    if (!power_of_two(L.page_rows) || !power_of_two(L.block_rows) || L.block_rows < 16 || L.block_rows > 256 || L.page_rows < L.block_rows) return MKA_ERR_SHAPE;
    if (L.pool_pages <= 0 || L.pool_pages > 0x7fffffffLL || L.table_stride < 0 || L.table_head_stride < 0) return MKA_ERR_SHAPE;
    if (L.stride_n < d || L.stride_page <= 0 || L.stride_h < 0 || (H_kv > 1 && L.stride_h <= 0)) return MKA_ERR_SHAPE;
    if (L.exp_stride_page < 0 || L.exp_stride_h < 0) return MKA_ERR_SHAPE;
    if (!aligned(L.k, 16) || !aligned(L.v, 16) || L.stride_n % 16 || L.stride_page % 16 || L.stride_h % 16) return MKA_ERR_ALIGN;
    return MKA_OK;
}
mka_status check_levels8(const mka_shape* s, int H_kv, const mka_paged_level8 L[3], int& code) {
    if (!L) return MKA_ERR_ARG;
    code = -1;
    for (int l = 0; l < 3; ++l) {
        if (L[l].n < 0 || L[l].n > 0x7fffffffLL) return MKA_ERR_SHAPE;
        if (L[l].n == 0) continue;
        const mka_status st = check_level8(L[l], s->d, H_kv);
        if (st != MKA_OK) return st;
        const int64_t width = L[l].table_head_stride > 0 ? L[l].table_head_stride : L[l].table_stride;
        if (width < (L[l].n + L[l].page_rows - 1) / L[l].page_rows) return MKA_ERR_SHAPE;
        if (code >= 0 && code != L[l].code) return MKA_ERR_UNSUPPORTED;
        code = L[l].code;
    }
    return MKA_OK;
}
mka_status check_shape8(const mka_shape* s, int H_kv, bool decode) {
    if (!s) return MKA_ERR_ARG;
    if (s->dtype != MKA_BF16 && s->dtype != MKA_F32) return MKA_ERR_ARG;
    if (s->mode != MKA_MODE_FAST && s->mode != MKA_MODE_FULL) return MKA_ERR_ARG;
    if (s->dtype != MKA_BF16 || s->mode != MKA_MODE_FAST || (s->flags & MKA_FLAG_FORCE_SIMT)) return MKA_ERR_UNSUPPORTED;
    if (s->B < 0 || s->H < 0 || s->T < 0 || (s->d != 64 && s->d != 128)) return MKA_ERR_SHAPE;
    if (decode ? s->T != 1 : (s->window < 1 || s->q_offset < 0)) return MKA_ERR_SHAPE;
    if (H_kv <= 0 || s->H % H_kv != 0 || (decode && s->H / H_kv > 16)) return MKA_ERR_SHAPE;
    if (s->B > 65535 || s->H > 65535 || (int64_t)s->B * s->H > 0x7fffffffLL) return MKA_ERR_SHAPE;
    return MKA_OK;
}
float resolve_scale(const mka_shape* s) { return s->scale > 0.f ? s->scale : 1.0f / sqrtf((float)s->d); }
mka_status status_of(cudaError_t e) { return e == cudaSuccess ? MKA_OK : (e == cudaErrorNotSupported ? MKA_ERR_UNSUPPORTED : MKA_ERR_CUDA); }

// Entries per query head of the decode's partials: a count, and one for every share that a list can touch.  The H_kv lists of one sequence are
// equally long, so a share (all tiles / 296, at least two) is no less than H_kv / 296 of a list.
int64_t decode8_tiles(const int64_t n_level[3], int32_t d) {
    int64_t tiles = 0;
    for (int l = 0; l < 3; ++l) tiles += (n_level[l] + tile_rows8(d) - 1) / tile_rows8(d);
    return tiles;
}
int64_t decode8_slots(const int64_t n_level[3], int32_t H_kv, int32_t d) {
    const int64_t tiles = decode8_tiles(n_level, d);
    const int64_t by_share = kDealCtas / H_kv + 2, by_list = tiles / 2 + 2;
    return 1 + (by_share < by_list ? by_share : by_list);
}

// Which kernel adds them up: a warp to a row (launch_combine8) where a list of a batch of equal lengths has up to three of them (more than 98 lists), the dense decode's CTA
// to a row else.  Dense decode's / this one, us, 600,000 rows in all, by lists:
//   28 on 4, d = 128    64  37.0 / 37.7    148  39.1 / 38.6    296  40.0 / 37.3    512  45.6 / 41.1    2048  77.9 / 57.9
//   16 on 16, d = 128   64  34.3 / 36.0    144  34.3 / 33.6    288  34.9 / 34.1    512  37.1 / 36.2    2048  49.5 / 47.8
//   8 on 1, d = 64      4  43.8 / 54.6    104  41.2 / 36.3    296  40.4 / 37.3    512  44.6 / 42.8    2048  71.3 / 59.9
//   32 on 8, d = 64     64  34.1 / 35.1    104  37.7 / 34.4    296  36.6 / 34.4    512  39.2 / 38.4    2048  54.9 / 50.0
bool few_partials(int64_t lists) { return kDealCtas / lists + 1 <= 3; }
void fill_levels8(DecodePaged8Params& p, const mka_paged_level8 L[3], const int64_t n[3]) {
    for (int l = 0; l < 3; ++l) {
        if (n[l] == 0) continue;
        PagedLevelDev& x = p.base.L[l];
        x.k = L[l].k; x.v = L[l].v; x.table = L[l].page_table; x.rows = L[l].rows; x.n = n[l];
        x.table_stride = L[l].table_stride; x.table_head_stride = L[l].table_head_stride;
        x.sp = L[l].stride_page; x.sh = L[l].stride_h; x.sn = L[l].stride_n;
        x.pool_pages = L[l].pool_pages; x.page_shift = log2_of(L[l].page_rows);
        p.k_exp[l] = L[l].k_exp; p.v_exp[l] = L[l].v_exp; p.esp[l] = L[l].exp_stride_page; p.esh[l] = L[l].exp_stride_h;
        p.block_shift[l] = log2_of(L[l].block_rows);
    }
}

// Rows of the levels that a chunk can see: [lo, hi).
bool visible8(const mka_shape* s, const int64_t n_level[3], int64_t (&lo)[3], int64_t (&hi)[3]) {
    for (int l = 0; l < 3; ++l) {
        if (n_level[l] < 0 || n_level[l] > 0x7fffffffLL) return false;
        const int64_t last = (int64_t)s->q_offset + s->T;                 // rows in front of it are visible to some row of the chunk
        lo[l] = 0;
        hi[l] = l < 2 && n_level[l] > last ? last : n_level[l];
        if (l == 0 && (int64_t)s->q_offset - s->window + 1 > 0) lo[l] = (int64_t)s->q_offset - s->window + 1;
        if (hi[l] <= lo[l]) lo[l] = hi[l] = 0;
    }
    return true;
}

// Few tokens go through the single-token kernel, in blocks of up to sixteen rows (heads x tokens of a KV head) that each walk the keys.  Every block reads the codes again,
// mostly from the L2 cache; the other way costs the expansion, and tiles of 128 rows whatever the rows.  Over 612 sizes (4 to 100 tokens on 100 to 60,000 rows of
// context, heads 28 on 4, 32 on 8, 16 on 16 and 8 on 1, one or four sequences, pages and blocks of 32 rows) the pick takes 1.0 % more than the better one on
// average, 66 % at most (8 on 1, 24 tokens at 15,000 rows).  This way / through the forward, us, chosen in brackets, at d = 128:
//   28 on 4, 15,000 rows, 4 / 16 / 32 tokens      [28.2] / 59.9    [53.9] / 60.9    86.7 / [61.0]      (pages of 16 rows: 4 tokens 23.1, 8 32.8, 16 53.7)
//   16 on 16, 15,000 rows, 24 / 64 / 100          [59.2] / 99.9    101 / [104]      161 / [105]
//   8 on 1, 1000 rows, 4 / 64                     [12.9] / 17.5    23.1 / [21.0]
//   d = 64, 28 on 4, 15,000 rows, 8 / 16 tokens   [39.5] / 49.0    52.2 / [49.4]
constexpr int kMaxChunkRows = 512;
bool walk_in_blocks(int d, int64_t blocks, int group, double mbytes) {
    return blocks == 1 || (double)blocks * mbytes < (d == 128 ? 3.0 + (2.5 + 0.7 * group) * mbytes : 1.0 + 0.8 * group * mbytes);
}
struct Chunk8 {
    int blocks;                      // to a KV head; 0: the tensor-core forward
    int64_t lo, hi[3], skip[3];
    size_t total;
};
bool chunk8_layout(const mka_shape* s, int H_kv, const int64_t n_level[3], Chunk8& c) {
    int64_t lo[3], span[3];
    if (!visible8(s, n_level, lo, c.hi)) return false;
    const int64_t rows = s->H / H_kv * (int64_t)s->T;
    c.blocks = 0;
    if (rows > kMaxChunkRows || rows == 0) return true;
    const int64_t blocks = (rows + block_rows8((int)rows) - 1) / block_rows8((int)rows);
    if (blocks * H_kv > 65535 || (int64_t)s->B * s->H * s->T > 0x7fffffffLL || (int64_t)s->q_offset + s->T > 0x7fffffffLL) return true;
    for (int l = 0; l < 3; ++l) {
        c.skip[l] = lo[l] / 64 * 64;
        span[l] = c.hi[l] - c.skip[l];
    }
    c.lo = lo[0];
    double mbytes = 0.0;                                     // of codes that the chunk sees
    for (int l = 0; l < 3; ++l) mbytes += (double)span[l] * s->B * H_kv * (2e-6 * s->d);
    if (!walk_in_blocks(s->d, blocks, s->H / H_kv, mbytes) || !deal_fits(s->B, blocks * H_kv, decode8_tiles(span, s->d))) return true;
    c.blocks = (int)blocks;
    c.total = kWsHeader + (size_t)s->B * s->H * s->T * (size_t)decode8_slots(span, (int)(blocks * H_kv), s->d) * (s->d + 2) * sizeof(float);
    return true;
}

// The forward's workspace: header | tables | keys and values of the visible rows, level by level | scratch of the forward, as much as is left.
struct Fwd8Layout {
    int64_t lo[3], hi[3];            // the visible rows of each level
    int first[3], count[3];          // pages of 128 rows that hold visible ones
    size_t table[3], k[3], v[3], scratch;
};
bool fwd8_layout(const mka_shape* s, int H_kv, const int64_t n_level[3], Fwd8Layout& w) {
    size_t at = kWsHeader;
    if (!visible8(s, n_level, w.lo, w.hi)) return false;
    for (int l = 0; l < 3; ++l) {
        w.first[l] = (int)(w.lo[l] / 128);
        w.count[l] = w.hi[l] > 0 ? (int)((w.hi[l] + 127) / 128) - w.first[l] : 0;
        if ((int64_t)s->B * w.count[l] > 0x7fffffffLL) return false;
        const size_t bytes = (size_t)s->B * w.count[l] * H_kv * 128 * s->d * 2;
        w.table[l] = at; at += round_up((size_t)s->B * (w.first[l] + w.count[l]) * 4, 256);
        w.k[l] = at; at += bytes;
        w.v[l] = at; at += bytes;
    }
    w.scratch = at;
    return true;
}

// What serves a chunk and every one that is nowhere larger (sequences, tokens, q_offset, window, rows of the levels), whichever way each of them goes.  Neither way's own need
// grows with every size: the window's rows touch one page more or less by where they lie, partials get fewer where the blocks get more, and a shorter
// context may go through the single-token kernel where a longer one is expanded.
size_t fwd8_most(const mka_shape* s, int H_kv, const int64_t n_level[3]) {
    int64_t lo[3], hi[3], span[3];
    if (!visible8(s, n_level, lo, hi)) return 0;
    const int64_t last = (int64_t)s->q_offset + s->T, wide = (int64_t)s->window + s->T - 1;          // rows that windows cover together
    size_t expand = kWsHeader + fwd_tc_scratch_most(s->d);
    double mbytes = 0.0;
    for (int l = 0; l < 3; ++l) {
        hi[l] = l < 2 && n_level[l] > last ? last : n_level[l];
        int64_t pages = (hi[l] + 127) / 128;
        span[l] = hi[l];
        if (l == 0) {                                        // `wide` rows lie in so many pages at most, and with the rest of a block of 64 in front of them are so many
            if (pages > (wide + 126) / 128 + 1) pages = (wide + 126) / 128 + 1;
            if (span[l] > wide + 63) span[l] = wide + 63;
        }
        if ((int64_t)s->B * pages > 0x7fffffffLL) return 0;
        expand += round_up((size_t)s->B * ((hi[l] + 127) / 128) * 4, 256) + 2 * (size_t)s->B * pages * H_kv * 128 * s->d * 2;
        mbytes += (double)span[l] * s->B * H_kv * (2e-6 * s->d);
    }
    const int64_t rows = s->H / H_kv * (int64_t)s->T;
    size_t walk = kWsHeader;
    for (int64_t b = 1; 16 * (b - 1) < rows && 16 * (b - 1) < kMaxChunkRows && b * H_kv <= 65535; ++b) {
        const int64_t here = 16 * b < rows ? 16 * b : rows;
        const size_t bytes = kWsHeader + (size_t)s->B * H_kv * here * (size_t)decode8_slots(span, (int)(b * H_kv), s->d) * (s->d + 2) * sizeof(float);
        if (bytes > walk) walk = bytes;
    }
    const int64_t blocks = (rows + 15) / 16;
    const bool all_walk = rows <= kMaxChunkRows && blocks * H_kv <= 65535 && (int64_t)s->B * s->H * s->T <= 0x7fffffffLL && last <= 0x7fffffffLL &&
                          (rows == 0 || (walk_in_blocks(s->d, blocks, s->H / H_kv, mbytes) && deal_fits(s->B, blocks * H_kv, decode8_tiles(span, s->d))));
    return all_walk || walk > expand ? walk : expand;
}

mka_status check_tables(const mka_page_tables* t) {
    if (!t) return MKA_ERR_ARG;
    if (t->pages < 0 || t->pages > 0x7fffff00LL || t->seqs < 0 || t->width < 0 || t->width > 0x7ff00000 || t->table_stride < t->width || t->page_rows <= 0) return MKA_ERR_SHAPE;
    return MKA_OK;
}
mka_status check_planes(const mka_page_plane* planes, int n, int64_t pages, CopyPagesParams& c) {
    if (n < 0 || n > kMaxPlanes) return MKA_ERR_SHAPE;
    if (n > 0 && !planes) return MKA_ERR_ARG;
    memset(&c, 0, sizeof(c));
    for (int j = 0; j < n; ++j) {
        const mka_page_plane& x = planes[j];
        if (x.heads < 0 || x.bytes < 0 || x.stride_page < 0 || x.stride_h < 0) return MKA_ERR_SHAPE;
        if (x.heads == 0 || x.bytes == 0 || pages == 0) continue;
        if (!x.base) return MKA_ERR_ARG;
        c.plane[c.planes++] = {static_cast<char*>(x.base), x.stride_page, x.stride_h, x.heads, x.bytes};
    }
    return MKA_OK;
}
void fill_tables(PagesParams& p, const mka_page_tables* t) {
    memset(&p, 0, sizeof(p));
    p.refs = t->refs; p.table = t->table; p.rows = t->rows;
    p.table_stride = t->table_stride;
    p.pages = (int)t->pages; p.seqs = t->seqs; p.width = t->width; p.page_rows = t->page_rows;
}
void fill_scratch(PagesParams& p, void* ws) {
    int* w = reinterpret_cast<int*>(static_cast<char*>(ws) + kWsHeader);
    const size_t pairs = p.pages > p.seqs ? p.pages : p.seqs;
    p.count = static_cast<int*>(ws);
    p.list = w; w += p.pages;
    p.src = w; w += pairs;
    p.dst = w;
}

}  // namespace

extern "C" {

mka_status mka_append_kv_paged8(int32_t B, int32_t H, int64_t n, int32_t d, int32_t dtype, const mka_level* src, const mka_paged_level8* dst,
                                int64_t dst_offset, const int32_t* dst_offsets, void* stream) {
    if (dtype != MKA_BF16 && dtype != MKA_F32) return MKA_ERR_ARG;
    if (!src || !dst) return MKA_ERR_ARG;
    if (B < 0 || H < 0 || n < 0 || n > 0x7fffffffLL || dst_offset < 0) return MKA_ERR_SHAPE;
    if (d != 64 && d != 128) return MKA_ERR_SHAPE;
    if (src->n != n) return MKA_ERR_SHAPE;
    if (B == 0 || H == 0 || n == 0) return MKA_OK;
    const mka_status st = check_level8(*dst, d, H);
    if (st != MKA_OK) return st;
    if (dst->n < 0 || (dst->table_stride < (dst->n + dst->page_rows - 1) / dst->page_rows)) return MKA_ERR_SHAPE;
    if (dst_offset > 0x7fffffffffffLL || (!dst_offsets && dst->n < dst_offset + n)) return MKA_ERR_SHAPE;
    const int elems = dtype == MKA_BF16 ? 8 : 4;
    if (!src->k || !src->v) return MKA_ERR_ARG;
    if (src->stride_n < d || src->stride_b < 0 || src->stride_h < 0) return MKA_ERR_SHAPE;
    if (!aligned(src->k, 16) || !aligned(src->v, 16) || src->stride_n % elems || src->stride_b % elems || src->stride_h % elems) return MKA_ERR_ALIGN;
    Append8Params p;
    memset(&p, 0, sizeof(p));
    p.k = src->k; p.v = src->v; p.sb = src->stride_b; p.sh = src->stride_h; p.sn = src->stride_n;
    p.pool_k = static_cast<uint8_t*>(dst->k); p.pool_v = static_cast<uint8_t*>(dst->v); p.k_exp = dst->k_exp; p.v_exp = dst->v_exp;
    p.table = dst->page_table; p.offsets = dst_offsets;
    p.n = n; p.dst_offset = dst_offset; p.table_stride = dst->table_stride; p.rows_held = dst->n;
    p.pool_sp = dst->stride_page; p.pool_sh = dst->stride_h; p.pool_sn = dst->stride_n; p.esp = dst->exp_stride_page; p.esh = dst->exp_stride_h;
    p.B = B; p.H = H; p.d = d; p.page_shift = log2_of(dst->page_rows); p.block_shift = log2_of(dst->block_rows);
    p.pool_pages = (int)dst->pool_pages; p.s8 = dst->code == MKA_CODE_S8;
    return status_of(launch_append8(p, dtype, static_cast<cudaStream_t>(stream)));
}

size_t mka_decode_paged8_workspace_bytes(const mka_shape* s, int32_t H_kv, const int64_t n_level[3]) {
    if (!s || !n_level || H_kv <= 0 || s->B < 0 || s->H < 0 || s->d <= 0) return 0;
    for (int l = 0; l < 3; ++l) if (n_level[l] < 0) return 0;
    return kWsHeader + (size_t)s->B * s->H * (size_t)decode8_slots(n_level, H_kv, s->d) * (s->d + 2) * sizeof(float);
}

mka_status mka_decode_paged8(const mka_shape* s, int32_t H_kv, const void* q, const mka_paged_level8 L[3], const float* gate, void* O, float* LSE,
                             void* ws, size_t ws_bytes, void* stream) {
    mka_status st = check_shape8(s, H_kv, true);
    if (st != MKA_OK) return st;
    int code;
    if ((st = check_levels8(s, H_kv, L, code)) != MKA_OK) return st;
    if (s->B == 0 || s->H == 0) return MKA_OK;
    if (!q || !gate || !O) return MKA_ERR_ARG;
    if (!aligned(q, 16) || !aligned(O, 16) || !aligned(ws, 4)) return MKA_ERR_ALIGN;
    const int64_t n_level[3] = {L[0].n, L[1].n, L[2].n};
    if (!deal_fits(s->B, H_kv, decode8_tiles(n_level, s->d))) return MKA_ERR_SHAPE;
    if (!ws || ws_bytes < mka_decode_paged8_workspace_bytes(s, H_kv, n_level)) return MKA_ERR_WORKSPACE;
    DecodePaged8Params p;
    memset(&p, 0, sizeof(p));
    fill_levels8(p, L, n_level);
    p.s8 = code == MKA_CODE_S8;
    p.base.q = q; p.base.gate = gate;
    p.base.B = s->B; p.base.H = s->H; p.base.H_kv = H_kv; p.base.d = s->d; p.base.scale = resolve_scale(s);
    p.base.test_stall = (s->flags & MKA_FLAG_TEST_STALL) ? 1 : 0;
    p.base.total_chunks = decode8_slots(n_level, H_kv, s->d);
    p.base.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + kWsHeader);
    p.base.status = static_cast<unsigned int*>(ws); p.base.wait_limit_ns = wait_limit_ns();
    DecodeParams c;                                    // the combine kernel of the dense decode finishes the job
    memset(&c, 0, sizeof(c));
    c.O = O; c.LSE = LSE; c.gate = gate; c.B = s->B; c.H = s->H; c.d = s->d;
    c.partial = p.base.partial; c.total_chunks = p.base.total_chunks;
    const bool any = code >= 0;                        // (no level with rows: only the combine kernel runs, over no partials)
    c.counted = any ? 1 : 0;
    c.expected = (int)(kDealCtas / ((int64_t)s->B * H_kv)) + 1;
    if (!any) { c.total_chunks = 0; c.status = p.base.status; }
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    p.O = O; p.LSE = LSE;
    cudaError_t e = any ? launch_decode_paged8(p, cs) : cudaSuccess;
    if (e == cudaSuccess) e = any && few_partials((int64_t)s->B * H_kv) ? launch_combine8(p, cs) : launch_decode_combine(c, cs);
    return status_of(e);
}

static mka_status run_chunk8(const mka_shape* s, int32_t H_kv, const void* Q, const mka_paged_level8 L[3], const float* gate, void* O, float* LSE, void* ws,
                             const Chunk8& k, bool s8, cudaStream_t cs) {
    DecodePaged8Params p;
    memset(&p, 0, sizeof(p));
    fill_levels8(p, L, k.hi);
    int64_t span[3];
    bool any = false;
    for (int l = 0; l < 3; ++l) {
        p.base.skip[l] = (int)k.skip[l];
        span[l] = k.hi[l] - k.skip[l];
        any |= k.hi[l] > 0;
    }
    p.s8 = s8; p.T = s->T; p.window = s->window; p.q_offset = s->q_offset; p.blocks = k.blocks; p.from = (int)k.lo;
    p.base.q = Q; p.base.gate = gate;
    p.base.B = s->B; p.base.H = s->H * s->T; p.base.H_kv = H_kv * k.blocks; p.base.d = s->d; p.base.scale = resolve_scale(s);
    p.base.test_stall = (s->flags & MKA_FLAG_TEST_STALL) ? 1 : 0;
    p.base.total_chunks = decode8_slots(span, H_kv * k.blocks, s->d);
    p.base.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + kWsHeader);
    p.base.status = static_cast<unsigned int*>(ws); p.base.wait_limit_ns = wait_limit_ns();
    DecodeParams c;
    memset(&c, 0, sizeof(c));
    c.O = O; c.LSE = LSE; c.gate = gate; c.B = s->B; c.H = p.base.H; c.d = s->d;
    c.partial = p.base.partial; c.total_chunks = any ? p.base.total_chunks : 0; c.counted = any ? 1 : 0;
    c.expected = (int)(kDealCtas / ((int64_t)s->B * p.base.H_kv)) + 1;
    c.nan_is_none = 1;
    if (!any) c.status = p.base.status;
    p.O = O; p.LSE = LSE;
    cudaError_t e = any ? launch_chunk_paged8(p, cs) : cudaSuccess;
    if (e == cudaSuccess) e = any && few_partials((int64_t)s->B * p.base.H_kv) ? launch_combine8(p, cs) : launch_decode_combine(c, cs);
    return status_of(e);
}

size_t mka_fwd_paged8_workspace_bytes(const mka_shape* s, int32_t H_kv, const int64_t n_level[3]) {
    if (!n_level || check_shape8(s, H_kv, false) != MKA_OK) return 0;
    return fwd8_most(s, H_kv, n_level);
}

mka_status mka_fwd_paged8(const mka_shape* s, int32_t H_kv, const void* Q, const mka_paged_level8 L[3], const float* gate, void* O, float* LSE,
                          void* ws, size_t ws_bytes, void* stream) {
    mka_status st = check_shape8(s, H_kv, false);
    if (st != MKA_OK) return st;
    int code;
    if ((st = check_levels8(s, H_kv, L, code)) != MKA_OK) return st;
    if (s->B == 0 || s->H == 0 || s->T == 0) return MKA_OK;
    if (!Q || !gate || !O) return MKA_ERR_ARG;
    if (!aligned(Q, 16) || !aligned(O, 16) || !aligned(ws, 256)) return MKA_ERR_ALIGN;
    const int64_t n_level[3] = {L[0].n, L[1].n, L[2].n};
    Chunk8 k;
    if (!chunk8_layout(s, H_kv, n_level, k)) return MKA_ERR_SHAPE;
    if (k.blocks) {
        if (!ws || ws_bytes < k.total) return MKA_ERR_WORKSPACE;
        return run_chunk8(s, H_kv, Q, L, gate, O, LSE, ws, k, code == MKA_CODE_S8, static_cast<cudaStream_t>(stream));
    }
    Fwd8Layout w;
    if (!fwd8_layout(s, H_kv, n_level, w)) return MKA_ERR_SHAPE;
    if (!ws || ws_bytes < w.scratch) return MKA_ERR_WORKSPACE;
    if ((double)((s->T + 127LL) / 128) * s->H * s->B > 2147483647.0) return MKA_ERR_SHAPE;     // the kernel numbers its blocks in an int
    char* const base = static_cast<char*>(ws);
    Expand8Params x;
    memset(&x, 0, sizeof(x));
    x.B = s->B; x.H_kv = H_kv; x.d = s->d; x.s8 = code == MKA_CODE_S8;
    FwdParams p;
    memset(&p, 0, sizeof(p));
    PagedLevelDev P[3];
    memset(P, 0, sizeof(P));
    for (int l = 0; l < 3; ++l) {
        if (w.count[l] == 0) continue;                 // no row, or none that the chunk can see
        Expand8Level& X = x.L[l];
        X.k = static_cast<const uint8_t*>(L[l].k); X.v = static_cast<const uint8_t*>(L[l].v); X.k_exp = L[l].k_exp; X.v_exp = L[l].v_exp;
        X.table = L[l].page_table; X.rows = L[l].rows; X.n = L[l].n;
        X.table_stride = L[l].table_stride; X.table_head_stride = L[l].table_head_stride;
        X.sp = L[l].stride_page; X.sh = L[l].stride_h; X.sn = L[l].stride_n; X.esp = L[l].exp_stride_page; X.esh = L[l].exp_stride_h;
        X.page_shift = log2_of(L[l].page_rows); X.block_shift = log2_of(L[l].block_rows); X.pool_pages = (int)L[l].pool_pages;
        X.first = w.first[l]; X.count = w.count[l]; X.from = w.lo[l];
        X.out_k = reinterpret_cast<__nv_bfloat16*>(base + w.k[l]); X.out_v = reinterpret_cast<__nv_bfloat16*>(base + w.v[l]);
        X.out_table = reinterpret_cast<int*>(base + w.table[l]);
        p.L[l].n = w.hi[l];
        P[l].k = X.out_k; P[l].v = X.out_v; P[l].table = X.out_table; P[l].rows = L[l].rows; P[l].n = w.hi[l];
        P[l].table_stride = w.first[l] + w.count[l];
        P[l].sn = s->d; P[l].sh = 128LL * s->d; P[l].sp = (long long)H_kv * 128 * s->d;
        P[l].pool_pages = (long long)s->B * w.count[l]; P[l].page_shift = 7;
    }
    p.Q = Q; p.O = O; p.LSE = LSE; p.gate = gate;
    p.B = s->B; p.H = s->H; p.T = s->T; p.d = s->d;
    p.window = s->window; p.q_offset = s->q_offset; p.scale = resolve_scale(s);
    p.mode = s->mode; p.kv_group = s->H / H_kv; p.paged = P;
    if (ws_bytes > w.scratch) { p.scratch = base + w.scratch; p.scratch_bytes = ws_bytes - w.scratch; }
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    cudaError_t e = launch_expand8(x, cs);
    if (e == cudaSuccess) e = launch_fwd_tc(p, static_cast<unsigned int*>(ws), cs);
    return status_of(e);
}

size_t mka_pages_workspace_bytes(int64_t pages, int32_t seqs) {
    if (pages < 0 || pages > 0x7fffff00LL || seqs < 0) return 0;
    const size_t pairs = pages > seqs ? (size_t)pages : (size_t)seqs;
    return kWsHeader + 4 * ((size_t)pages + 2 * pairs);
}

mka_status mka_pages_resize(const mka_page_tables* t, const mka_page_plane* planes, int32_t n_planes, const int32_t* new_rows, int32_t* missing,
                            void* ws, size_t ws_bytes, void* stream) {
    mka_status st = check_tables(t);
    if (st != MKA_OK) return st;
    CopyPagesParams c;
    if ((st = check_planes(planes, n_planes, t->pages, c)) != MKA_OK) return st;
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    if (t->seqs == 0) return missing && cudaMemsetAsync(missing, 0, 4, cs) != cudaSuccess ? MKA_ERR_CUDA : MKA_OK;
    if (t->seqs > kMaxSeqs) return MKA_ERR_SHAPE;
    if ((!t->refs && t->pages > 0) || (!t->table && t->width > 0) || !t->rows || !new_rows) return MKA_ERR_ARG;
    if (!aligned(ws, 4)) return MKA_ERR_ALIGN;
    if (!ws || ws_bytes < mka_pages_workspace_bytes(t->pages, t->seqs)) return MKA_ERR_WORKSPACE;
    PagesParams p;
    fill_tables(p, t);
    fill_scratch(p, ws);
    p.new_rows = new_rows; p.missing = missing;
    p.copies = c.planes > 0;
    return status_of(launch_pages_resize(p, c, cs));
}

mka_status mka_pages_fork(const mka_page_tables* t, const int32_t* parents, const int32_t* children, int32_t n, void* stream) {
    const mka_status st = check_tables(t);
    if (st != MKA_OK) return st;
    if (n < 0) return MKA_ERR_SHAPE;
    if (n == 0 || t->seqs == 0) return MKA_OK;
    if ((!t->refs && t->pages > 0) || (!t->table && t->width > 0) || !t->rows || !parents || !children) return MKA_ERR_ARG;
    PagesParams p;
    fill_tables(p, t);
    p.parents = parents; p.children = children; p.n = n;
    return status_of(launch_pages_fork(p, static_cast<cudaStream_t>(stream)));
}

mka_status mka_pages_compact(const mka_page_tables* t, const mka_page_plane* planes, int32_t n_planes, int32_t* refs_out, int32_t* table_out,
                             int64_t table_out_stride, int32_t* remap, int32_t* live, void* ws, size_t ws_bytes, void* stream) {
    mka_status st = check_tables(t);
    if (st != MKA_OK) return st;
    CopyPagesParams c;
    if ((st = check_planes(planes, n_planes, t->pages, c)) != MKA_OK) return st;
    if (table_out_stride < t->width) return MKA_ERR_SHAPE;
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    const bool tables = t->seqs > 0 && t->width > 0;         // (of an empty pool too: table_out receives their entries as they are)
    if (t->pages == 0 && !tables) return live && cudaMemsetAsync(live, 0, 4, cs) != cudaSuccess ? MKA_ERR_CUDA : MKA_OK;
    if (t->pages > 0 && (!t->refs || !refs_out || !remap)) return MKA_ERR_ARG;
    if (t->seqs > 0 && (!t->rows || (t->width > 0 && (!t->table || !table_out)))) return MKA_ERR_ARG;
    if (!aligned(ws, 4)) return MKA_ERR_ALIGN;
    if (!ws || ws_bytes < mka_pages_workspace_bytes(t->pages, t->seqs)) return MKA_ERR_WORKSPACE;
    PagesParams p;
    fill_tables(p, t);
    fill_scratch(p, ws);
    p.refs_out = refs_out; p.table_out = table_out; p.table_out_stride = table_out_stride; p.remap = remap; p.live = live;
    return status_of(launch_pages_compact(p, c, cs));
}

}  // extern "C"
