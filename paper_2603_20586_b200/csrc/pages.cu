// Pages of a paged cache: which of them are in use (reference counts), and the sequences' tables.
//
// All of it is whole numbers, decided on the device without the host looking on, and the same every time: pages are taken lowest first, in the order of
// the sequences.  The counts are few bytes (4 per page); what bounds a plan is the number of times its threads must agree, so one
// cluster of eight CTAs makes it, meeting at cluster barriers instead of ends of kernels.  A warp owns a
// stretch of the pool: ballots give its free pages, shuffles and one exchange through distributed shared memory the place of each among
// all.  What the plan says to copy is copied by a second kernel over the whole chip, bound by HBM at twice the pages' bytes.
#include "tc_ptx.cuh"

namespace mka {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kChunk = 256;                                              // table entries that a warp takes at a time

template <int kC> __device__ __forceinline__ int cluster_rank() {
    if (kC == 1) return 0;
    int r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// (meet, of_rank: with one CTA a barrier of the CTA and its own shared memory)
template <int kC> __device__ __forceinline__ void meet() {
    if (kC > 1) cluster_sync(); else __syncthreads();
}
template <int kC> __device__ __forceinline__ int of_rank(const int* p, int rank) {
    if (kC == 1) return *p;
    uint32_t remote;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(remote) : "memory");
    return v;
}
template <typename T> __device__ __forceinline__ T warp_scan(T x, int lane) {     // sum up to and with this lane
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}
// Exclusive sum over the CTA's threads, and the total; `sums` [kWarps + 1] in shared memory.
template <typename T> __device__ __forceinline__ T cta_scan(T x, T* sums, int lane, int warp, T& total) {
    const T up_to = warp_scan(x, lane);
    __syncthreads();
    if (lane == 31) sums[warp] = up_to;
    __syncthreads();
    if (warp == 0) {
        const T own = sums[lane], s = warp_scan(own, lane);
        __syncwarp();
        sums[lane] = s - own;
        if (lane == 31) sums[kWarps] = s;
    }
    __syncthreads();
    total = sums[kWarps];
    return sums[warp] + up_to - x;
}
__device__ __forceinline__ int pages_of(long long rows, int page_rows) { return rows <= 0 ? 0 : (int)((rows + page_rows - 1) / page_rows); }
__device__ __forceinline__ bool in_pool(int page, int pages) { return (unsigned int)page < (unsigned int)pages; }

// Pages of a warp's stretch: whole words of 32.
template <int kC> __device__ __forceinline__ void stretch(int pages, int rank, int warp, int& first, int& end) {
    const int words = (int)(((long long)pages + 31) / 32), per = (words + kC * kWarps - 1) / (kC * kWarps);
    const long long at = (long long)(rank * kWarps + warp) * per * 32;
    first = (int)(at < pages ? at : pages);
    end = (int)(at + per * 32LL < pages ? at + per * 32LL : pages);
}
// Word of the stretch at `at`: bit i set where page at + i is in use.  Pages behind the pool count as in use.
__device__ __forceinline__ uint32_t used_word(const int* refs, int at, int pages, int lane) {
    return __ballot_sync(0xffffffffu, at + lane >= pages || __ldcg(refs + at + lane) > 0);
}
// A warp's stretch: how many of its pages are free, and the words of the first kWords of it, kept for the second look (pools of up to 65,536 pages: all).
constexpr int kWords = 8;
__device__ __forceinline__ int count_free(const int* refs, int first, int end, int pages, int lane, uint32_t (&words)[kWords]) {
    int n = 0;
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
        words[k] = first + k * 32 < end ? used_word(refs, first + k * 32, pages, lane) : 0xffffffffu;
        n += __popc(~words[k]);
    }
#pragma unroll 4
    for (int at = first + kWords * 32; at < end; at += 32) n += __popc(~used_word(refs, at, pages, lane));
    return n;
}
// f(first page of a word, word) for all words of a stretch
template <typename F>
__device__ __forceinline__ void each_word(const int* refs, int first, int end, int pages, int lane, const uint32_t (&words)[kWords], F f) {
#pragma unroll
    for (int k = 0; k < kWords; ++k)
        if (first + k * 32 < end) f(first + k * 32, words[k]);
    for (int at = first + kWords * 32; at < end; at += 32) f(at, used_word(refs, at, pages, lane));
}

// 2 KB or less, by a warp; a plane of up to 256 bytes a page (exponents) is one slice.
constexpr int kSlice = 2048, kSmall = 256;
__host__ __device__ __forceinline__ bool small_plane(const PlaneDev& pl) { return (long long)pl.bytes * pl.heads <= kSmall; }
__host__ __device__ __forceinline__ int slices_of(const PlaneDev& pl) { return small_plane(pl) ? 1 : (pl.bytes + kSlice - 1) / kSlice * pl.heads; }
__device__ __forceinline__ void copy_slice(char* dst, const char* src, int bytes, int lane) {
    if (((reinterpret_cast<uintptr_t>(dst) | reinterpret_cast<uintptr_t>(src) | (uintptr_t)bytes) & 15) == 0) {
        uint4 x[kSlice / 512];
#pragma unroll
        for (int i = 0; i < kSlice / 512; ++i)
            if ((i * 32 + lane) * 16 < bytes) x[i] = __ldcg(reinterpret_cast<const uint4*>(src) + i * 32 + lane);
#pragma unroll
        for (int i = 0; i < kSlice / 512; ++i)
            if ((i * 32 + lane) * 16 < bytes) reinterpret_cast<uint4*>(dst)[i * 32 + lane] = x[i];
        return;
    }
    for (int i = lane; i < bytes; i += 32) dst[i] = src[i];
}

// ---------------------------------------------------------------------------------------------------------------- resize
// 1. pages behind the new ends are given back   2. what every sequence needs; the free pages are counted   3. the free pages that are
// needed are listed in order   4. the sequences take theirs   5. few pages to copy (copy_here) are copied on the spot: a kernel of their own costs 4 us.
// Every CTA works out for itself what every sequence has and needs, in shared memory: handed on through global memory, it cost two more ways there and a barrier.
// Where no sequence takes a page, 2 to 5 are left out; where none gives one back, the barrier behind 1 (64 tables of 2000 pages, half of a step's two calls
// shrinking: 35.9 -> 30.2 us).  Giving back by a kernel over the whole chip in front cost two to seven microseconds and gained one at 500,000 entries.
__device__ __forceinline__ bool may_resize(const PagesParams& p, int n) { return n >= 0 && (long long)n <= (long long)p.width * p.page_rows; }

// What all sequences ask for together may be more than 32 bits hold (2049 tables of 2^20 entries), though no more than `pages` of it is ever served: it is summed in 64,
// and a place behind the pool's last page is kept as pages + 1.
struct SeqPlan { int have, grow, first, from; };             // pages it has and takes, the place of its first in the list (< 0: left alone), the page it has to copy (or -1)
template <int kC>
__global__ void __launch_bounds__(kThreads) pages_resize_kernel(const PagesParams p, const CopyPagesParams planes, const int slices, const int copy_here) {
    chain_enter();
    extern __shared__ SeqPlan plan[];                        // [seqs]
    __shared__ int sums[kWarps + 1], free_here;
    __shared__ long long need_sums[kWarps + 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = cluster_rank<kC>();
    const int gw = rank * kWarps + warp;
    constexpr int kAll = kC * kWarps;
    bool take_any = false, give_any = false;
    for (int s = tid; s < p.seqs; s += kThreads) {
        const int rows = p.rows[s], n = p.new_rows[s], have = min(pages_of(rows, p.page_rows), p.width);
        const bool fits = may_resize(p, n);                  // else the sequence is left alone
        int last = -1;                                       // growing inside a page: it may have to be copied
        if (p.copies && fits && rows > 0 && n > rows && rows % p.page_rows != 0) last = p.table[s * p.table_stride + have - 1];
        plan[s] = {have, fits ? pages_of(n, p.page_rows) - have : 0, fits ? 0 : -1, in_pool(last, p.pages) ? last : -1};
        take_any |= plan[s].grow > 0 || plan[s].from >= 0;
        give_any |= plan[s].grow < 0;
    }
    take_any = __syncthreads_or(take_any);
    give_any = __syncthreads_or(give_any);
    // `per` warps to a sequence, kChunk of its table's entries at a time
    const int per = max(1, min(kAll / p.seqs, (p.width + kChunk - 1) / kChunk)), j0 = gw % per, s0 = gw < kAll / per * per ? gw / per : p.seqs;
    for (int s = s0; give_any && s < p.seqs; s += kAll / per) {
        const SeqPlan q = plan[s];
        const int* const row = p.table + s * p.table_stride;
        for (int c0 = q.have + q.grow + j0 * kChunk; c0 < q.have; c0 += per * kChunk) {
            int page[kChunk / 32];
#pragma unroll
            for (int k = 0; k < kChunk / 32; ++k) page[k] = c0 + k * 32 + lane < q.have ? row[c0 + k * 32 + lane] : -1;
#pragma unroll
            for (int k = 0; k < kChunk / 32; ++k)
                if (in_pool(page[k], p.pages)) atomicSub(p.refs + page[k], 1);
        }
    }
    if (give_any || !take_any) meet<kC>();
    if (!take_any) {                                         // (all CTAs have read the rows)
        for (int s = rank * kThreads + tid; s < p.seqs; s += kC * kThreads) {
            if (plan[s].first >= 0) p.rows[s] = p.new_rows[s];
            if (p.copies && !copy_here) p.src[s] = -1;
        }
        if (rank == 0 && tid == 0 && p.missing) *p.missing = 0;
        return;
    }
    int first, end;
    stretch<kC>(p.pages, rank, warp, first, end);
    uint32_t words[kWords];
    const int mine = count_free(p.refs, first, end, p.pages, lane, words);
    long long need = 0;
    for (int b0 = 0; b0 < p.seqs; b0 += kThreads) {
        const int s = b0 + tid;
        SeqPlan q = {0, 0, -1, -1};
        if (s < p.seqs) {
            q = plan[s];
            if (q.from >= 0 && __ldcg(p.refs + q.from) <= 1) q.from = -1;             // nobody else holds it
        }
        const long long own = max(q.grow, 0) + (q.from >= 0 ? 1 : 0);
        long long total;
        const long long at = need + cta_scan(own, need_sums, lane, warp, total);
        if (s < p.seqs) { plan[s].from = q.from; plan[s].first = q.first < 0 ? -1 : (int)min(at, p.pages + 1LL); }
        need += total;
    }
    int total;
    int at = cta_scan(lane == 0 ? mine : 0, sums, lane, warp, total);    // free pages of the CTA in front of this warp
    at = __shfl_sync(0xffffffffu, at, 0);
    if (tid == 0) free_here = total;
    meet<kC>();
    int all = 0;
    for (int r = 0; r < kC; ++r) {
        const int n = of_rank<kC>(&free_here, r);
        at += r < rank ? n : 0;
        all += n;
    }
    if (at < need)
        each_word(p.refs, first, end, p.pages, lane, words, [&](int a, uint32_t used) {
            const int place = at + __popc(~used & low_bits(lane));
            if (!(used >> lane & 1) && place < need) p.list[place] = a + lane;
            at += __popc(~used);
        });
    if (rank == 0 && tid == 0 && p.missing) *p.missing = (int)min(max(need - all, 0LL), 0x7fffffffLL);
    meet<kC>();                                                      // (also: nobody leaves while its shared memory is read)
    auto served = [&](const SeqPlan& q) { const int take = max(q.grow, 0) + (q.from >= 0 ? 1 : 0); return take == 0 || (long long)q.first + take <= all; };
    for (int s = s0; s < p.seqs; s += kAll / per) {
        const SeqPlan q = plan[s];
        const int copy = q.from >= 0 ? 1 : 0;
        const bool yes = served(q);
        int* const row = p.table + s * p.table_stride;
        for (int c0 = j0 * kChunk; yes && c0 < q.grow; c0 += per * kChunk) {
            int page[kChunk / 32];
#pragma unroll
            for (int k = 0; k < kChunk / 32; ++k) page[k] = c0 + k * 32 + lane < q.grow ? __ldcg(p.list + q.first + copy + c0 + k * 32 + lane) : -1;
#pragma unroll
            for (int k = 0; k < kChunk / 32; ++k)
                if (page[k] >= 0) {
                    row[q.have + c0 + k * 32 + lane] = page[k];
                    p.refs[page[k]] = 1;
                }
        }
        if (j0 == 0 && lane == 0) {
            int to = -1;
            if (yes && copy) {
                to = __ldcg(p.list + q.first);
                row[q.have - 1] = to;
                p.refs[to] = 1;
                atomicSub(p.refs + q.from, 1);
            }
            if (p.copies && !copy_here) { p.src[s] = q.from; p.dst[s] = to; }
            if (yes && q.first >= 0) p.rows[s] = p.new_rows[s];
        }
    }
    // the pages to copy, 2 KB to a warp
    for (int i = gw; i < p.seqs * slices; i += kAll) {
        const int s = i / slices;
        int slice = i - s * slices, j = 0;
        const SeqPlan q = plan[s];
        if (q.from < 0 || !served(q)) continue;
        const int to = __ldcg(p.list + q.first);
        for (; j < planes.planes - 1; ++j) {
            const int own = slices_of(planes.plane[j]);
            if (slice < own) break;
            slice -= own;
        }
        const PlaneDev& pl = planes.plane[j];
        if (small_plane(pl)) {
            for (int i = lane; i < pl.bytes * pl.heads; i += 32) {
                const long long off = i / pl.bytes * pl.stride_h + i % pl.bytes;
                pl.base[to * pl.stride_page + off] = pl.base[q.from * pl.stride_page + off];
            }
            continue;
        }
        const int of = (pl.bytes + kSlice - 1) / kSlice, h = slice / of, off = (slice - h * of) * kSlice;
        copy_slice(pl.base + to * pl.stride_page + h * pl.stride_h + off, pl.base + q.from * pl.stride_page + h * pl.stride_h + off, min(kSlice, pl.bytes - off), lane);
    }
}

// ------------------------------------------------------------------------------------------------------------------ fork
// One CTA per child.  Left out: numbers that are no sequence, a child that is a parent in the same call, all but the first mention of a child.
constexpr int kForkThreads = 1024;
__global__ void __launch_bounds__(kForkThreads) pages_fork_kernel(const PagesParams p) {
    chain_enter();
    const int i = blockIdx.x, tid = threadIdx.x;
    const int child = p.children[i], parent = p.parents[i];
    bool bad = (unsigned int)child >= (unsigned int)p.seqs || (unsigned int)parent >= (unsigned int)p.seqs;
    for (int j = tid; j < p.n; j += kForkThreads) bad = bad || (j < i && p.children[j] == child) || p.parents[j] == child;
    if (__syncthreads_or(bad)) return;
    const int rows = p.rows[parent], have = min(pages_of(rows, p.page_rows), p.width), had = min(pages_of(p.rows[child], p.page_rows), p.width);
    int* const to = p.table + child * p.table_stride;
    const int* const from = p.table + parent * p.table_stride;
    __syncthreads();                                                     // (all have read the child's rows)
#pragma unroll 2
    for (int k = tid; k < max(have, had); k += kForkThreads) {
        if (k < had && in_pool(to[k], p.pages)) atomicSub(p.refs + to[k], 1);
        if (k < have) {
            const int page = from[k];
            to[k] = page;
            if (in_pool(page, p.pages)) atomicAdd(p.refs + page, 1);
        }
    }
    if (tid == 0) p.rows[child] = max(rows, 0);
}

// --------------------------------------------------------------------------------------------------------------- compact
// The page at place a of the pool has u pages in use in front of it.  With n in use in all, a free page in front of n is hole number a - u, and a page in use
// from n on has number u - (those in use in front of n): one count of the pages is enough for both.
template <int kC>
__global__ void __launch_bounds__(kThreads) pages_compact_kernel(const PagesParams p) {
    chain_enter();
    __shared__ int sums[kWarps + 1], used_here;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = cluster_rank<kC>();
    int first, end;
    stretch<kC>(p.pages, rank, warp, first, end);
    uint32_t words[kWords];
    const int mine = (end - first) - count_free(p.refs, first, end, p.pages, lane, words);
    int total;
    int u = cta_scan(lane == 0 ? mine : 0, sums, lane, warp, total);
    u = __shfl_sync(0xffffffffu, u, 0);
    if (tid == 0) used_here = total;
    meet<kC>();
    int n = 0;
    for (int r = 0; r < kC; ++r) {
        const int x = of_rank<kC>(&used_here, r);
        u += r < rank ? x : 0;
        n += x;
    }
    // holes -> dst in order; pages that move -> list, at the place u
    each_word(p.refs, first, end, p.pages, lane, words, [&](int a, uint32_t used) {
        const int at = a + lane, before = u + __popc(used & low_bits(lane));
        if (at < p.pages) {
            const bool in_use = used >> lane & 1;
            if (at == n) *p.count = n - before;                          // as many holes as pages that move
            if (!in_use && at < n) p.dst[at - before] = at;
            if (in_use && at >= n) p.list[before] = at;
            if (!in_use || at < n) p.remap[at] = in_use ? at : -1;
            // counts that no move concerns; a hole's and a moving page's come with the move
            if (in_use == (at < n) && (p.refs_out != p.refs || !in_use)) p.refs_out[at] = in_use ? __ldcg(p.refs + at) : 0;
        }
        u += __popc(used & (p.pages - a >= 32 ? 0xffffffffu : low_bits(p.pages - a)));
    });
    if (rank == 0 && tid == 0) {
        if (p.live) *p.live = n;
        if (n == p.pages) *p.count = 0;
    }
    meet<kC>();
    const int moves = __ldcg(p.count);
    for (int k = rank * kThreads + tid; k < moves; k += kC * kThreads) {
        const int from = __ldcg(p.list + n - moves + k), to = __ldcg(p.dst + k);
        p.src[k] = from;
        p.remap[from] = to;
        p.refs_out[to] = __ldcg(p.refs + from);
        p.refs_out[from] = 0;
    }
}

// The sequences' tables after a compaction, by `ctas` CTAs of 256 threads.
__device__ __forceinline__ void rename_pages(const PagesParams& p, int cta, int ctas) {
    const long long total = (long long)p.seqs * p.width;
    for (long long i = (long long)cta * 256 + threadIdx.x; i < total; i += (long long)ctas * 256) {
        const int s = (int)(i / p.width), k = (int)(i - (long long)s * p.width);
        if (k >= pages_of(p.rows[s], p.page_rows)) continue;
        const int page = p.table[s * p.table_stride + k];
        p.table_out[s * p.table_out_stride + k] = in_pool(page, p.pages) ? __ldcg(p.remap + page) : page;
    }
}

// ------------------------------------------------------------------------------------------------------------------ copy
// A page's bytes in the large planes are cut into pieces of 4 KB, sixteen bytes to a thread, two pieces to a CTA: where the pieces lie is worked out
// once.  (Four pieces took 64 registers and left half as many threads: 75 us for 150 MB against 58.)  Planes of up to 256 bytes a page (exponents) go along with
// its first pieces, a thread to a byte: as pieces of their own they took as long as the large ones.
// After a compaction (rename) the last row of the grid's CTAs rewrites the tables meanwhile.
constexpr int kPiece = 4096, kPieces = 2;
__global__ void __launch_bounds__(256, 6) pages_copy_kernel(const CopyPagesParams p, const PagesParams tables, const int rename) {
    chain_enter();
    if (rename && blockIdx.y == gridDim.y - 1) {
        rename_pages(tables, blockIdx.x, gridDim.x);
        return;
    }
    const int n = p.count ? *p.count : p.n, tid = threadIdx.x;
    char* base[kPieces];
    long long stride[kPieces];
    int bytes[kPieces];                                      // from this thread's on; 0: nothing
    bool wide = true;
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
        int piece = blockIdx.y * kPieces + u, j = 0, of = 0;
        for (; j < p.large; ++j) {
            of = (p.plane[j].bytes + kPiece - 1) / kPiece;
            if (piece < of * p.plane[j].heads) break;
            piece -= of * p.plane[j].heads;
        }
        base[u] = nullptr; stride[u] = 0; bytes[u] = 0;
        if (j == p.large) continue;
        const PlaneDev& pl = p.plane[j];
        const int h = piece / of, at = (piece - h * of) * kPiece;
        base[u] = pl.base + h * pl.stride_h + at + tid * 16;
        stride[u] = pl.stride_page;
        bytes[u] = max(0, min(kPiece, pl.bytes - at) - tid * 16);
        wide &= ((reinterpret_cast<uintptr_t>(pl.base) | (uintptr_t)pl.stride_page | (uintptr_t)pl.stride_h | (uintptr_t)pl.bytes) & 15) == 0;
    }
    auto small_planes = [&](long long f, long long t) {
        if (blockIdx.y != 0) return;
        for (int j = p.large; j < p.planes; ++j) {
            const PlaneDev& pl = p.plane[j];
            if (tid >= pl.bytes * pl.heads) continue;
            const int h = tid / pl.bytes;
            const long long at = h * pl.stride_h + tid - h * pl.bytes;
            pl.base[t * pl.stride_page + at] = pl.base[f * pl.stride_page + at];
        }
    };
    if (!wide) {
        for (int k = blockIdx.x; k < n; k += gridDim.x) {
            const long long f = p.src[k], t = p.dst[k];
            if (f < 0 || t < 0) continue;
#pragma unroll
            for (int u = 0; u < kPieces; ++u)
#pragma unroll 1
                for (int i = 0; i < min(bytes[u], 16); ++i) base[u][t * stride[u] + i] = base[u][f * stride[u] + i];
            small_planes(f, t);
        }
        return;
    }
    int k = blockIdx.x, from = -1, to = -1;
    if (k < n) { from = p.src[k]; to = p.dst[k]; }
    while (k < n) {
        const long long f = from, t = to;
        k += gridDim.x;
        if (k < n) { from = p.src[k]; to = p.dst[k]; }       // the next one's
        if (f < 0 || t < 0) continue;
        uint4 x[kPieces];
#pragma unroll
        for (int u = 0; u < kPieces; ++u)
            if (bytes[u] > 0) x[u] = __ldcs(reinterpret_cast<const uint4*>(base[u] + f * stride[u]));
#pragma unroll
        for (int u = 0; u < kPieces; ++u)
            if (bytes[u] > 0) *reinterpret_cast<uint4*>(base[u] + t * stride[u]) = x[u];
        small_planes(f, t);
    }
}

}  // namespace

static cudaError_t launch_pages_copy(const CopyPagesParams& p, const PagesParams* rename, cudaStream_t st) {
    // large planes first
    CopyPagesParams q = p;
    q.planes = 0;
    for (int small = 0; small < 2; ++small) {
        for (int j = 0; j < p.planes; ++j)
            if (small_plane(p.plane[j]) == (small == 1)) q.plane[q.planes++] = p.plane[j];
        if (!small) q.large = q.planes;
    }
    long long pieces = 0;
    for (int j = 0; j < q.large; ++j) pieces += (long long)((q.plane[j].bytes + kPiece - 1) / kPiece) * q.plane[j].heads;
    long long groups = pieces > 0 ? (pieces + kPieces - 1) / kPieces : (q.planes > 0 ? 1 : 0);
    if (q.n == 0) groups = 0;
    if (groups > 65534) return cudaErrorInvalidValue;        // (a page of a gigabyte)
    if (groups == 0 && !rename) return cudaSuccess;
    // (a CTA takes four pages of a move of 10,000 rather than sixteen: 66 us for the whole call, 78 so)
    const long long fill = 148 * 32 / (groups + (rename ? 1 : 0)) + 1, most = q.n > 0 ? q.n : 1;
    PagesParams none = {};
    return launch_chained(pages_copy_kernel, dim3((unsigned)(most < fill ? most : fill), (unsigned)(groups + (rename ? 1 : 0))), dim3(256), 0, st, 0, q,
                          rename ? *rename : none, rename ? 1 : 0);
}

// One CTA or a cluster of eight: one where its warps hold all of the pool's words (8192 pages) and the tables, and the copies that may come, are few.
// Up to four slices (2 KB) to a warp of a cluster, eight to a warp of one CTA, are copied on the spot.
constexpr int kCluster = 8, kOnePages = kWords * 32 * kWarps;
template <int kC>
static cudaError_t launch_resize(const PagesParams& p, const CopyPagesParams& c, long long slices, int here, cudaStream_t st) {
    const size_t smem = (size_t)p.seqs * sizeof(SeqPlan);
    if (smem > 32768) {
        cudaError_t e = cudaFuncSetAttribute(pages_resize_kernel<kC>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kMaxSeqs * sizeof(SeqPlan)));
        if (e != cudaSuccess) return e;
    }
    return launch_chained(pages_resize_kernel<kC>, dim3(kC), dim3(kThreads), smem, st, kC > 1 ? kC : 0, p, c, here ? (int)slices : 0, here);
}
cudaError_t launch_pages_resize(const PagesParams& p, CopyPagesParams c, cudaStream_t st) {
    long long slices = 0;
    for (int j = 0; j < c.planes; ++j) slices += slices_of(c.plane[j]);
    const bool one = p.pages <= kOnePages && p.seqs <= 64 && (long long)p.seqs * p.width <= 16384 && slices * p.seqs <= 8 * kWarps;
    const int here = c.planes > 0 && (one || slices * p.seqs <= 4 * kCluster * kWarps);
    cudaError_t e = one ? launch_resize<1>(p, c, slices, here, st) : launch_resize<kCluster>(p, c, slices, here, st);
    if (e != cudaSuccess || c.planes == 0 || here) return e;
    c.src = p.src; c.dst = p.dst; c.n = p.seqs;
    return launch_pages_copy(c, nullptr, st);
}
cudaError_t launch_pages_fork(const PagesParams& p, cudaStream_t st) {
    return launch_chained(pages_fork_kernel, dim3(p.n), dim3(kForkThreads), 0, st, 0, p);
}
cudaError_t launch_pages_compact(const PagesParams& p, CopyPagesParams c, cudaStream_t st) {
    cudaError_t e = p.pages <= kOnePages ? launch_chained(pages_compact_kernel<1>, dim3(1), dim3(kThreads), 0, st, 0, p)
                                         : launch_chained(pages_compact_kernel<kCluster>, dim3(kCluster), dim3(kThreads), 0, st, kCluster, p);
    if (e != cudaSuccess) return e;
    c.src = p.src; c.dst = p.dst; c.count = p.count; c.n = p.pages / 2;          // (at most half of the pages can move)
    return launch_pages_copy(c, (long long)p.seqs * p.width > 0 ? &p : nullptr, st);
}

}  // namespace mka
