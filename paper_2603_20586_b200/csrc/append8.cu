// Appends key and value rows to a paged cache of 8-bit codes (code8.cuh): per block of rows and KV head the largest magnitude, its exponent, the codes.
//
// HBM-bound: a row is read once (2 or 4 bytes a column) and written once (1 byte).  A unit = one block of one head of keys or of values that the call's
// rows touch; as many threads as keep eight or sixteen 8-column vectors each hold all of it in registers, so the second look at the rows (the first
// finds the magnitude) costs no memory.  A block that holds rows already keeps its exponent or takes a larger one; its codes are read and written
// again only when it grows.  No two units write the same block, and nothing is accumulated: results do not depend on the order of the units.
// 32,768 rows of 8 heads at d = 128 (201 MB) in blocks of 64: 37.0 us with other rows every time, 5.4 TB/s (0.83 of a copy); the next rows of 32 sequences: 3.8 us (4.1 where they
// lie inside blocks, 5.0 and 5.7 at d = 64 and 128 where they make these grow).  Back to back on the same rows, us, for the floor of a copy: 65,536 rows of 8 heads at d = 64, blocks of 16 / 64 / 256:
// bf16 36.6 / 33.3 / 34.0 (30.7), f32 52.7 / 52.9 / 53.4 (51.2); d = 128, 32,768 rows: bf16 33.4 / 34.5 / 33.1, f32 52.0 / 52.6 / 72.0 (the last: units of 512 threads, one CTA to an SM).
#include <cuda_fp16.h>

#include "code8.cuh"

namespace mka {
namespace {


// Eight columns as they are in memory.  top(): a number that grows with the largest magnitude, over the type's infinity where an element is not finite.
template <typename T> struct Row8;
template <> struct Row8<__nv_bfloat16> {
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { u = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void clear() { u = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ uint32_t word(int i) const { return i < 2 ? (i ? u.y : u.x) : (i == 2 ? u.z : u.w); }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? word(i >> 1) & 0xffff0000u : word(i >> 1) << 16); }
    // bits of two magnitudes side by side
    __device__ __forceinline__ uint32_t top(uint32_t t) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) t = __vmaxu2(t, word(i) & 0x7fff7fffu);
        return t;
    }
    static __device__ __forceinline__ uint32_t top_bits(uint32_t t) { return max(t & 0xffff0000u, t << 16); }       // as the bits of a float
};
template <> struct Row8<float> {
    uint4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = __ldcs(reinterpret_cast<const uint4*>(p)); b = __ldcs(reinterpret_cast<const uint4*>(p) + 1); }
    __device__ __forceinline__ void clear() { a = b = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ uint32_t word(int i) const { return i < 4 ? (i < 2 ? (i ? a.y : a.x) : (i == 2 ? a.z : a.w)) : (i < 6 ? (i == 4 ? b.x : b.y) : (i == 6 ? b.z : b.w)); }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(word(i)); }
    __device__ __forceinline__ uint32_t top(uint32_t t) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, word(i) & 0x7fffffffu);
        return t;
    }
    static __device__ __forceinline__ uint32_t top_bits(uint32_t t) { return t; }
};

// Codes of four values that are finite and fit, in units of 2^-e already up to the factor `up`.  s8: adding 1.5 2^23 rounds to a whole number, whose low byte is
// the code (one instruction; a conversion to an integer is a sixteenth of the rate).
template <bool kS8>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float up) {
    if (kS8) {
        const float magic = 12582912.f;
        const uint32_t x = __float_as_uint(fmaf(a, up, magic)), y = __float_as_uint(fmaf(b, up, magic));
        const uint32_t z = __float_as_uint(fmaf(c, up, magic)), w = __float_as_uint(fmaf(d, up, magic));
        return __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
    }
    return encode2<false>(a * up, b * up) | encode2<false>(c * up, d * up) << 16;
}

// kUnit: threads of a unit, as many as hold the block with kVecs vectors of eight columns each (16 x 64 take half a warp).  In bf16 sixteen for blocks of 32 rows and more,
// two CTAs to an SM: 65,536 rows of eight heads at d = 64 in blocks of 64 38.2 -> 35.6 us against eight and three CTAs, 32,768 rows of eight heads at d = 128 in blocks of 32, 64, 128
// and 256 36.6 -> 34.5, 36.4 -> 36.2, 35.0 -> 35.4, 49.8 -> 34.4 (eight: units of 512 threads, one CTA to an SM).  f32 rows keep eight; in e4m3
// they are up to 5 % slower since (13.2 -> 13.8, blocks of 256 68.3 -> 72.1).
template <typename T, int kUnit, int kVecs> struct Shape8 {
    static constexpr int kThreads = kUnit > 256 ? kUnit : 256, kCtas = kUnit > 256 ? 1 : (sizeof(T) == 2 && kVecs == 8 ? 3 : 2);
};
template <typename T, bool kS8, int kUnit, int kVecs, int DH>
__global__ void __launch_bounds__(Shape8<T, kUnit, kVecs>::kThreads, Shape8<T, kUnit, kVecs>::kCtas) append8_kernel(const Append8Params p, const long long units, const int blocks) {
    chain_enter();
    constexpr int kCtaThreads = Shape8<T, kUnit, kVecs>::kThreads, kWarps = kUnit / 32, kVecsOfRow = DH / 8;       // kWarps: 0 for half a warp
    constexpr int kRowsApart = kUnit / kVecsOfRow;            // rows between a lane's vectors
    constexpr int kPart = kWarps > 1 ? kWarps : 1;
    __shared__ uint32_t tops[kCtaThreads / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int ut = tid % kUnit;
    const uint32_t lanes = kUnit == 16 ? 0xffffu << (lane & 16) : 0xffffffffu;       // the unit's in this warp
    long long u = (long long)blockIdx.x * (kCtaThreads / kUnit) + tid / kUnit;
    const bool real = u < units;
    if (!real) u = 0;
    const bool values = u & 1;
    const long long bh = (u >> 1) / blocks;
    const int blk_i = (int)((u >> 1) - bh * blocks), b = (int)(bh / p.H), h = (int)(bh - (long long)b * p.H);
    constexpr int block = kRowsApart * kVecs;                        // its rows
    const long long r0 = p.dst_offset + (p.offsets ? (long long)p.offsets[b] : 0);
    const long long base = ((r0 >> p.block_shift) + blk_i) << p.block_shift;         // the block's first row
    const long long lo = r0 > base ? r0 : base, hi = r0 + p.n < base + block ? r0 + p.n : base + block;
    // where the block lies; rows that the table does not hold, or whose page is not in the pool, are dropped
    bool write = real && r0 >= 0 && lo < hi && hi <= p.rows_held;
    int page = -1;
    if (write) page = p.table[b * p.table_stride + (base >> p.page_shift)];
    write = write && page >= 0 && page < p.pool_pages;
    const int in_page = (int)(base & ((1LL << p.page_shift) - 1));
    const int row = ut / kVecsOfRow, col = ut % kVecsOfRow * 8;      // of the lane's first vector
    const int first = (int)(lo - base), end = write ? (int)(hi - base) : 0;          // the new rows of the block
    const T* const src = static_cast<const T*>(values ? p.v : p.k) + b * p.sb + h * p.sh + (base - r0) * p.sn + col;
    Row8<T> x[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int r = row + i * kRowsApart;
        if (r >= first && r < end) x[i].load(src + r * p.sn);
        else x[i].clear();
    }
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) t = x[i].top(t);
    t = __reduce_max_sync(lanes, Row8<T>::top_bits(t));
    if (kWarps > 1) {
        if (lane == 0) tops[warp] = t;
        __syncthreads();
        const int w0 = warp / kPart * kPart;
#pragma unroll
        for (int w = 0; w < kPart; ++w) t = max(t, tops[w0 + w]);
    }
    float top = __uint_as_float(t);
    const bool odd = t >= 0x7f800000u;                               // of the whole unit: an element is not finite
    if (kWarps > 1 && __syncthreads_or(odd)) {                       // (the other units of the CTA go along)
        uint32_t f = 0;
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t m = __float_as_uint(x[i].at(j)) & 0x7fffffffu;
                f = m < 0x7f800000u ? max(f, m) : f;
            }
        f = __reduce_max_sync(0xffffffffu, f);
        __syncthreads();
        if (lane == 0) tops[warp] = f;
        __syncthreads();
        const int w0 = warp / kPart * kPart;
#pragma unroll
        for (int w = 0; w < kPart; ++w) f = max(f, tops[w0 + w]);
        top = __uint_as_float(f);
    } else if (kWarps <= 1 && odd) {
        uint32_t f = 0;
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t m = __float_as_uint(x[i].at(j)) & 0x7fffffffu;
                f = m < 0x7f800000u ? max(f, m) : f;
            }
        top = __uint_as_float(__reduce_max_sync(lanes, f));
    }
    if (!write) return;
    uint8_t* const exp_at = (values ? p.v_exp : p.k_exp) + page * p.esp + h * p.esh + (in_page >> p.block_shift);
    uint8_t* const dst = (values ? p.pool_v : p.pool_k) + page * p.pool_sp + h * p.pool_sh + in_page * p.pool_sn + col;
    int e = exponent_for<kS8>(top);
    if (first > 0) {                                                 // the block holds rows already
        const int old = block_exponent(*exp_at);
        if (e > old) {
            const float down = pow2i(old - e);
            for (int r = row; r < first; r += kRowsApart) {
                uint2* const at = reinterpret_cast<uint2*>(dst + r * p.pool_sn);
                const uint2 c = *at;
                uint32_t out[2];
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    uint32_t a, z;
                    decode4<kS8, 0>(w ? c.y : c.x, a, z);
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&a)), g = __half22float2(*reinterpret_cast<const __half2*>(&z));
                    out[w] = encode2<kS8>(f.x * down, f.y * down) | encode2<kS8>(g.x * down, g.y * down) << 16;
                }
                *at = make_uint2(out[0], out[1]);
            }
        } else {
            e = old;
        }
        // (every lane has read the exponent before one of them writes it)
        if (kWarps > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / kPart), "r"(kUnit) : "memory");
        else __syncwarp(lanes);
    }
    const float up = pow2i(-e);
    if (odd || e == kExpHigh) {                                      // infinities, NaN, magnitudes beyond the largest exponent
#pragma unroll 1
        for (int i = 0; i < kVecs; ++i) {
            const int r = row + i * kRowsApart;
            if (r < first || r >= end) continue;
            Row8<T> y;
            y.load(src + r * p.sn);
            uint32_t out[2];
#pragma unroll
            for (int w = 0; w < 2; ++w)
                out[w] = encode2<kS8>(y.at(4 * w) * up, y.at(4 * w + 1) * up) | encode2<kS8>(y.at(4 * w + 2) * up, y.at(4 * w + 3) * up) << 16;
            *reinterpret_cast<uint2*>(dst + r * p.pool_sn) = make_uint2(out[0], out[1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int r = row + i * kRowsApart;
            if (r < first || r >= end) continue;
            *reinterpret_cast<uint2*>(dst + r * p.pool_sn) =
                make_uint2(encode4<kS8>(x[i].at(0), x[i].at(1), x[i].at(2), x[i].at(3), up), encode4<kS8>(x[i].at(4), x[i].at(5), x[i].at(6), x[i].at(7), up));
        }
    }
    if (ut == 0) *exp_at = (uint8_t)(e + 127);
}

template <typename T, bool kS8, int kUnit, int kVecs, int DH>
cudaError_t launch_t(const Append8Params& p, cudaStream_t st) {
    constexpr int kThreads = Shape8<T, kUnit, kVecs>::kThreads;
    constexpr int block = kUnit * kVecs * 8 / DH;                    // 1 << p.block_shift
    const long long blocks = (p.n + block - 2) / block + 1;          // that a sequence's rows touch at most
    const long long units = 2 * blocks * p.B * p.H, per = kThreads / kUnit, ctas = (units + per - 1) / per;
    if (ctas > 0x7fffffffLL || blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
    return launch_chained(append8_kernel<T, kS8, kUnit, kVecs, DH>, dim3((unsigned)ctas), dim3(kThreads), 0, st, 0, p, units, (int)blocks);
}
template <typename T, bool kS8, int DH>
cudaError_t launch_w(const Append8Params& p, cudaStream_t st) {
    constexpr int kVecs = sizeof(T) == 2 ? 16 : 8;
    switch (p.block_shift) {
        case 4: return launch_t<T, kS8, DH / 4, 8, DH>(p, st);
        case 5: return launch_t<T, kS8, 32 * DH / 8 / kVecs, kVecs, DH>(p, st);
        case 6: return launch_t<T, kS8, 64 * DH / 8 / kVecs, kVecs, DH>(p, st);
        case 7: return launch_t<T, kS8, 128 * DH / 8 / kVecs, kVecs, DH>(p, st);
        default: return launch_t<T, kS8, 256 * DH / 8 / kVecs, kVecs, DH>(p, st);
    }
}
template <typename T, int DH>
cudaError_t launch_c(const Append8Params& p, cudaStream_t st) { return p.s8 ? launch_w<T, true, DH>(p, st) : launch_w<T, false, DH>(p, st); }

}  // namespace

cudaError_t launch_append8(const Append8Params& p, int dtype, cudaStream_t st) {
    if (dtype == MKA_BF16) return p.d == 128 ? launch_c<__nv_bfloat16, 128>(p, st) : launch_c<__nv_bfloat16, 64>(p, st);
    return p.d == 128 ? launch_c<float, 128>(p, st) : launch_c<float, 64>(p, st);
}

}  // namespace mka
