// Activations as channels-last tensors [n][h][w][c] of three types, and their 8-bit checkpoints.
//
// A checkpoint holds blocks of 32 consecutive channels of one position (the last block of a row may be shorter): one byte per value
// and one byte E per block, value = code * 2^(E - 127).  E is the smallest exponent with which the block's largest magnitude stays
// within 127 (int8) or 448 (e4m3); the codes are rounded to nearest even.  The scale is a power of two, so dividing by it is exact, a code
// follows from the values alone (no reciprocal whose last bit decides a tie), and a decoded value is exact in bf16 (both codes have at
// most seven significant bits; only e4m3 blocks with E below 3, values below 2^-116, have steps finer than bf16's last).  A block with an infinity or a NaN gets E = 255 and codes 0 and stands for NaN throughout.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ptx.cuh"

namespace op {

using kn::f2;
using kn::add2; using kn::mul2; using kn::fma2; using kn::mk2; using kn::un2;
enum { kSrcSame = 0, kSrcInt8 = 1, kSrcE4m3 = 2 };      // what a backward pass reads x from (and the two formats of codes)

// ---------------------------------------------------------------- vectors of V elements
template <int BYTES> struct RawOf;
template <> struct RawOf<1> { using type = uint8_t; };
template <> struct RawOf<2> { using type = uint16_t; };
template <> struct RawOf<4> { using type = uint32_t; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<16> { using type = uint4; };
struct alignas(16) Raw32 { uint4 a, b; };
template <> struct RawOf<32> { using type = Raw32; };
template <typename T, int V> using Raw = typename RawOf<sizeof(T) * V>::type;

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(float v) { return v; }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }

template <typename T, int V>
__device__ __forceinline__ void unpack(const Raw<T, V>& r, float* f) {
    if constexpr (V > 1 && sizeof(T) == 2) {
        const uint32_t* u = (const uint32_t*)&r;
        #pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) { f[2 * i] = kn::bf_lo(u[i]); f[2 * i + 1] = kn::bf_hi(u[i]); }
            else { const float2 t = __half22float2(*(const __half2*)&u[i]); f[2 * i] = t.x; f[2 * i + 1] = t.y; }
        }
    } else {
        const T* e = (const T*)&r;
        #pragma unroll
        for (int i = 0; i < V; ++i) f[i] = to_f<T>(e[i]);
    }
}
// rounds to nearest, as a cast does
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> pack(const float* f) {
    Raw<T, V> r;
    if constexpr (V > 1 && sizeof(T) == 2) {
        uint32_t* u = (uint32_t*)&r;
        #pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) { const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]); u[i] = *(const uint32_t*)&h; }
            else { const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]); u[i] = *(const uint32_t*)&h; }
        }
    } else {
        T* e = (T*)&r;
        #pragma unroll
        for (int i = 0; i < V; ++i) e[i] = from_f<T>(f[i]);
    }
    return r;
}

// ---------------------------------------------------------------- positions
struct FastDiv {               // x / d for x < 2^31
    uint32_t d, mul, shift;
    __device__ __forceinline__ uint32_t div(uint32_t x) const { return (uint32_t)(((uint64_t)x * mul) >> shift); }
};
inline FastDiv fast_div(uint32_t d) {
    // m = floor(2^(31 + s) / d) + 1 with 2^s >= d: x m / 2^(31 + s) is below x / d + x / 2^(31 + s) < x / d + 1 / d
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return {d, (uint32_t)(((1ull << (31 + s)) / d) + 1), 31 + s};
}
// strides in elements; flat: position p of a sample lies at p * sw
// step: positions between a thread's; inc = step * sw, wrap = sh - w * sw (0: flat)
struct Geo {
    long long sn, sh, sw, inc, wrap;
    FastDiv w;
    int flat, step;
    __device__ __forceinline__ long long at(uint32_t p) const {
        if (flat) return (long long)p * sw;
        const uint32_t h = w.div(p);
        return (long long)h * sh + (long long)(p - h * w.d) * sw;
    }
};

// A thread's walk over positions that lie g.step apart: its offset in a tensor, by one addition, and another where it passes the end of a row.
struct Cursor {
    long long off;
    int x;
    __device__ __forceinline__ Cursor(const Geo& g, uint32_t p) : off(g.at(p)), x(g.flat ? 0 : (int)(p - g.w.div(p) * g.w.d)) {}
    __device__ __forceinline__ void next(const Geo& g) {
        off += g.inc;
        if (!g.flat) {
            x += g.step;
            while (x >= (int)g.w.d) { x -= (int)g.w.d; off += g.wrap; }
        }
    }
};

// ---------------------------------------------------------------- codes
__device__ __forceinline__ float scale_of(uint32_t e) {         // 2^(e - 127); e = 0: a subnormal; 255: NaN
    return e == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(e ? e << 23 : 1u << 22);
}
// exponent byte of a block from the bits of its largest magnitude.  amax = m 2^k with m in [1, 2): amax / 2^(k - 6) = 64 m stays within 127 for
// m up to 127/64, whose mantissa field is 0x7E0000: adding 0x1FFFF carries into the exponent exactly for larger ones.  e4m3: 256 m
// within 448, 0x600000.
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return 255u;
    const int e = FMT == kSrcInt8 ? (int)((amax_bits + 0x1ffffu) >> 23) - 6 : (int)((amax_bits + 0x1fffffu) >> 23) - 8;
    return (uint32_t)max(e, 0);
}
__device__ __forceinline__ float inverse_scale(uint32_t e) { return e == 255u ? 0.f : __uint_as_float((254u - e) << 23); }      // 2^(127 - e), e <= 249

// codes of V values.  int8: 1.5 * 2^23 + v has v, rounded to nearest even, in its low byte.  A block that stands for NaN has inv = 0;
// its infinities and NaN give 0 * inf = NaN, so its codes are set to 0 by the caller's `nan`.
template <int FMT, int V>
__device__ __forceinline__ Raw<uint8_t, V> codes_of(const float* f, float inv, bool nan) {
    Raw<uint8_t, V> r;
    if constexpr (FMT == kSrcInt8) {
        uint32_t b[V];
        if constexpr (V >= 2) {
            const f2 i2 = mk2(inv, inv), m2 = mk2(12582912.f, 12582912.f);
            #pragma unroll
            for (int i = 0; i < V; i += 2) {
                float lo, hi;
                un2(fma2(mk2(f[i], f[i + 1]), i2, m2), lo, hi);
                b[i] = __float_as_uint(lo); b[i + 1] = __float_as_uint(hi);
            }
        } else b[0] = __float_as_uint(fmaf(f[0], inv, 12582912.f));
        if constexpr (V >= 4) {
            uint32_t* u = (uint32_t*)&r;
            #pragma unroll
            for (int i = 0; i < V / 4; ++i) {
                const uint32_t lo = __byte_perm(b[4 * i], b[4 * i + 1], 0x0040), hi = __byte_perm(b[4 * i + 2], b[4 * i + 3], 0x0040);
                u[i] = nan ? 0u : __byte_perm(lo, hi, 0x5410);
            }
        } else {
            uint8_t* u = (uint8_t*)&r;
            #pragma unroll
            for (int i = 0; i < V; ++i) u[i] = nan ? 0 : (uint8_t)b[i];
        }
    } else {
        if constexpr (V >= 2) {
            uint16_t* u = (uint16_t*)&r;
            #pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                uint16_t q;
                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q) : "f"(f[2 * i + 1] * inv), "f"(f[2 * i] * inv));
                u[i] = nan ? 0 : q;
            }
        } else {
            uint16_t q;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q) : "f"(0.f), "f"(f[0] * inv));
            *(uint8_t*)&r = nan ? 0 : (uint8_t)q;
        }
    }
    return r;
}
// the integers or e4m3 numbers that V codes are, without their scale
template <int FMT, int V>
__device__ __forceinline__ void code_values(const Raw<uint8_t, V>& r, float* f) {
    if constexpr (FMT == kSrcInt8) {
        if constexpr (V >= 4) {
            const uint32_t* u = (const uint32_t*)&r;
            #pragma unroll
            for (int i = 0; i < V / 4; ++i) {
                const uint32_t t = u[i] ^ 0x80808080u;       // code + 128 as an unsigned byte, then 2^23 + that as a float
                #pragma unroll
                for (int k = 0; k < 4; k += 2)
                    un2(add2(mk2(__uint_as_float(__byte_perm(t, 0x4b000000u, 0x7440u | k)), __uint_as_float(__byte_perm(t, 0x4b000000u, 0x7441u | k))), mk2(-8388736.f, -8388736.f)),
                        f[4 * i + k], f[4 * i + k + 1]);
            }
        } else {
            const int8_t* u = (const int8_t*)&r;
            #pragma unroll
            for (int i = 0; i < V; ++i) f[i] = (float)u[i];
        }
    } else {
        if constexpr (V >= 2) {
            const uint16_t* u = (const uint16_t*)&r;
            #pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                uint32_t h;
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(u[i]));
                const float2 t = __half22float2(*(const __half2*)&h);
                f[2 * i] = t.x; f[2 * i + 1] = t.y;
            }
        } else {
            uint32_t h;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t) * (const uint8_t*)&r));
            f[0] = __half22float2(*(const __half2*)&h).x;
        }
    }
}
// The largest magnitude of eight values as the bits of a float.  Magnitudes compare as unsigned integers, NaN above infinity above all others; 16-bit
// types are compared in pairs (a NaN stays one).
template <typename T>
__device__ __forceinline__ uint32_t amax_bits(const Raw<T, 8>& r) {
    const uint32_t* u = (const uint32_t*)&r;
    if constexpr (sizeof(T) == 2) {
        uint32_t m = u[0] & 0x7fff7fffu;
        #pragma unroll
        for (int i = 1; i < 4; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(u[i] & 0x7fff7fffu));
            else asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(m) : "r"(u[i] & 0x7fff7fffu));
        }
        const uint32_t top = max(m >> 16, m & 0xffffu);
        if constexpr (std::is_same<T, __nv_bfloat16>::value) return top << 16;
        else return __float_as_uint(__half2float(__ushort_as_half((unsigned short)top)));
    } else {
        uint32_t m = 0;
        #pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, u[i] & 0x7fffffffu);
        return m;
    }
}
// Codes and exponent of a vector, called by the four lanes of a block together (the lanes of a row's last block that hold no channels pass zeros and
// store nothing).  r, f: the vector as it is stored, and its values; codes, scales: where its codes and its block's exponent go.
template <typename T, int FMT>
__device__ __forceinline__ void store_codes(const Raw<T, 8>& r, const float* f, bool has, uint8_t* codes, uint8_t* scales) {
    const uint32_t quad = 0xfu << (threadIdx.x & 28);
    uint32_t m = amax_bits<T>(r);
    m = max(m, __shfl_xor_sync(quad, m, 1));
    m = max(m, __shfl_xor_sync(quad, m, 2));
    const uint32_t e = scale_byte<FMT>(m);
    if (has) {
        *(uint2*)codes = codes_of<FMT, 8>(f, inverse_scale(e), e == 255u);
        if ((threadIdx.x & 3) == 0) *scales = (uint8_t)e;
    }
}
// where a thread's codes go, position by position, `step` positions apart
struct Dense { int C, blocks, inc_scales; long long inc_codes; };
inline Dense dense_of(int C, int step) { return {C, (C + 31) / 32, (C + 31) / 32 * step, (long long)C * step}; }
struct CodesCursor {
    uint8_t *codes, *scales;
    __device__ __forceinline__ CodesCursor(uint8_t* c, uint8_t* s, long long row, int vec, const Dense& d) : codes(c + row * d.C + 8 * vec), scales(s + row * d.blocks + (vec >> 2)) {}
    __device__ __forceinline__ void next(const Dense& d) { codes += d.inc_codes; scales += d.inc_scales; }
};

// How a launch walks a tensor: a block takes the positions [chunk * ppc, + ppc) of a sample and `cols` vectors of V channels; thread
// (row, col) takes every `rows`-th position of its vector.  With V = 8 the vectors of a row are counted up to a multiple of four, so that
// the four lanes of a checkpoint block are neighbours in one warp.
struct Walk {
    int C, HW, vecs, cols, rows, colblocks, ppc;
    long long chunks;           // per sample
    Dense dense;                // codes of positions `rows` apart
};
struct Spot { int col, row, v, p0, p1; long long n, chunk; bool on, has; };
__device__ __forceinline__ Spot spot(const Walk& w, int skip = 0) {
    Spot s;
    const long long b = blockIdx.x - skip;
    const long long t = b / w.colblocks;
    const int cb = (int)(b - t * w.colblocks);
    s.n = t / w.chunks;
    s.chunk = t - s.n * w.chunks;
    s.row = threadIdx.x / w.cols;
    s.col = threadIdx.x - s.row * w.cols;
    s.v = cb * w.cols + s.col;
    s.on = s.row < w.rows;
    s.has = s.on && s.v < w.vecs;
    s.p0 = (int)s.chunk * w.ppc;
    s.p1 = min(w.HW, s.p0 + w.ppc);
    return s;
}

// ---------------------------------------------------------------- encode, decode
// Rows of a multiple of eight channels at 16-byte boundaries: four lanes per block.  HBM-bound: 2 bytes read and 1.03 written per bf16 value
// (512 x 55 x 55 x 96: encode 83 us, decode 76, of 69 at the copy rate).
template <typename T, int FMT>
__global__ void __launch_bounds__(256) checkpoint_encode_kernel(const T* __restrict__ x, const Geo g, const Walk w, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    kn::pdl_sync();
    const Spot s = spot(w);
    if (!s.on) return;
    const T* xp = x + s.n * g.sn + 8 * s.v;
    constexpr int U = 4;
    Cursor c(g, s.p0 + s.row);
    CodesCursor k(codes, scales, s.n * w.HW + s.p0 + s.row, s.v, w.dense);
    for (int p = s.p0 + s.row; p < s.p1; p += U * w.rows) {
        Raw<T, 8> r[U] = {};
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s.has && p + u * w.rows < s.p1) r[u] = *(const Raw<T, 8>*)(xp + c.off);
            c.next(g);
        }
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * w.rows < s.p1) {
                float f[8];
                unpack<T, 8>(r[u], f);
                store_codes<T, FMT>(r[u], f, s.has, k.codes, k.scales);
            }
            k.next(w.dense);
        }
    }
}
template <typename T, int FMT>
__global__ void __launch_bounds__(256) checkpoint_decode_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const Geo g, const Walk w, T* __restrict__ out) {
    kn::pdl_sync();
    const Spot s = spot(w);
    if (!s.has) return;
    T* op = out + s.n * g.sn + 8 * s.v;
    constexpr int U = 4;
    Cursor c(g, s.p0 + s.row);
    CodesCursor k(const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales), s.n * w.HW + s.p0 + s.row, s.v, w.dense);
    for (int p = s.p0 + s.row; p < s.p1; p += U * w.rows) {
        uint2 r[U];
        uint8_t e[U];
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * w.rows < s.p1) { r[u] = *(const uint2*)k.codes; e[u] = *k.scales; }
            k.next(w.dense);
        }
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * w.rows < s.p1) {
                float f[8];
                code_values<FMT, 8>(r[u], f);
                const float sc = scale_of(e[u]);
                #pragma unroll
                for (int i = 0; i < 8; i += 2) un2(mul2(mk2(f[i], f[i + 1]), mk2(sc, sc)), f[i], f[i + 1]);
                *(Raw<T, 8>*)(op + c.off) = pack<T, 8>(f);
            }
            c.next(g);
        }
    }
}
// Any other rows: a warp per block (Walk's vectors), a lane per value; a warp walks down the positions of its block.  Bound by instructions, one value each
// (64 x 31 x 31 x 75 bf16: encode 15 us, decode 11).
struct WarpSpot { int lane, c, p0, p1; long long n; bool on; };
__device__ __forceinline__ WarpSpot warp_spot(const Walk& w) {
    const long long b = blockIdx.x, t = b / w.colblocks, n = t / w.chunks;
    const int warp = threadIdx.x >> 5, row = warp / w.cols, block = (int)(b - t * w.colblocks) * w.cols + warp - row * w.cols, p0 = (int)(t - n * w.chunks) * w.ppc;
    WarpSpot s;
    s.lane = threadIdx.x & 31;
    s.c = block * 32 + s.lane;
    s.n = n;
    s.p0 = p0 + row;
    s.p1 = min(w.HW, p0 + w.ppc);
    s.on = row < w.rows && block < w.vecs;
    return s;
}
template <typename T, int FMT>
__global__ void __launch_bounds__(256) checkpoint_encode_any_kernel(const T* __restrict__ x, const Geo g, const Walk w, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    kn::pdl_sync();
    const WarpSpot s = warp_spot(w);
    if (!s.on) return;
    const bool has = s.c < w.C;
    const T* xp = x + s.n * g.sn + s.c;
    const long long row0 = s.n * w.HW + s.p0;
    uint8_t *cp = codes + row0 * w.C + s.c, *ep = scales + row0 * w.dense.blocks + (s.c >> 5);
    Cursor c(g, s.p0);
    constexpr int U = 8;
    for (int p = s.p0; p < s.p1; p += U * w.rows) {
        float f[U];
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            f[u] = has && p + u * w.rows < s.p1 ? to_f<T>(xp[c.off]) : 0.f;
            c.next(g);
        }
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * w.rows >= s.p1) break;
            const uint32_t e = scale_byte<FMT>(__reduce_max_sync(~0u, __float_as_uint(f[u]) & 0x7fffffffu));
            if (has) *cp = codes_of<FMT, 1>(f + u, inverse_scale(e), e == 255u);
            if (s.lane == 0) *ep = (uint8_t)e;
            cp += w.dense.inc_codes;
            ep += w.dense.inc_scales;
        }
    }
}
template <typename T, int FMT>
__global__ void __launch_bounds__(256) checkpoint_decode_any_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const Geo g, const Walk w, T* __restrict__ out) {
    kn::pdl_sync();
    const WarpSpot s = warp_spot(w);
    if (!s.on || s.c >= w.C) return;
    T* op = out + s.n * g.sn + s.c;
    const long long row0 = s.n * w.HW + s.p0;
    const uint8_t *cp = codes + row0 * w.C + s.c, *ep = scales + row0 * w.dense.blocks + (s.c >> 5);
    Cursor c(g, s.p0);
    constexpr int U = 8;
    for (int p = s.p0; p < s.p1; p += U * w.rows) {
        uint8_t q[U], e[U];
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * w.rows < s.p1) { q[u] = *cp; e[u] = *ep; }
            cp += w.dense.inc_codes;
            ep += w.dense.inc_scales;
        }
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * w.rows >= s.p1) break;
            float f;
            code_values<FMT, 1>(q[u], &f);
            op[c.off] = from_f<T>(f * scale_of(e[u]));
            c.next(g);
        }
    }
}

}  // namespace op
