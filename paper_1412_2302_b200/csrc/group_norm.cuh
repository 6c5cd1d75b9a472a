// Group normalisation with an activation over channels-last tensors, forward and backward.
//
//   mean, var over the positions and the C / groups channels of a group of one sample;  rstd = 1 / sqrt(var + eps)
//   z = (x - mean) rstd w + b,  y = act(z)
//   dz = dy act'(z);  db = sum dz,  dw = sum dz xhat with xhat = (x - mean) rstd
//   dx = rstd (dz w - c1 - xhat c2),  c1 = mean(dz w), c2 = mean(dz w xhat) over the group
//
// Written with d = x - mean and a = rstd w as  z = d a + b  and  dx = dz a + (d (-rstd^2 c2) - rstd c1): two packed instructions per pair
// of channels each.  Both directions are HBM-bound: x in and y out; dy and x in and dx out.  Measured, bf16 (at the copy rate): 128 x 27 x 27 x 256, a launch per
// direction, forward 27 us (14.6), SiLU 32, backward 44 (21.9), SiLU 63; 512 x 55 x 55 x 96, read twice from memory, forward 164 (91), backward 255 (136), ReLU 274, SiLU 316.
// Small calls are bound by their launches and a chain of sums and barriers: 1 x 13 x 13 x 384 7.4 us.
//
// Sums.  Where a block keeps its values, it goes over them twice, the second time with the first's mean as the shift.  Elsewhere a thread sums, for
// each of its channels, the differences from the first value and their squares, in fp32; after 8 values, 40, 72 and so on it moves to those from the mean
// so far.  So nothing cancels as it would in E[x^2] - mean^2, however far the mean is from
// zero, nor where the first value lies far from all others: differences
// from that one alone left rstd off by 1.7e-3 at 444 x 256 x 256 x 8.
// From there on parts of n values are joined by their means, each held as hi + lo, and their squared
// deviations M2 from them (Part below): means as differences from one of them, M2 = sum M2_i + n_i (mean_i - mean)^2, all of one sign.  The order is
// fixed, so results repeat bit for bit.  (fp64 sums of values and squares do as well but took 3 to 8 us of a call: conversions, divisions, roots.)
#pragma once
#include "checkpoint.cuh"

namespace op {

enum { kActNone = 0, kActRelu = 1, kActSilu = 2, kActAny = 3 };

template <int V> __device__ __forceinline__ void v_add(const float* a, const float* b, float* o) {
    if constexpr (V == 1) o[0] = a[0] + b[0];
    else {
        #pragma unroll
        for (int i = 0; i < V; i += 2) un2(add2(mk2(a[i], a[i + 1]), mk2(b[i], b[i + 1])), o[i], o[i + 1]);
    }
}
template <int V> __device__ __forceinline__ void v_mul(const float* a, const float* b, float* o) {
    if constexpr (V == 1) o[0] = a[0] * b[0];
    else {
        #pragma unroll
        for (int i = 0; i < V; i += 2) un2(mul2(mk2(a[i], a[i + 1]), mk2(b[i], b[i + 1])), o[i], o[i + 1]);
    }
}
template <int V> __device__ __forceinline__ void v_fma(const float* a, const float* b, const float* c, float* o) {
    if constexpr (V == 1) o[0] = fmaf(a[0], b[0], c[0]);
    else {
        #pragma unroll
        for (int i = 0; i < V; i += 2) un2(fma2(mk2(a[i], a[i + 1]), mk2(b[i], b[i + 1]), mk2(c[i], c[i + 1])), o[i], o[i + 1]);
    }
}
// s = 1 / (1 + e^-z).  fp32 tensors take the accurate functions; 16-bit ones the hardware's approximate ones, without their care for subnormal
// numbers (relative error below 2^-20 for |z| < 16, next to a rounding of 2^-9 or 2^-12; below z = -87 the result is 0).  SiLU's passes are bound by the
// instructions they issue: two values sharing a reciprocal (1 / a = b / (a b)) save half of those, but take 20 instructions more per eight values.
template <typename T, int V> __device__ __forceinline__ void sigmoid(const float* z, float* s) {
    if constexpr (sizeof(T) == 4) {
        #pragma unroll
        for (int i = 0; i < V; ++i) s[i] = __fdiv_rn(1.f, 1.f + expf(-z[i]));
    } else {
        float t[V], one[V], ls[V];
        #pragma unroll
        for (int i = 0; i < V; ++i) { one[i] = 1.f; ls[i] = -1.44269504f; }
        v_mul<V>(z, ls, t);
        #pragma unroll
        for (int i = 0; i < V; ++i) asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(t[i]));
        v_add<V>(t, one, t);
        #pragma unroll
        for (int i = 0; i < V; ++i) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s[i]) : "f"(t[i]));
    }
}
// ACT: the activation, or kActAny to take it from `act`
template <typename T, int V, int ACT> __device__ __forceinline__ void activate(int act, float* z) {
    if (ACT != kActAny) act = ACT;
    if (act == kActRelu) {
        #pragma unroll
        for (int i = 0; i < V; ++i) z[i] = z[i] < 0.f ? 0.f : z[i];          // keeps NaN
    } else if (act == kActSilu) {
        float s[V];
        sigmoid<T, V>(z, s);
        v_mul<V>(z, s, z);
    }
}

struct NormShape {
    int C, HW, groups, cg;
    FastDiv by_cg;
    float eps;
    int act;
    __device__ __forceinline__ int group(int c) const { return (int)by_cg.div((uint32_t)c); }
};

// per-channel constants of a thread's vector
template <int V> struct Chan { float nm[V], a[V], b[V]; uint32_t negative; };      // negative: (backward) the sign bit where an a is
template <int V>
__device__ __forceinline__ void load_chan(Chan<V>& k, const NormShape& s, const float* mean, const float* rstd, const float* weight, const float* bias, long long n, int c0) {
    #pragma unroll
    for (int i = 0; i < V; ++i) {
        const long long g = n * s.groups + s.group(c0 + i);
        k.nm[i] = -mean[g];
        k.a[i] = rstd[g] * (weight ? weight[c0 + i] : 1.f);
        k.b[i] = bias ? bias[c0 + i] : 0.f;
    }
}

// ---------------------------------------------------------------- forward, any size: sums, statistics, result
// n values by their mean hi + lo and their squared deviations from it
struct Part { float hi, lo, m2; };
// a thread's values of a channel: n of them, S the sum of their differences from K (nK = -K), Q that of the squares
__device__ __forceinline__ Part moments(int n, float nK, float S, float Q) {
    const float d = n ? __fdividef(S, (float)n) : 0.f, hi = d - nK;
    return {hi, (-nK - hi) + d, fmaf(-S, d, Q)};
}
// The parts get(0) .. get(count - 1) of n(i) values each, joined; inv = 1 / all their values.  The mean is first taken to fp32, then what is left over:
// the second pass sums small differences whatever the first part was.
template <int UNROLL, typename G, typename N> __device__ __forceinline__ Part join(int count, float inv, G get, N n) {
    const float ref = get(0).hi;
    float m = 0.f, e = 0.f, q = 0.f;
    #pragma unroll UNROLL
    for (int i = 0; i < count; ++i) m = fmaf(n(i), get(i).hi - ref, m);
    const float hi = fmaf(m, inv, ref);
    #pragma unroll UNROLL
    for (int i = 0; i < count; ++i) {
        const Part t = get(i);
        const float d = (t.hi - hi) + t.lo, w = n(i) * d;
        e += w;
        q += fmaf(w, d, t.m2);
    }
    const float lo = e * inv;
    return {hi, lo, fmaf(-e, lo, q)};
}
// A running sum whose roundings are summed beside it (the error of an fp32 addition is an fp32 number), for sums that are as long as a caller's
// tensor has samples: a plain one is off by 2^-25 of its value per term where the terms are alike, 65536 samples of 9 x 9 x 32 by 1.1e-4.
struct LongSum {
    float s = 0.f, e = 0.f;
    __device__ __forceinline__ void add(float v) {
        const float t = s + v, b = t - s;
        e += (s - (t - b)) + (v - b);
        s = t;
    }
    __device__ __forceinline__ float value() const { return e == e ? s + e : s; }      // (beside an infinity there is no error to speak of)
};
template <int N> __device__ __forceinline__ float sum_of(float* v) {      // N a power of two, in pairs
    #pragma unroll
    for (int o = N / 2; o; o /= 2) {
        #pragma unroll
        for (int i = 0; i < o; ++i) v[i] += v[i + o];
    }
    return v[0];
}
// the sum over `lanes` neighbouring lanes (a power of two; all 32 of the warp call it)
__device__ __forceinline__ float lanes_sum(float t, int lanes) {
    for (int o = lanes >> 1; o; o >>= 1) t += __shfl_xor_sync(~0u, t, o);
    return t;
}
// Per-thread sums of a block in shared memory, by vector element and thread: pitch = threads + 4, so that neighbouring threads' stores and the
// reads of neighbouring channels (elements of neighbouring threads) each fall into different banks.
template <int V> struct Table {
    float* p;
    int pitch;
    __device__ __forceinline__ float& at(int k, int i, int t) const { return p[(k * V + i) * pitch + t]; }
};
__device__ __forceinline__ float warp_sum(float t) {
    #pragma unroll
    for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(~0u, t, o);
    return t;
}
__device__ __forceinline__ float2 warp_sum(float2 t) {
    #pragma unroll
    for (int o = 16; o; o >>= 1) { t.x += __shfl_xor_sync(~0u, t.x, o); t.y += __shfl_xor_sync(~0u, t.y, o); }
    return t;
}
// the threads' parts of channel c (element c % V of column c / V), joined: the first `more` rows of threads have n_lo + 1 values, the others n_lo
template <int V> __device__ __forceinline__ Part join_rows(const Table<V>& s, int c, int rows, int cols, int more, float n_lo, float inv) {
    const int i = c % V, t = c / V;
    return join<4>(rows, inv, [&](int r) { return Part{s.at(0, i, r * cols + t), s.at(1, i, r * cols + t), s.at(2, i, r * cols + t)}; }, [&](int r) { return r < more ? n_lo + 1.f : n_lo; });
}
__device__ __forceinline__ float2 statistics(const Part& t, const NormShape& s) {
    const float var = __fdiv_rn(t.m2, (float)s.HW * (float)s.cg);
    return make_float2(t.hi + t.lo, __frsqrt_rn((var < 0.f ? 0.f : var) + s.eps));      // (keeps NaN)
}

// From n values' sums of differences from K, S, and of their squares, Q, to those from a K nearer to their mean: with d the step, sum (x - K - d)
// = S - n d and sum (x - K - d)^2 = Q - d (2 S - n d).
template <int V> __device__ __forceinline__ void move_mean(float n, float* nK, float* S, float* Q) {
    const float per = -__fdividef(1.f, n);
    #pragma unroll
    for (int i = 0; i < V; ++i) {
        const float k = fmaf(S[i], per, nK[i]), nd = k - nK[i], r = fmaf(n, nd, S[i]);
        Q[i] = fmaf(nd, S[i] + r, Q[i]);
        S[i] = r;
        nK[i] = k;
    }
}
template <typename T, int V>
__global__ void __launch_bounds__(256) gn_sums_kernel(const T* __restrict__ x, const Geo g, const Walk w, float4* __restrict__ partial) {
    kn::pdl_sync();
    __shared__ float sums[3 * V * 260];
    const Table<V> table{sums, 260};
    const Spot s = spot(w);
    constexpr int U = 8;
    float nK[V], S[V], Q[V];                   // a number near the mean, negative; the sums of the differences from it and of their squares
    #pragma unroll
    for (int i = 0; i < V; ++i) nK[i] = S[i] = Q[i] = 0.f;
    int cnt = 0;
    if (s.has && s.p0 + s.row < s.p1) {
        const T* xp = x + s.n * g.sn + V * s.v;
        Cursor c(g, s.p0 + s.row);
        unpack<T, V>(*(const Raw<T, V>*)(xp + c.off), nK);
        #pragma unroll
        for (int i = 0; i < V; ++i) nK[i] = -nK[i];
        cnt = (s.p1 - s.p0 - s.row + w.rows - 1) / w.rows;
        for (int it = 0; it < cnt; it += U) {
            Raw<T, V> r[U];
            #pragma unroll
            for (int u = 0; u < U; ++u) {
                if (it + u < cnt) r[u] = *(const Raw<T, V>*)(xp + c.off);
                c.next(g);
            }
            #pragma unroll
            for (int u = 0; u < U; ++u)
                if (it + u < cnt) {
                    float f[V];
                    unpack<T, V>(r[u], f);
                    v_add<V>(f, nK, f);
                    v_add<V>(S, f, S);
                    v_fma<V>(f, f, Q, Q);
                }
            if (it % (4 * U) == 0) move_mean<V>((float)min(it + U, cnt), nK, S, Q);
        }
    }
    #pragma unroll
    for (int i = 0; i < V; ++i) {
        const Part t = moments(cnt, nK[i], S[i], Q[i]);
        table.at(0, i, threadIdx.x) = t.hi; table.at(1, i, threadIdx.x) = t.lo; table.at(2, i, threadIdx.x) = t.m2;
    }
    __syncthreads();
    const int nch = w.cols * V, c0 = (s.v - s.col) * V, np = s.p1 - s.p0;
    for (int j = threadIdx.x; j < nch && c0 + j < w.C; j += 256) {
        const Part t = join_rows<V>(table, j, min(w.rows, np), w.cols, np % w.rows, (float)(np / w.rows), __fdividef(1.f, (float)np));
        partial[(s.n * w.chunks + s.chunk) * w.C + c0 + j] = make_float4(t.hi, t.lo, t.m2, 0.f);
    }
}
__device__ __forceinline__ float2 block_sum(float2 t, float2* red) {        // of all 256 threads
    t = warp_sum(t);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = t;
    __syncthreads();
    t = red[0];
    #pragma unroll
    for (int k = 1; k < 8; ++k) { t.x += red[k].x; t.y += red[k].y; }
    return t;
}
// The chunks' parts [chunks][C] of a group's channels, joined by a block, or by a warp where there are groups enough (4096 groups of 30 parts: 7.6 -> 2.5 us).
template <bool BLOCK>
__global__ void __launch_bounds__(256) gn_statistics_kernel(const float4* __restrict__ partial, const NormShape s, long long all_groups, int chunks, int ppc, float* __restrict__ mean, float* __restrict__ rstd) {
    kn::pdl_sync();
    __shared__ float2 red[8];
    const long long id = BLOCK ? blockIdx.x : blockIdx.x * 8ll + (threadIdx.x >> 5);
    if (id >= all_groups) return;
    constexpr int N = BLOCK ? 256 : 32;
    const int me = threadIdx.x % N;
    const long long n = id / s.groups;
    const int g = (int)(id - n * s.groups), total = chunks * s.cg;
    const float4* p = partial + n * chunks * s.C + (long long)g * s.cg;
    const float ref = p[0].x, lo = (float)ppc, last = (float)(s.HW - (chunks - 1) * ppc), count = (float)s.HW * (float)s.cg;
    auto sum = [&](float2 t) { return BLOCK ? block_sum(t, red) : warp_sum(t); };
    float2 t = make_float2(0.f, 0.f);
    #pragma unroll 4
    for (int i = me; i < total; i += N) {
        const int k = s.group(i);
        t.x = fmaf(k == chunks - 1 ? last : lo, p[(long long)k * s.C + (i - k * s.cg)].x - ref, t.x);
    }
    const float hi = ref + __fdiv_rn(sum(t).x, count);
    LongSum t1, t2;
    for (int i = me; i < total; i += 4 * N) {
        float u1[4], u2[4];
        #pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = i + u * N;
            u1[u] = u2[u] = 0.f;
            if (j < total) {
                const int k = s.group(j);
                const float4 q = p[(long long)k * s.C + (j - k * s.cg)];
                const float d = (q.x - hi) + q.y, w = (k == chunks - 1 ? last : lo) * d;
                u1[u] = w;
                u2[u] = fmaf(w, d, q.z);
            }
        }
        t1.add(sum_of<4>(u1));
        t2.add(sum_of<4>(u2));
    }
    t = make_float2(t1.value(), t2.value());
    t = sum(t);
    if (me == 0) {
        const float l = __fdiv_rn(t.x, count);
        const float2 r = statistics(Part{hi, l, fmaf(-t.x, l, t.y)}, s);
        mean[id] = r.x;
        rstd[id] = r.y;
    }
}
struct Keep { uint8_t *codes, *scales; int fmt; };        // codes == nullptr: nothing kept
template <typename T>
__device__ __forceinline__ void keep_codes(const Keep& k, const Raw<T, 8>& r, const float* f, bool has, CodesCursor& c) {
    if (k.fmt == kSrcInt8) store_codes<T, kSrcInt8>(r, f, has, c.codes, c.scales);
    else store_codes<T, kSrcE4m3>(r, f, has, c.codes, c.scales);
}
template <typename T, int V, int ACT, bool KEEP>
__global__ void __launch_bounds__(256, V == 8 && !KEEP ? 4 : 3) gn_apply_kernel(const T* __restrict__ x, const Geo gx, const Walk w, const NormShape sh, const float* __restrict__ weight,
                                                                              const float* __restrict__ bias, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                                              T* __restrict__ y, const Geo gy, const Keep kx, const Keep ky) {
    kn::pdl_sync();
    const Spot s = spot(w);
    const int p0 = s.p0 + s.row;
    if (!s.on || p0 >= s.p1) return;
    Chan<V> k = {};
    if (s.has) load_chan<V>(k, sh, mean, rstd, weight, bias, s.n, V * s.v);
    const T* xp = x + s.n * gx.sn + V * s.v;
    T* yp = y + s.n * gy.sn + V * s.v;
    Cursor cx(gx, p0), cy(gy, p0);
    CodesCursor ckx(kx.codes, kx.scales, s.n * w.HW + p0, s.v, w.dense), cky(ky.codes, ky.scales, s.n * w.HW + p0, s.v, w.dense);
    constexpr int U = 4;                       // vectors in flight: bound by their number (two: 155 us for 512 x 55 x 55 x 96, 3.8 TB/s; four: 96)
    for (int p = p0; p < s.p1; p += U * w.rows) {
        Raw<T, V> r[U] = {};
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s.has && p + u * w.rows < s.p1) r[u] = *(const Raw<T, V>*)(xp + cx.off);
            cx.next(gx);
        }
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * w.rows >= s.p1) break;
            float f[V], z[V];
            unpack<T, V>(r[u], f);
            if constexpr (V == 8 && KEEP)
                if (kx.codes) { keep_codes<T>(kx, r[u], f, s.has, ckx); ckx.next(w.dense); }
            v_add<V>(f, k.nm, f);
            v_fma<V>(f, k.a, k.b, z);
            activate<T, V, ACT>(sh.act, z);
            Raw<T, V> out = pack<T, V>(z);
            if (s.has) *(Raw<T, V>*)(yp + cy.off) = out;
            cy.next(gy);
            if constexpr (V == 8 && KEEP)
                if (ky.codes) {                     // of y as it is stored
                    if (!s.has) out = Raw<T, V>{};
                    unpack<T, 8>(out, f);
                    keep_codes<T>(ky, out, f, s.has, cky);
                    cky.next(w.dense);
                }
        }
    }
}

// ---------------------------------------------------------------- backward
// where a backward pass reads x: a tensor, or the codes and exponents of a checkpoint (dense)
struct Source { const void* x; const uint8_t *codes, *scales; };
template <typename T, int V, int SRC> struct Fetch {
    using R = typename std::conditional<SRC == kSrcSame, Raw<T, V>, Raw<uint8_t, V>>::type;
    R r;
    uint8_t e;
    // f = x, or the code that stands for it (x = f * scale(), exactly); d = x - mean, rounded once
    __device__ __forceinline__ float scale() const {
        if constexpr (SRC == kSrcSame) return 1.f;
        else return scale_of(e);
    }
    __device__ __forceinline__ void value(const float* nm, float* f, float* d) const {
        if constexpr (SRC == kSrcSame) {
            unpack<T, V>(r, f);
            v_add<V>(f, nm, d);
        } else {
            code_values<SRC, V>(r, f);
            const float sc = scale();
            float s[V];
            #pragma unroll
            for (int i = 0; i < V; ++i) s[i] = sc;
            v_fma<V>(f, s, nm, d);
        }
    }
};
// a thread's walk over x in either form
template <typename T, int V, int SRC> struct SourceCursor {
    Cursor c;
    const T* x;
    const uint8_t *codes, *scales;
    template <typename W> __device__ __forceinline__ SourceCursor(const Source& s, const Geo& g, const W& w, long long n, int p, int v)
        : c(g, SRC == kSrcSame ? p : 0), x(SRC == kSrcSame ? (const T*)s.x + n * g.sn + V * v : nullptr), codes(SRC == kSrcSame ? nullptr : s.codes + (n * w.HW + p) * w.C + V * v),
          scales(SRC == kSrcSame ? nullptr : s.scales + (n * w.HW + p) * w.dense.blocks + V * v / 32) {}
    __device__ __forceinline__ void load(Fetch<T, V, SRC>& f) const {
        using R = typename Fetch<T, V, SRC>::R;
        if constexpr (SRC == kSrcSame) f.r = *(const R*)(x + c.off);
        else { f.r = *(const R*)codes; f.e = *scales; }
    }
    __device__ __forceinline__ const void* place() const { return SRC == kSrcSame ? (const void*)(x + c.off) : (const void*)codes; }
    template <typename W> __device__ __forceinline__ void next(const Geo& g, const W& w) {
        if constexpr (SRC == kSrcSame) c.next(g);
        else { codes += w.dense.inc_codes; scales += w.dense.inc_scales; }
    }
};
struct BackwardArgs {
    const float *mean, *rstd, *weight, *bias;
};
// A thread's channels in a backward pass: nm, a and b, where ReLU has in the place of b a number to compare with.  z > 0 holds for x > theta (w > 0) or x < theta
// (w < 0) with theta = mean - b / (rstd w): theta in fp64, rounded to fp32 downwards (upwards), decides for every fp32 x as the real one does, where
// z in fp32 is off by 2^-23 |b| about zero.  b holds -theta; x - theta with a's sign has z's (their product may be too small for fp32).  Where w is zero z is
// the bias, for all x: b holds an infinity that gives x + b the sign that is wanted.
template <int V, int ACT>
__device__ __forceinline__ void load_backward_chan(Chan<V>& k, const NormShape& sh, const BackwardArgs& A, long long n, int c0) {
    load_chan<V>(k, sh, A.mean, A.rstd, A.weight, A.bias, n, c0);
    k.negative = 0;
    if (ACT == kActRelu || (ACT == kActAny && sh.act == kActRelu)) {
        #pragma unroll
        for (int i = 0; i < V; ++i) {
            const double a = (double)A.rstd[n * sh.groups + sh.group(c0 + i)] * (A.weight ? (double)A.weight[c0 + i] : 1.);
            const double theta = -(double)k.nm[i] - (double)k.b[i] / a;
            k.b[i] = a == 0. ? copysignf(__uint_as_float(0x7f800000u), k.b[i] <= 0.f ? -k.a[i] : k.a[i]) : -(a > 0. ? __double2float_rd(theta) : __double2float_ru(theta));
            k.negative |= __float_as_uint(k.a[i]) & 0x80000000u;
        }
    }
}
// d = x - mean, and dz in the place of dy
template <typename T, int V, int SRC, int ACT>
__device__ __forceinline__ void activation_gradient(int act, const Chan<V>& k, const Fetch<T, V, SRC>& fx, float* d, float* dy) {
    float x[V];
    fx.value(k.nm, x, d);
    if (ACT != kActAny) act = ACT;
    if (act == kActNone) return;
    float z[V];
    if (act == kActRelu) {
        const float sc = fx.scale();
        if constexpr (SRC != kSrcSame) {
            #pragma unroll
            for (int i = 0; i < V; ++i) x[i] *= sc;
        }
        v_add<V>(x, k.b, z);
        if constexpr (V == 1) z[0] = __uint_as_float(__float_as_uint(z[0]) ^ k.negative);
        else if (k.negative) {
            #pragma unroll
            for (int i = 0; i < V; ++i) z[i] = __uint_as_float(__float_as_uint(z[i]) ^ (__float_as_uint(k.a[i]) & 0x80000000u));
        }
        #pragma unroll
        for (int i = 0; i < V; ++i) dy[i] = z[i] <= 0.f ? 0.f : dy[i];      // (passes NaN)
    } else {
        v_fma<V>(d, k.a, k.b, z);
        float s[V], u[V], one[V], minus[V];
        #pragma unroll
        for (int i = 0; i < V; ++i) { one[i] = 1.f; minus[i] = -1.f; }
        sigmoid<T, V>(z, s);
        v_fma<V>(s, minus, one, u);
        v_mul<V>(z, s, z);
        v_fma<V>(z, u, s, u);                  // s + z s (1 - s)
        v_mul<V>(dy, u, dy);
    }
}
// Positions whose loads a thread of the two kernels below has under way, of two tensors each, and blocks per SM (two with 128 registers, three with 80).
// 512 x 55 x 55 x 96 bf16, ReLU, both kernels: four and two from x 275 us, from int8 codes 303, from e4m3 301; three and two 297, 327 and 324; two and three
// 322, 389 and 376.  In fp32 (a quarter of the samples, from x): three and two 131, four and two 143.
template <int V> constexpr int kBackwardBlocks = V == 8 ? 2 : 3;
template <typename T, int V> constexpr int kBackwardLoads = V == 8 && sizeof(T) == 4 ? 3 : 4;
template <typename T, int V, int SRC, int ACT>
__global__ void __launch_bounds__(256, kBackwardBlocks<V>) gn_backward_sums_kernel(const T* __restrict__ dy, const Geo gdy, const Source src, const Geo gx, const Walk w, const NormShape sh,
                                                               const BackwardArgs A, float* __restrict__ partial) {
    kn::pdl_sync();
    __shared__ float sums[2 * V * 260];
    const Table<V> table{sums, 260};
    const Spot s = spot(w);
    constexpr int U = kBackwardLoads<T, V>;
    float S1[V], S2[V];
    #pragma unroll
    for (int i = 0; i < V; ++i) S1[i] = S2[i] = 0.f;
    if (s.has) {
        Chan<V> k;
        load_backward_chan<V, ACT>(k, sh, A, s.n, V * s.v);
        const T* dp = dy + s.n * gdy.sn + V * s.v;
        Cursor c(gdy, s.p0 + s.row);
        SourceCursor<T, V, SRC> cx(src, gx, w, s.n, s.p0 + s.row, s.v);
        for (int p = s.p0 + s.row; p < s.p1; p += U * w.rows) {
            Raw<T, V> r[U];
            Fetch<T, V, SRC> fx[U];
            #pragma unroll
            for (int u = 0; u < U; ++u) {
                if (p + u * w.rows < s.p1) {
                    r[u] = *(const Raw<T, V>*)(dp + c.off);
                    cx.load(fx[u]);
                }
                c.next(gdy);
                cx.next(gx, w);
            }
            #pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * w.rows < s.p1) {
                    float f[V], q[V];
                    unpack<T, V>(r[u], q);
                    activation_gradient<T, V, SRC, ACT>(sh.act, k, fx[u], f, q);
                    v_add<V>(S1, q, S1);
                    v_fma<V>(f, q, S2, S2);
                }
        }
    }
    #pragma unroll
    for (int i = 0; i < V; ++i) { table.at(0, i, threadIdx.x) = S1[i]; table.at(1, i, threadIdx.x) = S2[i]; }
    __syncthreads();
    const int nch = w.cols * V, c0 = (s.v - s.col) * V;
    for (int j = threadIdx.x; j < nch; j += 256) {
        if (c0 + j >= w.C) break;
        float t1[4] = {}, t2[4] = {};                       // four chains: up to 256 rows
        for (int r = 0; r < w.rows; r += 4) {
            #pragma unroll
            for (int q = 0; q < 4; ++q)
                if (r + q < w.rows) { t1[q] += table.at(0, j % V, (r + q) * w.cols + j / V); t2[q] += table.at(1, j % V, (r + q) * w.cols + j / V); }
        }
        float* o = partial + (s.n * w.chunks + s.chunk) * 2 * w.C + c0 + j;
        o[0] = (t1[0] + t1[1]) + (t1[2] + t1[3]);
        o[w.C] = ((t2[0] + t2[1]) + (t2[2] + t2[3])) * A.rstd[s.n * sh.groups + sh.group(c0 + j)];       // of xhat
    }
}
// c1 and c2 of a group from the chunks' sums [chunks][2][C], by a block or a warp
template <bool BLOCK>
__global__ void __launch_bounds__(256) gn_backward_group_kernel(const float* __restrict__ partial, const NormShape sh, long long all_groups, int chunks, const BackwardArgs A, float2* __restrict__ c12) {
    kn::pdl_sync();
    __shared__ float2 red[8];
    const long long id = BLOCK ? blockIdx.x : blockIdx.x * 8ll + (threadIdx.x >> 5);
    if (id >= all_groups) return;
    constexpr int N = BLOCK ? 256 : 32;
    const int me = threadIdx.x % N;
    const long long n = id / sh.groups;
    const int g = (int)(id - n * sh.groups), total = chunks * sh.cg;
    const float* p = partial + n * chunks * 2 * sh.C + (long long)g * sh.cg;
    LongSum t1, t2;
    for (int i = me; i < total; i += 4 * N) {
        float u1[4], u2[4];
        #pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = i + u * N;
            u1[u] = u2[u] = 0.f;
            if (j < total) {
                const int k = sh.group(j), c = j - k * sh.cg;
                const float wt = A.weight ? A.weight[g * sh.cg + c] : 1.f;
                const float* q = p + (long long)k * 2 * sh.C + c;
                u1[u] = wt * q[0];
                u2[u] = wt * q[sh.C];
            }
        }
        t1.add(sum_of<4>(u1));
        t2.add(sum_of<4>(u2));
    }
    float2 t = make_float2(t1.value(), t2.value());
    t = BLOCK ? block_sum(t, red) : warp_sum(t);
    const float m = (float)sh.HW * (float)sh.cg;
    if (me == 0) c12[id] = make_float2(__fdiv_rn(t.x, m), __fdiv_rn(t.y, m));
}
// dweight and dbias: the sums [n][2][C] of the samples (or of their chunks).  A block takes 32 channels, its warps every WARPS-th row.
template <int WARPS>
__device__ __forceinline__ void parameter_gradient(const float* __restrict__ partial, int C, long long n, int block, float2* red /* [WARPS][33] */, float* __restrict__ dweight, float* __restrict__ dbias) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = block * 32 + lane;
    LongSum b, w;
    if (c < C) {
        const float* p = partial + c;
        for (long long i = warp; i < n; i += 8 * WARPS) {
            float v[8], q[8];
            #pragma unroll
            for (int u = 0; u < 8; ++u) {
                const long long k = i + u * WARPS;
                v[u] = k < n ? p[k * 2 * C] : 0.f;
                q[u] = k < n ? p[k * 2 * C + C] : 0.f;
            }
            b.add(sum_of<8>(v));
            w.add(sum_of<8>(q));
        }
    }
    float2 t = make_float2(b.value(), w.value());
    red[warp * 33 + lane] = t;
    __syncthreads();
    if (warp == 0 && c < C) {
        #pragma unroll 8
        for (int k = 1; k < WARPS; ++k) { t.x += red[k * 33 + lane].x; t.y += red[k * 33 + lane].y; }
        if (dbias) dbias[c] = t.x;
        if (dweight) dweight[c] = t.y;
    }
}
__global__ void __launch_bounds__(1024) gn_parameter_gradient_kernel(const float* __restrict__ partial, int C, long long n, float* __restrict__ dweight, float* __restrict__ dbias) {
    kn::pdl_sync();
    __shared__ float2 red[32 * 33];
    parameter_gradient<32>(partial, C, n, blockIdx.x, red, dweight, dbias);
}
template <typename T, int V, int SRC, int ACT>
__global__ void __launch_bounds__(256, kBackwardBlocks<V>) gn_backward_apply_kernel(const T* __restrict__ dy, const Geo gdy, const Source src, const Geo gx, const Walk w, const NormShape sh,
                                                                const BackwardArgs A, const float2* __restrict__ c12, T* __restrict__ dx, const Geo gdx, const float* __restrict__ partial,
                                                                long long partials, int extra, float* __restrict__ dweight, float* __restrict__ dbias) {
    kn::pdl_sync();
    // the first `extra` blocks add up the parameters' gradients beside the others' work (a launch of their own took 8 us)
    __shared__ float2 red[8 * 33];
    if (blockIdx.x < extra) { parameter_gradient<8>(partial, w.C, partials, blockIdx.x, red, dweight, dbias); return; }
    const Spot s = spot(w, extra);
    if (!s.has) return;
    Chan<V> k;
    load_backward_chan<V, ACT>(k, sh, A, s.n, V * s.v);
    float B[V], D[V];
    #pragma unroll
    for (int i = 0; i < V; ++i) {
        const long long g = s.n * sh.groups + sh.group(V * s.v + i);
        const float2 c = c12[g];
        const float r = A.rstd[g];
        B[i] = -r * (r * c.y);
        D[i] = -r * c.x;
    }
    const T* dp = dy + s.n * gdy.sn + V * s.v;
    T* op = dx + s.n * gdx.sn + V * s.v;
    constexpr int U = kBackwardLoads<T, V>;
    Cursor c(gdy, s.p0 + s.row), co(gdx, s.p0 + s.row);
    SourceCursor<T, V, SRC> cx(src, gx, w, s.n, s.p0 + s.row, s.v);
    for (int p = s.p0 + s.row; p < s.p1; p += U * w.rows) {
        Raw<T, V> r[U];
        Fetch<T, V, SRC> fx[U];
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * w.rows < s.p1) {
                r[u] = *(const Raw<T, V>*)(dp + c.off);
                cx.load(fx[u]);
            }
            c.next(gdy);
            cx.next(gx, w);
        }
        #pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u * w.rows < s.p1) {
                float f[V], q[V];
                unpack<T, V>(r[u], q);
                activation_gradient<T, V, SRC, ACT>(sh.act, k, fx[u], f, q);
                v_fma<V>(f, B, D, f);
                v_fma<V>(q, k.a, f, q);
                *(Raw<T, V>*)(op + co.off) = pack<T, V>(q);
                co.next(gdx);
            }
    }
}


// ---------------------------------------------------------------- one launch per direction: whole groups of a sample per block
//
// A block takes a slice of the channels (of whole groups, and of whole checkpoint blocks) of a sample and keeps it: a thread's vectors stay raw in its own slots
// of shared memory, filled by asynchronous copies, while the block forms its groups' sums, and are then turned into the result, so every value is
// read from memory once.  Slots are private to a thread: no barrier stands between its copies and its reads.  Blocks are persistent: while a
// sample's results are formed, the vectors of the block's next sample are copied into the slots that have been read, so memory is read and
// written at the same time and does not wait for the sums.
//
// Slices that do not fit take the launches above, which read x twice.  (Spread over a cluster of up to eight blocks, with the sums going around it
// through distributed shared memory, they took longer than that: 128 x 55 x 55 x 96 forward 68 us against 57, backward from a checkpoint 149
// against 112.  The fixed work per sample, some 2000 instructions of each warp, was then paid for 20 vectors per thread.)
struct SliceWalk {
    int C, HW;                                // of the tensor
    int slices, Cs, groups;                   // channel slices; channels and groups of one
    int vecs, cols, rows, threads;            // vectors of a slice's row; rows = threads / cols
    int its;                                  // positions of a thread, at most
    int lanes, lc, lc_shift;                  // lanes that join a group's sums, lc = 2^lc_shift of them over its channels (powers of two)
    Dense dense;                              // codes of positions `rows` apart
};
constexpr int kSlThreads = 256;               // at most; two blocks per SM with 128 registers

template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
    if constexpr (BYTES == 32) { copy_async<16>(dst, src); copy_async<16>(dst + 16, (const uint8_t*)src + 16); }
    else if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
// a vector into its slot: asynchronously where it has at least four bytes
template <typename R> __device__ __forceinline__ void fill_slot(R* slot, const void* src) {
    if constexpr (sizeof(R) >= 4) copy_async<sizeof(R)>(tc::smem_u32(slot), src);
    else *slot = *(const R*)src;
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// waits until at most `pending` of the newest groups are still under way
__device__ __forceinline__ void copies_wait(int pending) {
    if (pending == 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else if (pending == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (pending == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else asm volatile("cp.async.wait_group 3;" ::: "memory");
}
constexpr int kSlBatches = 4;                 // groups of copies

// Shared memory behind the slots: the groups' results, two sums per thread and vector element; backward also two sums per channel, those of the block's last samples, the
// channels' weights and the groups' rstd.
template <int V> struct SliceSmem {
    float2* res;
    Table<V> part;
    float *chan, *acc, *weight, *rstd;
    __device__ __forceinline__ SliceSmem(uint8_t* p, const SliceWalk& w) {
        res = (float2*)p;
        part = {(float*)(res + w.groups), w.threads + 4};
        chan = part.p + 2 * V * part.pitch;
        acc = chan + 2 * w.Cs;
        weight = acc + 2 * w.Cs;
        rstd = weight + w.Cs;
    }
};
template <int V> inline size_t slice_scratch(const SliceWalk& w, bool backward) {
    return ((size_t)2 * V * (w.threads + 4) + (backward ? 5 * w.Cs + w.groups : 0)) * sizeof(float) + w.groups * sizeof(float2);
}
// a block's work: a slice (from channel c0, group g0 on) of the samples n0, n0 + step, ...
struct SliceSpot {
    long long n0, step;
    int c0, g0;
    __device__ __forceinline__ SliceSpot(const SliceWalk& w) {
        const uint32_t slice = blockIdx.x % (uint32_t)w.slices;
        n0 = blockIdx.x / (uint32_t)w.slices;
        step = gridDim.x / (uint32_t)w.slices;
        c0 = slice * w.Cs;
        g0 = slice * w.groups;
    }
};
// What the lanes of a group add up: the table's K sums of the channels c0 .. c0 + cg - 1 over the rows of threads r < rows, dealt to lanes by channel
// (w.lc of them) and by row.  These loops run a warp at a time with nothing to hide their latency, so they are kept to a load and an addition.
template <int V, int K> __device__ __forceinline__ void group_sums(const SliceWalk& w, const Table<V>& table, uint32_t c0, uint32_t cg, int rows, uint32_t lane, float* out) {
    const uint32_t ci = lane & (w.lc - 1);
    const int ri = lane >> w.lc_shift, lr = w.lanes >> w.lc_shift, step = lr * w.cols, next = V * table.pitch;
    for (uint32_t c = c0 + ci; c < c0 + cg; c += w.lc) {
        const float* p = table.p + (c % V) * table.pitch + c / V + ri * w.cols;
        #pragma unroll 4
        for (int r = ri; r < rows; r += lr, p += step) {
            #pragma unroll
            for (int k = 0; k < K; ++k) out[k] += p[k * next];
        }
    }
}
// V channels' parameters, or `other` where there are none
template <int V> __device__ __forceinline__ void load_parameters(const float* p, int c, float other, float* out) {
    if (V == 8 && p && ((uintptr_t)p & 15) == 0) {
        *(float4*)out = *(const float4*)(p + c);
        *(float4*)(out + 4) = *(const float4*)(p + c + 4);
    } else {
        #pragma unroll
        for (int i = 0; i < V; ++i) out[i] = p ? p[c + i] : other;
    }
}

// The values are at hand, so the sums go over them twice: the first sum's mean, off by some 2^-24 of the values' size, is the shift of the second, whose sums of
// differences and of squares then cancel nothing and can simply be added up.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kSlThreads, 2) gn_slice_forward_kernel(const T* __restrict__ x, const Geo gx, const SliceWalk w, const NormShape sh, long long samples,
                                                                         const float* __restrict__ weight, const float* __restrict__ bias, T* __restrict__ y, const Geo gy,
                                                                         float* __restrict__ mean, float* __restrict__ rstd, const Keep kx, const Keep ky) {
    kn::pdl_sync();
    extern __shared__ __align__(16) uint8_t smem[];
    using R = Raw<T, V>;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = w.threads >> 5;
    R* slots = (R*)smem + tid;
    const SliceSmem<V> m(smem + (size_t)w.its * w.threads * sizeof(R), w);
    const SliceSpot b(w);
    const int row = tid / w.cols, v = tid - row * w.cols, cv = b.c0 / V + v;      // cv: vector within the tensor's row
    const bool on = row < w.rows, has = on && v < w.vecs;
    const int cnt = on && row < w.HW ? (w.HW - row + w.rows - 1) / w.rows : 0;  // positions of this thread
    const int filled = has ? cnt : 0, batch = (w.its + kSlBatches - 1) / kSlBatches;
    const int rows = min(w.rows, w.HW), at_once = 32 / w.lanes, lane_g = lane / w.lanes, lane_i = lane % w.lanes;
    const float count = (float)w.HW * (float)sh.cg, per = __frcp_rn(count);
    if (b.n0 < samples) {
        Cursor c(gx, row);
        const T* xp = x + b.n0 * gx.sn + V * cv;
        #pragma unroll 1
        for (int bt = 0; bt < kSlBatches; ++bt) {
            const int e = min(filled, (bt + 1) * batch);
            #pragma unroll 4
            for (int it = bt * batch; it < e; ++it) {
                fill_slot(slots + it * w.threads, xp + c.off);
                c.next(gx);
            }
            copies_commit();
        }
    }
    #pragma unroll 1
    for (long long n = b.n0; n < samples; n += b.step) {
        float nK[V], S[V], Q[V];
        // the shift
        #pragma unroll
        for (int i = 0; i < V; ++i) S[i] = Q[i] = 0.f;
        #pragma unroll 1
        for (int bt = 0; bt < kSlBatches; ++bt) {
            copies_wait(kSlBatches - 1 - bt);
            const int e = min(filled, (bt + 1) * batch);
            #pragma unroll 4
            for (int it = bt * batch; it < e; ++it) {
                float f[V];
                unpack<T, V>(slots[it * w.threads], f);
                v_add<V>(S, f, S);
            }
        }
        #pragma unroll
        for (int i = 0; i < V; ++i) { m.part.at(0, i, tid) = S[i]; S[i] = 0.f; }
        __syncthreads();
        for (int g0 = warp * at_once; g0 < w.groups; g0 += warps * at_once) {
            const int g = g0 + lane_g;
            float t = 0.f;
            if (g < w.groups) group_sums<V, 1>(w, m.part, g * sh.cg, sh.cg, rows, lane_i, &t);
            t = lanes_sum(t, w.lanes);
            if (lane_i == 0 && g < w.groups) m.res[g].x = t * per;
        }
        __syncthreads();
        // sums
        #pragma unroll
        for (int i = 0; i < V; ++i) nK[i] = -m.res[sh.group(min(V * v + i, w.Cs - 1))].x;
        #pragma unroll 4
        for (int it = 0; it < filled; ++it) {
            float f[V];
            unpack<T, V>(slots[it * w.threads], f);
            v_add<V>(f, nK, f);
            v_add<V>(S, f, S);
            v_fma<V>(f, f, Q, Q);
        }
        #pragma unroll
        for (int i = 0; i < V; ++i) { m.part.at(0, i, tid) = S[i]; m.part.at(1, i, tid) = Q[i]; }
        __syncthreads();
        for (int g0 = warp * at_once; g0 < w.groups; g0 += warps * at_once) {
            const int g = g0 + lane_g;
            float sq[2] = {0.f, 0.f};
            if (g < w.groups) group_sums<V, 2>(w, m.part, g * sh.cg, sh.cg, rows, lane_i, sq);
            const float s = lanes_sum(sq[0], w.lanes), q = lanes_sum(sq[1], w.lanes);
            if (lane_i == 0 && g < w.groups) {
                const float d = s * per, mu = m.res[g].x + d;
                const float var = fmaf(-s, d, q) * per;
                const float2 r = make_float2(mu, __frsqrt_rn((var < 0.f ? 0.f : var) + sh.eps));      // (keeps NaN)
                m.res[g] = r;
                mean[n * sh.groups + b.g0 + g] = r.x;
                rstd[n * sh.groups + b.g0 + g] = r.y;
            }
        }
        __syncthreads();

        // results, and the next sample's copies
        Chan<V> k = {};
        if (has) {
            load_parameters<V>(weight, V * cv, 1.f, k.a);
            load_parameters<V>(bias, V * cv, 0.f, k.b);
        }
        #pragma unroll
        for (int i = 0; i < V; ++i) {
            const float2 r = m.res[sh.group(min(V * v + i, w.Cs - 1))];
            k.nm[i] = -r.x;
            k.a[i] *= r.y;
        }
        const bool more = n + b.step < samples;
        const T* xn = x + (n + b.step) * gx.sn + V * cv;
        T* yp = y + n * gy.sn + V * cv;
        Cursor cy(gy, row), cx(gx, row);
        CodesCursor ckx(kx.codes, kx.scales, n * w.HW + row, cv, w.dense), cky(ky.codes, ky.scales, n * w.HW + row, cv, w.dense);
        #pragma unroll 1
        for (int bt = 0; bt < kSlBatches; ++bt) {
            const int e = min(cnt, (bt + 1) * batch);
            #pragma unroll 1
            for (int it = bt * batch; it < e; ++it) {
                const R r = has ? slots[it * w.threads] : R{};
                float f[V], z[V];
                unpack<T, V>(r, f);
                if constexpr (V == 8)
                    if (kx.codes) { keep_codes<T>(kx, r, f, has, ckx); ckx.next(w.dense); }
                v_add<V>(f, k.nm, f);
                v_fma<V>(f, k.a, k.b, z);
                activate<T, V, ACT>(sh.act, z);
                R out = pack<T, V>(z);
                if (has) *(R*)(yp + cy.off) = out;
                cy.next(gy);
                if constexpr (V == 8)
                    if (ky.codes) {                     // of y as it is stored
                        if (!has) out = R{};
                        unpack<T, 8>(out, f);
                        keep_codes<T>(ky, out, f, has, cky);
                        cky.next(w.dense);
                    }
                if (more && has) fill_slot(slots + it * w.threads, xn + cx.off);
                cx.next(gx);
            }
            copies_commit();
        }
    }
}

// The same for the backward pass: sums of dz and dz d per channel, c1 and c2 of the groups, then dx.  A block's sums for dweight and dbias are added up in
// shared memory and go to sum1 and sum2 every kSlSamples of its samples (so these running sums are short), to rows sum_pitch apart, first those of the
// blocks' first kSlSamples samples, block by block; a single row is the gradients.
constexpr int kSlSamples = 64;
inline long long slice_sums(long long samples, long long step) {      // rows that a launch with `step` blocks per slice writes
    const long long full = (samples - 1) / (kSlSamples * step);
    return full * step + (samples - full * kSlSamples * step < step ? samples - full * kSlSamples * step : step);
}
template <typename T, int V, int SRC, int ACT>
__global__ void __launch_bounds__(kSlThreads, 2) gn_slice_backward_kernel(const T* __restrict__ dy, const Geo gdy, const Source src, const Geo gx, const SliceWalk w, const NormShape sh,
                                                                          long long samples, const BackwardArgs A, T* __restrict__ dx, const Geo gdx, float* __restrict__ sum1,
                                                                          float* __restrict__ sum2, long long sum_pitch) {
    kn::pdl_sync();
    extern __shared__ __align__(16) uint8_t smem[];
    using R = Raw<T, V>;
    using X = typename Fetch<T, V, SRC>::R;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = w.threads >> 5;
    const size_t slab = (size_t)w.its * w.threads;
    R* slots = (R*)smem + tid;
    X* xslots = (X*)(smem + slab * sizeof(R)) + tid;
    uint8_t* eslots = smem + slab * (sizeof(R) + sizeof(X)) + tid;
    const SliceSmem<V> m(smem + slab * (sizeof(R) + sizeof(X) + (SRC == kSrcSame ? 0 : 1)), w);       // (slab is a multiple of 32)
    const SliceSpot b(w);
    const int row = tid / w.cols, v = tid - row * w.cols, cv = b.c0 / V + v;
    const bool has = row < w.rows && v < w.vecs;
    const int cnt = has && row < w.HW ? (w.HW - row + w.rows - 1) / w.rows : 0, batch = (w.its + kSlBatches - 1) / kSlBatches;
    if (b.n0 < samples) {
        Cursor cdy(gdy, row);
        SourceCursor<T, V, SRC> cx(src, gx, w, b.n0, row, cv);
        const T* dp = dy + b.n0 * gdy.sn + V * cv;
        #pragma unroll 1
        for (int bt = 0; bt < kSlBatches; ++bt) {
            const int e = min(cnt, (bt + 1) * batch);
            #pragma unroll 2
            for (int it = bt * batch; it < e; ++it) {
                fill_slot(slots + it * w.threads, dp + cdy.off);
                cdy.next(gdy);
                fill_slot(xslots + it * w.threads, cx.place());
                cx.next(gx, w);
            }
            copies_commit();
        }
        if constexpr (SRC != kSrcSame) {
            const uint8_t* ep = src.scales + (b.n0 * w.HW + row) * w.dense.blocks + V * cv / 32;
            #pragma unroll 8
            for (int it = 0; it < cnt; ++it, ep += w.dense.inc_scales) eslots[it * w.threads] = *ep;
        }
    }
    for (int c = tid; c < w.Cs; c += w.threads) {
        m.acc[c] = m.acc[w.Cs + c] = 0.f;
        m.weight[c] = A.weight ? A.weight[b.c0 + c] : 1.f;
    }
    #pragma unroll 1
    for (long long n = b.n0, out = b.n0; n < samples; out += b.step) {
        const long long end = min(samples, n + kSlSamples * b.step);
        #pragma unroll 1
        for (; n < end; n += b.step) {
            const long long gb = n * sh.groups + b.g0;              // this block's first group
            for (int g = tid; g < w.groups; g += w.threads) m.rstd[g] = A.rstd[gb + g];
            Chan<V> k;
            if (has) load_backward_chan<V, ACT>(k, sh, A, n, V * cv);
            // d and dz of the thread's position `it`
            auto values = [&](int it, float* f, float* q) {
                Fetch<T, V, SRC> fx;
                fx.r = xslots[it * w.threads];
                if constexpr (SRC != kSrcSame) fx.e = eslots[it * w.threads];
                unpack<T, V>(slots[it * w.threads], q);
                activation_gradient<T, V, SRC, ACT>(sh.act, k, fx, f, q);
            };
            float S1[V], S2[V];
            #pragma unroll
            for (int i = 0; i < V; ++i) S1[i] = S2[i] = 0.f;
            #pragma unroll 1
            for (int bt = 0; bt < kSlBatches; ++bt) {
                copies_wait(kSlBatches - 1 - bt);
                const int e = min(cnt, (bt + 1) * batch);
                #pragma unroll 1
                for (int it = bt * batch; it < e; ++it) {
                    float f[V], q[V];
                    values(it, f, q);
                    v_add<V>(S1, q, S1);
                    v_fma<V>(f, q, S2, S2);
                }
            }
            #pragma unroll
            for (int i = 0; i < V; ++i) { m.part.at(0, i, tid) = S1[i]; m.part.at(1, i, tid) = S2[i]; }
            __syncthreads();
            for (uint32_t c = tid; c < (uint32_t)w.Cs; c += w.threads) {
                const float* p = m.part.p + (c % V) * m.part.pitch + c / V;
                float2 t = make_float2(0.f, 0.f);
                #pragma unroll 8
                for (int r = 0; r < w.rows; ++r, p += w.cols) { t.x += p[0]; t.y += p[V * m.part.pitch]; }
                t.y *= m.rstd[sh.group(c)];                         // of xhat
                m.chan[c] = t.x;
                m.chan[w.Cs + c] = t.y;
                m.acc[c] += t.x;
                m.acc[w.Cs + c] += t.y;
            }
            __syncthreads();
            const float per = __frcp_rn((float)sh.HW * (float)sh.cg);
            for (int g0 = warp * (32 / w.lanes); g0 < w.groups; g0 += warps * (32 / w.lanes)) {
                const int g = g0 + lane / w.lanes;
                float2 t = make_float2(0.f, 0.f);
                if (g < w.groups)
                    #pragma unroll 2
                    for (int c = g * sh.cg + lane % w.lanes; c < (g + 1) * sh.cg; c += w.lanes) {
                        t.x = fmaf(m.weight[c], m.chan[c], t.x);
                        t.y = fmaf(m.weight[c], m.chan[w.Cs + c], t.y);
                    }
                t.x = lanes_sum(t.x, w.lanes);
                t.y = lanes_sum(t.y, w.lanes);
                if (g < w.groups && lane % w.lanes == 0) m.res[g] = make_float2(t.x * per, t.y * per);
            }
            __syncthreads();
            float B[V], D[V];
            if (has) {
                #pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int g = sh.group(V * v + i);
                    const float2 c = m.res[g];
                    const float r = m.rstd[g];
                    B[i] = -r * (r * c.y);
                    D[i] = -r * c.x;
                }
            }
            const bool more = n + b.step < samples;
            const long long n1 = n + b.step;
            const T* dn = dy + n1 * gdy.sn + V * cv;
            T* op = dx + n * gdx.sn + V * cv;
            Cursor c(gdx, row), cdy(gdy, row);
            SourceCursor<T, V, SRC> cx(src, gx, w, n1, row, cv);
            uint8_t e_next = 0;                                     // the exponent of the next sample's copies, stored a position after it was asked for
            #pragma unroll 1
            for (int bt = 0; bt < kSlBatches; ++bt) {
                const int e = min(cnt, (bt + 1) * batch);
                #pragma unroll 1
                for (int it = bt * batch; it < e; ++it) {
                    float f[V], q[V];
                    values(it, f, q);
                    if (SRC != kSrcSame && more) {
                        if (it > 0) eslots[(it - 1) * w.threads] = e_next;
                        e_next = *cx.scales;
                    }
                    v_fma<V>(f, B, D, f);
                    v_fma<V>(q, k.a, f, q);
                    *(R*)(op + c.off) = pack<T, V>(q);
                    c.next(gdx);
                    if (more) {
                        fill_slot(slots + it * w.threads, dn + cdy.off);
                        cdy.next(gdy);
                        fill_slot(xslots + it * w.threads, cx.place());
                        cx.next(gx, w);
                    }
                }
                copies_commit();
            }
            if (SRC != kSrcSame && more && cnt > 0) eslots[(cnt - 1) * w.threads] = e_next;
            __syncthreads();                                        // (the groups' rstd and results are free for the next sample)
        }
        for (int c = tid; c < w.Cs; c += w.threads) {               // (this thread's sums)
            if (sum1) sum1[out * sum_pitch + b.c0 + c] = m.acc[c];
            if (sum2) sum2[out * sum_pitch + b.c0 + c] = m.acc[w.Cs + c];
            m.acc[c] = m.acc[w.Cs + c] = 0.f;
        }
    }
}

}  // namespace op
