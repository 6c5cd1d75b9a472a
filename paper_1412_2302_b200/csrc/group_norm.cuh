// Group normalisation with an activation over channels-last tensors, forward and backward.
//
//   mean, var over the positions and the C / groups channels of a group of one sample;  rstd = 1 / sqrt(var + eps)
//   z = (x - mean) rstd w + b,  y = act(z)
//   dz = dy act'(z);  db = sum dz,  dw = sum dz xhat with xhat = (x - mean) rstd
//   dx = rstd (dz w - c1 - xhat c2),  c1 = mean(dz w), c2 = mean(dz w xhat) over the group
//
// Written with d = x - mean and a = rstd w as  z = d a + b  and  dx = dz a + (d (-rstd^2 c2) - rstd c1): two packed instructions per pair
// of channels each.  Both directions are HBM-bound: x in and y out; dy and x in and dx out.
//
// Sums.  A thread sums, for each of its channels, the differences from the first value it reads and their squares, in fp32.  That value
// is one of the summed, so the sum of squares is at most (1 + n) times the true one about the mean, however far the mean is from zero: nothing
// cancels as it would in E[x^2] - mean^2.  Between threads sums are joined in fp64 with a fixed order, so results repeat bit for bit.
#pragma once
#include "checkpoint.cuh"

namespace op {

enum { kActNone = 0, kActRelu = 1, kActSilu = 2 };

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
// numbers (relative error below 2^-20 for |z| < 16, next to a rounding of 2^-9 or 2^-12; below z = -87 the result is 0).
template <typename T, int V> __device__ __forceinline__ void sigmoid(const float* z, float* s) {
    if constexpr (sizeof(T) == 4) {
        #pragma unroll
        for (int i = 0; i < V; ++i) s[i] = __fdiv_rn(1.f, 1.f + expf(-z[i]));
    } else {
        const float l = -1.44269504f;
        float t[V], one[V], ls[V];
        #pragma unroll
        for (int i = 0; i < V; ++i) { one[i] = 1.f; ls[i] = l; }
        v_mul<V>(z, ls, t);
        #pragma unroll
        for (int i = 0; i < V; ++i) asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(t[i]));
        v_add<V>(t, one, t);
        #pragma unroll
        for (int i = 0; i < V; ++i) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s[i]) : "f"(t[i]));
    }
}
template <typename T, int V> __device__ __forceinline__ void activate(int act, float* z) {
    if (act == kActRelu) {
        #pragma unroll
        for (int i = 0; i < V; ++i) z[i] = z[i] < 0.f ? 0.f : z[i];          // keeps NaN
    } else if (act == kActSilu) {
        float s[V];
        sigmoid<T, V>(z, s);
        v_mul<V>(z, s, z);
    }
}

struct NormShape { int C, HW, groups, cg; float eps; int act; };

// per-channel constants of a thread's vector
template <int V> struct Chan { float nm[V], a[V], b[V]; };
template <int V>
__device__ __forceinline__ void load_chan(Chan<V>& k, const NormShape& s, const float* mean, const float* rstd, const float* weight, const float* bias, long long n, int c0) {
    #pragma unroll
    for (int i = 0; i < V; ++i) {
        const long long g = n * s.groups + (c0 + i) / s.cg;
        k.nm[i] = -mean[g];
        k.a[i] = rstd[g] * (weight ? weight[c0 + i] : 1.f);
        k.b[i] = bias ? bias[c0 + i] : 0.f;
    }
}

// ---------------------------------------------------------------- forward, any size: sums, statistics, result
// The sums of one thread for one channel, as sums of all values and of their squares (fp64: the squares' cancellation is harmless there
// up to |mean| / std of 10^6).
__device__ __forceinline__ double2 raw_moments(int n, float K, float S, float Q) {
    if (n == 0) return make_double2(0., 0.);
    const double s1 = (double)n * K + S, m2 = (double)Q - (double)S * S / n;
    return make_double2(s1, m2 + s1 * s1 / n);
}
template <typename T, int V>
__global__ void __launch_bounds__(256) gn_sums_kernel(const T* __restrict__ x, const Geo g, const Walk w, double2* __restrict__ partial) {
    kn::pdl_sync();
    __shared__ double2 sums[256 * V];
    const Spot s = spot(w);
    constexpr int U = V == 8 ? 4 : 8;
    float nK[V], S[V], Q[V];
    #pragma unroll
    for (int i = 0; i < V; ++i) nK[i] = S[i] = Q[i] = 0.f;
    int cnt = 0;
    if (s.has) {
        const T* xp = x + s.n * g.sn + V * s.v;
        for (int p = s.p0 + s.row; p < s.p1; p += U * w.rows) {
            Raw<T, V> r[U];
            #pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * w.rows < s.p1) r[u] = *(const Raw<T, V>*)(xp + g.at(p + u * w.rows));
            #pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * w.rows < s.p1) {
                    float f[V];
                    unpack<T, V>(r[u], f);
                    if (cnt == 0) {
                        #pragma unroll
                        for (int i = 0; i < V; ++i) nK[i] = -f[i];
                    }
                    v_add<V>(f, nK, f);
                    v_add<V>(S, f, S);
                    v_fma<V>(f, f, Q, Q);
                    ++cnt;
                }
        }
    }
    #pragma unroll
    for (int i = 0; i < V; ++i) sums[threadIdx.x * V + i] = raw_moments(cnt, -nK[i], S[i], Q[i]);
    __syncthreads();
    const int nch = w.cols * V, c0 = (s.v - s.col) * V;
    for (int j = threadIdx.x; j < nch; j += 256) {
        if (c0 + j >= w.C) break;
        double2 t = make_double2(0., 0.);
        for (int r = 0; r < w.rows; ++r) { const double2 q = sums[r * nch + j]; t.x += q.x; t.y += q.y; }
        partial[(s.n * w.chunks + s.chunk) * w.C + c0 + j] = t;
    }
}
// a block per group
__global__ void __launch_bounds__(128) gn_statistics_kernel(const double2* __restrict__ partial, const NormShape s, long long chunks, float* __restrict__ mean, float* __restrict__ rstd) {
    kn::pdl_sync();
    const long long n = blockIdx.x / s.groups;
    const int g = (int)(blockIdx.x - n * s.groups);
    const double2* p = partial + n * chunks * s.C + (long long)g * s.cg;
    double2 t = make_double2(0., 0.);
    const long long total = chunks * s.cg;
    for (long long i = threadIdx.x; i < total; i += 128) {
        const long long k = i / s.cg;
        const double2 q = p[k * s.C + (i - k * s.cg)];
        t.x += q.x; t.y += q.y;
    }
    #pragma unroll
    for (int o = 16; o; o >>= 1) { t.x += __shfl_xor_sync(~0u, t.x, o); t.y += __shfl_xor_sync(~0u, t.y, o); }
    __shared__ double2 ws[4];
    if ((threadIdx.x & 31) == 0) ws[threadIdx.x >> 5] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        t = make_double2(ws[0].x + ws[1].x + ws[2].x + ws[3].x, ws[0].y + ws[1].y + ws[2].y + ws[3].y);
        const double m = (double)s.HW * s.cg, mu = t.x / m;
        double var = t.y / m - mu * mu;
        if (var < 0.) var = 0.;
        mean[blockIdx.x] = (float)mu;
        rstd[blockIdx.x] = (float)(1. / sqrt(var + (double)s.eps));
    }
}
struct Keep { uint8_t *codes, *scales; int fmt; };        // codes == nullptr: nothing kept
template <typename T>
__device__ __forceinline__ void keep_codes(const Keep& k, const Raw<T, 8>& r, const float* f, bool has, CodesCursor& c) {
    if (k.fmt == kSrcInt8) store_codes<T, kSrcInt8>(r, f, has, c.codes, c.scales);
    else store_codes<T, kSrcE4m3>(r, f, has, c.codes, c.scales);
}
// A thread's positions from p on, `rows` apart, `cnt` of them: results (and checkpoints) of the vectors that fetch(it) gives.
template <typename T, int V, typename F>
__device__ __forceinline__ void apply_positions(const Chan<V>& k, const NormShape& sh, int p, int rows, int it0, int cnt, long long row0, int v, bool has, T* y, const Geo& gy, const Keep& kx, const Keep& ky,
                                                F fetch) {
    Cursor c(gy, p + it0 * rows);
    CodesCursor cx(kx.codes, kx.scales, row0 + p + it0 * rows, v, sh.C), cy(ky.codes, ky.scales, row0 + p + it0 * rows, v, sh.C);
    #pragma unroll 2
    for (int it = it0; it < cnt; ++it) {
        const Raw<T, V> r = fetch(it);
        float f[V], z[V];
        unpack<T, V>(r, f);
        if constexpr (V == 8)
            if (kx.codes) { keep_codes<T>(kx, r, f, has, cx); cx.next(rows, sh.C); }
        v_add<V>(f, k.nm, f);
        v_fma<V>(f, k.a, k.b, z);
        activate<T, V>(sh.act, z);
        Raw<T, V> out = pack<T, V>(z);
        if (has) *(Raw<T, V>*)(y + c.off) = out;
        c.next(gy, rows);
        if constexpr (V == 8)
            if (ky.codes) {                     // of y as it is stored
                if (!has) out = Raw<T, 8>{};
                unpack<T, 8>(out, f);
                keep_codes<T>(ky, out, f, has, cy);
                cy.next(rows, sh.C);
            }
    }
}
template <typename T, int V>
__global__ void __launch_bounds__(256) gn_apply_kernel(const T* __restrict__ x, const Geo gx, const Walk w, const NormShape sh, const float* __restrict__ weight,
                                                       const float* __restrict__ bias, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                       T* __restrict__ y, const Geo gy, const Keep kx, const Keep ky) {
    kn::pdl_sync();
    const Spot s = spot(w);
    const int p = s.p0 + s.row;
    if (!s.on || p >= s.p1) return;
    Chan<V> k = {};
    if (s.has) load_chan<V>(k, sh, mean, rstd, weight, bias, s.n, V * s.v);
    const T* xp = x + s.n * gx.sn + V * s.v;
    Cursor c(gx, p);
    apply_positions<T, V>(k, sh, p, w.rows, 0, (s.p1 - p + w.rows - 1) / w.rows, s.n * w.HW, s.v, s.has, y + s.n * gy.sn + V * s.v, gy, kx, ky, [&](int) {
        Raw<T, V> r = {};
        if (s.has) r = *(const Raw<T, V>*)(xp + c.off);
        c.next(gx, w.rows);
        return r;
    });
}

// ---------------------------------------------------------------- backward
// where a backward pass reads x: a tensor, or the codes and exponents of a checkpoint (dense)
struct Source { const void* x; const uint8_t *codes, *scales; };
template <typename T, int V, int SRC> struct Fetch {
    using R = typename std::conditional<SRC == kSrcSame, Raw<T, V>, Raw<uint8_t, V>>::type;
    R r;
    uint8_t e;
    __device__ __forceinline__ void load(const Source& s, const Geo& g, const Walk& w, long long n, int p, int v) {
        if constexpr (SRC == kSrcSame) r = *(const R*)((const T*)s.x + n * g.sn + g.at(p) + V * v);
        else {
            const long long row = n * w.HW + p;
            r = *(const R*)(s.codes + row * w.C + V * v);
            e = s.scales[row * ((w.C + 31) / 32) + V * v / 32];
        }
    }
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
// The side of ReLU's kink that a value is on, where fp32 cannot tell: d and a carry a rounding each, so z = d a + b is off by up to
// 2^-23 |b| or so when it is near zero.  Such values (a few in a million) are taken again in fp64 from x itself.
struct BackwardArgs {
    const float *mean, *rstd, *weight, *bias;
};
// d = x - mean, and dz in the place of dy
template <typename T, int V, int SRC>
__device__ __forceinline__ void activation_gradient(const NormShape& sh, const Chan<V>& k, const BackwardArgs& A, long long n, int c0, const Fetch<T, V, SRC>& fx, float* d, float* dy) {
    float x[V];
    fx.value(k.nm, x, d);
    if (sh.act == kActNone) return;
    float z[V];
    v_fma<V>(d, k.a, k.b, z);
    if (sh.act == kActRelu) {
        bool near = false;
        #pragma unroll
        for (int i = 0; i < V; ++i) near = near || fabsf(z[i]) < fabsf(1e-6f * k.b[i]);
        if (near) {
            #pragma unroll
            for (int i = 0; i < V; ++i) {
                const double side = ((double)(x[i] * fx.scale()) + (double)k.nm[i]) * (double)A.rstd[n * sh.groups + (c0 + i) / sh.cg] * (A.weight ? (double)A.weight[c0 + i] : 1.) + (double)k.b[i];
                if (fabsf(z[i]) < fabsf(1e-6f * k.b[i])) z[i] = side > 0. ? 1.f : -1.f;
            }
        }
        #pragma unroll
        for (int i = 0; i < V; ++i) dy[i] = z[i] <= 0.f ? 0.f : dy[i];
    } else {
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
template <typename T, int V, int SRC>
__global__ void __launch_bounds__(256) gn_backward_sums_kernel(const T* __restrict__ dy, const Geo gdy, const Source src, const Geo gx, const Walk w, const NormShape sh,
                                                               const BackwardArgs A, float* __restrict__ partial) {
    kn::pdl_sync();
    __shared__ float sums[2][256 * V];
    const Spot s = spot(w);
    constexpr int U = V == 8 ? 2 : 4;
    float S1[V], S2[V];
    #pragma unroll
    for (int i = 0; i < V; ++i) S1[i] = S2[i] = 0.f;
    if (s.has) {
        Chan<V> k;
        load_chan<V>(k, sh, A.mean, A.rstd, A.weight, A.bias, s.n, V * s.v);
        const T* dp = dy + s.n * gdy.sn + V * s.v;
        for (int p = s.p0 + s.row; p < s.p1; p += U * w.rows) {
            Raw<T, V> r[U];
            Fetch<T, V, SRC> fx[U];
            #pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * w.rows < s.p1) {
                    r[u] = *(const Raw<T, V>*)(dp + gdy.at(p + u * w.rows));
                    fx[u].load(src, gx, w, s.n, p + u * w.rows, s.v);
                }
            #pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * w.rows < s.p1) {
                    float f[V], q[V];
                    unpack<T, V>(r[u], q);
                    activation_gradient<T, V, SRC>(sh, k, A, s.n, V * s.v, fx[u], f, q);
                    v_add<V>(S1, q, S1);
                    v_fma<V>(f, q, S2, S2);
                }
        }
    }
    #pragma unroll
    for (int i = 0; i < V; ++i) { sums[0][threadIdx.x * V + i] = S1[i]; sums[1][threadIdx.x * V + i] = S2[i]; }
    __syncthreads();
    const int nch = w.cols * V, c0 = (s.v - s.col) * V;
    for (int j = threadIdx.x; j < nch; j += 256) {
        if (c0 + j >= w.C) break;
        float t1 = 0.f, t2 = 0.f;
        for (int r = 0; r < w.rows; ++r) { t1 += sums[0][r * nch + j]; t2 += sums[1][r * nch + j]; }
        float* o = partial + (s.n * w.chunks + s.chunk) * 2 * w.C + c0 + j;
        o[0] = t1;
        o[w.C] = t2 * A.rstd[s.n * sh.groups + (c0 + j) / sh.cg];       // of xhat
    }
}
// Blocks below n * groups: c1 and c2 of a group.  The others: dweight and dbias of 32 channels, over samples and chunks.
__global__ void __launch_bounds__(256) gn_backward_final_kernel(const float* __restrict__ partial, const NormShape sh, long long n_total, long long chunks, const BackwardArgs A,
                                                                float2* __restrict__ c12, float* __restrict__ dweight, float* __restrict__ dbias) {
    kn::pdl_sync();
    __shared__ double2 red[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long nblk = n_total * sh.groups;
    double2 t = make_double2(0., 0.);
    if (blockIdx.x < nblk) {
        const long long n = blockIdx.x / sh.groups;
        const int g = (int)(blockIdx.x - n * sh.groups);
        const float* p = partial + n * chunks * 2 * sh.C + (long long)g * sh.cg;
        for (long long i = threadIdx.x; i < chunks * sh.cg; i += 256) {
            const long long k = i / sh.cg;
            const int c = (int)(i - k * sh.cg);
            const double wt = A.weight ? A.weight[g * sh.cg + c] : 1.f;
            t.x += wt * p[k * 2 * sh.C + c];
            t.y += wt * p[k * 2 * sh.C + sh.C + c];
        }
        #pragma unroll
        for (int o = 16; o; o >>= 1) { t.x += __shfl_xor_sync(~0u, t.x, o); t.y += __shfl_xor_sync(~0u, t.y, o); }
        if (lane == 0) red[warp][0] = t;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int k = 1; k < 8; ++k) { t.x += red[k][0].x; t.y += red[k][0].y; }
            const double m = (double)sh.HW * sh.cg;
            c12[blockIdx.x] = make_float2((float)(t.x / m), (float)(t.y / m));
        }
        return;
    }
    const int c = (int)(blockIdx.x - nblk) * 32 + lane;
    if (c < sh.C)
        for (long long i = warp; i < n_total * chunks; i += 8) { t.x += partial[i * 2 * sh.C + c]; t.y += partial[i * 2 * sh.C + sh.C + c]; }
    red[warp][lane] = t;
    __syncthreads();
    if (warp == 0 && c < sh.C) {
        for (int k = 1; k < 8; ++k) { t.x += red[k][lane].x; t.y += red[k][lane].y; }
        if (dbias) dbias[c] = (float)t.x;
        if (dweight) dweight[c] = (float)t.y;
    }
}
template <typename T, int V, int SRC>
__global__ void __launch_bounds__(256) gn_backward_apply_kernel(const T* __restrict__ dy, const Geo gdy, const Source src, const Geo gx, const Walk w, const NormShape sh,
                                                                const BackwardArgs A, const float2* __restrict__ c12, T* __restrict__ dx, const Geo gdx) {
    kn::pdl_sync();
    const Spot s = spot(w);
    if (!s.has) return;
    Chan<V> k;
    load_chan<V>(k, sh, A.mean, A.rstd, A.weight, A.bias, s.n, V * s.v);
    float B[V], D[V];
    #pragma unroll
    for (int i = 0; i < V; ++i) {
        const long long g = s.n * sh.groups + (V * s.v + i) / sh.cg;
        const float2 c = c12[g];
        const float r = A.rstd[g];
        B[i] = -r * r * c.y;
        D[i] = -r * c.x;
    }
    const T* dp = dy + s.n * gdy.sn + V * s.v;
    T* op = dx + s.n * gdx.sn + V * s.v;
    constexpr int U = V == 8 ? 2 : 4;
    for (int p = s.p0 + s.row; p < s.p1; p += U * w.rows) {
        Raw<T, V> r[U];
        Fetch<T, V, SRC> fx[U];
        #pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u * w.rows < s.p1) {
                r[u] = *(const Raw<T, V>*)(dp + gdy.at(p + u * w.rows));
                fx[u].load(src, gx, w, s.n, p + u * w.rows, s.v);
            }
        #pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u * w.rows < s.p1) {
                float f[V], q[V];
                unpack<T, V>(r[u], q);
                activation_gradient<T, V, SRC>(sh, k, A, s.n, V * s.v, fx[u], f, q);
                v_fma<V>(f, B, D, f);
                v_fma<V>(q, k.a, f, q);
                *(Raw<T, V>*)(op + gdx.at(p + u * w.rows)) = pack<T, V>(q);
            }
    }
}


// ---------------------------------------------------------------- one launch per direction: a sample per cluster
//
// The CTAs of a cluster share the positions of one sample.  A thread keeps the vectors it has read (raw, in its own slots of shared memory, filled by
// asynchronous copies) while the sums go around the cluster through distributed shared memory, then turns them into the result:
// every value is read from memory once.  Slots are private to a thread, so no barrier stands between its copies and its reads.
// Iterations beyond `keep` (samples too large for the cluster's shared memory) are read again, from L2.
struct ClusterWalk {
    int C, HW, vecs, cols, rows, threads;     // rows = threads / cols
    int k, ppc, its, keep;                    // CTAs of the cluster; positions of a CTA, at most; iterations of a thread, and those whose vectors stay
};
constexpr int kClThreads = 384;               // at most; two CTAs per SM with 80 registers

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
constexpr int kClBatches = 4;                 // groups of copies

__device__ __forceinline__ double2 ld_cluster_d2(uint32_t addr, uint32_t rank) {
    double2 v;
    asm volatile("ld.shared::cluster.v2.f64 {%0, %1}, [%2];" : "=d"(v.x), "=d"(v.y) : "r"(tc::mapa_u32(addr, rank)) : "memory");
    return v;
}
__device__ __forceinline__ double2 warp_sum(double2 t) {
    #pragma unroll
    for (int o = 16; o; o >>= 1) { t.x += __shfl_xor_sync(~0u, t.x, o); t.y += __shfl_xor_sync(~0u, t.y, o); }
    return t;
}
// shared memory behind the slots: per-thread sums, per-channel sums, per-group sums of this CTA, per-group results
struct ClusterSmem { float2* part; double2 *chan, *grp; float2* res; };
template <int V> __device__ __forceinline__ ClusterSmem cluster_smem(uint8_t* p, const ClusterWalk& w, int groups) {
    ClusterSmem s;
    s.chan = (double2*)p;
    s.grp = s.chan + w.C;
    s.part = (float2*)(s.grp + groups);
    s.res = s.part + w.threads * V;
    return s;
}
template <int V> inline size_t cluster_scratch(const ClusterWalk& w, int groups) { return (size_t)(w.C + groups) * 16 + ((size_t)w.threads * V + groups) * 8; }

template <typename T, int V>
__global__ void __launch_bounds__(kClThreads, 2) gn_cluster_forward_kernel(const T* __restrict__ x, const Geo gx, const ClusterWalk w, const NormShape sh, const float* __restrict__ weight,
                                                                           const float* __restrict__ bias, T* __restrict__ y, const Geo gy, float* __restrict__ mean,
                                                                           float* __restrict__ rstd, const Keep kx, const Keep ky) {
    kn::pdl_sync();
    extern __shared__ __align__(16) uint8_t smem[];
    using R = Raw<T, V>;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = w.threads >> 5;
    R* slots = (R*)smem + tid;
    const ClusterSmem m = cluster_smem<V>(smem + (size_t)w.keep * w.threads * sizeof(R), w, sh.groups);
    const int rank = w.k > 1 ? (int)tc::cluster_ctarank() : 0;
    const long long n = blockIdx.x / w.k;
    const int row = tid / w.cols, v = tid - row * w.cols;
    const bool on = row < w.rows, has = on && v < w.vecs;
    const int p0 = rank * w.ppc, np = max(0, min(w.HW - p0, w.ppc));
    const int cnt = on && row < np ? (np - row + w.rows - 1) / w.rows : 0;      // iterations of this thread
    const T* xp = x + n * gx.sn + V * v;

    // sums
    float nK[V], S[V], Q[V];
    #pragma unroll
    for (int i = 0; i < V; ++i) nK[i] = S[i] = Q[i] = 0.f;
    const int kept = has ? min(cnt, w.keep) : 0, batch = (w.keep + kClBatches - 1) / kClBatches;
    Cursor cur(gx, p0 + row);
    #pragma unroll 1
    for (int b = 0; b < kClBatches; ++b) {
        const int e = min(kept, (b + 1) * batch);
        #pragma unroll 4
        for (int it = b * batch; it < e; ++it) {
            fill_slot(slots + it * w.threads, xp + cur.off);
            cur.next(gx, w.rows);
        }
        copies_commit();
    }
    auto shift = [&](const R& r) {             // the first value
        unpack<T, V>(r, nK);
        #pragma unroll
        for (int i = 0; i < V; ++i) nK[i] = -nK[i];
    };
    auto add = [&](const R& r) {
        float f[V];
        unpack<T, V>(r, f);
        v_add<V>(f, nK, f);
        v_add<V>(S, f, S);
        v_fma<V>(f, f, Q, Q);
    };
    #pragma unroll 1
    for (int b = 0; b < kClBatches; ++b) {
        copies_wait(kClBatches - 1 - b);
        const int e = min(kept, (b + 1) * batch);
        if (b == 0 && kept > 0) shift(slots[0]);
        #pragma unroll 2
        for (int it = b * batch; it < e; ++it) add(slots[it * w.threads]);
    }
    if (has) {
        if (kept == 0 && cnt > 0) shift(*(const R*)(xp + cur.off));
        constexpr int U = 4;
        for (int it = kept; it < cnt; it += U) {
            R r[U];
            #pragma unroll
            for (int u = 0; u < U; ++u) {
                if (it + u < cnt) r[u] = *(const R*)(xp + cur.off);
                cur.next(gx, w.rows);
            }
            #pragma unroll
            for (int u = 0; u < U; ++u)
                if (it + u < cnt) add(r[u]);
        }
    }
    {
        const float nf = (float)cnt, inv = cnt ? __fdividef(1.f, nf) : 0.f;
        #pragma unroll
        for (int i = 0; i < V; ++i) {         // the mean of this thread's values and their squared deviations from it
            const float d = S[i] * inv;
            m.part[tid * V + i] = make_float2(d - nK[i], fmaf(-S[i], d, Q[i]));
        }
    }
    __syncthreads();
    const int more = np % w.rows;
    const double n_lo = (double)(np / w.rows);
    for (int c = tid; c < w.C; c += w.threads) {
        double2 t = make_double2(0., 0.);
        for (int r = 0; r < w.rows; ++r) {          // the first `more` rows of threads have one position more than the others
            const float2 q = m.part[r * w.cols * V + c];
            const double nr = r < more ? n_lo + 1. : n_lo, mu = q.x;
            t.x += nr * mu;
            t.y += (double)q.y + nr * mu * mu;
        }
        m.chan[c] = t;
    }
    __syncthreads();
    for (int g = warp; g < sh.groups; g += warps) {
        double2 t = make_double2(0., 0.);
        for (int c = lane; c < sh.cg; c += 32) { const double2 q = m.chan[g * sh.cg + c]; t.x += q.x; t.y += q.y; }
        t = warp_sum(t);
        if (lane == 0) m.grp[g] = t;
    }
    __syncwarp();
    if (w.k > 1) tc::cluster_sync_all();
    else __syncthreads();
    for (int g = warp; g < sh.groups; g += warps) {
        double2 t = make_double2(0., 0.);
        if (w.k == 1) t = m.grp[g];
        else {
            if (lane < w.k) t = ld_cluster_d2(tc::smem_u32(m.grp + g), lane);
            t = warp_sum(t);
        }
        const double count = (double)sh.HW * sh.cg, mu = t.x / count;
        double var = t.y / count - mu * mu;
        if (var < 0.) var = 0.;
        const float2 r = make_float2((float)mu, (float)(1. / sqrt(var + (double)sh.eps)));
        if (lane == 0) {
            m.res[g] = r;
            if (rank == 0) { mean[n * sh.groups + g] = r.x; rstd[n * sh.groups + g] = r.y; }
        }
    }
    if (w.k > 1) { __syncwarp(); tc::cluster_arrive(); }        // this CTA has read the others' sums
    __syncthreads();

    // result
    if (cnt > 0) {
        Chan<V> k;
        #pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = min(V * v + i, w.C - 1);
            const float2 r = m.res[c / sh.cg];
            k.nm[i] = -r.x;
            k.a[i] = r.y * (weight ? weight[c] : 1.f);
            k.b[i] = bias ? bias[c] : 0.f;
        }
        T* yp = y + n * gy.sn + V * v;
        const int split = min(cnt, w.keep);
        apply_positions<T, V>(k, sh, p0 + row, w.rows, 0, split, n * w.HW, v, has, yp, gy, kx, ky, [&](int it) { return has ? slots[it * w.threads] : R{}; });
        if (split < cnt) {
            Cursor c(gx, p0 + row + split * w.rows);
            apply_positions<T, V>(k, sh, p0 + row, w.rows, split, cnt, n * w.HW, v, has, yp, gy, kx, ky, [&](int) {
                R r = {};
                if (has) r = *(const R*)(xp + c.off);
                c.next(gx, w.rows);
                return r;
            });
        }
    }
    if (w.k > 1) { __syncwarp(); tc::cluster_wait(); }          // no CTA leaves while another may read its sums
}

// The same for the backward pass: sums of dz and dz d per channel, around the cluster for c1 and c2, then dx.  The samples' sums for dweight and
// dbias go to partial [n][2][C] (a CTA joins the channels rank, rank + k, ... of its cluster) and are added over the samples by a second launch.
template <typename T, int V, int SRC>
__global__ void __launch_bounds__(kClThreads, 2) gn_cluster_backward_kernel(const T* __restrict__ dy, const Geo gdy, const Source src, const Geo gx, const ClusterWalk w, const NormShape sh,
                                                                            const BackwardArgs A, T* __restrict__ dx, const Geo gdx, float* __restrict__ partial) {
    kn::pdl_sync();
    extern __shared__ __align__(16) uint8_t smem[];
    using R = Raw<T, V>;
    using X = typename Fetch<T, V, SRC>::R;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = w.threads >> 5;
    const size_t slab = (size_t)w.keep * w.threads;
    R* slots = (R*)smem + tid;
    X* xslots = (X*)(smem + slab * sizeof(R)) + tid;
    uint8_t* eslots = smem + slab * (sizeof(R) + sizeof(X)) + tid;
    const ClusterSmem m = cluster_smem<V>(smem + slab * (sizeof(R) + sizeof(X)) + (SRC == kSrcSame ? 0 : (slab + 15) / 16 * 16), w, sh.groups);
    const int rank = w.k > 1 ? (int)tc::cluster_ctarank() : 0;
    const long long n = blockIdx.x / w.k;
    const int row = tid / w.cols, v = tid - row * w.cols;
    const bool has = row < w.rows && v < w.vecs;
    const int p0 = rank * w.ppc, np = max(0, min(w.HW - p0, w.ppc));
    const int cnt = has && row < np ? (np - row + w.rows - 1) / w.rows : 0;
    const T* dp = dy + n * gdy.sn + V * v;
    const int blocks = (w.C + 31) / 32, kept = min(cnt, w.keep), batch = (w.keep + kClBatches - 1) / kClBatches;
    const T* xp = SRC == kSrcSame ? (const T*)src.x + n * gx.sn + V * v : nullptr;
    const uint8_t* cp = SRC == kSrcSame ? nullptr : src.codes + (n * w.HW + p0 + row) * w.C + V * v;
    Cursor cdy(gdy, p0 + row), cx(gx, p0 + row);
    #pragma unroll 1
    for (int b = 0; b < kClBatches; ++b) {
        const int e = min(kept, (b + 1) * batch);
        #pragma unroll 2
        for (int it = b * batch; it < e; ++it) {
            fill_slot(slots + it * w.threads, dp + cdy.off);
            cdy.next(gdy, w.rows);
            if constexpr (SRC == kSrcSame) {
                fill_slot(xslots + it * w.threads, xp + cx.off);
                cx.next(gx, w.rows);
            } else {
                fill_slot(xslots + it * w.threads, cp);
                cp += (long long)w.rows * w.C;
            }
        }
        copies_commit();
    }
    if constexpr (SRC != kSrcSame) {
        const uint8_t* ep = src.scales + (n * w.HW + p0 + row) * blocks + V * v / 32;
        #pragma unroll 8
        for (int it = 0; it < kept; ++it) eslots[it * w.threads] = ep[(long long)it * w.rows * blocks];
    }
    Chan<V> k;
    if (has) load_chan<V>(k, sh, A.mean, A.rstd, A.weight, A.bias, n, V * v);
    float S1[V], S2[V];
    #pragma unroll
    for (int i = 0; i < V; ++i) S1[i] = S2[i] = 0.f;
    // d and dz of iteration it
    auto values = [&](int it, float* f, float* q) {
        Fetch<T, V, SRC> fx;
        R r;
        if (it < kept) {
            r = slots[it * w.threads];
            fx.r = xslots[it * w.threads];
            if constexpr (SRC != kSrcSame) fx.e = eslots[it * w.threads];
        } else {
            const int p = p0 + row + it * w.rows;
            r = *(const R*)(dp + gdy.at(p));
            fx.load(src, gx, Walk{w.C, w.HW}, n, p, v);
        }
        unpack<T, V>(r, q);
        activation_gradient<T, V, SRC>(sh, k, A, n, V * v, fx, f, q);
    };
    auto add = [&](int it) {
        float f[V], q[V];
        values(it, f, q);
        v_add<V>(S1, q, S1);
        v_fma<V>(f, q, S2, S2);
    };
    #pragma unroll 1
    for (int b = 0; b < kClBatches; ++b) {
        copies_wait(kClBatches - 1 - b);
        const int e = min(kept, (b + 1) * batch);
        #pragma unroll 1
        for (int it = b * batch; it < e; ++it) add(it);
    }
    #pragma unroll 2
    for (int it = kept; it < cnt; ++it) add(it);
    #pragma unroll
    for (int i = 0; i < V; ++i) m.part[tid * V + i] = make_float2(S1[i], S2[i]);
    __syncthreads();
    for (int c = tid; c < w.C; c += w.threads) {
        double2 t = make_double2(0., 0.);
        for (int r = 0; r < w.rows; ++r) { const float2 q = m.part[r * w.cols * V + c]; t.x += q.x; t.y += q.y; }
        t.y *= A.rstd[n * sh.groups + c / sh.cg];              // of xhat
        m.chan[c] = t;
    }
    __syncthreads();
    for (int g = warp; g < sh.groups; g += warps) {
        double2 t = make_double2(0., 0.);
        for (int c = lane; c < sh.cg; c += 32) {
            const double2 q = m.chan[g * sh.cg + c];
            const double wt = A.weight ? A.weight[g * sh.cg + c] : 1.f;
            t.x += wt * q.x;
            t.y += wt * q.y;
        }
        t = warp_sum(t);
        if (lane == 0) m.grp[g] = t;
    }
    __syncwarp();
    if (w.k > 1) tc::cluster_sync_all();
    else __syncthreads();
    for (int g = warp; g < sh.groups; g += warps) {
        double2 t = make_double2(0., 0.);
        if (w.k == 1) t = m.grp[g];
        else {
            if (lane < w.k) t = ld_cluster_d2(tc::smem_u32(m.grp + g), lane);
            t = warp_sum(t);
        }
        const double count = (double)sh.HW * sh.cg;
        if (lane == 0) m.res[g] = make_float2((float)(t.x / count), (float)(t.y / count));
    }
    for (int c = rank + w.k * tid; c < w.C; c += w.k * w.threads) {
        double2 t = m.chan[c];
        if (w.k > 1) {
            t = make_double2(0., 0.);
            for (int r = 0; r < w.k; ++r) { const double2 q = ld_cluster_d2(tc::smem_u32(m.chan + c), r); t.x += q.x; t.y += q.y; }
        }
        partial[n * 2 * w.C + c] = (float)t.x;
        partial[n * 2 * w.C + w.C + c] = (float)t.y;
    }
    if (w.k > 1) { __syncwarp(); tc::cluster_arrive(); }
    __syncthreads();
    if (has) {
        float B[V], D[V];
        #pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = (V * v + i) / sh.cg;
            const float2 c = m.res[g];
            const float r = A.rstd[n * sh.groups + g];
            B[i] = -r * r * c.y;
            D[i] = -r * c.x;
        }
        T* op = dx + n * gdx.sn + V * v;
        Cursor c(gdx, p0 + row);
        #pragma unroll 1
        for (int it = 0; it < cnt; ++it) {
            float f[V], q[V];
            values(it, f, q);
            v_fma<V>(f, B, D, f);
            v_fma<V>(q, k.a, f, q);
            *(R*)(op + c.off) = pack<T, V>(q);
            c.next(gdx, w.rows);
        }
    }
    if (w.k > 1) { __syncwarp(); tc::cluster_wait(); }
}
// dweight and dbias: the samples' sums, added in fp64.  A block takes 32 channels, its warps every 32nd sample.
__global__ void __launch_bounds__(1024) gn_parameter_gradient_kernel(const float* __restrict__ partial, int C, long long n, float* __restrict__ dweight, float* __restrict__ dbias) {
    kn::pdl_sync();
    __shared__ double2 red[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    double2 t = make_double2(0., 0.);
    if (c < C) {
        const float* p = partial + c;
        #pragma unroll 8
        for (long long i = warp; i < n; i += 32) { t.x += p[i * 2 * C]; t.y += p[i * 2 * C + C]; }
    }
    red[warp][lane] = t;
    __syncthreads();
    t = red[lane][warp];               // lane: part, warp: channel
    t = warp_sum(t);
    const int cw = blockIdx.x * 32 + warp;
    if (lane == 0 && cw < C) {
        if (dbias) dbias[cw] = (float)t.x;
        if (dweight) dweight[cw] = (float)t.y;
    }
}

}  // namespace op
