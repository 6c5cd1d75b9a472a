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
template <int V> __device__ __forceinline__ void v_fma(const float* a, const float* b, const float* c, float* o) {
    if constexpr (V == 1) o[0] = fmaf(a[0], b[0], c[0]);
    else {
        #pragma unroll
        for (int i = 0; i < V; i += 2) un2(fma2(mk2(a[i], a[i + 1]), mk2(b[i], b[i + 1]), mk2(c[i], c[i + 1])), o[i], o[i + 1]);
    }
}
// 1 / (1 + e^-z).  fp32 tensors take the accurate functions; for 16-bit ones the hardware's approximate ones (relative error below 2^-20 for
// |z| < 16, next to a rounding of 2^-9 or 2^-12)
template <typename T> __device__ __forceinline__ float sigmoid(float z) {
    if constexpr (sizeof(T) == 4) return __fdiv_rn(1.f, 1.f + expf(-z));
    else return __fdividef(1.f, 1.f + __expf(-z));
}
template <typename T, int V> __device__ __forceinline__ void activate(int act, float* z) {
    if (act == kActRelu) {
        #pragma unroll
        for (int i = 0; i < V; ++i) z[i] = z[i] < 0.f ? 0.f : z[i];          // keeps NaN
    } else if (act == kActSilu) {
        #pragma unroll
        for (int i = 0; i < V; ++i) z[i] *= sigmoid<T>(z[i]);
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
template <typename T, int V>
__global__ void __launch_bounds__(256) gn_apply_kernel(const T* __restrict__ x, const Geo gx, const Walk w, const NormShape sh, const float* __restrict__ weight,
                                                       const float* __restrict__ bias, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                       T* __restrict__ y, const Geo gy, const Keep kx, const Keep ky) {
    kn::pdl_sync();
    const Spot s = spot(w);
    if (!s.on) return;
    Chan<V> k;
    if (s.has) load_chan<V>(k, sh, mean, rstd, weight, bias, s.n, V * s.v);
    const T* xp = x + s.n * gx.sn + V * s.v;
    T* yp = y + s.n * gy.sn + V * s.v;
    const int blocks = (w.C + 31) / 32;
    constexpr int U = V == 8 ? 2 : 8;
    for (int p = s.p0 + s.row; p < s.p1; p += U * w.rows) {
        Raw<T, V> r[U];
        #pragma unroll
        for (int u = 0; u < U; ++u)
            if (s.has && p + u * w.rows < s.p1) r[u] = *(const Raw<T, V>*)(xp + gx.at(p + u * w.rows));
        #pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u * w.rows < s.p1) {
                const int q = p + u * w.rows;
                float f[V], z[V];
                if (s.has) unpack<T, V>(r[u], f);
                if constexpr (V == 8)
                    if (kx.codes) {
                        float t[8];
                        #pragma unroll
                        for (int i = 0; i < 8; ++i) t[i] = s.has ? f[i] : 0.f;
                        store_codes(kx.fmt, t, s.has, kx.codes, kx.scales, s.n * w.HW + q, s.v, w.C, blocks);
                    }
                Raw<T, V> out;
                if (s.has) {
                    v_add<V>(f, k.nm, f);
                    v_fma<V>(f, k.a, k.b, z);
                    activate<T, V>(sh.act, z);
                    out = pack<T, V>(z);
                    *(Raw<T, V>*)(yp + gy.at(q)) = out;
                }
                if constexpr (V == 8)
                    if (ky.codes) {                     // of y as it is stored
                        float t[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                        if (s.has) unpack<T, 8>(out, t);
                        store_codes(ky.fmt, t, s.has, ky.codes, ky.scales, s.n * w.HW + q, s.v, w.C, blocks);
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
    __device__ __forceinline__ void load(const Source& s, const Geo& g, const Walk& w, long long n, int p, int v) {
        if constexpr (SRC == kSrcSame) r = *(const R*)((const T*)s.x + n * g.sn + g.at(p) + V * v);
        else {
            const long long row = n * w.HW + p;
            r = *(const R*)(s.codes + row * w.C + V * v);
            e = s.scales[row * ((w.C + 31) / 32) + V * v / 32];
        }
    }
    __device__ __forceinline__ void value(float* f) const {
        if constexpr (SRC == kSrcSame) unpack<T, V>(r, f);
        else {
            code_values<SRC, V>(r, f);
            const float sc = scale_of(e);
            #pragma unroll
            for (int i = 0; i < V; ++i) f[i] *= sc;
        }
    }
};
// The side of ReLU's kink that a value is on, where fp32 cannot tell: d and a carry a rounding each, so z = d a + b is off by up to
// 2^-23 |b| or so when it is near zero.  Such values (a few in a million) are taken again in fp64 from x itself.
__device__ __noinline__ bool relu_side(float x, float nm, float rstd, float weight, float b) {
    return ((double)x + (double)nm) * (double)rstd * (double)weight + (double)b > 0.;
}
struct BackwardArgs {
    const float *mean, *rstd, *weight, *bias;
};
// d = x - mean and dz from x and dy (in place: x becomes d, dy becomes dz)
template <typename T, int V>
__device__ __forceinline__ void activation_gradient(const NormShape& sh, const Chan<V>& k, const BackwardArgs& A, long long n, int c0, float* x, float* dy) {
    if (sh.act == kActRelu) {
        #pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = x[i] + k.nm[i], z = fmaf(d, k.a[i], k.b[i]);
            bool on = !(z <= 0.f);
            if (fabsf(z) < 1e-6f * fabsf(k.b[i]))
                on = relu_side(x[i], k.nm[i], A.rstd[n * sh.groups + (c0 + i) / sh.cg], A.weight ? A.weight[c0 + i] : 1.f, k.b[i]);
            x[i] = d;
            dy[i] = on ? dy[i] : 0.f;
        }
    } else {
        v_add<V>(x, k.nm, x);
        if (sh.act == kActSilu) {
            float z[V];
            v_fma<V>(x, k.a, k.b, z);
            #pragma unroll
            for (int i = 0; i < V; ++i) { const float s = sigmoid<T>(z[i]); dy[i] *= fmaf(z[i] * s, 1.f - s, s); }
        }
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
                    fx[u].value(f);
                    unpack<T, V>(r[u], q);
                    activation_gradient<T, V>(sh, k, A, s.n, V * s.v, f, q);
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
                fx[u].value(f);
                unpack<T, V>(r[u], q);
                activation_gradient<T, V>(sh, k, A, s.n, V * s.v, f, q);
                v_fma<V>(f, B, D, f);
                v_fma<V>(q, k.a, f, q);
                *(Raw<T, V>*)(op + gdx.at(p + u * w.rows)) = pack<T, V>(q);
            }
    }
}

}  // namespace op
