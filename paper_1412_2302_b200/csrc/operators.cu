// Host side of the operators on caller-owned tensors declared at the end of include/alexnet.h: group normalisation with an activation, 8-bit
// activation checkpoints, and the weight gradient of a linear layer from a checkpoint.  No handle and no device memory of their own: the
// caller gives every buffer, the workspace included, so calls on different streams share nothing.
#include "../../include/alexnet.h"

#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>
#include <utility>

#include "checkpoint.cuh"
#include "group_norm.cuh"
#include "linear_grad.cuh"

namespace {
using namespace op;
using bf16 = __nv_bfloat16;
constexpr int kSms = 148;

struct Err {
    char* buf; size_t len; const char* who;
    int arg(const char* msg) const { if (buf && len) snprintf(buf, len, "%s: %s", who, msg); return ALEXNET_ERR_ARG; }
    int cuda(cudaError_t e) const { cudaGetLastError(); if (buf && len) snprintf(buf, len, "%s: %s", who, cudaGetErrorString(e)); return ALEXNET_ERR_CUDA; }
};

// launches of one call, in order; the first refused launch ends it
struct Launcher {
    cudaStream_t st;
    cudaError_t e = cudaSuccess;
    size_t smem = 0;            // of the next launch
    int cluster = 1;
    template <typename... KArgs, typename... Args>
    void operator()(void (*kernel)(KArgs...), long long grid, int block, Args&&... args) {
        if (e != cudaSuccess) return;
        cudaLaunchConfig_t lc{};
        lc.gridDim = dim3((unsigned)grid); lc.blockDim = block; lc.dynamicSmemBytes = smem; lc.stream = st;
        cudaLaunchAttribute at[2]{};
        at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[0].val.programmaticStreamSerializationAllowed = 1;
        at[1].id = cudaLaunchAttributeClusterDimension;
        at[1].val.clusterDim.x = cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
        lc.attrs = at; lc.numAttrs = cluster > 1 ? 2 : 1;
        smem = 0; cluster = 1;
        e = cudaLaunchKernelEx(&lc, kernel, std::forward<Args>(args)...);
    }
};

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }
bool is_fmt(int f) { return f == ALEXNET_CODES_INT8 || f == ALEXNET_CODES_E4M3; }
int elem_bytes(int dtype) { return dtype == ALEXNET_DTYPE_F32 ? 4 : 2; }
int src_of(int fmt) { return fmt == ALEXNET_CODES_INT8 ? kSrcInt8 : kSrcE4m3; }

struct Dims { long long n; int h, w, C; };
const char* check_dims(const Dims& d) {
    if (d.n < 0) return "n must not be negative";
    if (d.h < 1 || d.w < 1) return "h and w must be at least 1";
    if (d.C < 1 || d.C > (1 << 20)) return "channels must be 1 to 1048576";
    if ((long long)d.h * d.w > (1ll << 30)) return "h * w exceeds 2^30";
    if (d.n > (1ll << 31) || (d.n > 0 && d.n * d.h * d.w > (1ll << 48) / d.C)) return "the tensor is too large";
    return nullptr;
}
const char* check_view(const alexnet_view_t& v, const Dims& d, int dtype, bool output) {
    if (d.n == 0) return nullptr;
    if (!v.data) return "NULL pointer";
    if ((uintptr_t)v.data % elem_bytes(dtype)) return "a tensor is not aligned to its elements";
    long long size[3] = {d.n, d.h, d.w}, st[3] = {v.stride_n, v.stride_h, v.stride_w};
    for (int i = 0; i < 3; ++i)
        if (size[i] > 1 && (st[i] < 0 || st[i] > (1ll << 48))) return "a stride is negative or too large";
    if (output) {      // positions must not share memory: by rising stride, each dimension steps over all of the ones below
        for (int i = 0; i < 3; ++i)
            for (int j = i + 1; j < 3; ++j)
                if (st[j] < st[i]) { std::swap(st[i], st[j]); std::swap(size[i], size[j]); }
        long long extent = d.C;
        for (int i = 0; i < 3; ++i)
            if (size[i] > 1) {
                if (st[i] < extent) return "positions of an output overlap";
                extent += (size[i] - 1) * st[i];
            }
    }
    return nullptr;
}
Geo geo_of(const alexnet_view_t& v, const Dims& d, int step) {
    Geo g{};
    g.sn = d.n > 1 ? v.stride_n : 0;
    g.sh = d.h > 1 ? v.stride_h : 0;
    g.sw = d.w > 1 ? v.stride_w : 0;
    g.w = fast_div((uint32_t)d.w);
    g.flat = d.h == 1 || d.w == 1 || g.sh == (long long)d.w * g.sw;
    if (d.w == 1) g.sw = g.sh;
    g.step = step;
    g.inc = step * g.sw;
    g.wrap = g.flat ? 0 : g.sh - d.w * g.sw;
    return g;
}
// vectors of eight channels at 16-byte boundaries everywhere
bool vec_ok(const alexnet_view_t& v, const Dims& d, int dtype) {
    const int step = 16 / elem_bytes(dtype);
    return d.C % 8 == 0 && (uintptr_t)v.data % 16 == 0 && (d.n <= 1 || v.stride_n % step == 0) && (d.h <= 1 || v.stride_h % step == 0) && (d.w <= 1 || v.stride_w % step == 0);
}
bool vec_ok(const alexnet_checkpoint_t& k, const Dims& d) { return d.C % 8 == 0 && (uintptr_t)k.codes % 8 == 0; }

// How a launch walks [n][h w][C] with vectors of V channels.  Elementwise passes (blocks_per_sm = 0): eight blocks per SM, of at least four positions per thread.
// Passes whose blocks end with a reduction: whole rounds of what an SM holds of them (`blocks_per_sm` with vectors of eight, six with single channels), a block being as dear as
// its positions and ten more, and a thread adds up at most kMostTerms of them, for the sake of the sums' roundings.
constexpr int kElementwise = 0, kForwardSums = 3, kMostTerms = 192;
Walk find_walk(const Dims& d, int V, int blocks_per_sm) {
    Walk w{};
    w.C = d.C; w.HW = d.h * d.w; w.vecs = d.C / V;
    const int q = V == 8 ? 4 : 1, padded = (int)ceil_div(w.vecs, q) * q;
    w.colblocks = (int)ceil_div(padded, 256);
    w.cols = (int)ceil_div(ceil_div(padded, w.colblocks), q) * q;
    w.rows = 256 / w.cols;
    const long long blocks = std::max<long long>(1, d.n * w.colblocks), most = std::max<long long>(1, ceil_div(w.HW, 4 * w.rows));
    long long chunks = std::min(most, ceil_div(8 * kSms, blocks));
    if (blocks_per_sm) {
        const int slots = (V == 8 ? blocks_per_sm : 6) * kSms;
        const long long least = ceil_div(w.HW, (long long)kMostTerms * w.rows);
        long long cost = 1ll << 62;
        for (long long c = least; c <= std::max(least, std::min(most, ceil_div(32 * kSms, blocks))); ++c) {
            const long long t = ceil_div(blocks * c, slots) * (ceil_div(ceil_div(w.HW, c), w.rows) + 10);
            if (t < cost) { cost = t; chunks = c; }
        }
    }
    chunks = std::max<long long>(1, std::min<long long>(chunks, w.HW));
    w.ppc = (int)ceil_div(w.HW, chunks);
    w.chunks = ceil_div(w.HW, w.ppc);
    w.dense = dense_of(d.C, w.rows);
    return w;
}
// (found once for the sizes of a thread's last calls, three or four walks each: with few large samples the search takes 15 to 60 us)
const Walk& walk_of(const Dims& d, int V, int blocks_per_sm) {
    struct Known { long long n = -1; int HW, C, V, blocks_per_sm; Walk walk; };
    static thread_local Known known[64];
    static thread_local unsigned next = 0;
    const int HW = d.h * d.w;
    for (const Known& q : known)
        if (q.n == d.n && q.HW == HW && q.C == d.C && q.V == V && q.blocks_per_sm == blocks_per_sm) return q.walk;
    Known& q = known[next++ % 64];
    q = {d.n, HW, d.C, V, blocks_per_sm, find_walk(d, V, blocks_per_sm)};
    return q.walk;
}
// the same for rows of any length: a vector is a checkpoint block, taken by a warp
Walk walk_any(const Dims& d) {
    Walk w{};
    w.C = d.C; w.HW = d.h * d.w; w.vecs = (int)ceil_div(d.C, 32);
    w.colblocks = (int)ceil_div(w.vecs, 8);
    w.cols = (int)ceil_div(w.vecs, w.colblocks);
    w.rows = 8 / w.cols;
    const long long chunks = std::max<long long>(1, std::min(ceil_div(w.HW, 8 * w.rows), ceil_div(8 * kSms, std::max<long long>(1, d.n * w.colblocks))));
    w.ppc = (int)ceil_div(w.HW, chunks);
    w.chunks = ceil_div(w.HW, w.ppc);
    w.dense = dense_of(d.C, w.rows);
    return w;
}
long long grid_of(const Walk& w, const Dims& d) { return d.n * w.chunks * w.colblocks; }
constexpr long long kMaxGrid = 0x7fffffffll;

template <typename T>
void encode(Launcher& go, const Dims& d, const alexnet_view_t& x, const alexnet_checkpoint_t& k, int dtype) {
    const bool vec = vec_ok(x, d, dtype) && vec_ok(k, d), int8 = k.format == ALEXNET_CODES_INT8;
    const Walk w = vec ? walk_of(d, 8, kElementwise) : walk_any(d);
    const Geo g = geo_of(x, d, w.rows);
    if (vec) go(int8 ? checkpoint_encode_kernel<T, kSrcInt8> : checkpoint_encode_kernel<T, kSrcE4m3>, grid_of(w, d), 256, (const T*)x.data, g, w, (uint8_t*)k.codes, k.scales);
    else go(int8 ? checkpoint_encode_any_kernel<T, kSrcInt8> : checkpoint_encode_any_kernel<T, kSrcE4m3>, grid_of(w, d), 256, (const T*)x.data, g, w, (uint8_t*)k.codes, k.scales);
}
template <typename T>
void decode(Launcher& go, const Dims& d, const alexnet_view_t& x, const alexnet_checkpoint_t& k, int dtype) {
    const bool vec = vec_ok(x, d, dtype) && vec_ok(k, d), int8 = k.format == ALEXNET_CODES_INT8;
    const Walk w = vec ? walk_of(d, 8, kElementwise) : walk_any(d);
    const Geo g = geo_of(x, d, w.rows);
    const uint8_t *codes = (const uint8_t*)k.codes, *scales = k.scales;
    if (vec) go(int8 ? checkpoint_decode_kernel<T, kSrcInt8> : checkpoint_decode_kernel<T, kSrcE4m3>, grid_of(w, d), 256, codes, scales, g, w, (T*)x.data);
    else go(int8 ? checkpoint_decode_any_kernel<T, kSrcInt8> : checkpoint_decode_any_kernel<T, kSrcE4m3>, grid_of(w, d), 256, codes, scales, g, w, (T*)x.data);
}
const char* check_codes(const alexnet_checkpoint_t& k, const Dims& d) {
    if (!is_fmt(k.format)) return "unknown checkpoint format";
    if (d.n > 0 && (!k.codes || !k.scales)) return "NULL pointer in a checkpoint";
    return nullptr;
}
bool is_dtype(int t) { return t == ALEXNET_DTYPE_BF16 || t == ALEXNET_DTYPE_F16 || t == ALEXNET_DTYPE_F32; }

int checkpoint_call(const alexnet_checkpoint_args_t* a, cudaStream_t st, const Err& err, bool enc) {
    if (!a) return err.arg("NULL arguments");
    const Dims d{a->n, a->h, a->w, a->channels};
    if (const char* m = check_dims(d)) return err.arg(m);
    if (!is_dtype(a->dtype)) return err.arg("unknown dtype");
    if (const char* m = check_view(a->x, d, a->dtype, !enc)) return err.arg(m);
    if (const char* m = check_codes(a->checkpoint, d)) return err.arg(m);
    if (d.n == 0) return ALEXNET_OK;
    if (grid_of(walk_any(d), d) > kMaxGrid || grid_of(walk_of(d, 1, kElementwise), d) > kMaxGrid) return err.arg("the tensor is too large");
    Launcher go{st};
    switch (a->dtype) {
    case ALEXNET_DTYPE_BF16: enc ? encode<bf16>(go, d, a->x, a->checkpoint, a->dtype) : decode<bf16>(go, d, a->x, a->checkpoint, a->dtype); break;
    case ALEXNET_DTYPE_F16: enc ? encode<__half>(go, d, a->x, a->checkpoint, a->dtype) : decode<__half>(go, d, a->x, a->checkpoint, a->dtype); break;
    default: enc ? encode<float>(go, d, a->x, a->checkpoint, a->dtype) : decode<float>(go, d, a->x, a->checkpoint, a->dtype); break;
    }
    return go.e == cudaSuccess ? ALEXNET_OK : err.cuda(go.e);
}

// ---------------------------------------------------------------- group norm
const char* check_shape(const alexnet_group_norm_t& s) {
    if (const char* m = check_dims({s.n, s.h, s.w, s.channels})) return m;
    if (s.groups < 1 || s.channels % s.groups) return "groups must divide the channels";
    if (!is_dtype(s.dtype)) return "unknown dtype";
    if (s.activation < ALEXNET_ACT_NONE || s.activation > ALEXNET_ACT_SILU) return "unknown activation";
    if (!(s.eps > 0.f)) return "eps must be positive";
    if (s.n * s.groups > kMaxGrid / 2) return "the tensor is too large";
    return nullptr;
}
NormShape norm_shape(const alexnet_group_norm_t& s) { return {s.channels, s.h * s.w, s.groups, s.channels / s.groups, fast_div((uint32_t)(s.channels / s.groups)), s.eps, s.activation}; }
constexpr size_t kSmSmem = 228 * 1024, kCtaSmem = 227 * 1024;
// How blocks that keep whole groups of a sample walk a tensor, `slot` bytes kept per vector of V channels; threads = 0: not at all.  As many slices as there are
// (powers of two) until a slice takes at most 112 KB, so that two blocks share an SM, and further while the device is not full; but no rows below 64
// bytes, which cost more sectors than they use.
template <int V>
SliceWalk find_slice_walk(const Dims& d, int groups, int slot, int elem, bool backward) {
    SliceWalk best{}, w{};
    w.C = d.C; w.HW = d.h * d.w;
    const int cg = d.C / groups;
    for (w.slices = 1; w.slices <= 64; w.slices *= 2) {
        w.Cs = d.C / w.slices; w.groups = groups / w.slices;
        if (w.slices > 1 && (groups % w.slices || w.Cs % 32 || w.Cs * elem < 64)) break;
        w.vecs = w.Cs / V;
        w.cols = (int)ceil_div(w.vecs, V == 8 ? 4 : 1) * (V == 8 ? 4 : 1);
        if (w.cols > kSlThreads || w.groups > 1024 || d.n > kMaxGrid / 64) continue;
        // threads: the fewest slots, and among alike the most
        long long slots = 1ll << 60;
        SliceWalk t = w;
        for (t.threads = 128; t.threads <= kSlThreads; t.threads += 32) {
            if (t.threads < w.cols) continue;
            t.rows = t.threads / w.cols;
            t.its = (int)ceil_div(w.HW, t.rows);
            if (t.its * (long long)t.threads <= slots + slots / 16) { slots = std::min(slots, t.its * (long long)t.threads); w.threads = t.threads; w.rows = t.rows; w.its = t.its; }
        }
        if (!w.threads || (size_t)w.its * w.threads * slot + slice_scratch<V>(w, backward) > kSmSmem / 2 - 1024) continue;
        best = w;
        if (d.n * w.slices >= 2 * kSms) break;
    }
    if (!best.threads) return best;
    best.dense = dense_of(d.C, best.rows);
    best.lanes = 1;
    while (best.lanes < 32 && best.lanes * 2 * best.groups <= best.threads && best.lanes < cg * best.rows) best.lanes *= 2;
    for (best.lc = 1; best.lc < best.lanes && best.lc < cg; best.lc *= 2) ++best.lc_shift;
    return best;
}
// (found once for the sizes of a thread's last calls: the search takes 2 us)
template <int V>
const SliceWalk& slice_walk(const Dims& d, int groups, int slot, int elem, bool backward) {
    struct Known { long long n = -1; int h, w, C, groups, slot, elem; bool backward; SliceWalk walk; };
    static thread_local Known known[16];
    static thread_local unsigned next = 0;
    for (const Known& q : known)
        if (q.n == d.n && q.h == d.h && q.w == d.w && q.C == d.C && q.groups == groups && q.slot == slot && q.elem == elem && q.backward == backward) return q.walk;
    Known& q = known[next++ % 16];
    q = {d.n, d.h, d.w, d.C, groups, slot, elem, backward, find_slice_walk<V>(d, groups, slot, elem, backward)};
    return q.walk;
}
// Forward passes: samples of more than 64 positions are kept by blocks where they are read in vectors of eight.  (With single channels the three launches are
// faster or alike: 1 x 13 x 13 x 75 6.2 us against 17, 512 x 9 x 9 x 75 15.4 against 18.9, 512 x 13 x 13 x 75 24 against 22.5; 512 x 7 x 7 x 75 takes 12.9
// against 10.7.)
template <int V>
const SliceWalk& forward_slices(const Dims& d, int groups, int elem) {
    static const SliceWalk none{};
    if (d.h * d.w > 64 && V == 1) return none;
    return slice_walk<V>(d, groups, elem * V, elem, false);
}
// Backward passes: samples of more than 64 positions are kept by blocks where x is read as it is, in vectors of eight.  (From int8 codes, or with single
// channels, the three launches are faster, SiLU: 128 x 27 x 27 x 256 61 us against 71, 512 x 13 x 13 x 384 93 against 99, 512 x 11 x 11 x 256 47 against 50,
// 512 x 9 x 9 x 75 from x 25 against 30; with fewer positions they are not: 512 x 9 x 9 x 256 36 against 34, 2048 x 7 x 7 x 512 159 against 133; nor from x:
// 512 x 27 x 27 x 256 without an activation 168 against 139.)
template <int V>
const SliceWalk& backward_slices(const Dims& d, int groups, int elem, bool kept) {
    static const SliceWalk none{};
    if (d.h * d.w > 64 && (kept || V == 1)) return none;
    return slice_walk<V>(d, groups, elem * V + (kept ? V + 1 : elem * V), kept ? 2 : elem, true);
}
// Samples that are under way at once: as many blocks per slice as the device holds (asked once per kernel and launch shape).
template <typename K>
long long slice_rows(Launcher& go, K* kernel, const SliceWalk& w, const Dims& d, size_t smem) {
    struct Known { const void* kernel = nullptr; int device, threads, blocks; size_t smem; };
    static thread_local Known known[16];      // (of all kernels with this signature)
    static thread_local unsigned next = 0;
    int dev = 0, blocks = 0;
    if (go.e == cudaSuccess) go.e = cudaGetDevice(&dev);
    for (const Known& q : known)
        if (q.kernel == (const void*)kernel && q.device == dev && q.threads == w.threads && q.smem == smem) blocks = q.blocks;
    if (!blocks && go.e == cudaSuccess) {
        go.e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kCtaSmem);
        if (go.e == cudaSuccess) go.e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, kernel, w.threads, smem);
        if (go.e == cudaSuccess) known[next++ % 16] = {(const void*)kernel, dev, w.threads, blocks, smem};
    }
    return std::min<long long>(d.n, std::max(1, std::min(blocks, 32) * kSms / w.slices));
}

// Bytes of workspace of a call with vectors of V channels; 0 where it takes one launch and leaves nothing between.
template <int V>
size_t forward_ws(const Dims& d, int groups, int dtype) {
    if (forward_slices<V>(d, groups, elem_bytes(dtype)).threads) return 0;
    const Walk w = walk_of(d, V, kForwardSums);
    return (size_t)(d.n * w.chunks) * d.C * sizeof(float4);
}
template <int V>
size_t backward_ws(const Dims& d, int groups, int dtype, bool kept) {
    const int elem = elem_bytes(dtype);
    const SliceWalk& s = backward_slices<V>(d, groups, elem, kept);
    // (never more blocks of a slice than 32 per SM; slice_sums grows with them by less than their number)
    if (s.threads) return d.n == 1 ? 0 : (size_t)(std::min<long long>(d.n, 32 * kSms) + d.n / kSlSamples) * 2 * d.C * sizeof(float);
    return (size_t)(d.n * groups) * sizeof(float2) + (size_t)(d.n * walk_of(d, V, kBackwardBlocks<V>).chunks) * 2 * d.C * sizeof(float);
}
size_t reported(size_t bytes) { return bytes ? (bytes + 511) / 256 * 256 : 256; }
// whether a call reads and writes vectors of eight channels
bool forward_in_vectors(const alexnet_group_norm_forward_t& a, const Dims& d) {
    return vec_ok(a.x, d, a.shape.dtype) && vec_ok(a.y, d, a.shape.dtype) && (!a.keep_x.codes || vec_ok(a.keep_x, d)) && (!a.keep_y.codes || vec_ok(a.keep_y, d));
}
bool backward_in_vectors(const alexnet_group_norm_backward_t& a, const Dims& d) {
    return vec_ok(a.dy, d, a.shape.dtype) && vec_ok(a.dx, d, a.shape.dtype) && (a.kept.codes || a.kept.scales ? vec_ok(a.kept, d) : vec_ok(a.x, d, a.shape.dtype));
}
template <typename T, int V, int ACT>
void forward(Launcher& go, const alexnet_group_norm_forward_t* a, const Dims& d) {
    const Walk w = walk_of(d, V, kForwardSums);
    const NormShape s = norm_shape(a->shape);
    Keep kx{}, ky{};
    if (V == 8) {
        if (a->keep_x.codes) kx = {(uint8_t*)a->keep_x.codes, a->keep_x.scales, src_of(a->keep_x.format)};
        if (a->keep_y.codes) ky = {(uint8_t*)a->keep_y.codes, a->keep_y.scales, src_of(a->keep_y.format)};
    }
    const SliceWalk& sw = forward_slices<V>(d, s.groups, (int)sizeof(T));
    if (sw.threads) {
        const size_t smem = (size_t)sw.its * sw.threads * sizeof(T) * V + slice_scratch<V>(sw, false);
        const long long rows = slice_rows(go, gn_slice_forward_kernel<T, V, ACT>, sw, d, smem);
        go.smem = smem;
        go(gn_slice_forward_kernel<T, V, ACT>, rows * sw.slices, sw.threads, (const T*)a->x.data, geo_of(a->x, d, sw.rows), sw, s, (long long)d.n, a->weight, a->bias, (T*)a->y.data,
           geo_of(a->y, d, sw.rows), a->mean, a->rstd, kx, ky);
        if (V != 8) {
            if (a->keep_x.codes) encode<T>(go, d, a->x, a->keep_x, a->shape.dtype);
            if (a->keep_y.codes) encode<T>(go, d, a->y, a->keep_y, a->shape.dtype);
        }
        return;
    }
    const Walk wa = walk_of(d, V, kElementwise);
    const Geo gx = geo_of(a->x, d, w.rows), gy = geo_of(a->y, d, w.rows);      // (the same threads' rows in both walks)
    float4* partial = (float4*)a->workspace;
    const T *x = (const T*)a->x.data;
    go(gn_sums_kernel<T, V>, grid_of(w, d), 256, x, gx, w, partial);
    const long long groups = d.n * s.groups;
    const bool block = groups < 8 * kSms;
    go(block ? gn_statistics_kernel<true> : gn_statistics_kernel<false>, block ? groups : ceil_div(groups, 8), 256, (const float4*)partial, s, groups, (int)w.chunks, w.ppc, a->mean, a->rstd);
    const bool keep = kx.codes || ky.codes;
    go(keep ? gn_apply_kernel<T, V, ACT, V == 8> : gn_apply_kernel<T, V, ACT, false>, grid_of(wa, d), 256, x, gx, wa, s, a->weight, a->bias, (const float*)a->mean, (const float*)a->rstd, (T*)a->y.data, gy, kx, ky);
    if (V != 8) {
        if (a->keep_x.codes) encode<T>(go, d, a->x, a->keep_x, a->shape.dtype);
        if (a->keep_y.codes) encode<T>(go, d, a->y, a->keep_y, a->shape.dtype);
    }
}
template <typename T, int V, int SRC, int ACT>
void backward(Launcher& go, const alexnet_group_norm_backward_t* a, const Dims& d) {
    const Walk w = walk_of(d, V, kBackwardBlocks<V>);
    const NormShape s = norm_shape(a->shape);
    float2* c12 = (float2*)a->workspace;
    float* partial = (float*)(c12 + d.n * s.groups);
    const Source src{a->x.data, (const uint8_t*)a->kept.codes, a->kept.scales};
    const BackwardArgs A{a->mean, a->rstd, a->weight, a->bias};
    const T* dy = (const T*)a->dy.data;
    constexpr int kSlot = (int)sizeof(T) * V + (SRC == kSrcSame ? (int)sizeof(T) * V : V + 1);
    const SliceWalk& sw = backward_slices<V>(d, s.groups, (int)sizeof(T), SRC != kSrcSame);
    if (sw.threads) {
        partial = (float*)a->workspace;
        auto* kernel = gn_slice_backward_kernel<T, V, SRC, ACT>;
        const size_t smem = (size_t)sw.its * sw.threads * kSlot + slice_scratch<V>(sw, true);
        const long long rows = slice_rows(go, kernel, sw, d, smem);
        go.smem = smem;
        go(kernel, rows * sw.slices, sw.threads, dy, geo_of(a->dy, d, sw.rows), src, geo_of(a->x, d, sw.rows), sw, s, (long long)d.n, A, (T*)a->dx.data, geo_of(a->dx, d, sw.rows),
           rows > 1 ? partial : a->dbias, rows > 1 ? partial + d.C : a->dweight, rows > 1 ? 2ll * d.C : 0ll);
        if (rows > 1 && (a->dweight || a->dbias)) go(gn_parameter_gradient_kernel, ceil_div(d.C, 32), 1024, (const float*)partial, d.C, slice_sums(d.n, rows), a->dweight, a->dbias);
        return;
    }
    const Geo gdy = geo_of(a->dy, d, w.rows), gx = geo_of(a->x, d, w.rows), gdx = geo_of(a->dx, d, w.rows);
    go(gn_backward_sums_kernel<T, V, SRC, ACT>, grid_of(w, d), 256, dy, gdy, src, gx, w, s, A, partial);
    const long long groups = d.n * s.groups;
    const bool block = groups < 8 * kSms;
    go(block ? gn_backward_group_kernel<true> : gn_backward_group_kernel<false>, block ? groups : ceil_div(groups, 8), 256, (const float*)partial, s, groups, (int)w.chunks, A, c12);
    const int extra = a->dweight || a->dbias ? (int)ceil_div(d.C, 32) : 0;
    go(gn_backward_apply_kernel<T, V, SRC, ACT>, grid_of(w, d) + extra, 256, dy, gdy, src, gx, w, s, A, (const float2*)c12, (T*)a->dx.data, gdx, (const float*)partial, d.n * w.chunks, extra, a->dweight,
       a->dbias);
}
template <typename T, int V, int SRC>
void backward(Launcher& go, const alexnet_group_norm_backward_t* a, const Dims& d) {
    if constexpr (V == 1) backward<T, V, SRC, kActAny>(go, a, d);
    else if (a->shape.activation == ALEXNET_ACT_NONE) backward<T, V, SRC, kActNone>(go, a, d);
    else if (a->shape.activation == ALEXNET_ACT_RELU) backward<T, V, SRC, kActRelu>(go, a, d);
    else backward<T, V, SRC, kActSilu>(go, a, d);
}
template <typename T, int V>
void backward(Launcher& go, const alexnet_group_norm_backward_t* a, const Dims& d) {
    if (a->x.data) backward<T, V, kSrcSame>(go, a, d);
    else if (a->kept.format == ALEXNET_CODES_INT8) backward<T, V, kSrcInt8>(go, a, d);
    else backward<T, V, kSrcE4m3>(go, a, d);
}
template <typename T, int V>
void forward(Launcher& go, const alexnet_group_norm_forward_t* a, const Dims& d) {
    if constexpr (V == 1) forward<T, V, kActAny>(go, a, d);
    else if (a->shape.activation == ALEXNET_ACT_NONE) forward<T, V, kActNone>(go, a, d);
    else if (a->shape.activation == ALEXNET_ACT_RELU) forward<T, V, kActRelu>(go, a, d);
    else forward<T, V, kActSilu>(go, a, d);
}

// ---------------------------------------------------------------- linear weight gradient
const char* check_linear(const alexnet_linear_weight_grad_t& a) {
    if (a.rows < 0 || a.rows > (1ll << 30)) return "rows must be 0 to 2^30";
    if (a.n_in < 1 || a.n_out < 1 || a.n_in > (1 << 20) || a.n_out > (1 << 20)) return "features must be 1 to 1048576";
    if (!is_fmt(a.x.format)) return "unknown checkpoint format";
    if ((uintptr_t)a.dy % 2) return "dy is not aligned to its elements";
    if (a.rows > 1 && (a.dy_stride < 0 || a.dy_stride > (1ll << 38))) return "the stride of dy is negative or too large";
    return nullptr;
}
PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
    static std::atomic<void*> cached{nullptr};
    void* fn = cached.load();
    if (!fn) {
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) { cudaGetLastError(); return nullptr; }
        cached.store(fn);
    }
    return (PFN_cuTensorMapEncodeTiled_v12000)fn;
}
struct LinearPlan {
    int cg, BN, m_tiles, tiles, steps, whole, splits, per, stages;
    bool move_dy, move_x;               // copies with rows on 16-byte boundaries, where the rows are not
    long long dy_pitch, x_pitch;        // bytes
    size_t dy_at, x_at, bytes, smem;    // places in the workspace, behind the partial sums
};
LinearPlan find_linear_plan(const alexnet_linear_weight_grad_t& a) {
    LinearPlan b{};
    b.steps = (int)ceil_div(a.rows, kLgRows);
    // The tile's width, pairs or single CTAs and the splits of the last round by a model of the launch in cycles, fitted to measurements (BN 128 to
    // 256): a step of 64 rows costs 480 + 1.6 BN, in a pair 420 + 1.4 BN (half of dy's way through shared memory); a tile no less
    // than its stores, and 1500 or 2500 around them; a second launch 4000, and its partial sums 2500 bytes a cycle.
    double best = 1e30;
    for (int cg = 1; cg <= 2; ++cg)
        for (int BN = 256; BN >= 32; BN -= 32) {
            if (BN > 32 && BN - 32 >= a.n_out) continue;
            if (cg == 2 && (BN < 128 || a.n_in <= 128)) continue;
            const long long tiles = ceil_div(a.n_in, 128 * cg) * ceil_div(a.n_out, BN), slots = kSms / cg;
            const double step = cg == 2 ? 420 + 1.4 * BN : 480 + 1.6 * BN, around = cg == 2 ? 2500 : 1500;
            auto round = [&](long long steps) { return std::max(steps * step, 22.0 * BN) + around; };
            for (int s = 1; s <= 64; ++s) {
                const long long per = ceil_div(std::max(1, b.steps), s);
                const int splits = (int)ceil_div(std::max(1, b.steps), per);
                const long long whole = splits > 1 ? tiles / slots * slots : tiles, rest = tiles - whole;
                if (s > 1 && (per < 4 || rest * (s - 1) >= slots)) break;
                double cost = (double)ceil_div(whole, slots) * round(b.steps);
                if (rest) cost += (double)ceil_div(rest * splits, slots) * round(per) + 4000 + (double)splits * rest * 128 * cg * BN * 8 / 2500;
                if (cost < best) { best = cost; b.cg = cg; b.BN = BN; b.tiles = (int)tiles; b.whole = (int)whole; b.splits = splits; b.per = (int)per; }
            }
        }
    b.m_tiles = (int)ceil_div(a.n_in, 128 * b.cg);
    const int stage = kLgA + (b.BN / b.cg + 63) / 64 * 8192;
    b.stages = std::min(kLgMaxStages, (227 * 1024 - 1024 - 256) / stage);
    b.smem = tc::own_sm(1024 + (size_t)b.stages * stage + 256);
    b.dy_pitch = ceil_div(a.n_out, 8) * 16;
    b.x_pitch = ceil_div(a.n_in, 16) * 16;
    b.dy_at = (size_t)b.splits * (b.tiles - b.whole) * b.BN * 128 * b.cg * sizeof(float);
    return b;
}
// (found once for the sizes of a thread's last calls: with few tiles the search takes 10 us; what goes by alignment is added)
LinearPlan linear_plan(const alexnet_linear_weight_grad_t& a) {
    struct Known { long long rows = -1; int n_in, n_out; LinearPlan plan; };
    static thread_local Known known[16];
    static thread_local unsigned next = 0;
    const Known* found = nullptr;
    for (const Known& q : known)
        if (q.rows == a.rows && q.n_in == a.n_in && q.n_out == a.n_out) found = &q;
    if (!found) {
        known[next % 16] = {a.rows, a.n_in, a.n_out, find_linear_plan(a)};
        found = &known[next++ % 16];
    }
    LinearPlan b = found->plan;
    b.move_dy = (uintptr_t)a.dy % 16 != 0 || (a.rows > 1 && (a.dy_stride % 8 != 0 || a.dy_stride < a.n_out));
    b.move_x = (uintptr_t)a.x.codes % 16 != 0 || a.n_in % 16 != 0;
    b.x_at = b.dy_at + (b.move_dy ? ((size_t)a.rows * b.dy_pitch + 255) / 256 * 256 : 0);
    b.bytes = b.x_at + (b.move_x ? ((size_t)a.rows * b.x_pitch + 255) / 256 * 256 : 0);      // 0: none needed
    return b;
}
long long repitch_grid(long long rows, long long pitch) { return std::min<long long>(16 * kSms, ceil_div(rows * (pitch / 16), 256)); }
int linear_call(const alexnet_linear_weight_grad_t* a, cudaStream_t st, const Err& err, int drop) {
    if (!a) return err.arg("NULL arguments");
    if (const char* m = check_linear(*a)) return err.arg(m);
    if (!a->dw || (uintptr_t)a->dw % 4) return err.arg("dw is NULL or not aligned");
    if (a->rows > 0 && (!a->dy || !a->x.codes || !a->x.scales)) return err.arg("NULL pointer");
    const LinearPlan pl = linear_plan(*a);
    if (pl.bytes && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < pl.bytes)) return err.arg("the workspace is too small or not 16-byte aligned");
    if (a->rows == 0) {
        const cudaError_t e = cudaMemsetAsync(a->dw, 0, (size_t)a->n_in * a->n_out * sizeof(float), st);
        return e == cudaSuccess ? ALEXNET_OK : err.cuda(e);
    }
    LinearGradParams p{};
    Launcher go{st};
    const void* dy = a->dy;
    long long dy_pitch = a->dy_stride * 2;
    if (pl.move_dy) {
        uint8_t* t = (uint8_t*)a->workspace + pl.dy_at;
        go(repitch_kernel<uint16_t>, repitch_grid(a->rows, pl.dy_pitch), 256, (const uint8_t*)a->dy, a->rows > 1 ? a->dy_stride * 2 : 0ll, a->n_out * 2, pl.dy_pitch, a->rows, t);
        dy = t; dy_pitch = pl.dy_pitch;
    } else if (a->rows == 1) dy_pitch = ceil_div(a->n_out, 8) * 16;
    p.codes = (const uint8_t*)a->x.codes;
    p.code_pitch = a->n_in;
    if (pl.move_x) {
        uint8_t* t = (uint8_t*)a->workspace + pl.x_at;
        go(repitch_kernel<uint8_t>, repitch_grid(a->rows, pl.x_pitch), 256, p.codes, (long long)a->n_in, a->n_in, pl.x_pitch, a->rows, t);
        p.codes = t; p.code_pitch = pl.x_pitch;
    }
    PFN_cuTensorMapEncodeTiled_v12000 enc = tensor_map_encoder();
    if (!enc) return err.cuda(cudaErrorNotSupported);
    const cuuint64_t dims[2] = {(cuuint64_t)a->n_out, (cuuint64_t)a->rows}, strides[1] = {(cuuint64_t)dy_pitch};
    const cuuint32_t box[2] = {64, kLgRows}, one[2] = {1, 1};
    if (enc(&p.tmD, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(dy), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return err.arg("the driver refused the tensor map of dy");
    p.scales = a->x.scales;
    p.blocks = (int)ceil_div(a->n_in, 32);
    p.rows = (int)a->rows; p.n_in = a->n_in; p.n_out = a->n_out;
    p.BN = pl.BN; p.m_tiles = pl.m_tiles; p.tiles = pl.tiles; p.steps = pl.steps; p.whole = pl.whole; p.splits = pl.splits; p.per = pl.per; p.stages = pl.stages;
    p.out = a->dw;
    p.drop = drop;
    p.partial = (float*)a->workspace;
    auto* kernel = a->x.format == ALEXNET_CODES_INT8 ? (pl.cg == 2 ? linear_grad_kernel<kSrcInt8, 2> : linear_grad_kernel<kSrcInt8, 1>)
                                                     : (pl.cg == 2 ? linear_grad_kernel<kSrcE4m3, 2> : linear_grad_kernel<kSrcE4m3, 1>);
    if (go.e == cudaSuccess) go.e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
    go.smem = pl.smem;
    go.cluster = pl.cg;
    const long long rest = pl.tiles - pl.whole;
    go(kernel, pl.cg * std::min<long long>(kSms / pl.cg, pl.whole + rest * pl.splits), kLgThreads, p);
    if (rest) {      // four columns at a time where there are enough tiles to fill the device so
        const int rows = 128 * pl.cg, at_once = 1024 / rows;
        const bool four = rest * (pl.BN / (4 * at_once)) >= kSms;
        go(four ? linear_grad_join_kernel<4> : linear_grad_join_kernel<1>, rest * ceil_div(pl.BN, (four ? 4 : 1) * at_once), 256, (const float*)p.partial, p.out, p.n_in, p.n_out, p.m_tiles, p.whole,
           (int)rest, p.splits, p.BN, rows);
    }
    return go.e == cudaSuccess ? ALEXNET_OK : err.cuda(go.e);
}
}  // namespace

extern "C" {

int alexnet_checkpoint_encode(const alexnet_checkpoint_args_t* args, void* stream, char* err, size_t err_len) {
    return checkpoint_call(args, (cudaStream_t)stream, {err, err_len, "checkpoint_encode"}, true);
}
int alexnet_checkpoint_decode(const alexnet_checkpoint_args_t* args, void* stream, char* err, size_t err_len) {
    return checkpoint_call(args, (cudaStream_t)stream, {err, err_len, "checkpoint_decode"}, false);
}

size_t alexnet_group_norm_workspace_bytes(const alexnet_group_norm_t* s, int backward) {
    if (!s || check_shape(*s)) return 0;
    const Dims d{s->n, s->h, s->w, s->channels};
    // by sizes alone, so for any alignment, and for x in either form
    size_t bytes = 0;
    for (int kept = 0; kept <= (backward ? 1 : 0); ++kept) {
        if (d.C % 8 == 0) bytes = std::max(bytes, backward ? backward_ws<8>(d, s->groups, s->dtype, kept) : forward_ws<8>(d, s->groups, s->dtype));
        bytes = std::max(bytes, backward ? backward_ws<1>(d, s->groups, s->dtype, kept) : forward_ws<1>(d, s->groups, s->dtype));
    }
    return reported(bytes);
}

size_t alexnet_group_norm_forward_workspace_bytes(const alexnet_group_norm_forward_t* a) {
    if (!a || check_shape(a->shape)) return 0;
    const alexnet_group_norm_t& s = a->shape;
    const Dims d{s.n, s.h, s.w, s.channels};
    return reported(forward_in_vectors(*a, d) ? forward_ws<8>(d, s.groups, s.dtype) : forward_ws<1>(d, s.groups, s.dtype));
}
size_t alexnet_group_norm_backward_workspace_bytes(const alexnet_group_norm_backward_t* a) {
    if (!a || check_shape(a->shape)) return 0;
    const alexnet_group_norm_t& s = a->shape;
    const Dims d{s.n, s.h, s.w, s.channels};
    const bool kept = a->kept.codes || a->kept.scales;
    return reported(backward_in_vectors(*a, d) ? backward_ws<8>(d, s.groups, s.dtype, kept) : backward_ws<1>(d, s.groups, s.dtype, kept));
}

int alexnet_group_norm_forward(const alexnet_group_norm_forward_t* a, void* stream, char* err_buf, size_t err_len) {
    const Err err{err_buf, err_len, "group_norm_forward"};
    if (!a) return err.arg("NULL arguments");
    const alexnet_group_norm_t& s = a->shape;
    const Dims d{s.n, s.h, s.w, s.channels};
    if (const char* m = check_shape(s)) return err.arg(m);
    if (const char* m = check_view(a->x, d, s.dtype, false)) return err.arg(m);
    if (const char* m = check_view(a->y, d, s.dtype, true)) return err.arg(m);
    for (const alexnet_checkpoint_t* k : {&a->keep_x, &a->keep_y})
        if (k->codes || k->scales)
            if (const char* m = check_codes(*k, d)) return err.arg(m);
    if (d.n == 0) return ALEXNET_OK;
    if (!a->mean || !a->rstd) return err.arg("NULL pointer");
    if (a->x.data == a->y.data) return err.arg("y must not share memory with x");
    if (grid_of(walk_of(d, 1, kElementwise), d) > kMaxGrid) return err.arg("the tensor is too large");
    const bool vec = forward_in_vectors(*a, d);
    const size_t need = vec ? forward_ws<8>(d, s.groups, s.dtype) : forward_ws<1>(d, s.groups, s.dtype);
    if (need && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < need)) return err.arg("the workspace is too small or not 16-byte aligned");
    Launcher go{(cudaStream_t)stream};
    switch (s.dtype) {
    case ALEXNET_DTYPE_BF16: vec ? forward<bf16, 8>(go, a, d) : forward<bf16, 1>(go, a, d); break;
    case ALEXNET_DTYPE_F16: vec ? forward<__half, 8>(go, a, d) : forward<__half, 1>(go, a, d); break;
    default: vec ? forward<float, 8>(go, a, d) : forward<float, 1>(go, a, d); break;
    }
    return go.e == cudaSuccess ? ALEXNET_OK : err.cuda(go.e);
}

int alexnet_group_norm_backward(const alexnet_group_norm_backward_t* a, void* stream, char* err_buf, size_t err_len) {
    const Err err{err_buf, err_len, "group_norm_backward"};
    if (!a) return err.arg("NULL arguments");
    const alexnet_group_norm_t& s = a->shape;
    const Dims d{s.n, s.h, s.w, s.channels};
    if (const char* m = check_shape(s)) return err.arg(m);
    const bool kept = a->kept.codes || a->kept.scales;
    if (kept && a->x.data) return err.arg("x is given twice, as a tensor and as a checkpoint");
    if (const char* m = kept ? check_codes(a->kept, d) : check_view(a->x, d, s.dtype, false)) return err.arg(m);
    if (const char* m = check_view(a->dy, d, s.dtype, false)) return err.arg(m);
    if (const char* m = check_view(a->dx, d, s.dtype, true)) return err.arg(m);
    if (d.n == 0) {          // no samples: the parameters' gradients are empty sums
        cudaError_t e = cudaSuccess;
        for (float* p : {a->dweight, a->dbias})
            if (p && e == cudaSuccess) e = cudaMemsetAsync(p, 0, (size_t)d.C * sizeof(float), (cudaStream_t)stream);
        return e == cudaSuccess ? ALEXNET_OK : err.cuda(e);
    }
    if (!a->mean || !a->rstd) return err.arg("NULL pointer");
    if (a->dx.data == a->x.data || a->dx.data == a->dy.data) return err.arg("dx must not share memory with x or dy");
    if (grid_of(walk_of(d, 1, kElementwise), d) > kMaxGrid) return err.arg("the tensor is too large");
    const bool vec = backward_in_vectors(*a, d);
    const size_t need = vec ? backward_ws<8>(d, s.groups, s.dtype, kept) : backward_ws<1>(d, s.groups, s.dtype, kept);
    if (need && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < need)) return err.arg("the workspace is too small or not 16-byte aligned");
    Launcher go{(cudaStream_t)stream};
    switch (s.dtype) {
    case ALEXNET_DTYPE_BF16: vec ? backward<bf16, 8>(go, a, d) : backward<bf16, 1>(go, a, d); break;
    case ALEXNET_DTYPE_F16: vec ? backward<__half, 8>(go, a, d) : backward<__half, 1>(go, a, d); break;
    default: vec ? backward<float, 8>(go, a, d) : backward<float, 1>(go, a, d); break;
    }
    return go.e == cudaSuccess ? ALEXNET_OK : err.cuda(go.e);
}

size_t alexnet_linear_weight_grad_workspace_bytes(const alexnet_linear_weight_grad_t* a) {
    if (!a || check_linear(*a)) return 0;
    const size_t bytes = linear_plan(*a).bytes;
    return bytes ? bytes + 256 : 256;
}

int alexnet_linear_weight_grad(const alexnet_linear_weight_grad_t* args, void* stream, char* err, size_t err_len) {
    return linear_call(args, (cudaStream_t)stream, {err, err_len, "linear_weight_grad"}, -1);
}
int alexnet_operators_debug_expire_wait(const alexnet_linear_weight_grad_t* args, int block, void* stream, char* err, size_t err_len) {
    const Err e{err, err_len, "operators_debug_expire_wait"};
    if (block < 0 || block > 1) return e.arg("block must be 0 or 1");
    return linear_call(args, (cudaStream_t)stream, e, block);
}

int alexnet_operators_check(void) {
    int expired = 0;
    // (torch's streams, like all non-blocking ones, do not wait for the default stream's copy, nor it for them)
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&expired, g_expired, sizeof(int)) != cudaSuccess) { cudaGetLastError(); return ALEXNET_ERR_CUDA; }
    return expired ? ALEXNET_ERR_DEVICE_TIMEOUT : ALEXNET_OK;
}

}  // extern "C"
