// Weight gradient of a linear layer whose input was kept as an 8-bit checkpoint: dw[o][i] = sum_r dy[r][o] x[r][i].
//
// A GEMM whose reduction runs over the rows of both operands, so both reach the tensor cores MN-major, 64 rows at a time.  dy comes by
// TMA; the codes of x are read to registers, decoded there (exact in bf16: seven significant bits times a power of two) and written to
// the same swizzled tile that TMA would write, so x is never in memory as bf16: its traffic is a byte per value.
//
// The tile is 128 input features (rows of the accumulator) by BN output features: the decoded side is the narrow one, as each CTA decodes
// its own tile of x again for every BN outputs.  An accumulator column then is 32 consecutive inputs of one output for each warp, which
// leaves as one full 128-byte line.
//
// Warps: 0 = TMA producer (dy), 1 = MMA issuer and TMEM owner, 2..9 = epilogue (two sets of four), 10..25 = decoders, four groups
// that take the steps in turn (a step takes a warp over 1000 cycles from its wait to its arrival, and the tensor cores 512).  Persistent
// over tiles with two accumulators, so a tile's stores overlap the next one's products.  Where the tiles do not fill the last round of CTAs
// (or any), those of that round are split over the rows; a second kernel adds their partial sums in a fixed order.  Every wait is
// bounded; a CTA whose wait runs out writes NaN from there on and raises g_expired.  It arrives on no barrier any more, so that the other CTA of a pair comes to
// the same end instead of working on tiles and sums that are not there.
//
// Measured: 8192 rows, 4096 x 4096: 225 us, 1220 TFLOP/s; the library's product alone, with x in bf16 already, 181 us, and the decoding and
// writing of x before it another 25.  128 rows, 9216 x 4096: 29.5 us, 5.2 TB/s, all but 11 % of them the fp32 stores of dw.  173 rows, 4096 x 1000:
// 7.5 us, of which the first loads, one chain of steps and the stores are the most: a latency.  Long products are bound by the shared memory
// (the decoded tile's stores and the operands' reads), then by the power limit; short ones by the stores of dw.
#pragma once
#include "checkpoint.cuh"

namespace op {

constexpr int kLgRows = 64, kLgEpilogue = 8, kLgDecoders = 4, kLgGroups = 4;      // decoder warps of a step; groups of them
constexpr int kLgThreads = 32 * (2 + kLgEpilogue + kLgGroups * kLgDecoders);
constexpr int kLgShare = kLgRows * 4 / (32 * kLgDecoders);     // checkpoint blocks of a step that a decoder takes: rows 8 kLgDecoders apart
constexpr int kLgA = 128 * kLgRows * 2;            // bytes of the decoded tile of a stage: two boxes of 64 features x 64 rows
constexpr int kLgMaxStages = 6;
// Steps whose products one accumulator takes up.  The tensor cores cut their running sums off instead of rounding them, so an error grows with
// every row (2.2e-10 of the result per row: 1.8e-6 after 8192, where an fp32 product with rounded sums has 2.4e-7): after 2048 rows the sums are
// added, rounded, to those before.
constexpr int kLgChunk = 32;
struct LinearGradParams {
    CUtensorMap tmD;                               // dy [rows][n_out], boxes of 64 features x 64 rows
    const uint8_t *codes, *scales;
    long long code_pitch;                          // bytes; a multiple of 16
    int blocks;                                    // scales per row
    int rows, n_in, n_out;
    int BN, m_tiles, tiles, steps;                 // steps of 64 rows
    int whole, splits, per;                        // the first `whole` tiles take all rows; each of the others is `splits` units of `per` steps
    int stages;
    float* out;
    float* partial;                                // sums of the split tiles: [split][tile - whole][BN][128 CG]
    int drop;                                      // self-test: the CTA whose decoders leave out their first arrival, or -1
};
__device__ int g_expired;

// A unit of work, in the order in which the CTAs take them: the whole tiles (input tile fastest), then the split ones, split by split.
struct LinearGradTile {
    int m, n, k0, k1, part;                        // part: index of the unit's partial sums, or -1
    __device__ __forceinline__ void set(const LinearGradParams& p, int unit) {
        int tile = unit, z = 0;
        part = -1;
        if (unit >= p.whole) {
            const int rest = p.tiles - p.whole;
            z = (unit - p.whole) / rest;
            tile = unit - z * rest;
            if (p.splits > 1) part = unit - p.whole;
        }
        m = tile % p.m_tiles;
        n = tile / p.m_tiles;
        k0 = z * p.per;
        k1 = part < 0 ? p.steps : min(p.steps, k0 + p.per);
    }
};
struct LinearGradCodes { uint4 c[2]; uint32_t e; };      // a checkpoint block of one row

// Sixteen codes to bf16 pairs, s2 = the scale twice.  int8: the code + 128 as the low byte of 2^23 + that, times the scale, less (2^23 + 128)
// times the scale, in one multiply-add: exact, unless the product passes fp32's range (exponents that only magnitudes above 2^109 have).
template <int FMT, bool FUSED>
__device__ __forceinline__ void decode16(const uint4& c, f2 s2, f2 o2, uint32_t* w) {
    if constexpr (FUSED) {
        const uint32_t* u = (const uint32_t*)&c;
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t t = u[i] ^ 0x80808080u;
            #pragma unroll
            for (int q = 0; q < 2; ++q) {
                float lo, hi;
                un2(fma2(mk2(__uint_as_float(__byte_perm(t, 0x4b000000u, 0x7440u | 2 * q)), __uint_as_float(__byte_perm(t, 0x4b000000u, 0x7441u | 2 * q))), s2, o2), lo, hi);
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[2 * i + q]) : "f"(hi), "f"(lo));
            }
        }
    } else {
        float v[16];
        code_values<FMT, 16>(c, v);
        #pragma unroll
        for (int q = 0; q < 8; ++q) {
            float lo, hi;
            un2(mul2(mk2(v[2 * q], v[2 * q + 1]), s2), lo, hi);
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[q]) : "f"(hi), "f"(lo));
        }
    }
}
// a block of 32 codes into its place in the stage: addr = row k of a box, the block's chunks 4 b .. 4 b + 3 (b = 0, 1), swizzled by k
template <int FMT, bool FUSED>
__device__ __forceinline__ void decode_block(const LinearGradCodes& r, uint32_t addr, uint32_t swz) {
    const float sc = scale_of(r.e), off = -8388736.f * sc;
    const f2 s2 = mk2(sc, sc), o2 = mk2(off, off);
    #pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t w[8];
        decode16<FMT, FUSED>(r.c[h], s2, o2, w);
        tc::st_shared_v4(addr + (swz ^ (uint32_t)(32 * h)), w[0], w[1], w[2], w[3]);
        tc::st_shared_v4(addr + (swz ^ (uint32_t)(32 * h + 16)), w[4], w[5], w[6], w[7]);
    }
}

// CG = 2: CTA pairs.  The two CTAs (cluster of two) share a tile of 256 inputs: each decodes its own 128 and loads half of the BN columns of dy;
// the leader's instructions cover both, so a CTA's shared memory takes half the traffic of dy.
template <int FMT, int CG>
__global__ void __launch_bounds__(kLgThreads, 1) linear_grad_kernel(const __grid_constant__ LinearGradParams p) {
    kn::pdl_trigger();
    if (CG == 2) tc::cluster_arrive();                 // (this CTA runs)
    const int rank = CG == 2 ? (int)tc::cluster_ctarank() : 0;
    const int tile0 = (int)blockIdx.x / CG, tile_step = (int)gridDim.x / CG;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = tc::smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    const int nb = (p.BN / CG + 63) >> 6, stages = p.stages;
    const uint32_t stage_bytes = kLgA + (uint32_t)nb * 8192u;
    // barriers behind the stages: full[8] @0, empty[8] @64, acc_full[2] @128, acc_empty[2] @144, tmem slot @160, abort flag @168
    const uint32_t bar = base + stages * stage_bytes;
    uint8_t* gen = smem_raw + (bar - raw);
    volatile int* abort_flag = (volatile int*)(gen + 168);
    volatile uint32_t* tmem_slot = (volatile uint32_t*)(gen + 160);
    const uint32_t full0 = bar, empty0 = bar + 64u, accf0 = bar + 128u, acce0 = bar + 144u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tiles = p.whole + (p.tiles - p.whole) * p.splits;      // units
    uint32_t ncols = 32;
    while ((int)ncols < 2 * p.BN) ncols <<= 1;

    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int s = 0; s < stages; ++s) { tc::mbar_init(full0 + 8u * s, 1 + CG * kLgDecoders); tc::mbar_init(empty0 + 8u * s, 1); }
        for (int s = 0; s < 2; ++s) { tc::mbar_init(accf0 + 8u * s, 1); tc::mbar_init(acce0 + 8u * s, CG * kLgEpilogue); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        tc::tma_prefetch_desc(&p.tmD);
    }
    __syncwarp();
    if (CG == 2) tc::cluster_wait();                   // the peer runs
    if (warp == 1) {
        if (CG == 2) tc::tmem_alloc_pair(tc::smem_u32((const void*)tmem_slot), ncols);
        else tc::tmem_alloc(tc::smem_u32((const void*)tmem_slot), ncols);
    }
    tc::tc_fence_before();
    __syncthreads();
    __syncwarp();
    if (CG == 2) tc::cluster_arrive();
    kn::pdl_wait();
    if (CG == 2) {
        tc::cluster_wait();                            // the peer has its tensor memory, and its barriers exist before anything arrives on them
        if (warp == 1) tc::tmem_relinquish_pair();
    }
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        if (lane == 0) {
            int st = 0; uint32_t ph = 0;
            bool ok = true;
            LinearGradTile t;
            for (int tile = tile0; tile < tiles && ok; tile += tile_step) {
                t.set(p, tile);
                for (int k = t.k0; k < t.k1; ++k) {
                    if (!(ok = tc::mbar_wait(empty0 + 8u * st, ph ^ 1u, abort_flag))) break;
                    const uint32_t sb = base + st * stage_bytes + kLgA, fb = full0 + 8u * st;
                    if (rank == 0) tc::mbar_expect_tx(fb, (uint32_t)(CG * nb) * 8192u);
                    const int col = t.n * p.BN + rank * (p.BN / CG);
                    for (int j = 0; j < nb; ++j) {
                        if (CG == 2) tc::tma_load_2d_pair(sb + j * 8192, &p.tmD, col + 64 * j, k * kLgRows, tc::mapa_u32(fb, 0));
                        else tc::tma_load_2d(sb + j * 8192, &p.tmD, col + 64 * j, k * kLgRows, fb);
                    }
                    if (++st == stages) { st = 0; ph ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
        // A unit's first chunk goes to accumulator `ab`, the others to the other one, whence the epilogue adds them to the first; the next unit's
        // first chunk goes to that other one, while the epilogue stores this unit's result.  fill: bit a is the parity of accumulator a's next use.
        const uint32_t idesc = tc::instr_desc(p.BN, 1, 1, 128 * CG);
        int st = 0; uint32_t ph = 0;
        int ab = 0; uint32_t fill = 0;
        bool ok = true;
        LinearGradTile t;
        for (int tile = tile0; tile < tiles && ok; tile += tile_step, ab ^= 1) {
            t.set(p, tile);
            for (int c0 = t.k0; c0 < t.k1 && ok; c0 += kLgChunk) {
                const int a = c0 == t.k0 ? ab : ab ^ 1, c1 = min(t.k1, c0 + kLgChunk);
                if (!(ok = tc::mbar_wait_warp(acce0 + 8u * a, (fill >> a & 1u) ^ 1u, abort_flag))) break;
                if (CG == 2) tc::fence_acq_rel_cluster();  // the peer's epilogue arrived from the other CTA
                tc::tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(a * p.BN);
                for (int k = c0; k < c1; ++k) {
                    if (!(ok = CG == 2 ? tc::mbar_wait_warp_cluster(full0 + 8u * st, ph, abort_flag) : tc::mbar_wait_warp(full0 + 8u * st, ph, abort_flag))) break;
                    tc::tc_fence_after();
                    const uint32_t sa = base + st * stage_bytes, sb = sa + kLgA;
                    #pragma unroll
                    for (int j = 0; j < 4; ++j)
                        tc::umma_cg<CG>(d, tc::smem_desc(sa + j * 2048, 8192, 1024), tc::smem_desc(sb + j * 2048, 8192, 1024), idesc, (k > c0 || j > 0) ? 1u : 0u);
                    tc::umma_commit_cg<CG>(empty0 + 8u * st);
                    if (++st == stages) { st = 0; ph ^= 1u; }
                }
                if (!ok) break;
                tc::umma_commit_cg<CG>(accf0 + 8u * a);
                fill ^= 1u << a;
            }
        }
        }
    } else if (warp < 2 + kLgEpilogue) {
        const int quad = warp & 3, set = (warp - 2) >> 2;
        int ab = 0; uint32_t fill = 0;
        bool ok = true;
        LinearGradTile t;
        auto filled = [&](int a) {                     // the accumulator's current use is complete
            ok = ok && tc::mbar_wait_idle(accf0 + 8u * a, fill >> a & 1u, abort_flag);
            fill ^= 1u << a;
            tc::tc_fence_after();
        };
        auto release = [&](int a) {
            tc::tc_fence_before();
            __syncwarp();
            if (ok && lane == 0) {
                if (CG == 2) tc::mbar_arrive_cluster(tc::mapa_u32(acce0 + 8u * a, 0));
                else tc::mbar_arrive(acce0 + 8u * a);
            }
        };
        for (int tile = tile0; tile < tiles; tile += tile_step, ab ^= 1) {
            t.set(p, tile);
            const int i = (t.m * CG + rank) * 128 + quad * 32 + lane, o0 = t.n * p.BN, nv = min(p.BN, p.n_out - o0);
            const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16), ta = lanes + (uint32_t)(ab * p.BN), tb = lanes + (uint32_t)((ab ^ 1) * p.BN);
            for (int c0 = t.k0 + kLgChunk; c0 < t.k1; c0 += kLgChunk) {
                filled(ab ^ 1);                        // (the first chunk's products are complete as well: they were issued before)
                if (ok) {
                    #pragma unroll 1
                    for (int c = 32 * set; c < nv; c += c & 16 ? 48 : 16) {  // the columns that this warp stores below
                        uint32_t u[16], v[16];
                        tc::tmem_ld16(ta + (uint32_t)c, u);
                        tc::tmem_ld16(tb + (uint32_t)c, v);
                        tc::tmem_ld_wait();
                        #pragma unroll
                        for (int q = 0; q < 16; ++q) u[q] = __float_as_uint(__uint_as_float(u[q]) + __uint_as_float(v[q]));
                        tc::tmem_st16(ta + (uint32_t)c, u);
                    }
                    tc::tmem_st_wait();
                }
                release(ab ^ 1);
            }
            filled(ab);
            // dw[o][i], or the unit's partial sums [column][input]
            const bool part = t.part >= 0, mine = part || i < p.n_in;
            const long long pitch = part ? 128 * CG : p.n_in;
            float* out = part ? p.partial + ((long long)t.part * p.BN + 32 * set) * (128 * CG) + rank * 128 + quad * 32 + lane : p.out + (long long)(o0 + 32 * set) * p.n_in + i;
            #pragma unroll 1
            for (int c = 32 * set; c < nv; c += 64, out += 64 * pitch) {
                uint32_t v[32];
                if (ok) { tc::tmem_ld32(ta + (uint32_t)c, v); tc::tmem_ld_wait(); }
                else {
                    #pragma unroll
                    for (int q = 0; q < 32; ++q) v[q] = 0x7fffffffu;
                }
                if (mine) {
                    float* o = out;
                    if (c + 32 <= nv) {
                        #pragma unroll
                        for (int q = 0; q < 32; ++q) { *o = __uint_as_float(v[q]); o += pitch; }
                    } else {
                        #pragma unroll
                        for (int q = 0; q < 32; ++q) { if (c + q < nv) *o = __uint_as_float(v[q]); o += pitch; }
                    }
                }
            }
            release(ab);
        }
    } else {
        // thread: checkpoint block cb (32 codes) of row kr of a step.  With the 128-byte swizzle, 16-byte chunk j of row k lies at j ^ (k & 7);
        // the threads of the second box take rows two apart from those of the first, so that eight neighbouring lanes (four blocks, two
        // rows) write to eight different bank groups.
        const int group = (warp - 2 - kLgEpilogue) / kLgDecoders, td = (threadIdx.x - 32 * (2 + kLgEpilogue)) % (32 * kLgDecoders);
        const int cb = td & 3, kr = (td >> 2) ^ (cb & 2);
        LinearGradCodes f[kLgShare];           // of the group's next step: in flight while the other groups decode theirs
        int total = 0, tile = tile0, left = 0, row = 0;
        LinearGradTile t;
        for (int k = tile0; k < tiles; k += tile_step) { t.set(p, k); total += t.k1 - t.k0; }
        const uint8_t *cp = nullptr, *ep = nullptr;
        int halves = 0;                        // of the block's two halves of 16 codes, how many there are in memory
        auto enter = [&] {                     // the next tile whose codes are to be loaded
            t.set(p, tile);
            tile += tile_step;
            left = t.k1 - t.k0;
            row = t.k0 * kLgRows + kr;
            const int col = (t.m * CG + rank) * 128 + cb * 32;
            halves = col >= p.n_in ? 0 : col + 16 < p.n_in ? 2 : 1;
            cp = p.codes + row * p.code_pitch + col;
            ep = p.scales + (long long)row * p.blocks + (col >> 5);
        };
        const long long step_c = kLgRows * p.code_pitch, step_e = (long long)kLgRows * p.blocks;
        auto forward = [&](int steps) {
            while (steps >= left && tile < tiles) { steps -= left; enter(); }
            left -= steps;
            row += steps * kLgRows;
            cp += steps * step_c;
            ep += steps * step_e;
        };
        enter();
        int to_load = total - group;
        if (to_load > 0) forward(group);
        auto load = [&] {
            #pragma unroll
            for (int u = 0; u < kLgShare; ++u) {
                LinearGradCodes& r = f[u];
                const bool in = row + 8 * kLgDecoders * u < p.rows;
                const uint8_t *c = cp + u * (step_c / kLgShare), *e = ep + u * (step_e / kLgShare);
                r.c[0] = in && halves > 0 ? __ldg((const uint4*)c) : make_uint4(0u, 0u, 0u, 0u);
                r.c[1] = in && halves > 1 ? __ldg((const uint4*)c + 1) : make_uint4(0u, 0u, 0u, 0u);
                r.e = in && halves > 0 ? __ldg(e) : 0u;
            }
            to_load -= kLgGroups;
            if (to_load > 0) forward(kLgGroups);
        };
        if (to_load > 0) load();
        const uint32_t off = (uint32_t)(cb >> 1) * 8192u + (uint32_t)kr * 128u, swz = (uint32_t)((4 * (cb & 1)) ^ (kr & 7)) << 4;
        int st = group; uint32_t ph = 0;
        for (int s = group; s < total; s += kLgGroups) {
            while (st >= stages) { st -= stages; ph ^= 1u; }
            if (!tc::mbar_wait_idle(empty0 + 8u * st, ph ^ 1u, abort_flag)) break;
            const uint32_t addr = base + st * stage_bytes + off;
            bool small = true;
            #pragma unroll
            for (int u = 0; u < kLgShare; ++u) small = small && f[u].e < 230u;
            if (FMT == kSrcInt8 && __all_sync(~0u, small)) {
                #pragma unroll
                for (int u = 0; u < kLgShare; ++u) decode_block<FMT, FMT == kSrcInt8>(f[u], addr + 1024u * kLgDecoders * u, swz);
            } else {
                #pragma unroll
                for (int u = 0; u < kLgShare; ++u) decode_block<FMT, false>(f[u], addr + 1024u * kLgDecoders * u, swz);
            }
            tc::fence_async_smem();
            __syncwarp();
            if (lane == 0 && (s > 0 || (int)blockIdx.x != p.drop)) {
                if (CG == 2) tc::mbar_arrive_remote(tc::mapa_u32(full0 + 8u * st, 0));
                else tc::mbar_arrive(full0 + 8u * st);
            }
            st += kLgGroups;
            if (to_load > 0) load();
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    if (*abort_flag) {                              // copies in flight land before the shared memory is given back
        if (threadIdx.x == 0) atomicExch(&g_expired, 1);
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000LL) { }
        __syncthreads();
    }
    __syncwarp();
    if (CG == 2) tc::cluster_sync_all();               // no CTA leaves while its peer may still arrive on its barriers
    if (warp == 1) {
        tc::tc_fence_after();
        if (CG == 2) tc::tmem_dealloc_pair(tmem, ncols);
        else tc::tmem_dealloc(tmem, ncols);
    }
    if (CG == 2) { __syncwarp(); tc::cluster_sync_all(); }      // nor before both have deallocated
}

// dw of the split tiles: the sums of their splits, added in that order.  A thread takes four inputs of a column and J columns in turn, with the loads of
// eight partial sums in flight; bound by their way from L2.  (One value per thread: 36 us for the 18 MB of 34 tiles of 256 x 256 in two
// splits, four times as long: the blocks' set-up.)
template <int J>
__global__ void __launch_bounds__(256) linear_grad_join_kernel(const float* __restrict__ partial, float* __restrict__ dw, int n_in, int n_out, int m_tiles, int whole, int rest, int splits, int BN,
                                                               int rows /* 128 CG */) {
    kn::pdl_sync();
    const int lanes = rows / 4, at_once = 256 / lanes, blocks = (BN + J * at_once - 1) / (J * at_once);
    const int t = blockIdx.x / blocks, tile = whole + t, n = tile / m_tiles, m = tile - n * m_tiles;
    const int c0 = (blockIdx.x - t * blocks) * J * at_once + threadIdx.x / lanes, r = threadIdx.x % lanes * 4, i = m * rows + r;
    if (i >= n_in) return;
    const long long stride = (long long)rest * BN * rows;
    const float* src = partial + (long long)t * BN * rows + r;
    constexpr int Z = 8 / J;                           // splits whose sums are in flight
    float4 s[J];
    #pragma unroll
    for (int j = 0; j < J; ++j) s[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int z0 = 0; z0 < splits; z0 += Z) {
        float4 v[Z][J];
        #pragma unroll
        for (int q = 0; q < Z; ++q)
            #pragma unroll
            for (int j = 0; j < J; ++j) {
                const int c = c0 + j * at_once;
                v[q][j] = z0 + q < splits && c < BN ? __ldcg((const float4*)(src + (z0 + q) * stride + (long long)c * rows)) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
        #pragma unroll
        for (int q = 0; q < Z; ++q)
            #pragma unroll
            for (int j = 0; j < J; ++j) { s[j].x += v[q][j].x; s[j].y += v[q][j].y; s[j].z += v[q][j].z; s[j].w += v[q][j].w; }
    }
    const bool vec = n_in % 4 == 0 && ((uintptr_t)dw & 15) == 0;
    #pragma unroll
    for (int j = 0; j < J; ++j) {
        const int c = c0 + j * at_once, o = n * BN + c;
        if (c >= BN || o >= n_out) continue;
        float* d = dw + (long long)o * n_in + i;
        if (vec) *(float4*)d = s[j];
        else {
            d[0] = s[j].x;
            if (i + 1 < n_in) d[1] = s[j].y;
            if (i + 2 < n_in) d[2] = s[j].z;
            if (i + 3 < n_in) d[3] = s[j].w;
        }
    }
}

// Rows of `bytes` bytes (a multiple of UNIT), `src_pitch` apart, to rows `pitch` apart that start on 16-byte boundaries, zeros behind them: for
// operands whose rows the copies above cannot read in place.  One thread per 16 bytes.
template <typename UNIT>
__global__ void __launch_bounds__(256) repitch_kernel(const uint8_t* __restrict__ src, long long src_pitch, int bytes, long long pitch, long long rows, uint8_t* __restrict__ dst) {
    kn::pdl_sync();
    const int per_row = (int)(pitch / 16);
    const long long total = rows * per_row;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < total; t += (long long)gridDim.x * 256) {
        const long long r = t / per_row;
        const int b0 = (int)(t - r * per_row) * 16;
        const UNIT* s = (const UNIT*)(src + r * src_pitch + b0);
        UNIT v[16 / sizeof(UNIT)];
        #pragma unroll
        for (int i = 0; i < (int)(16 / sizeof(UNIT)); ++i) v[i] = b0 + i * (int)sizeof(UNIT) < bytes ? s[i] : UNIT(0);
        *(uint4*)(dst + r * pitch + b0) = *(const uint4*)v;
    }
}

}  // namespace op
