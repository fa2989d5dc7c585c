// The FC on the rows of a prompt: y = act(x W + b) + r for any number of rows, on the 5th-generation tensor cores.
//
// The library's other FC kernels take up to 16 rows, where the weights are the only traffic that counts.  With the rows of a prompt
// the product itself is the work, so this is a matrix product: x[M,K] and W[K,N] are both moved by TMA (128-byte swizzle), W exactly
// as it lies in memory, and the accumulators live in TMEM.
//
// The weight tile is the M operand of the MMA (128 output channels, MN-major), the rows of x are its N operand (BN of them,
// K-major).  So an accumulator lane is one output channel and its columns are rows of y: a warp of the epilogue holds 32 consecutive
// channels of a row, which it can read (residual) and write in one contiguous piece without a turn through shared memory, and the bias of a
// lane is one register.  It also makes BN, the rows per tile, a free number in steps of 16 from a single row up.
//
//   warps 0-7  epilogue: accumulators to registers, bias, activation, residual, rounding, store.  Two accumulators in TMEM, so
//              the MMAs of the next tile run meanwhile
//   warp 8     boxes: per block of 128 channels two of W (64 columns x 128 channels) and two of x (64 channels x BN rows)
//   warp 9     MMAs
//
// Two forms, one source:
//   CG = 2  two CTAs of a cluster share a tile of 256 channels x BN rows (tcgen05 cta_group::2): each loads its own 128 channels
//           of W and half of the rows, the MMA of the pair reads both, so a row of x crosses from L2 once per pair.  For many rows.
//   CG = 1  one CTA, 128 channels x BN rows; where the tiles are too few for the device, a cluster of S CTAs splits the
//           channels (K) and adds its S partial tiles through distributed shared memory, in rank order.  For few rows.
// Accumulation in fp32 (TMEM), one rounding at the end to the type of y.  No atomics: the same bits each time.
//
// Every wait is bounded: one that runs out sets the status word, the CTA stops issuing work, waits for the copies and MMAs
// under way, and frees its TMEM.
#include <math.h>
#include <string.h>

#include <atomic>
#include <type_traits>

#include "scap_tc.cuh"

namespace scap {

constexpr int FA_EPI_WARPS = 8;
constexpr int FA_THREADS = (FA_EPI_WARPS + 2) * 32;
constexpr int FA_BK = 128;                   // channels per stage: eight MMAs per round of waits (64: the issuing lanes fall behind the tensor core)
constexpr int FA_TN = 128;                   // output channels per CTA
constexpr int FA_ABYTES = FA_TN * FA_BK * 2; // 32 KB of W per stage
// The tensor core truncates where it adds to an accumulator, always towards zero, so a sum is off by about 2^-25 of itself per addition: 3e-6
// at K = 2560, nothing beside a rounding to 16 bits but much beside one to fp32, and 2e-4 at K = 2^18.  For an fp32 result, and where a sum over all channels would be
// off by more than an eighth of half a step of the 16-bit result (fa_long), an accumulator takes 512 channels (32
// additions) and the epilogue warps add those sums up in registers, rounding to nearest, while the next 512 are under way.
constexpr int FA_CHUNK = 4;
constexpr int FA_MAX_BN_CHUNKED = 192;       // rows per tile then: the sums of half of them are a thread's registers
// K / 16 additions of 2^-25: an eighth of 2^-12 for fp16, of 2^-9 for bf16.
static bool fa_long(int K, bool bf16) { return K > (bf16 ? 131072 : 16384); }
constexpr int FA_MAX_STAGES = 12;
constexpr int FA_SMEM = 226 * 1024;          // of the 227 KB that a CTA may have; the barriers are inside

struct FaArgs {
    const float *b;
    const void *r;
    void *y;
    long long ldr, ldy;
    int M, K, N;
    int act;
    int BN, stages, S;
    int tiles_n, tiles_m, groups;  // groups: row tiles that are walked together, for reuse in L2
    uint32_t tmem_cols;
    uint32_t limit;
    int *status;
};

struct FaShared {
    unsigned long long full[FA_MAX_STAGES], empty[FA_MAX_STAGES], tfull[2], tempty[2], drain;
    uint32_t tmem_base;
    int abort_flag;
    int sent, peer_sent, peer_abort;  // stages asked for; with CG = 2 also what the other CTA leaves here at the end
};

__device__ __forceinline__ bool fa_wait(uint32_t bar, uint32_t parity, const FaArgs &a, volatile int *abort_flag) {
    for (uint32_t i = 0; i < a.limit; ++i) {
        if (mbarrier_try_wait(bar, parity)) return true;
        if (*abort_flag) return false;
    }
    if (a.status) atomicCAS(a.status, 0, 40);
    *abort_flag = 1;
    return false;
}

__device__ __forceinline__ bool fa_elect() {
    uint32_t on;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(on));
    return on != 0;
}

template <int CG>
__device__ __forceinline__ void fa_box(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    if constexpr (CG == 2)  // the barrier may be the other CTA's
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

template <int CG>
__device__ __forceinline__ void fa_mma(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t acc) {
    if constexpr (CG == 2)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5, %5, %5, %5, %5}, p;\n\t}\n" ::"r"(d), "l"(da), "l"(db), "r"(idesc),
            "r"(acc), "r"(0u) : "memory");
    else
        tc_mma(d, da, db, idesc, acc);
}

// Arrival on a barrier when the MMAs issued so far are done; with CG = 2 on both CTAs' barriers at this offset.
template <int CG>
__device__ __forceinline__ void fa_commit(uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((unsigned short)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void fa_arrive_cluster(uint32_t addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}

__device__ __forceinline__ void fa_ld16(uint32_t (&v)[16], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
          "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr));
}

__device__ __forceinline__ float fa_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float fa_rcp(float x) {  // 0 of an infinity
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// (1 - erf(u / sqrt 2)) / 2 of u >= 0, as e^(-u^2 / 2) times a polynomial in t = 1 / (1 + p u) whose coefficients are a fit, by reweighted least
// squares, with the smallest relative error over u = 0 .. 14: 1e-7, and 9e-7 with the roundings of the exponential up to u = 4, 3e-6 up to 8.
__device__ __forceinline__ float fa_upper_tail(float u) {
    const float t = fa_rcp(fmaf(u, 0.23334524f, 1.0f));
    float s = -0.0676725209f;
    s = fmaf(s, t, 0.230117321f);
    s = fmaf(s, t, -0.175572917f);
    s = fmaf(s, t, 0.204248384f);
    s = fmaf(s, t, 0.0236110892f);
    s = fmaf(s, t, 0.100611739f);
    s = fmaf(s, t, 0.0914779976f);
    s = fmaf(s, t, 0.0931788981f);
    return s * t * fa_exp2(u * u * -0.72134752f);
}

// Activations of R values, in line, in about 5 to 18 instructions each: sixteen copies have to fit the instruction cache in an epilogue's loop (with
// expf, erfcf and a function call per four values relu took 2.8 us of 13.6 and gelu 8.4 us of 19.2, at 832 x 1280 x 3328).  Off by at most
// (4 z + 16) 2^-24 of themselves, z being the argument of the exponential (u, u^2 / 2, 1.6 u + 0.07 u^3): 2^-20 where it is small, 2^-17 at gelu(-8).
template <int R>
__device__ __forceinline__ void fa_act(float (&u)[R], int act) {
    if (act == SCAP_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < R; ++j) u[j] = u[j] < 0.0f ? 0.0f : u[j];
    } else if (act == SCAP_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < R; ++j) u[j] *= fa_rcp(1.0f + fa_exp2(-1.44269504f * u[j]));
    } else if (act == SCAP_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const float q = fa_upper_tail(fabsf(u[j]));
            u[j] *= u[j] < 0.0f ? q : 1.0f - q;
        }
    } else if (act == SCAP_ACT_GELU_TANH) {  // (1 + tanh a) / 2 = 1 / (1 + e^(-2a))
#pragma unroll
        for (int j = 0; j < R; ++j) u[j] *= fa_rcp(1.0f + fa_exp2(u[j] * fmaf(u[j] * u[j], -0.10294324f, -2.3022082f)));
    }
}

// Elements of y and r: fp32, or 16 bits of the type of x.  A load gives the bits, 0 where it is off (no branch, and nothing that
// waits for them, so that a batch of loads is under way together); fa_widen makes the number of them.
template <bool F32>
__device__ __forceinline__ uint32_t fa_load(const void *p, long long i, bool on) {
    if constexpr (F32) return __float_as_uint(ld_act_if(reinterpret_cast<const float *>(p) + i, on));
    else return ld_act_if_u16(reinterpret_cast<const unsigned short *>(p) + i, on);
}
template <bool BF16, bool F32>
__device__ __forceinline__ float fa_widen(uint32_t u) {
    if constexpr (F32) return __uint_as_float(u);
    else return widen_bits<BF16>((unsigned short)u);
}
template <bool BF16, bool F32>
__device__ __forceinline__ void fa_store(void *p, long long i, float v) {
    if constexpr (F32) reinterpret_cast<float *>(p)[i] = v;
    else if constexpr (BF16) reinterpret_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
    else reinterpret_cast<__half *>(p)[i] = __float2half_rn(v);
}
// Two rows of a lane's channel against one row of a pair of channels: lanes 2i and 2i+1 hold channels c and c+1, each with row a in the lower and
// row a+1 in the upper half.  Lane 2i gets row a, lane 2i+1 row a+1, of both channels.  The same step again undoes it.
__device__ __forceinline__ uint32_t fa_swap(uint32_t v, uint32_t sel) { return __byte_perm(v, __shfl_xor_sync(0xffffffffu, v, 1), sel); }
template <bool BF16>
__device__ __forceinline__ uint32_t fa_pack(float lo, float hi) {
    if constexpr (BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    } else {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
}

// Tile number -> channel tile and row tile.  Row tiles are walked in groups: the tiles that run at the same time then share both
// their rows of x and their columns of W in L2.
__device__ __forceinline__ void fa_tile(const FaArgs &a, int t, int &tn, int &tm) {
    const int per = a.groups * a.tiles_n, g = t / per, in = t - g * per;
    const int rows = min(a.groups, a.tiles_m - g * a.groups);
    tn = in / rows;
    tm = g * a.groups + in - tn * rows;
}

template <bool BF16, int CG, bool F32, bool CHUNKED>
__global__ void __launch_bounds__(FA_THREADS, 1) fc_act_kernel(const FaArgs a, const __grid_constant__ CUtensorMap wmap,
                                                                const __grid_constant__ CUtensorMap xmap) {
    extern __shared__ unsigned char fa_raw[];
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(fa_raw) + 1023) & ~(uintptr_t)1023);
    const int bn_cta = a.BN / CG;                                   // rows of x that this CTA loads
    const uint32_t stage = FA_ABYTES + (uint32_t)bn_cta * FA_BK * 2;
    FaShared *sh = reinterpret_cast<FaShared *>(ring + (size_t)a.stages * stage);
    // (the shuffles tell the compiler that these are the same in the whole warp: addresses and descriptors then stay in uniform registers)
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int clusters = CG == 2 ? (int)gridDim.x / 2 : (int)gridDim.x;  // (CG = 1: one tile per CTA of x; y = K ranks)
    const int rank = CG == 2 ? (int)(blockIdx.x & 1) : 0;
    const int first = CG == 2 ? (int)blockIdx.x / 2 : (int)blockIdx.x;
    const int S = CG == 2 ? 1 : a.S, srank = CG == 2 ? 0 : (int)blockIdx.y;
    const int tiles = a.tiles_n * a.tiles_m;
    const int nkb_all = (a.K + FA_BK - 1) / FA_BK;
    const int kb0 = (int)((long long)nkb_all * srank / S), nkb = (int)((long long)nkb_all * (srank + 1) / S) - kb0;
    const int chunk = CHUNKED ? FA_CHUNK : nkb;  // stages that are added up in one accumulator
    volatile int *abort_flag = &sh->abort_flag;

    if (tid == 0) {
        for (int i = 0; i < a.stages; ++i) {
            mbar_init(&sh->full[i], 1);
            mbar_init(&sh->empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh->tfull[i], 1);
            mbar_init(&sh->tempty[i], FA_EPI_WARPS * CG);
        }
        mbar_init(&sh->drain, 1);
        sh->abort_flag = sh->sent = sh->peer_sent = sh->peer_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == FA_EPI_WARPS + 1) {
        if constexpr (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)), "r"(a.tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)), "r"(a.tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2 || S > 1) { cluster_arrive(); cluster_wait(); }  // the partner's barriers are ready before anything can arrive on them
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh->tmem_base, 0);

    if (warp == FA_EPI_WARPS) {
        // ---- boxes, by one elected lane.  W is a constant of the layer: its first stages are asked for before the work that this call
        // follows has finished.
        if (fa_elect()) {
            const uint32_t ring_at = smem_u32(ring);
            const uint32_t bytes = (uint32_t)CG * stage;
            const uint32_t full0 = CG == 2 ? cluster_addr(smem_u32(&sh->full[0]), 0) : smem_u32(&sh->full[0]);
            const uint32_t empty0 = smem_u32(&sh->empty[0]);
            auto ask_w = [&](int st, int n0, int k0) {
                if (rank == 0) mbar_arrive_expect_tx(&sh->full[st], bytes);
                fa_box<CG>(ring_at + st * stage, &wmap, n0, k0, full0 + 8 * st);
                fa_box<CG>(ring_at + st * stage + FA_ABYTES / 2, &wmap, n0 + 64, k0, full0 + 8 * st);
            };
            auto ask_x = [&](int st, int m0, int k0) {
                fa_box<CG>(ring_at + st * stage + FA_ABYTES, &xmap, k0, m0, full0 + 8 * st);
                fa_box<CG>(ring_at + st * stage + FA_ABYTES + bn_cta * 128, &xmap, k0 + 64, m0, full0 + 8 * st);
            };
            const int ahead = nkb < a.stages ? nkb : a.stages;  // stages of the first tile that go out at once
            int sent = 0, st = 0, tn = 0, tm = 0;
            uint32_t par = 1;  // of the round before: a fresh barrier passes
            if (first < tiles) {
                fa_tile(a, first, tn, tm);
                const int n0 = tn * FA_TN * CG + rank * FA_TN, m0 = tm * a.BN + rank * bn_cta;
                for (int i = 0; i < ahead; ++i) ask_w(i, n0, (kb0 + i) * FA_BK);
                griddep_wait();
                for (int i = 0; i < ahead; ++i) ask_x(i, m0, (kb0 + i) * FA_BK);
                sent = st = ahead;
                if (st == a.stages) { st = 0; par ^= 1u; }
            }
            bool ok = true;
            for (int t = first; t < tiles && ok; t += clusters) {
                fa_tile(a, t, tn, tm);
                const int n0 = tn * FA_TN * CG + rank * FA_TN, m0 = tm * a.BN + rank * bn_cta;
                for (int kb = t == first ? ahead : 0; kb < nkb; ++kb) {
                    ok = fa_wait(empty0 + 8 * st, par, a, abort_flag);
                    if (!ok) break;
                    ask_w(st, n0, (kb0 + kb) * FA_BK);
                    ask_x(st, m0, (kb0 + kb) * FA_BK);
                    ++sent;
                    if (++st == a.stages) { st = 0; par ^= 1u; }
                }
            }
            griddep_launch_dependents();
            sh->sent = sent;
        }
        __syncwarp();
    } else if (warp == FA_EPI_WARPS + 1) {
        // ---- MMAs, by one elected lane; with CG = 2 only in the first CTA of the pair.  The elected form matters: with `lane == 0` the four
        // MMAs and the commit of a stage took 345 cycles to issue, with elect.sync 180, and a box 85 and 25.
        if (rank == 0 && fa_elect()) {
            const uint32_t idesc = (1u << 4) | ((BF16 ? 1u : 0u) << 7) | ((BF16 ? 1u : 0u) << 10) | (1u << 15) | (0u << 16) |
                                   ((uint32_t)(a.BN >> 3) << 17) | ((uint32_t)((FA_TN * CG) >> 4) << 24);
            const uint64_t dw0 = tc_desc(smem_u32(ring), FA_ABYTES / 2, 1024, 2), dx0 = tc_desc(smem_u32(ring) + FA_ABYTES, 16, 1024, 2);
            const uint32_t full0 = smem_u32(&sh->full[0]), empty0 = smem_u32(&sh->empty[0]);
            int st = 0, n = 0;  // n: accumulations so far, in turn in the two accumulators
            uint32_t par = 0;
            bool ok = true, issued = false;
            for (int t = first; t < tiles && ok; t += clusters) {
                for (int kb = 0; kb < nkb;) {
                    const int acc = n & 1, stop = min(nkb, kb + chunk);
                    if (n >= 2) {
                        ok = fa_wait(smem_u32(&sh->tempty[acc]), (uint32_t)((n >> 1) - 1) & 1u, a, abort_flag);
                        if (!ok) break;
                        tc_fence_after();
                    }
                    const uint32_t d = tmem + (uint32_t)acc * (uint32_t)a.BN;
                    bool more = false;
                    for (; kb < stop; ++kb) {
                        ok = fa_wait(full0 + 8 * st, par, a, abort_flag);
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t dw = dw0 + (uint64_t)((uint32_t)st * (stage >> 4)), dx = dx0 + (uint64_t)((uint32_t)st * (stage >> 4));
                        // (the channels beyond K of the last block are zeros in both operands)
#pragma unroll
                        for (uint32_t k = 0; k < FA_BK / 16; ++k)
                            fa_mma<CG>(d, dw + k * (2048 >> 4), dx + (k >> 2) * ((uint32_t)bn_cta * 128 >> 4) + (k & 3) * (32 >> 4), idesc, (more || k > 0) ? 1u : 0u);
                        fa_commit<CG>(empty0 + 8 * st);
                        more = issued = true;
                        if (++st == a.stages) { st = 0; par ^= 1u; }
                    }
                    if (!ok) break;
                    fa_commit<CG>(smem_u32(&sh->tfull[acc]));
                    ++n;
                }
            }
            if (!ok && issued) {  // let the MMAs under way finish before shared memory and TMEM go
                if constexpr (CG == 2)
                    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(&sh->drain)) : "memory");
                else
                    fa_commit<CG>(smem_u32(&sh->drain));
                for (uint32_t i = 0; i < TRIES / 16 && !mbarrier_try_wait(smem_u32(&sh->drain), 0); ++i) {}
            }
        }
        __syncwarp();
    } else {
        // ---- epilogue: warp w reads the 32 lanes of its quarter, and every other 16 columns
        const int quarter = warp & 3, half = warp >> 2;
        const uint32_t lane_at = tmem + ((uint32_t)(quarter * 32) << 16);
        griddep_wait();  // b and r may come from the work just before; y may still be read by it
        int n = 0;
        for (int t = first; t < tiles; t += clusters) {
            int tn, tm;
            fa_tile(a, t, tn, tm);
            const int col = tn * FA_TN * CG + rank * FA_TN + quarter * 32 + lane;  // output channel of this lane
            const bool on = col < a.N;
            const float bias = on && a.b ? ld_act(a.b + col) : 0.0f;
            const int m0 = tm * a.BN, rows = min(a.BN, a.M - m0);
            // The residual of 16 rows is asked for ahead of their accumulators: while the MMAs run, and while the 16 rows before are worked on.
            // 16-bit rows move four bytes per lane: a pair of channels, of even rows in even lanes and of odd rows in odd ones.  (A lane with one
            // channel and two bytes per store took 45 cycles per row of a tile, 11.2 us in place of 13.3 at 832 x 1280 x 3328.)
            uint32_t r[F32 ? 16 : 8];
            const uint32_t sel = lane & 1 ? 0x3276u : 0x5410u;
            const int colp = col & ~1;
            auto ask_r = [&](int c) {
                if constexpr (F32) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) r[j] = fa_load<F32>(a.r, (long long)(m0 + c + j) * a.ldr + col, on && c + j < rows);
                } else {
                    const int left = on ? rows - c - (lane & 1) : 0;
                    const unsigned short *p = reinterpret_cast<const unsigned short *>(a.r) + (long long)(m0 + c + (lane & 1)) * a.ldr + colp;
                    if (a.ldr & 1) {  // (rows that begin between two words)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            r[j] = ld_act_if_u16(p + 2 * j * a.ldr, 2 * j < left) | (uint32_t)ld_act_if_u16(p + 2 * j * a.ldr + 1, 2 * j < left) << 16;
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) r[j] = __float_as_uint(ld_act_if(reinterpret_cast<const float *>(p + 2 * j * a.ldr), 2 * j < left));
                    }
                }
            };
            if (S == 1 && a.r) ask_r(half * 16);
            bool ok = true;
            auto wait_acc = [&]() {
                ok = fa_wait(smem_u32(&sh->tfull[n & 1]), (uint32_t)(n >> 1) & 1u, a, abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                tc_fence_after();
                return ok;
            };
            auto done_acc = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (CG == 2) fa_arrive_cluster(cluster_addr(smem_u32(&sh->tempty[n & 1]), 0));
                    else mbar_arrive(&sh->tempty[n & 1]);
                }
                ++n;
            };
            // sixteen rows: either into y, or (a rank of several) as part of the sum into the ring, which nobody uses any more: [row of y][channel]
            auto finish = [&](int c, const float (&v)[16]) {
                if (S > 1) {
                    float *part = reinterpret_cast<float *>(ring);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c + j < rows) part[(c + j) * FA_TN + quarter * 32 + lane] = v[j];
                    return;
                }
                float u[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) u[j] = v[j] + bias;
                fa_act(u, a.act);
                if constexpr (F32) {
                    if (a.r) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) u[j] += fa_widen<BF16, F32>(r[j]);
                        ask_r(c + 32);
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (on && c + j < rows) fa_store<BF16, F32>(a.y, (long long)(m0 + c + j) * a.ldy + col, u[j]);
                } else {
                    if (a.r) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const uint32_t w = fa_swap(r[j], sel);
                            u[2 * j] += widen_bits<BF16>((unsigned short)w);
                            u[2 * j + 1] += widen_bits<BF16>((unsigned short)(w >> 16));
                        }
                        ask_r(c + 32);
                    }
                    uint32_t w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = fa_swap(fa_pack<BF16>(u[2 * j], u[2 * j + 1]), sel);
                    const int left = on ? rows - c - (lane & 1) : 0;
                    unsigned short *p = reinterpret_cast<unsigned short *>(a.y) + (long long)(m0 + c + (lane & 1)) * a.ldy + colp;
                    if (a.ldy & 1) {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (2 * j < left) { p[2 * j * a.ldy] = (unsigned short)w[j]; p[2 * j * a.ldy + 1] = (unsigned short)(w[j] >> 16); }
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (2 * j < left) *reinterpret_cast<uint32_t *>(p + 2 * j * a.ldy) = w[j];
                    }
                }
            };
            if constexpr (CHUNKED) {
                constexpr int NC = FA_MAX_BN_CHUNKED / 32;
                float sum[NC][16];
#pragma unroll
                for (int i = 0; i < NC; ++i)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[i][j] = 0.0f;
                for (int kb = 0; kb < nkb; kb += chunk) {
                    if (!wait_acc()) break;
#pragma unroll
                    for (int i = 0; i < NC; i += 2) {
                        const int c = half * 16 + 32 * i;
                        if (c < rows) {
                            uint32_t v[2][16];
                            const bool both = c + 32 < rows;
                            fa_ld16(v[0], lane_at + (uint32_t)((n & 1) * a.BN + c));
                            fa_ld16(v[1], lane_at + (uint32_t)((n & 1) * a.BN + (both ? c + 32 : c)));
                            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                sum[i][j] += __uint_as_float(v[0][j]);
                                sum[i + 1][j] += both ? __uint_as_float(v[1][j]) : 0.0f;
                            }
                        }
                    }
                    done_acc();
                }
                if (!ok) break;
#pragma unroll 1
                for (int c = half * 16; c < rows; c += 32) {  // (rolled, the sums move up: the code unrolled does not fit the instruction cache)
                    finish(c, sum[0]);
#pragma unroll
                    for (int i = 0; i + 1 < NC; ++i)
#pragma unroll
                        for (int j = 0; j < 16; ++j) sum[i][j] = sum[i + 1][j];
                }
            } else {
                if (!wait_acc()) break;
                for (int c = half * 16; c < rows; c += 32) {
                    uint32_t v[16];
                    fa_ld16(v, lane_at + (uint32_t)((n & 1) * a.BN + c));
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                    float x[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[j] = __uint_as_float(v[j]);
                    finish(c, x);
                }
                done_acc();
            }
        }
    }
    if (CG == 1 && S > 1) {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        if (!*abort_flag && warp < FA_EPI_WARPS) {
            int tn, tm;
            fa_tile(a, first, tn, tm);
            const int m0 = tm * a.BN, rows = min(a.BN, a.M - m0);
            const int ch = (warp & 3) * 32 + lane, col = tn * FA_TN + ch;
            const float bias = col < a.N && a.b ? ld_act(a.b + col) : 0.0f;
            const uint32_t part = smem_u32(ring);
            // rank s finishes rows s, s + S, ... of the tile, a warp four of them at a time: a remote load takes several hundred cycles
            for (int c0 = srank + S * (warp >> 2); c0 < rows; c0 += 8 * S) {
                float u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                uint32_t r[4];
                if (a.r) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int c = c0 + 2 * S * i;
                        r[i] = fa_load<F32>(a.r, (long long)(m0 + c) * a.ldr + col, c < rows && col < a.N);
                    }
                }
                for (int s0 = 0; s0 < S; s0 += 4) {
                    float v[4][4];
#pragma unroll
                    for (int s = 0; s < 4; ++s) {  // (a rank or a row that there is not reads the first one, and is not used)
                        const uint32_t at = cluster_addr(part + (uint32_t)ch * 4, s0 + s < S ? s0 + s : s0);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int c = c0 + 2 * S * i;
                            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[s][i]) : "r"(at + (uint32_t)(c < rows ? c : c0) * (FA_TN * 4)) : "memory");
                        }
                    }
#pragma unroll
                    for (int s = 0; s < 4; ++s)
#pragma unroll
                        for (int i = 0; i < 4; ++i) u[i] += s0 + s < S ? v[s][i] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] += bias;
                fa_act(u, a.act);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = c0 + 2 * S * i;
                    if (c < rows && col < a.N) {
                        float w = u[i];
                        if (a.r) w += fa_widen<BF16, F32>(r[i]);
                        fa_store<BF16, F32>(a.y, (long long)(m0 + c) * a.ldy + col, w);
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) {
        if (tid == 0) {
            const uint32_t other = (uint32_t)rank ^ 1u;
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(smem_u32(&sh->peer_sent), other)), "r"(sh->sent) : "memory");
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(smem_u32(&sh->peer_abort), other)), "r"(sh->abort_flag) : "memory");
        }
    }
    if (CG == 2 || S > 1) { cluster_arrive(); cluster_wait(); }  // nobody leaves while the other may still use its shared memory
    // After a wait that ran out nobody consumes the stages, but the copies under way still write here: wait for them, with a limit.  With
    // CG = 2 those of both CTAs count on the first one's barriers; for stages that only the other one asked for there was no announcement yet.
    if (*abort_flag || (CG == 2 && sh->peer_abort)) {
        if (rank == 0 && tid == 0) {
            const int mine_sent = sh->sent, all = CG == 2 ? max(mine_sent, sh->peer_sent) : mine_sent;
            for (int i = all > a.stages ? all - a.stages : 0; i < all; ++i) {
                if (i >= mine_sent) mbar_arrive_expect_tx(&sh->full[i % a.stages], stage);
                for (uint32_t n = 0; n < TRIES / 16 && !mbarrier_try_wait(smem_u32(&sh->full[i % a.stages]), (uint32_t)(i / a.stages) & 1u); ++n) {}
            }
        }
        __syncthreads();
        if constexpr (CG == 2) { cluster_arrive(); cluster_wait(); }
    }
    tc_fence_after();
    if (warp == FA_EPI_WARPS + 1) {
        if constexpr (CG == 2)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(a.tmem_cols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(a.tmem_cols) : "memory");
    }
}

// Rows of x whose stride TMA cannot take (not a multiple of 16 bytes), copied to rows that it can.
__global__ void fc_act_repack_kernel(const unsigned short *x, long long ldx, unsigned short *out, int ldo, int M, int K) {
    griddep_wait();
    griddep_launch_dependents();  // (the product asks for its first weights meanwhile, and waits for this kernel before it looks at x)
    const long long n = (long long)M * ldo;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const long long m = i / ldo;
        const int k = (int)(i - m * ldo);
        out[i] = k < K ? __ldcg(x + m * ldx + k) : (unsigned short)0;
    }
}

struct FaPlan {
    int cg, BN, S, stages;
};

static int fa_stages(int cg, int BN) {
    const int stage = FA_ABYTES + BN / cg * FA_BK * 2;
    const int n = (FA_SMEM - 1024 - (int)sizeof(FaShared)) / stage;
    return n < FA_MAX_STAGES ? n : FA_MAX_STAGES;
}

// Clusters of S CTAs that the device holds at once, as the runtime reports it.  A CTA takes a whole SM, and the S of a cluster come from one group
// of SMs, so the larger sizes leave SMs over: on 148, 74 clusters of 2, 33 of 4, 22 of 6 and 15 of 8.  One cluster more is a second turn of
// them all: 18 of 8 took 18.7 us where 9 of them with twice the rows take 10.2 (28 rows, 8736 x 1048).
// The current device, -1 where there is none; asked for once per call (once per size it was 0.3 us of the host's time).
static int fa_device() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); dev = -1; }
    return dev;
}
static int fa_clusters(int S, int dev) {
    static std::atomic<int> cached_by_dev[64][MAX_CLUSTER + 1];
    if (dev >= 0 && dev < 64) {
        const int hit = cached_by_dev[dev][S].load(std::memory_order_relaxed);
        if (hit) return hit;
    }
    int n = sm_count() / S;
    static SmemOptIn opt_in;
    auto kern = fc_act_kernel<true, 1, false, false>;
    if (S > 1 && ensure_dynamic_smem(kern, FA_SMEM, opt_in) == cudaSuccess) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(1, S);
        cfg.blockDim = dim3(FA_THREADS);
        cfg.dynamicSmemBytes = FA_SMEM;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 1;
        attr[0].val.clusterDim.y = S;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int found = 0;
        if (cudaOccupancyMaxActiveClusters(&found, kern, &cfg) == cudaSuccess && found > 0) n = found;
        else cudaGetLastError();
    } else if (S > 1) {
        cudaGetLastError();
    }
    if (dev >= 0 && dev < 64) cached_by_dev[dev][S].store(n, std::memory_order_relaxed);
    return n;
}

// The form with the shortest estimate, in cycles: waves of tiles x blocks of 128 channels x the slower of a block's MMAs and its loads (58
// bytes per cycle and SM, from L2), W at the rate of the memory, the epilogue of the last wave (18 cycles a row; more with a function to compute or
// fp32 rows), and what a pair or the sum over ranks costs.  A sum reads
// its peers four at a time, and clusters of 5 and 7 were never the best.  Over 70 drawn shapes with every form measured the choice is 4% off the best.
static FaPlan fa_plan(int M, int K, int N, bool chunked, int act, int dev) {
    const int nkb = (K + FA_BK - 1) / FA_BK;
    FaPlan best = {1, 16, 1, 0};
    const double floor = 0.45 * K * (double)N * 2 / 1000.0;  // W at the rate of the memory, in cycles
    const double row = (chunked ? 25.0 : 18.0) + (act > SCAP_ACT_RELU ? 10.0 : 0.0);
    double best_t = 1e300;
    int slots_of[MAX_CLUSTER + 1];
    for (int S = 1; S <= MAX_CLUSTER; ++S) slots_of[S] = fa_clusters(S, dev);
    for (int cg = 1; cg <= 2; ++cg)
        for (int BN = 16 * cg; BN <= (chunked ? FA_MAX_BN_CHUNKED : 256); BN += 16 * cg) {
            if (BN >= M + 16 * cg) break;
            const long long tiles = (long long)((N + FA_TN * cg - 1) / (FA_TN * cg)) * ((M + BN - 1) / BN);
            const int most = cg == 1 ? MAX_CLUSTER : 1;
            for (int S = 1; S <= most; ++S) {
                if (S > nkb) break;
                if (S == 5 || S == 7) continue;
                const int slots = slots_of[cg == 2 ? 2 : S];
                if (S > 1 && tiles > slots) continue;
                const double waves = (double)((tiles + slots - 1) / slots);
                const double mma = 8.0 * (BN / 2 < 46 ? 46 : BN / 2), load = (FA_ABYTES + BN / cg * FA_BK * 2) / 58.0;
                double t = waves * ((nkb + S - 1) / S) * (mma > load ? mma : load);
                t = sqrt(t * t + floor * floor);  // the closer to the memory's rate, the slower each SM's share
                if (S > 1) t += 2500.0 + 35.0 * BN + (S > 4 ? 2500.0 : 0.0);
                else t += row * BN + (cg == 2 ? 3500.0 : 0.0);
                if (t < best_t) { best_t = t; best = {cg, BN, S, 0}; }
            }
        }
    best.stages = fa_stages(best.cg, best.BN);
    return best;
}

static bool fa_map(CUtensorMap *map, const void *p, long long inner, long long outer, long long ld, int box_inner, int box_outer, bool bf16) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
    const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_outer};
    const cuuint32_t estr[2] = {1, 1};
    return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(p), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool BF16, int CG, bool F32, bool CHUNKED>
static cudaError_t fa_launch_y(const FaArgs &a, int slots, const CUtensorMap &wmap, const CUtensorMap &xmap, cudaStream_t st) {
    static SmemOptIn opt_in;
    auto kern = fc_act_kernel<BF16, CG, F32, CHUNKED>;
    cudaError_t e = ensure_dynamic_smem(kern, FA_SMEM, opt_in);
    if (e != cudaSuccess) return e;
    const int tiles = a.tiles_n * a.tiles_m;
    cudaLaunchConfig_t cfg = {};
    if (CG == 2) {
        cfg.gridDim = dim3(2 * (tiles < slots ? tiles : slots));
    } else {
        cfg.gridDim = a.S > 1 ? dim3(tiles, a.S) : dim3(tiles < slots ? tiles : slots);
    }
    cfg.blockDim = dim3(FA_THREADS);
    cfg.dynamicSmemBytes = FA_SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = g_tune.pdl ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CG;
    attr[1].val.clusterDim.y = CG == 1 ? a.S : 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CG == 2 || a.S > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, a, wmap, xmap);
}

template <bool BF16, int CG>
static cudaError_t fa_launch(const FaArgs &a, int slots, bool f32, const CUtensorMap &wmap, const CUtensorMap &xmap, cudaStream_t st) {
    if (f32) return fa_launch_y<BF16, CG, true, true>(a, slots, wmap, xmap, st);
    return fa_long(a.K, BF16) ? fa_launch_y<BF16, CG, false, true>(a, slots, wmap, xmap, st) : fa_launch_y<BF16, CG, false, false>(a, slots, wmap, xmap, st);
}

}  // namespace scap

using namespace scap;

extern "C" size_t scap_fc_act_workspace(int M, int K, int N, int64_t ldx) {
    if (M < 0 || M > SCAP_MAX_ROWS || K < 1 || K > SCAP_MAX_K || N < 1 || ldx < K) return 0;
    return ldx % 8 == 0 ? 16 : (size_t)(M > 0 ? M : 1) * align_up((size_t)K, 8) * 2;
}

extern "C" scap_status scap_fc_act(const void *x, int64_t ldx, const void *W, const float *b, scap_act act, const void *r, int64_t ldr, void *y,
                                   int64_t ldy, int M, int K, int N, scap_dtype dt, scap_dtype ydt, void *ws, size_t ws_bytes, scap_stream_t stream) {
    if (M < 0 || M > SCAP_MAX_ROWS || K < 1 || K > SCAP_MAX_K || N < 1 || ldx < K || ldy < N || (r && ldr < N)) return SCAP_ERR_SHAPE;
    if ((unsigned)act > (unsigned)SCAP_ACT_GELU_TANH) return SCAP_ERR_INVALID_ARG;
    if ((dt != SCAP_F16 && dt != SCAP_BF16) || (ydt != SCAP_F32 && ydt != dt)) return SCAP_ERR_DTYPE;
    if (M == 0) return SCAP_OK;
    if (!x || !W || !y || !ws) return SCAP_ERR_INVALID_ARG;
    if (N % 8 != 0 || !aligned16(x) || !aligned16(W) || !aligned16(y) || !aligned16(b) || !aligned16(r) || !aligned16(ws)) return SCAP_ERR_ALIGN;
    // a tensor map takes strides below 2^40 bytes; offsets of y and r are 64-bit
    if (ldx >= (1ll << 38) || ldy >= (1ll << 38) || (r && ldr >= (1ll << 38)) || N > (1 << 30)) return SCAP_ERR_SHAPE;
    if (ws_bytes < scap_fc_act_workspace(M, K, N, ldx)) return SCAP_ERR_WORKSPACE;
    scap_status dev = check_device();
    if (dev != SCAP_OK) return dev;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);

    const int device = fa_device();
    const FaPlan p = fa_plan(M, K, N, ydt == SCAP_F32 || fa_long(K, dt == SCAP_BF16), act, device);
    const int slots = fa_clusters(p.cg == 2 ? 2 : 1, device);  // tiles that run at once, where S is 1
    FaArgs a = {};
    a.b = b; a.r = r; a.y = y; a.ldr = ldr; a.ldy = ldy;
    a.M = M; a.K = K; a.N = N; a.act = act;
    a.BN = p.BN; a.S = p.S; a.stages = p.stages;
    const long long tn = ((long long)N + FA_TN * p.cg - 1) / (FA_TN * p.cg), tm = ((long long)M + p.BN - 1) / p.BN;
    if (tn * tm > (1ll << 30)) return SCAP_ERR_SHAPE;
    a.tiles_n = (int)tn; a.tiles_m = (int)tm;
    a.groups = a.tiles_m < 8 ? a.tiles_m : 8;
    a.tmem_cols = 32;
    while (a.tmem_cols < 2u * (uint32_t)p.BN) a.tmem_cols *= 2;
    a.limit = g_tune.tc_spin ? (uint32_t)g_tune.tc_spin : TRIES;
    a.status = tc_status_ptr();

    const void *xs = x;
    long long ldxs = ldx;
    const bool repack = ldx % 8 != 0;
    if (repack) { xs = ws; ldxs = (long long)align_up((size_t)K, 8); }
    CUtensorMap wmap, xmap;
    const bool bf16 = dt == SCAP_BF16;
    if (!fa_map(&wmap, W, N, K, N, 64, FA_BK, bf16) || !fa_map(&xmap, xs, K, M, ldxs, 64, p.BN / p.cg, bf16)) return SCAP_ERR_CUDA;
    if (repack) {
        const long long n = (long long)M * ldxs;
        const long long blocks = (n + 255) / 256;
        const cudaError_t e = launch(fc_act_repack_kernel, dim3((unsigned)(blocks < 8 * sm_count() ? blocks : 8 * sm_count())), dim3(256), 0, st, g_tune.pdl != 0,
                                     reinterpret_cast<const unsigned short *>(x), (long long)ldx, reinterpret_cast<unsigned short *>(ws), (int)ldxs, M, K);
        if (e != cudaSuccess) return cuda_status(e);
    }
    const bool f32 = ydt == SCAP_F32;
    cudaError_t e;
    if (bf16) e = p.cg == 2 ? fa_launch<true, 2>(a, slots, f32, wmap, xmap, st) : fa_launch<true, 1>(a, slots, f32, wmap, xmap, st);
    else e = p.cg == 2 ? fa_launch<false, 2>(a, slots, f32, wmap, xmap, st) : fa_launch<false, 1>(a, slots, f32, wmap, xmap, st);
    return cuda_status(e);
}
