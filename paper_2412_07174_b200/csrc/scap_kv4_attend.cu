// Attention of new tokens over the 4-bit cache: out = softmax(scale q k^T + mask) v, one to sixteen new tokens per sequence.
//
// The rows of a key head (its query heads x the new tokens) are the M rows of mma.m16n8k16, up to 16 at a time; the cache is
// dequantised by nothing but a mask: a code is an fp16 subnormal (see scap_kv4.cuh), and what belongs to a group of channels is
// applied once per token:
//   scores  s_t = ks_t (sum_c q_c code_tc - zero_t sum_c q_c)
//   output  o_c = sum_t (p_t vs_t) code_tc - sum_t (p_t vs_t) zero_t, the second sum by one more MMA whose columns are the zero points.
// p vs is rounded to fp16 (11 bits) once and used in both sums, so the rounding acts on the value v, not on its code part; the queries
// are scaled by a power of two per row and are exact.  Scores, maxima, sums and accumulators are fp32.
//
// What bounds it: the bytes of the cache, D/2 + 4 groups per token, head and side - if the instructions keep up: per tile of 32 tokens a
// warp issues 64 MMAs (D = 128), 160 mask and shift instructions and about 150 for the softmax.
//
// Work is cut into equal parts, whatever the lengths: a unit is one tile of 32 tokens of one (sequence, 16 rows, head), all units are
// numbered, and CTA i of C takes the units [U i / C, U (i + 1) / C).  Inside a CTA the tiles of an item go round the four warps, each
// of which has its own ring of tiles, filled by cp.async.bulk (one copy per tile, 4.3 KB at D = 128), its own running maximum and sum, and no barrier with
// the others until the item ends.  An item that lies in one CTA is finished there; the parts of one that is cut go to the
// workspace, and a second kernel joins them in order.  No atomics: the same bits each time.
//
// Every wait is bounded; one that runs out sets the status word and leaves its tile out.
#include "scap_kv4.cuh"

namespace scap {

constexpr int AT_WARPS = 4;
constexpr int AT_THREADS = AT_WARPS * 32;
constexpr int AT_ROWS = 16;
constexpr int AT_MIN_UNITS = 4;  // tiles per CTA at least

template <int D>
__host__ __device__ constexpr int at_resident() { return D == 256 ? 2 : 3; }
template <int D, int G>
__host__ __device__ constexpr int at_stages() { return D == 64 ? 6 : (D == 128 ? (G == 4 ? 3 : 4) : 3); }

struct AtArgs {
    KvCache c;
    const unsigned short *q;
    unsigned short *out;
    float *lse;
    long long ldq, ldo;   // elements between tokens
    float *part;          // [2 C][16][D] weighted sums, then [2 C][16][2] maximum and sum
    int nq, g, row_tiles, window;
    float scale;          // times log2 e
    int ctas;
    bool bf16;
    uint32_t limit;
    int *status;
};

// Tiles that the new tokens of sequence b can see: first one and number.
__device__ __forceinline__ int at_tiles(const AtArgs &a, int b, int &first) {
    const int len = __ldcg(a.c.lens + b);
    first = 0;
    if (len <= 0) return 0;
    if (a.window > 0) {
        const long long lo = (long long)len - a.nq + 1 - a.window;  // of the first new token
        first = lo > 0 ? (int)(lo / KV_TILE) : 0;
    }
    return (int)(((long long)len + KV_TILE - 1) / KV_TILE) - first;
}

// Sum over the block; every thread gets it.
__device__ __forceinline__ long long at_block_sum(long long v, long long *s) {
#pragma unroll
    for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < AT_WARPS; ++w) v += s[w];
    return v;
}

// The sequence that unit u belongs to and the first unit of that sequence (the whole block takes part); per = items per sequence.
__device__ __forceinline__ void at_find(const AtArgs &a, long long u, int per, long long *s, int &seq, long long &base) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long before = 0;
    for (int b0 = 0; b0 < a.c.n_seqs; b0 += AT_THREADS) {
        const int b = b0 + (int)threadIdx.x;
        int first;
        const long long n = b < a.c.n_seqs ? (long long)at_tiles(a, b, first) * per : 0;
        long long incl = n;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const long long up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        __syncthreads();
        if (lane == 31) s[warp] = incl;
        __syncthreads();
        long long off = before, all = before;
        for (int w = 0; w < AT_WARPS; ++w) {
            if (w < warp) off += s[w];
            all += s[w];
        }
        if (n > 0 && off + incl - n <= u && u < off + incl) {
            s[AT_WARPS] = b;
            s[AT_WARPS + 1] = off + incl - n;
        }
        before = all;
        __syncthreads();
        if (u < before) break;
    }
    seq = (int)s[AT_WARPS];
    base = s[AT_WARPS + 1];
    __syncthreads();
}

__device__ __forceinline__ long long at_cut(long long units, int i, int ctas) { return units * i / ctas; }
__device__ __forceinline__ int at_cta_of(long long units, long long u, int ctas) { return (int)(((u + 1) * ctas - 1) / units); }
__device__ __forceinline__ int at_ctas(long long units, int ctas) {
    const long long n = (units + AT_MIN_UNITS - 1) / AT_MIN_UNITS;
    return n < ctas ? (int)n : ctas;
}

__device__ __forceinline__ void at_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t at_pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float at_ex2(float v) {  // 2^v; -inf gives 0
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float at_widen(unsigned short u, bool bf16) { return bf16 ? widen_bits<true>(u) : widen_bits<false>(u); }
__device__ __forceinline__ void at_store(unsigned short *p, float v, bool bf16) {
    *p = bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}
// 2^e for -126 <= e <= 127
__device__ __forceinline__ float at_pow2(int e) { return __int_as_float((e + 127) << 23); }

template <int D, int G>
__global__ void __launch_bounds__(AT_THREADS, at_resident<D>()) kv4_attend_kernel(const AtArgs a) {
    constexpr int W = D / 32;            // words of a K row per lane
    constexpr int TILE = kv_tile_bytes(D, G);
    constexpr int ST = at_stages<D, G>();
    constexpr int NT = D / 8;            // blocks of eight channels
    constexpr float LN2 = 0.69314718055994531f;
    static_assert(ST * TILE >= AT_ROWS * D * 4, "a warp's part of the join goes where its ring was");
    extern __shared__ __align__(128) unsigned char at_raw[];
    __shared__ unsigned long long s_full[AT_WARPS][ST];
    __shared__ long long s_sum[AT_WARPS + 2];
    __shared__ float s_m[AT_WARPS][AT_ROWS], s_l[AT_WARPS][AT_ROWS];

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, qg = lane >> 2, qt = lane & 3;
    unsigned char *ring = at_raw + warp * ST * TILE;
    if (lane == 0)
        for (int i = 0; i < ST; ++i) mbarrier_init(smem_addr(&s_full[warp][i]), 1);
    __syncthreads();
    griddep_wait();
    griddep_launch_dependents();

    const int per = a.c.heads * a.row_tiles;
    long long mine = 0;
    for (int b = tid; b < a.c.n_seqs; b += AT_THREADS) {
        int first;
        mine += at_tiles(a, b, first);
    }
    const long long units = at_block_sum(mine, s_sum) * per;
    const int ctas = at_ctas(units, a.ctas);
    if ((int)blockIdx.x < ctas) {
        long long u = at_cut(units, blockIdx.x, ctas);
        const long long u1 = at_cut(units, blockIdx.x + 1, ctas);
        int seq;
        long long base;
        at_find(a, u, per, s_sum, seq, base);
        int slot = 0, phase = 0;  // of this warp's ring, over all items
        bool dead = false;        // a wait of this warp ran out

        while (u < u1) {
            int first_tile;
            const int tiles = at_tiles(a, seq, first_tile);
            if (tiles == 0) { ++seq; continue; }  // (an empty sequence has no units; its rows are the second kernel's)
            const int item = (int)((u - base) / tiles), t0 = (int)(u - base - (long long)item * tiles);
            const int t1 = (int)min((long long)tiles, t0 + (u1 - u));
            const int rt = item / a.c.heads, h = item - rt * a.c.heads;
            const int len = __ldcg(a.c.lens + seq), rows = min(AT_ROWS, a.nq * a.g - rt * AT_ROWS);
            const int count = !dead && t1 - t0 - warp > 0 ? (t1 - t0 - warp + AT_WARPS - 1) / AT_WARPS : 0;  // tiles t0 + warp, + 4, ... are this warp's

            // ---- pages of the next 32 tiles of this warp, one per lane, and the first copies
            auto pos_of = [&](int i) { return (first_tile + t0 + warp + AT_WARPS * i) * KV_TILE; };
            int pages = lane < count ? kv_page(a.c, seq, pos_of(lane)) : -1;
            int next_pages = 32 + lane < count ? kv_page(a.c, seq, pos_of(32 + lane)) : -1;
            auto ask = [&](int i, int page, int st) {
                if (page >= 0 && lane == 0) {
                    const uint32_t bar = smem_addr(&s_full[warp][st]);
                    const unsigned char *src = kv_tile(a.c, page, h, pos_of(i), TILE);
                    mbarrier_arrive_expect(bar, TILE);
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_addr(ring + st * TILE)), "l"(src), "r"(TILE), "r"(bar)
                                 : "memory");
                } else if (lane == 0) {
                    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(&s_full[warp][st])) : "memory");  // no page: the tile is empty
                }
            };
            {
                int st = slot;
                for (int i = 0; i < ST && i < count; ++i) {
                    ask(i, __shfl_sync(0xffffffffu, pages, i), st);
                    if (++st == ST) st = 0;
                }
            }

            // ---- queries: rows qg and qg + 8 as A operands, scaled to just below 2^15 by a power of two; channels 32 j + 8 qt + i, the
            // even and odd nibbles of a code word in the two k halves of an MMA, the odd ones 16 times smaller as their codes are larger
            uint32_t qa[2 * W][4];
            float f[2], qz[2][G];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = qg + 8 * r;
                uint4 raw[W];
                const int in = rt * AT_ROWS + row, tok = in / a.g, hd = in - tok * a.g;
                const unsigned short *src = a.q + ((long long)seq * a.nq + tok) * a.ldq + (long long)(h * a.g + hd) * D + 8 * qt;
#pragma unroll
                for (int j = 0; j < W; ++j) raw[j] = ld_act16_if(src + 32 * j, row < rows);
                float v[W][8], top = 0.0f;
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t w = (&raw[j].x)[i >> 1];
                        v[j][i] = at_widen((unsigned short)(i & 1 ? w >> 16 : w), a.bf16);
                        top = fmaxf(top, fabsf(v[j][i]));
                    }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                int e = top > 0.0f ? 14 - ((__float_as_int(top) >> 23) - 127) : 0;
                e = e > 100 ? 100 : (e < -100 ? -100 : e);
                const float up = at_pow2(e);
                float sum[G];
#pragma unroll
                for (int n = 0; n < G; ++n) sum[n] = 0.0f;
#pragma unroll
                for (int j = 0; j < W; ++j) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[j * G / W] += v[j][i];
#pragma unroll
                    for (int hi = 0; hi < 2; ++hi) {
                        qa[2 * j + hi][r] = at_pack(v[j][2 * hi] * up, v[j][2 * hi + 4] * up);
                        qa[2 * j + hi][2 + r] = at_pack(v[j][2 * hi + 1] * (up * 0.0625f), v[j][2 * hi + 5] * (up * 0.0625f));
                    }
                }
                f[r] = at_pow2(24 - e) * a.scale;
#pragma unroll
                for (int n = 0; n < G; ++n) {
                    sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 1);
                    sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 2);
                    qz[r][n] = sum[n] * a.scale;
                }
            }
            // keys that a row sees: lo[r] .. hi[r]
            int hi[2], lo[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int in = min(rt * AT_ROWS + qg + 8 * r, a.nq * a.g - 1), at = len - a.nq + in / a.g;
                hi[r] = at;
                lo[r] = a.window > 0 && at >= a.window ? at - a.window + 1 : 0;
            }
            const int hi_all = len - a.nq, lo_all = a.window > 0 && len > a.window ? len - a.window : 0;  // what every row sees

            float o[NT][4], z[G][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
            int top_e = 1;  // exponent field of the largest scale of values so far: p vs is held as p vs 2^(14 + 127 - top_e)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][i] = 0.0f;
#pragma unroll
            for (int n = 0; n < G; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[n][i] = 0.0f;

            for (int i = 0; i < count; ++i) {
                const uint32_t bar = smem_addr(&s_full[warp][slot]);
                const int page = __shfl_sync(0xffffffffu, pages, i & 31);
                bool landed = false;
                for (uint32_t n = 0; n < a.limit && !landed; ++n) landed = mbarrier_try_wait(bar, phase);
                if (!__all_sync(0xffffffffu, landed)) {
                    // It ran out: no further work for this warp, but the copies under way still write here - wait for them, with a limit.
                    if (lane == 0 && a.status) atomicCAS(a.status, 0, 41);
                    dead = true;
                    int st = slot, ph = phase;
                    for (int k = i; k < i + ST && k < count; ++k) {
                        for (uint32_t n = 0; n < TRIES / 16 && !mbarrier_try_wait(smem_addr(&s_full[warp][st]), ph); ++n) {}
                        if (++st == ST) { st = 0; ph ^= 1; }
                    }
                    __syncwarp();
                    break;
                }
                const unsigned char *tile = ring + slot * TILE;
                const int pos = pos_of(i);
                if (page >= 0) {
                    // ---- scores
                    float s[4][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float acc[G][4];
#pragma unroll
                        for (int n = 0; n < G; ++n)
#pragma unroll
                            for (int k = 0; k < 4; ++k) acc[n][k] = 0.0f;
                        const unsigned char *krow = tile + (8 * j + qg) * (D / 2) + qt * (D / 8);
                        uint32_t w[W];
                        if constexpr (W == 2) *reinterpret_cast<uint2 *>(w) = *reinterpret_cast<const uint2 *>(krow);
                        else
#pragma unroll
                            for (int k = 0; k < W / 4; ++k) *reinterpret_cast<uint4 *>(w + 4 * k) = *reinterpret_cast<const uint4 *>(krow + 16 * k);
#pragma unroll
                        for (int k = 0; k < W; ++k) {
                            at_mma(acc[k * G / W], qa[2 * k], w[k] & 0x000f000fu, w[k] & 0x00f000f0u);
                            at_mma(acc[k * G / W], qa[2 * k + 1], (w[k] >> 8) & 0x000f000fu, (w[k] >> 8) & 0x00f000f0u);
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) s[j][k] = 0.0f;
#pragma unroll
                        for (int n = 0; n < G; ++n) {
                            const uint2 kw = *reinterpret_cast<const uint2 *>(tile + kv_k_words(D) + (n * KV_TILE + 8 * j + 2 * qt) * 4);
                            const float k0 = __uint_as_float(kw.x & ~15u), k1 = __uint_as_float(kw.y & ~15u);
                            const float z0 = (float)(kw.x & 15u), z1 = (float)(kw.y & 15u);
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                s[j][2 * r] += k0 * (acc[n][2 * r] * f[r] - z0 * qz[r][n]);
                                s[j][2 * r + 1] += k1 * (acc[n][2 * r + 1] * f[r] - z1 * qz[r][n]);
                            }
                        }
                    }
                    // ---- keys that not every row sees: tokens behind the last, before a window, or newer than the row's own
                    const bool edge = pos + KV_TILE - 1 > hi_all || pos < lo_all;
                    if (edge) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int at = pos + 8 * j + 2 * qt + (k & 1), r = k >> 1;
                                if (at > hi[r] || at < lo[r]) s[j][k] = -INFINITY;
                            }
                    }
                    // ---- running maximum and sum
                    float scale_o[2];
                    bool same = true;
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float t = m[r];
#pragma unroll
                        for (int j = 0; j < 4; ++j) t = fmaxf(t, fmaxf(s[j][2 * r], s[j][2 * r + 1]));
                        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
                        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
                        const float ref = t == -INFINITY ? 0.0f : t;  // nothing seen so far: all weights are 0
                        scale_o[r] = at_ex2(m[r] - ref);
                        same = same && t == m[r];
                        m[r] = t;
                        l[r] *= scale_o[r];
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                s[j][2 * r + k] = at_ex2(s[j][2 * r + k] - ref);
                                l[r] += s[j][2 * r + k];
                            }
                    }
                    // ---- scales of the values; tokens behind the last one have none, whatever lies there
                    uint2 vw[4][G];
                    uint32_t big = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int n = 0; n < G; ++n) {
                            vw[j][n] = *reinterpret_cast<const uint2 *>(tile + kv_v_words(D, G) + (n * KV_TILE + 8 * j + 2 * qt) * 4);
                            if (edge) {
                                const int at = pos + 8 * j + 2 * qt;
                                if (at >= len || at <= lo_all - a.nq) vw[j][n].x = 0;
                                if (at + 1 >= len || at + 1 <= lo_all - a.nq) vw[j][n].y = 0;
                            }
                            big = max(big, vw[j][n].x < 0x7f800000u ? vw[j][n].x : 0u);
                            big = max(big, vw[j][n].y < 0x7f800000u ? vw[j][n].y : 0u);
                        }
                    const int e = (int)(__reduce_max_sync(0xffffffffu, big) >> 23);
                    if (e > top_e) {
                        const int d = top_e - e < -126 ? -126 : top_e - e;
                        const float down = at_pow2(d);
                        scale_o[0] *= down;
                        scale_o[1] *= down;
                        same = false;
                        top_e = e;
                    }
                    if (!__all_sync(0xffffffffu, same)) {
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int k = 0; k < 4; ++k) o[n][k] *= scale_o[k >> 1];
#pragma unroll
                        for (int n = 0; n < G; ++n)
#pragma unroll
                            for (int k = 0; k < 4; ++k) z[n][k] *= scale_o[k >> 1];
                    }
                    // ---- weighted values.  2^(14 + 127 - top_e) in two factors: the exponent may lie anywhere
                    const int es = 141 - top_e, e1 = es / 2, e2 = es - e1;
                    const float up1 = at_pow2(e1), up2 = at_pow2(e2);
#pragma unroll
                    for (int n = 0; n < G; ++n) {
                        uint32_t pa[2][4];
#pragma unroll
                        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const int j = 2 * ks + half;
                                const float down = half ? 0.0625f : 1.0f;
                                const float v0 = __uint_as_float(vw[j][n].x & ~15u) * up1 * (up2 * down), v1 = __uint_as_float(vw[j][n].y & ~15u) * up1 * (up2 * down);
#pragma unroll
                                for (int r = 0; r < 2; ++r) {
                                    float x0 = s[j][2 * r] * v0, x1 = s[j][2 * r + 1] * v1;
                                    if (edge) {  // a row does not see what another one does: not even a NaN
                                        const int at = pos + 8 * j + 2 * qt;
                                        if (at > hi[r] || at < lo[r]) x0 = 0.0f;
                                        if (at + 1 > hi[r] || at + 1 < lo[r]) x1 = 0.0f;
                                    }
                                    pa[ks][2 * half + r] = at_pack(x0, x1);
                                }
                            }
#pragma unroll
                        for (int ks = 0; ks < 2; ++ks) {
                            const uint2 w0 = vw[2 * ks][n], w1 = vw[2 * ks + 1][n];
                            at_mma(z[n], pa[ks], (w0.x & 15u) | ((w0.y & 15u) << 16), ((w1.x & 15u) << 4) | ((w1.y & 15u) << 20));
                        }
#pragma unroll
                        for (int b4 = n * (NT / 4) / G; b4 < (n + 1) * (NT / 4) / G; ++b4) {
                            const uint4 w4 = *reinterpret_cast<const uint4 *>(tile + kv_v_codes(D) + (b4 * 32 + lane) * 16);
                            const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                at_mma(o[4 * b4 + k], pa[0], w[k] & 0x000f000fu, w[k] & 0x00f000f0u);
                                at_mma(o[4 * b4 + k], pa[1], (w[k] >> 8) & 0x000f000fu, (w[k] >> 8) & 0x00f000f0u);
                            }
                        }
                    }
                }
                // ---- the slot is free: the tile ST further on
                __syncwarp();
                if (i + ST < count) {
                    const int ni = i + ST;
                    // (pages holds those of the block of 32 that tile i lies in, next_pages the following block)
                    const int from = (ni >> 5) == (i >> 5) ? pages : next_pages;
                    ask(ni, __shfl_sync(0xffffffffu, from, ni & 31), slot);
                }
                if ((i & 31) == 31) {
                    pages = next_pages;
                    const int n = i + 33 + lane;
                    next_pages = n < count ? kv_page(a.c, seq, pos_of(n)) : -1;
                }
                if (++slot == ST) { slot = 0; phase ^= 1; }
            }

            // ---- join of the four warps: each puts its sums where its ring was (all of its copies have landed)
            const int es = top_e - 141 + 24, e1 = es / 2, e2 = es - e1;
            const float back1 = at_pow2(e1), back2 = at_pow2(e2);
            float *part = reinterpret_cast<float *>(ring);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
                if (qt == 0) {
                    s_m[warp][qg + 8 * r] = m[r];
                    s_l[warp][qg + 8 * r] = l[r];
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float zz = z[n * G / NT][2 * r];
                    *reinterpret_cast<float2 *>(part + (qg + 8 * r) * D + 8 * n + 2 * qt) =
                        make_float2((o[n][2 * r] - zz) * back1 * back2, (o[n][2 * r + 1] - zz) * back1 * back2);
                }
            }
            __syncthreads();
            const bool whole = t0 == 0 && t1 == tiles;
            const int slot_out = 2 * (int)blockIdx.x + (t0 == 0 ? 1 : 0);
            float *sums = a.part + (size_t)slot_out * AT_ROWS * D, *ml = a.part + (size_t)2 * a.ctas * AT_ROWS * D + (size_t)slot_out * AT_ROWS * 2;
            for (int row = warp; row < rows; row += AT_WARPS) {
                float top = -INFINITY, wt[AT_WARPS], sum = 0.0f;
#pragma unroll
                for (int w = 0; w < AT_WARPS; ++w) top = fmaxf(top, s_m[w][row]);
                const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
                for (int w = 0; w < AT_WARPS; ++w) {
                    wt[w] = at_ex2(s_m[w][row] - ref);
                    sum += wt[w] * s_l[w][row];
                }
                const float by = whole ? (sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f) : 1.0f;
                const int in = rt * AT_ROWS + row, tok = in / a.g, hd = in - tok * a.g;
                const long long tokrow = (long long)seq * a.nq + tok;
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    float v = 0.0f;
#pragma unroll
                    for (int w = 0; w < AT_WARPS; ++w) {
                        const float x = reinterpret_cast<const float *>(at_raw + w * ST * TILE)[row * D + c + lane];
                        v += wt[w] > 0.0f || x != x ? wt[w] * x : 0.0f;
                    }
                    if (whole) at_store(a.out + tokrow * a.ldo + (long long)(h * a.g + hd) * D + c + lane, v * by, a.bf16);
                    else sums[row * D + c + lane] = v;
                }
                if (lane == 0) {
                    if (!whole) {
                        ml[2 * row] = top;
                        ml[2 * row + 1] = sum;
                    } else if (a.lse) {
                        a.lse[tokrow * (a.c.heads * a.g) + h * a.g + hd] = sum > 0.0f || sum != sum ? top * LN2 + logf(sum) : -INFINITY;
                    }
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the next copies may overwrite what was read and written here
            __syncthreads();
            u += t1 - t0;
            if (u - base >= (long long)tiles * per) { base += (long long)tiles * per; ++seq; }
        }
    }
}

// Joins the parts of the items that were cut, and writes the rows of sequences without tokens.  One block per row of an item.
template <int D>
__global__ void __launch_bounds__(AT_THREADS) kv4_join_kernel(const AtArgs a) {
    constexpr float LN2 = 0.69314718055994531f;
    __shared__ long long s_sum[AT_WARPS + 2];
    __shared__ float s_w[AT_THREADS];
    __shared__ int s_at[AT_THREADS];
    griddep_wait();
    griddep_launch_dependents();
    const int seq = blockIdx.x, item = blockIdx.y, rt = item / a.c.heads, h = item - rt * a.c.heads, row = blockIdx.z, tid = threadIdx.x;
    const int in = rt * AT_ROWS + row;
    if (in >= a.nq * a.g) return;
    const int tok = in / a.g, hd = in - tok * a.g, per = a.c.heads * a.row_tiles;
    const long long tokrow = (long long)seq * a.nq + tok;
    unsigned short *out = a.out + tokrow * a.ldo + (long long)(h * a.g + hd) * D;
    float *lse = a.lse ? a.lse + tokrow * (a.c.heads * a.g) + h * a.g + hd : nullptr;
    int first;
    const int tiles = at_tiles(a, seq, first);
    if (tiles == 0) {
        for (int c = tid; c < D; c += AT_THREADS) at_store(out + c, 0.0f, a.bf16);
        if (lse && tid == 0) *lse = -INFINITY;
        return;
    }
    long long all = 0, before = 0;
    for (int b = tid; b < a.c.n_seqs; b += AT_THREADS) {
        int f;
        const int n = at_tiles(a, b, f);
        all += n;
        if (b < seq) before += n;
    }
    const long long units = at_block_sum(all, s_sum) * per, u0 = at_block_sum(before, s_sum) * per + (long long)item * tiles;
    const int ctas = at_ctas(units, a.ctas), i0 = at_cta_of(units, u0, ctas), i1 = at_cta_of(units, u0 + tiles - 1, ctas);
    if (i0 == i1) return;  // finished by its CTA
    const float *ml = a.part + (size_t)2 * a.ctas * AT_ROWS * D;
    auto slot_of = [&](int i) { return 2 * i + (i == i0 ? 1 : 0); };
    // maximum over the parts
    float top = -INFINITY;
    for (int i = i0 + tid; i <= i1; i += AT_THREADS) top = fmaxf(top, __ldcg(ml + ((size_t)slot_of(i) * AT_ROWS + row) * 2));
#pragma unroll
    for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if ((tid & 31) == 0) s_w[tid >> 5] = top;
    __syncthreads();
    top = s_w[0];
#pragma unroll
    for (int w = 1; w < AT_WARPS; ++w) top = fmaxf(top, s_w[w]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, v[(D + AT_THREADS - 1) / AT_THREADS];
#pragma unroll
    for (int k = 0; k < (D + AT_THREADS - 1) / AT_THREADS; ++k) v[k] = 0.0f;
    for (int i = i0; i <= i1; i += AT_THREADS) {
        const int n = min(AT_THREADS, i1 - i + 1);
        __syncthreads();
        float part_l = 0.0f;
        if (tid < n) {
            const float2 p = __ldcg(reinterpret_cast<const float2 *>(ml + ((size_t)slot_of(i + tid) * AT_ROWS + row) * 2));
            s_w[tid] = at_ex2(p.x - ref);
            s_at[tid] = slot_of(i + tid);
            part_l = s_w[tid] * p.y;
        }
        __syncthreads();
        sum += part_l;
#pragma unroll 8
        for (int k = 0; k < n; ++k) {
            const float w = s_w[k];
            const float *src = a.part + ((size_t)s_at[k] * AT_ROWS + row) * D;
#pragma unroll
            for (int c = 0; c < (D + AT_THREADS - 1) / AT_THREADS; ++c)
                if (D % AT_THREADS == 0 || tid < D) {
                    const float x = __ldcg(src + c * AT_THREADS + tid);
                    v[c] += w > 0.0f || x != x ? w * x : 0.0f;
                }
        }
    }
    // the sums of the threads in one order
#pragma unroll
    for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncthreads();
    if ((tid & 31) == 0) s_w[tid >> 5] = sum;
    __syncthreads();
    sum = s_w[0];
#pragma unroll
    for (int w = 1; w < AT_WARPS; ++w) sum += s_w[w];
    const bool any = sum > 0.0f || sum != sum;
    const float by = any ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int c = 0; c < (D + AT_THREADS - 1) / AT_THREADS; ++c)
        if (D % AT_THREADS == 0 || tid < D) at_store(out + c * AT_THREADS + tid, v[c] * by, a.bf16);
    if (lse && tid == 0) *lse = any ? top * LN2 + logf(sum) : -INFINITY;
}

template <int D, int G>
static cudaError_t at_launch(const AtArgs &a, cudaStream_t st) {
    static SmemOptIn opt_in;
    constexpr int SMEM = AT_WARPS * at_stages<D, G>() * kv_tile_bytes(D, G);
    auto kern = kv4_attend_kernel<D, G>;
    cudaError_t e = ensure_dynamic_smem(kern, SMEM, opt_in);
    if (e != cudaSuccess) return e;
    e = launch(kern, dim3(a.ctas), dim3(AT_THREADS), SMEM, st, g_tune.pdl != 0, a);
    if (e != cudaSuccess) return e;
    const int rows = a.nq * a.g < AT_ROWS ? a.nq * a.g : AT_ROWS;
    return launch(kv4_join_kernel<D>, dim3(a.c.n_seqs, a.c.heads * a.row_tiles, rows), dim3(AT_THREADS), 0, st, g_tune.pdl != 0, a);
}

static int at_grid(int D) { return sm_count() * (D == 256 ? at_resident<256>() : at_resident<128>()); }

}  // namespace scap

using namespace scap;

extern "C" size_t scap_kv4_attend_workspace(int n_seqs, int nq, int q_heads, int heads, int head_dim) {
    if (n_seqs < 1 || n_seqs > SCAP_MAX_SEQS || nq < 1 || nq > SCAP_MAX_BATCH || heads < 1 || heads > 1024 || q_heads < heads || q_heads % heads || q_heads > 1024) return 0;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return 0;
    return (size_t)2 * at_grid(head_dim) * AT_ROWS * (head_dim + 2) * sizeof(float);
}

extern "C" scap_status scap_kv4_attend(const scap_kv4 *cache, const void *q, int64_t ldq, void *out, int64_t ldo, float *lse, int nq, int q_heads, double scale, int window,
                                       scap_dtype dt, void *ws, size_t ws_bytes, scap_stream_t stream) {
    scap_status s = kv_check(cache);
    if (s != SCAP_OK) return s;
    if (nq < 1 || nq > SCAP_MAX_BATCH || q_heads < cache->heads || q_heads % cache->heads || q_heads > 1024 || window < 0) return SCAP_ERR_SHAPE;
    if (!(scale == scale) || scale > 1e30 || scale < -1e30) return SCAP_ERR_INVALID_ARG;
    if (dt != SCAP_F16 && dt != SCAP_BF16) return SCAP_ERR_DTYPE;
    const int64_t width = (int64_t)q_heads * cache->head_dim;
    if (ldq < width || ldo < width || ldq >= (1ll << 38) || ldo >= (1ll << 38)) return SCAP_ERR_SHAPE;
    if (!q || !out || !ws) return SCAP_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out) || !aligned16(lse) || !aligned16(ws) || ldq % 8) return SCAP_ERR_ALIGN;
    if (ws_bytes < scap_kv4_attend_workspace(cache->n_seqs, nq, q_heads, cache->heads, cache->head_dim)) return SCAP_ERR_WORKSPACE;
    s = check_device();
    if (s != SCAP_OK) return s;
    AtArgs a = {};
    a.c = kv_cache(cache);
    a.q = reinterpret_cast<const unsigned short *>(q);
    a.out = reinterpret_cast<unsigned short *>(out);
    a.lse = lse; a.ldq = ldq; a.ldo = ldo;
    a.part = reinterpret_cast<float *>(ws);
    a.nq = nq; a.g = q_heads / cache->heads;
    a.row_tiles = (nq * a.g + AT_ROWS - 1) / AT_ROWS;
    a.window = window;
    a.scale = (float)(scale * 1.4426950408889634);
    a.ctas = at_grid(cache->head_dim);
    a.bf16 = dt == SCAP_BF16;
    a.limit = g_tune.tc_spin ? (uint32_t)g_tune.tc_spin : TRIES;
    a.status = tc_status_ptr();
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    switch (cache->head_dim * 8 + a.c.groups) {
        case 64 * 8 + 1: return cuda_status(at_launch<64, 1>(a, st));
        case 64 * 8 + 2: return cuda_status(at_launch<64, 2>(a, st));
        case 128 * 8 + 1: return cuda_status(at_launch<128, 1>(a, st));
        case 128 * 8 + 2: return cuda_status(at_launch<128, 2>(a, st));
        case 128 * 8 + 4: return cuda_status(at_launch<128, 4>(a, st));
        case 256 * 8 + 2: return cuda_status(at_launch<256, 2>(a, st));
        default: return cuda_status(at_launch<256, 4>(a, st));
    }
}
