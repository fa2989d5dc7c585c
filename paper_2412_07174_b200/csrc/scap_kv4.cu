// The 4-bit key / value cache: new tokens into it, and the values it holds out of it.
//
// Both kernels take their rows in runs: the rows of one sequence that fall into one 32-token tile.  One warp has a run and one head,
// because a word of V codes holds eight tokens: whoever writes one of them has to write back the other seven.  A lane has D/32
// neighbouring channels.  Bound by memory (prompts) or by the latency of a few dependent loads (single tokens).
//
// Quantisation is decided exactly as its definition in real numbers: (hi - lo) / 15 in binary64 and rounded to 20 bits there, and
// x / s in binary32 unless it comes near a tie, which is then decided in binary64.
#include "scap_kv4.cuh"

namespace scap {

constexpr int KV_THREADS = 128;

struct KvRows {
    const void *k, *v;       // append: read; read: written
    long long ldk, ldv;      // elements between tokens
    const int *row_start;    // [n_seqs + 1], or NULL: row b is the one new token of sequence b
    int rows, per_warp;      // rows of k and v; rows a warp looks through for the beginnings of runs
};

struct KvRun {
    int row, seq, pos, n;  // first row, its sequence and position, number of rows
};

// Sequence of a row: the last one that does not begin behind it (one load of 32 lanes per factor of 32).
__device__ __forceinline__ int kv_find(const int *start, int n, int row, int lane) {
    int lo = 0, len = n;  // start[lo] <= row (or lo = 0), the answer in lo .. lo + len - 1
    while (len > 1) {
        const int step = (len + 31) / 32, at = lo + lane * step;
        const unsigned below = __ballot_sync(0xffffffffu, lane * step < len && __ldcg(start + at) <= row);
        const int k = below ? 31 - __clz(below) : 0;
        lo += k * step;
        len = min(step, len - k * step);
    }
    return lo;
}

// The run that begins at `row`, if one does.
__device__ __forceinline__ bool kv_run(const KvCache &c, const KvRows &r, int row, int lane, KvRun &run) {
    int first = row, end = row + 1;
    run.seq = row;
    if (r.row_start) {
        run.seq = kv_find(r.row_start, c.n_seqs, row, lane);
        first = __ldcg(r.row_start + run.seq);
        end = min(__ldcg(r.row_start + run.seq + 1), r.rows);
    }
    if (row < first || row >= end) return false;  // before the first sequence, or behind the last one
    const int all = r.row_start ? __ldcg(r.row_start + run.seq + 1) - first : 1;
    run.row = row;
    run.pos = __ldcg(c.lens + run.seq) - all + (row - first);
    if (run.pos < 0) return false;
    if (row != first && run.pos % KV_TILE != 0) return false;
    run.n = min(KV_TILE - run.pos % KV_TILE, end - row);
    return true;
}

// s of a group whose values reach from lo to hi: (hi - lo) / 15 to 20 significant bits (to a multiple of 2^-145 where that is coarser).
__device__ __forceinline__ float kv_scale(float lo, float hi) {
    const double r = ((double)hi - (double)lo) / 15.0;
    if (r < 1.1754943508222875e-38) return (float)(rint(r * 0x1p145) * 0x1p-145);
    unsigned long long u = (unsigned long long)__double_as_longlong(r);
    u += 0xffffffffull + ((u >> 33) & 1ull);
    return (float)__longlong_as_double((long long)(u & ~0x1ffffffffull));
}

// round(x / s), ties to even, as in real numbers.  inv = 1 / s; |x / s| is at most a little over 15, so the product is off by less than
// 3e-6, and a result that far from a tie is right.
__device__ __forceinline__ float kv_round(float x, float s, float inv) {
    const float t = x * inv, n = rintf(t);
    if (fabsf(t - n) < 0.4999f) return n;
    return (float)rint((double)x / (double)s);
}

template <bool BF16>
__device__ __forceinline__ uint32_t kv_min2(uint32_t a, uint32_t b) {  // of both halves; a NaN stays
    uint32_t r;
    if constexpr (BF16) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

template <int CPL>
struct KvVec {
    uint32_t w[CPL / 2];
};
template <int CPL>
__device__ __forceinline__ KvVec<CPL> kv_load(const void *p, long long i, bool on) {
    KvVec<CPL> r;
    const unsigned short *q = reinterpret_cast<const unsigned short *>(p) + i;
#pragma unroll
    for (int k = 0; k < CPL / 2; ++k) r.w[k] = 0;
    if (on) {
        if constexpr (CPL == 2) r.w[0] = __ldcg(reinterpret_cast<const uint32_t *>(q));
        else if constexpr (CPL == 4) { const uint2 u = __ldcg(reinterpret_cast<const uint2 *>(q)); r.w[0] = u.x; r.w[1] = u.y; }
        else { const uint4 u = __ldcg(reinterpret_cast<const uint4 *>(q)); r.w[0] = u.x; r.w[1] = u.y; r.w[2] = u.z; r.w[3] = u.w; }
    }
    return r;
}

// Codes of a lane's channels (nibble i = channel i) and the word of its group.  All lanes of the warp take part.
template <int CPL, bool BF16>
__device__ __forceinline__ uint32_t kv_quantise(const KvVec<CPL> &x, int group_lanes, uint32_t &word) {
    // smallest value and smallest negative in one register, per group of lanes
    uint32_t m = 0;  // (0, 0): the range always holds zero
#pragma unroll
    for (int k = 0; k < CPL / 2; ++k) {
        const uint32_t a = x.w[k];
        m = kv_min2<BF16>(m, __byte_perm(a, a ^ 0x80008000u, 0x5410));  // (x0, -x0)
        m = kv_min2<BF16>(m, __byte_perm(a, a ^ 0x80008000u, 0x7632));  // (x1, -x1)
    }
#pragma unroll
    for (int o = 1; o < 32; o *= 2)
        if (o < group_lanes) m = kv_min2<BF16>(m, __shfl_xor_sync(0xffffffffu, m, o));
    float lo, hi;
    widen2<BF16>(m, lo, hi);
    hi = -hi;
    if (!(fabsf(lo) < __int_as_float(0x7f800000) && fabsf(hi) < __int_as_float(0x7f800000))) {  // an infinity or a NaN: the group reads as NaN
        word = 0x7fc00000u;
        return 0;
    }
    const float s = kv_scale(lo, hi);
    if (s == 0.0f) {
        word = 0;
        return 0;
    }
    const bool tiny = s < 0x1p-100f;  // no use of 1 / s: binary64 throughout
    const float inv = tiny ? 0.0f : 1.0f / s;
    auto rnd = [&](float v) { return tiny ? (float)rint((double)v / (double)s) : kv_round(v, s, inv); };
    const float zero = fminf(15.0f, fmaxf(0.0f, rnd(-lo)));
    word = __float_as_uint(s) | (uint32_t)zero;
    uint32_t codes = 0;
#pragma unroll
    for (int k = 0; k < CPL / 2; ++k) {
        float a, b;
        widen2<BF16>(x.w[k], a, b);
        codes |= (uint32_t)fminf(15.0f, fmaxf(0.0f, rnd(a) + zero)) << (8 * k);
        codes |= (uint32_t)fminf(15.0f, fmaxf(0.0f, rnd(b) + zero)) << (8 * k + 4);
    }
    return codes;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(KV_THREADS) kv4_append_kernel(const KvCache c, const KvRows r, int group) {
    constexpr int CPL = D / 32;  // channels of a lane
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, h = blockIdx.y;
    const int group_lanes = group / CPL, tile_bytes = kv_tile_bytes(D, c.groups);
    const long long row0 = ((long long)blockIdx.x * (KV_THREADS / 32) + (threadIdx.x >> 5)) * r.per_warp;
    for (long long row = row0; row < row0 + r.per_warp && row < r.rows; ++row) {
        KvRun run;
        if (!kv_run(c, r, (int)row, lane, run)) continue;
        const int page = kv_page(c, run.seq, run.pos);
        if (page < 0) continue;
        unsigned char *tile = kv_tile(c, page, h, run.pos, tile_bytes);
        uint32_t *kw = reinterpret_cast<uint32_t *>(tile + kv_k_words(D)), *vw = reinterpret_cast<uint32_t *>(tile + kv_v_words(D, c.groups));
        const int tok0 = run.pos % KV_TILE, ch = lane * CPL, g = ch / group;
        const bool writes = lane % group_lanes == 0;
        for (int t = 0; t < 4; ++t) {
            // the eight tokens 8 j + 2 t + o of a word of V codes
            KvVec<CPL> kx[8], vx[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int n = 8 * (i >> 1) + 2 * t + (i & 1) - tok0;  // row of the run
                const bool on = n >= 0 && n < run.n;
                kx[i] = kv_load<CPL>(r.k, (long long)(run.row + n) * r.ldk + (long long)h * D + ch, on);
                vx[i] = kv_load<CPL>(r.v, (long long)(run.row + n) * r.ldv + (long long)h * D + ch, on);
            }
            uint32_t vcode[CPL], mask = 0;
#pragma unroll
            for (int k = 0; k < CPL; ++k) vcode[k] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int tok = 8 * (i >> 1) + 2 * t + (i & 1);
                if (tok < tok0 || tok >= tok0 + run.n) continue;  // (the same for all lanes)
                const int nib = 4 * ((i >> 1) + 4 * (i & 1));
                uint32_t word;
                const uint32_t kc = kv_quantise<CPL, BF16>(kx[i], group_lanes, word);
                unsigned char *to = tile + tok * (D / 2) + kv_k_byte(D, ch);
                if constexpr (CPL == 2) *to = (unsigned char)kc;
                else if constexpr (CPL == 4) *reinterpret_cast<unsigned short *>(to) = (unsigned short)kc;
                else *reinterpret_cast<uint32_t *>(to) = kc;
                if (writes) kw[g * KV_TILE + kv_word_at(tok)] = word;
                const uint32_t vc = kv_quantise<CPL, BF16>(vx[i], group_lanes, word);
                if (writes) vw[g * KV_TILE + kv_word_at(tok)] = word;
#pragma unroll
                for (int k = 0; k < CPL; ++k) vcode[k] |= ((vc >> (4 * k)) & 15u) << nib;
                mask |= 15u << nib;
            }
            if (mask) {
                uint32_t *vcodes = reinterpret_cast<uint32_t *>(tile + kv_v_codes(D));
#pragma unroll
                for (int k = 0; k < CPL; ++k) {
                    uint32_t *at = vcodes + kv_v_word(ch + k, t);
                    *at = mask == 0xffffffffu ? vcode[k] : (__ldcg(at) & ~mask) | vcode[k];
                }
            }
        }
    }
}

template <int D, bool BF16>
__device__ __forceinline__ unsigned short kv_narrow(float v) {
    if constexpr (BF16) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
    else return __half_as_ushort(__float2half_rn(v));
}

template <int D, bool BF16>
__global__ void __launch_bounds__(KV_THREADS) kv4_read_kernel(const KvCache c, const KvRows r, int group) {
    constexpr int CPL = D / 32;
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, h = blockIdx.y, tile_bytes = kv_tile_bytes(D, c.groups);
    unsigned short *ko = reinterpret_cast<unsigned short *>(const_cast<void *>(r.k)), *vo = reinterpret_cast<unsigned short *>(const_cast<void *>(r.v));
    const long long row0 = ((long long)blockIdx.x * (KV_THREADS / 32) + (threadIdx.x >> 5)) * r.per_warp;
    for (long long row = row0; row < row0 + r.per_warp && row < r.rows; ++row) {
        KvRun run;
        if (!kv_run(c, r, (int)row, lane, run)) continue;
        const int page = kv_page(c, run.seq, run.pos);
        if (page < 0) continue;
        const unsigned char *tile = kv_tile(c, page, h, run.pos, tile_bytes);
        const int tok0 = run.pos % KV_TILE, ch = lane * CPL, g = ch / group;
        const uint32_t *kw = reinterpret_cast<const uint32_t *>(tile + kv_k_words(D)) + g * KV_TILE, *vw = reinterpret_cast<const uint32_t *>(tile + kv_v_words(D, c.groups)) + g * KV_TILE;
        for (int t = 0; t < 4; ++t) {
            uint32_t vcode[CPL], kcode[8], kword[8], vword[8];
#pragma unroll
            for (int k = 0; k < CPL; ++k) vcode[k] = __ldcg(reinterpret_cast<const uint32_t *>(tile + kv_v_codes(D)) + kv_v_word(ch + k, t));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int tok = 8 * (i >> 1) + 2 * t + (i & 1);
                kcode[i] = kword[i] = vword[i] = 0;
                if (tok < tok0 || tok >= tok0 + run.n) continue;
                const unsigned char *from = tile + tok * (D / 2) + kv_k_byte(D, ch);
                if constexpr (CPL == 2) kcode[i] = __ldcg(from);
                else if constexpr (CPL == 4) kcode[i] = __ldcg(reinterpret_cast<const unsigned short *>(from));
                else kcode[i] = __ldcg(reinterpret_cast<const uint32_t *>(from));
                kword[i] = __ldcg(kw + kv_word_at(tok));
                vword[i] = __ldcg(vw + kv_word_at(tok));
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int tok = 8 * (i >> 1) + 2 * t + (i & 1), n = tok - tok0;
                if (n < 0 || n >= run.n) continue;
                const int nib = 4 * ((i >> 1) + 4 * (i & 1));
                const float ks = __uint_as_float(kword[i] & ~15u), kz = (float)(kword[i] & 15u);
                const float vs = __uint_as_float(vword[i] & ~15u), vz = (float)(vword[i] & 15u);
                uint32_t ka[CPL / 2], va[CPL / 2];
#pragma unroll
                for (int k = 0; k < CPL / 2; ++k) {
                    const float a = ks * ((float)((kcode[i] >> (8 * k)) & 15u) - kz), b = ks * ((float)((kcode[i] >> (8 * k + 4)) & 15u) - kz);
                    ka[k] = (uint32_t)kv_narrow<D, BF16>(a) | ((uint32_t)kv_narrow<D, BF16>(b) << 16);
                    const float e = vs * ((float)((vcode[2 * k] >> nib) & 15u) - vz), f = vs * ((float)((vcode[2 * k + 1] >> nib) & 15u) - vz);
                    va[k] = (uint32_t)kv_narrow<D, BF16>(e) | ((uint32_t)kv_narrow<D, BF16>(f) << 16);
                }
                unsigned short *kt = ko + (long long)(run.row + n) * r.ldk + (long long)h * D + ch, *vt = vo + (long long)(run.row + n) * r.ldv + (long long)h * D + ch;
                if constexpr (CPL == 2) {
                    *reinterpret_cast<uint32_t *>(kt) = ka[0];
                    *reinterpret_cast<uint32_t *>(vt) = va[0];
                } else if constexpr (CPL == 4) {
                    *reinterpret_cast<uint2 *>(kt) = make_uint2(ka[0], ka[1]);
                    *reinterpret_cast<uint2 *>(vt) = make_uint2(va[0], va[1]);
                } else {
                    *reinterpret_cast<uint4 *>(kt) = make_uint4(ka[0], ka[1], ka[2], ka[3]);
                    *reinterpret_cast<uint4 *>(vt) = make_uint4(va[0], va[1], va[2], va[3]);
                }
            }
        }
    }
}

scap_status kv_check(const scap_kv4 *c) {
    if (!c || !c->pages || !c->table || !c->lens) return SCAP_ERR_INVALID_ARG;
    if (c->n_pages < 1 || c->page_tokens < KV_TILE || c->page_tokens > 4096 || c->page_tokens % KV_TILE || c->heads < 1 || c->heads > 1024 || c->table_stride < 1 || c->n_seqs < 1 ||
        c->n_seqs > SCAP_MAX_SEQS)
        return SCAP_ERR_SHAPE;
    const size_t need = scap_kv4_page_bytes(c->page_tokens, c->heads, c->head_dim, c->group);
    if (need == 0 || c->page_stride < need || c->page_stride > ((size_t)1 << 40)) return SCAP_ERR_SHAPE;
    if (!aligned16(c->pages) || c->page_stride % 16 || !aligned16(c->table) || !aligned16(c->lens)) return SCAP_ERR_ALIGN;
    return SCAP_OK;
}

// Rows a warp looks through: few where there are few, so that single tokens of many sequences go side by side.
static int kv_per_warp(long long rows, int heads) {
    const long long warps = rows * heads / (16LL * sm_count());
    return warps < 1 ? 1 : (warps > 8 ? 8 : (int)warps);
}

template <int D>
static cudaError_t kv_launch(bool append, bool bf16, const KvCache &c, const KvRows &r, int group, cudaStream_t st) {
    const long long warps = ((long long)r.rows + r.per_warp - 1) / r.per_warp;
    const dim3 grid((unsigned)((warps + KV_THREADS / 32 - 1) / (KV_THREADS / 32)), c.heads), block(KV_THREADS);
    const bool pdl = g_tune.pdl != 0;
    if (append) return bf16 ? launch(kv4_append_kernel<D, true>, grid, block, 0, st, pdl, c, r, group) : launch(kv4_append_kernel<D, false>, grid, block, 0, st, pdl, c, r, group);
    return bf16 ? launch(kv4_read_kernel<D, true>, grid, block, 0, st, pdl, c, r, group) : launch(kv4_read_kernel<D, false>, grid, block, 0, st, pdl, c, r, group);
}

static scap_status kv_rows(bool append, const scap_kv4 *cache, const void *k, int64_t ldk, const void *v, int64_t ldv, const int *row_start, int rows, scap_dtype dt, scap_stream_t stream) {
    scap_status s = kv_check(cache);
    if (s != SCAP_OK) return s;
    if (rows < 0 || rows > SCAP_MAX_ROWS || (!row_start && rows > cache->n_seqs)) return SCAP_ERR_SHAPE;
    if (dt != SCAP_F16 && dt != SCAP_BF16) return SCAP_ERR_DTYPE;
    const int64_t width = (int64_t)cache->heads * cache->head_dim;
    if (ldk < width || ldv < width || ldk >= (1ll << 38) || ldv >= (1ll << 38)) return SCAP_ERR_SHAPE;
    if (rows == 0) return SCAP_OK;
    if (!k || !v) return SCAP_ERR_INVALID_ARG;
    if (!aligned16(k) || !aligned16(v) || ldk % 8 || ldv % 8 || (reinterpret_cast<uintptr_t>(row_start) & 3u)) return SCAP_ERR_ALIGN;
    s = check_device();
    if (s != SCAP_OK) return s;
    const KvCache c = kv_cache(cache);
    KvRows r = {};
    r.k = k; r.v = v; r.ldk = ldk; r.ldv = ldv; r.row_start = row_start; r.rows = rows;
    r.per_warp = kv_per_warp(rows, cache->heads);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool bf16 = dt == SCAP_BF16;
    switch (cache->head_dim) {
        case 64: return cuda_status(kv_launch<64>(append, bf16, c, r, cache->group, st));
        case 128: return cuda_status(kv_launch<128>(append, bf16, c, r, cache->group, st));
        default: return cuda_status(kv_launch<256>(append, bf16, c, r, cache->group, st));
    }
}

}  // namespace scap

using namespace scap;

extern "C" size_t scap_kv4_page_bytes(int page_tokens, int heads, int head_dim, int group) {
    if (page_tokens < KV_TILE || page_tokens > 4096 || page_tokens % KV_TILE || heads < 1 || heads > 1024) return 0;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return 0;
    if ((group != 32 && group != 64 && group != 128) || group > head_dim || head_dim > 4 * group) return 0;
    return (size_t)heads * (page_tokens / KV_TILE) * kv_tile_bytes(head_dim, head_dim / group);
}

extern "C" scap_status scap_kv4_append(const scap_kv4 *cache, const void *k, int64_t ldk, const void *v, int64_t ldv, const int *row_start, int rows, scap_dtype dt,
                                       scap_stream_t stream) {
    return kv_rows(true, cache, k, ldk, v, ldv, row_start, rows, dt, stream);
}

extern "C" scap_status scap_kv4_read(const scap_kv4 *cache, void *k, int64_t ldk, void *v, int64_t ldv, const int *row_start, int rows, scap_dtype dt, scap_stream_t stream) {
    return kv_rows(false, cache, k, ldk, v, ldv, row_start, rows, dt, stream);
}
