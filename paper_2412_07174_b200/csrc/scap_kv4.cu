// The 4-bit key / value cache: new tokens into it, and the values it holds out of it.
//
// Both kernels take their rows in runs: the rows of one sequence that fall into one 32-token tile.  A block has a run and one head: a
// word of V codes holds the eight tokens 8 j + 2 t + o, and whoever writes one of them has to write back the other seven, so warp t of
// four has those.  A lane has D/32 neighbouring channels.  Bound by instruction issue (prompts: about 170 instructions of a warp per token,
// head and side, 524000 of these for 8191 tokens of 32 heads) or by the latency of a few dependent loads (single tokens).
//
// Quantisation is decided exactly as its definition in real numbers: (hi - lo) / 15 in binary64 and rounded to 20 bits there, and
// x / s in binary32 unless it comes near a tie, which is then decided in binary64.
#include "scap_kv4.cuh"

namespace scap {

constexpr int KV_THREADS = 128;  // four warps: one for each word of eight tokens

struct KvRows {
    const void *k, *v;       // append: read; read: written
    long long ldk, ldv;      // elements between tokens
    const int *row_start;    // [n_seqs + 1], or NULL: row b is the one new token of sequence b
    int rows, per_block;     // rows of k and v; rows among which a block looks for the beginnings of runs
};

struct KvRun {
    int seq, pos, n;  // sequence and position of the first row, number of rows; 0 rows: no run begins here
    int next;         // where to look on
};

// The run that begins at `row`, if one does.  Its sequence is the last one that does not begin behind the row: every look at 32 places of
// row_start narrows it down by a factor of 32, and the last look brings the lengths with it.
__device__ __forceinline__ KvRun kv_run(const KvCache &c, const KvRows &r, int row, int lane) {
    KvRun run;
    int first = row, stop = row + 1, len;
    run.seq = row;
    if (r.row_start) {
        int lo = 0, many = c.n_seqs;  // row_start[lo] <= row (or lo = 0), the answer in lo .. lo + many - 1
        while (many > 31) {
            const int step = (many + 31) / 32;
            const unsigned below = __ballot_sync(0xffffffffu, lane * step < many && __ldcg(r.row_start + lo + lane * step) <= row);
            const int k = below ? 31 - __clz(below) : 0;
            lo += k * step;
            many = min(step, many - k * step);
        }
        const bool on = lane <= many;  // (one place more: where the last sequence ends)
        const int at = on ? __ldcg(r.row_start + lo + lane) : 0, tokens = lane < many ? __ldcg(c.lens + lo + lane) : 0;
        const unsigned below = __ballot_sync(0xffffffffu, lane < many && at <= row);
        const int k = below ? 31 - __clz(below) : 0;
        run.seq = lo + k;
        first = __shfl_sync(0xffffffffu, at, k);
        stop = __shfl_sync(0xffffffffu, at, k + 1);
        len = __shfl_sync(0xffffffffu, tokens, k);
    } else {
        len = __ldcg(c.lens + run.seq);
    }
    const int end = min(stop, r.rows);
    run.n = 0;
    run.pos = 0;
    run.next = row < first ? first : r.rows;  // before the first sequence, or behind the last one
    if (row < first || row >= end) return run;
    const long long pos = (long long)len - ((long long)stop - first) + (row - first);
    if (pos < 0) {  // (more rows than the sequence has tokens: those in front have no place)
        run.next = (int)min((long long)end, row - pos);
        return run;
    }
    run.pos = (int)pos;
    run.next = min(end, row + KV_TILE - run.pos % KV_TILE);
    if (row == first || run.pos % KV_TILE == 0) run.n = run.next - row;
    return run;
}

// s of a group whose values reach from lo to hi: (hi - lo) / 15 to 20 significant bits (to a multiple of 2^-145 where that is coarser).
// The quotient is a product with the rounded 1 / 15 and one correction of it, which gives the correctly rounded one (Markstein).
__device__ __forceinline__ float kv_scale(float lo, float hi) {
    const double d = (double)hi - (double)lo, q = d * (1.0 / 15.0), r = fma(fma(-15.0, q, d), 1.0 / 15.0, q);
    if (r < 1.1754943508222875e-38) return (float)(rint(r * 0x1p145) * 0x1p-145);
    unsigned long long u = (unsigned long long)__double_as_longlong(r);
    u += 0xffffffffull + ((u >> 33) & 1ull);
    return (float)__longlong_as_double((long long)(u & ~0x1ffffffffull));
}

template <bool BF16>
__device__ __forceinline__ uint32_t kv_min2(uint32_t a, uint32_t b) {  // of both halves; a NaN stays
    uint32_t r;
    if constexpr (BF16) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

__device__ __forceinline__ float kv_rcp(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
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
template <int CPL, int GL, bool BF16>
__device__ __forceinline__ uint32_t kv_quantise(const KvVec<CPL> &v, uint32_t &word) {
    // smallest value and smallest negative in one register, per group of lanes
    uint32_t m = 0;  // (0, 0): the range always holds zero
#pragma unroll
    for (int k = 0; k < CPL / 2; ++k) {
        const uint32_t a = v.w[k];
        m = kv_min2<BF16>(m, __byte_perm(a, a ^ 0x80008000u, 0x5410));  // (x0, -x0)
        m = kv_min2<BF16>(m, __byte_perm(a, a ^ 0x80008000u, 0x7632));  // (x1, -x1)
    }
#pragma unroll
    for (int o = 1; o < GL; o *= 2) m = kv_min2<BF16>(m, __shfl_xor_sync(0xffffffffu, m, o));
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
    // round(x / s), ties to even, as in real numbers: by the product with 1 / s (good to 2^-23), which is at most a little over 15, so
    // it is off by less than 3e-6 - right unless it comes that near a tie; rounded by adding 1.5 2^23, whose last bit is one.
    constexpr float BIG = 12582912.0f;
    const float inv = kv_rcp(s);
    float x[CPL];
#pragma unroll
    for (int k = 0; k < CPL / 2; ++k) widen2<BF16>(v.w[k], x[2 * k], x[2 * k + 1]);
    const float tz = -lo * inv, nz = (tz + BIG) - BIG;
    bool near = fabsf(tz - nz) > 0.4999f || s < 0x1p-100f;  // (no use of 1 / s there)
    int zero = (int)(__float_as_uint(tz + BIG) - __float_as_uint(BIG)), n[CPL];
#pragma unroll
    for (int k = 0; k < CPL; ++k) {
        const float t = x[k] * inv, m = t + BIG;
        n[k] = (int)(__float_as_uint(m) - __float_as_uint(BIG));
        near = near || fabsf(t - (m - BIG)) > 0.4999f;
    }
    if (near) {
        zero = (int)rint(-(double)lo / (double)s);
#pragma unroll 1
        for (int k = 0; k < CPL; ++k) {
            const int q = (int)rint((double)x[0] / (double)s);
#pragma unroll
            for (int i = 0; i < CPL; ++i) n[i] = i == k ? q : n[i];
#pragma unroll
            for (int i = 0; i + 1 < CPL; ++i) x[i] = x[i + 1];  // (rolled: one copy of the division)
        }
    }
    zero = min(15, max(0, zero));
    word = __float_as_uint(s) | (uint32_t)zero;
    uint32_t codes = 0;
#pragma unroll
    for (int k = 0; k < CPL; ++k) codes |= (uint32_t)min(15, max(0, n[k] + zero)) << (4 * k);
    return codes;
}

template <int D, int GROUP, bool BF16>
__global__ void __launch_bounds__(KV_THREADS) kv4_append_kernel(const KvCache c, const KvRows r) {
    constexpr int CPL = D / 32, GL = GROUP / CPL, GROUPS = D / GROUP;  // channels of a lane, lanes of a group
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, t = threadIdx.x >> 5, h = blockIdx.y;
    constexpr int tile_bytes = kv_tile_bytes(D, GROUPS);
    const int ch = lane * CPL, g = ch / GROUP;
    const bool writes = lane % GL == 0;
    const int row0 = blockIdx.x * r.per_block, row1 = min(row0 + r.per_block, r.rows);
    for (int row = row0; row < row1;) {
        const KvRun run = kv_run(c, r, row, lane);
        const int first = row, tok0 = run.pos % KV_TILE;
        row = run.next;
        if (run.n == 0) continue;
        // this warp's tokens 8 j + 2 t + o that lie in the run, as nibbles of the words of V codes
        uint32_t mask = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int n = 8 * (i >> 1) + 2 * t + (i & 1) - tok0;
            if (n >= 0 && n < run.n) mask |= 15u << (4 * ((i >> 1) + 4 * (i & 1)));
        }
        if (mask == 0) continue;
        const int page = kv_page(c, run.seq, run.pos);
        if (page < 0) continue;
        unsigned char *tile = kv_tile(c, page, h, run.pos, tile_bytes);
        uint32_t *kw = reinterpret_cast<uint32_t *>(tile + kv_k_words(D)) + g * KV_TILE, *vw = reinterpret_cast<uint32_t *>(tile + kv_v_words(D, GROUPS)) + g * KV_TILE;
        uint32_t *vcodes = reinterpret_cast<uint32_t *>(tile + kv_v_codes(D));
        uint32_t vcode[CPL];
#pragma unroll
        for (int k = 0; k < CPL; ++k) vcode[k] = mask == 0xffffffffu ? 0u : __ldcg(vcodes + kv_v_word(ch + k, t)) & ~mask;
        // (rolled, with the next token's values under way: unrolled the code does not fit the instruction cache)
        auto tok_of = [&](int i) { return 8 * (i >> 1) + 2 * t + (i & 1); };
        auto ask = [&](int i, KvVec<CPL> &kx, KvVec<CPL> &vx) {
            const int n = tok_of(i) - tok0;
            const bool on = i < 8 && n >= 0 && n < run.n;
            kx = kv_load<CPL>(r.k, (long long)(first + n) * r.ldk + (long long)h * D + ch, on);
            vx = kv_load<CPL>(r.v, (long long)(first + n) * r.ldv + (long long)h * D + ch, on);
        };
        KvVec<CPL> kx[2], vx[2];
        ask(0, kx[0], vx[0]);
        ask(1, kx[1], vx[1]);
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            const KvVec<CPL> k0 = kx[0], v0 = vx[0];
            kx[0] = kx[1];
            vx[0] = vx[1];
            ask(i + 2, kx[1], vx[1]);
            const int tok = tok_of(i);
            if (tok < tok0 || tok >= tok0 + run.n) continue;  // (the same for all lanes)
            uint32_t word;
            const uint32_t kc = kv_quantise<CPL, GL, BF16>(k0, word);
            unsigned char *to = tile + tok * (D / 2) + kv_k_byte(D, ch);
            if constexpr (CPL == 2) *to = (unsigned char)kc;
            else if constexpr (CPL == 4) *reinterpret_cast<unsigned short *>(to) = (unsigned short)kc;
            else *reinterpret_cast<uint32_t *>(to) = kc;
            if (writes) kw[kv_word_at(tok)] = word;
            const uint32_t vc = kv_quantise<CPL, GL, BF16>(v0, word);
            if (writes) vw[kv_word_at(tok)] = word;
            const int nib = 4 * ((i >> 1) + 4 * (i & 1));
#pragma unroll
            for (int k = 0; k < CPL; ++k) vcode[k] |= ((vc >> (4 * k)) & 15u) << nib;
        }
#pragma unroll
        for (int k = 0; k < CPL; ++k) vcodes[kv_v_word(ch + k, t)] = vcode[k];
    }
}

// Two values to a word of two 16-bit ones.
template <bool BF16>
__device__ __forceinline__ uint32_t kv_narrow2(float a, float b) {
    uint32_t r;
    if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
template <int CPL>
__device__ __forceinline__ void kv_put(void *p, long long i, const uint32_t (&w)[CPL / 2]) {
    unsigned short *q = reinterpret_cast<unsigned short *>(p) + i;
    if constexpr (CPL == 2) *reinterpret_cast<uint32_t *>(q) = w[0];
    else if constexpr (CPL == 4) *reinterpret_cast<uint2 *>(q) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint4 *>(q) = make_uint4(w[0], w[1], w[2], w[3]);
}

template <int D, int GROUP, bool BF16>
__global__ void __launch_bounds__(KV_THREADS) kv4_read_kernel(const KvCache c, const KvRows r) {
    constexpr int CPL = D / 32, GROUPS = D / GROUP, tile_bytes = kv_tile_bytes(D, GROUPS);
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, t = threadIdx.x >> 5, h = blockIdx.y, ch = lane * CPL, g = ch / GROUP;
    const int row0 = blockIdx.x * r.per_block, row1 = min(row0 + r.per_block, r.rows);
    for (int row = row0; row < row1;) {
        const KvRun run = kv_run(c, r, row, lane);
        const int first = row, tok0 = run.pos % KV_TILE;
        row = run.next;
        if (run.n == 0) continue;
        const int page = kv_page(c, run.seq, run.pos);
        if (page < 0) continue;
        const unsigned char *tile = kv_tile(c, page, h, run.pos, tile_bytes);
        const uint32_t *kw = reinterpret_cast<const uint32_t *>(tile + kv_k_words(D)) + g * KV_TILE, *vw = reinterpret_cast<const uint32_t *>(tile + kv_v_words(D, GROUPS)) + g * KV_TILE;
        uint32_t vcode[CPL], kcode[8], kword[8], vword[8];
#pragma unroll
        for (int k = 0; k < CPL; ++k) vcode[k] = __ldcg(reinterpret_cast<const uint32_t *>(tile + kv_v_codes(D)) + kv_v_word(ch + k, t));
#pragma unroll
        for (int i = 0; i < 8; i += 4) {  // the words of tokens 2 t + o lie side by side
            *reinterpret_cast<uint4 *>(kword + i) = __ldcg(reinterpret_cast<const uint4 *>(kw + kv_word_at(2 * t + i / 4)));
            *reinterpret_cast<uint4 *>(vword + i) = __ldcg(reinterpret_cast<const uint4 *>(vw + kv_word_at(2 * t + i / 4)));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {  // (in the order of the words: token 8 (i % 4) + 2 t + i / 4; the tile is there whether the token is or not)
            const unsigned char *from = tile + (8 * (i & 3) + 2 * t + (i >> 2)) * (D / 2) + kv_k_byte(D, ch);
            if constexpr (CPL == 2) kcode[i] = __ldcg(from);
            else if constexpr (CPL == 4) kcode[i] = __ldcg(reinterpret_cast<const unsigned short *>(from));
            else kcode[i] = __ldcg(reinterpret_cast<const uint32_t *>(from));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int j = i & 3, o = i >> 2, n = 8 * j + 2 * t + o - tok0;
            if (n < 0 || n >= run.n) continue;
            const int nib = 4 * (j + 4 * o);
            const float ks = __uint_as_float(kword[i] & ~15u), vs = __uint_as_float(vword[i] & ~15u);
            const int kz = kword[i] & 15u, vz = vword[i] & 15u;
            uint32_t ka[CPL / 2], va[CPL / 2];
#pragma unroll
            for (int k = 0; k < CPL / 2; ++k) {
                ka[k] = kv_narrow2<BF16>(ks * (float)((int)((kcode[i] >> (8 * k)) & 15u) - kz), ks * (float)((int)((kcode[i] >> (8 * k + 4)) & 15u) - kz));
                va[k] = kv_narrow2<BF16>(vs * (float)((int)((vcode[2 * k] >> nib) & 15u) - vz), vs * (float)((int)((vcode[2 * k + 1] >> nib) & 15u) - vz));
            }
            kv_put<CPL>(const_cast<void *>(r.k), (long long)(first + n) * r.ldk + (long long)h * D + ch, ka);
            kv_put<CPL>(const_cast<void *>(r.v), (long long)(first + n) * r.ldv + (long long)h * D + ch, va);
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

// Rows a block looks through: a tile's worth, fewer where there are few, so that single tokens of many sequences go side by side.
static int kv_per_block(long long rows, int heads) {
    const long long n = rows * heads / (8LL * sm_count());
    return n < 1 ? 1 : (n > KV_TILE ? KV_TILE : (int)n);
}

template <int D, int GROUP>
static cudaError_t kv_launch(bool append, bool bf16, const KvCache &c, const KvRows &r, cudaStream_t st) {
    const dim3 grid((r.rows + r.per_block - 1) / r.per_block, c.heads), block(KV_THREADS);
    const bool pdl = g_tune.pdl != 0;
    if (append) return bf16 ? launch(kv4_append_kernel<D, GROUP, true>, grid, block, 0, st, pdl, c, r) : launch(kv4_append_kernel<D, GROUP, false>, grid, block, 0, st, pdl, c, r);
    return bf16 ? launch(kv4_read_kernel<D, GROUP, true>, grid, block, 0, st, pdl, c, r) : launch(kv4_read_kernel<D, GROUP, false>, grid, block, 0, st, pdl, c, r);
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
    r.per_block = kv_per_block(rows, cache->heads);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool bf16 = dt == SCAP_BF16;
    switch (cache->head_dim + cache->group) {
        case 64 + 32: return cuda_status(kv_launch<64, 32>(append, bf16, c, r, st));
        case 64 + 64: return cuda_status(kv_launch<64, 64>(append, bf16, c, r, st));
        case 128 + 32: return cuda_status(kv_launch<128, 32>(append, bf16, c, r, st));
        case 128 + 64: return cuda_status(kv_launch<128, 64>(append, bf16, c, r, st));
        case 128 + 128: return cuda_status(kv_launch<128, 128>(append, bf16, c, r, st));
        case 256 + 64: return cuda_status(kv_launch<256, 64>(append, bf16, c, r, st));
        default: return cuda_status(kv_launch<256, 128>(append, bf16, c, r, st));
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
