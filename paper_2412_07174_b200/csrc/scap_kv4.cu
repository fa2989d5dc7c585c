// The 4-bit key / value cache: new tokens into it, and the values it holds out of it.
//
// Both kernels take their rows in runs: the rows of one sequence that fall into one 32-token tile.  A block has a run and one head: a
// word of V codes holds the eight tokens 8 j + 2 t + o, and whoever writes one of them has to write back the other seven, so warp t of
// four has those.  A lane has eight neighbouring channels of a token (append) or D/32 of every token (read).  Bound by instruction issue
// (prompts: 8191 tokens of 32 heads take 88 us, 48 of them without the quantisation; the bytes alone are 26) or by the latency of a few
// dependent loads (single tokens).
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

// Codes of a lane's channels (nibble i = channel i) and the word of its group.  All lanes of the warp take part.  True where they
// come too near a tie, and kv_quantise_near has to look.
template <int CPL, int GL, bool BF16>
__device__ __forceinline__ bool kv_quantise(const KvVec<CPL> &v, uint32_t &codes, uint32_t &word, float &lo, float &s) {
    // smallest value and smallest negative in one register, per group of lanes
    uint32_t m2 = 0;  // (0, 0): the range always holds zero
#pragma unroll
    for (int k = 0; k < CPL / 2; ++k) {
        const uint32_t a = v.w[k];
        m2 = kv_min2<BF16>(m2, __byte_perm(a, a ^ 0x80008000u, 0x5410));  // (x0, -x0)
        m2 = kv_min2<BF16>(m2, __byte_perm(a, a ^ 0x80008000u, 0x7632));  // (x1, -x1)
    }
#pragma unroll
    for (int o = 1; o < GL; o *= 2) m2 = kv_min2<BF16>(m2, __shfl_xor_sync(0xffffffffu, m2, o));
    float hi;
    widen2<BF16>(m2, lo, hi);
    hi = -hi;
    const float inf = __int_as_float(0x7f800000);
    const bool bad = !(fabsf(lo) < inf && fabsf(hi) < inf);  // an infinity or a NaN: the group reads as NaN
    s = kv_scale(lo, hi);
    // round(x / s) + zero, ties to even, as in real numbers: by the product with 1 / s (good to 2^-23) added to 1.5 2^23 + zero, whose last bit is
    // one.  The product is at most a little over 15, so it is off by less than 2e-6 - right unless it comes that near a tie, which is seen from
    // what the rounding took off.  Codes lie at or above 0 by themselves: x >= lo, so round(x / s) >= round(lo / s) = -zero.
    constexpr float BIG = 12582912.0f;
    const uint32_t big = __float_as_uint(BIG);
    const float inv = kv_rcp(s), mz = fmaf(-lo, inv, BIG);
    float off = fabsf(fmaf(-lo, inv, BIG - mz));
    const float base = fminf(mz, BIG + 15.0f);
    uint32_t sum = 0;
#pragma unroll
    for (int k = 0; k < CPL; ++k) {
        float x[2];
        widen2<BF16>(v.w[k / 2], x[0], x[1]);
        const float m = fmaf(x[k & 1], inv, base);
        off = fmaxf(off, fabsf(fmaf(x[k & 1], inv, base - m)));
        sum += min(__float_as_uint(m), big + 15u) << (4 * k);
    }
    const bool none = bad || s == 0.0f;
    codes = none ? 0u : sum - big * (0x11111111u >> (32 - 4 * CPL));
    word = bad ? 0x7fc00000u : (none ? 0u : __float_as_uint(s) | (__float_as_uint(base) - big));
    return !none && (off > 0.49999f || s < 0x1p-100f);  // (no use of 1 / s below)
}
template <int CPL, bool BF16>
__device__ __forceinline__ void kv_quantise_near(KvVec<CPL> v, uint32_t &codes, uint32_t &word, float lo, float s) {
    const int zero = min(15, max(0, (int)rint(-(double)lo / (double)s)));
    word = __float_as_uint(s) | (uint32_t)zero;
    codes = 0;
#pragma unroll 1
    for (int k = 0; k < CPL; ++k) {  // (rolled: one copy of the division)
        float x, next;
        widen2<BF16>(v.w[0], x, next);
        codes |= (uint32_t)min(15, max(0, (int)rint((double)x / (double)s) + zero)) << (4 * k);
#pragma unroll
        for (int i = 0; i < CPL / 2; ++i) v.w[i] = __funnelshift_r(v.w[i], i + 1 < CPL / 2 ? v.w[i + 1] : 0u, 16);
    }
}

template <int D, int GROUP, bool BF16, int CPL>
__global__ void __launch_bounds__(KV_THREADS, CPL == D / 32 ? 7 : 6) kv4_append_kernel(const KvCache c, const KvRows r) {
    // Many rows: eight channels of a lane, so what a group costs whatever its size (its range over the lanes, its scale, its zero point) is paid for
    // several at once, as a warp takes 256 / D tokens at a time (one token of a warp: 111 us; six CTAs of an SM, 85 registers: 94 -> 88).
    // Few rows, so that a block looks for one: all lanes for the one token that there is, a shorter way (64 tokens of 32 heads, with the read
    // behind it: 12.0 -> 10.2 us; seven CTAs of an SM, or the 2048 of them take three waves).
    constexpr int LPT = D / CPL, TPW = 32 / LPT, GL = GROUP / CPL, GROUPS = D / GROUP;  // lanes of a token, tokens of a warp, lanes of a group
    constexpr int OUT = CPL / TPW;                                                      // words of V codes that a lane stores
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, t = threadIdx.x >> 5, h = blockIdx.y, sub = lane / LPT;
    constexpr int tile_bytes = kv_tile_bytes(D, GROUPS);
    const int ch = lane % LPT * CPL, g = ch / GROUP;
    const bool writes = lane % GL == 0;
    int out = 0;  // first of its channels whose word of V codes this lane stores
#pragma unroll
    for (int d = LPT, have = CPL / 2; d < 32; d *= 2, have /= 2) out += lane & d ? have : 0;
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
        // (rolled, with the next token's values under way: unrolled the code does not fit the instruction cache)
        auto tok_of = [&](int i) { return 8 * (i >> 1) + 2 * t + (i & 1); };
        auto ask = [&](int i, KvVec<CPL> &kx, KvVec<CPL> &vx) {
            const int n = tok_of(i) - tok0;
            const bool on = i < 8 && n >= 0 && n < run.n;
            kx = kv_load<CPL>(r.k, (long long)(first + n) * r.ldk + (long long)h * D + ch, on);
            vx = kv_load<CPL>(r.v, (long long)(first + n) * r.ldv + (long long)h * D + ch, on);
        };
        KvVec<CPL> kx[2], vx[2];
        ask(sub, kx[0], vx[0]);
        ask(sub + TPW, kx[1], vx[1]);
        const int page = kv_page(c, run.seq, run.pos);
        if (page < 0) continue;
        unsigned char *tile = kv_tile(c, page, h, run.pos, tile_bytes);
        uint32_t *kw = reinterpret_cast<uint32_t *>(tile + kv_k_words(D)) + g * KV_TILE, *vw = reinterpret_cast<uint32_t *>(tile + kv_v_words(D, GROUPS)) + g * KV_TILE;
        uint32_t *vcodes = reinterpret_cast<uint32_t *>(tile + kv_v_codes(D));
        uint32_t old[OUT], vcode[CPL];
#pragma unroll
        for (int k = 0; k < OUT; ++k) old[k] = mask == 0xffffffffu ? 0u : __ldcg(vcodes + kv_v_word(ch + out + k, t)) & ~mask;
#pragma unroll
        for (int k = 0; k < CPL; ++k) vcode[k] = 0;
#pragma unroll 1
        for (int i = sub; i < 8; i += TPW) {  // (as often in all lanes)
            const KvVec<CPL> k0 = kx[0], v0 = vx[0];
            kx[0] = kx[1];
            vx[0] = vx[1];
            ask(i + 2 * TPW, kx[1], vx[1]);
            const int tok = tok_of(i);
            const bool on = tok >= tok0 && tok < tok0 + run.n;
            if (!__any_sync(0xffffffffu, on)) continue;
            // (nothing but zeros where there is no token)
            uint32_t kc, vc, kword, vword;
            float klo, ks, vlo, vs;
            const bool knear = kv_quantise<CPL, GL, BF16>(k0, kc, kword, klo, ks), vnear = kv_quantise<CPL, GL, BF16>(v0, vc, vword, vlo, vs);
            if (knear) kv_quantise_near<CPL, BF16>(k0, kc, kword, klo, ks);
            if (vnear) kv_quantise_near<CPL, BF16>(v0, vc, vword, vlo, vs);
            if (on) {
                unsigned char *to = tile + tok * (D / 2) + kv_k_byte(D, ch);
                if constexpr (CPL == 2) *to = (unsigned char)kc;
                else if constexpr (CPL == 4) *reinterpret_cast<unsigned short *>(to) = (unsigned short)kc;
                else *reinterpret_cast<uint32_t *>(to) = kc;
            }
            if (on && writes) {
                kw[kv_word_at(tok)] = kword;
                vw[kv_word_at(tok)] = vword;
            }
            const int nib = 4 * ((i >> 1) + 4 * (i & 1));
#pragma unroll
            for (int k = 0; k < CPL; ++k) vcode[k] |= ((vc >> (4 * k)) & 15u) << nib;
        }
        // The tokens of a word from all lanes that have some; each keeps the words that it stores.
#pragma unroll
        for (int d = LPT, have = CPL / 2; d < 32; d *= 2, have /= 2)
#pragma unroll
            for (int k = 0; k < have; ++k) {
                const bool upper = lane & d;
                const uint32_t away = __shfl_xor_sync(0xffffffffu, upper ? vcode[k] : vcode[k + have], d);
                vcode[k] = (upper ? vcode[k + have] : vcode[k]) | away;
            }
#pragma unroll
        for (int k = 0; k < OUT; ++k) vcodes[kv_v_word(ch + out + k, t)] = vcode[k] | old[k];
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
    if (append && r.per_block > 1)
        return bf16 ? launch(kv4_append_kernel<D, GROUP, true, 8>, grid, block, 0, st, pdl, c, r) : launch(kv4_append_kernel<D, GROUP, false, 8>, grid, block, 0, st, pdl, c, r);
    if (append)
        return bf16 ? launch(kv4_append_kernel<D, GROUP, true, D / 32>, grid, block, 0, st, pdl, c, r) : launch(kv4_append_kernel<D, GROUP, false, D / 32>, grid, block, 0, st, pdl, c, r);
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
