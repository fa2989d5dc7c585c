// Attention of new tokens over the 4-bit cache: out = softmax(scale q k^T + mask) v, one to sixteen new tokens per sequence.
//
// The rows of a key head (its query heads x the new tokens) are the N columns of mma.m16n8k16, eight at a time (RN = 1 or 2 such groups), and
// the codes its A operand: tokens are the M rows of the scores, channels those of the output.  The cache is dequantised by nothing but a
// mask: a code is an fp16 subnormal (see scap_kv4.cuh), and what belongs to a group of channels is applied once per token:
//   scores  s_t = ks_t (sum_c q_c code_tc - zero_t sum_c q_c), the second sum by one more MMA with the zero points as codes
//   output  o_c = sum_t (p_t vs_t) code_tc - sum_t (p_t vs_t) zero_t, likewise.
// p vs is rounded to fp16 (11 bits) once and used in both sums, so the rounding acts on the value v, not on its code part; its size is kept by a
// reference per row (below).  The queries are scaled by a power of two per row and are exact.  Scores, references, sums and accumulators are fp32.
// (With the rows as the M rows of the MMA a head with eight or fewer of them pays for sixteen: twice the MMAs, accumulators and
// exponentials; 131001 tokens, 8 key heads, 8 rows: 57 us against 45 at that time.)
//
// What bounds it: latency inside a warp, with four warps per scheduler to cover it; no unit is saturated.  The bytes of the cache are D/2 + 4 groups per token, head
// and side; per tile of 32 tokens (D = 128, RN = 1, one group) a warp issues about 600 instructions, 36 of them MMAs and 192 masks and shifts - six for eight codes, and the
// pipe that runs them takes two cycles each.  48 sequences of together 196608 tokens, 8 key heads, groups of 64: 73 us at 228 MB = 3.1 TB/s, issue slots
// 57 % busy with 1.1 of 3.6 warps ready, the mask pipe 45 %, tensor pipe 20 %, DRAM 40 %; of 6.3 cycles between two instructions of a warp 1.5 go to results of fixed latency,
// 1.0 to other warps, 0.7 to the mask pipe, 0.6 to memory.  131001 tokens of one sequence, groups of 128: 40 us at 143 MB = 3.6 TB/s.  With
// the copies alone, no arithmetic, these took 48 and 33 us: 4 to 6 us until the first tiles of all warps have come, then 5.7 TB/s.
//
// Work is cut into equal parts, whatever the lengths: a unit is one tile of 32 tokens of one (sequence, 8 RN rows, head), all units are
// numbered, and worker i of w takes the units [U i / w, U (i + 1) / w).  A worker is a CTA: the tiles of an item go round its four warps,
// each of which has its own ring of tiles, filled by cp.async.bulk (one copy per tile, 4.3 KB at D = 128), its own running maximum and sum, and no
// barrier with the others until the item ends.  Or (SOLO), with many items, a warp.  An item that lies in one worker is finished there; the
// parts of one that is cut go to the workspace, and a second kernel joins them in order.  No atomics: the same bits each time.
// (Tried and slower: the first tiles of the next item asked for while the last ones of the present one are worked on: 77 -> 85 us, the loop
// over tiles pays for it; a fifth CTA per SM: the same; the shifts as multiplications on the idle pipe: 77 -> 82.)
//
// Every wait is bounded; one that runs out sets the status word and leaves its tile out.
#include "scap_kv4.cuh"

namespace scap {

constexpr int AT_WARPS = 4;
constexpr int AT_THREADS = AT_WARPS * 32;
constexpr int AT_MIN_UNITS = 4;  // tiles per CTA, one for each warp, unless the items are shorter: an item after another takes 4 us each
// The reference m of a row is such that a weight p = 2^(s - m) times the scale of its value (exponent field e: 2^(e - 127) .. 2^(e - 126)) times 2^-24 is
// 2^10 .. 2^11 for the largest product seen, s + e = m + AT_TOP, and it moves when one would reach 2^15, s + e > m + AT_MOST.  (With 2^-24 the weights of values
// as large as binary32 holds are still 33 bits above 2^-126, where 2^x becomes 0.)  A scale below 2^-56 counts as 2^-56 here, so that weights stay below
// 2^94 and the sum of any number of them is finite.
constexpr float AT_TOP = 161.0f, AT_MOST = 165.0f, AT_DOWN = 0x1p-24f;
constexpr uint32_t AT_LEAST = 71u << 23;

// CTAs per SM and tiles in a warp's ring, as registers and shared memory allow (RN groups of eight rows, G groups of channels).
__host__ __device__ constexpr int at_resident(int D, int G, int RN) {
    return D == 64 ? (RN == 1 ? 5 : 4) : (D == 128 ? (RN == 1 && G < 4 ? 4 : 3) : (RN == 1 ? 3 : 2));
}
__host__ __device__ constexpr int at_stages(int D, int G, int RN) {
    return D == 64 ? 4 : (D == 128 ? 3 : 2);
}

struct AtArgs {
    KvCache c;
    const unsigned short *q;
    unsigned short *out;
    float *lse;
    long long ldq, ldo;   // elements between tokens
    float *part, *ml;     // parts of items that were cut, two per worker: [8 RN][D] weighted sums, [8 RN][2] reference and sum
    int2 *where;          // [n_seqs][items]: first and last worker of an item that was cut, equal where it was not
    int nq, g, row_tiles, window;
    float scale;          // times log2 e
    int tile_cap;         // tiles that a row of the table has room for
    int resident, waves;  // CTAs that the device holds at once, and how many times that there may be
    bool bf16;
    uint32_t limit;
    int *status;
};

// Tiles that a warp adds up in its accumulators before it puts the sums where parts go and begins anew.  The tensor core truncates as it adds: a sum of n
// numbers of one sign is off by up to n 2^-23 of itself, and code and zero-point part of an output are two such sums whose difference may be small (the mean of
// 400000 values, a third of them in each warp, was off by 4.7 % of itself; with 256 tiles by 1.0e-3, with 128 by less than the two roundings to 11 bits allow).  Only warps with
// so many tiles of one item pay for it: 120 sequences of 100000 tokens, 8 key heads: 3763 -> 3865 us (256 tiles: 3811, 64: 3961).
constexpr int AT_RUN = 128;

// What a warp is at: units [u, u1) of its worker `id`.  Tiles t0 .. t1 - 1 of an item of sequence seq are next, a stretch of the tiles i0 .. i1 - 1 that the
// worker has of it.
struct AtWork {
    long long u, u1, base;
    int id, seq, len, item, tiles, t0, t1, i0, i1;
};

// Tiles that the new tokens of a sequence of `len` tokens can see: first one and number.
__device__ __forceinline__ int at_tiles_of(const AtArgs &a, int len, int &first) {
    first = 0;
    if (len <= 0) return 0;
    if (a.window > 0) {
        const long long lo = (long long)len - a.nq + 1 - a.window;  // of the first new token
        first = lo > 0 ? (int)(lo / KV_TILE) : 0;
    }
    // (what a table has no room for is not seen)
    return max(0, min((int)(((long long)len + KV_TILE - 1) / KV_TILE), a.tile_cap) - first);
}

__device__ __forceinline__ long long at_cut(long long units, int i, int workers) { return units * i / workers; }
// CTAs that share the units, and workers in them: the CTA, or (SOLO) each of its warps.  Where there is much to do there are twice as many CTAs as
// the device holds: the SMs favour the older ones of their CTAs, and the younger ones of a second wave take over from those.  It helps where CTAs end items
// of their own (us with one wave and two, 128 channels, 80 units per resident CTA; 70 sequences: 85 and 80, 32: 74 and 72, 16: 68 and 67) and costs the time of the
// more and shorter parts where few items are cut into many (8: 59 and 65, one: 58 and 67), so it takes half as many items as there are resident CTAs.  With
// less to do it varies (20 to 60 units, 48 and 70 sequences: from 12 better to 9 worse).
constexpr int AT_TWO_WAVES = 64;  // units per resident CTA
__host__ __device__ constexpr bool at_two_waves(long long units, long long items, int resident) { return units >= (long long)AT_TWO_WAVES * resident && 2 * items >= resident; }
template <bool SOLO>
__device__ __forceinline__ int at_workers(const AtArgs &a, long long units, long long items, int &ctas) {
    constexpr int PER = SOLO ? AT_WARPS : 1;
    const long long n = max((units + AT_MIN_UNITS - 1) / AT_MIN_UNITS, items);
    const int most = at_two_waves(units, items, a.resident) ? a.waves * a.resident : a.resident;
    const int workers = n < (long long)PER * most ? (int)n : PER * most;
    ctas = min(most, workers);  // (SOLO: worker w is warp w / ctas of CTA w % ctas, so that few of them lie in different CTAs)
    return workers;
}

__device__ __forceinline__ int at_tiles(const AtArgs &a, int b, int &first) { return at_tiles_of(a, __ldcg(a.c.lens + b), first); }

// Number of tiles of all sequences, and of the sequences that have any (the whole block takes part).
__device__ __forceinline__ long long at_count(const AtArgs &a, long long *s, int &some) {
    long long all = 0;
    some = 0;
    for (int b0 = 0; b0 < a.c.n_seqs; b0 += AT_THREADS) {
        const int b = b0 + (int)threadIdx.x;
        int first;
        const int n = b < a.c.n_seqs ? at_tiles(a, b, first) : 0;
        all += n;
        some += __syncthreads_count(n > 0);
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) all += __shfl_xor_sync(0xffffffffu, all, o);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = all;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int w = 0; w < AT_WARPS; ++w) all += s[w];
    __syncthreads();
    return all;
}

// The units of a worker, the number of the worker, the sequence that its first unit belongs to, that sequence's length and first unit.
struct AtPlace {
    long long u, u1, base;
    int id, seq, len;
};
// This worker's place (the whole block takes part); per = items per sequence.  False: there is nothing for this CTA.
template <bool SOLO>
__device__ __forceinline__ bool at_begin(const AtArgs &a, int per, long long *s, AtPlace &p) {
    constexpr int PER = SOLO ? AT_WARPS : 1;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long units = 0, before = 0;
    const bool one = a.c.n_seqs <= AT_THREADS;  // one look at the lengths gives the sum and the place
    int some = 0, ctas = 0, workers = 0;
    if (!one) units = at_count(a, s, some) * per;
    for (int b0 = 0; b0 < a.c.n_seqs; b0 += AT_THREADS) {
        const int b = b0 + (int)threadIdx.x;
        int first;
        const int tokens = b < a.c.n_seqs ? __ldcg(a.c.lens + b) : 0;
        const long long n = (long long)at_tiles_of(a, tokens, first) * per;
        long long incl = n;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const long long up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 31) s[warp] = incl;
        const int here = __syncthreads_count(n > 0);
        if (one) some = here;
        long long off = before, all = before;
#pragma unroll
        for (int w = 0; w < AT_WARPS; ++w) {
            if (w < warp) off += s[w];
            all += s[w];
        }
        if (one) units = all;
        workers = at_workers<SOLO>(a, units, (long long)some * per, ctas);
        if ((int)blockIdx.x >= ctas) return false;
        // (SOLO: a cut is moved to a border between items that lies within half a share of it, so that short items stay whole)
        const long long near = SOLO ? units / workers / 2 : 0, tiles = per > 0 ? n / per : 0;
        long long last = 0;
#pragma unroll
        for (int w = 0; w < PER; ++w)
#pragma unroll
            for (int e = 0; e < (SOLO ? 2 : 1); ++e) {
                const int id = (int)blockIdx.x + w * ctas + e;
                if (id >= workers) break;
                const long long u = at_cut(units, id, workers);
                if (n > 0 && off + incl - n <= u && u < off + incl) {
                    long long moved = u;
                    if (SOLO) {
                        const long long over = (u - (off + incl - n)) % tiles;
                        moved = over <= near ? u - over : (tiles - over <= near ? u + tiles - over : u);
                    }
                    if (e == 0) {
                        s[AT_WARPS + 5 * w] = b;
                        s[AT_WARPS + 5 * w + 1] = off + incl - n;
                        s[AT_WARPS + 5 * w + 2] = tokens;
                    }
                    s[AT_WARPS + 5 * w + 3 + e] = moved;
                }
                last = u;
            }
        before = all;
        __syncthreads();
        if (last < before) break;
    }
    const int w = SOLO ? warp : 0;
    p.id = (int)blockIdx.x + w * ctas;
    p.u = p.u1 = 0;
    p.seq = p.len = 0;
    p.base = 0;
    if (p.id < workers) {
        p.u = s[AT_WARPS + 5 * w + 3];
        p.u1 = p.id + 1 == workers ? units : (SOLO ? s[AT_WARPS + 5 * w + 4] : at_cut(units, p.id + 1, workers));
        p.seq = (int)s[AT_WARPS + 5 * w];
        p.base = s[AT_WARPS + 5 * w + 1];
        p.len = (int)s[AT_WARPS + 5 * w + 2];
    }
    return true;
}

__device__ __forceinline__ void at_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Transposes an 8 x 8 matrix of 16-bit elements, two neighbours of a row per lane.
__device__ __forceinline__ uint32_t at_trans(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
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
// x 2^d for d <= 0, in two steps: 2^d alone is 0 below -126, where a sum of weights may have 94 bits to spare
__device__ __forceinline__ float at_lower(float x, float d) {
    const float h = at_ex2(0.5f * d);
    return x * h * h;
}
__device__ __forceinline__ float at_widen(unsigned short u, bool bf16) { return bf16 ? widen_bits<true>(u) : widen_bits<false>(u); }
__device__ __forceinline__ void at_store(unsigned short *p, float v, bool bf16) {
    *p = bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}
// 2^e for -126 <= e <= 127
__device__ __forceinline__ float at_pow2(int e) { return __int_as_float((e + 127) << 23); }

// Adds the sums of the stretches before to those that a warp has put into shared memory, for the rows own, own + STEP, ... that this warp puts out (and put
// where parts go, a channel the same lane).  Out of line: in line it costs the loop over tiles registers (four new tokens of 32 key heads: 80 -> 82 us).
// The codes of a word as pairs of subnormal numbers.  Of the products that it adds at a time the tensor core drops what lies below 2^-24 of the largest exponent, and a subnormal
// number counts with 2^-14 there, so codes lie as high as one shift for each half of a word puts them: 2^-22 and 2^-18.  (At 2^-24 and 2^-20, without the first shift,
// sums lose four times as much: 15 others added with a token of nine tenths of the weight were off by 2^-13 of its scale together; 72.6 -> 75.9 us for 48 sequences of 196608 tokens.)
constexpr uint32_t AT_LOW = 0x003c003cu, AT_HIGH = 0x03c003c0u;
__device__ __forceinline__ uint32_t at_place(uint32_t w, int second) { return second ? w >> 6 : w << 2; }

template <int D, int STEP, int PITCH>
__device__ __noinline__ void at_fold(int own, int rows, int lane, float *part, float *s_m, float *s_l, const float *sums, const float *ml) {
    __syncwarp();
#pragma unroll 1
    for (int row = own; row < rows; row += STEP) {
        const float had = ml[2 * row], had_l = ml[2 * row + 1], now = s_m[row], now_l = s_l[row], top = fmaxf(now, had), ref = top == -INFINITY ? 0.0f : top;
        const float w_now = at_ex2(now - ref), w_had = at_ex2(had - ref);
#pragma unroll 1
        for (int c = lane; c < D; c += 32) {
            const float x = part[row * PITCH + c], y = sums[row * D + c];
            part[row * PITCH + c] = (w_now > 0.0f || x != x ? w_now * x : 0.0f) + (w_had > 0.0f || y != y ? w_had * y : 0.0f);
        }
        __syncwarp();
        if (lane == 0) {
            s_m[row] = top;
            s_l[row] = at_lower(now_l, now - ref) + at_lower(had_l, had - ref);
        }
    }
}

template <int D, int G, int RN, bool SOLO>
__global__ void __launch_bounds__(AT_THREADS, at_resident(D, G, RN)) kv4_attend_kernel(const AtArgs a) {
    constexpr int W = D / 32;            // words of a K row per lane
    constexpr int TILE = kv_tile_bytes(D, G);
    constexpr int ST = at_stages(D, G, RN);
    constexpr int MT = D / 16;           // blocks of sixteen channels
    constexpr int ROWS = 8 * RN;
    constexpr int PITCH = D + 4;         // of a row of the join
    constexpr float LN2 = 0.69314718055994531f;
    static_assert(ST * TILE >= ROWS * PITCH * 4, "a warp's part of the join goes where its ring was");
    // Sixteen rows: the queries are B operands in shared memory, one 16-byte load for two MMAs, where their registers would spill.
    constexpr bool QS = RN == 2;
    static_assert(!(SOLO && QS), "a warp on its own has its queries in registers");
    constexpr int STEP = SOLO ? 1 : AT_WARPS;  // the tiles of an item go round so many warps
    extern __shared__ __align__(128) unsigned char at_raw[];
    uint4 *s_q = reinterpret_cast<uint4 *>(at_raw + AT_WARPS * ST * TILE);  // [RN][W][32 lanes]
    __shared__ uint32_t s_zq[QS ? RN : 1][G][32];
    // What turns an accumulator of a row into a score in units of log 2, by warp (QS: by eight rows).  Read once per tile: in registers, one more of them
    // than before, the kernel for 256 channels spilled (300 sequences of together 30000 tokens, 8 key heads: 66 -> 82 us).
    __shared__ __align__(8) float s_f[QS ? RN : AT_WARPS][8];
    __shared__ unsigned long long s_full[AT_WARPS][ST];
    __shared__ long long s_sum[AT_WARPS + 5 * (SOLO ? AT_WARPS : 1)];
    __shared__ float s_m[AT_WARPS][ROWS], s_l[AT_WARPS][ROWS];
    __shared__ AtWork s_work[AT_WARPS];

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, qg = lane >> 2, qt = lane & 3;
    unsigned char *ring = at_raw + warp * ST * TILE;
    if (lane == 0)
        for (int i = 0; i < ST; ++i) mbarrier_init(smem_addr(&s_full[warp][i]), 1);
    __syncthreads();
    griddep_wait();
    griddep_launch_dependents();  // (after the wait: the second kernel may rely on all work before this one)

    const int per = a.c.heads * a.row_tiles;
    // What a warp is at lives in shared memory: none of it is needed while it goes through its tiles, whose registers are scarce.
    volatile AtWork &work = s_work[warp];
    {
        AtPlace place;
        if (!at_begin<SOLO>(a, per, s_sum, place)) return;
        if (lane == 0) {
            work.u = place.u;
            work.u1 = place.u1;
            work.base = place.base;
            work.id = place.id;
            work.t1 = work.i1 = 0;
            work.seq = place.seq;
            work.len = place.len;
        }
        __syncwarp();
    }
    int slot = 0, phase = 0;  // of this warp's ring, over all items
    bool dead = false;        // a wait of this warp ran out
    const int own = SOLO ? 0 : warp;  // this warp's first tile of those that its worker has of an item

    while (work.u < work.u1) {
        const int len = work.len;
        int count, pos0;
        {
            int first_tile;
            const int tiles = at_tiles_of(a, len, first_tile);
            const long long in_seq = work.u - work.base;
            if (in_seq >= (long long)tiles * per) {  // the next sequence (an empty one has no units; its rows are the second kernel's)
                const int next = __ldcg(a.c.lens + work.seq + 1);
                __syncwarp();
                if (lane == 0) {
                    work.base += (long long)tiles * per;
                    work.seq += 1;
                    work.len = next;
                }
                __syncwarp();
                continue;
            }
            const int item = (int)(in_seq / tiles), t0 = (int)(in_seq - (long long)item * tiles);
            const int i1 = (int)min((long long)tiles, t0 + (work.u1 - work.u)), t1 = min(i1, t0 + AT_RUN * STEP);
            count = !dead && t1 - t0 - own > 0 ? (t1 - t0 - own + STEP - 1) / STEP : 0;  // tiles t0 + own, + STEP, ... are this warp's
            pos0 = (first_tile + t0 + own) * KV_TILE;
            if (lane == 0) {
                work.item = item;
                work.tiles = tiles;
                if (work.t1 == work.i1) work.i0 = t0;  // (else the stretch before this one ended inside the item)
                work.i1 = i1;
                work.t0 = t0;
                work.t1 = t1;
            }
            __syncwarp();
        }

        // ---- addresses of the next 32 tiles of this warp, one per lane (0: no page), and the first copies
        auto where = [&](int i) -> unsigned long long {
            if (i >= count) return 0ull;
            const int per_page = a.c.page_tokens / KV_TILE, t = pos0 / KV_TILE + STEP * i, at = t / per_page;
            if (at >= a.c.table_stride) return 0ull;
            const int page = __ldcg(a.c.table + (long long)work.seq * a.c.table_stride + at);
            if (page < 0 || page >= a.c.n_pages) return 0ull;
            const int h = work.item % a.c.heads;
            return (unsigned long long)(a.c.pages + (long long)page * a.c.page_stride + (long long)(h * per_page + t - at * per_page) * TILE);
        };
        unsigned long long at_now = where(lane), at_next = where(32 + lane);
        unsigned there = __ballot_sync(0xffffffffu, at_now != 0);  // which of the present 32 tiles have a page
        auto ask = [&](unsigned long long src, int st) {  // by the lane that has the address
            const uint32_t bar = smem_addr(&s_full[warp][st]);
            if (src) {
                mbarrier_arrive_expect(bar, TILE);
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_addr(ring + st * TILE)), "l"(src), "r"(TILE), "r"(bar)
                             : "memory");
            } else {
                asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");  // the tile is empty
            }
        };
        // (the first tile alone: those of all warps of the device are then under way before anybody's second)
        if (lane == 0 && count > 0) ask(at_now, slot);

        // ---- queries: rows 8 rn + qg as B operands, each scaled by a power of two of its own so that its largest channel lies in 2^11 .. 2^12 (a
        // row does not depend on those it is taken with); channels 32 j + 8 qt + i, the
        // even and odd nibbles of a code word in the two k halves of an MMA, the odd ones 16 times smaller as their codes are larger: a channel is exact
        // down to 2^-21 of the largest of its row, and off by 2^-32 of that below.
        // zq: minus the sum of a group, in two fp16 parts, against the zero points (times 2^4, as zero 2^-18 is the subnormal used and code 2^-22 the other)
        uint32_t qb[QS ? 1 : 2 * W][2], zq[QS ? 1 : G];
        if (!QS || warp < RN) {  // (in shared memory: warp rn for its eight rows)
            const int rn = QS ? warp : 0, row = 8 * rn + qg;
            uint4 raw[W];
            const int rt = work.item / a.c.heads, h = work.item - rt * a.c.heads, in = rt * ROWS + row, tok = in / a.g, hd = in - tok * a.g;
            const unsigned short *src = a.q + ((long long)work.seq * a.nq + tok) * a.ldq + (long long)(h * a.g + hd) * D + 8 * qt;
#pragma unroll
            for (int j = 0; j < W; ++j) raw[j] = ld_act16_if(src + 32 * j, in < a.nq * a.g);
            float v[W][8], top = 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t w = (&raw[j].x)[i >> 1];
                    v[j][i] = at_widen((unsigned short)(i & 1 ? w >> 16 : w), a.bf16);
                    top = fmaxf(top, fabsf(v[j][i]));
                }
            if (!(top < INFINITY)) top = 0.0f;  // (a row that is not finite stays so, whatever its scale)
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));  // of the four lanes that have the row
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = top > 0.0f ? min(126, 11 - ((__float_as_int(top) >> 23) - 127)) : 0;  // at least -116
            const float up = at_pow2(e), up16 = up * 0.0625f;
            float sum[G];
#pragma unroll
            for (int n = 0; n < G; ++n) sum[n] = 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j) {
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[j * G / W] = fmaf(v[j][i], up, sum[j * G / W]);
                uint32_t w[2][2];
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) {
                    w[hi][0] = at_pack(v[j][2 * hi] * up, v[j][2 * hi + 4] * up);
                    w[hi][1] = at_pack(v[j][2 * hi + 1] * up16, v[j][2 * hi + 5] * up16);
                    if constexpr (!QS) { qb[2 * j + hi][0] = w[hi][0]; qb[2 * j + hi][1] = w[hi][1]; }
                }
                if constexpr (QS) s_q[(rn * W + j) * 32 + lane] = make_uint4(w[0][0], w[0][1], w[1][0], w[1][1]);
            }
#pragma unroll
            for (int n = 0; n < G; ++n) {
                sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 1);
                sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 2);
                const float x = -sum[n] * 0.0625f, x_hi = __half2float(__float2half_rn(x));
                if constexpr (QS) s_zq[rn][n][lane] = at_pack(x_hi, x - x_hi);
                else zq[n] = at_pack(x_hi, x - x_hi);
            }
            const float back = a.scale * at_pow2((22 - e) / 2) * at_pow2(22 - e - (22 - e) / 2);
            if (qt == 0) s_f[warp][qg] = back;
            __syncwarp();
        }
        if (lane > 0 && lane < ST && lane < count) ask(at_now, slot + lane < ST ? slot + lane : slot + lane - ST);
        if constexpr (QS) __syncthreads();
        // keys that row 8 rn + 2 qt + k sees: up to that of its own token, hi, and with a window from lo on
        uint32_t tok_of[RN];
#pragma unroll
        for (int rn = 0; rn < RN; ++rn) {
            const int in = work.item / a.c.heads * ROWS + 8 * rn + 2 * qt, last = a.nq * a.g - 1;
            tok_of[rn] = (uint32_t)(min(in, last) / a.g) | (uint32_t)(min(in + 1, last) / a.g) << 16;
        }
        auto unseen = [&](int at, int rn, int k) {
            const int hi = len - a.nq + (int)((tok_of[rn] >> (16 * k)) & 0xffffu);
            return at > hi || (a.window > 0 && at <= hi - a.window);
        };
        const int hi_all = len - a.nq, lo_all = a.window > 0 && len > a.window ? len - a.window : 0;  // what every row sees

        float o[RN][MT][4], z[RN][G][4], m[RN][2], l[RN][2];
#pragma unroll
        for (int rn = 0; rn < RN; ++rn) {
#pragma unroll
            for (int n = 0; n < MT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[rn][n][i] = 0.0f;
#pragma unroll
            for (int n = 0; n < G; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[rn][n][i] = 0.0f;
            m[rn][0] = m[rn][1] = -INFINITY;
            l[rn][0] = l[rn][1] = 0.0f;
        }

        const uint32_t zmask = qt == 0 ? 15u : 0u;
        for (int i = 0; i < count; ++i) {
            const uint32_t bar = smem_addr(&s_full[warp][slot]);
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
            const int pos = pos0 + STEP * KV_TILE * i;
            if ((there >> (i & 31)) & 1u) {
                // keys that not every row sees: tokens behind the last, before a window, or newer than the row's own
                const bool edge = pos + KV_TILE - 1 > hi_all || pos < lo_all;
                // ---- scores: s[rn][j][k] is row 8 rn + 2 qt + k at token 8 j + qg.  The four blocks of eight tokens are two A operands.
                float s[RN][4][2];
                uint32_t kw[G][4];
#pragma unroll
                for (int n = 0; n < G; ++n)
                    *reinterpret_cast<uint4 *>(kw[n]) = *reinterpret_cast<const uint4 *>(tile + kv_k_words(D) + (n * KV_TILE + 4 * qg) * 4);
                // (MB of the two A operands at a time: the chains of MMAs are independent, but their registers are scarce)
                constexpr int MB = G <= 2 ? 2 : 1;
#pragma unroll
                for (int m0 = 0; m0 < 2; m0 += MB) {
                    float acc[MB][RN][G][4];
                    uint32_t w[2 * MB][W];
#pragma unroll
                    for (int j = 0; j < 2 * MB; ++j) {
                        const unsigned char *krow = tile + (8 * (2 * m0 + j) + qg) * (D / 2) + qt * (D / 8);
                        if constexpr (W == 2) *reinterpret_cast<uint2 *>(w[j]) = *reinterpret_cast<const uint2 *>(krow);
                        else
#pragma unroll
                            for (int k = 0; k < W / 4; ++k) *reinterpret_cast<uint4 *>(w[j] + 4 * k) = *reinterpret_cast<const uint4 *>(krow + 16 * k);
                    }
#pragma unroll
                    for (int n = 0; n < G; ++n)
#pragma unroll
                        for (int mt = 0; mt < MB; ++mt) {
                            const uint32_t z0 = (kw[n][2 * (m0 + mt)] & zmask) * 0x00400040u, z1 = (kw[n][2 * (m0 + mt) + 1] & zmask) * 0x00400040u;
#pragma unroll
                            for (int rn = 0; rn < RN; ++rn) {
#pragma unroll
                                for (int k = 0; k < 4; ++k) acc[mt][rn][n][k] = 0.0f;
                                at_mma(acc[mt][rn][n], z0, z1, 0u, 0u, QS ? s_zq[QS ? rn : 0][n][lane] : zq[QS ? 0 : n], 0u);
                            }
                        }
                    // (the words of a group lie W / G apart from those of the next: in turn, so that neighbouring MMAs have different accumulators)
#pragma unroll
                    for (int kk = 0; kk < W; ++kk) {
                        const int k = kk % G * (W / G) + kk / G;
                        uint32_t q[RN][2][2];
#pragma unroll
                        for (int rn = 0; rn < RN; ++rn) {
                            if constexpr (QS) {
                                const uint4 x = s_q[(rn * W + k) * 32 + lane];
                                q[rn][0][0] = x.x; q[rn][0][1] = x.y; q[rn][1][0] = x.z; q[rn][1][1] = x.w;
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i) q[rn][i >> 1][i & 1] = qb[2 * k + (i >> 1)][i & 1];
                            }
                        }
#pragma unroll
                        for (int hi8 = 0; hi8 < 2; ++hi8)
#pragma unroll
                            for (int mt = 0; mt < MB; ++mt) {
                                const uint32_t x = at_place(w[2 * mt][k], hi8), y = at_place(w[2 * mt + 1][k], hi8);
                                const uint32_t a0 = x & AT_LOW, a1 = y & AT_LOW, a2 = x & AT_HIGH, a3 = y & AT_HIGH;
#pragma unroll
                                for (int rn = 0; rn < RN; ++rn) at_mma(acc[mt][rn][k * G / W], a0, a1, a2, a3, q[rn][hi8][0], q[rn][hi8][1]);
                            }
                    }
#pragma unroll
                    for (int j = 0; j < 2 * MB; ++j)
#pragma unroll
                        for (int n = 0; n < G; ++n) {
                            const float ks = __uint_as_float(kw[n][2 * m0 + j] & ~15u);
#pragma unroll
                            for (int rn = 0; rn < RN; ++rn)
#pragma unroll
                                for (int k = 0; k < 2; ++k) {
                                    const float x = acc[j >> 1][rn][n][2 * (j & 1) + k];
                                    s[rn][2 * m0 + j][k] = n == 0 ? ks * x : fmaf(ks, x, s[rn][2 * m0 + j][k]);
                                }
                        }
                }
#pragma unroll
                for (int rn = 0; rn < RN; ++rn) {
                    const float2 f = *reinterpret_cast<const float2 *>(&s_f[QS ? rn : warp][2 * qt]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[rn][j][0] *= f.x;
                        s[rn][j][1] *= f.y;
                    }
                }
                uint32_t vw[G][4];
#pragma unroll
                for (int n = 0; n < G; ++n) *reinterpret_cast<uint4 *>(vw[n]) = *reinterpret_cast<const uint4 *>(tile + kv_v_words(D, G) + (n * KV_TILE + 4 * qg) * 4);
                if (edge) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int at = pos + 8 * j + qg;
#pragma unroll
                        for (int rn = 0; rn < RN; ++rn)
#pragma unroll
                            for (int k = 0; k < 2; ++k)
                                if (unseen(at, rn, k)) s[rn][j][k] = -INFINITY;
                        if (at >= len || at <= lo_all - a.nq) {  // tokens that no row sees have no scale, whatever lies there
#pragma unroll
                            for (int n = 0; n < G; ++n) vw[n][j] = 0;
                        }
                    }
                }
                // ---- reference of a row: by its largest product of a weight and a scale, so that a large value that has next to no weight takes no bits
                // of the others.  It is left as it is while products stay below 2^15, so that the accumulators are rarely rescaled.
                float top[RN][2];
                auto largest = [&](const float (&e)[4]) {
#pragma unroll
                    for (int rn = 0; rn < RN; ++rn)
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            top[rn][k] = fmaxf(fmaxf(s[rn][0][k] + e[0], s[rn][1][k] + e[1]), fmaxf(s[rn][2][k] + e[2], s[rn][3][k] + e[3]));
                };
                float e[4];
                bool fine = true;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t big = AT_LEAST;
#pragma unroll
                    for (int n = 0; n < G; ++n) big = max(big, vw[n][j]);
                    fine = fine && big < 0x7f800000u;
                    e[j] = (float)(big >> 23);
                }
                largest(e);
                bool keep = fine;
#pragma unroll
                for (int rn = 0; rn < RN; ++rn)
#pragma unroll
                    for (int k = 0; k < 2; ++k) keep = keep && !(top[rn][k] > m[rn][k] + AT_MOST);
                if (!__all_sync(0xffffffffu, keep)) {
                    if (!__all_sync(0xffffffffu, fine)) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {  // (a scale that is NaN has no say)
                            uint32_t big = AT_LEAST;
#pragma unroll
                            for (int n = 0; n < G; ++n) big = max(big, vw[n][j] < 0x7f800000u ? vw[n][j] : 0u);
                            e[j] = (float)(big >> 23);
                        }
                        largest(e);
                    }
#pragma unroll
                    for (int rn = 0; rn < RN; ++rn) {
                        float down[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float x = top[rn][k];
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                            const float ref = x > m[rn][k] + AT_MOST ? x - AT_TOP : m[rn][k];  // (every row by itself)
                            const float by = ref == -INFINITY ? 0.0f : m[rn][k] - ref;
                            l[rn][k] = at_lower(l[rn][k], by);
                            down[k] = at_ex2(by);
                            m[rn][k] = ref;
                        }
#pragma unroll
                        for (int n = 0; n < MT; ++n)
#pragma unroll
                            for (int k = 0; k < 4; ++k) o[rn][n][k] *= down[k & 1];
#pragma unroll
                        for (int n = 0; n < G; ++n)
#pragma unroll
                            for (int k = 0; k < 4; ++k) z[rn][n][k] *= down[k & 1];
                    }
                }
                // ---- weights, those of blocks whose codes are 16 times larger as held made 16 times smaller
#pragma unroll
                for (int rn = 0; rn < RN; ++rn)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float ref = m[rn][k] == -INFINITY ? 0.0f : m[rn][k], ref16 = ref + 4.0f;  // nothing seen so far: all weights are 0
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            s[rn][j][k] = at_ex2(s[rn][j][k] - (j & 1 ? ref16 : ref));
                            l[rn][k] = j & 1 ? fmaf(s[rn][j][k], 16.0f, l[rn][k]) : l[rn][k] + s[rn][j][k];
                        }
                    }
                // ---- weighted values: p vs as B operands (a block of eight tokens x eight rows is transposed in registers)
                uint32_t pb[G][RN][4];
#pragma unroll
                for (int n = 0; n < G; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float vs = __uint_as_float(vw[n][j] & ~15u) * AT_DOWN;
#pragma unroll
                        for (int rn = 0; rn < RN; ++rn) pb[n][rn][j] = at_pack(s[rn][j][0] * vs, s[rn][j][1] * vs);
                    }
                if (edge) {  // a row does not see what another one does: not even a NaN
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int rn = 0; rn < RN; ++rn) {
                            const int at = pos + 8 * j + qg;
                            const uint32_t seen = (unseen(at, rn, 0) ? 0u : 0xffffu) | (unseen(at, rn, 1) ? 0u : 0xffff0000u);
#pragma unroll
                            for (int n = 0; n < G; ++n) pb[n][rn][j] &= seen;
                        }
                }
#pragma unroll
                for (int n = 0; n < G; ++n) {
#pragma unroll
                    for (int rn = 0; rn < RN; ++rn)
#pragma unroll
                        for (int j = 0; j < 4; ++j) pb[n][rn][j] = at_trans(pb[n][rn][j]);
                    uint32_t w0[4], w1[4];  // tokens 8 j + 2 qt and the next
                    *reinterpret_cast<uint4 *>(w0) = *reinterpret_cast<const uint4 *>(tile + kv_v_words(D, G) + (n * KV_TILE + 8 * qt) * 4);
                    *reinterpret_cast<uint4 *>(w1) = *reinterpret_cast<const uint4 *>(tile + kv_v_words(D, G) + (n * KV_TILE + 8 * qt + 4) * 4);
#pragma unroll
                    for (int ks = 0; ks < 2; ++ks) {
                        const uint32_t z0 = (__byte_perm(w0[2 * ks], w1[2 * ks], 0x5410) & 0x000f000fu) << 2, z1 = (__byte_perm(w0[2 * ks + 1], w1[2 * ks + 1], 0x5410) & 0x000f000fu) << 6;
#pragma unroll
                        for (int rn = 0; rn < RN; ++rn) at_mma(z[rn][n], z0, z0, z1, z1, pb[n][rn][2 * ks], pb[n][rn][2 * ks + 1]);
                    }
#pragma unroll
                    for (int b4 = n * W / G; b4 < (n + 1) * W / G; ++b4) {
                        const uint4 w4 = *reinterpret_cast<const uint4 *>(tile + kv_v_codes(D) + (b4 * 32 + lane) * 16);
                        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const uint32_t x = at_place(w[2 * half], ks), y = at_place(w[2 * half + 1], ks);
                                const uint32_t a0 = x & AT_LOW, a1 = y & AT_LOW, a2 = x & AT_HIGH, a3 = y & AT_HIGH;
#pragma unroll
                                for (int rn = 0; rn < RN; ++rn) at_mma(o[rn][2 * b4 + half], a0, a1, a2, a3, pb[n][rn][2 * ks], pb[n][rn][2 * ks + 1]);
                            }
                    }
                }
            }
            // ---- the slot is free: the tile ST further on
            __syncwarp();
            const int ni = i + ST;
            // (at_now has the addresses of the block of 32 that tile i lies in, at_next those of the block behind it)
            if (ni < count && lane == (ni & 31)) ask((ni >> 5) == (i >> 5) ? at_now : at_next, slot);
            if ((i & 31) == 31) {
                at_now = at_next;
                there = __ballot_sync(0xffffffffu, at_now != 0);
                at_next = where(i + 33 + lane);
            }
            if (++slot == ST) { slot = 0; phase ^= 1; }
        }

        // ---- join of the four warps: each puts its sums where its ring was (all of its copies have landed)
        constexpr float BACK = 0x1p22f / AT_DOWN;  // codes are held times 2^-22
        float *part = reinterpret_cast<float *>(ring);
#pragma unroll
        for (int rn = 0; rn < RN; ++rn)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int row = 8 * rn + 2 * qt + k;
                float x = l[rn][k];
                x += __shfl_xor_sync(0xffffffffu, x, 4);
                x += __shfl_xor_sync(0xffffffffu, x, 8);
                x += __shfl_xor_sync(0xffffffffu, x, 16);
                if (qg == 0) {
                    s_m[warp][row] = m[rn][k];
                    s_l[warp][row] = x;
                }
#pragma unroll
                for (int n = 0; n < MT; ++n) {
                    const float zz = z[rn][n * G / MT][k];
                    part[row * PITCH + 16 * n + qg] = (o[rn][n][k] - zz) * BACK;
                    part[row * PITCH + 16 * n + 8 + qg] = (o[rn][n][2 + k] - zz) * BACK;
                }
            }
        const int seq = work.seq, item = work.item, i0 = work.i0, i1 = work.i1, rt = item / a.c.heads, h = item - rt * a.c.heads, rows = min(ROWS, a.nq * a.g - rt * ROWS);
        const int slot_out = 2 * work.id + (i0 == 0 ? 1 : 0);
        float *sums = a.part + (size_t)slot_out * ROWS * D, *ml = a.ml + (size_t)slot_out * ROWS * 2;
        if (work.t0 != i0) at_fold<D, STEP, PITCH>(own, rows, lane, part, s_m[warp], s_l[warp], sums, ml);
        if constexpr (SOLO) __syncwarp();
        else __syncthreads();
        const bool all = i0 == 0 && i1 == work.tiles, whole = all && work.t1 == i1;  // the item lies in this worker; this is the end of it
        if (SOLO ? lane == 0 : tid == 0) {
            int2 *at = a.where + (long long)seq * per + item;
            if (all) *at = make_int2(-1, -1);
            else if (i0 == 0) at->x = work.id;
            else if (i1 == work.tiles) at->y = work.id;
        }
        constexpr int NW = SOLO ? 1 : AT_WARPS;
        for (int row = own; row < rows; row += STEP) {
            float top = -INFINITY, wt[NW], sum = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) top = fmaxf(top, s_m[SOLO ? warp : w][row]);
            const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float by = s_m[SOLO ? warp : w][row] - ref;
                wt[w] = at_ex2(by);
                sum += at_lower(s_l[SOLO ? warp : w][row], by);
            }
            const float by = whole ? (sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f) : 1.0f;
            const int in = rt * ROWS + row, tok = in / a.g, hd = in - tok * a.g;
            const long long tokrow = (long long)seq * a.nq + tok;
#pragma unroll
            for (int c = 0; c < D; c += 32) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const float x = reinterpret_cast<const float *>(at_raw + (SOLO ? warp : w) * ST * TILE)[row * PITCH + c + lane];
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
        __syncwarp();
        if (lane == 0) work.u += work.t1 - work.t0;
        if constexpr (SOLO) __syncwarp();
        else __syncthreads();
    }
}

// A row of an item that was cut, from its parts i0 .. i1: `warps` warps (this one being number w of them) take every warps-th part, several
// under way at a time, a lane D/32 neighbouring channels.  top, sum, v: reference, sum of weights and weighted sums of these parts.
template <int D, int ROWS>
__device__ __forceinline__ void at_parts(const AtArgs &a, int i0, int i1, int row, int w, int warps, float &top, float &sum, float (&v)[D / 32]) {
    constexpr int CPL = D / 32, AHEAD = 8;
    const int lane = threadIdx.x & 31, parts = i1 - i0 + 1;
    top = -INFINITY;
    sum = 0.0f;
#pragma unroll
    for (int k = 0; k < CPL; ++k) v[k] = 0.0f;
    for (int i = w; i < parts; i += warps * AHEAD) {
        float2 p[AHEAD];
        float x[AHEAD][CPL];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int part = i0 + min(i + k * warps, parts - 1);
            const size_t at = ((size_t)2 * part + (part == i0 ? 1 : 0)) * ROWS + row;
            p[k] = __ldcg(reinterpret_cast<const float2 *>(a.ml + at * 2));
            const float *src = a.part + at * D + lane * CPL;
#pragma unroll
            for (int c = 0; c < CPL; c += 2) {
                const float2 y = __ldcg(reinterpret_cast<const float2 *>(src + c));
                x[k][c] = y.x;
                x[k][c + 1] = y.y;
            }
        }
        float t = top;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) t = i + k * warps < parts ? fmaxf(t, p[k].x) : t;
        const float ref = t == -INFINITY ? 0.0f : t, down = at_ex2(top - ref);
        sum = at_lower(sum, top - ref);
        top = t;
#pragma unroll
        for (int c = 0; c < CPL; ++c) v[c] *= down;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i + k * warps < parts) {
                const float wt = at_ex2(p[k].x - ref);
                sum += at_lower(p[k].y, p[k].x - ref);
#pragma unroll
                for (int c = 0; c < CPL; ++c) v[c] += wt > 0.0f || x[k][c] != x[k][c] ? wt * x[k][c] : 0.0f;
            }
    }
}

// Joins the parts of the items that were cut, and writes the rows of sequences without tokens.  A block has a row of an item, its four
// warps a quarter of the parts each; SOLO, where there are many items and few parts of any, it has an item and a warp every fourth row.
template <int D, int ROWS, bool SOLO>
__global__ void __launch_bounds__(AT_THREADS) kv4_join_kernel(const AtArgs a) {
    constexpr float LN2 = 0.69314718055994531f;
    constexpr int CPL = D / 32;
    __shared__ float s_w[AT_WARPS], s_top[AT_WARPS], s_v[SOLO ? 1 : AT_WARPS][D];
    const int seq = blockIdx.x, item = blockIdx.y, rt = item / a.c.heads, h = item - rt * a.c.heads, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int per = a.c.heads * a.row_tiles, rows = min(ROWS, a.nq * a.g - rt * ROWS), q_heads = a.c.heads * a.g;
    griddep_wait();
    griddep_launch_dependents();
    const int2 range = __ldcg(a.where + (long long)seq * per + item);
    int first;
    const bool empty = at_tiles(a, seq, first) == 0;
    const int i0 = range.x, i1 = range.y;
    if (!empty && i0 == i1) return;  // finished by its worker
    for (int row = SOLO ? warp : (int)blockIdx.z; row < rows; row += SOLO ? AT_WARPS : ROWS) {
        const int in = rt * ROWS + row, tok = in / a.g, hd = in - tok * a.g;
        const long long tokrow = (long long)seq * a.nq + tok;
        unsigned short *out = a.out + tokrow * a.ldo + (long long)(h * a.g + hd) * D;
        float *lse = a.lse ? a.lse + tokrow * q_heads + h * a.g + hd : nullptr;
        if (empty) {
            for (int c = SOLO ? lane : tid; c < D; c += SOLO ? 32 : AT_THREADS) at_store(out + c, 0.0f, a.bf16);
            if (lse && (SOLO ? lane : tid) == 0) *lse = -INFINITY;
            continue;
        }
        float top, sum, v[CPL];
        at_parts<D, ROWS>(a, i0, i1, row, SOLO ? 0 : warp, SOLO ? 1 : AT_WARPS, top, sum, v);
        if constexpr (SOLO) {
            const bool any = sum > 0.0f || sum != sum;
            const float by = any ? 1.0f / sum : 0.0f;
#pragma unroll
            for (int c = 0; c < CPL; ++c) at_store(out + lane * CPL + c, v[c] * by, a.bf16);
            if (lse && lane == 0) *lse = any ? top * LN2 + logf(sum) : -INFINITY;
        } else {
            if (lane == 0) s_top[warp] = top;
            __syncthreads();
            float own = top;
#pragma unroll
            for (int w = 0; w < AT_WARPS; ++w) top = fmaxf(top, s_top[w]);
            own -= top == -INFINITY ? 0.0f : top;
            const float wt = at_ex2(own);
#pragma unroll
            for (int c = 0; c < CPL; ++c) s_v[warp][lane * CPL + c] = v[c] * wt;
            if (lane == 0) s_w[warp] = at_lower(sum, own);
            __syncthreads();
            sum = ((s_w[0] + s_w[1]) + s_w[2]) + s_w[3];  // the four warps in order
            const bool any = sum > 0.0f || sum != sum;
            const float by = any ? 1.0f / sum : 0.0f;
            for (int c = tid; c < D; c += AT_THREADS) at_store(out + c, (((s_v[0][c] + s_v[1][c]) + s_v[2][c]) + s_v[3][c]) * by, a.bf16);
            if (lse && tid == 0) *lse = any ? top * LN2 + logf(sum) : -INFINITY;
        }
    }
}

template <int D, int G, int RN, bool SOLO>
static cudaError_t at_launch_rn(const AtArgs &a, int grid, cudaStream_t st) {
    static SmemOptIn opt_in;
    constexpr int SMEM = AT_WARPS * at_stages(D, G, RN) * kv_tile_bytes(D, G) + (RN == 2 ? RN * D / 32 * 32 * 16 : 0);
    auto kern = kv4_attend_kernel<D, G, RN, SOLO>;
    cudaError_t e = ensure_dynamic_smem(kern, SMEM, opt_in);
    if (e != cudaSuccess) return e;
    e = launch(kern, dim3(grid), dim3(AT_THREADS), SMEM, st, g_tune.pdl != 0, a);
    if (e != cudaSuccess) return e;
    const int rows = a.nq * a.g < 8 * RN ? a.nq * a.g : 8 * RN;
    return launch(kv4_join_kernel<D, 8 * RN, SOLO>, dim3(a.c.n_seqs, a.c.heads * a.row_tiles, SOLO ? 1 : rows), dim3(AT_THREADS), 0, st, g_tune.pdl != 0, a);
}

// How the rows and items of a call are taken.  Eight rows at a time where a head has no more than that, else sixteen: the cache is then
// read (and unpacked) half as often.  Warps work on their own (SOLO) where there are more items than CTAs that the device holds: an item then
// costs no barriers, its queries are prepared once, and its tiles need not be a multiple of four (100 sequences of together 40000 tokens,
// 8 key heads: 57 -> 44 us; 512 of 60000: 148 -> 76; 64 of 128000, where there are fewer items than CTAs: 61 -> 66).
struct AtPlan {
    int rn, items, resident;
    bool solo;
    int waves() const { return solo ? 1 : 2; }
    size_t workers() const { return (size_t)(solo ? AT_WARPS : 1) * waves() * resident; }  // at most; two parts for each
    size_t bytes(int n_seqs, int D) const { return workers() * 2 * 8 * rn * (D + 2) * sizeof(float) + (size_t)n_seqs * items * sizeof(int2); }
};
static AtPlan at_plan(int n_seqs, int nq, int q_heads, int heads, int D, int G) {
    AtPlan p;
    const int rows = nq * (q_heads / heads);
    p.rn = rows <= 8 ? 1 : 2;
    p.items = heads * ((rows + 8 * p.rn - 1) / (8 * p.rn));  // per sequence
    p.resident = sm_count() * at_resident(D, G, p.rn);
    p.solo = p.rn == 1 && (long long)n_seqs * p.items > p.resident;
    return p;
}

template <int D, int G>
static cudaError_t at_launch(const AtArgs &a, const AtPlan &p, int grid, cudaStream_t st) {
    if (p.solo) return at_launch_rn<D, G, 1, true>(a, grid, st);
    return p.rn == 1 ? at_launch_rn<D, G, 1, false>(a, grid, st) : at_launch_rn<D, G, 2, false>(a, grid, st);
}

}  // namespace scap

using namespace scap;

extern "C" size_t scap_kv4_attend_workspace(int n_seqs, int nq, int q_heads, int heads, int head_dim) {
    if (n_seqs < 1 || n_seqs > SCAP_MAX_SEQS || nq < 1 || nq > SCAP_MAX_BATCH || heads < 1 || heads > 1024 || q_heads < heads || q_heads % heads || q_heads > 1024) return 0;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return 0;
    size_t most = 0;
    for (int G = 1; G <= 4; G *= 2) {  // (the number of groups decides how many CTAs the device holds)
        const AtPlan p = at_plan(n_seqs, nq, q_heads, heads, head_dim, G);
        const size_t bytes = p.bytes(n_seqs, head_dim);
        most = bytes > most ? bytes : most;
    }
    return most;
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
    const AtPlan p = at_plan(cache->n_seqs, nq, q_heads, cache->heads, cache->head_dim, a.c.groups);
    a.row_tiles = p.items / cache->heads;
    a.window = window;
    a.scale = (float)(scale * 1.4426950408889634);
    a.resident = p.resident;
    a.waves = p.waves();
    // What the tables have room for bounds the work: no more CTAs than that takes.
    const long long cap = (long long)cache->table_stride * (cache->page_tokens / KV_TILE), seen = window > 0 ? ((long long)window + nq) / KV_TILE + 2 : cap;
    a.tile_cap = (int)(cap < (1ll << 30) ? cap : (1ll << 30));
    const long long items = (long long)cache->n_seqs * cache->heads * a.row_tiles, units = (cap < seen ? cap : seen) * items;
    const long long few = (units + AT_MIN_UNITS - 1) / AT_MIN_UNITS > items ? (units + AT_MIN_UNITS - 1) / AT_MIN_UNITS : items;
    const int most = at_two_waves(units, items, a.resident) ? a.waves * a.resident : a.resident;  // (both at least what the kernel counts)
    const int grid = few < most ? (int)few : most;
    a.ml = a.part + 2 * p.workers() * 8 * p.rn * cache->head_dim;
    a.where = reinterpret_cast<int2 *>(a.ml + 2 * p.workers() * 8 * p.rn * 2);
    a.bf16 = dt == SCAP_BF16;
    a.limit = g_tune.tc_spin ? (uint32_t)g_tune.tc_spin : TRIES;
    a.status = tc_status_ptr();
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    switch (cache->head_dim * 8 + a.c.groups) {
        case 64 * 8 + 1: return cuda_status(at_launch<64, 1>(a, p, grid, st));
        case 64 * 8 + 2: return cuda_status(at_launch<64, 2>(a, p, grid, st));
        case 128 * 8 + 1: return cuda_status(at_launch<128, 1>(a, p, grid, st));
        case 128 * 8 + 2: return cuda_status(at_launch<128, 2>(a, p, grid, st));
        case 128 * 8 + 4: return cuda_status(at_launch<128, 4>(a, p, grid, st));
        case 256 * 8 + 2: return cuda_status(at_launch<256, 2>(a, p, grid, st));
        default: return cuda_status(at_launch<256, 4>(a, p, grid, st));
    }
}
