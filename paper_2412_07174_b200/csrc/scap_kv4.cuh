// The 4-bit key / value cache: layout of a page, and what its kernels share (internal header).
//
// A page holds page_tokens tokens (a multiple of 32) of every key head.  Head by head, then tile by tile, a tile being 32 tokens:
//   K codes  32 rows of D/2 bytes
//   V codes  32 D/2 bytes
//   K words  [groups][32]   one 32-bit word per token and group of channels: the scale, whose low four bits are the zero point;
//   V words  [groups][32]   token 8 j + i at place 4 i + j, so that the four tokens of a lane are one 16-byte load
// A code q in 0..15 stands for s (q - zero).  s has 20 significant bits, so the low four bits of its binary32 form are free for the
// zero point, and s (q - zero) is exact in binary32.
//
// The order of the codes inside a tile is that of the tensor core's operand registers, so that the attention kernel gets them with plain
// wide loads and a mask (mma.m16n8k16: lane (g, t), g = lane / 4, t = lane % 4, holds column g at k = 2t, 2t+1, 2t+8, 2t+9):
//   K  row = token.  Word t (D/32) + j of a row holds the eight channels 32 j + 8 t .. + 7, channel i in nibble i: lane (g, t) reads
//      D/32 consecutive words of token g.
//   V  word ((nt / 4) 32 + 4 g + t) 4 + nt % 4 holds the eight tokens 8 j + 2 t + o of channel 8 nt + g, in nibble j + 4 o (j = 0..3,
//      o = 0, 1): lane (g, t) reads four consecutive words, for four blocks of eight channels.
// In both, the nibbles i and i + 4 of a word are the two halves of one operand register: w << 2 and w >> 6 under the masks 0x003c003c and 0x03c003c0
// are pairs of fp16 subnormals, code 2^-22 and code 2^-18, which the tensor core multiplies exactly.  No code is converted.
#pragma once

#include "scap_common.cuh"

namespace scap {

constexpr int KV_TILE = 32;  // tokens

__host__ __device__ constexpr int kv_tile_bytes(int D, int groups) { return KV_TILE * D + 2 * groups * KV_TILE * 4; }
__host__ __device__ constexpr int kv_v_codes(int D) { return KV_TILE * D / 2; }
__host__ __device__ constexpr int kv_k_words(int D) { return KV_TILE * D; }
__host__ __device__ constexpr int kv_v_words(int D, int groups) { return KV_TILE * D + groups * KV_TILE * 4; }

// Byte of a K row that holds channels c, c + 1 (c even).
__host__ __device__ constexpr int kv_k_byte(int D, int c) { return (((c >> 3) & 3) * (D / 32) + (c >> 5)) * 4 + ((c & 7) >> 1); }
// Place of a token's word.
__host__ __device__ constexpr int kv_word_at(int tok) { return (tok & 7) * 4 + (tok >> 3); }
// Word of the V codes that holds channel c of the tokens 8 j + 2 t + o.
__host__ __device__ constexpr int kv_v_word(int c, int t) { return (((c >> 5) * 32 + (c & 7) * 4 + t) << 2) + ((c >> 3) & 3); }

struct KvCache {
    unsigned char *pages;
    long long page_stride;
    int n_pages, page_tokens, heads, groups;
    const int *table;
    const int *lens;
    int table_stride, n_seqs;
};

inline KvCache kv_cache(const scap_kv4 *c) {
    KvCache k;
    k.pages = reinterpret_cast<unsigned char *>(c->pages);
    k.page_stride = (long long)c->page_stride;
    k.n_pages = c->n_pages; k.page_tokens = c->page_tokens; k.heads = c->heads;
    k.groups = c->group > 0 ? c->head_dim / c->group : 0;
    k.table = c->table; k.lens = c->lens;
    k.table_stride = c->table_stride; k.n_seqs = c->n_seqs;
    return k;
}

// The page of token `pos` of sequence b: -1 where the table has none (beyond its row, or an entry that is no page of the pool).
__device__ __forceinline__ int kv_page(const KvCache &c, int b, int pos) {
    const int at = pos / c.page_tokens;
    if (pos < 0 || at >= c.table_stride) return -1;
    const int p = __ldcg(c.table + (long long)b * c.table_stride + at);
    return p >= 0 && p < c.n_pages ? p : -1;
}

// The tile of head h that holds token pos, in page p.
__device__ __forceinline__ unsigned char *kv_tile(const KvCache &c, int p, int h, int pos, int tile_bytes) {
    return c.pages + (long long)p * c.page_stride + (long long)(h * (c.page_tokens / KV_TILE) + (pos % c.page_tokens) / KV_TILE) * tile_bytes;
}

// Checks of a cache description that all calls on keys and values share.
scap_status kv_check(const scap_kv4 *c);

}  // namespace scap
