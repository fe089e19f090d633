// Attention over the paged low-bit cache: the call as the kernels see it, and the order that its work is numbered in.
//
// A pair is (row tile, key head): up to kTileRows query rows that share a key head, a row being (token, query head of the group), tokens
// outermost.  Row tiles of the shared prefix come first (their rows are those of all tokens), then those of each sequence.  A pair's
// keys are cut into units of kUnit; units are numbered pair by pair and every CTA takes an equal run of them, wherever sequences end.
// What a CTA has of a pair is a partial result: per row the reference m, the sum l of exp2(s - m) and the sum of exp2(s - m) V.  It is
// entry (CTA + pair) of the workspace, which no other CTA writes: the CTA after it starts at this pair or a later one.
#pragma once
#include "bfq_kv.cuh"

namespace bfq {
namespace kv {

constexpr int kUnit = 64;  // keys of a unit
constexpr int kTileRows = 16;

struct AttendParams {
    Cache cache;
    Heads q, out;
    float* lse;  // [tokens][q heads] or null
    const int32_t* block_table;
    int64_t table_ld;
    int table_width;
    const int32_t* lengths;
    const int32_t* q_starts;  // [batch + 1], or null: one token for each sequence
    const int32_t* prefix;
    int prefix_pages, prefix_length;
    int64_t tokens;  // rows of q: at least those of the sequences
    int batch, group, max_new;
    int tiles_prefix, tiles_seq;  // row tiles of the prefix, and of each sequence
    float scale_log2;             // softmax scale * log2 e
    const float2* tw;
    int2* pairs;        // [pairs] first CTA, CTAs
    float2* sums;       // [entries][kTileRows] m, l
    float* parts;       // [entries][kTileRows][D]
    int* status;
    __host__ __device__ int entries() const { return tiles_prefix + batch * tiles_seq; }
};

__device__ __forceinline__ int first_token(const AttendParams& p, int b) {
    if (p.q_starts == nullptr) return b;
    const int t = load_plain(p.q_starts + b);
    return t < 0 ? 0 : (t > p.tokens ? static_cast<int>(p.tokens) : t);
}
__device__ __forceinline__ int cached_keys(const AttendParams& p, int b) {
    const int n = load_plain(p.lengths + b), most = p.table_width << p.cache.page_shift;
    return n < 0 ? 0 : (n > most ? most : n);
}

// One row tile: its rows and the keys that any of them has.
struct Tile {
    int row0, rows;      // of the sequence's rows (prefix: of all rows)
    int token0;          // token of the sequence's row 0
    int keys;            // keys 0 .. keys - 1
    int last0;           // row r has keys 0 .. last0 + (row0 + r) / group; prefix: all
    const int32_t* pages;
};
__device__ __forceinline__ Tile tile_of(const AttendParams& p, int e) {
    Tile t;
    if (e < p.tiles_prefix) {
        const int tokens = first_token(p, p.batch);
        t.row0 = e * kTileRows, t.token0 = 0;
        const int left = tokens * p.group - t.row0;
        t.rows = left < 0 ? 0 : (left < kTileRows ? left : kTileRows);
        t.keys = t.rows > 0 ? p.prefix_length : 0;
        t.last0 = 1 << 30;
        t.pages = p.prefix;
        return t;
    }
    const int b = (e - p.tiles_prefix) / p.tiles_seq, rt = (e - p.tiles_prefix) % p.tiles_seq;
    const int t0 = first_token(p, b), news = first_token(p, b + 1) - t0, n = cached_keys(p, b);
    t.row0 = rt * kTileRows, t.token0 = t0;
    const int left = news * p.group - t.row0;
    t.rows = left < 0 ? 0 : (left < kTileRows ? left : kTileRows);
    t.last0 = n - news;
    const int need = t.rows > 0 ? t.last0 + (t.row0 + t.rows - 1) / p.group + 1 : 0;
    t.keys = need < 0 ? 0 : need;
    t.pages = p.block_table + b * p.table_ld;
    return t;
}
__device__ __forceinline__ int units_of(const Tile& t) { return (t.keys + kUnit - 1) / kUnit; }

}  // namespace kv
}  // namespace bfq
