// Attention over the paged low-bit cache: the call as the kernels see it, and the order that its work is numbered in.
//
// A pair is (row tile, key head): up to `rows` query rows that share a key head, a row being (token, query head of the group), tokens
// outermost.  Row tiles of the shared prefix come first (their rows are those of all tokens), then those of each sequence.  A pair's
// keys are cut into units; units are numbered pair by pair and every CTA takes an equal run of them, wherever sequences end.
// What a CTA has of a pair is a partial result: per row the reference m, the sum l of exp2(s - m) and the sum of exp2(s - m) V.  It is
// entry (CTA + pair) of the workspace, which no other CTA writes: the CTA after it starts at this pair or a later one.  Pairs have their numbers there
// from the places of their tiles: row tiles counted for each sequence alike, or, where most sequences have far fewer tokens than the most that
// one may have, by the tokens in front of them, (first row of the sequence) / rows + sequence + tile, which rises from tile to tile too.
// What is numbered in 32 bits is bounded by the tokens, not by what every sequence might have: the host refuses a call whose tokens in any order could
// have more.  Starts that fall can have more all the same (they are reported, and their outputs mean nothing): sums stop at that bound, what
// lies behind it is not done, and what the joins read of such a pair's place is brought into range.
//
// Two kernels do this: one for few rows (tiles of 8 or 16 rows), one for many (256 rows); each has its own Part of the work.  A call gives the
// prefix's tiles to one of them, and each sequence goes by its own rows, seen on the device: a batch may hold chunks of prompts beside single tokens.
#pragma once
#include "bfq_kv.cuh"
#include "bfq_kvmma.cuh"

namespace bfq {
namespace kv {

constexpr int kFewUnit = 128, kTallUnit = 64;  // keys
constexpr int kTallRows = 256;
constexpr int kFewMost = 48;  // rows that share their keys: more go to the kernel for many

struct Part {
    int rows, rows_shift;         // of a tile, 1 << rows_shift
    int unit_shift;               // keys of a unit: 1 << unit_shift
    int tiles_prefix, tiles_seq;  // row tiles of the prefix, and of each sequence
    int seq_from, seq_to;         // rows of the sequences that are this part's
    int by_tokens;                // how tiles are placed in the workspace
    int most;                     // units of a key head, at most
    int ctas;                     // of the launch
    int2* pairs;                  // [pairs] first CTA, CTAs
    float2* sums;                 // [entries][rows] m, l
    float* parts;                 // [entries][rows][D]
};

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
    float scale_log2;  // softmax scale * log2 e
    const float2* tw;
    Part few, tall;
    int prefix_tall, seq_tall;  // the kernel for many rows has the prefix; has sequences (those of more than kFewMost rows)
    int join_tall;              // k_join_tall joins the sequences of the kernel for many rows
    int beside_tall;            // the kernel for few rows follows the one for many
    int* status;
    __host__ __device__ int entries(const Part& part) const { return part.tiles_prefix + batch * part.tiles_seq; }
    __host__ __device__ int64_t places_by_tokens(const Part& part) const { return part.tiles_prefix + (tokens * group >> part.rows_shift) + batch; }
    __host__ __device__ int64_t places(const Part& part) const { return part.by_tokens ? places_by_tokens(part) : entries(part); }
};

__device__ __forceinline__ int first_token(const AttendParams& p, int b) {
    if (p.q_starts == nullptr) return b;
    const int t = load_plain(p.q_starts + b);
    return t < 0 ? 0 : (t > p.tokens ? static_cast<int>(p.tokens) : t);
}
__device__ __forceinline__ int cached_keys(const AttendParams& p, int b) {
    const int n = load_plain(p.lengths + b), most = p.cache.pages > 0 ? p.table_width << p.cache.page_shift : 0;
    return n < 0 ? 0 : (n > most ? most : n);
}
// Starts that do not rise from 0 to the tokens, more new tokens than the call was told, a length outside its range: the kernels take the nearest one
// inside, or rows are left out
__device__ __forceinline__ bool out_of_range(const AttendParams& p, int b) {
    if (p.q_starts != nullptr) {
        const int64_t from = load_plain(p.q_starts + b), to = load_plain(p.q_starts + b + 1);
        if (from < 0 || to < from || to > p.tokens || to - from > p.max_new) return true;
        if (to == from) return false;  // its length does not matter
    }
    return load_plain(p.lengths + b) != cached_keys(p, b);
}

// One row tile: its rows and the keys that any of them has.
struct Tile {
    int place;           // in the workspace
    int row0, rows;      // of the sequence's rows (prefix: of all rows)
    int token0;          // token of the sequence's row 0
    int keys;            // keys 0 .. keys - 1
    int last0;           // row r has keys 0 .. last0 + (row0 + r) / group; prefix: all
    const int32_t* pages;
};
__device__ __forceinline__ Tile tile_of(const AttendParams& p, const Part& part, int e) {
    Tile t;
    const int rows = part.rows;
    if (e < part.tiles_prefix) {
        const int tokens = first_token(p, p.batch);
        t.place = e, t.row0 = e * rows, t.token0 = 0;
        const int left = tokens * p.group - t.row0;
        t.rows = left < 0 ? 0 : (left < rows ? left : rows);
        t.keys = t.rows > 0 ? p.prefix_length : 0;
        t.last0 = 1 << 30;
        t.pages = p.prefix;
        return t;
    }
    const int b = (e - part.tiles_prefix) / part.tiles_seq, rt = (e - part.tiles_prefix) % part.tiles_seq;
    const int t0 = first_token(p, b), news = first_token(p, b + 1) - t0, n = cached_keys(p, b);
    t.place = part.by_tokens ? part.tiles_prefix + (t0 * p.group >> part.rows_shift) + b + rt : e;
    t.row0 = rt * rows, t.token0 = t0;
    const int all = news * p.group, left = all >= part.seq_from && all <= part.seq_to ? all - t.row0 : 0;
    t.rows = left < 0 ? 0 : (left < rows ? left : rows);
    t.last0 = n - news;
    const int need = t.rows > 0 ? t.last0 + (t.row0 + t.rows - 1) / p.group + 1 : 0;
    t.keys = need < 0 ? 0 : need;
    t.pages = p.block_table + b * p.table_ld;
    return t;
}

// The entry whose tile has a place behind the prefix's; -1: none has.
__device__ __forceinline__ int entry_at(const AttendParams& p, const Part& part, int place) {
    if (!part.by_tokens) return place;
    auto first_place = [&](int b) { return part.tiles_prefix + (first_token(p, b) * p.group >> part.rows_shift) + b; };
    int lo = 0, hi = p.batch;  // the last sequence whose places begin at or before this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (first_place(mid) <= place) lo = mid;
        else hi = mid;
    }
    const int rt = place - first_place(lo);
    return rt >= 0 && rt < part.tiles_seq ? part.tiles_prefix + lo * part.tiles_seq + rt : -1;
}
// What a pair's place holds: its first CTA and how many have a part of it.
__device__ __forceinline__ int2 ctas_of(const Part& part, int pair) {
    const int2 v = load_plain(part.pairs + pair);
    const int first = min(max(v.x, 0), part.ctas - 1);
    return make_int2(first, min(max(v.y, 0), part.ctas - first));
}

// the entry to look at after e: a sequence's tiles without rows are its last ones
__device__ __forceinline__ int after(const Part& part, int e, const Tile& t) {
    if (t.rows > 0 || e < part.tiles_prefix) return e + 1;
    return part.tiles_prefix + ((e - part.tiles_prefix) / part.tiles_seq + 1) * part.tiles_seq;
}

// Where in the numbering of units a role of a CTA is.
struct Walk {
    int entry, head, unit, units;  // unit of units within the pair
    Tile tile;
    __device__ __forceinline__ void enter(const AttendParams& p, const Part& part, int e) {  // the first entry from e on that has units
        const int last = p.entries(part);
        for (entry = e, units = 0; entry < last; entry = after(part, entry, tile)) {
            tile = tile_of(p, part, entry);
            units = (tile.keys + (1 << part.unit_shift) - 1) >> part.unit_shift;
            if (units > 0) break;
        }
    }
    __device__ __forceinline__ void next_pair(const AttendParams& p, const Part& part) {
        unit = 0;
        if (++head < p.cache.heads) return;
        head = 0;
        enter(p, part, entry + 1);
    }
    __device__ __forceinline__ void next(const AttendParams& p, const Part& part) {
        if (++unit == units) next_pair(p, part);
    }
    __device__ __forceinline__ int pair(const AttendParams& p) const { return tile.place * p.cache.heads + head; }
};

// A CTA's run of units, found by all its threads together from the lengths.  Units of a head are at most part.most, which times the heads is below 2^30.
struct Run {
    int from;   // the first one's number
    int per;    // units of every CTA but the last
    int count;  // 0: none
};
template <int THREADS>
__device__ __forceinline__ Run find_run(const AttendParams& p, const Part& part, int* scan, Walk* walk) {  // scan: shared, THREADS / 32 + 2
    constexpr int kWarps = THREADS / 32;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, entries = p.entries(part), heads = p.cache.heads;
    const int each = (entries + THREADS - 1) / THREADS;
    auto units_of = [&](const Tile& t) { return (t.keys + (1 << part.unit_shift) - 1) >> part.unit_shift; };
    int mine = 0;
    for (int e = tid * each; e < entries && e < (tid + 1) * each;) {
        const Tile t = tile_of(p, part, e);
        mine = min(mine + units_of(t), part.most), e = after(part, e, t);
    }
    int before = mine, total = 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, before, o);
        if (lane >= o) before = min(before + v, part.most);
    }
    if (lane == 31) scan[warp] = before;
    before = __shfl_up_sync(0xFFFFFFFFu, before, 1);
    if (lane == 0) before = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w == warp) before = min(before + total, part.most);
        total = min(total + scan[w], part.most);
    }
    total *= heads;
    Run run;
    run.per = total > 0 ? (total + static_cast<int>(gridDim.x) - 1) / static_cast<int>(gridDim.x) : 1;
    run.from = run.per * static_cast<int>(blockIdx.x);
    run.count = run.from < total ? (run.per < total - run.from ? run.per : total - run.from) : 0;
    if (run.count == 0) return run;
    if (run.from >= before * heads && run.from - before * heads < mine * heads) {  // one thread: the entry that holds `from` is one of its own
        int e = tid * each;
        if (each > 1)
            for (;;) {
                const Tile t = tile_of(p, part, e);
                const int u = units_of(t);
                if (run.from - before * heads < u * heads) break;
                before += u, e = after(part, e, t);
            }
        scan[kWarps] = e, scan[kWarps + 1] = run.from - before * heads;
    }
    __syncthreads();
    walk->enter(p, part, scan[kWarps]);
    walk->head = scan[kWarps + 1] / walk->units, walk->unit = scan[kWarps + 1] - walk->head * walk->units;
    return run;
}

// the tall kernel (bfq_kvtall.cu): CTAs of a launch, and the launch
cudaError_t tall_ctas(const bfq_plan* plan, int bits, int* ctas);
cudaError_t tall_launch(const bfq_plan* plan, const AttendParams& p, int ctas, cudaStream_t st);
// joins its results where there is no prefix (bfq_kvjoin.cu)
cudaError_t join_tall_launch(const bfq_plan* plan, const AttendParams& p, cudaStream_t st);

}  // namespace kv
}  // namespace bfq
