// How the attention over pages cuts its work: sequences, tiles, shares of blocks.  Host and device code.
#pragma once
#include <stdint.h>

#include "../../include/sdv.h"

#ifdef __CUDACC__
#include "ptx.cuh"
#define SDV_HD __host__ __device__ __forceinline__
#else
#define SDV_HD inline
#endif
namespace sdv {

#ifndef __CUDACC__
template <typename T> inline T min(T a, T b) { return b < a ? b : a; }
template <typename T> inline T max(T a, T b) { return a < b ? b : a; }
#endif

constexpr int kTreeKeys = 64;          // keys of a tile
constexpr int kTreeTileRows = 128;     // query rows of a tile: one query head of one row each, all heads of a group of as many rows as fit

// The caller's index arrays and sizes.
struct TreeLists {
    const int *kv_len, *cu_rows;
    int n_seqs, n_rows, n_kv, g, table_width, page_size;   // g: query heads per KV head (at most 128)
    int chunk;                                             // rows of a tile: kTreeTileRows / g
    int whole;                                             // items (KV head, row chunk) are dealt out whole, not tile by tile
};

// An entry of the caller's lists; EARLY: for a kernel that has not waited for the one ahead of it yet (which does not write them, and began behind who did).
template <bool EARLY>
SDV_HD int list_entry(const int* p) {
#ifdef __CUDA_ARCH__
    if (EARLY) return ld_global_l2(p);
#endif
    return *p;
}
// Rows of sequence b, whatever cu_rows holds: within [0, n_rows), none where the array descends.
template <bool EARLY = false>
SDV_HD int rows_begin(const int* cu, int b, int n_rows) { return min(max(list_entry<EARLY>(cu + b), 0), n_rows); }
SDV_HD int rows_count(const int* cu, int b, int n_rows) { return max(0, rows_begin(cu, b + 1, n_rows) - rows_begin(cu, b, n_rows)); }

// One sequence as the kernels see it, whatever the arrays hold.
struct TreeSeq {
    int first, rows, length, keys;     // first row, rows, committed tokens, tokens in all (those the block table has room for)
    int chunks, tiles;                 // tiles of query rows, tiles of keys
};
template <bool EARLY = false>
SDV_HD TreeSeq tree_seq(const TreeLists& P, int b) {
    TreeSeq s;
    s.first = rows_begin<EARLY>(P.cu_rows, b, P.n_rows);
    s.rows = min(max(0, rows_begin<EARLY>(P.cu_rows, b + 1, P.n_rows) - s.first), SDV_TREE_ROWS);
    const long long room = min((long long)P.table_width * P.page_size, 0x7fffffffll - kTreeKeys);
    s.length = (int)min((long long)max(list_entry<EARLY>(P.kv_len + b), 0), room);
    s.keys = (int)min((long long)s.length + s.rows, room);
    s.chunks = (s.rows + P.chunk - 1) / P.chunk;
    s.tiles = s.rows ? (s.keys + kTreeKeys - 1) / kTreeKeys : 0;
    return s;
}
// What a sequence adds to the list that is dealt out: tiles, or items.
SDV_HD int tree_tiles(const TreeLists& P, const TreeSeq& s) { return (P.whole ? (s.tiles ? 1 : 0) : s.tiles) * s.chunks * P.n_kv; }

// The tiles (or items) of all sequences, KV heads and row chunks in a row are cut into shares, one a block: the first blocks have one more than the last.  (The host refuses calls
// that could have 2^31 tiles.)
struct TreeCut {
    int base, more;        // tiles of the last blocks, blocks with one more
    SDV_HD TreeCut(int total, int blocks) {
        base = (int)((unsigned)total / (unsigned)blocks);
        more = total - base * blocks;
    }
    SDV_HD int begin(int block) const { return block * base + min(block, more); }
    SDV_HD int owner(int tile) const {
        const int split = more * (base + 1);   // tiles of the blocks with one more
        return tile < split ? (int)((unsigned)tile / (unsigned)(base + 1)) : more + (int)((unsigned)(tile - split) / (unsigned)base);
    }
};

// Cursor over a block's tiles: sequence, KV head, row chunk, key tile.
struct TreeCursor {
    int left;                          // tiles (items) of the block still to do, this one included
    int b, h, c, tile;
    TreeSeq s;
    // n tiles (items) from the offset-th of sequence b0 on (which has more than that)
    SDV_HD void start(const TreeLists& P, int b0, const TreeSeq& seq, int offset, int n) {
        left = n;
        b = b0;
        s = seq;
        const int item = P.whole ? offset : (int)((unsigned)offset / (unsigned)s.tiles);
        tile = P.whole ? 0 : offset - item * s.tiles;
        h = s.chunks == 1 ? item : (int)((unsigned)item / (unsigned)s.chunks);
        c = item - h * s.chunks;
    }
    // Tiles of the present item that belong to this block, from the present one on.
    SDV_HD int run(const TreeLists& P) const { return P.whole ? s.tiles : min(left, s.tiles - tile); }
    SDV_HD void skip(const TreeLists& P, int n) {   // n = run()
        left -= P.whole ? 1 : n;
        if (left <= 0) return;
        tile = 0;
        if (++c < s.chunks) return;
        c = 0;
        if (++h < P.n_kv) return;
        h = 0;
        do s = tree_seq(P, ++b); while (s.tiles == 0 && b + 1 < P.n_seqs);
        if (s.tiles == 0) left = 0;
    }
};

}  // namespace sdv
