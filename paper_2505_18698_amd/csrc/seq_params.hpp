// Arguments of the kernels of the exact attention over sequences and of the
// paged cache.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ma {

// Row starts of packed sequences (device memory; clamped to 0..total, so that
// no value in it leads out of range).
struct Seqs {
    const int *cu;
    int B, total;
    __device__ inline int start(int s) const { return max(0, min(cu[s], total)); }
    __device__ inline int length(int s) const { return max(0, start(s + 1) - start(s)); }
};

// Where the keys of the query rows are: in the same rows; in pages; or, for cross attention, in rows
// of their own.
enum Keys { kSelf, kPaged, kCross };

// The key rows of cross attention: the ranges of packed sequences, of which the first lens[s] rows
// are keys (null: all of them) and the others padding.
struct KeySeqs : Seqs {
    const int *lens;
    __device__ inline int count(int s) const
    {
        const int n = length(s);
        return lens ? max(0, min(lens[s], n)) : n;
    }
};

struct SeqFwd {
    const void *q, *k, *v;  // packed, cross: rows of ldq, ldk, ldv elements; paged: k, v are [pages, Hkv, page, d]
    void *out;              // [total, Hq, d]
    float *lse;             // [Hq, total] or null
    void *rest;             // as out, or null: what rounding out to 16 bits leaves
    Seqs seqs;              // the query rows
    KeySeqs keys;           // cross: the key rows
    const int *kv_lens;     // paged: keys of every sequence
    const int *table;       // paged: [B, blocks] page numbers
    int Hkv, G, d;          // Hq = Hkv G
    int64_t ldq, ldk, ldv;  // elements
    int page_log2, pages, blocks;
    float c;                // s log2(e)
    int causal;
    int clear;              // packed, cross: write zeros in the rows of no sequence
    int tiles;              // row tiles of one key head (an upper bound)
    // split over the keys: workgroups of one key head; their segments' rows,
    // normalised, and their log2-sum-exp; and what every row tile is made of
    int shares;
    float *part_o, *part_l;
    struct SeqTileParts *parts;
};

// parts[0].count: how many row tiles there are; parts[1 + i]: of tile i the sequence's first row, the
// tile's first packed row and their number, the first and the number of the shares that have a
// segment of it, and how many first packed rows of the sequence see no key.
struct SeqTileParts {
    int row0, at, rows, first, count, blind, unused[2];
};

struct SeqBwd {
    const void *q, *k, *v, *out, *dout;  // q, k, v: rows of ldq, ldk, ldv elements
    const float *lse;                    // [Hq, total]; total: of the query rows, total_k of the key rows (self: the same)
    const void *rest;                    // as out, or null
    void *dq, *dk, *dv;
    Seqs seqs;
    KeySeqs keys;                        // cross: the key rows
    int Hkv, G, d;
    int64_t ldq, ldk, ldv;
    float c;                             // s log2(e)
    int causal;
    int clear;                           // write zeros in the gradients' rows of no sequence
    int tiles_q, tiles_k;                // row and key tiles of one key head (upper bounds)
    float *lse2, *delta;                 // [Hq, total]: lse in log2 units, delta
    float *norm_g, *norm_v;              // fp16: |dO_i|^2 [Hq, total] and |v_j|^2 [Hkv, total_k], 0 where not finite
    int stat_blocks;                     // workgroups of the row statistics
    // pieces that the query rows of a key tile are cut into; with more than one, their sums:
    // dK and dV of every piece, row and key head, in rows of the tile width
    int pieces;
    float *part_k, *part_v;
    // cross: pieces that the keys of a row tile are cut into; with more than one, dQ of every piece, row
    // and head, in rows of the tile width
    int pieces_q;
    float *part_q;
};

struct PagedPlan {
    const int *past, *fresh;  // [B] cached and new tokens
    const int *ring;          // [ring_len] free pages, in a ring
    const int *free_in;       // (first, count) of the free ones
    int *table;               // [B, blocks]
    int *cu, *kv_lens;        // [B + 1], [B]
    int64_t *slots;           // [capacity]
    int *free_out, *status;
    int B, ring_len, blocks, page_log2, capacity;
};

struct PagedWrite {
    const void *k, *v;  // [rows, Hkv, d], rows ldk, ldv elements apart
    void *k_pages, *v_pages;
    const int64_t *slots;
    int rows, Hkv, d, page_log2, pages, size;  // size: bytes an element
    int64_t ldk, ldv;
};

}  // namespace ma
