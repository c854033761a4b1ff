// Arguments and launches of a decoder's other operators: the rotation of queries and keys, the
// selection of beams, and the paged cache in their order (decoder.hip, decoder_abi.hip).
#pragma once

#include "seq_host.hpp"
#include "seq_params.hpp"

namespace ma {

struct Rotate {
    const void *q, *k, *v;  // rows of ldq, ldk, ldv elements; v: append only
    void *q_out;            // [total, Hq, d]
    void *k_out, *v_out;    // [total, Hk, d] and null; append: [pages, Hk, page, d] both
    const float *inv_freq;  // [rot / 2]
    Seqs seqs;
    const int *kv_lens;     // tokens of every sequence, its rows the last of them; null: its rows are all
    const int64_t *slots;   // append: of every row
    int Hq, Hk, d, rot;
    int64_t ldq, ldk, ldv;
    int page_log2, pages;
    int interleaved, inverse, clear;
    int rows;               // rows a workgroup takes, up to kRotateRows
};

struct BeamSelect {
    const void *logits;     // [B K] rows of ld elements, the first V of them
    const float *scores;    // [B, K]
    const uint8_t *done;    // [B, K] or null
    float *scores_out;      // [B, M]
    int *tokens, *parents;  // [B, M]
    uint8_t *done_out;      // [B, M] or null
    int64_t ld;
    int B, K, V, M, eos;
    int parts, part_vectors;  // parts of a row, and 16-byte vectors a part
    uint64_t *keys;         // [B K, parts, M] the best of every part, as keys
    float *part_max, *part_sum;  // [B K, parts] its largest logit and the sum of exp(logit - largest)
};

struct PagedReorder {
    void *k_pages, *v_pages;  // [pages, Hkv, page, d]
    int *table;               // [B K, blocks]
    const int *parents;       // [B, K]
    const int *lens;          // [B K]
    int B, K, chunks;         // chunks of 16 bytes of a row of one head
    int Hkv, page_log2, pages, blocks;
    int move_table;
};

constexpr int kRotateRows = 16;
constexpr int kBeamMax = MONARCH_ATTN_BEAM_MAX;

}  // namespace ma

namespace ma_host {

enum DecoderKind { kRotate = 17, kBeamParts = 18, kBeamJoin = 19, kReorder = 20 };

int run_rotate(Launcher &L, const ma::Rotate &p, int32_t dtype, bool append);
int run_beam_select(Launcher &L, const ma::BeamSelect &p, int32_t dtype);
int run_paged_reorder(Launcher &L, const ma::PagedReorder &p);

}  // namespace ma_host
