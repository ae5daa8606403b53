// What the serving operators (include/etc.h, etc_serving_*) pass from the host checks to the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/etc.h"

namespace etc {

constexpr int kServingMaxSeqs = 1024;
constexpr int kServingMaxTokens = 1 << 20;
constexpr int kServingMaxKv = 1 << 30;
constexpr int kServingMaxVocab = 1 << 20;

// Operators in the error word, and what they refuse.
enum ServingOp { SRV_TABLES = 1, SRV_APPEND = 2, SRV_ATTENTION = 3, SRV_SAMPLE = 4, SRV_APPEND_CODES = 5, SRV_ATTENTION_CODES = 6, SRV_SCORE = 7 };
enum ServingError { SRV_BAD_SLOT = 1, SRV_BAD_LENGTH = 2, SRV_BAD_PAGE = 3, SRV_BAD_TOKEN = 4 };

// A handle's part in every launch.
struct ServingDev {
    int nq, nkv, d, page_shift, qk_norm, vocab;
    float eps;
    int max_kv_len;
    int n_cus;
    const double *inv_freq;      // [d / 2] theta^(-2i/d)
    int32_t *error;              // pinned host memory, 4 words
    int32_t *arrive;             // [2] zero between launches: workgroups of a launch that have read their inputs
    // attention: partial results of items whose keys are cut, a slot each, and per item how many have arrived (zero between launches)
    float *attn_part;
    int32_t *attn_arrive;
    int attn_slots;              // no cut takes more
    int32_t *taken;              // [8 * kTakenApart] pieces that a die's workgroups have taken behind their first ones (zero between launches)
    // sampling of long rows: statistics and bins of the slices
    void *smp_stats;
    uint64_t *smp_bins;
    // and of the rows that several workgroups share: [row] tokens listed, [row] workgroups that have listed theirs (zero between launches),
    // [row][kSampleList] the tokens
    int32_t *smp_listed, *smp_done, *smp_list;
    int32_t *score_arrived;      // [kScoreRows * kScoreApart] slices of a row that have arrived (zero between launches); a slice's results in smp_bins
};
constexpr int kTakenApart = 32;              // counters stand a cache line apart: 512 arrivals at neighbours took 3 us longer
constexpr int kScoreTop = 64;                // likeliest tokens of a row, at most
constexpr int kScoreRows = 512;              // rows that are cut
constexpr int kScoreParts = 1024;            // slices of a launch, at most; a slice leaves 16 + 8 * kScoreTop bytes
constexpr int kScoreApart = 32;
constexpr int kSampleList = 8192;
constexpr int kSampleSharedRows = 128;
constexpr int kAttnMaxSlots = 1024;
constexpr int kCaRows = 256;                // of attention: rows of a block
constexpr int kCaKeys = 64;                 // keys of a tile
constexpr int kCaMinTiles = 2;              // of a piece, where keys are cut
constexpr int kCaWholeTiles = 6;            // of an item that is not cut (chunk_attn.hip says why)
// Slots a handle can need: an item's keys are cut into pieces of kCaMinTiles at least, a sequence's rows into blocks.
inline int attention_slots(int nq, int nkv, const etc_serving_limits &l)
{
    const int64_t tiles = ((int64_t)l.max_kv_len + kCaKeys - 1) / kCaKeys, seqs = l.max_seqs < l.max_tokens ? l.max_seqs : l.max_tokens;
    if (tiles <= kCaWholeTiles) return 0;
    const int64_t items = ((int64_t)l.max_tokens * (nq / nkv) / kCaRows + seqs) * nkv, slots = items * ((tiles + kCaMinTiles - 1) / kCaMinTiles);
    return slots < kAttnMaxSlots ? (int)slots : kAttnMaxSlots;
}
int64_t attention_slot_bytes(int head_dim);
int64_t sample_slices(int vocab, int max_rows);
int64_t sample_stat_bytes();
int64_t sample_bins_bytes();

hipError_t launch_serving_tables(const ServingDev &S, const etc_serving_tables_io &io, hipStream_t s);
hipError_t launch_serving_append(const ServingDev &S, const etc_serving_append_io &io, hipStream_t s);
hipError_t launch_serving_attention(const ServingDev &S, const etc_serving_attention_io &io, hipStream_t s);
hipError_t launch_serving_sample(const ServingDev &S, const etc_serving_sample_io &io, hipStream_t s);
hipError_t launch_serving_append_codes(const ServingDev &S, const etc_serving_append_codes_io &io, hipStream_t s);
hipError_t launch_serving_attention_codes(const ServingDev &S, const etc_serving_attention_codes_io &io, hipStream_t s);
hipError_t launch_serving_score(const ServingDev &S, const etc_serving_score_io &io, hipStream_t s);

}  // namespace etc
