// What the calls of the prompts' attention and its kernels share (prompt_attention.hip, prompt_kernel.h).
#pragma once

#include "kv_common.h"

namespace paro {

typedef float F4 __attribute__((ext_vector_type(4)));
typedef float F16 __attribute__((ext_vector_type(16)));
typedef uint32_t U4 __attribute__((ext_vector_type(4)));
typedef uint32_t U2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4, kPromptThreads = 64 * kWaves;
constexpr int kMaxSplits = 32;
constexpr int kSplitBlocks = 512;               // tiles are split while there are fewer of them
constexpr int kMostParts = 2 * kSplitBlocks;     // that a call can have
constexpr int kChip = 256;                       // compute units
constexpr int kLeastTokens = 256;                // that a part has at least
constexpr float kShift = 10.0f;                  // p is held 2^10 times
constexpr float kSlack = 5.0f;                   // the maximum that p is taken from may lie so far below the true one (2^15 is an fp16 number)
constexpr float kFarMax = 65536.0f;              // |maximum| above which scores are rounded before it is taken off
constexpr int kPromptRaw = 0x00020000;           // raw buffer, 32-bit data format
constexpr int kPromptAgent = 16;                 // agent scope: past the L2 of the XCD

// The shape of a block: each of its waves holds 32 pairs, WN of them hold the same ones and have every WN-th run of NB x 32 tokens.
template <int D_, int NB_, int WN_>
struct Shape {
    static constexpr int D = D_, NB = NB_, WN = WN_, WM = kWaves / WN_;
    static constexpr int Pairs = 32 * WM, Tokens = 32 * NB * WN, Quarters = Tokens / 64;   // 16-token runs of a tile that a wave moves
    static constexpr int TileBytes = Tokens * D * 2;     // of keys, and of values, as fp16 in LDS
    static constexpr int PartFloats = Pairs * (D + 2);
    static constexpr int Blocks = 4 * TileBytes <= 65536 ? 2 : 1;      // of a compute unit: their waves take turns at its pipes
};

struct PromptArgs {
    const uint8_t *k, *v, *ks, *vs;
    const _Float16 *q;
    const int32_t *starts, *table, *lengths, *prefix, *first;
    _Float16 *o;
    float *lse;
    uint32_t *arrived;                           // [tiles][kv_heads]
    float *partial;                              // [tiles][kv_heads][splits] of PartFloats
    int64_t ldq, ldo, ld_table;
    int page_log, n_pages, kv_heads, group, width, batch, window, T, tiles, splits;
    float scale;                                 // with log2(e)
    Scores scores;
};

// Most tiles of `pairs` pairs that T rows of `batch` sequences can have.
inline int64_t prompt_tiles(int64_t T, int64_t group, int64_t batch, int pairs)
{
    const int64_t all = T * group;
    return batch == 1 ? (all + pairs - 1) / pairs : all / pairs + (batch < T ? batch : T);
}
// Most parts that a tile is cut into.
inline int64_t prompt_splits(int64_t tiles, int64_t kv_heads)
{
    const int64_t heads = tiles * kv_heads, n = (kSplitBlocks + heads - 1) / heads;
    return n < kMaxSplits ? n : kMaxSplits;
}

// The shapes that calls choose from, by what they have of pairs: blocks of many, whose waves have pairs of their own, or of few, whose waves share
// pairs and have tokens of their own.  8 sequences of 16 rows x 4 heads of 128 channels behind 4000 tokens take 33 us in the latter, 36 in the former,
// of 32 rows 50 and 39; 16 sequences of 16 rows x 2 heads of 64 channels 35 and 40, of 32 rows 53 and 42; of 256 channels 56 and 69, 142 and 86.  The choice
// is by the mean of a call's sequences and the same for all of them: 200 single rows beside a prompt of 2000 take 170 us in blocks of few, 148 in the others;
// 15 of them beside a prompt of 4096 take 190 in blocks of many, 264 in the others.
// Two blocks to a compute unit where LDS holds them: one's first and last memory accesses are the other's products (four drafts of 5 rows of 128
// channels: 20 us, 28 with one of twice the tokens; 16 sequences of 4 rows behind 4000 tokens 49 either way, MXFP4 40 and 47).
template <int D> struct Shapes;
template <> struct Shapes<64> { typedef Shape<64, 2, 1> Many; typedef Shape<64, 1, 4> Few; };
template <> struct Shapes<128> { typedef Shape<128, 2, 1> Many; typedef Shape<128, 1, 2> Few; };
template <> struct Shapes<256> { typedef Shape<256, 2, 1> Many; typedef Shape<256, 1, 2> Few; };
constexpr int kFewPairs = 64;                    // of a sequence on average, up to which a call's are few

// By the cache's format (prompt_fp16.hip, prompt_e4m3.hip, prompt_mxfp4.hip, which take a minute each to compile).
hipError_t launch_prompt_fp16(int head_dim, bool scored, PromptArgs &a, hipStream_t s);
hipError_t launch_prompt_e4m3(int head_dim, bool scored, PromptArgs &a, hipStream_t s);
hipError_t launch_prompt_mxfp4(int head_dim, bool scored, PromptArgs &a, hipStream_t s);

}  // namespace paro
