// Attention over the 4-bit cache of keys and values and windowed attention of prompts: how the cache lies in
// memory, what the kernels are given, and how a call is cut into workgroups.
//
// Cache.  A block of 32 features of one token and head shares a scale 2^e, e = floor(log2(largest magnitude)) - 2,
// at least 2^-126, kept as the byte e + 127; 255 marks a block that held an infinity or a NaN and reads as NaN.  Its values are a sign and
// one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale in four bits.  A page holds `page` tokens of every head; what one
// head has in it lies together, so that a workgroup streams whole pieces of memory:
//   codes of the keys, codes of the values (page * D / 2 bytes each), scales of the keys, of the values (page * scale_bytes(D) each).
// A 32-bit word holds 8 neighbouring features of one token, 32 s + 8 q and up, feature i in bits 4 i and up: what
// one lane hands to a matrix instruction as 8 steps of the reduction, all under one scale.  The words of 16 tokens lie in lane
// order: lane 16 q + (token % 16) of a wavefront finds its words s = 0 .. D/32 - 1 side by side, so that one load instruction fetches 16
// tokens (32 where D = 64) as one contiguous piece.  The values' words have another order of lanes (value_lane), that of
// which the unpacked rows go to the LDS without bank conflicts.  No byte belongs to two tokens: tokens are written
// independently of each other.
#pragma once
#include <cstdint>

#include "shflbw.h"

#if defined(__HIP__) || defined(__HIPCC__)
#define SHFLBW_HD __host__ __device__
#else
#define SHFLBW_HD
#endif

namespace shflbw {

// The largest scale byte of a finite block: of 65504 (binary16), of exponent 127 (bfloat16).  Larger ones are in slots that were never written, or 255:
// 16 bits may not hold their values, so attention keeps them from queries that do not see them as it does NaN.
SHFLBW_HD constexpr unsigned most_scale(bool bf16) { return bf16 ? 252 : 140; }
SHFLBW_HD constexpr int scale_bytes(int D) { return D == 64 ? 2 : 4; }   // a token's scales, as one load
SHFLBW_HD constexpr int64_t page_head_bytes(int page, int D) { return (int64_t)page * (D + 2 * scale_bytes(D)); }
// Which 16-byte (12 for D = 96; 8 of 16 for D = 64) piece of its 16 tokens a token's words of q (0..3) are
SHFLBW_HD constexpr int key_lane(int token, int q) { return q * 16 + (token & 15); }
SHFLBW_HD constexpr int value_lane(int token, int q) { return (q >> 1) * 32 + ((token >> 3) & 1) * 16 + (token & 7) * 2 + (q & 1); }
// Where the first word of lane `lane` of the 16 tokens around `token` lies, in bytes from the codes' start
SHFLBW_HD constexpr int code_offset(int D, int token, int lane)
{
    return D == 64 ? (token >> 5) * 1024 + lane * 16 + ((token >> 4) & 1) * 8 : (token >> 4) * (D * 8) + lane * (D / 8);
}

// What both attention kernels are given.  Keys and values come from the cache, or (prompt) lie as the queries do.
struct AttnArgs {
    const uint16_t* q;        // [q_heads * D][tokens], tokens innermost
    const uint16_t* k;        // prompt: [heads * D][tokens]
    const uint16_t* v;
    const char* cache;
    const int32_t* table;     // pages of every sequence
    const int32_t* lengths;   // cached tokens of every sequence
    const int32_t* starts;    // first query of every sequence and the end; nullptr: one query each (prompt: one sequence)
    uint16_t* out;
    float* part_o;            // nullptr: out takes the results.  Otherwise [split][q_head][token][D] sums that are not divided yet ..
    float* part_ml;           // .. and [split][q_head][token][2], their maximum and sum of weights
    int64_t ldq, ldk, ldv, ldo, table_ld;
    int64_t tokens;           // columns of q
    int table_width;          // pages a sequence can have
    int batch, heads, group;  // group: query heads per key head
    int pages, page_shift;
    int window, sinks;        // window INT32_MAX: none
    float scale;              // log2(e) / sqrt(D)
    int splits, split_tiles;  // parts a sequence's keys are cut into, key tiles of a part
    int col_blocks;           // blocks of columns of a sequence and key head
    // Prefixes: a "sequence" is a prefix, whose queries are those of sequences members[b] to members[b + 1] - 1 (nullptr: of all) and see all of its keys
    bool shared;
    const int32_t* members;
    int sequences;            // of `starts`
    // Sequences behind prefixes: their keys are the prefix's, from 0 on, and their own, from the next multiple of a tile on
    bool behind;
    const int32_t *prefix_table, *prefix_lengths;
    int64_t prefix_ld;
    int prefix_width, prefixes;
    // Parts of other keys (prefixes') to be joined with what the decoding kernel finds: `joined` of them, up to ATTN_JOINED, as part_o and part_ml
    const float *joined_o, *joined_ml;
    int joined;
};
constexpr int ATTN_JOINED = 32;

// Wavefronts per SIMD of the decoding kernel that the plan counts on.  Its registers allow no more, but for heads of 64 with 32 and 48
// columns, which compile to 119 and 155: 4 and 3 would fit.
SHFLBW_HD constexpr int decode_residency(int col_tiles, int D) { return col_tiles == 1 ? 4 : col_tiles == 2 && D < 128 ? 3 : col_tiles == 4 && D == 128 ? 1 : 2; }
// Of the other; where it is 3, a CU holds three workgroups of 4 wavefronts: two prompts of 16384 under a window of 1024, 16 heads of 64 take
// 302 us in these, 340 in workgroups of 8, of which it holds one, 329 in two of 4.  Of 4 for heads of 128 the LDS holds one.
SHFLBW_HD constexpr int tile_residency(int D, bool cache, int waves) { return waves == 4 && D == 128 ? 1 : waves == 4 && D == 64 && !cache ? 3 : 2; }
// Rows of a join up to which a row has a workgroup: calls with 128 rows of 32 parts take 52.2 us with it, 54.0 without, with 4096 of 8 30.5 and 27.1 (between
// these nothing was measured)
constexpr int ATTN_FEW_ROWS = 2048;
constexpr int ATTN_DECODE_KEYS = 32;     // keys of a tile of the decoding kernel
constexpr int ATTN_TILE_KEYS = 64;       // keys of a tile of the other
constexpr int ATTN_TILE_QUERIES = 32;    // queries of an item there
constexpr int64_t ATTN_MAX_LD = 1 << 26;  // of a prompt's keys and values: 32 rows span less than 4 GiB

struct AttnPlan {
    bool decode;              // the kernel for few queries
    int col_tiles;            // its 16-column tiles per wavefront
    int waves;                // wavefronts per workgroup
    bool tiny;                // the other's form for a prompt of fewer than 64 columns in all
    int col_blocks, splits, split_tiles;
    int64_t groups;           // workgroups
    int64_t workspace;        // bytes
};

// Which sequence and key head (pair), and which of its per_pair workgroups, workgroup `block` of the tile kernel is.  The GPU deals workgroups
// to its eight XCDs in turn.  Where heads come in fours, a pair's workgroups are on one XCD, whose L2 holds its keys and values, and every XCD
// has much the same share of each sequence: 8 prompts of 400 to 4000 tokens, 16 query heads of 128 over 4, 298 us, dealt to all XCDs 315.
// Other pairs, and what eights of pairs leave over, are dealt to all XCDs alike: 16 over 2 heads of 4 such prompts 171 us, on one XCD each
// 285; one prompt of 8000, 5 over 1 head, 166 and 870.
struct AttnPlace {
    int pair, inner;
};
SHFLBW_HD inline AttnPlace attn_place(int block, int pairs, int heads, int per_pair)
{
    const int dealt = heads % 4 ? pairs : pairs % 8, at = block - dealt * per_pair;
    if (at >= 0) return AttnPlace{dealt + at % 8 + at / 8 / per_pair * 8, at / 8 % per_pair};
    // round r begins on XCD dealt * r % 8, which comes back after 8 / (dealt's power of two) rounds: then all move on by one
    const int round = block / dealt, two = dealt & -dealt, on = (int)((int64_t)round * (two < 8 ? two : 8) / 8 % dealt);
    return AttnPlace{(block % dealt + on) % dealt, round};
}

// How attention over the cache is cut.  max_queries, max_length: of any sequence.
AttnPlan plan_cache_attention(int batch, int heads, int group, int D, int64_t tokens, int max_queries, int64_t max_length, int window, int sinks);
// The same for prompts, which need no workspace.  tokens: columns in all.
AttnPlan plan_prompt(int sequences, int heads, int group, int D, int64_t max_tokens, int window, int sinks, int64_t tokens = ATTN_TILE_KEYS);
// Which forms of the tile kernel there are: the launcher has these and no others, and a plan names one of them
constexpr bool tile_kernel_exists(int D, bool cache, int waves, bool tiny)
{
    return tiny ? !cache && waves == 4 : waves == 4 || (waves == 8 && (cache || D > 64));
}

// Attention over shared prefixes: the prefixes' part and the sequences' own part; or (behind) both at once, as `own`.  workspace: of all parts
struct SharedPlan {
    AttnPlan prefix, own;
    bool behind;
    bool joins;               // the own part's kernel joins the prefixes' parts
    int64_t workspace;
};
// keys_fit: a sequence's keys behind its prefix's are counted in 32 bits
SharedPlan plan_shared_attention(int prefixes, int64_t max_sharing, int64_t max_prefix, int batch, int heads, int group, int D, int64_t tokens, int max_queries,
                                 int64_t max_length, bool keys_fit);

// SHFLBW_OK, or why the cache cannot be used (host checks of its fields)
int check_cache(const shflbw_kv_cache* cache);
// The launchers of attention_kernel.hip, one translation unit per operand format: the kernel that the plan says, and the join of
// its parts.  prompt: keys and values in a.k and a.v.
int run_attention_f16(const AttnArgs& a, const AttnPlan& plan, int head_dim, bool prompt, void* stream);
int run_attention_bf16(const AttnArgs& a, const AttnPlan& plan, int head_dim, bool prompt, void* stream);
// The same for both parts of attention over shared prefixes, whose parts lie one behind the other, and the join of all
int run_shared_attention_f16(const AttnArgs& prefix, const AttnArgs& own, const SharedPlan& plan, int head_dim, void* stream);
int run_shared_attention_bf16(const AttnArgs& prefix, const AttnArgs& own, const SharedPlan& plan, int head_dim, void* stream);

}  // namespace shflbw
