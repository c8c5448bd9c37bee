// How a call of the attention over the KV4 cache is cut: a rule on sizes alone, in plain C++ (no HIP), so that a CPU
// test can ask it for any shape.
#pragma once
#include <stdint.h>

namespace reqat {

// The rows of a KV head (queries x heads of its group) go to qtiles of 16 x tiles rows; the tokens of
// a sequence to `splits` pieces of `chunk`, a workgroup each, whose results a second kernel joins (splits > 1).
//
// Up to 32 rows (tiles 1, 2) a wave does all by itself, 32 tokens a step; beyond, the kernel for prompts, in which waves
// without rows only unpack (16 sequences of up to 4000 tokens, 8 KV heads: 28.5 us with 25 rows, 48 to 53 with 35 to 80, 69 with 160, where the
// bytes take 11: no kernel here is made for 33 to 255 rows).
//
// Pieces: 512 workgroups of four waves, two per CU, where there are fewer units (sequence x KV head): 30000 tokens of one
// sequence with 8 KV heads take 16.4 us in 472 pieces, 20.5 in 944, whose results the join reads too.  Several
// sequences differ in length and max_kv is the longest's: pieces of at most 1536 tokens (64 sequences of up to
// 16384 tokens, 8 KV heads: 139 us, 170 in one piece each, 148 in pieces of 1024, 145 of 2048).  At most 256 pieces, of 256 tokens or
// more: shorter contexts are one piece and need no join; from 257 to 512 tokens eight waves take it (500
// tokens: 8.1 us, 8.6 in two pieces of four waves and a join; 250 tokens: 6.9 against 6.3).
struct Kv4Plan {
    int tiles;
    int64_t qtiles;                     // in an int where the launch fits
    int waves, splits, chunk;
};
constexpr int kKv4MaxSplits = 256;
constexpr int64_t kKv4MaxPieces = 8192; // in all, where the longest of several sequences asks for them
constexpr int kKv4Prompt = 16;          // tiles of the kernel for prompts: 256 rows

inline Kv4Plan kv4_plan(int64_t B, int64_t max_q, int64_t max_kv, int q_heads, int kv_heads) {
    Kv4Plan p;
    const int64_t rows = max_q * (q_heads / kv_heads);
    p.tiles = rows > 32 ? kKv4Prompt : rows > 16 ? 2 : 1;
    p.qtiles = (rows + 16 * p.tiles - 1) / (16 * p.tiles);
    const int64_t groups = B * kv_heads * p.qtiles;
    p.waves = 4;
    int64_t splits = 1;
    if (p.tiles == kKv4Prompt) {
        splits = groups > 0 ? (256 + groups - 1) / groups : 1;
    } else if (p.tiles == 1 && max_kv > 256 && max_kv <= 512 && groups <= 256) {
        p.waves = 8;
    } else {
        splits = groups > 0 ? (512 + groups - 1) / groups : 1;
        if (B > 1 && max_kv > 2048) {
            int64_t finer = (max_kv + 1535) / 1536;
            finer = finer * groups > kKv4MaxPieces ? kKv4MaxPieces / groups : finer;
            splits = splits < finer ? finer : splits;
        }
    }
    const int64_t most = (max_kv + 255) / 256;
    splits = splits > most ? most : splits;
    splits = splits > kKv4MaxSplits ? kKv4MaxSplits : splits;
    splits = splits < 1 ? 1 : splits;
    const int64_t chunk = ((max_kv + splits - 1) / splits + 127) / 128 * 128;
    p.chunk = (int)(chunk < 128 ? 128 : chunk);                          // max_kv <= 2^30
    p.splits = (int)((max_kv + p.chunk - 1) / p.chunk);
    if (p.splits < 1) p.splits = 1;
    return p;
}

// Rows of partial results (query x head x piece) that a workspace has room for: enough for the plan of a call and of every
// call with fewer sequences, queries or tokens, since fewer of them can mean more pieces.  Each bound below holds for
// the plans it names and grows with B, max_q and max_kv.  At most 8192 x 32 rows, 138 MB with heads of 128.
inline int64_t kv4_piece_rows(int64_t B, int64_t max_q, int64_t max_kv, int q_heads, int kv_heads) {
    const auto least = [](int64_t a, int64_t b) { return a < b ? a : b; };
    if (max_kv <= 256 || B <= 0 || max_q <= 0) return 0;                 // one piece
    const int64_t group = q_heads / kv_heads, units = B * kv_heads;      // units of up to 32 rows
    const int64_t most = least((max_kv + 255) / 256, kKv4MaxSplits);     // pieces of a unit
    // up to 32 rows: ceil(512 / units) pieces of fewer than 512 units, or pieces of 1536 tokens of several sequences
    int64_t pieces = least(511 + units, 1022);
    if (B > 1 && max_kv > 2048) {
        const int64_t finer = least(units * ((max_kv + 1535) / 1536), kKv4MaxPieces);
        pieces = pieces > finer ? pieces : finer;
    }
    const int64_t rows = group > 32 ? 0 : least(max_q, 32 / group) * group;
    const int64_t few = least(pieces, units * most) * rows;
    if (max_q * group <= 32) return few;
    // prompts: ceil(256 / tiles) pieces of fewer than 256 tiles of 256 rows
    const int64_t all = max_q * group, tiles = units * ((all + 255) / 256);
    const int64_t prompts = least(least(255 + tiles, 510) * least(all, 256), least(units * all, int64_t(1) << 40) * most);
    return few > prompts ? few : prompts;
}

// Whether the launch of a plan holds fewer than 2^32 threads (workgroups of up to 512).
inline bool kv4_plan_fits(const Kv4Plan &p, int64_t B, int kv_heads) {
    const int64_t n = B * kv_heads * p.splits;                           // below 2^40
    return n < (int64_t(1) << 23) && n * p.qtiles < (int64_t(1) << 23);  // qtiles below 2^40; 1 but for prompts
}

}  // namespace reqat
