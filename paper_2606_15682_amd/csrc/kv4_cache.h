// The paged 4-bit cache: where a token's codes and scales lie, for its writer and reader
// (kv4_cache.hip) and for the attention over it (kv4_attention.hip).
//
// A page holds page_size = 2^page_log2 tokens of every KV head; per page and head
//   keys    codes  [token][D / 2],               element 2i in bits 3:0 of byte i
//           scales [token][D / 16]
//   values  codes  [token / 4][D / 8][4][4]      dword (w, t): channels 8w .. 8w+7 of token t of four
//           scales [token / 4][D / 16][4]
// A matrix-core tile of scores takes 16 or 32 bytes of one token's keys per lane, and the product
// with the values wants four tokens of the same channels in a lane: both are one wide load here.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace reqat {

struct Kv4View {
    uint8_t *kc, *ks, *vc, *vs;
    const float *gk, *gv, *shift;          // shift: kv_heads x D, or null
    int64_t pages;
    int page_log2, heads, D;

    __host__ __device__ int64_t slots() const { return pages << page_log2; }
    // first token of a (page, head) pair, in tokens
    __host__ __device__ int64_t run(int64_t page, int head) const { return (page * heads + head) << page_log2; }
};

// Token `tok` of the (page, head) run that starts at token `run`: byte offsets of its
// first key code and key scale, and of the value codes and scales of channel block b (of 16).
__host__ __device__ __forceinline__ int64_t kv4_k_codes(int64_t run, int tok, int D) { return (run + tok) * (D / 2); }
__host__ __device__ __forceinline__ int64_t kv4_k_scales(int64_t run, int tok, int D) { return (run + tok) * (D / 16); }
__host__ __device__ __forceinline__ int64_t kv4_v_codes(int64_t run, int tok, int b, int D) {
    return run * (D / 2) + (int64_t)(tok >> 2) * (2 * D) + b * 32 + (tok & 3) * 4;   // and 16 bytes on: channels 8 .. 15
}
__host__ __device__ __forceinline__ int64_t kv4_v_scales(int64_t run, int tok, int b, int D) {
    return run * (D / 16) + (int64_t)(tok >> 2) * (D / 4) + b * 4 + (tok & 3);
}

}  // namespace reqat
