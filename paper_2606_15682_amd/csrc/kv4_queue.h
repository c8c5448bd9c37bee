// The queue in LDS through which a wave of the decode attention (kv4_attention.hip) takes its codes and scales: direct
// loads, each lane's where the lane finds them again, so that what is on its way takes no registers (106 of the up to 128 that
// sixteen waves a CU may have; 64 more with loads into registers).
#pragma once

#include "g2l.h"

namespace reqat {

// g2l16 past the caches: codes are read once.  64 sequences of up to 16384 tokens (8 KV heads) 153 -> 137 us, 131072
// tokens of one 37.5 -> 34.9, when it was changed; with the scales' loads, several to a line, so too: no further gain.
__device__ __forceinline__ void g2l16_once(const uint8_t *base, uint32_t voff, uint8_t *l) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(voff), "s"(base), "{m0}"((uint32_t)(uintptr_t)l));
}

struct Kv4Queue {
    static constexpr int kDepth = 1;                                     // steps on their way beside the one computed on (2: no faster)
    static constexpr int kLoads = 8;                                     // of a step, in each wave
    static constexpr int kKeys = 0, kValues = 2048, kKeyScales = 4096, kValueScales = 4608;
    static constexpr int kStage = 5120;                                  // twice 16 tokens

    // Loads the 16 tokens whose codes and scales begin at these (scalar) addresses as half u of a stage.
    __device__ __forceinline__ static void put(const uint8_t *kc, uint32_t k_at, const uint8_t *vc, uint32_t v_at, const uint8_t *ks,
                                               uint32_t ks_at, const uint8_t *vs, uint32_t vs_at, uint8_t *stage, int u) {
        g2l16_once(kc, k_at, stage + kKeys + u * 1024);
        g2l16_once(vc, v_at, stage + kValues + u * 1024);
        g2l4(ks, ks_at, stage + kKeyScales + u * 256);
        g2l4(vs, vs_at, stage + kValueScales + u * 256);
    }
};

}  // namespace reqat
