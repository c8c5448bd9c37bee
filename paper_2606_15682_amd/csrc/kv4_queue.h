// The queue in LDS through which a wave of the decode attention (kv4_attention.hip) takes its codes and scales: direct
// loads, each lane's where the lane finds them again, so that what is on its way takes no registers (102 instead of 166:
// sixteen waves a CU rather than twelve).
#pragma once

#include "g2l.h"

namespace reqat {

struct Kv4Queue {
    static constexpr int kDepth = 1;                                     // steps on their way beside the one computed on (2: no faster)
    static constexpr int kLoads = 8;                                     // of a step, in each wave
    static constexpr int kKeys = 0, kValues = 2048, kKeyScales = 4096, kValueScales = 4608;
    static constexpr int kStage = 5120;                                  // twice 16 tokens

    // Loads the 16 tokens whose codes and scales begin at these (scalar) addresses as half u of a stage.
    __device__ __forceinline__ static void put(const uint8_t *kc, uint32_t k_at, const uint8_t *vc, uint32_t v_at, const uint8_t *ks,
                                               uint32_t ks_at, const uint8_t *vs, uint32_t vs_at, uint8_t *stage, int u) {
        g2l16(kc, k_at, stage + kKeys + u * 1024);
        g2l16(vc, v_at, stage + kValues + u * 1024);
        g2l4(ks, ks_at, stage + kKeyScales + u * 256);
        g2l4(vs, vs_at, stage + kValueScales + u * 256);
    }
};

}  // namespace reqat
