// How the norm kernels cut a call, in plain C++ (no HIP): a function of the sizes alone, so that workspace and launch agree.
#pragma once
#include <stdint.h>

namespace reqat {

constexpr int64_t kNormMaxCols = 32768;    // 1024 threads of four vectors of bfloat16, or eight of FP32

struct NormPlan {
    int threads;                           // of a row's group: 64 (four groups a workgroup), 256 or 1024
    int vpt;                               // 16-byte vectors of a row a thread holds: 1 to 4, of 1024 threads and FP32 to 8
    int64_t workgroups, groups;
};

inline NormPlan norm_plan(int64_t M, int64_t K, bool bf16) {
    const int64_t vectors = (K + (bf16 ? 7 : 3)) / (bf16 ? 8 : 4);
    NormPlan p;
    p.threads = vectors <= 4 * 64 ? 64 : (vectors <= 4 * 256 ? 256 : 1024);
    p.vpt = (int)((vectors + p.threads - 1) / p.threads);
    const int64_t rows = p.threads == 64 ? 4 : 1, most = p.threads == 1024 ? 256 : 512;
    p.workgroups = (M + rows - 1) / rows;
    if (p.workgroups > most) p.workgroups = most;
    p.groups = p.workgroups * rows;
    return p;
}

}  // namespace reqat
