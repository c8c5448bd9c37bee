// How the norm kernels cut a call, in plain C++ (no HIP): a function of the sizes alone, so that workspace and launch agree.
#pragma once
#include <stdint.h>

namespace reqat {

constexpr int64_t kNormMaxCols = 32768;    // 512 threads of eight vectors of bfloat16, or 1024 of eight of FP32

// Groups of G threads, a row each, that a workgroup of the backward pass has.
constexpr int norm_groups(int G) { return G == 64 ? 4 : 1; }

// Vectors of a row that a thread of such a group holds: the kernels that there are.
constexpr int norm_least_vectors(int G) { return G == 64 ? 1 : (G == 256 ? 2 : (G == 512 ? 3 : 5)); }
constexpr int norm_most_vectors(int G) { return G <= 256 ? 4 : 8; }

struct NormPlan {
    int threads;                           // of a row's group: 64 (four groups a workgroup), 256, 512 or 1024
    int vpt;                               // 16-byte vectors of a row a thread holds
    int64_t forward, backward;             // workgroups
    bool columns;                          // dw and db by columns, in a launch of their own
    int64_t sums;                          // rows of partial sums of dw, and of db
};

// Forward: eight workgroups of 256 threads a compute unit (9001 x 3584 bfloat16 in 27 us; with two, 39 us).  Backward: as
// many as keep a row ahead in flight, for each leaves a row of sums that the second launch reads (8192 x 5120: two
// workgroups of 256 threads a compute unit 54 us, four 110 us; 4096 x 8960: one of 512 threads 54 us, two 62 us), and
// from 128 rows on two rows each for the same reason (256 x 5120: 12.2 us for 15.3).
inline NormPlan norm_plan(int64_t M, int64_t K, bool bf16) {
    const int64_t vectors = (K + (bf16 ? 7 : 3)) / (bf16 ? 8 : 4);
    NormPlan p;
    p.threads = vectors <= 4 * 64 ? 64 : (vectors <= 4 * 256 ? 256 : (vectors <= 8 * 512 ? 512 : 1024));
    p.vpt = (int)((vectors + p.threads - 1) / p.threads);
    const int64_t groups = norm_groups(p.threads), units = (M + groups - 1) / groups;
    p.columns = p.vpt > 4;
    const int64_t forward = p.threads <= 256 ? 2048 : (p.columns ? 256 : 1024);
    const int64_t backward = p.threads <= 256 || p.columns ? 512 : 256;
    p.forward = units < forward ? units : forward;
    const int64_t wanted = p.threads == 64 || units <= 128 ? units : (units < 256 ? 128 : (units + 1) / 2);
    p.backward = wanted < backward ? wanted : backward;
    p.sums = !p.columns ? p.backward : (M < 64 ? M : 64);
    return p;
}

}  // namespace reqat
