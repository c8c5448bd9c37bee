// How the policy loss cuts its rows, in plain C++ (no HIP): a function of the sizes alone, so that workspace and launch agree.
#pragma once
#include <stdint.h>

namespace reqat {

struct PolicyPlan {
    int64_t slices, slice;                 // workgroups to a row, and the elements of each; 1: whole rows
};

// Up to 128 rows are cut into slices of at least 8 KB, 32 a row at most, for some 1024 workgroups in all: a row of 152064
// bfloat16 logits by itself takes one compute unit 23 us with its gradient.  Loss and gradient in a graph, whole rows and
// slices, us: 1 row 22.8 and 10.5, 24 rows 23.7 and 14.2, 128 rows 26.1 and 25.3, 256 rows 41.9 and 45.1, 512 rows 74.6 and
// 95.8 (FP32: 35.9 and 12.2, 40.6 and 19.3, 66.0 and 52.0, 96.4 and 104, 181 and 216).
inline PolicyPlan policy_plan(int64_t T, int64_t V, bool bf16) {
    const int64_t unit = bf16 ? 4096 : 2048, units = (V + unit - 1) / unit;
    PolicyPlan p = {1, V};
    if (T <= 0 || T > 128 || units < 2) return p;
    int64_t slices = (1024 + T - 1) / T;
    if (slices > 32) slices = 32;
    if (slices > units) slices = units;
    p.slice = (units + slices - 1) / slices * unit;
    p.slices = (V + p.slice - 1) / p.slice;
    return p;
}

}  // namespace reqat
