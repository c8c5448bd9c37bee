// How the policy loss cuts its rows, in plain C++ (no HIP): a function of the sizes alone, so that workspace and launch agree.
#pragma once
#include <stdint.h>

namespace reqat {

struct PolicyPlan {
    int64_t slices, slice;                 // workgroups to a row, and the elements of each; 1: whole rows
};

// Up to 128 rows are cut into slices of at least 8 KB, 32 a row at most, for some 1024 workgroups in all: a row of 152064
// bfloat16 logits by itself takes one compute unit 24 us with its gradient.  Loss and gradient of such rows in a graph, whole
// rows and slices, us: 1 row 24.5 and 10.0, 24 rows 25.0 and 13.3, 64 rows 25.4 and 19.0, 96 rows 25.9 and 22.1, 128 rows 27.0
// and 26.4, 160 rows 28.3 and 31.1, 256 rows 34.5 and 43.9, 512 rows 60.5 and 78.8 (FP32: 35.0 and 11.6, 36.6 and 17.6, 41.1 and
// 26.4, 42.9 and 35.6, 45.0 and 45.1, 48.4 and 52.3, 66.6 and 78.5, 163 and 208).  300 rows are two rounds of 256 workgroups,
// the second nearly empty: 55.3 and 51.3 (111 and 108), which no rule takes care of.
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
