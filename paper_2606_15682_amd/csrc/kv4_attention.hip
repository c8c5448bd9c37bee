// Attention over the paged 4-bit cache (W4A4KV4 serving, Sec. 4.3; layout in kv4_cache.h):
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i . k_j - max),  j over the row's visible tokens.
// The shift of the keys is left out of the scores: q . m is the same for every key of a row,
// and a softmax does not change when its scores all move by as much.
//
// The simple kernel: one wave per query and head; 64 tokens a step, one lane each for the scores,
// then D / 64 channels a lane for the values.
#include "internal.h"
#include "fp4_device.h"

namespace reqat {

namespace {

__device__ __forceinline__ float code_value(uint32_t c) {
    const float m = 0.5f * (float)(c & 7u);
    return (c & 8u) ? -m : m;
}

template <int D>
__global__ __launch_bounds__(64) void kv4_attention_simple_kernel(const Kv4AttnArgs a) {
    const int i = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, lane = threadIdx.x;
    int64_t q0 = b, q1 = b + 1;
    if (a.q_start) {
        q0 = a.q_start[b] < 0 ? 0 : a.q_start[b];
        q1 = a.q_start[b + 1] > a.T ? a.T : a.q_start[b + 1];
    }
    if (q0 + i >= q1) return;
    const int64_t row = q0 + i, nq = q1 - q0;
    const int64_t len = a.kv_len[b] < 0 ? 0 : a.kv_len[b];
    const bool lost = len > a.max_kv || len > (a.table_cols << a.c.page_log2);
    int64_t n = a.causal ? len - nq + i + 1 : len;
    if (n < 0) n = 0;
    const int h = hq / (a.q_heads / a.c.heads);
    __shared__ float q[D], p[64];
    for (int d = lane; d < D; d += 64) q[d] = f32_from_bits((uint32_t)a.q[row * a.ldq + hq * D + d] << 16);
    __syncthreads();
    float top = -__builtin_inff(), total = 0.0f, o[D / 64] = {};
    for (int64_t j0 = 0; j0 < n && !lost; j0 += 64) {
        const int64_t j = j0 + lane;
        float s = -__builtin_inff();
        if (j < n) {
            const int64_t page = a.table[b * a.ld_table + (j >> a.c.page_log2)];
            s = __builtin_nanf("");
            if (page >= 0 && page < a.c.pages) {
                const int tok = (int)(j & ((1 << a.c.page_log2) - 1));
                const int64_t run = a.c.run(page, h);
                s = 0.0f;
                for (int g = 0; g < D / 16; ++g) {
                    float t = 0.0f;
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t w = a.c.kc[kv4_k_codes(run, tok, D) + 8 * g + e];
                        t += q[16 * g + 2 * e] * code_value(w & 15u) + q[16 * g + 2 * e + 1] * code_value(w >> 4);
                    }
                    s += t * e4m3_value(a.c.ks[kv4_k_scales(run, tok, D) + g]);
                }
                s *= a.scale * *a.c.gk;
            }
        }
        float m = s;
        for (int off = 32; off > 0; off >>= 1) m = __builtin_elementwise_maximum(m, __shfl_xor(m, off, 64));
        const float next = __builtin_elementwise_maximum(m, top);
        const float keep = top == -__builtin_inff() ? 0.0f : __expf(top - next);
        const float w = j < n ? __expf(s - next) : 0.0f;
        float sum = w;
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
        total = total * keep + sum;
        top = next;
        __syncthreads();
        p[lane] = w;
        __syncthreads();
        for (int e = 0; e < D / 64; ++e) {
            const int d = lane * (D / 64) + e;
            float acc = 0.0f;
            for (int u = 0; u < 64 && j0 + u < n; ++u) {
                const int64_t page = a.table[b * a.ld_table + ((j0 + u) >> a.c.page_log2)];
                if (page < 0 || page >= a.c.pages) continue;
                const int tok = (int)((j0 + u) & ((1 << a.c.page_log2) - 1));
                const int64_t run = a.c.run(page, h);
                const uint32_t byte = a.c.vc[kv4_v_codes(run, tok, d / 16, D) + (d % 16 / 8) * 16 + d % 8 / 2];
                acc += p[u] * (code_value((d & 1) ? byte >> 4 : byte & 15u) * e4m3_value(a.c.vs[kv4_v_scales(run, tok, d / 16, D)]));
            }
            o[e] = o[e] * keep + acc;
        }
    }
    const float inv = n == 0 && !lost ? 0.0f : *a.c.gv / total;
    for (int e = 0; e < D / 64; ++e) {
        const float y = lost ? __builtin_nanf("") : n == 0 ? 0.0f : o[e] * inv;
        a.out[row * a.ldo + hq * D + lane * (D / 64) + e] = (uint16_t)bf16_rne_from_float(y);
    }
    if (a.lse && lane == 0)
        a.lse[row * a.q_heads + hq] = lost ? __builtin_nanf("") : n == 0 ? -__builtin_inff() : top + __logf(total);
}

}  // namespace

size_t kv4_attention_workspace_bytes(int64_t, int64_t, int64_t, int64_t, int, int, int) { return 0; }

hipError_t launch_kv4_attention(const Kv4AttnArgs &a, hipStream_t stream) {
    const dim3 grid((unsigned)a.max_q, (unsigned)a.q_heads, (unsigned)a.B);
    if (a.c.D == 128) kv4_attention_simple_kernel<128><<<grid, 64, 0, stream>>>(a);
    else kv4_attention_simple_kernel<64><<<grid, 64, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace reqat
