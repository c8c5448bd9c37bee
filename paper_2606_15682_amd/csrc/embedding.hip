// Embedding lookup with a factor and its gradient, for gfx950:
//   out_t = RN(scale table[id_t]),   dtable_v = RN([dtable_v +] scale sum_{t: id_t = v} dy_t), in the order of t.
// An id outside the table is padding: a row of zeros, and no gradient.
//
// The gradient sorts the tokens by id (a counting sort in one launch), then adds up each id's rows.  A run of equal ids
// is cut into pieces of kPiece tokens, so that a frequent token is not one workgroup's work; the pieces' sums are joined in
// order by a last launch.  Every sum has a fixed order.
#include "internal.h"
#include "row_io.h"

namespace reqat {

namespace {

constexpr int kPiece = kEmbedPiece;

// ------------------------------------------------------------------ lookup: a wave per token

template <typename T> __global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
    constexpr int N = kVec<T>;
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= a.T) return;
    const int32_t id = a.ids[t];
    const bool known = id >= 0 && id < a.V;
    const T *row = reinterpret_cast<const T *>(a.table) + (int64_t)(known ? id : 0) * a.ld_table;
    T *out = reinterpret_cast<T *>(a.out) + t * a.ld_out;
    const int D = (int)a.D;
    for (int j = (threadIdx.x & 63) * N; j < D; j += 64 * N) {
        const int n = D - j;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (known) {
            v = n >= N ? load_vec(row + j) : load_part(row + j, n);
            if (a.scale != 1.0f) {
                float z[N];
                unpack<T>(v, z);
#pragma unroll
                for (int e = 0; e < N; ++e) z[e] *= a.scale;
                v = pack<T>(z);
            }
        }
        if (n >= N) store_vec(out + j, v);
        else store_part(out + j, v, n);
    }
}

// ------------------------------------------------------------------ tokens by id

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;

// Workgroup g owns the ids [g R, g R + R).  Each reads all ids twice (the caches hold them): it counts the tokens of lower
// ids, which is where its own begin, and its own by wave and id; then every wave goes through its part of the tokens
// again, in order, and puts each into its place.  No workgroup waits for another.
//   row_start [V + 1]: first place of an id;  order, sorted [T]: token and id at a place.
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const int32_t *__restrict__ ids, int64_t T, int32_t V, int R,
                                                                  int32_t *__restrict__ row_start,
                                                                  int32_t *__restrict__ order, int32_t *__restrict__ sorted) {
    extern __shared__ int32_t count[];                  // [kSortWaves][R]
    __shared__ int32_t below_of[kSortWaves], sum_of[kSortWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t lo = (int32_t)blockIdx.x * R;
    const uint32_t width = (uint32_t)(V - lo < R ? V - lo : R);
    for (int k = threadIdx.x; k < kSortWaves * R; k += kSortThreads) count[k] = 0;
    __syncthreads();
    const int64_t part = (T + kSortThreads - 1) / kSortThreads * 64;
    const int64_t begin = wave * part, end = begin + part < T ? begin + part : T;
    int32_t *mine = count + wave * R;
    int32_t below = 0;
    for (int64_t t = begin + lane; t < end; t += 64) {
        const int32_t id = ids[t];
        if (id >= 0 && id < lo) ++below;
        const uint32_t k = (uint32_t)id - (uint32_t)lo;                     // out of range for padding too
        if (k < width) atomicAdd(&mine[k], 1);          // a count: the order of the additions does not show
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) below += __shfl_xor(below, off, 64);
    if (lane == 0) below_of[wave] = below;
    __syncthreads();
    // thread k: the tokens of id lo + k; places of its waves' parts
    int32_t total = 0;
    if ((int)threadIdx.x < R)
        for (int w = 0; w < kSortWaves; ++w) total += count[w * R + threadIdx.x];
    int32_t incl = total;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int32_t u = __shfl_up(incl, off, 64);
        if (lane >= off) incl += u;
    }
    if (lane == 63) sum_of[wave] = incl;
    __syncthreads();
    int32_t place = incl - total;
    for (int w = 0; w < kSortWaves; ++w) place += below_of[w] + (w < wave ? sum_of[w] : 0);
    if (threadIdx.x < width) {
        row_start[lo + threadIdx.x] = place;
        if (lo + (int32_t)threadIdx.x == V - 1) row_start[V] = place + total;
    }
    if ((int)threadIdx.x < R)
        for (int w = 0; w < kSortWaves; ++w) {
            const int32_t n = count[w * R + threadIdx.x];
            count[w * R + threadIdx.x] = place;
            place += n;
        }
    __syncthreads();
    for (int64_t t0 = begin; t0 < end; t0 += 64) {
        const int64_t t = t0 + lane;
        const int32_t id = t < end ? ids[t] : -1;
        uint64_t left = __ballot((uint32_t)id - (uint32_t)lo < width);
        while (left) {                                  // one turn for each different id among the 64
            const int first = __builtin_ctzll(left);
            const int32_t one = __shfl(id, first, 64);
            const uint64_t same = __ballot(id == one);
            volatile int32_t *at = &mine[one - lo];     // the wave's own counter
            const int32_t base = *at;
            if (id == one) {
                const int32_t p = base + __builtin_popcountll(same & ((1ull << lane) - 1));
                order[p] = (int32_t)t;
                sorted[p] = id;
            }
            __builtin_amdgcn_wave_barrier();
            if (lane == first) *at = base + __builtin_popcountll(same);
            __builtin_amdgcn_wave_barrier();
            left &= ~same;
        }
    }
}

// ------------------------------------------------------------------ sums of rows

// Adds dy of the tokens order[p .. p + n) to acc, elements j .. j + kVec - 1 (m of them exist).
template <typename T>
__device__ __forceinline__ void add_rows(const EmbedGradArgs &a, int64_t p, int n, int64_t j, int m, float (&acc)[kVec<T>]) {
    constexpr int N = kVec<T>;
    const T *dy = reinterpret_cast<const T *>(a.dy) + j;
    for (int k = 0; k < n; k += 4) {
        uint4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            v[u] = make_uint4(0, 0, 0, 0);
            if (k + u < n) {
                const T *row = dy + (int64_t)a.order[p + k + u] * a.ld_dy;
                v[u] = m >= N ? load_vec(row) : load_part(row, m);
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (k + u >= n) break;
            float z[N];
            unpack<T>(v[u], z);
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += z[e];
        }
    }
}

// dtable[id][j ..] = RN([old +] scale acc).
template <typename T, typename G>
__device__ __forceinline__ void put_row(const EmbedGradArgs &a, int32_t id, int64_t j, int m, const float (&acc)[kVec<T>]) {
    G *out = reinterpret_cast<G *>(a.dtable) + (int64_t)id * a.ld_table + j;
#pragma unroll
    for (int e0 = 0; e0 < kVec<T>; e0 += kVec<G>) {
        constexpr int NG = kVec<G> < kVec<T> ? kVec<G> : kVec<T>;
        const int n = m - e0;
        if constexpr (NG == kVec<G>) {
            float z[NG];
            if (a.accumulate && n > 0) unpack<G>(n >= NG ? load_vec(out + e0) : load_part(out + e0, n), z);
#pragma unroll
            for (int e = 0; e < NG; ++e) z[e] = (a.accumulate ? z[e] : 0.0f) + a.scale * acc[e0 + e];
            if (n >= NG) store_vec(out + e0, pack<G>(z));
            else if (n > 0) store_part(out + e0, pack<G>(z), n);
        } else {                                        // FP32 rows into a bfloat16 table
#pragma unroll
            for (int e = 0; e < NG; ++e)
                if (e < n) out[e] = from_f32<G>((a.accumulate ? to_f32(out[e]) : 0.0f) + a.scale * acc[e]);
        }
    }
}

// Workgroups 0 .. T - 1: the piece that begins at a place, if one does.  A run of at most kPiece tokens is finished here;
// a longer one's pieces leave their sums in the workspace, in row 2 (p / kPiece) + [first piece]: pieces of one run are
// kPiece apart, and a second run's first piece is the only other one that can begin between them.
// Workgroups T .. T + V - 1 (a fresh table): zeros for ids without tokens.
template <typename T, typename G> __global__ __launch_bounds__(256) void embed_sum_kernel(EmbedGradArgs a) {
    constexpr int N = kVec<T>;
    const int64_t D = a.D;
    if ((int64_t)blockIdx.x >= a.T) {
        const int32_t id = (int32_t)(blockIdx.x - a.T);
        if (a.row_start[id] != a.row_start[id + 1]) return;
        const float none[N] = {};
        for (int64_t j = threadIdx.x * N; j < D; j += 256 * N) put_row<T, G>(a, id, j, (int)(D - j), none);
        return;
    }
    const int64_t p = blockIdx.x;
    if (p >= a.row_start[a.V]) return;
    const int32_t id = a.sorted[p], start = a.row_start[id], n = a.row_start[id + 1] - start;
    const int32_t k = (int32_t)p - start;
    if (k % kPiece) return;
    const int len = n - k < kPiece ? n - k : kPiece;
    for (int64_t j = threadIdx.x * N; j < D; j += 256 * N) {
        float acc[N] = {};
        add_rows<T>(a, p, len, j, (int)(D - j), acc);
        if (n <= kPiece) {
            put_row<T, G>(a, id, j, (int)(D - j), acc);
        } else {
            float *part = a.partials + (2 * (p / kPiece) + (k == 0)) * D + j;
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (j + e < D) part[e] = acc[e];
        }
    }
}

// Workgroup f joins the pieces of the run of more than kPiece tokens that begins at a place from f kPiece on, below
// (f + 1) kPiece, if there is one: there cannot be two.
template <typename G> __global__ __launch_bounds__(256) void embed_join_kernel(EmbedGradArgs a) {
    const int64_t valid = a.row_start[a.V];
    int64_t head = -1;
    int32_t id = 0, n = 0;
    const int64_t p = (int64_t)blockIdx.x * kPiece + (threadIdx.x & 63);
    bool is = false;
    if (p < valid) {
        id = a.sorted[p];
        n = a.row_start[id + 1] - a.row_start[id];
        is = a.row_start[id] == p && n > kPiece;
    }
    const uint64_t found = __ballot(is);
    if (!found) return;
    const int lane = __builtin_ctzll(found);
    head = (int64_t)blockIdx.x * kPiece + lane;
    id = __shfl(id, lane, 64);
    n = __shfl(n, lane, 64);
    for (int64_t j = (int64_t)blockIdx.y * 1024 + threadIdx.x * 4; j < a.D && j < (int64_t)(blockIdx.y + 1) * 1024; j += 1024) {
        float acc[4] = {};
        for (int64_t q = head; q < head + n; q += kPiece) {
            const float *part = a.partials + (2 * (q / kPiece) + (q == head)) * a.D + j;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e < a.D) acc[e] += part[e];
        }
        put_row<float, G>(a, id, j, (int)(a.D - j), acc);
    }
}

}  // namespace

hipError_t launch_embedding(const EmbedArgs &a, bool bf16, hipStream_t stream) {
    if (a.T == 0 || a.D == 0) return hipSuccess;
    const dim3 grid((unsigned)((a.T + 3) / 4)), block(256);
    if (bf16) hipLaunchKernelGGL(embed_kernel<uint16_t>, grid, block, 0, stream, a);
    else hipLaunchKernelGGL(embed_kernel<float>, grid, block, 0, stream, a);
    return hipGetLastError();
}

namespace {

template <typename T, typename G> hipError_t launch_sums(const EmbedGradArgs &a, hipStream_t stream) {
    const int64_t groups = a.T + (a.accumulate ? 0 : a.V);
    hipLaunchKernelGGL((embed_sum_kernel<T, G>), dim3((unsigned)groups), dim3(256), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.T <= kPiece) return e;       // no run of more than a piece
    hipLaunchKernelGGL(embed_join_kernel<G>, dim3((unsigned)((a.T + kPiece - 1) / kPiece), (unsigned)((a.D + 1023) / 1024)), dim3(256),
                       0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding_backward(const EmbedGradArgs &a, const int32_t *ids, bool bf16, bool table_bf16, hipStream_t stream) {
    if (a.V == 0 || a.D == 0 || (a.T == 0 && a.accumulate)) return hipSuccess;
    // ids a workgroup sorts: at most 960 (one a thread, 60 KB of LDS), and some 256 workgroups where that allows it
    int R = (int)((a.V + 255) / 256);
    R = R > 960 ? 960 : R;
    hipLaunchKernelGGL(embed_sort_kernel, dim3((unsigned)((a.V + R - 1) / R)), dim3(kSortThreads), (size_t)(kSortWaves * R * 4), stream,
                       ids, a.T, (int32_t)a.V, R, a.row_start, a.order, a.sorted);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (bf16) return table_bf16 ? launch_sums<uint16_t, uint16_t>(a, stream) : launch_sums<uint16_t, float>(a, stream);
    return table_bf16 ? launch_sums<float, uint16_t>(a, stream) : launch_sums<float, float>(a, stream);
}

// [row_start V + 1 | order T | sorted T] int32, then the pieces' sums on a 16-byte boundary.
size_t embedding_workspace_bytes(int64_t T, int64_t V, int64_t D) {
    return embedding_workspace_head(T, V) + (T > kPiece ? (size_t)(2 * ((T + kPiece - 1) / kPiece)) * (size_t)D * 4 : 0);
}

size_t embedding_workspace_head(int64_t T, int64_t V) { return ((size_t)(V + 1 + 2 * T) * 4 + 15) & ~(size_t)15; }

}  // namespace reqat
