// Embedding lookup with a factor and its gradient, for gfx950:
//   out_t = RN(scale table[id_t]),   dtable_v = RN([dtable_v +] scale sum_{t: id_t = v} dy_t), in the order of t.
// An id outside the table is padding: a row of zeros, and no gradient.
//
// The gradient sorts the tokens by id (a counting sort in one launch), then goes through them kPiece at a time: a wave adds
// up the rows of its piece, id by id, and finishes the ids whose tokens all lie in it; so every wave has the same work,
// however frequent an id is.  A run of equal ids that goes on into the next pieces is joined in order by a last launch.
// Up to kFewTokens tokens, each token's workgroup looks through all ids instead, and the first of an id adds up its rows.
// Every sum has a fixed order.
#include "internal.h"
#include "row_io.h"

namespace reqat {

namespace {

constexpr int kPiece = kEmbedPiece;
constexpr int kFewTokens = 512;

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

// ------------------------------------------------------------------ a fresh table

// Zeros; the ids' rows are written again by the sums.  One store a thread, workgroup after workgroup: 152064 x 5120 FP32 in
// 454 us, 6.9 TB/s.  Longer runs a workgroup write slower (4 stores a thread 517 us, 16 557 us, a persistent grid of 2048
// workgroups 670 us): more places are open at once.  A table without gaps goes as one row.
template <typename G> __global__ __launch_bounds__(256) void embed_zero_kernel(G *table, int64_t ld, int64_t cols) {
    constexpr int N = kVec<G>;
    G *row = table + (int64_t)blockIdx.y * ld;
    const int64_t j = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N;
    if (j + N <= cols) store_vec(row + j, make_uint4(0, 0, 0, 0));
    else
        for (int64_t k = j; k < cols; ++k) row[k] = G(0);
}

template <typename G> hipError_t launch_zero(const EmbedGradArgs &a, hipStream_t stream) {
    const bool dense = a.ld_table == a.D;
    const int64_t rows = dense ? 1 : a.V, cols = dense ? a.V * a.D : a.D, step = 256 * kVec<G>;
    constexpr int64_t kMostX = 1 << 23, kMostY = 65535;      // a launch's threads stay below 2^32
    for (int64_t r = 0; r < rows; r += kMostY)
        for (int64_t c = 0; c < cols; c += kMostX * step) {
            const int64_t ny = rows - r < kMostY ? rows - r : kMostY;
            const int64_t left = cols - c < kMostX * step ? cols - c : kMostX * step;
            hipLaunchKernelGGL(embed_zero_kernel<G>, dim3((unsigned)((left + step - 1) / step), (unsigned)ny), dim3(256), 0, stream,
                               reinterpret_cast<G *>(a.dtable) + r * a.ld_table + c, a.ld_table, left);
        }
    return hipGetLastError();
}

// ------------------------------------------------------------------ tokens by id

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kAhead = 8;

// The ids of tokens t, t + 64, ..., asked for together; padding behind the end.
__device__ __forceinline__ void load_ids(const int32_t *__restrict__ ids, int64_t t, int64_t end, int32_t (&out)[kAhead]) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) out[u] = t + u * 64 < end ? ids[t + u * 64] : -1;
}

// Workgroup g owns the ids [g R, g R + R).  Each reads all ids twice (the caches hold them): it counts the tokens of lower
// ids, which is where its own begin, and its own by wave and id; then every wave goes through its part of the tokens
// again, in order, and puts each into its place.  No workgroup waits for another.
//   places [T]: token, id, first place of the id and its number of tokens;  *valid: the places that hold a token.
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const int32_t *__restrict__ ids, int64_t T, int32_t V, int R,
                                                                  int32_t *__restrict__ valid, int4 *__restrict__ places) {
    extern __shared__ int32_t count[];                  // [kSortWaves][R], first place [R], number [R]
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
    for (int64_t t0 = begin; t0 < end; t0 += 64 * kAhead) {
        int32_t some[kAhead];
        load_ids(ids, t0 + lane, end, some);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int32_t id = some[u];
            if (id >= 0 && id < lo) ++below;
            const uint32_t k = (uint32_t)id - (uint32_t)lo;                 // out of range for padding too
            if (k < width) atomicAdd(&mine[k], 1);      // a count: the order of the additions does not show
        }
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
    int32_t *first = count + kSortWaves * R, *number = first + R;
    if (threadIdx.x < width && lo + (int32_t)threadIdx.x == V - 1) *valid = place + total;
    if ((int)threadIdx.x < R) {
        first[threadIdx.x] = place;
        number[threadIdx.x] = total;
        for (int w = 0; w < kSortWaves; ++w) {
            const int32_t n = count[w * R + threadIdx.x];
            count[w * R + threadIdx.x] = place;
            place += n;
        }
    }
    __syncthreads();
    const int bits = 32 - __builtin_clz((uint32_t)R | 1u);
    for (int64_t t0 = begin; t0 < end; t0 += 64 * kAhead) {
        int32_t some[kAhead];
        load_ids(ids, t0 + lane, end, some);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t k = (uint32_t)some[u] - (uint32_t)lo;
            const bool own = k < width;
            uint64_t same = __ballot(own);              // after the loop: the lanes of the same id
            if (!same) continue;
            for (int b = 0; b < bits; ++b) {
                const uint64_t set = __ballot(own && ((k >> b) & 1u));
                same &= (k >> b) & 1u ? set : ~set;
            }
            if (own) {
                volatile int32_t *at = &mine[k];        // the wave's own counter
                const int32_t base = *at;
                const int before = __builtin_popcountll(same & ((1ull << lane) - 1));
                __builtin_amdgcn_wave_barrier();        // all have read before the first of an id moves it on
                if (before == 0) *at = base + __builtin_popcountll(same);
                places[base + before] = make_int4((int32_t)(t0 + u * 64 + lane), some[u], first[k], number[k]);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// ------------------------------------------------------------------ sums of rows

// Elements that a lane takes at a time: 16 bytes of the table, or of dy where a bfloat16 table has FP32 gradients.
template <typename T, typename G> constexpr int kTake = sizeof(T) == 2 && sizeof(G) == 2 ? 8 : 4;

// E elements from p on, m of them exist.
template <typename T, int E> __device__ __forceinline__ void load_some(const T *p, int m, T (&e)[E]) {
    if (m >= E) {
        __builtin_memcpy(e, p, sizeof(e));
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) e[i] = i < m ? p[i] : T(0);
    }
}

template <typename T, int E> __device__ __forceinline__ void store_some(T *p, int m, const T (&e)[E]) {
    if (m >= E) {
        __builtin_memcpy(p, e, sizeof(e));
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < m) p[i] = e[i];
    }
}

template <typename G> __device__ __forceinline__ G *table_at(const EmbedGradArgs &a, int32_t id, int j) {
    return reinterpret_cast<G *>(a.dtable) + (int64_t)id * a.ld_table + j;
}

// dtable[id][j ..] = RN([old +] scale acc), E elements, m of them exist.
template <typename G, int E>
__device__ __forceinline__ void put_row(const EmbedGradArgs &a, int32_t id, int j, int m, const G (&old)[E], const float (&acc)[E]) {
    G e[E];
#pragma unroll
    for (int i = 0; i < E; ++i) e[i] = from_f32<G>((a.accumulate ? to_f32(old[i]) : 0.0f) + a.scale * acc[i]);
    if (m > 0) store_some(table_at<G>(a, id, j), m, e);
}

// A wave per piece f and 64 E columns.  Sums of runs that began before the piece go into row 2 f of the workspace, of a run
// that goes on behind it and began here into row 2 f + 1.
template <typename T, typename G> __global__ __launch_bounds__(256) void embed_sum_kernel(EmbedGradArgs a, uint32_t tiles) {
    constexpr int E = kTake<T, G>, U = 8;
    static_assert(kPiece % U == 0 && kPiece <= 64, "whole turns, a lane to a place");
    const int lane = threadIdx.x & 63;
    const int64_t wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    const int64_t f = wave / tiles, p0 = f * kPiece;
    const int left = (int)(a.T - p0 < kPiece ? a.T - p0 : kPiece);
    if (left <= 0) return;
    const int4 place = a.places[p0 + (lane < left ? lane : 0)];      // not a place of this call from *valid on
    const int32_t valid = *a.valid;
    const int count = __builtin_amdgcn_readfirstlane((int)(valid - p0 < left ? valid - p0 : left));
    const int j = ((int)(wave % tiles) * 64 + lane) * E, D = (int)a.D, m = D - j;
    const T *dy = reinterpret_cast<const T *>(a.dy) + j;
    const bool ends = p0 + lane + 1 - place.z == place.w;           // whether the place is its id's last
    const uint64_t end_mask = __ballot(ends);
    float acc[E] = {};
    const auto part = [&](int64_t row) {
        float *out = a.partials + row * D + j;
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < m) out[i] = acc[i];
    };
#pragma unroll 1
    for (int k0 = 0; k0 < count; k0 += U) {
        T e[U][E] = {};
        G old[U][E] = {};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u;
            if (k < count && m > 0) {
                load_some(dy + (int64_t)__builtin_amdgcn_readlane(place.x, k) * a.ld_dy, m, e[u]);
                if (a.accumulate && (end_mask >> k & 1)) load_some(table_at<G>(a, __builtin_amdgcn_readlane(place.y, k), j), m, old[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u;
            if (k >= count) break;
#pragma unroll
            for (int i = 0; i < E; ++i) acc[i] += to_f32(e[u][i]);
            if (end_mask >> k & 1) {
                if (__builtin_amdgcn_readlane(place.z, k) >= p0) put_row<G, E>(a, __builtin_amdgcn_readlane(place.y, k), j, m, old[u], acc);
                else part(2 * f);
#pragma unroll
                for (int i = 0; i < E; ++i) acc[i] = 0.0f;
            }
        }
    }
    if (count > 0 && !(end_mask >> (count - 1) & 1)) part(2 * f + (__builtin_amdgcn_readlane(place.z, count - 1) >= p0));
}

// Workgroup f: the run that begins in piece f and goes on behind it, if there is one: its sums there and in the next pieces.
template <typename G> __global__ __launch_bounds__(256) void embed_join_kernel(EmbedGradArgs a) {
    const int64_t f = blockIdx.x, p = (f + 1) * kPiece - 1;
    if (p >= a.T) return;
    const int4 place = a.places[p];
    if (p >= *a.valid || place.z < f * kPiece || p + 1 - place.z == place.w) return;
    const int64_t j = (int64_t)blockIdx.y * 1024 + threadIdx.x * 4;
    const int m = (int)(a.D - j);
    if (m <= 0) return;
    float acc[4] = {};
    G old[4] = {};
    if (a.accumulate) load_some(table_at<G>(a, place.y, (int)j), m, old);
    const int pieces = (int)((place.z + place.w - 1) / kPiece - f) + 1;
    for (int k = 0; k < pieces; k += 8) {
        float z[8][4] = {};
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (k + u < pieces) load_some(a.partials + (2 * (f + k + u) + (k + u == 0)) * a.D + j, m, z[u]);
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += z[u][e];
    }
    put_row<G, 4>(a, place.y, (int)j, m, old, acc);
}

// ------------------------------------------------------------------ few tokens

// Workgroup p: if token p is the first of its id, the sum of all its rows, in order.
template <typename T, typename G> __global__ __launch_bounds__(256) void embed_few_kernel(EmbedGradArgs a, const int32_t *__restrict__ ids) {
    constexpr int E = kTake<T, G>, kChunks = kFewTokens / 64;
    const int p = blockIdx.x, lane = threadIdx.x & 63, count = (int)a.T;
    int32_t all[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) all[c] = c * 64 + lane < count ? ids[c * 64 + lane] : -1;
    const int32_t id = ids[p];
    if (id < 0 || id >= a.V) return;
    __shared__ int32_t list[kFewTokens];
    int n = 0;
    uint64_t earlier = 0;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const uint64_t same = __ballot(all[c] == id);
        if (p >= c * 64) earlier |= p - c * 64 >= 64 ? same : same & ((1ull << (p - c * 64)) - 1);
        // every wave writes the same list
        if ((same >> lane) & 1) list[n + __builtin_popcountll(same & ((1ull << lane) - 1))] = c * 64 + lane;
        n += __builtin_popcountll(same);
    }
    if (earlier) return;
    __syncthreads();
    const int j = ((int)blockIdx.y * 256 + (int)threadIdx.x) * E, m = (int)a.D - j;
    if (m <= 0) return;
    const T *dy = reinterpret_cast<const T *>(a.dy) + j;
    G old[E] = {};
    if (a.accumulate) load_some(table_at<G>(a, id, j), m, old);
    float acc[E] = {};
    for (int k = 0; k < n; k += 8) {
        T e[8][E] = {};
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (k + u < n) load_some(dy + (int64_t)list[k + u] * a.ld_dy, m, e[u]);
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (k + u < n) acc[i] += to_f32(e[u][i]);
    }
    put_row<G, E>(a, id, j, m, old, acc);
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

template <typename T, typename G> hipError_t launch_backward(const EmbedGradArgs &a, const int32_t *ids, hipStream_t stream) {
    hipError_t e = hipSuccess;
    if (!a.accumulate && (e = launch_zero<G>(a, stream)) != hipSuccess) return e;
    constexpr int kFewTile = 256 * kTake<T, G>, kTile = 64 * kTake<T, G>;
    if (a.T <= kFewTokens) {
        if (a.T > 0) hipLaunchKernelGGL((embed_few_kernel<T, G>), dim3((unsigned)a.T, (unsigned)((a.D + kFewTile - 1) / kFewTile)), dim3(256), 0, stream, a, ids);
        return hipGetLastError();
    }
    // ids a workgroup sorts: at most 768 (54 KB of LDS), and some 256 workgroups where that allows it
    int R = (int)((a.V + 255) / 256);
    R = R > 768 ? 768 : R;
    hipLaunchKernelGGL(embed_sort_kernel, dim3((unsigned)((a.V + R - 1) / R)), dim3(kSortThreads), (size_t)((kSortWaves + 2) * R * 4), stream,
                       ids, a.T, (int32_t)a.V, R, a.valid, a.places);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const unsigned tiles = (unsigned)((a.D + kTile - 1) / kTile);
    const int64_t waves = (a.T + kPiece - 1) / kPiece * tiles;
    hipLaunchKernelGGL((embed_sum_kernel<T, G>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, stream, a, tiles);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(embed_join_kernel<G>, dim3((unsigned)((a.T + kPiece - 1) / kPiece), (unsigned)((a.D + 1023) / 1024)), dim3(256),
                       0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding_backward(const EmbedGradArgs &a, const int32_t *ids, bool bf16, bool table_bf16, hipStream_t stream) {
    if (a.V == 0 || a.D == 0 || (a.T == 0 && a.accumulate)) return hipSuccess;
    if (bf16) return table_bf16 ? launch_backward<uint16_t, uint16_t>(a, ids, stream) : launch_backward<uint16_t, float>(a, ids, stream);
    return table_bf16 ? launch_backward<float, uint16_t>(a, ids, stream) : launch_backward<float, float>(a, ids, stream);
}

// [number of places, 16 bytes | places, 16 T bytes | the pieces' sums, FP32]
size_t embedding_workspace_bytes(int64_t T, int64_t V, int64_t D) {
    (void)V;
    return T > kFewTokens ? 16 + (size_t)T * 16 + (size_t)(2 * ((T + kPiece - 1) / kPiece)) * (size_t)D * 4 : 0;
}

}  // namespace reqat
