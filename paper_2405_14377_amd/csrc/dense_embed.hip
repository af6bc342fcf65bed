// Dense embedding table T [V, E] with a scale:
//   forward   Y[t, :]  = scale * T[ids[t], :]
//   backward  dT[v, :] = scale * sum over { t : ids[t] = v, v != pad } dY[t, :]
// The forward copies rows: it is bound by the HBM bytes of its rows.  The
// backward groups the tokens by id first (no floating-point atomics: every
// row is summed in token order in fp32 and rounded once), then writes every
// row of dT, the rows without tokens as zeros.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "internal.h"
#include "rowops.h"

namespace comera {
namespace {

constexpr int kRowsPerBlock = 8;       // forward: rows of one workgroup

// One workgroup copies kRowsPerBlock rows: items of VEC columns, row by row,
// over its 256 threads.  chunks = ceil(E / VEC); the last item of a row is
// moved back to end at the row's end (its first entries are written twice
// with the same values), so E >= VEC.
template <class TT, class TY, int VEC>
__global__ __launch_bounds__(256) void dense_rows_kernel(const int64_t *ids, int64_t n, const TT *T, int64_t V,
                                                         int64_t E, int64_t chunks, float scale, TY *Y,
                                                         int32_t *err_flag) {
    for (int64_t row0 = int64_t(blockIdx.x) * kRowsPerBlock; row0 < n; row0 += int64_t(gridDim.x) * kRowsPerBlock) {
        const int rows = int(min(int64_t(kRowsPerBlock), n - row0));
        for (int r = 0; r < rows; ++r) {
            const int64_t id = ids[row0 + r];
            const bool in = id >= 0 && id < V;
            if (!in && err_flag && threadIdx.x == 0) *err_flag = 1;
            const TT *src = T + (in ? id : 0) * E;
            TY *dst = Y + (row0 + r) * E;
            for (int64_t i = threadIdx.x; i < chunks; i += 256) {
                const int64_t c = min(i * VEC, E - VEC);
                float v[VEC];
                if (in) {
                    Pack<TT, VEC> p;
                    p.load(src + c);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[e] = scale * p.get(e);
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[e] = 0.f;
                }
                Pack<TY, VEC>::store(dst + c, v);
            }
        }
    }
}

// ---------------------------------------------------------------- tokens by id
constexpr int kGroupWaves = 8;
constexpr int kGroupThreads = 64 * kGroupWaves;
constexpr int kGroupQ = 1024;          // most ids of one workgroup: 32 KiB of counters
constexpr int kGroupUnroll = 4;        // ids in flight per lane

// Groups the tokens by id in one launch, in token order within an id.
// Workgroup g owns the ids with id mod G = g (G a power of two), so that
// frequent ids, which are often neighbours, fall to different workgroups.
// Every workgroup reads all n ids (they stay in the L2): wave w takes a
// contiguous part of the tokens and counts the owned ids in its own LDS
// counters, and the tokens of lower workgroups, which end where this one's
// begin.  A prefix sum over (id, wave) turns the counters into places, and a
// second walk in the same order writes each owned token to its place; tokens
// of one id in one step of 64 are ranked by their lanes.  Bound by the reads
// of the ids: 2 x 8 n bytes by each of 256 CUs.
__global__ __launch_bounds__(kGroupThreads) void dense_group_kernel(const int64_t *ids, int64_t n, int64_t V, int lg,
                                                                    int Q, int64_t pad, uint32_t *perm,
                                                                    uint32_t *start, uint32_t *count,
                                                                    int32_t *err_flag) {
    extern __shared__ uint32_t cnt[];                  // [kGroupWaves][Q]
    __shared__ uint32_t wsum[kGroupWaves], wbelow[kGroupWaves];
    const int t = threadIdx.x, w = t >> 6, lane = t & 63;
    const uint32_t g = blockIdx.x, mask = (1u << lg) - 1;
    for (int i = t; i < kGroupWaves * Q; i += kGroupThreads) cnt[i] = 0;
    __syncthreads();
    constexpr int kStep = 64 * kGroupUnroll;
    const int64_t seg = ((n + kGroupWaves - 1) / kGroupWaves + kStep - 1) / kStep * kStep;
    const int64_t s0 = w * seg, s1 = min(n, s0 + seg);
    uint32_t below = 0;
    bool bad = false;
    for (int64_t b = s0; b < s1; b += kStep) {
        int64_t id[kGroupUnroll];
#pragma unroll
        for (int u = 0; u < kGroupUnroll; ++u) {
            const int64_t at = b + u * 64 + lane;
            id[u] = at < s1 ? ids[at] : pad;
        }
#pragma unroll
        for (int u = 0; u < kGroupUnroll; ++u) {
            const bool in = id[u] >= 0 && id[u] < V;
            const bool here = b + u * 64 + lane < s1;
            bad = bad || (here && !in);
            if (here && in && id[u] != pad) {
                const uint32_t k = uint32_t(id[u]) & mask;
                if (k < g) ++below;
                if (k == g) atomicAdd(&cnt[w * Q + int(uint32_t(id[u]) >> lg)], 1u);
            }
        }
    }
    if (g == 0 && bad && err_flag) *err_flag = 1;
    for (int o = 32; o; o >>= 1) below += __shfl_xor(below, o);
    if (lane == 0) wbelow[w] = below;
    __syncthreads();
    // thread t owns kPer consecutive ids; their totals are summed up over the
    // workgroup
    constexpr int kPer = kGroupQ / kGroupThreads;
    uint32_t tot[kPer], mine = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int q = t * kPer + i;
        tot[i] = 0;
        if (q < Q)
            for (int x = 0; x < kGroupWaves; ++x) tot[i] += cnt[x * Q + q];
        mine += tot[i];
    }
    uint32_t upto = mine;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(upto, o);
        if (lane >= o) upto += y;
    }
    if (lane == 63) wsum[w] = upto;
    __syncthreads();
    uint32_t base = upto - mine;
    for (int x = 0; x < kGroupWaves; ++x) {
        base += wbelow[x];
        if (x < w) base += wsum[x];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int q = t * kPer + i;
        const int64_t id = (int64_t(q) << lg) + g;
        if (q < Q && id < V) {
            start[id] = base;
            count[id] = tot[i];
        }
        if (q < Q)
            for (int x = 0; x < kGroupWaves; ++x) {
                const uint32_t c = cnt[x * Q + q];
                cnt[x * Q + q] = base;
                base += c;
            }
    }
    __syncthreads();
    volatile uint32_t *place = cnt + w * Q;            // this wave's places
    for (int64_t b = s0; b < s1; b += kStep) {
        int64_t id[kGroupUnroll];
#pragma unroll
        for (int u = 0; u < kGroupUnroll; ++u) {
            const int64_t at = b + u * 64 + lane;
            id[u] = at < s1 ? ids[at] : pad;
        }
#pragma unroll
        for (int u = 0; u < kGroupUnroll; ++u) {
            const bool own = b + u * 64 + lane < s1 && id[u] >= 0 && id[u] < V && id[u] != pad &&
                             (uint32_t(id[u]) & mask) == g;
            const uint32_t q = uint32_t(id[u]) >> lg;
            uint64_t left = __ballot(own);
            while (left) {                             // once per distinct owned id among the 64
                const int leader = __ffsll((unsigned long long)left) - 1;
                const uint32_t ql = uint32_t(__builtin_amdgcn_readlane(int(q), leader));
                const uint64_t same = __ballot(own && q == ql);
                const uint32_t first = place[ql];
                if (own && q == ql) {
                    const uint32_t rank = uint32_t(__popcll(same & ((uint64_t(1) << lane) - 1)));
                    perm[first + rank] = uint32_t(b + u * 64 + lane);
                    if (lane == leader) place[ql] = first + uint32_t(__popcll(same));
                }
                left &= ~same;
            }
        }
    }
}

// dT rows: workgroup rows of ids blockIdx.x, + gridDim.x, ...; columns over
// the threads, tokens of an id in order.
template <class TY, class TT, int VEC>
__global__ __launch_bounds__(256) void dense_sum_kernel(const TY *dY, int64_t V, int64_t E, int64_t chunks,
                                                        float scale, const uint32_t *perm, const uint32_t *start,
                                                        const uint32_t *count, TT *dT) {
    for (int64_t id = blockIdx.x; id < V; id += gridDim.x) {
        const uint32_t s = start[id], m = count[id];
        for (int64_t i = threadIdx.x; i < chunks; i += 256) {
            const int64_t c = min(i * VEC, E - VEC);
            float v[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = 0.f;
            for (uint32_t k = 0; k < m; ++k) {
                Pack<TY, VEC> p;
                p.load(dY + int64_t(perm[s + k]) * E + c);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[e] += p.get(e);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] *= scale;
            Pack<TT, VEC>::store(dT + id * E + c, v);
        }
    }
}

// ---------------------------------------------------------------- host side
size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

struct DenseLayout_ {
    size_t perm, start, count, total;
    int lg, Q;          // ids mod 2^lg per workgroup, ids of one workgroup
};

bool dense_ok(const comera_dense_embed_shape *s) {
    return s && s->V >= 1 && s->E >= 1 && (s->table == COMERA_F32 || s->table == COMERA_BF16) &&
           (s->act == COMERA_F32 || s->act == COMERA_BF16);
}

// rows and widths below 2^31: ids and tokens are kept in 32 bits, a row's
// items in int; offsets into T, Y and dT are 64 bits
bool dense_supported(const comera_dense_embed_shape *s) { return s->V < 2147483647 && s->E < 2147483647; }

void dense_layout(const comera_dense_embed_shape *s, int64_t n, DenseLayout_ &L) {
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t o = off;
        off = align_up(off + bytes);
        return o;
    };
    // 256 workgroups, more where one would own more ids than its LDS counts
    L.lg = 8;
    while (((s->V - 1) >> L.lg) >= kGroupQ) ++L.lg;
    L.Q = int((s->V - 1) >> L.lg) + 1;
    L.perm = take(4 * size_t(std::max<int64_t>(n, 1)));
    L.start = take(4 * size_t(s->V));
    L.count = take(4 * size_t(s->V));
    L.total = off;
}

comera_status dense_status() { return note_hip(launch_status(), "dense embedding") ? COMERA_ERR_HIP : COMERA_OK; }

template <class TT, class TY>
void launch_rows(const comera_dense_embed_shape *s, const int64_t *ids, int64_t n, const void *T, float scale, void *Y,
                 int32_t *err_flag, hipStream_t st) {
    const unsigned grid = unsigned(std::min<int64_t>((n + kRowsPerBlock - 1) / kRowsPerBlock, 1 << 16));
    if (s->E >= 8)
        COMERA_LAUNCH((dense_rows_kernel<TT, TY, 8>), dim3(grid), dim3(256), 0, st, ids, n,
                      static_cast<const TT *>(T), s->V, s->E, (s->E + 7) / 8, scale, static_cast<TY *>(Y), err_flag);
    else
        COMERA_LAUNCH((dense_rows_kernel<TT, TY, 1>), dim3(grid), dim3(256), 0, st, ids, n,
                      static_cast<const TT *>(T), s->V, s->E, s->E, scale, static_cast<TY *>(Y), err_flag);
}

template <class TY, class TT>
void launch_sum(const comera_dense_embed_shape *s, const void *dY, float scale, const uint32_t *perm,
                const uint32_t *start, const uint32_t *count, void *dT, hipStream_t st) {
    const unsigned grid = unsigned(std::min<int64_t>(s->V, 1 << 16));
    if (s->E >= 4)
        COMERA_LAUNCH((dense_sum_kernel<TY, TT, 4>), dim3(grid), dim3(256), 0, st, static_cast<const TY *>(dY), s->V,
                      s->E, (s->E + 3) / 4, scale, perm, start, count, static_cast<TT *>(dT));
    else
        COMERA_LAUNCH((dense_sum_kernel<TY, TT, 1>), dim3(grid), dim3(256), 0, st, static_cast<const TY *>(dY), s->V,
                      s->E, s->E, scale, perm, start, count, static_cast<TT *>(dT));
}

}  // namespace
}  // namespace comera

using namespace comera;

extern "C" {

size_t comera_dense_embed_workspace_bytes(const comera_dense_embed_shape *s, int64_t n_tokens) {
    if (!dense_ok(s) || !dense_supported(s) || n_tokens < 0 || n_tokens >= 2147483647) return 0;
    DenseLayout_ L;
    dense_layout(s, n_tokens, L);
    return L.total;
}

comera_status comera_dense_embed_forward(const comera_dense_embed_shape *s, const int64_t *ids, int64_t n_tokens,
                                         const void *T, float scale, void *Y, int32_t *err_flag, void *stream) {
    if (!dense_ok(s) || n_tokens < 0 || n_tokens >= 2147483647 || !std::isfinite(scale)) return COMERA_ERR_INVALID_ARG;
    if (!dense_supported(s)) return COMERA_ERR_UNSUPPORTED;
    if (n_tokens == 0) return COMERA_OK;
    if (!ids || !T || !Y) return COMERA_ERR_INVALID_ARG;
    hipStream_t st = hipStream_t(stream);
    if (s->table == COMERA_F32 && s->act == COMERA_F32)
        launch_rows<float, float>(s, ids, n_tokens, T, scale, Y, err_flag, st);
    else if (s->table == COMERA_F32)
        launch_rows<float, bf16>(s, ids, n_tokens, T, scale, Y, err_flag, st);
    else if (s->act == COMERA_F32)
        launch_rows<bf16, float>(s, ids, n_tokens, T, scale, Y, err_flag, st);
    else
        launch_rows<bf16, bf16>(s, ids, n_tokens, T, scale, Y, err_flag, st);
    return dense_status();
}

comera_status comera_dense_embed_backward(const comera_dense_embed_shape *s, const int64_t *ids, int64_t n_tokens,
                                          const void *dY, float scale, int64_t pad_id, void *dT, void *ws,
                                          size_t ws_bytes, int32_t *err_flag, void *stream) {
    if (!dense_ok(s) || n_tokens < 0 || n_tokens >= 2147483647 || !std::isfinite(scale) || pad_id < -1 ||
        pad_id >= s->V)
        return COMERA_ERR_INVALID_ARG;
    if (!dense_supported(s)) return COMERA_ERR_UNSUPPORTED;
    if (!dT || (n_tokens > 0 && (!ids || !dY))) return COMERA_ERR_INVALID_ARG;
    DenseLayout_ L;
    dense_layout(s, n_tokens, L);
    if (!ws || ws_bytes < L.total || reinterpret_cast<uintptr_t>(ws) % 8) return COMERA_ERR_WORKSPACE;
    char *base = static_cast<char *>(ws);
    uint32_t *perm = reinterpret_cast<uint32_t *>(base + L.perm);
    uint32_t *start = reinterpret_cast<uint32_t *>(base + L.start);
    uint32_t *count = reinterpret_cast<uint32_t *>(base + L.count);
    hipStream_t st = hipStream_t(stream);
    const unsigned groups = unsigned(std::min<int64_t>(int64_t(1) << L.lg, s->V));
    COMERA_LAUNCH(dense_group_kernel, dim3(groups), dim3(kGroupThreads), size_t(4) * kGroupWaves * L.Q, st, ids,
                  n_tokens, s->V, L.lg, L.Q, pad_id, perm, start, count, err_flag);
    if (s->table == COMERA_F32 && s->act == COMERA_F32)
        launch_sum<float, float>(s, dY, scale, perm, start, count, dT, st);
    else if (s->table == COMERA_F32)
        launch_sum<bf16, float>(s, dY, scale, perm, start, count, dT, st);
    else if (s->act == COMERA_F32)
        launch_sum<float, bf16>(s, dY, scale, perm, start, count, dT, st);
    else
        launch_sum<bf16, bf16>(s, dY, scale, perm, start, count, dT, st);
    return dense_status();
}

}  // extern "C"
