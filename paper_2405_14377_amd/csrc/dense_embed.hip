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
constexpr int kGroupWaves = 16;
constexpr int kGroupThreads = 64 * kGroupWaves;
constexpr int kGroupBits = 9;
constexpr int kGroupQ = 1 << kGroupBits;   // most ids of one workgroup: 32 KiB of counters
constexpr int kGroupUnroll = 8;        // ids in flight per lane
constexpr int kGroupList = 160;        // owned tokens that a wave keeps: 20 KiB
constexpr int kGroupStep = 64 * kGroupUnroll;

struct GroupArgs {
    const int64_t *ids;
    int64_t n, V, pad;
    int lg, Q;
    uint2 *order;       // (token, id) by id
    uint2 *range;       // (first place, tokens) of each id
    uint32_t *total;    // tokens with an id
    int32_t *err_flag;
};

// one step of a wave's walk over its tokens: kGroupUnroll ids a lane
__device__ __forceinline__ void load_ids(const GroupArgs &a, int64_t b, int64_t s1, int lane,
                                         int64_t (&id)[kGroupUnroll]) {
#pragma unroll
    for (int u = 0; u < kGroupUnroll; ++u) {
        const int64_t at = b + u * 64 + lane;
        id[u] = a.ids[min(at, s1 - 1)];
    }
}

// Puts 64 owned tokens (those lanes with `own`) to their places: lanes of one
// id are ranked by their lane number, their first lane moves the id's place
// on.  Every id bit halves the set of lanes that agree with this one.
__device__ __forceinline__ void put_tokens(const GroupArgs &a, volatile uint32_t *place, bool own, uint32_t token,
                                           uint32_t q, uint32_t id, int lane) {
    uint64_t same = __ballot(own);
#pragma unroll
    for (int b = 0; b < kGroupBits; ++b) {
        const uint64_t m = __ballot((q >> b) & 1);
        same &= (q >> b) & 1 ? m : ~m;
    }
    if (own) {
        const uint32_t rank = uint32_t(__popcll(same & ((uint64_t(1) << lane) - 1)));
        const uint32_t first = place[q];
        a.order[first + rank] = make_uint2(token, id);
        if (rank == 0) place[q] = first + uint32_t(__popcll(same));
    }
}

// Groups the tokens by id in one launch, in token order within an id.
// Workgroup g owns the ids with id mod G = g (G a power of two), so that
// frequent ids, which are often neighbours, fall to different workgroups.
// Every workgroup reads all n ids (they stay in the L2): wave w takes a
// contiguous part of the tokens, counts the owned ids in its own LDS
// counters, lists the owned tokens, and counts the tokens of lower
// workgroups, which end where this one's begin.  A prefix sum over (id, wave)
// turns the counters into places, and the lists, in the order of the walk, go
// to them; a wave that owns more tokens than its list holds walks its part
// again.  Bound by the latency and the L2 reads of the ids, 8 n bytes by each
// of 256 CUs.
__global__ __launch_bounds__(kGroupThreads) void dense_group_kernel(GroupArgs a) {
    extern __shared__ uint32_t cnt[];                  // [kGroupWaves][Q]
    __shared__ uint32_t wsum[kGroupWaves], wbelow[kGroupWaves];
    __shared__ uint2 list[kGroupWaves][kGroupList];    // (token, id)
    const int t = threadIdx.x, w = t >> 6, lane = t & 63, Q = a.Q;
    const uint32_t g = blockIdx.x, mask = (1u << a.lg) - 1;
    for (int i = t; i < kGroupWaves * Q; i += kGroupThreads) cnt[i] = 0;
    __syncthreads();
    const int64_t seg = ((a.n + kGroupWaves - 1) / kGroupWaves + kGroupStep - 1) / kGroupStep * kGroupStep;
    const int64_t s0 = w * seg, s1 = min(a.n, s0 + seg);
    uint32_t below = 0, listed = 0;
    bool bad = false;
    for (int64_t b = s0; b < s1; b += kGroupStep) {
        int64_t id[kGroupUnroll];
        load_ids(a, b, s1, lane, id);
#pragma unroll
        for (int u = 0; u < kGroupUnroll; ++u) {
            const int64_t at = b + u * 64 + lane;
            const bool in = uint64_t(id[u]) < uint64_t(a.V);
            const bool here = at < s1;
            bad = bad || !in;                          // lanes behind the end repeat an id
            const uint32_t k = uint32_t(id[u]) & mask;
            const bool counts = here && in && id[u] != a.pad;
            below += counts && k < g ? 1 : 0;
            const bool own = counts && k == g;
            const uint64_t m = __ballot(own);
            if (m) {
                if (own) {
                    atomicAdd(&cnt[w * Q + int(uint32_t(id[u]) >> a.lg)], 1u);
                    const uint32_t i = listed + uint32_t(__popcll(m & ((uint64_t(1) << lane) - 1)));
                    if (i < kGroupList) list[w][i] = make_uint2(uint32_t(at), uint32_t(id[u]));
                }
                listed += uint32_t(__popcll(m));
            }
        }
    }
    if (g == 0 && bad && a.err_flag) *a.err_flag = 1;
    for (int o = 32; o; o >>= 1) below += __shfl_xor(below, o);
    if (lane == 0) wbelow[w] = below;
    __syncthreads();
    // thread q < Q owns one id: its total, and those of the ids before it
    uint32_t mine = 0;
    if (t < Q)
        for (int x = 0; x < kGroupWaves; ++x) mine += cnt[x * Q + t];
    uint32_t base = mine;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(base, o);
        if (lane >= o) base += y;
    }
    if (lane == 63) wsum[w] = base;
    __syncthreads();
    base -= mine;
    for (int x = 0; x < kGroupWaves; ++x) {
        base += wbelow[x];
        if (x < w) base += wsum[x];
    }
    if (t < Q) {
        const int64_t id = (int64_t(t) << a.lg) + g;
        if (id < a.V) a.range[id] = make_uint2(base, mine);
        for (int x = 0; x < kGroupWaves; ++x) {
            const uint32_t c = cnt[x * Q + t];
            cnt[x * Q + t] = base;
            base += c;
        }
    }
    // all tokens with an id end behind the last id of the last workgroup
    if (g == gridDim.x - 1 && t == kGroupThreads - 1) *a.total = base;
    __syncthreads();
    volatile uint32_t *place = cnt + w * Q;            // this wave's places
    if (listed <= kGroupList) {
        for (uint32_t i0 = 0; i0 < listed; i0 += 64) {
            const bool own = i0 + lane < listed;
            const uint2 x = list[w][own ? i0 + lane : 0];
            put_tokens(a, place, own, x.x, x.y >> a.lg, x.y, lane);
        }
        return;
    }
    for (int64_t b = s0; b < s1; b += kGroupStep) {
        int64_t id[kGroupUnroll];
        load_ids(a, b, s1, lane, id);
#pragma unroll 1
        for (int u = 0; u < kGroupUnroll; ++u) {
            int64_t x = id[0];
#pragma unroll
            for (int k = 1; k < kGroupUnroll; ++k) x = u == k ? id[k] : x;
            const int64_t at = b + u * 64 + lane;
            const uint32_t i = uint32_t(x);
            const bool own = at < s1 && uint64_t(x) < uint64_t(a.V) && x != a.pad && (i & mask) == g;
            if (__ballot(own)) put_tokens(a, place, own, uint32_t(at), i >> a.lg, i, lane);
        }
    }
}

// ---------------------------------------------------------------- sums by id
// Column slice of a wave: 64 lanes x VEC columns.  The last lane with columns
// is moved back to end at the row's end, as in the forward.
constexpr int kSumVec = 4;
constexpr int kSumLoads = 16;          // rows in flight per wave

// One wave adds the rows of C consecutive places of the order, one column
// slice of them, in order.  An id whose places all lie in the chunk gets its
// row of dT; what an id has here that goes on in the next chunk goes to
// last[chunk], what came from the chunk before (and perhaps goes on) to
// first[chunk], fp32 and unscaled, for dense_finish_kernel.  Chunks of equal
// length keep every wave busy alike however the ids are distributed.
template <class TY, class TT, int VEC>
__device__ __forceinline__ void sum_chunk(const TY *dY, int64_t E, int64_t chunk, int slice, int C, uint32_t nv,
                                          float scale, const uint2 *order, TT *dT, float *first, float *last) {
    const int lane = threadIdx.x & 63;
    const int64_t p0 = chunk * C;
    const int cnt = int(min(int64_t(C), int64_t(nv) - p0));
    // entry p0 - 1 + lane: the chunk's places and one on either side
    uint2 me = make_uint2(0, 0xffffffffu);             // an id that no place has
    const int64_t at = p0 - 1 + lane;
    if (at >= 0 && at < nv && lane <= C + 1) me = order[at];
    const int64_t c0 = int64_t(slice) * (64 * VEC) + lane * VEC;
    const bool on = c0 < E;
    const int64_t c = on ? min(c0, E - VEC) : 0;
    const uint32_t next = __shfl_down(me.y, 1);
    const uint64_t ends = __ballot(lane >= 1 && lane <= cnt && me.y != next) >> 1;   // bit k: place k is its id's last
    const bool goes_in = __builtin_amdgcn_readlane(int(me.y), 0) == __builtin_amdgcn_readlane(int(me.y), 1);
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
    bool from_before = goes_in;
    for (int k0 = 0; k0 < cnt; k0 += kSumLoads) {
        Pack<TY, VEC> x[kSumLoads];
#pragma unroll
        for (int k = 0; k < kSumLoads; ++k) {
            // places behind the chunk's end read its last row again
            const uint32_t tok = uint32_t(__builtin_amdgcn_readlane(int(me.x), 1 + min(k0 + k, cnt - 1)));
            x[k].load(dY + int64_t(tok) * E + c);
        }
#pragma unroll
        for (int k = 0; k < kSumLoads; ++k) {
            if (k0 + k < cnt) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] += x[k].get(e);
                const bool end = (ends >> (k0 + k)) & 1;
                if (end || k0 + k == cnt - 1) {
                    if (on) {
                        if (end && !from_before) {
                            const uint32_t id = uint32_t(__builtin_amdgcn_readlane(int(me.y), 1 + k0 + k));
                            float v[VEC];
#pragma unroll
                            for (int e = 0; e < VEC; ++e) v[e] = scale * acc[e];
                            Pack<TT, VEC>::store(dT + int64_t(id) * E + c, v);
                        } else {
                            Pack<float, VEC>::store((from_before ? first : last) + chunk * E + c, acc);
                        }
                    }
                    from_before = false;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
                }
            }
        }
    }
}

template <class TY, class TT, int VEC>
__global__ __launch_bounds__(256) void dense_chunk_kernel(const TY *dY, int64_t E, int slices, int C, float scale,
                                                          const uint2 *order, const uint32_t *total, TT *dT,
                                                          float *first, float *last) {
    const uint32_t nv = *total;
    const int64_t jobs = (int64_t(nv) + C - 1) / C * slices;
    for (int64_t job = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6); job < jobs; job += int64_t(gridDim.x) * 4) {
        const int64_t chunk = job / slices;
        sum_chunk<TY, TT, VEC>(dY, E, chunk, int(job - chunk * slices), C, nv, scale, order, dT, first, last);
    }
}

constexpr int kFinishWaves = 8;
constexpr int kFinishIds = 32;         // ids of one workgroup
constexpr int kFinishAlone = 16;       // partial rows that one wave adds by itself
constexpr uint32_t kDone = 0xffffffffu, kNone = 0xfffffffeu;

// rows [i, end) of `part` added in order, eight loads in flight
template <int VEC>
__device__ __forceinline__ void add_rows(const float *part, int64_t i, int64_t end, int64_t E, int64_t c,
                                         float (&acc)[VEC]) {
    for (; i < end; i += 8) {
        Pack<float, VEC> x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k].load(part + min(i + k, end - 1) * E + c);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + k < end)
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] += x[k].get(e);
    }
}

// Rows of dT that dense_chunk_kernel left: zeros for ids without tokens, and
// the sum of the partials of ids that lie in several chunks (last[a], then
// first[a + 1 .. a + more]).  A workgroup takes kFinishIds ids, spread over
// the table (frequent ids are often neighbours).  blockIdx.y = 0: a wave per
// row, all columns; every blockIdx.y: all waves on each row that has many
// partials, its own column slices.
template <class TT, int VEC>
__global__ __launch_bounds__(64 * kFinishWaves) void dense_finish_kernel(int64_t V, int64_t E, int lgC, float scale,
                                                                         const uint2 *range, const float *first,
                                                                         const float *last, TT *dT) {
    __shared__ uint2 rows[kFinishIds];                 // (a, more), or kDone, kNone for more
    __shared__ uint32_t many_rows;
    __shared__ float red[kFinishWaves][64 * VEC];
    const int t = threadIdx.x, w = t >> 6, lane = t & 63;
    const int64_t stride = (V + kFinishIds - 1) / kFinishIds;      // groups of ids, and the distance of a group's ids
    constexpr int64_t kCols = 64 * VEC;
    for (int64_t group = blockIdx.x; group < stride; group += gridDim.x) {
        __syncthreads();                               // the last group's rows are no longer read
        if (w == 0) {
            uint2 x = make_uint2(0, kDone);
            const int64_t id = group + lane * stride;
            if (lane < kFinishIds && id < V) {
                const uint2 r = range[id];
                const uint32_t a = r.x >> lgC, z = (r.x + r.y - 1) >> lgC;
                x = make_uint2(a, r.y == 0 ? kNone : z == a ? kDone : z - a);
            }
            const uint64_t many = __ballot(x.y >= kFinishAlone && x.y < kNone);
            if (lane < kFinishIds) rows[lane] = x;
            if (lane == 0) many_rows = uint32_t(many);
        }
        __syncthreads();
        for (uint32_t m = many_rows; m; m &= m - 1) {  // the same rows in every wave
            const int r = __ffs(int(m)) - 1;
            const int64_t a = rows[r].x, more = rows[r].y;
            for (int64_t s = blockIdx.y; s * kCols < E; s += gridDim.y) {
                const int64_t c0 = s * kCols + lane * VEC, c = c0 < E ? min(c0, E - VEC) : 0;
                float acc[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
                if (w == 0) add_rows<VEC>(last, a, a + 1, E, c, acc);
                add_rows<VEC>(first, a + 1 + more * w / kFinishWaves, a + 1 + more * (w + 1) / kFinishWaves, E, c,
                              acc);
#pragma unroll
                for (int e = 0; e < VEC; ++e) red[w][lane * VEC + e] = acc[e];
                __syncthreads();
                if (w == 0 && c0 < E) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        for (int k = 1; k < kFinishWaves; ++k) acc[e] += red[k][lane * VEC + e];
                        acc[e] *= scale;
                    }
                    Pack<TT, VEC>::store(dT + (group + r * stride) * E + c, acc);
                }
                __syncthreads();
            }
        }
        if (blockIdx.y) continue;
        for (int r = w; r < kFinishIds; r += kFinishWaves) {
            const uint32_t a = uint32_t(__builtin_amdgcn_readfirstlane(int(rows[r].x)));
            const uint32_t more = uint32_t(__builtin_amdgcn_readfirstlane(int(rows[r].y)));
            if (more == kDone || (more >= kFinishAlone && more != kNone)) continue;
            TT *row = dT + (group + r * stride) * E;
            for (int64_t c0 = lane * VEC; c0 < E; c0 += kCols) {
                const int64_t c = min(c0, E - VEC);
                float acc[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
                if (more != kNone) {
                    add_rows<VEC>(last, a, int64_t(a) + 1, E, c, acc);
                    add_rows<VEC>(first, int64_t(a) + 1, int64_t(a) + 1 + more, E, c, acc);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[e] *= scale;
                }
                Pack<TT, VEC>::store(row + c, acc);
            }
        }
    }
}

// ---------------------------------------------------------------- host side
size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

struct DenseLayout_ {
    size_t order, range, total, first, last, bytes;
    int lg, Q;          // ids mod 2^lg per workgroup, ids of one workgroup
    int lgC;            // log2 of the places of one chunk
    int64_t chunks;
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
    // longer chunks leave fewer partial rows, shorter ones more waves
    L.lgC = n < 32768 ? 4 : 5;
    L.chunks = (n + (1 << L.lgC) - 1) >> L.lgC;
    L.order = take(8 * size_t(n));
    L.range = take(8 * size_t(s->V));
    L.total = take(4);
    L.first = take(sizeof(float) * size_t(L.chunks) * size_t(s->E));
    L.last = take(sizeof(float) * size_t(L.chunks) * size_t(s->E));
    L.bytes = off;
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

struct SumArgs {
    const void *dY;
    int64_t V, E;
    float scale;
    const uint2 *order, *range;
    const uint32_t *total;
    float *first, *last;
    void *dT;
};

template <class TY, class TT, int VEC>
void launch_sum(const SumArgs &a, const DenseLayout_ &L, hipStream_t st) {
    constexpr int64_t kMost = 1 << 20;                 // workgroups; the kernels walk on from there
    const int64_t slices = (a.E + 64 * VEC - 1) / (64 * VEC);
    if (L.chunks > 0)
        COMERA_LAUNCH((dense_chunk_kernel<TY, TT, VEC>), dim3(unsigned(std::min(kMost, (L.chunks * slices + 3) / 4))),
                      dim3(256), 0, st, static_cast<const TY *>(a.dY), a.E, int(slices), 1 << L.lgC, a.scale, a.order,
                      a.total, static_cast<TT *>(a.dT), a.first, a.last);
    COMERA_LAUNCH((dense_finish_kernel<TT, VEC>),
                  dim3(unsigned(std::min<int64_t>((a.V + kFinishIds - 1) / kFinishIds, 1 << 16)),
                       unsigned(std::min<int64_t>(slices, 16))),
                  dim3(64 * kFinishWaves), 0, st, a.V, a.E, L.lgC, a.scale, a.range, a.first, a.last,
                  static_cast<TT *>(a.dT));
}

template <class TY, class TT>
void launch_sum(const SumArgs &a, const DenseLayout_ &L, hipStream_t st) {
    if (a.E >= kSumVec)
        launch_sum<TY, TT, kSumVec>(a, L, st);
    else
        launch_sum<TY, TT, 1>(a, L, st);
}

}  // namespace
}  // namespace comera

using namespace comera;

extern "C" {

size_t comera_dense_embed_workspace_bytes(const comera_dense_embed_shape *s, int64_t n_tokens) {
    if (!dense_ok(s) || !dense_supported(s) || n_tokens < 0 || n_tokens >= 2147483647) return 0;
    DenseLayout_ L;
    dense_layout(s, n_tokens, L);
    return L.bytes;
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
    if (!ws || ws_bytes < L.bytes || reinterpret_cast<uintptr_t>(ws) % 8) return COMERA_ERR_WORKSPACE;
    char *base = static_cast<char *>(ws);
    hipStream_t st = hipStream_t(stream);
    SumArgs a{dY, s->V, s->E, scale, reinterpret_cast<uint2 *>(base + L.order),
              reinterpret_cast<uint2 *>(base + L.range), reinterpret_cast<uint32_t *>(base + L.total),
              reinterpret_cast<float *>(base + L.first), reinterpret_cast<float *>(base + L.last), dT};
    const unsigned groups = unsigned(std::min<int64_t>(int64_t(1) << L.lg, s->V));
    const GroupArgs ga{ids, n_tokens, s->V, pad_id, L.lg, L.Q, reinterpret_cast<uint2 *>(base + L.order),
                       reinterpret_cast<uint2 *>(base + L.range), reinterpret_cast<uint32_t *>(base + L.total),
                       err_flag};
    COMERA_LAUNCH(dense_group_kernel, dim3(groups), dim3(kGroupThreads), size_t(4) * kGroupWaves * L.Q, st, ga);
    if (s->table == COMERA_F32 && s->act == COMERA_F32)
        launch_sum<float, float>(a, L, st);
    else if (s->table == COMERA_F32)
        launch_sum<bf16, float>(a, L, st);
    else if (s->act == COMERA_F32)
        launch_sum<float, bf16>(a, L, st);
    else
        launch_sum<bf16, bf16>(a, L, st);
    return dense_status();
}

}  // extern "C"
