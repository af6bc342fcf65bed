// Dense embedding table T [V, E] with a scale:
//   forward   Y[t, :]  = scale * T[ids[t], :]
//   backward  dT[v, :] = scale * sum over { t : ids[t] = v, v != pad } dY[t, :]
// The forward copies rows: it is bound by the HBM bytes of its rows.  The
// backward groups the tokens by id first (no floating-point atomics: every
// row is summed in fp32 in a fixed order and rounded once: token by token, or
// where an id has many tokens in partial sums over runs of them that are added
// in order), then writes every row of dT, the rows without tokens as zeros.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "internal.h"
#include "rowops.h"

namespace comera {
namespace {

constexpr int kRowsVec = 8;            // columns of a lane

// LPR lanes copy a row, LPR x VEC columns at a time.  The last lane with
// columns is moved back to end at the row's end (its first entries are
// written twice with the same values), so E >= VEC.  Bound by HBM: 65536
// uniform ids of a 50000 x 1536 fp32 table to bf16 94 us, 5.4 TB/s (two or
// four rows a wave, whose loads are in flight together: 95 and 96 us).
template <class TT, class TY, int VEC, int LPR>
__global__ __launch_bounds__(256) void dense_rows_kernel(const int64_t *ids, int64_t n, const TT *T, int64_t V,
                                                         int64_t E, float scale, TY *Y, int32_t *err_flag) {
    // one row a wave: its number and its id are uniform
    const int r = LPR == 64 ? __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6) : int(threadIdx.x) / LPR;
    const int lane = threadIdx.x % LPR;
    constexpr int kRows = 256 / LPR;
    for (int64_t row = int64_t(blockIdx.x) * kRows + r; row < n; row += int64_t(gridDim.x) * kRows) {
        const int64_t id = ids[row];
        const bool in = uint64_t(id) < uint64_t(V);
        if (!in && err_flag && lane == 0) *err_flag = 1;
        const TT *src = T + (in ? id : 0) * E;
        for (int64_t c0 = lane * VEC; c0 < E; c0 += LPR * VEC) {
            const int64_t c = min(c0, E - VEC);
            Pack<TT, VEC> p;
            p.load(src + c);
            float v[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = in ? scale * p.get(e) : 0.f;
            Pack<TY, VEC>::store(Y + row * E + c, v);
        }
    }
}

// ---------------------------------------------------------------- tokens by id
constexpr int kGroupWaves = 16;
constexpr int kGroupThreads = 64 * kGroupWaves;
constexpr int kGroupBits = 9;
constexpr int kGroupQ = 1 << kGroupBits;   // most ids of one workgroup: 32 KiB of counters
constexpr int kGroupUnroll = 8;        // ids in flight per lane
constexpr int kGroupList = 192;        // owned tokens that a wave keeps: 24 KiB
constexpr int kGroupStep = 64 * kGroupUnroll;

struct GroupArgs {
    const int64_t *ids;
    int64_t n, V;
    uint32_t pad;       // 2^32 - 1: none
    int lg, Q;
    int parts;          // the tokens are walked in so many parts, by workgroups of their own
    uint32_t few;       // an id with more tokens goes to the list of long ones
    uint4 *order;       // (token, id, first place and tokens of the id) by id
    uint2 *range;       // (first place, tokens) of each id
    uint4 *many;        // [workgroup][most_many] its long ids, (id, first place, tokens, 0)
    int most_many;
    uint32_t *n_many;   // [workgroup] how many
    uint32_t *total;    // tokens with an id
    uint32_t *count;    // [part][workgroup][Q] tokens of each id (more than one part)
    uint32_t *sum;      // [part][workgroup] tokens
    int32_t *err_flag;
};

constexpr uint32_t kNoId = 0xffffffffu;

// one step of a wave's walk over its tokens: kGroupUnroll ids a lane (b is
// uniform; behind the last token the last id is read again)
__device__ __forceinline__ void load_ids(const GroupArgs &a, int64_t b, uint32_t lane, int64_t (&id)[kGroupUnroll]) {
    if (b + kGroupStep <= a.n) {
        const int64_t *p = a.ids + b;
#pragma unroll
        for (int u = 0; u < kGroupUnroll; ++u) id[u] = p[u * 64 + lane];
    } else {
#pragma unroll
        for (int u = 0; u < kGroupUnroll; ++u) id[u] = a.ids[min(b + u * 64 + lane, a.n - 1)];
    }
}

// the id, or kNoId for padding and ids out of range
__device__ __forceinline__ uint32_t good_id(const GroupArgs &a, int64_t id) {
    const uint32_t x = uint64_t(id) < uint64_t(a.V) ? uint32_t(id) : kNoId;
    return x == a.pad ? kNoId : x;
}

// set bits of m below this lane
__device__ __forceinline__ uint32_t bits_below(uint64_t m) {
    return __builtin_amdgcn_mbcnt_hi(uint32_t(m >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(m), 0));
}

// the tokens of a wave, of part p
struct Segment {
    int64_t s0, s1;
    __device__ __forceinline__ Segment(const GroupArgs &a, int p, int w) {
        const int64_t waves = int64_t(kGroupWaves) * a.parts;
        const int64_t len = ((a.n + waves - 1) / waves + kGroupStep - 1) / kGroupStep * kGroupStep;
        s0 = min(a.n, (int64_t(p) * kGroupWaves + w) * len);
        s1 = min(a.n, s0 + len);
    }
};

// Walks the tokens [s0, s1) of a wave; take(own, m, token, id) is called for
// every 64 tokens of which some lanes (m) hold ids of workgroup g.  Returns
// the number of tokens of the workgroups before it.
template <class Take>
__device__ __forceinline__ uint32_t walk(const GroupArgs &a, int64_t s0, int64_t s1, uint32_t lane, uint32_t g,
                                         Take take) {
    const uint32_t mask = (1u << a.lg) - 1;
    uint32_t below = 0;
    int64_t next[kGroupUnroll];
    if (s0 < s1) load_ids(a, s0, lane, next);
    for (int64_t b = s0; b < s1; b += kGroupStep) {
        uint32_t id[kGroupUnroll];
#pragma unroll
        for (int u = 0; u < kGroupUnroll; ++u) id[u] = good_id(a, next[u]);
        if (b + kGroupStep > a.n) {
#pragma unroll
            for (int u = 0; u < kGroupUnroll; ++u)
                if (b + u * 64 + lane >= a.n) id[u] = kNoId;
        }
        if (b + kGroupStep < s1) load_ids(a, b + kGroupStep, lane, next);
#pragma unroll
        for (int u = 0; u < kGroupUnroll; ++u) {
            const uint32_t k = id[u] & mask;           // kNoId: the last workgroup's, and below none
            below += uint32_t(__popcll(__ballot(k < g)));
            if (__ballot(k == g)) {
                const bool own = k == g && id[u] != kNoId;
                take(own, __ballot(own), uint32_t(b + u * 64 + lane), id[u]);
            }
        }
    }
    return below;
}

// What the lanes of a wave hand each other through LDS without a barrier, by
// an LDS address: volatile accesses by a generic one stay flat instructions.
typedef volatile __attribute__((address_space(3))) uint32_t LdsWord;
typedef volatile __attribute__((address_space(3))) uint64_t LdsPair;

// Puts 64 owned tokens (those lanes with `own`) to their places: lanes of one
// id are ranked by their lane number, their first lane moves the id's place
// on.  Every id bit halves the set of lanes that agree with this one.
__device__ __forceinline__ void put_tokens(const GroupArgs &a, LdsWord *place, const uint2 *ids, bool own,
                                           uint64_t token_id, uint32_t lane) {
    const uint32_t q = uint32_t(token_id) >> a.lg;
    uint64_t same = __ballot(own);
#pragma unroll
    for (int b = 0; b < kGroupBits; ++b) {
        const uint64_t m = __ballot((q >> b) & 1);
        same &= (q >> b) & 1 ? m : ~m;
    }
    if (own) {
        const uint32_t rank = bits_below(same);
        const uint32_t first = place[q];
        a.order[first + rank] = make_uint4(uint32_t(token_id >> 32), uint32_t(token_id), ids[q].x, ids[q].y);
        if (rank == 0) place[q] = first + uint32_t(__popcll(same));
    }
}

// the first `n` tokens of a wave's list
__device__ __forceinline__ void put_list(const GroupArgs &a, LdsWord *place, const uint2 *ids,
                                         const LdsPair *list, uint32_t n, uint32_t lane) {
    for (uint32_t i = 0; i < n; i += 64) {
        const bool own = i + lane < n;
        put_tokens(a, place, ids, own, own ? list[i + lane] : 0, lane);
    }
}

// Tokens of each id in each part, for dense_group_kernel.
__global__ __launch_bounds__(kGroupThreads) void dense_count_kernel(GroupArgs a) {
    __shared__ uint32_t cnt[kGroupQ], all;
    const int t = threadIdx.x, w = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t g = blockIdx.x, p = blockIdx.y;
    if (t < a.Q) cnt[t] = 0;
    if (t == 0) all = 0;
    __syncthreads();
    const Segment seg(a, int(p), w);
    uint32_t mine = 0;
    walk(a, seg.s0, seg.s1, t & 63, g, [&](bool own, uint64_t m, uint32_t, uint32_t id) {
        if (own) atomicAdd(&cnt[id >> a.lg], 1u);
        mine += uint32_t(__popcll(m));
    });
    if ((t & 63) == 0) atomicAdd(&all, mine);
    __syncthreads();
    const int64_t at = int64_t(p) * gridDim.x + g;
    if (t < a.Q) a.count[at * a.Q + t] = cnt[t];
    if (t == 0) a.sum[at] = all;
}

// Groups the tokens by id, in token order within an id.  Workgroup (g, p)
// owns the ids with id mod G = g (G a power of two), so that frequent ids,
// which are often neighbours, fall to different workgroups, in part p of the
// tokens.  Wave w takes a contiguous share of the part, counts the owned ids
// in its own LDS counters and lists the owned tokens.  A prefix sum over (id,
// wave) turns the counters into places, and the lists, in the order of the
// walk, go to them; a wave that owns more tokens than its list holds (an id
// that is a good part of the batch) walks its share again, list by list.
// Where the workgroup's places begin: with one part it counts the tokens of
// lower workgroups on the walk, which needs no other launch; with more parts
// it adds up what dense_count_kernel counted.  Every id is read by G
// workgroups, from the L2; bound by the instructions of the walk, about 10
// per 64 ids and wave, and by its chain of waits: 9.1 us for 16384 ids of 256
// workgroups.
__global__ __launch_bounds__(kGroupThreads) void dense_group_kernel(GroupArgs a) {
    extern __shared__ uint32_t cnt[];                  // [kGroupWaves][Q]
    __shared__ uint32_t wsum[kGroupWaves], wbelow[kGroupWaves], longs;
    __shared__ uint64_t lists[kGroupWaves][kGroupList];            // token << 32 | id
    __shared__ uint2 ids[kGroupQ];                     // first place and tokens of the workgroup's ids
    const int t = threadIdx.x, w = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, Q = a.Q;
    const uint32_t groups = gridDim.x, g = blockIdx.x, p = blockIdx.y, all = groups * a.parts;
    for (int i = t; i < kGroupWaves * Q; i += kGroupThreads) cnt[i] = 0;
    if (t == 0) longs = 0;
    __syncthreads();
    const Segment seg(a, int(p), w);
    LdsPair *list = (LdsPair *)lists[w];
    uint32_t listed = 0;
    auto append = [&](bool own, uint64_t m, uint32_t token, uint32_t id) {
        const uint32_t i = listed + bits_below(m);
        if (own && i < kGroupList) list[i] = uint64_t(token) << 32 | id;
        listed += uint32_t(__popcll(m));
    };
    uint32_t below = walk(a, seg.s0, seg.s1, lane, g, [&](bool own, uint64_t m, uint32_t token, uint32_t id) {
        if (own) atomicAdd(&cnt[w * Q + int(id >> a.lg)], 1u);
        append(own, m, token, id);
    });
    // this thread's id in all parts and in the parts before this one
    uint32_t whole = 0, before = 0;
    if (a.parts > 1) {
        if (t < Q)
#pragma unroll 8
            for (int x = 0; x < a.parts; ++x) {
                const uint32_t c = a.count[(int64_t(x) * groups + g) * Q + t];
                whole += c;
                before += x < int(p) ? c : 0;
            }
        below = 0;                                     // tokens of lower workgroups, all parts
        for (uint32_t i = t; i < all; i += kGroupThreads) below += i % groups < g ? a.sum[i] : 0;
        for (int o = 32; o; o >>= 1) below += __shfl_xor(below, o);
    }
    if (lane == 0) wbelow[w] = below;
    __syncthreads();
    // thread q < Q owns one id: its total, and those of the ids before it
    if (a.parts == 1 && t < Q)
        for (int x = 0; x < kGroupWaves; ++x) whole += cnt[x * Q + t];
    uint32_t base = whole;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(base, o);
        if (lane >= o) base += y;
    }
    if (lane == 63) wsum[w] = base;
    __syncthreads();
    base -= whole;
    for (int x = 0; x < kGroupWaves; ++x) {
        base += wbelow[x];
        if (x < w) base += wsum[x];
    }
    if (t < Q) {
        ids[t] = make_uint2(base, whole);
        if (p == 0) {
            const int64_t id = (int64_t(t) << a.lg) + g;
            if (id < a.V) a.range[id] = make_uint2(base, whole);
            if (whole > a.few)                         // in any order
                a.many[int64_t(g) * a.most_many + atomicAdd(&longs, 1u)] = make_uint4(uint32_t(id), base, whole, 0);
        }
        uint32_t at = base + before;
        for (int x = 0; x < kGroupWaves; ++x) {
            const uint32_t c = cnt[x * Q + t];
            cnt[x * Q + t] = at;
            at += c;
        }
    }
    // all tokens with an id end behind the last id of the last workgroup
    if (g == groups - 1 && p == 0 && t == kGroupThreads - 1) *a.total = base + whole;
    __syncthreads();
    if (t == 0 && p == 0) a.n_many[g] = longs;
    LdsWord *place = (LdsWord *)(cnt + w * Q);            // this wave's places
    if (listed > kGroupList) {
        listed = 0;
        walk(a, seg.s0, seg.s1, lane, g, [&](bool own, uint64_t m, uint32_t token, uint32_t id) {
            append(own, m, token, id);
            if (listed > kGroupList - 64) {
                put_list(a, place, ids, list, listed, lane);
                listed = 0;
            }
        });
    }
    put_list(a, place, ids, list, listed, lane);
    // ids out of range: every workgroup looks at its share of the tokens
    if (a.err_flag)
        for (int64_t at = int64_t(p * groups + g) * kGroupThreads + t; at < a.n; at += int64_t(all) * kGroupThreads)
            if (uint64_t(a.ids[at]) >= uint64_t(a.V)) *a.err_flag = 1;
}

// ---------------------------------------------------------------- sums by id
constexpr int kSumVec = 4;             // columns of a lane
constexpr int kSumLoads = 16;          // rows in flight per wave
constexpr int kFillIds = 64;           // ids of one workgroup that writes zeros

struct SumArgs {
    const void *dY;
    int64_t n, V, E;
    int64_t jobs;       // chunks times slices
    int slices;         // column slices of a row: 64 lanes x VEC columns
    int lgC;            // log2 of the places of one chunk
    uint32_t few;       // tokens of an id that one wave adds alone
    float scale;
    const uint4 *order;
    const uint2 *range;
    const uint4 *many;
    const uint32_t *n_many, *total;
    int most_many;
    float *first, *last;
    void *dT;
    uint32_t sum_blocks;               // of the grid's workgroups, the ones that add
};

// One wave adds, in order, one column slice of the rows of the ids that begin
// in C consecutive places of the order.  An id of at most `few` tokens is
// added to its end, also behind the chunk's end (which 64 lanes, one place
// each, reach); an id of more tokens is cut at the chunks' ends and leaves
// fp32 unscaled partials, last[chunk] where it begins and first[chunk] where
// it goes on, for dense_finish_kernel.  Chunks of equal length keep every
// wave busy alike however the ids are distributed.
template <class TY, class TT, int VEC>
__device__ __forceinline__ void sum_chunk(const SumArgs &a, int64_t chunk, int slice, const uint4 &me, uint32_t nv) {
    const int lane = threadIdx.x & 63, C = 1 << a.lgC;
    const int64_t E = a.E, p0 = chunk << a.lgC, c0 = int64_t(slice) * (64 * VEC) + lane * VEC;
    const bool on = c0 < E;
    const int64_t c = on ? min(c0, E - VEC) : 0;
    const bool here = p0 + lane < nv;
    const uint2 rg = here ? make_uint2(me.z, me.w) : make_uint2(0, 0);
    const uint32_t pos = uint32_t(p0) + lane;
    const bool few = rg.y <= a.few;
    const bool mine = here && (few ? rg.x >= uint32_t(p0) && rg.x < uint32_t(p0) + C : lane < C);
    const uint64_t todo = __ballot(mine);
    if (!todo) return;
    const int k1 = 64 - __clzll((long long)todo);
    int k0 = __ffsll((unsigned long long)todo) - 1;    // the places of one run of lanes
    const bool ends = pos + 1 == rg.x + rg.y;
    const uint64_t cut = __ballot(mine && (ends || (!few && lane == C - 1)));
    const uint64_t whole = __ballot(few);
    const uint64_t begun = __ballot(rg.x >= uint32_t(p0));         // the id begins in this chunk
    const TY *dY = static_cast<const TY *>(a.dY);
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
    for (; k0 < k1; k0 += kSumLoads) {
        Pack<TY, VEC> x[kSumLoads];
#pragma unroll
        for (int k = 0; k < kSumLoads; ++k) {
            // places behind the last one read its row again
            const uint32_t tok = uint32_t(__builtin_amdgcn_readlane(int(me.x), min(k0 + k, k1 - 1)));
            x[k].load(dY + int64_t(tok) * E + c);
        }
#pragma unroll
        for (int k = 0; k < kSumLoads; ++k) {
            if (k0 + k < k1) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] += x[k].get(e);
                if ((cut >> (k0 + k)) & 1) {
                    if (on) {
                        if ((whole >> (k0 + k)) & 1) {
                            const uint32_t id = uint32_t(__builtin_amdgcn_readlane(int(me.y), k0 + k));
                            float v[VEC];
#pragma unroll
                            for (int e = 0; e < VEC; ++e) v[e] = a.scale * acc[e];
                            Pack<TT, VEC>::store(static_cast<TT *>(a.dT) + int64_t(id) * E + c, v);
                        } else {
                            float *to = (begun >> (k0 + k)) & 1 ? a.last : a.first;
                            Pack<float, VEC>::store(to + chunk * E + c, acc);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
                }
            }
        }
    }
}

// Sums of ids and, in workgroups of their own behind the adding ones, zeros
// for the ids without tokens.
template <class TY, class TT, int VEC>
__global__ __launch_bounds__(256) void dense_sum_kernel(SumArgs a) {
    const int w = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), lane = threadIdx.x & 63;
    if (blockIdx.x < a.sum_blocks) {
        const uint32_t nv = *a.total;
        for (int64_t job = int64_t(blockIdx.x) * 4 + w; job < a.jobs; job += int64_t(a.sum_blocks) * 4) {
            const int64_t chunk = job / a.slices;
            // places behind the grouped tokens hold anything and are not used
            const uint4 me = a.order[min((chunk << a.lgC) + lane, a.n - 1)];
            if ((chunk << a.lgC) < nv) sum_chunk<TY, TT, VEC>(a, chunk, int(job - chunk * a.slices), me, nv);
        }
        return;
    }
    constexpr int kPer = kFillIds / 4;
    TT *dT = static_cast<TT *>(a.dT);
    for (int64_t id0 = int64_t(blockIdx.x - a.sum_blocks) * kFillIds + w * kPer; id0 < a.V;
         id0 += int64_t(gridDim.x - a.sum_blocks) * kFillIds) {
        const bool empty = lane < kPer && id0 + lane < a.V && a.range[id0 + lane].y == 0;
        for (uint64_t m = __ballot(empty); m; m &= m - 1) {
            TT *row = dT + (id0 + __ffsll((unsigned long long)m) - 1) * a.E;
            const float zero[VEC] = {};
            for (int64_t c0 = lane * VEC; c0 < a.E; c0 += 64 * VEC)
                Pack<TT, VEC>::store(row + min(c0, a.E - VEC), zero);
        }
    }
}

// ---------------------------------------------------------------- few tokens
constexpr int kFewTokens = 1024;       // one id a thread
constexpr int kFewQ = 64;              // most ids of one workgroup: a bit each
constexpr int kFewLoads = 16;          // rows in flight per wave

// All of a small batch's gradient in one launch.  Workgroup g owns the ids
// with id mod G = g: it lists its tokens in order, adds the rows of its ids
// that have any, a wave per id and column slice (or several, where tokens are
// many and pairs few), and writes zeros for the others, a wave per row.
// Bound by launch latency and the zeros: 300 uniform ids of 2000 x 640 bf16
// 7.7 us (three launches: 14.5), 1000 Zipf ids of 8000 x 768 10.9 us (17.7),
// 64 ids of 20000 x 768 10.7 us (19.5); 300 tokens of two ids 9.9 us (with a
// wave per pair 14.9).
template <class TY, class TT, int VEC>
__global__ __launch_bounds__(kFewTokens) void dense_few_kernel(GroupArgs a, SumArgs b) {
    constexpr int kWaves = kFewTokens / 64;
    __shared__ uint2 list[kFewTokens];                 // (token, id)
    __shared__ uint32_t wcount[kWaves];
    __shared__ unsigned long long present;
    __shared__ float red[kWaves][64 * VEC];
    const int t = threadIdx.x, w = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
    const uint32_t g = blockIdx.x, mask = (1u << a.lg) - 1;
    if (t == 0) present = 0;
    __syncthreads();
    uint32_t id = kNoId;
    if (t < a.n) {
        id = good_id(a, a.ids[t]);
        if (g == 0 && a.err_flag && uint64_t(a.ids[t]) >= uint64_t(a.V)) *a.err_flag = 1;
    }
    const bool own = id != kNoId && (id & mask) == g;
    const uint64_t m = __ballot(own);
    if (own) atomicOr(&present, 1ull << (id >> a.lg));
    if (lane == 0) wcount[w] = uint32_t(__popcll(m));
    __syncthreads();
    uint32_t at = 0, n = 0;
    for (int x = 0; x < kWaves; ++x) {
        if (x == w) at = n;
        n += wcount[x];
    }
    if (own) list[at + bits_below(m)] = make_uint2(uint32_t(t), id);
    __syncthreads();
    n = uint32_t(__builtin_amdgcn_readfirstlane(int(n)));
    const unsigned long long all = present;
    const int64_t E = b.E;
    const TY *dY = static_cast<const TY *>(b.dY);
    TT *dT = static_cast<TT *>(b.dT);
    // acc += the rows of id q's tokens at places [i, end) of the list
    auto add = [&](uint32_t q, uint32_t i, uint32_t end, int64_t c, float (&acc)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
        for (; i < end; i += 64) {
            const uint2 x = list[min(i + lane, end - 1)];
            uint64_t todo = __ballot(i + lane < end && (x.y >> a.lg) == q);
            while (todo) {
                Pack<TY, VEC> r[kFewLoads];
                int k1 = 0, bit = 0;
#pragma unroll
                for (int k = 0; k < kFewLoads; ++k) {
                    // behind the last token its row is read again
                    if (todo) {
                        bit = __ffsll((unsigned long long)todo) - 1;
                        todo &= todo - 1;
                        k1 = k + 1;
                    }
                    r[k].load(dY + int64_t(uint32_t(__builtin_amdgcn_readlane(int(x.x), bit))) * E + c);
                }
#pragma unroll
                for (int k = 0; k < kFewLoads; ++k)
                    if (k < k1)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) acc[e] += r[k].get(e);
            }
        }
    };
    auto store = [&](uint32_t q, int64_t c, float (&acc)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] *= b.scale;
        Pack<TT, VEC>::store(dT + ((int64_t(q) << a.lg) + g) * E + c, acc);
    };
    // ids with tokens first: their loads are on their way while zeros are written
    const int jobs = __builtin_amdgcn_readfirstlane(min(__popcll(all) * b.slices, kWaves));
    if (n <= 2 * kFewLoads || jobs > kWaves / 2) {
        int job = 0;
        for (unsigned long long p = all; p; p &= p - 1) {
            const uint32_t q = uint32_t(__ffsll(p)) - 1;
            for (int s = 0; s < b.slices; ++s, ++job) {
                if (job % kWaves != w) continue;
                const int64_t c0 = int64_t(s) * 64 * VEC + lane * VEC, c = c0 < E ? min(c0, E - VEC) : 0;
                float acc[VEC];
                add(q, 0, n, c, acc);
                if (c0 < E) store(q, c, acc);
            }
        }
    } else {
        // ids and slices for half of the waves at most: several waves a pair,
        // their sums added in order
        const int split = min(kWaves / jobs, int(n) / kFewLoads), mine = w / split, part = w % split;
        uint32_t q = 0;
        int64_t c0 = E;
        int job = 0;
        for (unsigned long long p = all; p; p &= p - 1, job += b.slices)
            if (mine >= job && mine < job + b.slices) {
                q = uint32_t(__ffsll(p)) - 1;
                c0 = int64_t(mine - job) * 64 * VEC + lane * VEC;
            }
        const int64_t c = c0 < E ? min(c0, E - VEC) : 0;
        float acc[VEC];
        if (mine < jobs) {
            add(q, n * part / split, n * (part + 1) / split, c, acc);
#pragma unroll
            for (int e = 0; e < VEC; ++e) red[w][lane * VEC + e] = acc[e];
        }
        __syncthreads();
        if (mine < jobs && part == 0 && c0 < E) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                for (int k = 1; k < split; ++k) acc[e] += red[w + k][lane * VEC + e];
            store(q, c, acc);
        }
    }
    for (int q = w; q < a.Q; q += kWaves) {
        const int64_t row = (int64_t(q) << a.lg) + g;
        if (row >= a.V || ((all >> q) & 1)) continue;
        const float zero[VEC] = {};
        for (int64_t c0 = lane * VEC; c0 < E; c0 += 64 * VEC)
            Pack<TT, VEC>::store(dT + row * E + min(c0, E - VEC), zero);
    }
}

constexpr int kFinishWaves = 8;

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

// Rows of the ids with many tokens: last[a] of the chunk where the id begins,
// then first[a + 1 .. z], a part of them by each wave of a workgroup, the
// waves' sums added in order.  Workgroup (g, y, z) takes every gridDim.z-th of
// the long ids that workgroup g of dense_group_kernel listed, column slices y,
// y + gridDim.y, ...
template <class TT, int VEC>
__global__ __launch_bounds__(64 * kFinishWaves) void dense_finish_kernel(SumArgs a, int groups) {
    __shared__ float red[kFinishWaves][64 * VEC];
    const int w = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), lane = threadIdx.x & 63;
    const int64_t E = a.E;
    for (int g = blockIdx.x; g < groups; g += gridDim.x) {
        const uint32_t n = a.n_many[g];
        for (uint32_t i = blockIdx.z; i < n; i += gridDim.z) {
            const uint4 r = a.many[int64_t(g) * a.most_many + i];
            const uint32_t id = r.x;
            const int64_t at = r.y >> a.lgC, more = ((r.y + r.z - 1) >> a.lgC) - at;
            for (int s = blockIdx.y; s < a.slices; s += gridDim.y) {
                const int64_t c0 = int64_t(s) * 64 * VEC + lane * VEC, c = c0 < E ? min(c0, E - VEC) : 0;
                float acc[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
                if (w == 0) add_rows<VEC>(a.last, at, at + 1, E, c, acc);
                add_rows<VEC>(a.first, at + 1 + more * w / kFinishWaves, at + 1 + more * (w + 1) / kFinishWaves, E, c,
                              acc);
#pragma unroll
                for (int e = 0; e < VEC; ++e) red[w][lane * VEC + e] = acc[e];
                __syncthreads();
                if (w == 0 && c0 < E) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        for (int k = 1; k < kFinishWaves; ++k) acc[e] += red[k][lane * VEC + e];
                        acc[e] *= a.scale;
                    }
                    Pack<TT, VEC>::store(static_cast<TT *>(a.dT) + int64_t(id) * E + c, acc);
                }
                __syncthreads();
            }
        }
    }
}

// ---------------------------------------------------------------- host side
// From here on one more launch costs less than the walk of all ids by every
// workgroup: 16384 Zipf ids 39.0 us in one part, 40.5 in two launches; 32768:
// 51.2 and 50.0; 131072: 132 and 92 (table of 32768 x 768)
constexpr int64_t kSplitTokens = 24576;
// From here on chunks of 32 places instead of 16: fewer partial rows, where
// there are waves enough.  16 and 32 places, a table of 32768 x 768: 16384
// uniform ids in fp32 44.2 and 47.0 us, in bf16 22.1 and 22.9 (Zipf ids 52.9
// and 53.4, 30.5 and 28.2); 65536 uniform 82.6 and 83.0, 52.1 and 51.6 (Zipf
// 99.9 and 93.6, 68.1 and 60.9); 131072 of a 5000 x 128 fp32 table 56.7 and
// 36.1.  Between 24576 and here 32 would be level or up to 9 % faster.
constexpr int64_t kLongChunks = 32768;

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

struct DenseLayout_ {
    size_t order, range, many, n_many, total, count, sum, first, last, bytes;
    int lg, Q, parts;   // ids mod 2^lg per workgroup, ids of one workgroup, parts of the tokens
    int lgC;            // log2 of the places of one chunk
    int few;            // tokens of an id that is never cut
    int most_many;      // most ids of one workgroup with more tokens
    int64_t chunks;
    bool few_tokens;    // all in one launch
    int64_t groups() const { return int64_t(1) << lg; }
};

bool dense_ok(const comera_dense_embed_shape *s) {
    return s && s->V >= 1 && s->E >= 1 && (s->table == COMERA_F32 || s->table == COMERA_BF16) &&
           (s->act == COMERA_F32 || s->act == COMERA_BF16);
}

// Ids and tokens are kept in 32 bits; offsets into T, Y and dT are 64 bits.
bool dense_supported(const comera_dense_embed_shape *s) { return s->V < 2147483647 && s->E < 2147483647; }
// 2^21 workgroups of 1024 threads group the tokens of 2^30 ids; twice as many
// would not fit a launch.
bool dense_backward_supported(const comera_dense_embed_shape *s) {
    return dense_supported(s) && s->V <= int64_t(kGroupQ) << 21;
}

// the longest batch that one launch does, where the table is not too long for it
int64_t most_few_tokens(const comera_dense_embed_shape *s) { return std::min<int64_t>(kFewTokens, 256 * s->V); }

void dense_layout(const comera_dense_embed_shape *s, int64_t n, DenseLayout_ &L) {
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t o = off;
        off = align_up(off + bytes);
        return o;
    };
    // 256 workgroups (more where one would own more ids than its LDS counts).
    // A long batch is cut into parts, each id read by fewer workgroups: as
    // few as own all ids, in as many parts as make 256 of them (32 at most);
    // so is a shorter one of a few ids, whose tokens few workgroups own: 16384
    // of 2 ids 41.3 -> 33.4 us, of 16 20.2 -> 22.7, 8192 of 2 26.2 -> 29.9.
    // A batch of one id a thread is done by one launch (with more tables rows
    // than 2^22 its workgroups would be too many), unless a few ids leave it
    // to a few CUs: 1000 tokens of 2 ids 20.2 us, 14.8 by the general way; 300
    // 10.2 and 14.1.
    L.few_tokens = n <= most_few_tokens(s) && s->V <= int64_t(kFewQ) << 16;
    L.lg = n < kSplitTokens ? 8 : 5;
    while (((s->V - 1) >> L.lg) >= (L.few_tokens ? kFewQ : kGroupQ)) ++L.lg;
    const bool split = n >= (s->V > 4 ? kSplitTokens : kSplitTokens / 2);
    L.parts = split ? int(std::min<int64_t>(32, std::max<int64_t>(1, 256 / std::min(L.groups(), s->V)))) : 1;
    L.Q = int((s->V - 1) >> L.lg) + 1;
    L.lgC = n < kLongChunks ? 4 : 5;
    // an id that begins at a chunk's last place ends within the 64 lanes
    L.few = std::min(64 - (1 << L.lgC), 1 << L.lgC);
    L.chunks = (n + (1 << L.lgC) - 1) >> L.lgC;
    L.order = take(16 * size_t(n));
    L.range = take(8 * size_t(s->V));
    L.most_many = int(std::min<int64_t>(L.Q, n / L.few + 1));
    L.many = take(16 * size_t(L.most_many) * size_t(L.groups()));
    L.n_many = take(4 * size_t(L.groups()));
    L.total = take(4);
    if (L.parts > 1) {
        L.count = take(4 * size_t(L.Q) * size_t(L.groups()) * size_t(L.parts));
        L.sum = take(4 * size_t(L.groups()) * size_t(L.parts));
    }
    L.first = take(sizeof(float) * size_t(L.chunks) * size_t(s->E));
    L.last = take(sizeof(float) * size_t(L.chunks) * size_t(s->E));
    L.bytes = off;
}

// The most that any batch of up to n tokens needs, so that the workspace of a
// program's longest batch serves its shorter ones.  What a batch needs grows
// with it except where dense_layout changes its form, which may halve it.
size_t dense_most_bytes(const comera_dense_embed_shape *s, int64_t n) {
    size_t most = 0;
    for (const int64_t last : {most_few_tokens(s), kSplitTokens / 2 - 1, kSplitTokens - 1, kLongChunks - 1, n}) {
        if (last > n) continue;
        DenseLayout_ L{};
        dense_layout(s, last, L);
        most = std::max(most, L.bytes);
    }
    return most;
}

comera_status dense_status() { return note_hip(launch_status(), "dense embedding") ? COMERA_ERR_HIP : COMERA_OK; }

template <class TT, class TY, int VEC, int LPR>
void launch_rows(const comera_dense_embed_shape *s, const int64_t *ids, int64_t n, const void *T, float scale, void *Y,
                 int32_t *err_flag, hipStream_t st) {
    constexpr int kRows = 256 / LPR;
    const dim3 grid(unsigned(std::min<int64_t>((n + kRows - 1) / kRows, 1 << 20)));
    COMERA_LAUNCH((dense_rows_kernel<TT, TY, VEC, LPR>), grid, dim3(256), 0, st, ids, n, static_cast<const TT *>(T),
                  s->V, s->E, scale, static_cast<TY *>(Y), err_flag);
}

// Narrow rows share a wave: 65536 ids of 50000 x 64 7.2 us, 13.1 with a wave each
template <class TT, class TY>
void launch_rows(const comera_dense_embed_shape *s, const int64_t *ids, int64_t n, const void *T, float scale, void *Y,
                 int32_t *err_flag, hipStream_t st) {
    if (s->E < kRowsVec)
        launch_rows<TT, TY, 1, 8>(s, ids, n, T, scale, Y, err_flag, st);
    else if (s->E <= 16 * kRowsVec)
        launch_rows<TT, TY, kRowsVec, 16>(s, ids, n, T, scale, Y, err_flag, st);
    else if (s->E <= 32 * kRowsVec)
        launch_rows<TT, TY, kRowsVec, 32>(s, ids, n, T, scale, Y, err_flag, st);
    else
        launch_rows<TT, TY, kRowsVec, 64>(s, ids, n, T, scale, Y, err_flag, st);
}

template <class TY, class TT, int VEC>
void launch_sum(const GroupArgs &ga, SumArgs a, const DenseLayout_ &L, hipStream_t st) {
    a.slices = int((a.E + 64 * VEC - 1) / (64 * VEC));
    const int64_t groups = std::min(L.groups(), a.V);
    if (L.few_tokens) {
        COMERA_LAUNCH((dense_few_kernel<TY, TT, VEC>), dim3(unsigned(groups)), dim3(kFewTokens), 0, st, ga, a);
        return;
    }
    const dim3 grid(unsigned(groups), unsigned(L.parts));
    if (L.parts > 1) COMERA_LAUNCH(dense_count_kernel, grid, dim3(kGroupThreads), 0, st, ga);
    COMERA_LAUNCH(dense_group_kernel, grid, dim3(kGroupThreads), size_t(4) * kGroupWaves * L.Q, st, ga);
    // workgroups up to 2^20 of each kind; the kernels walk on from there
    constexpr int64_t kMost = 1 << 20;
    a.jobs = L.chunks * a.slices;
    a.sum_blocks = uint32_t(std::min(kMost, (a.jobs + 3) / 4));
    const uint32_t fill = uint32_t(std::min(kMost, (a.V + kFillIds - 1) / kFillIds));
    COMERA_LAUNCH((dense_sum_kernel<TY, TT, VEC>), dim3(a.sum_blocks + fill), dim3(256), 0, st, a);
    const auto finish = [&](auto kernel) {
        COMERA_LAUNCH(kernel, dim3(unsigned(std::min<int64_t>(groups, 1 << 16)), unsigned(std::min(a.slices, 16)),
                                   unsigned(std::max<int64_t>(1, 256 / groups))),
                      dim3(64 * kFinishWaves), 0, st, a, int(groups));
    };
    // a table of a few rows: narrower slices, more workgroups (131072 tokens
    // of one id 168 -> 113 us, of 16 ids 66 -> 60, with the parts above)
    if (a.V * a.slices >= 64) {
        finish(dense_finish_kernel<TT, VEC>);
    } else {
        a.slices = int((a.E + 63) / 64);
        finish(dense_finish_kernel<TT, 1>);
    }
}

template <class TY, class TT>
void launch_sum(const GroupArgs &ga, const SumArgs &a, const DenseLayout_ &L, hipStream_t st) {
    if (a.E >= kSumVec)
        launch_sum<TY, TT, kSumVec>(ga, a, L, st);
    else
        launch_sum<TY, TT, 1>(ga, a, L, st);
}

}  // namespace
}  // namespace comera

using namespace comera;

extern "C" {

size_t comera_dense_embed_workspace_bytes(const comera_dense_embed_shape *s, int64_t n_tokens) {
    if (!dense_ok(s) || !dense_backward_supported(s) || n_tokens < 0 || n_tokens >= 2147483647) return 0;
    return dense_most_bytes(s, n_tokens);
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
    if (!dense_backward_supported(s)) return COMERA_ERR_UNSUPPORTED;
    if (!dT || (n_tokens > 0 && (!ids || !dY))) return COMERA_ERR_INVALID_ARG;
    DenseLayout_ L{};
    dense_layout(s, n_tokens, L);
    if (!ws || ws_bytes < L.bytes || reinterpret_cast<uintptr_t>(ws) % 16) return COMERA_ERR_WORKSPACE;
    char *base = static_cast<char *>(ws);
    hipStream_t st = hipStream_t(stream);
    GroupArgs ga{};
    ga.ids = ids;
    ga.n = n_tokens;
    ga.V = s->V;
    ga.pad = pad_id < 0 ? kNoId : uint32_t(pad_id);
    ga.lg = L.lg;
    ga.Q = L.Q;
    ga.few = uint32_t(L.few);
    ga.order = reinterpret_cast<uint4 *>(base + L.order);
    ga.range = reinterpret_cast<uint2 *>(base + L.range);
    ga.many = reinterpret_cast<uint4 *>(base + L.many);
    ga.most_many = L.most_many;
    ga.n_many = reinterpret_cast<uint32_t *>(base + L.n_many);
    ga.total = reinterpret_cast<uint32_t *>(base + L.total);
    ga.parts = L.parts;
    ga.count = reinterpret_cast<uint32_t *>(base + L.count);
    ga.sum = reinterpret_cast<uint32_t *>(base + L.sum);
    ga.err_flag = err_flag;
    SumArgs a{};
    a.dY = dY;
    a.n = n_tokens;
    a.V = s->V;
    a.E = s->E;
    a.lgC = L.lgC;
    a.few = ga.few;
    a.scale = scale;
    a.order = ga.order;
    a.range = ga.range;
    a.many = ga.many;
    a.n_many = ga.n_many;
    a.total = ga.total;
    a.most_many = L.most_many;
    a.first = reinterpret_cast<float *>(base + L.first);
    a.last = reinterpret_cast<float *>(base + L.last);
    a.dT = dT;
    if (s->table == COMERA_F32 && s->act == COMERA_F32)
        launch_sum<float, float>(ga, a, L, st);
    else if (s->table == COMERA_F32)
        launch_sum<bf16, float>(ga, a, L, st);
    else if (s->act == COMERA_F32)
        launch_sum<float, bf16>(ga, a, L, st);
    else
        launch_sum<bf16, bf16>(ga, a, L, st);
    return dense_status();
}

}  // extern "C"
