// Global norm of a step's gradients, and their clipping:
//   norm  = s * sqrt(sum_i sum_j g_i[j]^2)
//   out_i = s * min(1, max_norm / norm) * g_i
// Squares and their sum are taken in 64 bits: neither overflows or vanishes
// for any fp32 gradient, and the norm has the last digit of fp32 right
// whatever the number of entries.  A norm that is not finite leaves the
// clipping out (out_i = s g_i) and sets the flag.
//
// Two passes: grad_squares_kernel leaves one partial sum per workgroup, then
// every workgroup of grad_scale_kernel adds all the partials in the same
// fixed order (a few KiB from the L2), so no launch stands between them and
// the result is the same bits every time.  Bound by HBM: the gradients are
// read twice and written once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "internal.h"
#include "rowops.h"

namespace comera {
namespace {

constexpr int kChunkTensors = 120;     // tensors of one launch whose table is a kernel argument of under 4 KiB
constexpr int kTile = 8192;            // entries that a workgroup takes at a time
constexpr int kGradThreads = 256;
constexpr int kGradParts = 2048;       // workgroups of the first pass over all launches, up to twice as many
// Up to so many tiles one workgroup does both passes: 5 tiles 8.1 us a call
// (two launches: 9.6), 9 tiles 9.3 (9.6), 18 tiles 15.5 (9.6)
constexpr uint32_t kSmallTiles = 8;
constexpr int kSmallThreads = 1024;
constexpr int kScaleBlocks = 2048;     // workgroups of one launch of the second pass, at most
// From here on (bytes read and written) the clipped gradients are stored
// around the last-level cache: their lines would leave it only during the
// next pass, and throw out what that pass could still find there.  272 MB:
// both passes together 90.7 -> 76.5 us, with an update behind them that reads
// the results and a state of their size 155 -> 148.  One tensor, with such an
// update, ordinary and streamed: 128 MB 79.9 and 81.6, 160 MB 96.8 and 98.7,
// 192 MB 120 and 118, 224 MB 146 and 136.  Clipping in place, whose two
// accesses meet the same lines, is level either way from 24 to 250 MB of
// gradients (136 MB 65.2 and 65.2, with an update 161.0 and 162.0).
constexpr double kStreamBytes = 192.0 * 1048576;
constexpr int64_t kBf16 = int64_t(1) << 62;

struct Entry {
    const void *g;
    void *out;
    int64_t n;                         // entries, and kBf16
    uint32_t tile0, tile1;             // its tiles, among those of the launch
    __host__ __device__ __forceinline__ int64_t size() const { return n & ~kBf16; }
    __host__ __device__ __forceinline__ bool is_bf16() const { return n & kBf16; }
};

struct Work {
    int count;
    uint32_t tiles;
    uint32_t per;                      // tiles of a workgroup of the first pass
    int part0, parts;                  // this launch's partials
    int all_parts;
};

// a launch's tensors as a kernel argument, and in device memory
struct GradChunk : Work {
    Entry e[kChunkTensors];
    __device__ __forceinline__ Entry at(int i) const { return e[i]; }
    __device__ __forceinline__ uint32_t tile0(int i) const { return e[i].tile0; }
};
static_assert(sizeof(GradChunk) <= 3968, "the table is passed as a kernel argument");

struct GradTable : Work {
    const Entry *e;
    __device__ __forceinline__ Entry at(int i) const { return e[i]; }
    __device__ __forceinline__ uint32_t tile0(int i) const { return e[i].tile0; }
};

// Tensor that holds tile t (the last one that starts at or before it): the
// lanes compare 64 entries of the table at a time, so 64 tensors take one
// round trip, 4096 two.
template <class List>
__device__ __forceinline__ int tensor_of(const List &c, uint32_t t) {
    const int lane = threadIdx.x & 63;
    int lo = 0, len = c.count;
    while (len > 1) {
        const int step = (len + 63) / 64;
        const bool le = lane * step < len && c.tile0(lo + min(lane * step, len - 1)) <= t;
        const int k = __popcll(__ballot(le)) - 1;
        lo += k * step;
        len = min(step, len - k * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// entries of one launch's table to their place in the whole list's
__global__ __launch_bounds__(128) void grad_table_kernel(GradChunk c, Entry *table, uint32_t tile_base) {
    if (int(threadIdx.x) >= c.count) return;
    Entry x = c.at(threadIdx.x);
    x.tile0 += tile_base;
    x.tile1 += tile_base;
    table[threadIdx.x] = x;
}

// sum over a workgroup in a fixed order, in every thread
template <int THREADS = kGradThreads>
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double red[THREADS / 64];
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < THREADS / 64; ++w) v += red[w];
    return v;
}

// One tile: each thread's 16-byte pieces, all in flight at once.  use(p, i) is
// called for every whole piece at entry i, rest(j) for the entries behind the
// last one.
template <class T, class Use, class Rest>
__device__ __forceinline__ void for_tile(const T *g, int64_t at, int64_t n, Use use, Rest rest) {
    constexpr int V = 16 / sizeof(T), U = kTile / (V * kGradThreads);
    const int tid = threadIdx.x % kGradThreads;        // a small list's workgroup takes several tiles side by side
    const int64_t i0 = at + int64_t(tid) * V;
    if (at + kTile <= n) {
        Pack<T, V> p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) p[u].load(g + i0 + u * kGradThreads * V);
#pragma unroll
        for (int u = 0; u < U; ++u) use(p[u], i0 + u * kGradThreads * V);
        return;
    }
    // the last tile of a tensor: pieces behind its last whole one read that
    // one (or nothing) and are not used
    const int64_t whole = at + (n - at) / V * V;
    if (whole > at) {
        Pack<T, V> p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) p[u].load(g + min(i0 + u * kGradThreads * V, whole - V));
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * kGradThreads * V < whole) use(p[u], i0 + u * kGradThreads * V);
    }
    if (whole + tid < n) rest(whole + tid);
}

template <class T>
__device__ __forceinline__ double tile_squares(const T *g, int64_t at, int64_t n) {
    constexpr int V = 16 / sizeof(T);
    double s[2] = {0, 0};
    auto add = [&](float x, int k) { s[k & 1] += double(x) * double(x); };
    for_tile<T>(
        g, at, n,
        [&](const Pack<T, V> &p, int64_t) {
#pragma unroll
            for (int e = 0; e < V; ++e) add(p.get(e), e);
        },
        [&](int64_t j) {
            Pack<T, 1> p;
            p.load(g + j);
            add(p.get(0), 0);
        });
    return s[0] + s[1];
}

template <class List>
__global__ __launch_bounds__(kGradThreads) void grad_squares_kernel(List c, double *part) {
    const uint32_t t0 = blockIdx.x * c.per, t1 = min(t0 + c.per, c.tiles);
    double s = 0;
    int i = tensor_of(c, t0);
    Entry x = c.at(i);
    for (uint32_t t = t0; t < t1; ++t) {
        while (t >= x.tile1) x = c.at(++i);
        const int64_t at = int64_t(t - x.tile0) * kTile;
        s += x.is_bf16() ? tile_squares(static_cast<const bf16 *>(x.g), at, x.size())
                         : tile_squares(static_cast<const float *>(x.g), at, x.size());
    }
    s = block_sum(s);
    if (threadIdx.x == 0) part[c.part0 + blockIdx.x] = s;
}

// norm of all partials; every workgroup that calls it gets the same bits
__device__ __forceinline__ double total_norm(const double *part, int parts, float scale) {
    double s = 0;
    for (int i = threadIdx.x; i < parts; i += kGradThreads) s += part[i];
    return double(scale) * sqrt(block_sum(s));
}

__device__ __forceinline__ void write_norm(double norm, float *out, int32_t *flag) {
    const float f = float(norm);
    if (out) *out = f;
    if (flag && !isfinite(f)) *flag = 1;
}

__global__ __launch_bounds__(kGradThreads) void grad_norm_kernel(const double *part, int parts, float scale,
                                                                 float *norm, int32_t *flag) {
    const double v = total_norm(part, parts, scale);
    if (threadIdx.x == 0) write_norm(v, norm, flag);
}

template <class T, bool STREAM>
__device__ __forceinline__ void tile_scale(const T *g, T *out, int64_t at, int64_t n, float c) {
    constexpr int V = 16 / sizeof(T);
    for_tile<T>(
        g, at, n,
        [&](const Pack<T, V> &p, int64_t i) {
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = c * p.get(e);
            Pack<T, V>::template store<STREAM>(out + i, v);
        },
        [&](int64_t j) {
            Pack<T, 1> p;
            p.load(g + j);
            const float v[1] = {c * p.get(0)};
            Pack<T, 1>::store(out + j, v);
        });
}

// the factor of every entry
__device__ __forceinline__ float factor(double norm, float scale, float max_norm) {
    const bool clip = isfinite(float(norm)) && norm > double(max_norm);
    return clip ? float(double(scale) * (double(max_norm) / norm)) : scale;
}

template <class List, bool STREAM>
__global__ __launch_bounds__(kGradThreads) void grad_scale_kernel(List c, const double *part, float scale,
                                                                  float max_norm, float *norm, int32_t *flag) {
    const double v = total_norm(part, c.all_parts, scale);
    if (c.part0 == 0 && blockIdx.x == 0 && threadIdx.x == 0) write_norm(v, norm, flag);
    const float f = factor(v, scale, max_norm);
    // from the last tile back: what the first pass read last is still cached
    const uint32_t b = gridDim.x - 1 - blockIdx.x;
    const uint32_t t0 = uint32_t(uint64_t(c.tiles) * b / gridDim.x);
    const uint32_t t1 = uint32_t(uint64_t(c.tiles) * (b + 1) / gridDim.x);
    int i = tensor_of(c, t1 - 1);
    Entry x = c.at(i);
    for (uint32_t t = t1; t-- > t0;) {
        while (t < x.tile0) x = c.at(--i);
        if (f == 1.f && x.out == x.g) continue;
        const int64_t at = int64_t(t - x.tile0) * kTile;
        if (x.is_bf16())
            tile_scale<bf16, STREAM>(static_cast<const bf16 *>(x.g), static_cast<bf16 *>(x.out), at, x.size(), f);
        else
            tile_scale<float, STREAM>(static_cast<const float *>(x.g), static_cast<float *>(x.out), at, x.size(), f);
    }
}

// A small list's norm and clipping in one launch of one workgroup, four tiles
// side by side; the second pass reads from the L2.
__global__ __launch_bounds__(kSmallThreads) void grad_small_kernel(GradChunk c, float scale, float max_norm,
                                                                   float *norm, int32_t *flag) {
    constexpr uint32_t kSide = kSmallThreads / kGradThreads;
    const uint32_t t0 = uint32_t(__builtin_amdgcn_readfirstlane(int(threadIdx.x) / kGradThreads));
    double s = 0;
    for (uint32_t t = t0; t < c.tiles; t += kSide) {
        const Entry x = c.at(tensor_of(c, t));
        const int64_t at = int64_t(t - x.tile0) * kTile;
        s += x.is_bf16() ? tile_squares(static_cast<const bf16 *>(x.g), at, x.size())
                         : tile_squares(static_cast<const float *>(x.g), at, x.size());
    }
    const double v = double(scale) * sqrt(block_sum<kSmallThreads>(s));
    if (threadIdx.x == 0) write_norm(v, norm, flag);
    const float f = factor(v, scale, max_norm);
    for (uint32_t t = t0; t < c.tiles; t += kSide) {
        const Entry x = c.at(tensor_of(c, t));
        if (f == 1.f && x.out == x.g) continue;
        const int64_t at = int64_t(t - x.tile0) * kTile;
        if (x.is_bf16())
            tile_scale<bf16, false>(static_cast<const bf16 *>(x.g), static_cast<bf16 *>(x.out), at, x.size(), f);
        else
            tile_scale<float, false>(static_cast<const float *>(x.g), static_cast<float *>(x.out), at, x.size(), f);
    }
}

}  // namespace
}  // namespace comera

// the tensors' table, cut into launches (host memory), and all of it in the
// caller's device memory
struct comera_grad_plan_s {
    std::vector<comera::GradChunk> chunks;
    int64_t count = 0;
    int parts = 0;
    bool stream = false;                   // more bytes than the last-level cache holds
    comera::GradTable table{};             // e: null without one
    bool written = false;                  // not where launch check mode only recorded the table's launches
    bool has_table() const { return table.e && (written || comera::launch_check_mode()); }
};

using namespace comera;

namespace {

struct Range {
    uintptr_t begin, end;
};

comera_status grad_args(comera_grad_plan_t p, float scale, const void *ws, size_t ws_bytes) {
    if (!p || !std::isfinite(scale) || !(scale > 0.f)) return COMERA_ERR_INVALID_ARG;
    if (!ws || ws_bytes < comera_grad_workspace_bytes(p) || reinterpret_cast<uintptr_t>(ws) % 16)
        return COMERA_ERR_WORKSPACE;
    return COMERA_OK;
}

// the first pass; returns the number of partials
int launch_squares(comera_grad_plan_t p, double *part, hipStream_t st) {
    if (p->has_table()) {
        COMERA_LAUNCH((grad_squares_kernel<GradTable>), dim3(unsigned(p->table.parts)), dim3(kGradThreads), 0, st,
                      p->table, part);
        return p->table.parts;
    }
    for (const GradChunk &c : p->chunks)
        COMERA_LAUNCH((grad_squares_kernel<GradChunk>), dim3(unsigned(c.parts)), dim3(kGradThreads), 0, st, c, part);
    return p->parts;
}

template <class List>
void launch_scale(comera_grad_plan_t p, const List &c, const double *part, float scale, float max_norm,
                         float *norm, int32_t *flag, hipStream_t st) {
    const dim3 grid(std::min<unsigned>(c.tiles, kScaleBlocks));
    if (p->stream)
        COMERA_LAUNCH((grad_scale_kernel<List, true>), grid, dim3(kGradThreads), 0, st, c, part, scale, max_norm, norm,
                      flag);
    else
        COMERA_LAUNCH((grad_scale_kernel<List, false>), grid, dim3(kGradThreads), 0, st, c, part, scale, max_norm,
                      norm, flag);
}

}  // namespace

extern "C" {

comera_status comera_grad_plan(const comera_grad_tensor *tensors, int64_t count, comera_grad_plan_t *out) {
    if (!out) return COMERA_ERR_INVALID_ARG;
    *out = nullptr;
    if (count < 0 || (count > 0 && !tensors)) return COMERA_ERR_INVALID_ARG;
    try {
        std::vector<Range> ranges;
        std::vector<int64_t> order;
        double tiles = 0, bytes_in = 0;
        for (int64_t i = 0; i < count; ++i) {
            const comera_grad_tensor &t = tensors[i];
            if (t.n < 0 || (t.dtype != COMERA_F32 && t.dtype != COMERA_BF16)) return COMERA_ERR_INVALID_ARG;
            if (t.n == 0) continue;
            if (!t.g || t.n >= (int64_t(1) << 42)) return COMERA_ERR_INVALID_ARG;
            const uintptr_t esz = t.dtype == COMERA_F32 ? 4 : 2, bytes = uintptr_t(t.n) * esz;
            const uintptr_t g = reinterpret_cast<uintptr_t>(t.g), o = reinterpret_cast<uintptr_t>(t.out);
            if (g % esz || o % esz) return COMERA_ERR_INVALID_ARG;
            ranges.push_back({g, g + bytes});
            if (o && o != g) ranges.push_back({o, o + bytes});
            tiles += double((t.n + kTile - 1) / kTile);
            order.push_back(i);
            bytes_in += double(bytes);
        }
        // no buffer twice: an entry would count twice in the norm, or be
        // scaled by two workgroups at once
        std::sort(ranges.begin(), ranges.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
        for (size_t i = 1; i < ranges.size(); ++i)
            if (ranges[i].begin < ranges[i - 1].end) return COMERA_ERR_INVALID_ARG;
        if (tiles > 2147483647.0) return COMERA_ERR_UNSUPPORTED;
        comera_grad_plan_s *p = new comera_grad_plan_s;
        try {
            // the largest tensors first: they fill the card, and the launches
            // for the many small ones behind them are short
            std::stable_sort(order.begin(), order.end(),
                             [&](int64_t a, int64_t b) { return tensors[a].n > tensors[b].n; });
            for (const int64_t i : order) {
                const comera_grad_tensor &t = tensors[i];
                if (p->chunks.empty() || p->chunks.back().count == kChunkTensors) p->chunks.emplace_back();
                GradChunk &c = p->chunks.back();
                const uint32_t nt = uint32_t((t.n + kTile - 1) / kTile);
                c.e[c.count++] = {t.g, t.out ? t.out : const_cast<void *>(t.g),
                                  t.n | (t.dtype == COMERA_BF16 ? kBf16 : 0), c.tiles, c.tiles + nt};
                c.tiles += nt;
            }
            const uint32_t per = uint32_t(std::max(1.0, std::floor(tiles / kGradParts)));
            for (GradChunk &c : p->chunks) {
                c.per = per;
                c.part0 = p->parts;
                c.parts = int((c.tiles + per - 1) / per);
                p->parts += c.parts;
            }
            for (GradChunk &c : p->chunks) c.all_parts = p->parts;
            p->count = int64_t(order.size());
            p->stream = 2 * bytes_in > kStreamBytes;
            // one launch over the whole table: as many tiles a workgroup
            p->table.count = int(p->count);
            p->table.tiles = uint32_t(tiles);
            p->table.per = per;
            p->table.parts = p->table.all_parts = int((p->table.tiles + per - 1) / per);
        } catch (...) {
            delete p;
            throw;
        }
        *out = p;
        return COMERA_OK;
    } catch (...) {
        return COMERA_ERR_INTERNAL;
    }
}

void comera_grad_plan_destroy(comera_grad_plan_t p) { delete p; }

size_t comera_grad_table_bytes(comera_grad_plan_t p) {
    return p && p->chunks.size() > 1 ? sizeof(Entry) * size_t(p->count) : 0;
}

comera_status comera_grad_plan_set_table(comera_grad_plan_t p, void *table, size_t bytes, void *stream) {
    if (!p) return COMERA_ERR_INVALID_ARG;
    p->table.e = nullptr;
    const size_t need = comera_grad_table_bytes(p);
    if (!table || need == 0) return COMERA_OK;
    if (bytes < need || reinterpret_cast<uintptr_t>(table) % 8) return COMERA_ERR_WORKSPACE;
    // a captured table would be written by replays alone, and calls before
    // the first one would read it
    if (!launch_check_mode()) {
        hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
        if (note_hip(int(hipStreamIsCapturing(hipStream_t(stream), &capture)), "gradient table")) {
            (void)hipGetLastError();       // noted: not the next call's
            return COMERA_ERR_HIP;
        }
        if (capture != hipStreamCaptureStatusNone) return COMERA_ERR_INVALID_ARG;
    }
    Entry *e = static_cast<Entry *>(table);
    uint32_t tiles = 0;
    for (const GradChunk &c : p->chunks) {
        COMERA_LAUNCH(grad_table_kernel, dim3(1), dim3(128), 0, hipStream_t(stream), c, e, tiles);
        e += c.count;
        tiles += c.tiles;
    }
    if (note_hip(launch_status(), "gradient table")) return COMERA_ERR_HIP;
    p->table.e = static_cast<const Entry *>(table);
    p->written = !launch_check_mode();
    return COMERA_OK;
}

size_t comera_grad_workspace_bytes(comera_grad_plan_t p) {
    return p ? sizeof(double) * size_t(std::max(1, p->parts)) : 0;
}

comera_status comera_grad_norm(comera_grad_plan_t p, float scale, float *norm, int32_t *flag, void *ws,
                               size_t ws_bytes, void *stream) {
    if (comera_status e = grad_args(p, scale, ws, ws_bytes)) return e;
    if (!norm && !flag) return COMERA_ERR_INVALID_ARG;
    hipStream_t st = hipStream_t(stream);
    double *part = static_cast<double *>(ws);
    const int parts = launch_squares(p, part, st);
    COMERA_LAUNCH(grad_norm_kernel, dim3(1), dim3(kGradThreads), 0, st, part, parts, scale, norm, flag);
    return note_hip(launch_status(), "gradient norm") ? COMERA_ERR_HIP : COMERA_OK;
}

comera_status comera_grad_clip(comera_grad_plan_t p, float scale, float max_norm, float *norm, int32_t *flag, void *ws,
                               size_t ws_bytes, void *stream) {
    if (!(max_norm >= 0.f)) return COMERA_ERR_INVALID_ARG;
    if (comera_status e = grad_args(p, scale, ws, ws_bytes)) return e;
    if (p->chunks.empty()) {               // nothing to scale: a norm of zero
        if (!norm && !flag) return COMERA_OK;
        return comera_grad_norm(p, scale, norm, flag, ws, ws_bytes, stream);
    }
    hipStream_t st = hipStream_t(stream);
    double *part = static_cast<double *>(ws);
    if (p->chunks.size() == 1 && p->chunks[0].tiles <= kSmallTiles) {
        COMERA_LAUNCH(grad_small_kernel, dim3(1), dim3(kSmallThreads), 0, st, p->chunks[0], scale, max_norm, norm,
                      flag);
        return note_hip(launch_status(), "gradient clipping") ? COMERA_ERR_HIP : COMERA_OK;
    }
    launch_squares(p, part, st);
    if (p->has_table())
        launch_scale(p, p->table, part, scale, max_norm, norm, flag, st);
    else
        for (size_t i = p->chunks.size(); i-- > 0;)    // last read, first scaled
            launch_scale(p, p->chunks[i], part, scale, max_norm, norm, flag, st);
    return note_hip(launch_status(), "gradient clipping") ? COMERA_ERR_HIP : COMERA_OK;
}

}  // extern "C"
