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

constexpr int kChunkTensors = 128;     // tensors of one launch: their table is a kernel argument of under 4 KiB
constexpr int kTile = 8192;            // entries that a workgroup takes at a time
constexpr int kGradThreads = 256;
constexpr int kGradParts = 2048;       // workgroups of the first pass over all launches (about)
constexpr int kChunkParts = 256;       // and at least so many of one launch, while it has tiles: one per CU
constexpr int kScaleBlocks = 2048;     // workgroups of one launch of the second pass, at most

struct GradChunk {
    const void *g[kChunkTensors];
    void *out[kChunkTensors];
    int64_t n[kChunkTensors];
    uint32_t tile0[kChunkTensors + 1]; // first tile of each tensor; behind the last one, the tiles and then 2^32 - 1
    uint32_t tiles;
    uint64_t is_bf16[kChunkTensors / 64];
    int count;
    int part0, parts;                  // this launch's partials
    int all_parts;
};
static_assert(sizeof(GradChunk) <= 3968, "the table is passed as a kernel argument");

// tensor that holds tile t (the last one that starts at or before it): every
// lane compares two entries of the table, so it takes one round trip
__device__ __forceinline__ int tensor_of(const GradChunk &c, uint32_t t) {
    static_assert(kChunkTensors == 128, "two entries a lane");
    const int lane = threadIdx.x & 63;
    const uint32_t x = c.tile0[lane], y = c.tile0[64 + lane];
    return __popcll(__ballot(x <= t)) + __popcll(__ballot(y <= t)) - 1;
}

// sum over a workgroup of 256 threads in a fixed order, in every thread
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double red[kGradThreads / 64];
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < kGradThreads / 64; ++w) v += red[w];
    return v;
}

// One tile: each thread's 16-byte pieces, all in flight at once.  use(p, i) is
// called for every whole piece at entry i, rest(j) for the entries behind the
// last one.
template <class T, class Use, class Rest>
__device__ __forceinline__ void for_tile(const T *g, int64_t at, int64_t n, Use use, Rest rest) {
    constexpr int V = 16 / sizeof(T), U = kTile / (V * kGradThreads);
    const int64_t i0 = at + int64_t(threadIdx.x) * V;
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
    if (whole + threadIdx.x < n) rest(whole + threadIdx.x);
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

__global__ __launch_bounds__(kGradThreads) void grad_squares_kernel(GradChunk c, double *part) {
    const uint32_t t0 = uint32_t(uint64_t(c.tiles) * blockIdx.x / c.parts);
    const uint32_t t1 = uint32_t(uint64_t(c.tiles) * (blockIdx.x + 1) / c.parts);
    double s = 0;
    int i = tensor_of(c, t0);
    for (uint32_t t = t0; t < t1; ++t) {
        while (t >= c.tile0[i + 1]) ++i;
        const int64_t at = int64_t(t - c.tile0[i]) * kTile;
        s += (c.is_bf16[i >> 6] >> (i & 63)) & 1 ? tile_squares(static_cast<const bf16 *>(c.g[i]), at, c.n[i])
                                                 : tile_squares(static_cast<const float *>(c.g[i]), at, c.n[i]);
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

template <class T>
__device__ __forceinline__ void tile_scale(const T *g, T *out, int64_t at, int64_t n, float c) {
    constexpr int V = 16 / sizeof(T);
    for_tile<T>(
        g, at, n,
        [&](const Pack<T, V> &p, int64_t i) {
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = c * p.get(e);
            Pack<T, V>::store(out + i, v);
        },
        [&](int64_t j) {
            Pack<T, 1> p;
            p.load(g + j);
            const float v[1] = {c * p.get(0)};
            Pack<T, 1>::store(out + j, v);
        });
}

__global__ __launch_bounds__(kGradThreads) void grad_scale_kernel(GradChunk c, const double *part, float scale,
                                                                  float max_norm, float *norm, int32_t *flag) {
    const double v = total_norm(part, c.all_parts, scale);
    if (c.part0 == 0 && blockIdx.x == 0 && threadIdx.x == 0) write_norm(v, norm, flag);
    const bool clip = isfinite(float(v)) && v > double(max_norm);
    const float f = clip ? float(double(scale) * (double(max_norm) / v)) : scale;
    // from the last tile back: what the first pass read last is still cached
    const uint32_t b = gridDim.x - 1 - blockIdx.x;
    const uint32_t t0 = uint32_t(uint64_t(c.tiles) * b / gridDim.x);
    const uint32_t t1 = uint32_t(uint64_t(c.tiles) * (b + 1) / gridDim.x);
    int i = tensor_of(c, t1 - 1);
    for (uint32_t t = t1; t-- > t0;) {
        while (t < c.tile0[i]) --i;
        if (f == 1.f && c.out[i] == c.g[i]) continue;
        const int64_t at = int64_t(t - c.tile0[i]) * kTile;
        if ((c.is_bf16[i >> 6] >> (i & 63)) & 1)
            tile_scale(static_cast<const bf16 *>(c.g[i]), static_cast<bf16 *>(c.out[i]), at, c.n[i], f);
        else
            tile_scale(static_cast<const float *>(c.g[i]), static_cast<float *>(c.out[i]), at, c.n[i], f);
    }
}

}  // namespace
}  // namespace comera

// the tensors' table, cut into launches (host memory only)
struct comera_grad_plan_s {
    std::vector<comera::GradChunk> chunks;
    int parts = 0;
};

using namespace comera;

namespace {

struct Range {
    uintptr_t begin, end;
    int64_t tensor;
    bool written;
};

}  // namespace

extern "C" {

comera_status comera_grad_plan(const comera_grad_tensor *tensors, int64_t count, comera_grad_plan_t *out) {
    if (!out) return COMERA_ERR_INVALID_ARG;
    *out = nullptr;
    if (count < 0 || (count > 0 && !tensors)) return COMERA_ERR_INVALID_ARG;
    try {
        std::vector<Range> ranges;
        double tiles = 0;
        for (int64_t i = 0; i < count; ++i) {
            const comera_grad_tensor &t = tensors[i];
            if (t.n < 0 || (t.dtype != COMERA_F32 && t.dtype != COMERA_BF16)) return COMERA_ERR_INVALID_ARG;
            if (t.n == 0) continue;
            if (!t.g || t.n >= (int64_t(1) << 42)) return COMERA_ERR_INVALID_ARG;
            const uintptr_t esz = t.dtype == COMERA_F32 ? 4 : 2, bytes = uintptr_t(t.n) * esz;
            const uintptr_t g = reinterpret_cast<uintptr_t>(t.g), o = reinterpret_cast<uintptr_t>(t.out);
            if (g % esz || o % esz) return COMERA_ERR_INVALID_ARG;
            ranges.push_back({g, g + bytes, i, !o || o == g});
            if (o && o != g) ranges.push_back({o, o + bytes, i, true});
            tiles += double((t.n + kTile - 1) / kTile);
        }
        // no buffer twice: an entry would count twice in the norm, or be
        // scaled by two workgroups at once
        std::sort(ranges.begin(), ranges.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
        for (size_t i = 1; i < ranges.size(); ++i)
            if (ranges[i].begin < ranges[i - 1].end) return COMERA_ERR_INVALID_ARG;
        if (tiles > 2147483647.0) return COMERA_ERR_UNSUPPORTED;
        comera_grad_plan_s *p = new comera_grad_plan_s;
        try {
            for (int64_t i = 0; i < count; ++i) {
                const comera_grad_tensor &t = tensors[i];
                if (t.n == 0) continue;
                if (p->chunks.empty() || p->chunks.back().count == kChunkTensors) {
                    p->chunks.emplace_back();
                    std::fill(p->chunks.back().tile0 + 1, p->chunks.back().tile0 + kChunkTensors + 1, 0xffffffffu);
                }
                GradChunk &c = p->chunks.back();
                const int k = c.count++;
                c.g[k] = t.g;
                c.out[k] = t.out ? t.out : const_cast<void *>(t.g);
                c.n[k] = t.n;
                c.tile0[k + 1] = c.tile0[k] + uint32_t((t.n + kTile - 1) / kTile);
                if (t.dtype == COMERA_BF16) c.is_bf16[k >> 6] |= uint64_t(1) << (k & 63);
            }
            for (GradChunk &c : p->chunks) {
                c.tiles = c.tile0[c.count];
                const int64_t n = c.tiles;
                c.part0 = p->parts;
                c.parts = int(std::min(n, std::max<int64_t>(kChunkParts, int64_t(double(n) / tiles * kGradParts))));
                p->parts += c.parts;
            }
            for (GradChunk &c : p->chunks) c.all_parts = p->parts;
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

size_t comera_grad_workspace_bytes(comera_grad_plan_t p) {
    return p ? sizeof(double) * size_t(std::max(1, p->parts)) : 0;
}

static comera_status grad_args(comera_grad_plan_t p, float scale, const void *ws, size_t ws_bytes) {
    if (!p || !std::isfinite(scale) || !(scale > 0.f)) return COMERA_ERR_INVALID_ARG;
    if (!ws || ws_bytes < comera_grad_workspace_bytes(p) || reinterpret_cast<uintptr_t>(ws) % sizeof(double))
        return COMERA_ERR_WORKSPACE;
    return COMERA_OK;
}

comera_status comera_grad_norm(comera_grad_plan_t p, float scale, float *norm, int32_t *flag, void *ws,
                               size_t ws_bytes, void *stream) {
    if (comera_status e = grad_args(p, scale, ws, ws_bytes)) return e;
    if (!norm && !flag) return COMERA_ERR_INVALID_ARG;
    hipStream_t st = hipStream_t(stream);
    double *part = static_cast<double *>(ws);
    for (const GradChunk &c : p->chunks)
        COMERA_LAUNCH(grad_squares_kernel, dim3(unsigned(c.parts)), dim3(kGradThreads), 0, st, c, part);
    COMERA_LAUNCH(grad_norm_kernel, dim3(1), dim3(kGradThreads), 0, st, part, p->parts, scale, norm, flag);
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
    for (const GradChunk &c : p->chunks)
        COMERA_LAUNCH(grad_squares_kernel, dim3(unsigned(c.parts)), dim3(kGradThreads), 0, st, c, part);
    for (size_t i = p->chunks.size(); i-- > 0;) {      // last read, first scaled
        const GradChunk &c = p->chunks[i];
        COMERA_LAUNCH(grad_scale_kernel, dim3(std::min<unsigned>(c.tiles, kScaleBlocks)), dim3(kGradThreads), 0, st, c,
                      part, scale, max_norm, norm, flag);
    }
    return note_hip(launch_status(), "gradient clipping") ? COMERA_ERR_HIP : COMERA_OK;
}

}  // extern "C"
