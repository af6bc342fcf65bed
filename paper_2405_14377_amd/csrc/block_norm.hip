// Norms before and after a block, with its gate and residual scale:
//   z  = Npost(F)                     (z = F without a post-norm)
//   Xn = a X + beta * gate * z
//   H  = Npre(Xn)
// RMS:   N(v)_c = v_c r w_c + bias_c,           r = 1 / sqrt(mean(v^2) + eps)
// LAYER: N(v)_c = (v_c - mean) r w_c + bias_c,  r = 1 / sqrt(var + eps)
//
// Backward, with y the normalised row (before w and bias) and u = dN * w:
//   RMS   dv = r (u - y mean(u y))
//   LAYER dv = r (u - mean(u) - y mean(u y))
//   T = dXn + Npre'(dH);  dX = a T;  dgate = beta T z;  dF = Npost'(beta gate T)
//   dpost_w = sum_t beta gate T y_F,  dpost_b = sum_t beta gate T,
//   dpre_w = sum_t dH y_X,            dpre_b = sum_t dH
// The statistics are taken again from Xn and F, whose rows the backward reads
// in any case, so nothing is saved between the two calls.
//
// A row is held in the registers of LPR lanes (a wave, or several waves of
// one workgroup), CH chunks of VEC entries a lane: every input is read once
// and every output written once.  Bound by HBM: 4 rows forward, 6 backward.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "internal.h"
#include "rowops.h"

namespace comera {
namespace {

constexpr int kMaxWidth = 8192;
constexpr int kMaxParts = 256;         // backward workgroups: one per CU
constexpr int kWaveRows = 4;           // forward: rows side by side when a row is one wave's
constexpr int kBwdWaves = 8;           // backward: waves of a workgroup, two on every SIMD of its CU

struct NormArgs {
    const void *X, *F, *gate;          // X: the residual stream (forward), Xn (backward)
    const float *gate_ch, *post_w, *post_b, *pre_w, *pre_b;
    const void *dXn, *dH;
    void *Xn, *H;                      // forward
    void *dX, *dF, *dgate;             // backward (dgate of a per-token gate)
    float *part;                       // [workgroup][sums][N]
    int want;                          // bit s: sum s is asked for
    int64_t b;
    int N, lpr, post, pre;
    float eps, a, beta;
};

// The parameters' gradients, from the sums of all workgroups.
struct FinishArgs {
    const float *part;
    int parts, N, want;
    const float *gate_ch, *post_w, *post_b;
    float beta;
    float *dgate, *dpost_w, *dpost_b, *dpre_w, *dpre_b;

    // at column c, from the sums of y_F times T and of T
    __device__ __forceinline__ void post(int c, float yt, float t) const {
        const float gate = gate_ch ? gate_ch[c] : 1.f;
        if (dpost_w) dpost_w[c] = beta * gate * yt;
        if (dpost_b) dpost_b[c] = beta * gate * t;
        if (dgate) dgate[c] = beta * (yt * (post_w ? post_w[c] : 1.f) + (post_b ? post_b[c] * t : 0.f));
    }
    // of dH times y_X and of dH
    __device__ __forceinline__ void pre(int c, float yh, float h) const {
        if (dpre_w) dpre_w[c] = yh;
        if (dpre_b) dpre_b[c] = h;
    }
};

// Sums of NV (1, 2 or 4) values over the lanes of a row, the same bits in
// every lane of it.  Rows of LPR = 16 or 32 lanes: exchanges within them.
// Over a wave: the values are folded into one register, each in
// the rows of 16 lanes of its own, then summed within the rows, which takes
// 10 instructions for four values (four sums by themselves: about 50).  Rows
// of several waves: the waves' sums go through one of two LDS buffers in turn
// (a buffer is written again only after a barrier that every reader of its
// last use has passed), eight lanes read them and exchange them.  Every
// thread of the workgroup calls it equally often when a row has several
// waves.
template <int LPR, int NV>
__device__ __forceinline__ void row_sum(float (&v)[NV], float (*red)[8][4], int &turn, int waves) {
    static_assert(NV == 1 || NV == 2 || NV == 4, "one, two or four sums");
    static_assert(LPR == 0 || LPR == 16 || LPR == 32, "parts of a wave, or whole waves");
    if constexpr (LPR > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            v[i] = sum_of_16(v[i]);
            if constexpr (LPR == 32) v[i] = fold_16(v[i], v[i]);
        }
        return;
    }
    float s;
    if constexpr (NV == 4) {
        s = fold_16(fold_32(v[0], v[1]), fold_32(v[2], v[3]));     // rows: v0, v2, v1, v3
    } else {
        s = fold_32(v[0], v[NV - 1]);
        s = fold_16(s, s);
    }
    s = sum_of_16(s);
    if (waves > 1) {
        const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, w0 = w - w % waves, x = lane & 7;
        if ((lane & 15) == 0) red[turn][w][lane >> 4] = s;
        __syncthreads();
        s = red[turn][min(w0 + x, 7)][lane >> 4];
        s = sum_of_8(x < waves ? s : 0.f);
        turn ^= 1;
    }
    v[0] = lane_value(s, 0);
    if constexpr (NV > 1) v[1] = lane_value(s, 32);
    if constexpr (NV > 2) {
        v[2] = lane_value(s, 16);
        v[3] = lane_value(s, 48);
    }
}

// columns of a lane: chunk j starts at col[j]; the last chunk of a row whose
// width is no multiple of VEC is moved back to the row's end, and its first
// skip entries, which the chunk before also holds, are left out of sums.
// Lanes behind the row's end hold nothing (on = false).
template <int VEC, int CH>
struct Columns {
    int col[CH], skip[CH];
    bool on[CH];
    __device__ __forceinline__ Columns(int lane, int lpr, int N) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * lpr + lane) * VEC;
            on[j] = c < N;
            col[j] = on[j] ? min(c, N - VEC) : 0;
            skip[j] = on[j] ? c - col[j] : VEC;
        }
    }
    // zeros for the entries that are not the lane's own
    __device__ __forceinline__ void clear(float (&v)[CH * VEC]) const {
#pragma unroll
        for (int j = 0; j < CH; ++j)
            if (skip[j])
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[j * VEC + e] = e < skip[j] ? 0.f : v[j * VEC + e];
    }
    // whether entry e of chunk j counts in sums
    __device__ __forceinline__ bool counts(int j, int e) const { return e >= skip[j]; }
};

template <class T, int VEC, int CH>
__device__ __forceinline__ void load_row(const void *p, int64_t at, const Columns<VEC, CH> &k, float (&v)[CH * VEC]) {
    const T *row = static_cast<const T *>(p) + at;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        Pack<T, VEC> x;
        x.load(row + k.col[j]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[j * VEC + e] = x.get(e);
    }
}

// Every entry is stored by one lane alone, so an output may be the buffer of
// an input: what another lane of the row reads of an entry it does not own is
// neither summed nor stored.  Ordinary stores, although the forward alone is
// faster with streamed ones (16384 x 768, fp32 stream: 31.5 -> 24.3 us; 40001 x
// 1024: 76.4 -> 74.3): the next reader of Xn and H loses more than that (both
// together 48.8 -> 53.8 and 113 -> 119).
template <class T, int VEC, int CH>
__device__ __forceinline__ void store_row(void *p, int64_t at, const Columns<VEC, CH> &k,
                                          const float (&v)[CH * VEC]) {
    T *row = static_cast<T *>(p) + at;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        float x[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = v[j * VEC + e];
        if (k.skip[j] == 0) {
            Pack<T, VEC>::store(row + k.col[j], x);
        } else {
#pragma unroll
            for (int e = 1; e < VEC; ++e)
                if (k.counts(j, e)) {
                    const float y[1] = {x[e]};
                    Pack<T, 1>::store(row + k.col[j] + e, y);
                }
        }
    }
}

template <int VEC, int CH>
__device__ __forceinline__ void load_param(const float *p, float otherwise, const Columns<VEC, CH> &k,
                                           float (&v)[CH * VEC]) {
    if (p) {
        load_row<float, VEC, CH>(p, 0, k, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < CH * VEC; ++i) v[i] = otherwise;
}

// mean and reciprocal root of a row (mean 0 for RMS); two passes over the
// registers for LAYER, so that no digits are lost where the mean is large.
// Entries that are not the lane's own are zeros in v.
template <int LPR, int VEC, int CH>
__device__ __forceinline__ void row_stats(const float (&v)[CH * VEC], const Columns<VEC, CH> &k, int kind, float inv_n,
                                          float eps, float (*red)[8][4], int &turn, int waves, float &mean,
                                          float &r) {
    mean = 0.f;
    float q[1] = {0.f};
    if (kind == COMERA_NORM_LAYER) {
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < CH * VEC; ++i) s[0] += v[i];
        row_sum<LPR>(s, red, turn, waves);
        mean = s[0] * inv_n;
        float d[CH * VEC];
#pragma unroll
        for (int i = 0; i < CH * VEC; ++i) d[i] = v[i] - mean;
        k.clear(d);
#pragma unroll
        for (int i = 0; i < CH * VEC; ++i) q[0] += d[i] * d[i];
    } else {
#pragma unroll
        for (int i = 0; i < CH * VEC; ++i) q[0] += v[i] * v[i];
    }
    row_sum<LPR>(q, red, turn, waves);
    r = rsqrtf(q[0] * inv_n + eps);
}

// the rows of one token that the forward reads, as loaded
template <class TS, class TA, int VEC, int CH>
struct FwdRows {
    Pack<TS, VEC> x[CH];
    Pack<TA, VEC> f[CH], g[CH];
    __device__ __forceinline__ void load(const NormArgs &p, int64_t row, const Columns<VEC, CH> &k) {
        const int64_t at = row * p.N;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            x[j].load(static_cast<const TS *>(p.X) + at + k.col[j]);
            if (p.F) f[j].load(static_cast<const TA *>(p.F) + at + k.col[j]);
            if (p.gate) g[j].load(static_cast<const TA *>(p.gate) + at + k.col[j]);
        }
    }
};

// LPR: lanes of a row that is a part of a wave; 0 for rows of p.lpr lanes,
// whole waves.
template <class TS, class TA, int VEC, int CH, int LPR>
__global__ __launch_bounds__(512) void block_norm_fwd_kernel(NormArgs p) {
    constexpr int NE = VEC * CH;
    __shared__ __attribute__((aligned(16))) float red[2][8][4];
    int turn = 0;
    const int lpr = LPR ? LPR : p.lpr, waves = lpr >> 6, rows = int(blockDim.x) / lpr;
    const int lane = int(threadIdx.x) % lpr;
    const Columns<VEC, CH> k(lane, lpr, p.N);
    const float inv_n = 1.f / float(p.N);
    float pw[NE], pb[NE], w[NE], wb[NE];
    load_param<VEC, CH>(p.gate_ch, 1.f, k, pw);
    load_param<VEC, CH>(p.post_b, 0.f, k, pb);
#pragma unroll
    for (int i = 0; i < NE; ++i) pb[i] *= pw[i];
    {
        float x[NE];
        load_param<VEC, CH>(p.post_w, 1.f, k, x);
#pragma unroll
        for (int i = 0; i < NE; ++i) pw[i] *= x[i];
    }
    load_param<VEC, CH>(p.pre_w, 1.f, k, w);
    load_param<VEC, CH>(p.pre_b, 0.f, k, wb);
    // every thread takes equally many rows: those behind the last one read
    // it again and write nothing
    const int64_t step = int64_t(gridDim.x) * rows;
    int64_t row = int64_t(blockIdx.x) * rows + int(threadIdx.x) / lpr;
    FwdRows<TS, TA, VEC, CH> next;
    next.load(p, min(row, p.b - 1), k);
    for (int64_t base = int64_t(blockIdx.x) * rows; base < p.b; base += step, row += step) {
        const bool live = row < p.b;
        const FwdRows<TS, TA, VEC, CH> in = next;
        if (base + step < p.b) next.load(p, min(row + step, p.b - 1), k);
        const int64_t at = row * p.N;
        float x[NE];
#pragma unroll
        for (int i = 0; i < NE; ++i) x[i] = in.x[i / VEC].get(i % VEC);
        if (p.F) {
            float f[NE];
#pragma unroll
            for (int i = 0; i < NE; ++i) f[i] = in.f[i / VEC].get(i % VEC);
            k.clear(f);
            float mean = 0.f, r = 1.f;
            if (p.post != COMERA_NORM_NONE)
                row_stats<LPR, VEC, CH>(f, k, p.post, inv_n, p.eps, red, turn, waves, mean, r);
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                float z = (f[i] - mean) * r * pw[i] + pb[i];
                if (p.gate) z *= in.g[i / VEC].get(i % VEC);
                x[i] = p.a * x[i] + p.beta * z;
            }
        }
        k.clear(x);
        // the pre-norm takes Xn before its rounding to the stream's type
        float mean = 0.f, r = 1.f;
        if (p.pre != COMERA_NORM_NONE) row_stats<LPR, VEC, CH>(x, k, p.pre, inv_n, p.eps, red, turn, waves, mean, r);
        if (p.Xn && live) store_row<TS, VEC, CH>(p.Xn, at, k, x);
        if (p.H && live) {
#pragma unroll
            for (int i = 0; i < NE; ++i) x[i] = (x[i] - mean) * r * w[i] + wb[i];
            store_row<TA, VEC, CH>(p.H, at, k, x);
        }
    }
}

// the rows of one token that the backward reads, as loaded; entries that the
// lane does not own are zeros
template <class TS, class TA, int VEC, int CH>
struct BwdRows {
    Pack<TS, VEC> x[CH], t[CH];
    Pack<TA, VEC> h[CH], f[CH], g[CH];
    __device__ __forceinline__ void load(const NormArgs &p, int64_t row, const Columns<VEC, CH> &k) {
        const int64_t at = row * p.N;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            if (p.dXn) t[j].load(static_cast<const TS *>(p.dXn) + at + k.col[j]);
            if (p.dH) {
                x[j].load(static_cast<const TS *>(p.X) + at + k.col[j]);
                h[j].load(static_cast<const TA *>(p.dH) + at + k.col[j]);
            }
            if (p.F) f[j].load(static_cast<const TA *>(p.F) + at + k.col[j]);
            if (p.gate) g[j].load(static_cast<const TA *>(p.gate) + at + k.col[j]);
        }
    }
    __device__ __forceinline__ void arrive(const NormArgs &p) const {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            if (p.dXn) t[j].arrive();
            if (p.dH) {
                x[j].arrive();
                h[j].arrive();
            }
            if (p.F) f[j].arrive();
            if (p.gate) g[j].arrive();
        }
    }
    // zeros for the entries that are not the lane's own; a row that is not
    // live adds nothing to any sum
    __device__ __forceinline__ void clear(const NormArgs &p, const Columns<VEC, CH> &k, bool live) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int n = live ? k.skip[j] : VEC;
            if (n == 0) continue;
            t[j].clear(n);
            x[j].clear(n);
            h[j].clear(n);
            f[j].clear(n);
            g[j].clear(n);
        }
    }
};

// Per token two rounds of sums over the row for RMS (squares of both rows and
// sum(u x) at once, then the post-norm's), a third one ahead for the means of
// LAYER; the next token's rows are on their way meanwhile.  The sums over the
// tokens that the parameters' gradients need stay in registers over the rows
// of a workgroup: of y_F times T (times the token's gate), of T alike, of dH
// times y_X and of dH.  FULL: means and the sums for biases; without it (RMS
// norms, no bias) a third of the arithmetic and half of the sums fall away.
// block_norm_finish_kernel adds the workgroups' sums in order; a workgroup
// that is alone forms the gradients from its own.
// More arguments: FinishArgs of a workgroup that is alone, or none.
template <class TS, class TA, int VEC, int CH, bool FULL, int LPR, class... Alone>
__global__ __launch_bounds__(512) void block_norm_bwd_kernel(NormArgs p, Alone... alone) {
    constexpr int NE = VEC * CH, NS = FULL ? 4 : 2;
    // two tokens' rows do not fit the registers with 16 entries a lane, nor with
    // 12 in fp32 and every sum (4096 x 768 LAYER: 27.4 us with spills, 20.0)
    constexpr bool AHEAD = NE <= 8 || (NE <= 12 && !(FULL && sizeof(TS) == 4 && sizeof(TA) == 4));
    // The loop's end waits for the next token's rows, and with them for stores
    // behind those loads.  All stores after that wait: 16384 x 4096 155.1 ->
    // 149.1 us, 32768 x 512 45.6 -> 44.7.  Not in fp32 (8192 x 2048 81.3 ->
    // 82.0), nor with every sum (8191 x 1001 50.5 -> 51.7) or narrow rows
    // (65536 x 128 24.6 -> 25.2).
    constexpr bool LATE = !FULL && VEC == 8 && CH == 1 && LPR == 0 && sizeof(TS) == 2 && sizeof(TA) == 2;
    __shared__ __attribute__((aligned(16))) float red[2][8][4];
    extern __shared__ float share[];       // [2][rows][N] when rows > 1
    int turn = 0;
    const int lpr = LPR ? LPR : p.lpr, waves = lpr >> 6, rows = int(blockDim.x) / lpr;
    const int lane = int(threadIdx.x) % lpr;
    const Columns<VEC, CH> k(lane, lpr, p.N);
    const float inv_n = 1.f / float(p.N);
    const bool pre_mean = FULL && p.dH && p.pre == COMERA_NORM_LAYER;
    const bool post_mean = FULL && p.F && p.post == COMERA_NORM_LAYER;
    float pw[NE], w[NE], acc[NS][NE];
    load_param<VEC, CH>(p.gate_ch, 1.f, k, pw);
    {
        float x[NE];
        load_param<VEC, CH>(p.post_w, 1.f, k, x);
#pragma unroll
        for (int i = 0; i < NE; ++i) pw[i] *= p.beta * x[i];
    }
    load_param<VEC, CH>(p.pre_w, 1.f, k, w);
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < NE; ++i) acc[s][i] = 0.f;
    // every thread takes equally many rows: those behind the last one read
    // it again and write nothing
    const int64_t step = int64_t(gridDim.x) * rows;
    int64_t row = int64_t(blockIdx.x) * rows + int(threadIdx.x) / lpr;
    BwdRows<TS, TA, VEC, CH> next;
    if constexpr (AHEAD) next.load(p, min(row, p.b - 1), k);
    for (int64_t base = int64_t(blockIdx.x) * rows; base < p.b; base += step, row += step) {
        const bool live = row < p.b;
        BwdRows<TS, TA, VEC, CH> in;
        if constexpr (AHEAD) {
            in = next;
            if (base + step < p.b) next.load(p, min(row + step, p.b - 1), k);
        } else {
            in.load(p, min(row, p.b - 1), k);
        }
        in.clear(p, k, live);
        const int64_t at = row * p.N;
        float x[NE], f[NE], t[NE];
        float mean[2] = {0.f, 0.f};
        if (FULL && (pre_mean || post_mean)) {
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                if (pre_mean) mean[0] += in.x[i / VEC].get(i % VEC);
                if (post_mean) mean[1] += in.f[i / VEC].get(i % VEC);
            }
            row_sum<LPR>(mean, red, turn, waves);
            mean[0] *= inv_n;
            mean[1] *= inv_n;
        }
        if (p.dH)
#pragma unroll
            for (int i = 0; i < NE; ++i) x[i] = in.x[i / VEC].get(i % VEC) - (FULL ? mean[0] : 0.f);
        if (p.F)
#pragma unroll
            for (int i = 0; i < NE; ++i) f[i] = in.f[i / VEC].get(i % VEC) - (FULL ? mean[1] : 0.f);
        if constexpr (FULL) {
            if (p.dH) k.clear(x);          // the mean is not theirs
            if (p.F) k.clear(f);
        }
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        if (p.dH)
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                const float u = in.h[i / VEC].get(i % VEC) * w[i];
                s[0] += x[i] * x[i];
                s[1] += u * x[i];
                if constexpr (FULL) s[2] += u;
            }
        if (p.F)
#pragma unroll
            for (int i = 0; i < NE; ++i) s[3] += f[i] * f[i];
        if (p.dH || (p.F && p.post != COMERA_NORM_NONE)) row_sum<LPR>(s, red, turn, waves);
#pragma unroll
        for (int i = 0; i < NE; ++i) t[i] = 0.f;
        if (p.dXn)
#pragma unroll
            for (int i = 0; i < NE; ++i) t[i] = in.t[i / VEC].get(i % VEC);
        if (p.dH) {
            const float r = rsqrtf(s[0] * inv_n + p.eps);
            const float sy = s[1] * r * inv_n, su = pre_mean ? s[2] * inv_n : 0.f;
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                const float h = in.h[i / VEC].get(i % VEC), y = x[i] * r;
                acc[NS / 2][i] += h * y;
                if constexpr (FULL) acc[3][i] += h;
                t[i] += r * (FULL ? h * w[i] - su - y * sy : h * w[i] - y * sy);
            }
        }
        float dx[NE];
        {
            const float a = p.F ? p.a : 1.f;
#pragma unroll
            for (int i = 0; i < NE; ++i) dx[i] = a * t[i];
        }
        if ((!LATE || !p.F) && p.dX && live) store_row<TS, VEC, CH>(p.dX, at, k, dx);
        if (!p.F) continue;
        if constexpr (FULL) k.clear(t);
        const float r = p.post != COMERA_NORM_NONE ? rsqrtf(s[3] * inv_n + p.eps) : 1.f;
#pragma unroll
        for (int i = 0; i < NE; ++i) f[i] *= r;
        if (p.gate) {
            float z[NE], o[NE];
            load_param<VEC, CH>(p.post_w, 1.f, k, z);
            load_param<VEC, CH>(p.post_b, 0.f, k, o);
#pragma unroll
            for (int i = 0; i < NE; ++i) {
                z[i] = p.beta * t[i] * (f[i] * z[i] + o[i]);
                t[i] *= in.g[i / VEC].get(i % VEC);
            }
            if constexpr (LATE) next.arrive(p);
            if (p.dgate && live) store_row<TA, VEC, CH>(p.dgate, at, k, z);
        }
        float q[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            acc[0][i] += t[i] * f[i];
            if constexpr (FULL) acc[1][i] += t[i];
            t[i] *= pw[i];
            q[0] += t[i] * f[i];
            if constexpr (FULL) q[1] += t[i];
        }
        if (p.post != COMERA_NORM_NONE) {
            row_sum<LPR>(q, red, turn, waves);
            const float sy = q[0] * inv_n, su = post_mean ? q[1] * inv_n : 0.f;
#pragma unroll
            for (int i = 0; i < NE; ++i) t[i] = r * (FULL ? t[i] - su - f[i] * sy : t[i] - f[i] * sy);
        }
        if constexpr (LATE) {
            next.arrive(p);
            if (p.dX && live) store_row<TS, VEC, CH>(p.dX, at, k, dx);
        }
        if (p.dF && live) store_row<TA, VEC, CH>(p.dF, at, k, t);
    }
    if (!p.part) return;
    // the workgroup's sums, those that are asked for: its rows added in order
    // through LDS, a pair of sums at a time
    float *out = p.part + int64_t(blockIdx.x) * NS * p.N;
    if (rows == 1) {
#pragma unroll
        for (int s = 0; s < NS; ++s)
            if ((p.want >> s) & 1) store_row<float, VEC, CH>(out, int64_t(s) * p.N, k, acc[s]);
    } else {
        const int mine = int(threadIdx.x) / lpr;
#pragma unroll
        for (int s0 = 0; s0 < NS; s0 += 2) {
            if (!((p.want >> s0) & 3)) continue;
#pragma unroll
            for (int s = 0; s < 2; ++s)
                store_row<float, VEC, CH>(share, int64_t(s * rows + mine) * p.N, k, acc[s0 + s]);
            __syncthreads();
            for (int c = threadIdx.x; c < 2 * p.N; c += int(blockDim.x)) {
                const int s = c >= p.N, col = c - s * p.N;
                const float *x = share + s * rows * p.N + col;
                float v = x[0];
                for (int r = 1; r < rows; ++r) v += x[r * p.N];
                out[int64_t(s0 + s) * p.N + col] = v;
            }
            __syncthreads();
        }
    }
    if constexpr (sizeof...(Alone) > 0) {
        __syncthreads();
        for (int c = threadIdx.x; c < p.N; c += int(blockDim.x)) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};         // sums that are not asked for stay zeros
#pragma unroll
            for (int s = 0; s < NS; ++s)
                if ((p.want >> s) & 1) v[FULL ? s : 2 * s] = out[int64_t(s) * p.N + c];
            (alone.post(c, v[0], v[1]), ...);
            (alone.pre(c, v[2], v[3]), ...);
        }
    }
}

constexpr int kFinCols = 32, kFinGroups = 32;

// Sums of the workgroups' partials and the parameters' gradients from them:
// 32 columns x 32 groups of partials per workgroup (a thread has all its
// loads in flight at once), the groups added in order.  blockIdx.y = 0: the
// NP sums of the post-norm and the gate; 1: those of the pre-norm.
template <int NP>
__global__ __launch_bounds__(kFinCols *kFinGroups) void block_norm_finish_kernel(FinishArgs a) {
    constexpr int kPer = kMaxParts / kFinGroups, NS = 2 * NP;
    __shared__ float red[NP][kFinGroups][kFinCols];
    const int s0 = blockIdx.y * NP;
    if (!((a.want >> s0) & (NP == 2 ? 3 : 1))) return;
    const int l = threadIdx.x % kFinCols, g = threadIdx.x / kFinCols;
    const int c = blockIdx.x * kFinCols + l;
    float x[kPer][NP];
    const int cc = min(c, a.N - 1);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int p = g + i * kFinGroups;
#pragma unroll
        for (int s = 0; s < NP; ++s)
            x[i][s] = p < a.parts ? a.part[(int64_t(p) * NS + s0 + s) * a.N + cc] : 0.f;
    }
#pragma unroll
    for (int s = 0; s < NP; ++s) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) v += x[i][s];
        red[s][g][l] = v;
    }
    __syncthreads();
    if (g < NP) {                          // group s adds sum s ...
        float sum = 0.f;
        for (int i = 0; i < kFinGroups; ++i) sum += red[g][i][l];
        red[g][0][l] = sum;                // read by this thread alone so far
    }
    __syncthreads();
    if (g != 0 || c >= a.N) return;        // ... and group 0 forms the gradients
    const float first = red[0][0][l], second = NP == 2 ? red[NP - 1][0][l] : 0.f;
    if (blockIdx.y == 0)
        a.post(c, first, second);
    else
        a.pre(c, first, second);
}

// ---------------------------------------------------------------- host side
bool norm_kind(int k) { return k == COMERA_NORM_NONE || k == COMERA_NORM_RMS || k == COMERA_NORM_LAYER; }

bool norm_shape_ok(const comera_block_norm_shape *s) {
    return s && s->width >= 1 && (s->stream == COMERA_F32 || s->stream == COMERA_BF16) &&
           (s->act == COMERA_F32 || s->act == COMERA_BF16) && norm_kind(s->post) && norm_kind(s->pre) &&
           (s->gate == COMERA_GATE_NONE || s->gate == COMERA_GATE_CHANNEL || s->gate == COMERA_GATE_TOKEN) &&
           std::isfinite(s->eps) && s->eps > 0.f && std::isfinite(s->res_scale) && std::isfinite(s->branch_scale);
}

// a bf16 stream between fp32 blocks has no kernels
bool norm_supported(const comera_block_norm_shape *s) {
    return s->width <= kMaxWidth && !(s->stream == COMERA_BF16 && s->act == COMERA_F32);
}

// How a row is spread: lanes per row and entries per lane.
struct Spread {
    int vec, ch, lpr, rows;
    int threads() const { return lpr * rows; }
};

// Rows of up to 256 columns: 16 or 32 lanes with 8 entries each, several rows
// a wave.  65536 rows of 64, 100, 256 columns with LAYER norms and a token
// gate: forward 13.3, 14.0, 32.4 us (a wave each: 35.4, 36.9, 41.8), backward
// 31.9, 42.6, 75.4 (96.9, 117, 114).  Single entries below 8 columns.
Spread narrow_spread(int N, int waves) {
    if (N < 8) return {1, 1, 64, waves};
    const int lpr = N <= 128 ? 16 : 32;
    return {8, 1, lpr, 64 * waves / lpr};
}

// Forward: 8 entries a lane up to 512 columns; above, 12 or 16, whichever
// leaves fewer idle lanes (768 columns: 64 lanes x 12).  RMS, 24 M entries,
// with 12 and with 16: 768 columns bf16 41.0 and 42.9 us, fp32 73.3 and 74.9;
// 1001 59.5 and 41.2, 78.6 and 75.3; 2304 41.0 and 42.4, 72.1 and 77.8; 4096
// 64.9 and 38.5, 80.9 and 74.5.
Spread fwd_spread(int N) {
    if (N <= 256) return narrow_spread(N, kWaveRows);
    if (N <= 512) return {8, 1, 64, kWaveRows};
    const int l12 = (N + 767) / 768 * 64, l16 = (N + 1023) / 1024 * 64;
    const Spread sp = l12 * 12 < l16 * 16 && l12 <= 512 ? Spread{4, 3, l12, 1} : Spread{8, 2, l16, 1};
    return {sp.vec, sp.ch, sp.lpr, sp.lpr == 64 ? kWaveRows : 1};
}

// Backward: its registers hold two rows of four tensors and up to four sums,
// so 8 entries a lane as long as eight waves cover the row (4096 columns), 12
// where one wave then does (up to 768) or eight waves do (up to 6144), and 16
// above, which read one row at a time: 2048 x 5000 LAYER fp32 with 16 entries
// and two rows spilled registers (165 us; 50 with 12).
Spread bwd_spread(int N) {
    if (N <= 256) return narrow_spread(N, kBwdWaves);
    if (N > 512 && N <= 768) return {4, 3, 64, kBwdWaves};
    if (N > 6144) return {8, 2, (N + 1023) / 1024 * 64, 1};
    if (N > 4096) return {4, 3, (N + 767) / 768 * 64, 1};
    const int waves = (N + 511) / 512;
    return {8, 1, 64 * waves, kBwdWaves / waves};
}

// One workgroup that takes up to two turns forms the parameters' gradients
// itself and saves a launch.  One launch and two, us a call in a row of calls,
// which the host's launches bound, and the kernels alone (a replayed graph),
// fp32: 8 rows of 768 columns RMS 8.1 and 10.5, kernels 5.9 and 7.6, LAYER 8.5
// and 10.9, 7.1 and 8.9; 16 rows LAYER 9.3 and 10.8, 9.0 and 9.1.  The second
// turn of wide rows costs the kernels alone more than a launch (two rows of
// 4096 LAYER 9.6 and 10.7, 9.3 and 7.3), four turns cost more in any case (32
// rows of 768 RMS 11.7 and 11.3, 11.2 and 7.7; LAYER 13.4 and 11.5, 13.2 and
// 9.1).  Not above 4096 columns: one row of 8192 14.9 and 13.6, with LAYER
// 20.1 and 14.4.
bool bwd_alone(const Spread &sp, int N, int64_t b) { return b > 0 && b <= 2 * sp.rows && N <= 4096; }

int64_t bwd_parts(const Spread &sp, int N, int64_t b) {
    return bwd_alone(sp, N, b) ? 1 : std::min<int64_t>((b + sp.rows - 1) / sp.rows, kMaxParts);
}

template <class TS, class TA>
void launch_fwd(const NormArgs &p, const Spread &sp, hipStream_t st) {
    // Up to 4096 workgroups, with two rows each at least (four where a row is
    // eight waves) so that loads run ahead, but no CU left without its four:
    // 4096 x 8192 fp32 119 us with one row each, 105 with four; 40001 x 1024
    // bf16 81 us with five, 77 with two or three.
    const int64_t groups = (p.b + sp.rows - 1) / sp.rows, least = sp.lpr >= 512 ? 4 : 2;
    const unsigned grid =
        unsigned(std::min<int64_t>(4096, std::max(std::min<int64_t>(groups, 1024), groups / least)));
    const dim3 block(sp.threads());
    if (sp.vec == 1)
        COMERA_LAUNCH((block_norm_fwd_kernel<TS, TA, 1, 1, 0>), dim3(grid), block, 0, st, p);
    else if (sp.vec == 4)
        COMERA_LAUNCH((block_norm_fwd_kernel<TS, TA, 4, 3, 0>), dim3(grid), block, 0, st, p);
    else if (sp.ch == 2)
        COMERA_LAUNCH((block_norm_fwd_kernel<TS, TA, 8, 2, 0>), dim3(grid), block, 0, st, p);
    else if (sp.lpr == 16)
        COMERA_LAUNCH((block_norm_fwd_kernel<TS, TA, 8, 1, 16>), dim3(grid), block, 0, st, p);
    else if (sp.lpr == 32)
        COMERA_LAUNCH((block_norm_fwd_kernel<TS, TA, 8, 1, 32>), dim3(grid), block, 0, st, p);
    else
        COMERA_LAUNCH((block_norm_fwd_kernel<TS, TA, 8, 1, 0>), dim3(grid), block, 0, st, p);
}

template <class TS, class TA, bool FULL, class... Alone>
void launch_bwd(const NormArgs &p, const Spread &sp, hipStream_t st, const Alone &...alone) {
    const unsigned grid = unsigned(bwd_parts(sp, p.N, p.b));
    const dim3 block(sp.threads());
    const size_t lds = sp.rows > 1 ? sizeof(float) * 2 * sp.rows * p.N : 0;
    auto launch = [&](auto kernel) { COMERA_LAUNCH(kernel, dim3(grid), block, lds, st, p, alone...); };
    if (sp.vec == 1)
        launch(block_norm_bwd_kernel<TS, TA, 1, 1, FULL, 0, Alone...>);
    else if (sp.vec == 4)
        launch(block_norm_bwd_kernel<TS, TA, 4, 3, FULL, 0, Alone...>);
    else if (sp.ch == 1 && sp.lpr == 16)
        launch(block_norm_bwd_kernel<TS, TA, 8, 1, FULL, 16, Alone...>);
    else if (sp.ch == 1 && sp.lpr == 32)
        launch(block_norm_bwd_kernel<TS, TA, 8, 1, FULL, 32, Alone...>);
    else if (sp.ch == 1)
        launch(block_norm_bwd_kernel<TS, TA, 8, 1, FULL, 0, Alone...>);
    else if constexpr (sizeof...(Alone) == 0)
        launch(block_norm_bwd_kernel<TS, TA, 8, 2, FULL, 0>);
}

}  // namespace
}  // namespace comera

using namespace comera;

extern "C" {

size_t comera_block_norm_workspace_bytes(const comera_block_norm_shape *s, int64_t b) {
    if (!norm_shape_ok(s) || !norm_supported(s) || b < 0) return 0;
    return sizeof(float) * 4 * size_t(s->width) * size_t(std::max<int64_t>(1, bwd_parts(bwd_spread(int(s->width)), int(s->width), b)));
}

comera_status comera_block_norm_forward(const comera_block_norm_shape *s, int64_t b, const void *X, const void *F,
                                        const float *post_w, const float *post_b, const void *gate, const float *pre_w,
                                        const float *pre_b, void *Xn, void *H, void *stream) {
    if (!norm_shape_ok(s) || b < 0) return COMERA_ERR_INVALID_ARG;
    if (!norm_supported(s)) return COMERA_ERR_UNSUPPORTED;
    const bool gated = s->gate != COMERA_GATE_NONE;
    // what the shape leaves out is not passed, what it names is
    if ((!F && b > 0 && (Xn || post_w || post_b || gate)) || (F && gated != (gate != nullptr)) ||
        (s->post == COMERA_NORM_NONE && (post_w || post_b)) || (s->pre == COMERA_NORM_NONE && (pre_w || pre_b || H)) ||
        (s->pre != COMERA_NORM_NONE && !H && b > 0))
        return COMERA_ERR_INVALID_ARG;
    if (b == 0) return COMERA_OK;
    if (!X || (!Xn && !H)) return COMERA_ERR_INVALID_ARG;
    NormArgs p{};
    p.X = X;
    p.F = F;
    if (gated && s->gate == COMERA_GATE_CHANNEL) p.gate_ch = static_cast<const float *>(gate);
    if (gated && s->gate == COMERA_GATE_TOKEN) p.gate = gate;
    p.post_w = post_w;
    p.post_b = post_b;
    p.pre_w = pre_w;
    p.pre_b = pre_b;
    p.Xn = Xn;
    p.H = H;
    p.b = b;
    p.N = int(s->width);
    p.post = s->post;
    p.pre = s->pre;
    p.eps = s->eps;
    p.a = s->res_scale;
    p.beta = s->branch_scale;
    const Spread sp = fwd_spread(p.N);
    p.lpr = sp.lpr;
    hipStream_t st = hipStream_t(stream);
    if (s->stream == COMERA_F32 && s->act == COMERA_F32)
        launch_fwd<float, float>(p, sp, st);
    else if (s->stream == COMERA_F32)
        launch_fwd<float, bf16>(p, sp, st);
    else
        launch_fwd<bf16, bf16>(p, sp, st);
    return note_hip(launch_status(), "block norm") ? COMERA_ERR_HIP : COMERA_OK;
}

comera_status comera_block_norm_backward(const comera_block_norm_shape *s, int64_t b, const void *Xn, const void *F,
                                         const float *post_w, const float *post_b, const void *gate,
                                         const float *pre_w, const void *dXn, const void *dH, void *dX, void *dF,
                                         void *dgate, float *dpost_w, float *dpost_b, float *dpre_w, float *dpre_b,
                                         void *ws, size_t ws_bytes, void *stream) {
    if (!norm_shape_ok(s) || b < 0) return COMERA_ERR_INVALID_ARG;
    if (!norm_supported(s)) return COMERA_ERR_UNSUPPORTED;
    const bool gated = s->gate != COMERA_GATE_NONE, channel = s->gate == COMERA_GATE_CHANNEL;
    const bool pre = s->pre != COMERA_NORM_NONE, post = s->post != COMERA_NORM_NONE;
    if ((!F && b > 0 && (dF || dgate || dpost_w || dpost_b || post_w || post_b || gate)) ||
        (F && gated != (gate != nullptr)) || (!gated && dgate) ||
        (!post && (post_w || post_b || dpost_w || dpost_b)) || (!pre && (pre_w || dpre_w || dpre_b || dH)))
        return COMERA_ERR_INVALID_ARG;
    const bool params = dpost_w || dpost_b || dpre_w || dpre_b || (channel && dgate);
    const Spread sp = bwd_spread(int(s->width));
    const int64_t parts = bwd_parts(sp, int(s->width), b);
    if (b > 0 && ((!dXn && !dH) || (dH && !Xn))) return COMERA_ERR_INVALID_ARG;
    if (params && b > 0 &&
        (!ws || ws_bytes < comera_block_norm_workspace_bytes(s, b) || reinterpret_cast<uintptr_t>(ws) % 16))
        return COMERA_ERR_WORKSPACE;
    hipStream_t st = hipStream_t(stream);
    const bool full = dpost_b || dpre_b || (channel && dgate && post_b) || s->pre == COMERA_NORM_LAYER ||
                      s->post == COMERA_NORM_LAYER;
    NormArgs p{};
    p.X = Xn;
    p.F = F;
    if (channel) p.gate_ch = static_cast<const float *>(gate);
    if (s->gate == COMERA_GATE_TOKEN) p.gate = gate;
    p.post_w = post_w;
    p.post_b = post_b;
    p.pre_w = pre_w;
    p.dXn = dXn;
    p.dH = dH;
    p.dX = dX;
    p.dF = dF;
    if (!channel) p.dgate = dgate;
    p.part = params ? static_cast<float *>(ws) : nullptr;
    const bool ch_gate = channel && dgate;
    if (full)
        p.want = (dpost_w || ch_gate ? 1 : 0) | (dpost_b || ch_gate ? 2 : 0) | (dpre_w ? 4 : 0) | (dpre_b ? 8 : 0);
    else
        p.want = (dpost_w || ch_gate ? 1 : 0) | (dpre_w ? 2 : 0);
    p.b = b;
    p.N = int(s->width);
    p.post = s->post;
    p.pre = s->pre;
    p.eps = s->eps;
    p.a = s->res_scale;
    p.beta = s->branch_scale;
    p.lpr = sp.lpr;
    FinishArgs f{};
    f.part = p.part;
    f.parts = int(parts);
    f.N = p.N;
    f.want = p.want;
    f.gate_ch = p.gate_ch;
    f.post_w = post_w;
    f.post_b = post_b;
    f.beta = p.beta;
    f.dgate = channel ? static_cast<float *>(dgate) : nullptr;
    f.dpost_w = dpost_w;
    f.dpost_b = dpost_b;
    f.dpre_w = dpre_w;
    f.dpre_b = dpre_b;
    const bool alone = params && bwd_alone(sp, p.N, b);
    if (b > 0 && (params || dX || dF || p.dgate)) {
        auto launch = [&](const auto &...in_it) {
            if (s->stream == COMERA_F32 && s->act == COMERA_F32)
                full ? launch_bwd<float, float, true>(p, sp, st, in_it...)
                     : launch_bwd<float, float, false>(p, sp, st, in_it...);
            else if (s->stream == COMERA_F32)
                full ? launch_bwd<float, bf16, true>(p, sp, st, in_it...)
                     : launch_bwd<float, bf16, false>(p, sp, st, in_it...);
            else
                full ? launch_bwd<bf16, bf16, true>(p, sp, st, in_it...)
                     : launch_bwd<bf16, bf16, false>(p, sp, st, in_it...);
        };
        if (alone)
            launch(f);
        else
            launch();
    }
    if (params && !alone) {                // (no rows: zeros)
        const dim3 grid(unsigned((p.N + kFinCols - 1) / kFinCols), 2), block(kFinCols * kFinGroups);
        if (full)
            COMERA_LAUNCH((block_norm_finish_kernel<2>), grid, block, 0, st, f);
        else
            COMERA_LAUNCH((block_norm_finish_kernel<1>), grid, block, 0, st, f);
    }
    return note_hip(launch_status(), "block norm") ? COMERA_ERR_HIP : COMERA_OK;
}

}  // extern "C"
