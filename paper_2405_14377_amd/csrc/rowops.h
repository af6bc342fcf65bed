// Device helpers of the row operators (dense embedding, block norms, gradient
// clipping): wide loads and stores of fp32 and bf16 entries at any element
// alignment, and sums over a wave.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace comera {

struct bf16 {
    uint16_t bits;
};

// Wide accesses that need no more than the entries' own alignment: gfx950
// runs with unaligned global access on, so one instruction serves rows of
// any width and tensors that start anywhere.
template <int BYTES, int ALIGN>
struct Wide;

// a store that leaves no line in the caches (STREAM), or an ordinary one
template <bool STREAM, class W, class T>
__device__ __forceinline__ void store_wide(T *p, const W &u) {
    if constexpr (STREAM)
        __builtin_nontemporal_store(u, reinterpret_cast<W *>(p));
    else
        *reinterpret_cast<W *>(p) = u;
}

template <>
struct Wide<16, 4> {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct Wide<16, 2> {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
};
template <>
struct Wide<8, 2> {
    typedef uint32_t type __attribute__((ext_vector_type(2), aligned(2)));
};

__device__ __forceinline__ float lo_bf16(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

// two fp32 values rounded to nearest even (v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
}

// V consecutive entries as loaded (registers of 32 bits), and as fp32 values
template <class T, int V>
struct Pack;

template <int V>
struct Pack<float, V> {
    float x[V];
    __device__ __forceinline__ void load(const float *p) {
        if constexpr (V % 4 == 0) {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const auto u = *reinterpret_cast<const typename Wide<16, 4>::type *>(p + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i + e] = __uint_as_float(u[e]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = p[i];
        }
    }
    __device__ __forceinline__ float get(int i) const { return x[i]; }
    __device__ __forceinline__ void clear(int first) {     // entries [0, first)
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = i < first ? 0.f : x[i];
    }
    template <bool STREAM = false>
    static __device__ __forceinline__ void store(float *p, const float (&v)[V]) {
        if constexpr (V % 4 == 0) {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                typename Wide<16, 4>::type u;
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = __float_as_uint(v[i + e]);
                store_wide<STREAM>(p + i, u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) p[i] = v[i];
        }
    }
};

template <int V>
struct Pack<bf16, V> {
    uint32_t x[(V + 1) / 2];
    __device__ __forceinline__ void load(const bf16 *p) {
        if constexpr (V % 8 == 0) {
#pragma unroll
            for (int i = 0; i < V; i += 8) {
                const auto u = *reinterpret_cast<const typename Wide<16, 2>::type *>(p + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i / 2 + e] = u[e];
            }
        } else if constexpr (V % 4 == 0) {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const auto u = *reinterpret_cast<const typename Wide<8, 2>::type *>(p + i);
                x[i / 2] = u[0];
                x[i / 2 + 1] = u[1];
            }
        } else {
            static_assert(V == 1, "bf16 packs of 1, or of a multiple of 4");
            x[0] = p->bits;
        }
    }
    __device__ __forceinline__ void arrive() const {       // waits for the load
#pragma unroll
        for (int i = 0; i < (V + 1) / 2; ++i) asm volatile("" ::"v"(x[i]) : "memory");
    }
    __device__ __forceinline__ float get(int i) const { return i & 1 ? hi_bf16(x[i / 2]) : lo_bf16(x[i / 2]); }
    __device__ __forceinline__ void clear(int first) {     // entries [0, first)
#pragma unroll
        for (int i = 0; i < V; i += 2)
            x[i / 2] = i + 1 < first ? 0u : i < first ? x[i / 2] & 0xffff0000u : x[i / 2];
    }
    template <bool STREAM = false>
    static __device__ __forceinline__ void store(bf16 *p, const float (&v)[V]) {
        if constexpr (V % 8 == 0) {
#pragma unroll
            for (int i = 0; i < V; i += 8) {
                typename Wide<16, 2>::type u;
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = pack_bf16(v[i + 2 * e], v[i + 2 * e + 1]);
                store_wide<STREAM>(p + i, u);
            }
        } else if constexpr (V % 4 == 0) {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                typename Wide<8, 2>::type u;
                u[0] = pack_bf16(v[i], v[i + 1]);
                u[1] = pack_bf16(v[i + 2], v[i + 3]);
                store_wide<STREAM>(p + i, u);
            }
        } else {
            p->bits = uint16_t(pack_bf16(v[0], 0.f));
        }
    }
};

// v of the lane that the DPP control `ctrl` names (within a row of 16 lanes)
template <int ctrl>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float(uint32_t(__builtin_amdgcn_update_dpp(0, int(__float_as_uint(v)), ctrl, 0xf, 0xf, true)));
}

// sum over 8 lanes in a row, the same bits in each of them
__device__ __forceinline__ float sum_of_8(float v) {
    v += dpp<0xb1>(v);      // quad_perm 1,0,3,2
    v += dpp<0x4e>(v);      // quad_perm 2,3,0,1
    v += dpp<0x141>(v);     // row_half_mirror
    return v;
}

// sum over the 16 lanes of a row
__device__ __forceinline__ float sum_of_16(float v) {
    v = sum_of_8(v);
    v += dpp<0x140>(v);     // row_mirror
    return v;
}

// Lanes 0-31: a of this lane and of the one 32 above; lanes 32-63: the same
// of b.  One exchange and one addition for two values.
__device__ __forceinline__ float fold_32(float a, float b) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}

// Rows 0 and 2 of 16 lanes: a of this lane and of the one 16 above; rows 1
// and 3: b of the one 16 below and of this lane.
__device__ __forceinline__ float fold_16(float a, float b) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}

__device__ __forceinline__ float lane_value(float v, int lane) {
    return __uint_as_float(uint32_t(__builtin_amdgcn_readlane(int(__float_as_uint(v)), lane)));
}

}  // namespace comera
