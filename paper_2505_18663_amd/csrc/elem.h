// Element types of the operators around the quantized layer (rope.hip, group_norm.hip, linear16.hip): conversions to and from
// fp32, 16-byte pieces of a row at any element's address, activations.
#pragma once
#include <type_traits>

#include "dvdq_internal.h"

namespace dvdq {

struct Bf16 {
    using Raw = uint16_t;
    static constexpr int kVec = 8;   // elements in 16 bytes
    static __device__ __forceinline__ float to_f32(Raw v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
    static __device__ __forceinline__ Raw from_f32(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }   // nearest even
};
struct Fp16 {
    using Raw = uint16_t;
    static constexpr int kVec = 8;
    static __device__ __forceinline__ float to_f32(Raw v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ __forceinline__ Raw from_f32(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }   // nearest even
};
struct Fp32 {
    using Raw = float;
    static constexpr int kVec = 4;
    static __device__ __forceinline__ float to_f32(Raw v) { return v; }
    static __device__ __forceinline__ Raw from_f32(float f) { return f; }
};

// V elements of a row.  Global loads and stores of 16 bytes take any element's address, so rows of any pitch and views that begin
// at any element are moved in whole pieces; only the piece across a row's end goes by element.
template <typename E, int V = E::kVec>
struct __attribute__((packed, aligned(sizeof(typename E::Raw)))) Piece {
    typename E::Raw e[V];
};

template <typename E, int V = E::kVec>
static __device__ __forceinline__ Piece<E, V> load_piece(const typename E::Raw *p, int n) {
    if (n >= V) return *reinterpret_cast<const Piece<E, V> *>(p);
    Piece<E, V> r = {};
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < n) r.e[i] = p[i];
    return r;
}
// STREAM: past the caches, for outputs that are larger than those and whose pieces make whole lines between them
template <typename E, int V = E::kVec, bool STREAM = false>
static __device__ __forceinline__ void store_piece(typename E::Raw *p, const Piece<E, V> &v, int n) {
    if (n >= V) {
        if constexpr (STREAM && sizeof(v) == 16) {
            typedef uint32_t Quad __attribute__((ext_vector_type(4)));
            typedef Quad Anywhere __attribute__((aligned(2)));
            __builtin_nontemporal_store(__builtin_bit_cast(Quad, v), reinterpret_cast<Anywhere *>(p));
        } else {
            *reinterpret_cast<Piece<E, V> *>(p) = v;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < n) p[i] = v.e[i];
}

// Activations, fp32 in and out.  exp and the division are the hardware's (relative error of 1e-6 at most where the result is a
// normal number), an order of magnitude below the rounding to 16 bits; the limits are exact: exp overflows to inf, z / inf = 0.
//   silu(z) = z / (1 + e^-z)
//   gelu_tanh(z) = z/2 (1 + tanh u) = z / (1 + e^-2u), u = sqrt(2/pi) (z + 0.044715 z^3)
//   gelu(z) = z/2 (1 + erf(z / sqrt 2))
static __device__ __forceinline__ float sigmoid_times(float z, float t) {   // z / (1 + e^-t)
    return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * t));
}
template <int ACT>
static __device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == DVDQ_ACT_SILU) return sigmoid_times(z, z);
    else if constexpr (ACT == DVDQ_ACT_GELU_TANH) {
        // e^-2u = 2^(z (a + b z^2)), the constants multiplied out
        const float t = z * fmaf(z * z, -0.10294324f, -2.3022082f);
        return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
    }
    else if constexpr (ACT == DVDQ_ACT_GELU) return 0.5f * z * (1.0f + erff(0.70710678118654752f * z));
    else return z;
}

// Calls f with the element type of a DVDQ_BF16 / DVDQ_FP16 / DVDQ_FP32 code (already validated).
template <class F>
inline int with_type(int dtype, F f) {
    switch (dtype) {
        case DVDQ_BF16: return f(Bf16());
        case DVDQ_FP16: return f(Fp16());
        default: return f(Fp32());
    }
}

// The same for an activation.
template <class F>
inline int with_act(int act, F f) {
    switch (act) {
        case DVDQ_ACT_SILU: return f(std::integral_constant<int, DVDQ_ACT_SILU>());
        case DVDQ_ACT_GELU_TANH: return f(std::integral_constant<int, DVDQ_ACT_GELU_TANH>());
        case DVDQ_ACT_GELU: return f(std::integral_constant<int, DVDQ_ACT_GELU>());
        default: return f(std::integral_constant<int, DVDQ_ACT_NONE>());
    }
}

}  // namespace dvdq
