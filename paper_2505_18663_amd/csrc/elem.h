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

// Activations, fp32 in and out.  exp and the division are the hardware's.  The result's relative error is at most 2^-20, and (4 |t| + 16) 2^-24
// where it falls like e^-|t| (t is rounded on its way into the exponential): 2^-15 at t = 87, where a rounding to bf16 is 2^-9.  What is
// smaller still, below 2^-118, may come out as zero: the reciprocal's argument is then beyond 2^126.  exp overflows to inf, z / inf = 0.
//   silu(z) = z / (1 + e^-z)
//   gelu_tanh(z) = z/2 (1 + tanh u) = z / (1 + e^-2u), u = sqrt(2/pi) (z + 0.044715 z^3)
//   gelu(z) = z/2 (1 + erf(z / sqrt 2)) = z Q(-z) = z (1 - Q(z)), Q the normal distribution's upper tail: 1 + erf has no digits left
//     below z = -5.  Q(a) = e^(-a^2 / 2) P(1 / (1 + 0.3 a)) for a >= 0, P the polynomial of degree 8 with the smallest largest relative error
//     up to a = 14 (5.8e-8), beyond which the exponential is below 2^-126.
//     32760 x 1536 x 8960 with it 837 us, with erff 952, with erfcf 1060.
static __device__ __forceinline__ float sigmoid_times(float z, float t) {   // z / (1 + e^-t)
    return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * t));
}
static __device__ __forceinline__ float upper_tail(float a) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, a, 1.0f));
    float p = 0.0383793637f;
    p = fmaf(p, t, -0.169170782f);
    p = fmaf(p, t, 0.228668645f);
    p = fmaf(p, t, -0.0765151531f);
    p = fmaf(p, t, 0.142540798f);
    p = fmaf(p, t, 0.0946815684f);
    p = fmaf(p, t, 0.121920779f);
    p = fmaf(p, t, 0.119487643f);
    p = fmaf(p, t, 7.17154398e-06f);
    return p * __builtin_amdgcn_exp2f(a * a * -0.721347520f);
}
template <int ACT>
static __device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == DVDQ_ACT_SILU) return sigmoid_times(z, z);
    else if constexpr (ACT == DVDQ_ACT_GELU_TANH) {
        // e^-2u = 2^(z (a + b z^2)), the constants multiplied out
        const float t = z * fmaf(z * z, -0.10294324f, -2.3022082f);
        return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
    }
    else if constexpr (ACT == DVDQ_ACT_GELU) {
        const float q = upper_tail(fminf(fabsf(z), 20.0f));   // (0 from 20 on)
        return z * (z < 0.0f ? q : 1.0f - q);
    }
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
