// Element types of the operators around the quantized layer (rope.hip, group_norm.hip, rows8.hip, linear_tiles.h): conversions to and from
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
// 16 bytes without the first `by` (fewer than 16), zero behind.  (load_end has the same written out: of words in memory the compiler then makes loads of the
// words that are wanted, an eighth less code; 3 x 202 x 912 in 8 bits 3.4 -> 3.2 us.)
static __device__ __forceinline__ uint4 shifted_down(const uint4 &v, uint32_t by) {
    const uint32_t words = by >> 2, bytes = by & 3;
    const uint32_t a = words == 0 ? v.x : words == 1 ? v.y : words == 2 ? v.z : v.w;
    const uint32_t b = words == 0 ? v.y : words == 1 ? v.z : words == 2 ? v.w : 0u;
    const uint32_t c = words == 0 ? v.z : words == 1 ? v.w : 0u, d = words == 0 ? v.w : 0u;
    return make_uint4(__builtin_amdgcn_alignbyte(b, a, bytes), __builtin_amdgcn_alignbyte(c, b, bytes), __builtin_amdgcn_alignbyte(d, c, bytes),
                      __builtin_amdgcn_alignbyte(0u, d, bytes));
}
// 16 bytes of a row of bytes, the last n (fewer than 16) of which end it, as words, zero past the end.  Loads that each hang on a condition are waited
// for one by one (8 bytes took a copy of 6242 rows 6 us), so where the row has them the 16 bytes that end with it are loaded and shifted down; in a
// shorter row the elements (E bytes each) come at once, the last one in the place of those past it.
template <int E>
static __device__ __forceinline__ uint4 load_end(const uint8_t *p, int n, bool whole_before) {
    if (n <= 0) return make_uint4(0, 0, 0, 0);
    if (whole_before) {
        struct __attribute__((packed, aligned(E))) Sixteen {
            uint32_t w[4];
        };
        const Sixteen v = *reinterpret_cast<const Sixteen *>(p + n - 16);
        const uint32_t by = 16 - n, words = by >> 2, bytes = by & 3;
        const uint32_t a = words == 0 ? v.w[0] : words == 1 ? v.w[1] : words == 2 ? v.w[2] : v.w[3];
        const uint32_t b = words == 0 ? v.w[1] : words == 1 ? v.w[2] : words == 2 ? v.w[3] : 0u;
        const uint32_t c = words == 0 ? v.w[2] : words == 1 ? v.w[3] : 0u, d = words == 0 ? v.w[3] : 0u;
        return make_uint4(__builtin_amdgcn_alignbyte(b, a, bytes), __builtin_amdgcn_alignbyte(c, b, bytes), __builtin_amdgcn_alignbyte(d, c, bytes),
                          __builtin_amdgcn_alignbyte(0u, d, bytes));
    }
    using Raw = std::conditional_t<E == 1, uint8_t, std::conditional_t<E == 2, uint16_t, uint32_t>>;
    uint32_t e[16 / E], w[4] = {};
#pragma unroll
    for (int i = 0; i < 16 / E; ++i) e[i] = reinterpret_cast<const Raw *>(p)[min(i, n / E - 1)];
#pragma unroll
    for (int i = 0; i < 16 / E; ++i) w[i * E / 4] |= i < n / E ? e[i] << 8 * (i * E % 4) : 0u;
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// STREAM: past the caches, for outputs that are larger than those and whose pieces make whole lines between them
template <typename E, int V = E::kVec, bool STREAM = false>
static __device__ __forceinline__ void store_piece(typename E::Raw *p, const Piece<E, V> &v, int n) {
    if (n >= V) {
        if constexpr (STREAM && sizeof(v) == 32) {   // (fp32: two pieces)
            typedef uint32_t Quad __attribute__((ext_vector_type(4)));
            typedef Quad Anywhere __attribute__((aligned(4)));
            struct Two { Quad q[2]; };
            const Two t = __builtin_bit_cast(Two, v);
            __builtin_nontemporal_store(t.q[0], reinterpret_cast<Anywhere *>(p));
            __builtin_nontemporal_store(t.q[1], reinterpret_cast<Anywhere *>(p) + 1);
        } else if constexpr (STREAM && sizeof(v) == 16) {
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
