// Rows normed by their root mean square, with the residual's addition, and rows to 8 bits with a scale each:
//
//   h = T(x + residual)        rounded to the tensors' type T (x itself without a residual)
//   y = T(h weight / root)     root = sqrt(mean h^2 + eps)
//   codes = rne(127 z / max|z|), scale = f max|z| / 127
//       z = h weight, f = 1 / root for the norm: the root is the same for the whole row and does not touch the codes
//       z = act(x) up, f = 1 for activations that no norm precedes, and for weights
//
// Codes are those of the real numbers: values next to the border between two codes are worked out again in 64 bits (a product of two
// 24-bit numbers is exact there), so codes depend neither on the launch nor on how well fp32 activations are computed.  An element costs four
// operations for that, its code by the magic number, the distance from it and a maximum of those; what is near (7 elements in 10^5; behind an activation one in
// 10^4) is read again.
//
// A row is read once, as 16-byte pieces that its threads hold in registers, and each output is written once: bound by memory, at 5.4 to 6.2 TB/s where a
// large copy reaches 5.2 to 5.9.  us: 118800 x 1536 bf16 norm 123, with the residual 256 (1.46 GB), its codes 93 and 229, quant8 101; 393120 x 128 33 (norm);
// 32760 x 8960 quant8 155 to 179; 13824 x 5120 fp32 quant8 73.  With an activation vector operations bound it: 118800 x 1536 tanh GELU with a factor 185 to 207
// (floor 160), GELU 207 (106).  Few rows: 3.2 to 5.5, a launch.
#include <algorithm>

#include "elem.h"
#include "wave_reduce.h"

namespace dvdq {

namespace {

struct RowArgs {
    const void *x, *second, *weight;                 // second: the residual, or the factor `up`
    void *h, *y;
    int8_t *codes;
    float *scale;
    int32_t *rowsum;
    int64_t x_batch, x_row, s_batch, s_row, h_batch, h_row, y_batch, y_row, c_batch, c_row;
    int64_t first, rows;                             // of this launch's rows; all rows
    uint32_t S, S_mul, S_shift;                      // rows of a batch; row / S = row * S_mul >> 32 + S_shift for rows below 2^31 (S > 1)
    int C, act;
    float eps, share;                                // share: 1 / C
};

struct Code {
    using Raw = int8_t;
};

enum { kNorm = 0, kNormCodes = 1, kQuant = 2, kQuantAct = 3 };   // (kQuantAct: with an activation)
constexpr bool is_norm(int mode) { return mode <= kNormCodes; }

static __device__ __forceinline__ float act32(float z, int act) {
    switch (act) {
        case DVDQ_ACT_SILU: return activate<DVDQ_ACT_SILU>(z);
        case DVDQ_ACT_GELU_TANH: return activate<DVDQ_ACT_GELU_TANH>(z);
        case DVDQ_ACT_GELU: return activate<DVDQ_ACT_GELU>(z);
        default: return z;
    }
}

static __device__ __forceinline__ double act64(double z, int act) {
    switch (act) {
        case DVDQ_ACT_SILU: return z / (1.0 + exp(-z));
        case DVDQ_ACT_GELU_TANH: return z / (1.0 + exp(-1.5957691216057308 * (z + 0.044715 * z * z * z)));
        case DVDQ_ACT_GELU: return 0.5 * z * erfc(z * -0.70710678118654752);
        default: return z;
    }
}

// A row's elements: h or x, and z in 32 and in 64 bits
template <typename E, int MODE>
struct Row {
    using Raw = typename E::Raw;
    static constexpr bool kWide = sizeof(Raw) == 4;
    const Raw *x, *second, *weight;
    Raw *h, *y;
    int8_t *codes;
    int act;
    bool exact;                                      // fp32 holds z as it is: a product of two 16-bit values, or no product

    __device__ __forceinline__ Row(const RowArgs &a, uint32_t row) {
        const int64_t b = a.S == 1 ? row : __umulhi(row, a.S_mul) >> a.S_shift, s = row - (uint32_t)b * a.S;
        x = static_cast<const Raw *>(a.x) + b * a.x_batch + s * a.x_row;
        second = a.second ? static_cast<const Raw *>(a.second) + b * a.s_batch + s * a.s_row : nullptr;
        weight = static_cast<const Raw *>(a.weight);
        h = a.h ? static_cast<Raw *>(a.h) + b * a.h_batch + s * a.h_row : nullptr;
        y = static_cast<Raw *>(a.y) + b * a.y_batch + s * a.y_row;
        codes = a.codes + b * a.c_batch + s * a.c_row;
        act = a.act;
        exact = MODE == kQuantAct ? false : !kWide || !(is_norm(MODE) ? weight : second);
    }
    // the value that z is made of, from memory; summed: h is there already
    __device__ __forceinline__ float value(int c, bool summed) const {
        if (is_norm(MODE) && second) return E::to_f32(summed ? h[c] : E::from_f32(E::to_f32(x[c]) + E::to_f32(second[c])));
        return E::to_f32(x[c]);
    }
    __device__ __forceinline__ float z32(int c, float v) const {
        if (MODE == kQuantAct) v = act32(v, act);
        if (!is_norm(MODE)) return second ? v * E::to_f32(second[c]) : v;
        return weight ? v * E::to_f32(weight[c]) : v;
    }
    __device__ __forceinline__ double z64(int c, float v) const {
        if (!is_norm(MODE)) return (MODE == kQuantAct ? act64(v, act) : (double)v) * (second ? (double)E::to_f32(second[c]) : 1.0);
        return weight ? (double)v * E::to_f32(weight[c]) : (double)v;
    }
    // How far fp32 may have 127 z / max|z| = t off: the quotient 127 / max|z| by 2^-24 of t (twice that where the maximum is not an fp32 number), products by 2^-24, activations by 2^-15 of themselves
    // where they fall like an exponential (see activate).
    __device__ __forceinline__ float margin(float t) const {
        if (MODE != kQuantAct) return exact ? 0x1p-16f : 0x1p-15f;
        return 0x1p-15f + fabsf(t) * 0x1p-15f;
    }
};
// An activation is good to 2^-18 of itself up to where it has fallen to 7.5e-5 (e^-12 times an argument of 12; see activate); beyond, it is that small.
constexpr float kGood = 0x1p-18f, kFallen = 7.5e-5f;
constexpr float kTiny = 0x1p-60f;                    // below, products in fp32 may have lost digits
// An activation below 2^-118 may come out as zero (see activate).  Where the largest of a thread's factors times that is 2^-9 of the row's largest |z|
// (1/4 of a code) or more, fp32 does not know the thread's elements, and all of them are worked out in 64 bits.
static __device__ __forceinline__ bool lost_digits(float up_top, float top) { return up_top * 0x1p-118f > top * 0x1p-9f; }
constexpr float kNearTop = 1.0f - 0x1p-13f;          // what may turn out to be the largest, as a share of the largest in fp32

// Reductions over the T threads of a row (8 to 1024); every thread gets the result.  Beyond a wave through LDS, whose two halves take turns (`turn`).
template <int T, class V, class Op>
static __device__ __forceinline__ V over_row(V v, Op op, uint64_t *lds, int &turn) {
    v = op(v, dpp<DPP_XOR1>(v));
    v = op(v, dpp<DPP_XOR2>(v));
    v = op(v, dpp<DPP_HALF_MIRROR>(v));
    if constexpr (T >= 16) v = op(v, dpp<DPP_MIRROR>(v));
    if constexpr (T >= 32) v = swap_rows<false>(v, op);
    if constexpr (T >= 64) v = swap_rows<true>(v, op);
    if constexpr (T > 64) {
        V *slots = reinterpret_cast<V *>(lds + (turn ^= 16));
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
        __syncthreads();
        V w[T / 64];
#pragma unroll
        for (int i = 0; i < T / 64; ++i) w[i] = slots[i];
        v = w[0];
#pragma unroll
        for (int i = 1; i < T / 64; ++i) v = op(v, w[i]);
    }
    return v;
}
struct Add {
    template <class V>
    __device__ V operator()(V a, V b) const { return a + b; }
};
struct Larger {
    template <class V>
    __device__ V operator()(V a, V b) const { return a > b ? a : b; }
};

// What becomes of a row once its largest |z| is known in fp32
struct Scale {
    double top;      // max|z|
    float reach;     // 127 / top
    bool fine, tiny; // no NaN or infinity; products may have lost digits
};
static __device__ __forceinline__ float scale_of(const Scale &s, float factor) {
    return !s.fine ? __builtin_nanf("") : s.top > 0.0 ? (float)(s.top * (1.0 / 127.0) * factor) : 0.0f;   // one rounding
}
static __device__ __forceinline__ Scale scale_from(uint32_t top_bits) {
    const float top = __builtin_bit_cast(float, top_bits);
    return {(double)top, 0.0f, top_bits < 0x7F800000u, top < kTiny};
}

// 16 bytes of a row as four words, which stay four registers also where branches meet (as an array of elements each has a register).
template <typename E>
static __device__ __forceinline__ uint4 load_words(const typename E::Raw *p, int n, bool whole_before) {
    constexpr int kBytes = sizeof(typename E::Raw);
    if (n >= E::kVec) return __builtin_bit_cast(uint4, *reinterpret_cast<const Piece<E> *>(p));
    return load_end<kBytes>(reinterpret_cast<const uint8_t *>(p), n * kBytes, whole_before);
}
static __device__ __forceinline__ uint32_t word_of(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
template <typename E>
static __device__ __forceinline__ float element(const uint4 &v, int e) {
    if constexpr (E::kVec == 8) return E::to_f32((uint16_t)(word_of(v, e / 2) >> 16 * (e % 2)));
    else return __builtin_bit_cast(float, word_of(v, e));
}
template <typename E>
static __device__ __forceinline__ uint4 rounded(const float (&v)[E::kVec]) {
    if constexpr (E::kVec == 8) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = E::from_f32(v[2 * i]) | (uint32_t)E::from_f32(v[2 * i + 1]) << 16;
        return make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        return __builtin_bit_cast(uint4, v);
    }
}
template <typename E>
static __device__ __forceinline__ void store_words(typename E::Raw *p, const uint4 &v, int n) {
    constexpr int V = E::kVec;
    if (n >= V) {
        *reinterpret_cast<Piece<E> *>(p) = __builtin_bit_cast(Piece<E>, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e < n) {
            if constexpr (V == 8) p[e] = (uint16_t)(word_of(v, e / 2) >> 16 * (e % 2));
            else p[e] = element<E>(v, e);
        }
}

// the larger of |a|, |b| and c; NaN if one of them is
static __device__ __forceinline__ float maximum3(float a, float b, float c) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(a), fabsf(b)), c);
}
template <typename E, int ACT, int NP, int V>
static __device__ __forceinline__ void activate_all(float (&z)[NP][V], const uint4 (&x)[NP]) {
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) z[i][e] = activate<ACT>(element<E>(x[i], e));
}

// T threads a row, which they hold: NP pieces of 16 bytes each.
template <typename E, int MODE, int T, int NP>
__global__ __launch_bounds__(T < 256 ? 256 : T) void row_held(RowArgs a) {
    constexpr int V = E::kVec, R = T < 256 ? 256 / T : 1;
    // the row's end lies in a thread's last piece, or where not every number of pieces has a kernel, in its last two
    constexpr int kWhole = T == 64 || (T == 256 && NP < 8) ? NP - 1 : std::max(NP - 2, 0);
    __shared__ uint64_t lds[32];
    int turn = 0;
    const int l = threadIdx.x % T;
    const int64_t mine = a.first + (int64_t)blockIdx.x * R + threadIdx.x / T;
    const bool there = R == 1 || mine < a.rows;
    uint32_t row = (uint32_t)(there ? mine : a.rows - 1);
    if (T >= 64) row = __builtin_amdgcn_readfirstlane(row);
    const Row<E, MODE> r(a, row);
    const bool long_row = a.C >= V;
    uint4 px[NP], ps[NP], pw[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int c = (l + T * i) * V, n = i < kWhole ? V : a.C - c;
        px[i] = load_words<E>(r.x + c, n, long_row);
        if (r.second) ps[i] = load_words<E>(r.second + c, n, long_row);
        if (is_norm(MODE) && r.weight) pw[i] = load_words<E>(r.weight + c, n, long_row);
    }
    float z[NP][V], sum = 0.0f, top = 0.0f, up_top = 0.0f;
    if constexpr (MODE == kQuantAct) {
        switch (a.act) {
            case DVDQ_ACT_SILU: activate_all<E, DVDQ_ACT_SILU>(z, px); break;
            case DVDQ_ACT_GELU_TANH: activate_all<E, DVDQ_ACT_GELU_TANH>(z, px); break;
            default: activate_all<E, DVDQ_ACT_GELU>(z, px);
        }
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int c = (l + T * i) * V, n = i < kWhole ? V : a.C - c;
        if (is_norm(MODE)) {
            if (r.second) {
                float v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = element<E>(px[i], e) + element<E>(ps[i], e);
                px[i] = rounded<E>(v);
                if (there) store_words<E>(r.h + c, px[i], n);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                z[i][e] = element<E>(px[i], e);
                sum = fmaf(z[i][e], z[i][e], sum);
            }
            if (r.weight)
#pragma unroll
                for (int e = 0; e < V; ++e) z[i][e] *= element<E>(pw[i], e);
        } else {
            if (MODE == kQuant)
#pragma unroll
                for (int e = 0; e < V; ++e) z[i][e] = element<E>(px[i], e);
            if (r.second)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float up = element<E>(ps[i], e);
                    if (MODE == kQuantAct) up_top = fmaxf(up_top, fabsf(up));
                    z[i][e] *= up;
                }
        }
        if (MODE != kNorm)
#pragma unroll
            for (int e = 0; e < V; e += 2) top = maximum3(z[i][e], z[i][e + 1], top);
    }
    float factor = 1.0f;
    if (is_norm(MODE)) factor = rsqrtf(fmaf(over_row<T>(sum, Add(), lds, turn), a.share, a.eps));
    if (MODE == kNorm) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (l + T * i) * V, n = i < kWhole ? V : a.C - c;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = z[i][e] * factor;
            if (there) store_words<E>(r.y + c, rounded<E>(v), n);
        }
        return;
    }
    // Which of a thread's elements need a second look: bit V i + e.  That goes by the values in memory, so that there is one place for it.
    static_assert(NP * V <= 64, "a bit each");
    using Mask = std::conditional_t<NP * V <= 32, uint32_t, uint64_t>;
    const auto place = [&](Mask which) {
        const int bit = sizeof(Mask) == 4 ? __builtin_ctz((uint32_t)which) : __builtin_ctzll(which);
        return (l + T * (bit / V)) * V + bit % V;
    };
    Scale s = scale_from(over_row<T>(__builtin_bit_cast(uint32_t, top) & 0x7FFFFFFFu, Larger(), lds, turn));   // (a NaN's bits are above infinity's)
    const bool wide = s.tiny || (MODE == kQuantAct && lost_digits(up_top, (float)s.top));   // (up_top is 0 where there is no factor)
    if (!r.exact || s.tiny) {
        double t = 0.0;
        if (s.fine) {
            const float near = wide ? 0.0f : (float)s.top * kNearTop;
            Mask which = 0;
            if (top >= near)
#pragma unroll
                for (int i = 0; i < NP; ++i)
#pragma unroll
                    for (int e = 0; e < V; ++e) which |= (Mask)(fabsf(z[i][e]) >= near ? 1 : 0) << (V * i + e);
            for (; which; which &= which - 1) {
                const int c = place(which);
                if (c < a.C) t = Larger()(t, fabs(r.z64(c, r.value(c, true))));
            }
        }
        t = over_row<T>(t, Larger(), lds, turn);
        if (s.fine) s.top = t;
    }
    s.reach = s.top > 0.0 ? 127.0f / (float)s.top : 0.0f;
    int total = 0;
    float far = 0.0f;                            // the furthest that t is from a whole number
    constexpr float kMagic = 12582912.0f;        // 1.5 2^23: t + that has the whole number next to t in its lowest bits
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int c = (l + T * i) * V, n = i < kWhole ? V : a.C - c;
        uint32_t m[V], word[V / 4];
        float off[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float t = fmaf(z[i][e], s.reach, kMagic), q = t - kMagic;
            m[e] = __builtin_bit_cast(uint32_t, t);
            off[e] = fabsf(fmaf(z[i][e], s.reach, -q));
            if (MODE == kQuantAct) off[e] = fmaf(fabsf(q), kGood, off[e]);
        }
#pragma unroll
        for (int e = 0; e < V; e += 2) far = maximum3(off[e], off[e + 1], far);
#pragma unroll
        for (int w = 0; w < V / 4; ++w) {
            word[w] = __builtin_amdgcn_perm(m[4 * w + 1], m[4 * w], 0x0C0C0400u) | __builtin_amdgcn_perm(m[4 * w + 3], m[4 * w + 2], 0x04000C0Cu);
            if (!s.fine) word[w] = 0;
            if (a.rowsum) total = __builtin_amdgcn_sdot4((int)word[w], 0x01010101, total, false);
        }
        Piece<Code, V> o;
        __builtin_memcpy(&o, word, V);
        if (there) store_piece<Code, V>(r.codes + c, o, n);
    }
    // (a part that is not there is z = 0)
    const bool fallen = MODE == kQuantAct && (r.second ? up_top : 1.0f) * kFallen * s.reach > 0.25f;
    if (s.fine && s.top > 0.0 && (wide || fallen || far > 0.5f - (r.exact ? 0x1p-16f : 0x1p-15f))) {
        Mask near = 0;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float t = z[i][e] * s.reach;
                near |= (Mask)(wide || fabsf(t - rintf(t)) > 0.5f - r.margin(t) ? 1 : 0) << (V * i + e);
            }
        for (; near; near &= near - 1) {
            const int c = place(near);
            if (c >= a.C) break;
            const int code = (int)rint(127.0 * r.z64(c, r.value(c, true)) / s.top);
            if (there) {
                total += code - r.codes[c];
                r.codes[c] = (int8_t)code;
            }
        }
    }
    if (a.rowsum) {
        total = over_row<T>(total, Add(), lds, turn);
        if (l == 0 && there) a.rowsum[row] = total;
    }
    if (l == 0 && there) a.scale[row] = scale_of(s, factor);
}

// Longer rows: a workgroup per row, which it reads again for each step.
template <typename E, int MODE>
__global__ __launch_bounds__(1024) void row_long(RowArgs a) {
    constexpr int T = 1024, V = E::kVec;
    __shared__ uint64_t lds[32];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const Row<E, MODE> r(a, (uint32_t)row);
        float up_top = 0.0f;
        // the values and z of the n elements from c on, zero past them
        const auto piece = [&](int c, int n, float (&v)[V], float (&z)[V]) {
            const uint4 px = load_words<E>(r.x + c, n, true);
            uint4 ps = {}, pw = {};
            if (r.second) ps = load_words<E>(r.second + c, n, true);
            if (is_norm(MODE) && r.weight) pw = load_words<E>(r.weight + c, n, true);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[e] = element<E>(px, e);
                if (is_norm(MODE)) {
                    if (r.second) v[e] = E::to_f32(E::from_f32(v[e] + element<E>(ps, e)));
                    z[e] = r.weight ? v[e] * element<E>(pw, e) : v[e];
                } else {
                    z[e] = MODE == kQuantAct ? act32(v[e], a.act) : v[e];
                    if (r.second) z[e] *= element<E>(ps, e);
                    if (MODE == kQuantAct && r.second) up_top = fmaxf(up_top, fabsf(element<E>(ps, e)));
                }
            }
        };
        float v[V], z[V], sum = 0.0f, top = 0.0f;
        for (int c = threadIdx.x * V; c < a.C; c += T * V) {
            piece(c, a.C - c, v, z);
            if (is_norm(MODE))
#pragma unroll
                for (int e = 0; e < V; ++e) sum = fmaf(v[e], v[e], sum);
            if (MODE != kNorm)
#pragma unroll
                for (int e = 0; e < V; e += 2) top = maximum3(z[e], z[e + 1], top);
        }
        float factor = 1.0f;
        if (is_norm(MODE)) factor = rsqrtf(fmaf(over_row<T>(sum, Add(), lds, turn), a.share, a.eps));
        Scale s = {};
        bool wide = false;
        if (MODE != kNorm) {
            s = scale_from(over_row<T>(__builtin_bit_cast(uint32_t, top) & 0x7FFFFFFFu, Larger(), lds, turn));
            wide = s.tiny || (MODE == kQuantAct && lost_digits(up_top, (float)s.top));
            if (!r.exact || s.tiny) {
                const float near = wide ? 0.0f : (float)s.top * kNearTop;
                double t = 0.0;
                if (s.fine && top >= near)
                    for (int c = threadIdx.x * V; c < a.C; c += T * V)
#pragma unroll 1
                        for (int at = c; at < min(c + V, a.C); ++at) {
                            const float value = r.value(at, false);
                            if (fabsf(r.z32(at, value)) >= near) t = Larger()(t, fabs(r.z64(at, value)));
                        }
                t = over_row<T>(t, Larger(), lds, turn);
                if (s.fine) s.top = t;
            }
            s.reach = s.top > 0.0 ? 127.0f / (float)s.top : 0.0f;
        }
        int total = 0;
        for (int c = threadIdx.x * V; c < a.C; c += T * V) {
            const int n = a.C - c;
            piece(c, n, v, z);
            if (is_norm(MODE) && r.h) store_words<E>(r.h + c, rounded<E>(v), n);
            if (MODE == kNorm) {
#pragma unroll
                for (int e = 0; e < V; ++e) z[e] *= factor;
                store_words<E>(r.y + c, rounded<E>(z), n);
                continue;
            }
            uint32_t near = 0;
            Piece<Code, V> o;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float t = z[e] * s.reach, q = rintf(t);
                near |= (wide || fabsf(t - q) > 0.5f - r.margin(t) ? 1u : 0u) << e;
                o.e[e] = s.fine ? (int8_t)(int)q : 0;
                total += o.e[e];
            }
            store_piece<Code, V>(r.codes + c, o, n);
            if (s.fine && s.top > 0.0)
                for (; near; near &= near - 1) {
                    const int at = c + __builtin_ctz(near);
                    if (at >= a.C) break;
                    const int code = (int)rint(127.0 * r.z64(at, r.value(at, true)) / s.top);
                    total += code - r.codes[at];
                    r.codes[at] = (int8_t)code;
                }
        }
        if (MODE != kNorm) {
            if (a.rowsum) {
                total = over_row<T>(total, Add(), lds, turn);
                if (threadIdx.x == 0) a.rowsum[row] = total;
            }
            if (threadIdx.x == 0) a.scale[row] = scale_of(s, factor);
        }
    }
}

template <typename E, int MODE>
int launch_held(const RowArgs &a, hipStream_t stream) {
    const int pieces = (a.C + E::kVec - 1) / E::kVec;
    const auto launch = [&](auto t, auto np) {
        constexpr int T = decltype(t)::value, NP = decltype(np)::value, R = T < 256 ? 256 / T : 1;
        // (a launch has less than 2^32 threads; a loop in the kernel instead costs it 20 registers of constants)
        for (RowArgs part = a; part.first < a.rows; part.first += (int64_t)R << 21) {
            const int64_t workgroups = std::min<int64_t>((a.rows - part.first + R - 1) / R, 1 << 21);
            row_held<E, MODE, T, NP><<<dim3((unsigned)workgroups), T < 256 ? 256 : T, 0, stream>>>(part);
            const int rc = check_launch();
            if (rc != DVDQ_OK) return rc;
        }
        return (int)DVDQ_OK;
    };
    using std::integral_constant;
    // As few threads as hold the row in registers, up to 8 pieces each: no exchange through LDS up to 256 pieces, and more rows at once on a
    // compute unit.  32760 x 8960 bf16 with 256 threads of 5 pieces against 512 of 3, us: norm 203 and 199, its codes 163 and 216, quant8 179 and 188,
    // gated 323 and 424; 32760 x 13824 fp32 with 512 threads of 8 against 1024 of 4: 617 and 622, 509 and 669, 392 and 390, 835 and 915;
    // 3000 x 30000 bf16 74 and 72, 83 and 73, 81 and 69, 146 and 130.  Longer rows are read again: 3000 x 30000 fp32 187, 227, 138, 358.
    if (pieces <= 8) return launch(integral_constant<int, 8>(), integral_constant<int, 1>());
    if (pieces <= 16) return launch(integral_constant<int, 16>(), integral_constant<int, 1>());
    if (pieces <= 32) return launch(integral_constant<int, 32>(), integral_constant<int, 1>());
    const integral_constant<int, 64> wave;
    if (pieces <= 64) return launch(wave, integral_constant<int, 1>());
    if (pieces <= 128) return launch(wave, integral_constant<int, 2>());
    if (pieces <= 192) return launch(wave, integral_constant<int, 3>());
    if (pieces <= 256) return launch(wave, integral_constant<int, 4>());
    const integral_constant<int, 256> four;
    if (pieces <= 512) return launch(four, integral_constant<int, 2>());
    if (pieces <= 768) return launch(four, integral_constant<int, 3>());
    if (pieces <= 1024) return launch(four, integral_constant<int, 4>());
    if (pieces <= 1280) return launch(four, integral_constant<int, 5>());
    if (pieces <= 1536) return launch(four, integral_constant<int, 6>());
    if (pieces <= 2048) return launch(four, integral_constant<int, 8>());
    if constexpr (E::kVec == 8) {
        if (pieces <= 4096) return launch(integral_constant<int, 1024>(), integral_constant<int, 4>());
    } else {
        if (pieces <= 6 * 512) return launch(integral_constant<int, 512>(), integral_constant<int, 6>());
        if (pieces <= 8 * 512) return launch(integral_constant<int, 512>(), integral_constant<int, 8>());
    }
    row_long<E, MODE><<<dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), 1024, 0, stream>>>(a);
    return check_launch();
}

template <int MODE>
int launch_rows(RowArgs a, int dtype, hipStream_t stream) {
    if (a.S > 1) {                                   // 2^(31 + l) / S rounded up, 2^l >= S
        int l = 1;
        while (((uint64_t)1 << l) < a.S) ++l;
        a.S_mul = (uint32_t)((((uint64_t)1 << (31 + l)) + a.S - 1) / a.S), a.S_shift = l - 1;
    }
    return with_type(dtype, [&](auto type) {
        using E = decltype(type);
        return launch_held<E, MODE>(a, stream);
    });
}

}  // namespace

int launch_rms_norm(const void *x, int64_t B, int64_t S, int64_t C, int64_t x_batch, int64_t x_row, const void *residual, int64_t r_batch,
                    int64_t r_row, void *h, int64_t h_batch, int64_t h_row, const void *weight, float eps, int dtype, void *y, int64_t y_batch,
                    int64_t y_row, int8_t *codes, int64_t c_batch, int64_t c_row, float *x_scale, int32_t *code_rowsum, hipStream_t stream) {
    RowArgs a = {};
    a.x = x, a.second = residual, a.weight = weight, a.h = h, a.y = y;
    a.codes = codes, a.scale = x_scale, a.rowsum = code_rowsum;
    a.x_batch = x_batch, a.x_row = x_row, a.s_batch = r_batch, a.s_row = r_row, a.h_batch = h_batch, a.h_row = h_row;
    a.y_batch = y_batch, a.y_row = y_row, a.c_batch = c_batch, a.c_row = c_row;
    a.rows = B * S, a.S = (uint32_t)S, a.C = (int)C, a.eps = eps, a.share = 1.0f / (float)C;
    return y ? launch_rows<kNorm>(a, dtype, stream) : launch_rows<kNormCodes>(a, dtype, stream);
}

int launch_quant8(const void *x, int64_t ldx, const void *up, int64_t ldu, int act, int64_t M, int64_t C, int dtype, int8_t *codes, int64_t ldc,
                  float *x_scale, int32_t *code_rowsum, hipStream_t stream) {
    RowArgs a = {};
    a.x = x, a.second = up;
    a.codes = codes, a.scale = x_scale, a.rowsum = code_rowsum;
    a.x_row = ldx, a.s_row = ldu, a.c_row = ldc;
    a.rows = M, a.S = (uint32_t)M, a.C = (int)C, a.act = act;
    return act == DVDQ_ACT_NONE ? launch_rows<kQuant>(a, dtype, stream) : launch_rows<kQuantAct>(a, dtype, stream);
}

}  // namespace dvdq
