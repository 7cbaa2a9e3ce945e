// Rows normed by their root mean square, with the residual's addition, and rows to 8 bits with a scale each:
//
//   h = T(x + residual)        rounded to the tensors' type T (x itself without a residual)
//   y = T(h weight / root)     root = sqrt(mean h^2 + eps)
//   codes = rne(127 z / max|z|), scale = f max|z| / 127
//       z = h weight, f = 1 / root for the norm: the root is the same for the whole row and does not touch the codes
//       z = act(x) up, f = 1 for activations that no norm precedes, and for weights
//
// Codes are those of the real numbers: values next to the border between two codes are worked out again in 64 bits (a product of two
// 24-bit numbers is exact there), so codes depend neither on the launch nor on how well fp32 activations are computed.
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
    int64_t rows;
    uint32_t S;                                      // rows of a batch
    int C, act;
    float eps;
};

enum { kNorm = 0, kNormCodes = 1, kQuant = 2 };

static __device__ __forceinline__ float act32(float z, int act) {
    switch (act) {
        case DVDQ_ACT_SILU: return activate<DVDQ_ACT_SILU>(z);
        case DVDQ_ACT_GELU_TANH: return activate<DVDQ_ACT_GELU_TANH>(z);
        case DVDQ_ACT_GELU: return activate<DVDQ_ACT_GELU>(z);
        default: return z;
    }
}

static __device__ __noinline__ double act64(double z, int act) {
    switch (act) {
        case DVDQ_ACT_SILU: return z / (1.0 + exp(-z));
        case DVDQ_ACT_GELU_TANH: return z / (1.0 + exp(-1.5957691216057308 * (z + 0.044715 * z * z * z)));
        case DVDQ_ACT_GELU: return 0.5 * z * erfc(z * -0.70710678118654752);
        default: return z;
    }
}

// Reductions over a workgroup; every thread gets the result.
template <class T, class Op>
static __device__ __forceinline__ T all(T v, T *lds, Op op) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v = op(v, __shfl_xor(v, m));
    const int waves = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int i = 1; i < waves; ++i) v = op(v, lds[i]);
    __syncthreads();
    return v;
}

// A workgroup per row, which it reads again for each step.
template <typename E, int MODE>
__global__ __launch_bounds__(256) void row_any(RowArgs a) {
    using Raw = typename E::Raw;
    constexpr bool WIDE = sizeof(Raw) == 4;
    __shared__ double lds[4];
    const auto add = [](auto p, auto q) { return p + q; };
    const auto larger = [](auto p, auto q) { return p > q ? p : q; };
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t b = (uint32_t)row / a.S, s = (uint32_t)row % a.S;
        const Raw *x = static_cast<const Raw *>(a.x) + b * a.x_batch + s * a.x_row;
        const Raw *second = a.second ? static_cast<const Raw *>(a.second) + b * a.s_batch + s * a.s_row : nullptr;
        const Raw *weight = static_cast<const Raw *>(a.weight);
        const bool plain = MODE == kQuant && a.act == DVDQ_ACT_NONE;
        // whether fp32 holds z as it is: a product of two 16-bit values, or no product
        const bool exact = MODE == kQuant ? plain && (!WIDE || !second) : !WIDE || !weight;
        auto value = [&](int c) {
            float v = E::to_f32(x[c]);
            if (MODE != kQuant && second) v = E::to_f32(E::from_f32(v + E::to_f32(second[c])));
            return v;
        };
        auto z32 = [&](int c, float v) {
            if (MODE == kQuant) return act32(v, a.act) * (second ? E::to_f32(second[c]) : 1.0f);
            return weight ? v * E::to_f32(weight[c]) : v;
        };
        auto z64 = [&](int c, float v) {
            if (MODE == kQuant) return act64(v, a.act) * (second ? (double)E::to_f32(second[c]) : 1.0);
            return weight ? (double)v * E::to_f32(weight[c]) : (double)v;
        };
        float sum = 0.0f;
        uint32_t top_bits = 0;
        for (int c = threadIdx.x; c < a.C; c += 256) {
            const float v = value(c);
            if (MODE != kQuant) sum += v * v;
            if (MODE != kNorm) top_bits = max(top_bits, __builtin_bit_cast(uint32_t, z32(c, v)) & 0x7FFFFFFFu);   // (a NaN is above infinity)
        }
        float factor = 1.0f;
        if (MODE != kQuant) factor = 1.0f / sqrtf(all(sum, reinterpret_cast<float *>(lds), add) / (float)a.C + a.eps);
        double top = 0.0;
        bool fine = true, tiny = false;
        if (MODE != kNorm) {
            top_bits = all(top_bits, reinterpret_cast<uint32_t *>(lds), larger);
            const float top32 = __builtin_bit_cast(float, top_bits);
            fine = top_bits < 0x7F800000u;
            top = top32;
            tiny = top32 < 0x1p-60f;                 // (products of small numbers: fp32 may have lost digits)
            if (fine && (!exact || tiny)) {
                const float near = tiny ? 0.0f : top32 * (1.0f - 0x1p-13f);
                double t = 0.0;
                for (int c = threadIdx.x; c < a.C; c += 256) {
                    const float v = value(c);
                    if (fabsf(z32(c, v)) >= near) t = larger(t, fabs(z64(c, v)));
                }
                top = all(t, lds, larger);
            }
        }
        const float reach = top > 0.0 ? (float)(127.0 / top) : 0.0f;
        int codes = 0;
        for (int c = threadIdx.x; c < a.C; c += 256) {
            const float v = value(c);
            if (MODE != kQuant && a.h) static_cast<Raw *>(a.h)[b * a.h_batch + s * a.h_row + c] = E::from_f32(v);
            if (MODE == kNorm) {
                static_cast<Raw *>(a.y)[b * a.y_batch + s * a.y_row + c] = E::from_f32(weight ? v * factor * E::to_f32(weight[c]) : v * factor);
            } else {
                const float t = z32(c, v) * reach;
                float q = rintf(t);
                if (fine && top > 0.0 && (tiny || fabsf(t - q) > 0.5f - 0x1p-14f - fabsf(t) * 0x1p-15f)) q = (float)rint(127.0 * z64(c, v) / top);
                const int code = fine ? (int)q : 0;
                a.codes[b * a.c_batch + s * a.c_row + c] = (int8_t)code;
                codes += code;
            }
        }
        if (MODE != kNorm) {
            if (a.rowsum) {
                const int total = all(codes, reinterpret_cast<int *>(lds), add);
                if (threadIdx.x == 0) a.rowsum[row] = total;
            }
            if (threadIdx.x == 0) a.scale[row] = !fine ? __builtin_nanf("") : top > 0.0 ? (float)(top / 127.0) * factor : 0.0f;
        }
    }
}

template <int MODE>
int launch_rows(const RowArgs &a, int dtype, hipStream_t stream) {
    return with_type(dtype, [&](auto type) {
        using E = decltype(type);
        row_any<E, MODE><<<dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), 256, 0, stream>>>(a);
        return check_launch();
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
    a.rows = B * S, a.S = (uint32_t)S, a.C = (int)C, a.eps = eps;
    return y ? launch_rows<kNorm>(a, dtype, stream) : launch_rows<kNormCodes>(a, dtype, stream);
}

int launch_quant8(const void *x, int64_t ldx, const void *up, int64_t ldu, int act, int64_t M, int64_t C, int dtype, int8_t *codes, int64_t ldc,
                  float *x_scale, int32_t *code_rowsum, hipStream_t stream) {
    RowArgs a = {};
    a.x = x, a.second = up;
    a.codes = codes, a.scale = x_scale, a.rowsum = code_rowsum;
    a.x_row = ldx, a.s_row = ldu, a.c_row = ldc;
    a.rows = M, a.S = (uint32_t)M, a.C = (int)C, a.act = act;
    return launch_rows<kQuant>(a, dtype, stream);
}

}  // namespace dvdq
