// C ABI of the operators around the quantized layer: argument validation on the host, then kernel launches.
#include "dvdq_internal.h"
#include "../../include/dvdq_bench.h"

namespace {

constexpr int64_t kMaxInt = 0x7FFFFFFF;
constexpr int64_t kMaxTokens = (int64_t)1 << 23, kMaxChannels = (int64_t)1 << 22, kMaxPitch = (int64_t)1 << 26;   // what a launch's grid and 32-bit indices hold

inline bool aligned_to(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline size_t element_bytes(int dtype) { return dtype == DVDQ_FP32 ? 4 : 2; }

int check_heads(const dvdq_rope_heads *h, int64_t B, int64_t T, int dtype) {
    if (!h->in || !h->out) return DVDQ_ERR_NULL;
    if (h->heads < 1) return DVDQ_ERR_SHAPE;
    if (h->heads > 65536) return DVDQ_ERR_UNSUPPORTED;
    const int64_t size[3] = {B, T, h->heads};
    for (int i = 0; i < 3; ++i) {
        if (size[i] > 1 && h->out_stride[i] == 0) return DVDQ_ERR_UNSUPPORTED;
        if (size[i] > 1 && h->in == h->out && h->in_stride[i] != h->out_stride[i]) return DVDQ_ERR_UNSUPPORTED;
    }
    if (!aligned_to(h->in, element_bytes(dtype)) || !aligned_to(h->out, element_bytes(dtype))) return DVDQ_ERR_ALIGN;
    return DVDQ_OK;
}

}  // namespace

extern "C" {

int dvdq_rope_table(const double *freq, int64_t n_pos, int64_t half, double magnitude, float *table, void *hip_stream) {
    if (!freq || !table) return DVDQ_ERR_NULL;
    if (n_pos < 1 || half < 1) return DVDQ_ERR_SHAPE;
    if (half > 512 || n_pos > ((int64_t)1 << 31) / half) return DVDQ_ERR_UNSUPPORTED;
    if (!aligned_to(freq, 16) || !aligned_to(table, 16)) return DVDQ_ERR_ALIGN;
    return dvdq::launch_rope_table(freq, n_pos, half, magnitude, table, static_cast<hipStream_t>(hip_stream));
}

int dvdq_rope(const dvdq_rope_heads *q, const dvdq_rope_heads *k, int64_t B, int64_t T, int64_t head_dim, const float *table,
              int64_t n_pos, int64_t rot_dim, const int32_t *positions, int64_t pos_batch, int n_axes, const int32_t *sections,
              int flags, int dtype, void *hip_stream) {
    if (!q || (n_axes > 1 && !sections)) return DVDQ_ERR_NULL;
    if (B < 0 || T < 0 || head_dim < 1 || n_pos < 1 || rot_dim < 2 || rot_dim % 2 || rot_dim > head_dim || n_axes < 1 || pos_batch < 0)
        return DVDQ_ERR_SHAPE;
    if (head_dim > 1024 || n_axes > 4 || n_pos > kMaxInt || (flags & ~(DVDQ_ROPE_INTERLEAVED | DVDQ_ROPE_INVERSE)) ||
        dtype < DVDQ_BF16 || dtype > DVDQ_FP32)
        return DVDQ_ERR_UNSUPPORTED;
    if (sections) {
        int64_t sum = 0;
        for (int i = 0; i < n_axes; ++i) {
            if (sections[i] < 0 || sections[i] % 2) return DVDQ_ERR_SHAPE;
            sum += sections[i];
        }
        if (sum != rot_dim) return DVDQ_ERR_SHAPE;
    }
    if (B == 0 || T == 0) return DVDQ_OK;
    if (B > kMaxTokens || T > kMaxTokens / B || pos_batch > kMaxInt) return DVDQ_ERR_UNSUPPORTED;
    if (!table || !positions) return DVDQ_ERR_NULL;
    if (pos_batch != 0 && pos_batch < T * n_axes) return DVDQ_ERR_SHAPE;
    for (const dvdq_rope_heads *h : {q, k}) {
        const int rc = h ? check_heads(h, B, T, dtype) : DVDQ_OK;
        if (rc != DVDQ_OK) return rc;
    }
    if (!aligned_to(table, 16) || !aligned_to(positions, 4)) return DVDQ_ERR_ALIGN;
    return dvdq::launch_rope(q, k, B, T, head_dim, table, n_pos, rot_dim, positions, pos_batch, n_axes, sections,
                             (flags & DVDQ_ROPE_INTERLEAVED) != 0, (flags & DVDQ_ROPE_INVERSE) != 0, dtype,
                             static_cast<hipStream_t>(hip_stream));
}

size_t dvdq_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (M < 1 || N < 1 || K < 1 || M > kMaxTokens || N > kMaxChannels || K > kMaxChannels) return 0;
    return dvdq::linear_workspace_bytes(M, N, K);
}

int dvdq_linear(const void *x, int64_t ldx, const void *w, int64_t ldw, const void *bias, int act, const void *gate,
                int64_t gate_rows, int64_t ldg, const void *residual, int64_t ldr, int64_t M, int64_t N, int64_t K, int dtype, void *y,
                int64_t ldy, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (M < 0 || N < 1 || K < 1) return DVDQ_ERR_SHAPE;
    if (M == 0) return DVDQ_OK;
    if (!x || !w || !y) return DVDQ_ERR_NULL;
    if (gate && (gate_rows < 1 || M % gate_rows)) return DVDQ_ERR_SHAPE;
    if ((M > 1 && (ldx < K || ldy < N || (residual && ldr < N))) || (N > 1 && ldw < K) || (gate && gate_rows > 1 && ldg < N))
        return DVDQ_ERR_SHAPE;
    if (M > kMaxTokens || N > kMaxChannels || K > kMaxChannels || act < DVDQ_ACT_NONE || act > DVDQ_ACT_GELU || (dtype != DVDQ_BF16 && dtype != DVDQ_FP16) ||
        (residual == y && M > 1 && ldr != ldy) || (M > 1 && (ldy > kMaxPitch || (residual && ldr > kMaxPitch))))
        return DVDQ_ERR_UNSUPPORTED;
    // operands of which other outputs still need what an output would overwrite
    if (y == x || y == w || (y == bias && M > 1) || (y == gate && (gate_rows != M || (M > 1 && ldg != ldy)))) return DVDQ_ERR_UNSUPPORTED;
    for (const void *p : {x, w, bias, gate, residual, static_cast<const void *>(y)})
        if (!aligned_to(p, 2)) return DVDQ_ERR_ALIGN;
    const size_t need = dvdq::linear_workspace_bytes(M, N, K);
    if (need) {
        if (!workspace) return DVDQ_ERR_NULL;
        if (!aligned_to(workspace, 16)) return DVDQ_ERR_ALIGN;
        if (workspace_bytes < need) return DVDQ_ERR_WORKSPACE;
    }
    return dvdq::launch_linear(x, ldx, w, ldw, bias, act, gate, gate_rows, ldg, residual, ldr, M, N, K, dtype, y, ldy, workspace,
                               static_cast<hipStream_t>(hip_stream));
}

int dvdq_bench_linear_choice(int64_t M, int64_t N, int64_t K, int any) {
    if (M < 1 || N < 1 || K < 1 || M > kMaxTokens || N > kMaxChannels || K > kMaxChannels) return -2;
    return dvdq::linear_choice(M, N, K, any || K % 8 != 0);
}

size_t dvdq_group_norm_workspace_bytes(int64_t B, int64_t S, int64_t C, int64_t groups) {
    if (B < 1 || S < 1 || C < 1 || groups < 1 || C % groups || C > 4096 || B > 65535) return 0;
    return dvdq::group_norm_workspace_bytes(B, S, C, groups);
}

int dvdq_group_norm(const void *x, int64_t B, int64_t S, int64_t C, int64_t x_batch, int64_t x_row, int64_t groups,
                    const void *weight, const void *bias, float eps, int act, int dtype, void *y, int64_t y_batch, int64_t y_row,
                    void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (B < 0 || S < 0 || C < 1 || groups < 1 || C % groups || !(eps >= 0.0f)) return DVDQ_ERR_SHAPE;
    if (C > 4096 || B > 65535 || (act != DVDQ_ACT_NONE && act != DVDQ_ACT_SILU) || dtype < DVDQ_BF16 || dtype > DVDQ_FP32)
        return DVDQ_ERR_UNSUPPORTED;
    if (B == 0 || S == 0) return DVDQ_OK;
    if (!x || !y || !workspace) return DVDQ_ERR_NULL;
    if (S > 1 && (x_row < C || y_row < C)) return DVDQ_ERR_SHAPE;
    if ((B > 1 && y_batch == 0) || (x == y && ((S > 1 && x_row != y_row) || (B > 1 && x_batch != y_batch)))) return DVDQ_ERR_UNSUPPORTED;
    for (const void *p : {x, weight, bias, static_cast<const void *>(y)})
        if (!aligned_to(p, element_bytes(dtype))) return DVDQ_ERR_ALIGN;
    if (!aligned_to(workspace, 16)) return DVDQ_ERR_ALIGN;
    if (workspace_bytes < dvdq::group_norm_workspace_bytes(B, S, C, groups)) return DVDQ_ERR_WORKSPACE;
    return dvdq::launch_group_norm(x, B, S, C, x_batch, x_row, groups, weight, bias, eps, act, dtype, y, y_batch, y_row, workspace,
                                   static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
