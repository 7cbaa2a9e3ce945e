// Matrix product of 16-bit activations and weights with its epilogue:
//
//   y[m, n] = residual[m, n] + gate[m / (M / G), n] * act(sum_k x[m, k] w[n, k] + bias[n])
//
// Products on the matrix cores, sums and epilogue in fp32, one rounding to the tensors' type.
#include "elem.h"
#include "gemm_common.h"

namespace dvdq {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

template <typename E>
static __device__ __forceinline__ v4f mfma(uint4 a, uint4 b, v4f c) {
    if constexpr (std::is_same<E, Bf16>::value)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

struct LinearArgs {
    const uint16_t *x, *w, *bias, *gate, *residual;
    uint16_t *y;
    int64_t ldx, ldw, ldr, ldy, ldg;   // elements between rows
    int M, N, K;
    int gate_rows;                     // tokens of one row of the gate
    int act;
};

// Bias, activation, gate, residual and store of 8 consecutive channels of a token.
template <typename E, int ACT>
static __device__ __forceinline__ void finish(const LinearArgs &a, float (&v)[8], const float (&bias)[8], int m, int n, int count) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = activate<ACT>(v[i] + bias[i]);
    if (a.gate) {
        const Piece<E> p = load_piece<E>(a.gate + (m / a.gate_rows) * a.ldg + n, count);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= E::to_f32(p.e[i]);
    }
    if (a.residual) {
        const Piece<E> p = load_piece<E>(a.residual + m * a.ldr + n, count);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += E::to_f32(p.e[i]);
    }
    Piece<E> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.e[i] = E::from_f32(v[i]);
    store_piece<E>(a.y + m * a.ldy + n, o, count);
}

// A wave's 64 channels x 16 FM tokens: the lane's token of fragment j is m + 16 j, its channels n .. n + 15 (channel_of_row).
template <typename E, int ACT, int FM>
static __device__ __forceinline__ void finish_tile(const LinearArgs &a, v4f (&acc)[4][FM], int m, int n) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int count = min(8, a.N - n - 8 * h);
        if (count <= 0) return;
        float bias[8] = {};
        if (a.bias) {
            const Piece<E> p = load_piece<E>(a.bias + n + 8 * h, count);
#pragma unroll
            for (int i = 0; i < 8; ++i) bias[i] = E::to_f32(p.e[i]);
        }
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            if (m + 16 * j >= a.M) break;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = acc[2 * h + i / 4][j][i & 3];
            finish<E, ACT>(a, v, bias, m + 16 * j, n + 8 * h, count);
        }
    }
}
template <typename E, int FM>
static __device__ __forceinline__ void epilogue(const LinearArgs &a, v4f (&acc)[4][FM], int m, int n) {
    switch (a.act) {
        case DVDQ_ACT_SILU: finish_tile<E, DVDQ_ACT_SILU>(a, acc, m, n); break;
        case DVDQ_ACT_GELU_TANH: finish_tile<E, DVDQ_ACT_GELU_TANH>(a, acc, m, n); break;
        case DVDQ_ACT_GELU: finish_tile<E, DVDQ_ACT_GELU>(a, acc, m, n); break;
        default: finish_tile<E, DVDQ_ACT_NONE>(a, acc, m, n);
    }
}

// The weights are the matrix instruction's rows, the tokens its columns, so that a lane's four results are four channels of one
// token.  Row r of fragment f of 64 channels is channel 16 (r / 4) + 4 f + r % 4: over the four fragments a lane then holds 16
// consecutive channels of a token, and the four lanes of a token 64, which are stored without a detour.
static __device__ __forceinline__ int channel_of_row(int row) { return (row & ~63) + 16 * ((row & 15) >> 2) + 4 * ((row & 63) >> 4) + (row & 3); }

// Any sizes, pitches and addresses: 128 x 128 outputs of four waves, 64 x 64 each, operands through registers into LDS rows of 64
// elements of K.  The 16-byte pieces of an LDS row are permuted by its row number, so that the 16 rows that a read takes at once
// lie in different banks.
template <typename E>
__global__ __launch_bounds__(256) void linear_any(LinearArgs a) {
    constexpr int BK = 64;
    __shared__ uint4 lds_w[128 * 8], lds_x[128 * 8];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n_tiles = (a.N + 127) / 128, tile_m = blockIdx.x / n_tiles;
    const int n0 = (blockIdx.x - tile_m * n_tiles) * 128, m0 = tile_m * 128;
    const int wn = (wave & 1) * 64, wm = (wave >> 1) * 64;
    v4f acc[4][4] = {};
    const int piece = tid & 7, row0 = tid >> 3;
    for (int k0 = 0; k0 < a.K; k0 += BK) {
        const int k = k0 + piece * 8, count = min(8, a.K - k);
        Piece<E> pw[4], px[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + 32 * i;
            const int n = min(n0 + channel_of_row(row), a.N - 1), m = min(m0 + row, a.M - 1);
            pw[i] = load_piece<E>(a.w + n * a.ldw + k, count);
            px[i] = load_piece<E>(a.x + m * a.ldx + k, count);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + 32 * i, at = row * 8 + (piece ^ ((row >> 1) & 7));
            lds_w[at] = __builtin_bit_cast(uint4, pw[i]);
            lds_x[at] = __builtin_bit_cast(uint4, px[i]);
        }
        __syncthreads();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            uint4 fw[4], fx[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const int rw = wn + 16 * f + (lane & 15), rx = wm + 16 * f + (lane & 15), p = 4 * ks + (lane >> 4);
                fw[f] = lds_w[rw * 8 + (p ^ ((rw >> 1) & 7))];
                fx[f] = lds_x[rx * 8 + (p ^ ((rx >> 1) & 7))];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma<E>(fw[i], fx[j], acc[i][j]);
        }
    }
    epilogue<E>(a, acc, m0 + wm + (lane & 15), n0 + wn + 16 * (lane >> 4));
}

// ---- rows of whole 16-byte pieces: operands straight into LDS

// 16 bytes per lane from each lane's own address to LDS address lds_base + 16 * lane (completion awaited by hand, as with
// lds_direct_load16)
static __device__ __forceinline__ void lds_direct_load16_at(const void *p, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds_base) : "memory");
}

__device__ uint4 zero_piece;   // what the pieces past K of the last slice are read from

// Tiles of 64 WN channels x 16 FM WM tokens, WN x WM waves of 64 channels x 16 FM tokens each; slices of 64 elements of K, two of
// them in LDS.  A slice is worked off in phases of 16 (or fewer) matrix instructions, and a phase begins by requesting the fragments
// of the next one, so that the matrix cores have operands when it ends.  Before the last phase of a slice, whose fragments
// are then in registers, stands the slice's one barrier: behind it the next slice is in LDS for every wave, and the buffer of this one is free for
// the slice after that.
template <typename E, int FM, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM, FM * WN * WM == 64 ? 2 : 2) void linear_tiles(LinearArgs a) {
    constexpr int W = WN * WM, BN = 64 * WN, BM = 16 * FM * WM, FH = FM < 4 ? FM : 4, NH = FM / FH, P = 2 * NH;
    constexpr int LW = BN / 8 / W, LX = BM / 8 / W;          // loads of a wave per slice, 8 rows each
    constexpr uint32_t kBufBytes = (BN + BM) * 128;
    extern __shared__ uint4 lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n_tiles = (a.N + BN - 1) / BN, m_tiles = (a.M + BM - 1) / BM;
    int m0, n0;
    {
        // consecutive workgroups go to different XCDs: each XCD takes one run of tiles, 4 columns wide
        const int total = gridDim.x, xcd = blockIdx.x & 7, i = blockIdx.x >> 3;
        const int t = xcd * (total >> 3) + min(xcd, total & 7) + i;
        tile_origin(t, m_tiles, n_tiles, 4, BM, BN, m0, n0);
    }
    const int wn = wave % WN * 64, wm = wave / WN * 16 * FM;

    const uint32_t lds0 = lds_address(lds);
    const uint8_t *src_w = reinterpret_cast<const uint8_t *>(uniform_ptr(a.w + n0 * a.ldw));
    const uint8_t *src_x = reinterpret_cast<const uint8_t *>(uniform_ptr(a.x + m0 * a.ldx));
    uint32_t off_w[LW], off_x[LX];
#pragma unroll
    for (int j = 0; j < LW; ++j) {
        const int row = wave * (8 * LW) + 8 * j + (lane >> 3);
        off_w[j] = (uint32_t)(min(channel_of_row(row), a.N - 1 - n0) * a.ldw * 2) + 16 * ((lane & 7) ^ ((row >> 1) & 7));
    }
#pragma unroll
    for (int j = 0; j < LX; ++j) {
        const int row = wave * (8 * LX) + 8 * j + (lane >> 3);
        off_x[j] = (uint32_t)(min(row, a.M - 1 - m0) * a.ldx * 2) + 16 * ((lane & 7) ^ ((row >> 1) & 7));
    }
    const int slices = (a.K + 63) >> 6;
    auto load = [&](int q) {
        const uint32_t to_w = lds0 + (q & 1) * kBufBytes + wave * (1024 * LW), to_x = lds0 + (q & 1) * kBufBytes + BN * 128 + wave * (1024 * LX);
        const uint8_t *sw = src_w + (uint32_t)q * 128u, *sx = src_x + (uint32_t)q * 128u;
        if ((q + 1) * 64 <= a.K) {
#pragma unroll
            for (int j = 0; j < LW; ++j) lds_direct_load16(sw, off_w[j], to_w + 1024 * j);
#pragma unroll
            for (int j = 0; j < LX; ++j) lds_direct_load16(sx, off_x[j], to_x + 1024 * j);
        } else {
            const uint32_t left = (uint32_t)(a.K - q * 64) * 2;   // bytes of a row that there are
#pragma unroll
            for (int j = 0; j < LW; ++j) {
                const uint32_t piece = 16 * ((lane & 7) ^ (((wave * (8 * LW) + 8 * j + (lane >> 3)) >> 1) & 7));
                lds_direct_load16_at(piece < left ? static_cast<const void *>(sw + off_w[j]) : &zero_piece, to_w + 1024 * j);
            }
#pragma unroll
            for (int j = 0; j < LX; ++j) {
                const uint32_t piece = 16 * ((lane & 7) ^ (((wave * (8 * LX) + 8 * j + (lane >> 3)) >> 1) & 7));
                lds_direct_load16_at(piece < left ? static_cast<const void *>(sx + off_x[j]) : &zero_piece, to_x + 1024 * j);
            }
        }
    };

    // fragment reads: LDS row r of 128 bytes holds its 16-byte piece c at c ^ ((r >> 1) & 7)
    const int at = (lane & 15) * 8 + ((lane >> 4) ^ ((lane & 15) >> 1));   // of k-step 0; k-step 1 is piece ^ 4
    const int at_w = wn * 8 + at, at_x = BN * 8 + wm * 8 + at;
    v4f acc[4][FM] = {};
    uint4 fw[2][4], fx[2][FH];
    auto read = [&](int buf, int p) {   // the fragments of phase p of the slice in `buf`
        const int ks = p / NH, h = p % NH;
        const uint4 *base = lds + buf * (kBufBytes / 16);
        if (h == 0)
#pragma unroll
            for (int f = 0; f < 4; ++f) fw[ks][f] = base[(at_w ^ (4 * ks)) + 128 * f];
#pragma unroll
        for (int f = 0; f < FH; ++f) fx[p & 1][f] = base[(at_x ^ (4 * ks)) + 128 * (h * FH + f)];
    };

    load(0);
    if (slices > 1) {
        load(1);
        wait_vmcnt<LW + LX>();
    } else {
        wait_vmcnt<0>();
    }
    asm volatile("s_barrier" ::: "memory");
    read(0, 0);
    for (int q = 0; q < slices; ++q) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (p < P - 1) {
                read(q & 1, p + 1);
            } else if (q + 1 < slices) {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                if (q + 2 < slices) load(q + 2);
                read((q + 1) & 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < FH; ++j) acc[i][(p % NH) * FH + j] = mfma<E>(fw[p / NH][i], fx[p & 1][j], acc[i][(p % NH) * FH + j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    epilogue<E>(a, acc, m0 + wm + (lane & 15), n0 + wn + 16 * (lane >> 4));
}

template <typename E, int FM, int WN, int WM>
int launch_tiles(const LinearArgs &a, hipStream_t stream) {
    constexpr size_t kLds = 2 * (64 * WN + 16 * FM * WM) * 128;
    static std::atomic<uint64_t> done{0};
    const auto kernel = linear_tiles<E, FM, WN, WM>;
    allow_dynamic_lds(reinterpret_cast<const void *>(kernel), kLds, done);
    const unsigned tiles = (unsigned)((a.N + 64 * WN - 1) / (64 * WN)) * (unsigned)((a.M + 16 * FM * WM - 1) / (16 * FM * WM));
    kernel<<<dim3(tiles), 64 * WN * WM, kLds, stream>>>(a);
    return check_launch();
}

}  // namespace

size_t linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    (void)M, (void)N, (void)K;
    return 0;
}

int launch_linear(const void *x, int64_t ldx, const void *w, int64_t ldw, const void *bias, int act, const void *gate, int64_t gate_rows,
                  int64_t ldg, const void *residual, int64_t ldr, int64_t M, int64_t N, int64_t K, int dtype, void *y, int64_t ldy,
                  void *workspace, hipStream_t stream) {
    (void)workspace;
    LinearArgs a = {};
    a.x = static_cast<const uint16_t *>(x), a.w = static_cast<const uint16_t *>(w), a.bias = static_cast<const uint16_t *>(bias);
    a.gate = static_cast<const uint16_t *>(gate), a.residual = static_cast<const uint16_t *>(residual), a.y = static_cast<uint16_t *>(y);
    a.ldx = ldx, a.ldw = ldw, a.ldr = ldr, a.ldy = ldy, a.ldg = ldg;
    a.M = (int)M, a.N = (int)N, a.K = (int)K;
    a.gate_rows = gate ? (int)(M / gate_rows) : 1;
    a.act = act;
    const auto whole = [](const void *p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld & 7) == 0 && ld < (int64_t)1 << 22; };
    const bool pieces = K % 8 == 0 && whole(x, M > 1 ? ldx : 0) && whole(w, N > 1 ? ldw : 0);
    return with_type(dtype, [&](auto type) {
        using E = decltype(type);
        if constexpr (sizeof(typename E::Raw) == 2) {
            if (pieces) {
                if (((M + 255) / 256) * ((N + 255) / 256) >= 256) return launch_tiles<E, 8, 4, 2>(a, stream);
                return launch_tiles<E, 4, 2, 2>(a, stream);
            }
            linear_any<E><<<dim3((unsigned)(((N + 127) / 128) * ((M + 127) / 128))), 256, 0, stream>>>(a);
            return check_launch();
        } else {
            return (int)DVDQ_ERR_UNSUPPORTED;
        }
    });
}

}  // namespace dvdq
