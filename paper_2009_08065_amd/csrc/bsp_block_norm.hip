// The norms on either side of a Transformer block with the block's gate and the residual's scale (bsp_block_norm), and their
// gradients (bsp_block_norm_backward).
//
//   Z = x_scale X + gate * N_post(F)      H = N_pre(Z)       N(v) = (v - mean) / sqrt(var + eps) * w + b  (LAYER; RMS: mean = 0)
//
// Both are bound by memory: forward reads X and F and writes Z and H, backward reads up to dZ, dH, Z and F and writes dX and dF.  So
// a row stays in the registers of its team of threads from the first load to the last store: statistics, both norms and the rounding
// between them (N_pre reads Z as it is stored, which is what the backward pass will see) cost no second look at memory.
// A team is 16 lanes for the narrowest rows, one wavefront while a row has no more than 32 values for a lane (backward 16), else a workgroup.
// Measured (MI355X, us, of a pass among others): forward 8192 x 1024 in bf16, BERT's form 14.3 (4.7 TB/s), both norms and a gate 16; in fp32 23.0 (5.8
// TB/s); 16384 x 4096 in bf16 95 (5.6).  Backward 8192 x 1024, BERT's form 19.6 to 20.3 (16.9 and 3.9 for the columns; 4.2 TB/s), both norms and a gate 30 (3.4: its
// vectors are asked for behind the first row sum, one row of a team is on its way at a time); 16384 x 4096 143 (4.7 TB/s) and 187 to 192 (4.2).
// Sums are fp32: of a row by the lanes and then across them; the mean first, then the squares of what is left, which a
// sum of squares less the square of the sum would lose where the mean is large.  The sums down the columns (gradients of w, b and gate) are kept
// in registers over the rows of a workgroup, and a second launch adds the workgroups' sums in ascending order: equal calls give equal bits.
#include "bsp_common.h"
#include "bsp_mfma_device.h"

namespace bsp {
namespace {

constexpr int kMaxH = 8192;
constexpr int kVec = 8;  // values of a piece

// How a thread has its pieces of a row.  kWhole: 8 neighbouring columns, 16 or 32 bytes in one go (at any address: loads and stores need no
// alignment).  kWords: the same from a buffer that ends with the row, word by word.  kApart: 8 columns a team's width apart.
// Widths that are multiples of 8: kWords forward (us, 16384 x 4096 in fp32, both norms and gate rows 224, kWhole 239; 4096 x 2048 in bf16 15.8, 16.9),
// kWhole backward (16384 x 4096 in fp32 378, kWords 403).  16-bit rows of an even width: kWords (353 x 6462 forward 10.3, kApart 12.9, backward 29.4,
// 33.5; in fp32 it is the other way round, 12.3 and 11.3, 32.4 and 29.2).  Else kApart.
enum { kApart, kWhole, kWords };

// Column of value j of piece u of thread t's share of a row.
template <int TPR, int HOW>
__device__ __forceinline__ int column(int u, int j, int t) {
    return HOW != kApart ? (u * TPR + t) * kVec + j : (u * kVec + j) * TPR + t;
}

// The row of H elements at element `at`, as a buffer: past its end loads give 0 and stores write nothing, word by word.  (A team's row is the same for all
// lanes of a wavefront.  With a comparison and a branch for every element the kernel's code, which a short call runs through once, took
// most of its time.)
template <int SIZE>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of_row(const void *p, int64_t at, int H) {
    const uint64_t a = (uint64_t)p + at * SIZE;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void *)((uint64_t)hi << 32 | lo), 0, H * SIZE, 0x00020000);
}

// A piece as it lies in memory.
template <int DT, int TPR, int HOW>
struct Raw {
    uint4 d[DT == BSP_F32 ? 2 : 1];
    // of the row of H columns at element `at`
    __device__ __forceinline__ void load(const void *p, int64_t at, int u, int t, int H) {
        constexpr int size = DT == BSP_F32 ? 4 : 2;
        if constexpr (HOW == kWhole) {
            const int c = column<TPR, HOW>(u, 0, t);
            if (c < H) {
                __builtin_memcpy(d, (const uint8_t *)p + (at + c) * size, sizeof(d));
            } else {
#pragma unroll
                for (uint4 &x : d) x = make_uint4(0u, 0u, 0u, 0u);
            }
        } else if constexpr (HOW == kWords) {
            const __amdgpu_buffer_rsrc_t row = buffer_of_row<size>(p, at, H);
            const int c = size * column<TPR, HOW>(u, 0, t);
#pragma unroll
            for (int i = 0; i < (int)(sizeof(d) / 16); ++i) d[i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(row, c + 16 * i, 0, 0));
        } else {
            uint32_t w[8];
            if constexpr (TPR < 64) {  // (several rows in a wavefront: the last column in the place of those past it, and zeros after that)
#pragma unroll
                for (int j = 0; j < kVec; ++j) {
                    const int c = column<TPR, HOW>(u, j, t);
                    if constexpr (DT == BSP_F32) w[j] = ((const uint32_t *)p)[at + (c < H ? c : H - 1)];
                    else w[j] = ((const uint16_t *)p)[at + (c < H ? c : H - 1)];
                }
#pragma unroll
                for (int j = 0; j < kVec; ++j) w[j] = column<TPR, HOW>(u, j, t) < H ? w[j] : 0u;
            } else {
                const __amdgpu_buffer_rsrc_t row = buffer_of_row<size>(p, at, H);
#pragma unroll
                for (int j = 0; j < kVec; ++j) {
                    const int c = size * column<TPR, HOW>(u, j, t);
                    if constexpr (DT == BSP_F32) w[j] = __builtin_amdgcn_raw_buffer_load_b32(row, c, 0, 0);
                    else w[j] = __builtin_amdgcn_raw_buffer_load_b16(row, c, 0, 0);
                }
            }
            if constexpr (DT == BSP_F32) {
                d[0] = make_uint4(w[0], w[1], w[2], w[3]);
                d[1] = make_uint4(w[4], w[5], w[6], w[7]);
            } else {
                d[0] = make_uint4(w[0] | (w[1] << 16), w[2] | (w[3] << 16), w[4] | (w[5] << 16), w[6] | (w[7] << 16));
            }
        }
    }
    __device__ __forceinline__ float operator[](int j) const {
        if constexpr (DT == BSP_F32) {
            const uint32_t w[8] = {d[0].x, d[0].y, d[0].z, d[0].w, d[1].x, d[1].y, d[1].z, d[1].w};
            return __uint_as_float(w[j]);
        } else {
            const uint32_t w[4] = {d[0].x, d[0].y, d[0].z, d[0].w};
            const uint16_t h = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
            return elem<DT>::load(&h, 0);
        }
    }
};

template <int DT, int TPR, int HOW>
__device__ __forceinline__ void store_piece(const float (&v)[kVec], void *p, int64_t at, int u, int t, int H) {
    if constexpr (HOW == kWhole) {
        const int c = column<TPR, HOW>(u, 0, t);
        if (c >= H) return;
        if constexpr (DT == BSP_F32) {
            __builtin_memcpy((float *)p + at + c, v, 32);
        } else {
            uint32_t d[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) d[j] = cvt_pk<DT>(v[2 * j], v[2 * j + 1]);
            __builtin_memcpy((uint16_t *)p + at + c, d, 16);
        }
    } else if constexpr (HOW == kWords) {
        constexpr int size = DT == BSP_F32 ? 4 : 2;
        const __amdgpu_buffer_rsrc_t row = buffer_of_row<size>(p, at, H);
        const int c = size * column<TPR, HOW>(u, 0, t);
        if constexpr (DT == BSP_F32) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])},
                                                       row, c + 16 * i, 0, 0);
        } else {
            __builtin_amdgcn_raw_buffer_store_b128(u32x4{cvt_pk<DT>(v[0], v[1]), cvt_pk<DT>(v[2], v[3]), cvt_pk<DT>(v[4], v[5]), cvt_pk<DT>(v[6], v[7])}, row, c, 0, 0);
        }
    } else if constexpr (TPR < 64) {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            if (column<TPR, HOW>(u, j, t) < H) elem<DT>::store(p, at + column<TPR, HOW>(u, j, t), v[j]);
    } else {
        constexpr int size = DT == BSP_F32 ? 4 : 2;
        const __amdgpu_buffer_rsrc_t row = buffer_of_row<size>(p, at, H);
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            const int c = size * column<TPR, HOW>(u, j, t);
            if constexpr (DT == BSP_F32) __builtin_amdgcn_raw_buffer_store_b32(elem<DT>::bits(v[j]), row, c, 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b16((uint16_t)elem<DT>::bits(v[j]), row, c, 0, 0);
        }
    }
}

template <int DT>
__device__ __forceinline__ float rounded(float v) {
    if constexpr (DT == BSP_F32) return v;
    else {
        const uint16_t b = (uint16_t)elem<DT>::bits(v);
        return elem<DT>::load(&b, 0);
    }
}

// The sum of 64 lanes' values, in every lane: within rows of 16 lanes and then across them (an exchange through LDS takes ten times as long, and
// a row waits for up to four of these in turn).
template <int CTRL, int ROWS>
__device__ __forceinline__ float add_dpp(float x) {
    return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float x) {
    x = add_dpp<0x111, 0xf>(x);  // row_shr 1, 2, 4, 8: lane 15 of a row has the row's
    x = add_dpp<0x112, 0xf>(x);
    x = add_dpp<0x114, 0xf>(x);
    x = add_dpp<0x118, 0xf>(x);
    x = add_dpp<0x142, 0xa>(x);  // row_bcast 15 into rows 1 and 3, 31 into rows 2 and 3
    x = add_dpp<0x143, 0xc>(x);
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), 63));
}

// The sum of 16 lanes' values, in every one of them: rotations within the row.
__device__ __forceinline__ float sum_of_16(float x) {
    x = add_dpp<0x121, 0xf>(x);
    x = add_dpp<0x122, 0xf>(x);
    x = add_dpp<0x124, 0xf>(x);
    return add_dpp<0x128, 0xf>(x);
}

// Sums of K values over the TPR threads of a team, in every one of them.  LDS: `red` of 2 * K * TPR / 64 floats, its halves in turn, so that
// one barrier a sum is enough.
template <int TPR, int K>
__device__ __forceinline__ void team_sum(float (&v)[K], float *red, int &turn) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = TPR == 16 ? sum_of_16(v[k]) : wave_sum(v[k]);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        float *r = red + turn * K * W;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) r[k * W + (threadIdx.x >> 6)] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) s += r[k * W + w];
            v[k] = s;
        }
    }
}

struct Forward {
    const void *X, *F, *gate, *w_post, *b_post, *w_pre, *b_pre;
    void *Z, *H;
    float *stats_post, *stats_pre;
    int64_t T, rows_per_gate;
    float x_scale, eps;
    int32_t width, rms, norms;
};

// One team's row: mean and 1 / deviation of the values v (columns past the width hold 0 and are not part of it).
template <int TPR, int ITER, int HOW>
__device__ __forceinline__ void statistics(const float (&v)[ITER][kVec], int t, const Forward &a, float &mean, float &rstd, float *red, int &turn) {
    mean = 0.0f;
    const float n = 1.0f / (float)a.width;
    if (!a.rms) {
        float s[1] = {0.0f};
#pragma unroll
        for (int u = 0; u < ITER; ++u)
#pragma unroll
            for (int j = 0; j < kVec; ++j) s[0] += v[u][j];
        team_sum<TPR, 1>(s, red, turn);
        mean = s[0] * n;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int u = 0; u < ITER; ++u)
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            const float d = v[u][j] - mean;
            q[0] = column<TPR, HOW>(u, j, t) < a.width ? __builtin_fmaf(d, d, q[0]) : q[0];
        }
    team_sum<TPR, 1>(q, red, turn);
    rstd = 1.0f / __builtin_sqrtf(q[0] * n + a.eps);
}

template <int DT, int TPR, int ITER, int HOW>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void block_norm_kernel(Forward a) {
    constexpr int kTeams = TPR < 256 ? 256 / TPR : 1;
    __shared__ float red[TPR > 64 ? 2 * (TPR / 64) : 1];
    int turn = 0;
    const int t = threadIdx.x % TPR, H = a.width;
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kTeams + threadIdx.x / TPR;
    if (row >= a.T) return;  // (whole teams)
    const int64_t at = row * H;
    const bool post = a.F && (a.norms & BSP_NORM_POST), pre = (a.norms & BSP_NORM_PRE) != 0;
    // everything is asked for before the first sum is waited for
    using Piece = Raw<DT, TPR, HOW>;
    Piece rx[ITER], rf[ITER], rg[ITER], w1[ITER], b1[ITER], w2[ITER], b2[ITER];
    auto ask = [&](Piece(&r)[ITER], const void *p, int64_t from) {
        if (p)
#pragma unroll
            for (int u = 0; u < ITER; ++u) r[u].load(p, from, u, t, H);
    };
    ask(rx, a.X, at);
    ask(rf, a.F, at);
    ask(w1, a.w_post, 0);
    ask(b1, a.b_post, 0);
    if (a.gate) ask(rg, a.gate, row / a.rows_per_gate * H);
    ask(w2, a.w_pre, 0);
    ask(b2, a.b_pre, 0);
    auto normalise = [&](float(&v)[ITER][kVec], float mean, float rstd, const void *w, const Piece(&rw)[ITER], const void *b, const Piece(&rb)[ITER]) {
#pragma unroll
        for (int u = 0; u < ITER; ++u)
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                v[u][j] = (v[u][j] - mean) * rstd;
                if (w) v[u][j] *= rw[u][j];
                if (b) v[u][j] += rb[u][j];
            }
    };
    float x[ITER][kVec], f[ITER][kVec];
    if (a.F) {
#pragma unroll
        for (int u = 0; u < ITER; ++u)
#pragma unroll
            for (int j = 0; j < kVec; ++j) f[u][j] = rf[u][j];
        if (post) {
            float mean, rstd;
            statistics<TPR, ITER, HOW>(f, t, a, mean, rstd, red, turn);
            if (a.stats_post && t == 0) *reinterpret_cast<float2 *>(a.stats_post + 2 * row) = make_float2(mean, rstd);
            normalise(f, mean, rstd, a.w_post, w1, a.b_post, b1);
        }
    }
#pragma unroll
    for (int u = 0; u < ITER; ++u)
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            float z = a.x_scale * rx[u][j];
            if (a.F) z += a.gate ? f[u][j] * rg[u][j] : f[u][j];
            x[u][j] = column<TPR, HOW>(u, j, t) < H ? rounded<DT>(z) : 0.0f;
        }
    if (a.Z)
#pragma unroll
        for (int u = 0; u < ITER; ++u) store_piece<DT, TPR, HOW>(x[u], a.Z, at, u, t, H);
    if (pre) {
        float mean, rstd;
        statistics<TPR, ITER, HOW>(x, t, a, mean, rstd, red, turn);
        if (a.stats_pre && t == 0) *reinterpret_cast<float2 *>(a.stats_pre + 2 * row) = make_float2(mean, rstd);
        normalise(x, mean, rstd, a.w_pre, w2, a.b_pre, b2);
#pragma unroll
        for (int u = 0; u < ITER; ++u) store_piece<DT, TPR, HOW>(x[u], a.H, at, u, t, H);
    }
}

// ---- backward -----------------------------------------------------------------------------------------------------------------
// With d the gradient of N's output, g = d w and hat = (v - mean) rstd:
//   dv = rstd (g - hat mean(g hat) - mean(g))     dw = sum d hat     db = sum d        (RMS: without mean(g))
enum { kDwPost, kDbPost, kDwPre, kDbPre, kDgate, kSums };

struct Backward {
    const void *dZ, *dH, *Z, *F, *gate, *w_post, *b_post, *w_pre;
    const float *stats_post, *stats_pre;
    void *dX, *dF;
    float *sums;   // [kSums][workgroups][width], what each workgroup has
    float *dgate;  // where a team owns whole rows of the gate
    int64_t T, rows_per_gate, rows_per_piece;
    float x_scale;
    int32_t width, rms, norms, pieces, groups, per_wg;  // pieces of a gate row's rows; gate rows; gate rows of a workgroup (pieces == 1)
    uint32_t want;                                      // bit i: sums of kind i
};

// Whether a row is for 16 lanes, four of them in a wavefront.  (us, bf16, BERT's form and both norms with a gate: 32768 x 64 forward 7.0 and 8.6, with a
// wavefront for a row 16.6 and 22.4, backward 11.4 and 16.9, 22.3 and 45; 32768 x 256 13.7 and 15.7, 18.4 and 23, backward 19.4 and 28, 23.4 and 46; 17221
// x 79 13.0 and 20.4, 24 and 37; but 14904 x 228, which is no multiple of 8, 18.5 and 42, 18.2 and 26.)
bool of_16(int64_t H) { return H <= 128 || (H <= 256 && H % kVec == 0); }

constexpr int kBackTeams = 4;  // wavefronts of a workgroup where a row is one's (their sums meet before they leave it)
constexpr int teams_of(int tpr) { return tpr <= 64 ? 64 * kBackTeams / tpr : 1; }

// SIMPLE: BERT's form, N_pre without a gate (no F, and two sums).
template <int DT, int TPR, int ITER, int HOW, bool SIMPLE>
__global__ __launch_bounds__(TPR * teams_of(TPR)) void block_norm_back_kernel(Backward a) {
    constexpr int kTeams = teams_of(TPR);
    __shared__ float red[TPR > 64 ? 4 * (TPR / 64) : 1];
    constexpr int kColumns = TPR * ITER * kVec;
    __shared__ __align__(16) float share[kTeams > 1 ? 2 * kTeams * kColumns : 4];
    int turn = 0;
    const int t = threadIdx.x % TPR, team = threadIdx.x / TPR, H = a.width;
    const bool pre = SIMPLE || (a.norms & BSP_NORM_PRE), post = !SIMPLE && (a.norms & BSP_NORM_POST);
    const void *F = SIMPLE ? nullptr : a.F, *gate = SIMPLE ? nullptr : a.gate;
    const float inv = 1.0f / (float)H;
    float acc[kSums][ITER][kVec];
    auto clear = [&](int i) {
#pragma unroll
        for (int u = 0; u < ITER; ++u)
#pragma unroll
            for (int j = 0; j < kVec; ++j) acc[i][u][j] = 0.0f;
    };
#pragma unroll
    for (int i = 0; i < kSums; ++i) clear(i);
    using Piece = Raw<DT, TPR, HOW>;
    Piece w2[ITER];
    if (pre && a.w_pre)
#pragma unroll
        for (int u = 0; u < ITER; ++u) w2[u].load(a.w_pre, 0, u, t, H);

    struct Row {
        Piece dz[ITER], dh[ITER], z[ITER], f[ITER];
        float2 pre, post;
    };
    auto ask = [&](Row &r, int64_t row) {
        const int64_t at = row * H;
        auto each = [&](Piece(&x)[ITER], const void *p) {
#pragma unroll
            for (int u = 0; u < ITER; ++u) x[u].load(p, at, u, t, H);
        };
        if (a.dZ) each(r.dz, a.dZ);
        if (pre) {
            each(r.dh, a.dH);
            each(r.z, a.Z);
            r.pre = *reinterpret_cast<const float2 *>(a.stats_pre + 2 * row);
        }
        if (F) each(r.f, F);
        if (post) r.post = *reinterpret_cast<const float2 *>(a.stats_post + 2 * row);
    };
    auto one_row = [&](const Row &r, int64_t row, int64_t group) {
        const int64_t at = row * H;
        float d[ITER][kVec];
#pragma unroll
        for (int u = 0; u < ITER; ++u)
#pragma unroll
            for (int j = 0; j < kVec; ++j) d[u][j] = a.dZ ? r.dz[u][j] : 0.0f;
        if (pre) {
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int u = 0; u < ITER; ++u)
#pragma unroll
                for (int j = 0; j < kVec; ++j) {
                    const float hat = (r.z[u][j] - r.pre.x) * r.pre.y, dh = r.dh[u][j];
                    acc[kDwPre][u][j] = __builtin_fmaf(dh, hat, acc[kDwPre][u][j]);
                    acc[kDbPre][u][j] += dh;
                    const float g = a.w_pre ? dh * w2[u][j] : dh;
                    s[0] = __builtin_fmaf(g, hat, s[0]);  // (past the width dh is 0)
                    s[1] += g;
                }
            team_sum<TPR, 2>(s, red, turn);
            const float c1 = s[0] * inv, c2 = a.rms ? 0.0f : s[1] * inv;
#pragma unroll
            for (int u = 0; u < ITER; ++u)
#pragma unroll
                for (int j = 0; j < kVec; ++j) {
                    const float hat = (r.z[u][j] - r.pre.x) * r.pre.y, dh = r.dh[u][j];
                    d[u][j] += r.pre.y * ((a.w_pre ? dh * w2[u][j] : dh) - hat * c1 - c2);
                }
        }
        if (a.dX)
#pragma unroll
            for (int u = 0; u < ITER; ++u) {
                float x[kVec];
#pragma unroll
                for (int j = 0; j < kVec; ++j) x[j] = a.x_scale * d[u][j];
                store_piece<DT, TPR, HOW>(x, a.dX, at, u, t, H);
            }
        if constexpr (!SIMPLE) {
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int u = 0; u < ITER; ++u) {
                Piece w, b, y;
                if (gate) y.load(gate, group * H, u, t, H);
                if (post && a.w_post) w.load(a.w_post, 0, u, t, H);
                if (post && a.b_post) b.load(a.b_post, 0, u, t, H);
#pragma unroll
                for (int j = 0; j < kVec; ++j) {
                    if (column<TPR, HOW>(u, j, t) >= H) {
                        d[u][j] = 0.0f;
                        continue;
                    }
                    float n = F ? r.f[u][j] : 0.0f, hat = 0.0f;
                    if (post) {
                        hat = (n - r.post.x) * r.post.y;
                        n = a.w_post ? hat * w[j] : hat;
                        if (a.b_post) n += b[j];
                    }
                    if (gate) {
                        acc[kDgate][u][j] = __builtin_fmaf(d[u][j], n, acc[kDgate][u][j]);
                        d[u][j] *= y[j];
                    }
                    if (post) {
                        acc[kDwPost][u][j] = __builtin_fmaf(d[u][j], hat, acc[kDwPost][u][j]);
                        acc[kDbPost][u][j] += d[u][j];
                        if (a.w_post) d[u][j] *= w[j];
                        s[0] = __builtin_fmaf(d[u][j], hat, s[0]);
                        s[1] += d[u][j];
                    }
                }
            }
            if (post) {
                team_sum<TPR, 2>(s, red, turn);
                const float c1 = s[0] * inv, c2 = a.rms ? 0.0f : s[1] * inv;
#pragma unroll
                for (int u = 0; u < ITER; ++u)
#pragma unroll
                    for (int j = 0; j < kVec; ++j) d[u][j] = r.post.y * (d[u][j] - (r.f[u][j] - r.post.x) * r.post.y * c1 - c2);
            }
        }
        if (a.dF)
#pragma unroll
            for (int u = 0; u < ITER; ++u) store_piece<DT, TPR, HOW>(d[u], a.dF, at, u, t, H);
    };

    // The rows of this team, one loop for both ways they are dealt (the kernel's code is what a short call waits for): every kTeams-th row of a
    // piece of one gate row's rows (of all rows where there is no gate), or every kTeams-th gate row of the workgroup's, whole.
    const bool whole = a.per_wg != 0;
    const int64_t first_group = whole ? (int64_t)blockIdx.x * a.per_wg : blockIdx.x / a.pieces;
    const int64_t r0 = whole ? 0 : (blockIdx.x - first_group * a.pieces) * a.rows_per_piece;
    int64_t r1 = whole ? a.rows_per_gate : r0 + a.rows_per_piece;
    if (r1 > a.rows_per_gate) r1 = a.rows_per_gate;
    const int64_t stride = whole ? 1 : kTeams, begin = whole ? 0 : r0 + team;
    int64_t last_group = whole ? first_group + a.per_wg : first_group + 1;
    if (last_group > a.groups) last_group = a.groups;
    int64_t group = whole ? first_group + team : first_group, r = begin;
    // the next row is on its way while one is worked on, where the registers have room for it
    constexpr bool kAhead = SIMPLE || TPR == 256;
    Row cur;
    bool more = r < r1 && group < last_group;
    if (kAhead && more) ask(cur, group * a.rows_per_gate + r);
    while (more) {
        const int64_t at_group = group, at_row = group * a.rows_per_gate + r;
        r += stride;
        const bool end = r >= r1;  // of this team's part of the gate row
        if (end) {
            r = begin;
            group += kTeams;
        }
        more = group < last_group && !(end && !whole);
        if constexpr (kAhead) {
            Row next;
            if (more) ask(next, group * a.rows_per_gate + r);
            one_row(cur, at_row, at_group);
            cur = next;
        } else {
            ask(cur, at_row);
            one_row(cur, at_row, at_group);
        }
        if (whole && end) {
            if (a.dgate)
#pragma unroll
                for (int u = 0; u < ITER; ++u) store_piece<BSP_F32, TPR, HOW>(acc[kDgate][u], a.dgate, at_group * H, u, t, H);
            clear(kDgate);
        }
    }
    // the workgroup's sums: the teams' by columns in LDS, each thread adds up some columns' in ascending order
    int half = 0;
    static_for<0, kSums>([&](auto kind) {
        constexpr int i = decltype(kind)::value;
        if (SIMPLE && i != kDwPre && i != kDbPre) return;
        if (!((a.want >> i) & 1u)) return;  // uniform
        float *out = a.sums + ((int64_t)i * gridDim.x + blockIdx.x) * H;
        if constexpr (kTeams > 1) {
            float *mine = share + (half * kTeams + team) * kColumns, *first = share + half * kTeams * kColumns;
            half ^= 1;  // (the other half is read no more: everybody has passed the barrier of the kind before)
#pragma unroll
            for (int u = 0; u < ITER; ++u)
#pragma unroll
                for (int j = 0; j < kVec; ++j) mine[column<TPR, HOW>(u, j, t)] = acc[i][u][j];
            __syncthreads();
            for (int c = threadIdx.x; c < H; c += TPR * kTeams) {
                float s = first[c];
#pragma unroll
                for (int o = 1; o < kTeams; ++o) s += first[o * kColumns + c];
                out[c] = s;
            }
        } else {
#pragma unroll
            for (int u = 0; u < ITER; ++u) store_piece<BSP_F32, TPR, HOW>(acc[i][u], out, 0, u, t, H);
        }
    });
}

// out[k][row][c] = sum over `n` workgroups' sums, ascending in each of 16 interleaved parts, then the parts.
struct Columns {
    const float *sums;
    float *out[kSums];
    int64_t wgs;
    int32_t width, pieces, groups;
};

constexpr int kParts = 16;

__global__ __launch_bounds__(64 * kParts) void block_norm_columns_kernel(Columns a) {
    __shared__ float part[kParts][64];
    const int lane = threadIdx.x & 63, p = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    const int row = blockIdx.y;  // a norm's sums, then the gate's rows
    const int kind = row < kDgate ? row : kDgate;
    float *out = a.out[kind];
    if (!out) return;
    const int64_t first = kind == kDgate ? (int64_t)(row - kDgate) * a.pieces : 0, n = kind == kDgate ? a.pieces : a.wgs;
    const float *in = a.sums + ((int64_t)kind * a.wgs + first) * a.width + (c < a.width ? c : 0);
    float s = 0.0f;
    const float *q = in + p * (int64_t)a.width;
    const int64_t step = kParts * (int64_t)a.width;
    int32_t left = n > p ? (int32_t)((n - p + kParts - 1) / kParts) : 0;
    auto add = [&](auto count) {  // that many loads on their way together (8192 x 1024: with four only 0.8 us longer)
        constexpr int N = decltype(count)::value;
        for (; left >= N; left -= N) {
            float v[N];
#pragma unroll
            for (int k = 0; k < N; ++k, q += step) v[k] = *q;
#pragma unroll
            for (int k = 0; k < N; ++k) s += v[k];
        }
    };
    add(std::integral_constant<int, 16>{});
    add(std::integral_constant<int, 4>{});
    add(std::integral_constant<int, 1>{});
    part[p][lane] = s;
    __syncthreads();
    if (p || c >= a.width) return;
    for (int i = 1; i < kParts; ++i) s += part[i][lane];
    out[(int64_t)(kind == kDgate ? row - kDgate : 0) * a.width + c] = s;
}

// Workgroups of the backward pass, at most where the gate's rows allow it.  Two for a compute unit; one where they are of 512 threads (us, 2048 x 8192
// in bf16, BERT's form 38.5, with two 45, both norms and a gate 74, 87), and where they would have a row or two each, because each has sums to write and
// to be read again (512 x 4096 15.2, 19.3, both norms and a gate in fp32 25.5, 33.6; but 2048 x 2048 28.4, 27.1).
int64_t ranges_of(int64_t T, int64_t H) { return H > 4096 || (H > 1024 && T <= 1024) ? 256 : 512; }

// Workgroups, and how the rows are dealt to them.
struct Deal {
    int64_t wgs, rows_per_gate, rows_per_piece;
    int32_t pieces, groups, per_wg;
};

Deal deal(int64_t T, int64_t H, int64_t gate_rows) {
    Deal d;
    const int64_t teams = teams_of(of_16(H) ? 16 : H <= 1024 ? 64 : 256);
    d.groups = (int32_t)(gate_rows > 0 ? gate_rows : 1);
    d.rows_per_gate = T / d.groups;
    const int64_t ranges = ranges_of(T, H);
    int64_t rows = (T + ranges - 1) / ranges;
    rows = (rows + teams - 1) / teams * teams;
    if (d.rows_per_gate >= rows || d.groups == 1) {
        d.pieces = (int32_t)((d.rows_per_gate + rows - 1) / rows);
        d.rows_per_piece = (d.rows_per_gate + d.pieces - 1) / d.pieces;
        d.per_wg = 0;
        d.wgs = (int64_t)d.groups * d.pieces;
    } else {
        d.pieces = 1;
        d.rows_per_piece = d.rows_per_gate;
        d.per_wg = (int32_t)((rows + d.rows_per_gate - 1) / d.rows_per_gate);
        d.wgs = ((int64_t)d.groups + d.per_wg - 1) / d.per_wg;
    }
    return d;
}

int check(int64_t T, int64_t H, int dt, int norms, int kind, const void *gate, int64_t gate_rows) {
    if (!valid_dtype(dt) || (kind != BSP_NORM_LAYER && kind != BSP_NORM_RMS)) return BSP_ERR_DTYPE;
    if (norms < 1 || norms > 3) return BSP_ERR_DTYPE;
    if (T < 0 || H <= 0 || H > kMaxH || T >= ((int64_t)1 << 31)) return BSP_ERR_SHAPE;
    if (gate && (gate_rows < 1 || T % gate_rows != 0 || gate_rows > 0x7fffffff)) return BSP_ERR_SHAPE;
    if (gate && gate_rows > (T ? T : 65535 - kDgate)) return BSP_ERR_SHAPE;  // (of no rows: the launch that clears the sums has a line of workgroups for each)
    return BSP_OK;
}

// f(how).  words: whether the rows and vectors are at addresses of 32-bit words, and (16 bits) the rows of whole ones.
template <int DT, int TPR, bool FORWARD, typename F>
void how_of(int64_t width, bool words, F f) {
    constexpr bool kAlone = TPR >= 64, kNarrow = DT != BSP_F32;  // (buffers are for rows that have a wavefront to themselves)
    if (width % kVec == 0 && (!FORWARD || !kAlone || words)) f(std::integral_constant<int, FORWARD && kAlone ? kWords : kWhole>{});
    else if (kAlone && kNarrow && words) f(std::integral_constant<int, kAlone && kNarrow ? kWords : kApart>{});
    else f(std::integral_constant<int, kApart>{});
}

template <int DT, int TPR, int ITER>
void launch_forward(const Forward &a, bool words, hipStream_t s) {
    constexpr int kTeams = TPR < 256 ? 256 / TPR : 1;
    const int64_t wgs = (a.T + kTeams - 1) / kTeams, most = (int64_t)1 << 20;  // (a launch has less than 2^32 threads along x)
    const dim3 grid((unsigned)(wgs < most ? wgs : most), (unsigned)((wgs + most - 1) / most));
    how_of<DT, TPR, true>(a.width, words, [&](auto how) { block_norm_kernel<DT, TPR, ITER, decltype(how)::value><<<grid, TPR < 256 ? 256 : TPR, 0, s>>>(a); });
}

template <int DT, int TPR, int ITER>
void launch_backward(const Backward &a, bool words, unsigned grid, hipStream_t s) {
    constexpr int kThreads = TPR * teams_of(TPR);
    const bool simple = a.norms == BSP_NORM_PRE && !a.gate;
    how_of<DT, TPR, false>(a.width, words, [&](auto how) {
        if (simple) block_norm_back_kernel<DT, TPR, ITER, decltype(how)::value, true><<<grid, kThreads, 0, s>>>(a);
        else block_norm_back_kernel<DT, TPR, ITER, decltype(how)::value, false><<<grid, kThreads, 0, s>>>(a);
    });
}

}  // namespace
}  // namespace bsp

using namespace bsp;

extern "C" int bsp_block_norm(const void *X, const void *F, int dt, int64_t T, int64_t H, int norms, int kind, float eps, float x_scale,
                              const void *gate, int64_t gate_rows, const void *w_post, const void *b_post, const void *w_pre,
                              const void *b_pre, void *Z, void *Hn, float *stats_post, float *stats_pre, void *stream) {
    const bool post = (norms & BSP_NORM_POST) != 0, pre = (norms & BSP_NORM_PRE) != 0;
    if (int st = check(T, H, dt, norms, kind, gate, gate_rows)) return st;
    if (T == 0) return BSP_OK;
    if (!X || (!F && (post || gate)) || (pre && !Hn) || (!Z && !pre)) return BSP_ERR_NULL;
    const size_t size = dtype_size(dt);
    bool words = H % 2 == 0;
    for (const void *p : {X, F, gate, w_post, b_post, w_pre, b_pre, (const void *)Z, (const void *)Hn}) {
        if (!aligned(p, size)) return BSP_ERR_SHAPE;
        words &= aligned(p, 4);
    }
    if (!aligned(stats_post, 8) || !aligned(stats_pre, 8)) return BSP_ERR_SHAPE;
    const Forward a = {X, F, gate, w_post, b_post, w_pre, b_pre, Z, Hn, stats_post, stats_pre,
                       T, gate ? T / gate_rows : T, x_scale, eps, (int32_t)H, kind == BSP_NORM_RMS, norms};
    hipStream_t s = (hipStream_t)stream;
    BSP_DISPATCH_DTYPE(dt, DT, {
        if (H <= 128) launch_forward<DT, 16, 1>(a, words, s);
        else if (of_16(H)) launch_forward<DT, 16, 2>(a, words, s);
        else if (H <= 512) launch_forward<DT, 64, 1>(a, words, s);
        else if (H <= 1024) launch_forward<DT, 64, 2>(a, words, s);
        else if (H <= 2048) launch_forward<DT, 64, 4>(a, words, s);
        else if (H <= 4096) launch_forward<DT, 256, 2>(a, words, s);
        else launch_forward<DT, 256, 4>(a, words, s);
    });
    return check_launch();
}

extern "C" size_t bsp_block_norm_backward_workspace_bytes(int64_t T, int64_t H, int64_t gate_rows) {
    if (T <= 0 || H <= 0 || H > kMaxH || gate_rows < 0 || (gate_rows && T % gate_rows)) return 0;
    return (size_t)kSums * (size_t)deal(T, H, gate_rows).wgs * (size_t)H * 4;
}

extern "C" int bsp_block_norm_backward(const void *dZ, const void *dH, const void *Z, const void *F, int dt, int64_t T, int64_t H, int norms,
                                       int kind, float x_scale, const void *gate, int64_t gate_rows, const void *w_post,
                                       const void *b_post, const void *w_pre, const float *stats_post, const float *stats_pre, void *dX,
                                       void *dF, float *dw_post, float *db_post, float *dw_pre, float *db_pre, float *dgate, void *ws,
                                       size_t ws_bytes, void *stream) {
    const bool post = (norms & BSP_NORM_POST) != 0, pre = (norms & BSP_NORM_PRE) != 0;
    if (int st = check(T, H, dt, norms, kind, gate, gate_rows)) return st;
    if ((!post && (dw_post || db_post)) || (!pre && (dw_pre || db_pre)) || (!gate && dgate)) return BSP_ERR_SHAPE;
    hipStream_t s = (hipStream_t)stream;
    const bool any = dw_post || db_post || dw_pre || db_pre || dgate;
    if ((pre && T && (!dH || !Z || !stats_pre)) || (post && T && (!F || !stats_post)) || (dgate && T && !F)) return BSP_ERR_NULL;
    if (!pre && !dZ && T) return BSP_ERR_NULL;
    const size_t size = dtype_size(dt);
    bool words = H % 2 == 0;
    for (const void *p : {dZ, dH, Z, F, gate, w_post, b_post, w_pre, (const void *)dX, (const void *)dF}) {
        if (!aligned(p, size)) return BSP_ERR_SHAPE;
        words &= aligned(p, 4);
    }
    for (const float *p : {stats_post, stats_pre})
        if (!aligned(p, 8)) return BSP_ERR_SHAPE;
    for (const float *p : {(const float *)dw_post, (const float *)db_post, (const float *)dw_pre, (const float *)db_pre, (const float *)dgate})
        if (!aligned(p, 4)) return BSP_ERR_SHAPE;
    Columns c = {(const float *)ws, {dw_post, db_post, dw_pre, db_pre, dgate}, 0, (int32_t)H, 0, gate ? (int32_t)gate_rows : 1};
    Deal d = {0, 0, 0, 0, 1, 0};
    if (T) {
        d = deal(T, H, gate ? gate_rows : 0);
        if (any) {
            if (!ws) return BSP_ERR_NULL;
            if (ws_bytes < (size_t)kSums * (size_t)d.wgs * (size_t)H * 4) return BSP_ERR_CAPACITY;
            if (!aligned(ws, 256)) return BSP_ERR_SHAPE;
        }
    }
    const bool direct = d.per_wg > 0;  // whole gate rows in a workgroup: written by the first launch
    if (T) {
        Backward a = {dZ, pre ? dH : nullptr, pre ? Z : nullptr, (post || dgate) ? F : nullptr, gate, w_post, b_post, w_pre, stats_post, stats_pre, dX, dF,
                      (float *)ws, direct ? dgate : nullptr, T, d.rows_per_gate, d.rows_per_piece, x_scale, (int32_t)H,
                      kind == BSP_NORM_RMS, norms, d.pieces, d.groups, d.per_wg, 0};
        for (int i = 0; i < kSums; ++i)
            if (c.out[i] && !(direct && i == kDgate)) a.want |= 1u << i;
        BSP_DISPATCH_DTYPE(dt, DT, {
            if (H <= 128) launch_backward<DT, 16, 1>(a, words, (unsigned)d.wgs, s);
            else if (of_16(H)) launch_backward<DT, 16, 2>(a, words, (unsigned)d.wgs, s);
            else if (H <= 512) launch_backward<DT, 64, 1>(a, words, (unsigned)d.wgs, s);
            else if (H <= 1024) launch_backward<DT, 64, 2>(a, words, (unsigned)d.wgs, s);
            else if (H <= 2048) launch_backward<DT, 256, 1>(a, words, (unsigned)d.wgs, s);
            else if (H <= 4096) launch_backward<DT, 256, 2>(a, words, (unsigned)d.wgs, s);
            else launch_backward<DT, 512, 2>(a, words, (unsigned)d.wgs, s);
        });
        if (int st = check_launch()) return st;
    }
    if (any) {  // (of no rows: zeros)
        c.wgs = d.wgs;
        c.pieces = d.pieces;
        if (direct) c.out[kDgate] = nullptr;
        const unsigned rows = kDgate + (c.out[kDgate] ? (unsigned)c.groups : 0u);
        block_norm_columns_kernel<<<dim3((unsigned)((H + 63) / 64), rows), 64 * kParts, 0, s>>>(c);
        return check_launch();
    }
    return BSP_OK;
}
