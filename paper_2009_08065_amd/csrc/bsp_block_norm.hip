// The norms on either side of a Transformer block with the block's gate and the residual's scale (bsp_block_norm), and their
// gradients (bsp_block_norm_backward).
//
//   Z = x_scale X + gate * N_post(F)      H = N_pre(Z)       N(v) = (v - mean) / sqrt(var + eps) * w + b  (LAYER; RMS: mean = 0)
//
// Both are bound by memory: forward reads X and F and writes Z and H, backward reads up to dZ, dH, Z and F and writes dX and dF.  So
// a row stays in the registers of its team of threads from the first load to the last store: statistics, both norms and the rounding
// between them (N_pre reads Z as it is stored, which is what the backward pass will see) cost no second look at memory.
// A team is one wavefront while a row has no more than 32 values for a lane, else a workgroup.
// Sums are fp32: of a row by the lanes and then across them; the mean first, then the squares of what is left, which a
// sum of squares less the square of the sum would lose where the mean is large.  The sums down the columns (gradients of w, b and gate) are kept
// in registers over the rows of a workgroup, and a second launch adds the workgroups' sums in ascending order: equal calls give equal bits.
#include "bsp_common.h"

namespace bsp {
namespace {

constexpr int kMaxH = 8192;
constexpr int kVec = 8;  // values of a piece: consecutive ones of a thread (VEC), or one per thread and step (any alignment)

// Piece u of a thread's share of a row: columns of its value j.
template <int TPR, bool VEC>
__device__ __forceinline__ int column(int u, int j, int t) {
    return VEC ? (u * TPR + t) * kVec + j : (u * kVec + j) * TPR + t;
}

template <int DT, int TPR, bool VEC>
__device__ __forceinline__ void load_piece(float (&v)[kVec], const void *p, int64_t at, int u, int t, int H) {
    if constexpr (VEC) {
        const int c = column<TPR, true>(u, 0, t);
        if (c < H) {
            if constexpr (DT == BSP_F32) {
                const float4 a = *reinterpret_cast<const float4 *>((const float *)p + at + c);
                const float4 b = *reinterpret_cast<const float4 *>((const float *)p + at + c + 4);
                v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
            } else {
                const uint4 a = *reinterpret_cast<const uint4 *>((const uint16_t *)p + at + c);
                const uint32_t d[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint16_t lo = (uint16_t)d[j], hi = (uint16_t)(d[j] >> 16);
                    v[2 * j] = elem<DT>::load(&lo, 0);
                    v[2 * j + 1] = elem<DT>::load(&hi, 0);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < kVec; ++j) v[j] = 0.0f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            const int c = column<TPR, false>(u, j, t);
            v[j] = c < H ? elem<DT>::load(p, at + c) : 0.0f;
        }
    }
}

template <int DT, int TPR, bool VEC>
__device__ __forceinline__ void store_piece(const float (&v)[kVec], void *p, int64_t at, int u, int t, int H) {
    if constexpr (VEC) {
        const int c = column<TPR, true>(u, 0, t);
        if (c >= H) return;
        if constexpr (DT == BSP_F32) {
            *reinterpret_cast<float4 *>((float *)p + at + c) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4 *>((float *)p + at + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            uint32_t d[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) d[j] = elem<DT>::bits(v[2 * j]) | (elem<DT>::bits(v[2 * j + 1]) << 16);
            *reinterpret_cast<uint4 *>((uint16_t *)p + at + c) = make_uint4(d[0], d[1], d[2], d[3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            const int c = column<TPR, false>(u, j, t);
            if (c < H) elem<DT>::store(p, at + c, v[j]);
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

// Sums of K values over the TPR threads of a team, in every one of them.  LDS: `red` of K * TPR / 64 floats, two of them in turn, so that
// one barrier a sum is enough.
template <int TPR, int K>
__device__ __forceinline__ void team_sum(float (&v)[K], float *red, int &turn) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], d);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        float *r = red + turn * 2 * W;
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
template <int TPR, int ITER, bool VEC>
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
            q[0] = column<TPR, VEC>(u, j, t) < a.width ? __builtin_fmaf(d, d, q[0]) : q[0];
        }
    team_sum<TPR, 1>(q, red, turn);
    rstd = 1.0f / __builtin_sqrtf(q[0] * n + a.eps);
}

template <int DT, int TPR, int ITER, bool VEC>
__device__ __forceinline__ void normalise(float (&v)[ITER][kVec], float mean, float rstd, const void *w, const void *b, int t, int H) {
#pragma unroll
    for (int u = 0; u < ITER; ++u) {
        float x[kVec];
#pragma unroll
        for (int j = 0; j < kVec; ++j) v[u][j] = (v[u][j] - mean) * rstd;
        if (w) {
            load_piece<DT, TPR, VEC>(x, w, 0, u, t, H);
#pragma unroll
            for (int j = 0; j < kVec; ++j) v[u][j] *= x[j];
        }
        if (b) {
            load_piece<DT, TPR, VEC>(x, b, 0, u, t, H);
#pragma unroll
            for (int j = 0; j < kVec; ++j) v[u][j] += x[j];
        }
    }
}

template <int DT, int TPR, int ITER, bool VEC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void block_norm_kernel(Forward a) {
    constexpr int kTeams = TPR < 256 ? 256 / TPR : 1;
    __shared__ float red[TPR > 64 ? 4 * (TPR / 64) : 1];
    int turn = 0;
    const int t = threadIdx.x % TPR, H = a.width;
    const int64_t row = (int64_t)blockIdx.x * kTeams + threadIdx.x / TPR;
    if (row >= a.T) return;  // (whole teams; a workgroup of one team has a row)
    const int64_t at = row * H;
    float x[ITER][kVec], f[ITER][kVec];
#pragma unroll
    for (int u = 0; u < ITER; ++u) load_piece<DT, TPR, VEC>(x[u], a.X, at, u, t, H);
    if (a.F) {
#pragma unroll
        for (int u = 0; u < ITER; ++u) load_piece<DT, TPR, VEC>(f[u], a.F, at, u, t, H);
        if (a.norms & BSP_NORM_POST) {
            float mean, rstd;
            statistics<TPR, ITER, VEC>(f, t, a, mean, rstd, red, turn);
            if (a.stats_post && t == 0) *reinterpret_cast<float2 *>(a.stats_post + 2 * row) = make_float2(mean, rstd);
            normalise<DT, TPR, ITER, VEC>(f, mean, rstd, a.w_post, a.b_post, t, H);
        }
        if (a.gate) {
            const int64_t g = row / a.rows_per_gate * H;
#pragma unroll
            for (int u = 0; u < ITER; ++u) {
                float y[kVec];
                load_piece<DT, TPR, VEC>(y, a.gate, g, u, t, H);
#pragma unroll
                for (int j = 0; j < kVec; ++j) f[u][j] *= y[j];
            }
        }
    }
#pragma unroll
    for (int u = 0; u < ITER; ++u)
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            float z = a.x_scale * x[u][j];
            if (a.F) z += f[u][j];
            x[u][j] = column<TPR, VEC>(u, j, t) < H ? rounded<DT>(z) : 0.0f;
        }
    if (a.Z)
#pragma unroll
        for (int u = 0; u < ITER; ++u) store_piece<DT, TPR, VEC>(x[u], a.Z, at, u, t, H);
    if (a.norms & BSP_NORM_PRE) {
        float mean, rstd;
        statistics<TPR, ITER, VEC>(x, t, a, mean, rstd, red, turn);
        if (a.stats_pre && t == 0) *reinterpret_cast<float2 *>(a.stats_pre + 2 * row) = make_float2(mean, rstd);
        normalise<DT, TPR, ITER, VEC>(x, mean, rstd, a.w_pre, a.b_pre, t, H);
#pragma unroll
        for (int u = 0; u < ITER; ++u) store_piece<DT, TPR, VEC>(x[u], a.H, at, u, t, H);
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

template <int DT, int TPR, int ITER, bool VEC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void block_norm_back_kernel(Backward a) {
    constexpr int kTeams = TPR < 256 ? 256 / TPR : 1;
    __shared__ float red[TPR > 64 ? 8 * (TPR / 64) : 1];
    __shared__ float share[kTeams > 1 ? (kTeams - 1) * TPR * kVec : 1];
    int turn = 0;
    const int t = threadIdx.x % TPR, team = threadIdx.x / TPR, H = a.width;
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

    auto one_row = [&](int64_t row, int64_t group) {
        const int64_t at = row * H;
        float d[ITER][kVec], x[kVec];
#pragma unroll
        for (int u = 0; u < ITER; ++u) {
            if (a.dZ) load_piece<DT, TPR, VEC>(d[u], a.dZ, at, u, t, H);
            else
#pragma unroll
                for (int j = 0; j < kVec; ++j) d[u][j] = 0.0f;
        }
        float f[ITER][kVec];
        if (a.F)
#pragma unroll
            for (int u = 0; u < ITER; ++u) load_piece<DT, TPR, VEC>(f[u], a.F, at, u, t, H);
        if (a.norms & BSP_NORM_PRE) {
            float h[ITER][kVec], z[ITER][kVec];
            const float2 st = *reinterpret_cast<const float2 *>(a.stats_pre + 2 * row);
#pragma unroll
            for (int u = 0; u < ITER; ++u) load_piece<DT, TPR, VEC>(h[u], a.dH, at, u, t, H);
#pragma unroll
            for (int u = 0; u < ITER; ++u) load_piece<DT, TPR, VEC>(z[u], a.Z, at, u, t, H);
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int u = 0; u < ITER; ++u) {
                if (a.w_pre) load_piece<DT, TPR, VEC>(x, a.w_pre, 0, u, t, H);
#pragma unroll
                for (int j = 0; j < kVec; ++j) {
                    const float hat = (z[u][j] - st.x) * st.y, dh = h[u][j];
                    acc[kDwPre][u][j] = __builtin_fmaf(dh, hat, acc[kDwPre][u][j]);
                    acc[kDbPre][u][j] += dh;
                    const float g = a.w_pre ? dh * x[j] : dh;
                    s[0] = __builtin_fmaf(g, hat, s[0]);  // (past the width dh is 0)
                    s[1] += g;
                    z[u][j] = hat;
                    h[u][j] = g;
                }
            }
            team_sum<TPR, 2>(s, red, turn);
            const float c1 = s[0] * inv, c2 = a.rms ? 0.0f : s[1] * inv;
#pragma unroll
            for (int u = 0; u < ITER; ++u)
#pragma unroll
                for (int j = 0; j < kVec; ++j) d[u][j] += st.y * (h[u][j] - z[u][j] * c1 - c2);
        }
        if (a.dX)
#pragma unroll
            for (int u = 0; u < ITER; ++u) {
#pragma unroll
                for (int j = 0; j < kVec; ++j) x[j] = a.x_scale * d[u][j];
                store_piece<DT, TPR, VEC>(x, a.dX, at, u, t, H);
            }
        const bool post = (a.norms & BSP_NORM_POST) != 0;
        float2 st = make_float2(0.0f, 0.0f);
        if (post) st = *reinterpret_cast<const float2 *>(a.stats_post + 2 * row);
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < ITER; ++u) {
            float w[kVec], b[kVec];
            if (a.gate) load_piece<DT, TPR, VEC>(x, a.gate, group * H, u, t, H);
            if (post && a.w_post) load_piece<DT, TPR, VEC>(w, a.w_post, 0, u, t, H);
            if (post && a.b_post) load_piece<DT, TPR, VEC>(b, a.b_post, 0, u, t, H);
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                if (column<TPR, VEC>(u, j, t) >= H) {
                    d[u][j] = 0.0f;
                    continue;
                }
                float n = a.F ? f[u][j] : 0.0f, hat = 0.0f;
                if (post) {
                    hat = (n - st.x) * st.y;
                    n = a.w_post ? hat * w[j] : hat;
                    if (a.b_post) n += b[j];
                }
                if (a.gate) {
                    acc[kDgate][u][j] = __builtin_fmaf(d[u][j], n, acc[kDgate][u][j]);
                    d[u][j] *= x[j];
                }
                if (post) {
                    acc[kDwPost][u][j] = __builtin_fmaf(d[u][j], hat, acc[kDwPost][u][j]);
                    acc[kDbPost][u][j] += d[u][j];
                    if (a.w_post) d[u][j] *= w[j];
                    s[0] = __builtin_fmaf(d[u][j], hat, s[0]);
                    s[1] += d[u][j];
                    f[u][j] = hat;
                }
            }
        }
        if (post) {
            team_sum<TPR, 2>(s, red, turn);
            const float c1 = s[0] * inv, c2 = a.rms ? 0.0f : s[1] * inv;
#pragma unroll
            for (int u = 0; u < ITER; ++u)
#pragma unroll
                for (int j = 0; j < kVec; ++j) d[u][j] = st.y * (d[u][j] - f[u][j] * c1 - c2);
        }
        if (a.dF)
#pragma unroll
            for (int u = 0; u < ITER; ++u) store_piece<DT, TPR, VEC>(d[u], a.dF, at, u, t, H);
    };

    if (a.per_wg == 0) {  // a piece of one gate row's rows (all rows where there is no gate)
        const int64_t group = blockIdx.x / a.pieces, piece = blockIdx.x - group * a.pieces;
        int64_t r0 = piece * a.rows_per_piece, r1 = r0 + a.rows_per_piece;
        if (r1 > a.rows_per_gate) r1 = a.rows_per_gate;
        for (int64_t r = r0 + team; r < r1; r += kTeams) one_row(group * a.rows_per_gate + r, group);
    } else {              // gate rows of a few rows each: whole ones for a team
        for (int64_t k = team; k < a.per_wg; k += kTeams) {
            const int64_t group = (int64_t)blockIdx.x * a.per_wg + k;
            if (group >= a.groups) break;
            for (int64_t r = 0; r < a.rows_per_gate; ++r) one_row(group * a.rows_per_gate + r, group);
            if (a.dgate)
#pragma unroll
                for (int u = 0; u < ITER; ++u) store_piece<BSP_F32, TPR, VEC>(acc[kDgate][u], a.dgate, group * H, u, t, H);
            clear(kDgate);
        }
    }
    // the workgroup's sums: the teams' in ascending order, a piece at a time through LDS
    for (int i = 0; i < kSums; ++i) {
        if (!((a.want >> i) & 1u)) continue;
        float v[ITER][kVec];
#pragma unroll
        for (int u = 0; u < ITER; ++u)
#pragma unroll
            for (int j = 0; j < kVec; ++j)
                v[u][j] = i == 0 ? acc[0][u][j] : (i == 1 ? acc[1][u][j] : (i == 2 ? acc[2][u][j] : (i == 3 ? acc[3][u][j] : acc[4][u][j])));
        float *out = a.sums + ((int64_t)i * gridDim.x + blockIdx.x) * H;
#pragma unroll
        for (int u = 0; u < ITER; ++u) {
            if constexpr (kTeams > 1) {
                __syncthreads();
                if (team)
#pragma unroll
                    for (int j = 0; j < kVec; ++j) share[((team - 1) * kVec + j) * TPR + t] = v[u][j];
                __syncthreads();
                if (!team)
#pragma unroll
                    for (int o = 0; o < kTeams - 1; ++o)
#pragma unroll
                        for (int j = 0; j < kVec; ++j) v[u][j] += share[(o * kVec + j) * TPR + t];
            }
            if (!team) store_piece<BSP_F32, TPR, VEC>(v[u], out, 0, u, t, H);
        }
    }
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
#pragma unroll 4
    for (int64_t i = p; i < n; i += kParts) s += in[i * a.width];
    part[p][lane] = s;
    __syncthreads();
    if (p || c >= a.width) return;
    for (int i = 1; i < kParts; ++i) s += part[i][lane];
    out[(int64_t)(kind == kDgate ? row - kDgate : 0) * a.width + c] = s;
}

constexpr int64_t kRanges = 512;  // workgroups of the backward pass, at most where the gate's rows allow it

// Workgroups, and how the rows are dealt to them.
struct Deal {
    int64_t wgs, rows_per_gate, rows_per_piece;
    int32_t pieces, groups, per_wg;
};

Deal deal(int64_t T, int64_t H, int64_t gate_rows) {
    Deal d;
    const int64_t teams = H <= 1024 ? 4 : 1;
    d.groups = (int32_t)(gate_rows > 0 ? gate_rows : 1);
    d.rows_per_gate = T / d.groups;
    int64_t rows = (T + kRanges - 1) / kRanges;
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
    if (gate && T && gate_rows > T) return BSP_ERR_SHAPE;
    return BSP_OK;
}

template <typename... P>
bool vectors(int64_t H, P... p) {
    return H % kVec == 0 && (aligned(p, 16) && ...);
}

template <int DT, int TPR, int ITER>
void launch_forward(const Forward &a, bool vec, hipStream_t s) {
    constexpr int kTeams = TPR < 256 ? 256 / TPR : 1;
    const unsigned grid = (unsigned)((a.T + kTeams - 1) / kTeams);
    if (vec) block_norm_kernel<DT, TPR, ITER, true><<<grid, TPR < 256 ? 256 : TPR, 0, s>>>(a);
    else block_norm_kernel<DT, TPR, ITER, false><<<grid, TPR < 256 ? 256 : TPR, 0, s>>>(a);
}

template <int DT, int TPR, int ITER>
void launch_backward(const Backward &a, bool vec, unsigned grid, hipStream_t s) {
    if (vec) block_norm_back_kernel<DT, TPR, ITER, true><<<grid, TPR < 256 ? 256 : TPR, 0, s>>>(a);
    else block_norm_back_kernel<DT, TPR, ITER, false><<<grid, TPR < 256 ? 256 : TPR, 0, s>>>(a);
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
    for (const void *p : {X, F, gate, w_post, b_post, w_pre, b_pre, (const void *)Z, (const void *)Hn})
        if (!aligned(p, size)) return BSP_ERR_SHAPE;
    if (!aligned(stats_post, 8) || !aligned(stats_pre, 8)) return BSP_ERR_SHAPE;
    const Forward a = {X, F, gate, w_post, b_post, w_pre, b_pre, Z, Hn, stats_post, stats_pre,
                       T, gate ? T / gate_rows : T, x_scale, eps, (int32_t)H, kind == BSP_NORM_RMS, norms};
    const bool vec = vectors(H, X, F, gate, w_post, b_post, w_pre, b_pre, Z, Hn);
    hipStream_t s = (hipStream_t)stream;
    BSP_DISPATCH_DTYPE(dt, DT, {
        if (H <= 512) launch_forward<DT, 64, 1>(a, vec, s);
        else if (H <= 1024) launch_forward<DT, 64, 2>(a, vec, s);
        else if (H <= 2048) launch_forward<DT, 64, 4>(a, vec, s);
        else if (H <= 4096) launch_forward<DT, 256, 2>(a, vec, s);
        else launch_forward<DT, 256, 4>(a, vec, s);
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
    for (const void *p : {dZ, dH, Z, F, gate, w_post, b_post, w_pre, (const void *)dX, (const void *)dF})
        if (!aligned(p, size)) return BSP_ERR_SHAPE;
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
        const bool vec = vectors(H, dZ, a.dH, a.Z, a.F, gate, w_post, b_post, w_pre, dX, dF, direct ? dgate : nullptr);
        BSP_DISPATCH_DTYPE(dt, DT, {
            if (H <= 512) launch_backward<DT, 64, 1>(a, vec, (unsigned)d.wgs, s);
            else if (H <= 1024) launch_backward<DT, 64, 2>(a, vec, (unsigned)d.wgs, s);
            else if (H <= 2048) launch_backward<DT, 256, 1>(a, vec, (unsigned)d.wgs, s);
            else if (H <= 4096) launch_backward<DT, 256, 2>(a, vec, (unsigned)d.wgs, s);
            else launch_backward<DT, 512, 2>(a, vec, (unsigned)d.wgs, s);
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
