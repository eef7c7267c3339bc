// Products of 8-bit matrices: Y = act(A B^T + bias) + residual (bsp_matmul_fp8), and the layer on 16- or 32-bit inputs
// (bsp_linear_fp8).
//
// Both operands have 128-column segments of one power of two each (bsp_fp8.hip), so a step of 128 columns is two
// v_mfma_scale_f32_32x32x64 per 32 x 32 piece, which take the codes and, per lane, the biased exponents of the lane's row: the sums come
// out scaled, in fp32, without a vector instruction.
//
// That instruction (like the unscaled ones on 8-bit codes) brings the products of eight neighbouring columns to the largest one's exponent before it adds
// them and drops what is 14 binades below: 1.3e-5 of the result (2-norm, N(0, 1) operands) whatever the length, far below the rounding to 16
// bits and below that of the operands, but not fp32; of products that cancel it is the largest ones that the loss goes by.  So results in fp32 take the same
// codes through v_mfma_f32_32x32x16_bf16: a code times its scale is a bfloat16, the conversion applies it, and 6e-9 of the result is what is lost, at half the
// rate.  (Against 64 bits bf16 results are off by 1.66224e-3 in the 2-norm, by 1.66196e-3 where the sums are fp32: 8192 x 4096, K = 1024, GELU.)
//
// The roles: B's rows (output columns) are the instruction's rows, A's rows (tokens) its columns, so that a lane ends with groups of four
// consecutive outputs of one token.
//
// A workgroup owns 32 FB WB tokens x 32 FA WA outputs; both tiles go straight from memory to LDS, 128 bytes of a row at a time, two to four steps
// in turn.  A row's 16-byte pieces are rotated by half its number, which the loads bring about by what each lane asks for, so that
// the operand reads of 16 lanes meet all banks.
//
// Measured (MI355X, us): 16384 x 4096, K = 4096 225 to 235 (2.4 PFLOP/s), 8192 x 4096, K = 1024 44 (1.6), with GELU 55, 8192 x 1024, K = 4096 37
// (1.9); in fp32 4096 x 4096, K = 8192 200 (1.4 PFLOP/s), 1024 x 4096, K = 8192 66 to 68 (1.0); one token, 4096 x 1024 4.1 with its quantisation.
// What bounds the large ones: of 231 us in tiles of 256 x 256 182 are left without the loads (the matrix cores at the clock that their power leaves), 210
// without the LDS reads; tiles of 128 x 128 fall from 266 to 162 without the loads, 16 TB/s of them.  Halves of steps in a ring of four, read into
// registers ahead of the barrier, took 250, the first half of
// the next step read ahead of this step's last products 224: the caches' rows and the wait for them stay.
#include "bsp_common.h"
#include "bsp_fp8_device.h"
#include "bsp_mfma_device.h"
#include "bsp_tile_device.h"

namespace bsp {
namespace {

struct Product {
    const uint8_t *A, *SA, *B, *SB;
    const void *bias, *residual;
    void *Y;
    float *partial;  // [splits][T][M up to a multiple of 8] where the columns are split, else null
    int64_t T, M;
    int32_t steps, pitch, split_steps;  // steps of 128 columns; bytes of a row; steps of a split
    int32_t block, act;                 // B has a scale per 128 rows
};

__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }

__device__ __forceinline__ f32x16 mfma_scaled(i32x8 a, i32x8 b, f32x16 c, uint32_t sa, uint32_t sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, (int)sa, 0, (int)sb);
}

// Eight codes times their scale as bfloat16: exact for what is a whole multiple of 2^-133, its least number (only scales below 2^-124 have codes that are none).
__device__ __forceinline__ uint4 widen8(uint32_t lo, uint32_t hi, uint32_t scale) {
    const float f = __uint_as_float(scale << 23);  // (the conversion takes the exponent: 0 is 2^-127)
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, true)));
}

// The tile's place: workgroup ids go round the 8 XCDs; each XCD has an eighth of the tiles in the order of groups of kGroup token tiles that walk
// their output ranges.  (With whole token tiles for each XCD 88 tokens, two tiles, kept two of the eight busy.)
constexpr uint32_t kGroup = 4;

template <int DT, int FA, int FB, int WA, int WB, int NS>
__global__ __launch_bounds__(64 * WA * WB) void fp8_tile_kernel(Product p) {
    constexpr int kWaves = WA * WB, kThreads = 64 * kWaves;
    constexpr int TA = 32 * FA * WA, TB = 32 * FB * WB;  // outputs, tokens
    constexpr int kCodes = (TA + TB) * 128, kStage = kCodes + (TA + TB) * 4, kLoads = (TA + TB) / 8 / kWaves;
    constexpr int kPitch = TA + 4;  // floats of a token's row in the output pass
    static_assert((TA + TB) / 8 % kWaves == 0);
    extern __shared__ __align__(16) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int wa = wave % WA, wb = wave / WA;

    const uint32_t ranges = (uint32_t)((p.M + TA - 1) / TA), tiles = (uint32_t)((p.T + TB - 1) / TB);
    const uint32_t n = tiles * ranges, place = (blockIdx.x & 7) * ((n + 7) / 8) + (blockIdx.x >> 3);
    if (place >= n || (blockIdx.x >> 3) >= (n + 7) / 8) return;  // uniform: before any barrier
    const uint32_t group = place / (kGroup * ranges), in_group = place - group * kGroup * ranges;
    const uint32_t height = tiles - group * kGroup < kGroup ? tiles - group * kGroup : kGroup;
    const int64_t t0 = (int64_t)(group * kGroup + in_group % height) * TB, m0 = (int64_t)(in_group / height) * TA;
    const int first = blockIdx.y * p.split_steps, last = first + p.split_steps < p.steps ? first + p.split_steps : p.steps;

    // the loads of this wavefront: 8 rows each, first B's, then A's; a row past the end reads the last one
    const uint8_t *base[2] = {p.B + m0 * p.pitch, p.A + t0 * p.pitch};
    uint32_t at[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int r8 = wave * kLoads + i, op = 8 * r8 >= TA, r = 8 * r8 + (lane >> 3) - (op ? TA : 0);
        const int64_t left = op ? p.T - t0 : p.M - m0;
        const uint32_t row = r < left ? r : (uint32_t)(left - 1);
        at[i] = row * (uint32_t)p.pitch + ((((uint32_t)lane & 7) ^ ((r >> 1) & 7)) << 4);
    }
    // and 64 rows' scales to a piece (in tiles of fewer pieces than wavefronts several load the same one)
    constexpr int kScalePieces = (TA + TB) / 64, kScaleLoads = (kScalePieces + kWaves - 1) / kWaves;
    static_assert(TA % 64 == 0 && TB % 64 == 0);
    const uint8_t *scale_base[kScaleLoads];
    uint32_t scale_at[kScaleLoads], scale_lds[kScaleLoads];
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        const int piece = (wave * kScaleLoads + i) % kScalePieces, op = 64 * piece >= TA, r = 64 * piece + lane - (op ? TA : 0);
        const int64_t row0 = op ? t0 : m0, left = (op ? p.T : p.M) - row0, row = r < left ? r : left - 1;
        const bool blocks = !op && p.block;
        scale_base[i] = op ? p.SA + t0 * p.steps : p.SB + (blocks ? m0 / 128 : m0) * p.steps;
        scale_at[i] = (uint32_t)(blocks ? (m0 + row) / 128 - m0 / 128 : row) * (uint32_t)p.steps;
        scale_lds[i] = (uint32_t)(kCodes + piece * 256);
    }
    constexpr int kEach = kLoads + kScaleLoads;  // loads of a wavefront and step
    auto load_one = [&](auto which, int step, int slot) {
        constexpr int i = decltype(which)::value;
        if constexpr (i < kLoads) {
            const int r8 = wave * kLoads + i, op = 8 * r8 >= TA;
            load_to_lds(slot * kStage + r8 * 1024, base[op] + (int64_t)step * 128, at[i]);
        } else {
            load_bytes_to_lds(slot * kStage + scale_lds[i - kLoads], scale_base[i - kLoads] + step, scale_at[i - kLoads]);
        }
    };
    auto load = [&](int step, int slot) { static_for<0, kEach>([&](auto i) { load_one(i, step, slot); }); };
    f32x16 acc[FA][FB];
#pragma unroll
    for (int i = 0; i < FA; ++i)
#pragma unroll
        for (int j = 0; j < FB; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.0f;

    const uint32_t cell = (uint32_t)l32 * 128 + ((((uint32_t)half * 2) ^ ((l32 >> 1) & 7)) << 4);
    const uint32_t cell_a = cell + (uint32_t)(wa * FA) * 4096, cell_b = cell + TA * 128 + (uint32_t)(wb * FB) * 4096;
    auto operand = [&](uint32_t c, int slot, int f, int sub) {
        const uint8_t *q = smem + slot * kStage + f * 4096;
        const uint4 lo = *reinterpret_cast<const uint4 *>(q + (c ^ (sub << 6))), hi = *reinterpret_cast<const uint4 *>(q + (c ^ (sub << 6) ^ 16));
        return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
    };

    // the bias of the tile's outputs, one per thread, asked for before the operands
    static_assert(TA <= kThreads);
    float own_bias = 0.0f;
    if (p.bias && !p.partial && tid < TA) own_bias = elem<DT>::load(p.bias, m0 + tid < p.M ? m0 + tid : p.M - 1);
    static_for<0, NS - 1>([&](auto n) {
        if (first + n < last) load(first + n, n);  // uniform
    });
    const uint32_t scale_a = kCodes + (uint32_t)(wa * FA * 32 + l32) * 4, scale_b = kCodes + (uint32_t)(TA + wb * FB * 32 + l32) * 4;
    struct Operands {
        i32x8 a[FA], b[FB];
    };
    uint32_t sc[FA + FB];
    auto read_scales = [&](int slot) {
#pragma unroll
        for (int f = 0; f < FA + FB; ++f)
            sc[f] = *reinterpret_cast<const uint32_t *>(smem + slot * kStage + (f < FA ? scale_a + 128 * f : scale_b + 128 * (f - FA)));
    };
    auto read = [&](Operands &o, int slot, int sub) {
#pragma unroll
        for (int i = 0; i < FA; ++i) o.a[i] = operand(cell_a, slot, i, sub);
#pragma unroll
        for (int j = 0; j < FB; ++j) o.b[j] = operand(cell_b, slot, j, sub);
    };
    // The products of half a step; after each of them `between` may put something else: a step's loads in a row would hold up the next product, on
    // all wavefronts at once (fp32, 1024 x 4096, K = 8192 in tiles of 256: 4 % longer).
    constexpr int kProducts = FA * FB * (DT == BSP_F32 ? 4 : 1);
    auto multiply = [&](const Operands &o, auto between) {
        if constexpr (DT == BSP_F32) {
            // (the next 16 columns are widened between the products of these: 1024 x 4096, K = 8192 3 % shorter)
            uint4 wide[2][FA + FB];
            auto widen = [&](int to, int f, int k) {
                const i32x8 &x = f < FA ? o.a[f] : o.b[f - FA];
                wide[to][f] = widen8((uint32_t)x[2 * k], (uint32_t)x[2 * k + 1], sc[f]);
            };
            static_for<0, FA + FB>([&](auto f) { widen(0, f, 0); });
            static_for<0, 4>([&](auto kk) {
                constexpr int k = decltype(kk)::value;
                static_for<0, FA * FB>([&](auto n) {
                    constexpr int N = decltype(n)::value, i = N / FB, j = N % FB;
                    acc[i][j] = mfma32<BSP_BF16>(wide[k & 1][i], wide[k & 1][FA + j], acc[i][j]);
                    if constexpr (k < 3)
                        static_for<N * (FA + FB) / (FA * FB), (N + 1) * (FA + FB) / (FA * FB)>([&](auto f) { widen(1 - (k & 1), f, k + 1); });
                    between(std::integral_constant<int, k * FA * FB + N>{});
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
        } else {
            static_for<0, FA * FB>([&](auto n) {
                constexpr int i = decltype(n)::value / FB, j = decltype(n)::value % FB;
                acc[i][j] = mfma_scaled(o.a[i], o.b[j], acc[i][j], sc[i], sc[FA + j]);
                between(n);
            });
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto nothing = [](auto) {};
    // n others dealt evenly over the products
    auto dealt = [&](auto n, auto other) {
        return [=](auto product) {
            constexpr int N = decltype(n)::value, P = decltype(product)::value;
            static_for<P * N / kProducts, (P + 1) * N / kProducts>([&](auto o) { other(o); });
            __builtin_amdgcn_sched_barrier(0);
        };
    };
    using Others = std::integral_constant<int, kEach>;
    int slot = 0;
    if constexpr (NS == 2) {
        auto step = [&](int s, auto more) {
            wait_loads<0>();
            barrier();  // this step is in LDS, and nobody reads the other slot any more
            read_scales(slot);
            constexpr bool kBoth = DT != BSP_F32 || FA * FB < 8;  // both halves are read at once, where the registers have room for them
            Operands o[kBoth ? 2 : 1];
            read(o[0], slot, 0);
            if constexpr (kBoth) read(o[1], slot, 1);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (decltype(more)::value) multiply(o[0], dealt(Others{}, [&](auto i) { load_one(i, s + 1, slot ^ 1); }));
            else multiply(o[0], nothing);
            if constexpr (!kBoth) read(o[0], slot, 1);
            multiply(o[kBoth ? 1 : 0], nothing);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            slot ^= 1;
        };
        for (int s = first; s + 1 < last; ++s) step(s, std::true_type{});
        step(last - 1, std::false_type{});
    } else {
        // The first half of a step is read while the second half of the one before it is multiplied: a step is in LDS, for everybody, half a
        // step before its turn.
        Operands o[2];
        if (first + NS - 1 <= last) wait_loads<(NS - 2) * kEach>();
        else wait_loads<0>();
        barrier();
        read_scales(0);
        read(o[0], 0, 0);
        // (The products stay on their side of the barrier: the compiler would move them behind it, where everything waits for everything.)
        auto step = [&](int s, auto behind) {  // behind: whether all the steps that the ring has room for are behind this one
            constexpr bool kFull = decltype(behind)::value;
            const int next = slot == NS - 1 ? 0 : slot + 1, free = slot == 0 ? NS - 1 : slot - 1;
            read(o[1], slot, 1);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kFull) multiply(o[0], dealt(Others{}, [&](auto i) { load_one(i, s + NS - 1, free); }));
            else multiply(o[0], nothing);
            // the next step's loads are done where no more are left than those of the steps behind it
            wait_loads<kFull ? (NS - 2) * kEach : 0>();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            barrier();
            if (kFull || s + 1 < last) read(o[0], next, 0);
            __builtin_amdgcn_sched_barrier(0);
            multiply(o[1], nothing);
            if (kFull || s + 1 < last) read_scales(next);
            slot = next;
        };
        int s = first;
        for (; s + NS - 1 < last; ++s) step(s, std::true_type{});
        for (; s < last; ++s) step(s, std::false_type{});
    }

    // 16-bit results without a residual: finished where they are, rounded into a tile of all tokens in LDS, and out in whole rows.
    if constexpr (DT != BSP_F32) {
        constexpr int kRow = TA * 2 + 16;
        static_assert(TB * kRow <= NS * kStage);
        if (!p.partial && !p.residual) {
            float *biases = reinterpret_cast<float *>(smem + NS * kStage);
            if (tid < TA) biases[tid] = own_bias;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < FA; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = (wa * FA + i) * 32 + 8 * q + 4 * half;
                    const f32x4 b = *reinterpret_cast<const f32x4 *>(biases + c);
#pragma unroll
                    for (int j = 0; j < FB; ++j) {
                        float v[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            v[k] = acc[i][j][4 * q + k] + b[k];
                            if (p.act == BSP_ACT_GELU) v[k] = gelu_fit(v[k]);
                        }
                        *reinterpret_cast<uint2 *>(smem + ((wb * FB + j) * 32 + l32) * kRow + c * 2) = make_uint2(cvt_pk<DT>(v[0], v[1]), cvt_pk<DT>(v[2], v[3]));
                    }
                }
            __syncthreads();
            const int cols = p.M - m0 < TA ? (int)(p.M - m0) : TA, rows = p.T - t0 < TB ? (int)(p.T - t0) : TB;
            uint16_t *y = (uint16_t *)p.Y + t0 * p.M + m0;
            const bool vec = (p.M & 7) == 0 && (reinterpret_cast<uintptr_t>(p.Y) & 15) == 0;
            for (int n = tid; n < TB * (TA / 8); n += kThreads) {
                const int r = n / (TA / 8), c = n % (TA / 8) * 8;
                if (r >= rows || c >= cols) continue;
                const uint4 x = *reinterpret_cast<const uint4 *>(smem + r * kRow + c * 2);
                uint16_t *o = y + (int64_t)r * p.M + c;
                if (vec) {
                    store_y16(o, x);
                } else if (c + 8 <= cols) {
                    __builtin_memcpy(o, &x, 16);  // (stores need no alignment either)
                } else {
                    for (int k = 0; k < cols - c; ++k) o[k] = *reinterpret_cast<const uint16_t *>(smem + r * kRow + (c + k) * 2);
                }
            }
            return;
        }
    }
    // Else a pass of 32 WB tokens: sums to LDS, then whole rows leave with bias, activation and residual
    float *out = reinterpret_cast<float *>(smem);
    const bool vec = (p.M & 7) == 0;
    constexpr int kPiece = TA / 8;  // threads of a row
    const int c = (tid % kPiece) * 8;
    const int64_t m = m0 + c;
    const int cols = p.M - m > 8 ? 8 : (int)(p.M - m);
    float *biases = reinterpret_cast<float *>(smem + (NS * kStage > 32 * WB * kPitch * 4 ? NS * kStage : 32 * WB * kPitch * 4));
    if (tid < TA) biases[tid] = own_bias;
    __syncthreads();
    float bias[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) bias[k] = biases[c + k];
#pragma unroll
    for (int j = 0; j < FB; ++j) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4 *>(out + (wb * 32 + l32) * kPitch + (wa * FA + i) * 32 + 8 * q + 4 * half) =
                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __syncthreads();
        for (int r = tid / kPiece; r < 32 * WB; r += kThreads / kPiece) {
            const int64_t t = t0 + (r >> 5) * 32 * FB + 32 * j + (r & 31);
            if (t >= p.T || cols <= 0) continue;
            float v[8];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(out + r * kPitch + c + 4 * k);
#pragma unroll
                for (int n = 0; n < 4; ++n) v[4 * k + n] = x[n];
            }
            if (p.partial) {
                float *y = p.partial + ((int64_t)blockIdx.y * p.T + t) * ((p.M + 7) / 8 * 8) + m;
                *reinterpret_cast<float4 *>(y) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4 *>(y + 4) = make_float4(v[4], v[5], v[6], v[7]);
                continue;
            }
            const int64_t y = t * p.M + m;
            finish8<DT>(v, bias, p.act, p.residual, p.Y, y, vec, cols);
        }
    }
}

// ---- few tokens ---------------------------------------------------------------------------------------------------------------
// Up to 16 NT tokens: B is read once and straight into registers (a wavefront's 16 rows x 128 columns are whole lines), the steps of 128
// columns dealt to the workgroup's wavefronts in turn, whose sums meet in LDS in ascending order.  What bounds it is B's way from memory,
// and for small matrices the launch.
// RAW: the tokens come as they are and are quantised here, in registers, by every workgroup for itself: 32 values of a lane, four lanes to
// a segment.  That is less than a launch of its own.
constexpr int kFewWaves = 8;

template <int XDT>
__device__ __forceinline__ i32x8 quantise_segment(const void *X, int64_t at, int cols, uint32_t &e) {
    float v[32];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (cols >= 8 * (k + 1)) {
            load8<XDT>(X, at + 8 * k, v + 8 * k);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[8 * k + j] = 8 * k + j < cols ? elem<XDT>::load(X, at + 8 * k + j) : 0.0f;
        }
    }
    float m = 0.0f;
#pragma unroll
    for (int k = 0; k < 32; ++k) m = __builtin_fmaxf(m, magnitude(v[k]));
    if (XDT != BSP_F16) keep_below<32>(v, m);
    m = __builtin_fmaxf(m, __shfl_xor(m, 16));
    m = __builtin_fmaxf(m, __shfl_xor(m, 32));
    e = scale_exponent(m);
    const float s = inverse_scale(e);
    i32x8 c;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float y[4] = {s * v[4 * k], s * v[4 * k + 1], s * v[4 * k + 2], s * v[4 * k + 3]};
        c[k] = (int)codes4(y);
    }
    return c;
}

template <int DT, int NT, bool RAW>
__global__ __launch_bounds__(64 * kFewWaves) void fp8_few_kernel(Product p, const void *X, int64_t N) {
    __shared__ __align__(16) float sums[kFewWaves][NT * 16][20];  // (20: a token's 16 outputs and a gap, for the banks)
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int l16 = lane & 15, quarter = lane >> 4;
    const int64_t m0 = (int64_t)blockIdx.x * 16;
    const int64_t row = m0 + l16 < p.M ? m0 + l16 : p.M - 1;
    const uint8_t *b = p.B + row * p.pitch + 32 * quarter;
    const uint8_t *sb = p.SB + (p.block ? row / 128 : row) * p.steps;
    int64_t token[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) token[t] = 16 * t + l16 < p.T ? 16 * t + l16 : p.T - 1;

    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    u32x4 next0, next1;
    uint32_t next_e;
    auto ask = [&](int s) {
        next0 = *reinterpret_cast<const u32x4 *>(b + (int64_t)s * 128);
        next1 = *reinterpret_cast<const u32x4 *>(b + (int64_t)s * 128 + 16);
        next_e = sb[s];
    };
    ask(wave);  // (there are no more wavefronts than steps)
    // One tile of tokens: what the first output of this thread is finished with is on its way before the products (1 token, 4096 x 1024 4.7 us, 4.45;
    // two tiles 5.7, 5.95: their tokens' loads wait for these).
    constexpr bool kEarly = NT == 1;
    const bool mine = kEarly && (tid >> 4) < p.T && m0 + (tid & 15) < p.M;
    float bias = 0.0f, residual = 0.0f;
    if (mine && p.bias) bias = elem<DT>::load(p.bias, m0 + (tid & 15));
    if (mine && p.residual) residual = elem<DT>::load(p.residual, (tid >> 4) * p.M + m0 + (tid & 15));
    for (int s = wave; s < p.steps; s += waves) {
        const u32x4 w0 = next0, w1 = next1;
        const uint32_t es = next_e;
        if (s + waves < p.steps) ask(s + waves);
        const i32x8 w = {(int)w0[0], (int)w0[1], (int)w0[2], (int)w0[3], (int)w1[0], (int)w1[1], (int)w1[2], (int)w1[3]};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            i32x8 x;
            uint32_t e;
            if constexpr (RAW) {
                const int64_t k = (int64_t)s * 128 + 32 * quarter;
                x = quantise_segment<DT>(X, token[t] * N + k, N - k > 32 ? 32 : (int)(N - k), e);
            } else {
                const uint8_t *a = p.A + token[t] * p.pitch + (int64_t)s * 128 + 32 * quarter;
                const u32x4 x0 = *reinterpret_cast<const u32x4 *>(a), x1 = *reinterpret_cast<const u32x4 *>(a + 16);
                x = i32x8{(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], (int)x1[0], (int)x1[1], (int)x1[2], (int)x1[3]};
                e = p.SA[token[t] * p.steps + s];
            }
            if constexpr (DT == BSP_F32) {
#pragma unroll
                for (int k = 0; k < 8; k += 2)
                    acc[t] = mfma16<BSP_BF16>(widen8((uint32_t)w[k], (uint32_t)w[k + 1], es), widen8((uint32_t)x[k], (uint32_t)x[k + 1], e), acc[t]);
            } else {
                acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc[t], 0, 0, 0, (int)es, 0, (int)e);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4 *>(&sums[wave][16 * t + l16][4 * quarter]) = acc[t];
    __syncthreads();
    for (int i = tid; i < NT * 256; i += blockDim.x) {
        const int t = i >> 4, c = i & 15;
        const int64_t m = m0 + c;
        if (t >= p.T || m >= p.M) continue;
        float v = 0.0f;
        for (int w = 0; w < waves; ++w) v += sums[w][t][c];
        if (!kEarly || i != tid) {  // (where there are fewer threads than outputs)
            if (p.bias) bias = elem<DT>::load(p.bias, m);
            if (p.residual) residual = elem<DT>::load(p.residual, t * p.M + m);
        }
        if (p.bias) v += bias;
        if (p.act == BSP_ACT_GELU) v = gelu_fit(v);
        if (p.residual) v += residual;
        elem<DT>::store(p.Y, t * p.M + m, v);
    }
}

// The splits' sums, ascending, then bias, activation and residual.
template <int DT>
__global__ __launch_bounds__(256) void fp8_join_kernel(Product p, int splits) {
    const uint32_t per_row = (uint32_t)((p.M + 7) / 8), i = blockIdx.x * 256u + threadIdx.x;
    const uint32_t t = i / per_row, m = (i - t * per_row) * 8;
    if (t >= p.T) return;
    const int cols = p.M - m > 8 ? 8 : (int)(p.M - m);
    float v[8], bias[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        v[k] = 0.0f;
        bias[k] = p.bias && k < cols ? elem<DT>::load(p.bias, m + k) : 0.0f;
    }
    const float *x = p.partial + (int64_t)i * 8;
    const int64_t stride = p.T * per_row * 8;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const float4 a = *reinterpret_cast<const float4 *>(x + s * stride), b = *reinterpret_cast<const float4 *>(x + s * stride + 4);
        v[0] += a.x, v[1] += a.y, v[2] += a.z, v[3] += a.w, v[4] += b.x, v[5] += b.y, v[6] += b.z, v[7] += b.w;
    }
    finish8<DT>(v, bias, p.act, p.residual, p.Y, (int64_t)t * p.M + m, (p.M & 7) == 0, cols);
}

constexpr int64_t kFewTokens = 32;  // of fp8_few_kernel

// Whether its workgroups quantise the tokens themselves: where a wavefront has one step of it to do, or two for one tile of tokens.  (us, in
// one launch / in two: 1 token of 1024 columns, 4096 rows 4.1 / 5.3; 32 tokens 6.0 / 6.4; 1 token of 4096 columns 10.5 / 8.1, 32 tokens 18.4 / 12.8.)
bool quantised_inside(int64_t T, int64_t steps) { return T <= 16 ? steps <= 2 * kFewWaves : T <= kFewTokens && steps <= kFewWaves; }

struct Shape {
    int tile;    // 256, 128, 64; 127 and 63: 128 and 64 with their steps three and four deep in LDS; 0: few tokens
    int splits, split_steps;
};

// Rounds of `n` workgroups of which the compute units take `together` at once; in the last one up to 256 have a compute unit each and take
// `alone` of a round.
double rounds_of(double n, double together, double alone) {
    const double whole = __builtin_floor(n / together), left = n - whole * together;
    return left == 0.0 ? whole : whole + alone + (1.0 - alone) * (left > 256.0 ? (left - 256.0) / (together - 256.0) : 0.0);
}

// Microseconds of a product in `n` tiles (with the splits) of `steps` steps; fitted to 127 shapes of 33 to 16384 rows, 64 to 8192 outputs and 64 to
// 16384 columns, where the tile that is chosen takes 1 % longer than the best one in the mean (3 % at
// 115 others).  `wide`: fp32 results, whose instructions take
// twice as long.  A larger tile loads less for a product, but its workgroups leave compute units idle at the end of a round, and one of 256 x 256
// fills a compute unit, so that its epilogue (GELU: 8 us a round) hides nothing.  Two steps in LDS let two workgroups of 128 x 128 share a compute
// unit and wait for each other; with three a workgroup that is alone on it reads half a step ahead.  Measured, 256 / 128 / 127 / 64 / 63: 16384 x
// 4096, K = 4096 231 / 280 / 315 / 438 / 442; 8192 x 4096, K = 1024 44 / 44 / 62 / 66 / 82, with GELU 58 / 55 / 73 / 75 / 94; 2048 x 1024, K = 4096
// 49 / 28 / 20 / 22 / 18; 512 x 1024, K = 4096 49 / 28 / 19 / 21 / 11; 1024 x 4096, K = 8192 in fp32 147 / 75 / 66 / 82 / 84.  The estimates are of rounds that fill the
// chip: 4096 x 4096, K = 8192 in fp32 is one of 256 x 256 on all compute units and takes 199 (estimated 198); 64 or 128 such workgroups are faster, 147,
// but there smaller tiles are faster still.
double tile_us(int tile, double n, double steps, bool wide, bool gelu) {
    const double rounds = __builtin_ceil(n / 256.0);
    switch (tile) {
        case 256: return 4.0 + rounds * ((wide ? 2.95 : 1.46) * steps + 5.0 + (gelu ? 10.0 : 0.0));
        case 128: return 4.0 + rounds_of(n, 512.0, 0.6) * ((wide ? 2.1 : 0.98) * steps + 3.0 + (gelu ? 2.0 : 0.0));
        case 127: return 4.0 + rounds * ((wide ? 0.98 : n <= 256.0 ? 0.37 : 0.54) * steps + 2.7 + (gelu ? 1.0 : 0.0));
        case 64: return 4.0 + rounds_of(n, 1024.0, 0.42) * ((wide ? 1.28 : 0.8) * steps + 1.6 + (gelu ? 1.5 : 0.0));
        default:
            if (n <= 256.0) return 5.0 + (wide ? 0.49 : 0.215) * steps;
            return 4.0 + rounds_of(n, 512.0, 0.61) * ((wide ? 0.68 : 0.36) * steps + 2.2 + (gelu ? 0.5 : 0.0));
    }
}

// The tile, and into how many runs the steps are split where there are too few tiles for the compute units (256 x 256, K = 16384 in fp32: 60 us,
// 15.7 in eight runs; 1024 x 1024, K = 8192 34.9 and 30.5 in two).  A split costs a launch and its sums' way to memory and back.
Shape choose(int64_t T, int64_t M, int64_t steps, bool wide, bool gelu) {
    Shape best = {0, 1, (int)steps};
    if (T <= kFewTokens) return best;
    double least = 0.0;
    for (int tile : {256, 128, 127, 64, 63}) {
        const double side = (double)((tile + 1) / 2 * 2), n = __builtin_ceil((double)T / side) * __builtin_ceil((double)M / side);
        for (int k = 1; k <= 16; k *= 2) {
            if (k > 1 && (steps < 4 * k || n * k > 512.0)) break;
            const int64_t each = (steps + k - 1) / k;
            double us = tile_us(tile, n * k, (double)each, wide, gelu);
            if (k > 1) us += 4.7 + (double)T * (double)M * (8.0 * k + 4.0) / 4.3e6;
            if (least != 0.0 && us >= least) continue;
            least = us;
            best = {tile, (int)((steps + each - 1) / each), (int)each};
        }
    }
    return best;
}

template <int DT, int FA, int FB, int WA, int WB, int NS>
int launch_tile(const Product &p, int splits, hipStream_t s) {
    constexpr int TA = 32 * FA * WA, TB = 32 * FB * WB;
    constexpr size_t stages = NS * (size_t)(TA + TB) * 132, out = (size_t)32 * WB * (TA + 4) * 4, lds = (stages > out ? stages : out) + TA * 4;
    auto k = fp8_tile_kernel<DT, FA, FB, WA, WB, NS>;
    if (lds > 65536) {  // (asking again is harmless)
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) {
            set_last_hip_error((int)e);
            return BSP_ERR_HIP;
        }
    }
    const int64_t wgs = ((p.T + TB - 1) / TB * ((p.M + TA - 1) / TA) + 7) / 8 * 8;
    if (wgs * splits * (64 * WA * WB) >= ((int64_t)1 << 32)) return BSP_ERR_SHAPE;
    k<<<dim3((unsigned)wgs, (unsigned)splits), 64 * WA * WB, lds, s>>>(p);
    return check_launch();
}

template <int DT, bool RAW>
int launch_few(const Product &p, const void *X, int64_t N, hipStream_t s) {
    const unsigned grid = (unsigned)((p.M + 15) / 16), threads = 64u * (unsigned)(p.steps < kFewWaves ? p.steps : kFewWaves);
    if ((uint64_t)grid * threads >= ((uint64_t)1 << 32)) return BSP_ERR_SHAPE;
    if (p.T <= 16) fp8_few_kernel<DT, 1, RAW><<<grid, threads, 0, s>>>(p, X, N);
    else fp8_few_kernel<DT, 2, RAW><<<grid, threads, 0, s>>>(p, X, N);
    return check_launch();
}

template <int DT>
int launch_product(const Product &p, const Shape &c, hipStream_t s) {
    int st;
    if (c.tile == 0) return launch_few<DT, false>(p, nullptr, 0, s);
    if (c.tile == 256) st = launch_tile<DT, 2, 4, 4, 2, 2>(p, c.splits, s);
    else if (c.tile == 128) st = launch_tile<DT, 2, 1, 2, 4, 2>(p, c.splits, s);
    else if (c.tile == 127) st = launch_tile<DT, 2, 1, 2, 4, 3>(p, c.splits, s);
    else if (c.tile == 64) st = launch_tile<DT, 1, 1, 2, 2, 2>(p, c.splits, s);
    else st = launch_tile<DT, 1, 1, 2, 2, 4>(p, c.splits, s);
    if (st || c.splits == 1) return st;
    const int64_t n = p.T * ((p.M + 7) / 8);
    fp8_join_kernel<DT><<<(unsigned)((n + 255) / 256), 256, 0, s>>>(p, c.splits);
    return check_launch();
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }
int64_t steps_of(int64_t K) { return (K + 127) / 128; }

size_t partial_bytes(const Shape &c, int64_t T, int64_t M) {
    return c.splits > 1 ? (size_t)c.splits * (size_t)T * (size_t)((M + 7) / 8 * 8) * 4 : 0;
}

// (for either kind of result: the query does not know it)
size_t split_bytes(int64_t T, int64_t M, int64_t K) {
    size_t most = 0;
    for (bool wide : {false, true})
        for (bool gelu : {false, true}) {
            const size_t n = partial_bytes(choose(T, M, steps_of(K), wide, gelu), T, M);
            most = n > most ? n : most;
        }
    return most;
}

int check_sizes(int64_t T, int64_t M, int64_t K, int layout, int ydt, int act) {
    if (!valid_dtype(ydt) || (layout != BSP_FP8_ROW && layout != BSP_FP8_BLOCK) || (act != BSP_ACT_NONE && act != BSP_ACT_GELU)) return BSP_ERR_DTYPE;
    if (T < 0 || M <= 0 || K <= 0 || T >= ((int64_t)1 << 31) || M >= ((int64_t)1 << 31) || K > ((int64_t)1 << 23)) return BSP_ERR_SHAPE;
    return BSP_OK;
}

int product(const void *A, const uint8_t *SA, const void *B, const uint8_t *SB, int layout, int64_t T, int64_t M, int64_t K, const void *bias,
            int act, const void *residual, void *Y, int ydt, void *ws, size_t ws_bytes, hipStream_t s) {
    Shape c = choose(T, M, steps_of(K), ydt == BSP_F32, act == BSP_ACT_GELU);
    if (ws_bytes < partial_bytes(c, T, M)) c.splits = 1, c.split_steps = (int)steps_of(K);
    const Product p = {(const uint8_t *)A, SA, (const uint8_t *)B, SB, bias, residual, Y, c.splits > 1 ? (float *)ws : nullptr, T, M,
                       (int32_t)steps_of(K), (int32_t)(128 * steps_of(K)), c.split_steps, layout == BSP_FP8_BLOCK, act};
    switch (ydt) {
        case BSP_F32: return launch_product<BSP_F32>(p, c, s);
        case BSP_BF16: return launch_product<BSP_BF16>(p, c, s);
        default: return launch_product<BSP_F16>(p, c, s);
    }
}

}  // namespace
}  // namespace bsp

using namespace bsp;

extern "C" size_t bsp_matmul_fp8_workspace_bytes(int64_t T, int64_t M, int64_t K) {
    return T > 0 && !check_sizes(T, M, K, BSP_FP8_ROW, BSP_F32, BSP_ACT_NONE) ? split_bytes(T, M, K) : 0;
}

extern "C" int bsp_matmul_fp8(const void *A, const uint8_t *SA, const void *B, const uint8_t *SB, int b_layout, int64_t T, int64_t M, int64_t K,
                              const void *bias, int act, const void *residual, void *Y, int ydt, void *ws, size_t ws_bytes, void *stream) {
    if (int st = check_sizes(T, M, K, b_layout, ydt, act)) return st;
    if (T == 0) return BSP_OK;
    if (!A || !SA || !B || !SB || !Y) return BSP_ERR_NULL;
    const size_t size = dtype_size(ydt);
    if (!aligned(A, 16) || !aligned(B, 16) || !aligned(Y, size) || !aligned(bias, size) || !aligned(residual, size) || !aligned(ws, 256)) return BSP_ERR_SHAPE;
    if (!ws) ws_bytes = 0;
    if (ws_bytes && ws_bytes < split_bytes(T, M, K)) return BSP_ERR_CAPACITY;
    return product(A, SA, B, SB, b_layout, T, M, K, bias, act, residual, Y, ydt, ws, ws_bytes, (hipStream_t)stream);
}

extern "C" int bsp_matmul_fp8_form(int64_t T, int64_t M, int64_t K, int ydt, int act, int32_t *side, int32_t *depth, int32_t *splits) {
    if (int st = check_sizes(T, M, K, BSP_FP8_ROW, ydt, act)) return st;
    if (!side || !depth || !splits) return BSP_ERR_NULL;
    const Shape c = choose(T, M, steps_of(K), ydt == BSP_F32, act == BSP_ACT_GELU);
    *side = (c.tile + 1) / 2 * 2;
    *depth = c.tile == 0 ? 0 : c.tile == 127 ? 3 : c.tile == 63 ? 4 : 2;
    *splits = c.splits;
    return BSP_OK;
}

extern "C" size_t bsp_linear_fp8_workspace_bytes(int64_t T, int64_t M, int64_t N) {
    if (T <= 0 || check_sizes(T, M, N, BSP_FP8_ROW, BSP_F32, BSP_ACT_NONE)) return 0;
    if (quantised_inside(T, steps_of(N))) return 0;
    return up256((size_t)T * 128 * steps_of(N)) + up256((size_t)T * steps_of(N)) + split_bytes(T, M, N);
}

extern "C" int bsp_linear_fp8(const void *X, int xdt, int64_t T, int64_t M, int64_t N, const void *W, const uint8_t *SW, int w_layout,
                              const void *bias, int act, const void *residual, void *Y, void *ws, size_t ws_bytes, void *stream) {
    if (int st = check_sizes(T, M, N, w_layout, xdt, act)) return st;
    if (T == 0) return BSP_OK;
    const bool raw = quantised_inside(T, steps_of(N));
    if (!X || !W || !SW || !Y || (!raw && !ws)) return BSP_ERR_NULL;
    const size_t size = dtype_size(xdt);
    if (!aligned(X, size) || !aligned(W, 16) || !aligned(Y, size) || !aligned(bias, size) || !aligned(residual, size) || !aligned(ws, 256)) return BSP_ERR_SHAPE;
    if (ws_bytes < bsp_linear_fp8_workspace_bytes(T, M, N)) return BSP_ERR_CAPACITY;
    if (raw) {
        const Product p = {nullptr, nullptr, (const uint8_t *)W, SW, bias, residual, Y, nullptr, T, M, (int32_t)steps_of(N), (int32_t)(128 * steps_of(N)), 0,
                           w_layout == BSP_FP8_BLOCK, act};
        switch (xdt) {
            case BSP_F32: return launch_few<BSP_F32, true>(p, X, N, (hipStream_t)stream);
            case BSP_BF16: return launch_few<BSP_BF16, true>(p, X, N, (hipStream_t)stream);
            default: return launch_few<BSP_F16, true>(p, X, N, (hipStream_t)stream);
        }
    }
    uint8_t *codes = (uint8_t *)ws, *scales = codes + up256((size_t)T * 128 * steps_of(N)), *rest = scales + up256((size_t)T * steps_of(N));
    if (int st = bsp_fp8_quant(X, xdt, T, N, BSP_FP8_ROW, codes, scales, nullptr, nullptr, stream)) return st;
    return product(codes, scales, W, SW, w_layout, T, M, N, bias, act, residual, Y, xdt, rest, split_bytes(T, M, N), (hipStream_t)stream);
}
