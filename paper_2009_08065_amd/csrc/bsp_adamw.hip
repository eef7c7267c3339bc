// One Adam step with decoupled weight decay over many tensors (bsp_adamw_step): the moments in fp32, or as 8-bit codes with a
// scale for every 256 elements.
//
// A model's step is hundreds of small tensors beside a few large ones, so the tensors' addresses go to the kernel as its
// arguments (kMaxTensors to a launch: nothing is copied to the device and a captured step needs no memory of its own) and a
// workgroup finds its tensor by its number.
//
// fp32 moments: the arithmetic of bsp_adam_step, one rounding per operation, the decay before the update.
// 8-bit moments: m and r = sqrt(v) are kept, r because the update divides by it: the codes of e4m3 span 2^18, those of v would
// span a range of gradients of 2^9 only.  They are rounded up or down at random in proportion to the distance: v changes by a
// thousandth in a step, a code by a sixteenth, and rounded to the nearest a moment would never move.  The random bits are mixed from the
// element's place, the step and the seed, so equal calls give equal bits.  A positive r does not become 0: the next step
// would divide by eps alone.
//
// Both are bound by memory.  Measured (MI355X, us): 302 M weights of 288 tensors with masks, 16-bit gradients and copies, fp32 moments 1830 (4.6 TB/s of
// 28 bytes a weight), 8-bit ones 1031 (4.7 of 16; some 90 vector instructions a weight, about what the memory leaves time for); 750000 weights 6.5.
#include "bsp_common.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <utility>

namespace bsp {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTensors = 40;            // 40 entries of 88 bytes: a launch has 4 KB of arguments
constexpr int kBlock = 256;                // elements of an 8-bit scale: one wavefront, 4 per lane
constexpr int64_t kMostWorkgroups = (int64_t)1 << 24;  // of a launch, which has less than 2^32 threads
constexpr int64_t kChunk8 = (kThreads / kWave) * kBlock;  // elements of a workgroup that has a block for each wavefront

struct Entry {
    float *w;
    const void *g;
    void *m, *v;
    float *scales;
    void *copy;
    const uint8_t *keep;
    const float *alpha;
    int64_t n;
    uint32_t N, R;
    float decay;  // lr * weight decay where the host knows lr, else the weight decay
};

struct Table {
    Entry e[kMaxTensors];
    uint32_t first[kMaxTensors];  // first workgroup of each tensor
    int32_t count;
};

struct Hyper {
    float lr, beta1, beta2, omb1, omb2, c1, c2, eps, lambda, log1, log2;
    uint32_t seed, t;
    const float *lr_t, *grad_scale;
};

// What a step has in common, and whether it is taken at all.
struct Step {
    float lr, c1, c2, gs;
    uint32_t salt;
};

__device__ __forceinline__ bool begin_step(const Hyper &h, Step &s) {
    s.gs = h.grad_scale ? *h.grad_scale : 1.0f;
    if (!(__builtin_fabsf(s.gs) <= 3.402823466e38f)) return false;
    uint32_t t = h.t;
    s.lr = h.lr;
    s.c1 = h.c1;
    s.c2 = h.c2;
    if (h.lr_t) {  // 1 - beta^t without the cancellation of the difference
        s.lr = h.lr_t[0];
        const float tf = h.lr_t[1];
        t = (uint32_t)tf;
        s.c1 = -expm1f(tf * h.log1);
        s.c2 = -expm1f(tf * h.log2);
    }
    s.salt = h.seed * 0x9E3779B1u + t * 0x6A09E667u;
    return true;
}

// The tensor of this workgroup (its index; uniform).
__device__ __forceinline__ int find_tensor(const Table &tab) {
    const int lane = threadIdx.x & 63;
    const bool before = lane < tab.count && tab.first[lane < kMaxTensors ? lane : 0] <= blockIdx.x;
    return __builtin_popcountll(__ballot(before)) - 1;
}

// Place of an element in the group arrays [M / R, N], carried along a walk in equal strides: row-block, row in it and column.
struct Groups {
    uint32_t col, row, N, R;
    int64_t block;
    __device__ __forceinline__ Groups(const Entry &e, int64_t base) : N(e.N), R(e.R) {
        const int64_t r = e.n <= 0xffffffffll ? (int64_t)((uint32_t)base / N) : base / N;
        block = r <= 0xffffffffll ? (int64_t)((uint32_t)r / R) : r / R;
        col = (uint32_t)(base - r * N);
        row = (uint32_t)(r - block * R);
    }
    // (a division where a stride passes several rows only: divisions for every element were a third of the masked kernel's instructions)
    __device__ __forceinline__ void advance(uint32_t stride) {
        col += stride;
        if (col < N) return;
        if (N >= stride) {
            col -= N;
            if (++row == R) {
                row = 0;
                ++block;
            }
        } else {
            const uint32_t q = col / N;
            col -= q * N;
            row += q;
            const uint32_t b = row / R;
            row -= b * R;
            block += b;
        }
    }
    __device__ __forceinline__ int64_t at() const { return block * N + col; }
};

__device__ __forceinline__ float update(float w, float m, float v, float lr, float c1, float c2, float eps) {
    const float mh = m / c1;
    const float vh = v / c2;
    const float num = lr * mh;
    const float den = __builtin_sqrtf(vh) + eps;
    const float q = num / den;
    return w - q;
}

template <int CDT>
__device__ __forceinline__ void store_copy(void *p, int64_t i, float v) {
    if (p) elem<CDT>::store(p, i, v);
}

// PER: elements of a thread, 256 apart.  Four for large models (302 M weights 1889 us, with eight 1974); two where the launch would have few workgroups (750000 weights of 12 tensors:
// 10.4 us with eight).
template <int GDT, int CDT, int PER>
__global__ __launch_bounds__(kThreads) void adamw32_kernel(Table tab, Hyper h) {
    Step s;
    if (!begin_step(h, s)) return;
    const int k = find_tensor(tab);
    const Entry &e = tab.e[k];
    const int64_t base = (int64_t)(blockIdx.x - tab.first[k]) * (kThreads * PER);
    float *w = e.w + base, *m = (float *)e.m + base, *v = (float *)e.v + base;
    const int64_t left = e.n - base;
    const bool grouped = e.keep || e.alpha;
    Groups groups(e, grouped ? base : 0);
    if (grouped) groups.advance(threadIdx.x);
    const float decay = h.lr_t ? s.lr * e.decay : e.decay;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const uint32_t i = j * kThreads + threadIdx.x;
        if (i >= left) break;
        const float w0 = w[i];
        float g = elem<GDT>::load(e.g, base + i);
        if (h.grad_scale) g = g * s.gs;
        int64_t at = 0;
        if (grouped) {
            at = groups.at();
            groups.advance(kThreads);
        }
        if (e.alpha) g = __builtin_fmaf(h.lambda * e.alpha[at], w0, g);
        const float t1 = h.beta1 * m[i];
        const float t2 = h.omb1 * g;
        const float mn = t1 + t2;
        const float t3 = h.beta2 * v[i];
        float t4 = h.omb2 * g;
        t4 = t4 * g;
        const float vn = t3 + t4;
        float wn = w0;
        if (decay != 0.0f) {
            const float d = decay * w0;
            wn = w0 - d;
        }
        wn = update(wn, mn, vn, s.lr, s.c1, s.c2, h.eps);
        if (e.keep && !e.keep[at]) wn = 0.0f;
        w[i] = wn;
        m[i] = mn;
        v[i] = vn;
        store_copy<CDT>(e.copy, base + i, wn);
    }
}

// ---- 8-bit moments ------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x = (x ^ (x >> 16)) * 0xBB67AE85u;
    x = (x ^ (x >> 15)) * 0x3C6EF373u;
    return x ^ (x >> 16);
}

// The largest of 64 lanes' values (all >= 0, as their bits, whose order is theirs), in every lane: within rows of 16 lanes and then across them,
// without LDS.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
    const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
    return x > y ? x : y;
}
__device__ __forceinline__ float wave_max(uint32_t x) {
    x = max_dpp<0x111, 0xf>(x);  // row_shr 1, 2, 4, 8: lane 15 of a row has the row's
    x = max_dpp<0x112, 0xf>(x);
    x = max_dpp<0x114, 0xf>(x);
    x = max_dpp<0x118, 0xf>(x);
    x = max_dpp<0x142, 0xa>(x);  // row_bcast 15 into rows 1 and 3, 31 into rows 2 and 3
    x = max_dpp<0x143, 0xc>(x);
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)x, 63));
}

// The square root to the nearest number: the instruction's is one of three neighbours, and the sign of s' s - v for the lower and the
// upper one says which.  (What is stored is a decision on r: with a root that is off by an ulp here and there, the same step elsewhere gives other codes.)
__device__ __forceinline__ float nearest_root(float v) {
    const float s = __builtin_amdgcn_sqrtf(v);
    const float down = __uint_as_float(__float_as_uint(s) - 1u), up = __uint_as_float(__float_as_uint(s) + 1u);
    float r = __builtin_fmaf(-down, s, v) <= 0.0f ? down : s;
    return __builtin_fmaf(-up, s, v) > 0.0f ? up : r;
}

// |y| <= 448 to one of the two codes' values next to it, up where what y has above the lower one and the 16 bits (of 2^16) make a whole step.
// From 2^-6 on the carry out of the 20 bits that the code does not have says so.  Below it a step is 2^-9, and a comparison decides (an addition
// would round, and one code in a million would differ from what it has to be); few values are so far below their block's largest, so that is
// looked for in a wavefront as a whole.
constexpr float kLeastNormal = 0.015625f;
__device__ __forceinline__ float round_normal(float a, uint32_t bits16) {
    return __uint_as_float((__float_as_uint(a) + (bits16 << 4)) & 0xfff00000u);
}
__device__ __forceinline__ float round_small(float a, uint32_t bits16) {
    const float t = a * 512.0f, whole = __builtin_floorf(t), missing = (float)(65536u - bits16) * 0x1p-16f;
    return (t - whole >= missing ? whole + 1.0f : whole) * 0x1p-9f;
}

// four values, each an e4m3 number, as codes
__device__ __forceinline__ uint32_t codes4(const float (&x)[4]) {
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], p, true);
}
template <int I>
__device__ __forceinline__ float value_of(uint32_t codes) {
    return __builtin_amdgcn_cvt_f32_fp8((int)codes, I);
}

// BLOCKS: blocks of a wavefront, one after the other: four for large models (302 M weights 1040 us, with one 1093), one where the launch would have
// few workgroups (750000 weights of 12 tensors 7.8, with four 9.3; 10 layers of width 142 21, 29).
template <int GDT, int CDT, int BLOCKS>
__global__ __launch_bounds__(kThreads) void adamw8_kernel(Table tab, Hyper h) {
    Step s;
    if (!begin_step(h, s)) return;
    const int k = find_tensor(tab);
    const Entry &e = tab.e[k];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t base = (int64_t)(blockIdx.x - tab.first[k]) * (BLOCKS * kChunk8) + wave * (BLOCKS * kBlock);
    const bool grouped = e.keep || e.alpha;
    Groups groups(e, grouped ? base : 0);
    if (grouped) groups.advance(4 * lane);
    const int64_t blocks = (e.n + kBlock - 1) / kBlock;
    const float decay = h.lr_t ? s.lr * e.decay : e.decay, rate = s.lr / s.c1, root = 1.0f / __builtin_sqrtf(s.c2);
    uint8_t *m8 = (uint8_t *)e.m, *v8 = (uint8_t *)e.v;
    for (int b = 0; b < BLOCKS; ++b) {
        const int64_t i0 = base + b * kBlock + 4 * lane, block = base / kBlock + b;
        if (block >= blocks) break;  // uniform in a wavefront
        const int have = e.n - i0 >= 4 ? 4 : (e.n > i0 ? (int)(e.n - i0) : 0);
        const bool four = have == 4;  // (loads and stores of several elements need no alignment here)
        float w[4] = {0, 0, 0, 0}, g[4] = {0, 0, 0, 0}, m[4], r[4];
        uint32_t mc = 0, vc = 0;
        if (four) {
            __builtin_memcpy(w, e.w + i0, 16);
            __builtin_memcpy(&mc, m8 + i0, 4);
            __builtin_memcpy(&vc, v8 + i0, 4);
            if constexpr (GDT == BSP_F32) {
                __builtin_memcpy(g, (const float *)e.g + i0, 16);
            } else {
                uint16_t c[4];
                __builtin_memcpy(c, (const uint16_t *)e.g + i0, 8);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[j] = elem<GDT>::load(&c[j], 0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < have) {
                    w[j] = e.w[i0 + j];
                    g[j] = elem<GDT>::load(e.g, i0 + j);
                    mc |= (uint32_t)m8[i0 + j] << (8 * j);
                    vc |= (uint32_t)v8[i0 + j] << (8 * j);
                }
        }
        const float sm = e.scales[block], sv = e.scales[blocks + block];
        const float m0[4] = {value_of<0>(mc), value_of<1>(mc), value_of<2>(mc), value_of<3>(mc)};
        const float r0[4] = {value_of<0>(vc), value_of<1>(vc), value_of<2>(vc), value_of<3>(vc)};
        uint32_t kept = 0xfu;
        float coef[4] = {0, 0, 0, 0};
        if (grouped) {
            Groups at = groups;
            groups.advance(kBlock);
            if (four && at.col + 4 <= at.N) {  // neighbours in the group arrays
                if (e.keep) {
                    uint32_t k4;
                    __builtin_memcpy(&k4, e.keep + at.at(), 4);
                    kept = ((k4 & 0xffu) != 0) | ((k4 & 0xff00u) != 0) << 1 | ((k4 & 0xff0000u) != 0) << 2 | ((k4 & 0xff000000u) != 0) << 3;
                }
                if (e.alpha) __builtin_memcpy(coef, e.alpha + at.at(), 16);
            } else if (have) {  // (a row ends among them, or the tensor: all places, then all loads)
                int64_t place[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    place[j] = j < have ? at.at() : place[0];
                    at.advance(1);
                }
                if (e.keep) {
                    uint8_t k[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) k[j] = e.keep[place[j]];
                    kept = 0u;
#pragma unroll
                    for (int j = 0; j < 4; ++j) kept |= (k[j] ? 1u : 0u) << j;
                }
                if (e.alpha)
#pragma unroll
                    for (int j = 0; j < 4; ++j) coef[j] = e.alpha[place[j]];
            }
        }
        uint32_t bits_m = 0, bits_r = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float x = g[j];
            if (h.grad_scale) x = x * s.gs;
            if (e.alpha) x = __builtin_fmaf(h.lambda * coef[j], w[j], x);
            m[j] = h.beta1 * (m0[j] * sm) + h.omb1 * x;
            const float ro = r0[j] * sv;
            const float v = h.beta2 * (ro * ro) + h.omb2 * x * x;
            r[j] = nearest_root(v);
            float wn = w[j];
            if (decay != 0.0f) {
                const float d = decay * wn;
                wn = wn - d;
            }
            // (in this grouping and with the instruction's reciprocal, 1 ulp: nine roundings of the update at most, the other kernel's five and a half)
            wn = wn - rate * m[j] * __builtin_amdgcn_rcpf(__builtin_fmaf(r[j], root, h.eps));
            w[j] = (kept >> j) & 1u ? wn : 0.0f;
            const uint32_t um = __float_as_uint(m[j]) & 0x7fffffffu, ur = __float_as_uint(r[j]);
            bits_m = bits_m > um ? bits_m : um;
            bits_r = bits_r > ur ? bits_r : ur;
        }
        const float top_m = wave_max(bits_m), top_r = wave_max(bits_r);
        // (2^-100: below it 448 / largest has no number, and such moments move nothing.  A block with a moment that is not finite starts afresh: a
        // scale of infinity would make all its other weights NaN in the next step, zeros of r alone would let m move them without bound.)
        const bool finite = top_m <= 3.402823466e38f && top_r <= 3.402823466e38f;
        const bool has_m = finite && top_m >= 0x1p-100f, has_r = finite && top_r >= 0x1p-100f;
        const float im = has_m ? 448.0f * (1.0f / top_m) : 0.0f, ir = has_r ? 448.0f * (1.0f / top_r) : 0.0f;
        uint32_t bits[4];
        float ym[4], yr[4];  // (y of m with its sign)
        bool small = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bits[j] = mix((uint32_t)(i0 + j) + s.salt);
            ym[j] = __builtin_fminf(__builtin_fmaxf(m[j] * im, -448.0f), 448.0f);
            yr[j] = __builtin_fminf(r[j] * ir, 448.0f);
            m[j] = round_normal(__builtin_fabsf(ym[j]), bits[j] & 0xffffu);
            r[j] = round_normal(yr[j], bits[j] >> 16);
            small |= __builtin_fminf(__builtin_fabsf(ym[j]), yr[j]) < kLeastNormal;
        }
        if (__ballot(small)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a = __builtin_fabsf(ym[j]);
                m[j] = a < kLeastNormal ? round_small(a, bits[j] & 0xffffu) : m[j];
                const float least = yr[j] > 0.0f ? __builtin_fmaxf(round_small(yr[j], bits[j] >> 16), 0x1p-9f) : 0.0f;
                r[j] = yr[j] < kLeastNormal ? least : r[j];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) m[j] = __builtin_copysignf(m[j], ym[j]);
        const uint32_t mn = codes4(m), vn = codes4(r);
        if (lane == 0) {
            e.scales[block] = has_m ? top_m * (1.0f / 448.0f) : 0.0f;
            e.scales[blocks + block] = has_r ? top_r * (1.0f / 448.0f) : 0.0f;
        }
        if (four) {
            __builtin_memcpy(e.w + i0, w, 16);
            __builtin_memcpy(m8 + i0, &mn, 4);
            __builtin_memcpy(v8 + i0, &vn, 4);
            if (e.copy) {
                const uint2 c = make_uint2(elem<CDT>::bits(w[0]) | (elem<CDT>::bits(w[1]) << 16), elem<CDT>::bits(w[2]) | (elem<CDT>::bits(w[3]) << 16));
                __builtin_memcpy((uint16_t *)e.copy + i0, &c, 8);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < have) {
                    e.w[i0 + j] = w[j];
                    m8[i0 + j] = (uint8_t)(mn >> (8 * j));
                    v8[i0 + j] = (uint8_t)(vn >> (8 * j));
                    store_copy<CDT>(e.copy, i0 + j, w[j]);
                }
        }
    }
}

template <int GDT, int CDT>
void launch(const Table &tab, const Hyper &h, unsigned wgs, int bits, int per, hipStream_t s) {
    if (bits == 8 && per == 4) adamw8_kernel<GDT, CDT, 4><<<wgs, kThreads, 0, s>>>(tab, h);
    else if (bits == 8) adamw8_kernel<GDT, CDT, 1><<<wgs, kThreads, 0, s>>>(tab, h);
    else if (per == 4) adamw32_kernel<GDT, CDT, 4><<<wgs, kThreads, 0, s>>>(tab, h);
    else adamw32_kernel<GDT, CDT, 2><<<wgs, kThreads, 0, s>>>(tab, h);
}

// Whether anything that the step writes shares memory: the same tensor listed twice, say, would be updated by two workgroups at once.
// 0 no, 1 yes, -1 no memory to find out.  Each kind in ascending order and apart from the others, as models allocate them or cut them out of buffers, is
// seen in one look; else all are sorted (us on the host, 12 and 288 tensors with copies: 0.25 and 5, sorted 1.2 and 45).
using Range = std::pair<uintptr_t, uintptr_t>;
constexpr int kWritten = 5;
inline Range written(const bsp_adamw_tensor &x, int kind, int bits) {
    const int64_t n = x.M * x.N;
    const void *at = nullptr;
    int64_t bytes = 0;
    switch (kind) {
        case 0: at = x.w, bytes = 4 * n; break;
        case 1: at = x.m, bytes = bits / 8 * n; break;
        case 2: at = x.v, bytes = bits / 8 * n; break;
        case 3: at = x.copy, bytes = 2 * n; break;
        default: at = bits == 8 ? x.scales : nullptr, bytes = (n + kBlock - 1) / kBlock * 8; break;
    }
    const uintptr_t a = reinterpret_cast<uintptr_t>(at);
    return {a, a ? a + (uintptr_t)bytes : a};  // (empty where there is none)
}

int overlapping(const bsp_adamw_tensor *x, int64_t count, int bits) {
    Range span[kWritten];
    bool apart = true;
    for (int k = 0; k < kWritten; ++k) {
        span[k] = {0, 0};
        for (int64_t i = 0; i < count; ++i) {
            const Range r = written(x[i], k, bits);
            if (r.first == r.second) continue;
            if (span[k].second == 0) span[k].first = r.first;
            apart &= r.first >= span[k].second;
            span[k].second = r.second;
        }
        for (int o = 0; o < k; ++o) apart &= span[o].second <= span[k].first || span[k].second <= span[o].first;
    }
    if (apart) return 0;
    Range *all = new (std::nothrow) Range[(size_t)(kWritten * count)];
    if (!all) return -1;
    int64_t n = 0;
    for (int k = 0; k < kWritten; ++k)
        for (int64_t i = 0; i < count; ++i) {
            const Range r = written(x[i], k, bits);
            if (r.first != r.second) all[n++] = r;
        }
    std::sort(all, all + n);
    int found = 0;
    for (int64_t i = 1; i < n; ++i) found |= all[i].first < all[i - 1].second;
    delete[] all;
    return found;
}

}  // namespace
}  // namespace bsp

using namespace bsp;

extern "C" int bsp_adamw_step(const bsp_adamw_tensor *tensors, int64_t count, int gdt, int cdt, int state_bits, double lambda, double lr,
                              double beta1, double beta2, double eps, int64_t t, uint32_t seed, const float *lr_t,
                              const float *grad_scale, void *stream) {
    if (count < 0 || (state_bits != 32 && state_bits != 8)) return BSP_ERR_SHAPE;
    if (count && !tensors) return BSP_ERR_NULL;
    if (!valid_dtype(gdt) || (cdt != BSP_BF16 && cdt != BSP_F16)) return BSP_ERR_DTYPE;
    if (!lr_t && t < 1) return BSP_ERR_SHAPE;
    const int64_t largest = state_bits == 32 ? kThreads * 4 : 4 * kChunk8;
    int64_t all = 0, most = 0;
    for (int64_t i = 0; i < count; ++i) {  // all of them before the first launch
        const bsp_adamw_tensor &x = tensors[i];
        if (x.M < 0 || x.N < 0 || x.N > 0x7fffffff || (x.M && x.N > 0x7fffffffffffll / x.M)) return BSP_ERR_SHAPE;
        if (x.M == 0 || x.N == 0) continue;
        if (!x.w || !x.g || !x.m || !x.v || (state_bits == 8 && !x.scales)) return BSP_ERR_NULL;
        if ((x.keep || x.alpha) && (x.R <= 0 || x.M % x.R != 0)) return BSP_ERR_SHAPE;
        const int64_t n = (x.M * x.N + largest - 1) / largest;
        if (n >= kMostWorkgroups) return BSP_ERR_SHAPE;
        all += n;
        most = n > most ? n : most;
        if (!aligned(x.w, 4) || !aligned(x.g, dtype_size(gdt)) || (state_bits == 32 && (!aligned(x.m, 4) || !aligned(x.v, 4))) ||
            !aligned(x.scales, 4) || !aligned(x.copy, 2) || !aligned(x.alpha, 4))
            return BSP_ERR_SHAPE;
    }
    if (const int shared = overlapping(tensors, count, state_bits)) return shared > 0 ? BSP_ERR_SHAPE : BSP_ERR_CAPACITY;
    // (a tensor beside very many small ones: its part of a launch has to stay below the most there are)
    const int per = all >= 1024 * ((count + kMaxTensors - 1) / kMaxTensors) || most >= kMostWorkgroups / 4 ? 4 : (state_bits == 32 ? 2 : 1);
    const int64_t chunk = per * (state_bits == 32 ? (int64_t)kThreads : kChunk8);
    Hyper h;
    h.lr = (float)lr;
    h.beta1 = (float)beta1;
    h.beta2 = (float)beta2;
    h.omb1 = (float)(1.0 - beta1);  // (of 0.999 in fp32 it would be 1.3e-5 off)
    h.omb2 = (float)(1.0 - beta2);
    h.c1 = (float)(1.0 - std::pow(beta1, (double)t));
    h.c2 = (float)(1.0 - std::pow(beta2, (double)t));
    h.eps = (float)eps;
    h.lambda = (float)lambda;
    h.log1 = (float)std::log(beta1);
    h.log2 = (float)std::log(beta2);
    h.seed = seed;
    h.t = (uint32_t)t;
    h.lr_t = lr_t;
    h.grad_scale = grad_scale;
    hipStream_t s = (hipStream_t)stream;
    Table tab;
    int64_t wgs = 0;
    tab.count = 0;
    auto flush = [&]() -> int {
        if (!tab.count) return BSP_OK;
        BSP_DISPATCH_DTYPE(gdt, GDT, {
            if (cdt == BSP_F16) launch<GDT, BSP_F16>(tab, h, (unsigned)wgs, state_bits, per, s);
            else launch<GDT, BSP_BF16>(tab, h, (unsigned)wgs, state_bits, per, s);
        });
        tab.count = 0;
        wgs = 0;
        return check_launch();
    };
    for (int64_t i = 0; i < count; ++i) {
        const bsp_adamw_tensor &x = tensors[i];
        const int64_t n = x.M * x.N;
        if (n == 0) continue;
        const int64_t need = (n + chunk - 1) / chunk;
        if (tab.count == kMaxTensors || wgs + need >= kMostWorkgroups)
            if (int st = flush()) return st;
        Entry &e = tab.e[tab.count];
        e.w = x.w;
        e.g = x.g;
        e.m = x.m;
        e.v = x.v;
        e.scales = x.scales;
        e.copy = x.copy;
        e.keep = x.keep;
        e.alpha = x.alpha;
        e.n = n;
        e.N = (uint32_t)x.N;
        e.R = (uint32_t)(x.R > 0 ? x.R : 1);
        e.decay = lr_t ? x.weight_decay : (float)(lr * (double)x.weight_decay);
        tab.first[tab.count++] = (uint32_t)wgs;
        wgs += need;
    }
    return flush();
}
