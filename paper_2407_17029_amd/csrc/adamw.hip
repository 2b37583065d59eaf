// The optimizer's step over many tensors at once: the list on the device, the norm of all gradients, and AdamW with moments in
// 32 or 8 bits (qblora_adamw_plan, qblora_grad_norm, qblora_adamw_step; the formulas stand in include/qblora.h).
//
// Bound by HBM: a step reads every gradient, moment and weight once and writes them once, the norm in front of it reads the gradients
// once more.  120 million elements in 84 tensors, moments in 8 bits, fp32 masters and bf16 copies (18 bytes an element): the step 378 us,
// 5.7 TB/s, the norm 95 to 127 + 5; 5 million in 14 tensors with moments in 32 bits (30 bytes): 23 us and 5 + 2.  Without masters (12 and 24
// bytes) 318 us (4.5 TB/s) and 20.  With step and rate on the device every thread forms the corrections' powers in 64 bits: 400 to 412 us
// and 25.  Element by element with pointers that might have been LDS ones the step took 784 and 39 us.
#include <algorithm>

#include "adapters.h"

namespace qblora {

namespace {

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t bf16x4_at_any __attribute__((ext_vector_type(2), aligned(2)));

constexpr int kThreads = 256, kMomentBlock = 256;

// ---- the list ----------------------------------------------------------------------------------------------------

__global__ __launch_bounds__(256) void k_adamw_plan(PlanDesc d, int64_t units) {
    if (blockIdx.x == 0 && (int)threadIdx.x < d.n) d.out[threadIdx.x] = d.entry[threadIdx.x];
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
        int i = 0;
        while (i + 1 < d.n && d.entry[i + 1].first_unit <= u) ++i;         // the last that begins here or before: empty ones are passed
        d.units[u] = {d.first + i, (int32_t)(u - d.entry[i].first_unit)};
    }
}

// ---- the norm ----------------------------------------------------------------------------------------------------
//
// Squares of fp32 numbers are exact in fp64, where they are added up: the result is the same number, to fp32's precision,
// whatever the order, and the order is fixed all the same.
//
// Squares of units from, from + step, ... as far as thread t of 256 reads them
__device__ __forceinline__ double squares(const PlanEntry* entries, const PlanUnit* units, int64_t n_units, int64_t from, int64_t step, int t) {
    double sum = 0.0;
    constexpr int kLoads = kUnit / (4 * kThreads);
    // where a unit lies is looked up while the one before it is on its way
    struct Piece { const __attribute__((address_space(1))) float* grad; int n; };
    auto piece = [&](int64_t u) __attribute__((always_inline)) {
        const PlanUnit unit = units[min(u, n_units - 1)];
        return Piece{in_memory(entries[unit.tensor].grad) + (int64_t)unit.index * kUnit,
                     (int)min((int64_t)kUnit, entries[unit.tensor].n - (int64_t)unit.index * kUnit)};
    };
    Piece now = piece(from);
    for (int64_t u = from; u < n_units; u += step) {
        if (now.n == kUnit) {
            f32x4_any v[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) v[i] = *(const __attribute__((address_space(1))) f32x4_any*)(now.grad + 4 * (t + i * kThreads));
            now = piece(u + step);
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += (double)v[i][j] * v[i][j];
            continue;
        }
        float v[4 * kLoads];                                                   // behind the end the last element once more, not counted
#pragma unroll
        for (int i = 0; i < 4 * kLoads; ++i) v[i] = now.grad[min(t + i * kThreads, now.n - 1)];
        const int n = now.n;
        now = piece(u + step);
#pragma unroll
        for (int i = 0; i < 4 * kLoads; ++i)
            if (t + i * kThreads < n) sum += (double)v[i] * v[i];
    }
    return sum;
}

// The sum over a workgroup, in its first thread; `slots`: one number a wave
__device__ __forceinline__ double group_sum(double v, double* slots) {
    for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    if (threadIdx.x == 0)
        for (int i = 0; i < (int)(blockDim.x >> 6); ++i) v += slots[i];
    return v;
}
__device__ __forceinline__ void write_norm(double sum, double max_norm, float* out) {
    const float norm = (float)__dsqrt_rn(sum);
    const double factor = max_norm / (__dsqrt_rn(sum) + 1e-6);
    out[0] = norm;
    out[1] = isfinite(norm) ? (float)(factor < 1.0 ? factor : 1.0) : __uint_as_float(0x7fc00000u);
}

__global__ __launch_bounds__(kThreads) void k_norm_parts(const PlanEntry* entries, const PlanUnit* units, int64_t n_units, double* part) {
    __shared__ double slots[kThreads / 64];
    const double sum = group_sum(squares(entries, units, n_units, blockIdx.x, gridDim.x, threadIdx.x), slots);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void k_norm_sum(const double* part, int parts, double max_norm, float* out) {
    __shared__ double slots[kSumThreads / 64];
    double v[kNormParts / kSumThreads], sum = 0.0;
#pragma unroll
    for (int i = 0; i < kNormParts / kSumThreads; ++i) v[i] = (int)threadIdx.x + i * kSumThreads < parts ? part[threadIdx.x + i * kSumThreads] : 0.0;
#pragma unroll
    for (int i = 0; i < kNormParts / kSumThreads; ++i) sum += v[i];
    sum = group_sum(sum, slots);
    if (threadIdx.x == 0) write_norm(sum, max_norm, out);
}

// Few units: one workgroup, four units at a time, in one launch (14 units 5.8 us; two launches 3.1 + 2.0, and 3.4 more on the host: norm and
// step of those 17.6 us with two, 15.4 with one).
constexpr int kNormFew = 32;
__global__ __launch_bounds__(kSumThreads) void k_norm_few(const PlanEntry* entries, const PlanUnit* units, int n_units, double max_norm, float* out) {
    __shared__ double slots[kSumThreads / 64];
    const int group = threadIdx.x / kThreads;
    const double mine = n_units ? squares(entries, units, n_units, group, kSumThreads / kThreads, threadIdx.x % kThreads) : 0.0;
    const double sum = group_sum(mine, slots);
    if (threadIdx.x == 0) write_norm(sum, max_norm, out);
}

// ---- the step ----------------------------------------------------------------------------------------------------
//
// A wave has 1024 neighbouring elements: four blocks of 256, of which a lane has 4 each, so that a block of 8-bit moments is one
// wave's and its largest value is found across the lanes.  What the four blocks need is loaded before anything is computed.  A
// piece that ends inside its unit goes element by element through the same arithmetic.

// Smallest power of two, 2^-126 at least, that brings x within 1.75 * 2^top, and its inverse
struct Scale { float scale, inverse; };
__device__ __forceinline__ Scale scale_for(uint32_t bits, int top) {         // of x >= 0
    int e = (int)(bits >> 23) - top + ((bits & 0x7fffffu) > 0x600000u);     // biased exponent of the scale
    e = max(e, 1);
    return {__uint_as_float((uint32_t)e << 23), __uint_as_float((uint32_t)(254 - e) << 23)};
}

// a >= 0 in units of its block's scale, rounded by 16 random bits to a neighbour with 23 - DROP mantissa bits, equally spaced ones
// below LOW_EXP
template <int DROP, int LOW_EXP, bool NEVER_ZERO>
__device__ __forceinline__ float round_by_chance(float a, uint32_t r) {
    const float up = __uint_as_float((__float_as_uint(a) + (r << (DROP - 16)) + (1u << (DROP - 17))) >> DROP << DROP);
    const float steps = __uint_as_float((uint32_t)(127 + 23 - DROP - LOW_EXP) << 23);          // per unit, below 2^LOW_EXP
    float q = floorf(a * steps + ((float)r + 0.5f) * 0x1p-16f);
    if (NEVER_ZERO) q = a > 0.0f ? fmaxf(q, 1.0f) : 0.0f;
    return a >= __uint_as_float((uint32_t)(127 + LOW_EXP) << 23) ? up : q * __uint_as_float((uint32_t)(127 - (23 - DROP - LOW_EXP)) << 23);
}

// The largest of the wave's numbers, the same in every lane: within rows of 16 by rotations, then across the four rows
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, false));
    return max(max((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16)),
               max((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48)));
}
__device__ __forceinline__ uint32_t size_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// What a step needs beside the tensors
struct Numbers { float f, beta1, one_beta1, beta2, one_beta2, eps, inv_sqrt_c2, keep, move; uint32_t key; };

// One element's step; its random bits.  The root and the quotient are the hardware's, a unit in the last place off each: they move the
// weight's step by as little, and no moment.
__device__ __forceinline__ uint32_t step_element(const Numbers& a, uint32_t e, float g, float& m, float& v, float& w) {
    uint32_t x = e * 0x9E3779B1u + a.key;
    x = (x ^ x >> 16) * 0x6C8E9CF5u;
    x = (x ^ x >> 15) * 0xB5297A4Du;
    x ^= x >> 16;
    const bool fine = size_bits(g) < 0x7f800000u;
    const float gf = g * a.f;
    const float m1 = __builtin_amdgcn_fmed3f(m * a.beta1 + gf * a.one_beta1, -0x1p127f, 0x1p127f);
    const float v1 = fminf(v * a.beta2 + (gf * gf) * a.one_beta2, 0x1p127f);
    const float w1 = w * a.keep - a.move * (m1 * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v1) * a.inv_sqrt_c2 + a.eps));
    m = fine ? m1 : m;
    v = fine ? v1 : v;
    w = fine ? w1 : w;
    return x;
}
// A bf16 weight without master: w rounded to a neighbour by 16 random bits; what is not finite is cut
__device__ __forceinline__ uint32_t bf16_by_chance(float w, uint32_t random) {
    const uint32_t bits = __float_as_uint(w), r = random * 0x9E3779B1u >> 16;
    return (size_bits(w) < 0x7f800000u ? bits + r : bits) >> 16;
}
__device__ __forceinline__ uint32_t m_code(float m, const Scale& s, uint32_t random) {
    const float a = round_by_chance<20, -6, false>(fabsf(m) * s.inverse, random & 0xffffu);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(copysignf(a, m), 0.0f, 0, false) & 0xffu;
}
__device__ __forceinline__ uint32_t v_code(float v, const Scale& s, uint32_t random) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(round_by_chance<21, -14, true>(v * s.inverse, random >> 16), 0.0f, 0, false) & 0xffu;
}

// The wave's 1024 elements from element e0 of the tensor on, all of which exist
template <int BITS, bool MASTER, bool PARAM>
__device__ __forceinline__ void step_whole(const PlanEntry& t, const Numbers& a, int64_t e0) {
    const int lane = threadIdx.x & 63;
    const int64_t at = e0 + 4 * lane, block = e0 / kMomentBlock;
    f32x4_any g[4], w[4], m32[4], v32[4];
    bf16x4_at_any p[4];
    uint32_t m8[4], v8[4];
    float ms[4], vs[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        g[b] = *(const __attribute__((address_space(1))) f32x4_any*)(t.grad + at + 256 * b);
        if constexpr (MASTER) w[b] = *(const __attribute__((address_space(1))) f32x4_any*)(t.master + at + 256 * b);
        else p[b] = *(const __attribute__((address_space(1))) bf16x4_at_any*)(t.param + at + 256 * b);
        if constexpr (BITS == 32) {
            m32[b] = *(const __attribute__((address_space(1))) f32x4_any*)(reinterpret_cast<const float*>(t.m) + at + 256 * b);
            v32[b] = *(const __attribute__((address_space(1))) f32x4_any*)(reinterpret_cast<const float*>(t.v) + at + 256 * b);
        } else {
            m8[b] = *(const __attribute__((address_space(1))) u32_any*)(reinterpret_cast<const uint8_t*>(t.m) + at + 256 * b);
            v8[b] = *(const __attribute__((address_space(1))) u32_any*)(reinterpret_cast<const uint8_t*>(t.v) + at + 256 * b);
            ms[b] = in_memory(t.m_scale)[block + b];
            vs[b] = in_memory(t.v_scale)[block + b];
        }
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        float m[4], v[4];
        if constexpr (BITS == 32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) { m[j] = m32[b][j]; v[j] = v32[b][j]; }
        } else {
            m[0] = __builtin_amdgcn_cvt_f32_fp8(m8[b], 0) * ms[b]; m[1] = __builtin_amdgcn_cvt_f32_fp8(m8[b], 1) * ms[b];
            m[2] = __builtin_amdgcn_cvt_f32_fp8(m8[b], 2) * ms[b]; m[3] = __builtin_amdgcn_cvt_f32_fp8(m8[b], 3) * ms[b];
            v[0] = __builtin_amdgcn_cvt_f32_bf8(v8[b], 0) * vs[b]; v[1] = __builtin_amdgcn_cvt_f32_bf8(v8[b], 1) * vs[b];
            v[2] = __builtin_amdgcn_cvt_f32_bf8(v8[b], 2) * vs[b]; v[3] = __builtin_amdgcn_cvt_f32_bf8(v8[b], 3) * vs[b];
        }
        if constexpr (!MASTER) w[b] = f32x4_any{bf16_lo(p[b][0]), bf16_hi(p[b][0]), bf16_lo(p[b][1]), bf16_hi(p[b][1])};
        uint32_t random[4];
        bf16x4_at_any old = p[b];
        float was[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float x = w[b][j];
            was[j] = x;
            random[j] = step_element(a, (uint32_t)(at + 256 * b + j), g[b][j], m[j], v[j], x);
            w[b][j] = x;
        }
        if constexpr (MASTER) {
            *(__attribute__((address_space(1))) f32x4_any*)(t.master + at + 256 * b) = w[b];
            if constexpr (PARAM)
                *(__attribute__((address_space(1))) bf16x4_at_any*)(t.param + at + 256 * b) =
                    bf16x4_at_any{pack_bf16(w[b][0], w[b][1]), pack_bf16(w[b][2], w[b][3])};
        } else {
            uint32_t c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                c[j] = size_bits(g[b][j]) < 0x7f800000u ? bf16_by_chance(w[b][j], random[j]) : __float_as_uint(was[j]) >> 16;
            old = bf16x4_at_any{c[0] | c[1] << 16, c[2] | c[3] << 16};
            *(__attribute__((address_space(1))) bf16x4_at_any*)(t.param + at + 256 * b) = old;
        }
        if constexpr (BITS == 32) {
            *(__attribute__((address_space(1))) f32x4_any*)(reinterpret_cast<float*>(t.m) + at + 256 * b) = f32x4_any{m[0], m[1], m[2], m[3]};
            *(__attribute__((address_space(1))) f32x4_any*)(reinterpret_cast<float*>(t.v) + at + 256 * b) = f32x4_any{v[0], v[1], v[2], v[3]};
        } else {
            const Scale sm = scale_for(wave_max(max(max(size_bits(m[0]), size_bits(m[1])), max(size_bits(m[2]), size_bits(m[3])))), 8);
            const Scale sv = scale_for(wave_max(max(max(size_bits(v[0]), size_bits(v[1])), max(size_bits(v[2]), size_bits(v[3])))), 15);
            uint32_t cm = 0, cv = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) { cm |= m_code(m[j], sm, random[j]) << (8 * j); cv |= v_code(v[j], sv, random[j]) << (8 * j); }
            *(__attribute__((address_space(1))) u32_any*)(reinterpret_cast<uint8_t*>(t.m) + at + 256 * b) = cm;
            *(__attribute__((address_space(1))) u32_any*)(reinterpret_cast<uint8_t*>(t.v) + at + 256 * b) = cv;
            if (lane == 0) { in_memory(t.m_scale)[block + b] = sm.scale; in_memory(t.v_scale)[block + b] = sv.scale; }
        }
    }
}

// The wave's elements from e0 on where the tensor ends among them: a block at a time, lane i has its elements i, i + 64, ...
template <int BITS>
__device__ __forceinline__ void step_end(const PlanEntry& t, const Numbers& a, int64_t e0) {
    const int lane = threadIdx.x & 63;
    for (int b = 0; b < 4 && e0 + 256 * b < t.n; ++b) {
        const int64_t base = e0 + 256 * b, block = base / kMomentBlock;
        const float ms = BITS == 8 ? in_memory(t.m_scale)[block] : 1.0f, vs = BITS == 8 ? in_memory(t.v_scale)[block] : 1.0f;
        float g[4], w[4], m[4], v[4];
        uint32_t random[4], top_m = 0, top_v = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {                                          // behind the end the last element once more, not kept
            const int64_t e = min(base + 64 * j + lane, t.n - 1);
            g[j] = in_memory(t.grad)[e];
            w[j] = t.master ? in_memory(t.master)[e] : bf16_bits_to_float(in_memory(t.param)[e]);
            if constexpr (BITS == 32) {
                m[j] = in_memory(reinterpret_cast<float*>(t.m))[e];
                v[j] = in_memory(reinterpret_cast<float*>(t.v))[e];
            } else {
                m[j] = __builtin_amdgcn_cvt_f32_fp8(in_memory(reinterpret_cast<uint8_t*>(t.m))[e], 0) * ms;
                v[j] = __builtin_amdgcn_cvt_f32_bf8(in_memory(reinterpret_cast<uint8_t*>(t.v))[e], 0) * vs;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t e = base + 64 * j + lane;
            random[j] = step_element(a, (uint32_t)e, g[j], m[j], v[j], w[j]);
            if (e >= t.n) continue;
            if (t.master) {
                in_memory(t.master)[e] = w[j];
                if (t.param) in_memory(t.param)[e] = (qblora_bf16)pack_bf16(w[j], 0.0f);
            } else if (size_bits(g[j]) < 0x7f800000u) {
                in_memory(t.param)[e] = (qblora_bf16)bf16_by_chance(w[j], random[j]);
            }
            if constexpr (BITS == 32) {
                in_memory(reinterpret_cast<float*>(t.m))[e] = m[j];
                in_memory(reinterpret_cast<float*>(t.v))[e] = v[j];
            }
            top_m = max(top_m, size_bits(m[j]));
            top_v = max(top_v, size_bits(v[j]));
        }
        if constexpr (BITS == 8) {
            const Scale sm = scale_for(wave_max(top_m), 8), sv = scale_for(wave_max(top_v), 15);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t e = base + 64 * j + lane;
                if (e >= t.n) continue;
                in_memory(reinterpret_cast<uint8_t*>(t.m))[e] = (uint8_t)m_code(m[j], sm, random[j]);
                in_memory(reinterpret_cast<uint8_t*>(t.v))[e] = (uint8_t)v_code(v[j], sv, random[j]);
            }
            if (lane == 0) { in_memory(t.m_scale)[block] = sm.scale; in_memory(t.v_scale)[block] = sv.scale; }
        }
    }
}

template <int BITS>
__global__ __launch_bounds__(kThreads) void k_adamw(StepDesc d) {
    const PlanUnit unit = d.units[blockIdx.x];
    const PlanEntry t = d.entries[unit.tensor];
    const float f = d.clip ? d.clip[1] : 1.0f;
    if (!isfinite(f)) return;                                              // a broken gradient: nothing is changed
    const double lr = d.device_lr ? (double)*d.device_lr : d.lr;
    double lr_c1 = d.lr_c1;
    Numbers a{f, d.beta1, d.one_beta1, d.beta2, d.one_beta2, d.eps, d.inv_sqrt_c2, 0.0f, 0.0f, d.key};
    if (d.device_step) {
        int64_t step = *d.device_step;
        if (step < 1) step = 1;
        lr_c1 = lr / (1.0 - pow(d.beta1d, (double)step));
        a.inv_sqrt_c2 = (float)(1.0 / sqrt(1.0 - pow(d.beta2d, (double)step)));
        a.key = d.seed_key + (uint32_t)step * 0xD168AAADu;
    } else if (d.device_lr) {
        lr_c1 = lr / (1.0 - pow(d.beta1d, (double)d.step));
    }
    a.keep = (float)(1.0 - lr * t.rate * t.decay);
    a.move = (float)(lr_c1 * t.rate);
    a.key += (uint32_t)unit.tensor * 0x632BE5ABu;
    const int64_t e0 = (int64_t)unit.index * kUnit + (int)(threadIdx.x >> 6) * (kUnit / (kThreads / 64));
    if (e0 + kUnit / (kThreads / 64) > t.n) step_end<BITS>(t, a, e0);
    else if (!t.master) step_whole<BITS, false, true>(t, a, e0);
    else if (t.param) step_whole<BITS, true, true>(t, a, e0);
    else step_whole<BITS, true, false>(t, a, e0);
}

}  // namespace

int launch_adamw_plan(const PlanDesc& d, int64_t units, hipStream_t st) {
    k_adamw_plan<<<(unsigned)std::max<int64_t>(1, std::min<int64_t>(1024, (units + 255) / 256)), 256, 0, st>>>(d, units);
    return launch_status();
}

int launch_grad_norm(const PlanEntry* entries, const PlanUnit* units, int64_t n_units, double max_norm, double* part, float* out,
                     hipStream_t st) {
    if (n_units <= kNormFew) {
        k_norm_few<<<1, kSumThreads, 0, st>>>(entries, units, (int)n_units, max_norm, out);
        return launch_status();
    }
    const int parts = (int)std::min<int64_t>(n_units, kNormParts);
    k_norm_parts<<<parts, kThreads, 0, st>>>(entries, units, n_units, part);
    k_norm_sum<<<1, kSumThreads, 0, st>>>(part, parts, max_norm, out);
    return launch_status();
}

int launch_adamw(const StepDesc& d, hipStream_t st) {
    const int64_t most = kMostThreads / kThreads;
    for (int64_t at = 0; at < d.n_units; at += most) {
        StepDesc e = d;
        e.units += at;
        const unsigned blocks = (unsigned)std::min(most, d.n_units - at);
        if (d.bits == 8) k_adamw<8><<<blocks, kThreads, 0, st>>>(e);
        else k_adamw<32><<<blocks, kThreads, 0, st>>>(e);
    }
    return launch_status();
}

}  // namespace qblora
