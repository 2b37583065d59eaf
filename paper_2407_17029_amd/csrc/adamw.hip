// The optimizer's step over many tensors at once: the list on the device, the norm of all gradients, and AdamW with moments in
// 32 or 8 bits (qblora_adamw_plan, qblora_grad_norm, qblora_adamw_step; the formulas stand in include/qblora.h).
#include <algorithm>

#include "adapters.h"

namespace qblora {

namespace {

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

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
__device__ __forceinline__ double group_sum(double v, double* slots) {
    for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slots[0] + slots[1] + slots[2] + slots[3];
    __syncthreads();
    return v;
}

__global__ __launch_bounds__(kThreads) void k_norm_parts(const PlanEntry* entries, const PlanUnit* units, int64_t n_units, double* part) {
    __shared__ double slots[kThreads / 64];
    double sum = 0.0;
    for (int64_t u = blockIdx.x; u < n_units; u += gridDim.x) {
        const PlanUnit unit = units[u];
        const float* const grad = entries[unit.tensor].grad + (int64_t)unit.index * kUnit;
        const int n = (int)min((int64_t)kUnit, entries[unit.tensor].n - (int64_t)unit.index * kUnit);
#pragma unroll
        for (int i = 0; i < kUnit / (4 * kThreads); ++i) {
            const int e = 4 * (threadIdx.x + i * kThreads);
            if (e + 4 <= n) {
                const f32x4_any v = *reinterpret_cast<const f32x4_any*>(grad + e);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += (double)v[j] * v[j];
            } else {
                for (int j = e; j < n; ++j) sum += (double)grad[j] * grad[j];
            }
        }
    }
    sum = group_sum(sum, slots);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kThreads) void k_norm_sum(const double* part, int parts, double max_norm, float* out) {
    __shared__ double slots[kThreads / 64];
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) sum += part[i];
    sum = group_sum(sum, slots);
    if (threadIdx.x == 0) {
        const float norm = (float)__dsqrt_rn(sum);
        const double factor = max_norm / (__dsqrt_rn(sum) + 1e-6);
        out[0] = norm;
        out[1] = isfinite(norm) ? (float)(factor < 1.0 ? factor : 1.0) : __uint_as_float(0x7fc00000u);
    }
}

// ---- the step ----------------------------------------------------------------------------------------------------
//
// A wave has 256 neighbouring elements, 4 a lane: one block of 8-bit moments, whose largest values are found across the wave.

// Smallest power of two, 2^-126 at least, that brings x within 1.75 * 2^top, and its inverse
struct Scale { float scale, inverse; };
__device__ __forceinline__ Scale scale_for(float x, int top) {
    const uint32_t bits = __float_as_uint(x);                              // x >= 0
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

__device__ __forceinline__ float wave_max(float v) {
    for (int s = 32; s; s >>= 1) v = fmaxf(v, __shfl_xor(v, s));
    return v;
}

template <int BITS>
__global__ __launch_bounds__(kThreads) void k_adamw(StepDesc d) {
    const PlanUnit unit = d.units[blockIdx.x];
    const PlanEntry t = d.entries[unit.tensor];
    const float f = d.clip ? d.clip[1] : 1.0f;
    if (!isfinite(f)) return;                                              // a broken gradient: nothing is changed
    double lr = d.device_lr ? (double)*d.device_lr : d.lr;
    double lr_c1 = d.lr_c1;
    float inv_sqrt_c2 = d.inv_sqrt_c2;
    uint32_t key = d.key;
    if (d.device_step) {
        int64_t step = *d.device_step;
        if (step < 1) step = 1;
        lr_c1 = lr / (1.0 - pow(d.beta1d, (double)step));
        inv_sqrt_c2 = (float)(1.0 / sqrt(1.0 - pow(d.beta2d, (double)step)));
        key = d.seed_key + (uint32_t)step * 0xD168AAADu;
    } else if (d.device_lr) {
        lr_c1 = lr / (1.0 - pow(d.beta1d, (double)d.step));
    }
    const float keep = (float)(1.0 - lr * t.rate * t.decay), move = (float)(lr_c1 * t.rate);
    key += (uint32_t)unit.tensor * 0x632BE5ABu;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int b = wave; b < kUnit / kMomentBlock; b += kThreads / 64) {
        const int64_t block = (int64_t)unit.index * (kUnit / kMomentBlock) + b;
        const int64_t e0 = block * kMomentBlock + 4 * lane;
        if (block * kMomentBlock >= t.n) break;
        const int n = (int)max((int64_t)0, min((int64_t)4, t.n - e0));     // elements of this lane
        float g[4] = {0, 0, 0, 0}, m[4] = {0, 0, 0, 0}, v[4] = {0, 0, 0, 0}, w[4] = {0, 0, 0, 0};
        for (int j = 0; j < n; ++j) {
            g[j] = t.grad[e0 + j];
            w[j] = t.master ? t.master[e0 + j] : bf16_bits_to_float(t.param[e0 + j]);
        }
        if constexpr (BITS == 32) {
            for (int j = 0; j < n; ++j) { m[j] = reinterpret_cast<const float*>(t.m)[e0 + j]; v[j] = reinterpret_cast<const float*>(t.v)[e0 + j]; }
        } else {
            const float ms = t.m_scale[block], vs = t.v_scale[block];
            for (int j = 0; j < n; ++j) {
                m[j] = __builtin_amdgcn_cvt_f32_fp8(reinterpret_cast<const uint8_t*>(t.m)[e0 + j], 0) * ms;
                v[j] = __builtin_amdgcn_cvt_f32_bf8(reinterpret_cast<const uint8_t*>(t.v)[e0 + j], 0) * vs;
            }
        }
        uint32_t random[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t x = (uint32_t)(e0 + j) * 0x9E3779B1u + key;
            x = (x ^ x >> 16) * 0x6C8E9CF5u;
            x = (x ^ x >> 15) * 0xB5297A4Du;
            random[j] = x ^ x >> 16;
            const float gf = g[j] * f;
            if (!isfinite(g[j]) || j >= n) continue;
            m[j] = fminf(fmaxf(m[j] * d.beta1 + gf * d.one_beta1, -0x1p127f), 0x1p127f);
            v[j] = fminf(v[j] * d.beta2 + (gf * gf) * d.one_beta2, 0x1p127f);
            w[j] = w[j] * keep - move * (m[j] / (__fsqrt_rn(v[j]) * inv_sqrt_c2 + d.eps));
        }
        for (int j = 0; j < n; ++j) {
            if (!isfinite(g[j])) continue;
            if (t.master) {
                t.master[e0 + j] = w[j];
                if (t.param) t.param[e0 + j] = (qblora_bf16)(pack_bf16(w[j], 0.0f));
            } else {
                const uint32_t r = random[j] * 0x9E3779B1u >> 16, bits = __float_as_uint(w[j]);
                t.param[e0 + j] = (qblora_bf16)((isfinite(w[j]) ? bits + r : bits) >> 16);
            }
        }
        if constexpr (BITS == 32) {
            for (int j = 0; j < n; ++j) { reinterpret_cast<float*>(t.m)[e0 + j] = m[j]; reinterpret_cast<float*>(t.v)[e0 + j] = v[j]; }
        } else {
            const Scale sm = scale_for(wave_max(fmaxf(fmaxf(fabsf(m[0]), fabsf(m[1])), fmaxf(fabsf(m[2]), fabsf(m[3])))), 8);
            const Scale sv = scale_for(wave_max(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]))), 15);
            for (int j = 0; j < n; ++j) {
                const float a = round_by_chance<20, -6, false>(fabsf(m[j]) * sm.inverse, random[j] & 0xffffu);
                const float b = round_by_chance<21, -14, true>(v[j] * sv.inverse, random[j] >> 16);
                reinterpret_cast<uint8_t*>(t.m)[e0 + j] =
                    (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(copysignf(a, m[j]), 0.0f, 0, false);
                reinterpret_cast<uint8_t*>(t.v)[e0 + j] = (uint8_t)__builtin_amdgcn_cvt_pk_bf8_f32(b, 0.0f, 0, false);
            }
            if (lane == 0) { t.m_scale[block] = sm.scale; t.v_scale[block] = sv.scale; }
        }
    }
}

}  // namespace

int launch_adamw_plan(const PlanDesc& d, int64_t units, hipStream_t st) {
    k_adamw_plan<<<(unsigned)std::max<int64_t>(1, std::min<int64_t>(1024, (units + 255) / 256)), 256, 0, st>>>(d, units);
    return launch_status();
}

int launch_grad_norm(const PlanEntry* entries, const PlanUnit* units, int64_t n_units, double max_norm, double* part, float* out,
                     hipStream_t st) {
    const int parts = (int)std::min<int64_t>(n_units, kNormParts);
    if (parts) k_norm_parts<<<parts, kThreads, 0, st>>>(entries, units, n_units, part);
    k_norm_sum<<<1, kThreads, 0, st>>>(part, parts, max_norm, out);
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
