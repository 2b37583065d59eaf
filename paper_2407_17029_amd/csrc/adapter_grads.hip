// Gradients of every adapter's matrices: reductions over the adapter's own tokens.
//
//   dA_a[m][r] = (1/lambda1) * pool( X^T dU ),   dB_a[r][j] = pool( dY^T (s U) ),   pool: sums of lambda adjacent features
//
// X and dY are contracted as they are (exact products), the narrow factors as three bf16 parts, and the features are added up in the
// result's registers.  A workgroup has 128 features of X or dY and 128 r of one adapter and walks the adapter's tokens, 32 a
// step, through LDS; both operands come out of the transposing read.  Few adapters with many tokens: the tokens go in slices, whose
// partial sums a second launch adds up in a fixed order.
#include <algorithm>

#include "adapters.h"

namespace qblora {

namespace {

typedef __attribute__((ext_vector_type(4))) short s16x4;

constexpr int kThreads = 256, kBT = 32, kWide = 128, kNarrow = 128;
constexpr int kStride = 2 * kWide + 32;                        // bytes of a token's row in LDS: four rows lie in different banks
constexpr int kTile = kBT * kStride;

__device__ __forceinline__ bf16x8 tokens_of(const unsigned char* p) {
    const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p)));
    const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 4 * kStride)));
    return __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
}
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Sums of LAM adjacent ones of a value that 16 neighbouring lanes hold, in every LAM-th of them
template <int LAM>
__device__ __forceinline__ float pool_lanes(float v) {
    if constexpr (LAM >= 2) v += __shfl_xor(v, 1);
    if constexpr (LAM >= 4) v += __shfl_xor(v, 2);
    if constexpr (LAM >= 8) v += __shfl_xor(v, 4);
    return v;
}

struct Job { const qblora_bf16* wide; int64_t ld; const qblora_bf16* narrow; float* out; int width, rows; float factor; };

// IS_B: the result is [R][width / LAM] (rows of the product are features), else [width / LAM][R] (rows are r)
template <int LAM, bool IS_B>
__device__ void gradient(const Grouped& g, const Job& job, int R, int ld_out, int p0, int p1, int i0, int r0, unsigned char* smem) {
    unsigned char* const sw = smem; unsigned char* const sh = smem + kTile; unsigned char* const sm = smem + 2 * kTile;
    unsigned char* const sl = smem + 3 * kTile;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, q = lane >> 4, s = lane & 15;
    const int64_t slice = (int64_t)g.T * g.R;
    f32x4 acc[4][4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int chunk = t & 15, row = t >> 4;                    // rows row and row + 16
    const bool wide_in = i0 + 8 * chunk < job.width, narrow_in = r0 + 8 * chunk < R;
    uint4 rw[2], rh[2], rm[2], rl[2];
    auto fetch = [&](int p) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = p + row + 16 * i;
            rw[i] = rh[i] = rm[i] = rl[i] = make_uint4(0, 0, 0, 0);
            if (at >= p1) continue;
            const int token = g.order[at];
            if (token < 0 || token >= g.T) continue;
            if (wide_in) rw[i] = *reinterpret_cast<const uint4*>(job.wide + (int64_t)token * job.ld + i0 + 8 * chunk);
            if (narrow_in) {
                const int64_t from = (int64_t)at * g.R + r0 + 8 * chunk;
                rh[i] = *reinterpret_cast<const uint4*>(job.narrow + from);
                rm[i] = *reinterpret_cast<const uint4*>(job.narrow + slice + from);
                rl[i] = *reinterpret_cast<const uint4*>(job.narrow + 2 * slice + from);
            }
        }
    };
    const int w0 = 64 * (wave & 1), n0 = 64 * (wave >> 1);     // of the wave: 64 features, 64 r
    const uint32_t at = (8 * q + (s >> 2)) * kStride + 8 * (s & 3);
    if (p0 < p1) fetch(p0);
    for (int p = p0; p < p1; p += kBT) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t to = (row + 16 * i) * kStride + 16 * chunk;
            *reinterpret_cast<uint4*>(sw + to) = rw[i];
            *reinterpret_cast<uint4*>(sh + to) = rh[i];
            *reinterpret_cast<uint4*>(sm + to) = rm[i];
            *reinterpret_cast<uint4*>(sl + to) = rl[i];
        }
        __syncthreads();
        if (p + kBT < p1) fetch(p + kBT);
        bf16x8 wf[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) wf[a] = tokens_of(sw + at + 2 * (w0 + 16 * a));
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const bf16x8 h = tokens_of(sh + at + 2 * (n0 + 16 * b)), m = tokens_of(sm + at + 2 * (n0 + 16 * b)),
                         l = tokens_of(sl + at + 2 * (n0 + 16 * b));
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                acc[a][b] = IS_B ? mma(wf[a], h, acc[a][b]) : mma(h, wf[a], acc[a][b]);
                acc[a][b] = IS_B ? mma(wf[a], m, acc[a][b]) : mma(m, wf[a], acc[a][b]);
                acc[a][b] = IS_B ? mma(wf[a], l, acc[a][b]) : mma(l, wf[a], acc[a][b]);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            f32x4 v = acc[a][b];
            if constexpr (IS_B) {                              // four neighbouring features of one r
                const int i = i0 + w0 + 16 * a + 4 * q, r = r0 + n0 + 16 * b + s;
                if constexpr (LAM == 8) {
                    float sum = v[0] + v[1] + v[2] + v[3];
                    sum += __shfl_xor(sum, 16);
                    if (!(q & 1) && i < job.width && r < R) job.out[(int64_t)r * ld_out + i / 8] = job.factor * sum;
                } else if (i < job.width && r < R) {
                    float* o = job.out + (int64_t)r * ld_out + i / LAM;
                    if constexpr (LAM == 1) *reinterpret_cast<float4*>(o) = make_float4(job.factor * v[0], job.factor * v[1], job.factor * v[2], job.factor * v[3]);
                    if constexpr (LAM == 2) *reinterpret_cast<float2*>(o) = make_float2(job.factor * (v[0] + v[1]), job.factor * (v[2] + v[3]));
                    if constexpr (LAM == 4) *o = job.factor * (v[0] + v[1] + v[2] + v[3]);
                }
            } else {                                           // four neighbouring r of one feature
                const int i = i0 + w0 + 16 * a + s, r = r0 + n0 + 16 * b + 4 * q;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = job.factor * pool_lanes<LAM>(v[e]);
                if (s % LAM == 0 && i < job.width && r < R) *reinterpret_cast<float4*>(job.out + (int64_t)(i / LAM) * ld_out + r) = make_float4(v[0], v[1], v[2], v[3]);
            }
        }
}

template <int LAM1, int LAM2>
__global__ __launch_bounds__(kThreads) void k_adapter_grads(AdapterGradDesc d, int tiles_a, int tiles_b) {
    __shared__ __align__(16) unsigned char smem[4 * kTile];
    const int a = blockIdx.y, z = blockIdx.z;
    const AdapterEntry e = d.g.table[a];
    if (!e.dA || !e.dB || e.R <= 0 || e.R > d.g.R) return;
    const bool is_b = (int)blockIdx.x >= tiles_a;
    int tile = blockIdx.x - (is_b ? tiles_a : 0);
    const int n_wide = ((is_b ? d.d_out : d.d_in) + kWide - 1) / kWide;
    const int i0 = tile % n_wide * kWide, r0 = tile / n_wide * kNarrow;
    if (r0 >= e.R) return;
    const int f0 = min(max(d.g.first[a], 0), d.g.T), f1 = min(max(d.g.first[a + 1], f0), d.g.T);
    const int steps = (f1 - f0 + kBT - 1) / kBT;
    const int p0 = f0 + (int)((int64_t)steps * z / d.splits) * kBT, p1 = min(f1, f0 + (int)((int64_t)steps * (z + 1) / d.splits) * kBT);
    const int K = d.d_in / LAM1, J = d.d_out / LAM2;
    float* const part = d.splits > 1 ? d.part + ((int64_t)z * d.g.count + a) * (K + J) * d.g.R : nullptr;
    if (is_b) {
        const Job job{d.dY, d.lddy, d.su, part ? part + (int64_t)K * d.g.R : e.dB, d.d_out, 0, 1.0f};
        gradient<LAM2, true>(d.g, job, e.R, J, p0, p1, i0, r0, smem);
    } else {
        const Job job{d.X, d.ldx, d.du, part ? part : e.dA, d.d_in, 0, 1.0f / LAM1};
        gradient<LAM1, false>(d.g, job, e.R, e.R, p0, p1, i0, r0, smem);
    }
}

// The slices' sums; a workgroup takes 1024 numbers of one adapter's dA and dB, which lie one behind the other
__global__ __launch_bounds__(256) void k_adapter_grad_sums(AdapterGradDesc d, int K, int J) {
    const int a = blockIdx.y;
    const AdapterEntry e = d.g.table[a];
    if (!e.dA || !e.dB || e.R <= 0 || e.R > d.g.R) return;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, n_a = (int64_t)K * e.R, n_b = (int64_t)J * e.R;
    const bool is_b = at >= n_a;
    const int64_t i = is_b ? at - n_a : at;
    if (is_b && i >= n_b) return;
    const int64_t slice = (int64_t)d.g.count * (K + J) * d.g.R;
    const float* p = d.part + (int64_t)a * (K + J) * d.g.R + (is_b ? (int64_t)K * d.g.R : 0) + i;
    float4 v = *reinterpret_cast<const float4*>(p);
    for (int z = 1; z < d.splits; ++z) {
        const float4 w = *reinterpret_cast<const float4*>(p + z * slice);
        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
    }
    *reinterpret_cast<float4*>((is_b ? e.dB : e.dA) + i) = v;
}

template <int LAM1, int LAM2>
int grads(const AdapterGradDesc& d, hipStream_t st) {
    const int blocks_r = (d.g.R + kNarrow - 1) / kNarrow;
    const int tiles_a = (d.d_in + kWide - 1) / kWide * blocks_r, tiles_b = (d.d_out + kWide - 1) / kWide * blocks_r;
    k_adapter_grads<LAM1, LAM2><<<dim3(tiles_a + tiles_b, d.g.count, d.splits), kThreads, 0, st>>>(d, tiles_a, tiles_b);
    if (d.splits > 1) {
        const int K = d.d_in / LAM1, J = d.d_out / LAM2;
        k_adapter_grad_sums<<<dim3((unsigned)(((int64_t)(K + J) * d.g.R / 4 + 255) / 256), d.g.count), 256, 0, st>>>(d, K, J);
    }
    return launch_status();
}
template <int LAM1>
int grads_by_lam2(const AdapterGradDesc& d, hipStream_t st) {
    switch (d.lam2) {
        case 1: return grads<LAM1, 1>(d, st);
        case 2: return grads<LAM1, 2>(d, st);
        case 4: return grads<LAM1, 4>(d, st);
        default: return grads<LAM1, 8>(d, st);
    }
}

}  // namespace

int adapter_grad_splits(int count, int64_t T, int d_in, int d_out, int R) {
    const int64_t blocks_r = (R + kNarrow - 1) / kNarrow;
    const int64_t units = ((d_in + kWide - 1) / kWide + (d_out + kWide - 1) / kWide) * blocks_r * count;
    return (int)std::max<int64_t>(1, std::min<int64_t>({8, 512 / units, T / 512}));
}

int launch_adapter_grads(const AdapterGradDesc& d, hipStream_t st) {
    switch (d.lam1) {
        case 1: return grads_by_lam2<1>(d, st);
        case 2: return grads_by_lam2<2>(d, st);
        case 4: return grads_by_lam2<4>(d, st);
        default: return grads_by_lam2<8>(d, st);
    }
}

}  // namespace qblora
