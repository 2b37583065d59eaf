// Gradients of every adapter's matrices: reductions over the adapter's own tokens.
//
//   dA_a[m][r] = (1/lambda1) * pool( X^T dU ),   dB_a[r][j] = pool( dY^T (s U) ),   pool: sums of lambda adjacent features
//
// X and dY are contracted as they are (exact products), the narrow factors as three bf16 parts, and the features are added up in the
// result's registers.  A workgroup has 256 features of X or dY and 128 r of one adapter and walks the adapter's tokens, 32 a
// step, through a ring in LDS that the rows are copied straight into; both operands come out of the transposing read.  Few adapters
// with many tokens: the tokens go in slices, whose partial sums a second launch adds up in a fixed order.
//
// Bound by the matrix pipe, which contracts every product three times: two parts (16 bits) left dA and dB 1.5 to 2 times as far from
// 64 bits as fp32 products are, three (24 bits) are closer than those (4e-7
// against 9e-7, 7810 tokens).  7842 tokens, 8192 + 22016 features, R = 256: 364 GFLOP in 342 us, 312 at best
// (1060 and 1170 TFLOP/s, where a large library product reaches 1210); 7810 tokens of 4096 + 4096, R = 128, four adapters: 60 us.
// The slices follow the adapters of the table: 8192 tokens of one adapter take 59 + 5 us in a table of one, 304 in one of 16.
// Tiles of 128 x 128 through registers took 510 and 84, with 1.6 times the traffic into LDS and no copy under way during a product.
#include <algorithm>

#include "adapters.h"

namespace qblora {

namespace {

typedef __attribute__((ext_vector_type(4))) short s16x4;

constexpr int kThreads = 512, kBT = 32, kWide = 256, kNarrow = 128, kParts = 3;
constexpr int kWideBytes = kBT * 2 * kWide, kNarrowBytes = kBT * 2 * kNarrow, kStage = kWideBytes + kParts * kNarrowBytes;
constexpr int kStages = 3, kCopies = 2 + kParts;               // of a wave for a stage
constexpr int kOrder = 2048;                                   // tokens whose numbers lie in LDS
constexpr int kLds = kStages * kStage + 4 * kOrder;

__device__ __align__(16) const uint32_t g_nothing[4] = {0u, 0u, 0u, 0u};

__device__ __forceinline__ void copy16_to_lds(const void* p, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds_base), "v"(p) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Eight tokens of this lane's feature or r: rows + 0 .. 3 and + 4 .. 7, `four` bytes on
template <int FOUR>
__device__ __forceinline__ bf16x8 tokens_of(const unsigned char* p) {
    const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p)));
    const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + FOUR)));
    return __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
}
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Where the 16-byte chunks of a token's row go (chunk c to c ^ swap): half a wave's transposing read takes two chunks of rows
// 0 .. 3 and 8 .. 11, which then lie in different banks
__device__ __forceinline__ int token_swap(int row) { return ((row & 3) | (row >> 1 & 4)) << 1; }

// Sums of LAM adjacent ones of a value that 16 neighbouring lanes hold, in every LAM-th of them
template <int LAM>
__device__ __forceinline__ float pool_lanes(float v) {
    if constexpr (LAM >= 2) v += __shfl_xor(v, 1);
    if constexpr (LAM >= 4) v += __shfl_xor(v, 2);
    if constexpr (LAM >= 8) v += __shfl_xor(v, 4);
    return v;
}

struct Job { const qblora_bf16* wide; int64_t ld; const qblora_bf16* narrow; float* out; int width; float factor; };

// IS_B: the result is [R][width / LAM] (rows of the product are features), else [width / LAM][R] (rows are r)
template <int LAM, bool IS_B>
__device__ void gradient(const Grouped& g, const Job& job, int R, int ld_out, int p0, int p1, int i0, int r0, unsigned char* smem) {
    int* const order = reinterpret_cast<int*>(smem + kStages * kStage);
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), q = lane >> 4, s = lane & 15;
    const int64_t slice = (int64_t)g.T * g.R;
    f32x4 acc[8][2];
#pragma unroll
    for (int a = 0; a < 8; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // A wave copies two rows of the wide array twice, and four rows of each part of the narrow one.  Features behind the last fetch the
    // first ones, whose sums they repeat; r behind the last, and tokens behind the last, are zero in the narrow array.
    int wide_row[2], wide_col[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        wide_row[i] = 2 * (wave + 8 * i) + (lane >> 5);
        const int col = i0 + 8 * ((lane & 31) ^ token_swap(wide_row[i]));
        wide_col[i] = col < job.width ? col : 0;
    }
    const int narrow_row = 4 * wave + (lane >> 4), narrow_col = r0 + 8 * ((lane & 15) ^ token_swap(narrow_row));
    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(smem)) + wave * 1024;
    // the wave's 128 features and 32 r
    const int w0 = 128 * (wave & 1), n0 = 32 * (wave >> 1), row = 8 * q + (s >> 2);
    const int inside = 16 * (((s & 3) >> 1) ^ token_swap(row)) + 8 * (s & 1);
    int w_off[8], n_off[2];
#pragma unroll
    for (int a = 0; a < 8; ++a) w_off[a] = row * (2 * kWide) + (inside ^ (2 * (w0 + 16 * a)));
#pragma unroll
    for (int b = 0; b < 2; ++b) n_off[b] = kWideBytes + row * (2 * kNarrow) + (inside ^ (2 * (n0 + 16 * b)));
    const bool busy = r0 + n0 < R;

    for (int base = p0; base < p1; base += kOrder) {
        const int end = min(base + kOrder, p1), steps = (end - base + kBT - 1) / kBT;
        for (int i = t; i < end - base; i += kThreads) order[i] = g.order[base + i];
        __syncthreads();
        auto issue = [&](int step, int buf) __attribute__((always_inline)) {
            const uint32_t to = lds + buf * kStage;
            const int from = base + step * kBT;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int token = min(max(order[min(from + wide_row[i], end - 1) - base], 0), g.T - 1);
                copy16_to_lds(job.wide + (int64_t)token * job.ld + wide_col[i], to + i * 8192);
            }
            const int at = from + narrow_row, token = order[min(at, end - 1) - base];
            const bool real = at < end && narrow_col < R && token >= 0 && token < g.T;
            const qblora_bf16* const narrow = job.narrow + (int64_t)at * g.R + narrow_col;
#pragma unroll
            for (int p = 0; p < kParts; ++p)
                copy16_to_lds(real ? (const void*)(narrow + p * slice) : (const void*)g_nothing, to + kWideBytes + p * kNarrowBytes);
        };
        issue(0, 0);
        if (steps > 1) issue(1, 1);
        int buf = 0;
        for (int step = 0; step < steps; ++step) {
            static_assert(kCopies == 5, "the copies of one stage may be under way");
            if (step + 1 < steps) asm volatile("s_waitcnt vmcnt(5)" ::: "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            meet();                                            // this stage is in, the one before it is free
            if (step + 2 < steps) issue(step + 2, buf == 0 ? 2 : buf - 1);
            if (busy) {
                const unsigned char* const from = smem + buf * kStage;
                bf16x8 wf[8];
#pragma unroll
                for (int a = 0; a < 8; ++a) wf[a] = tokens_of<8 * kWide>(from + w_off[a]);
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int p = 0; p < kParts; ++p) {
                        const bf16x8 nf = tokens_of<8 * kNarrow>(from + n_off[b] + p * kNarrowBytes);
#pragma unroll
                        for (int a = 0; a < 8; ++a) acc[a][b] = IS_B ? mma(wf[a], nf, acc[a][b]) : mma(nf, wf[a], acc[a][b]);
                    }
            }
            buf = buf == kStages - 1 ? 0 : buf + 1;
        }
        __syncthreads();
    }
    if (!busy) return;
#pragma unroll
    for (int a = 0; a < 8; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
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
    extern __shared__ __align__(16) unsigned char smem[];
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
        const Job job{d.dY, d.lddy, d.su, part ? part + (int64_t)K * d.g.R : e.dB, d.d_out, 1.0f};
        gradient<LAM2, true>(d.g, job, e.R, J, p0, p1, i0, r0, smem);
    } else {
        const Job job{d.X, d.ldx, d.du, part ? part : e.dA, d.d_in, 1.0f / LAM1};
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
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(k_adapter_grads<LAM1, LAM2>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess)
        return QBLORA_ERR_LAUNCH;
    k_adapter_grads<LAM1, LAM2><<<dim3(tiles_a + tiles_b, d.g.count, d.splits), kThreads, kLds, st>>>(d, tiles_a, tiles_b);
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
    return (int)std::max<int64_t>(1, std::min<int64_t>({8, 256 / units, T / 512}));
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
