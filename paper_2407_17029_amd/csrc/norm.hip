// Addition of the residual and root-mean-square norm, forward and backward (qblora_rms_norm_fwd / _bwd).
//
//   total = bf16(x + residual),  r = 1 / sqrt(mean(total^2) + eps),  y = total * r * w
//   dx = r (g - h mean(g h)) + dtotal,  dw = sum_t dy h,  with h = total * r, g = dy * w
//
// Everything between the bf16 arrays is fp32; the sum is rounded before it is normed, as it is what the next layer and the
// backward pass get.
//
// Bound by HBM: one pass over each array.  A workgroup holds a row in registers, 8 features a thread and chunk, so the mean
// is known before anything is written; the only other traffic is dw.  Rows of any length and alignment: a 16-byte access
// takes any address in one instruction; the features behind the last whole chunk are read with the row's last eight and written
// one by one.  8192 rows of 8192 both ways (1.07 GB): 192 us, 5.6 TB/s, where a large copy reaches 4.9 (93 forward, 97 backward, 4
// the sum of dw); 4001 rows of 4097, an odd length, 84 us (30 forward, 45 backward); 64 rows of 4096: 4 us, of which 3.5 are an
// empty launch.
#include <algorithm>

#include "decoder.h"

namespace qblora {

namespace {

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// The eight features from e on of a row of d, as four dwords, 0 behind the end
__device__ __forceinline__ uint4 load_chunk(const qblora_bf16* row, int e, int d) {
    if (e + 8 <= d) {
        const bf16x8_any v = *reinterpret_cast<const bf16x8_any*>(row + e);
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
    if (d >= 8) {                                                      // the row's last eight, those of this chunk to the front
        const bf16x8_any v = *reinterpret_cast<const bf16x8_any*>(row + d - 8);
        uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
        const int bits = 16 * (e + 8 - d);                             // 16 to 112
        if (bits >= 64) { lo = hi; hi = 0; }
        const int left = bits & 63;
        if (left) { lo = lo >> left | hi << (64 - left); hi >>= left; }
        return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
    }
    uint32_t w[4] = {0, 0, 0, 0};
    for (int j = 0; j < 8; ++j)
        if (e + j < d) w[j / 2] |= (uint32_t)row[e + j] << (16 * (j & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool PAST>
__device__ __forceinline__ void store_chunk(qblora_bf16* row, int e, int d, uint4 v) {
    if (e + 8 <= d) {
        const bf16x8_any o = {v.x, v.y, v.z, v.w};
        if (PAST) __builtin_nontemporal_store(o, reinterpret_cast<bf16x8_any*>(row + e));
        else *reinterpret_cast<bf16x8_any*>(row + e) = o;
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    for (int j = 0; j < 8; ++j)
        if (e + j < d) row[e + j] = (qblora_bf16)(w[j / 2] >> (16 * (j & 1)));
}
__device__ __forceinline__ uint32_t word(const uint4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }
__device__ __forceinline__ void set_word(uint4& v, int j, uint32_t x) {
    if (j == 0) v.x = x; else if (j == 1) v.y = x; else if (j == 2) v.z = x; else v.w = x;
}

// sum over the workgroup; `slots`: one float a wave, not reused before the next barrier but one
__device__ __forceinline__ float block_sum(float v, float* slots) {
    for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
    for (int w = 0; w < waves; ++w) v += slots[w];
    return v;
}

template <int NC, bool PAST>                  // PAST: stores go past the caches
__global__ __launch_bounds__(1024) void k_rms_norm(NormDesc a) {
    __shared__ float slots[16];
    const int64_t row = blockIdx.x;
    const int d = a.d;
    const qblora_bf16* x = a.x + row * d;
    uint4 v[NC], w[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = 8 * (threadIdx.x + i * blockDim.x);
        v[i] = w[i] = make_uint4(0, 0, 0, 0);
        if (c < d) {
            v[i] = load_chunk(x, c, d);
            w[i] = load_chunk(a.w, c, d);
        }
    }
    if (a.residual) {
        const qblora_bf16* res = a.residual + row * d;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = 8 * (threadIdx.x + i * blockDim.x);
            if (c >= d) continue;
            const uint4 r = load_chunk(res, c, d);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t p = word(v[i], j), q = word(r, j);
                set_word(v[i], j, pack_bf16(bf16_lo(p) + bf16_lo(q), bf16_hi(p) + bf16_hi(q)));
            }
            store_chunk<PAST>(a.total + row * d, c, d, v[i]);
        }
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float lo = bf16_lo(word(v[i], j)), hi = bf16_hi(word(v[i], j));
            sum = __fmaf_rn(lo, lo, sum);
            sum = __fmaf_rn(hi, hi, sum);
        }
    const float mean = block_sum(sum / (float)d, slots);                 // each thread's part of it: their sum may pass fp32
    const float r = 1.0f / __fsqrt_rn(mean + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = r;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = 8 * (threadIdx.x + i * blockDim.x);
        if (c >= d) continue;
        uint4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t p = word(v[i], j), q = word(w[i], j);
            set_word(o, j, pack_bf16(bf16_lo(p) * r * bf16_lo(q), bf16_hi(p) * r * bf16_hi(q)));
        }
        store_chunk<PAST>(a.y + row * d, c, d, o);
    }
}

constexpr int kSumStride = 65;
// dw of 64 columns: every eighth thread takes the same eight, rows threads / 8 apart, which are added up in a fixed order.
__device__ __forceinline__ void column_sums(const NormBackDesc& a, int block, float* sums) {
    const int c = 64 * block + 8 * (threadIdx.x & 7), groups = blockDim.x >> 3, g = threadIdx.x >> 3;
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (c < a.d)
#pragma unroll 4
        for (int64_t row = g; row < a.T; row += groups) {
            const uint4 t = load_chunk(a.total + row * a.d, c, a.d), y = load_chunk(a.dy + row * a.d, c, a.d);
            const float r = a.rstd[row];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[2 * j] = __fmaf_rn(bf16_lo(word(y, j)), bf16_lo(word(t, j)) * r, s[2 * j]);
                s[2 * j + 1] = __fmaf_rn(bf16_hi(word(y, j)), bf16_hi(word(t, j)) * r, s[2 * j + 1]);
            }
        }
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[g * kSumStride + 8 * (threadIdx.x & 7) + j] = s[j];
    __syncthreads();
    if (threadIdx.x >= 64 || 64 * block + (int)threadIdx.x >= a.d) return;
    float sum = 0.0f;
    for (int i = 0; i < groups; ++i) sum += sums[i * kSumStride + threadIdx.x];
    a.dw[64 * block + threadIdx.x] = sum;
}

// The first a.rows workgroups take rows, the others, if any, 64 columns of dw each.
template <int NC, bool PAST>                  // PAST: stores go past the caches
__global__ __launch_bounds__(1024) void k_rms_norm_bwd(NormBackDesc a) {
    __shared__ float slots[2][16];
    extern __shared__ float sums[];                                      // of the workgroups with columns
    if ((int)blockIdx.x >= a.rows) return column_sums(a, blockIdx.x - a.rows, sums);
    const int d = a.d;
    uint4 w[NC];
    float dw[NC][8];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = 8 * (threadIdx.x + i * blockDim.x);
        w[i] = c < d ? load_chunk(a.w, c, d) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = 0.0f;
    }
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += a.rows, turn ^= 1) {
        const float r = a.rstd[row];
        uint4 t[NC], y[NC], e[NC];
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = 8 * (threadIdx.x + i * blockDim.x);
            t[i] = y[i] = e[i] = make_uint4(0, 0, 0, 0);
            if (c < d) {
                t[i] = load_chunk(a.total + row * d, c, d);
                y[i] = load_chunk(a.dy + row * d, c, d);
                if (a.dtotal) e[i] = load_chunk(a.dtotal + row * d, c, d);
            }
        }
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t tp = word(t[i], j / 2), yp = word(y[i], j / 2), wp = word(w[i], j / 2);
                const float h = ((j & 1) ? bf16_hi(tp) : bf16_lo(tp)) * r, dy = (j & 1) ? bf16_hi(yp) : bf16_lo(yp);
                dw[i][j] = __fmaf_rn(dy, h, dw[i][j]);
                sum = __fmaf_rn(dy * ((j & 1) ? bf16_hi(wp) : bf16_lo(wp)), h, sum);
            }
        const float mean = block_sum(sum / (float)d, slots[turn]);
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = 8 * (threadIdx.x + i * blockDim.x);
            if (c >= d) continue;
            uint4 o;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t tp = word(t[i], j), yp = word(y[i], j), wp = word(w[i], j), ep = word(e[i], j);
                const float lo = __fmaf_rn(-bf16_lo(tp) * r, mean, bf16_lo(yp) * bf16_lo(wp));
                const float hi = __fmaf_rn(-bf16_hi(tp) * r, mean, bf16_hi(yp) * bf16_hi(wp));
                set_word(o, j, pack_bf16(__fmaf_rn(r, lo, bf16_lo(ep)), __fmaf_rn(r, hi, bf16_hi(ep))));
            }
            store_chunk<PAST>(a.dx + row * d, c, d, o);
        }
    }
    if (!a.part) return;
    float* part = a.part + (int64_t)blockIdx.x * d;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = 8 * (threadIdx.x + i * blockDim.x);
        if (c + 8 <= d) {
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
                const f32x4_any v = {dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]};
                *reinterpret_cast<f32x4_any*>(part + c + j) = v;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < d) part[c + j] = dw[i][j];
        }
    }
}

// dw[c] = sum over the rows of `part`, 16 columns and 64 rows at a time
__global__ __launch_bounds__(1024) void k_rms_norm_dw(const float* __restrict__ part, int rows, int d, float* __restrict__ dw) {
    __shared__ float sums[64][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), r0 = threadIdx.x >> 4;
    float s = 0.0f;
    if (c < d)
#pragma unroll 4
        for (int r = r0; r < rows; r += 64) s += part[(int64_t)r * d + c];
    sums[r0][threadIdx.x & 15] = s;
    __syncthreads();
    if (r0 == 0 && c < d) {
        s = 0.0f;
        for (int i = 0; i < 64; ++i) s += sums[i][threadIdx.x & 15];
        dw[c] = s;
    }
}

struct Plan { int threads, chunks; };          // threads of a row, chunks of a thread
Plan plan_of(int d) {
    const int chunks = (d + 7) / 8, t = (chunks + 63) / 64 * 64;
    return {t < 1024 ? t : 1024, t <= 1024 ? 1 : 2};
}
// From so many bytes an array on, no L2 holds the outputs when they are read: 8192 rows of 8192 both ways 199 us through the
// caches, 190 past them; 2001 rows of 4096 31 and 28.
constexpr int64_t kPastBytes = 8 << 20;
bool past_caches(int64_t T, int d) { return T * d * 2 >= kPastBytes; }

// Up to so many rows whose arrays stay in the caches, dw is summed by columns in the same launch, which reads total and dy a
// second time: 1000 rows of 4096 both ways 22.1 us and 23.5 with the second launch, 64 rows 21.4 and 23.8; but 1000 rows of 8192
// 33.3 and 31.6, 2001 of 600 26.4 and 25.4.  The columns take as many threads at least, which share out the rows.
constexpr int64_t kColumnRows = 1024;
constexpr int kColumnThreads = 512;

}  // namespace

int launch_rms_norm(const NormDesc& a, hipStream_t st) {
    const Plan p = plan_of(a.d);
    const bool past = past_caches(a.T, a.d);
    const int64_t most = kMostThreads / p.threads;                       // rows of a launch
    for (int64_t row = 0; row < a.T; row += most) {
        NormDesc b = a;
        b.x += row * a.d;
        if (a.residual) b.residual += row * a.d;
        if (a.residual) b.total += row * a.d;
        b.y += row * a.d;
        if (a.rstd) b.rstd += row;
        const dim3 grid((unsigned)std::min(most, a.T - row)), threads(p.threads);
        const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, threads, 0, st, b); };
        if (p.chunks == 1) go(past ? k_rms_norm<1, true> : k_rms_norm<1, false>);
        else go(past ? k_rms_norm<2, true> : k_rms_norm<2, false>);
    }
    return launch_status();
}

int64_t rms_norm_bwd_parts(int64_t T, int d) {
    // 1024 threads of rows a CU.  With 4096 or 8192 features every CU has as many workgroups (4001 rows both ways 52 and 103 us); where
    // the threads of a row do not divide 1024, some CUs have one more than others: 5120 features 82 us, 6144 100, 7168 119.
    const int64_t full = 256 * 1024 / plan_of(d).threads;
    const int64_t some = (T + 3) / 4;                                    // four rows at least: 8001 x 600 25 us, with one 28.7
    return some < full ? some : full;
}

int launch_rms_norm_bwd(const NormBackDesc& desc, hipStream_t st) {
    NormBackDesc a = desc;
    const Plan p = plan_of(a.d);
    const bool past = past_caches(a.T, a.d);
    const auto launch = [&](int threads, int columns) {
        const size_t lds = columns ? threads / 8 * kSumStride * sizeof(float) : 0;
        const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.rows + columns), dim3(threads), lds, st, a); };
        if (p.chunks == 1) go(past ? k_rms_norm_bwd<1, true> : k_rms_norm_bwd<1, false>);
        else go(past ? k_rms_norm_bwd<2, true> : k_rms_norm_bwd<2, false>);
    };
    if (a.dw && a.T && a.T <= kColumnRows && !past && a.dx != a.dy) {    // (dy is read by both)
        a.rows = (int)a.T;
        a.part = nullptr;
        launch(std::max(p.threads, kColumnThreads), (a.d + 63) / 64);
        return launch_status();
    }
    a.rows = (int)rms_norm_bwd_parts(a.T, a.d);
    if (a.rows) launch(p.threads, 0);
    if (a.dw) hipLaunchKernelGGL(k_rms_norm_dw, dim3((a.d + 15) / 16), dim3(1024), 0, st, a.part, a.rows, a.d, a.dw);
    return launch_status();
}

}  // namespace qblora
