// Rotary positions (qblora_rope_fwd / _bwd) and their serving form, which writes k and v to the paged cache
// (qblora_rope_cache).
//
//   pair (a, b) of a head at position p:  a' = scale (a cos x - b sin x),  b' = scale (b cos x + a sin x),  x = p * freq
//
// Bound by HBM, each element read and written once, or by the launch with few tokens.  A workgroup takes kTokens tokens,
// forms their sines and cosines once for all heads in LDS, and moves 8 features a thread.
#include "decoder.h"

namespace qblora {

namespace {

constexpr int kThreads = 256;

// cos and sin of p * freq: in 64 bits down to one turn, then by the hardware's functions of turns
__device__ __forceinline__ void turn(int32_t p, float freq, float scale, float& c, float& s) {
    double r = (double)p * (double)freq * 0.15915494309189533577;
    r -= __builtin_rint(r);
    c = __builtin_amdgcn_cosf((float)r) * scale;
    s = __builtin_amdgcn_sinf((float)r) * scale;
}
__device__ __forceinline__ float to_float(qblora_bf16 x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ qblora_bf16 to_bf16(float x) { return (qblora_bf16)pack_bf16(x, 0.0f); }

__device__ __forceinline__ bool in_cache(const RopeDesc& d, int64_t slot) { return slot >= 0 && slot < d.cache_slots; }
// element offset of head h's part of a slot's page, and the place in the page
__device__ __forceinline__ int64_t page_of(const RopeDesc& d, int64_t slot, int h, int& place) {
    place = (int)(slot & ((1 << d.page_shift) - 1));
    return (((slot >> d.page_shift) * d.kv_heads + h) << d.page_shift) * d.head_dim;
}
__device__ __forceinline__ int64_t key_at(const RopeDesc& d, int place, int f) {
    return ((int64_t)(f >> 3 << d.page_shift) + place) * 8 + (f & 7);
}
__device__ __forceinline__ int64_t value_at(const RopeDesc& d, int place, int f) {
    return ((int64_t)(place >> 3) * d.head_dim + f) * 8 + (place & 7);
}

// One feature pair (or one feature beside the pairs) a thread, any width and layout.  `pass`: 0 q, 1 k, 2 v.
__global__ __launch_bounds__(kThreads) void k_rope_any(RopeDesc d) {
    const int64_t t = blockIdx.x;
    const int32_t p = d.positions[t];
    const int half = d.rot >> 1, per_head = half + (d.head_dim - d.rot), hk = d.k ? d.kv_heads : 0;
    const int64_t slot = d.slots ? d.slots[t] : -1;
    for (int i = threadIdx.x; i < (d.heads + hk) * per_head; i += kThreads) {
        const int hh = i / per_head, u = i - hh * per_head;
        const bool is_k = hh >= d.heads;
        const int h = is_k ? hh - d.heads : hh;
        const qblora_bf16* in = (is_k ? d.k + t * d.ldk : d.q + t * d.ldq) + (int64_t)h * d.head_dim;
        qblora_bf16* out = is_k ? d.k_out + t * d.ldk_out + (int64_t)h * d.head_dim
                                : d.q_out + t * d.ldq_out + (int64_t)h * d.head_dim;
        const bool cached = is_k && d.kc;
        if (cached && !in_cache(d, slot)) continue;
        int place = 0;
        if (cached) out = d.kc + page_of(d, slot, h, place);
        if (u < half) {
            const int f0 = d.interleaved ? 2 * u : u, f1 = d.interleaved ? 2 * u + 1 : u + half;
            float c, s;
            turn(p, d.freq[u], d.scale, c, s);
            s *= d.sign;
            const float a = to_float(in[f0]), b = to_float(in[f1]);
            out[cached ? key_at(d, place, f0) : f0] = to_bf16(__fmaf_rn(a, c, -(b * s)));
            out[cached ? key_at(d, place, f1) : f1] = to_bf16(__fmaf_rn(b, c, a * s));
        } else {
            const int f = d.rot + u - half;
            out[cached ? key_at(d, place, f) : f] = in[f];
        }
    }
    if (!d.vc || !in_cache(d, slot)) return;
    for (int i = threadIdx.x; i < d.kv_heads * d.head_dim; i += kThreads) {
        const int h = i / d.head_dim, f = i - h * d.head_dim;
        int place;
        qblora_bf16* out = d.vc + page_of(d, slot, h, place);
        out[value_at(d, place, f)] = d.v[t * d.ldv + i];
    }
}

}  // namespace

int launch_rope(const RopeDesc& d, hipStream_t st) {
    hipLaunchKernelGGL(k_rope_any, dim3((unsigned)d.T), dim3(kThreads), 0, st, d);
    return launch_status();
}

}  // namespace qblora
