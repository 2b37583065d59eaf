// What the operators between the projections share (not part of the C ABI): descriptions and launchers.
#pragma once
#include "common.h"

namespace qblora {

// Eight bf16 at any address: a global access takes any in one instruction.
typedef uint32_t bf16x8_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t bf16x4_any __attribute__((ext_vector_type(2), aligned(2)));

__device__ __forceinline__ float bf16_lo(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

// Threads of one launch.  A grid dimension has fewer than 2^32, and one of more is cut to its low 32 bits without an error: 2^24 + 77
// tokens in workgroups of 256 left all but 77 unwritten.  Calls on more rows than this takes go in several launches.
constexpr int64_t kMostThreads = (int64_t)1 << 30;

struct TablesDesc {
    const int32_t* context; const int32_t* fresh; int n;
    int page_shift;
    const int32_t* free_pages; int n_free;
    int32_t* table; int width;
    int tokens;
    int32_t* starts; int32_t* positions; int64_t* slots; int32_t* taken;
};
int launch_page_tables(const TablesDesc& d, hipStream_t st);

struct RopeDesc {
    const float* freq; int rot, interleaved; float scale; float sign;      // sign -1: the transposed operator
    const qblora_bf16* q; int64_t ldq; int heads;
    const qblora_bf16* k; int64_t ldk; int kv_heads;
    int head_dim;
    const int32_t* positions; int64_t T;
    qblora_bf16* q_out; int64_t ldq_out;
    qblora_bf16* k_out; int64_t ldk_out;
    // serving: k and v go to the cache instead
    const qblora_bf16* v; int64_t ldv; const int64_t* slots;
    qblora_bf16* kc; qblora_bf16* vc; int64_t cache_slots; int page_shift;
};
int launch_rope(const RopeDesc& d, hipStream_t st);

struct NormDesc {
    const qblora_bf16* x; const qblora_bf16* residual; const qblora_bf16* w;
    int64_t T; int d; float eps;
    qblora_bf16* total; qblora_bf16* y; float* rstd;
};
int launch_rms_norm(const NormDesc& d, hipStream_t st);
struct NormBackDesc {
    const qblora_bf16* total; const qblora_bf16* w; const float* rstd; const qblora_bf16* dy; const qblora_bf16* dtotal;
    int64_t T; int d;
    qblora_bf16* dx; float* dw; float* part;
    int rows;                                      // workgroups that take rows
};
int64_t rms_norm_bwd_parts(int64_t T, int d);      // rows of [d] partial sums of dw
int launch_rms_norm_bwd(const NormBackDesc& d, hipStream_t st);

struct AttnDesc {
    const qblora_bf16* q; int64_t ldq; int heads, kv_heads, group;          // group: query heads per key / value head
    uint32_t group_magic;                                                    // 2^32 / group + 1
    const qblora_bf16* kc; const qblora_bf16* vc; int pages, page_shift, head_dim;
    const int32_t* table; int width;
    const int32_t* starts; const int32_t* context; int n, T;
    float scale_log2;                                                        // scale * log2(e)
    int window, max_new;
    qblora_bf16* out; int64_t ldo; float* lse;
    float* part;
};
size_t attention_part_bytes(int head_dim, int kv_heads, int group, int max_new);
int launch_attention(const AttnDesc& d, hipStream_t st);

}  // namespace qblora
