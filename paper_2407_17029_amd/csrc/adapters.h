// What the operators on many adapters and the optimizer's step share (not part of the C ABI): descriptions and launchers.
#pragma once
#include "decoder.h"

namespace qblora {

// A pointer that was read from memory, as one to device memory: through a pointer that might lie anywhere the compiler makes accesses
// that count as LDS accesses too, and waits for all of them at each one's first use (256 single tokens on 100 adapters, the outputs' part: 473 us instead of 186).
template <typename T>
__device__ __forceinline__ __attribute__((address_space(1))) T* in_memory(T* p) { return (__attribute__((address_space(1))) T*)p; }
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load16(const void* p) {
    const u32x4 v = *in_memory(reinterpret_cast<const u32x4*>(p));
    return make_uint4(v.x, v.y, v.z, v.w);
}

constexpr int kTileTokens = 64;                    // tokens of a tile of the groups
constexpr int kMostAdapters = 8192, kMostGroupRequests = 8192;
constexpr int kMostInnerRank = 512;
constexpr int64_t kMostGroupTokens = (int64_t)1 << 20;

// An entry of the adapters' table, on the device
struct AdapterEntry {
    const qblora_bf16* A; const qblora_bf16* B;    // NULL and R = 0: adds nothing
    float* dA; float* dB;
    int R; float s;
    int64_t spare;
};
static_assert(sizeof(AdapterEntry) == 48, "the table's entries are packed by the host");

constexpr int kTableChunk = 32;                    // entries that one launch writes
struct TableDesc { AdapterEntry entry[kTableChunk]; AdapterEntry* out; int n; };
int launch_adapter_table(const TableDesc& d, hipStream_t st);

struct GroupsDesc {
    const int32_t* starts; const int32_t* which; int n, count, T;
    int32_t* first; int32_t* order; int32_t* tiles; int tile_room;
};
int launch_adapter_groups(const GroupsDesc& d, hipStream_t st);

// The batch as the kernels on tiles see it
struct Grouped {
    const AdapterEntry* table; int count;
    const int32_t* first; const int32_t* order; const int32_t* tiles; int tile_room;
    int T, R;                                      // R: row length of the arrays by place in `order`
};

// part[z][place][r] = factor * s * sum over slice z of the inputs of Z[token][k] * W[k / lam][r]; W is A, or (back) the transpose of B
struct RankDesc {
    Grouped g;
    const qblora_bf16* Z; int64_t ldz; int width, lam, back;
    float factor;
    float* part; int splits;
};
int rank_splits(int tiles, int width, int R);
// no fewer rows of partial sums, slices x tokens, than any number of tokens up to T takes
int64_t rank_part_rows(int64_t T, int width);
int launch_rank_sums(const RankDesc& d, hipStream_t st);

// U, the sum of the slices, as three bf16 parts [3][T][R]: high part and what is left of it, twice.  The second array may be absent.
struct PartsDesc {
    Grouped g;
    const float* part; int splits; qblora_bf16* out;
    const float* part2; int splits2; qblora_bf16* out2;
};
int launch_rank_parts(const PartsDesc& d, hipStream_t st);
// Whether a call makes the parts although nobody keeps them; every call with an inner rank above 256 does
bool rank_parts_pay(int count, int64_t T, int R);

// out[token][n] += factor * sum_r U[place][r] * W[r][n / lam], U the parts that launch_rank_parts made, or (u NULL) the sum of
// `splits` slices of part; W is B, or (back) the transpose of A
struct SpreadDesc {
    Grouped g;
    const qblora_bf16* u;
    const float* part; int splits;
    qblora_bf16* out; int64_t ldo; int width, lam, back;
    float factor;
};
int launch_spread(const SpreadDesc& d, hipStream_t st);
// Whether W = B without parts goes through the form for few tokens of a tile
bool spread_few_applies(int count, int64_t T);

// dA and dB of every entry that has a place for them, from X, dY and the three bf16 parts of s U and of dU
struct AdapterGradDesc {
    Grouped g;
    const qblora_bf16* X; int64_t ldx; int d_in, lam1;
    const qblora_bf16* dY; int64_t lddy; int d_out, lam2;
    const qblora_bf16* su; const qblora_bf16* du;
    float* part; int splits;                       // splits > 1: [splits][count][(d_in/lam1 + d_out/lam2) * R] partial sums
};
int adapter_grad_splits(int count, int64_t T, int d_in, int d_out, int R);
int launch_adapter_grads(const AdapterGradDesc& d, hipStream_t st);

// ---- the optimizer's step

constexpr int kUnit = 4096;                        // elements of a unit
struct PlanEntry {
    int64_t n;
    qblora_bf16* param; float* master; const float* grad; void* m; void* v; float* m_scale; float* v_scale;
    float rate, decay;
    int64_t first_unit;                            // among those of its launch
};
static_assert(sizeof(PlanEntry) == 80, "the plan's entries are packed by the host");
struct PlanUnit { int32_t tensor, index; };        // a unit's tensor and its number in it
constexpr int kPlanChunk = 32;
struct PlanDesc { PlanEntry entry[kPlanChunk]; PlanEntry* out; PlanUnit* units; int first, n; };
int launch_adamw_plan(const PlanDesc& d, int64_t units, hipStream_t st);

constexpr int kNormParts = 2048;                   // partial sums of the norm at most
int launch_grad_norm(const PlanEntry* entries, const PlanUnit* units, int64_t n_units, double max_norm, double* part, float* out,
                     hipStream_t st);

struct StepDesc {
    const PlanEntry* entries; const PlanUnit* units; int64_t n_units; int bits;
    double lr, beta1d, beta2d;
    float beta1, one_beta1, beta2, one_beta2, eps;
    double lr_c1; float inv_sqrt_c2;               // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    uint32_t seed_key, key;                        // seed * 0x85157AF5, and with t's part
    const int64_t* device_step; const float* device_lr; const float* clip;
    int64_t step;
};
int launch_adamw(const StepDesc& d, hipStream_t st);

}  // namespace qblora
