// Many adapters on one projection: the table, the batch's tokens by adapter, and the two halves of the adapter term.
//
//   rank sums   U[t][r] = factor * s_a * sum_k Z[t][k] W_a[k / lam][r]      (W = A on X; W = B transposed on dY)
//   spread      out[t][n] += factor * sum_r U[t][r] W_a[r][n / lam]         (W = B on Y; W = A transposed on dX)
//
// Mean and repetition are never made: a matrix operand's row of W serves lam inputs, a result lam outputs.  Both halves go tile
// by tile, a tile being up to 64 tokens of one adapter, so that W is read once for them.
#include <algorithm>

#include "adapters.h"

namespace qblora {

namespace {

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;

// ---- the table ---------------------------------------------------------------------------------------------------

__global__ __launch_bounds__(64) void k_adapter_table(TableDesc d) {
    if ((int)threadIdx.x < d.n) d.out[threadIdx.x] = d.entry[threadIdx.x];
}

// ---- tokens by adapter -------------------------------------------------------------------------------------------
//
// Every workgroup reads all requests into LDS and adds up the tokens of each adapter (integer sums: any order), scans them, and
// then serves 64 requests of its own: 16 threads a request add up what earlier requests of its adapter have, a wave writes its
// tokens.
constexpr int kGroupThreads = 1024, kGroupRequests = kGroupThreads / 16;

// exclusive scan over the workgroup of a value each thread brings, and the sum of all; `slots`: one int a wave
__device__ __forceinline__ int scan_group(int v, int* slots, int* all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
    for (int s = 1; s < 64; s <<= 1) {
        const int y = __shfl_up(x, s);
        if (lane >= s) x += y;
    }
    __syncthreads();
    if (lane == 63) slots[wave] = x;
    __syncthreads();
    int before = 0, sum = 0;
    for (int w = 0; w < kGroupThreads / 64; ++w) {
        if (w < wave) before += slots[w];
        sum += slots[w];
    }
    *all = sum;
    return before + x - v;
}

__global__ __launch_bounds__(kGroupThreads) void k_adapter_groups(GroupsDesc d) {
    extern __shared__ __align__(16) int mem[];
    int* const slot = mem;                                     // of each request; -1: none
    int* const length = slot + ((d.n + 3) & ~3);
    int* const tokens = length + ((d.n + 3) & ~3);             // of each adapter, then where they begin
    int* const begin_tile = tokens + d.count;
    int* const slots = begin_tile + d.count;
    const int t = threadIdx.x;
    for (int a = t; a < d.count; a += kGroupThreads) tokens[a] = 0;
    __syncthreads();
    // What starts holds is cut to 0 .. T.  Requests that share tokens may list more than there is room for, or than 32 bits count:
    // every place is compared as an unsigned number before it is written to.
    const uint32_t T = d.T;
    for (int i = t; i < d.n; i += kGroupThreads) {
        const int from = min(max(d.starts[i], 0), d.T), to = min(max(d.starts[i + 1], 0), d.T);
        const int a = d.which[i], m = max(to - from, 0);
        const bool has = a >= 0 && a < d.count && m > 0;
        slot[i] = has ? a : -1;
        length[i] = has ? m : 0;
        if (has) atomicAdd(&tokens[a], m);
    }
    __syncthreads();
    // each thread's adapters are neighbours
    const int per = (d.count + kGroupThreads - 1) / kGroupThreads;
    int mine = 0, tiles = 0;
    for (int i = 0; i < per; ++i) {
        const int a = t * per + i;
        if (a < d.count) { mine += tokens[a]; tiles += (tokens[a] + kTileTokens - 1) / kTileTokens; }
    }
    int all, all_tiles;
    int at = scan_group(mine, slots, &all), at_tile = scan_group(tiles, slots, &all_tiles);
    for (int i = 0; i < per; ++i) {
        const int a = t * per + i;
        if (a >= d.count) break;
        const int m = tokens[a];
        tokens[a] = at;
        begin_tile[a] = at_tile;
        if (a % gridDim.x == blockIdx.x) {                     // the adapters' tiles are shared out among the workgroups
            d.first[a] = min(max(at, 0), d.T);
            for (int j = 0; j * kTileTokens < m; ++j) {
                const int from = at + j * kTileTokens;
                if ((uint32_t)from >= T || (uint32_t)(at_tile + j) >= (uint32_t)d.tile_room) break;
                reinterpret_cast<int4*>(d.tiles)[at_tile + j] =
                    make_int4(a, from, min(min(m - j * kTileTokens, kTileTokens), d.T - from), 0);
            }
        }
        at += m;
        at_tile += (m + kTileTokens - 1) / kTileTokens;
    }
    __syncthreads();
    all = min(max(all, 0), d.T);
    all_tiles = min(max(all_tiles, 0), d.tile_room);
    if (blockIdx.x == 0 && t == 0) d.first[d.count] = all;
    for (int i = all + blockIdx.x * kGroupThreads + t; i < d.T; i += gridDim.x * kGroupThreads) d.order[i] = -1;
    for (int i = all_tiles + blockIdx.x * kGroupThreads + t; i < d.tile_room; i += gridDim.x * kGroupThreads)
        reinterpret_cast<int4*>(d.tiles)[i] = make_int4(0, 0, 0, 0);
    // where each of this workgroup's requests begins in its adapter's run
    const int r0 = blockIdx.x * kGroupRequests, me = r0 + (t >> 4), sub = t & 15;
    const int a = me < d.n ? slot[me] : -1;
    int before = 0;
    if (a >= 0)
        for (int i = sub; i < me; i += 16)
            if (slot[i] == a) before += length[i];
    for (int s = 8; s; s >>= 1) before += __shfl_xor(before, s);
    __syncthreads();
    if (sub == 0 && a >= 0) slots[t >> 4] = tokens[a] + before;
    __syncthreads();
    for (int i = t >> 6; i < kGroupRequests && r0 + i < d.n; i += kGroupThreads / 64) {
        const int m = length[r0 + i];
        if (!m) continue;
        const int to = slots[i], from = max(d.starts[r0 + i], 0);
        for (int j = t & 63; j < m; j += 64)
            if ((uint32_t)(to + j) < T) d.order[to + j] = from + j;
    }
}

// ---- what the halves share ---------------------------------------------------------------------------------------

struct Tile { int begin, tokens, R; const AdapterEntry* entry; };

// The tile's description, if it is one: numbers out of range make none.
__device__ __forceinline__ bool read_tile(const Grouped& g, int at, Tile* tile) {
    const int4 e = reinterpret_cast<const int4*>(g.tiles)[at];
    if (e.x < 0 || e.x >= g.count || e.y < 0 || e.z <= 0 || e.z > kTileTokens || e.y > g.T - e.z) return false;
    const AdapterEntry* entry = g.table + e.x;
    const int R = entry->R;
    if (R <= 0 || R > g.R) return false;
    *tile = {e.y, e.z, R, entry};
    return true;
}

// Eight values of four of them, each twice; and so on: the operand of eight inputs from the lam-th part of as many rows
template <int LAM>
__device__ __forceinline__ bf16x8 repeated(uint2 v, int which) {
    uint4 o;
    if constexpr (LAM == 2) {
        o.x = __builtin_amdgcn_perm(v.x, v.x, 0x01000100u); o.y = __builtin_amdgcn_perm(v.x, v.x, 0x03020302u);
        o.z = __builtin_amdgcn_perm(v.y, v.y, 0x01000100u); o.w = __builtin_amdgcn_perm(v.y, v.y, 0x03020302u);
    } else if constexpr (LAM == 4) {
        const uint32_t p = which & 1 ? v.y : v.x;
        o.x = o.y = __builtin_amdgcn_perm(p, p, 0x01000100u);
        o.z = o.w = __builtin_amdgcn_perm(p, p, 0x03020302u);
    } else {
        const uint32_t p = which & 2 ? v.y : v.x;
        o.x = o.y = o.z = o.w = which & 1 ? __builtin_amdgcn_perm(p, p, 0x03020302u) : __builtin_amdgcn_perm(p, p, 0x01000100u);
    }
    return __builtin_bit_cast(bf16x8, o);
}

// Column lane & 15 of four rows of a 16-bit array in LDS: lane s of a group of 16 points at row s >> 2, elements 4 (s & 3) on
__device__ __forceinline__ uint2 columns_of(const unsigned char* p) {
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p)));
}

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// ---- rank sums ---------------------------------------------------------------------------------------------------
//
// Many tokens: steps of 64 inputs, Z's rows and W's through registers into LDS, double-buffered.  The matrix product's rows are r
// (16 a block, blocks dealt to the four waves), its columns tokens.  W's rows lie by input (A: the transposing read makes
// the operand) or by r (B).  Both factors are bf16 as they are, the products exact, the sums fp32.
constexpr int kRankThreads = 256, kRankRows = 256;         // r of a workgroup at most
constexpr int kZStride = 128 + 16;                         // bytes of a token's 64 inputs in LDS

template <int LAM, bool BACK>
constexpr int rank_w_bytes() { return BACK ? kRankRows * (128 / LAM + 16) : 64 / LAM * (kRankRows * 2 + 32); }
template <int LAM, bool BACK>
constexpr int rank_lds() { return 2 * (kTileTokens * kZStride + rank_w_bytes<LAM, BACK>()); }

template <int LAM, bool BACK>
__device__ void rank_many(const RankDesc& d, const Tile& tile, int step0, int step1, int r_base, float* part, unsigned char* smem) {
    constexpr int kWBytes = rank_w_bytes<LAM, BACK>();
    constexpr int kWRows = 64 / LAM;                       // of A for a step
    constexpr int kMost = BACK ? kRankRows * (8 / LAM) / kRankThreads : kWRows * (kRankRows / 8) / kRankThreads;   // copies a thread
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int R = min(tile.R - r_base, kRankRows);
    const int J = d.width / LAM;
    // Z: rows t >> 3 and 32 further, 16 bytes each
    const unsigned char* z[2];
    uint32_t z_to[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int l = (t >> 3) + 32 * i;
        const int token = min(max(d.g.order[tile.begin + min(l, tile.tokens - 1)], 0), d.g.T - 1);
        z[i] = reinterpret_cast<const unsigned char*>(d.Z + (int64_t)token * d.ldz) + 16 * (t & 7);
        z_to[i] = l * kZStride + 16 * (t & 7);
    }
    const bool two = tile.tokens > 32;
    // W: chunks of 16 bytes
    const int stride = BACK ? 128 / LAM + 16 : 2 * R + 32;                     // of a row in LDS
    const int chunks = BACK ? R * (8 / LAM) : kWRows * (R / 8);
    const unsigned char* w[kMost];
    uint32_t w_to[kMost];
    bool w_has[kMost];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int c = t + i * kRankThreads;
        w_has[i] = c < chunks;
        const int per = BACK ? 8 / LAM : R / 8, row = c / per, col = c % per;
        w[i] = BACK ? reinterpret_cast<const unsigned char*>(tile.entry->B + (int64_t)(r_base + row) * J) + 16 * col
                    : reinterpret_cast<const unsigned char*>(tile.entry->A + (int64_t)row * tile.R + r_base) + 16 * col;
        w_to[i] = row * stride + 16 * col;
    }
    const int64_t w_step = BACK ? 128 / LAM : (int64_t)kWRows * tile.R * 2;    // bytes to the next step
    const int blocks = (R + 15) / 16, mine = (blocks - wave + 3) / 4;          // blocks wave, wave + 4, ...
    const int tb_n = (tile.tokens + 15) / 16;
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[i][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    uint4 zr[2], wr[kMost];
    auto fetch = [&](int step) __attribute__((always_inline)) {
        zr[0] = *reinterpret_cast<const uint4*>(z[0] + (int64_t)step * 128);
        if (two) zr[1] = *reinterpret_cast<const uint4*>(z[1] + (int64_t)step * 128);
#pragma unroll
        for (int i = 0; i < kMost; ++i)
            if (w_has[i]) wr[i] = *reinterpret_cast<const uint4*>(w[i] + step * w_step);
    };
    auto put = [&](int buf) __attribute__((always_inline)) {
        unsigned char* const zs = smem + buf * (kTileTokens * kZStride + kWBytes);
        *reinterpret_cast<uint4*>(zs + z_to[0]) = zr[0];
        if (two) *reinterpret_cast<uint4*>(zs + z_to[1]) = zr[1];
#pragma unroll
        for (int i = 0; i < kMost; ++i)
            if (w_has[i]) *reinterpret_cast<uint4*>(zs + kTileTokens * kZStride + w_to[i]) = wr[i];
    };
    const int g = lane >> 4, s = lane & 15;
    auto products = [&](int buf) __attribute__((always_inline)) {
        const unsigned char* const zs = smem + buf * (kTileTokens * kZStride + kWBytes);
        const unsigned char* const ws = zs + kTileTokens * kZStride;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            bf16x8 zf[4];
#pragma unroll
            for (int b = 0; b < 4; ++b)
                if (b < tb_n) zf[b] = *reinterpret_cast<const bf16x8*>(zs + (16 * b + s) * kZStride + 64 * ks + 16 * g);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= mine) break;
                const int r0 = 16 * (wave + 4 * i);
                bf16x8 wf;
                const int k = (32 * ks + 8 * g) / LAM;                         // first row of W of this lane's eight inputs
                if constexpr (BACK) {
                    const unsigned char* row = ws + (r0 + s) * stride;         // a row of the last block may lie behind R: its sums are not kept
                    if constexpr (LAM == 1) wf = *reinterpret_cast<const bf16x8*>(row + 2 * k);
                    else wf = repeated<LAM>(*reinterpret_cast<const uint2*>(row + 2 * (k & ~3)), k & 3 ? (LAM == 4 ? (k & 3) >> 1 : k & 3) : 0);
                } else {
                    const unsigned char* at = ws + ((k & ~3) + (s >> 2)) * stride + 2 * r0 + 8 * (s & 3);
                    if constexpr (LAM == 1) {
                        const uint2 lo = columns_of(at), hi = columns_of(at + 4 * stride);
                        wf = __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
                    } else {
                        wf = repeated<LAM>(columns_of(at), LAM == 4 ? (k & 3) >> 1 : k & 3);
                    }
                }
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    if (b < tb_n) acc[i][b] = mma(wf, zf[b], acc[i][b]);
            }
        }
    };
    fetch(step0);
    put(0);
    __syncthreads();
    for (int step = step0; step < step1; ++step) {
        const int buf = (step - step0) & 1;
        if (step + 1 < step1) fetch(step + 1);
        products(buf);
        if (step + 1 < step1) put(buf ^ 1);
        __syncthreads();
    }
    const float f = d.factor * tile.entry->s;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= mine) break;
        const int r = 16 * (wave + 4 * i) + 4 * g;
        if (r >= R) continue;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int l = 16 * b + s;
            if (l >= tile.tokens) continue;
            *reinterpret_cast<float4*>(part + (int64_t)(tile.begin + l) * d.g.R + r_base + r) =
                make_float4(f * acc[i][b][0], f * acc[i][b][1], f * acc[i][b][2], f * acc[i][b][3]);
        }
    }
}

template <int LAM, bool BACK>
__global__ __launch_bounds__(kRankThreads) void k_rank_sums(RankDesc d) {
    extern __shared__ __align__(16) unsigned char smem[];
    Tile tile;
    if (!read_tile(d.g, blockIdx.x, &tile)) return;
    const int r_base = blockIdx.z * kRankRows, split = blockIdx.y;
    if (r_base >= tile.R) return;
    const int all = d.width / 64;
    const int step0 = (int)((int64_t)all * split / d.splits), step1 = (int)((int64_t)all * (split + 1) / d.splits);
    float* const part = d.part + (int64_t)split * d.g.T * d.g.R;
    rank_many<LAM, BACK>(d, tile, step0, step1, r_base, part, smem);
}

// ---- spread ------------------------------------------------------------------------------------------------------
//
// Many tokens: U as a bf16 pair (high part and what is left: 16 significant bits) in registers, 16 tokens a wave, all r; steps of
// 64 rows of outputs over W through LDS.  The matrix product's rows are outputs / lam, its columns tokens, so that a lane has 4
// neighbouring rows of one token, 4 lam outputs.
constexpr int kSpreadThreads = 256;

template <int KS>
constexpr int spread_u_stride() { return 64 * KS + 16; }                       // bytes of a token's U in LDS
template <int KS, bool BACK>
constexpr int spread_w_bytes() { return BACK ? 64 * (64 * KS + 16) : 32 * KS * (128 + 32); }
template <int KS, bool BACK>
constexpr int spread_lds() { return std::max(2 * kTileTokens * spread_u_stride<KS>(), 2 * spread_w_bytes<KS, BACK>()); }

__device__ __forceinline__ void split_pair(float4 v, uint2* hi, uint2* lo) {
    hi->x = pack_bf16(v.x, v.y); hi->y = pack_bf16(v.z, v.w);
    lo->x = pack_bf16(v.x - bf16_lo(hi->x), v.y - bf16_hi(hi->x));
    lo->y = pack_bf16(v.z - bf16_lo(hi->y), v.w - bf16_hi(hi->y));
}

// Four neighbouring r of the sum of the slices
__device__ __forceinline__ float4 sum_slices(const float* part, int splits, int64_t slice, int64_t at) {
    float4 v = *reinterpret_cast<const float4*>(part + at);
    for (int z = 1; z < splits; ++z) {
        const float4 w = *reinterpret_cast<const float4*>(part + z * slice + at);
        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
    }
    return v;
}

// The rows of one tile as a bf16 pair
__device__ __forceinline__ void write_pairs(const Grouped& g, const Tile& tile, const float* part, int splits, qblora_bf16* hi) {
    const int quads = tile.R / 4;
    const int64_t slice = (int64_t)g.T * g.R;
    for (int i = threadIdx.x; i < tile.tokens * quads; i += kSpreadThreads) {
        const int64_t at = (int64_t)(tile.begin + i / quads) * g.R + 4 * (i % quads);
        uint2 h, l;
        split_pair(sum_slices(part, splits, slice, at), &h, &l);
        *reinterpret_cast<uint2*>(hi + at) = h;
        *reinterpret_cast<uint2*>(hi + slice + at) = l;
    }
}

// LAM values of a row: out += v
template <int LAM>
__device__ __forceinline__ void add_outputs(qblora_bf16* out, const f32x4& v, float f) {
    // 4 rows of LAM outputs each
    if constexpr (LAM == 1) {
        uint2 o = *reinterpret_cast<uint2*>(out);
        o.x = pack_bf16(bf16_lo(o.x) + f * v[0], bf16_hi(o.x) + f * v[1]);
        o.y = pack_bf16(bf16_lo(o.y) + f * v[2], bf16_hi(o.y) + f * v[3]);
        *reinterpret_cast<uint2*>(out) = o;
    } else {
#pragma unroll
        for (int i = 0; i < LAM / 2; ++i) {
            uint4 o = *reinterpret_cast<uint4*>(out + 8 * i);
            uint32_t* w = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float x = f * v[(8 * i + 2 * j) / LAM];
                w[j] = pack_bf16(bf16_lo(w[j]) + x, bf16_hi(w[j]) + x);
            }
            *reinterpret_cast<uint4*>(out + 8 * i) = o;
        }
    }
}

template <int LAM, bool BACK, int KS>
__device__ void spread_many(const SpreadDesc& d, const Tile& tile, int j0, int j1, unsigned char* smem) {
    constexpr int kUStride = spread_u_stride<KS>(), kWBytes = spread_w_bytes<KS, BACK>();
    constexpr int kWStride = BACK ? 64 * KS + 16 : 128 + 32;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, g = lane >> 4, s = lane & 15;
    const int R = tile.R, J = d.width / LAM;
    const int64_t slice = (int64_t)d.g.T * d.g.R;
    // token blocks: 1, 2 or 4 of them side by side, the other waves take other rows of W
    const int tbs = tile.tokens <= 16 ? 1 : tile.tokens <= 32 ? 2 : 4;
    for (int i = t; i < 16 * tbs * KS * 8; i += kSpreadThreads) {
        const int l = i / (KS * 8), r = 4 * (i % (KS * 8));
        uint2 h = make_uint2(0, 0), lo = h;
        if (l < tile.tokens && r < R) split_pair(sum_slices(d.part, d.splits, slice, (int64_t)(tile.begin + l) * d.g.R + r), &h, &lo);
        *reinterpret_cast<uint2*>(smem + l * kUStride + 2 * r) = h;
        *reinterpret_cast<uint2*>(smem + (kTileTokens + l) * kUStride + 2 * r) = lo;
    }
    __syncthreads();
    const int tb = wave % tbs, jb0 = wave / tbs, jb_step = 4 / tbs;
    bf16x8 uh[KS], ul[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        uh[k] = *reinterpret_cast<const bf16x8*>(smem + (16 * tb + s) * kUStride + 64 * k + 16 * g);
        ul[k] = *reinterpret_cast<const bf16x8*>(smem + (kTileTokens + 16 * tb + s) * kUStride + 64 * k + 16 * g);
    }
    __syncthreads();
    // W by chunks of 16 bytes: 8 a row of r (B), R / 8 a row of outputs (A); r behind R are zero
    const unsigned char* w[KS];
    uint32_t w_to[KS];
    int w_row[KS];
    bool w_has[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        const int c = t + i * kSpreadThreads;
        const int row = BACK ? c / (4 * KS) : c >> 3, col = BACK ? c % (4 * KS) : c & 7;
        w_row[i] = BACK ? row : 8 * col;                                       // first of its outputs / lam in the step
        w_has[i] = BACK ? 8 * col < R : row < R;
        w[i] = BACK ? reinterpret_cast<const unsigned char*>(tile.entry->A + (int64_t)row * R) + 16 * col
                    : reinterpret_cast<const unsigned char*>(tile.entry->B + (int64_t)row * J) + 16 * col;
        w_to[i] = row * kWStride + 16 * col;
    }
    uint4 wr[KS];
    auto fetch = [&](int j) __attribute__((always_inline)) {
        const int64_t by = BACK ? (int64_t)j * R * 2 : (int64_t)j * 2;
#pragma unroll
        for (int i = 0; i < KS; ++i)
            wr[i] = w_has[i] && j + w_row[i] < J ? *reinterpret_cast<const uint4*>(w[i] + by) : make_uint4(0, 0, 0, 0);
    };
    auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < KS; ++i) *reinterpret_cast<uint4*>(smem + buf * kWBytes + w_to[i]) = wr[i];
    };
    const int l = 16 * tb + s;
    const int token = l < tile.tokens ? d.g.order[tile.begin + l] : -1;
    const bool real = token >= 0 && token < d.g.T;
    qblora_bf16* const out = d.out + (int64_t)(real ? token : 0) * d.ldo;
    fetch(j0);
    put(0);
    __syncthreads();
    for (int j = j0; j < j1; j += 64) {
        const int buf = ((j - j0) >> 6) & 1;
        if (j + 64 < j1) fetch(j + 64);
        for (int jb = jb0; jb < 4; jb += jb_step) {
            f32x4 acc{0.0f, 0.0f, 0.0f, 0.0f};
            const unsigned char* const ws = smem + buf * kWBytes;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                bf16x8 wf;
                if constexpr (BACK) {
                    wf = *reinterpret_cast<const bf16x8*>(ws + (16 * jb + s) * kWStride + 64 * k + 16 * g);
                } else {
                    const unsigned char* at = ws + (32 * k + 8 * g + (s >> 2)) * kWStride + 32 * jb + 8 * (s & 3);
                    const uint2 lo = columns_of(at), hi = columns_of(at + 4 * kWStride);
                    wf = __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
                }
                acc = mma(wf, uh[k], acc);
                acc = mma(wf, ul[k], acc);
            }
            const int at = j + 16 * jb + 4 * g;
            if (real && at < J) add_outputs<LAM>(out + (int64_t)at * LAM, acc, d.factor);
        }
        if (j + 64 < j1) put(buf ^ 1);
        __syncthreads();
    }
}

template <int LAM, bool BACK, int KS>
__global__ __launch_bounds__(kSpreadThreads) void k_spread(SpreadDesc d, int rows) {       // rows: outputs / lam of a workgroup
    extern __shared__ __align__(16) unsigned char smem[];
    Tile tile;
    if (!read_tile(d.g, blockIdx.x, &tile)) return;
    if (blockIdx.y == 0) {
        if (d.hi) write_pairs(d.g, tile, d.part, d.splits, d.hi);
        if (d.hi2) write_pairs(d.g, tile, d.part2, d.splits2, d.hi2);
    }
    if (!d.out) return;
    const int j0 = blockIdx.y * rows, j1 = min(j0 + rows, d.width / LAM);
    if (j0 >= j1) return;
    spread_many<LAM, BACK, KS>(d, tile, j0, j1, smem);
}

template <typename K>
int allow_lds(K kernel, int bytes) {
    return bytes <= 65536 || hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess
               ? QBLORA_OK : QBLORA_ERR_LAUNCH;
}

template <int LAM, bool BACK>
int rank_sums(const RankDesc& d, hipStream_t st) {
    constexpr int lds = rank_lds<LAM, BACK>();
    const int rc = allow_lds(k_rank_sums<LAM, BACK>, lds);
    if (rc) return rc;
    k_rank_sums<LAM, BACK><<<dim3(d.g.tile_room, d.splits, (d.g.R + kRankRows - 1) / kRankRows), kRankThreads, lds, st>>>(d);
    return launch_status();
}

template <int LAM, bool BACK, int KS>
int spread(const SpreadDesc& d, hipStream_t st) {
    constexpr int lds = spread_lds<KS, BACK>();
    const int rc = allow_lds(k_spread<LAM, BACK, KS>, lds);
    if (rc) return rc;
    const int J = d.width / LAM, steps = (J + 63) / 64;
    const int parts = std::min(steps, std::max(1, 1024 / d.g.tile_room));
    const int rows = (steps + parts - 1) / parts * 64;
    k_spread<LAM, BACK, KS><<<dim3(d.g.tile_room, d.out ? (J + rows - 1) / rows : 1), kSpreadThreads, lds, st>>>(d, rows);
    return launch_status();
}
template <int LAM, bool BACK>
int spread_by_rank(const SpreadDesc& d, hipStream_t st) {
    if (d.g.R <= 64) return spread<LAM, BACK, 2>(d, st);
    if (d.g.R <= 128) return spread<LAM, BACK, 4>(d, st);
    if (d.g.R <= 256) return spread<LAM, BACK, 8>(d, st);
    return spread<LAM, BACK, 16>(d, st);
}

}  // namespace

int launch_adapter_table(const TableDesc& d, hipStream_t st) {
    k_adapter_table<<<1, 64, 0, st>>>(d);
    return launch_status();
}

int launch_adapter_groups(const GroupsDesc& d, hipStream_t st) {
    const int lds = (2 * ((d.n + 3) & ~3) + 2 * d.count + kGroupRequests) * 4;
    const int rc = allow_lds(k_adapter_groups, lds);
    if (rc) return rc;
    k_adapter_groups<<<std::max(1, (d.n + kGroupRequests - 1) / kGroupRequests), kGroupThreads, lds, st>>>(d);
    return launch_status();
}

int rank_splits(int tiles, int width, int R) {
    const int steps = width / 64, wanted = std::max(1, 512 / std::max(1, tiles));
    return std::min({steps, wanted, 16});
}

int launch_rank_sums(const RankDesc& d, hipStream_t st) {
    if (d.back) switch (d.lam) {
        case 1: return rank_sums<1, true>(d, st);
        case 2: return rank_sums<2, true>(d, st);
        case 4: return rank_sums<4, true>(d, st);
        default: return rank_sums<8, true>(d, st);
    }
    switch (d.lam) {
        case 1: return rank_sums<1, false>(d, st);
        case 2: return rank_sums<2, false>(d, st);
        case 4: return rank_sums<4, false>(d, st);
        default: return rank_sums<8, false>(d, st);
    }
}

int launch_spread(const SpreadDesc& d, hipStream_t st) {
    if (d.back) switch (d.lam) {
        case 1: return spread_by_rank<1, true>(d, st);
        case 2: return spread_by_rank<2, true>(d, st);
        case 4: return spread_by_rank<4, true>(d, st);
        default: return spread_by_rank<8, true>(d, st);
    }
    switch (d.lam) {
        case 1: return spread_by_rank<1, false>(d, st);
        case 2: return spread_by_rank<2, false>(d, st);
        case 4: return spread_by_rank<4, false>(d, st);
        default: return spread_by_rank<8, false>(d, st);
    }
}

}  // namespace qblora
