// Many adapters on one projection: the table, the batch's tokens by adapter, and the two halves of the adapter term.
//
//   rank sums   U[t][r] = factor * s_a * sum_k Z[t][k] W_a[k / lam][r]      (W = A on X; W = B transposed on dY)
//   spread      out[t][n] += factor * sum_r U[t][r] W_a[r][n / lam]         (W = B on Y; W = A transposed on dX)
//
// Mean and repetition are never made: a matrix operand's row of W serves lam inputs, a result lam outputs.  Both halves go tile
// by tile, a tile being up to 64 tokens of one adapter, so that W is read once for them.
//
// What bounds them and what they take, on one MI355X (a large copy reaches 5.1 TB/s there, read + write): single tokens are the stream of
// the adapters (256 tokens on 100 adapters, 8192 to 22016, R = 256: 210 MB of A in 41 us, 5.1 TB/s, 564 MB of B in 119, 4.7; eight tokens
// on eight adapters, 4096 square, 6.3 and 7.0 us, where an empty launch takes 3.5).  Training batches are X, dY and the outputs (7810
// tokens, 4096 square, R = 128: 64 MB in 21 us, 128 MB of outputs in and out in 38) until the products count (7842 tokens to 22016
// features, R = 256: 88 GFLOP and 345 MB in 153 us, 88 GFLOP in two parts and 690 MB in 240).  Grids are sized by the adapters of the table:
// 1500 tokens of one of them, 4096 square, R = 128, take 11 + 5 + 15 us in a table of one and 49 + 9 + 51 in one of 500.
#include <algorithm>

#include "adapters.h"

namespace qblora {

namespace {

typedef __attribute__((ext_vector_type(4))) short s16x4;

// ---- the table ---------------------------------------------------------------------------------------------------

__global__ __launch_bounds__(64) void k_adapter_table(TableDesc d) {
    if ((int)threadIdx.x < d.n) d.out[threadIdx.x] = d.entry[threadIdx.x];
}

// ---- tokens by adapter -------------------------------------------------------------------------------------------
//
// Every workgroup reads all requests into LDS and adds up the tokens of each adapter (integer sums: any order), scans them, and
// then serves 64 requests of its own: 16 threads a request add up what earlier requests of its adapter have, a wave writes its
// tokens.  64 single tokens 5.5 us, 1000 requests with 50000 tokens 11.9: reads that wait for one another, not bytes.
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
    int* const slots = tokens + d.count;
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

// A tile and its adapter, with numbers that keep all accesses inside the arrays; ok: they are those of a tile with an adapter
struct Tile { int begin, tokens, R; float s; const qblora_bf16* A; const qblora_bf16* B; bool ok; };

// Nothing here waits for the adapter's description, so that a caller may ask for the tile's tokens at the same time.
__device__ __forceinline__ Tile read_tile(const Grouped& g, int at) {
    const int4 e = reinterpret_cast<const int4*>(g.tiles)[at];
    const AdapterEntry* const entry = g.table + min(max(e.x, 0), g.count - 1);
    const uint4 matrices = *reinterpret_cast<const uint4*>(entry);
    const uint2 rank = *reinterpret_cast<const uint2*>(&entry->R);
    Tile tile;
    tile.begin = min(max(e.y, 0), g.T - 1);
    tile.tokens = min(min(max(e.z, 1), kTileTokens), g.T - tile.begin);
    tile.A = reinterpret_cast<const qblora_bf16*>((uint64_t)matrices.y << 32 | matrices.x);
    tile.B = reinterpret_cast<const qblora_bf16*>((uint64_t)matrices.w << 32 | matrices.z);
    tile.R = (int)rank.x;
    tile.s = __uint_as_float(rank.y);
    tile.ok = e.x >= 0 && e.x < g.count && e.y == tile.begin && e.z == tile.tokens && tile.R > 0 && tile.R <= g.R;
    return tile;
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

// ---- copies into LDS ----------------------------------------------------------------------------------------------

// 16 bytes a lane to lds_base + 16 * lane; no register is written
__device__ __forceinline__ void copy16_to_lds(const void* p, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds_base), "v"(p) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
// At most n (uniform) of this wave's copies are under way; an odd n waits for one more
__device__ __forceinline__ void wait_copies(int n) {
    switch (n >> 1) {
        case 0: asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); break;
        case 1: asm volatile("s_waitcnt vmcnt(2)" ::: "memory"); break;
        case 2: asm volatile("s_waitcnt vmcnt(4)" ::: "memory"); break;
        case 3: asm volatile("s_waitcnt vmcnt(6)" ::: "memory"); break;
        case 4: asm volatile("s_waitcnt vmcnt(8)" ::: "memory"); break;
        case 5: asm volatile("s_waitcnt vmcnt(10)" ::: "memory"); break;
        default: asm volatile("s_waitcnt vmcnt(12)" ::: "memory"); break;
    }
}
// Every wave is here, with its reads of LDS behind it
__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// ---- rank sums ---------------------------------------------------------------------------------------------------
//
// Many tokens: steps of 64 inputs, Z's rows and W's copied straight into a ring of three stages in LDS.  The matrix product's rows are r
// (16 a block, blocks dealt to the four waves), its columns tokens.  W's rows lie by input (A: the transposing read makes
// the operand) or by r (B).  Both factors are bf16 as they are, the products exact, the sums fp32.  The 16-byte chunks of
// a row change places by its number, so that what a wave reads at once lies in different banks.
constexpr int kRankThreads = 256, kRankRows = 256;         // r of a workgroup at most
constexpr int kRankStages = 3;
constexpr int kZBytes = kTileTokens * 128;

// Copies of W that a wave makes for a step, for so many r
template <int LAM>
__host__ __device__ constexpr int rank_w_copies(int R) { return (R * (8 / LAM) + kRankThreads - 1) / kRankThreads; }
template <int LAM>
int rank_lds(int R) { return kRankStages * (kZBytes + rank_w_copies<LAM>(std::min(R, kRankRows)) * kRankThreads * 16); }

// Where the 16-byte chunks of a row in LDS go: chunk c of row `row` lies at c ^ swap(row, chunks of a row), so that what half a wave
// reads at once fills all banks.  A transposing read takes two chunks of four neighbouring rows, and of four more `APART` rows on;
// a row read takes one chunk of 16 rows.
template <int APART>
__device__ __forceinline__ int column_swap(int row, int chunks) {
    const int u = (row & 3) | (APART == 8 ? row >> 1 & 4 : row & 4);
    return chunks % 16 == 0 ? u << 1 : chunks % 8 == 0 ? u & 6 : chunks % 4 == 0 ? u >> 1 & 2 : 0;
}
__device__ __forceinline__ int row_swap(int row, int chunks) {
    return chunks % 16 == 0 ? row & 15 : chunks % 8 == 0 ? row >> 1 & 7 : chunks % 4 == 0 ? row >> 2 & 3 : chunks % 2 == 0 ? row >> 3 & 1 : 0;
}

template <int LAM, bool BACK>
__device__ void rank_many(const RankDesc& d, const Tile& tile, const int (&tokens)[2], int step0, int step1, int r_base, float* part, unsigned char* smem) {
    constexpr int kWRows = 64 / LAM;                       // of A for a step
    constexpr int kMost = rank_w_copies<LAM>(kRankRows);
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int R = min(tile.R - r_base, kRankRows);
    const int J = d.width / LAM;
    const int tb_n = (tile.tokens + 15) / 16;
    // Z: copy i of a wave takes rows 8 (wave + 4 i) .. + 7, 128 bytes each
    const int z_copies = tile.tokens > 32 ? 2 : 1;
    const unsigned char* z[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int token = min(max(tokens[i], 0), d.g.T - 1);
        z[i] = reinterpret_cast<const unsigned char*>(d.Z + (int64_t)token * d.ldz) + (int64_t)step0 * 128 + 16 * ((lane & 7) ^ (lane >> 3));
    }
    // W: chunks of 16 bytes, `per` of them a row; places behind the last chunk fetch the first
    const int per = BACK ? 8 / LAM : R / 8, chunks = R * (8 / LAM);
    const int w_copies = rank_w_copies<LAM>(R);
    const unsigned char* const w = reinterpret_cast<const unsigned char*>(BACK ? tile.B + (int64_t)r_base * J : tile.A + r_base);
    uint32_t w_from[kMost];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        int c = (i * 4 + wave) * 64 + lane;
        if (c >= chunks) c = 0;
        const int row = c / per, col = c % per ^ (BACK ? row_swap(row, per) : column_swap<LAM == 1 ? 8 : 4>(row, per));
        w_from[i] = (uint32_t)row * (uint32_t)((BACK ? J : tile.R) * 2) + 16 * col;
    }
    const int64_t w_step = BACK ? 128 / LAM : (int64_t)kWRows * tile.R * 2;    // bytes to the next step
    const unsigned char* w_at = w + step0 * w_step;
    const int stage_bytes = kZBytes + w_copies * kRankThreads * 16;
    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(smem)) + wave * 1024;
    auto issue = [&](int buf) __attribute__((always_inline)) {
        const uint32_t to = lds + buf * stage_bytes;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i >= z_copies) break;
            copy16_to_lds(z[i], to + i * 4096);
            z[i] += 128;
        }
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            if (i >= w_copies) break;
            copy16_to_lds(w_at + w_from[i], to + kZBytes + i * 4096);
        }
        w_at += w_step;
    };
    const int blocks = (R + 15) / 16, mine = (blocks - wave + 3) / 4;          // blocks wave, wave + 4, ...
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[i][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // Offsets of this lane's operands in a stage: of Z by the half of a step, of W by that and by whether the block is an odd one of the
    // wave's (blocks 4 further lie 8 chunks on, which a swap may turn; 16 chunks on it does not).  Rows of W behind R, and what lies
    // behind the copied ones, make sums that are not kept.
    const int g = lane >> 4, s = lane & 15, stride = 16 * per;
    int z_off[2], w_off[2][2], which[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        z_off[ks] = s * 128 + 16 * ((4 * ks + g) ^ (s & 7));
        const int k = (32 * ks + 8 * g) / LAM;                                 // first row of W of this lane's eight inputs
        which[ks] = LAM == 4 ? (k & 3) >> 1 : k & 3;
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
            if constexpr (BACK) {
                const int row = 16 * (wave + 4 * odd) + s;
                w_off[ks][odd] = kZBytes + row * stride + 16 * (k >> 3 ^ row_swap(row, per)) + 2 * (k & 4);
            } else {
                const int row = (k & ~3) + (s >> 2);
                w_off[ks][odd] = kZBytes + row * stride + 16 * ((2 * (wave + 4 * odd) + ((s & 3) >> 1)) ^ column_swap<LAM == 1 ? 8 : 4>(row, per)) + 8 * (s & 1);
            }
        }
    }
    const int w_two = BACK ? 128 * stride : 256;                               // from a block to the second next of the wave's
    auto products = [&](int buf) __attribute__((always_inline)) {
        const unsigned char* const at = smem + buf * stage_bytes;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            bf16x8 zf[4];
#pragma unroll
            for (int b = 0; b < 4; ++b)
                if (b < tb_n) zf[b] = *reinterpret_cast<const bf16x8*>(at + z_off[ks] + b * 2048);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= mine) break;
                const unsigned char* const from = at + w_off[ks][i & 1] + (i >> 1) * w_two;
                bf16x8 wf;
                if constexpr (BACK && LAM == 1) {
                    wf = *reinterpret_cast<const bf16x8*>(from);
                } else if constexpr (BACK) {
                    wf = repeated<LAM>(*reinterpret_cast<const uint2*>(from), which[ks]);
                } else if constexpr (LAM == 1) {
                    const uint2 lo = columns_of(from), hi = columns_of(from + 4 * stride);     // four rows on the chunks are moved alike
                    wf = __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
                } else {
                    wf = repeated<LAM>(columns_of(from), which[ks]);
                }
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    if (b < tb_n) acc[i][b] = mma(wf, zf[b], acc[i][b]);
            }
        }
    };
    const int steps = step1 - step0, per_stage = z_copies + w_copies;
    issue(0);
    if (steps > 1) issue(1);
    int buf = 0;
    for (int step = 0; step < steps; ++step) {
        wait_copies(step + 1 < steps ? per_stage : 0);
        meet();                                                                // this stage is in, the one before it is free
        if (step + 2 < steps) issue(buf == 0 ? 2 : buf - 1);
        products(buf);
        buf = buf == 2 ? 0 : buf + 1;
    }
    const float f = d.factor * tile.s;
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
    const Tile tile = read_tile(d.g, blockIdx.x);
    int tokens[2];                                             // of the rows that this lane copies
#pragma unroll
    for (int i = 0; i < 2; ++i) tokens[i] = d.g.order[tile.begin + min(8 * ((int)(threadIdx.x >> 6) + 4 * i) + (int)(threadIdx.x >> 3 & 7), tile.tokens - 1)];
    const int r_base = blockIdx.z * kRankRows, split = blockIdx.y;
    if (!tile.ok || r_base >= tile.R) return;
    const int all = d.width / 64;
    const int step0 = (int)((int64_t)all * split / d.splits), step1 = (int)((int64_t)all * (split + 1) / d.splits);
    float* const part = d.part + (int64_t)split * d.g.T * d.g.R;
    rank_many<LAM, BACK>(d, tile, tokens, step0, step1, r_base, part, smem);
}

// ---- spread ------------------------------------------------------------------------------------------------------
//
// U as a bf16 pair (high part and what is left: 16 significant bits) in registers, 16 tokens a wave, all r.  Steps of 128 outputs
// (64 with lam = 1): the rows of W that serve them and the outputs as they were go straight into a ring in LDS.  The matrix
// product's rows are outputs / lam, its columns tokens, so that a lane has 4 neighbouring rows of one token, 4 lam outputs.
// The results of a step are stored behind the next barrier, before the next copies are issued: the newest operations a wave waits
// around are then its copies alone, whose number it knows.
constexpr int kWideWaves = 8, kFewWaves = 4;                                  // of a workgroup, for tiles of up to 64 tokens and of up to 16
constexpr int kFewThreads = 64 * kFewWaves;
// Rows of W for a step of a tile of up to ROOM tokens.  Half as many for inner ranks above 256, of which two whole stages would take all of a
// CU's LDS, and with ROOM = 16 above 128, where they would leave a CU one workgroup.  Tiles of 64 tokens keep whole steps up to 256
// although a CU then has one workgroup too (R = 256, lambda = 2: three stages of 48 KB).
template <int LAM, int KS, int ROOM>
__host__ __device__ constexpr int spread_rows() {
    return (ROOM == 16 ? KS < 8 : KS <= 8) ? (LAM == 1 ? 64 : 128 / LAM) : LAM == 1 ? 32 : LAM == 8 ? 16 : 64 / LAM;
}
template <int LAM, int KS, int ROOM>
__host__ __device__ constexpr int spread_out_bytes() { return 2 * LAM * spread_rows<LAM, KS, ROOM>(); }     // of a token, for a step
// Copies of W that a wave makes for a step
template <int LAM, int KS, int ROOM>
__host__ __device__ constexpr int spread_w_copies(int R) {
    constexpr int threads = 64 * (ROOM == 16 ? kFewWaves : kWideWaves);
    return (R * (spread_rows<LAM, KS, ROOM>() / 8) + threads - 1) / threads;
}
// Bytes of a stage that hold outputs of up to ROOM tokens: a copy of each wave at least
template <int LAM, int KS, int ROOM>
__host__ __device__ constexpr int spread_out_room() {
    constexpr int least = 1024 * (ROOM == 16 ? kFewWaves : kWideWaves), bytes = ROOM * spread_out_bytes<LAM, KS, ROOM>();
    return bytes < least ? least : bytes;
}
template <int LAM, int KS, int ROOM>
__host__ __device__ constexpr int spread_stage_bytes(int R) {
    return spread_out_room<LAM, KS, ROOM>() + spread_w_copies<LAM, KS, ROOM>(R) * 1024 * (ROOM == 16 ? kFewWaves : kWideWaves);
}
// U of a tile in LDS, where the workgroup adds up the slices
__host__ __device__ constexpr int spread_u_bytes(int tokens, int R) { return (tokens < kTileTokens ? tokens : kTileTokens) * 4 * R; }

// The bf16 value next to v that a finite v leaves finite, and what it leaves: nothing of an infinity, which would make NaN of it
__device__ __forceinline__ float high_part(float v) {
    const float h = bf16_lo(pack_bf16(v, 0.0f));
    return __builtin_isinf(h) && !__builtin_isinf(v) ? copysignf(0x1.fep127f, v) : h;
}
__device__ __forceinline__ float left_of(float v, float high) { return __builtin_isinf(high) ? 0.0f : v - high; }
__device__ __forceinline__ void split_pair(float4 v, uint2* hi, uint2* lo) {
    const float4 h = make_float4(high_part(v.x), high_part(v.y), high_part(v.z), high_part(v.w));
    hi->x = pack_bf16(h.x, h.y); hi->y = pack_bf16(h.z, h.w);
    lo->x = pack_bf16(left_of(v.x, h.x), left_of(v.y, h.y));
    lo->y = pack_bf16(left_of(v.z, h.z), left_of(v.w, h.w));
}

// Four neighbouring r of the sum of the slices, always in the same order; eight loads under way together
__device__ __forceinline__ float4 sum_slices(const float* part, int splits, int64_t slice, int64_t at) {
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int z0 = 0; z0 < splits; z0 += 8) {
        float4 w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const float4*>(part + (int64_t)min(z0 + i, splits - 1) * slice + at);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (z0 + i < splits) { v.x += w[i].x; v.y += w[i].y; v.z += w[i].z; v.w += w[i].w; }
    }
    return v;
}

// The U of a tile in LDS, 4 R bytes a token; where R is a multiple of 32 the 16-byte chunks change places by the token
__device__ __forceinline__ int u_at(int l, int quad, int R) { return 4 * R * l + 16 * (quad ^ (R % 32 == 0 ? l & 7 : 0)); }
__device__ __forceinline__ void sum_tile(const SpreadDesc& d, const Tile& tile, unsigned char* us, int threads) {
    const int quads = tile.R / 4;
    const int64_t slice = (int64_t)d.g.T * d.g.R;
    for (int i = threadIdx.x; i < tile.tokens * quads; i += threads)
        *reinterpret_cast<float4*>(us + u_at(i / quads, i % quads, tile.R)) =
            sum_slices(d.part, d.splits, slice, (int64_t)(tile.begin + i / quads) * d.g.R + 4 * (i % quads));
    __syncthreads();
}

// 4 rows of LAM outputs each: what was there, at `from`, and f * v
template <int LAM>
__device__ __forceinline__ void add_outputs(uint4* o, const unsigned char* from, const f32x4& v, float f, int chunk, int swap) {
    if constexpr (LAM == 1) {
        const uint2 w = *reinterpret_cast<const uint2*>(from + 16 * ((chunk >> 1) ^ swap) + 8 * (chunk & 1));
        o->x = pack_bf16(bf16_lo(w.x) + f * v[0], bf16_hi(w.x) + f * v[1]);
        o->y = pack_bf16(bf16_lo(w.y) + f * v[2], bf16_hi(w.y) + f * v[3]);
    } else {
#pragma unroll
        for (int i = 0; i < LAM / 2; ++i) {
            const uint4 w = *reinterpret_cast<const uint4*>(from + 16 * ((chunk * (LAM / 2) + i) ^ swap));
            const float x = f * v[8 * i / LAM], y = f * v[(8 * i + 2) / LAM], z = f * v[(8 * i + 4) / LAM], u = f * v[(8 * i + 6) / LAM];
            o[i] = make_uint4(pack_bf16(bf16_lo(w.x) + x, bf16_hi(w.x) + x), pack_bf16(bf16_lo(w.y) + y, bf16_hi(w.y) + y),
                              pack_bf16(bf16_lo(w.z) + z, bf16_hi(w.z) + z), pack_bf16(bf16_lo(w.w) + u, bf16_hi(w.w) + u));
        }
    }
}

// Rows j0 .. j1 - 1 of W for a tile of at most ROOM tokens; `rows_u`: LDS behind the ring
template <int LAM, bool BACK, int KS, int ROOM>
__device__ void spread_tile(const SpreadDesc& d, const Tile& tile, int j0, int j1, int stages, unsigned char* smem, unsigned char* rows_u) {
    constexpr int kRows = spread_rows<LAM, KS, ROOM>(), kOutBytes = spread_out_bytes<LAM, KS, ROOM>(), kOutChunks = kOutBytes / 16;
    constexpr int kBlocks = kRows / 16;                                        // of 16 rows of W, for a step
    constexpr int kMost = spread_w_copies<LAM, KS, ROOM>(32 * KS), kWaves = ROOM == 16 ? kFewWaves : kWideWaves;
    const int J = d.width / LAM;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4, s = lane & 15;
    const int R = tile.R;
    const int64_t slice = (int64_t)d.g.T * d.g.R;
    // token blocks: 1, 2 or 4 of them side by side, the other waves take other rows of W
    const int tbs = ROOM == 16 || tile.tokens <= 16 ? 1 : tile.tokens <= 32 ? 2 : 4;
    // outputs: a copy is 1 KB of neighbouring tokens' 128 (64) outputs; what lies behind the row's end fetches its last chunk
    constexpr int kTokensACopy = 1024 / kOutBytes;
    constexpr int kOutCopies = ROOM / (kWaves * kTokensACopy) > 0 ? ROOM / (kWaves * kTokensACopy) : 1;
    const int o_copies = max(1, tbs * 16 / (kWaves * kTokensACopy));
    const unsigned char* o_from[kOutCopies];
    int o_col[kOutCopies];
    const int o_last = 2 * d.width - 16;
#pragma unroll
    for (int i = 0; i < kOutCopies; ++i) {
        const int l = kTokensACopy * (wave + kWaves * i) + lane / kOutChunks;
        const int token = min(max(d.g.order[tile.begin + min(l, tile.tokens - 1)], 0), d.g.T - 1);
        o_from[i] = reinterpret_cast<const unsigned char*>(d.out + (int64_t)token * d.ldo);
        o_col[i] = 2 * LAM * j0 + 16 * (lane % kOutChunks ^ (l & (kOutChunks - 1)));
    }
    // W: chunks of 16 bytes, `per` of them a row; places behind the last chunk, or behind the last row of outputs, fetch the first
    const int per = BACK ? R / 8 : kRows / 8, chunks = R * (kRows / 8);
    const int w_copies = spread_w_copies<LAM, KS, ROOM>(R);
    const unsigned char* const w = reinterpret_cast<const unsigned char*>(BACK ? tile.A : tile.B);
    uint32_t w_from[kMost];
    int w_row[kMost];                                                          // first of the step's outputs / lam that the chunk holds
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        int c = (i * kWaves + wave) * 64 + lane;
        if (c >= chunks) c = 0;
        const int row = c / per, col = c % per ^ (BACK ? row_swap(row, per) : column_swap<8>(row, per));
        w_from[i] = (uint32_t)row * (uint32_t)((BACK ? R : J) * 2) + 16 * col;
        w_row[i] = BACK ? row : 8 * col;
    }
    constexpr int kWAt = spread_out_room<LAM, KS, ROOM>();
    const int stage_bytes = kWAt + w_copies * kWaves * 1024;
    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(smem)) + wave * 1024;
    auto issue = [&](int j, int buf) __attribute__((always_inline)) {
        const uint32_t to = lds + buf * stage_bytes;
#pragma unroll
        for (int i = 0; i < kOutCopies; ++i) {
            if (i >= o_copies) break;
            copy16_to_lds(o_from[i] + min(o_col[i] + 2 * LAM * (j - j0), o_last), to + i * kWaves * 1024);
        }
        const unsigned char* const at = w + (BACK ? (int64_t)j * R * 2 : (int64_t)j * 2);
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            if (i >= w_copies) break;
            copy16_to_lds(j + w_row[i] < J ? at + w_from[i] : w, to + kWAt + i * kWaves * 1024);
        }
    };
    issue(j0, 0);
    if (stages == 3 && j0 + kRows < j1) issue(j0 + kRows, 1);

    const int tb = wave % tbs, jb0 = wave / tbs, jb_step = kWaves / tbs;
    const int l = 16 * tb + s;
    const int token = l < tile.tokens ? d.g.order[tile.begin + l] : -1;
    const bool real = token >= 0 && token < d.g.T;
    qblora_bf16* const out = d.out + (int64_t)(real ? token : 0) * d.ldo;
    bf16x8 uh[KS], ul[KS];
    const int l_real = min(l, tile.tokens - 1);
    if (!d.u) {
        sum_tile(d, tile, rows_u, 64 * kWaves);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int r = 32 * k + 8 * g;
            uint2 h0 = make_uint2(0, 0), h1 = h0, l0 = h0, l1 = h0;
            if (r < R) {
                split_pair(*reinterpret_cast<const float4*>(rows_u + u_at(l_real, r / 4, R)), &h0, &l0);
                split_pair(*reinterpret_cast<const float4*>(rows_u + u_at(l_real, r / 4 + 1, R)), &h1, &l1);
            }
            uh[k] = __builtin_bit_cast(bf16x8, make_uint4(h0.x, h0.y, h1.x, h1.y));
            ul[k] = __builtin_bit_cast(bf16x8, make_uint4(l0.x, l0.y, l1.x, l1.y));
        }
    } else {
        const qblora_bf16* const row = d.u + (int64_t)(tile.begin + l_real) * d.g.R;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int r = 32 * k + 8 * g;
            uint4 h = make_uint4(0, 0, 0, 0), lo = h;
            if (r < R) {
                h = *reinterpret_cast<const uint4*>(row + r);
                lo = *reinterpret_cast<const uint4*>(row + slice + r);
            }
            uh[k] = __builtin_bit_cast(bf16x8, h);
            ul[k] = __builtin_bit_cast(bf16x8, lo);
        }
    }
    const int last = (R - 1) / 32;                                             // step of r that may hold r behind R
    const bool behind = 32 * last + 8 * g >= R;
    // Offsets of this lane's operands in a stage.  B: the rows of 32 r lie a whole number of times 16 rows on, where the chunks are
    // moved alike, and so do four rows; a block's chunks change places with the block's number.  A: 8 chunks on, likewise.
    int w_off[BACK ? 4 : 1];
    if constexpr (BACK) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w_off[k] = kWAt + s * 2 * R + 16 * ((4 * k + g) ^ row_swap(s, per));
    } else {
        const int row = 8 * g + (s >> 2);
        w_off[0] = row * (2 * kRows) + 16 * (((s & 3) >> 1) ^ column_swap<8>(row, kRows / 8)) + 8 * (s & 1);
    }
    uint4 result[kBlocks][LAM == 1 ? 1 : LAM / 2];
    int result_at[kBlocks];
    auto store = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
            if (jb0 + i * jb_step >= kBlocks || result_at[i] >= J || !real) continue;
            qblora_bf16* const o = out + (int64_t)result_at[i] * LAM;
            if constexpr (LAM == 1) *reinterpret_cast<uint2*>(o) = make_uint2(result[i][0].x, result[i][0].y);
            else
#pragma unroll
                for (int e = 0; e < LAM / 2; ++e) *reinterpret_cast<uint4*>(o + 8 * e) = result[i][e];
        }
    };
    const int per_stage = o_copies + w_copies;
    int buf = 0;
    for (int j = j0; j < j1; j += kRows) {
        wait_copies(stages == 3 && j + kRows < j1 ? per_stage : 0);
        meet();                                                                // this step is in, the stage of the one before is free
        if (j > j0) store();
        const int ahead = j + (stages - 1) * kRows;
        if (ahead < j1) issue(ahead, buf == 0 ? stages - 1 : buf - 1);
        const unsigned char* const os = smem + buf * stage_bytes;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
            const int jb = jb0 + i * jb_step;
            if (jb >= kBlocks) continue;
            f32x4 acc{0.0f, 0.0f, 0.0f, 0.0f}, acc_lo = acc;                        // two chains of products
            const unsigned char* const block = BACK ? os + jb * (32 * R) : os + kWAt + (w_off[0] ^ (32 * jb));
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                if (k > last) continue;
                bf16x8 wf;
                if constexpr (BACK) {
                    wf = *reinterpret_cast<const bf16x8*>(block + w_off[k & 3] + 256 * (k >> 2));
                } else {
                    const uint2 lo = columns_of(block + 64 * k * kRows), hi = columns_of(block + 64 * k * kRows + 8 * kRows);
                    wf = __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
                }
                if (k == last && behind) wf = __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0));    // U is 0 there, W may be anything
                acc = mma(wf, uh[k], acc);
                acc_lo = mma(wf, ul[k], acc_lo);
            }
            acc += acc_lo;
            result_at[i] = j + 16 * jb + 4 * g;
            add_outputs<LAM>(result[i], os + l * kOutBytes, acc, d.factor, 4 * jb + g, l & (kOutChunks - 1));
        }
        buf = buf == stages - 1 ? 0 : buf + 1;
    }
    store();
}

template <int LAM, bool BACK, int KS>
__global__ __launch_bounds__(64 * kWideWaves) void k_spread(SpreadDesc d, int rows, int stages) {       // rows: of W, for a workgroup
    extern __shared__ __align__(16) unsigned char smem[];
    const Tile tile = read_tile(d.g, blockIdx.x);
    const int j0 = blockIdx.y * rows, j1 = min(j0 + rows, d.width / LAM);
    if (!tile.ok || j0 >= j1) return;
    spread_tile<LAM, BACK, KS, kTileTokens>(d, tile, j0, j1, stages, smem, smem + stages * spread_stage_bytes<LAM, KS, kTileTokens>(d.g.R));
}

// Few tokens of a batch.  Up to kFewTile of a tile, the usual thing while requests decode, are multiplied in the vector ALU: bound by the
// stream of B, of which every row is read once, straight into registers, eight loads a thread under way at any time, the first of
// them before U is there.  A piece is 256 rows of outputs: a thread has 8 neighbouring ones and every eighth r, and the eight
// shares are added in LDS.  Tiles of more tokens go 16 at a time through the matrix pipe.
constexpr int kFewTile = 4, kFewRows = 256, kFewAhead = 8;

template <int LAM, int KS, int MT>
__device__ void spread_few(const SpreadDesc& d, const Tile& tile, int j0, int j1, unsigned char* smem) {
    constexpr int kLoads = 4 * KS, kAhead = kLoads < kFewAhead ? kLoads : kFewAhead;
    const int t = threadIdx.x, share = t >> 5, R = tile.R, J = d.width / LAM, col = 8 * (t & 31);
    float* const us = reinterpret_cast<float*>(smem);                          // [R][MT]
    float* const sums = us + 32 * KS * MT;                                     // [8 shares][MT][256]
    const qblora_bf16* const B = tile.B + (int64_t)share * J;
    // No load is conditional, as loads behind a branch are waited for together: rows behind R and outputs behind the last fetch others
    // once more, which are not used.
    uint4 w[kAhead];
    auto load = [&](int i, int j) __attribute__((always_inline)) {            // row share + 8 i of the piece at j
        w[i % kAhead] = load16(B + (int64_t)(8 * i < R ? 8 * i : 0) * J + min(j + col, J - 8));
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(i, j0);
    qblora_bf16* out[MT];
    bool real[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int token = d.g.order[tile.begin + min(m, tile.tokens - 1)];
        real[m] = m < tile.tokens && token >= 0 && token < d.g.T;
        out[m] = d.out + (int64_t)min(max(token, 0), d.g.T - 1) * d.ldo;
    }
    const int quads = R / 4;
    const int64_t slice = (int64_t)d.g.T * d.g.R;
    for (int i = t; i < MT * quads; i += kFewThreads) {
        const int m = i / quads, r = 4 * (i % quads);
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (m < tile.tokens) v = sum_slices(d.part, d.splits, slice, (int64_t)(tile.begin + m) * d.g.R + r);
        us[r * MT + m] = v.x; us[(r + 1) * MT + m] = v.y; us[(r + 2) * MT + m] = v.z; us[(r + 3) * MT + m] = v.w;
    }
    __syncthreads();
    for (int j = j0; j < j1; j += kFewRows) {
        const bool mine = j + t < j1;
        const int64_t at = (int64_t)min(j + t, J - 1) * LAM;                     // the outputs of row j + t
        qblora_bf16 was[MT][LAM];
#pragma unroll
        for (int m = 0; m < MT; ++m) __builtin_memcpy(was[m], __builtin_assume_aligned(out[m] + at, 2 * LAM), 2 * LAM);
        float acc[MT][8];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[m][e] = 0.0f;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint4 v = w[i % kAhead];
            if (i + kAhead < kLoads) load(i + kAhead, j);
            else load(i + kAhead - kLoads, j + kFewRows);
            if (8 * i >= R) continue;
            const float b[8] = {bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y), bf16_lo(v.z), bf16_hi(v.z), bf16_lo(v.w), bf16_hi(v.w)};
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float u = us[(share + 8 * i) * MT + m];
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[m][e] = __fmaf_rn(u, b[e], acc[m][e]);
            }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float4* const to = reinterpret_cast<float4*>(sums + (share * MT + m) * kFewRows + col);
            to[0] = make_float4(acc[m][0], acc[m][1], acc[m][2], acc[m][3]);
            to[1] = make_float4(acc[m][4], acc[m][5], acc[m][6], acc[m][7]);
        }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (!mine || !real[m]) continue;
            float v = 0.0f;
#pragma unroll
            for (int q = 0; q < 8; ++q) v += sums[(q * MT + m) * kFewRows + t];
            v *= d.factor;
            qblora_bf16* const o = out[m] + at;
            if constexpr (LAM == 1) {
                o[0] = (qblora_bf16)pack_bf16(bf16_bits_to_float(was[m][0]) + v, 0.0f);
            } else {
                uint32_t pair[LAM / 2];
#pragma unroll
                for (int e = 0; e < LAM / 2; ++e) pair[e] = pack_bf16(bf16_bits_to_float(was[m][2 * e]) + v, bf16_bits_to_float(was[m][2 * e + 1]) + v);
                __builtin_memcpy(__builtin_assume_aligned(o, 2 * LAM), pair, 2 * LAM);
            }
        }
        __syncthreads();
    }
}

template <int LAM, int KS>
__device__ __forceinline__ void spread_few(const SpreadDesc& d, const Tile& tile, int j0, int j1, unsigned char* smem) {
    if (tile.tokens == 1) spread_few<LAM, KS, 1>(d, tile, j0, j1, smem);
    else if (tile.tokens == 2) spread_few<LAM, KS, 2>(d, tile, j0, j1, smem);
    else spread_few<LAM, KS, kFewTile>(d, tile, j0, j1, smem);
}

template <int LAM, int KS>
__global__ __launch_bounds__(kFewThreads, 2) void k_spread_few(SpreadDesc d, int rows, int stages) {
    extern __shared__ __align__(16) unsigned char smem[];
    const Tile whole = read_tile(d.g, blockIdx.y);
    const int j0 = blockIdx.x * rows, j1 = min(j0 + rows, d.width / LAM);
    if (!whole.ok || j0 >= j1) return;
    for (int from = 0; from < whole.tokens; from += 16) {
        Tile tile = whole;
        tile.begin += from;
        tile.tokens = min(whole.tokens - from, 16);
        if (from) __syncthreads();
        if (tile.tokens > kFewTile) spread_tile<LAM, false, KS, 16>(d, tile, j0, j1, stages, smem, smem + stages * spread_stage_bytes<LAM, KS, 16>(d.g.R));
        else if (KS > 1 && tile.R <= 32) spread_few<LAM, 1>(d, tile, j0, j1, smem);
        else if (KS > 2 && tile.R <= 64) spread_few<LAM, 2>(d, tile, j0, j1, smem);
        else if (KS > 4 && tile.R <= 128) spread_few<LAM, 4>(d, tile, j0, j1, smem);
        else spread_few<LAM, KS>(d, tile, j0, j1, smem);
    }
}
constexpr int few_bytes(int KS, int MT) { return 4 * MT * (32 * KS + 8 * kFewRows); }

// U as three bf16 parts, 24 significant bits: the sums of the slices of one or two arrays
__global__ __launch_bounds__(256) void k_rank_parts(PartsDesc d) {
    const Tile tile = read_tile(d.g, blockIdx.x);
    if (!tile.ok) return;
    const bool second = blockIdx.y != 0;
    const float* const part = second ? d.part2 : d.part;
    qblora_bf16* const out = second ? d.out2 : d.out;
    const int splits = second ? d.splits2 : d.splits, quads = tile.R / 4;
    const int64_t slice = (int64_t)d.g.T * d.g.R;
    for (int i = blockIdx.z * 256 + threadIdx.x; i < tile.tokens * quads; i += gridDim.z * 256) {
        const int64_t at = (int64_t)(tile.begin + i / quads) * d.g.R + 4 * (i % quads);
        const float4 v = sum_slices(part, splits, slice, at);
        uint2 h, m, l;
        split_pair(v, &h, &m);
        l.x = pack_bf16(left_of(v.x, bf16_lo(h.x)) - bf16_lo(m.x), left_of(v.y, bf16_hi(h.x)) - bf16_hi(m.x));
        l.y = pack_bf16(left_of(v.z, bf16_lo(h.y)) - bf16_lo(m.y), left_of(v.w, bf16_hi(h.y)) - bf16_hi(m.y));
        *reinterpret_cast<uint2*>(out + at) = h;
        *reinterpret_cast<uint2*>(out + slice + at) = m;
        *reinterpret_cast<uint2*>(out + 2 * slice + at) = l;
    }
}

// More than 64 KB of LDS has to be asked for, up to the whole of a CU's
template <typename K>
int allow_lds(K kernel, int bytes) {
    return bytes <= 64 * 1024 || hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) == hipSuccess
               ? QBLORA_OK : QBLORA_ERR_LAUNCH;
}

template <int LAM, bool BACK>
int rank_sums(const RankDesc& d, hipStream_t st) {
    const int lds = rank_lds<LAM>(d.g.R);
    const int rc = allow_lds(k_rank_sums<LAM, BACK>, lds);
    if (rc) return rc;
    k_rank_sums<LAM, BACK><<<dim3(d.g.tile_room, d.splits, (d.g.R + kRankRows - 1) / kRankRows), kRankThreads, lds, st>>>(d);
    return launch_status();
}

// Stages of a ring beside `more` bytes of LDS: three where two workgroups still fit a CU, else two if these do, else three if they fit at all
int ring_stages(int stage, int more) {
    const int half = 80 * 1024;
    return 3 * stage + more <= half ? 3 : 2 * stage + more <= half ? 2 : 3 * stage + more <= 2 * half ? 3 : 2;
}

template <int LAM, bool BACK, int KS>
int spread(const SpreadDesc& d, hipStream_t st) {
    constexpr int kRows = spread_rows<LAM, KS, kTileTokens>();
    const int J = d.width / LAM, steps = (J + kRows - 1) / kRows;
    const int more = d.u ? 0 : spread_u_bytes(std::min(d.g.T, kTileTokens), d.g.R), stage = spread_stage_bytes<LAM, KS, kTileTokens>(d.g.R);
    const int stages = ring_stages(stage, more);
    const int rc = allow_lds(k_spread<LAM, BACK, KS>, stages * stage + more);
    if (rc) return rc;
    // one round of workgroups where that fills nine tenths of the chip with eight steps each at least, else smaller ones in about
    // 1024: 125 tiles of 2048 rows 39 us with 500 workgroups, 42 with 1000 (4096 rows, R = 256: 94 with 250, 106 with 1000);
    // 88 of 2560 rows 25.4 with 440, 22.4 with 970
    const int slots = stages * stage + more <= 80 * 1024 ? 512 : 256;
    int parts = slots / d.g.tile_room;
    if (10 * parts * d.g.tile_room < 9 * slots || steps < 8 * parts) parts = 1024 / d.g.tile_room;
    parts = std::min(steps, std::max(1, parts));
    const int rows = (steps + parts - 1) / parts * kRows;
    k_spread<LAM, BACK, KS><<<dim3(d.g.tile_room, (J + rows - 1) / rows), 64 * kWideWaves, stages * stage + more, st>>>(d, rows, stages);
    return launch_status();
}

template <int LAM, int KS>
int spread_few_tokens(const SpreadDesc& d, hipStream_t st) {
    // Pieces of 256 rows of outputs, or of 64 where those would leave most CUs idle.  One round of workgroups, two a CU, while that gives
    // each few pieces (40 adapters, 860 pieces: 512 workgroups 12.6 us, 2048 16.2); else more and smaller ones, which even out at
    // the end (100 adapters, 4500 pieces: 1024 125 us, 2048 119).
    const int J = d.width / LAM, piece = d.g.tile_room * ((J + kFewRows - 1) / kFewRows) < 256 ? 64 : kFewRows;
    const int pieces = (J + piece - 1) / piece;
    const int parts = std::min(pieces, std::max(1, (pieces * d.g.tile_room <= 2048 ? 512 : 2048) / d.g.tile_room));
    const int rows = (pieces + parts - 1) / parts * piece;
    const int more = spread_u_bytes(16, d.g.R), stage = spread_stage_bytes<LAM, KS, 16>(d.g.R), stages = ring_stages(stage, more);
    const int lds = std::max(d.g.T > kFewTile ? stages * stage + more : 0, few_bytes(KS, d.g.T >= 3 ? 4 : d.g.T));
    const int rc = allow_lds(k_spread_few<LAM, KS>, lds);
    if (rc) return rc;
    k_spread_few<LAM, KS><<<dim3((J + rows - 1) / rows, d.g.tile_room), kFewThreads, lds, st>>>(d, rows, stages);
    return launch_status();
}
template <int LAM, bool BACK>
int spread_by_rank(const SpreadDesc& d, hipStream_t st) {
    if constexpr (!BACK)
        if (!d.u && spread_few_applies(d.g.count, d.g.T)) return d.g.R <= 64 ? spread_few_tokens<LAM, 2>(d, st) : d.g.R <= 128 ? spread_few_tokens<LAM, 4>(d, st) : spread_few_tokens<LAM, 8>(d, st);
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
    const int lds = (2 * ((d.n + 3) & ~3) + d.count + kGroupRequests) * 4;
    const int rc = allow_lds(k_adapter_groups, lds);
    if (rc) return rc;
    k_adapter_groups<<<std::max(1, (d.n + kGroupRequests - 1) / kGroupRequests), kGroupThreads, lds, st>>>(d);
    return launch_status();
}

// Slices of the inputs: as many workgroups as the CUs take at once (three each up to R = 128, by LDS, two above), but 16 steps a slice where
// that makes 512 workgroups all the same.  85 tiles of 13824 inputs: 5 slices 39 us, 8 32; 123 tiles of 4096: 4 slices 21.5 us, 6 23.5; of
// 8192 with R = 256: 2 slices 73 us, 4 48, 6 66.
int rank_splits(int tiles, int width, int R) {
    const int steps = width / 64, wanted = std::min((R <= 128 ? 768 : 512) / std::max(1, tiles), std::max(steps / 16, 512 / std::max(1, tiles)));
    return std::max(1, std::min({steps, wanted, std::max(16, std::min(steps / 4, 32))}));
}

int64_t rank_part_rows(int64_t T, int width) {
    return std::max(T, std::min(std::min<int64_t>(32, width / 64) * T, (int64_t)768 * kTileTokens));
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

int launch_rank_parts(const PartsDesc& d, hipStream_t st) {
    const int z = std::max(1, std::min(kTileTokens * d.g.R / 1024, 512 / d.g.tile_room));
    k_rank_parts<<<dim3(d.g.tile_room, d.out2 ? 2 : 1, z), 256, 0, st>>>(d);
    return launch_status();
}

// From so many tokens on, or inner ranks whose sums do not fit LDS beside the rest, sums that are cut into slices are added up once, in
// a launch of their own, and not by every workgroup that needs them
bool rank_parts_pay(int count, int64_t T, int R) { return T >= 1024 || R > 256 || (T > 8 * (int64_t)count && R > 64); }

// The kernel for few tokens of a tile where the batch has so few for each adapter, as far as their number tells (167 tokens on two
// adapters: 66 us with it, 230 tokens 40)
bool spread_few_applies(int count, int64_t T) { return T <= 8 * (int64_t)count; }

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
