// Attention of new tokens over the paged cache (qblora_paged_attention).
//
//   out = sum_j e_j v_j / sum_j e_j,  e_j = exp(scale q.k_j - m),  over the positions j a row sees, in one pass: m is the
//   maximum so far, and what was summed under a smaller one is multiplied by 2^(old - new) (the exponents are in base 2).
//
// Scores, maxima, sums and parts are fp32.  The matrix instruction takes the second product's operands in bf16.  attend_few, whose
// matrix pipe is idle most of the time, multiplies a weight e_j in two parts, cut to bf16 and what that leaves: 2^-16 of it is lost
// (64 tokens of 40 heads over 100 to 8000: 367 us with one part, 369 with two; one of 4095 16.8 and 17.0).  attend_many, which that pipe
// bounds, rounds it once: up to 2^-8 of each, which many positions average out (0.0024 of the result's size in all, where an output's
// own rounding is 0.0017).  The sum below the line is of the unrounded ones.
//
// A row is a query head of a new token; the rows of one request that share a key / value head go together, token by token
// (row r: token r / group, head r % group of the group), so that the cache is read once for all of them.
//
// attend_few takes 16 rows, the width of the matrix instruction, and is bound by the stream of the cache: a wave takes 32
// positions at a time straight from the pages into registers, in the operand order that the cache is stored in, with the
// next 32 in flight behind them.  Scores are formed transposed, S^T = K Q^T, so that a lane holds eight positions of one row,
// the operand of O^T = V^T P^T but for four exchanges between lanes.  The four waves of a workgroup take turns on the positions
// and are joined in LDS.  64 single tokens of 40 heads over 100 to 8000 positions (2.3 GB): 369 us, 6.2 TB/s of what a kernel
// that only reads gets 6.3 of; four of 64 heads, 8 of them with keys, over 30000 to 131000 (0.8 GB): 131 us, 6.2 TB/s; one of
// 4095 (67 MB): 12.4 to 14.6 us and 4 of the join.
//
// attend_many takes 128 rows, 32 a wave, and is bound by the matrix pipe and by the exponentials beside it.  64 positions at a
// time go through LDS, in the order of the pages (copies of 1 KB that need no registers, two tiles in turn, one barrier a
// tile); scores are transposed here too, so that a row's maximum and sum are a lane's own but for one exchange of halves.
// 4096 tokens over 12288, 32 heads (962 GFLOP): 865 us, 1110 TFLOP/s, 0.83 of what the library's large product reaches on the
// chip; two workgroups a CU, the matrix pipe busy for 0.59 of the cycles and the vector ALU for 0.48, at a power-limited 1.7
// GHz.  In small calls a tile takes 1.1 us of a workgroup alone on its CU and 1.9 of each of two, its start 3 to 5 us, the
// store of a part up to 1.7.  Heads of 64 are bound by the exponentials (4096 tokens over 4000, 32 heads, 203 GFLOP: 243 us, 840
// TFLOP/s), heads of 256 by one wave a SIMD (2000 over 2000, 16 heads, 98 GFLOP: 175 us, 560 TFLOP/s).
//
// Work: requests differ by orders of magnitude, and only the device knows their lengths.  Every workgroup adds up the work
// of all requests, which gives the number of positions that a workgroup takes if there are to be `target` of them, and finds
// its own (request, rows, range of positions) from the prefix sums.  A context that is cut this way leaves partial results
// in the workspace, which k_attn_join adds up.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "attn_units.h"
#include "decoder.h"

namespace qblora {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kFewRows = 16;
constexpr int kBlock = kAttnBlock;             // positions of a step
constexpr int kManyRows = 128;
constexpr float kNegInf = -__builtin_inff();
// A maximum may grow by 2^8 before what was summed is rescaled: the weights stay below 2^8 and most steps do without the 64
// products.  4096 tokens over 12288 took 974 us with every growth followed, 927 so.
constexpr float kSlack = 8.0f;

// Which requests a form takes, and how their work is shared out: units of `rows` rows, about `target` of them for a key /
// value head, at least `least` blocks each.  A tile that is longer than a unit is cut into parts no longer than one, or, with
// `slack`, into as many as come nearest.  Cut tiles leave their parts in `part` and themselves in `cut`; `cuts` counts them.
struct CutTile { int token0, rem0, rows, splits, slot, pad[3]; };
enum { FEW = 1, LOT = 2, ALL = 3 };            // the requests of few rows, those of more, or all
struct Share { int rows, target, least, slack, form, grid_units; int* cuts; CutTile* cut; float* part; };   // grid_units: a key / value head
// Few rows: with 512 units 4 contexts of 30000 to 131000 take 151 us, with 1024 131, with 2048 139; single tokens of 16 x 1000 to
// 8000 positions 55.9, 51.3 and 54.9.  With 4 blocks at least, one of 4095 takes 20.5, with 8 17.4, with 16 17.4.
// Heads of 256 leave one workgroup a CU: 4 of 16 / 4 heads over 10000 to 60000 120 us with 1024, 112 with 512, 145 with 256 (64 of
// 16 over 500 to 3000 242, 248 and 248).
constexpr int kFewTarget = 1024, kFewWideTarget = 512, kFewLeast = 8;
// More rows: every part costs 66 KB of writes and as many of reads, so there are fewer units than places.  175 tokens of 64 / 8
// heads over 3985 take 42 us with 384, 60 with 512, 47 with 256; 128 of 32 heads over 2000 22.6 with 16 blocks at least, 30.0 with 12,
// 24.3 with 24.  Without the slack, 175 over 3985 take 50 us, 128 over 2000 30.7, and 1000 of 40 heads without a context 39.1 instead of 29.8.
// Heads of 256: 512 tokens of 16 heads over 2000 79 us with 384, which is one round and a half, and 51 with 256.
constexpr int kManyTarget = 384, kManyWideTarget = 256, kManyLeast = 16;
// Requests of up to kSomeRows rows go to attend_few, 16 rows at a time, if they do not make more than kSomeBlocks blocks in all:
// what the chip takes at once in units of kFewLeast.  Four tokens of 8 heads a key head over 4000: 14.0 us that way, 17.7 in one
// tile of 128 rows; 16 of those requests over 1000 to 4000, above the limit, 49.7 and 37.3.
constexpr int kSomeRows = 64, kSomeBlocks = 512 * kFewLeast;
static_assert(2 * kFewTarget < 1 << 15 && 2 * kManyTarget < 1 << 15, "parts and cut tiles are counted in halves of a word");

// x / group for x < 128 + group: the magic number is 2^32 / group + 1, whose excess is less than x * group / 2^32 < 1
__device__ __forceinline__ int quotient(const AttnDesc& d, int x) { return d.group == 1 ? x : (int)__umulhi((uint32_t)x, d.group_magic); }

// A workgroup's rows and range of positions; slot: its place among the parts, cut: its tile's among those that are cut
struct Unit { int request, tile, split, splits, slot, cut; };

struct Span { int start, fresh, context; };
__device__ __forceinline__ Span span_of(const AttnDesc& d, int i) {
    const int s0 = min(max(d.starts[i], 0), d.T), s1 = min(max(d.starts[i + 1], s0), d.T);
    return {s0, s1 - s0, context_of(d.context[i])};
}

// of a request that the whole wave works on
__device__ __forceinline__ Span uniform_span_of(const AttnDesc& d, int i) {
    const Span s = span_of(d, i);
    return {__builtin_amdgcn_readfirstlane(s.start), __builtin_amdgcn_readfirstlane(s.fresh), __builtin_amdgcn_readfirstlane(s.context)};
}

// sum over the lanes up to this one
__device__ __forceinline__ int scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);    // from 1, 2, 4 and 8 lanes before, in rows of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);    // the last lane of a row to the next one
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);    // lane 31 to the upper half
    return x;
}
__device__ __forceinline__ int64_t sum_of_wave(int64_t x) {
    if (__all((uint64_t)x < 1u << 25)) return __builtin_amdgcn_readlane(scan((int)x), 63);
    for (int s = 32; s; s >>= 1) x += __shfl_xor(x, s);
    return x;
}

// of a tile of `rows` rows of this request.  (Charged with what all of the request's tokens see, 1500 tokens of 12 / 4 heads over 2000
// with a window of 64 are cut in three parts a tile, two of them empty: 22.6 us where this takes 16.0.)
__device__ __forceinline__ int tile_blocks(const AttnDesc& d, const Span& s, int rows) {
    return blocks_of_tile(s.context, s.fresh, d.width << d.page_shift, d.window, quotient(d, rows - 2 + d.group));
}
// `some`: the rows up to which requests go to attend_few in this call, where both forms are there
__device__ __forceinline__ Cost cost_of(const AttnDesc& d, const Span& s, const Share& w, int some) {
    const int64_t rows = (int64_t)s.fresh * d.group;
    if (rows == 0 || (w.form == FEW && rows > some) || (w.form == LOT && rows <= some)) return {0, 0};
    return {(int)((rows + w.rows - 1) / w.rows), tile_blocks(d, s, w.rows)};
}

// The unit number `want` of the batch; false: there are not so many.  With `first`, the number of cut tiles is left where
// k_attn_join looks for it: 0 if there are more units than the grid runs, as an entry that no workgroup writes is not to be read.  All threads call it.  Up to 64 requests every wave finds it by itself, a request a lane; more
// are taken a workgroup's threads at a time.
struct Finder {
    int64_t sums[kWaves];
    int ends[2][kWaves], found[6];
};
__device__ __forceinline__ bool find_unit(const AttnDesc& d, const Share& share, int want, bool first, Finder& f, Unit& u) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (d.n <= 64) {
        Span s{0, 0, 0};
        if (lane < d.n) s = span_of(d, lane);
        int some = kFewRows;
        if (share.form != ALL) {
            const int64_t rows = (int64_t)s.fresh * d.group;
            const bool between = rows > kFewRows && rows <= kSomeRows;
            if (__any(between)) {
                const int64_t blocks = between ? (rows + kFewRows - 1) / kFewRows * tile_blocks(d, s, kFewRows) : 0;
                if (sum_of_wave(blocks) * d.kv_heads <= kSomeBlocks) some = kSomeRows;
            }
        }
        const Cost c = cost_of(d, s, share, some);
        const Units v = units_of(c, blocks_per_unit(sum_of_wave((int64_t)c.tiles * c.blocks), share.target, share.least), share.slack);
        const int mine = units_within(v.count, share.grid_units);
        const int a = scan(mine), b = scan(v.cuts);
        if (first && tid == 63) *share.cuts = cut_tiles(b, a, share.grid_units);
        const uint64_t hit = __ballot(mine && a - mine <= want && want < a);
        if (!hit) return false;
        const int at = __builtin_ctzll(hit);
        const int number = want - __builtin_amdgcn_readlane(a - mine, at);
        const int before = __builtin_amdgcn_readlane(b - v.cuts, at);
        u.request = at;
        u.splits = __builtin_amdgcn_readlane(v.splits, at);
        u.tile = number / u.splits;
        u.split = number - u.tile * u.splits;
        u.slot = (before & 0xffff) + number;
        u.cut = (before >> 16) + u.tile;
        return true;
    }
    int64_t all = 0;
    for (int i = tid; i < d.n; i += kThreads) {
        all = add_blocks(all, cost_of(d, span_of(d, i), share, kFewRows));
    }
    all = sum_of_wave(all);
    if (lane == 0) f.sums[wave] = all;
    if (tid == 0) f.found[0] = -1;
    __syncthreads();
    all = 0;
    for (int w = 0; w < kWaves; ++w) all += f.sums[w];
    const int per = blocks_per_unit(all, share.target, share.least);
    int units = 0, cuts = 0;                                           // in front of these requests
    for (int base = 0; base < d.n; base += kThreads) {
        const int i = base + tid;
        Cost c{0, 0};
        if (i < d.n) c = cost_of(d, span_of(d, i), share, kFewRows);
        const Units v = units_of(c, per, share.slack);
        const int mine = units_within(v.count, share.grid_units);
        int a = scan(mine), b = scan(v.cuts);
        __syncthreads();
        if (lane == 63) { f.ends[0][wave] = a; f.ends[1][wave] = b; }
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) {
            if (w == wave) { a += units; b += cuts; }
            units = add_units(units, f.ends[0][w]);
            cuts += f.ends[1][w];
        }
        if (mine && a - mine <= want && want < a) {
            const int number = want - (a - mine), before = b - v.cuts;
            f.found[0] = i;
            f.found[1] = number / v.splits;
            f.found[2] = number % v.splits;
            f.found[3] = v.splits;
            f.found[4] = (before & 0xffff) + number;
            f.found[5] = (before >> 16) + number / v.splits;
        }
        __syncthreads();
        if (f.found[0] >= 0 && !first) break;
    }
    if (first && tid == 0) *share.cuts = cut_tiles(cuts, units, share.grid_units);
    u.request = __builtin_amdgcn_readfirstlane(f.found[0]);
    if (u.request < 0) return false;
    u.tile = __builtin_amdgcn_readfirstlane(f.found[1]);
    u.split = __builtin_amdgcn_readfirstlane(f.found[2]);
    u.splits = __builtin_amdgcn_readfirstlane(f.found[3]);
    u.slot = __builtin_amdgcn_readfirstlane(f.found[4]);
    u.cut = __builtin_amdgcn_readfirstlane(f.found[5]);
    return true;
}

// the rows of a tile (row0 is row `rem0` of token `token0`) and the positions that any of them sees
struct Tile { int row0, token0, rem0, rows, pos0, pos1, full0, full1; };       // full: positions that every row sees, as far as lengths go
__device__ __forceinline__ Tile tile_of(const AttnDesc& d, const Span& s, int tile, int rows) {
    Tile t;
    t.row0 = tile * rows;
    t.token0 = t.row0 / d.group;
    t.rem0 = t.row0 - t.token0 * d.group;
    t.rows = min(rows, s.fresh * d.group - t.row0);
    const int first = s.context + t.token0, last = first + quotient(d, t.rem0 + t.rows - 1);
    const int limit = d.width << d.page_shift;
    t.pos1 = min(last + 1, limit);
    t.pos0 = d.window ? max(first + 1 - d.window, 0) : 0;
    t.full1 = min(first + 1, limit);
    t.full0 = d.window ? max(last + 1 - d.window, 0) : 0;
    return t;
}

// A cut tile goes to where k_attn_join finds it.
__device__ __forceinline__ void note_cut(const Share& share, const Unit& u, int kvh, const Span& s, const Tile& t) {
    if (u.splits > 1 && u.split == 0 && kvh == 0 && threadIdx.x == 0) {
        CutTile c{s.start + t.token0, t.rem0, t.rows, u.splits, u.slot, {0, 0, 0}};
        share.cut[u.cut] = c;
    }
}

__device__ __forceinline__ bool not_finite(uint32_t pair) { return (((pair & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0; }

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 exponents(uint32_t pair) { return __builtin_bit_cast(u16x2, pair & 0x7f807f80u); }
__device__ __forceinline__ u16x2 larger(u16x2 a, u16x2 b) { return __builtin_elementwise_max(a, b); }

// all bits of an element or none
__device__ __forceinline__ uint32_t mask_of(uint32_t bits) { return (bits & 1u) * 0xffffu | (bits >> 1 & 1u) * 0xffff0000u; }
__device__ __forceinline__ uint32_t without_not_finite(uint32_t pair) {
    const uint32_t bad = ((pair & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
    return pair & ~((bad >> 15) * 0xffffu);
}

// an infinity or NaN, or 0
__device__ __forceinline__ float if_not_finite(qblora_bf16 x) { return (x & 0x7f80u) == 0x7f80u ? __uint_as_float((uint32_t)x << 16) : 0.0f; }
// feature 0 of a position's value (feature f is 8 f elements further); null where no page is listed
template <int D>
__device__ __forceinline__ const qblora_bf16* value_row(const AttnDesc& d, const int32_t* table, int kvh, int pos) {
    const int id = table[pos >> d.page_shift], in_page = pos & ((1 << d.page_shift) - 1);
    if ((uint32_t)id >= (uint32_t)d.pages) return nullptr;
    return d.vc + (((int64_t)id * d.kv_heads + kvh) * D << d.page_shift) + (in_page >> 3) * D * 8 + (in_page & 7);
}

// A part of the cache, of which no line is kept: the call reads it once, or, with more than 16 rows to a key head, once for every 16 of
// them, by workgroups that run side by side.  64 tokens of 40 heads over 100 to 8000: 411 us without,
// 376 with values that way, 368 with both.
__device__ __forceinline__ uint4 stream(const qblora_bf16* p) {
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p)));
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

template <int D>
struct FewShared {
    float o[kWaves][kFewRows][D + 4];
    float m[kWaves][kFewRows], l[kWaves][kFewRows];
};

template <int D>
__device__ __forceinline__ void attend_few(const AttnDesc& d, const Share& share, int block, Finder& finder, FewShared<D>& sh) {
    constexpr int KS = D / 32, DT = D / 16;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, col = lane & 15;
    const int kvh = block % d.kv_heads;
    Unit u;
    if (!find_unit(d, share, block / d.kv_heads, block == 0, finder, u)) return;
    const Span s = uniform_span_of(d, u.request);
    const Tile t = tile_of(d, s, u.tile, kFewRows);
    note_cut(share, u, kvh, s, t);
    const int b_first = t.pos0 / kBlock, b_last = (t.pos1 + kBlock - 1) / kBlock;
    const int per = (max(b_last - b_first, 0) + u.splits - 1) / u.splits;
    const int b0 = b_first + u.split * per, b1 = min(b0 + per, b_last);

    // rows: operand B, row = lane & 15, features 32 s + 8 g ..
    bf16x8 qf[KS];
    const int among = t.rem0 + col, ahead = quotient(d, among);            // tokens behind the tile's first
    const int token = t.token0 + ahead, head = kvh * d.group + among - ahead * d.group;
    const int here = s.context + token;
    const bool real = col < t.rows;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (real) v = *reinterpret_cast<const uint4*>(d.q + (int64_t)(s.start + token) * d.ldq + (int64_t)head * D + 32 * i + 8 * g);
        qf[i] = __builtin_bit_cast(bf16x8, v);
    }
    const int row_low = d.window ? here - d.window : -1;               // sees positions row_low < j <= here

    const int shift = d.page_shift, page = 1 << shift;
    const int64_t page_elems = (int64_t)d.kv_heads * D << shift, head_elems = ((int64_t)kvh * D) << shift;
    const int32_t* table = d.table + (int64_t)u.request * d.width;
    const int steps = b0 + wave < b1 ? (b1 - b0 - wave + kWaves - 1) / kWaves : 0;

    f32x4 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
    float m = kNegInf, l = 0.0f;
    int odd0 = INT_MAX, odd1 = 0;                                      // positions among which values are not finite

    int ids0 = -1, ids1 = -1;                                          // pages of the steps' halves, a step a lane
    uint4 kf[2][KS], vf[DT];

    // pages of a step (step 64 k first)
    auto find_pages = [&](int step, int& id0, int& id1) {
        if ((step & 63) == 0) {
            const int pos = (b0 + wave + kWaves * (step + lane)) * kBlock;
            ids0 = ids1 = -1;
            if (pos < t.pos1) ids0 = table[pos >> shift];
            if (pos + 16 < t.pos1) ids1 = table[(pos + 16) >> shift];
            if ((uint32_t)ids0 >= (uint32_t)d.pages) ids0 = -1;
            if ((uint32_t)ids1 >= (uint32_t)d.pages) ids1 = -1;
        }
        id0 = __builtin_amdgcn_readlane(ids0, step & 63);
        id1 = __builtin_amdgcn_readlane(ids1, step & 63);
    };
    auto load_keys = [&](int step, int id0, int id1) {
        const int base = (b0 + wave + kWaves * step) * kBlock;
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            const int id = max(tt == 0 ? id0 : id1, 0);
            const qblora_bf16* k = d.kc + id * page_elems + head_elems + ((g << shift) + ((base + 16 * tt) & (page - 1)) + col) * 8;
#pragma unroll
            for (int i = 0; i < KS; ++i) kf[tt][i] = stream(k + ((4 * i) << shift) * 8);
        }
    };
    auto load_values = [&](int step, int id0, int id1) {
        const int base = (b0 + wave + kWaves * step) * kBlock;
        const int id = max(g < 2 ? id0 : id1, 0);
        const qblora_bf16* v = d.vc + id * page_elems + head_elems + ((((base + 8 * g) & (page - 1)) >> 3) * D + col) * 8;
#pragma unroll
        for (int i = 0; i < DT; ++i) vf[i] = stream(v + 16 * i * 8);
    };

    int id0 = -1, id1 = -1;
    if (steps > 0) {
        find_pages(0, id0, id1);
        load_keys(0, id0, id1);
        load_values(0, id0, id1);
    }
    for (int step = 0; step < steps; ++step) {
        const int base = (b0 + wave + kWaves * step) * kBlock;
        const bool listed0 = id0 >= 0, listed1 = id1 >= 0;
        f32x4 sc[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
                sc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[tt][i]), qf[i], sc[tt], 0, 0, 0);
        if (step + 1 < steps) {                                        // the next keys as soon as these are used
            find_pages(step + 1, id0, id1);
            load_keys(step + 1, id0, id1);
        }
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = sc[j >> 2][j & 3] * d.scale_log2;
        const bool masked = base < t.full0 || base + kBlock > t.full1 || !listed0 || !listed1;
        if (masked) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int pos = base + 16 * (j >> 2) + 4 * g + (j & 3);
                const bool seen = pos <= here && pos > row_low && pos < t.pos1 && (j < 4 ? listed0 : listed1);
                x[j] = seen ? x[j] : kNegInf;
            }
        }
        float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m, top), m_use = m_new == kNegInf ? 0.0f : m_new;
        const float a = exp2_of(m - m_use);
        m = m_new;
        l *= a;
        // The weights cut to bf16, and what that leaves: of the same sign, and not 0 either where the weight is not, so that both products
        // of an infinite value are that infinity.
        uint32_t pw[4], rest[4];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const float p0 = exp2_of(x[j] - m_use), p1 = exp2_of(x[j + 1] - m_use);
            l += p0 + p1;
            const uint32_t w0 = __float_as_uint(p0) & 0xffff0000u, w1 = __float_as_uint(p1) & 0xffff0000u;
            pw[j / 2] = w0 >> 16 | w1;
            rest[j / 2] = pack_bf16(fmaxf(p0 - __uint_as_float(w0), p0 * 0x1p-24f), fmaxf(p1 - __uint_as_float(w1), p1 * 0x1p-24f));
        }
        // lanes 16 g have the weights of positions 4 g .. and 16 + 4 g ..; their values are those of 8 g ..
        const auto to_octets = [](uint32_t& p, uint32_t& q) {
            const auto u = __builtin_amdgcn_permlane32_swap(p, q, false, false);
            const auto w = __builtin_amdgcn_permlane16_swap(u[0], u[1], false, false);
            p = w[0];
            q = w[1];
        };
        to_octets(pw[0], pw[2]);
        to_octets(pw[1], pw[3]);
        to_octets(rest[0], rest[2]);
        to_octets(rest[1], rest[3]);
        const bf16x8 pf = __builtin_bit_cast(bf16x8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
        const bf16x8 rf = __builtin_bit_cast(bf16x8, make_uint4(rest[0], rest[1], rest[2], rest[3]));
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] *= a;
        if (masked) {
            // A weight of 0 leaves nothing of a finite value.  If there are others: those that no row sees count as 0, 0 * NaN would
            // spread.  So do those of the other positions, which some rows may see and others not; they are added behind the loop.
            u16x2 most = {0, 0};
#pragma unroll
            for (int i = 0; i < DT; ++i)
                most = larger(larger(larger(most, exponents(vf[i].x)), larger(exponents(vf[i].y), exponents(vf[i].z))), exponents(vf[i].w));
            if (__any(most[0] == 0x7f80 || most[1] == 0x7f80)) {
                uint32_t any = 0;                                      // of the lane's octet of values: seen by some row
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int at = base + 8 * g + j;
                    if ((g < 2 ? listed0 : listed1) && at >= t.pos0 && at < t.pos1) any |= 1u << j;
                }
                bool odd = false;
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    const uint4 v = make_uint4(vf[i].x & mask_of(any), vf[i].y & mask_of(any >> 2), vf[i].z & mask_of(any >> 4), vf[i].w & mask_of(any >> 6));
                    odd |= not_finite(v.x) || not_finite(v.y) || not_finite(v.z) || not_finite(v.w);
                    vf[i] = make_uint4(without_not_finite(v.x), without_not_finite(v.y), without_not_finite(v.z), without_not_finite(v.w));
                }
                if (__any(odd)) {
                    odd0 = min(odd0, base);
                    odd1 = base + kBlock;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[i]), rf, o[i], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[i]), pf, o[i], 0, 0, 0);
        if (step + 1 < steps) load_values(step + 1, id0, id1);
    }

    for (int pos = odd0; pos < min(odd1, t.pos1); ++pos) {
        const qblora_bf16* v = value_row<D>(d, table, kvh, pos);
        if (!v || !real || pos > here || pos <= row_low) continue;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] += if_not_finite(v[(16 * i + 4 * g + j) * 8]);
    }

    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) { sh.m[wave][col] = m; sh.l[wave][col] = l; }
    if (real)
#pragma unroll
        for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4*>(&sh.o[wave][col][16 * i + 4 * g]) = o[i];
    __syncthreads();
    float* part = u.splits > 1 ? share.part + ((int64_t)u.slot * d.kv_heads + kvh) * (kFewRows * (D + 2)) : nullptr;
    for (int i = tid; i < t.rows * (D / 4); i += kThreads) {
        const int r = i / (D / 4), f = 4 * (i % (D / 4));
        float top = kNegInf;
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sh.m[w][r]);
        const float use = top == kNegInf ? 0.0f : top;
        float sum = 0.0f;
        f32x4 v = {0, 0, 0, 0};
        for (int w = 0; w < kWaves; ++w) {
            const float a = exp2_of(sh.m[w][r] - use);
            sum = __fmaf_rn(sh.l[w][r], a, sum);
            const f32x4 x = *reinterpret_cast<const f32x4*>(&sh.o[w][r][f]);
            for (int j = 0; j < 4; ++j) v[j] = __fmaf_rn(x[j], a, v[j]);
        }
        if (part) {
            *reinterpret_cast<f32x4*>(part + r * D + f) = v;
            if (f == 0) { part[kFewRows * D + r] = top; part[kFewRows * (D + 1) + r] = sum; }
        } else {
            const int ahead = quotient(d, t.rem0 + r);
            const int64_t tok = s.start + t.token0 + ahead, h = kvh * d.group + t.rem0 + r - ahead * d.group;
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            *reinterpret_cast<uint2*>(d.out + tok * d.ldo + h * D + f) = make_uint2(pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv));
            if (f == 0 && d.lse) d.lse[tok * d.heads + h] = (top + __builtin_log2f(sum)) * 0.69314718055994530942f;
        }
    }
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
// 64 lanes x 16 bytes from uniform_base + lane_offset to lds_base + 16 * lane
__device__ __forceinline__ void copy_to_lds(const void* uniform_base, uint32_t lane_offset, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(lds_base), "v"(lane_offset), "s"(uniform_base) : "memory", "m0");
}
// until none of the wave's copies is on its way
__device__ __forceinline__ void wait_for_copies() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);                      // vmcnt alone, 0
    asm volatile("" ::: "memory");
}

// A barrier that leaves copies on their way: what the wave has read of LDS it has.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// of both halves of the wave
__device__ __forceinline__ float max_of_halves(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_of_halves(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int D>
struct ManyShared {
    // positions of a tile: 64, or 32 where the registers hold no more beside 256 features
    static constexpr int kTile = D > 128 ? 32 : 64, kTileBytes = kTile * D * 2;
    __attribute__((aligned(16))) unsigned char buf[2][2][kTileBytes];          // [keys, values][turn]
};

template <int D>
__device__ __forceinline__ void attend_many(const AttnDesc& d, const Share& share, int block, Finder& finder, ManyShared<D>& sh) {
    constexpr int kTile = ManyShared<D>::kTile, kTileBytes = ManyShared<D>::kTileBytes;
    constexpr int KS = D / 16, DT = D / 32, TT = kTile / 32;
    constexpr int PS = kTile / 16, kSixteen = D * 32;                  // a tile's sixteens of positions, bytes of one
    constexpr int kSharers = kWaves / PS, kCopies = kSixteen / 1024 / kSharers;     // waves that copy a sixteen, copies of each
    constexpr int kBatch = 64 / PS;                                    // tiles whose pages a wave looks up at once
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, col = lane & 31;
    const int kvh = block % d.kv_heads;
    Unit u;
    if (!find_unit(d, share, block / d.kv_heads, block == 0, finder, u)) return;
    const Span s = uniform_span_of(d, u.request);
    const int tiles = (int)(((int64_t)s.fresh * d.group + kManyRows - 1) / kManyRows);
    const Tile t = tile_of(d, s, tiles - 1 - u.tile, kManyRows);       // the longest ranges first
    note_cut(share, u, kvh, s, t);
    const int limit = d.width << d.page_shift;
    const int n_first = t.pos0 / kTile, n_last = (t.pos1 + kTile - 1) / kTile;
    const int per = (max(n_last - n_first, 0) + u.splits - 1) / u.splits;
    const int n0 = n_first + u.split * per, n1 = min(n0 + per, n_last);

    // the wave's rows, and what of the positions all of them see
    const int w_rows = min(32, t.rows - 32 * wave);
    const int among = t.rem0 + 32 * wave + col, ahead = quotient(d, among), token = t.token0 + ahead, head = kvh * d.group + among - ahead * d.group;
    const bool real = col < w_rows;
    const int here = s.context + token;
    const int first = s.context + t.token0 + quotient(d, t.rem0 + 32 * wave), last = s.context + t.token0 + quotient(d, t.rem0 + 32 * wave + max(w_rows, 1) - 1);
    const int full0 = d.window ? max(last + 1 - d.window, 0) : 0, full1 = w_rows > 0 ? min(first + 1, limit) : 0;
    const int see0 = d.window ? max(first + 1 - d.window, 0) : 0, see1 = w_rows > 0 ? min(last + 1, limit) : 0;

    // rows: operand B, row = lane & 31, features 16 i + 8 h ..; a negative scale is the rows' sign, one of 0 makes them 0
    const float c = d.scale_log2 == 0.0f ? 1.0f : fabsf(d.scale_log2);
    const uint32_t flip = d.scale_log2 < 0.0f ? 0x80008000u : 0u, keep_q = d.scale_log2 == 0.0f ? 0u : 0xffffffffu;
    bf16x8 qf[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (real) v = *reinterpret_cast<const uint4*>(d.q + (int64_t)(s.start + token) * d.ldq + (int64_t)head * D + 16 * i + 8 * h);
        v = make_uint4((v.x ^ flip) & keep_q, (v.y ^ flip) & keep_q, (v.z ^ flip) & keep_q, (v.w ^ flip) & keep_q);
        qf[i] = __builtin_bit_cast(bf16x8, v);
    }

    // Copies: every wave has a sixteen of a tile's positions, or half of its features, so that it needs one page.
    const int shift = d.page_shift, page = 1 << shift;
    const int64_t page_bytes = (int64_t)d.kv_heads * D * 2 << shift;
    const int mine = wave % PS, part = wave / PS;                      // the sixteen, the half
    const int32_t* table = d.table + (int64_t)u.request * d.width;
    const unsigned char* k_head = reinterpret_cast<const unsigned char*>(d.kc) + ((int64_t)kvh * D * 2 << shift) + ((part * kCopies * 4) << shift) * 16;
    const unsigned char* v_head = reinterpret_cast<const unsigned char*>(d.vc) + ((int64_t)kvh * D * 2 << shift) + part * kCopies * 1024;
    const uint32_t k_lane = (((lane >> 4) << shift) + (lane & 15)) * 16, v_lane = lane * 16;
    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(sh.buf)) + mine * kSixteen + part * kCopies * 1024;
    int batch = 0;
    uint64_t batch_listed = 0;
    // A tile's values are copied later than its keys: all waves' copies at once would hold them up.
    const unsigned char* v_late = nullptr;
    uint32_t to_late = 0;
    auto copy_values = [&] {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy_to_lds(v_late + i * 1024, v_lane, to_late + i * 1024);
    };
    // copies tile j's keys, and says which of its sixteens are listed; for j = 0, 1, ..
    auto copy = [&](int j) {
        const int tile = n0 + j;
        if (j % kBatch == 0) {
            const int pos = (tile + lane / PS) * kTile + 16 * (lane % PS);
            batch = -1;
            if (pos < min(t.pos1, n1 * kTile)) batch = table[pos >> shift];
            const bool ok = (uint32_t)batch < (uint32_t)d.pages;
            batch_listed = __ballot(ok);
            batch = ok ? batch : 0;
        }
        const int id = __builtin_amdgcn_readlane(batch, j % kBatch * PS + mine), in_page = (tile * kTile + 16 * mine) & (page - 1);
        const unsigned char* k = k_head + id * page_bytes + in_page * 16;
        const unsigned char* v = v_head + id * page_bytes + in_page * (D * 2);
        const uint32_t to = lds + (j & 1) * kTileBytes;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            copy_to_lds(k, k_lane, to + i * 1024);
            k += (4 << shift) * 16;
        }
        v_late = v;
        to_late = to + 2 * kTileBytes;
        return (uint32_t)(batch_listed >> (j % kBatch * PS)) & ((1u << PS) - 1);
    };

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int k = 0; k < 16; ++k) o[i][k] = 0.0f;
    // Exponents are c s - ref, ref near the maximum of c s; l: the sum over this lane's positions; bound: the product up to
    // which ref serves as it is (NaN: none).  Where c s is so large that a product's rounding counts, ref is 0 and the maximum
    // `m` is taken off the products first.
    const float none = __builtin_nanf("");
    float ref = kNegInf, m = kNegInf, l = 0.0f, bound = none;
    bool large = false;
    int odd0 = INT_MAX, odd1 = 0;                                      // positions among which values are not finite

    // position of row `col` of a 32 x 32 tile, so that a lane's scores are of eight consecutive positions twice
    const int perm = 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
    const unsigned char* const k_from = sh.buf[0][0] + (perm >> 4) * kSixteen + h * 256 + (perm & 15) * 16;
    const unsigned char* const v_from = sh.buf[1][0] + (h * D + col) * 16;
    auto key = [&](int j, int i, int tt) {
        return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(k_from + (j & 1) * kTileBytes + tt * 2 * kSixteen + i * 512));
    };
    auto value = [&](int j, int s4, int i) { return *reinterpret_cast<const uint4*>(v_from + (j & 1) * kTileBytes + s4 * kSixteen + i * 512); };
    auto products = [&](int j, f32x16 (&sc)[TT]) {
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int k = 0; k < 16; ++k) sc[tt][k] = 0.0f;
        // keys in flight: heads of 128 865 us with two (4096 tokens over 12288), 851 with six, 860 with twelve; of 64 better without
        constexpr int kAhead = 6;
        bf16x8 ahead[kAhead];
        if constexpr (D >= 128) {
#pragma unroll
            for (int n = 0; n < kAhead; ++n) ahead[n] = key(j, n / TT, n % TT);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int n = 0; n < KS * TT; ++n) {
            sc[n % TT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(D >= 128 ? ahead[n % kAhead] : key(j, n / TT, n % TT), qf[n / TT], sc[n % TT], 0, 0, 0);
            if constexpr (D >= 128) {
                if (n + kAhead < KS * TT) ahead[n % kAhead] = key(j, (n + kAhead) / TT, (n + kAhead) % TT);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    auto weights = [&](f32x16 (&sc)[TT], bf16x8 (&pf)[PS]) {
        float top = sc[0][0];
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int k = 0; k < 16; ++k) top = fmaxf(top, sc[tt][k]);
        if (__any(!(top <= bound))) {
            top = max_of_halves(top);
            const float m_new = fmaxf(m, top), m_use = m_new == kNegInf ? 0.0f : m_new;
            const float a = m == kNegInf ? 0.0f : exp2_of(large ? (m - m_use) * c : ref - m_use * c);
            large = large || __any(fabsf(m_use) * c > 0x1p26f);
            m = m_new;
            ref = large ? 0.0f : m_use * c;
            bound = large || m_new == kNegInf ? none : m_use + kSlack / c;
            l *= a;
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int k = 0; k < 16; ++k) o[i][k] *= a;
            if (large) {
#pragma unroll
                for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                    for (int k = 0; k < 16; ++k) sc[tt][k] -= m_use;
            }
        }
#pragma unroll
        for (int s4 = 0; s4 < PS; ++s4) {
            uint32_t pw[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float p0 = exp2_of(__fmaf_rn(sc[s4 >> 1][8 * (s4 & 1) + 2 * k], c, -ref));
                const float p1 = exp2_of(__fmaf_rn(sc[s4 >> 1][8 * (s4 & 1) + 2 * k + 1], c, -ref));
                l += p0 + p1;
                pw[k] = pack_bf16(p0, p1);
            }
            pf[s4] = __builtin_bit_cast(bf16x8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
        }
    };

    const int turns = n1 - n0;
    uint32_t listed = 0, next_listed = 0;
    if (turns > 0) {
        next_listed = copy(0);
        copy_values();
    }
    auto full = [&](int j) {                                           // seen by all rows of the wave
        const int base = (n0 + j) * kTile;
        return base >= full0 && base + kTile <= full1 && next_listed == (1u << PS) - 1;
    };
    auto enter = [&](int j) {                                          // tile j is there, and the next one is copied
        listed = next_listed;
        wait_for_copies();
        meet();
        if (j + 1 < turns) next_listed = copy(j + 1);
    };
    for (int j = 0; j < turns;) {
        // tiles that some row sees in part, or none
        for (; j < turns && !full(j); ++j) {
            enter(j);
            const int base = (n0 + j) * kTile;
            if (j + 1 < turns) copy_values();
            if (base >= see1 || base + kTile <= see0) continue;
            f32x16 sc[TT];
            products(j, sc);
            // of a sixteen's positions 8 h + k this lane's row sees from low to high - 1, and the wave's rows see some of those of
            // `some` (what they all see is no matter of a mask)
            uint32_t some = 0, all = 0;                                // bit s4
#pragma unroll
            for (int s4 = 0; s4 < PS; ++s4) {
                const int at = base + 16 * s4;
                const bool there = listed >> s4 & 1;
                if (there && at < see1 && at + 16 > see0) some |= 1u << s4;
                if (there && at >= full0 && at + 16 <= full1) all |= 1u << s4;
                const int high = there ? min(here + 1, limit) - at - 8 * h : 0, low = d.window ? here + 1 - d.window - at - 8 * h : 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int at8 = 8 * (s4 & 1) + k;
                    sc[s4 >> 1][at8] = k < high ? sc[s4 >> 1][at8] : kNegInf;
                }
                if (d.window)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int at8 = 8 * (s4 & 1) + k;
                        sc[s4 >> 1][at8] = k >= low ? sc[s4 >> 1][at8] : kNegInf;
                    }
            }
            bf16x8 pf[PS];
            weights(sc, pf);
            // As in attend_few: values that no row sees are 0, and what is not finite is added behind the loop.  Sixteens that no row
            // sees are left out; in the others all is finite most of the time, and a weight of 0 leaves nothing of it.
#pragma unroll
            for (int s4 = 0; s4 < PS; ++s4) {
                if (!(some >> s4 & 1)) continue;
                uint4 v[DT];
#pragma unroll
                for (int i = 0; i < DT; ++i) v[i] = value(j, s4, i);
                if (!(all >> s4 & 1)) {
                    u16x2 most = {0, 0};
#pragma unroll
                    for (int i = 0; i < DT; ++i)
                        most = larger(larger(larger(most, exponents(v[i].x)), larger(exponents(v[i].y), exponents(v[i].z))), exponents(v[i].w));
                    if (__any(most[0] == 0x7f80 || most[1] == 0x7f80)) {
                        uint32_t bits = 0;                             // of the lane's eight positions, those that some row sees
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int pos = base + 16 * s4 + 8 * h + k;
                            if (pos >= see0 && pos < see1) bits |= 1u << k;
                        }
                        const uint32_t k0 = mask_of(bits), k1 = mask_of(bits >> 2), k2 = mask_of(bits >> 4), k3 = mask_of(bits >> 6);
                        bool odd = false;
#pragma unroll
                        for (int i = 0; i < DT; ++i) {
                            v[i] = make_uint4(v[i].x & k0, v[i].y & k1, v[i].z & k2, v[i].w & k3);
                            odd |= not_finite(v[i].x) || not_finite(v[i].y) || not_finite(v[i].z) || not_finite(v[i].w);
                            v[i] = make_uint4(without_not_finite(v[i].x), without_not_finite(v[i].y), without_not_finite(v[i].z), without_not_finite(v[i].w));
                        }
                        if (__any(odd)) {
                            odd0 = min(odd0, base);
                            odd1 = base + kTile;
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < DT; ++i)
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[i]), pf[s4], o[i], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // The others, nearly all of a long context: a loop of its own, so that its registers are its own.  The compiler puts the
        // second product's instructions among the exponentials.  (Halves of the tile in turn, the weights of one between the products
        // of the other, an instruction of each at a time, with operands read a quarter ahead: 903 us where this took 886.)
        for (; j < turns && full(j); ++j) {
            enter(j);
            f32x16 sc[TT];
            products(j, sc);
            if (j + 1 < turns) copy_values();
            bf16x8 pf[PS];
            weights(sc, pf);
#pragma unroll
            for (int s4 = 0; s4 < PS; ++s4) {
#pragma unroll
                for (int i = 0; i < DT; ++i)
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, value(j, s4, i)), pf[s4], o[i], 0, 0, 0);
                if (D > 128) __builtin_amdgcn_sched_barrier(0);
            }
        }
    }

    // (the lane's row again: the loop has no registers to keep it in)
    const int h2 = (int)opaque_bits((uint32_t)h), r = 32 * wave + (int)opaque_bits((uint32_t)col);
    const int past = quotient(d, t.rem0 + r), to = t.token0 + past, q_head = kvh * d.group + t.rem0 + r - past * d.group;
    for (int pos = odd0; pos < min(odd1, see1); ++pos) {
        const qblora_bf16* v = value_row<D>(d, table, kvh, pos);
        if (!v || r >= t.rows || pos > s.context + to || (d.window && pos <= s.context + to - d.window)) continue;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int k = 0; k < 16; ++k) o[i][k] += if_not_finite(v[(32 * i + 8 * (k >> 2) + 4 * h2 + (k & 3)) * 8]);
    }
    l = sum_of_halves(l);
    const float top = m == kNegInf ? kNegInf : large ? m * c : ref;    // what the sums are relative to
    if (r >= t.rows) return;
    if (u.splits > 1) {
        float* part_of = share.part + ((int64_t)u.slot * d.kv_heads + kvh) * (kManyRows * (D + 2));
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                *reinterpret_cast<float4*>(part_of + r * D + 32 * i + 8 * b + 4 * h2) = make_float4(o[i][4 * b], o[i][4 * b + 1], o[i][4 * b + 2], o[i][4 * b + 3]);
        if (h2 == 0) { part_of[kManyRows * D + r] = top; part_of[kManyRows * (D + 1) + r] = l; }
        return;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    qblora_bf16* out = d.out + (int64_t)(s.start + to) * d.ldo + (int64_t)q_head * D;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            *reinterpret_cast<uint2*>(out + 32 * i + 8 * b + 4 * h2) =
                make_uint2(pack_bf16(o[i][4 * b] * inv, o[i][4 * b + 1] * inv), pack_bf16(o[i][4 * b + 2] * inv, o[i][4 * b + 3] * inv));
    if (h2 == 0 && d.lse) d.lse[(int64_t)(s.start + to) * d.heads + q_head] = (top + __builtin_log2f(l)) * 0.69314718055994530942f;
}

// One of the forms, or both (ALL), so that chunks and single tokens of a batch run beside each other.
template <int D, int FORMS>
__global__ __launch_bounds__(kThreads, (D > 128 ? 1 : 2)) void k_attn(AttnDesc d, Share lot, Share few, int lot_blocks) {
    __shared__ Finder finder;
    __shared__ union Shared {
        std::conditional_t<(FORMS & LOT) != 0, ManyShared<D>, char> many;
        std::conditional_t<(FORMS & FEW) != 0, FewShared<D>, char> few;
    } sh;
    if constexpr ((FORMS & LOT) != 0) {
        if (FORMS == LOT || (int)blockIdx.x < lot_blocks) return attend_many<D>(d, lot, blockIdx.x, finder, sh.many);
    }
    if constexpr ((FORMS & FEW) != 0) attend_few<D>(d, few, blockIdx.x - (FORMS & LOT ? lot_blocks : 0), finder, sh.few);
}

// Adds up the parts of a cut tile, weights 2^(m - max m), four features a thread.  Few parts: a thread has them all in flight,
// and the threads that are left over take other rows; many: they share the parts, of every gridDim.y-th row, the first of
// them in flight while the weights are made.  512 tokens over 2000, three parts a tile: 46 us the first way, 67 the second.
constexpr int kFewParts = 4, kPartsAhead = 4;
template <int D>
__global__ __launch_bounds__(kThreads) void k_attn_join(AttnDesc d, Share lot, Share few, int lot_blocks) {
    constexpr int kQuads = D / 4, kGroups = kThreads / kQuads;
    __shared__ float weight[kFewTarget + 1];
    __shared__ float top_of[4], sum_of[4];
    __shared__ f32x4 sums[kGroups][kQuads];
    const bool of_lot = (int)blockIdx.x < lot_blocks;
    const Share& share = of_lot ? lot : few;
    const int block = blockIdx.x - (of_lot ? 0 : lot_blocks), kvh = block % d.kv_heads, number = block / d.kv_heads;
    const int cuts = *share.cuts;                                      // (both loads in flight: the grid fits the list)
    const CutTile t = share.cut[number];
    if (number >= cuts) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, quad = tid % kQuads, grp = tid / kQuads;
    const int rows = share.rows, part_floats = rows * (D + 2);
    const int64_t step = (int64_t)part_floats * d.kv_heads;
    const float* part = share.part + ((int64_t)t.slot * d.kv_heads + kvh) * part_floats;
    const auto store = [&](int r, float top, float sum, const f32x4& v) {
        const int ahead = quotient(d, t.rem0 + r);
        const int64_t tok = t.token0 + ahead, h = kvh * d.group + t.rem0 + r - ahead * d.group;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        *reinterpret_cast<uint2*>(d.out + tok * d.ldo + h * D + 4 * quad) =
            make_uint2(pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv));
        if (quad == 0 && d.lse) d.lse[tok * d.heads + h] = (top + __builtin_log2f(sum)) * 0.69314718055994530942f;
    };
    if (t.splits <= kFewParts) {                                       // a row for each group of threads
        for (int r = blockIdx.y * kGroups + grp; r < t.rows; r += gridDim.y * kGroups) {
            float tops[kFewParts], sums_of[kFewParts], top = kNegInf, sum = 0.0f;
            f32x4 x[kFewParts], v = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < kFewParts; ++k) {
                const float* p = part + min(k, t.splits - 1) * step;
                tops[k] = p[rows * D + r];
                sums_of[k] = p[rows * (D + 1) + r];
                x[k] = *reinterpret_cast<const f32x4*>(p + r * D + 4 * quad);
                top = fmaxf(top, tops[k]);
            }
            const float use = top == kNegInf ? 0.0f : top;
#pragma unroll
            for (int k = 0; k < kFewParts; ++k) {
                if (k >= t.splits) break;
                const float a = exp2_of(tops[k] - use);
                sum = __fmaf_rn(sums_of[k], a, sum);
                for (int j = 0; j < 4; ++j) v[j] = __fmaf_rn(x[k][j], a, v[j]);
            }
            store(r, top, sum, v);
        }
        return;
    }
    for (int r = blockIdx.y; r < t.rows; r += gridDim.y) {
        f32x4 ahead[kPartsAhead];                                      // in flight while the weights are made
#pragma unroll
        for (int i = 0; i < kPartsAhead; ++i)
            ahead[i] = *reinterpret_cast<const f32x4*>(part + min(grp + i * kGroups, t.splits - 1) * step + r * D + 4 * quad);
        float top = kNegInf;
        for (int k = tid; k < t.splits; k += kThreads) {
            weight[k] = part[k * step + rows * D + r];
            top = fmaxf(top, weight[k]);
        }
        for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
        if (lane == 0) top_of[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(top_of[0], top_of[1]), fmaxf(top_of[2], top_of[3]));
        const float use = top == kNegInf ? 0.0f : top;
        float sum = 0.0f;
        for (int k = tid; k < t.splits; k += kThreads) {
            weight[k] = exp2_of(weight[k] - use);
            sum = __fmaf_rn(part[k * step + rows * (D + 1) + r], weight[k], sum);
        }
        for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
        if (lane == 0) sum_of[wave] = sum;
        __syncthreads();
        sum = (sum_of[0] + sum_of[1]) + (sum_of[2] + sum_of[3]);
        f32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kPartsAhead; ++i) {
            if (grp + i * kGroups >= t.splits) break;
            const float a = weight[grp + i * kGroups];
            for (int j = 0; j < 4; ++j) v[j] = __fmaf_rn(ahead[i][j], a, v[j]);
        }
#pragma unroll 4
        for (int k = grp + kPartsAhead * kGroups; k < t.splits; k += kGroups) {
            const float a = weight[k];
            const f32x4 x = *reinterpret_cast<const f32x4*>(part + k * step + r * D + 4 * quad);
            for (int j = 0; j < 4; ++j) v[j] = __fmaf_rn(x[j], a, v[j]);
        }
        sums[grp][quad] = v;
        __syncthreads();
        if (grp == 0) {
            for (int g = 1; g < kGroups; ++g) v += sums[g][quad];
            store(r, top, sum, v);
        }
        __syncthreads();
    }
}

// `target` counts workgroups over all key / value heads
int target_of(int target, int kv_heads) { return (target + kv_heads - 1) / kv_heads; }
// More rows than this in a request, if the caller knows of any, and they go through LDS.
bool many_rows(int group, int max_new) { return (int64_t)group * max_new > kFewRows; }

// The workspace: counts, the cut tiles of both forms, their parts (at most two for each unit of the target: what is cut is
// longer than a unit).
struct Space {
    size_t bytes = 0;
    char* base;
    explicit Space(void* p) : base(static_cast<char*>(p)) {}
    template <typename T>
    T* take(size_t count) {
        T* r = reinterpret_cast<T*>(base + bytes);
        bytes += (count * sizeof(T) + 255) / 256 * 256;
        return r;
    }
};
void lay_out(Space& space, int kv_heads, int head_dim, bool many, Share& lot, Share& few) {
    int* cuts = space.take<int>(64);
    few.cuts = cuts;
    lot.cuts = cuts + 1;
    few.cut = space.take<CutTile>(few.target);
    few.part = space.take<float>((size_t)2 * few.target * kv_heads * kFewRows * (head_dim + 2));
    if (!many) return;
    lot.cut = space.take<CutTile>(lot.target);
    lot.part = space.take<float>((size_t)2 * lot.target * kv_heads * kManyRows * (head_dim + 2));
}
Share few_share(int kv_heads, int head_dim, bool many) {
    return Share{kFewRows, target_of(head_dim > 128 ? kFewWideTarget : kFewTarget, kv_heads), kFewLeast, 0, many ? FEW : ALL, 0, nullptr, nullptr, nullptr};
}
Share lot_share(int kv_heads, int head_dim) {
    return Share{kManyRows, target_of(head_dim > 128 ? kManyWideTarget : kManyTarget, kv_heads), kManyLeast, 1, LOT, 0, nullptr, nullptr, nullptr};
}

template <int D>
int launch(const AttnDesc& d, hipStream_t st) {
    const bool many = many_rows(d.group, d.max_new);
    Share few = few_share(d.kv_heads, D, many), lot = lot_share(d.kv_heads, D);
    Space space(d.part);
    lay_out(space, d.kv_heads, D, many, lot, few);
    // rows of m requests make at most (rows + m (size - 1)) / size tiles
    const int64_t rows = (int64_t)d.T * d.group, requests = std::min<int64_t>(d.n, d.T);
    const auto tiles_of = [&](int size) { return (rows + requests * (size - 1)) / size; };
    const int64_t lot_tiles = many ? tiles_of(kManyRows) : 0;
    const int64_t few_tiles = many ? std::min(tiles_of(kFewRows), requests * (d.n > 64 ? 1 : kSomeRows / kFewRows)) : tiles_of(kFewRows);
    const int64_t blocks_of_row = (((int64_t)d.width << d.page_shift) + kBlock - 1) / kBlock + 1;
    const int64_t lot_units = many ? units_of_grid(lot_tiles, blocks_of_row, lot.target, lot.least) : 0;
    const int64_t few_units = units_of_grid(few_tiles, blocks_of_row, few.target, few.least);
    const int64_t lot_blocks = lot_units * d.kv_heads, blocks = lot_blocks + few_units * d.kv_heads;
    if (blocks * kThreads > UINT32_MAX) return QBLORA_ERR_UNSUPPORTED;     // (a longer grid would be cut without an error)
    lot.grid_units = (int)lot_units;
    few.grid_units = (int)few_units;
    const auto go = [&](auto kernel, int64_t count) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3(kThreads), 0, st, d, lot, few, (int)lot_blocks);
    };
    if (!many) {
        go(k_attn<D, FEW>, blocks);
    } else if constexpr (D <= 128) {
        go(k_attn<D, ALL>, blocks);
    } else {                                                           // (one kernel of both would not have the registers)
        go(k_attn<D, LOT>, lot_blocks);
        go(k_attn<D, FEW>, blocks - lot_blocks);
    }
    // no context is long enough for a cut
    if ((int64_t)d.width << d.page_shift <= kFewLeast * kBlock) return launch_status();
    const int64_t lot_cuts = (lot_tiles < lot.target ? lot_tiles : lot.target) * d.kv_heads;
    const int64_t few_cuts = (few_tiles < few.target ? few_tiles : few.target) * d.kv_heads;
    hipLaunchKernelGGL(k_attn_join<D>, dim3((unsigned)(lot_cuts + few_cuts), many || d.group > kFewRows ? kFewRows : d.group), dim3(kThreads), 0, st,
                       d, lot, few, (int)lot_cuts);
    return launch_status();
}

}  // namespace

size_t attention_part_bytes(int head_dim, int kv_heads, int group, int max_new) {
    const bool many = many_rows(group, max_new);
    Share few = few_share(kv_heads, head_dim, many), lot = lot_share(kv_heads, head_dim);
    Space space(nullptr);
    lay_out(space, kv_heads, head_dim, many, lot, few);
    return space.bytes;
}

int launch_attention(const AttnDesc& d, hipStream_t st) {
    switch (d.head_dim) {
        case 64: return launch<64>(d, st);
        case 128: return launch<128>(d, st);
        default: return launch<256>(d, st);
    }
}

}  // namespace qblora
