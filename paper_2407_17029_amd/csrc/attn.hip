// Attention of new tokens over the paged cache (qblora_paged_attention).
//
//   out = sum_j e_j v_j / sum_j e_j,  e_j = exp(scale q.k_j - m),  over the positions j a row sees, in one pass: m is the
//   maximum so far, and what was summed under a smaller one is multiplied by 2^(old - new) (the exponents are in base 2).
//
// A row is a query head of a new token; the rows of one request that share a key / value head go together, token by token
// (row r: token r / group, head r % group of the group), so that the cache is read once for all of them.
//
// k_attn_few takes 16 rows, the width of the matrix instruction, and is bound by the stream of the cache: a wave takes 32
// positions at a time straight from the pages into registers, in the operand order that the cache is stored in, with the
// next 32 in flight behind them.  Scores are formed transposed, S^T = K Q^T, so that a lane holds eight consecutive positions
// of one row: that is the operand of O^T = V^T P^T as it stands.  The four waves of a workgroup take turns on the positions
// and are joined in LDS.
//
// Work: requests differ by orders of magnitude, and only the device knows their lengths.  Every workgroup adds up the work
// of all requests, which gives the number of positions that a workgroup takes if there are to be `target` of them, and finds
// its own (request, 16 rows, range of positions) from the prefix sums.  A context that is cut this way leaves partial results
// in the workspace, which k_attn_join adds up.
#include "decoder.h"

namespace qblora {

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kFewRows = 16;
constexpr int kBlock = 32;                     // positions of a step
constexpr int kFewTarget = 1024;               // workgroups that share the work
constexpr int kFewMin = 8;                     // least blocks of a workgroup
constexpr float kNegInf = -__builtin_inff();

struct Unit { int request, tile, split, splits, slot; };

struct Span { int start, fresh, context; };
__device__ __forceinline__ Span span_of(const AttnDesc& d, int i) {
    const int s0 = min(max(d.starts[i], 0), d.T), s1 = min(max(d.starts[i + 1], s0), d.T);
    return {s0, s1 - s0, min(max(d.context[i], 0), 1 << 30)};
}

struct Cost { int tiles, blocks; };
__device__ __forceinline__ Cost cost_of(const AttnDesc& d, int i, int rows) {
    const Span s = span_of(d, i);
    if (s.fresh == 0) return {0, 0};
    const int limit = d.width << d.page_shift;
    const int hi = min(s.context + s.fresh, limit), lo = d.window ? max(s.context + 1 - d.window, 0) : 0;
    const int blocks = hi > lo ? (hi + kBlock - 1) / kBlock - lo / kBlock : 1;
    return {(int)(((int64_t)s.fresh * d.group + rows - 1) / rows), blocks};
}

// The work of workgroup unit `want` (units counted over requests, tiles and splits, or with `joins` over the tiles of split
// requests alone); false: there is none.  All threads call it.
struct Finder {
    int64_t sums[kWaves];
    int found[6];
};
__device__ __forceinline__ bool find_unit(const AttnDesc& d, int rows, int target, int least, bool joins, int64_t want,
                                          Finder& f, Unit& u) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int64_t all = 0;
    for (int i = tid; i < d.n; i += kThreads) {
        const Cost c = cost_of(d, i, rows);
        all += (int64_t)c.tiles * c.blocks;
    }
    for (int s = 32; s; s >>= 1) all += __shfl_xor(all, s);
    if (lane == 0) f.sums[wave] = all;
    if (tid == 0) f.found[0] = -1;
    __syncthreads();
    all = 0;
    for (int w = 0; w < kWaves; ++w) all += f.sums[w];
    const int64_t per = max((all + target - 1) / target, (int64_t)least);       // blocks of a workgroup
    int64_t units = 0, slots = 0;                                               // in front of this round's requests
    for (int base = 0; base < d.n; base += kThreads) {
        const int i = base + tid;
        int64_t mine = 0, cut = 0;
        int tiles = 0, splits = 1;
        if (i < d.n) {
            const Cost c = cost_of(d, i, rows);
            tiles = c.tiles;
            splits = (int)((c.blocks + per - 1) / per);
            cut = splits > 1 ? (int64_t)tiles * splits : 0;
            mine = joins ? (splits > 1 ? tiles : 0) : (int64_t)tiles * splits;
        }
        int64_t a = mine, b = cut;
        for (int s = 1; s < 64; s <<= 1) {
            const int64_t x = __shfl_up(a, s), y = __shfl_up(b, s);
            if (lane >= s) { a += x; b += y; }
        }
        __shared__ int64_t ends[2][kWaves];
        __syncthreads();
        if (lane == 63) { ends[0][wave] = a; ends[1][wave] = b; }
        __syncthreads();
        int64_t u0 = units, s0 = slots;
        for (int w = 0; w < kWaves; ++w) {
            if (w == wave) { a += u0; b += s0; }
            u0 += ends[0][w];
            s0 += ends[1][w];
        }
        units = u0;
        slots = s0;
        if (mine && a - mine <= want && want < a) {
            const int at = (int)(want - (a - mine));
            f.found[0] = i;
            f.found[1] = joins ? at : at / splits;
            f.found[2] = joins ? 0 : at % splits;
            f.found[3] = splits;
            f.found[4] = (int)(b - cut) + (joins ? at * splits : at);
        }
        __syncthreads();
        if (f.found[0] >= 0) break;
    }
    u.request = __builtin_amdgcn_readfirstlane(f.found[0]);
    if (u.request < 0) return false;
    u.tile = __builtin_amdgcn_readfirstlane(f.found[1]);
    u.split = __builtin_amdgcn_readfirstlane(f.found[2]);
    u.splits = __builtin_amdgcn_readfirstlane(f.found[3]);
    u.slot = __builtin_amdgcn_readfirstlane(f.found[4]);
    return true;
}

// the rows of a tile and the positions that any of them sees
struct Tile { int row0, rows, pos0, pos1, full0, full1; };       // full: positions that every row sees, as far as lengths go
__device__ __forceinline__ Tile tile_of(const AttnDesc& d, const Span& s, int tile, int rows) {
    Tile t;
    t.row0 = tile * rows;
    t.rows = min(rows, s.fresh * d.group - t.row0);
    const int first = s.context + t.row0 / d.group, last = s.context + (t.row0 + t.rows - 1) / d.group;
    const int limit = d.width << d.page_shift;
    t.pos1 = min(last + 1, limit);
    t.pos0 = d.window ? max(first + 1 - d.window, 0) : 0;
    t.full1 = min(first + 1, limit);
    t.full0 = d.window ? max(last + 1 - d.window, 0) : 0;
    return t;
}

__device__ __forceinline__ bool not_finite(uint32_t pair) { return (((pair & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0; }

// bf16 ones where an element of the pair is NaN (kind 0), +inf (1) or -inf (2)
__device__ __forceinline__ uint32_t indicator(uint32_t pair, int kind) {
    uint32_t out = 0;
    for (int h = 0; h < 2; ++h) {
        const uint32_t x = (pair >> (16 * h)) & 0xffffu;
        const bool is = kind == 0 ? (x & 0x7fffu) > 0x7f80u : x == (kind == 1 ? 0x7f80u : 0xff80u);
        if (is) out |= 0x3f80u << (16 * h);
    }
    return out;
}
__device__ __forceinline__ uint32_t without_not_finite(uint32_t pair) {
    const uint32_t bad = ((pair & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
    return pair & ~((bad >> 15) * 0xffffu);
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

template <int D>
struct FewShared {
    float o[kWaves][kFewRows][D + 4];
    float m[kWaves][kFewRows], l[kWaves][kFewRows];
};

template <int D>
__global__ __launch_bounds__(kThreads, D > 128 ? 1 : 2) void k_attn_few(AttnDesc d, int target) {
    constexpr int KS = D / 32, DT = D / 16;
    __shared__ Finder finder;
    __shared__ FewShared<D> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, col = lane & 15;
    const int kvh = blockIdx.x % d.kv_heads;
    Unit u;
    if (!find_unit(d, kFewRows, target, kFewMin, false, blockIdx.x / d.kv_heads, finder, u)) return;
    const Span s = span_of(d, u.request);
    const Tile t = tile_of(d, s, u.tile, kFewRows);
    const int b_first = t.pos0 / kBlock, b_last = (t.pos1 + kBlock - 1) / kBlock;
    const int per = (max(b_last - b_first, 0) + u.splits - 1) / u.splits;
    const int b0 = b_first + u.split * per, b1 = min(b0 + per, b_last);

    // rows: operand B, row = lane & 15, features 32 s + 8 g ..
    bf16x8 qf[KS];
    const int row = t.row0 + col;
    const int token = row / d.group, head = kvh * d.group + row % d.group;
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
            const int at = 8 * (col >> 2) + 4 * tt + (col & 3);        // position of row `col` of this 16 x 16 tile
            const int id = max(at < 16 ? id0 : id1, 0);
            const qblora_bf16* k = d.kc + id * page_elems + head_elems + ((g << shift) + ((base + at) & (page - 1))) * 8;
#pragma unroll
            for (int i = 0; i < KS; ++i) kf[tt][i] = *reinterpret_cast<const uint4*>(k + ((4 * i) << shift) * 8);
        }
    };
    auto load_values = [&](int step, int id0, int id1) {
        const int base = (b0 + wave + kWaves * step) * kBlock;
        const int id = max(g < 2 ? id0 : id1, 0);
        const qblora_bf16* v = d.vc + id * page_elems + head_elems + ((((base + 8 * g) & (page - 1)) >> 3) * D + col) * 8;
#pragma unroll
        for (int i = 0; i < DT; ++i) vf[i] = *reinterpret_cast<const uint4*>(v + 16 * i * 8);
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
        uint32_t seen = 0xff;                                          // by this lane's row, of its eight positions
        uint32_t any = 0xff;                                           // by some row
        if (masked) {
            seen = any = 0;
            const bool listed = g < 2 ? listed0 : listed1;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int pos = base + 8 * g + j;
                if (listed && pos >= t.pos0 && pos < t.pos1) any |= 1u << j;
                if (pos <= here && pos > row_low) seen |= 1u << j;
            }
            seen &= any;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (seen >> j) & 1 ? x[j] : kNegInf;
        }
        float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m, top), m_use = m_new == kNegInf ? 0.0f : m_new;
        const float a = exp2_of(m - m_use);
        m = m_new;
        l *= a;
        uint32_t pw[4];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const float p0 = exp2_of(x[j] - m_use), p1 = exp2_of(x[j + 1] - m_use);
            l += p0 + p1;
            pw[j / 2] = pack_bf16(p0, p1);
        }
        const bf16x8 pf = __builtin_bit_cast(bf16x8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] *= a;
        if (masked) {
            // Values that no row sees count as 0 whatever they are: 0 * NaN would spread.  Those that some rows see and
            // others do not are 0 as well where they are not finite, and come in through products of indicators.
            uint32_t keep[4], vis[4];
            bool odd = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                keep[j] = ((any >> (2 * j)) & 1 ? 0xffffu : 0u) | ((any >> (2 * j + 1)) & 1 ? 0xffff0000u : 0u);
                vis[j] = ((seen >> (2 * j)) & 1 ? 0x3f80u : 0u) | ((seen >> (2 * j + 1)) & 1 ? 0x3f800000u : 0u);
            }
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                vf[i] = make_uint4(vf[i].x & keep[0], vf[i].y & keep[1], vf[i].z & keep[2], vf[i].w & keep[3]);
                odd |= not_finite(vf[i].x) || not_finite(vf[i].y) || not_finite(vf[i].z) || not_finite(vf[i].w);
            }
            if (__any(odd)) {
                const bf16x8 seen_ones = __builtin_bit_cast(bf16x8, make_uint4(vis[0], vis[1], vis[2], vis[3]));
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    const uint4 v = vf[i];
#pragma unroll
                    for (int kind = 0; kind < 3; ++kind) {
                        const uint4 is = make_uint4(indicator(v.x, kind), indicator(v.y, kind), indicator(v.z, kind), indicator(v.w, kind));
                        const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, is), seen_ones, f32x4{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (n[j] > 0.0f) o[i][j] += kind == 0 ? __builtin_nanf("") : kind == 1 ? -kNegInf : kNegInf;
                    }
                    vf[i] = make_uint4(without_not_finite(v.x), without_not_finite(v.y), without_not_finite(v.z), without_not_finite(v.w));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[i]), pf, o[i], 0, 0, 0);
        if (step + 1 < steps) load_values(step + 1, id0, id1);
    }

    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) { sh.m[wave][col] = m; sh.l[wave][col] = l; }
    if (real)
#pragma unroll
        for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4*>(&sh.o[wave][col][16 * i + 4 * g]) = o[i];
    __syncthreads();
    float* part = u.splits > 1 ? d.part + ((int64_t)u.slot * d.kv_heads + kvh) * (kFewRows * (D + 2)) : nullptr;
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
            for (int j = 0; j < 4; ++j) v[j] += sh.m[w][r] == kNegInf ? 0.0f : x[j] * a;
        }
        if (part) {
            *reinterpret_cast<f32x4*>(part + r * D + f) = v;
            if (f == 0) { part[kFewRows * D + r] = top; part[kFewRows * (D + 1) + r] = sum; }
        } else {
            const int64_t tok = s.start + (t.row0 + r) / d.group, h = kvh * d.group + (t.row0 + r) % d.group;
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            *reinterpret_cast<uint2*>(d.out + tok * d.ldo + h * D + f) = make_uint2(pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv));
            if (f == 0 && d.lse) d.lse[tok * d.heads + h] = (top + __builtin_log2f(sum)) * 0.69314718055994530942f;
        }
    }
}

// Adds up the partial results of a split tile: weights 2^(m - max m).
template <int D, int ROWS>
__global__ __launch_bounds__(kThreads) void k_attn_join(AttnDesc d, int target, int least) {
    __shared__ Finder finder;
    const int kvh = blockIdx.x % d.kv_heads;
    Unit u;
    if (!find_unit(d, ROWS, target, least, true, blockIdx.x / d.kv_heads, finder, u)) return;
    const Span s = span_of(d, u.request);
    const Tile t = tile_of(d, s, u.tile, ROWS);
    constexpr int64_t kPart = ROWS * (D + 2);
    const int64_t step = kPart * d.kv_heads;
    const float* part = d.part + ((int64_t)u.slot * d.kv_heads + kvh) * kPart;
    for (int i = threadIdx.x; i < t.rows * D; i += kThreads) {
        const int r = i / D, f = i % D;
        float top = kNegInf;
        for (int k = 0; k < u.splits; ++k) top = fmaxf(top, part[k * step + ROWS * D + r]);
        const float use = top == kNegInf ? 0.0f : top;
        float sum = 0.0f, v = 0.0f;
        for (int k = 0; k < u.splits; ++k) {
            const float mk = part[k * step + ROWS * D + r], a = exp2_of(mk - use);
            sum = __fmaf_rn(part[k * step + ROWS * (D + 1) + r], a, sum);
            if (mk != kNegInf) v = __fmaf_rn(part[k * step + i], a, v);
        }
        const int64_t tok = s.start + (t.row0 + r) / d.group, h = kvh * d.group + (t.row0 + r) % d.group;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        d.out[tok * d.ldo + h * D + f] = (qblora_bf16)pack_bf16(v * inv, 0.0f);
        if (f == 0 && d.lse) d.lse[tok * d.heads + h] = (top + __builtin_log2f(sum)) * 0.69314718055994530942f;
    }
}

// units over all key / value heads
int target_of(int kv_heads) { return (kFewTarget + kv_heads - 1) / kv_heads; }

template <int D>
int launch_few(const AttnDesc& d, hipStream_t st) {
    const int target = target_of(d.kv_heads);
    const int64_t tiles = (int64_t)d.T * d.group / kFewRows + d.n, grid = (tiles + target) * d.kv_heads;
    if (grid > INT32_MAX) return QBLORA_ERR_UNSUPPORTED;
    hipLaunchKernelGGL(k_attn_few<D>, dim3((unsigned)grid), dim3(kThreads), 0, st, d, target);
    const int64_t joins = (tiles < target ? tiles : target) * d.kv_heads;
    hipLaunchKernelGGL((k_attn_join<D, kFewRows>), dim3((unsigned)joins), dim3(kThreads), 0, st, d, target, kFewMin);
    return launch_status();
}

}  // namespace

size_t attention_part_bytes(int head_dim, int kv_heads, int group, int max_new) {
    (void)group; (void)max_new;
    return (size_t)2 * target_of(kv_heads) * kv_heads * kFewRows * (head_dim + 2) * sizeof(float);
}

int launch_attention(const AttnDesc& d, hipStream_t st) {
    switch (d.head_dim) {
        case 64: return launch_few<64>(d, st);
        case 128: return launch_few<128>(d, st);
        default: return launch_few<256>(d, st);
    }
}

}  // namespace qblora
