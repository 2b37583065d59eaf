// Rotary positions (qblora_rope_fwd / _bwd) and their serving form, which writes k and v to the paged cache
// (qblora_rope_cache).
//
//   pair (a, b) of a head at position p:  a' = scale (a cos x - b sin x),  b' = scale (b cos x + a sin x),  x = p * freq
//
// Bound by HBM, each element read and written once, or by the launch with few tokens.  k_rope: a thread keeps the sines and
// cosines of its 16 features (eight pairs) in registers and takes one head after another, four in flight, 16 bytes an
// access.  Tokens of a prompt that go to the cache come eight to a workgroup, neighbouring lanes one behind the other, so that
// eight keys' 16-byte octets are one 128-byte line of their page and eight values of a feature one 16-byte store; single
// tokens come one to a workgroup, which is four times as many of them.  k_rope_any: parts of a head that are no multiple of
// 16 features, a turn for every pair of every head (4096 tokens of 32 + 32 heads of 80, there and back: 105 us with 20 features
// turned, 33 by k_rope with all 80).  6693 tokens of 64 + 64 heads of 128 to the cache (658 MB): 130 us, 5.1 TB/s, where a large copy reaches 4.9; 1337 of 40 + 40 heads there and back (110 MB): 21.1 us, 5.2 TB/s; 64 single tokens of 32 + 32: 7 us, of which 3.5 are
// an empty launch.
#include <algorithm>

#include "decoder.h"

namespace qblora {

namespace {

constexpr int kThreads = 256;
// From here on, tokens that go to the cache are taken for prompts.  A chunk of 300: 10.3 us that way, 11.2 a token at a time, of
// 512: 10.4 and 19.9; but 256 single tokens (which no argument tells from a chunk) 12.4 and 10.7, 512 of them 25.6 and 23.7.
constexpr int kManyTokens = 256;

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

constexpr int kHeads = 4;                      // in flight
// From so many bytes of q and k on, nothing of the outputs is in an L2 when they are read: 1337 tokens of 40 + 40 heads (27 MB)
// both ways 23.7 us through the caches, 21.0 past them; 6693 tokens of 64 + 64 heads to the cache 155 and 147 (130 by now).
constexpr int64_t kPastBytes = 8 << 20;

template <bool PAST>
__device__ __forceinline__ void put(qblora_bf16* p, bf16x8_any v) {
    if (PAST) __builtin_nontemporal_store(v, reinterpret_cast<bf16x8_any*>(p));
    else *reinterpret_cast<bf16x8_any*>(p) = v;
}

// Whether a token begins a run: its slot does not follow that of the token before, or begins an octet.
__device__ __forceinline__ bool begins(const RopeDesc& d, int64_t t) {
    if (t == 0 || t >= d.T) return true;
    const int64_t slot = d.slots[t];
    return (slot & 7) == 0 || d.slots[t - 1] != slot - 1;
}
// The runs that begin among the eight tokens from t0 on: what a workgroup owns, so that an octet of a page has one writer.
// They end within seven more tokens.
__device__ __forceinline__ void owned_tokens(const RopeDesc& d, int64_t t0, int64_t& from, int64_t& to) {
    const int lane = threadIdx.x & 63;
    const uint32_t at = (uint32_t)__ballot(lane < 16 && begins(d, t0 + lane));
    from = t0 + (at & 0xff ? __builtin_ctz(at) : 8);
    to = t0 + 8 + (at >> 8 ? __builtin_ctz(at >> 8) : 8);
    if (to > d.T) to = d.T;
    if (!(at & 0xff)) from = to;
}

struct RopeGrid { int qk_blocks, v_blocks; };  // of blockIdx.y

template <int TB, bool PAIRS, bool PAST>                                // PAST: stores go past the caches
__global__ __launch_bounds__(kThreads) void k_rope(RopeDesc d, RopeGrid grid) {
    const int tid = threadIdx.x;
    const int64_t t0 = (int64_t)blockIdx.x * TB;
    if ((int)blockIdx.y < grid.qk_blocks) {
        // A thread's unit is two chunks of eight features, neighbouring lanes' chunks side by side: with half pairs chunk u of
        // the first and of the second members (or two of the chunks behind them), else chunks u and u + units.
        const int units = d.head_dim >> 4, chunks = d.rot >> 3, turning = d.rot >> 4, lanes = kThreads / (TB * units);
        const int tb = tid % TB, u = tid / TB % units, hl = tid / (TB * units);
        const int c0 = PAIRS || u < turning ? u : turning + u, c1 = PAIRS ? u + units : u < turning ? u + turning : u + units;
        const bool turns0 = c0 < chunks, turns1 = c1 < chunks;         // (half pairs: both or none)
        int64_t from = t0, to = t0 + TB < d.T ? t0 + TB : d.T;
        if (TB > 1) owned_tokens(d, t0, from, to);
        if (hl >= lanes) return;
        for (int64_t t = from + tb; t < to; t += TB) {
            const int all = d.heads + d.kv_heads;
            bf16x8_any x[kHeads][2];
            auto load = [&](int h0) {
#pragma unroll
                for (int i = 0; i < kHeads; ++i) {
                    const int h = h0 + i * lanes;
                    if (h >= all) continue;
                    const qblora_bf16* in = h < d.heads ? d.q + t * d.ldq + h * d.head_dim : d.k + t * d.ldk + (h - d.heads) * d.head_dim;
                    x[i][0] = *reinterpret_cast<const bf16x8_any*>(in + 8 * c0);
                    x[i][1] = *reinterpret_cast<const bf16x8_any*>(in + 8 * c1);
                }
            };
            const int begin = hl + (int)blockIdx.y * lanes * kHeads, step = grid.qk_blocks * lanes * kHeads;
            const int64_t slot = d.kc ? d.slots[t] : -1;
            // The first heads are on their way while the turns are made: 2000 tokens of 64 + 8 heads to the cache 17.3 us without, 16.0
            // with (512 single tokens, which pay for the registers: 22.1 and 25.6).  Not where many small workgroups do that for each
            // other: 8001 of 32 + 8 both ways 61 us without, 65 with.
            if (TB > 1) load(begin);
            float cs[8], sn[8];
            if (turns0) {
                const int32_t p = d.positions[t];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int pair = !PAIRS ? 8 * u + j : j < 4 ? 4 * c0 + j : 4 * c1 + j - 4;
                    if (PAIRS && j >= 4 && !turns1) break;
                    turn(p, d.freq[pair], d.scale, cs[j], sn[j]);
                    sn[j] *= d.sign;
                }
            }
            for (int h0 = begin; h0 < all; h0 += step) {
                if (TB == 1 || h0 != begin) load(h0);
#pragma unroll
                for (int i = 0; i < kHeads; ++i) {
                    const int h = h0 + i * lanes;
                    if (h >= all) continue;
                    bf16x8_any y[2] = {x[i][0], x[i][1]};
                    if (turns0) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (PAIRS) {                                   // a dword is a pair
#pragma unroll
                                for (int c = 0; c < 2; ++c) {
                                    if (c == 1 && !turns1) break;
                                    const float a = bf16_lo(x[i][c][j]), b = bf16_hi(x[i][c][j]);
                                    y[c][j] = pack_bf16(__fmaf_rn(a, cs[4 * c + j], -(b * sn[4 * c + j])), __fmaf_rn(b, cs[4 * c + j], a * sn[4 * c + j]));
                                }
                            } else {                                       // the two chunks are eight pairs
                                const float a0 = bf16_lo(x[i][0][j]), a1 = bf16_hi(x[i][0][j]), b0 = bf16_lo(x[i][1][j]), b1 = bf16_hi(x[i][1][j]);
                                const float k0 = cs[2 * j], k1 = cs[2 * j + 1], s0 = sn[2 * j], s1 = sn[2 * j + 1];
                                y[0][j] = pack_bf16(__fmaf_rn(a0, k0, -(b0 * s0)), __fmaf_rn(a1, k1, -(b1 * s1)));
                                y[1][j] = pack_bf16(__fmaf_rn(b0, k0, a0 * s0), __fmaf_rn(b1, k1, a1 * s1));
                            }
                        }
                    }
                    qblora_bf16 *o0, *o1;
                    if (h >= d.heads && d.kc) {
                        if (!in_cache(d, slot)) continue;
                        int place;
                        qblora_bf16* out = d.kc + page_of(d, slot, h - d.heads, place);
                        o0 = out + key_at(d, place, 8 * c0);
                        o1 = out + key_at(d, place, 8 * c1);
                    } else {
                        qblora_bf16* out = h < d.heads ? d.q_out + t * d.ldq_out + h * d.head_dim : d.k_out + t * d.ldk_out + (h - d.heads) * d.head_dim;
                        o0 = out + 8 * c0;
                        o1 = out + 8 * c1;
                    }
                    put<PAST>(o0, y[0]);
                    put<PAST>(o1, y[1]);
                }
            }
        }
        return;
    }

    // Values: four features a thread, and the run of tokens whose slots follow each other up to the end of an octet.  A whole
    // octet goes through LDS, so that a store is 64 features side by side rather than every fourth.
    __shared__ uint4 turned[kThreads / 64][TB > 1 ? 256 : 1];
    const int first = ((int)blockIdx.y - grid.qk_blocks) * kThreads + tid, step = grid.v_blocks * kThreads;
    const int quads = d.kv_heads * d.head_dim / 4;
    const int lane = tid & 63;
    int64_t slots = -1;                                                // of token t0 + lane
    uint32_t begin = 0x1ffff;                                          // which tokens begin a run; one ends within seven more
    if (TB > 1) {
        const int64_t t = t0 + lane;
        int64_t before = -1;
        if (lane < 16 && t < d.T) slots = d.slots[t];
        if (lane < 16 && t < d.T && t > 0) before = d.slots[t - 1];
        begin = (uint32_t)__ballot(lane >= 16 || t >= d.T || t == 0 || (slots & 7) == 0 || before != slots - 1) & 0x1ffff;
    }
    if (TB > 1 && (begin & 0x1ff) == 0x1ff) {
        // no slot follows another (single tokens): the eight tokens' values in flight together
        const uint32_t cached = (uint32_t)__ballot(lane < 8 && t0 + lane < d.T && in_cache(d, slots));
        for (int i = first; i - lane < quads; i += step) {
            const int h = 4 * i / d.head_dim, f = 4 * i - h * d.head_dim;
            bf16x4_any x[8];
#pragma unroll
            for (int b = 0; b < 8; ++b)
                if (i < quads && (cached >> b & 1)) x[b] = *reinterpret_cast<const bf16x4_any*>(d.v + (t0 + b) * d.ldv + 4 * i);
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                const int64_t slot = __shfl(slots, b);
                if (i >= quads || !(cached >> b & 1)) continue;
                int place;
                qblora_bf16* out = d.vc + page_of(d, slot, h, place);
                out += value_at(d, place, f);
#pragma unroll
                for (int j = 0; j < 4; ++j) out[8 * j] = (qblora_bf16)(j & 1 ? x[b][j >> 1] >> 16 : x[b][j >> 1]);
            }
        }
        return;
    }
    for (int b = 0; b < TB && t0 + b < d.T; ++b) {
        if (!(begin >> b & 1)) continue;                               // in another token's run
        const int64_t t = t0 + b, slot = TB > 1 ? __shfl(slots, b) : d.slots[t];
        if (!in_cache(d, slot)) continue;
        const int run = TB > 1 ? __builtin_ctz(begin >> (b + 1)) + 1 : 1;
        int place;
        (void)page_of(d, slot, 0, place);
        if (TB > 1 && run == 8) {
            uint4* mine = turned[tid >> 6];
            for (int i = first; i - lane < quads; i += step) {
                if (i < quads) {
                    const qblora_bf16* in = d.v + t * d.ldv + 4 * i;
                    bf16x4_any x[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = *reinterpret_cast<const bf16x4_any*>(in + k * d.ldv);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t y[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t lo = x[2 * k][j >> 1], hi = x[2 * k + 1][j >> 1];
                            y[k] = j & 1 ? (lo >> 16) | (hi & 0xffff0000u) : (lo & 0xffffu) | (hi << 16);
                        }
                        // feature 4 lane + j, its low bits turned by the lane: 16 lanes to every bank
                        mine[(4 * lane + j) ^ ((lane >> 1) & 3)] = make_uint4(y[0], y[1], y[2], y[3]);
                    }
                }
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int at = 64 * j + lane, f = 4 * (i - lane) + at;               // feature of all heads'
                    if (f < 4 * quads) {
                        const int h = f / d.head_dim;
                        int same;
                        qblora_bf16* out = d.vc + page_of(d, slot, h, same) + value_at(d, place, f - h * d.head_dim);
                        const uint4 y = mine[at ^ ((at >> 3) & 3)];
                        bf16x8_any o = {y.x, y.y, y.z, y.w};
                        put<PAST>(out, o);
                    }
                }
                __builtin_amdgcn_wave_barrier();
            }
            continue;
        }
        for (int i = first; i < quads; i += step) {
            const int h = 4 * i / d.head_dim, f = 4 * i - h * d.head_dim;
            int same;
            qblora_bf16* out = d.vc + page_of(d, slot, h, same) + value_at(d, place, f);
            const qblora_bf16* in = d.v + t * d.ldv + 4 * i;
            for (int k = 0; k < run; ++k) {
                const bf16x4_any x = *reinterpret_cast<const bf16x4_any*>(in + k * d.ldv);
#pragma unroll
                for (int j = 0; j < 4; ++j) out[8 * j + k] = (qblora_bf16)(j & 1 ? x[j >> 1] >> 16 : x[j >> 1]);
            }
        }
    }
}

// Launches for all tokens, as many at a time as a grid takes with `tb` of them a workgroup: go(those tokens, workgroups).  A run of
// slots that two launches share is written by one after the other.
template <typename Go>
void for_tokens(const RopeDesc& d, int tb, const Go& go) {
    const int64_t most = kMostThreads / kThreads * tb;
    for (int64_t t = 0; t < d.T; t += most) {
        RopeDesc e = d;
        e.T = std::min(most, d.T - t);
        e.q += t * d.ldq;
        e.q_out += t * d.ldq_out;
        e.positions += t;
        if (d.k) e.k += t * d.ldk;
        if (d.k_out) e.k_out += t * d.ldk_out;
        if (d.v) e.v += t * d.ldv;
        if (d.slots) e.slots += t;
        go(e, (unsigned)((e.T + tb - 1) / tb));
    }
}

}  // namespace

int launch_rope(const RopeDesc& d, hipStream_t st) {
    const int units = d.head_dim / 16, all = d.heads + d.kv_heads;
    const dim3 threads(kThreads);
    if (d.head_dim % 16 != 0 || d.rot % 16 != 0 || units > kThreads / 8) {
        for_tokens(d, 1, [&](const RopeDesc& e, unsigned blocks) { hipLaunchKernelGGL(k_rope_any, dim3(blocks), threads, 0, st, e); });
        return launch_status();
    }
    const bool prompts = d.kc && d.T >= kManyTokens;
    const int tb = prompts ? 8 : 1, lanes = kThreads / (tb * units);
    // workgroups of a token (or eight): one pass over the heads each
    const int groups = (all + lanes * kHeads - 1) / (lanes * kHeads);
    RopeGrid g{groups, 0};
    const bool past = d.T * all * d.head_dim * 2 >= kPastBytes;
    if (d.vc) g.v_blocks = (d.kv_heads * d.head_dim / 4 + kThreads - 1) / kThreads;
    const auto go = [&](auto kernel) {
        for_tokens(d, tb, [&](const RopeDesc& e, unsigned blocks) {
            hipLaunchKernelGGL(kernel, dim3(blocks, g.qk_blocks + g.v_blocks), threads, 0, st, e, g);
        });
    };
    if (tb == 8) {
        if (d.interleaved) go(past ? k_rope<8, true, true> : k_rope<8, true, false>);
        else go(past ? k_rope<8, false, true> : k_rope<8, false, false>);
    } else {
        if (d.interleaved) go(past ? k_rope<1, true, true> : k_rope<1, true, false>);
        else go(past ? k_rope<1, false, true> : k_rope<1, false, false>);
    }
    return launch_status();
}

}  // namespace qblora
