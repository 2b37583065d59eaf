// Block tables, slots and positions of a step, from the lengths of its requests (qblora_page_tables), in one launch.
//
//   first new token of request i:  start_i = sum_{j < i} fresh_j           page taken first:  first_i = sum_{j < i} more_j
//   more_i = max(0, min(ceil((context_i + fresh_i) / page), width) - ceil(context_i / page))
//   token t of request i:  p = context_i + t - start_i,  slot = id * page + p % page with the id of page p / page: the table's
//   where the request held it before, else free_pages[first_i + p / page - held]
//
// Bound by latency: 64 single tokens move 1.5 KB, 1000 requests with 50000 tokens 0.6 MB.  So there is one launch and no
// scratch: every workgroup forms the prefix sums of all requests in its own LDS (two values a request, read from L2) and then
// serves a share of the tokens and of the new pages, which find their request by bisection there.  Nothing waits for another
// workgroup, and no thread reads a table entry that the call writes.  With more than kGroups requests LDS holds the sums of
// groups of them, and the last steps of the search walk through a group's lengths.  64 single tokens: 3.7 us; 1000 requests with
// 50000 tokens: 7.6; an empty launch takes 3.5.
#include "decoder.h"

namespace qblora {

namespace {

constexpr int kThreads = 256;
constexpr int kGroups = 2048;

struct Request { uint32_t held, more, fresh; };

__device__ __forceinline__ Request request(const TablesDesc& d, int i) {
    const uint32_t c = (uint32_t)max(d.context[i], 0), m = (uint32_t)max(d.fresh[i], 0);
    const uint32_t mask = (1u << d.page_shift) - 1, total = c + m;       // at most 2^32 - 2
    const uint32_t held = (c >> d.page_shift) + ((c & mask) != 0);
    const uint32_t want = min((total >> d.page_shift) + ((total & mask) != 0), (uint32_t)d.width);
    return {held, want > held ? want - held : 0u, m};
}

// of two sums that are at most 2^31 - 1; more is as good as that
__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }

// the last of `groups` entries that is at most x (entry 0 is 0)
__device__ __forceinline__ int last_at_most(const uint32_t* v, int groups, uint32_t x) {
    int lo = 0, hi = groups;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (v[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(kThreads) void k_page_tables(TablesDesc d, int group) {
    __shared__ uint32_t tokens_at[kGroups], pages_at[kGroups];
    __shared__ uint32_t wave_tokens[kThreads / 64], wave_pages[kThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int groups = (d.n + group - 1) / group;
    const int per = (groups + kThreads - 1) / kThreads;                  // groups of a thread, one after another
    const int g0 = min(tid * per, groups), g1 = min(g0 + per, groups);

    uint32_t tokens = 0, pages = 0;
    for (int i = g0 * group; i < min(g1 * group, d.n); ++i) {
        const Request r = request(d, i);
        tokens = add(tokens, r.fresh);
        pages = add(pages, r.more);
    }
    uint32_t t_sum = tokens, p_sum = pages;
    for (int s = 1; s < 64; s <<= 1) {
        const uint32_t a = __shfl_up(t_sum, s), b = __shfl_up(p_sum, s);
        if (lane >= s) { t_sum = add(t_sum, a); p_sum = add(p_sum, b); }
    }
    if (lane == 63) { wave_tokens[wave] = t_sum; wave_pages[wave] = p_sum; }
    uint32_t t_at = __shfl_up(t_sum, 1), p_at = __shfl_up(p_sum, 1);
    if (lane == 0) t_at = p_at = 0;
    __syncthreads();
    uint32_t t_all = 0, p_all = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w == wave) { t_at = add(t_at, t_all); p_at = add(p_at, p_all); }
        t_all = add(t_all, wave_tokens[w]);
        p_all = add(p_all, wave_pages[w]);
    }
    const bool first_block = blockIdx.x == 0;
    for (int g = g0; g < g1; ++g) {
        tokens_at[g] = t_at;
        pages_at[g] = p_at;
        for (int i = g * group; i < min((g + 1) * group, d.n); ++i) {
            const Request r = request(d, i);
            if (first_block) d.starts[i] = (int32_t)min(t_at, (uint32_t)d.tokens);
            t_at = add(t_at, r.fresh);
            p_at = add(p_at, r.more);
        }
    }
    const uint32_t real = min(t_all, (uint32_t)d.tokens);
    if (first_block && tid == 0) {
        d.starts[d.n] = (int32_t)real;
        d.taken[0] = (int32_t)p_all;
    }
    __syncthreads();

    const int stride = gridDim.x * kThreads;
    for (int64_t x = (int64_t)blockIdx.x * kThreads + tid; x < p_all; x += stride) {      // the x-th page taken
        const int g = last_at_most(pages_at, groups, (uint32_t)x);
        uint32_t first = pages_at[g];
        int i = g * group;
        Request r = request(d, i);
        while (first + r.more <= x) {
            first += r.more;
            r = request(d, ++i);
        }
        d.table[(int64_t)i * d.width + r.held + ((uint32_t)x - first)] = x < d.n_free ? d.free_pages[x] : -1;
    }
    for (int64_t t = (int64_t)blockIdx.x * kThreads + tid; t < d.tokens; t += stride) {
        int32_t p = 0;
        int64_t slot = -1;
        if (t < real) {
            const int g = last_at_most(tokens_at, groups, (uint32_t)t);
            uint32_t start = tokens_at[g], first = pages_at[g];
            int i = g * group;
            Request r = request(d, i);
            while (start + r.fresh <= t) {
                start += r.fresh;
                first = add(first, r.more);
                r = request(d, ++i);
            }
            const uint32_t at = (uint32_t)max(d.context[i], 0) + ((uint32_t)t - start);
            const uint32_t page = at >> d.page_shift;
            p = (int32_t)min(at, 0x7fffffffu);
            if (page < (uint32_t)d.width) {
                int32_t id = -1;
                if (page < r.held) {
                    id = d.table[(int64_t)i * d.width + page];
                } else {
                    const uint32_t x = add(first, page - r.held);
                    if (x < (uint32_t)d.n_free) id = d.free_pages[x];
                }
                if (id >= 0) slot = ((int64_t)id << d.page_shift) + (at & ((1u << d.page_shift) - 1));
            }
        }
        d.positions[t] = p;
        d.slots[t] = slot;
    }
}

}  // namespace

int launch_page_tables(const TablesDesc& d, hipStream_t st) {
    const int group = d.n > kGroups ? (d.n + kGroups - 1) / kGroups : 1;
    const int64_t items = (int64_t)d.tokens + d.n;
    const int blocks = (int)(items < 512 ? 1 : items > 512 * 512 ? 512 : items / 512);
    hipLaunchKernelGGL(k_page_tables, dim3(blocks), dim3(kThreads), 0, st, d, group);
    return launch_status();
}

}  // namespace qblora
