// C-ABI entry points of the operators on many adapters and of the optimizer's step (include/qblora.h): host-side validation and
// descriptions.
#include <algorithm>
#include <cmath>

#include "adapters.h"

using namespace qblora;

namespace {

bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
bool lambda_ok(int l) { return l == 1 || l == 2 || l == 4 || l == 8; }
size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }

int check_adapters(const qblora_adapters* a) {
    if (!a) return QBLORA_ERR_NULL;
    if (a->count <= 0 || a->d_in <= 0 || a->d_out <= 0 || a->lambda1 <= 0 || a->lambda2 <= 0 || a->R <= 0) return QBLORA_ERR_SHAPE;
    if (a->d_in % 64 || a->d_out % 64 || a->R % 8) return QBLORA_ERR_SHAPE;
    if (!lambda_ok(a->lambda1) || !lambda_ok(a->lambda2) || a->R > kMostInnerRank || a->count > kMostAdapters || a->d_in > (1 << 20) ||
        a->d_out > (1 << 20))
        return QBLORA_ERR_UNSUPPORTED;
    if (!a->table) return QBLORA_ERR_NULL;
    if (!aligned(a->table, 16)) return QBLORA_ERR_SHAPE;
    return QBLORA_OK;
}
int check_batch(const int32_t* first, const int32_t* order, const int32_t* tiles, int64_t T) {
    if (T < 0) return QBLORA_ERR_SHAPE;
    if (T > kMostGroupTokens) return QBLORA_ERR_UNSUPPORTED;
    if (!first || (T && (!order || !tiles))) return QBLORA_ERR_NULL;
    if (T && !aligned(tiles, 16)) return QBLORA_ERR_SHAPE;
    return QBLORA_OK;
}
int check_rows(const void* p, int64_t ld, int width) {
    if (!p) return QBLORA_ERR_NULL;
    if (ld < width || ld % 8 || !aligned(p, 16)) return QBLORA_ERR_SHAPE;
    return QBLORA_OK;
}
// Runs of at most 64 tokens that a batch may have: any of the adapters may have tokens, which of them do is known on the device only
int tile_room(int count, int64_t T) { return (int)((T + kTileTokens - 1) / kTileTokens + std::min<int64_t>(count, T)); }

Grouped grouped(const qblora_adapters* a, const int32_t* first, const int32_t* order, const int32_t* tiles, int64_t T) {
    Grouped g{};
    g.table = reinterpret_cast<const AdapterEntry*>(a->table); g.count = a->count;
    g.first = first; g.order = order; g.tiles = tiles; g.tile_room = tile_room(a->count, T); g.T = (int)T; g.R = a->R;
    return g;
}

// The workspace, in this order: partial sums of the rank sums on X and on dY, the bf16 parts of s U and dU, partial gradients.  No
// size shrinks as T grows, so that one for the largest batch serves every smaller one.
struct Space { size_t part_x, part_y, su, du, grads, all; };
Space space_of(const qblora_adapters* a, int64_t T) {
    Space s{};
    s.part_x = up256((size_t)rank_part_rows(T, a->d_in) * a->R * 4);
    s.part_y = up256((size_t)rank_part_rows(T, a->d_out) * a->R * 4);
    s.su = s.du = up256((size_t)T * a->R * 6);
    const int splits = adapter_grad_splits(a->count, T, a->d_in, a->d_out, a->R);
    if (splits > 1)
        s.grads = up256((size_t)splits * a->count * ((size_t)a->d_in / a->lambda1 + a->d_out / a->lambda2) * a->R * 4);
    s.all = s.part_x + s.part_y + s.su + s.du + s.grads;
    return s;
}

int check_list(const qblora_adamw_list* l) {
    if (!l) return QBLORA_ERR_NULL;
    if (l->count < 0 || l->units < 0) return QBLORA_ERR_SHAPE;
    if (l->bits != 8 && l->bits != 32) return QBLORA_ERR_UNSUPPORTED;
    if (l->count && !l->plan) return QBLORA_ERR_NULL;
    if (!aligned(l->plan, 16)) return QBLORA_ERR_SHAPE;
    return QBLORA_OK;
}
const PlanEntry* entries_of(const qblora_adamw_list* l) { return reinterpret_cast<const PlanEntry*>(l->plan); }
const PlanUnit* units_of(const qblora_adamw_list* l) { return reinterpret_cast<const PlanUnit*>(entries_of(l) + l->count); }

constexpr int64_t kMostUnits = (int64_t)1 << 26;            // 2^30 blocks of 256

// units of a list, -1 if there are too many or a size is negative
int64_t count_units(const qblora_adamw_tensor* tensors, int32_t count) {
    int64_t units = 0;
    for (int i = 0; i < count; ++i) {
        const int64_t n = tensors[i].n;
        if (n < 0 || n > kMostUnits * kUnit) return -1;
        units += (n + kUnit - 1) / kUnit;
        if (units >= kMostUnits) return -1;
    }
    return units;
}

}  // namespace

extern "C" {

size_t qblora_adapter_table_bytes(int32_t count) { return count > 0 ? (size_t)count * sizeof(AdapterEntry) : 0; }

int qblora_adapter_table(const qblora_adapters* adapters, int32_t first, int32_t n, const qblora_adapter* list,
                         float* const* dA, float* const* dB, void* stream) {
    const int rc = check_adapters(adapters);
    if (rc) return rc;
    if (first < 0 || n < 0 || (int64_t)first + n > adapters->count) return QBLORA_ERR_SHAPE;
    if (n == 0) return QBLORA_OK;
    if (!list || (dA == nullptr) != (dB == nullptr)) return QBLORA_ERR_NULL;
    for (int i = 0; i < n; ++i) {
        const qblora_adapter& a = list[i];
        if (dA && ((dA[i] == nullptr) != (dB[i] == nullptr))) return QBLORA_ERR_NULL;
        if (!a.A || !a.B || a.R == 0) continue;
        if (a.lambda1 != adapters->lambda1 || a.lambda2 != adapters->lambda2 || a.R < 0 || a.R > adapters->R || a.R % 8) return QBLORA_ERR_SHAPE;
        if (a.scale_op != QBLORA_OP_AVGPOOL_REPEAT) return QBLORA_ERR_UNSUPPORTED;
        if (!aligned(a.A, 16) || !aligned(a.B, 16) || (dA && (!aligned(dA[i], 16) || !aligned(dB[i], 16)))) return QBLORA_ERR_SHAPE;
    }
    for (int at = 0; at < n; at += kTableChunk) {
        TableDesc d{};
        d.n = std::min(kTableChunk, n - at);
        d.out = reinterpret_cast<AdapterEntry*>(adapters->table) + first + at;
        for (int i = 0; i < d.n; ++i) {
            const qblora_adapter& a = list[at + i];
            if (!a.A || !a.B || a.R == 0) continue;
            d.entry[i] = {a.A, a.B, dA ? dA[at + i] : nullptr, dB ? dB[at + i] : nullptr, a.R, a.s, 0};
        }
        const int rc = launch_adapter_table(d, as_stream(stream));
        if (rc) return rc;
    }
    return QBLORA_OK;
}

int32_t qblora_adapter_tiles(int32_t count, int64_t T) {
    return count > 0 && T > 0 && T <= kMostGroupTokens ? tile_room(count, T) : 0;
}

int qblora_adapter_groups(const int32_t* starts, const int32_t* which, int32_t n, int32_t count, int64_t T, int32_t* first,
                          int32_t* order, int32_t* tiles, void* stream) {
    if (n < 0 || count <= 0 || T < 0) return QBLORA_ERR_SHAPE;
    if (n > kMostGroupRequests || count > kMostAdapters || T > kMostGroupTokens) return QBLORA_ERR_UNSUPPORTED;
    if (!starts || (n && !which) || !first || (T && (!order || !tiles))) return QBLORA_ERR_NULL;
    if (T && !aligned(tiles, 16)) return QBLORA_ERR_SHAPE;
    GroupsDesc d{};
    d.starts = starts; d.which = which; d.n = n; d.count = count; d.T = (int)T;
    d.first = first; d.order = order; d.tiles = tiles; d.tile_room = T ? tile_room(count, T) : 0;
    return launch_adapter_groups(d, as_stream(stream));
}

size_t qblora_adapters_saved_bytes(const qblora_adapters* a, int64_t T) {
    return check_adapters(a) || T < 0 || T > kMostGroupTokens ? 0 : (size_t)T * a->R * 6;
}

size_t qblora_adapters_workspace_bytes(const qblora_adapters* a, int64_t T) {
    return check_adapters(a) || T <= 0 || T > kMostGroupTokens ? 0 : space_of(a, T).all;
}

int qblora_adapters_fwd(const qblora_adapters* a, const int32_t* first, const int32_t* order, const int32_t* tiles,
                        const qblora_bf16* X, int64_t ldx, int64_t T, qblora_bf16* Y, int64_t ldy, qblora_bf16* saved,
                        void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_adapters(a);
    if (rc) return rc;
    rc = check_batch(first, order, tiles, T);
    if (rc || T == 0) return rc;
    if ((rc = check_rows(X, ldx, a->d_in))) return rc;
    if ((rc = check_rows(Y, ldy, a->d_out))) return rc;
    if (!aligned(saved, 16) || X == Y) return QBLORA_ERR_SHAPE;
    const Space s = space_of(a, T);
    if (!workspace || workspace_bytes < s.all || !aligned(workspace, 256)) return QBLORA_ERR_WORKSPACE;
    RankDesc u{};
    u.g = grouped(a, first, order, tiles, T);
    u.Z = X; u.ldz = ldx; u.width = a->d_in; u.lam = a->lambda1; u.back = 0; u.factor = 1.0f / a->lambda1;
    u.part = reinterpret_cast<float*>(workspace); u.splits = rank_splits(u.g.tile_room, a->d_in, a->R);
    if ((rc = launch_rank_sums(u, as_stream(stream)))) return rc;
    SpreadDesc v{};
    v.g = u.g; v.part = u.part; v.splits = u.splits;
    if (saved || rank_parts_pay(a->count, T, a->R)) {
        PartsDesc w{};
        w.g = u.g; w.part = u.part; w.splits = u.splits;
        w.out = saved ? saved : reinterpret_cast<qblora_bf16*>(reinterpret_cast<unsigned char*>(workspace) + s.part_x + s.part_y);
        if ((rc = launch_rank_parts(w, as_stream(stream)))) return rc;
        v.u = w.out;
    }
    v.out = Y; v.ldo = ldy; v.width = a->d_out; v.lam = a->lambda2; v.back = 0; v.factor = 1.0f;
    return launch_spread(v, as_stream(stream));
}

int qblora_adapters_bwd(const qblora_adapters* a, const int32_t* first, const int32_t* order, const int32_t* tiles,
                        const qblora_bf16* X, int64_t ldx, const qblora_bf16* dY, int64_t lddy, int64_t T,
                        const qblora_bf16* saved, qblora_bf16* dX, int64_t lddx, int32_t gradients, void* workspace,
                        size_t workspace_bytes, void* stream) {
    int rc = check_adapters(a);
    if (rc) return rc;
    rc = check_batch(first, order, tiles, T);
    if (rc) return rc;
    if (!dX && !gradients) return QBLORA_ERR_NULL;
    hipStream_t st = as_stream(stream);
    AdapterGradDesc w{};
    w.g = grouped(a, first, order, tiles, T);
    w.d_in = a->d_in; w.lam1 = a->lambda1; w.d_out = a->d_out; w.lam2 = a->lambda2; w.splits = 1;
    if (T == 0) return gradients ? launch_adapter_grads(w, st) : QBLORA_OK;
    if (gradients && (rc = check_rows(X, ldx, a->d_in))) return rc;
    if ((rc = check_rows(dY, lddy, a->d_out))) return rc;
    if (dX && (rc = check_rows(dX, lddx, a->d_in))) return rc;
    if (!aligned(saved, 16) || dX == dY || (gradients && dX == X)) return QBLORA_ERR_SHAPE;
    const Space s = space_of(a, T);
    if (!workspace || workspace_bytes < s.all || !aligned(workspace, 256)) return QBLORA_ERR_WORKSPACE;
    unsigned char* at = reinterpret_cast<unsigned char*>(workspace);
    float* part_x = reinterpret_cast<float*>(at);
    float* part_y = reinterpret_cast<float*>(at + s.part_x);
    qblora_bf16* su = reinterpret_cast<qblora_bf16*>(at + s.part_x + s.part_y);
    qblora_bf16* du = reinterpret_cast<qblora_bf16*>(at + s.part_x + s.part_y + s.su);
    const bool again = gradients && !saved;                     // s U has to be computed once more
    RankDesc u{};
    u.g = w.g;
    if (again) {
        u.Z = X; u.ldz = ldx; u.width = a->d_in; u.lam = a->lambda1; u.back = 0; u.factor = 1.0f / a->lambda1;
        u.part = part_x; u.splits = rank_splits(u.g.tile_room, a->d_in, a->R);
        if ((rc = launch_rank_sums(u, st))) return rc;
    }
    PartsDesc p{};
    p.g = w.g;
    if (again) { p.part2 = part_x; p.splits2 = u.splits; p.out2 = su; }
    u.Z = dY; u.ldz = lddy; u.width = a->d_out; u.lam = a->lambda2; u.back = 1; u.factor = 1.0f;
    u.part = part_y; u.splits = rank_splits(u.g.tile_room, a->d_out, a->R);
    if ((rc = launch_rank_sums(u, st))) return rc;
    SpreadDesc v{};
    v.g = w.g; v.part = part_y; v.splits = u.splits;
    if (gradients || rank_parts_pay(a->count, T, a->R)) {
        p.part = part_y; p.splits = u.splits; p.out = du;
        if ((rc = launch_rank_parts(p, st))) return rc;
        v.u = du;
    }
    if (dX) {
        v.out = dX; v.ldo = lddx; v.width = a->d_in; v.lam = a->lambda1; v.back = 1; v.factor = 1.0f / a->lambda1;
        if ((rc = launch_spread(v, st))) return rc;
    }
    if (!gradients) return QBLORA_OK;
    w.X = X; w.ldx = ldx; w.dY = dY; w.lddy = lddy; w.su = saved ? saved : su; w.du = du;
    w.part = reinterpret_cast<float*>(at + s.part_x + s.part_y + s.su + s.du);
    w.splits = adapter_grad_splits(a->count, T, a->d_in, a->d_out, a->R);
    return launch_adapter_grads(w, st);
}

size_t qblora_adamw_plan_bytes(const qblora_adamw_tensor* tensors, int32_t count) {
    if (count <= 0 || !tensors) return 0;
    const int64_t units = count_units(tensors, count);
    return units < 0 ? 0 : (size_t)count * sizeof(PlanEntry) + (size_t)units * sizeof(PlanUnit);
}

int qblora_adamw_plan(const qblora_adamw_tensor* tensors, int32_t count, int32_t bits, void* plan, size_t plan_bytes,
                      qblora_adamw_list* list, void* stream) {
    if (count < 0) return QBLORA_ERR_SHAPE;
    if (bits != 8 && bits != 32) return QBLORA_ERR_UNSUPPORTED;
    if (!list || (count && (!tensors || !plan))) return QBLORA_ERR_NULL;
    if (!aligned(plan, 16)) return QBLORA_ERR_SHAPE;
    const int64_t units = count_units(tensors, count);
    if (units < 0) return QBLORA_ERR_SHAPE;
    for (int i = 0; i < count; ++i) {
        const qblora_adamw_tensor& t = tensors[i];
        if (!std::isfinite(t.rate) || !std::isfinite(t.decay)) return QBLORA_ERR_SHAPE;
        if (t.n == 0) continue;
        if ((!t.param && !t.master) || !t.grad || !t.m || !t.v || (bits == 8 && (!t.m_scale || !t.v_scale))) return QBLORA_ERR_NULL;
        if (!aligned(t.param, 2) || !aligned(t.master, 4) || !aligned(t.grad, 4) || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4) ||
            (bits == 32 && (!aligned(t.m, 4) || !aligned(t.v, 4))))
            return QBLORA_ERR_SHAPE;
    }
    if (plan_bytes < (size_t)count * sizeof(PlanEntry) + (size_t)units * sizeof(PlanUnit)) return QBLORA_ERR_WORKSPACE;
    *list = {count, bits, units, plan};
    int64_t unit = 0;
    for (int at = 0; at < count; at += kPlanChunk) {
        PlanDesc d{};
        d.n = std::min(kPlanChunk, count - at);
        d.first = at;
        d.out = reinterpret_cast<PlanEntry*>(plan) + at;
        const int64_t begin = unit;
        d.units = reinterpret_cast<PlanUnit*>(reinterpret_cast<PlanEntry*>(plan) + count) + begin;
        for (int i = 0; i < d.n; ++i) {
            const qblora_adamw_tensor& t = tensors[at + i];
            d.entry[i] = {t.n, t.param, t.master, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.rate, t.decay, unit - begin};
            unit += (t.n + kUnit - 1) / kUnit;
        }
        const int rc = launch_adamw_plan(d, unit - begin, as_stream(stream));
        if (rc) return rc;
    }
    return QBLORA_OK;
}

size_t qblora_grad_norm_workspace_bytes(const qblora_adamw_list* list) {
    return check_list(list) ? 0 : (size_t)std::max<int64_t>(1, std::min<int64_t>(list->units, kNormParts)) * sizeof(double);
}

int qblora_grad_norm(const qblora_adamw_list* list, double max_norm, float* out, void* workspace, size_t workspace_bytes,
                     void* stream) {
    const int rc = check_list(list);
    if (rc) return rc;
    if (!out) return QBLORA_ERR_NULL;
    if (!(max_norm > 0.0)) return QBLORA_ERR_SHAPE;
    if (!workspace || workspace_bytes < qblora_grad_norm_workspace_bytes(list) || !aligned(workspace, 16)) return QBLORA_ERR_WORKSPACE;
    return launch_grad_norm(entries_of(list), units_of(list), list->units, max_norm, reinterpret_cast<double*>(workspace), out,
                            as_stream(stream));
}

int qblora_adamw_step(const qblora_adamw_list* list, const qblora_adamw* how, const float* clip, void* stream) {
    const int rc = check_list(list);
    if (rc) return rc;
    if (!how) return QBLORA_ERR_NULL;
    if (!(how->beta1 >= 0.0 && how->beta1 < 1.0) || !(how->beta2 >= 0.0 && how->beta2 < 1.0) || !(how->eps > 0.0) ||
        !std::isfinite(how->eps) || (!how->device_lr && !std::isfinite(how->lr)) || (!how->device_step && how->step < 1))
        return QBLORA_ERR_SHAPE;
    if ((float)how->beta1 == 1.0f || (float)how->beta2 == 1.0f || (float)how->eps < 1e-15f) return QBLORA_ERR_SHAPE;
    if (list->units == 0) return QBLORA_OK;
    StepDesc d{};
    d.entries = entries_of(list); d.units = units_of(list); d.n_units = list->units; d.bits = list->bits;
    d.lr = how->lr; d.beta1d = how->beta1; d.beta2d = how->beta2;
    d.beta1 = (float)how->beta1; d.one_beta1 = (float)(1.0 - how->beta1);
    d.beta2 = (float)how->beta2; d.one_beta2 = (float)(1.0 - how->beta2); d.eps = (float)how->eps;
    d.step = how->step; d.device_step = how->device_step; d.device_lr = how->device_lr; d.clip = clip;
    d.seed_key = how->seed * 0x85157AF5u;
    if (!how->device_step) {
        d.key = d.seed_key + (uint32_t)how->step * 0xD168AAADu;
        d.lr_c1 = how->lr / (1.0 - std::pow(how->beta1, (double)how->step));
        d.inv_sqrt_c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(how->beta2, (double)how->step)));
    }
    return launch_adamw(d, as_stream(stream));
}

}  // extern "C"
