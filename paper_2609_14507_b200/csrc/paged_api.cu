// C entry points of the paged cache: what they refuse, and how a call becomes launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/ipkv.h"
#include "kernels.h"
#include "paged.h"
#include "plan.hpp"

using namespace ipkvi;

namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bool shape_ok(const ipkv_attn_shape* sh) {
    return sh && sh->kind == IPKV_GQA && sh->n_q_heads > 0 && sh->n_kv_heads > 0 && sh->n_kv_heads <= (1 << 16) && sh->n_q_heads <= (1 << 20) &&
           sh->n_q_heads % sh->n_kv_heads == 0 && sh->dim_qk == sh->dim_v && (sh->dim_qk == 64 || sh->dim_qk == 128) && sh->block_tokens > 0 &&
           sh->block_tokens <= (1 << 20) && (sh->block_tokens == 16 || sh->block_tokens == 32 || sh->block_tokens % kTileTokens == 0);
}
bool capacity_ok(const ipkv_attn_shape* sh, int32_t n_rows, int32_t max_blocks) {
    return n_rows >= 0 && max_blocks >= 1 && int64_t(max_blocks) * sh->block_tokens <= kPagedMostSlots;
}
BlockGeom geom(const ipkv_attn_shape* sh) { return BlockGeom{sh->n_kv_heads, sh->dim_qk, sh->dim_v, sh->block_tokens}; }
bool cache_ok(const ipkv_attn_shape* sh, const ipkv_paged* c) {
    if (!shape_ok(sh) || !c || !capacity_ok(sh, c->n_rows, c->max_blocks)) return false;
    if (!c->pool_dev || !aligned(c->pool_dev, 16) || c->pool_bytes < geom(sh).block_bytes() || c->pool_bytes / geom(sh).block_bytes() > INT32_MAX) return false;
    if (!aligned(c->table_dev, 4) || !aligned(c->lengths_dev, 4) || (c->n_rows > 0 && (!c->table_dev || !c->lengths_dev))) return false;
    if (c->table_stride < c->max_blocks || c->table_stride > (int64_t(1) << 40)) return false;
    if (c->weights_dev || c->positions_dev) {
        if (!aligned(c->weights_dev, 16) || !aligned(c->positions_dev, 16)) return false;
        if (c->slot_stride < int64_t(c->max_blocks) * sh->block_tokens || c->slot_stride % 4 != 0 || c->slot_stride > (int64_t(1) << 32)) return false;
    }
    return true;
}
PagedCache cache_of(const ipkv_attn_shape* sh, const ipkv_paged* c) {
    PagedCache p;
    p.g = geom(sh);
    p.pool = static_cast<char*>(c->pool_dev); p.n_blocks = c->pool_bytes / p.g.block_bytes();
    p.table = c->table_dev; p.lengths = c->lengths_dev; p.table_stride = c->table_stride; p.slot_stride = c->slot_stride;
    p.weights = c->weights_dev; p.positions = c->positions_dev;
    p.n_rows = c->n_rows; p.max_blocks = c->max_blocks;
    return p;
}
// The cache of rows r0 .. r0 + n - 1.
void rows_from(PagedCache& p, const PagedCache& all, int32_t r0, int32_t n) {
    const int64_t slots = int64_t(r0) * all.g.n_kv_heads * all.slot_stride;
    p.table = all.table + r0 * all.table_stride; p.lengths = all.lengths + r0;
    p.weights = all.weights ? all.weights + slots : nullptr; p.positions = all.positions ? all.positions + slots : nullptr;
    p.n_rows = n;
}
// Whether an output array shaped like the cache's is the input itself or apart from it.
bool apart(const ipkv_attn_shape* sh, const ipkv_paged* c, const void* in, const void* out) {
    if (!in || in == out) return true;
    const uintptr_t bytes = uintptr_t(c->n_rows) * sh->n_kv_heads * c->slot_stride * 4, a = reinterpret_cast<uintptr_t>(in), b = reinterpret_cast<uintptr_t>(out);
    return a + bytes <= b || b + bytes <= a;
}

// Head groups of a row, rows of one launch and its scratch.
struct AttendPlan {
    int group, groups_per_kv, n_gh, rows_per_part, sixteens;
    int32_t unit;
    int64_t most_units;
    int32_t rows;                                // rows of a launch at most: shares held in shared memory, costs in 32 bits
    size_t header, partials, head_ml, scores;
    AttendPlan(const ipkv_attn_shape* sh, int32_t n_rows, int32_t max_blocks, int32_t window, int32_t first, bool weigh)
        : group(sh->n_q_heads / sh->n_kv_heads), groups_per_kv(paged_groups_per_kv(group)), n_gh(sh->n_kv_heads * groups_per_kv),
          rows_per_part(paged_rows_per_part(group)), sixteens(paged_sixteens(group)),
          unit(paged_unit(sh->dim_qk)),
          most_units(paged_most_units(int64_t(max_blocks) * sh->block_tokens, window, first, unit)) {
        const int64_t fit = int64_t(INT32_MAX) / (n_gh * (most_units + kPagedPairCost));
        const int64_t grid = int64_t(INT32_MAX) / 2 / sh->n_q_heads;      // the join's
        rows = int32_t(std::min<int64_t>(std::min<int64_t>(n_rows, kPagedRowsPerLaunch), std::min(fit, grid)));
        header = align_up(sizeof(PagedHeader), 256);
        const size_t parts = size_t(2) * kSmCount * kPagedCtasPerSm * rows_per_part;
        partials = align_up(parts * sh->dim_qk * sizeof(float), 256) + align_up(parts * sizeof(float2), 256);
        head_ml = weigh ? align_up(size_t(rows) * sh->n_q_heads * sizeof(float2), 256) : 0;
        scores = weigh ? size_t(rows) * n_gh * size_t(most_units) * unit * rows_per_part * sizeof(float) : 0;
    }
    size_t scratch() const { return header + partials + head_ml + scores; }
};

bool window_ok(int32_t window, int32_t first) { return window >= 0 && first >= 0; }

}  // namespace

extern "C" {

ipkv_status ipkv_paged_append(const ipkv_paged_append_call* call) {
    if (!call) return IPKV_EINVAL;
    const auto [sh, c, n_tokens, k_dev, v_dev, k_token_stride, v_token_stride, row_start_dev, token_positions_dev, status_dev, stream] = *call;
    if (!cache_ok(sh, c) || n_tokens < 0 || n_tokens > INT32_MAX) return IPKV_EINVAL;
    const int64_t row = int64_t(sh->n_kv_heads) * sh->dim_qk;
    for (int64_t stride : {k_token_stride, v_token_stride})
        if (stride != 0 && (stride < row || stride % 8 != 0 || stride > (int64_t(1) << 40))) return IPKV_EINVAL;
    if (!aligned(k_dev, 16) || !aligned(v_dev, 16) || !aligned(row_start_dev, 4) || !aligned(token_positions_dev, 4) || !aligned(status_dev, 4)) return IPKV_EINVAL;
    if (!row_start_dev && n_tokens != c->n_rows) return IPKV_EINVAL;
    if (n_tokens == 0 || c->n_rows == 0) return IPKV_OK;
    if (!k_dev || !v_dev || (c->positions_dev && !token_positions_dev)) return IPKV_EINVAL;
    PagedAppend a;
    a.c = cache_of(sh, c);
    a.k = static_cast<const char*>(k_dev); a.v = static_cast<const char*>(v_dev);
    a.k_token = 2 * (k_token_stride ? k_token_stride : row); a.v_token = 2 * (v_token_stride ? v_token_stride : row);
    a.n_tokens = n_tokens; a.row_start = row_start_dev; a.token_positions = token_positions_dev; a.status = status_dev;
    return launch_paged_append(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? IPKV_OK : IPKV_ECUDA;
}

ipkv_status ipkv_paged_scratch_bytes(const ipkv_attn_shape* sh, int32_t n_rows, int32_t max_blocks, int32_t window, int32_t first_tokens,
                                     int32_t weigh, size_t* out_bytes) {
    if (!shape_ok(sh) || !capacity_ok(sh, n_rows, max_blocks) || !window_ok(window, first_tokens) || !out_bytes) return IPKV_EINVAL;
    const AttendPlan plan(sh, n_rows, max_blocks, window, first_tokens, weigh != 0);
    if (n_rows > 0 && plan.rows < 1) return IPKV_EINVAL;
    *out_bytes = plan.scratch();
    return IPKV_OK;
}

ipkv_status ipkv_paged_attend(const ipkv_paged_attend_call* call) {
    if (!call) return IPKV_EINVAL;
    const auto [sh, c, q_dev, q_row_stride, window, first_tokens, weights_out_dev, scratch_dev, scratch_bytes, o_part_dev, lse_part_dev, status_dev, stream] = *call;
    if (!cache_ok(sh, c) || !window_ok(window, first_tokens)) return IPKV_EINVAL;
    if (!(sh->softmax_scale >= 0.f) || std::isinf(sh->softmax_scale)) return IPKV_EINVAL;
    const int64_t row = int64_t(sh->n_q_heads) * sh->dim_qk;
    if (q_row_stride != 0 && (q_row_stride < row || q_row_stride % 8 != 0 || q_row_stride > (int64_t(1) << 40))) return IPKV_EINVAL;
    if (!aligned(q_dev, 16) || !aligned(o_part_dev, 16) || !aligned(lse_part_dev, 4) || !aligned(status_dev, 4) || !aligned(weights_out_dev, 16)) return IPKV_EINVAL;
    if (!aligned(scratch_dev, 256) || (c->n_rows > 0 && !scratch_dev)) return IPKV_EINVAL;
    if (weights_out_dev) {
        if (c->slot_stride < int64_t(c->max_blocks) * sh->block_tokens || c->slot_stride % 4 != 0 || c->slot_stride > (int64_t(1) << 32)) return IPKV_EINVAL;
        if (!apart(sh, c, c->weights_dev, weights_out_dev)) return IPKV_EINVAL;
    }
    const AttendPlan plan(sh, c->n_rows, c->max_blocks, window, first_tokens, weights_out_dev != nullptr);
    if (c->n_rows == 0) return IPKV_OK;
    if (!q_dev || !o_part_dev || !lse_part_dev || plan.rows < 1) return IPKV_EINVAL;
    if (plan.scratch() > scratch_bytes) return IPKV_ENOMEM;

    PagedAttend a;
    a.c = cache_of(sh, c);
    const PagedCache all = a.c;
    char* at = static_cast<char*>(scratch_dev);
    a.header = reinterpret_cast<PagedHeader*>(at);
    const size_t parts = size_t(2) * kSmCount * kPagedCtasPerSm * plan.rows_per_part;
    a.part_o = reinterpret_cast<float*>(at + plan.header);
    a.part_ml = reinterpret_cast<float2*>(at + plan.header + align_up(parts * sh->dim_qk * sizeof(float), 256));
    a.head_ml = weights_out_dev ? reinterpret_cast<float2*>(at + plan.header + plan.partials) : nullptr;
    a.scores = weights_out_dev ? reinterpret_cast<float*>(at + plan.header + plan.partials + plan.head_ml) : nullptr;
    a.q_row = 2 * (q_row_stride ? q_row_stride : row);
    a.status = status_dev;
    a.window = window; a.first = window > 0 ? first_tokens : 0;
    a.unit = plan.unit; a.most_units = int32_t(plan.most_units);
    a.n_q_heads = sh->n_q_heads; a.group = plan.group; a.groups_per_kv = plan.groups_per_kv; a.n_gh = plan.n_gh;
    a.rows_per_part = plan.rows_per_part; a.sixteens = plan.sixteens;
    a.bt_shift = (sh->block_tokens & (sh->block_tokens - 1)) == 0 ? __builtin_ctz(unsigned(sh->block_tokens)) : -1;
    const float scale = sh->softmax_scale > 0.f ? sh->softmax_scale : 1.0f / std::sqrt(float(sh->dim_qk));
    a.scale_log2 = scale * 1.4426950408889634f;
    for (int32_t r0 = 0; r0 < c->n_rows; r0 += plan.rows) {
        const int32_t n = std::min(plan.rows, c->n_rows - r0);
        rows_from(a.c, all, r0, n);
        a.q = static_cast<const char*>(q_dev) + r0 * a.q_row;
        a.out_o = o_part_dev + r0 * row;
        a.out_lse = lse_part_dev + int64_t(r0) * sh->n_q_heads;
        a.weights_out = weights_out_dev ? weights_out_dev + int64_t(r0) * sh->n_kv_heads * c->slot_stride : nullptr;
        const int64_t pairs = int64_t(n) * plan.n_gh, most = int64_t(kSmCount) * kPagedCtasPerSm;
        a.cluster = paged_cluster(pairs, plan.most_units, plan.group, plan.sixteens, int(most));
        if (a.cluster > kPagedPortableCluster) {
            int largest = 0;
            if (paged_largest_cluster(a, largest) != cudaSuccess) return IPKV_ECUDA;
            a.cluster = paged_cluster(pairs, plan.most_units, plan.group, plan.sixteens, int(most), largest);
        }
        a.n_ctas = int32_t(a.cluster ? pairs * a.cluster : std::min(most, pairs * plan.most_units));
        a.per_cta = 1.f / float(a.n_ctas);
        a.per_gh = plan.n_gh > 1 ? uint32_t(((uint64_t(1) << 32) + plan.n_gh - 1) / plan.n_gh) : 0;
        a.cluster_shift = a.cluster > 1 ? __builtin_ctz(unsigned(a.cluster)) : 0;
        if (launch_paged_attend(a, static_cast<cudaStream_t>(stream)) != cudaSuccess) return IPKV_ECUDA;
    }
    return IPKV_OK;
}

ipkv_status ipkv_paged_evict_scratch_bytes(const ipkv_attn_shape* sh, int32_t n_rows, int32_t max_blocks, int32_t budget, size_t* out_bytes) {
    if (!shape_ok(sh) || !capacity_ok(sh, n_rows, max_blocks) || budget < 1 || !out_bytes) return IPKV_EINVAL;
    const int64_t slots = int64_t(max_blocks) * sh->block_tokens, most = std::max<int64_t>(0, std::min<int64_t>(budget, slots - budget));
    *out_bytes = align_up(size_t(n_rows) * sh->n_kv_heads * 2 * size_t(most) * sizeof(int32_t), 256);
    return IPKV_OK;
}

ipkv_status ipkv_paged_evict(const ipkv_paged_evict_call* call) {
    if (!call) return IPKV_EINVAL;
    const auto [sh, c, budget, first_tokens, recent, weights_out_dev, positions_out_dev, kept_dev, scratch_dev, scratch_bytes, status_dev, stream] = *call;
    if (!cache_ok(sh, c) || budget < 1 || first_tokens < 0 || recent < 0 || int64_t(first_tokens) + recent > budget) return IPKV_EINVAL;
    if (c->n_rows > 0 && (!c->weights_dev || !c->positions_dev)) return IPKV_EINVAL;
    if (!aligned(weights_out_dev, 16) || !aligned(positions_out_dev, 16) || !aligned(kept_dev, 4) || !aligned(status_dev, 4)) return IPKV_EINVAL;
    if (!aligned(scratch_dev, 256)) return IPKV_EINVAL;
    PagedEvict a;
    a.weights_out = weights_out_dev ? weights_out_dev : c->weights_dev;
    a.positions_out = positions_out_dev ? positions_out_dev : c->positions_dev;
    if (!apart(sh, c, c->weights_dev, a.weights_out) || !apart(sh, c, c->positions_dev, a.positions_out)) return IPKV_EINVAL;
    size_t need = 0;
    if (ipkv_paged_evict_scratch_bytes(sh, c->n_rows, c->max_blocks, budget, &need) != IPKV_OK) return IPKV_EINVAL;
    if (c->n_rows == 0) return IPKV_OK;
    if (int64_t(c->n_rows) * sh->n_kv_heads > INT32_MAX / 16) return IPKV_EINVAL;       // the grid
    if (need > scratch_bytes) return IPKV_ENOMEM;
    if (need > 0 && !scratch_dev) return IPKV_EINVAL;
    a.c = cache_of(sh, c);
    a.kept = kept_dev; a.moved = static_cast<int32_t*>(scratch_dev); a.status = status_dev;
    a.budget = budget; a.first = first_tokens; a.recent = recent;
    const int64_t slots = int64_t(c->max_blocks) * sh->block_tokens;
    a.most_moved = int32_t(std::max<int64_t>(0, std::min<int64_t>(budget, slots - budget)));
    return launch_paged_evict(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? IPKV_OK : IPKV_ECUDA;
}

}  // extern "C"
