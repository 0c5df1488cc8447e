// C entry points of the operators beside the cache: what they refuse, and how a call becomes launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <utility>
#include <vector>

#include "../../include/ipkv.h"
#include "kernels.h"
#include "ops.h"
#include "plan.hpp"

using namespace ipkvi;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// ---- head norm and rotation ---------------------------------------------------------------------------------------

// One side (input or output) of a part: [n_tokens][n_heads] heads of `dim` columns, strides in elements.
struct HeadView {
    __int128 base, token, head, n_tokens, n_heads, dim;      // bytes
    __int128 heads_span() const { return (n_heads - 1) * head + dim; }
    __int128 end() const { return base + (n_tokens - 1) * token + (n_heads - 1) * head + dim; }
    bool token_major() const { return n_tokens == 1 || token >= heads_span(); }
};

bool same_view(const HeadView& a, const HeadView& b) {
    return a.base == b.base && a.n_tokens == b.n_tokens && a.n_heads == b.n_heads && (a.n_tokens == 1 || a.token == b.token) &&
           (a.n_heads == 1 || a.head == b.head);
}

// Whether two views may share a byte.  Exact where their tokens lie equally far apart and so do their heads (views of one buffer, q, k
// and v of a token side by side or head by head among them); other interleavings count as shared.
bool may_overlap(const HeadView& a, const HeadView& b) {
    if (a.end() <= b.base || b.end() <= a.base) return false;
    if (a.n_tokens > 1 && a.token != b.token) return true;
    if (a.n_tokens > 1 && a.token_major() && b.token_major()) {
        __int128 d = (b.base - a.base) % a.token;
        if (d < 0) d += a.token;
        // a covers [0, span_a) of every period, b covers [d, d + span_b)
        if (d >= a.heads_span() && d + b.heads_span() <= a.token) return false;
    }
    if (a.n_heads > 1 && b.n_heads > 1 && a.head != b.head) return true;
    // two of their heads lie d + i token + j head apart: is that less than a head for any i and j?  (In 64 bits where the views fit them:
    // 128-bit divisions took 8 us of a call with four parts.)
    const __int128 token = a.n_tokens > 1 ? a.token : 0, head = a.n_heads > 1 ? a.head : b.head;
    auto meet = [&](auto d, auto token, auto head, auto dim) {
        using Int = decltype(d);
        const Int most = Int(a.n_tokens - 1), last = Int(b.n_heads);
        for (Int j = Int(1 - a.n_heads); j < last; ++j) {
            const Int x = d + j * head, i = token > 0 ? -x / token : 0;          // the nearest i is this or one beside it
            for (Int k = i - 1; k <= i + 1; ++k) {
                const Int gap = x + (k < -most ? -most : k > most ? most : k) * token;
                if (gap < dim && -gap < dim) return true;
            }
        }
        return false;
    };
    constexpr __int128 kFits = __int128(1) << 60;
    const __int128 d = b.base - a.base, reach = (a.n_heads + b.n_heads) * head + (a.n_tokens + 1) * token + a.dim;
    if (d < kFits && -d < kFits && reach < kFits) return meet(int64_t(d), int64_t(token), int64_t(head), int64_t(a.dim));
    return meet(d, token, head, a.dim);
}

// ---- the cache in 4 bits ------------------------------------------------------------------------------------------

bool nibble_shape_ok(const ipkv_attn_shape* sh) {
    return sh && sh->kind == IPKV_GQA && sh->n_q_heads > 0 && sh->n_kv_heads > 0 && sh->n_kv_heads <= (1 << 16) && sh->n_q_heads <= (1 << 20) &&
           sh->n_q_heads % sh->n_kv_heads == 0 && sh->dim_qk == sh->dim_v && (sh->dim_qk == 64 || sh->dim_qk == 128) && sh->block_tokens > 0 &&
           sh->block_tokens % kTileTokens == 0 && sh->block_tokens <= (1 << 20);
}
NibbleGeom nibble_geom(const ipkv_attn_shape* sh) { return NibbleGeom{sh->n_kv_heads, sh->dim_qk, sh->block_tokens}; }

constexpr int64_t kMaxRunTokens = int64_t(1) << 36;      // keeps every product with a block's bytes inside 63 bits

// Checks the arguments of pack and unpack and issues their launches.
ipkv_status move_spans(const ipkv_attn_shape* sh, int32_t n_spans, const ipkv_span* spans, int64_t n_tokens, const void* k, const void* v, int64_t k_token_stride,
                       int64_t v_token_stride, bool pack, cudaStream_t stream) {
    if (!nibble_shape_ok(sh) || n_spans < 0 || (n_spans > 0 && !spans)) return IPKV_EINVAL;
    const NibbleGeom g = nibble_geom(sh);
    const int64_t row = int64_t(g.n_kv_heads) * g.dim;
    for (int64_t stride : {k_token_stride, v_token_stride})
        if (stride != 0 && (stride < row || stride % 8 != 0 || stride > (int64_t(1) << 48))) return IPKV_EINVAL;
    if (!aligned16(k) || !aligned16(v)) return IPKV_EINVAL;
    int64_t tokens = 0;
    bool single = true;
    std::vector<std::pair<uintptr_t, uintptr_t>> touched;            // blocks that a span writes
    for (int32_t i = 0; i < n_spans; ++i) {
        const ipkv_span& sp = spans[i];
        if (sp.first_token < 0 || sp.n_tokens < 0 || sp.first_token > kMaxRunTokens || sp.n_tokens > INT32_MAX - 2 * kTileTokens) return IPKV_EINVAL;
        if (sp.n_tokens == 0) continue;
        if (!sp.blocks_dev || !aligned16(sp.blocks_dev)) return IPKV_EINVAL;
        tokens += sp.n_tokens;
        single = single && sp.n_tokens == 1;
        if (pack) {
            const uintptr_t base = reinterpret_cast<uintptr_t>(sp.blocks_dev);
            touched.emplace_back(base + uintptr_t(sp.first_token / g.bt * g.block_bytes()),
                                 base + uintptr_t(((sp.first_token + sp.n_tokens - 1) / g.bt + 1) * g.block_bytes()));
        }
    }
    if (tokens != n_tokens) return IPKV_EINVAL;
    if (tokens == 0) return IPKV_OK;
    if (!k || !v) return IPKV_EINVAL;
    std::sort(touched.begin(), touched.end());
    for (size_t i = 1; i < touched.size(); ++i)
        if (touched[i].first < touched[i - 1].second) return IPKV_EINVAL;
    NibbleMove a;
    a.g = g;
    a.k = static_cast<char*>(const_cast<void*>(k)); a.v = static_cast<char*>(const_cast<void*>(v));
    a.k_token = 2 * (k_token_stride ? k_token_stride : row); a.v_token = 2 * (v_token_stride ? v_token_stride : row);
    a.n_spans = 0; a.n_tiles = 0;
    int64_t src = 0;
    auto launch = [&]() {
        const cudaError_t e = a.n_spans == 0 ? cudaSuccess : pack ? launch_nibble_pack(a, single, stream) : launch_nibble_unpack(a, single, stream);
        a.n_spans = 0; a.n_tiles = 0;
        return e;
    };
    for (int32_t i = 0; i < n_spans; ++i) {
        const ipkv_span& sp = spans[i];
        if (sp.n_tokens == 0) continue;
        const int32_t tiles = int32_t((sp.first_token + sp.n_tokens - 1) / kTileTokens - sp.first_token / kTileTokens + 1);
        if (a.n_spans == kNibbleSpansPerLaunch || int64_t(a.n_tiles) + tiles > INT32_MAX / 2)
            if (launch() != cudaSuccess) return IPKV_ECUDA;
        a.span[a.n_spans++] = NibbleSpanArg{static_cast<char*>(sp.blocks_dev), sp.first_token, src, int32_t(sp.n_tokens), a.n_tiles};
        a.n_tiles += tiles;
        src += sp.n_tokens;
    }
    return launch() == cudaSuccess ? IPKV_OK : IPKV_ECUDA;
}

// Head groups of a row, partials that a launch of n_rows rows can have, and the scratch for them behind the tables.
struct NibblePlan {
    int group, groups_per_kv, n_gh, rows_per_part, octets, teams;
    explicit NibblePlan(const ipkv_attn_shape* sh)
        : group(sh->n_q_heads / sh->n_kv_heads), groups_per_kv(nibble_groups_per_kv(group)), n_gh(sh->n_kv_heads * groups_per_kv),
          rows_per_part(nibble_rows_per_part(group)), octets((rows_per_part + 7) / 8), teams(nibble_teams(octets)) {}
    static constexpr int kCtas = kSmCount * kNibbleCtasPerSm;
    size_t part_rows(int32_t n_rows) const { return (size_t(kCtas) + size_t(n_rows) * n_gh) * teams * rows_per_part; }
    static bool inlined(int32_t n_rows, int64_t n_runs) { return n_rows <= kNibbleInlineRows && n_runs <= kNibbleInlineRuns; }
    static size_t table_bytes(int32_t n_rows, int64_t n_runs) {
        return inlined(n_rows, n_runs) ? 0 : align_up(size_t(n_rows) * sizeof(NibbleRowArg) + size_t(n_runs) * sizeof(NibbleRunArg), 256);
    }
    size_t scratch(int32_t n_rows, int64_t n_runs, int dim) const {
        return table_bytes(n_rows, n_runs) + align_up(part_rows(n_rows) * dim * sizeof(float), 256) + align_up(part_rows(n_rows) * sizeof(float2), 256);
    }
};

ipkv_status attend_nibbles(const ipkv_attn_shape* sh, int32_t n_rows, const ipkv_run* runs, const int32_t* row_run_start, const void* q,
                           void* scratch, size_t scratch_bytes, float* o, float* lse, uint32_t* status, cudaStream_t stream) {
    if (!nibble_shape_ok(sh) || n_rows <= 0 || !row_run_start || !q || !scratch || !o || !lse) return IPKV_EINVAL;
    if (!(sh->softmax_scale >= 0.f) || std::isinf(sh->softmax_scale)) return IPKV_EINVAL;
    if (!aligned16(q) || !aligned16(o) || (reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(status) & 3u)) return IPKV_EINVAL;
    if (reinterpret_cast<uintptr_t>(scratch) & 255u) return IPKV_EINVAL;
    if (int64_t(n_rows) * sh->n_q_heads > INT32_MAX / 4) return IPKV_EINVAL;          // the join's grid
    const NibblePlan plan(sh);
    if (row_run_start[0] < 0) return IPKV_EINVAL;
    for (int r = 0; r < n_rows; ++r)
        if (row_run_start[r] > row_run_start[r + 1]) return IPKV_EINVAL;
    const int32_t k0 = row_run_start[0], k1 = row_run_start[n_rows];
    if (k1 > k0 && !runs) return IPKV_EINVAL;
    NibbleAttend a;
    int64_t live = 0;
    for (int32_t k = k0; k < k1; ++k) {
        if (runs[k].n_tokens < 0 || runs[k].n_tokens > INT32_MAX - 2 * kTileTokens) return IPKV_EINVAL;
        if (runs[k].n_tokens > 0 && (!runs[k].blocks_dev || !aligned16(runs[k].blocks_dev))) return IPKV_EINVAL;
        live += runs[k].n_tokens > 0;
    }
    const bool inlined = NibblePlan::inlined(n_rows, live);
    std::vector<char> image;
    NibbleRowArg* row = a.row;
    NibbleRunArg* run = a.run;
    const size_t table = NibblePlan::table_bytes(n_rows, live);
    if (plan.scratch(n_rows, live, sh->dim_qk) > scratch_bytes) return IPKV_ENOMEM;
    if (!inlined) {
        image.resize(table);
        row = reinterpret_cast<NibbleRowArg*>(image.data());
        run = reinterpret_cast<NibbleRunArg*>(row + n_rows);
    }
    int64_t units = 0, longest = 0;
    int32_t n_runs = 0, pairs = 0;
    for (int r = 0; r < n_rows; ++r) {
        int64_t tiles = 0;
        row[r].run0 = n_runs; row[r].pair0 = pairs; row[r].first = int32_t(units);
        for (int32_t k = row_run_start[r]; k < row_run_start[r + 1]; ++k) {
            if (runs[k].n_tokens == 0) continue;
            run[n_runs++] = NibbleRunArg{static_cast<const char*>(runs[k].blocks_dev), int32_t(runs[k].n_tokens), int32_t(tiles)};
            tiles += (runs[k].n_tokens + kTileTokens - 1) / kTileTokens;
            if (tiles > INT32_MAX) return IPKV_EINVAL;
        }
        row[r].tiles = int32_t(tiles);
        longest = std::max(longest, tiles);
        if (tiles > 0) units += (tiles + kNibblePairCost) * plan.n_gh;
        pairs += tiles > 0 ? plan.n_gh : 0;
        if (units > INT32_MAX) return IPKV_EINVAL;
    }
    a.n_ctas = units < NibblePlan::kCtas ? int32_t(units) : NibblePlan::kCtas;
    a.max_parts = units > 0 ? int32_t((((longest + kNibblePairCost) * a.n_ctas + units - 1) / units + 1) * plan.teams) : 0;
    const NibbleSplit split = nibble_split(row, n_rows, plan.n_gh, plan.teams, units, pairs, longest, kSmCount);
    a.whole = split.whole;
    a.share = split.share;
    if (a.whole) a.n_ctas = n_rows * plan.n_gh;
    if (a.share > 0) {
        int64_t ctas = 0;
        for (int r = 0; r < n_rows; ++r) { row[r].first = int32_t(ctas); ctas += plan.n_gh * ((row[r].tiles + a.share - 1) / a.share); }
        a.n_ctas = int32_t(ctas);
        a.max_parts = int32_t((longest + a.share - 1) / a.share * plan.teams);
    }
    a.rows = nullptr; a.runs = nullptr; a.plain_launch = 0; a.odd_tokens = 0xffff0000u;
    if (!inlined) {
        // as ipkv_attend_runs: a captured copy would be replayed from the image's address long after it is gone
        cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(stream, &capturing) != cudaSuccess) return IPKV_ECUDA;
        if (capturing == cudaStreamCaptureStatusNone) {
            if (cudaMemcpyAsync(scratch, image.data(), table, cudaMemcpyHostToDevice, stream) != cudaSuccess) return IPKV_ECUDA;
        } else if (launch_upload_by_value(scratch, image.data(), table, stream) != cudaSuccess) {
            return IPKV_ECUDA;
        } else {
            a.plain_launch = 1;
        }
        a.rows = static_cast<const NibbleRowArg*>(scratch);
        a.runs = reinterpret_cast<const NibbleRunArg*>(a.rows + n_rows);
    }
    a.g = nibble_geom(sh);
    a.q = static_cast<const char*>(q);
    char* partials = static_cast<char*>(scratch) + table;
    a.part_o = reinterpret_cast<float*>(partials);
    a.part_ml = reinterpret_cast<float2*>(partials + align_up(plan.part_rows(n_rows) * sh->dim_qk * sizeof(float), 256));
    a.part_rows = int64_t(plan.part_rows(n_rows));
    a.out_o = o; a.out_lse = lse; a.status = status;
    a.n_rows = n_rows; a.n_units = int32_t(units); a.n_runs = n_runs;
    a.n_q_heads = sh->n_q_heads; a.group = plan.group; a.groups_per_kv = plan.groups_per_kv; a.n_gh = plan.n_gh; a.rows_per_part = plan.rows_per_part;
    a.octets = plan.octets; a.teams = plan.teams;
    a.scale = sh->softmax_scale > 0.f ? sh->softmax_scale : 1.0f / std::sqrt(float(sh->dim_qk));
    return launch_nibble_attend(a, stream) == cudaSuccess ? IPKV_OK : IPKV_ECUDA;
}

// Nothing leaves a C entry as an exception: the tables on the host are the only thing here that can throw.
template <class F>
ipkv_status guarded(F&& f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return IPKV_ENOMEM;
    } catch (...) {
        return IPKV_EINTERNAL;
    }
}

}  // namespace

extern "C" {

ipkv_status ipkv_norm_rope(const ipkv_rope* rope, int64_t n_tokens, const ipkv_heads* parts, int32_t n_parts,
                           const int32_t* positions_dev, void* stream) {
    if (!rope || !parts || n_parts < 1 || n_parts > kRopeMaxParts || n_tokens < 0 || n_tokens > INT32_MAX) return IPKV_EINVAL;
    if (rope->dim != 64 && rope->dim != 128 && rope->dim != 256) return IPKV_EINVAL;
    if (rope->rot_dim < 0 || rope->rot_dim > rope->dim || rope->rot_dim % 16 != 0) return IPKV_EINVAL;
    if (rope->n_axes < 1 || rope->n_axes > 4) return IPKV_EINVAL;
    if (!(rope->eps >= 0.f) || std::isinf(rope->eps)) return IPKV_EINVAL;
    const int pairs = rope->rot_dim / 2;
    if (pairs > 0 && !rope->inv_freq && (!(rope->theta > 0.0) || std::isinf(rope->theta))) return IPKV_EINVAL;
    if (pairs > 0 && n_tokens > 0 && !positions_dev) return IPKV_EINVAL;
    if (reinterpret_cast<uintptr_t>(positions_dev) & 3u) return IPKV_EINVAL;
    for (int i = 0; i < pairs; ++i) {
        if (rope->inv_freq && !std::isfinite(rope->inv_freq[i])) return IPKV_EINVAL;
        if (rope->pair_axis && rope->pair_axis[i] >= rope->n_axes) return IPKV_EINVAL;
    }
    RopeLaunch a{};
    HeadView in[kRopeMaxParts], out[kRopeMaxParts];
    const int per_step = rope_heads_per_step(rope->dim);
    for (int i = 0; i < n_parts; ++i) {
        const ipkv_heads& h = parts[i];
        if (h.n_heads < 1 || h.n_heads > (1 << 20)) return IPKV_EINVAL;
        if (n_tokens > 0 && (!h.in_dev || !h.out_dev)) return IPKV_EINVAL;
        if (!aligned16(h.in_dev) || !aligned16(h.out_dev) || !aligned16(h.weight_dev)) return IPKV_EINVAL;
        const int64_t strides[4] = {h.in_token_stride, h.in_head_stride, h.out_token_stride, h.out_head_stride};
        for (int64_t x : strides)
            if (x < 0 || x % 8 != 0 || x > (int64_t(1) << 48)) return IPKV_EINVAL;
        in[i] = HeadView{__int128(reinterpret_cast<uintptr_t>(h.in_dev)), __int128(h.in_token_stride) * 2, __int128(h.in_head_stride) * 2,
                         n_tokens, h.n_heads, __int128(rope->dim) * 2};
        out[i] = HeadView{__int128(reinterpret_cast<uintptr_t>(h.out_dev)), __int128(h.out_token_stride) * 2, __int128(h.out_head_stride) * 2,
                          n_tokens, h.n_heads, __int128(rope->dim) * 2};
        // no two heads of an output may share bytes: tokens outside heads, or heads outside tokens
        const bool heads_apart = h.n_heads == 1 || out[i].head >= out[i].dim, tokens_apart = n_tokens <= 1 || out[i].token >= out[i].dim;
        const bool outer_token = n_tokens <= 1 || out[i].token >= out[i].heads_span();
        const bool outer_head = h.n_heads == 1 || out[i].head >= (__int128(n_tokens) - 1) * out[i].token + out[i].dim;
        if (n_tokens > 0 && !(heads_apart && tokens_apart && (outer_token || outer_head))) return IPKV_EINVAL;
        RopePart& q = a.part[i];
        q.in = static_cast<const char*>(h.in_dev); q.out = static_cast<char*>(h.out_dev); q.weight = static_cast<const char*>(h.weight_dev);
        q.in_token = h.in_token_stride * 2; q.in_head = h.in_head_stride * 2;
        q.out_token = h.out_token_stride * 2; q.out_head = h.out_head_stride * 2;
        q.n_heads = h.n_heads; q.step0 = a.n_steps;
        a.n_steps += (h.n_heads + per_step - 1) / per_step;
    }
    if (n_tokens == 0) return IPKV_OK;
    for (int i = 0; i < n_parts; ++i)
        for (int k = 0; k < n_parts; ++k) {
            if (i != k && may_overlap(out[i], out[k])) return IPKV_EINVAL;
            if (!(i == k && same_view(out[i], in[k])) && may_overlap(out[i], in[k])) return IPKV_EINVAL;
        }
    constexpr long double kTurnsPerRadian = 0.159154943091895335768883763372514362L;
    // theta^(-2i / rot_dim) by repeated multiplication (one power a call instead of one a pair): at most 127 roundings of 2^-64
    const long double ratio = pairs > 0 && !rope->inv_freq ? powl(static_cast<long double>(rope->theta), -2.0L / rope->rot_dim) : 1.0L;
    long double power = 1.0L;
    for (int i = 0; i < pairs; ++i) {
        long double turns = (rope->inv_freq ? static_cast<long double>(rope->inv_freq[i]) : power) * kTurnsPerRadian;
        power *= ratio;
        if (turns < 0.0L || turns >= 1.0L) turns -= floorl(turns);   // whole turns change nothing: positions are integers
        const long double scaled = turns * 18446744073709551616.0L + 0.5L;
        a.turn[i] = scaled >= 18446744073709551616.0L ? 0u : static_cast<uint64_t>(scaled);
        a.axis[i] = rope->pair_axis ? rope->pair_axis[i] : uint8_t(0);
    }
    a.positions = positions_dev; a.n_tokens = n_tokens; a.n_parts = n_parts; a.dim = rope->dim; a.rot_dim = rope->rot_dim;
    a.n_axes = rope->n_axes; a.interleaved = rope->interleaved != 0; a.eps = rope->eps;
    return launch_norm_rope(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? IPKV_OK : IPKV_ECUDA;
}

int64_t ipkv_nibble_block_bytes(const ipkv_attn_shape* sh) { return nibble_shape_ok(sh) ? nibble_geom(sh).block_bytes() : -1; }

ipkv_status ipkv_nibble_pack(const ipkv_attn_shape* sh, int32_t n_spans, const ipkv_span* spans, int64_t n_tokens,
                             const void* k_dev, const void* v_dev, int64_t k_token_stride, int64_t v_token_stride, void* stream) {
    return guarded([&] { return move_spans(sh, n_spans, spans, n_tokens, k_dev, v_dev, k_token_stride, v_token_stride, true, static_cast<cudaStream_t>(stream)); });
}

ipkv_status ipkv_nibble_unpack(const ipkv_attn_shape* sh, int32_t n_spans, const ipkv_span* spans, int64_t n_tokens,
                               void* k_dev, void* v_dev, int64_t k_token_stride, int64_t v_token_stride, void* stream) {
    return guarded([&] { return move_spans(sh, n_spans, spans, n_tokens, k_dev, v_dev, k_token_stride, v_token_stride, false, static_cast<cudaStream_t>(stream)); });
}

ipkv_status ipkv_nibble_scratch_bytes(const ipkv_attn_shape* sh, int32_t n_rows, int32_t n_runs, size_t* out_bytes) {
    if (!nibble_shape_ok(sh) || n_rows < 0 || n_runs < 0 || !out_bytes) return IPKV_EINVAL;
    *out_bytes = NibblePlan(sh).scratch(n_rows, n_runs, sh->dim_qk);
    return IPKV_OK;
}

ipkv_status ipkv_nibble_attend(const ipkv_attn_shape* sh, int32_t n_rows, const ipkv_run* runs, const int32_t* row_run_start, const void* q_dev,
                               void* scratch_dev, size_t scratch_bytes, float* o_part_dev, float* lse_part_dev, uint32_t* status_dev,
                               void* stream) {
    return guarded([&] { return attend_nibbles(sh, n_rows, runs, row_run_start, q_dev, scratch_dev, scratch_bytes, o_part_dev, lse_part_dev,
                                               status_dev, static_cast<cudaStream_t>(stream)); });
}

}  // extern "C"
