// C ABI of the cache and attention operators: checks of arguments, choice of kernels and grids.
#include "at_append.hpp"
#include "at_few.hpp"
#include "at_host.hpp"
#include "at_many.hpp"

namespace {

ap_status take_cache(const ap_kv_cache* c, Cache* out) {
    if (!c || c->dtype > AP_FP16 || (c->bits != 16 && c->bits != 4) || (c->head_dim != 64 && c->head_dim != 128)) return AP_ERR_INVALID;
    if (c->n_pages == 0 || c->page_size == 0 || c->kv_heads == 0 || !c->k || !c->v) return AP_ERR_INVALID;
    if (!multiple(c->k, 16) || !multiple(c->v, 16)) return AP_ERR_INVALID;
    if (!stride_ok(c->page_stride, 16) || !stride_ok(c->head_stride, 16) || !stride_ok(c->slot_stride, 16)) return AP_ERR_INVALID;
    if (c->bits == 4) {
        const int64_t n = 4 * (c->head_dim / 64);
        if (!c->k_pairs || !c->v_pairs || !multiple(c->k_pairs, n) || !multiple(c->v_pairs, n)) return AP_ERR_INVALID;
        if (!stride_ok(c->pair_page_stride, n) || !stride_ok(c->pair_head_stride, n) || !stride_ok(c->pair_slot_stride, n)) return AP_ERR_INVALID;
    }
    if (c->n_pages >= kMost || c->page_size >= kMost || c->kv_heads >= kMost) return AP_ERR_RANGE;
    *out = Cache{(char*)c->k, (char*)c->v, (char*)c->k_pairs, (char*)c->v_pairs, c->page_stride, c->head_stride, c->slot_stride,
                 c->pair_page_stride, c->pair_head_stride, c->pair_slot_stride, c->n_pages, c->page_size, 0, 0};
    divider(c->page_size, &out->magic, &out->shift);
    return AP_OK;
}

ap_status take_batch(const ap_kv_cache* c, const ap_seq_batch* b, Batch* out) {
    if (!b || b->n_seqs == 0 || b->max_kv == 0 || b->table_width == 0 || !b->new_first || !b->kv_len || !b->page_table) return AP_ERR_INVALID;
    if (b->n_tokens != 0 && b->max_new == 0) return AP_ERR_INVALID;
    if (b->table_stride < (int64_t)b->table_width || !multiple(b->new_first, 4) || !multiple(b->kv_len, 4) || !multiple(b->page_table, 4)) return AP_ERR_INVALID;
    if ((uint64_t)b->table_width * c->page_size < b->max_kv) return AP_ERR_RANGE;
    if (b->max_kv >= kMost - 4096 || b->n_tokens >= kMost || b->n_seqs >= kMost) return AP_ERR_RANGE;
    *out = Batch{b->new_first, b->kv_len, b->page_table, b->table_stride, b->n_seqs, b->n_tokens, std::min(b->max_new, b->n_tokens), b->max_kv};
    return AP_OK;
}

ap_status take_rows(const ap_rows* r, Rows* out) {
    if (!r || !r->data || !multiple(r->data, 16) || !stride_ok(r->token_stride, 16) || !stride_ok(r->head_stride, 16)) return AP_ERR_INVALID;
    *out = Rows{(char*)r->data, r->token_stride, r->head_stride};
    return AP_OK;
}

template <typename F> void for_type(uint32_t dtype, F f) { dtype == AP_BF16 ? f(bf16{}) : f(fp16{}); }
template <typename F> void for_dim(uint32_t d, F f) { d == 128 ? f(std::integral_constant<uint32_t, 128>{}) : f(std::integral_constant<uint32_t, 64>{}); }
template <typename F> void for_bits(uint32_t b, F f) { b == 16 ? f(std::integral_constant<uint32_t, 16>{}) : f(std::integral_constant<uint32_t, 4>{}); }
template <typename F> void for_cache(const ap_kv_cache* c, F f) {
    for_type(c->dtype, [&](auto e) { for_dim(c->head_dim, [&](auto d) { for_bits(c->bits, [&](auto b) { f(e, d, b); }); }); });
}

// Heads that a wavefront takes one after another: with few tokens a pass each, so that the call is as short as one pass;
// with many up to four, which share the look-up of the token and its cosines.
void row_grid(AppendParams* p, uint32_t heads, uint32_t heads_at_once, dim3* grid) {
    uint32_t passes = 1;
    while (passes < 4 && (uint64_t)p->batch.n_tokens * heads / (heads_at_once * passes) > 16384) passes *= 2;
    p->heads_per_wave = heads_at_once * passes;
    *grid = dim3((p->batch.n_tokens + kAppendThreads / kLanes - 1) / (kAppendThreads / kLanes), (heads + p->heads_per_wave - 1) / p->heads_per_wave);
}

uint32_t tiles_of(uint64_t n, uint32_t tile) { return (uint32_t)((n + tile - 1) / tile); }

// Tiles of keys that `span` neighbouring new tokens can see at most.
uint32_t most_tiles(const Batch& b, uint32_t window, uint32_t sinks, uint64_t span, uint32_t tile) {
    if (!window) return tiles_of(b.max_kv, tile);
    return tiles_of(std::min<uint64_t>(b.max_kv, (uint64_t)window + span - 1), tile) + tiles_of(std::min(sinks, b.max_kv), tile);
}

struct Plan {
    bool few, many;
    uint32_t few_tiles;                  // tiles of 16 rows
    uint32_t few_rows, few_stride, few_groups, few_seqs;
    bool few_team;                       // a workgroup for each (sequence, kv head)
    uint32_t many_chunk, many_chunks, row_tiles;
    uint64_t few_n, many_n;              // rows of results in the workspace
    uint64_t plan_bytes, bytes;
};

constexpr uint32_t kCus = 256;

// Workgroups on a CU of the kernel of few rows on the line.  Those of kFewDoubles take all that fit where a wavefront's share of
// the line stays kLeastPlaces, otherwise half as many, which leave less to join.  64 channels, up to 16 rows, four on a SIMD
// against two: 0.84 to 0.94 of the time with 12 to 24 places each, 0.99 to 1.02 with 3.4 to 6, 1.17 with 3; 128 channels,
// up to 32 rows, two against one: 0.70 to 0.82 with 12 places and more, 0.94 to 1.04 with 5 to 10, 1.20 with 3.  (A third one
// costs 16 bits with 64 channels 1.04 and 4 bits with 128 channels and 16 rows 1.2 of the time.)
constexpr uint32_t kLeastPlaces = 8;
uint32_t per_cu(uint32_t d, uint32_t bits, uint32_t tiles, uint64_t units) {
    uint32_t n = 0;
    bool doubles = false;
    auto of = [&](auto dim, auto b, auto t) { n = kFewPerSimd<dim(), b(), t(), false>, doubles = kFewDoubles<dim(), b(), t(), false>; };
    for_dim(d, [&](auto dim) {
        for_bits(bits, [&](auto b) { tiles == 1 ? of(dim, b, std::integral_constant<uint32_t, 1>{}) : of(dim, b, std::integral_constant<uint32_t, 2>{}); });
    });
    return doubles && units < (uint64_t)kLeastPlaces * n * kCus * kLineWaves ? n / 2 : n;
}

// How the kernel of few rows deals out its work.  32 heads on 8, 128 channels, bf16, sequences of one length, us:
//  - A team for each (sequence, head) while these are fewer than the chip's 256 CUs, and not so long that a ragged batch,
//    which takes as long as its longest, would wait for one.  Team / line: 8 sequences of 256 keys 7.1 / 11.8, of 512
//    9.4 / 13.2, of 1024 12.8 / 17.5, of 4096 48 / 37; 32 sequences of 512 14.8 / 21.2 (of 256 about 14 on the line).
//  - Otherwise short sequences go uncut to a wavefront each, so that nothing is left to join (which costs about 5 us, a tile
//    of a wavefront on its own about 1.1 us).  Uncut / line / team: 64 sequences of 128 keys 11.8 / 16.2 / 14.3, of 256
//    16.8 / 20.9 / -, of 512 34.5 / 36.6 / 32.2 (4 bits 25.7 / 20.9 / 19.7).
//  - Otherwise the line: each wavefront an equal piece.
constexpr uint32_t kTeamPairs = 256, kTeamTiles = 16, kTeamTilesOfFew = 32, kFewPairs = 128;
constexpr uint32_t kUncutTiles = 5, kUncutTilesOfMany = 8, kManyPairs = 512;
constexpr uint32_t kFewLeast = 2;        // places of the line that a wavefront of the kernel of few rows takes at least

// Into how many chunks the keys of each tile of rows are cut: where the workgroups (tiles of rows times heads) do not fill the
// chip, more of them are faster until joining costs more.  Estimated from what was measured (one chunk of 1024 tokens over 8192,
// 32 heads on 8, 128 channels, of 1 to 4 sequences, so 256 to 1024 workgroups: 227, 309, 519, 584 us): a tile of keys takes a
// workgroup kTileUs with the CU full of them, and 0.4 and a share of 0.6 of that with fewer; parts are written and read
// at about 4 TB/s, and joining them is a launch more.  Against as many chunks as whole workgroups still fit in: one sequence of
// those four 226 -> 177 us, two of 512 tokens over 16384 with 64 channels 392 -> 203 us, others 0.98 to 1.01 of the time.
uint32_t chunks_of(uint32_t d, uint32_t bits, uint64_t groups, uint32_t tiles, uint64_t rows) {
    constexpr double kTileUs = 2.4, kEnterTiles = 3, kLaunchUs = 5, kPartBytesPerUs = 4e6;
    constexpr uint32_t kLeastTiles = 8, kMostChunks = 64;
    uint32_t on_cu = 0, best = 1;
    for_dim(d, [&](auto dim) { for_bits(bits, [&](auto b) { on_cu = kManyPerCu<dim(), b()>; }); });
    double least = 0;
    for (uint32_t n = 1; n <= kMostChunks && (n == 1 || tiles >= n * kLeastTiles); ++n) {
        const uint64_t all = groups * n, full = all / (kCus * on_cu), rest = all % (kCus * on_cu);
        const double rounds = (double)full + (rest ? 0.4 + 0.6 * (double)((rest + kCus - 1) / kCus) / on_cu : 0.0);
        const double us = rounds * ((tiles + n - 1) / n + kEnterTiles) * kTileUs + (n > 1 ? kLaunchUs + 2.0 * (double)n * (double)rows * (4.0 * d + 8) / kPartBytesPerUs : 0.0);
        if (n == 1 || us < least) least = us, best = n;
    }
    return best;
}

ap_status plan_of(const ap_kv_cache* c, const Batch& b, uint32_t q_heads, uint32_t window, uint32_t sinks, Plan* out) {
    Plan r{};
    const uint32_t group = q_heads / c->kv_heads;
    const uint64_t rows = (uint64_t)b.max_new * group;
    if ((uint64_t)b.n_tokens * q_heads >= kMost || (uint64_t)b.n_seqs * c->kv_heads >= kMost) return AP_ERR_RANGE;
    // A batch of one sequence, or of sequences that all have few rows, needs one kernel only; in a mixed one each takes
    // the sequences that suit it.  The two launches for few rows are left out where as many tokens came as if all sequences had
    // max_new, and where the batch looks like whole prompts: no sequence holds more than max_new, and on average a quarter of that
    // is new.  A sequence of few rows then costs the kernel of many no longer than the last rows of the longest prompt: 16 prompts
    // of up to 512 57 -> 55 us, 5 of up to 300 17.5 -> 15.7, 4 of 1024 beside 12 single tokens over as many 83 -> 75 (4 bits 92 -> 93).
    const uint64_t most_tokens = (uint64_t)b.n_seqs * b.max_new;
    const bool prompts = b.n_tokens == most_tokens || (b.max_kv <= b.max_new && 4ull * b.n_tokens >= most_tokens);
    r.few = b.n_tokens && group <= kFewRows && (rows <= kFewRows || (b.n_seqs > 1 && !prompts));
    r.many = b.n_tokens && rows > kFewRows;
    if (r.few) {
        const uint64_t most = r.many ? (group <= 16 ? 16 : kFewRows) : rows;
        r.few_tiles = most <= 16 ? 1 : 2;
        r.few_rows = r.many ? (uint32_t)most : kFewRows;
        r.few_stride = (uint32_t)most;
        const uint32_t tiles = most_tiles(b, window, sinks, std::max<uint64_t>(1, most / group), kFewKeys);
        r.few_seqs = std::min(b.n_seqs, kFewSeqs);
        const uint64_t pairs = (uint64_t)r.few_seqs * c->kv_heads, units = pairs * ((uint64_t)tiles + kFewEnter);
        if (units >= kMost || pairs * r.few_stride >= kMostGroups) return AP_ERR_RANGE;
        if (pairs <= kTeamPairs && tiles <= (pairs <= kFewPairs ? kTeamTilesOfFew : kTeamTiles)) {
            r.few_team = true;
        } else if (tiles <= (pairs >= kManyPairs ? kUncutTilesOfMany : kUncutTiles)) {
            r.few_groups = (uint32_t)((pairs + kLineWaves - 1) / kLineWaves);
        } else {
            r.few_groups = (uint32_t)std::min<uint64_t>((units + kLineWaves - 1) / kLineWaves, kCus * per_cu(c->head_dim, c->bits, r.few_tiles, units));
            r.plan_bytes = (4ull * (r.few_seqs + 2) + 15) / 16 * 16;
            r.few_n = 2ull * r.few_groups * kLineWaves * r.few_stride;
        }
    }
    if (r.many) {
        r.row_tiles = (uint32_t)((uint64_t)b.n_tokens * group / kManyRows) + b.n_seqs;
        const uint32_t tiles = most_tiles(b, window, sinks, kManyRows / group + 2, kManyKeys);
        const uint64_t groups = ((uint64_t)b.n_tokens * group + kManyRows - 1) / kManyRows * c->kv_heads;
        const uint32_t chunks = chunks_of(c->head_dim, c->bits, groups, tiles, (uint64_t)b.n_tokens * q_heads);
        r.many_chunk = (tiles + chunks - 1) / chunks;
        r.many_chunks = (tiles + r.many_chunk - 1) / r.many_chunk;
        if (((uint64_t)r.row_tiles) * c->kv_heads * r.many_chunks >= kMostGroups) return AP_ERR_RANGE;
        if (r.many_chunks > 1) {
            r.many_n = (uint64_t)r.many_chunks * b.n_tokens * q_heads;
            if ((uint64_t)b.n_tokens * ((q_heads + 3) / 4) >= kMostGroups) return AP_ERR_RANGE;
        }
    }
    r.bytes = r.plan_bytes + (4ull * c->head_dim + 8) * (r.few_n + r.many_n);
    *out = r;
    return AP_OK;
}

}  // namespace

extern "C" {

ap_status ap_kv_append(const ap_kv_cache* cache, const ap_seq_batch* batch, const ap_rows* k, const ap_rows* v, const ap_rotation* rotation,
                       const ap_rows* q, const ap_rows* q_out, uint32_t q_heads, void* stream) {
    AppendParams p{};
    ap_status st = take_cache(cache, &p.cache);
    if (st == AP_OK) st = take_batch(cache, batch, &p.batch);
    if (st == AP_OK) st = take_rows(k, &p.k);
    if (st == AP_OK) st = take_rows(v, &p.v);
    if (st == AP_OK && q) {
        if (q_heads == 0) return AP_ERR_INVALID;
        st = take_rows(q, &p.q);
        if (st == AP_OK) st = take_rows(q_out, &p.q_out);
        p.q_heads = q_heads;
    }
    if (st != AP_OK) return st;
    p.kv_heads = cache->kv_heads;
    if (rotation) {
        if (!rotation->table || !multiple(rotation->table, 16) || rotation->rot_dim == 0 || rotation->rot_dim % 16 || rotation->rot_dim > cache->head_dim)
            return AP_ERR_INVALID;
        if (rotation->n_positions < batch->max_kv) return AP_ERR_RANGE;
        p.turn = rotation->table, p.rot = rotation->rot_dim;
    }
    const uint64_t heads = 2ull * cache->kv_heads + p.q_heads;
    if (heads >= 65536 || batch->n_tokens >= kMostGroups || (uint64_t)batch->n_tokens * heads >= kMost) return AP_ERR_RANGE;
    if (batch->n_tokens == 0) return AP_OK;
    dim3 grid;
    row_grid(&p, (uint32_t)heads, kLanes / (cache->head_dim / 16), &grid);
    const bool halves = !(rotation && rotation->neighbours);
    for_cache(cache, [&](auto e, auto d, auto b) {
        auto kernel = halves ? k_append<decltype(e), d(), b(), true> : k_append<decltype(e), d(), b(), false>;
        hipLaunchKernelGGL(kernel, grid, dim3(kAppendThreads), 0, (hipStream_t)stream, p);
    });
    return launched();
}

ap_status ap_kv_read(const ap_kv_cache* cache, const ap_seq_batch* batch, const ap_rows* k_out, const ap_rows* v_out, void* stream) {
    AppendParams p{};
    ap_status st = take_cache(cache, &p.cache);
    if (st == AP_OK) st = take_batch(cache, batch, &p.batch);
    if (st == AP_OK) st = take_rows(k_out, &p.k);
    if (st == AP_OK) st = take_rows(v_out, &p.v);
    if (st != AP_OK) return st;
    p.kv_heads = cache->kv_heads;
    const uint64_t heads = 2ull * cache->kv_heads;
    if (heads >= 65536 || batch->n_tokens >= kMostGroups || (uint64_t)batch->n_tokens * heads >= kMost) return AP_ERR_RANGE;
    if (batch->n_tokens == 0) return AP_OK;
    dim3 grid;
    row_grid(&p, (uint32_t)heads, kLanes / (cache->head_dim / 8), &grid);
    for_cache(cache, [&](auto e, auto d, auto b) {
        hipLaunchKernelGGL((k_read<decltype(e), d(), b()>), grid, dim3(kAppendThreads), 0, (hipStream_t)stream, p);
    });
    return launched();
}

ap_status ap_attention_workspace(const ap_kv_cache* cache, const ap_seq_batch* batch, uint32_t q_heads, uint32_t window, uint32_t sinks, uint64_t* bytes) {
    Cache c;
    Batch b;
    Plan plan;
    if (!bytes) return AP_ERR_INVALID;
    ap_status st = take_cache(cache, &c);
    if (st == AP_OK) st = take_batch(cache, batch, &b);
    if (st != AP_OK) return st;
    if (q_heads == 0 || q_heads % cache->kv_heads) return AP_ERR_INVALID;
    st = plan_of(cache, b, q_heads, window, sinks, &plan);
    if (st == AP_OK) *bytes = plan.bytes;
    return st;
}

ap_status ap_attention(const ap_kv_cache* cache, const ap_seq_batch* batch, const ap_rows* q, const ap_rows* out, uint32_t q_heads, float scale,
                       uint32_t window, uint32_t sinks, void* workspace, uint64_t workspace_bytes, void* stream) {
    AttnParams p{};
    Plan plan;
    ap_status st = take_cache(cache, &p.cache);
    if (st == AP_OK) st = take_batch(cache, batch, &p.batch);
    if (st == AP_OK) st = take_rows(q, &p.q);
    if (st == AP_OK) st = take_rows(out, &p.out);
    if (st != AP_OK) return st;
    const float scale_log2 = scale * 1.44269504088896341f;
    if (q_heads == 0 || q_heads % cache->kv_heads || !(scale > 0.0f) || !std::isfinite(scale_log2)) return AP_ERR_INVALID;
    st = plan_of(cache, p.batch, q_heads, window, sinks, &plan);
    if (st != AP_OK) return st;
    if (plan.bytes > 0 && (!workspace || !multiple(workspace, 16) || workspace_bytes < plan.bytes)) return AP_ERR_INVALID;
    if (batch->n_tokens == 0) return AP_OK;
    p.q_heads = q_heads, p.kv_heads = cache->kv_heads, p.group = q_heads / cache->kv_heads;
    divider(p.group, &p.group_magic, &p.group_shift);
    p.window = window, p.sinks = window ? sinks : 0;
    p.scale_log2 = scale_log2;
    p.few_rows = plan.few ? plan.few_rows : 0, p.few_stride = plan.few_stride;
    p.few_waves = plan.few_groups * kLineWaves, p.few_least = kFewLeast, p.many_chunk = plan.many_chunk;
    char* space = (char*)workspace;
    p.few_plan = plan.plan_bytes ? (uint32_t*)space : nullptr;
    p.few_o = (float*)(space + plan.plan_bytes), p.many_o = p.few_o + plan.few_n * cache->head_dim;
    p.few_ml = (f32x2*)(p.many_o + plan.many_n * cache->head_dim), p.many_ml = p.few_ml + plan.few_n;
    const hipStream_t on = (hipStream_t)stream;
    for_cache(cache, [&](auto e, auto d, auto b) {
        using E = decltype(e);
        if (plan.few) {
            auto kernel = plan.few_team ? (plan.few_tiles == 1 ? k_attend_few<E, d(), b(), 1, true> : k_attend_few<E, d(), b(), 2, true>)
                                        : (plan.few_tiles == 1 ? k_attend_few<E, d(), b(), 1, false> : k_attend_few<E, d(), b(), 2, false>);
            const uint32_t waves = !plan.few_team ? kLineWaves : plan.few_tiles == 1 ? kFewWaves<d(), b(), 1, true> : kFewWaves<d(), b(), 2, true>;
            for (uint32_t s = 0; s < batch->n_seqs; s += kFewSeqs) {    // so many sequences a launch, one launch after the other in one workspace
                AttnParams x = p;
                x.batch.n_seqs = std::min(kFewSeqs, batch->n_seqs - s);
                x.batch.first += s, x.batch.kv_len += s, x.batch.table += (int64_t)s * p.batch.table_stride;
                const uint32_t pairs = x.batch.n_seqs * p.kv_heads;
                hipLaunchKernelGGL(kernel, dim3(plan.few_team ? pairs : plan.few_groups), dim3(waves * kLanes), 0, on, x);
                if (p.few_plan) hipLaunchKernelGGL((k_join_few<E, d()>), dim3((pairs * plan.few_stride + 3) / 4), dim3(256), 0, on, x);
            }
        }
        if (plan.many) {
            hipLaunchKernelGGL((k_attend_many<E, d(), b()>), dim3(plan.row_tiles * cache->kv_heads * plan.many_chunks), dim3(kManyThreads), 0, on, p,
                               plan.row_tiles, plan.many_chunks);
            if (plan.many_chunks > 1) hipLaunchKernelGGL((k_join_many<E, d()>), dim3(batch->n_tokens * ((q_heads + 3) / 4)), dim3(256), 0, on, p);
        }
    });
    return launched();
}

}  // extern "C"
