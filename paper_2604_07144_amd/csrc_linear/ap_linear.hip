// C ABI of the operators on weights in 4 bits and of log probabilities: checks of arguments, choice of kernels and grids.
#include <algorithm>

#include "../csrc_attn/at_host.hpp"
#include "li_few.hpp"
#include "li_logprobs.hpp"
#include "li_many.hpp"
#include "li_pack.hpp"

namespace {

uint32_t tiles_of(uint64_t n, uint64_t tile) { return (uint32_t)((n + tile - 1) / tile); }

ap_status take_weights(const ap_weights* w, Weights* out) {
    if (!w || w->dtype > AP_FP16 || (w->group != 32 && w->group != 64 && w->group != 128)) return AP_ERR_INVALID;
    if (w->n_out == 0 || w->n_in == 0 || w->n_in % 8 || !w->codes || !w->pairs) return AP_ERR_INVALID;
    const int64_t n = 4 * kBlock / w->group;
    if (!multiple(w->codes, 16) || !stride_ok(w->code_stride, 16) || !multiple(w->pairs, n) || !stride_ok(w->pair_stride, n)) return AP_ERR_INVALID;
    if (w->n_out >= kMost || w->n_in >= kMost || (uint64_t)w->n_out * tiles_of(w->n_in, kBlock) >= kMost) return AP_ERR_RANGE;
    *out = Weights{(char*)w->codes, (char*)w->pairs, w->code_stride, w->pair_stride, w->n_out, w->n_in, tiles_of(w->n_in, kBlock)};
    return AP_OK;
}

ap_status take_vectors(const ap_vectors* v, uint32_t align, char** data, int64_t* stride) {
    if (!v || !v->data || !multiple(v->data, align) || !stride_ok(v->stride, align)) return AP_ERR_INVALID;
    *data = (char*)v->data, *stride = v->stride;
    return AP_OK;
}

// Rows that are written have to be apart: what two of them write to one place would go by timing.
bool apart(int64_t stride, uint64_t bytes, uint32_t n) { return n <= 1 || (uint64_t)stride >= bytes; }

template <typename F> void for_type(uint32_t dtype, F f) { dtype == AP_BF16 ? f(bf16{}) : f(fp16{}); }
template <typename F> void for_group(uint32_t g, F f) {
    if (g == 32) f(std::integral_constant<uint32_t, 32>{});
    else if (g == 64) f(std::integral_constant<uint32_t, 64>{});
    else f(std::integral_constant<uint32_t, 128>{});
}

ap_status pack_params(const ap_weights* weights, const ap_vectors* values, PackParams* p, dim3* grid) {
    char* data = nullptr;
    ap_status st = take_weights(weights, &p->w);
    if (st == AP_OK) st = take_vectors(values, 16, &data, &p->stride);
    if (st != AP_OK) return st;
    p->values = data;
    divider(p->w.blocks, &p->magic, &p->shift);
    const uint64_t groups = ((uint64_t)p->w.n_out * p->w.blocks + kPackThreads / 16 * kPackUnits - 1) / (kPackThreads / 16 * kPackUnits);
    if (groups >= kMostGroups) return AP_ERR_RANGE;
    *grid = dim3((uint32_t)groups);
    return AP_OK;
}

struct LinearPlan {
    bool many, held;
    uint32_t tokens;                                // of a workgroup
    uint32_t part_blocks, n_parts;
    uint32_t n_outs, n_tokens;                      // workgroups over the outputs and tokens
    uint64_t bytes;
};

constexpr uint32_t kCus = 256;

// Times beside the choices below are us a call, of calls in a graph with weights that come from memory.

// Up to kMostFew tokens go to the kernel of few rows, whose workgroup has all of them and 128 outputs or fewer; the other one's has
// 512 outputs.  64 tokens, few / many, bf16, groups of 128: 4096 outputs of 4096 inputs 15.2 / 19.7, 4096 of 14336 25 / 31, 10240 of 8192
// 31 / 34, gated 14336 of 4096 36 / 40.  (Other numbers of tokens and small groups were not compared.)
constexpr uint32_t kMostFew = 64;

// Estimates of the kernel of many rows, us: what a workgroup's step of 128 columns takes besides its tiles of 16 tokens and for each
// of them, what comes before the first and after the last step, what a second launch costs, and bytes of parts that are written and read a us.
// Expected / measured, groups of 128: 65, 100 tokens, 4096 outputs of 4096 inputs 24 / 20, 27 / 21; 128, 14336 of 4096 44 / 36; 331, 5120 of 13824
// 83 / 81; gated 14336 of 4096, 2048 tokens 530 / 521, 4999 1206 / 1120.  The terms are those of groups of 128: gated 14336 of 4096, 2048 tokens,
// groups of 64 and 32, 530 / 635 and 535 / 806.  And kEnterUs is more than a single tile takes to begin and to end (5): with 5 that product, in
// groups of 128, gets tiles of 64 for 96 and took 579 for 539; a round of workgroups that is not full, or not in step, has no term of its own.
constexpr double kStepUs = 0.3, kTileUs = 0.46, kEnterUs = 8, kJoinUs = 4, kPartBytesPerUs = 4e6;

ap_status linear_plan(const Weights& w, uint32_t n_tokens, uint32_t group, bool gated, LinearPlan* out) {
    LinearPlan r{};
    if (n_tokens >= kMost) return AP_ERR_RANGE;
    const uint64_t tiles = (uint64_t)tiles_of(w.n_out, 16) * (gated ? 2 : 1), sums = (uint64_t)n_tokens * w.n_out * (gated ? 2 : 1);
    r.many = n_tokens > kMostFew;
    uint32_t parts = 1;
    if (r.many) {
        // Tiles of 64, 96 or 112 tokens (small groups, whose pairs and sums leave fewer registers, up to 64 and 96), and the inputs in as many
        // parts, as the estimate likes best: little in the tiles that is no token, workgroups that fill the chip in whole rounds, few parts
        // to write and read.
        r.n_outs = tiles_of(tiles, kManyTiles * kManyWaves);
        double least = -1;
        for (const uint32_t tokens : {112u, 96u, 64u}) {
            if (tokens > (group == 32 ? 64 : group == 64 ? 96 : 112)) continue;
            const double step_us = kStepUs + kTileUs * (tokens / 16);
            for (uint32_t n = 1; n == 1 || (n <= 32 && n <= w.blocks && sums < 256 * kMostGroups); ++n) {
                const uint64_t rounds = ((uint64_t)r.n_outs * tiles_of(n_tokens, tokens) * n + kCus - 1) / kCus;
                const double us = rounds * (tiles_of(w.blocks, n) * step_us + kEnterUs) + (n > 1 ? kJoinUs + 8.0 * n * sums / kPartBytesPerUs : 0.0);
                if (least < 0 || us < least) least = us, parts = n, r.tokens = tokens;
            }
        }
        r.n_tokens = tiles_of(n_tokens, r.tokens);
    } else {
        r.tokens = n_tokens <= 4 ? 4 : n_tokens <= 8 ? 8 : n_tokens <= 16 ? 16 : n_tokens <= 32 ? 32 : 64;
        const uint32_t aside = r.tokens <= 16 ? (gated ? 2 : 1) : r.tokens / 8;
        r.n_outs = tiles_of(tiles, aside), r.n_tokens = 1;
        // With few outputs as many parts as fill the chip, of four steps of 16 wavefronts each at least, which are eight of the 8 wavefronts that
        // 5 to 16 tokens have (16 tokens, 2048 outputs of 14336 inputs stay one part, 11.0): 64 tokens, 4096 outputs of 14336 inputs in 1, 3
        // and 8 parts 94, 41 and 26; 10240 of 8192 in 1, 2 and 3 56, 37 and 32.  Where a workgroup has few tokens it has its outputs in
        // several tiles one after another, and no more workgroups are started than there are CUs.
        parts = std::max<uint32_t>(1, std::min(kCus / std::min(kCus, r.n_outs), w.blocks * aside / 64));
        if (r.tokens <= 16) r.n_outs = std::min(r.n_outs, kCus);
        // From three tiles on x is brought to LDS once, where it fits, and not with each.  Brought with each / once: gated 14336 of 4096, 1, 4
        // and 8 tokens 20.3 / 18.4, 20.2 / 18.2, 23.5 / 21.4; 128256 of 4096, 8 tokens 85 / 74; two tiles (6144 of 4096), 1 and 8 tokens 6.6 / 7.1
        // and 7.6 / 7.4; one tile (4096 of 4096) 4.8 / 5.4 and 5.4 / 5.7.
        r.held = r.tokens <= 8 && (uint64_t)tiles_of(w.blocks, parts) * r.tokens * 256 <= kHeldBytes && tiles > 2ull * kCus * aside;
    }
    r.part_blocks = tiles_of(w.blocks, parts), r.n_parts = tiles_of(w.blocks, r.part_blocks);
    if ((uint64_t)r.n_outs * r.n_tokens * r.n_parts >= kMostGroups / 4) return AP_ERR_RANGE;
    if (r.n_parts > 1) r.bytes = 4ull * r.n_parts * sums;
    *out = r;
    return AP_OK;
}

template <uint32_t... N, typename F> void for_one_of(uint32_t n, F f) { ((n == N ? f(std::integral_constant<uint32_t, N>{}) : void()), ...); }
template <typename F> void for_truth(bool b, F f) { b ? f(std::true_type{}) : f(std::false_type{}); }

ap_status run_linear(LinearParams p, const LinearPlan& plan, uint32_t dtype, uint32_t group, bool gated, void* workspace, hipStream_t on) {
    p.parts = (float*)workspace, p.part_blocks = plan.part_blocks, p.n_parts = plan.n_parts;
    for_type(dtype, [&](auto e) {
        for_group(group, [&](auto g) {
            for_truth(gated, [&](auto gates) {
                for_truth(p.w[0].n_in % kBlock == 0, [&](auto whole) {
                    using E = decltype(e);
                    if (plan.many) {
                        auto go = [&](auto tiles) {
                            hipLaunchKernelGGL((k_linear_many<E, g(), tiles(), gates(), whole()>), dim3(plan.n_outs * plan.n_tokens * plan.n_parts), dim3(kManyWaves * kLanes), 0,
                                               on, p, plan.n_outs, plan.n_tokens);
                        };
                        if (plan.tokens == 64) go(std::integral_constant<uint32_t, 4>{});
                        else if constexpr (g() == 64) go(std::integral_constant<uint32_t, 6>{});
                        else if constexpr (g() == 128) plan.tokens == 96 ? go(std::integral_constant<uint32_t, 6>{}) : go(std::integral_constant<uint32_t, 7>{});
                        return;
                    }
                    for_one_of<4, 8, 16, 32, 64>(plan.tokens, [&](auto t) {
                        for_truth(plan.held, [&](auto held) {
                            if constexpr (!held() || t() <= 8)
                                hipLaunchKernelGGL((k_linear_few<E, g(), t(), gates(), held(), whole()>), dim3(plan.n_outs, 1, plan.n_parts),
                                                   dim3(FewShape<g(), t(), gates(), held()>::kWaves * kLanes), 0, on, p);
                        });
                    });
                });
            });
        });
        if (plan.n_parts > 1) {
            auto join = gated ? k_join_parts<decltype(e), true> : k_join_parts<decltype(e), false>;
            hipLaunchKernelGGL(join, dim3(tiles_of((uint64_t)p.n_tokens * tiles_of(p.w[0].n_out, 4), 256)), dim3(256), 0, on, p);
        }
    });
    return launched();
}

bool space_ok(const void* workspace, uint64_t bytes, uint64_t need) { return need == 0 || (workspace && multiple(workspace, 16) && bytes >= need); }

constexpr uint32_t kMostPieces = 16;
struct LogPlan {
    uint32_t pieces, piece;
    uint64_t bytes;
};

ap_status take_logits(const ap_logits* x, uint32_t top, LogPlan* out) {
    if (!x || x->dtype > AP_FP32 || !x->data || x->vocab == 0 || top > kMostTop) return AP_ERR_INVALID;
    const uint32_t size = x->dtype == AP_FP32 ? 4 : 2;
    if (!multiple(x->data, size) || !stride_ok(x->stride, size)) return AP_ERR_INVALID;
    if (x->vocab >= kMost || x->n_rows >= kMost) return AP_ERR_RANGE;
    LogPlan r{};
    // Few rows are cut into pieces of whole spans of a workgroup, so that 1024 workgroups have something to do.
    const uint32_t units = tiles_of(x->vocab, kLogWaves * kSpan), groups = 1024 / std::min<uint32_t>(1024, std::max<uint32_t>(1, x->n_rows));
    r.piece = tiles_of(units, std::max<uint32_t>(1, std::min(std::min(groups, units), kMostPieces))) * kLogWaves * kSpan;
    r.pieces = tiles_of(x->vocab, r.piece);
    if ((uint64_t)x->n_rows * r.pieces >= kMostGroups) return AP_ERR_RANGE;
    if (r.pieces > 1) r.bytes = (uint64_t)x->n_rows * r.pieces * (16 + 8ull * top);
    *out = r;
    return AP_OK;
}

template <typename F> void for_logits(uint32_t dtype, F f) {
    if (dtype == AP_FP32) f(float{});
    else for_type(dtype, f);
}

}  // namespace

extern "C" {

ap_status ap_weights_pack(const ap_weights* weights, const ap_vectors* values, void* stream) {
    PackParams p{};
    dim3 grid;
    const ap_status st = pack_params(weights, values, &p, &grid);
    if (st != AP_OK) return st;
    const uint64_t codes = (uint64_t)p.w.blocks * (kBlock / 2), pairs = (uint64_t)p.w.blocks * (4 * kBlock / weights->group);
    if (!apart(p.w.code_stride, codes, p.w.n_out) || !apart(p.w.pair_stride, pairs, p.w.n_out)) return AP_ERR_INVALID;
    for_type(weights->dtype, [&](auto e) {
        for_group(weights->group, [&](auto g) { hipLaunchKernelGGL((k_pack<decltype(e), g()>), grid, dim3(kPackThreads), 0, (hipStream_t)stream, p); });
    });
    return launched();
}

ap_status ap_weights_read(const ap_weights* weights, const ap_vectors* values, void* stream) {
    PackParams p{};
    dim3 grid;
    const ap_status st = pack_params(weights, values, &p, &grid);
    if (st != AP_OK) return st;
    if (!apart(p.stride, 2ull * p.w.n_in, p.w.n_out)) return AP_ERR_INVALID;
    for_type(weights->dtype, [&](auto e) {
        for_group(weights->group, [&](auto g) { hipLaunchKernelGGL((k_unpack<decltype(e), g()>), grid, dim3(kPackThreads), 0, (hipStream_t)stream, p); });
    });
    return launched();
}

ap_status ap_linear_workspace(const ap_weights* weights, uint32_t n_tokens, uint64_t* bytes) {
    Weights w;
    LinearPlan plan;
    if (!bytes) return AP_ERR_INVALID;
    ap_status st = take_weights(weights, &w);
    if (st == AP_OK) st = linear_plan(w, n_tokens, weights->group, false, &plan);
    if (st == AP_OK) *bytes = plan.bytes;
    return st;
}

ap_status ap_linear(const ap_weights* weights, const ap_vectors* x, const ap_vectors* add, const ap_vectors* y, uint32_t n_tokens,
                    void* workspace, uint64_t workspace_bytes, void* stream) {
    LinearParams p{};
    LinearPlan plan;
    char *xs = nullptr, *adds = nullptr;
    ap_status st = take_weights(weights, &p.w[0]);
    if (st == AP_OK) st = take_vectors(x, 16, &xs, &p.x_stride);
    if (st == AP_OK && add) st = take_vectors(add, 2, &adds, &p.add_stride);
    if (st == AP_OK) st = take_vectors(y, 2, &p.y, &p.y_stride);
    if (st == AP_OK) st = linear_plan(p.w[0], n_tokens, weights->group, false, &plan);
    if (st != AP_OK) return st;
    if (!apart(p.y_stride, 2ull * p.w[0].n_out, n_tokens) || !space_ok(workspace, workspace_bytes, plan.bytes)) return AP_ERR_INVALID;
    if (n_tokens == 0) return AP_OK;
    p.x = xs, p.add = adds, p.n_tokens = n_tokens;
    return run_linear(p, plan, weights->dtype, weights->group, false, workspace, (hipStream_t)stream);
}

ap_status ap_gated_workspace(const ap_weights* gate, const ap_weights* up, uint32_t n_tokens, uint64_t* bytes) {
    Weights g, u;
    LinearPlan plan;
    if (!bytes) return AP_ERR_INVALID;
    ap_status st = take_weights(gate, &g);
    if (st == AP_OK) st = take_weights(up, &u);
    if (st != AP_OK) return st;
    if (gate->dtype != up->dtype || gate->group != up->group || g.n_out != u.n_out || g.n_in != u.n_in) return AP_ERR_INVALID;
    st = linear_plan(g, n_tokens, gate->group, true, &plan);
    if (st == AP_OK) *bytes = plan.bytes;
    return st;
}

ap_status ap_gated(const ap_weights* gate, const ap_weights* up, const ap_vectors* x, const ap_vectors* h, uint32_t n_tokens, uint32_t act,
                   void* workspace, uint64_t workspace_bytes, void* stream) {
    LinearParams p{};
    LinearPlan plan;
    char* xs = nullptr;
    ap_status st = take_weights(gate, &p.w[0]);
    if (st == AP_OK) st = take_weights(up, &p.w[1]);
    if (st == AP_OK) st = take_vectors(x, 16, &xs, &p.x_stride);
    if (st == AP_OK) st = take_vectors(h, 2, &p.y, &p.y_stride);
    if (st != AP_OK) return st;
    if (gate->dtype != up->dtype || gate->group != up->group || p.w[0].n_out != p.w[1].n_out || p.w[0].n_in != p.w[1].n_in || act > AP_GELU) return AP_ERR_INVALID;
    st = linear_plan(p.w[0], n_tokens, gate->group, true, &plan);
    if (st != AP_OK) return st;
    if (!apart(p.y_stride, 2ull * p.w[0].n_out, n_tokens) || !space_ok(workspace, workspace_bytes, plan.bytes)) return AP_ERR_INVALID;
    if (n_tokens == 0) return AP_OK;
    p.x = xs, p.n_tokens = n_tokens, p.act = act;
    return run_linear(p, plan, gate->dtype, gate->group, true, workspace, (hipStream_t)stream);
}

ap_status ap_logprobs_workspace(const ap_logits* logits, uint32_t top, uint64_t* bytes) {
    LogPlan plan;
    if (!bytes) return AP_ERR_INVALID;
    const ap_status st = take_logits(logits, top, &plan);
    if (st == AP_OK) *bytes = plan.bytes;
    return st;
}

ap_status ap_logprobs(const ap_logits* logits, const int32_t* tokens, float scale, uint32_t top, float* logprob, float* entropy,
                      int32_t* top_id, float* top_logprob, void* workspace, uint64_t workspace_bytes, void* stream) {
    LogPlan plan;
    const ap_status st = take_logits(logits, top, &plan);
    if (st != AP_OK) return st;
    if (!(scale * kLog2e >= kLeastScale) || !std::isfinite(scale * kLog2e) || (tokens == nullptr) != (logprob == nullptr) || (top && (!top_id || !top_logprob))) return AP_ERR_INVALID;
    if (!multiple(tokens, 4) || !multiple(logprob, 4) || !multiple(entropy, 4) || (top && (!multiple(top_id, 4) || !multiple(top_logprob, 4)))) return AP_ERR_INVALID;
    if (!space_ok(workspace, workspace_bytes, plan.bytes)) return AP_ERR_INVALID;
    if (logits->n_rows == 0) return AP_OK;
    LogParams p{};
    p.logits = (const char*)logits->data, p.stride = logits->stride, p.n_rows = logits->n_rows, p.vocab = logits->vocab;
    p.top = top, p.pieces = plan.pieces, p.piece = plan.piece;
    p.c = scale * kLog2e, p.scale = scale, p.beyond_c = p.scale / (p.c * kLn2) - 1.0;
    p.tokens = tokens, p.logprob = logprob, p.entropy = entropy, p.top_logprob = top_logprob, p.top_id = top_id;
    p.part_sums = (Sums*)workspace, p.part_keys = (uint64_t*)((char*)workspace + (uint64_t)p.n_rows * p.pieces * 16);
    for_logits(logits->dtype, [&](auto e) {
        using E = decltype(e);
        hipLaunchKernelGGL((k_logprobs<E>), dim3(p.n_rows * p.pieces), dim3(kLogThreads), 0, (hipStream_t)stream, p);
        // A wavefront for each piece, or four: 500 rows of 32000 in two pieces, 16 / 4 wavefronts 24.7 / 21.8 us; 8 rows of 128256 in 16 11.9 / 12.5.
        if (p.pieces > 4) hipLaunchKernelGGL((k_join_logprobs<E, 16>), dim3(p.n_rows), dim3(16 * kLanes), 0, (hipStream_t)stream, p);
        else if (p.pieces > 1) hipLaunchKernelGGL((k_join_logprobs<E, 4>), dim3(p.n_rows), dim3(4 * kLanes), 0, (hipStream_t)stream, p);
    });
    return launched();
}

}  // extern "C"
