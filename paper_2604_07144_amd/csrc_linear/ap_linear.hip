// C ABI of the operators on weights in 4 bits and of log probabilities: checks of arguments, choice of kernels and grids.
#include <algorithm>

#include "li_few.hpp"
#include "li_logprobs.hpp"
#include "li_pack.hpp"

namespace {

constexpr uint64_t kMost = 1ull << 31;              // rows, columns and blocks stay below
constexpr uint64_t kMostGroups = 1ull << 24;        // and workgroups (of 256 threads: a grid holds less than 2^32)

bool multiple(const void* p, uint64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool stride_ok(int64_t s, int64_t n) { return s >= 0 && s % n == 0; }
uint32_t tiles_of(uint64_t n, uint32_t tile) { return (uint32_t)((n + tile - 1) / tile); }

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

template <typename F> void for_type(uint32_t dtype, F f) { dtype == AP_BF16 ? f(bf16{}) : f(fp16{}); }
template <typename F> void for_group(uint32_t g, F f) {
    if (g == 32) f(std::integral_constant<uint32_t, 32>{});
    else if (g == 64) f(std::integral_constant<uint32_t, 64>{});
    else f(std::integral_constant<uint32_t, 128>{});
}

ap_status launched() { return hipGetLastError() == hipSuccess ? AP_OK : AP_ERR_DEVICE; }

// magic and shift of a division of numbers below 2^31 by `d`: n / d = ((2 n) * magic >> 32) >> shift
void divider(uint32_t d, uint32_t* magic, uint32_t* shift) {
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    *shift = l;
    *magic = (uint32_t)(((1ull << (31 + l)) + d - 1) / d);
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
    uint32_t token_tiles;
    dim3 grid;
    uint64_t bytes;
};

constexpr uint32_t kFewOuts = 2;                    // tiles of outputs of a workgroup

ap_status linear_plan(const Weights& w, uint32_t n_tokens, bool gated, LinearPlan* out) {
    LinearPlan r{};
    if (n_tokens >= kMost) return AP_ERR_RANGE;
    r.token_tiles = n_tokens <= 16 ? 1 : n_tokens <= 32 ? 2 : 4;
    const uint64_t outs = tiles_of(w.n_out, (gated ? kFewOuts / 2 : kFewOuts) * 16), tokens = tiles_of(n_tokens, r.token_tiles * 16);
    if (outs >= kMostGroups / 2 || tokens >= 65536) return AP_ERR_RANGE;
    r.grid = dim3((uint32_t)outs, (uint32_t)tokens);
    *out = r;
    return AP_OK;
}

ap_status run_linear(const LinearParams& p, const LinearPlan& plan, uint32_t dtype, uint32_t group, bool gated, hipStream_t on) {
    for_type(dtype, [&](auto e) {
        for_group(group, [&](auto g) {
            using E = decltype(e);
            auto pick = [&](auto tt) { return gated ? k_linear_few<E, g(), kFewOuts, tt(), true> : k_linear_few<E, g(), kFewOuts, tt(), false>; };
            auto kernel = plan.token_tiles == 1 ? pick(std::integral_constant<uint32_t, 1>{}) : plan.token_tiles == 2 ? pick(std::integral_constant<uint32_t, 2>{})
                                                                                                                   : pick(std::integral_constant<uint32_t, 4>{});
            hipLaunchKernelGGL(kernel, plan.grid, dim3(kFewWaves * kLanes), 0, on, p);
        });
    });
    return launched();
}

bool space_ok(const void* workspace, uint64_t bytes, uint64_t need) { return need == 0 || (workspace && multiple(workspace, 16) && bytes >= need); }

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
    r.pieces = 1;
    while (r.pieces < 32 && (uint64_t)x->n_rows * r.pieces < 512 && x->vocab / r.pieces > 8192) r.pieces *= 2;
    r.piece = (tiles_of(x->vocab, r.pieces) + 7) / 8 * 8;
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
    if (st == AP_OK) st = linear_plan(w, n_tokens, false, &plan);
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
    if (st == AP_OK) st = linear_plan(p.w[0], n_tokens, false, &plan);
    if (st != AP_OK) return st;
    if (!space_ok(workspace, workspace_bytes, plan.bytes)) return AP_ERR_INVALID;
    if (n_tokens == 0) return AP_OK;
    p.x = xs, p.add = adds, p.n_tokens = n_tokens;
    return run_linear(p, plan, weights->dtype, weights->group, false, (hipStream_t)stream);
}

ap_status ap_gated_workspace(const ap_weights* gate, const ap_weights* up, uint32_t n_tokens, uint64_t* bytes) {
    Weights g, u;
    LinearPlan plan;
    if (!bytes) return AP_ERR_INVALID;
    ap_status st = take_weights(gate, &g);
    if (st == AP_OK) st = take_weights(up, &u);
    if (st != AP_OK) return st;
    if (gate->dtype != up->dtype || gate->group != up->group || g.n_out != u.n_out || g.n_in != u.n_in) return AP_ERR_INVALID;
    st = linear_plan(g, n_tokens, true, &plan);
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
    st = linear_plan(p.w[0], n_tokens, true, &plan);
    if (st != AP_OK) return st;
    if (!space_ok(workspace, workspace_bytes, plan.bytes)) return AP_ERR_INVALID;
    if (n_tokens == 0) return AP_OK;
    p.x = xs, p.n_tokens = n_tokens, p.act = act;
    return run_linear(p, plan, gate->dtype, gate->group, true, (hipStream_t)stream);
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
    if (!(scale > 0.0f) || !std::isfinite(scale * kLog2e) || (tokens == nullptr) != (logprob == nullptr) || (top && (!top_id || !top_logprob))) return AP_ERR_INVALID;
    if (!multiple(tokens, 4) || !multiple(logprob, 4) || !multiple(entropy, 4) || (top && (!multiple(top_id, 4) || !multiple(top_logprob, 4)))) return AP_ERR_INVALID;
    if (!space_ok(workspace, workspace_bytes, plan.bytes)) return AP_ERR_INVALID;
    if (logits->n_rows == 0) return AP_OK;
    LogParams p{};
    p.logits = (const char*)logits->data, p.stride = logits->stride, p.n_rows = logits->n_rows, p.vocab = logits->vocab;
    p.top = top, p.pieces = plan.pieces, p.piece = plan.piece;
    p.tokens = tokens, p.scale = scale, p.logprob = logprob, p.entropy = entropy, p.top_logprob = top_logprob, p.top_id = top_id;
    p.part_sums = (f32x4*)workspace, p.part_keys = (uint64_t*)((char*)workspace + (uint64_t)p.n_rows * p.pieces * 16);
    for_logits(logits->dtype, [&](auto e) {
        using E = decltype(e);
        hipLaunchKernelGGL((k_logprobs<E>), dim3(p.n_rows * p.pieces), dim3(kLogThreads), 0, (hipStream_t)stream, p);
        if (p.pieces > 1) hipLaunchKernelGGL((k_join_logprobs<E>), dim3(p.n_rows), dim3(kLogThreads), 0, (hipStream_t)stream, p);
    });
    return launched();
}

}  // extern "C"
