// Entry points that norm and rotate heads, on their way into the cache or alone: argument checks and launches.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <string>

#include "append.h"
#include "attention_checks.h"

namespace gorgo {
namespace {

constexpr int64_t MOST_STRIDE = (int64_t)1 << 40;

int take_rotation(const gorgo_rotation* r, const gorgo_kv_batch* b, int32_t d, RotationArgs* out) {
    if (!r) return GORGO_OK;
    if (r->pairs < 1 || r->pairs > d / 2) return bad("rotation.pairs must be in 1..head_dim / 2");
    if (r->layout != GORGO_PAIRS_HALVES && r->layout != GORGO_PAIRS_NEIGHBOURS) return bad("rotation.layout must be 0 (halves) or 1 (neighbours)");
    if (r->axes < 1 || r->axes > 4) return bad("rotation.axes must be in 1..4");
    if (!r->frequencies || reinterpret_cast<uintptr_t>(r->frequencies) % 8) return bad("rotation.frequencies must be an 8-byte aligned array");
    if (reinterpret_cast<uintptr_t>(r->positions) % 4) return bad("rotation.positions must be 4-byte aligned");
    if (!r->positions && r->axes != 1 && b->tokens != 0) return bad("a rotation of several axes needs positions");
    if (!r->positions && b->sequences == 0 && b->tokens != 0) return bad("tokens of no sequence need rotation.positions");
    if (r->axis_stride < 0 || r->axis_stride > MOST_STRIDE) return bad("rotation.axis_stride must be in 0..2^40");
    if (!std::isfinite(r->magnitude)) return fail(GORGO_ERR_NONFINITE, "rotation.magnitude must be finite");
    for (int32_t i = 0; i < r->pairs; ++i) {
        if (r->axis_of_pair[i] >= r->axes) return bad("rotation.axis_of_pair must be below rotation.axes");
        out->axis_low |= (uint64_t)(r->axis_of_pair[i] & 1) << i;
        out->axis_high |= (uint64_t)(r->axis_of_pair[i] >> 1) << i;
    }
    out->frequencies = r->frequencies;
    out->positions = r->positions;
    out->axis_stride = r->axis_stride;
    out->magnitude = r->magnitude;
    out->pairs = r->pairs;
    out->neighbours = r->layout == GORGO_PAIRS_NEIGHBOURS;
    return GORGO_OK;
}

int take_norm(const gorgo_norm* n, const char* name, NormArgs* out) {
    if (!n) return GORGO_OK;
    if (!std::isfinite(n->eps) || n->eps <= 0.0f) return fail(GORGO_ERR_NONFINITE, std::string(name) + ".eps must be > 0 and finite");
    if (!aligned16(n->weight)) return bad(std::string(name) + ".weight must be 16-byte aligned");
    if (n->head_stride < 0 || n->head_stride > MOST_STRIDE || n->head_stride % 4) return bad(std::string(name) + ".head_stride must be a multiple of 4 in 0..2^40");
    out->weight = n->weight;
    out->head_stride = n->weight ? n->head_stride : 0;
    out->eps = n->eps;
    return GORGO_OK;
}

// Tokens of a workgroup, which share the look-ups of their places: 8 at most (16: 50,000 rows of 16 heads of 80 54.0 instead of 51.2 us; 4: 55.2), fewer where
// compute units would get less than four (3,747 rows of 12 heads of 72: 8.2 us, with two each 10.3).  And workgroups that share a block's rows, 32 each, where
// there are less than compute units (8 tokens of 32/8 heads of 128 in a captured graph: 4.0 us, 5.0 in one workgroup each; of 128/8 heads 4.1 and 8.2).
void deal(AppendArgs* a) {
    a->one_over_d = 1.0f / (float)a->cache.d;
    while ((1 << a->pair_bits) < a->rotation.pairs) ++a->pair_bits;
    const int32_t rows = a->q_heads.divisor + 2 * a->kv_heads.divisor;
    a->block = std::min(MOST_BLOCK, std::max(1, a->batch.tokens / (4 * COMPUTE_UNITS)));
    a->parts = std::min(std::max(1, COMPUTE_UNITS / std::max(1, a->batch.tokens)), (rows + 31) / 32);
}

}  // namespace
}  // namespace gorgo

using namespace gorgo;

extern "C" {

int gorgo_kv_append(const gorgo_kv_cache* cache, const gorgo_kv_batch* batch, const gorgo_rotation* rotation, const gorgo_norm* q_norm,
                    const gorgo_norm* k_norm, int32_t q_heads, const gorgo_kv_rows* q, const gorgo_kv_rows* q_out, const gorgo_kv_rows* k,
                    const gorgo_kv_rows* v, void* hip_stream) {
    clear_error();
    AppendArgs a;
    std::memset(static_cast<void*>(&a), 0, sizeof a);
    int rc = take_cache(cache, &a.cache);
    if (rc || (rc = take_batch(batch, cache, &a.batch)) || (rc = take_rotation(rotation, batch, cache->head_dim, &a.rotation)) ||
        (rc = take_norm(k_norm, "k_norm", &a.k_norm)) || (rc = take_rows(k, a.batch.tokens, "k", &a.k)) || (rc = take_rows(v, a.batch.tokens, "v", &a.v)))
        return rc;
    if (q_heads < 0 || q_heads > 4096) return bad("q_heads must be in 0..4096");
    if (q_heads > 0) {
        if ((rc = take_norm(q_norm, "q_norm", &a.q_norm)) || (rc = take_rows(q, a.batch.tokens, "q", &a.q)) ||
            (rc = take_rows(q_out, a.batch.tokens, "q_out", &a.q_out)))
            return rc;
        a.q_heads = divider(q_heads);
    }
    a.kv_heads = divider(cache->kv_heads);
    deal(&a);
    return a.batch.tokens == 0 ? GORGO_OK : launch_append(a, cache->type, hip_stream);
}

int gorgo_rotate_heads(const gorgo_kv_batch* batch, const gorgo_rotation* rotation, const gorgo_norm* norm, int32_t type, int32_t heads,
                       int32_t head_dim, const gorgo_kv_rows* x, const gorgo_kv_rows* out, void* hip_stream) {
    clear_error();
    AppendArgs a;
    std::memset(static_cast<void*>(&a), 0, sizeof a);
    if (!batch) return bad("batch is NULL");
    if (type != GORGO_KV_BF16 && type != GORGO_KV_F16) return bad("type must be 0 (bf16) or 1 (fp16)");
    if (heads < 1 || heads > 4096) return bad("heads must be in 1..4096");
    if (head_dim < 8 || head_dim > MAX_HEAD || head_dim % 8) return bad("head_dim must be a multiple of 8 in 8.." + std::to_string(MAX_HEAD));
    if (!rotation && !norm) return bad("neither rotation nor norm is given");
    if (batch->sequences < 0 || batch->sequences > (1 << 16)) return bad("batch.sequences must be in 0..2^16");
    if (batch->tokens < 0 || batch->tokens > (1 << 24)) return bad("batch.tokens must be in 0..2^24");
    if (batch->sequences > 0) {
        if (!batch->token_offsets && batch->tokens != batch->sequences) return bad("without token_offsets batch.tokens must equal batch.sequences");
        if (!batch->lengths) return bad("batch.lengths is NULL");
        a.batch.first = batch->token_offsets;
        a.batch.lengths = batch->lengths;
    }
    a.batch.S = batch->sequences;
    a.batch.tokens = batch->tokens;
    int rc = take_rotation(rotation, batch, head_dim, &a.rotation);
    if (rc || (rc = take_norm(norm, "norm", &a.q_norm)) || (rc = take_rows(x, batch->tokens, "x", &a.q)) || (rc = take_rows(out, batch->tokens, "out", &a.q_out)))
        return rc;
    a.cache.d = head_dim;
    a.q_heads = divider(heads);
    deal(&a);
    return batch->tokens == 0 ? GORGO_OK : launch_append(a, type, hip_stream);
}

}  // extern "C"
