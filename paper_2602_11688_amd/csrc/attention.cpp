// Entry points of the paged cache and the attention over it: argument checks, workspace, launches.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <string>

#include "attention.h"
#include "attention_checks.h"
#include "internal.h"

namespace gorgo {
namespace {

// Everything but the rows, the results and the workspace.
int take_attention(const gorgo_kv_cache* c, const gorgo_kv_batch* b, int32_t q_heads, AttendArgs* a) {
    std::memset(static_cast<void*>(a), 0, sizeof *a);
    int rc = take_cache(c, &a->cache);
    if (rc || (rc = take_batch(b, c, &a->batch))) return rc;
    if (q_heads < 1 || q_heads > 4096 || q_heads % c->kv_heads) return bad("q_heads must be a multiple of cache.kv_heads in 1..4096");
    const int32_t group = q_heads / c->kv_heads;
    if ((int64_t)b->tokens * group > 0x7fffffff - (1 << 21)) return bad("tokens times query heads of a cache head must be less than 2^31 - 2^21");
    // (workgroups of a launch times their threads stay below 2^32)
    if (((int64_t)b->tokens * group / PROMPT_ROWS + b->sequences) * c->kv_heads > (1 << 22))
        return bad("too many tokens, sequences and heads for one call: split the batch");
    a->q_heads = q_heads;
    a->group = divider(group);
    return GORGO_OK;
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

struct AttendPlan {
    int32_t tiles, splits;
    size_t workspace;                    // bytes, the counters at its beginning among them
};

int32_t padded(int32_t d) { return d <= 64 ? 64 : 128; }

// How many workgroups of attend_prompt_kernel the compute units hold at once, and the most pieces that the keys of a full table are worth.
int64_t prompt_groups(const AttendArgs& a) { return COMPUTE_UNITS * (padded(a.cache.d) == 64 && a.cache.page.divisor % PROMPT_KEYS == 0 ? 2 : 1); }
int64_t prompt_pieces(const AttendArgs& a, bool sinks) {
    int32_t tiles = a.batch.capacity / PROMPT_KEYS;
    // (with sinks: of a tile of rows' windows and of the sinks, which may both begin and end inside a tile)
    if (a.sinks) tiles = std::min(tiles, (int32_t)(((int64_t)a.window + PROMPT_ROWS) / PROMPT_KEYS) + a.sinks / PROMPT_KEYS + 3);
    return std::min<int64_t>(pieces_of(tiles, sinks), MOST_PIECES);
}
// Bytes of `rows` partial rows (each row in each of its pieces), behind the counts.
size_t prompt_bytes(const AttendArgs& a, int64_t rows) { return COUNTER_BYTES + (size_t)rows * (padded(a.cache.d) + 2) * 4; }

AttendPlan plan_prompt(const AttendArgs& a) {
    AttendPlan p;
    const int64_t rows = (int64_t)a.batch.tokens * a.group.divisor;
    p.tiles = (int32_t)(rows / PROMPT_ROWS) + a.batch.S;
    const int64_t full = rows / PROMPT_ROWS + std::min<int64_t>(a.batch.S, rows);
    const int64_t groups = std::max<int64_t>(1, full * a.cache.heads);
    // split where the tiles alone leave compute units idle, into as many workgroups as these hold at once (500 tokens of 32/8 heads of
    // 128 after 8,000: 85 us, with twice as many 98), 32 pieces at most (two times 30 tokens of 8 heads of one cache head after 30,000:
    // 88 us with 16, 58 with 32; 64 make 51 of it and a short call of 16 heads 1 % slower)
    const int64_t at_once = prompt_groups(a);
    p.splits = groups * 2 > at_once ? 1 : (int32_t)std::min<int64_t>(at_once / groups, prompt_pieces(a, a.sinks > 0));
    p.workspace = p.splits > 1 ? prompt_bytes(a, (int64_t)p.splits * a.batch.tokens * a.q_heads) : 0;
    return p;
}

// The most that plan_prompt asks for with at most these sequences, tokens and columns (few rows are split where many are not).  Pieces are
// at_once / groups at most, and groups are more than rows of a head / PROMPT_ROWS of each head: partial rows are less than at_once * PROMPT_ROWS.
size_t most_prompt_workspace(const AttendArgs& a) {
    const int64_t at_once = prompt_groups(a), pieces = prompt_pieces(a, true);      // (more of them than without sinks)
    if (pieces < 2 || a.cache.heads * 2 > at_once) return 0;
    return prompt_bytes(a, std::min(at_once * PROMPT_ROWS, pieces * a.batch.tokens * a.q_heads));
}

AttendPlan plan_token(const AttendArgs& a, int32_t type) {
    const int64_t UNIT = TOKEN_WAVES * token_keys(type == GORGO_KV_E4M3);
    AttendPlan p;
    p.tiles = 0;
    const int64_t units = (int64_t)a.batch.S * a.cache.heads * ((a.batch.capacity - 1) / UNIT + 1);
    p.splits = (int32_t)std::min<int64_t>(TOKEN_GROUPS, units);
    const size_t part = ((size_t)a.group.divisor * (padded(a.cache.d) + 2) + 3) & ~(size_t)3;
    p.workspace = COUNTER_BYTES + (size_t)p.splits * 2 * part * 4;
    return p;
}

// A token call of more query heads than its kernel holds side by side runs as a prompt of one token each.
bool token_suits(const AttendArgs& a) { return a.group.divisor <= TOKEN_ROWS; }

int attend(bool token, const gorgo_kv_cache* cache, const gorgo_kv_batch* batch, const gorgo_attention* how, const gorgo_kv_rows* q,
           const gorgo_kv_rows* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!how) return bad("attention is NULL");
    AttendArgs a;
    int rc = take_attention(cache, batch, how->q_heads, &a);
    if (rc) return rc;
    if (token && batch->token_offsets) return bad("gorgo_attend_token takes one token of each sequence: token_offsets must be NULL");
    const float scale_log2 = how->scale * 1.4426950408889634f;
    if (!std::isfinite(scale_log2) || how->scale <= 0.0f) return fail(GORGO_ERR_NONFINITE, "attention.scale must be > 0, and finite times log2(e)");
    if (how->window < 0) return bad("attention.window must be >= 0");
    if (how->sinks < 0) return bad("attention.sinks must be >= 0");
    if ((rc = take_rows(q, batch->tokens, "q", &a.q)) || (rc = take_rows(out, batch->tokens, "out", &a.out))) return rc;
    a.lse = lse;
    a.scale_log2 = scale_log2;
    a.window = how->window;
    a.sinks = how->window > 0 ? how->sinks : 0;      // (without a window all keys are seen)
    const bool by_token = token && token_suits(a);
    const AttendPlan p = by_token ? plan_token(a, cache->type) : plan_prompt(a);
    if (p.workspace > 0) {
        if (!workspace) return fail(GORGO_ERR_WORKSPACE, "workspace is NULL");
        if (reinterpret_cast<uintptr_t>(workspace) % 256) return fail(GORGO_ERR_WORKSPACE, "workspace must be 256-byte aligned");
        if (workspace_bytes < p.workspace)
            return fail(GORGO_ERR_WORKSPACE, "workspace has " + std::to_string(workspace_bytes) + " bytes, needs " + std::to_string(p.workspace));
    }
    if (batch->tokens == 0) return GORGO_OK;
    a.tiles = p.tiles;
    a.splits = p.splits;
    a.counters = static_cast<uint32_t*>(workspace);
    a.partial = p.workspace > 0 ? reinterpret_cast<float*>(static_cast<char*>(workspace) + COUNTER_BYTES) : nullptr;
    return by_token ? launch_attend_token(a, cache->type, stream) : launch_attend_prompt(a, cache->type, stream);
}

}  // namespace
}  // namespace gorgo

using namespace gorgo;

extern "C" {

int gorgo_kv_write(const gorgo_kv_cache* cache, const gorgo_kv_batch* batch, const gorgo_kv_rows* k, const gorgo_kv_rows* v, void* hip_stream) {
    clear_error();
    CacheArgs c;
    BatchArgs b;
    RowsArgs rk, rv;
    int rc = take_cache(cache, &c);
    if (rc || (rc = take_batch(batch, cache, &b)) || (rc = take_rows(k, b.tokens, "k", &rk)) || (rc = take_rows(v, b.tokens, "v", &rv))) return rc;
    return b.tokens == 0 ? GORGO_OK : launch_kv_write(c, b, rk, rv, cache->type, hip_stream);
}

int gorgo_kv_read(const gorgo_kv_cache* cache, const gorgo_kv_batch* batch, const gorgo_kv_rows* k, const gorgo_kv_rows* v, void* hip_stream) {
    clear_error();
    CacheArgs c;
    BatchArgs b;
    RowsArgs rk, rv;
    int rc = take_cache(cache, &c);
    if (rc || (rc = take_batch(batch, cache, &b)) || (rc = take_rows(k, b.tokens, "k", &rk)) || (rc = take_rows(v, b.tokens, "v", &rv))) return rc;
    return b.tokens == 0 ? GORGO_OK : launch_kv_read(c, b, rk, rv, cache->type, hip_stream);
}

int gorgo_attend_workspace_bytes(const gorgo_kv_cache* cache, const gorgo_kv_batch* batch, int32_t q_heads, size_t* bytes) {
    clear_error();
    if (!bytes) return bad("bytes is NULL");
    AttendArgs a;
    int rc = take_attention(cache, batch, q_heads, &a);
    if (rc) return rc;
    const size_t need = most_prompt_workspace(a);
    *bytes = up256(token_suits(a) ? std::max(need, plan_token(a, cache->type).workspace) : need);
    return GORGO_OK;
}

int gorgo_attend_prompt(const gorgo_kv_cache* cache, const gorgo_kv_batch* batch, const gorgo_attention* attention, const gorgo_kv_rows* q,
                        const gorgo_kv_rows* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    clear_error();
    return attend(false, cache, batch, attention, q, out, lse, workspace, workspace_bytes, hip_stream);
}

int gorgo_attend_token(const gorgo_kv_cache* cache, const gorgo_kv_batch* batch, const gorgo_attention* attention, const gorgo_kv_rows* q,
                       const gorgo_kv_rows* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    clear_error();
    return attend(true, cache, batch, attention, q, out, lse, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
