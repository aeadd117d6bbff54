// Entry points of the paged cache and the attention over it: argument checks, workspace, launches.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <string>

#include "attention.h"
#include "internal.h"

namespace gorgo {
namespace {

int bad(const std::string& what) { return fail(GORGO_ERR_INVALID_ARG, what); }

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// The cache, checked: what the kernels take for granted of it (16-byte loads, offsets in bytes that fit 64 bits, rows of one type).
int take_cache(const gorgo_kv_cache* c, CacheArgs* out) {
    if (!c) return bad("cache is NULL");
    if (c->type < GORGO_KV_BF16 || c->type > GORGO_KV_E4M3) return bad("cache.type must be 0 (bf16), 1 (fp16) or 2 (e4m3)");
    const bool e8 = c->type == GORGO_KV_E4M3;
    const int32_t step = e8 ? 16 : 8, bytes = e8 ? 1 : 2;
    if (c->pages < 1) return bad("cache.pages must be >= 1");
    if (c->page_tokens < 1 || c->page_tokens > 32767) return bad("cache.page_tokens must be in 1..32767");
    if (c->kv_heads < 1 || c->kv_heads > 1024) return bad("cache.kv_heads must be in 1..1024");
    if (c->head_dim < step || c->head_dim > MAX_HEAD || c->head_dim % step)
        return bad("cache.head_dim must be a multiple of " + std::to_string(step) + " in " + std::to_string(step) + ".." + std::to_string(MAX_HEAD));
    if (!c->k || !c->v) return bad("cache.k or cache.v is NULL");
    if (!aligned16(c->k) || !aligned16(c->v)) return bad("cache.k and cache.v must be 16-byte aligned");
    if (e8 && (!c->k_scale || !c->v_scale || reinterpret_cast<uintptr_t>(c->v_scale) % 4))
        return bad("an e4m3 cache needs k_scale and v_scale, v_scale 4-byte aligned");
    const int64_t strides[3] = {c->page_stride, c->head_stride, c->token_stride}, most = (int64_t)1 << 40;
    for (int64_t s : strides)
        if (s < 0 || s > most || s % step)
            return bad("cache strides must be multiples of " + std::to_string(step) + " elements in 0..2^40");
    if (c->token_stride * bytes > ((int64_t)1 << 26)) return bad("cache.token_stride must be at most 2^26 bytes");     // (64 of them: 32 bits)
    out->k = static_cast<char*>(c->k);
    out->v = static_cast<char*>(c->v);
    out->k_scale = c->k_scale;
    out->v_scale = c->v_scale;
    out->page_bytes = c->page_stride * bytes;
    out->head_bytes = c->head_stride * bytes;
    out->token_bytes = c->token_stride * bytes;
    out->page = divider(c->page_tokens);
    out->pages = c->pages;
    out->heads = c->kv_heads;
    out->d = c->head_dim;
    return GORGO_OK;
}

int take_batch(const gorgo_kv_batch* b, const gorgo_kv_cache* c, BatchArgs* out) {
    if (!b) return bad("batch is NULL");
    if (b->sequences < 0 || b->sequences > (1 << 16)) return bad("batch.sequences must be in 0..2^16");
    if (b->tokens < 0 || b->tokens > (1 << 24)) return bad("batch.tokens must be in 0..2^24");
    if (!b->token_offsets && b->tokens != b->sequences) return bad("without token_offsets batch.tokens must equal batch.sequences");
    if (b->sequences == 0 && b->tokens != 0) return bad("batch.tokens must be 0 without sequences");
    // (the kernels look up to two steps of 256 keys ahead, in 32 bits)
    if (b->table_columns < 1 || (int64_t)b->table_columns * c->page_tokens > MOST_POSITIONS)
        return bad("batch.table_columns must be >= 1, and table_columns * page_tokens at most 2^31 - 1024");
    if (b->sequences > 0 && (!b->page_table || !b->lengths)) return bad("batch.page_table or batch.lengths is NULL");
    out->table = b->page_table;
    out->first = b->token_offsets;
    out->lengths = b->lengths;
    out->S = b->sequences;
    out->tokens = b->tokens;
    out->columns = b->table_columns;
    out->capacity = b->table_columns * c->page_tokens;
    return GORGO_OK;
}

int take_rows(const gorgo_kv_rows* r, int32_t tokens, const char* name, RowsArgs* out) {
    if (!r) return bad(std::string(name) + " is NULL");
    if (tokens > 0 && !r->data) return bad(std::string(name) + ".data is NULL");
    if (!aligned16(r->data) || r->token_stride % 8 || r->head_stride % 8)
        return bad(std::string(name) + " must be 16-byte aligned, its strides multiples of 8 elements");
    const int64_t most = (int64_t)1 << 40;
    if (r->token_stride < 0 || r->head_stride < 0 || r->token_stride > most || r->head_stride > most)
        return bad(std::string(name) + ": strides must be in 0..2^40");
    out->base = static_cast<char*>(r->data);
    out->token_bytes = r->token_stride * 2;
    out->head_bytes = r->head_stride * 2;
    return GORGO_OK;
}

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
int64_t prompt_pieces(const AttendArgs& a) {
    return std::min<int64_t>(std::max<int64_t>(1, a.batch.capacity / (PIECE_TILES * PROMPT_KEYS)), MOST_PIECES);
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
    p.splits = groups * 2 > at_once ? 1 : (int32_t)std::min<int64_t>(at_once / groups, prompt_pieces(a));
    p.workspace = p.splits > 1 ? prompt_bytes(a, (int64_t)p.splits * a.batch.tokens * a.q_heads) : 0;
    return p;
}

// The most that plan_prompt asks for with at most these sequences, tokens and columns (few rows are split where many are not).  Pieces are
// at_once / groups at most, and groups are more than rows of a head / PROMPT_ROWS of each head: partial rows are less than at_once * PROMPT_ROWS.
size_t most_prompt_workspace(const AttendArgs& a) {
    const int64_t at_once = prompt_groups(a), pieces = prompt_pieces(a);
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
    if ((rc = take_rows(q, batch->tokens, "q", &a.q)) || (rc = take_rows(out, batch->tokens, "out", &a.out))) return rc;
    a.lse = lse;
    a.scale_log2 = scale_log2;
    a.window = how->window;
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
