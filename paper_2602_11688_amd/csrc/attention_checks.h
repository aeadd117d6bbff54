// Checks of the structures that the cache, attention and append entry points share, into what their kernels take.
#pragma once
#include <cstdint>
#include <string>

#include "attention.h"
#include "gorgo.h"
#include "internal.h"

namespace gorgo {

inline int bad(const std::string& what) { return fail(GORGO_ERR_INVALID_ARG, what); }

inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// The cache, checked: what the kernels take for granted of it (16-byte loads, offsets in bytes that fit 64 bits, rows of one type).
inline int take_cache(const gorgo_kv_cache* c, CacheArgs* out) {
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

inline int take_batch(const gorgo_kv_batch* b, const gorgo_kv_cache* c, BatchArgs* out) {
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

inline int take_rows(const gorgo_kv_rows* r, int32_t tokens, const char* name, RowsArgs* out) {
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

}  // namespace gorgo
