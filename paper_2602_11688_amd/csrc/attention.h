// What the host side of the cache and attention entry points (attention.cpp) hands to their kernels (attention.hip).
#pragma once
#include <cstddef>
#include <cstdint>

namespace gorgo {

// x / divisor for 0 <= x < 2^31 by a product: multiplier = ceil(2^(31 + shift) / divisor), 2^shift >= divisor.
struct Divider {
    uint64_t multiplier;
    int32_t shift, divisor;
};
inline Divider divider(int32_t by) {
    Divider d{0, 0, by};
    while (((int64_t)1 << d.shift) < by) ++d.shift;
    d.multiplier = (((uint64_t)1 << (31 + d.shift)) + (uint64_t)by - 1) / (uint64_t)by;
    return d;
}

struct CacheArgs {
    char *k, *v;                         // rows of `type`
    uint8_t *k_scale, *v_scale;          // [pages][heads][page tokens], 8 bits only
    int64_t page_bytes, head_bytes, token_bytes;
    Divider page;                        // tokens of a page
    int32_t pages, heads, d;
};

struct BatchArgs {
    const int32_t *table, *first, *lengths;    // [S][columns]; [S + 1], or null: one token each; [S]
    int32_t S, tokens, columns;
    int32_t capacity;                    // columns * page tokens
};

// Packed rows of a call's new tokens: base, and bytes from a token and a head to the next.
struct RowsArgs {
    char* base;
    int64_t token_bytes, head_bytes;
};

struct AttendArgs {
    CacheArgs cache;
    BatchArgs batch;
    RowsArgs q, out;
    float* lse;                          // [tokens][q heads] or null
    uint32_t* counters;                  // token: of the pairs that several workgroups share, zero between calls
    float* partial;                      // workspace behind them
    float scale_log2;                    // softmax scale * log2(e)
    int32_t q_heads, window;             // window 0: none
    int32_t sinks;                       // first keys that stay visible beside a window
    Divider group;                       // q heads of a cache head
    int32_t tiles;                       // prompt: slots for tiles of rows
    int32_t splits;                      // prompt: most pieces of a tile's keys; token: workgroups
};

enum CacheType { CACHE_BF16 = 0, CACHE_F16 = 1, CACHE_E4M3 = 2 };

constexpr int MAX_HEAD = 128;            // widest head of the kernels
constexpr int32_t MOST_POSITIONS = 0x7fffffff - 1023;                      // of a row of the table
constexpr int COMPUTE_UNITS = 256;
// attend_prompt_kernel: rows of a workgroup, keys of a tile, most pieces of a tile's keys
constexpr int PROMPT_ROWS = 256, PROMPT_KEYS = 64, KEYS_LOG2 = 6, MOST_PIECES = 32;
// Pieces that so many tiles of keys are worth: of four tiles each, with sinks (whose windows may be short) FEW_PIECES where that would be less.
// A window of 256 after 4 sinks, five prompts of 4 to 64 tokens: 25.3 us in pieces of four tiles, 20.1 of two, 19.0 with eight pieces at least;
// 130 tokens with a window of 4096: 24.8, 30.1 and 24.6.
constexpr int FEW_PIECES = 8;
constexpr int32_t pieces_of(int32_t tiles, bool sinks) {
    const int32_t pieces = tiles / 4 > 1 ? tiles / 4 : 1, few = tiles < FEW_PIECES ? tiles : FEW_PIECES;
    return sinks && few > pieces ? few : pieces;
}
// attend_token_kernel: wavefronts of a workgroup and keys of a wavefront's step (a workgroup's step is a unit of work), query heads
// of a cache head at most, workgroups that the registers let run at once.  Beyond TOKEN_ROWS, and only there, the call is a prompt of
// one token each.  With 32 of them, two cache heads of 128: 48 sequences of 16,000 keys 162 us here and 234 as prompts (8 bits: 103 and 232),
// 16 of 5,000 47 and 40 (41 and 40), one of 30,000 119 and 47 (62 and 46), one of 700 32 and 25 (33 and 25); with 16 query heads
// 147 and 234 (92 and 233), 37 and 40 (32 and 39).  The cache's bytes decide where many are served; for few the prompt form would be the better one from 17 on.
constexpr int TOKEN_WAVES = 4, TOKEN_ROWS = 32, TOKEN_GROUPS = 2 * COMPUTE_UNITS;
// The workspace's beginning: one count for each of them, the same for every call, whatever its batch.
constexpr size_t COUNTER_BYTES = TOKEN_GROUPS * 4;
constexpr int token_keys(bool e8) { return e8 ? 64 : 32; }

// attention.hip
int launch_kv_write(const CacheArgs& c, const BatchArgs& b, const RowsArgs& k, const RowsArgs& v, int type, void* stream);
int launch_kv_read(const CacheArgs& c, const BatchArgs& b, const RowsArgs& k, const RowsArgs& v, int type, void* stream);
int launch_attend_prompt(const AttendArgs& a, int type, void* stream);
int launch_attend_token(const AttendArgs& a, int type, void* stream);

}  // namespace gorgo
