// Random calls of the attention entry points with windows and sinks, with AddressSanitizer and UndefinedBehaviorSanitizer
// (tests/test_sanitized_append.py compiles and runs it).  usage: sinks_fuzz SEED ITERATIONS
// The launches are stand-ins that check what the kernels take for granted, above all that one workspace, of whose size nobody knows windows and
// sinks, holds the partial rows of every call.
#include <cmath>
#include <cstdio>
#include <cstdlib>

#include "attention.h"
#include "gorgo.h"
#include "internal.h"

static uint64_t rng_state;
static uint64_t rnd() {       // SplitMix64
    uint64_t z = (rng_state += 0x9E3779B97F4A7C15ull);
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
static uint64_t below(uint64_t n) { return n ? rnd() % n : 0; }
static int64_t some(int64_t most) { return (int64_t)std::exp((double)below(1 << 20) / (1 << 20) * std::log((double)most + 0.5)); }      // 1 .. most
static bool one_in(int n) { return below(n) == 0; }

#define CHECK(cond)                                                                                             \
    do {                                                                                                        \
        if (!(cond)) {                                                                                          \
            std::fprintf(stderr, "sinks_fuzz: check failed at line %d: %s (last error: %s)\n", __LINE__, #cond, gorgo_last_error()); \
            std::exit(3);                                                                                       \
        }                                                                                                       \
    } while (0)

static size_t workspace_size;
static int32_t window_given, sinks_given;
static int64_t split;

namespace gorgo {

static void check_mask(const AttendArgs& a) {
    CHECK(a.window == window_given && a.sinks == (window_given > 0 ? sinks_given : 0) && a.sinks >= 0);
}
int launch_kv_write(const CacheArgs&, const BatchArgs&, const RowsArgs&, const RowsArgs&, int, void*) { return GORGO_OK; }
int launch_kv_read(const CacheArgs&, const BatchArgs&, const RowsArgs&, const RowsArgs&, int, void*) { return GORGO_OK; }
int launch_attend_prompt(const AttendArgs& a, int, void*) {
    check_mask(a);
    CHECK(a.splits >= 1 && a.splits <= MOST_PIECES);
    const int64_t dp = a.cache.d <= 64 ? 64 : 128;
    if (a.splits > 1) {
        ++split;
        CHECK(COUNTER_BYTES + (size_t)(a.splits * (int64_t)a.batch.tokens * a.q_heads * (dp + 2)) * 4 <= workspace_size);
    }
    return GORGO_OK;
}
int launch_attend_token(const AttendArgs& a, int, void*) {
    check_mask(a);
    const int64_t dp = a.cache.d <= 64 ? 64 : 128, part = (a.group.divisor * (dp + 2) + 3) / 4 * 4;
    CHECK(a.splits >= 1 && a.splits <= TOKEN_GROUPS && COUNTER_BYTES + (size_t)(a.splits * 2 * part) * 4 <= workspace_size);
    return GORGO_OK;
}

}  // namespace gorgo

int main(int argc, char** argv) {
    if (argc < 3) return 2;
    rng_state = std::strtoull(argv[1], nullptr, 10);
    const int64_t iterations = std::strtoll(argv[2], nullptr, 10);
    char* const fake = reinterpret_cast<char*>((uintptr_t)1 << 20);            // (looked at by nobody)
    int64_t accepted = 0;
    for (int64_t i = 0; i < iterations; ++i) {
        const bool token = one_in(2);
        gorgo_kv_cache c{};
        c.type = (int32_t)below(3);
        c.k = c.v = fake;
        if (c.type == GORGO_KV_E4M3) c.k_scale = c.v_scale = (uint8_t*)fake;
        c.pages = (int32_t)some(0x7fffffff);
        c.page_tokens = (int32_t)some(32767);
        c.kv_heads = (int32_t)some(256);
        c.head_dim = 16 * (1 + (int32_t)below(8));
        c.token_stride = c.head_dim;
        c.head_stride = c.token_stride * c.page_tokens;
        c.page_stride = c.head_stride * c.kv_heads;
        const int32_t q_heads = c.kv_heads * (1 + (int32_t)below(12));
        gorgo_kv_batch b{};
        b.sequences = (int32_t)some(1000);
        b.tokens = token ? b.sequences : (int32_t)some(20000);
        b.table_columns = (int32_t)some((0x7fffffff - 1023) / c.page_tokens);
        b.page_table = b.lengths = (const int32_t*)fake;
        if (!token) b.token_offsets = (const int32_t*)fake;
        size_t need = 0;
        if (gorgo_attend_workspace_bytes(&c, &b, q_heads, &need) != GORGO_OK) continue;
        CHECK(need % 256 == 0 && need <= (35u << 20));
        workspace_size = need;
        if (one_in(2)) {                               // a smaller batch on this one's workspace
            b.sequences = (int32_t)some(b.sequences);
            b.tokens = token ? b.sequences : (int32_t)some(b.tokens);
            b.table_columns = (int32_t)some(b.table_columns);
        }
        window_given = one_in(8) ? (int32_t)rnd() : (int32_t)some(20000) - 1;
        sinks_given = one_in(8) ? (int32_t)rnd() : (int32_t)some(5000) - 1;
        gorgo_attention how{q_heads, window_given, 0.125f, sinks_given};
        gorgo_kv_rows q{fake, (int64_t)q_heads * c.head_dim, c.head_dim}, out = q;
        for (int rc : {gorgo_attend_prompt(&c, &b, &how, &q, &out, nullptr, fake, workspace_size, nullptr),
                       gorgo_attend_token(&c, &b, &how, &q, &out, nullptr, fake, workspace_size, nullptr)}) {
            CHECK(rc == GORGO_OK || rc == GORGO_ERR_INVALID_ARG);               // (never that the workspace is too small)
            CHECK(rc != GORGO_OK || (window_given >= 0 && sinks_given >= 0));
            accepted += rc == GORGO_OK;
        }
    }
    std::printf("%lld iterations, %lld calls accepted, %lld in pieces\n", (long long)iterations, (long long)accepted, (long long)split);
    return accepted > iterations / 4 && split > iterations / 20 ? 0 : 4;
}
