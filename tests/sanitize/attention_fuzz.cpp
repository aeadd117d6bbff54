// Random calls of the cache and attention entry points, ordinary and hostile, with AddressSanitizer and UndefinedBehaviorSanitizer
// (tests/test_sanitized_attention.py compiles and runs it).  usage: attention_fuzz SEED ITERATIONS
// The launches are stand-ins that check what the kernels take for granted: grids that a device accepts, offsets and partial rows
// that stay inside the workspace, positions that fit 32 bits.  Everything that is accepted has to pass them.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <limits>

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
// 1 .. most, evenly over the logarithm, or (one time in eight) anything near a power of two
static int64_t some(int64_t most) {
    if (below(8) == 0) {
        const int64_t x = ((int64_t)1 << below(33)) + (int64_t)below(5) - 2;
        return x < 1 ? 1 : x > most ? most : x;
    }
    return (int64_t)std::exp((double)below(1 << 20) / (1 << 20) * std::log((double)most + 0.5));
}
static bool one_in(int n) { return below(n) == 0; }

#define CHECK(cond)                                                                                             \
    do {                                                                                                        \
        if (!(cond)) {                                                                                          \
            std::fprintf(stderr, "attention_fuzz: check failed at line %d: %s (last error: %s)\n", __LINE__, #cond, gorgo_last_error()); \
            std::exit(3);                                                                                       \
        }                                                                                                       \
    } while (0)

static char* workspace_begin;
static size_t workspace_size;
static int64_t launches;

namespace gorgo {

static void check_cache(const CacheArgs& c, const BatchArgs& b, int type) {
    ++launches;
    CHECK(b.tokens > 0 && b.S > 0 && b.lengths && b.table && c.k && c.v && (type != CACHE_E4M3 || (c.k_scale && c.v_scale)));
    CHECK((int64_t)b.columns * c.page.divisor == b.capacity && b.capacity <= std::numeric_limits<int32_t>::max() - 1023);
    CHECK(c.d >= 8 && c.d <= MAX_HEAD && c.page_bytes % 16 == 0 && c.head_bytes % 16 == 0 && c.token_bytes % 16 == 0);
    CHECK(c.token_bytes * 63 + 256 <= (int64_t)0xffffffffu);
    for (int64_t x : {(int64_t)0, (int64_t)c.page.divisor - 1, (int64_t)c.page.divisor, (int64_t)b.capacity - 1, (int64_t)0x7fffffff})
        CHECK((int64_t)(((uint64_t)x * c.page.multiplier) >> (31 + c.page.shift)) == x / c.page.divisor);
}
int launch_kv_write(const CacheArgs& c, const BatchArgs& b, const RowsArgs&, const RowsArgs&, int type, void*) {
    check_cache(c, b, type);
    return GORGO_OK;
}
int launch_kv_read(const CacheArgs& c, const BatchArgs& b, const RowsArgs&, const RowsArgs&, int type, void*) {
    check_cache(c, b, type);
    return GORGO_OK;
}
static void check_workspace(const AttendArgs& a, int64_t floats) {
    CHECK((char*)a.counters == workspace_begin && (char*)a.partial == workspace_begin + COUNTER_BYTES);
    CHECK(COUNTER_BYTES + (size_t)floats * 4 <= workspace_size);
}
int launch_attend_prompt(const AttendArgs& a, int type, void*) {
    check_cache(a.cache, a.batch, type);
    const int64_t rows = (int64_t)a.batch.tokens * a.group.divisor, dp = a.cache.d <= 64 ? 64 : 128;
    CHECK(rows <= 0x7fffffff - PROMPT_ROWS && a.q_heads == a.group.divisor * a.cache.heads);
    // every sequence has a slot for each of its tiles, and a launch less than 2^32 threads
    CHECK(a.tiles >= rows / PROMPT_ROWS + a.batch.S && (int64_t)a.tiles * a.cache.heads * 2 * PROMPT_ROWS < ((int64_t)1 << 32));
    CHECK(a.splits >= 1 && a.splits <= MOST_PIECES);
    if (a.splits > 1) check_workspace(a, (int64_t)a.splits * a.batch.tokens * a.q_heads * (dp + 2));
    return GORGO_OK;
}
int launch_attend_token(const AttendArgs& a, int type, void*) {
    check_cache(a.cache, a.batch, type);
    const int64_t dp = a.cache.d <= 64 ? 64 : 128, part = (a.group.divisor * (dp + 2) + 3) / 4 * 4;
    CHECK(!a.batch.first && a.batch.tokens == a.batch.S && a.group.divisor <= TOKEN_ROWS);
    CHECK(a.splits >= 1 && a.splits <= TOKEN_GROUPS);
    check_workspace(a, (int64_t)a.splits * 2 * part);
    return GORGO_OK;
}

}  // namespace gorgo

static gorgo_kv_rows rows_of(char* base, int32_t heads, int32_t d) {
    gorgo_kv_rows r{base, (int64_t)heads * d, d};
    if (one_in(20)) r.token_stride = (int64_t)rnd();
    if (one_in(20)) r.head_stride = (int64_t)rnd();
    if (one_in(20)) r.data = base + below(16);
    if (one_in(40)) r.data = nullptr;
    return r;
}

int main(int argc, char** argv) {
    if (argc < 3) return 2;
    rng_state = std::strtoull(argv[1], nullptr, 10);
    const int64_t iterations = std::strtoll(argv[2], nullptr, 10);
    char* const fake = reinterpret_cast<char*>((uintptr_t)1 << 20);            // (looked at by nobody)
    workspace_begin = fake;
    int64_t accepted = 0;
    for (int64_t i = 0; i < iterations; ++i) {
        const bool token = one_in(2);
        gorgo_kv_cache c{};
        c.type = (int32_t)below(3);
        const int32_t step = c.type == GORGO_KV_E4M3 ? 16 : 8;
        c.k = c.v = fake;
        if (c.type == GORGO_KV_E4M3) c.k_scale = c.v_scale = (uint8_t*)fake;
        c.pages = (int32_t)some(0x7fffffff);
        c.page_tokens = (int32_t)some(32767);
        c.kv_heads = (int32_t)some(1024);
        c.head_dim = step * (1 + (int32_t)below(128 / step));
        c.token_stride = c.head_dim;
        c.head_stride = c.token_stride * c.page_tokens;
        c.page_stride = c.head_stride * c.kv_heads;
        const int32_t group = (int32_t)some(64), q_heads = one_in(20) ? (int32_t)rnd() : c.kv_heads * group;
        gorgo_kv_batch b{};
        b.sequences = (int32_t)some(1 << 16);
        b.tokens = token ? b.sequences : (int32_t)some(1 << 24);
        b.table_columns = (int32_t)some(0x7fffffff / c.page_tokens);
        b.page_table = b.lengths = (const int32_t*)fake;
        if (!token) b.token_offsets = (const int32_t*)fake;
        // one thing wrong, or near its end
        switch (below(24)) {
            case 0: c.type = (int32_t)rnd(); break;
            case 1: c.pages = (int32_t)rnd(); break;
            case 2: c.page_tokens = (int32_t)rnd(); break;
            case 3: c.kv_heads = (int32_t)rnd(); break;
            case 4: c.head_dim = (int32_t)rnd(); break;
            case 5: c.page_stride = (int64_t)rnd(); break;
            case 6: c.head_stride = (int64_t)rnd(); break;
            case 7: c.token_stride = (int64_t)rnd(); break;
            case 8: c.token_stride = (int64_t)below(1 << 26) / 16 * 16; break;
            case 9: b.sequences = (int32_t)rnd(); break;
            case 10: b.tokens = (int32_t)rnd(); break;
            case 11: b.table_columns = (int32_t)rnd(); break;
            case 12: b.lengths = nullptr; break;
            case 13: b.tokens = 0; break;
            default: break;
        }
        size_t need = 0;
        workspace_size = ~(size_t)0;
        if (gorgo_attend_workspace_bytes(&c, &b, q_heads, &need) == GORGO_OK) {
            CHECK(need % 256 == 0 && need <= (35u << 20));
            workspace_size = need;
            // a smaller batch on this one's workspace
            if (b.sequences > 0 && b.tokens > 0 && one_in(2)) {
                const int32_t all = b.tokens;
                b.sequences = (int32_t)some(b.sequences);
                b.tokens = b.token_offsets ? (int32_t)some(all) : b.sequences;
                b.table_columns = (int32_t)some(b.table_columns);
            }
        }
        gorgo_attention how{q_heads, one_in(8) ? (int32_t)rnd() : (int32_t)below(5000), 0.125f, 0};
        if (one_in(30)) how.scale = one_in(2) ? std::numeric_limits<float>::quiet_NaN() : std::numeric_limits<float>::max();
        gorgo_kv_rows q = rows_of(fake, q_heads > 0 && q_heads <= 4096 ? q_heads : 1, 128), out = q, k = rows_of(fake, 8, 128), v = rows_of(fake, 8, 128);
        const int written = gorgo_kv_write(&c, &b, &k, &v, nullptr);
        CHECK(written == gorgo_kv_read(&c, &b, &k, &v, nullptr) && (written == GORGO_OK || written == GORGO_ERR_INVALID_ARG));
        for (int rc : {gorgo_attend_prompt(&c, &b, &how, &q, &out, nullptr, fake, workspace_size, nullptr),
                       gorgo_attend_token(&c, &b, &how, &q, &out, nullptr, fake, workspace_size, nullptr)}) {
            CHECK(rc == GORGO_OK || rc == GORGO_ERR_INVALID_ARG || rc == GORGO_ERR_NONFINITE);     // (never that the workspace is too small)
            accepted += rc == GORGO_OK;
        }
    }
    std::printf("%lld iterations, %lld attention calls accepted, %lld launches\n", (long long)iterations, (long long)accepted, (long long)launches);
    return accepted > iterations / 4 ? 0 : 4;
}
