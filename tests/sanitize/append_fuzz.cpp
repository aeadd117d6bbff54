// Random calls of gorgo_kv_append and gorgo_rotate_heads, ordinary and hostile, with AddressSanitizer and UndefinedBehaviorSanitizer
// (tests/test_sanitized_append.py compiles and runs it).  usage: append_fuzz SEED ITERATIONS
// The launch is a stand-in that checks what the kernel takes for granted.  Everything that is accepted has to pass it.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <limits>

#include "append.h"
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
            std::fprintf(stderr, "append_fuzz: check failed at line %d: %s (last error: %s)\n", __LINE__, #cond, gorgo_last_error()); \
            std::exit(3);                                                                                       \
        }                                                                                                       \
    } while (0)

static int64_t launches;

namespace gorgo {

static void check_divider(const Divider& d, int64_t most) {
    for (int64_t x : {(int64_t)0, (int64_t)d.divisor - 1, (int64_t)d.divisor, most})
        CHECK((int64_t)(((uint64_t)x * d.multiplier) >> (31 + d.shift)) == x / d.divisor);
}
static bool whole(const RowsArgs& r) { return (uintptr_t)r.base % 16 == 0 && r.token_bytes % 16 == 0 && r.head_bytes % 16 == 0; }
int launch_append(const AppendArgs& a, int type, void*) {
    ++launches;
    const BatchArgs& b = a.batch;
    CHECK(b.tokens > 0 && a.cache.d >= 8 && a.cache.d <= MAX_HEAD && a.cache.d % 8 == 0);
    // every token has a workgroup, every row of a block a place in 32 bits, and a launch less than 2^32 threads
    const int64_t blocks = ((int64_t)b.tokens + a.block - 1) / a.block;
    CHECK(a.block >= 1 && a.block <= MOST_BLOCK && a.parts >= 1 && a.parts <= 65535 && blocks * a.parts * APPEND_THREADS < ((int64_t)1 << 32));
    CHECK(a.q_heads.divisor >= 0 && a.q_heads.divisor <= 4096 && a.kv_heads.divisor >= 0 && a.kv_heads.divisor <= 1024 && a.q_heads.divisor + a.kv_heads.divisor > 0);
    if (a.q_heads.divisor) {
        check_divider(a.q_heads, (int64_t)a.block * a.q_heads.divisor - 1);
        CHECK(a.q.base && a.q_out.base && whole(a.q) && whole(a.q_out));
    }
    if (a.kv_heads.divisor) {
        check_divider(a.kv_heads, (int64_t)a.block * a.kv_heads.divisor - 1);
        CHECK(a.k.base && a.v.base && whole(a.k) && whole(a.v) && a.cache.k && a.cache.v && b.table && b.S > 0);
        CHECK(type != CACHE_E4M3 || (a.cache.k_scale && a.cache.v_scale && a.cache.d % 16 == 0));
        CHECK((int64_t)b.columns * a.cache.page.divisor == b.capacity && b.capacity <= std::numeric_limits<int32_t>::max() - 1023);
        check_divider(a.cache.page, b.capacity - 1);
    } else {
        CHECK(!a.cache.k && type != CACHE_E4M3);       // (nothing is looked up in a table that may not be there)
    }
    if (b.S > 0) CHECK(b.lengths && (b.first || b.tokens == b.S));
    const RotationArgs& r = a.rotation;
    CHECK(r.pairs >= 0 && 2 * r.pairs <= a.cache.d && (1 << a.pair_bits) >= r.pairs && a.pair_bits <= 6 && (r.pairs == 0 || r.frequencies));
    CHECK(r.pairs == 0 || r.positions || b.S > 0);
    for (int i = 0; i < 64; ++i) {
        const int axis = (int)((r.axis_low >> i) & 1) + 2 * (int)((r.axis_high >> i) & 1);
        CHECK(axis == 0 || (i < r.pairs && r.positions));
    }
    for (const NormArgs* n : {&a.q_norm, &a.k_norm})
        CHECK(n->eps == 0.0f ? !n->weight : n->eps > 0.0f && std::isfinite(n->eps) && (uintptr_t)n->weight % 16 == 0 && n->head_stride % 4 == 0);
    return GORGO_OK;
}

}  // namespace gorgo

static char* const fake = reinterpret_cast<char*>((uintptr_t)1 << 20);            // (looked at by nobody)

static gorgo_kv_rows rows_of(int32_t heads, int32_t d) {
    gorgo_kv_rows r{fake, (int64_t)heads * d, d};
    if (one_in(30)) r.token_stride = (int64_t)rnd();
    if (one_in(30)) r.head_stride = (int64_t)rnd();
    if (one_in(30)) r.data = fake + below(32);
    if (one_in(60)) r.data = nullptr;
    return r;
}

static gorgo_norm norm_of(int32_t d) {
    gorgo_norm n{one_in(3) ? nullptr : (const float*)fake, one_in(2) ? d : 0, 1e-6f, 0};
    if (one_in(20)) n.eps = one_in(2) ? std::numeric_limits<float>::quiet_NaN() : -(float)below(2);
    if (one_in(20)) n.head_stride = (int64_t)rnd();
    if (one_in(20)) n.weight = (const float*)(fake + below(32));
    return n;
}

int main(int argc, char** argv) {
    if (argc < 3) return 2;
    rng_state = std::strtoull(argv[1], nullptr, 10);
    const int64_t iterations = std::strtoll(argv[2], nullptr, 10);
    int64_t accepted = 0;
    for (int64_t i = 0; i < iterations; ++i) {
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
        const bool token = one_in(2);
        gorgo_kv_batch b{};
        b.sequences = (int32_t)some(1 << 16);
        b.tokens = token ? b.sequences : (int32_t)some(1 << 24);
        b.table_columns = (int32_t)some((0x7fffffff - 1023) / c.page_tokens);
        b.page_table = b.lengths = (const int32_t*)fake;
        if (!token) b.token_offsets = (const int32_t*)fake;
        int32_t q_heads = one_in(4) ? 0 : (int32_t)some(4096);
        gorgo_rotation r{};
        r.frequencies = (const double*)fake;
        r.pairs = 1 + (int32_t)below(c.head_dim / 2);
        r.layout = (int32_t)below(2);
        r.axes = 1 + (int32_t)below(4);
        r.magnitude = 1.0f;
        if (r.axes > 1 || one_in(2)) r.positions = (const int32_t*)fake;
        r.axis_stride = b.tokens;
        for (auto& x : r.axis_of_pair) x = (uint8_t)below(r.axes);
        switch (below(24)) {             // one thing wrong, or near its end
            case 0: c.type = (int32_t)rnd(); break;
            case 1: c.head_dim = (int32_t)rnd(); break;
            case 2: c.page_tokens = (int32_t)rnd(); break;
            case 3: b.sequences = (int32_t)rnd(); break;
            case 4: b.tokens = (int32_t)rnd(); break;
            case 5: b.lengths = nullptr; break;
            case 6: b.tokens = 0; break;
            case 7: b.sequences = 0; break;
            case 8: q_heads = (int32_t)rnd(); break;
            case 9: r.pairs = (int32_t)rnd(); break;
            case 10: r.axes = (int32_t)rnd(); break;
            case 11: r.axis_of_pair[below(64)] = (uint8_t)rnd(); break;
            case 12: r.positions = nullptr; break;
            case 13: r.frequencies = (const double*)(fake + below(16)); break;
            case 14: r.magnitude = std::numeric_limits<float>::infinity(); break;
            case 15: r.layout = (int32_t)rnd(); break;
            case 16: r.axis_stride = (int64_t)rnd(); break;
            case 17: b.page_table = nullptr; break;
            case 18: b.tokens = 1 << 24, b.sequences = 1 << 16, b.token_offsets = (const int32_t*)fake; break;
            default: break;
        }
        gorgo_norm qn = norm_of(c.head_dim), kn = norm_of(c.head_dim);
        gorgo_kv_rows q = rows_of(8, 128), out = rows_of(8, 128), k = rows_of(8, 128), v = rows_of(8, 128);
        const gorgo_rotation* const rotation = one_in(4) ? nullptr : &r;
        const gorgo_norm *const q_norm = one_in(2) ? nullptr : &qn, *const k_norm = one_in(2) ? nullptr : &kn;
        for (int rc : {gorgo_kv_append(&c, &b, rotation, q_norm, k_norm, q_heads, &q, &out, &k, &v, nullptr),
                       gorgo_rotate_heads(&b, rotation, q_norm, c.type, q_heads, c.head_dim, &q, &out, nullptr)}) {
            CHECK(rc == GORGO_OK || rc == GORGO_ERR_INVALID_ARG || rc == GORGO_ERR_NONFINITE);
            accepted += rc == GORGO_OK;
        }
    }
    std::printf("%lld iterations, %lld calls accepted, %lld launches\n", (long long)iterations, (long long)accepted, (long long)launches);
    return accepted > iterations / 4 ? 0 : 4;
}
