// Heads that are normed and rotated, on their way into the cache or alone.
#pragma once
#include "append.h"
#include "kv_cache.h"

namespace gorgo {

// A row (token, head) lies in ROW neighbouring lanes, 2 * U values a lane: two runs of U that a rotation of halves turns by each other (values
// from u * U on and from pairs + u * U on), so that no value moves between lanes.
//   EVEN: halves that begin at a whole run (or nothing to rotate), U = 8, loads of 16 bytes.
//   UNEVEN: halves that begin anywhere, U = 8.  Loads and stores need not begin at a multiple of their size; the last run of a half (and of what is not
//   rotated) begins earlier where it would not be a whole one, and its first values are another lane's too, who stores the same.  Where
//   there are less than 8 values of a kind, they are stored one by one.  (Runs of 4 and of 1 need none of that and are bound by instructions: 64
//   million values in heads of 72 with norms took 92 us, now 72; of 80 with 13 pairs 205 and 65; of 128 with 63 pairs 146 and 77.)
//   SINGLE: U = 1, for heads of 8 values with halves of 1 to 4 (16 bits).
//   NEIGHBOURS: pairs within a run.
enum Runs { EVEN, UNEVEN, SINGLE, NEIGHBOURS };

// Sums and maxima over the lanes of a row: neighbours, pairs, then mirrors of 8 and 16 lanes.
template <int CTRL>
__device__ inline unsigned moved(unsigned x) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true); }
template <int CTRL>
__device__ inline float moved(float x) { return __builtin_bit_cast(float, moved<CTRL>(__builtin_bit_cast(unsigned, x))); }
template <int CTRL>
__device__ inline double moved(double x) {
    const uint2_t u = __builtin_bit_cast(uint2_t, x);
    return __builtin_bit_cast(double, (uint2_t){moved<CTRL>(u.x), moved<CTRL>(u.y)});
}
template <int ROW, class A, class F>
__device__ inline A over_row(A x, F f) {
    static_assert(ROW == 4 || ROW == 8 || ROW == 16);
    x = f(x, moved<0xb1>(x));                          // lanes i ^ 1
    x = f(x, moved<0x4e>(x));                          // i ^ 2
    if constexpr (ROW >= 8) x = f(x, moved<0x141>(x));      // 7 - i of 8
    if constexpr (ROW >= 16) x = f(x, moved<0x140>(x));     // 15 - i of 16
    return x;
}

// Cosine and sine in 64 bits: the nearest multiple of pi / 2 taken off in two steps, Taylor's series on what is left (at most pi / 4: the first
// terms left out are below 2^-45).  The instructions for 32 bits are off by more than a rounding, and take turns.
struct CosSin {
    double c, s;
};
__device__ inline CosSin cos_sin(double x) {
    const double k = __builtin_rint(x * 0.63661977236758134);
    double r = __builtin_fma(-k, 1.5707963267948966, x);
    r = __builtin_fma(-k, 6.123233995736766e-17, r);
    const double z = r * r;
    double s = 1.0 / 6227020800.0, c = -1.0 / 87178291200.0;
    s = __builtin_fma(s, z, -1.0 / 39916800.0);
    s = __builtin_fma(s, z, 1.0 / 362880.0);
    s = __builtin_fma(s, z, -1.0 / 5040.0);
    s = __builtin_fma(s, z, 1.0 / 120.0);
    s = __builtin_fma(s, z, -1.0 / 6.0);
    s = __builtin_fma(s * z, r, r);
    c = __builtin_fma(c, z, 1.0 / 479001600.0);
    c = __builtin_fma(c, z, -1.0 / 3628800.0);
    c = __builtin_fma(c, z, 1.0 / 40320.0);
    c = __builtin_fma(c, z, -1.0 / 720.0);
    c = __builtin_fma(c, z, 1.0 / 24.0);
    c = __builtin_fma(c, z, -0.5);
    c = __builtin_fma(c, z, 1.0);
    const double quarter = k - 4.0 * __builtin_floor(k * 0.25);
    const bool odd = quarter == 1.0 || quarter == 3.0;
    const double cos_ = odd ? s : c, sin_ = odd ? c : s;
    return {quarter == 1.0 || quarter == 2.0 ? -cos_ : cos_, quarter >= 2.0 ? -sin_ : sin_};
}

// To 32 bits so that a second rounding, to fewer, is that of the 64 bits: towards zero, with the last bit set where anything was lost.
__device__ inline float to_odd(double x) {
    const float f = (float)x;
    if (!((double)f != x)) return f;                   // (NaN too)
    if (x != x) return f;
    const unsigned u = __builtin_bit_cast(unsigned, f);
    const bool beyond = __builtin_fabs((double)f) > __builtin_fabs(x);
    return __builtin_bit_cast(float, (beyond ? u - 1 : u) | 1u);
}

// Sequences of a block of tokens: lane t's of token `token + t`, t < n, the last one that begins at or before it.
__device__ inline int32_t sequences_of(const BatchArgs& b, int32_t token, int32_t n) {
    const int lane = threadIdx.x & 63;
    if (!b.first) return min(token + lane, b.S - 1);
    int32_t s = 0;                                     // of the first token, 64 looked at at a time
    for (int32_t left = b.S; left > 1;) {
        const int32_t step = (left + 63) / 64, at = lane * step;
        const int before = __popcll(__ballot(at < left && b.first[s + min(at, left - 1)] <= token));
        const int32_t skip = max(before - 1, 0) * step;
        s += skip;
        left = min(step, left - skip);
    }
    s = uniform(s);
    int32_t more = 0;                                  // of the others: how many begin after it
    for (int32_t base = s + 1; base < b.S; base += 64) {
        const int32_t begin = base + lane < b.S ? b.first[base + lane] : 0x7fffffff;
        int last = 0;
        for (int32_t t = 0; t < n; ++t) {
            last = __popcll(__ballot(begin <= token + t));
            if (lane == t) more += last;
        }
        if (last < 64) break;
    }
    return s + more;
}

template <class T>
__device__ inline float value_of(unsigned pair, int which);
template <>
__device__ inline float value_of<Bf16>(unsigned pair, int which) { return __builtin_bit_cast(float, which ? pair & 0xffff0000u : pair << 16); }
template <>
__device__ inline float value_of<F16>(unsigned pair, int which) { return (float)__builtin_bit_cast(f16x2, pair)[which]; }

// U 16-bit values, two to a register; ALIGN: bytes that their address is a multiple of.
typedef uint4_t uint4_anywhere __attribute__((aligned(2)));
typedef uint2_t uint2_anywhere __attribute__((aligned(1)));
template <int U, int ALIGN>
struct Values {
    unsigned x[(U + 1) / 2];
    using Whole = std::conditional_t<ALIGN == 16, uint4_t, uint4_anywhere>;
    __device__ void load(const char* from) {
        if constexpr (U == 8) {
            const uint4_t v = *(const Whole*)from;
            x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
        } else {
            x[0] = *(const unsigned short*)from;
        }
    }
    __device__ void store(char* to) const {
        if constexpr (U == 8) *(Whole*)to = (uint4_t){x[0], x[1], x[2], x[3]};
        else *(unsigned short*)to = (unsigned short)x[0];
    }
    __device__ void zero() {
#pragma unroll
        for (unsigned& w : x) w = 0;
    }
};

enum Kind { QUERIES, KEYS, VALUES };

// A workgroup takes a block of tokens, or one of `parts` that share it.  Its wavefronts look up where the tokens lie (a lane a token), compute
// cosines and sines of their positions (a lane a pair, once for all heads), which go to LDS, and then take the tokens' rows, queries, keys
// and values one after the other, 64 / ROW a wavefront at a time; the rows of the next step are under way while one is worked on, the first
// before anything else is known.  Bound by bytes, every value being read once and written once: 29,555 tokens of 32/8 heads of 128 into an 8-bit
// cache take 147 us (4.5 TB/s read and written, where a copy reaches 4.9), 50,000 rows of 16 heads of 80 50.5 us (5.1); few tokens by the chain of a place, an
// angle, a row and its store (8 tokens: 4.0 us of a captured graph in 16 bits, 4.7 in 8).
template <class T, bool E8, int ROW, Runs RUNS>
__global__ __launch_bounds__(APPEND_THREADS) void append_kernel(AppendArgs a) {
    constexpr int WAVES = APPEND_THREADS / 64, ROWS = 64 / ROW;
    constexpr int U = RUNS == SINGLE ? 1 : 8, PAIRS = RUNS == NEIGHBOURS ? U / 2 : U;      // values of a run, and pairs that they belong to
    using Run = Values<U, RUNS == UNEVEN || U == 1 ? 2 : 16>;
    // cosine and sine of a token's pairs, in the order in which the lanes of a row read them
    __shared__ __attribute__((aligned(16))) float turns[MOST_BLOCK][2 * MOST_PAIRS];
    __shared__ __attribute__((aligned(16))) double turns64[E8 ? MOST_BLOCK : 1][2 * MOST_PAIRS];
    __shared__ int64_t row_at[MOST_BLOCK], scale_at[MOST_BLOCK];           // in the cache, -1: nowhere
    __shared__ int32_t counts[MOST_BLOCK];                                  // the token belongs to a sequence
    __shared__ __attribute__((aligned(16))) float weights[2][MAX_HEAD];    // that all heads share, of queries and keys

    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int32_t token0 = blockIdx.x * a.block, n = min(a.block, a.batch.tokens - token0);
    const int32_t pairs = a.rotation.pairs;

    // this lane's runs of a row: their first values, whether there is such a run, and which of its values count (UNEVEN)
    const int j = lane % ROW, d = a.cache.d, turned = RUNS == NEIGHBOURS ? 0 : (pairs + U - 1) / U;
    int start[2];
    unsigned valid = 0;                                // bit i * U + e: value e of run i counts
    bool inside[2], apart = false;                     // apart: to be stored one by one
    if constexpr (RUNS == UNEVEN) {
        const int rest = d - 2 * pairs;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int n = j < turned ? pairs : rest, at = j < turned ? j * U : (2 * (j - turned) + i) * U;      // values of the half, or the rest; where the run begins in it
            const int first = j < turned ? i * pairs : 2 * pairs;
            inside[i] = at < n;
            start[i] = n >= U ? first + min(at, n - U) : j < turned ? first : d - U;
            const int lo = n >= U ? at - min(at, n - U) : j < turned ? 0 : U - n, hi = n >= U || j >= turned ? U : n;
            if (inside[i]) valid |= ((1u << hi) - (1u << lo)) << (i * U);
            apart = n < U;
        }
    } else {
        start[0] = RUNS == NEIGHBOURS || j < turned ? j * U : 2 * j * U;
        start[1] = RUNS == NEIGHBOURS ? (j + ROW) * U : j < turned ? pairs + j * U : (2 * j + 1) * U;
        inside[0] = start[0] < d;
        inside[1] = start[1] < d;
    }
    // steps of a wavefront: of the block's queries, keys and values, in the order of tokens and heads
    const int32_t q_steps = (n * a.q_heads.divisor + ROWS - 1) / ROWS, kv_steps = (n * a.kv_heads.divisor + ROWS - 1) / ROWS, steps = q_steps + 2 * kv_steps;
    const int32_t stride = a.parts * WAVES;
    // A row's bytes from the block's first one; products of 32 bits where strides are as small as they mostly are (64 million
    // values in heads of 80 with norms: 58.5 us, 64.5 with products of 64 bits).
    auto from_first = [&](int64_t token_bytes, int64_t head_bytes, int32_t t, int32_t h) -> int64_t {
        if ((uint64_t)token_bytes >> 28 || (uint64_t)head_bytes >> 19) return t * token_bytes + h * head_bytes;
        return (int64_t)((uint32_t)t * (uint32_t)token_bytes + (uint32_t)h * (uint32_t)head_bytes);
    };
    struct Rows {                                      // of a wavefront's step
        Run x[2];
        int32_t t, h;                                  // token of the block, head
        bool is;
    };
    auto load = [&](int32_t at, Rows& rows) {
        rows.x[0].zero();
        rows.x[1].zero();
        if (at >= steps) return;
        const bool queries = at < q_steps, keys = !queries && at < q_steps + kv_steps;
        const RowsArgs& from = queries ? a.q : keys ? a.k : a.v;
        const Divider& heads = queries ? a.q_heads : a.kv_heads;
        const int32_t r = (queries ? at : keys ? at - q_steps : at - q_steps - kv_steps) * ROWS + lane / ROW, last = n * heads.divisor - 1;
        rows.is = r <= last;
        rows.t = quotient(heads, min(r, last));
        rows.h = min(r, last) - rows.t * heads.divisor;
        const char* const row = from.base + token0 * from.token_bytes + from_first(from.token_bytes, from.head_bytes, rows.t, rows.h);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (inside[i]) rows.x[i].load(row + start[i] * 2);
    };
    int32_t step = blockIdx.y * WAVES + wave;
    Rows now;
    load(step, now);
    if (threadIdx.x < 2 * MAX_HEAD / 4) {
        const NormArgs& norm = threadIdx.x < MAX_HEAD / 4 ? a.q_norm : a.k_norm;
        const int at = threadIdx.x % (MAX_HEAD / 4) * 4;
        if (norm.weight && !norm.head_stride && at < a.cache.d) *(float4_t*)&weights[threadIdx.x / (MAX_HEAD / 4)][at] = *(const float4_t*)(norm.weight + at);
    }

    // angles: a lane a pair, of as many tokens at once as their pairs leave room for
    const int32_t pair = lane & ((1 << a.pair_bits) - 1), tokens_at_once = 64 >> a.pair_bits;
    const double frequency = pair < pairs ? a.rotation.frequencies[pair] : 0.0;
    int32_t pos = 0;
    {
        int64_t at = -1, scale = 0;
        bool is = lane < n;
        if (a.batch.S) {
            int32_t s, length;
            const int32_t token = token0 + lane;
            Span span;
            if (a.batch.first && a.batch.S <= 64) {
                // a lane a sequence: one wait for all that there is to know of them (50,000 rows of 16 heads of 80: 50.8 us, 51.2 with a wait each)
                const int32_t mine = min(lane, a.batch.S - 1);
                const Span of = span_of(a.batch, mine);
                const int32_t begin = a.batch.first[mine], its_length = length_of(a.batch, mine);
                s = 0;
                for (int32_t t = 0; t < n; ++t) {
                    const int before = __popcll(__ballot(lane < a.batch.S && begin <= token0 + t));
                    if (lane == t) s = max(before - 1, 0);
                }
                span = {__shfl(of.begin, s), __shfl(of.end, s)};
                length = __shfl(its_length, s);
            } else {
                s = sequences_of(a.batch, token0, n);
                span = span_of(a.batch, s);
                length = length_of(a.batch, s);
            }
            is = is && token >= span.begin && token < span.end;
            pos = length - (span.end - token);
            if (a.cache.k && is && pos >= 0 && pos < a.batch.capacity) {
                const int32_t index = quotient(a.cache.page, pos), slot = pos - index * a.cache.page.divisor;
                const int32_t page = page_of(a.batch, a.cache, s, index);
                if (page >= 0) {
                    at = page * a.cache.page_bytes + slot * a.cache.token_bytes;
                    scale = ((int64_t)page * a.cache.heads) * a.cache.page.divisor + slot;
                }
            }
        }
        if (wave == 0 && lane < n) {
            row_at[lane] = at;
            scale_at[lane] = scale;
            counts[lane] = is;
        }
    }
    if (pairs) {
        // a pair stands beside the others that the lane of its run reads: in chunks of two pairs, one chunk of every lane after the other
        auto slot = [](int run, int nth) { return PAIRS == 1 ? run * 2 : nth / 2 * (MOST_PAIRS / PAIRS * 4) + run * 4 + (nth & 1) * 2; };
        const int to = slot(pair / PAIRS, pair % PAIRS);
        // (the last run of uneven halves begins earlier: its first pairs are the run before's too)
        const bool again = RUNS == UNEVEN && pairs > U && pair >= pairs - U, own = !(RUNS == UNEVEN && pairs > U && pair / PAIRS == turned - 1);
        const int to_again = slot(turned - 1, again ? pair - (pairs - U) : 0);
        const int axis = (int)((a.rotation.axis_low >> pair) & 1) | (int)((a.rotation.axis_high >> pair) & 1) << 1;
        for (int32_t first = wave * tokens_at_once; first < n; first += WAVES * tokens_at_once) {
            const int32_t t = first + (lane >> a.pair_bits);
            const bool is = t < n && pair < pairs;
            int32_t p = __shfl(pos, min(t, n - 1));
            if (a.rotation.positions && is) p = a.rotation.positions[axis * a.rotation.axis_stride + token0 + t];
            const CosSin x = cos_sin((double)p * frequency);
            const double c = x.c * a.rotation.magnitude, s = x.s * a.rotation.magnitude;
            auto put = [&](int at) {
                *(float2_t*)&turns[t][at] = (float2_t){(float)c, (float)s};
                if constexpr (E8) {
                    turns64[t][at] = c;
                    turns64[t][at + 1] = s;
                }
            };
            if (is && own) put(to);
            if (is && again) put(to_again);
        }
    }
    __syncthreads();

    auto work = [&](auto kind_, Rows& rows, const NormArgs& norm) {
        constexpr Kind KIND = decltype(kind_)::value;
        using A = std::conditional_t<E8 && KIND == KEYS, double, float>;
        // (its bits are looked at where they are needed: 16 masks kept from step to step would fill the scalar registers)
        unsigned bits = valid;
        if constexpr (RUNS == UNEVEN) asm volatile("" : "+v"(bits));
        auto counts_in = [&](int i, int e) { return RUNS != UNEVEN || ((bits >> (i * U + e)) & 1); };
        const int32_t t = rows.t, h = rows.h;
        const bool is = rows.is && (KIND == QUERIES ? counts[t] != 0 : row_at[t] >= 0);
        float out[2][U];
        if constexpr (KIND != VALUES) {
            A x[2][U];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < U; ++e) x[i][e] = value_of<T>(rows.x[i].x[e / 2], e & 1);
            if (norm.eps != 0.0f) {
                auto squares = [&]() {
                    A sum = 0;
#pragma unroll
                    for (int e = 0; e < U; ++e)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const A y = counts_in(i, e) ? x[i][e] : 0;
                            sum = __builtin_elementwise_fma(y, y, sum);
                        }
                    return over_row<ROW>(sum, [](A p, A q) { return p + q; });
                };
                A sum = squares(), by;
                if constexpr (std::is_same_v<A, double>) {
                    by = 1.0 / __builtin_sqrt(sum / a.cache.d + (double)norm.eps);
                } else {
                    float eps = norm.eps;
                    // Squares of bf16 values may be too large for 32 bits, or (with eps) so small that they lose bits or the root takes them for 0: such rows,
                    // and eps with them, are scaled by a power of two first, of which the quotient knows nothing.
                    if (__any(!(sum < 0x1p100f && (sum > 0x1p-80f || eps > 0x1p-70f)))) {
                        const float scale = sum <= 0x1p-80f ? (eps > 0x1p-70f ? 1.0f : 0x1p96f) : sum < 0x1p100f ? 1.0f : 0x1p-96f;
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int e = 0; e < U; ++e) x[i][e] *= scale;
                        sum = squares();
                        eps = eps * scale * scale;
                    }
                    by = __builtin_amdgcn_rsqf(sum * a.one_over_d + eps);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < U; ++e) x[i][e] *= by;
                if (norm.weight) {
                    auto weigh = [&](const float* w) {                     // (beyond a row's end there may be none)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if (inside[i]) {
#pragma unroll
                                for (int e = 0; e < U; ++e) x[i][e] *= w[start[i] + e];
                            }
                    };
                    if (norm.head_stride) weigh(norm.weight + h * norm.head_stride);
                    else weigh(weights[KIND]);
                }
            }
            auto turn = [&](A& p, A& q, A c, A s) {
                const A p_ = __builtin_elementwise_fma(p, c, -(q * s));
                q = __builtin_elementwise_fma(q, c, p * s);
                p = p_;
            };
            const A* table;
            if constexpr (std::is_same_v<A, double>) table = turns64[t];
            else table = turns[t];
            constexpr int CHUNK = MOST_PAIRS / PAIRS * 4;                  // values of a chunk of every lane
            if constexpr (RUNS != NEIGHBOURS) {
                if (j < turned) {
#pragma unroll
                    for (int e = 0; e < U; ++e) {
                        const A* const cs = table + (U == 1 ? j * 2 : e / 2 * CHUNK + j * 4 + (e & 1) * 2);
                        turn(x[0][e], x[1][e], cs[0], cs[1]);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < PAIRS; ++e) {
                        const A* const cs = table + e / 2 * CHUNK + (j + i * ROW) * 4 + (e & 1) * 2;
                        if ((j + i * ROW) * PAIRS + e < pairs) turn(x[i][2 * e], x[i][2 * e + 1], cs[0], cs[1]);
                    }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < U; ++e) {
                    if constexpr (std::is_same_v<A, double>) out[i][e] = to_odd(x[i][e]);
                    else out[i][e] = x[i][e];
                }
        }
        if constexpr (KIND == QUERIES || !E8) {
            if constexpr (KIND != VALUES) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < U; e += 2) rows.x[i].x[e / 2] = T::pack(out[i][e], U > 1 ? out[i][e + (U > 1)] : 0.0f);
            }
            char* const to = KIND == QUERIES ? a.q_out.base + token0 * a.q_out.token_bytes + from_first(a.q_out.token_bytes, a.q_out.head_bytes, t, h)
                                             : (KIND == KEYS ? a.cache.k : a.cache.v) + row_at[t] + from_first(0, a.cache.head_bytes, 0, h);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (!is || !inside[i]) continue;
                if (RUNS == UNEVEN && apart) {
#pragma unroll
                    for (int e = 0; e < U; ++e)
                        if (counts_in(i, e)) *(unsigned short*)(to + (start[i] + e) * 2) = (unsigned short)(rows.x[i].x[e / 2] >> (16 * (e & 1)));
                } else {
                    rows.x[i].store(to + start[i] * 2);
                }
            }
        } else {
            static_assert(U == 8 || !E8);
            if constexpr (KIND == VALUES) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < U; ++e) out[i][e] = value_of<T>(rows.x[i].x[e / 2], e & 1);
            }
            unsigned top = 0;                          // bits of the largest finite magnitude
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < U; ++e) {
                    const unsigned u = __builtin_bit_cast(unsigned, out[i][e]) & 0x7fffffffu;
                    if (u < 0x7f800000u && counts_in(i, e)) top = max(top, u);
                }
            top = over_row<ROW>(top, [](unsigned p, unsigned q) { return max(p, q); });
            const int byte = scale_byte(top);
            char* const to = (KIND == KEYS ? a.cache.k : a.cache.v) + row_at[t] + from_first(0, a.cache.head_bytes, 0, h);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                unsigned codes[2];
#pragma unroll
                for (int e = 0; e < U; e += 4) {
                    const float four[4] = {out[i][e], out[i][e + 1], out[i][e + 2], out[i][e + 3]};
                    codes[e / 4] = four_codes(four, byte);
                }
                if (!is || !inside[i]) continue;
                if (RUNS == UNEVEN && apart) {
#pragma unroll
                    for (int e = 0; e < U; ++e)
                        if (counts_in(i, e)) *(uint8_t*)(to + start[i] + e) = (uint8_t)(codes[e / 4] >> (8 * (e & 3)));
                } else {
                    *(std::conditional_t<RUNS == UNEVEN, uint2_anywhere, uint2_t>*)(to + start[i]) = (uint2_t){codes[0], codes[1]};
                }
            }
            if (is && j == 0) (KIND == KEYS ? a.cache.k_scale : a.cache.v_scale)[scale_at[t] + (int64_t)h * a.cache.page.divisor] = (uint8_t)byte;
        }
    };
    while (step < steps) {
        Rows next;
        load(step + stride, next);
        if (step < q_steps) work(std::integral_constant<Kind, QUERIES>{}, now, a.q_norm);
        else if (step < q_steps + kv_steps) work(std::integral_constant<Kind, KEYS>{}, now, a.k_norm);
        else work(std::integral_constant<Kind, VALUES>{}, now, a.k_norm);
        now = next;
        step += stride;
    }
}

}  // namespace gorgo
