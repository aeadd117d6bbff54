// Attention of one new token of each sequence over the pages of the cache.
#pragma once
#include "attention_common.h"

namespace gorgo {

// A row is a query head of one (sequence, cache head) pair, up to 16 * NB of them side by side.  Bound by the bytes of the cache:
// every key and value is read once.  A workgroup's four wavefronts stream disjoint runs of keys, 8 KB of keys and 8 KB of values at
// a time, in loads of whole rows (1 KB of neighbouring bytes each) that are in flight while the 16 KB before them are worked on.
// The products are the matrix unit's (16x16x32, S^T = K Q^T and O^T = V^T P^T as for prompts), whose operands want other shapes
// than rows: keys and then values pass through 8 KB of LDS that belongs to the wavefront alone, so nothing waits for anybody.
// 8-bit values are widened behind LDS; a key's power of two goes along with that, a value's is multiplied onto its weight.
//
// Work is dealt out in units (the keys of one step of a workgroup): all pairs' units stand in one line, and each workgroup takes
// an equal run of it, whatever the lengths are.  A pair that lies within one run is finished there.  Of a pair that several
// runs share each leaves a partial row, and the workgroup that leaves the last one joins them.
constexpr int TOKEN_THREADS = TOKEN_WAVES * 64;

struct KeySpan {
    int32_t lo, hi, sinks;               // keys [lo, hi) that the token sees, and [0, sinks), sinks <= lo
};
template <bool SINKS>
__device__ inline KeySpan keys_seen(const AttendArgs& a, int32_t s) {
    const int32_t length = length_of(a.batch, s), hi = min(length, a.batch.capacity);
    const int32_t lo = a.window ? min(max(0, length - a.window), hi) : 0;
    return {lo, hi, SINKS ? min(a.sinks, lo) : 0};
}
// Units of the sinks, but for one that holds keys of the window too.
template <int UNIT>
__device__ inline int32_t sink_units(KeySpan k) { return min((k.sinks + UNIT - 1) / UNIT, k.lo / UNIT); }
// Units of a pair: the sinks', and from the one that its window's first key lies in; one at least, so that somebody writes its rows.
template <int UNIT, bool SINKS>
__device__ inline int32_t units_of(KeySpan k) {
    return max(1, (k.hi + UNIT - 1) / UNIT - k.lo / UNIT + (SINKS ? sink_units<UNIT>(k) : 0));
}

// Sums over the lanes up to each.
__device__ inline int32_t prefix_sum(int32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);       // one, two, four and eight lanes to the right in a row of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // a row's last lane to the next row, then the half's
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// Quotient of uniform numbers that mostly fit 32 bits.
__device__ inline int64_t divide(int64_t x, int64_t by) {
    if (((x | by) >> 32) == 0) return (uint32_t)x / (uint32_t)by;
    return x / by;
}

// How the line of units is dealt out.
struct Shares {
    int64_t units, each, more;           // workgroups get `each` units, the first `more` of them one more
    int32_t groups;
    __device__ int64_t begin(int64_t group) const { return group * each + min(group, more); }
    __device__ int32_t holder(int64_t unit) const {
        const int64_t first = more * (each + 1);
        return (int32_t)(unit < first ? divide(unit, each + 1) : more + divide(unit - first, each));
    }
};

// A workgroup's partial rows of a pair (values, then maxima and sums): of the piece that its run begins with, or of a later one,
// which can only be its last.
template <int DP>
__device__ inline float* partial_of(const AttendArgs& a, int32_t group, bool later) {
    const int64_t size = ((int64_t)a.group.divisor * (DP + 2) + 3) & ~(int64_t)3;
    return a.partial + ((int64_t)group * 2 + later) * size;
}

// Partial values go from one workgroup to another past the caches that only some of the compute units share: stores and loads of
// agent scope, and a wait until they have arrived before they are counted.  (Fences instead would write back and drop all that
// such a cache holds.)
__device__ inline void give(float* to, float x, float y) {
    __hip_atomic_store((uint64_t*)to, __builtin_bit_cast(uint64_t, (float2_t){x, y}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline float2_t take(const float* from) {
    return __builtin_bit_cast(float2_t, __hip_atomic_load((const uint64_t*)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ inline void given() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// Wavefront-private LDS tile: rows of BYTES bytes in chunks of 16 that are moved within their row so that the lanes of one read
// touch every bank once: sixteen rows' same chunk (keys), or the rows and chunks of a transposing read (values: four rows of 16 bits,
// eight of 8 bits that are four and four, 16 apart).  The patterns are exclusive-ors of row bits: steps of rows or chunks by powers
// of two are exclusive-ors and sums with constants.
template <bool E8, int BYTES>
struct TokenTile {
    static constexpr int CHUNKS = BYTES / 16;
    static constexpr __device__ int k_turn(int row) { return BYTES == 256 ? row & 15 : BYTES == 128 ? (row >> 1) & 7 : (row >> 2) & 3; }
    static constexpr __device__ int v_turn(int row) {
        if (BYTES == 256) return (row & 3) << 2 | ((row >> 2) & 3);
        if (BYTES == 128 && !E8) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
        if (BYTES == 128) return ((row >> 1) & 1) | ((row >> 4) & 1) << 1 | ((row >> 2) & 1) << 2;
        return ((row >> 4) & 1) | ((row >> 2) & 1) << 1;
    }
    static __device__ int k_at(int row, int chunk) { return row * BYTES + ((chunk ^ k_turn(row)) << 4); }
    static __device__ int v_at(int row, int chunk) { return row * BYTES + ((chunk ^ v_turn(row)) << 4); }
};

// ALIGNED: the keys of a wavefront's step lie in one page.  SINKS: some first keys stay visible beside a window; units are numbered without those between
// (48 sequences with a window of 8192 and 64 sinks, 8 bits: 124.3 us, 5.6 TB/s; 127.2 with the steps loaded of which no key is seen).
template <class T, bool E8, int DP, int NB, bool ALIGNED, bool SINKS>
__global__ __launch_bounds__(TOKEN_THREADS, 2) void attend_token_kernel(AttendArgs a) {
    constexpr int KEYS = token_keys(E8), UNIT = KEYS * TOKEN_WAVES, NK = KEYS / 16;
    constexpr int STEPS = DP / 32, BLOCKS = DP / 16;
    constexpr int ROW = DP * (E8 ? 1 : 2);                                 // bytes
    using L = TokenTile<E8, ROW>;
    // Accumulators of 32 rows of 128 leave few registers.  What follows from a lane's number is computed again in every step and behind the loop, from copies
    // that the compiler does not see through: kept through it, it took up to 9 registers more than there are in 16 bits and 28 to 50 in 8, in scratch
    // memory.  48 sequences of 16,000 keys, 64 query heads over two cache heads: 162 us (163 then) in pages of 64, 161 (176) of 48, in 8 bits 103 (114)
    // and 109 (128).
    constexpr bool TIGHT = NB == 2 && DP == 128;
    constexpr int ROWS_A_LOAD = 64 / L::CHUNKS, LOADS = KEYS / ROWS_A_LOAD;
    constexpr int WAVE_LDS = KEYS * ROW > 16 * DP * 4 + 128 ? KEYS * ROW : 16 * DP * 4 + 128;
    __shared__ __attribute__((aligned(256))) char lds[TOKEN_WAVES * WAVE_LDS];
    __shared__ int32_t last_one;

    const int wave = uniform(threadIdx.x >> 6);
    int lane = threadIdx.x & 63, quarter = lane >> 4, l16 = lane & 15;
    const int32_t heads = a.cache.heads, G = a.group.divisor;
    char* const mine = lds + wave * WAVE_LDS;

    // this workgroup's run of units, and the sequence and head that it begins in
    Shares share;
    {
        int64_t all = 0;
        for (int32_t base = 0; base < a.batch.S; base += 64) {
            const int32_t x = base + lane < a.batch.S ? units_of<UNIT, SINKS>(keys_seen<SINKS>(a, base + lane)) : 0;
            all += (uint32_t)__builtin_amdgcn_readlane(prefix_sum(x), 63);
        }
        share.units = all * heads;
        share.groups = (int32_t)min<int64_t>(a.splits, share.units);      // (so that each has one at least)
        share.each = divide(share.units, share.groups);
        share.more = share.units - share.each * share.groups;
    }
    const int32_t group = blockIdx.x;
    if (group >= share.groups) return;
    const int64_t run = share.begin(group), run_end = share.begin(group + 1);
    int64_t at = run, before = 0;                                          // `before`: units of the sequences before s
    int32_t s = 0;
    for (int32_t base = 0; base < a.batch.S; base += 64) {
        const int32_t x = base + lane < a.batch.S ? units_of<UNIT, SINKS>(keys_seen<SINKS>(a, base + lane)) : 0;
        const int32_t upto = prefix_sum(x);
        const int64_t chunk = (int64_t)(uint32_t)__builtin_amdgcn_readlane(upto, 63) * heads;
        if (before + chunk <= at) {
            before += chunk;
            continue;
        }
        const int n = __popcll(__ballot(before + (int64_t)upto * heads <= at));      // sequences that end at or before `at`
        s = base + n;
        before += (int64_t)(__builtin_amdgcn_readlane(upto, n) - __builtin_amdgcn_readlane(x, n)) * heads;
        break;
    }

    while (at < run_end) {
        KeySpan seen = keys_seen<SINKS>(a, s);
        seen = {uniform(seen.lo), uniform(seen.hi), uniform(seen.sinks)};
        const int32_t n_units = units_of<UNIT, SINKS>(seen);
        const int32_t head = (int32_t)divide(at - before, n_units);
        const int64_t pair = before + (int64_t)head * n_units;             // its first unit
        const int32_t u0 = (int32_t)(at - pair), u1 = (int32_t)min<int64_t>(n_units, run_end - pair);
        const bool whole = u0 == 0 && u1 == n_units;
        // SINKS: keys are counted without the units that lie between the sinks' and the window's
        const int32_t sinks_end = SINKS ? sink_units<UNIT>(seen) * UNIT : 0, gap = SINKS ? seen.lo / UNIT * UNIT - sinks_end : 0;
        auto place = [&](int32_t key) { return SINKS && key >= sinks_end ? key + gap : key; };
        const int32_t unit0 = SINKS ? 0 : seen.lo / UNIT;
        // keys of this piece, and this wavefront's first ones
        const int32_t lo = seen.lo, hi = min(seen.hi - gap, (unit0 + u1) * UNIT);
        const int32_t first_key = SINKS ? 0 : lo, last_key = SINKS ? seen.hi - 1 : hi - 1;      // rows that exist
        int32_t key0 = (unit0 + u0) * UNIT + wave * KEYS;

        // Loads.  Load i takes rows i * ROWS_A_LOAD on, a lane 16 bytes of one.  Every load is done, from a row that exists; what must
        // be left out is masked, and values of such rows made zero on their way to LDS (their weight is 0, but 0 times an infinity
        // is not).
        const int chunk = lane % L::CHUNKS;
        const bool inside = chunk * 16 < a.cache.d * (E8 ? 1 : 2);
        int row_of = lane / L::CHUNKS;
        const int64_t head_at = head * a.cache.head_bytes;
        const uint32_t lane_at = (uint32_t)(lane / L::CHUNKS) * (uint32_t)a.cache.token_bytes + (inside ? chunk * 16 : 0);
        uint4_t k[LOADS], v[LOADS];
        unsigned k_byte[NK], v_bytes[NK];                                  // exponents: of key 16 n + l16, of keys 16 n + 4 quarter on
        int32_t page = -1;                                                 // ALIGNED: of the step's keys; else of key `lane` of them
        auto find_page = [&](int32_t key) {
            if (key >= hi) return;
            if constexpr (ALIGNED) page = uniform(page_of(a.batch, a.cache, s, quotient(a.cache.page, place(key))));
            else page = page_of(a.batch, a.cache, s, quotient(a.cache.page, max(first_key, min(place(key) + lane % KEYS, last_key))));
        };
        int64_t row_at = 0, scale_at = 0;                                  // ALIGNED: of the step's first key; else of key `lane`
        uint64_t next_held = 0;                                            // which keys of the step exist
        auto find_rows = [&](int32_t key_) {
            const int32_t key = place(key_);
            if constexpr (ALIGNED) {
                const int32_t slot = key - quotient(a.cache.page, key) * a.cache.page.divisor, id = max(page, 0);
                row_at = id * a.cache.page_bytes + slot * a.cache.token_bytes;
                scale_at = ((int64_t)id * heads + head) * a.cache.page.divisor + slot;
                const uint64_t below = hi - key_ >= KEYS ? ~(uint64_t)0 : ((uint64_t)1 << (hi - key_)) - 1;
                uint64_t from = lo <= key ? ~(uint64_t)0 : lo - key >= 64 ? 0 : ~(uint64_t)0 << (lo - key);
                if (SINKS && seen.sinks > key) from |= seen.sinks - key >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << (seen.sinks - key)) - 1;
                next_held = page >= 0 ? below & from : 0;
            } else {
                const int32_t mine_ = key + lane % KEYS, row_key = max(first_key, min(mine_, last_key)), id = max(page, 0);
                const int32_t slot = row_key - quotient(a.cache.page, row_key) * a.cache.page.divisor;
                row_at = id * a.cache.page_bytes + slot * a.cache.token_bytes;
                scale_at = ((int64_t)id * heads + head) * a.cache.page.divisor + slot;
                next_held = __ballot(page >= 0 && row_key == mine_ && (!SINKS || mine_ >= lo || mine_ < seen.sinks));
            }
            if (KEYS == 32) next_held |= ~(uint64_t)0 << 32;
        };
        auto load = [&](const char* from, uint4_t (&x)[LOADS]) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                if constexpr (ALIGNED)
                    x[i] = __builtin_nontemporal_load((const uint4_t*)(from + (row_at + head_at + i * ROWS_A_LOAD * a.cache.token_bytes) + lane_at));
                else
                    x[i] = __builtin_nontemporal_load((const uint4_t*)(from + (head_at + __shfl((long long)row_at, i * ROWS_A_LOAD + row_of)) + (inside ? chunk * 16 : 0)));
            }
        };
        // (a unit of sinks, and the window's first one, may hold no key for some of the wavefronts: what is in the registers then is left out like
        // any other key that is not seen)
        auto any_held = [&]() { return (KEYS == 32 ? (uint32_t)next_held : next_held) != 0; };
        auto load_scales = [&]() {
            if constexpr (E8) {
#pragma unroll
                for (int n = 0; n < NK; ++n) {
                    if constexpr (ALIGNED) {
                        k_byte[n] = a.cache.k_scale[scale_at + n * 16 + l16];
                        v_bytes[n] = *(const unsigned*)(a.cache.v_scale + scale_at + n * 16 + quarter * 4);
                    } else {
                        k_byte[n] = a.cache.k_scale[__shfl((long long)scale_at, n * 16 + l16)];
                        v_bytes[n] = 0;
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            v_bytes[n] |= (unsigned)a.cache.v_scale[__shfl((long long)scale_at, n * 16 + quarter * 4 + r)] << (8 * r);
                    }
                }
            }
        };

        find_page(key0);
        if (key0 < hi) {
            find_rows(key0);
            if (!SINKS || any_held()) {
                load(a.cache.k, k);
                load(a.cache.v, v);
                load_scales();
            } else {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) k[i] = v[i] = (uint4_t){0, 0, 0, 0};
#pragma unroll
                for (int n = 0; n < NK; ++n) k_byte[n] = v_bytes[n] = 0;
            }
        }
        // queries: row n * 16 + l16, in the order of values in which the keys are read from LDS
        uint4_t q[NB][STEPS];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int d = E8 ? (i / 2) * 64 + quarter * 16 + (i & 1) * 8 : i * 32 + quarter * 8;
                q[n][i] = (uint4_t){0, 0, 0, 0};
                if (n * 16 + l16 < G && d < a.cache.d)
                    q[n][i] = *(const uint4_t*)(a.q.base + s * a.q.token_bytes + (head * G + n * 16 + l16) * a.q.head_bytes + d * 2);
            }
        float4_t o[NB][BLOCKS];
        float top[NB], sum[NB];
        bool far[NB];                                                      // some row's maximum is far out
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            top[n] = NO_MAX;
            far[n] = false;
            sum[n] = 0.0f;
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) o[n][i] = (float4_t)(0.0f);
        }
        find_page(key0 + UNIT);

        // LDS addresses of this lane: a load's row and chunk; a key's chunk; a row and half a chunk of a transposing read.  (Kept
        // from being taken apart: the 32 sums and exclusive-ors with constants cost less in the loop than registers before it.)
        int k_to = L::k_at(row_of, chunk), v_to = L::v_at(row_of, chunk), k_from = L::k_at(l16, quarter);
        const int v_row = E8 ? quarter * 4 + ((l16 >> 1) & 3) + (l16 >> 3) * 16 : quarter * 4 + l16 / 4;
        int v_from = L::v_at(v_row, E8 ? 0 : (lane >> 1) & 1) + (lane & 1) * 8;

        for (; key0 < hi; key0 += UNIT) {
            asm volatile("" : "+v"(k_to), "+v"(v_to), "+v"(k_from), "+v"(v_from));
            if constexpr (TIGHT) asm volatile("" : "+v"(lane), "+v"(row_of), "+v"(quarter), "+v"(l16));
            const uint64_t held = next_held;
            const bool gaps = ~held != 0, more = key0 + UNIT < hi;
            if (a.cache.d < DP) {                                          // (beyond the row's end stand copies of its beginning)
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
                    if (!inside) k[i] = (uint4_t){0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < LOADS; ++i) *(uint4_t*)(mine + (k_to ^ (L::k_turn(i * ROWS_A_LOAD) << 4)) + i * ROWS_A_LOAD * ROW) = k[i];
            unsigned v_now[NK];
            float k_power[NK];
            if constexpr (E8) {
#pragma unroll
                for (int n = 0; n < NK; ++n) {
                    v_now[n] = v_bytes[n];
                    k_power[n] = power_of(k_byte[n]);
                }
            }
            if (more) {
                find_rows(key0 + UNIT);
                if (!SINKS || any_held()) load(a.cache.k, k);
            }
            float4_t sc[NB][NK];
#pragma unroll
            for (int n = 0; n < NK; ++n) {
                uint4_t x[STEPS];
#pragma unroll
                for (int i = 0; i < STEPS; i += E8 ? 2 : 1) {
                    const uint4_t raw = *(const uint4_t*)(mine + (k_from ^ (L::k_turn(n * 16) << 4) ^ ((E8 ? i / 2 : i) << 6)) + n * 16 * ROW);
                    if constexpr (E8) {
                        x[i] = widen8(raw.x, raw.y, k_power[n]);
                        x[i + 1] = widen8(raw.z, raw.w, k_power[n]);
                    } else {
                        x[i] = raw;
                    }
                }
#pragma unroll
                for (int m = 0; m < NB; ++m) {
                    sc[m][n] = (float4_t)(0.0f);
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) sc[m][n] = T::mfma16(as_x8<T>(x[i]), as_x8<T>(q[m][i]), sc[m][n]);
                }
            }
            // values take the keys' place in LDS
            if (gaps) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
                    if (!((held >> (i * ROWS_A_LOAD + row_of)) & 1)) v[i] = (uint4_t){0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < LOADS; ++i) *(uint4_t*)(mine + (v_to ^ (L::v_turn(i * ROWS_A_LOAD) << 4)) + i * ROWS_A_LOAD * ROW) = v[i];
            if (more) {
                if (!SINKS || any_held()) {
                    load(a.cache.v, v);
                    load_scales();
                }
                find_page(key0 + 2 * UNIT);
            }
            // lane: keys 16 n + 4 * quarter + r
            if (gaps) {
                const uint64_t mine_ = held >> (quarter * 4);
#pragma unroll
                for (int n = 0; n < NK; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!((mine_ >> (n * 16 + r)) & 1)) {
                            // (the byte that lies there may stand for an infinity, and its weight is 0: it becomes 0 too)
                            if constexpr (E8) v_now[n] &= ~(0xffu << (8 * r));
#pragma unroll
                            for (int m = 0; m < NB; ++m) sc[m][n][r] = -__builtin_inff();
                        }
            }
            uint4_t p[NB][NK / 2];
#pragma unroll
            for (int m = 0; m < NB; ++m) {
                float most = sc[m][0][0];
#pragma unroll
                for (int n = 0; n < NK; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) most = fmaxf(most, sc[m][n][r]);
                most *= a.scale_log2;
                if (__any(most - top[m] > T::RAISE + T::SLACK)) {
                    const float now = renewed<T>(top[m], quarters_max(most)), by = exp2_(top[m] - now);
                    top[m] = now;
                    far[m] = far_out(now);
                    sum[m] *= by;
#pragma unroll
                    for (int i = 0; i < BLOCKS; ++i) o[m][i] *= by;
                }
                float from_top = top[m], scale = a.scale_log2;
                if (far[m]) {
#pragma unroll
                    for (int n = 0; n < NK; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) sc[m][n][r] = sc[m][n][r] * a.scale_log2 - from_top;
                    from_top = 0.0f;
                    scale = 1.0f;
                }
#pragma unroll
                for (int n = 0; n < NK; ++n)
#pragma unroll
                    for (int r = 0; r < 4; r += 2) {
                        float x = exp2_(__builtin_fmaf(sc[m][n][r], scale, -from_top));
                        float y = exp2_(__builtin_fmaf(sc[m][n][r + 1], scale, -from_top));
                        sum[m] += x + y;
                        if constexpr (E8) {
                            x *= power_of((v_now[n] >> (8 * r)) & 0xffu);
                            y *= power_of((v_now[n] >> (8 * r + 8)) & 0xffu);
                        }
                        p[m][n / 2][(n & 1) * 2 + r / 2] = T::pack(x, y);
                    }
            }
#pragma unroll
            for (int n = 0; n < NK / 2; ++n)
#pragma unroll
                for (int i = 0; i < BLOCKS; ++i) {
                    uint4_t x;
                    if constexpr (E8) {
                        const uint2_t raw = column8(mine + (v_from ^ (L::v_turn(n * 32) << 4) ^ (i << 4)) + n * 32 * ROW);
                        x = widen8(raw.x, raw.y, 1.0f);
                    } else {
                        const uint2_t y = column4(mine + (v_from ^ (i << 5))), z = column4(mine + (v_from ^ (L::v_turn(16) << 4) ^ (i << 5)) + 16 * ROW);
                        x = (uint4_t){y.x, y.y, z.x, z.y};
                    }
#pragma unroll
                    for (int m = 0; m < NB; ++m) o[m][i] = T::mfma16(as_x8<T>(x), as_x8<T>(p[m][n]), o[m][i]);
                }
        }

        // The four wavefronts' rows are joined through LDS, 16 at a time: row l16, values i * 16 + 4 * quarter + r; their maxima and sums
        // behind them.
        float* const my_rows = (float*)mine;
        int thread = threadIdx.x;
        if constexpr (TIGHT) asm volatile("" : "+v"(thread), "+v"(quarter), "+v"(l16));
        const int out_row = thread / (DP / 8), out_d = (thread % (DP / 8)) * 8;
        auto finish = [&](int m, bool final) {
            __syncthreads();
            const int g = m * 16 + out_row;
            if (out_row < 16 && g < G) {
                float t[TOKEN_WAVES], most = NO_MAX, all = 0.0f, x[8] = {};
#pragma unroll
                for (int w = 0; w < TOKEN_WAVES; ++w) {
                    t[w] = ((const float*)(lds + w * WAVE_LDS))[16 * DP + out_row];
                    most = fmaxf(most, t[w]);
                }
#pragma unroll
                for (int w = 0; w < TOKEN_WAVES; ++w) {
                    const float* const from = (const float*)(lds + w * WAVE_LDS);
                    const float by = exp2_(t[w] - most);
                    all += by * from[16 * DP + 16 + out_row];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] += by * from[out_row * DP + out_d + e];
                }
                if (final) {
                    const float norm = all != 0.0f ? 1.0f / all : 0.0f;
                    if (out_d < a.cache.d)
                        *(uint4_t*)(a.out.base + s * a.out.token_bytes + (head * G + g) * a.out.head_bytes + out_d * 2) =
                            (uint4_t){T::pack(x[0] * norm, x[1] * norm), T::pack(x[2] * norm, x[3] * norm), T::pack(x[4] * norm, x[5] * norm),
                                      T::pack(x[6] * norm, x[7] * norm)};
                    if (a.lse && out_d == 0)
                        a.lse[(int64_t)s * a.q_heads + head * G + g] = log_of_sum<T>(most, all);
                } else {
                    float* const part = partial_of<DP>(a, group, at > run);
#pragma unroll
                    for (int e = 0; e < 8; e += 2) give(part + g * DP + out_d + e, x[e], x[e + 1]);
                    if (out_d == 0) give(part + G * DP + g * 2, most, all);
                }
            }
            __syncthreads();
        };
#pragma unroll
        for (int m = 0; m < NB; ++m) {
            const float total = quarters_sum(sum[m]);
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) *(float4_t*)(my_rows + l16 * DP + i * 16 + quarter * 4) = o[m][i];
            if (quarter == 0) {
                my_rows[16 * DP + l16] = top[m];
                my_rows[16 * DP + 16 + l16] = total;
            }
            finish(m, whole);
        }
        if (!whole) {
            const int32_t w0 = share.holder(pair), w1 = share.holder(pair + n_units - 1);
            uint32_t* const count = a.counters + w0;                       // (only the last pair of a run goes on in the next one)
            given();
            __syncthreads();
            if (threadIdx.x == 0) last_one = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(w1 - w0);
            __syncthreads();
            if (last_one) {
                if (threadIdx.x == 0) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // for the next call
                // Each wavefront joins every fourth piece, four rows at a time, sixteen pieces at a time: a quarter's lanes take a piece's
                // maximum and sum each, then all of them the values of one piece after the other, which no load waits for.  (Eight pairs of
                // 30,000 keys, 64 pieces each: 30 us in all; one piece after the other, each a step of a sum, 57 us.)
                for (int m = 0; m < NB; ++m) {
                    for (int r = quarter; r < 16; r += 4) {
                        const int g = m * 16 + r;
                        float most = NO_MAX, all = 0.0f;
                        float2_t x[DP / 32] = {};
                        if (g < G) {
                            for (int32_t first = w0 + wave; first <= w1; first += 16 * TOKEN_WAVES) {
                                const int32_t w = first + l16 * TOKEN_WAVES, w_ = min(w, w1);
                                float2_t stats = take(partial_of<DP>(a, w_, share.begin(w_) < pair) + G * DP + g * 2);
                                if (w > w1) stats = {NO_MAX, 0.0f};
                                float now = fmaxf(most, stats.x);
#pragma unroll
                                for (int step = 1; step < 16; step <<= 1) now = fmaxf(now, __shfl_xor(now, step));
                                const float old = exp2_(most - now), mine_by = w > w1 ? 0.0f : exp2_(stats.x - now);
                                float part_sum = stats.y * mine_by;
#pragma unroll
                                for (int step = 1; step < 16; step <<= 1) part_sum += __shfl_xor(part_sum, step);
                                most = now;
                                all = all * old + part_sum;
#pragma unroll
                                for (int e = 0; e < DP / 32; ++e) x[e] *= old;
#pragma unroll
                                for (int i0 = 0; i0 < 16; i0 += 8) {
                                    if (first + i0 * TOKEN_WAVES > w1) break;
                                    float2_t y[8][DP / 32];
#pragma unroll
                                    for (int i = 0; i < 8; ++i) {
                                        const int32_t from_w = min(first + (i0 + i) * TOKEN_WAVES, w1);
                                        const float* const from = partial_of<DP>(a, from_w, share.begin(from_w) < pair) + g * DP + l16 * 2;
#pragma unroll
                                        for (int e = 0; e < DP / 32; ++e) y[i][e] = take(from + e * 32);
                                    }
#pragma unroll
                                    for (int i = 0; i < 8; ++i) {
                                        const float by = __shfl(mine_by, quarter * 16 + i0 + i);
                                        if (first + (i0 + i) * TOKEN_WAVES <= w1) {
#pragma unroll
                                            for (int e = 0; e < DP / 32; ++e) x[e].x += y[i][e].x * by, x[e].y += y[i][e].y * by;
                                        }
                                    }
                                }
                            }
                        }
#pragma unroll
                        for (int e = 0; e < DP / 32; ++e) *(float2_t*)(my_rows + r * DP + l16 * 2 + e * 32) = x[e];
                        if (l16 == 0) {
                            my_rows[16 * DP + r] = most;
                            my_rows[16 * DP + 16 + r] = all;
                        }
                    }
                    finish(m, true);
                }
            }
        }
        at = pair + u1;
        if (at == before + (int64_t)n_units * heads) {
            before = at;
            ++s;
        }
    }
}

}  // namespace gorgo
