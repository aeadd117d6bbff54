// Attention of one new token of each sequence over the pages of the cache.
#pragma once
#include "attention_common.h"

namespace gorgo {

// A row is a query head of one (sequence, cache head) pair, up to 16 * NB of them side by side.  Bound by the bytes of the cache:
// every key and value is read once, and a workgroup's four wavefronts stream disjoint runs of 32 keys straight into registers.
// The products are the matrix unit's (16x16x32, S^T = K Q^T and O^T = V^T P^T as for prompts); only V passes through LDS, for
// the transposing read, in a part that belongs to the wavefront alone, so nothing waits for anybody until the end.
//
// Work is dealt out in units of UNIT keys: all pairs' units stand in one line, and each of the workgroups takes an equal run of
// it, whatever the lengths are.  A pair that lies within one run is finished there; what begins or ends in the middle of a run
// leaves a partial row, at most two a workgroup, and a second kernel joins them.
constexpr int TOKEN_THREADS = TOKEN_WAVES * 64;
constexpr int UNITS_A_GROUP = 8;         // units that make a workgroup worth while

struct KeySpan {
    int32_t lo, hi;                      // keys [lo, hi) that the token sees
};
__device__ inline KeySpan keys_seen(const AttendArgs& a, int32_t s) {
    const int32_t length = a.batch.lengths[s], hi = max(0, min(length, a.batch.capacity));
    return {a.window ? min(max(0, length - a.window), hi) : 0, hi};
}
// Units of a pair of sequence s: from the unit that its first key lies in; one at least, so that somebody writes its rows.
__device__ inline int32_t units_of(const AttendArgs& a, int32_t s) {
    const KeySpan k = keys_seen(a, s);
    return max(1, (k.hi + UNIT - 1) / UNIT - k.lo / UNIT);
}

__device__ inline int32_t wave_sum(int32_t x) {
#pragma unroll
    for (int step = 1; step < 64; step <<= 1) x += __shfl_xor(x, step);
    return x;
}
__device__ inline int64_t all_units(const AttendArgs& a) {
    const int lane = threadIdx.x & 63;
    int64_t all = 0;
    for (int32_t at = 0; at < a.batch.S; at += 64) all += wave_sum(at + lane < a.batch.S ? units_of(a, at + lane) : 0);
    return all * a.cache.heads;
}
// Workgroups that share the units: each pair has one of its own, or as many as its units are worth.
__device__ inline int32_t groups_at_work(const AttendArgs& a, int64_t units) {
    return (int32_t)min<int64_t>(a.splits, max<int64_t>((int64_t)a.batch.S * a.cache.heads, units / UNITS_A_GROUP));
}
__device__ inline int64_t run_begin(int64_t units, int32_t groups, int32_t group) { return units * group / groups; }

// A workgroup's partial rows of a pair (a row: DP values, a maximum and a sum): of the piece that its run begins with, or of a later
// one, which can only be its last.
template <int DP>
__device__ inline float* partial_of(const AttendArgs& a, int32_t group, bool later) {
    return a.partial + ((int64_t)group * 2 + later) * a.group.divisor * (DP + 2);
}

template <int DP>
__device__ inline int token_v_at(int row, int chunk) {
    const int turn = DP == 128 ? ((row & 3) << 2 | ((row >> 2) & 3)) : (((row >> 1) & 1) << 2 | ((row >> 2) & 3));
    return row * (DP * 2) + ((chunk ^ turn) << 4);
}

// ALIGNED: 32 keys lie in one page.
template <class T, bool E8, int DP, int NB, bool ALIGNED>
__global__ __launch_bounds__(TOKEN_THREADS, NB == 1 ? 3 : 2) void attend_token_kernel(AttendArgs a) {
    constexpr int KEYS = TOKEN_KEYS, STEPS = DP / 32, BLOCKS = DP / 16;
    constexpr int LOADS = E8 ? DP / 64 : DP / 32;                          // 16-byte loads of a lane for a row's quarter
    constexpr int WAVE_LDS = KEYS * DP * 2 > 16 * DP * 4 + 128 ? KEYS * DP * 2 : 16 * DP * 4 + 128;
    __shared__ __attribute__((aligned(256))) char lds[TOKEN_WAVES * WAVE_LDS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, l16 = lane & 15;
    const int32_t heads = a.cache.heads, G = a.group.divisor;
    const int64_t units = all_units(a);
    const int32_t groups = groups_at_work(a, units), group = blockIdx.x;
    if (group >= groups) return;
    int64_t at = run_begin(units, groups, group);
    const int64_t run_end = run_begin(units, groups, group + 1);
    char* const mine = lds + wave * WAVE_LDS;
    // this lane's first row and chunk of V in LDS, written and read (steps along a row are exclusive-ors, 16 rows a sum)
    const int to_lds = token_v_at<DP>(l16, E8 ? quarter * 2 : quarter);
    const int from_lds = token_v_at<DP>(quarter * 4 + l16 / 4, (lane >> 1) & 1) + (lane & 1) * 8;

    // the sequence that the run begins in
    int32_t s = 0, n_units = 0;
    int64_t before = 0;                                                    // units of the sequences before it
    for (int32_t base = 0; base < a.batch.S; base += 64) {
        int32_t x = base + lane < a.batch.S ? units_of(a, base + lane) : 0;
        const int32_t chunk = wave_sum(x);
        if (before + (int64_t)chunk * heads <= at) {
            before += (int64_t)chunk * heads;
            continue;
        }
        int32_t upto = x;                                                  // inclusive prefix sums over the lanes
#pragma unroll
        for (int step = 1; step < 64; step <<= 1) {
            const int32_t y = __shfl_up(upto, step);
            if (lane >= step) upto += y;
        }
        const int n = __popcll(__ballot(before + (int64_t)upto * heads <= at));      // sequences that end at or before `at`
        s = base + n;
        before += (int64_t)(__shfl(upto, n) - __shfl(x, n)) * heads;
        break;
    }
    s = __builtin_amdgcn_readfirstlane(s);

    const int64_t run = at;
    while (at < run_end) {
        const KeySpan seen = keys_seen(a, s);
        n_units = units_of(a, s);
        const int32_t head = (int32_t)((at - before) / n_units);
        const int64_t pair = before + (int64_t)head * n_units;             // its first unit
        const int32_t u0 = (int32_t)(at - pair), u1 = (int32_t)min<int64_t>(n_units, run_end - pair);
        const bool whole = u0 == 0 && u1 == n_units;
        const int32_t unit0 = seen.lo / UNIT;
        // keys of this piece, and this wavefront's first ones
        const int32_t lo = seen.lo, hi = min(seen.hi, (unit0 + u1) * UNIT);
        const int32_t key_begin = (unit0 + u0) * UNIT + wave * KEYS;

        // two rows of the cache a lane: keys l16 and 16 + l16 of the 32
        const char* const k_head = a.cache.k + head * a.cache.head_bytes + quarter * 16;
        const char* const v_head = a.cache.v + head * a.cache.head_bytes + quarter * 16;
        uint4_t k[2][LOADS], v[2][LOADS];
        unsigned ks[2], vs[2];
        int32_t page[2];
        auto find_pages = [&](int32_t key0) {
            if (key0 >= hi) return;
            if constexpr (ALIGNED) {
                page[0] = page[1] = page_of(a.batch, a.cache, s, quotient(a.cache.page, key0));
            } else {
#pragma unroll
                for (int n = 0; n < 2; ++n) page[n] = page_of(a.batch, a.cache, s, quotient(a.cache.page, max(lo, min(key0 + n * 16 + l16, hi - 1))));
            }
        };
        int64_t row[2], scale_at[2];
        bool next[2];
        auto find_rows = [&](int32_t key0) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int32_t key = max(lo, min(key0 + n * 16 + l16, hi - 1)), id = max(page[n], 0);
                next[n] = key == key0 + n * 16 + l16 && page[n] >= 0;
                const int32_t slot = key - quotient(a.cache.page, key) * a.cache.page.divisor;
                row[n] = id * a.cache.page_bytes + slot * a.cache.token_bytes;
                scale_at[n] = ((int64_t)id * heads + head) * a.cache.page.divisor + slot;
            }
        };
        // (every load is done, from the nearest key that exists; see below for what must be zero instead)
        auto load_rows = [&](const char* base, const uint8_t* scales, uint4_t (&x)[2][LOADS], unsigned (&power)[2]) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const char* const from = base + row[n];
                if (a.cache.d == DP) {
#pragma unroll
                    for (int i = 0; i < LOADS; ++i) x[n][i] = *(const uint4_t*)(from + i * 64);
                } else {
#pragma unroll
                    for (int i = 0; i < LOADS; ++i) {
                        x[n][i] = (uint4_t){0, 0, 0, 0};
                        if ((i * 4 + quarter) * (E8 ? 16 : 8) < a.cache.d) x[n][i] = *(const uint4_t*)(from + i * 64);
                    }
                }
                if constexpr (E8) power[n] = scales[scale_at[n]];
            }
        };

        int32_t key0 = key_begin;
        find_pages(key0);
        if (key0 < hi) {
            find_rows(key0);
            load_rows(k_head, a.cache.k_scale, k, ks);
            load_rows(v_head, a.cache.v_scale, v, vs);
        }
        // queries: row n * 16 + l16, in the order of values in which the keys lie in the registers
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
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            top[n] = NO_MAX;
            sum[n] = 0.0f;
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) o[n][i] = (float4_t)(0.0f);
        }
        find_pages(key0 + UNIT);

        for (; key0 < hi; key0 += UNIT) {
            const uint64_t held0 = __ballot(next[0]), held1 = __ballot(next[1]);      // (each quarter says the same of 16 keys)
            const int32_t key_next = key0 + UNIT;
            float4_t sc[NB][2];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int m = 0; m < NB; ++m) {
                    sc[m][n] = (float4_t)(0.0f);
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) {
                        uint4_t x;
                        if constexpr (E8) x = widen8(k[n][i / 2][(i & 1) * 2], k[n][i / 2][(i & 1) * 2 + 1], power_of(ks[n]));
                        else x = k[n][i];
                        sc[m][n] = T::mfma16(as_x8<T>(x), as_x8<T>(q[m][i]), sc[m][n]);
                    }
                }
            // V into LDS, row by row; zeros for keys that do not exist (their weight is 0, and 0 times an infinity is not)
            const bool gaps = (held0 & held1) != ~(uint64_t)0;
            if (gaps) {
#pragma unroll
                for (int n = 0; n < 2; ++n)
                    if (!next[n]) {
#pragma unroll
                        for (int i = 0; i < LOADS; ++i) v[n][i] = (uint4_t){0, 0, 0, 0};
                    }
            }
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    if constexpr (E8) {
                        const float power = power_of(vs[n]);
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            *(uint4_t*)(mine + (to_lds ^ (i << 7) ^ (e << 4)) + n * 16 * DP * 2) = widen8(v[n][i][2 * e], v[n][i][2 * e + 1], power);
                    } else {
                        *(uint4_t*)(mine + (to_lds ^ (i << 6)) + n * 16 * DP * 2) = v[n][i];
                    }
                }
            if (key_next < hi) {
                find_rows(key_next);
                load_rows(k_head, a.cache.k_scale, k, ks);
                load_rows(v_head, a.cache.v_scale, v, vs);
                find_pages(key_next + UNIT);
            }
            // lane: keys 4 * quarter + r of either sixteen
            if (gaps) {
#pragma unroll
                for (int m = 0; m < NB; ++m)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (!((held0 >> (quarter * 4 + r)) & 1)) sc[m][0][r] = -__builtin_inff();
                        if (!((held1 >> (quarter * 4 + r)) & 1)) sc[m][1][r] = -__builtin_inff();
                    }
            }
            uint4_t p[NB];
#pragma unroll
            for (int m = 0; m < NB; ++m) {
                float most = sc[m][0][0];
#pragma unroll
                for (int r = 0; r < 4; ++r) most = fmaxf(most, fmaxf(sc[m][0][r], sc[m][1][r]));
                most *= a.scale_log2;
                if (__any(most > top[m] + SLACK)) {
                    const float now = fmaxf(top[m], quarters_max(most)), by = exp2_(top[m] - now);
                    top[m] = now;
                    sum[m] *= by;
#pragma unroll
                    for (int i = 0; i < BLOCKS; ++i) o[m][i] *= by;
                }
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int r = 0; r < 4; r += 2) {
                        const float x = exp2_(__builtin_fmaf(sc[m][n][r], a.scale_log2, -top[m]));
                        const float y = exp2_(__builtin_fmaf(sc[m][n][r + 1], a.scale_log2, -top[m]));
                        sum[m] += x + y;
                        p[m][n * 2 + r / 2] = T::pack(x, y);
                    }
            }
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                const uint2_t x = column4(mine + (from_lds ^ (i << 5))), y = column4(mine + (from_lds ^ (i << 5)) + 16 * DP * 2);
#pragma unroll
                for (int m = 0; m < NB; ++m) o[m][i] = T::mfma16(as_x8<T>((uint4_t){x.x, x.y, y.x, y.y}), as_x8<T>(p[m]), o[m][i]);
            }
        }

        // the four wavefronts' rows are joined through LDS, 16 at a time: row l16, values i * 16 + 4 * quarter + r
#pragma unroll
        for (int m = 0; m < NB; ++m) {
            const float total = quarters_sum(sum[m]);
            __syncthreads();
            float* const rows = (float*)mine;
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) *(float4_t*)(rows + l16 * DP + i * 16 + quarter * 4) = o[m][i];
            if (quarter == 0) {
                rows[16 * DP + l16] = top[m];
                rows[16 * DP + 16 + l16] = total;
            }
            __syncthreads();
            const int r = threadIdx.x / (DP / 8), d = (threadIdx.x % (DP / 8)) * 8, g = m * 16 + r;
            if (r < 16 && g < G) {
                float t[TOKEN_WAVES], most = NO_MAX, all = 0.0f, x[8] = {};
#pragma unroll
                for (int w = 0; w < TOKEN_WAVES; ++w) {
                    t[w] = ((const float*)(lds + w * WAVE_LDS))[16 * DP + r];
                    most = fmaxf(most, t[w]);
                }
#pragma unroll
                for (int w = 0; w < TOKEN_WAVES; ++w) {
                    const float* const from = (const float*)(lds + w * WAVE_LDS);
                    const float by = exp2_(t[w] - most);
                    all += by * from[16 * DP + 16 + r];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] += by * from[r * DP + d + e];
                }
                if (whole) {
                    const float norm = all != 0.0f ? 1.0f / all : 0.0f;
                    if (d < a.cache.d)
                        *(uint4_t*)(a.out.base + s * a.out.token_bytes + (head * G + g) * a.out.head_bytes + d * 2) =
                            (uint4_t){T::pack(x[0] * norm, x[1] * norm), T::pack(x[2] * norm, x[3] * norm), T::pack(x[4] * norm, x[5] * norm),
                                      T::pack(x[6] * norm, x[7] * norm)};
                    if (a.lse && d == 0)
                        a.lse[(int64_t)s * a.q_heads + head * G + g] = all != 0.0f ? (most + log2_(all)) * 0.6931471805599453f : -__builtin_inff();
                } else {
                    float* const part = partial_of<DP>(a, group, at > run) + g * (DP + 2);
#pragma unroll
                    for (int e = 0; e < 8; ++e) part[d + e] = x[e];
                    if (d == 0) {
                        part[DP] = most;
                        part[DP + 1] = all;
                    }
                }
            }
        }
        __syncthreads();
        at = pair + u1;
        if (at == before + (int64_t)n_units * heads) {
            before = at;
            ++s;
        }
    }
}

// Joins the partial rows of the pairs that several workgroups shared.  One workgroup a pair; it finds the pair's place in the
// line of units as the kernel before did.
template <class T, int DP>
__global__ __launch_bounds__(TOKEN_THREADS) void join_token_kernel(AttendArgs a) {
    const int lane = threadIdx.x & 63;
    const int32_t heads = a.cache.heads, G = a.group.divisor, s = blockIdx.x / heads, head = blockIdx.x % heads;
    int64_t units = 0, before = 0;
    for (int32_t at = 0; at < a.batch.S; at += 64) {
        const int32_t x = at + lane < a.batch.S ? units_of(a, at + lane) : 0;
        units += wave_sum(x);
        before += wave_sum(at + lane < s ? x : 0);
    }
    units *= heads;
    const int32_t n = units_of(a, s), groups = groups_at_work(a, units);
    const int64_t begin = before * heads + (int64_t)head * n, end = begin + n;
    // the workgroups whose runs hold its first and its last unit
    auto holder = [&](int64_t unit) {
        int32_t w = (int32_t)(unit * groups / units);
        while (run_begin(units, groups, w + 1) <= unit) ++w;
        while (run_begin(units, groups, w) > unit) --w;
        return w;
    };
    const int32_t w0 = holder(begin), w1 = holder(end - 1);
    if (w0 == w1) return;
    const int d = (threadIdx.x % (DP / 8)) * 8;
    for (int32_t g = threadIdx.x / (DP / 8); g < G; g += TOKEN_THREADS / (DP / 8)) {
        auto part_of = [&](int32_t w) { return partial_of<DP>(a, w, run_begin(units, groups, w) < begin) + g * (DP + 2); };
        float most = NO_MAX, all = 0.0f, x[8] = {};
        for (int32_t w = w0; w <= w1; ++w) most = fmaxf(most, part_of(w)[DP]);
        for (int32_t w = w0; w <= w1; ++w) {
            const float* const part = part_of(w);
            const float by = exp2_(part[DP] - most);
            if (by == 0.0f) continue;
            all += by * part[DP + 1];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += by * part[d + e];
        }
        const float norm = all != 0.0f ? 1.0f / all : 0.0f;
        if (d < a.cache.d)
            *(uint4_t*)(a.out.base + s * a.out.token_bytes + (head * G + g) * a.out.head_bytes + d * 2) =
                (uint4_t){T::pack(x[0] * norm, x[1] * norm), T::pack(x[2] * norm, x[3] * norm), T::pack(x[4] * norm, x[5] * norm),
                          T::pack(x[6] * norm, x[7] * norm)};
        if (a.lse && d == 0)
            a.lse[(int64_t)s * a.q_heads + head * G + g] = all != 0.0f ? (most + log2_(all)) * 0.6931471805599453f : -__builtin_inff();
    }
}

}  // namespace gorgo
