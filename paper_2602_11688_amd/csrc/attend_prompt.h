// Attention of prompts: many new tokens of each sequence over the pages of the cache.
#pragma once
#include "attention_common.h"

namespace gorgo {

// Rows and keys.  A row is a (new token, query head) pair of one cache head, numbered token by token: the query heads that share
// a cache head also share the tile of its keys, and a causal tile of rows spans few tokens.  A workgroup takes ROWS consecutive
// rows of one sequence, a wavefront 32 of them, and walks the keys in tiles of KEYS.
//
// Scores are computed transposed, S^T = K Q^T, by 32x32x16 products: a lane then holds sixteen keys' scores of one row in its
// registers, so that maximum and sum are registers' work, and two halves of the wavefront share a row.  The second product,
// O^T = V^T P^T, wants eight keys of a row in each lane; which eight is free as long as both factors agree, since a sum over
// keys has no order.  With the keys (0-3, 8-11) in the lower half and (4-7, 12-15) in the upper one they are where the first
// product left them: P is never moved between lanes.  V^T comes from row-major LDS through transposing reads.
//
// Two phases a tile: products (of a tile's weights with V, of the next tile's K with Q) and the softmax in between (maximum, powers,
// sum, rounding), which also moves the next tile to LDS.  The matrix unit does the one, the vector unit the other, and they cost about the
// same: 32 products of 32 cycles, and 150 instructions of 4 with 32 powers that take 8.  Of a SIMD's two wavefronts one belongs
// to the upper half of the workgroup and one to the lower; the upper half runs one phase later, so that one unit's work hides the
// other's.  Barriers end the phases; the upper half stages K and V a tile further ahead, since its staging falls into the phase
// before the lower half's.
// 20,000 tokens of 32/8 heads of 128, bf16: 3050 to 3240 us by the card and its clock, 1010 to 1075 TFLOP/s (with all wavefronts in one
// phase 3313 where this took 3053; the products alone, with nothing to read and no softmax, 2064, as fast as a large library matrix
// product).  What is left, by copies that leave one part out: staging 440 us (through registers into LDS), reads of LDS 350 (each
// wavefront of 32 rows reads every tile), powers 260.
constexpr int PROMPT_THREADS = 2 * PROMPT_ROWS;      // a wavefront for 32 rows

// LDS tile of KEYS rows of DP 16-bit values, in chunks of 16 bytes that are moved within a row so that lanes which read one
// column of chunks (K: of 16 rows) or a 4 x 4 block of them (V: four rows) touch every bank once.
template <int DP>
struct Tile {
    static constexpr int CHUNKS = DP / 8, BYTES = PROMPT_KEYS * DP * 2;
    static __device__ int k_at(int row, int chunk) {
        return row * (DP * 2) + ((chunk ^ (DP == 128 ? row & 15 : (row >> 1) & 7)) << 4);
    }
    static __device__ int v_at(int row, int chunk) {
        const int turn = DP == 128 ? ((row & 3) << 2 | ((row >> 2) & 3)) : (((row >> 1) & 1) << 2 | ((row >> 2) & 3));
        return row * (DP * 2) + ((chunk ^ turn) << 4);
    }
};

// Tile of rows that a workgroup takes: slots are dealt out so that the sequence of a slot follows from `first` alone (sequence s
// begins at slot first[s] * group / ROWS + s; its tiles never reach the next one's).
struct RowTile {
    int32_t s, begin, rows;          // first row within the sequence, rows of this tile (0: none)
    Span span;
};
__device__ inline RowTile row_tile(const AttendArgs& a, int32_t slot) {
    const int lane = threadIdx.x & 63;
    const int32_t G = a.group.divisor;
    auto start = [&](int32_t s) { return (int32_t)(((int64_t)span_of(a.batch, s).begin * G) / PROMPT_ROWS) + s; };
    int32_t s = 0;
    for (int32_t at = 0; at < a.batch.S; at += 64) {
        const bool before = at + lane < a.batch.S && start(at + lane) <= slot;
        const int n = __popcll(__ballot(before));
        if (n) s = at + n - 1;
        if (n < 64) break;
    }
    s = __builtin_amdgcn_readfirstlane(s);
    RowTile t;
    t.s = s;
    t.span = span_of(a.batch, s);
    t.begin = (slot - start(s)) * PROMPT_ROWS;
    const int64_t all = (int64_t)(t.span.end - t.span.begin) * G;
    t.rows = t.begin < 0 || t.begin >= all ? 0 : (int32_t)min<int64_t>(PROMPT_ROWS, all - t.begin);
    return t;
}

// Keys [from, to) that some row of a tile of rows sees, and one piece's tiles of them.
struct KeyRange {
    int32_t from, to, pos_lo, pos_hi, begin, end, pieces;
};
__device__ inline KeyRange key_range(const AttendArgs& a, const RowTile& t, int32_t piece) {
    const int32_t length = length_of(a.batch, t.s), first_pos = length - (t.span.end - t.span.begin);
    KeyRange k;
    k.pos_lo = max(first_pos + quotient(a.group, t.begin), 0);             // (rows before position 0 see nothing)
    k.pos_hi = first_pos + quotient(a.group, t.begin + t.rows - 1);
    k.to = min(k.pos_hi + 1, min(length, a.batch.capacity));
    k.from = a.window ? max(0, k.pos_lo - a.window + 1) : 0;
    const int32_t begin = k.from / PROMPT_KEYS, count = k.to > k.from ? (k.to + PROMPT_KEYS - 1) / PROMPT_KEYS - begin : 0;
    k.pieces = max(1, min(a.splits, count / PIECE_TILES));
    k.begin = begin + (int32_t)((int64_t)count * piece / k.pieces);
    k.end = begin + (int32_t)((int64_t)count * (piece + 1) / k.pieces);
    return k;
}

// Two 16-bit values, zeros in the place of what is not finite.
template <class T>
__device__ unsigned tame(unsigned x) {
    return ((x & T::EXPONENT) == T::EXPONENT ? 0u : x & 0xffffu) | (((x >> 16) & T::EXPONENT) == T::EXPONENT ? 0u : x & 0xffff0000u);
}
// Four codes of 8 bits, zeros in the place of NaN.
__device__ inline unsigned tame_codes(unsigned x) {
#pragma unroll
    for (int i = 0; i < 32; i += 8)
        if (((x >> i) & 0x7fu) == 0x7fu) x &= ~(0xffu << i);
    return x;
}

// ALIGNED: a tile of keys lies in one page.  Heads of 64 have half the products and all of the softmax: the vector unit bounds them, and two
// workgroups at a time, 128 registers each, keep it busier (785 to 604 us then, see below; other pages than of whole tiles take more
// registers than that).  In scratch memory lie up to 11 registers of the variants for heads of 64 in whole pages, and up to 10 of those for wider
// heads in other pages.
template <class T, bool E8, int DP, bool ALIGNED>
__global__ __launch_bounds__(PROMPT_THREADS, DP == 64 && ALIGNED ? 4 : 2) void attend_prompt_kernel(AttendArgs a) {
    using L = Tile<DP>;
    constexpr int KEYS = PROMPT_KEYS, STEPS = DP / 16, BLOCKS = DP / 32;
    constexpr int ROW_LOADS = E8 ? DP / 16 : DP / 8;                       // 16-byte loads of a row
    constexpr int ITEMS = 2 * KEYS * ROW_LOADS;                            // of a tile of keys and values
    constexpr int LOADS = ITEMS / PROMPT_THREADS;                          // of a thread
    constexpr int KS = LOADS > 1 ? LOADS / 2 : 1;                          // rows that a thread takes of either
    static_assert(LOADS >= 1 && ITEMS % PROMPT_THREADS == 0);
    __shared__ __attribute__((aligned(256))) char lds[2][2 * L::BYTES];    // [buffer][K, V]

    const int32_t heads = a.cache.heads, G = a.group.divisor;
    const int32_t slot = a.tiles - 1 - (int32_t)(blockIdx.x / heads), head = blockIdx.x % heads;
    const RowTile tile = row_tile(a, slot);
    if (tile.rows <= 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    const int32_t piece = blockIdx.y;
    const KeyRange keys = key_range(a, tile, piece);
    if (piece >= keys.pieces) return;
    const int32_t first_pos = length_of(a.batch, tile.s) - (tile.span.end - tile.span.begin);    // of the sequence's first new token
    const int32_t from = keys.from, to = keys.to, end = keys.end, pieces = keys.pieces;

    // this lane's row
    const int32_t row = wave * 32 + l32;
    const bool is_row = row < tile.rows;
    const int32_t nth = quotient(a.group, tile.begin + min(row, tile.rows - 1));
    const int32_t q_head = head * G + (tile.begin + min(row, tile.rows - 1) - nth * G);
    const int32_t token = tile.span.begin + nth;
    const int32_t pos = first_pos + nth;
    // first and last position of this wavefront's rows
    const int32_t last_row = tile.rows - 1;
    const int32_t wave_first = min(wave * 32, last_row), wave_last = min(wave * 32 + 31, last_row);
    const int32_t wave_lo = max(first_pos + quotient(a.group, tile.begin + wave_first), 0);
    const int32_t wave_hi = wave * 32 < tile.rows ? first_pos + quotient(a.group, tile.begin + wave_last) : -1;

    uint4_t q[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int chunk = 2 * i + half;
        q[i] = (uint4_t){0, 0, 0, 0};
        if (is_row && chunk * 8 < a.cache.d)
            q[i] = *(const uint4_t*)(a.q.base + token * a.q.token_bytes + q_head * a.q.head_bytes + chunk * 16);
    }

    float16_t o[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) o[i] = (float16_t)(0.0f);
    float top = NO_MAX, sum = 0.0f;

    // Staging, of the keys of tile `next` and the values of the one before it: item i of a thread is 16 bytes of a row of either, in
    // one item's place where there are as many threads as items.  Every load is done, from a row that exists (before the first tile
    // and after the last one of any), so that none has to wait for another; what has to be zero is made so on the way to LDS.
    // Places in the cache go on from tile to tile by sums, and are looked up in the table where a page begins (ALIGNED).
    const int32_t begin = keys.begin;
    const int group = wave / (PROMPT_THREADS / 128);
    const int load_chunk = threadIdx.x % ROW_LOADS;
    const bool load_inside = load_chunk * (E8 ? 16 : 8) < a.cache.d;
    constexpr int ROWS_A_PASS = PROMPT_THREADS / ROW_LOADS;
    const int load_row = threadIdx.x / ROW_LOADS % KEYS;                  // (of the first of KS rows, ROWS_A_PASS apart)
    auto is_v = [&](int i) { return LOADS > 1 ? i >= KS : group == 1; };
    const int64_t head_at = head * a.cache.head_bytes;
    const int32_t* const table = a.batch.table + (int64_t)tile.s * a.batch.columns;
    uint4_t staged[LOADS];
    unsigned scales[LOADS];
    uint32_t lane_at[KS];                                                 // ALIGNED: of the thread's rows, from the tile's first
#pragma unroll
    for (int n = 0; n < KS; ++n)
        lane_at[n] = ALIGNED ? (uint32_t)(load_row + n * ROWS_A_PASS) * (uint32_t)a.cache.token_bytes + (load_inside ? load_chunk * 16 : 0)
                             : load_inside ? load_chunk * 16 : 0;
    constexpr int PLACES = ALIGNED ? 1 : KS;
    int64_t row_now[PLACES] = {}, row_last[PLACES] = {}, scale_now[PLACES] = {}, scale_last[PLACES] = {};    // of tile `next`, of the one before
    unsigned held[PLACES] = {};                                           // bit i: of tile next - i
    int32_t next = begin;
    int32_t page_index = 0, page_slot = 0, page_id = 0;                    // ALIGNED: of the tile after them, its page once it is looked up
    int32_t ids[PLACES] = {};                                             // !ALIGNED
    int32_t wild_first = 0x7fffffff, wild_last = -1;                       // tiles in which this thread found such values, see below
    auto find_pages = [&](int32_t tile_j) {
        if constexpr (!ALIGNED) {
            if (tile_j >= end) return;
#pragma unroll
            for (int i = 0; i < KS; ++i) ids[i] = table[quotient(a.cache.page, max(from, min(tile_j * KEYS + load_row + i * ROWS_A_PASS, to - 1)))];
        }
    };
    auto load = [&]() {
#pragma unroll
        for (int n = 0; n < PLACES; ++n) {
            row_last[n] = row_now[n];
            scale_last[n] = scale_now[n];
            held[n] <<= 1;
        }
        if (next < end) {
            if constexpr (ALIGNED) {
                if (page_slot == 0 || next == begin) {
                    const int32_t id = (uint32_t)page_id < (uint32_t)a.cache.pages ? page_id : 0;
                    row_now[0] = id * a.cache.page_bytes + page_slot * a.cache.token_bytes + head_at;
                    if constexpr (E8) scale_now[0] = ((int64_t)id * heads + head) * a.cache.page.divisor + page_slot;
                } else {
                    row_now[0] += KEYS * a.cache.token_bytes;
                    if constexpr (E8) scale_now[0] += KEYS;
                }
                held[0] |= (uint32_t)page_id < (uint32_t)a.cache.pages;
                page_slot += KEYS;
                if (page_slot == a.cache.page.divisor) {
                    page_slot = 0;
                    ++page_index;
                    if (next + 1 < end) page_id = constant(table)[page_index];
                }
            } else {
#pragma unroll
                for (int n = 0; n < PLACES; ++n) {
                    const int32_t key = max(from, min(next * KEYS + load_row + n * ROWS_A_PASS, to - 1));
                    const bool is = (uint32_t)ids[n] < (uint32_t)a.cache.pages;
                    const int32_t id = is ? ids[n] : 0, slot_ = key - quotient(a.cache.page, key) * a.cache.page.divisor;
                    row_now[n] = id * a.cache.page_bytes + slot_ * a.cache.token_bytes + head_at;
                    scale_now[n] = ((int64_t)id * heads + head) * a.cache.page.divisor + slot_;
                    held[n] |= is;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int n = ALIGNED ? 0 : i % KS;
            staged[i] = *(const uint4_t*)((is_v(i) ? a.cache.v + row_last[n] : a.cache.k + row_now[n]) + lane_at[i % KS]);
            if constexpr (E8)
                scales[i] = (is_v(i) ? a.cache.v_scale + scale_last[n] : a.cache.k_scale + scale_now[n])[ALIGNED ? (uint32_t)(load_row + i % KS * ROWS_A_PASS) : 0u];
        }
        find_pages(next + 1);
    };
    // Values of keys that nobody sees become zero: their weight is 0, but 0 times an infinity is not.  For the same reason, of a tile
    // whose keys only some of the rows see, only finite values are added up by the products.  The others are added at the end, to
    // the rows that see them.  Tiles whose values all rows see:
    const int32_t v_whole = a.window ? ((keys.pos_hi - a.window) >> KEYS_LOG2) + 1 : 0, v_whole_end = min(keys.pos_lo + 1, to) >> KEYS_LOG2;
    auto store = [&]() {
        const int32_t v_tile = next - 1, v_key0 = v_tile * KEYS;
        if (a.cache.d < DP) {                                              // (beyond the row's end stand copies of its beginning)
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                if (!load_inside) staged[i] = (uint4_t){0, 0, 0, 0}, scales[i] = 127;
        }
        if (!ALIGNED || v_tile < v_whole || v_tile >= v_whole_end || !(held[0] & 2)) {
#pragma unroll
            for (int i = LOADS / 2; i < LOADS; ++i) {
                const int r = load_row + i % KS * ROWS_A_PASS, n = ALIGNED ? 0 : i % KS;
                if (!is_v(i)) continue;
                if (v_key0 + r < from || v_key0 + r >= to || !(held[n] & 2)) staged[i] = (uint4_t){0, 0, 0, 0}, scales[i] = 127;
                if (v_tile >= v_whole && v_tile < v_whole_end) continue;
                bool found = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned x = E8 ? tame_codes(staged[i][e]) : tame<T>(staged[i][e]);
                    found |= x != staged[i][e];
                    staged[i][e] = x;
                }
                if (found && v_tile < end) {
                    wild_first = min(wild_first, v_tile);
                    wild_last = v_tile;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = load_row + i % KS * ROWS_A_PASS;
            char* const to_ = is_v(i) ? lds[v_tile & 1] + L::BYTES : lds[next & 1];
            if constexpr (E8) {
                const float power = power_of(scales[i]);
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const int chunk = load_chunk * 2 + n;
                    *(uint4_t*)(to_ + (is_v(i) ? L::v_at(r, chunk) : L::k_at(r, chunk))) = widen8(staged[i][2 * n], staged[i][2 * n + 1], power);
                }
            } else {
                *(uint4_t*)(to_ + (is_v(i) ? L::v_at(r, load_chunk) : L::k_at(r, load_chunk))) = staged[i];
            }
        }
        ++next;
    };

    // LDS addresses of this lane's reads.  A chunk's place is its number exclusive-or a pattern of its row, so a step along the
    // row is an exclusive-or with a constant, and a step of 32 (K) or 16 (V) rows a constant sum.
    const int k_lane = L::k_at(l32, half);
    const int v_lane = L::v_at(4 * half + (lane & 15) / 4, ((lane >> 4) & 1) * 2 + ((lane >> 1) & 1)) + (lane & 1) * 8;

    float16_t s[2];
    uint4_t p[4];
    auto scores = [&](int32_t tile_j) {
        const char* const lk = lds[tile_j & 1];
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const uint4_t kk = *(const uint4_t*)(lk + (k_lane ^ (i << 5)) + n * 32 * DP * 2);
                s[n] = T::mfma32(as_x8<T>(kk), as_x8<T>(q[i]), i ? s[n] : (float16_t)(0.0f));
            }
    };
    int32_t key_id = 0;                                                    // !ALIGNED: page of key `lane` of the tile
    // tiles that every row of this wavefront sees all of
    const int32_t whole = a.window ? ((wave_hi - a.window) >> KEYS_LOG2) + 1 : 0, whole_end = min(wave_lo + 1, to) >> KEYS_LOG2;
    auto weights = [&](int32_t tile_j) {
        uint64_t there;                                                    // keys whose page is
        if constexpr (ALIGNED) there = held[0] & (group ? 4 : 2) ? ~(uint64_t)0 : 0;
        else there = __ballot((uint32_t)key_id < (uint32_t)a.cache.pages);
        if (tile_j < whole || tile_j >= whole_end || ~there) {
            const int32_t key0 = tile_j * KEYS;
            // (heads of 64 are bound by this function: 677 us with, 712 without this on 16 heads, a window of 4096 and two prompts of 11,000 to
            // 24,000 tokens; wider ones lose 40 of 3060 by it, to the registers of a branch)
            if (DP == 64 && (key0 > wave_hi || (a.window && key0 + KEYS - 1 <= wave_lo - a.window) || !there)) {
#pragma unroll
                for (int t = 0; t < 4; ++t) p[t] = (uint4_t){0, 0, 0, 0};
                return;
            }
            // seen: first <= key < first + count (as unsigned numbers, one comparison)
            const int32_t first = (a.window ? max(max(pos, 0) - a.window + 1, 0) : 0) - key0;
            const uint32_t count = max(min(pos + 1, to) - key0 - first, 0);
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = n * 32 + (r >> 2) * 8 + half * 4 + (r & 3);
                    if ((uint32_t)(key - first) >= count) s[n][r] = -__builtin_inff();
                }
            if (~there) {
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (!((there >> (n * 32 + (r >> 2) * 8 + half * 4 + (r & 3))) & 1)) s[n][r] = -__builtin_inff();
            }
        }
        float most = s[0][0];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[n][r]);
        most *= a.scale_log2;
        if (__any(most - top > T::RAISE + T::SLACK)) {
            const float now_ = renewed<T>(top, both_max(most));
            const float by = exp2_(top - now_);
            top = now_;
            sum *= by;
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= by;
        }
        // (far out: the difference, divided by the scale that it is multiplied by again.  Tested on the maximum in every tile, 20,000 tokens of 32/8
        // heads of 128 take what they took without, 3030 us, and heads of 64 with a window 620 instead of 605; a flag renewed with the
        // maximum and a scale of 1 to choose cost the one 40 us, for want of scalar registers, and the other 13)
        float from_top = top;
        if (far_out(top)) {
            const float back = 1.0f / a.scale_log2;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] = (s[n][r] * a.scale_log2 - top) * back;
            from_top = 0.0f;
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float x = exp2_(__builtin_fmaf(s[n][r], a.scale_log2, -from_top)), y = exp2_(__builtin_fmaf(s[n][r + 1], a.scale_log2, -from_top));
                sum += x + y;
                p[n * 2 + r / 8][(r & 7) / 2] = T::pack(x, y);
            }
    };
    auto products = [&](int32_t tile_j) {
        const char* const lv = lds[tile_j & 1] + L::BYTES;
        auto v_part = [&](int t, int block) {
            // keys t * 16 + 4 * half + (0..3) and + 8, values block * 32 + l32
            const uint2_t x = column4(lv + (v_lane ^ (block << 6)) + t * 16 * DP * 2);
            const uint2_t y = column4(lv + (v_lane ^ (block << 6) ^ 32) + (t * 16 + 8) * DP * 2);
            return (uint4_t){x.x, x.y, y.x, y.y};
        };
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) o[i] = T::mfma32(as_x8<T>(v_part(t, i)), as_x8<T>(p[t]), o[i]);
    };
    auto phase_ends = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
    };

    if (begin < end) {
        if constexpr (ALIGNED) {
            page_index = quotient(a.cache.page, begin * KEYS);
            page_slot = begin * KEYS - page_index * a.cache.page.divisor;
            page_id = constant(table)[page_index];
        }
        find_pages(begin);
        load();
        store();
        load();
        __syncthreads();
        if (group) {
            store();
            load();
            phase_ends();
        }
        auto find_keys = [&](int32_t tile_j) {
            if constexpr (!ALIGNED) key_id = table[quotient(a.cache.page, max(from, min(tile_j * KEYS + lane, to - 1)))];
        };
        find_keys(begin);
        scores(begin);
        phase_ends();
        for (int32_t j = begin;; ++j) {
            if (E8) store();                           // (8 bits: 2860 us so, 2915 the other way round; 16 bits: 3085 and 3057)
            weights(j);
            if (!E8) store();
            phase_ends();
            __builtin_amdgcn_s_setprio(1);
            products(j);
            load();
            find_keys(j + 1);
            scores(j + 1);                             // (of the last tile: of what lies there, for nothing)
            __builtin_amdgcn_s_setprio(0);
            phase_ends();
            if (j + 1 == end) break;
        }
        if (!group) phase_ends();
    }

    // values that were not finite
    if (__syncthreads_or(wild_last >= 0)) {
        int* const range = (int*)lds[0];
        if (threadIdx.x == 0) range[0] = 0x7fffffff, range[1] = -1;
        __syncthreads();
        if (wild_last >= 0) {
            atomicMin(&range[0], wild_first);
            atomicMax(&range[1], wild_last);
        }
        __syncthreads();
        // (from the first tile to the last with such: what the products added in between is added again, which changes nothing)
        const int32_t upto = min((range[1] + 1) * KEYS, to);
        for (int32_t key = max(range[0] * KEYS, from); key < upto; ++key) {
            const int32_t index = quotient(a.cache.page, key), page = page_of(a.batch, a.cache, tile.s, index);
            if (page < 0) continue;
            const char* const v_row = a.cache.v + page * a.cache.page_bytes + head * a.cache.head_bytes + (key - index * a.cache.page.divisor) * a.cache.token_bytes;
            const bool sees = key <= pos && (!a.window || key > pos - a.window);
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int d = i * 32 + r * 2 + half * 4;
                    if (!sees || d >= a.cache.d) continue;
                    unsigned x[4];                                         // as 16-bit values
                    if constexpr (E8) {
                        const unsigned w = *(const unsigned*)(v_row + d);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = ((w >> (8 * e)) & 0x7fu) == 0x7fu ? T::EXPONENT + 1 : 0;
                    } else {
                        const uint2_t w = *(const uint2_t*)(v_row + d * 2);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = (w[e / 2] >> (16 * (e & 1))) & 0xffffu;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if ((x[e] & T::EXPONENT) == T::EXPONENT)
                            o[i][r + e] += x[e] & ~(T::EXPONENT | 0x8000u) ? __builtin_nanf("") : x[e] & 0x8000u ? -__builtin_inff() : __builtin_inff();
                }
        }
    }

    if (!is_row) return;
    sum = both_sum(sum);
    const int64_t out_row = (int64_t)token * a.q_heads + q_head;
    const float norm = sum != 0.0f ? 1.0f / sum : 0.0f;                    // (NaN stays)
    if (pieces > 1) {
        // partial rows: [piece][row][DP] and after them [piece][row] of maximum and sum of powers
        const int64_t rows = (int64_t)a.batch.tokens * a.q_heads;
        float* const part = a.partial + (piece * rows + out_row) * DP;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(float4_t*)(part + i * 32 + r * 2 + half * 4) = (float4_t){o[i][r] * norm, o[i][r + 1] * norm, o[i][r + 2] * norm, o[i][r + 3] * norm};
        if (half == 0) *(float2_t*)(a.partial + a.splits * rows * DP + (piece * rows + out_row) * 2) = (float2_t){top, sum};
        return;
    }
    char* const to_row = a.out.base + token * a.out.token_bytes + q_head * a.out.head_bytes;
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = i * 32 + r * 2 + half * 4;
            if (d < a.cache.d)
                *(uint2_t*)(to_row + d * 2) = (uint2_t){T::pack(o[i][r] * norm, o[i][r + 1] * norm), T::pack(o[i][r + 2] * norm, o[i][r + 3] * norm)};
        }
    if (a.lse && half == 0) a.lse[out_row] = log_of_sum<T>(top, sum);
}

// Joins the pieces of a tile of rows: weights sum * 2^(maximum - largest maximum), over their sum.  Eight values a lane; a
// workgroup takes as many rows as its lanes hold (blockIdx.y), and loads do not wait for each other: with one workgroup for all 256 rows and a loop of dependent
// steps the join was most of a call (64 tokens of 32/8 heads of 128 after 2,000, eight pieces: 61 us, now 25).
template <int DP>
constexpr int JOIN_ROWS = PROMPT_THREADS / (DP / 8);
template <class T, int DP>
__global__ __launch_bounds__(PROMPT_THREADS) void join_prompt_kernel(AttendArgs a) {
    const int32_t heads = a.cache.heads, G = a.group.divisor;
    const int32_t head = blockIdx.x % heads;
    const RowTile tile = row_tile(a, blockIdx.x / heads);
    if (tile.rows <= 0) return;
    const int32_t pieces = key_range(a, tile, 0).pieces;
    const int32_t row = blockIdx.y * JOIN_ROWS<DP> + threadIdx.x / (DP / 8);
    if (pieces == 1 || row >= tile.rows) return;
    const int64_t rows = (int64_t)a.batch.tokens * a.q_heads;
    const int d = (threadIdx.x % (DP / 8)) * 8;
    const int32_t nth = quotient(a.group, tile.begin + row), q_head = head * G + tile.begin + row - nth * G;
    const int32_t token = tile.span.begin + nth;
    const int64_t out_row = (int64_t)token * a.q_heads + q_head;
    // Of the row's lanes each takes the maximum and sum of every LANES-th piece; values of four pieces at a time, the first ones under way
    // before the weights are known.
    constexpr int LANES = DP / 8, EACH = MOST_PIECES / LANES;
    const int lane = threadIdx.x % LANES;
    const float* const stats = a.partial + a.splits * rows * DP + out_row * 2;
    float2_t w[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) w[e] = *(const float2_t*)(stats + min(lane + e * LANES, pieces - 1) * rows * 2);
    float4_t x[4][2];
    auto load = [&](int32_t piece) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4_t* const part = (const float4_t*)(a.partial + (min(piece + i, pieces - 1) * rows + out_row) * DP + d);
            x[i][0] = part[0];
            x[i][1] = part[1];
        }
    };
    load(0);
    float top = NO_MAX, sum = 0.0f, o[8] = {};
#pragma unroll
    for (int e = 0; e < EACH; ++e) top = fmaxf(top, w[e].x);
#pragma unroll
    for (int step = 1; step < LANES; step <<= 1) top = fmaxf(top, __shfl_xor(top, step, LANES));
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        w[e].y = lane + e * LANES < pieces ? w[e].y * exp2_(w[e].x - top) : 0.0f;
        sum += w[e].y;
    }
#pragma unroll
    for (int step = 1; step < LANES; step <<= 1) sum += __shfl_xor(sum, step, LANES);
    const float norm = sum != 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int e = 0; e < EACH; ++e)
#pragma unroll
        for (int i0 = 0; i0 < LANES; i0 += 4) {
            if (e * LANES + i0 >= pieces) break;
            if (e + i0 > 0) load(e * LANES + i0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float by = __shfl(w[e].y, i0 + i, LANES) * norm;
#pragma unroll
                for (int n = 0; n < 8; ++n) o[n] += by != 0.0f ? by * x[i][n / 4][n % 4] : 0.0f;      // (a piece without weight adds nothing, whatever is in it)
            }
        }
    if (d < a.cache.d)
        *(uint4_t*)(a.out.base + token * a.out.token_bytes + q_head * a.out.head_bytes + d * 2) =
            (uint4_t){T::pack(o[0], o[1]), T::pack(o[2], o[3]), T::pack(o[4], o[5]), T::pack(o[6], o[7])};
    if (a.lse && d == 0) a.lse[out_row] = log_of_sum<T>(top, sum);
}

}  // namespace gorgo
