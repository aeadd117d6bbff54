// Writing new tokens into a paged cache, and reading them back.
#pragma once
#include "attention_common.h"

namespace gorgo {

// Where a token of the packed rows, the same for a whole wavefront, lies in the cache.
struct Place {
    int64_t bytes;           // of its page and slot
    int64_t scale;           // index of its scale byte, of head 0
    bool held;               // false: no page, or no token
};
__device__ inline Place place_of(const CacheArgs& c, const BatchArgs& b, int32_t token) {
    int32_t s = token;
    if (b.first) {                                     // the last sequence that begins at or before it, 64 looked at at a time
        const int lane = threadIdx.x & 63;
        s = 0;
        for (int32_t n = b.S; n > 1;) {
            const int32_t step = (n + 63) / 64, at = lane * step;
            const int before = __popcll(__ballot(at < n && b.first[s + min(at, n - 1)] <= token));
            const int32_t skip = max(before - 1, 0) * step;
            s += skip;
            n = min(step, n - skip);
        }
        s = __builtin_amdgcn_readfirstlane(s);
    }
    Place at{0, 0, false};
    const Span span = span_of(b, s);
    if (token < span.begin || token >= span.end) return at;
    const int32_t pos = length_of(b, s) - (span.end - token);
    if (pos < 0 || pos >= b.capacity) return at;
    const int32_t index = quotient(c.page, pos), slot = pos - index * c.page.divisor;
    const int32_t page = page_of(b, c, s, index);
    if (page < 0) return at;
    at.bytes = page * c.page_bytes + slot * c.token_bytes;
    at.scale = ((int64_t)page * c.heads) * c.page.divisor + slot;
    at.held = true;
    return at;
}

// A row's scale byte, k + 127, from the bits of its largest finite magnitude: least k with it <= 448 * 2^k = 1.75 * 2^(k + 8); 119 at most, where
// 448 * 2^k is the largest value of such codes that bf16 holds.
__device__ inline int scale_byte(unsigned top) { return min(max((int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), 1), 119 + 127); }
// Codes of four values of such a row, to nearest, ties to even; what is not finite becomes the NaN code.
__device__ inline unsigned four_codes(const float (&x)[4], int byte) {
    const float down = __builtin_bit_cast(float, (unsigned)(254 - byte) << 23);      // 2^-k
    float f[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = x[e] * down;
    if (byte == 119 + 127) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (__builtin_fabsf(f[e]) < 512.0f) f[e] = fmaxf(fminf(f[e], 448.0f), -448.0f);      // (512 and more: not finite)
    }
    const int p = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], p, true);
}

constexpr int KV_THREADS = 256;

// One wavefront a token: ROW lanes a head, eight values a lane, keys and values.  Bound by bytes: every value is read once and
// written once, in pieces of 16 (8) bytes that lie side by side.  The row's largest magnitude is a butterfly over its ROW lanes.
template <bool E8, int ROW>
__global__ __launch_bounds__(KV_THREADS) void kv_write_kernel(CacheArgs c, BatchArgs b, RowsArgs k, RowsArgs v) {
    const int32_t token = blockIdx.x * (KV_THREADS / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (token >= b.tokens) return;
    const Place at = place_of(c, b, token);
    if (!at.held) return;
    const int lane = threadIdx.x & 63, chunk = lane % ROW;
    const bool inside = chunk * 8 < c.d;               // (lanes beyond a row's end stay for the butterfly)
    for (int32_t h = lane / ROW; h < c.heads; h += 64 / ROW) {
        uint4_t x[2] = {};
        if (inside) {
            x[0] = *(const uint4_t*)(k.base + token * k.token_bytes + h * k.head_bytes + chunk * 16);
            x[1] = *(const uint4_t*)(v.base + token * v.token_bytes + h * v.head_bytes + chunk * 16);
        }
        char* const to[2] = {c.k + at.bytes + h * c.head_bytes, c.v + at.bytes + h * c.head_bytes};
        if constexpr (!E8) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (inside) *(uint4_t*)(to[i] + chunk * 16) = x[i];
        } else {
            uint8_t* const scales[2] = {c.k_scale, c.v_scale};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                // bits of the largest finite magnitude: as integers they are ordered as the values are
                unsigned top = 0;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const unsigned lo = (x[i][w] << 16) & 0x7fff0000u, hi = x[i][w] & 0x7fff0000u;
                    if (lo < 0x7f800000u) top = max(top, lo);
                    if (hi < 0x7f800000u) top = max(top, hi);
                }
#pragma unroll
                for (int step = 1; step < ROW; step <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, step, ROW));
                const int byte = scale_byte(top);
                unsigned codes[2];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float f[4];
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        f[2 * w] = __builtin_bit_cast(float, x[i][2 * half + w] << 16);
                        f[2 * w + 1] = __builtin_bit_cast(float, x[i][2 * half + w] & 0xffff0000u);
                    }
                    codes[half] = four_codes(f, byte);
                }
                if (inside) *(uint2_t*)(to[i] + chunk * 8) = (uint2_t){codes[0], codes[1]};
                if (chunk == 0) scales[i][at.scale + (int64_t)h * c.page.divisor] = (uint8_t)byte;
            }
        }
    }
}

// The reverse: rows of the batch's tokens, in 16 bits; zeros where the cache holds none.
template <bool E8, int ROW>
__global__ __launch_bounds__(KV_THREADS) void kv_read_kernel(CacheArgs c, BatchArgs b, RowsArgs k, RowsArgs v) {
    const int32_t token = blockIdx.x * (KV_THREADS / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (token >= b.tokens) return;
    const Place at = place_of(c, b, token);
    const int lane = threadIdx.x & 63, chunk = lane % ROW;
    if (chunk * 8 >= c.d) return;
    for (int32_t h = lane / ROW; h < c.heads; h += 64 / ROW) {
        const char* const from[2] = {c.k + at.bytes + h * c.head_bytes, c.v + at.bytes + h * c.head_bytes};
        uint4_t x[2] = {};
        if (at.held) {
            if constexpr (!E8) {
#pragma unroll
                for (int i = 0; i < 2; ++i) x[i] = *(const uint4_t*)(from[i] + chunk * 16);
            } else {
                const uint8_t* const scales[2] = {c.k_scale, c.v_scale};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint2_t codes = *(const uint2_t*)(from[i] + chunk * 8);
                    x[i] = widen8(codes.x, codes.y, power_of(scales[i][at.scale + (int64_t)h * c.page.divisor]));
                }
            }
        }
        *(uint4_t*)(k.base + token * k.token_bytes + h * k.head_bytes + chunk * 16) = x[0];
        *(uint4_t*)(v.base + token * v.token_bytes + h * v.head_bytes + chunk * 16) = x[1];
    }
}

}  // namespace gorgo
