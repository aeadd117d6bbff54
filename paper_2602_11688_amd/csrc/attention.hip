// Kernels of the paged cache and of the attention over it, and their launches.
#include "attend_prompt.h"
#include "attend_token.h"
#include "gorgo.h"
#include "internal.h"
#include "kv_cache.h"

namespace gorgo {
namespace {

int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return GORGO_OK;
    (void)hipGetLastError();
    return fail(GORGO_ERR_DEVICE, std::string("launch ") + what + ": " + hipGetErrorString(e));
}

template <class T, bool E8, int DP>
void launch_prompt(const AttendArgs& a, bool aligned, hipStream_t s) {
    const dim3 grid((unsigned)(a.tiles * a.cache.heads), (unsigned)a.splits);
    if (aligned)
        hipLaunchKernelGGL((attend_prompt_kernel<T, E8, DP, true>), grid, dim3(PROMPT_THREADS), 0, s, a);
    else
        hipLaunchKernelGGL((attend_prompt_kernel<T, E8, DP, false>), grid, dim3(PROMPT_THREADS), 0, s, a);
    if (a.splits > 1) hipLaunchKernelGGL((join_prompt_kernel<T, DP>), dim3(grid.x, PROMPT_ROWS / JOIN_ROWS<DP>), dim3(PROMPT_THREADS), 0, s, a);
}

template <class T, bool E8, int DP, int NB>
void launch_token_rows(const AttendArgs& a, bool aligned, hipStream_t s) {
    if (aligned)
        hipLaunchKernelGGL((attend_token_kernel<T, E8, DP, NB, true>), dim3((unsigned)a.splits), dim3(TOKEN_THREADS), 0, s, a);
    else
        hipLaunchKernelGGL((attend_token_kernel<T, E8, DP, NB, false>), dim3((unsigned)a.splits), dim3(TOKEN_THREADS), 0, s, a);
}

template <class T, bool E8, int DP>
void launch_token(const AttendArgs& a, bool aligned, hipStream_t s) {
    if (a.group.divisor <= 16) launch_token_rows<T, E8, DP, 1>(a, aligned, s);
    else launch_token_rows<T, E8, DP, 2>(a, aligned, s);
}

// The kernels' variants: type of the cache (and with it of the rows), head size up to 64 or 128.
template <class F>
void by_type(int type, int32_t d, F f) {
    auto sized = [&](auto t, auto e8) {
        if (d <= 64) f(t, e8, std::integral_constant<int, 64>{});
        else f(t, e8, std::integral_constant<int, 128>{});
    };
    if (type == CACHE_BF16) sized(Bf16{}, std::false_type{});
    else if (type == CACHE_F16) sized(F16{}, std::false_type{});
    else sized(Bf16{}, std::true_type{});
}

}  // namespace

int launch_kv_write(const CacheArgs& c, const BatchArgs& b, const RowsArgs& k, const RowsArgs& v, int type, void* stream) {
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)((b.tokens + KV_THREADS / 64 - 1) / (KV_THREADS / 64)));
    by_type(type, c.d, [&](auto, auto e8, auto dp) {
        hipLaunchKernelGGL((kv_write_kernel<decltype(e8)::value, decltype(dp)::value / 8>), grid, dim3(KV_THREADS), 0, s, c, b, k, v);
    });
    return launched("kv_write_kernel");
}

int launch_kv_read(const CacheArgs& c, const BatchArgs& b, const RowsArgs& k, const RowsArgs& v, int type, void* stream) {
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)((b.tokens + KV_THREADS / 64 - 1) / (KV_THREADS / 64)));
    by_type(type, c.d, [&](auto, auto e8, auto dp) {
        hipLaunchKernelGGL((kv_read_kernel<decltype(e8)::value, decltype(dp)::value / 8>), grid, dim3(KV_THREADS), 0, s, c, b, k, v);
    });
    return launched("kv_read_kernel");
}

int launch_attend_prompt(const AttendArgs& a, int type, void* stream) {
    const bool aligned = a.cache.page.divisor % PROMPT_KEYS == 0;
    by_type(type, a.cache.d, [&](auto t, auto e8, auto dp) {
        launch_prompt<decltype(t), decltype(e8)::value, decltype(dp)::value>(a, aligned, static_cast<hipStream_t>(stream));
    });
    return launched("attend_prompt_kernel");
}

int launch_attend_token(const AttendArgs& a, int type, void* stream) {
    const bool aligned = a.cache.page.divisor % token_keys(type == CACHE_E4M3) == 0;
    by_type(type, a.cache.d, [&](auto t, auto e8, auto dp) {
        launch_token<decltype(t), decltype(e8)::value, decltype(dp)::value>(a, aligned, static_cast<hipStream_t>(stream));
    });
    return launched("attend_token_kernel");
}

}  // namespace gorgo
