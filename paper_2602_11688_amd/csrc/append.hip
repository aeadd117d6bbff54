// The kernel that norms and rotates heads, and its launch.
#include <type_traits>

#include "append_rows.h"
#include "gorgo.h"
#include "internal.h"

namespace gorgo {
namespace {

template <class T, bool E8, int ROW, Runs RUNS>
void launch(const AppendArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.batch.tokens + a.block - 1) / a.block), (unsigned)a.parts);
    hipLaunchKernelGGL((append_kernel<T, E8, ROW, RUNS>), grid, dim3(APPEND_THREADS), 0, s, a);
}

// Lanes of a row: as many as its runs need, a power of two.
template <class T, bool E8>
void launch_type(const AppendArgs& a, hipStream_t s) {
    const int32_t d = a.cache.d, pairs = a.rotation.pairs;
    if (a.rotation.neighbours) {
        d <= 64 ? launch<T, E8, 4, NEIGHBOURS>(a, s) : launch<T, E8, 8, NEIGHBOURS>(a, s);
    } else if (pairs % 8 == 0) {
        d <= 64 ? launch<T, E8, 4, EVEN>(a, s) : launch<T, E8, 8, EVEN>(a, s);
    } else if (d == 8) {
        if constexpr (!E8) launch<T, E8, 4, SINGLE>(a, s);       // (8-bit heads are multiples of 16)
    } else {
        const int32_t lanes = (pairs + 7) / 8 + ((d - 2 * pairs + 7) / 8 + 1) / 2;
        lanes <= 4 ? launch<T, E8, 4, UNEVEN>(a, s) : lanes <= 8 ? launch<T, E8, 8, UNEVEN>(a, s) : launch<T, E8, 16, UNEVEN>(a, s);
    }
}

}  // namespace

int launch_append(const AppendArgs& a, int type, void* stream) {
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (type == CACHE_BF16) launch_type<Bf16, false>(a, s);
    else if (type == CACHE_F16) launch_type<F16, false>(a, s);
    else launch_type<Bf16, true>(a, s);
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return GORGO_OK;
    (void)hipGetLastError();
    return fail(GORGO_ERR_DEVICE, std::string("launch append_kernel: ") + hipGetErrorString(e));
}

}  // namespace gorgo
