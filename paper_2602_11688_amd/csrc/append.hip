// The kernel that norms and rotates heads, and its launch.
#include <type_traits>

#include "append_rows.h"
#include "gorgo.h"
#include "internal.h"

namespace gorgo {
namespace {

template <class T, bool E8, int U, int ROW, bool HALVES>
void launch(const AppendArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((append_kernel<T, E8, U, ROW, HALVES>), dim3((unsigned)((a.batch.tokens + a.block - 1) / a.block), (unsigned)a.parts), dim3(APPEND_THREADS), 0, s, a);
}

// Lanes of a row: as many as its runs need (a power of two).
template <class T, bool E8>
void launch_type(const AppendArgs& a, hipStream_t s) {
    const bool small = a.cache.d <= 64;
    if (a.rotation.neighbours) {
        if (small) launch<T, E8, 8, 4, false>(a, s);
        else launch<T, E8, 8, 8, false>(a, s);
    } else if (a.rotation.pairs % 8 == 0) {
        if (small) launch<T, E8, 8, 4, true>(a, s);
        else launch<T, E8, 8, 8, true>(a, s);
    } else if (a.rotation.pairs % 4 == 0) {
        launch<T, E8, 4, 16, true>(a, s);
    } else {
        launch<T, E8, 1, 64, true>(a, s);
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
