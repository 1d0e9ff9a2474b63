// What the kernels of every translation unit share: mbarriers with bounded waits, small conversions, launches and the
// library's record of CUDA errors.
#ifndef BITCOS_COMMON_CUH
#define BITCOS_COMMON_CUH

#include "bitcos.h"

#include <cuda_runtime.h>

#include <cstdint>
#include <cstdlib>
#include <mutex>
#include <tuple>
#include <type_traits>

namespace bitcos_kernels {

constexpr uint64_t kWaitLimitNs = 500ull * 1000 * 1000;   // an mbarrier wait gives up after half a second

inline thread_local int g_last_cuda_error = 0;

// Largest magnitudes below this count as this in every quantiser, so that the quotient of the range and them is finite.
constexpr float kAmaxFloor = 7.888609052210118e-31f;      // 2^-100

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint64_t global_timer_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ uint32_t mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done;
}
// Polls until the phase completes, for at most limit_ns; false if it gave up.
__device__ __forceinline__ bool mbar_wait_limited(uint32_t bar, uint32_t parity, uint64_t limit_ns) {
    uint64_t t0 = 0;
    for (uint32_t i = 0;; ++i) {
        if (mbar_try(bar, parity)) return true;
        if ((i & 15u) == 15u) {
            const uint64_t now = global_timer_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > limit_ns) return false;
        }
    }
}
static __device__ __noinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity) { return mbar_wait_limited(bar, parity, kWaitLimitNs); }
// Waits for the given phase parity (bounded); the common case, an already completed phase, costs
// one instruction.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {
    if (mbar_try(bar, parity)) return true;
    return mbar_wait_slow(bar, parity);
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_cuda(cudaError_t e) {
    if (e == cudaSuccess) return BITCOS_OK;
    g_last_cuda_error = static_cast<int>(e);
    return BITCOS_ERR_CUDA;
}

// Number of multiprocessors of the current device.  The opt-in to large dynamic shared memory is
// done on the first call for a given kernel instantiation and device and remembered (so that
// first call must not happen during stream capture; later calls only read the cache).
template <auto kernel>
int prepare_kernel(int *sms_out, int *smem_budget_out) {
    constexpr int kMaxDev = 32;
    static int cache[kMaxDev][2];      // [0] multiprocessor count (0 = not prepared yet), [1] dynamic smem budget
    int dev = 0;
    int rc = check_cuda(cudaGetDevice(&dev));
    if (rc) return rc;
    if (dev < kMaxDev && cache[dev][0] > 0) {
        *sms_out = cache[dev][0];
        *smem_budget_out = cache[dev][1];
        return BITCOS_OK;
    }
    int sms = 0, max_smem = 0;
    rc = check_cuda(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    if (rc) return rc;
    rc = check_cuda(cudaDeviceGetAttribute(&max_smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev));
    if (rc) return rc;
    const int budget = max_smem - 1024;
    rc = check_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, budget));
    if (rc) return rc;
    if (dev < kMaxDev) {
        cache[dev][1] = budget;
        cache[dev][0] = sms;
    }
    *sms_out = sms;
    *smem_budget_out = budget;
    return BITCOS_OK;
}

// Launches with programmatic stream serialization, so that this kernel's prologue (barrier
// set-up, table and first weight copies) may overlap the tail of the previous kernel in the
// stream.  BITCOS_PDL=0 turns it off (for A/B runs).
// (arguments of exactly the kernel's types, taken by reference: the largest are 7 KB, and every copy on the way counts
// against launches of 2 us)
template <typename... KArgs, typename... Args>
int launch_pdl(void (*kernel)(KArgs...), dim3 grid, int threads, size_t smem, cudaStream_t stream, const Args &...args) {
    static_assert(std::is_same<std::tuple<typename std::remove_cv<KArgs>::type...>, std::tuple<Args...>>::value, "the kernel's own types");
    static const char *env = std::getenv("BITCOS_PDL");
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = (env && env[0] == '0') ? 0 : 1;
    void *pointers[] = {const_cast<void *>(static_cast<const void *>(&args))...};
    return check_cuda(cudaLaunchKernelExC(&cfg, reinterpret_cast<const void *>(kernel), pointers));
}

}  // namespace bitcos_kernels

#endif  // BITCOS_COMMON_CUH
