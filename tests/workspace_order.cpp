// What two host threads queue on one stream, without a GPU: the launch code (gemm_launch.hip,
// mx_gemm.hip) compiled for the host alone, over stand-ins for the HIP runtime and for the kernels'
// launchers that note each launch.  Every launch waits a while for the other thread's next one, so
// that calls which can interleave do.  Prints a line per case: its name and the launches in order,
// as <thread><launch>.
#include <stdio.h>
#include <string.h>

#include <chrono>
#include <condition_variable>
#include <mutex>
#include <string>
#include <thread>
#include <vector>

#include "../paper_2512_13282_amd/csrc/configs.h"
#include "../paper_2512_13282_amd/csrc/families.h"
#include "../paper_2512_13282_amd/csrc/mx_launch.h"

namespace {
std::mutex mu;
std::condition_variable cv;
std::string order;
int launches[2];
bool capturing;
thread_local int self = -1;

hipError_t note(char what) {
    if (self < 0) return hipSuccess;
    std::unique_lock<std::mutex> lk(mu);
    order += char('1' + self);
    order += what;
    order += ' ';
    const int mine = ++launches[self];
    cv.notify_all();
    cv.wait_for(lk, std::chrono::milliseconds(1000), [&] { return launches[1 - self] >= mine; });
    return hipSuccess;
}
}  // namespace

// ---- the HIP runtime
extern "C" {
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) {
    *s = capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    return hipSuccess;
}
hipError_t hipThreadExchangeStreamCaptureMode(hipStreamCaptureMode *) { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t) { *p = reinterpret_cast<void *>(uintptr_t(1) << 40); return hipSuccess; }
hipError_t hipMallocAsync(void **p, size_t n, hipStream_t) { return hipMalloc(p, n); }
hipError_t hipFree(void *) { return hipSuccess; }
hipError_t hipFreeAsync(void *, hipStream_t) { return hipSuccess; }
hipError_t hipGetSymbolAddress(void **, const void *) { return hipErrorInvalidValue; }
hipError_t hipLaunchKernel(const void *, dim3, dim3, void **, size_t, hipStream_t) { return note('c'); }
hipError_t __hipPushCallConfiguration(dim3, dim3, size_t, hipStream_t) { return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *n, hipStream_t *s) {
    *g = *b = dim3(1);
    *n = 0;
    *s = nullptr;
    return hipSuccess;
}
void **__hipRegisterFatBinary(const void *) { return nullptr; }
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, void *, void *, void *, void *, int *) {}
void __hipRegisterVar(void **, void *, char *, const char *, int, size_t, int, int) {}
void __hipUnregisterFatBinary(void **) {}
}

// ---- the kernels' launchers: 'p' a product, 'r' a separate reduction
namespace gemm {
hipError_t launch_mx_fwd(int32_t, const MxArgs &, int64_t, hipStream_t) { return note('p'); }
hipError_t launch_mx_dx(int32_t, const MxArgs &, int64_t, hipStream_t) { return note('p'); }
hipError_t launch_mx_dw(int32_t, const MxArgs &, int64_t, hipStream_t) { return note('p'); }
template <int DT> hipError_t launch_tile_family(int32_t, const KernelArgs &, int64_t, hipStream_t) { return note('p'); }
template <int DT> hipError_t launch_direct_family(int32_t, const KernelArgs &, int64_t, hipStream_t) { return note('p'); }
template <int DT, bool BT> hipError_t launch_ring_family(int32_t, const KernelArgs &, int64_t, hipStream_t) { return note('p'); }
template <int DT> hipError_t launch_small_family(int32_t, const KernelArgs &, int64_t, hipStream_t) { return note('p'); }
template <int DT> hipError_t launch_splitk_reduce(const KernelArgs &, int64_t, hipStream_t) { return note('r'); }
#define FAMILIES(DT)                                                                             \
    template hipError_t launch_tile_family<DT>(int32_t, const KernelArgs &, int64_t, hipStream_t);   \
    template hipError_t launch_direct_family<DT>(int32_t, const KernelArgs &, int64_t, hipStream_t); \
    template hipError_t launch_small_family<DT>(int32_t, const KernelArgs &, int64_t, hipStream_t);  \
    template hipError_t launch_ring_family<DT, true>(int32_t, const KernelArgs &, int64_t, hipStream_t);  \
    template hipError_t launch_ring_family<DT, false>(int32_t, const KernelArgs &, int64_t, hipStream_t); \
    template hipError_t launch_splitk_reduce<DT>(const KernelArgs &, int64_t, hipStream_t);
FAMILIES(DT_I8)
FAMILIES(DT_BF16)
}  // namespace gemm

namespace {
using namespace gemm;

int block_scaled(void *stream, int64_t a_offset, int32_t split) {
    MxArgs a{};
    a.g.dtype = DT_BF16;
    a.g.A = reinterpret_cast<const void *>((uintptr_t(1) << 41) + a_offset);
    a.g.B = reinterpret_cast<const void *>(uintptr_t(1) << 42);
    a.g.C = reinterpret_cast<void *>(uintptr_t(1) << 43);
    a.g.M = 256; a.g.N = 512; a.g.K = 1024;
    a.g.lda = 1024; a.g.ldb = 512; a.g.ldc = 512;
    a.scales = reinterpret_cast<const uint8_t *>(uintptr_t(1) << 44);
    a.ld_scales = 32;
    MxPlan plan{};
    if (!mx_select(MX_FWD, a.g.M, a.g.N, a.g.K, a_offset ? 2 * a.g.M * a.g.K : 0, 0, 6, split, &plan)) return -1;
    return launch_mx_gemm(a, MX_FWD, plan, stream);
}

int dense(void *stream) {
    KernelArgs a{};
    a.dtype = DT_BF16;
    a.M = a.N = 256; a.K = 1024;
    a.lda = 1024; a.ldb = 256; a.ldc = 256;
    a.split_k = 2;
    a.k_chunk = 512;
    a.tiles_m = a.tiles_n = 2;
    a.reduce_in_kernel = REDUCE_SEPARATE;
    return launch_gemm(a, 0, 8, stream);
}

template <typename F> void two_threads(const char *name, F f, bool same_stream) {
    order.clear();
    launches[0] = launches[1] = 0;
    int rc[2];
    std::thread t[2];
    for (int i = 0; i < 2; ++i)
        t[i] = std::thread([&, i] {
            self = i;
            rc[i] = f(reinterpret_cast<void *>(uintptr_t(same_stream ? 16 : 16 + 16 * i)));
        });
    for (auto &x : t) x.join();
    printf("%s: %s%s\n", name, order.c_str(), rc[0] == LAUNCH_OK && rc[1] == LAUNCH_OK ? "ok" : "failed");
}
}  // namespace

int main() {
    // The workspaces exist, so that a call's launches are its own alone.
    for (uintptr_t s : {16, 32}) {
        if (block_scaled(reinterpret_cast<void *>(s), 2, 3) != LAUNCH_OK || dense(reinterpret_cast<void *>(s)) != LAUNCH_OK) return 1;
    }
    two_threads("copied operand", [](void *s) { return block_scaled(s, 2, 1); }, true);
    two_threads("copied operand, slices", [](void *s) { return block_scaled(s, 2, 2); }, true);
    two_threads("dense, separate reduction", [](void *s) { return dense(s); }, true);
    two_threads("two streams", [](void *s) { return block_scaled(s, 2, 1); }, false);
    release_workspaces();
    capturing = true;       // without counters of its own: a separate reduction
    two_threads("captured slices", [](void *s) { return block_scaled(s, 0, 2); }, true);
    return 0;
}
