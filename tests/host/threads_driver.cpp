// Which launches the library enqueues on one stream when two threads make calls on it at once, without a device: the functions below stand in front of the runtime's own (a program's symbols come
// before those of its libraries). A launch takes a while, so that calls without an order between them mix. Prints a line per operator: launches of a call, calls whose launches were not next to each
// other on the stream, the kernel. Test infrastructure.
#include <hip/hip_runtime.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <unistd.h>

#include <functional>
#include <mutex>
#include <thread>
#include <vector>

#include "../../include/mlt_diag.h"

static std::mutex g_mu;
static std::vector<int> g_launches;            // the thread of each, in the stream's order
static thread_local int t_thread = 0;

extern "C" {
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600* p, int) {
  memset(p, 0, sizeof *p);
  strcpy(p->gcnArchName, "gfx950:sramecc+:xnack-");
  p->multiProcessorCount = 256;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t a, int) {
  *v = a == hipDeviceAttributeNumberOfXccs ? 8 : 256;
  return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* st) { *st = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) { *p = malloc(n); return hipSuccess; }
hipError_t hipFree(void* p) { free(p); return hipSuccess; }
static thread_local struct { dim3 g, b; size_t m; hipStream_t s; } t_conf;
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t m, hipStream_t s) { t_conf = {g, b, m, s}; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* m, hipStream_t* s) {
  *g = t_conf.g; *b = t_conf.b; *m = t_conf.m; *s = t_conf.s;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) {
  {
    std::lock_guard<std::mutex> lock(g_mu);
    g_launches.push_back(t_thread);
  }
  usleep(300);
  return hipSuccess;
}
}

static void* at(uintptr_t mib) { return (void*)(mib << 20); }   // operands: addresses that nobody follows
static const int32_t* ints(uintptr_t mib) { return (const int32_t*)at(mib); }

int main() {
  void* const s = (void*)0x1000;
  const float* const F = (const float*)at(3);
  const std::pair<const char*, std::function<int()>> ops[] = {
      {"packed", [&] { return mlt_mha_packed_fwd(20, 3000, 1, 8, 2, 128, at(1), 1024, at(2), 256, at(3), 256, ints(5), ints(6), at(9), 1024, 0.1f, 1, MLT_BF16, s); }},
      {"prompt", [&] { return mlt_paged_attn_prompt(30, 1, 8, 2, 128, 32, 100, 200, at(1), 1024, at(2), at(99), ints(5), ints(6), ints(7), at(199), 1024, 0.1f, MLT_BF16, s); }},
      {"prefix", [&] { return mlt_paged_attn_decode_prefix(70, 8, 2, 128, 32, 300, 9000, at(1), at(2), at(99), ints(5), 8500, ints(6), ints(7), at(199), 0.1f, nullptr, 0, MLT_BF16, s); }},
      {"w4", [&] { return mlt_gemm_w4(57, 900, 4096, at(1), 4096, at(2), 2048, 64, at(9), 900, (const uint8_t*)at(10), 900, at(11), 900, MLT_BF16, s); }},
      {"mha", [&] { return mlt_mha_fwd(1, 8, 1, 4096, 128, at(1), at(2), at(99), at(999), 0.1f, 0, MLT_BF16, s); }},
      {"paged", [&] { return mlt_paged_attn_decode(1, 8, 128, 16, 2048, 4096, at(1), at(2), at(99), ints(500), ints(501), at(999), 0.1f, MLT_BF16, s); }},
      {"paged_fp8", [&] { return mlt_paged_attn_decode_fp8(1, 8, 8, 128, 16, 2048, 4096, at(1), at(2), at(99), F, F, ints(500), ints(501), at(999), 0.1f, MLT_BF16, s); }},
  };
  for (const auto& op : ops) {
    if (op.second() != 0) { printf("%s refused\n", op.first); return 1; }            // (has its scratch now)
    g_launches.clear();
    op.second();
    const size_t each = g_launches.size(), calls = 40;
    g_launches.clear();
    std::thread threads[2];
    for (int t = 0; t < 2; ++t)
      threads[t] = std::thread([&, t] {
        t_thread = t;
        for (size_t i = 0; i < calls; ++i) op.second();
      });
    for (auto& t : threads) t.join();
    int mixed = 0;
    for (size_t i = 0; i < g_launches.size(); i += each)
      for (size_t k = 1; k < each; ++k)
        if (g_launches[i + k] != g_launches[i]) { ++mixed; break; }
    printf("%s %zu %d %s\n", op.first, each, g_launches.size() == 2 * calls * each ? mixed : -1, mlt_last_kernel());
  }
  return 0;
}
