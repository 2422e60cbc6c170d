// Host-only check of the launches of the calls between loss and step.  The library's host code runs on a recording
// stand-in for the HIP runtime: device memory is host memory, a launch is noted and not run.
#include <cstdio>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "grads.hpp"
#include "policy.hpp"
#include "status.hpp"

using namespace ffsnap;

struct Launch {
    std::string kernel;
    uint32_t groups, threads;
    uint64_t args[3];  // the first ones' first eight bytes
};
static std::vector<Launch> g_log;
// (filled by the objects' constructors, before this file's own)
static std::map<const void*, std::string>& names() { static std::map<const void*, std::string> m; return m; }
static struct { dim3 g, b; size_t s; hipStream_t q; } g_config;

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* h; return &h; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* f, char* name, const char*, unsigned, void*, void*, dim3*, dim3*, int*) { names()[f] = name; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t s, hipStream_t q) { g_config = {g, b, s, q}; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* s, hipStream_t* q) { *g = g_config.g; *b = g_config.b; *s = g_config.s; *q = g_config.q; return hipSuccess; }
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t)
{
    Launch l{names()[f], grid.x, block.x, {0, 0, 0}};
    const int n_args = l.kernel.find("policy_kernel") != std::string::npos ? 2 : l.kernel.find("grad_clip") != std::string::npos ? 3 : 0;
    for (int k = 0; k < n_args; k++) std::memcpy(&l.args[k], args[k], k == 1 ? 4 : 8);  // (the second of either is of 32 bits)
    g_log.push_back(l);
    return hipSuccess;
}
static hipError_t g_error = hipSuccess, g_malloc = hipErrorOutOfMemory;
hipError_t hipGetLastError() { const hipError_t e = g_error; g_error = hipSuccess; return e; }
hipError_t hipMalloc(void**, size_t) { return g_error = g_malloc; }
hipError_t hipFree(void*) { return hipSuccess; }
hipError_t hipMemcpy(void*, const void*, size_t, hipMemcpyKind) { return hipSuccess; }
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "stand-in"; }
// (of calls that are not made here)
hipError_t hipMemcpyAsync(void*, const void*, size_t, hipMemcpyKind, hipStream_t) { return hipSuccess; }
hipError_t hipGetSymbolAddress(void**, const void*) { return hipErrorNotFound; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* st) { *st = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { *e = nullptr; return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
}

#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)

// A launch's work items are counted in 32 bits.
static bool fits(const Launch& l) { return uint64_t(l.groups) * l.threads <= 0xFFFFFFFFull && l.groups > 0; }

static float* address(uint64_t a) { return reinterpret_cast<float*>(a); }

// Every token of a batch is some launch's, once.
static int policy_rows(uint64_t n, uint64_t vocab, uint32_t dtype, bool grad)
{
    g_log.clear();
    ff_policy_batch b = {address(1 << 20), n, vocab, vocab, dtype, 0, reinterpret_cast<int64_t*>(1 << 20), address(1 << 20), address(1 << 20),
                         address(1 << 20), address(1 << 20), 0.2f, 0.2f, 0.1f, 1.f};
    const int rc = ff_policy_loss(&b, address(1 << 20), address(1 << 21), grad ? address(1 << 22) : nullptr, vocab,
                                  reinterpret_cast<ff_policy_stats*>(1 << 20), address(1 << 20), nullptr);
    CHECK(rc == FF_OK && !g_log.empty());
    uint64_t next = 0;
    for (const Launch& l : g_log) {
        CHECK(fits(l));
        if (l.kernel.find("policy_kernel") == std::string::npos) continue;  // split rows
        CHECK(l.args[1] == next);
        next += l.groups;
    }
    CHECK(next == 0 || next == n);
    return 0;
}

int main()
{
    const uint64_t counts[] = {1, 64, 65, 4096, 4194303, 4194304, 8388607, 8388608, 16777215, 16777216, 67108863, 67108864, 200000000, (1ull << 31) - 1};
    for (uint64_t n : counts)
        for (uint64_t vocab : {1ull, 8ull, 1000ull, 8000ull, 16000ull, 32000ull, 64000ull, 128256ull, 1ull << 20})
            for (uint32_t dtype : {FF_BF16, FF_F16, FF_F32})
                for (bool grad : {false, true})
                    if (policy_rows(n, vocab, dtype, grad)) {
                        std::printf("%llu tokens, vocabulary %llu\n", static_cast<unsigned long long>(n), static_cast<unsigned long long>(vocab));
                        return 1;
                    }

    // Every item of a list is some launch's, once.
    GradWork work;
    const GradItem* const items = reinterpret_cast<const GradItem*>(1 << 20);
    work.items = items;
    for (uint64_t n : {1ull, 5ull, 4096ull, 67108860ull, 67108861ull, 67108864ull, 300000001ull, 1ull << 31}) {
        g_log.clear();
        work.launch = {0, static_cast<uint32_t>(n)};
        CHECK(launch_grad_clip(work, nullptr, nullptr, nullptr) == hipSuccess);
        uint64_t next = 0;
        for (const Launch& l : g_log) {
            CHECK(fits(l));
            CHECK(l.args[0] == reinterpret_cast<uint64_t>(items + next));
            CHECK(uint64_t(l.groups) * kGradWaves >= l.args[1] && l.args[1] > 0);
            next += l.args[1];
        }
        CHECK(next == n);
    }
    // A norm is one launch over all items, whose parts are joined in their order; the workspace holds the addresses of a long list's call.
    for (uint64_t n : {1ull, 2048ull, 2049ull, 5000ull}) {
        const std::vector<const void*> grads(n, address(1 << 20));
        work.n = n;
        work.launch = {0};
        for (uint64_t k = 2048; k < n; k += 2048) work.launch.push_back(static_cast<uint32_t>(3 * k));
        work.launch.push_back(static_cast<uint32_t>(3 * n));
        uint32_t groups[2];
        for (int given : {0, 1}) {
            g_log.clear();
            CHECK(launch_grad_norm(work, given ? grads.data() : nullptr, 1.0, 1.0, address(1 << 20), nullptr, nullptr) == hipSuccess);
            CHECK(g_log.back().kernel.find("grad_norm_kernel") != std::string::npos);
            for (size_t k = 0; k + 1 < g_log.size(); k++) CHECK(g_log[k].kernel.find("grad_norm_kernel") == std::string::npos);
            groups[given] = g_log.back().groups;
        }
        CHECK(groups[0] == groups[1]);
        CHECK(grad_workspace(work) >= groups[0] * sizeof(GradPart) + (n > 2048 ? 8 * n : 0));
    }

    // What a call has reported is not the next one's error.
    const ff_segment seg = {address(1 << 20), 64, FF_F32, FF_KIND_RAW, 0, 0};
    for (hipError_t e : {hipErrorOutOfMemory, hipErrorInvalidValue}) {
        g_malloc = e;
        ff_grad_list* list;
        CHECK(ff_grad_list_create(&seg, 1, 0, &list) == (e == hipErrorOutOfMemory ? FF_ERR_NOMEM : FF_ERR_HIP) && !list);
        ff_grad_stats* const stats = reinterpret_cast<ff_grad_stats*>(1 << 20);
        CHECK(ff_grad_norm_join(stats, 1, 1.0, 1.0, stats, nullptr) == FF_OK);
        ff_plan* plan;
        CHECK(ff_snapshot_plan(&seg, 1, 1024, 0, &plan) == (e == hipErrorOutOfMemory ? FF_ERR_NOMEM : FF_ERR_HIP) && !plan);
        CHECK(ff_grad_norm_join(stats, 1, 1.0, 1.0, stats, nullptr) == FF_OK);
    }
    std::printf("ok\n");
    return 0;
}
