// Host-only check of the launches of the head's loss.  The library's host code runs on a recording stand-in for the HIP runtime: a
// launch is noted and not run.
#include <cstdio>
#include <map>
#include <string>
#include <vector>

#include "../../include/ffsnap.h"
#include "status.hpp"

struct Launch {
    std::string kernel;
    uint32_t groups;
    uint32_t few_rows;  // of W that head_few_kernel packs
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
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3, void** args, size_t, hipStream_t)
{
    Launch l{names()[f], grid.x, 0};
    if (l.kernel.find("head_few_kernel") != std::string::npos) l.few_rows = *static_cast<const uint32_t*>(args[2]);
    g_log.push_back(l);
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "stand-in"; }
}

int ffsnap::hip_fail(hipError_t) { return FF_ERR_HIP; }

#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)

// Launches that read W to copy its rows.
static uint32_t copies()
{
    uint32_t n = 0;
    for (const Launch& l : g_log) n += l.kernel.find("head_pack_kernel") != std::string::npos || l.few_rows;
    return n;
}

int main()
{
    uint8_t* const at = reinterpret_cast<uint8_t*>(1ull << 30);  // never used
    ff_head_stats* const stats = reinterpret_cast<ff_head_stats*>(at + (6 << 20));
    struct { uint64_t vocab, width, stride; } heads[] = {{300, 64, 64}, {300, 65, 65}, {300, 64, 67}, {1, 1, 1}, {9000, 65521, 65528}, {128256, 5350, 5350}};
    for (auto h : heads)
        for (uint64_t n : {0ull, 1ull, 20ull, 100ull, 3000ull})
            for (int with_dh = 0; with_dh < 2; with_dh++) {
                const bool packed = h.width % 8 || h.stride % 8;
                ff_head_batch b = {n ? at : nullptr, n ? at + (1 << 20) : nullptr, n, h.vocab, h.width, h.width, h.stride, FF_BF16, 0, n ? reinterpret_cast<const int64_t*>(at) : nullptr,
                                   n ? reinterpret_cast<const float*>(at) : nullptr, 1.f, 0};
                g_log.clear();
                CHECK(ff_head_loss(&b, n ? reinterpret_cast<float*>(at + (2 << 20)) : nullptr, with_dh && n ? at + (3 << 20) : nullptr, h.width, at + (4 << 20), h.width, stats, at + (5 << 20),
                                   nullptr) == FF_OK);
                CHECK(!g_log.empty());
                // without tokens there is no W to read, and it may be absent
                CHECK((copies() > 0) == (packed && n > 0));
                for (const Launch& l : g_log) CHECK(l.groups > 0);
            }
    std::printf("ok\n");
    return 0;
}
