// A workgroup's threads on the CPU, one at a time: each runs until it comes to an exchange of its wavefront's lanes or to the workgroup's barrier.
// A wavefront runs for as long as it can before the next one does, in an order that the check chooses: what one reads and another
// overwrites without a barrier in between comes out wrong in one of the orders.  All lanes of a wavefront have to come to the same exchanges.
#pragma once
#include <stdint.h>
#include <setjmp.h>
#include <string.h>
#include <ucontext.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <memory>
#include <random>
#include <vector>

namespace lanes {

struct Index {
    uint32_t x, y, z;
};
enum Wait { kRuns, kLanes, kBarrier, kDone };
struct Thread {
    ucontext_t start;
    jmp_buf at;  // (from then on: a ucontext's switch is a call of the system)
    bool started = false;
    std::unique_ptr<char[]> stack;
    Wait wait = kDone;
    uint64_t given = 0;  // to the exchange
};

inline Index g_block, g_grid;
inline std::vector<Thread> g_threads;
inline uint32_t g_now, g_n;
inline jmp_buf g_back;
inline std::function<void()> g_body;
inline std::mt19937 g_order;
inline uint32_t g_kind;  // of order: wavefronts upwards, downwards, or a new order after every barrier
inline uint64_t g_given[64];

inline Index thread() { return {g_now, 0, 0}; }
inline int lane() { return static_cast<int>(g_now % 64); }

inline void wait(Wait why)
{
    Thread& me = g_threads[g_now];
    me.wait = why;
    if (!_setjmp(me.at)) _longjmp(g_back, 1);
}
inline void meet_workgroup() { wait(kBarrier); }

// The value of the lane `from`, in every lane.
template <class T>
T exchange(T v, int from)
{
    static_assert(sizeof(T) <= 8, "");
    memcpy(&g_threads[g_now].given, &v, sizeof(T));
    wait(kLanes);
    memcpy(&v, &g_given[from], sizeof(T));
    return v;
}
inline uint64_t ballot(bool x)
{
    g_threads[g_now].given = x;
    wait(kLanes);
    uint64_t all = 0;
    for (int k = 0; k < 64; k++) all |= (g_given[k] & 1) << k;
    return all;
}

inline void enter()
{
    g_body();
    wait(kDone);
}

inline void resume(Thread& t)
{
    if (_setjmp(g_back)) return;
    if (t.started) _longjmp(t.at, 1);
    t.started = true;
    setcontext(&t.start);
}

// Wavefront w until all its threads are at the barrier or done.
inline void run_wavefront(uint32_t w)
{
    for (;;) {
        const uint32_t first = w * 64;
        for (g_now = first; g_now < first + 64; g_now++)
            if (g_threads[g_now].wait == kRuns) resume(g_threads[g_now]);
        uint32_t count[4] = {};
        for (uint32_t k = 0; k < 64; k++) count[g_threads[first + k].wait]++;
        if (count[kLanes] == 0) return;
        if (count[kLanes] != 64) {
            std::printf("an exchange that not all lanes have come to\n");
            std::exit(1);
        }
        for (uint32_t k = 0; k < 64; k++) {
            g_given[k] = g_threads[first + k].given;
            g_threads[first + k].wait = kRuns;
        }
    }
}

template <class Dim, class Body>
void launch(Dim grid, Dim block, Body&& body)
{
    constexpr size_t kStack = 128 << 10;
    g_grid = {grid.x, grid.y, grid.z};
    g_n = block.x;
    g_body = body;
    if (g_threads.size() < g_n) g_threads.resize(g_n);
    for (uint32_t y = 0; y < grid.y; y++)
        for (uint32_t x = 0; x < grid.x; x++) {
            g_block = {x, y, 0};
            for (uint32_t t = 0; t < g_n; t++) {
                Thread& k = g_threads[t];
                if (!k.stack) k.stack.reset(new char[kStack]);
                getcontext(&k.start);
                k.start.uc_stack.ss_sp = k.stack.get();
                k.start.uc_stack.ss_size = kStack;
                k.start.uc_link = nullptr;
                makecontext(&k.start, enter, 0);
                k.started = false;
                k.wait = kRuns;
            }
            const uint32_t waves = g_n / 64;
            std::vector<uint32_t> order(waves);
            for (bool any = true; any;) {
                for (uint32_t w = 0; w < waves; w++) order[w] = g_kind == 1 ? waves - 1 - w : w;
                if (g_kind > 1) std::shuffle(order.begin(), order.end(), g_order);
                for (uint32_t w : order) run_wavefront(w);
                any = false;
                for (uint32_t t = 0; t < g_n; t++)
                    if (g_threads[t].wait == kBarrier) {
                        g_threads[t].wait = kRuns;
                        any = true;
                    }
            }
        }
}

}  // namespace lanes
