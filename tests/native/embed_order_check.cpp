// The embedding's kernels on the CPU, their wavefronts in several orders between barriers (lanes.hpp), against plain sums.  Values are
// small whole numbers: sums are exact in any order.
#include "embed.hip"

using namespace ffsnap;

static std::mt19937 g_rng(1);

static bool gradient(uint32_t n, uint32_t vocab, uint32_t width, bool add, const std::function<int64_t()>& id)
{
    std::vector<int64_t> ids(n);
    for (auto& x : ids) x = id();
    // (behind either, rows that are not the kernels' to read or write)
    constexpr uint32_t kGuard = 4096;
    std::vector<float> rows(size_t(n + kGuard) * width, NAN), start(size_t(vocab + kGuard) * width), want;
    for (size_t k = 0; k < size_t(n) * width; k++) rows[k] = float(int(g_rng() % 17) - 8);
    for (auto& x : start) x = float(int(g_rng() % 33) - 16);
    want = start;
    if (!add) std::fill_n(want.begin(), size_t(vocab) * width, 0.f);
    for (uint32_t t = 0; t < n; t++)
        if (ids[t] >= 0 && ids[t] < int64_t(vocab))
            for (uint32_t k = 0; k < width; k++) want[size_t(ids[t]) * width + k] += 2 * rows[size_t(t) * width + k];
    for (uint32_t kind = 0; kind < 4; kind++) {
        lanes::g_kind = kind;
        lanes::g_order.seed(kind);
        std::vector<float> out = start;
        std::vector<uint8_t> space(embed_workspace(n, vocab, width), 0xA5);
        const EmbedArgs a = {reinterpret_cast<const uint8_t*>(rows.data()), width, ids.data(), n, vocab, width, 2.f, reinterpret_cast<uint8_t*>(out.data()), width};
        launch_embed_grad(a, FF_F32, add, space.data(), nullptr);
        if (out != want) {
            std::printf("%u tokens, %u x %u, order %u: differs\n", n, vocab, width, kind);
            return false;
        }
    }
    return true;
}

int main()
{
    bool ok = true;
    // (placed in several rounds of a workgroup's threads: tokens of one word, of few, of a range)
    for (uint32_t n : {1u, 512u, 513u, 1100u, 4096u}) {
        ok = gradient(n, 40, 8, n % 2, [] { return 3; }) && ok;
        ok = gradient(n, 300, 9, true, [] { return int64_t(g_rng() % 5) - 1; }) && ok;
        ok = gradient(n, 64, 24, false, [] { return int64_t(g_rng() % 66) - 1; }) && ok;
    }
    // (ranges of 512 ids, 520 elements wide)
    ok = gradient(1500, 200000, 8, true, [] { return int64_t(200000 - g_rng() % 512); }) && ok;
    ok = gradient(600, 6, 520, true, [] { return 5; }) && ok;
    // (sorted lists, in several looks at the ids)
    ok = gradient(4097, 40, 8, true, [] { return 39; }) && ok;
    ok = gradient(17000, 300, 9, false, [] { return int64_t(g_rng() % 302) - 1; }) && ok;
    std::printf(ok ? "ok\n" : "failed\n");
    return !ok;
}
