// Layer norm's kernels on the CPU, their wavefronts in several orders between barriers (lanes.hpp), against sums in 64 bits; and rows of one
// value, whose outputs have no error to allow for.
#include "norm.hip"

using namespace ffsnap;

static std::mt19937 g_rng(1);
static float value() { return float(int(g_rng() % 2001) - 1000) / 256.f; }

static bool near(const char* what, uint32_t n, uint32_t width, uint32_t kind, const std::vector<float>& got, const std::vector<double>& want, double tol)
{
    for (size_t k = 0; k < want.size(); k++)
        if (!(std::fabs(got[k] - want[k]) <= tol)) {
            std::printf("%s of %u x %u, order %u: at %zu got %.9g, want %.9g\n", what, n, width, kind, k, double(got[k]), want[k]);
            return false;
        }
    return true;
}

// IN_PLACE: dx over dy
static bool both_ways(uint32_t n, uint32_t width, bool in_place)
{
    const double eps = double(1e-5f);
    std::vector<float> x(size_t(n) * width), w(width), b(width), dy(x.size()), y(x.size()), mean(n), rstd(n), dx(x.size()), dw(width), db(width);
    for (auto* v : {&x, &w, &b, &dy})
        for (auto& e : *v) e = value();
    std::vector<double> wy(x.size()), wdx(x.size()), wdw(width), wdb(width);
    for (uint32_t r = 0; r < n; r++) {
        const size_t at = size_t(r) * width;
        double m = 0, var = 0, c0 = 0, c1 = 0;
        for (uint32_t k = 0; k < width; k++) m += x[at + k];
        m /= width;
        for (uint32_t k = 0; k < width; k++) var += (x[at + k] - m) * (x[at + k] - m);
        const double rs = 1 / std::sqrt(var / width + eps);
        for (uint32_t k = 0; k < width; k++) {
            const double xh = (x[at + k] - m) * rs, g = double(dy[at + k]) * w[k];
            wy[at + k] = xh * w[k] + b[k];
            wdw[k] += dy[at + k] * xh;
            wdb[k] += dy[at + k];
            c0 += g;
            c1 += g * xh;
        }
        for (uint32_t k = 0; k < width; k++) {
            const double xh = (x[at + k] - m) * rs;
            wdx[at + k] = rs * (double(dy[at + k]) * w[k] - c0 / width - xh * (c1 / width));
        }
    }
    // Values are below 4, so sums over n rows or a row are below 16 times as many terms; 32-bit sums of N terms are off by at most N 2^-24 of that.
    // (Width 1 aside, where the variance is 0 and rstd 316, rows of these values have one beyond 1: rstd < 1.)
    const double off = 16 * 64 * std::ldexp(1.0, -24) * (width == 1 ? 1e3 : 1), rows = 16.0 * n * (n + 64) * std::ldexp(1.0, -24);
    bool ok = true;
    for (uint32_t kind = 0; kind < 4; kind++) {
        lanes::g_kind = kind;
        lanes::g_order.seed(kind);
        NormArgs a = {};
        auto bytes = [](std::vector<float>& v) { return reinterpret_cast<uint8_t*>(v.data()); };
        a.x = bytes(x);
        a.n_rows = n;
        a.width = a.x_stride = a.out_stride = a.dy_stride = width;
        a.weight = bytes(w);
        a.bias = bytes(b);
        a.eps = 1e-5f;
        a.mean = mean.data();
        a.rstd = rstd.data();
        a.out = bytes(y);
        launch_norm(a, FF_F32, nullptr);
        dx = dy;
        std::vector<float> parts(norm_workspace(n, width) / 4, NAN);
        std::vector<float> out(dx.size(), NAN);
        a.dy = bytes(dx);
        a.out = in_place ? bytes(dx) : bytes(out);
        a.dweight = bytes(dw);
        a.dbias = bytes(db);
        a.parts = parts.data();
        launch_norm_grad(a, FF_F32, nullptr);
        ok = near("y", n, width, kind, y, wy, off) && near("dx", n, width, kind, in_place ? dx : out, wdx, 4 * off) && near("dweight", n, width, kind, dw, wdw, rows + n * off) &&
             near("dbias", n, width, kind, db, wdb, rows) && ok;
    }
    return ok;
}

// A value of few bits: its sum over the row is exact, and so is the quotient.  y is the bias, whatever rstd is; and a row whose dy has one value
// under weights of one has no gradient.
static bool one_value(uint32_t width, float c)
{
    lanes::g_kind = 0;
    std::vector<float> x(width, c), w(width, 1.f), b(width), y(width), mean(1), rstd(1), dx(width, NAN);
    for (auto& e : b) e = value();
    NormArgs a = {};
    a.x = reinterpret_cast<uint8_t*>(x.data());
    a.n_rows = 1;
    a.width = a.x_stride = a.out_stride = a.dy_stride = width;
    a.weight = reinterpret_cast<uint8_t*>(w.data());
    a.bias = reinterpret_cast<uint8_t*>(b.data());
    a.eps = 1e-5f;
    a.mean = mean.data();
    a.rstd = rstd.data();
    a.out = reinterpret_cast<uint8_t*>(y.data());
    launch_norm(a, FF_F32, nullptr);
    a.dy = a.x;
    a.out = reinterpret_cast<uint8_t*>(dx.data());
    launch_norm_grad(a, FF_F32, nullptr);
    for (uint32_t k = 0; k < width; k++)
        if (mean[0] != c || y[k] != b[k] || dx[k] != 0.f) {
            std::printf("a row of %u times %g: mean %.9g, at %u y - b %g, dx %g\n", width, double(c), double(mean[0]), k, double(y[k] - b[k]), double(dx[k]));
            return false;
        }
    return true;
}

int main()
{
    bool ok = true;
    for (bool in_place : {false, true}) {
        for (uint32_t width : {1u, 7u, 64u, 520u, 1003u, 1500u, 4097u}) ok = both_ways(5, width, in_place) && ok;
        ok = both_ways(700, 40, in_place) && ok;
        ok = both_ways(2, 8200, in_place) && ok;
        ok = both_ways(9, 16384, in_place) && ok;
    }
    for (uint32_t width : {3u, 41u, 47u, 49u, 97u, 107u, 111u, 513u, 777u, 1003u, 1533u, 2049u, 4097u, 5000u, 8191u, 16383u})
        for (float c : {5.f, 300.f, 1000.f, 20000.f}) ok = one_value(width, c) && ok;
    std::printf(ok ? "ok\n" : "failed\n");
    return !ok;
}
