// extern "C" entry points of the operators at a model's two ends (see include/ffsnap.h for the contract).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "../../include/ffsnap.h"
#include "embed.hpp"
#include "head.hpp"
#include "norm.hpp"
#include "status.hpp"

using namespace ffsnap;

namespace {

uint32_t element_size(uint32_t dtype) { return dtype == FF_F32 ? 4 : dtype == FF_BF16 || dtype == FF_F16 ? 2 : 0; }
bool aligned(const void* p, uint64_t a) { return reinterpret_cast<uint64_t>(p) % a == 0; }
constexpr uint64_t kMost = 0x7FFFFFFFull;                // tokens, rows
constexpr uint64_t kMostStride = 1ull << 40;             // elements: addresses of rows fit 64 bits
bool rows_ok(uint64_t stride, uint64_t width) { return stride >= width && stride <= kMostStride; }
// A loss scale that is one in 32 bits.
bool scale_ok(float v) { return v > 0.f && std::isfinite(v); }

// Is an output's address, unless it is null, another output's or an input's?
bool shared(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs)
{
    for (auto o = outputs.begin(); o != outputs.end(); o++)
        if (*o && (std::find(o + 1, outputs.end(), *o) != outputs.end() || std::find(inputs.begin(), inputs.end(), *o) != inputs.end())) return true;
    return false;
}

int check_embed(const void* rows, uint64_t rows_stride, uint32_t dtype, const int64_t* ids, uint64_t n_tokens, uint64_t vocab, uint64_t width,
                float scale, const void* out, uint64_t out_stride, bool add, bool gradient)
{
    const uint32_t size = element_size(dtype);
    if (!size || !vocab || vocab > FF_EMBED_MAX_VOCAB || !width || width > FF_EMBED_MAX_WIDTH || n_tokens > kMost || !std::isfinite(scale)) return FF_ERR_INVALID;
    if (n_tokens && (!rows || !ids)) return FF_ERR_NULL;
    if ((n_tokens || (gradient && !add)) && !out) return FF_ERR_NULL;
    if (!aligned(rows, size) || !aligned(out, size) || !aligned(ids, 8)) return FF_ERR_INVALID;
    if (!rows_ok(rows_stride, width) || !rows_ok(out_stride, width)) return FF_ERR_INVALID;
    if (n_tokens && shared({out}, {rows, ids})) return FF_ERR_INVALID;
    return FF_OK;
}

int check_norm(const void* x, uint64_t n_rows, uint64_t width, uint64_t x_stride, uint32_t dtype, const void* weight, const void* out,
               uint64_t out_stride, const void* other)
{
    const uint32_t size = element_size(dtype);
    if (!size || !width || width > FF_NORM_MAX_WIDTH || n_rows > kMost || !rows_ok(x_stride, width) || !rows_ok(out_stride, width)) return FF_ERR_INVALID;
    if (!weight || (n_rows && (!x || !out))) return FF_ERR_NULL;
    if (!aligned(x, size) || !aligned(weight, size) || !aligned(other, size) || !aligned(out, size)) return FF_ERR_INVALID;
    return FF_OK;
}

int check_head(const ff_head_batch* b)
{
    if (b->dtype != FF_BF16 && b->dtype != FF_F16) return FF_ERR_INVALID;
    if (b->reserved || !b->vocab || b->vocab > FF_HEAD_MAX_VOCAB || !b->width || b->width > FF_HEAD_MAX_WIDTH || b->n_tokens > FF_HEAD_MAX_TOKENS)
        return FF_ERR_INVALID;
    if (!rows_ok(b->weight_stride, b->width) || !rows_ok(b->hidden_stride, b->width) || !scale_ok(b->loss_scale)) return FF_ERR_INVALID;
    return FF_OK;
}

}  // namespace

extern "C" {

int ff_embed(const void* table, uint64_t vocab, uint64_t width, uint64_t table_stride, uint32_t dtype, const int64_t* ids, uint64_t n_tokens,
             float scale, void* out, uint64_t out_stride, void* hip_stream)
{
    const int rc = check_embed(table, table_stride, dtype, ids, n_tokens, vocab, width, scale, out, out_stride, false, false);
    if (rc != FF_OK) return rc;
    const EmbedArgs a = {static_cast<const uint8_t*>(table), table_stride, ids, n_tokens, vocab, width, scale, static_cast<uint8_t*>(out), out_stride};
    FF_HIP_TRY(launch_embed(a, dtype, static_cast<hipStream_t>(hip_stream)));
    return FF_OK;
}

uint64_t ff_embed_workspace_bytes(uint64_t n_tokens, uint64_t vocab, uint64_t width) { return embed_workspace(n_tokens, vocab, width); }

int ff_embed_grad(const void* dout, uint64_t dout_stride, uint32_t dtype, const int64_t* ids, uint64_t n_tokens, uint64_t vocab, uint64_t width,
                  float scale, void* dtable, uint64_t dtable_stride, uint32_t flags, void* workspace, void* hip_stream)
{
    if (flags & ~FF_GRAD_ADD) return FF_ERR_INVALID;
    const bool add = flags & FF_GRAD_ADD;
    const int rc = check_embed(dout, dout_stride, dtype, ids, n_tokens, vocab, width, scale, dtable, dtable_stride, add, true);
    if (rc != FF_OK) return rc;
    if (!workspace) return FF_ERR_NULL;
    if (!aligned(workspace, 16)) return FF_ERR_INVALID;
    const EmbedArgs a = {static_cast<const uint8_t*>(dout), dout_stride, ids, n_tokens, vocab, width, scale, static_cast<uint8_t*>(dtable), dtable_stride};
    FF_HIP_TRY(launch_embed_grad(a, dtype, add, workspace, static_cast<hipStream_t>(hip_stream)));
    return FF_OK;
}

int ff_layer_norm(const void* x, uint64_t n_rows, uint64_t width, uint64_t x_stride, uint32_t dtype, const void* weight, const void* bias, float eps,
                  void* y, uint64_t y_stride, float* mean, float* rstd, void* hip_stream)
{
    const int rc = check_norm(x, n_rows, width, x_stride, dtype, weight, y, y_stride, bias);
    if (rc != FF_OK) return rc;
    if (!(eps >= 0.f) || !std::isfinite(eps) || !aligned(mean, 4) || !aligned(rstd, 4) || (x == y && x_stride != y_stride)) return FF_ERR_INVALID;
    if (n_rows && (shared({y, mean, rstd}, {weight, bias}) || shared({mean, rstd}, {x}))) return FF_ERR_INVALID;
    NormArgs a = {};
    a.x = static_cast<const uint8_t*>(x);
    a.n_rows = n_rows;
    a.width = width;
    a.x_stride = x_stride;
    a.weight = static_cast<const uint8_t*>(weight);
    a.bias = static_cast<const uint8_t*>(bias);
    a.eps = eps;
    a.mean = mean;
    a.rstd = rstd;
    a.out = static_cast<uint8_t*>(y);
    a.out_stride = y_stride;
    FF_HIP_TRY(launch_norm(a, dtype, static_cast<hipStream_t>(hip_stream)));
    return FF_OK;
}

uint64_t ff_layer_norm_workspace_bytes(uint64_t n_rows, uint64_t width)
{
    return width && width <= FF_NORM_MAX_WIDTH ? norm_workspace(n_rows, width) : 0;
}

int ff_layer_norm_grad(const void* x, uint64_t n_rows, uint64_t width, uint64_t x_stride, uint32_t dtype, const void* weight, const float* mean,
                       const float* rstd, const void* dy, uint64_t dy_stride, void* dx, uint64_t dx_stride, void* dweight, void* dbias, void* workspace,
                       void* hip_stream)
{
    const int rc = check_norm(x, n_rows, width, x_stride, dtype, weight, dx, dx_stride, dy);
    if (rc != FF_OK) return rc;
    if (n_rows && (!mean || !rstd || !dy)) return FF_ERR_NULL;
    if ((dweight || dbias) && !workspace) return FF_ERR_NULL;
    const uint32_t size = element_size(dtype);
    if (!rows_ok(dy_stride, width) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dweight, size) || !aligned(dbias, size) ||
        !aligned(workspace, 16) || (dx == dy && dx_stride != dy_stride) || (dx == x && dx_stride != x_stride))
        return FF_ERR_INVALID;
    if (shared({dweight, dbias}, {weight}) || (n_rows && (shared({dx, dweight, dbias}, {weight, mean, rstd}) || shared({dweight, dbias}, {x, dy})))) return FF_ERR_INVALID;
    NormArgs a = {};
    a.x = static_cast<const uint8_t*>(x);
    a.n_rows = n_rows;
    a.width = width;
    a.x_stride = x_stride;
    a.weight = static_cast<const uint8_t*>(weight);
    a.mean = const_cast<float*>(mean);
    a.rstd = const_cast<float*>(rstd);
    a.out = static_cast<uint8_t*>(dx);
    a.out_stride = dx_stride;
    a.dy = static_cast<const uint8_t*>(dy);
    a.dy_stride = dy_stride;
    a.dweight = static_cast<uint8_t*>(dweight);
    a.dbias = static_cast<uint8_t*>(dbias);
    a.parts = static_cast<float*>(workspace);
    FF_HIP_TRY(launch_norm_grad(a, dtype, static_cast<hipStream_t>(hip_stream)));
    return FF_OK;
}

uint64_t ff_head_workspace_bytes(const ff_head_batch* b, uint32_t gradient)
{
    return b && check_head(b) == FF_OK ? head_workspace(*b, gradient != 0) : 0;
}

int ff_head_loss(const ff_head_batch* b, float* logp, void* dhidden, uint64_t dhidden_stride, void* dweight, uint64_t dweight_stride,
                 ff_head_stats* stats, void* workspace, void* hip_stream)
{
    if (!b || !stats) return FF_ERR_NULL;
    const int rc = check_head(b);
    if (rc != FF_OK) return rc;
    if (!aligned(stats, 8)) return FF_ERR_INVALID;
    if (b->n_tokens) {
        if (!b->hidden || !b->weight || !b->targets || !b->weights || !logp) return FF_ERR_NULL;
        if (!aligned(b->hidden, 2) || !aligned(b->weight, 2) || !aligned(b->targets, 8) || !aligned(b->weights, 4) || !aligned(logp, 4) ||
            !aligned(dhidden, 2))
            return FF_ERR_INVALID;
        if (dhidden && (!rows_ok(dhidden_stride, b->width) || (dhidden == b->hidden && dhidden_stride != b->hidden_stride))) return FF_ERR_INVALID;
    }
    if (b->n_tokens || dweight) {
        if (!workspace) return FF_ERR_NULL;
        if (!aligned(workspace, 256)) return FF_ERR_INVALID;
    }
    if (dweight && (!aligned(dweight, 2) || !rows_ok(dweight_stride, b->width))) return FF_ERR_INVALID;
    if (shared({dweight, stats}, {b->weight}) ||
        (b->n_tokens && (shared({dhidden, dweight, logp, stats}, {b->weight, b->targets, b->weights}) || shared({dweight, logp, stats}, {b->hidden}))))
        return FF_ERR_INVALID;
    FF_HIP_TRY(launch_head(*b, logp, dhidden, dhidden_stride, dweight, dweight_stride, stats, workspace, static_cast<hipStream_t>(hip_stream)));
    return FF_OK;
}

}  // extern "C"
