// extern "C" entry points of the gradient lists and the policy loss (see include/ffsnap.h for the contract).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/ffsnap.h"
#include "grads.hpp"
#include "policy.hpp"
#include "status.hpp"

using namespace ffsnap;

struct ff_grad_list {
    bool host_only = false, has_addresses = false;
    int device = -1;
    void* dev_block = nullptr;  // items, then addresses
    GradWork work;
    uint64_t numel = 0;
    std::vector<uint32_t> item_size;  // of every tensor's elements; 0: it has none
};

namespace {

uint32_t element_size(uint32_t dtype) { return dtype == FF_F32 ? 4 : dtype == FF_BF16 || dtype == FF_F16 ? 2 : 0; }
bool aligned(const void* p, uint64_t a) { return reinterpret_cast<uint64_t>(p) % a == 0; }

int check_device(const ff_grad_list* list)
{
    if (list->host_only) return FF_ERR_HOST_ONLY;
    int dev = -1;
    FF_HIP_TRY(hipGetDevice(&dev));
    return dev == list->device ? FF_OK : FF_ERR_INVALID;
}

// Are the addresses of a call, or the list's own, all there?
int check_grads(const ff_grad_list* list, const void* const* grads)
{
    if (!grads) return list->has_addresses ? FF_OK : FF_ERR_NULL;
    for (size_t i = 0; i < list->item_size.size(); i++) {
        if (!list->item_size[i]) continue;
        if (!grads[i]) return FF_ERR_NULL;
        if (!aligned(grads[i], list->item_size[i])) return FF_ERR_INVALID;
    }
    return FF_OK;
}

bool positive(double v) { return v > 0.0; }  // not a NaN
// A loss scale, or its reciprocal, that is one in 32 bits as well.
bool scale_ok(double v) { return positive(static_cast<float>(v)) && std::isfinite(static_cast<float>(v)); }

int upload(ff_grad_list* list, const std::vector<GradItem>& items, const std::vector<uint64_t>& address)
{
    FF_HIP_TRY(hipGetDevice(&list->device));
    const uint64_t item_bytes = items.size() * sizeof(GradItem), address_bytes = address.size() * 8;
    if (item_bytes + address_bytes == 0) return FF_OK;
    std::vector<unsigned char> host(item_bytes + address_bytes);
    if (item_bytes) std::memcpy(host.data(), items.data(), item_bytes);
    if (address_bytes) std::memcpy(host.data() + item_bytes, address.data(), address_bytes);
    const hipError_t e = hipMalloc(&list->dev_block, host.size());
    if (e != hipSuccess) return alloc_fail(e);
    FF_HIP_TRY(hipMemcpy(list->dev_block, host.data(), host.size(), hipMemcpyHostToDevice));
    unsigned char* const d = static_cast<unsigned char*>(list->dev_block);
    list->work.items = reinterpret_cast<const GradItem*>(d);
    if (address_bytes) list->work.address = reinterpret_cast<const uint64_t*>(d + item_bytes);
    return FF_OK;
}

int create_list(const ff_segment* segs, uint64_t n, ff_grad_list* list)
{
    std::vector<uint64_t> address(n);
    list->has_addresses = true;
    for (uint64_t i = 0; i < n; i++) {
        const ff_segment& s = segs[i];
        const uint32_t size = element_size(s.dtype);
        if (!size || s.kind != FF_KIND_RAW || s.reserved || s.nbytes % size || !aligned(s.ptr, size)) return FF_ERR_INVALID;
        list->item_size.push_back(s.nbytes ? size : 0);
        list->numel += s.nbytes / size;
        address[i] = reinterpret_cast<uint64_t>(s.ptr);
        if (s.nbytes && !s.ptr) list->has_addresses = false;
    }
    if (!list->has_addresses) address.clear();
    list->work.n = n;
    std::vector<GradItem> items;
    if (!build_grad_items(segs, n, items, list->work.launch)) return FF_ERR_INVALID;
    if (list->host_only) return FF_OK;
    return upload(list, items, address);
}

}  // namespace

extern "C" {

int ff_grad_list_create(const ff_segment* segs, uint64_t n, uint32_t flags, ff_grad_list** out)
{
    if (!out) return FF_ERR_NULL;
    *out = nullptr;
    if (n && !segs) return FF_ERR_NULL;
    if (flags & ~FF_PLAN_HOST_ONLY || n > 0xFFFFFFFFull) return FF_ERR_INVALID;
    ff_grad_list* list = new (std::nothrow) ff_grad_list();
    if (!list) return FF_ERR_NOMEM;
    list->host_only = (flags & FF_PLAN_HOST_ONLY) != 0;
    int rc;
    try {
        rc = create_list(segs, n, list);
    } catch (const std::bad_alloc&) {
        rc = FF_ERR_NOMEM;
    }
    if (rc != FF_OK) {
        ff_grad_list_destroy(list);
        return rc;
    }
    *out = list;
    return FF_OK;
}

void ff_grad_list_destroy(ff_grad_list* list)
{
    if (!list) return;
    if (list->dev_block) (void)hipFree(list->dev_block);
    delete list;
}

uint64_t ff_grad_list_numel(const ff_grad_list* list) { return list ? list->numel : 0; }

uint64_t ff_grad_list_workspace_bytes(const ff_grad_list* list) { return list ? grad_workspace(list->work) : 0; }

int ff_grad_norm(const ff_grad_list* list, const void* const* grads, double inv_loss_scale, double max_norm,
                 void* workspace, ff_grad_stats* stats, void* hip_stream)
{
    if (!list || !workspace || !stats) return FF_ERR_NULL;
    if (!scale_ok(inv_loss_scale) || !positive(max_norm)) return FF_ERR_INVALID;
    if (!aligned(workspace, 16) || !aligned(stats, 8)) return FF_ERR_INVALID;
    int rc = check_grads(list, grads);
    if (rc == FF_OK) rc = check_device(list);
    if (rc != FF_OK) return rc;
    FF_HIP_TRY(launch_grad_norm(list->work, grads, inv_loss_scale, max_norm, workspace, stats,
                                static_cast<hipStream_t>(hip_stream)));
    return FF_OK;
}

int ff_grad_norm_join(const ff_grad_stats* parts, uint64_t n_parts, double inv_loss_scale, double max_norm,
                      ff_grad_stats* stats, void* hip_stream)
{
    if (!parts || !stats) return FF_ERR_NULL;
    if (!n_parts || !scale_ok(inv_loss_scale) || !positive(max_norm) || !aligned(parts, 8) || !aligned(stats, 8))
        return FF_ERR_INVALID;
    FF_HIP_TRY(launch_grad_join(parts, n_parts, inv_loss_scale, max_norm, stats, static_cast<hipStream_t>(hip_stream)));
    return FF_OK;
}

int ff_grad_clip(const ff_grad_list* list, const void* const* grads, const ff_grad_stats* stats, void* hip_stream)
{
    if (!list || !stats) return FF_ERR_NULL;
    if (!aligned(stats, 8)) return FF_ERR_INVALID;
    int rc = check_grads(list, grads);
    if (rc == FF_OK) rc = check_device(list);
    if (rc != FF_OK) return rc;
    FF_HIP_TRY(launch_grad_clip(list->work, grads, stats, static_cast<hipStream_t>(hip_stream)));
    return FF_OK;
}

uint64_t ff_policy_workspace_bytes(uint64_t n_tokens, uint64_t vocab) { return policy_workspace(n_tokens, vocab); }

int ff_policy_loss(const ff_policy_batch* b, float* logp, float* token_loss, void* dlogits, uint64_t grad_stride,
                   ff_policy_stats* stats, void* workspace, void* hip_stream)
{
    if (!b || !stats) return FF_ERR_NULL;
    const uint32_t size = element_size(b->dtype);
    if (!size || b->reserved || b->vocab == 0 || b->vocab > 0x7FFFFFFFull || b->n_tokens > 0x7FFFFFFFull) return FF_ERR_INVALID;
    if (!(b->clip_low >= 0.f && b->clip_low <= 1.f) || !(b->clip_high >= 0.f) || !(b->beta >= 0.f) || !std::isfinite(b->beta) ||
        !std::isfinite(b->clip_high) || !scale_ok(b->loss_scale))
        return FF_ERR_INVALID;
    if (b->beta > 0.f && !b->ref_logp) return FF_ERR_NULL;
    if (!aligned(stats, 8)) return FF_ERR_INVALID;
    if (b->n_tokens) {
        if (!b->logits || !b->targets || !b->old_logp || !b->advantages || !b->weights || !logp || !token_loss || !workspace)
            return FF_ERR_NULL;
        if (!aligned(b->logits, size) || !aligned(b->targets, 8) || !aligned(b->old_logp, 4) || !aligned(b->ref_logp, 4) ||
            !aligned(b->advantages, 4) || !aligned(b->weights, 4) || !aligned(logp, 4) || !aligned(token_loss, 4) ||
            !aligned(dlogits, size) || !aligned(workspace, 16))
            return FF_ERR_INVALID;
        if (b->row_stride < b->vocab || (dlogits && grad_stride < b->vocab)) return FF_ERR_INVALID;
        if (dlogits == b->logits && grad_stride != b->row_stride) return FF_ERR_INVALID;
    }
    FF_HIP_TRY(launch_policy(*b, logp, token_loss, dlogits, grad_stride, stats, workspace, static_cast<hipStream_t>(hip_stream)));
    return FF_OK;
}

}  // extern "C"
