// Host entry points of the operators of a length predictor: the workspace handle and the argument checks.
#include <new>

#include "experts.h"

using namespace gr;

namespace {

template <typename T>
bool dev_alloc(T** p, size_t n)
{
    if (hipMalloc(reinterpret_cast<void**>(p), (n ? n : 1) * sizeof(T)) == hipSuccess) return true;
    (void)hipGetLastError();      // (returned as GR_ERR_NOMEM: left behind, it would be the next launch's)
    return false;
}

// Rows and choices within what the handle was created for; *rc says what is wrong else.
bool slots_ok(const gr_experts* h, int64_t n_rows, int32_t top_k, int* rc)
{
    *rc = GR_ERR_INVALID_ARG;
    if (!h || n_rows < 0 || top_k < 1) return false;
    *rc = GR_ERR_TOO_LARGE;
    if (n_rows > h->max_rows || top_k > h->max_top_k) return false;
    *rc = GR_OK;
    return true;
}

bool route_ok(const gr_experts* h, int64_t n_rows, int32_t top_k, int32_t dtype, int32_t scoring, float scale, int* rc)
{
    if (!slots_ok(h, n_rows, top_k, rc)) return false;
    if (!type_ok(dtype) || (scoring != GR_SCORE_SOFTMAX && scoring != GR_SCORE_SIGMOID) || !(scale - scale == 0) || top_k > h->n_expert) {
        *rc = GR_ERR_INVALID_ARG;
        return false;
    }
    return true;
}

bool linear_ok(const gr_experts* h, int64_t n_pos, int32_t n_in, int32_t n_out, int32_t dtype, const int32_t* slot, int32_t top_k, int* rc)
{
    *rc = GR_ERR_INVALID_ARG;
    if (!h || n_pos < 0 || n_in < 1 || n_out < 1 || !type_ok(dtype) || (slot && top_k < 1)) return false;
    *rc = GR_ERR_TOO_LARGE;
    if (n_pos > h->max_slots || n_in > GR_MAX_WIDTH || n_out > GR_MAX_WIDTH) return false;
    *rc = GR_OK;
    return true;
}

}  // namespace

extern "C" {

int gr_experts_create(gr_experts** out, int32_t n_expert, int64_t max_rows, int32_t max_top_k)
{
    if (!out) return GR_ERR_INVALID_ARG;
    *out = nullptr;
    if (n_expert < 1 || max_rows < 0 || max_top_k < 1 || max_top_k > n_expert) return GR_ERR_INVALID_ARG;
    if (n_expert > GR_MAX_EXPERTS || max_top_k > GR_MAX_TOP_K || max_rows > (int64_t(1) << 30) / max_top_k) return GR_ERR_TOO_LARGE;
    gr_experts* h = new (std::nothrow) gr_experts;
    if (!h) return GR_ERR_NOMEM;
    h->n_expert = n_expert;
    h->max_rows = max_rows;
    h->max_top_k = max_top_k;
    h->max_slots = max_rows * max_top_k;
    if (!dev_alloc(&h->counts, (plan_units(n_expert, max_rows, h->max_slots) + 1) * (n_expert + 1)) || !dev_alloc(&h->squares, kClipParts) ||
        !dev_alloc(&h->parts, kPartFloats)) {
        gr_experts_destroy(h);
        return GR_ERR_NOMEM;
    }
    *out = h;
    return GR_OK;
}

int gr_experts_destroy(gr_experts* h)
{
    if (!h) return GR_OK;
    (void)hipDeviceSynchronize();
    int rc = GR_OK;
    for (void* p : {(void*)h->counts, (void*)h->squares, (void*)h->parts})
        if (p && hipFree(p) != hipSuccess) rc = GR_ERR_HIP;
    delete h;
    return rc;
}

int gr_expert_route(gr_experts* h, int64_t n_rows, int32_t top_k, const void* logits, int32_t dtype, const float* bias,
                    int32_t scoring, int32_t n_group, int32_t n_group_kept, int32_t renormalise, float scale,
                    float* out_weight, int32_t* out_expert, int32_t* out_off, int32_t* out_slot, int32_t* out_pos, void* hip_stream)
{
    int rc;
    if (!route_ok(h, n_rows, top_k, dtype, scoring, scale, &rc)) return rc;
    if (n_group < 1 || n_group_kept < 1 || n_group_kept > n_group || h->n_expert % n_group != 0) return GR_ERR_INVALID_ARG;
    if (n_group > GR_MAX_GROUPS) return GR_ERR_TOO_LARGE;
    const bool plan = out_off || out_slot || out_pos;
    if (plan && (!out_off || (n_rows > 0 && (!out_slot || !out_pos)))) return GR_ERR_INVALID_ARG;
    if (n_rows > 0 && (!logits || !out_weight || !out_expert)) return GR_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (n_rows == 0) return plan ? launch_plan(h, 0, out_expert, out_off, out_slot, out_pos, s) : GR_OK;
    const RouteIn in{logits, bias, n_rows, h->n_expert, top_k, scoring, n_group, n_group_kept, renormalise != 0, scale};
    return launch_route(h, in, dtype, out_weight, out_expert, out_off, out_slot, out_pos, s);
}

int gr_expert_route_backward(gr_experts* h, int64_t n_rows, int32_t top_k, const void* logits, int32_t dtype, int32_t scoring,
                             int32_t renormalise, float scale, const int32_t* expert, const float* dweight,
                             void* out_dlogits, void* hip_stream)
{
    int rc;
    if (!route_ok(h, n_rows, top_k, dtype, scoring, scale, &rc)) return rc;
    if (n_rows == 0) return GR_OK;
    if (!logits || !expert || !dweight || !out_dlogits) return GR_ERR_INVALID_ARG;
    const RouteIn in{logits, nullptr, n_rows, h->n_expert, top_k, scoring, 1, 1, renormalise != 0, scale};
    return launch_route_backward(in, dtype, expert, dweight, out_dlogits, static_cast<hipStream_t>(hip_stream));
}

int gr_expert_plan(gr_experts* h, int64_t n_rows, int32_t top_k, const int32_t* expert, int32_t* out_off, int32_t* out_slot,
                   int32_t* out_pos, void* hip_stream)
{
    int rc;
    if (!slots_ok(h, n_rows, top_k, &rc)) return rc;
    if (!out_off || (n_rows > 0 && (!expert || !out_slot || !out_pos))) return GR_ERR_INVALID_ARG;
    return launch_plan(h, n_rows * top_k, expert, out_off, out_slot, out_pos, static_cast<hipStream_t>(hip_stream));
}

int gr_expert_linear(gr_experts* h, int64_t n_pos, int32_t n_in, int32_t n_out, int32_t dtype, const int32_t* off,
                     const int32_t* slot, int32_t top_k, const void* x, const void* w, const void* bias, int32_t relu,
                     void* out_y, void* hip_stream)
{
    int rc;
    if (!linear_ok(h, n_pos, n_in, n_out, dtype, slot, top_k, &rc)) return rc;
    if (n_pos == 0) return GR_OK;
    if (!x || !w || !out_y) return GR_ERR_INVALID_ARG;
    LinearIn in{};
    in.off = off; in.slot = slot; in.x = x; in.w = w; in.bias = bias; in.n_pos = n_pos;
    in.n_expert = h->n_expert; in.n_in = n_in; in.n_out = n_out; in.top_k = slot ? top_k : 1; in.relu = relu != 0;
    return launch_linear(h, in, dtype, out_y, static_cast<hipStream_t>(hip_stream));
}

int gr_expert_linear_backward(gr_experts* h, int64_t n_pos, int32_t n_in, int32_t n_out, int32_t dtype, const int32_t* off,
                              const int32_t* slot, int32_t top_k, const void* x, const void* w, const void* y, const void* dy,
                              void* out_dz, void* out_dx, void* out_dw, void* out_db, void* hip_stream)
{
    int rc;
    if (!linear_ok(h, n_pos, n_in, n_out, dtype, slot, top_k, &rc)) return rc;
    // (with no positions the gradients of the weights are still written: 0)
    if (n_pos > 0 && (!dy || (out_dw && !x) || (out_dx && !w))) return GR_ERR_INVALID_ARG;
    if (n_pos > 0 && (y == nullptr) != (out_dz == nullptr)) return GR_ERR_INVALID_ARG;
    LinearIn in{};
    in.off = off; in.slot = slot; in.x = x; in.w = w; in.y = y; in.dy = dy; in.n_pos = n_pos;
    in.n_expert = h->n_expert; in.n_in = n_in; in.n_out = n_out; in.top_k = slot ? top_k : 1;
    return launch_linear_backward(h, in, dtype, out_dz, out_dx, out_dw, out_db, static_cast<hipStream_t>(hip_stream));
}

int gr_expert_combine(gr_experts* h, int64_t n_rows, int32_t top_k, int32_t n_out, int32_t dtype, const float* weight,
                      const int32_t* pos, const void* y, void* out, void* hip_stream)
{
    int rc;
    if (!slots_ok(h, n_rows, top_k, &rc)) return rc;
    if (n_out < 1 || !type_ok(dtype)) return GR_ERR_INVALID_ARG;
    if (n_out > GR_MAX_WIDTH) return GR_ERR_TOO_LARGE;
    if (n_rows == 0) return GR_OK;
    if (!pos || !y || !out) return GR_ERR_INVALID_ARG;
    return launch_combine(n_rows, top_k, n_out, dtype, weight, pos, y, out, static_cast<hipStream_t>(hip_stream));
}

int gr_expert_combine_backward(gr_experts* h, int64_t n_rows, int32_t top_k, int32_t n_out, int32_t dtype, const float* weight,
                               const int32_t* slot, const void* y, const void* dout, void* out_dy, float* out_dweight,
                               void* hip_stream)
{
    int rc;
    if (!slots_ok(h, n_rows, top_k, &rc)) return rc;
    if (n_out < 1 || !type_ok(dtype)) return GR_ERR_INVALID_ARG;
    if (n_out > GR_MAX_WIDTH) return GR_ERR_TOO_LARGE;
    if (n_rows == 0 || (!out_dy && !out_dweight)) return GR_OK;
    if (!slot || !dout || (out_dweight && !y)) return GR_ERR_INVALID_ARG;
    return launch_combine_backward(n_rows, top_k, n_out, dtype, weight, slot, y, dout, out_dy, out_dweight, static_cast<hipStream_t>(hip_stream));
}

int gr_clip_gradients(gr_experts* h, int32_t n_grad, const void* const* grad, void* const* out, const int64_t* count,
                      const int32_t* dtype, float max_norm, float* out_norm, void* hip_stream)
{
    if (!h || n_grad < 0 || !(max_norm >= 0) || (n_grad > 0 && (!grad || !out || !count || !dtype))) return GR_ERR_INVALID_ARG;
    if (n_grad > GR_MAX_GRADIENTS) return GR_ERR_TOO_LARGE;
    for (int i = 0; i < n_grad; ++i) {
        if (count[i] < 0 || !type_ok(dtype[i]) || (count[i] > 0 && (!grad[i] || !out[i]))) return GR_ERR_INVALID_ARG;
        if (count[i] > (int64_t(1) << 40)) return GR_ERR_TOO_LARGE;
    }
    return launch_clip(h, n_grad, grad, out, count, dtype, max_norm, out_norm, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
