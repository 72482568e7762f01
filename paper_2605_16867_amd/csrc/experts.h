// Internal declarations shared by the source files of the operators of a length predictor
// (experts.hip, linear.hip, clip.hip).  The public interface and the mathematics are in goodroute.h.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "goodroute.h"

struct gr_experts {
    int n_expert = 0, max_top_k = 0;
    int64_t max_rows = 0, max_slots = 0;
    int* counts = nullptr;       // [n_expert + 1][units of slots] slots of each expert, then those before the unit; behind them those of all units (see k_plan_*)
    double* squares = nullptr;   // [kClipParts] sums of squares (see k_norm)
    float* parts = nullptr;      // [kPartFloats] parts of long sums (see k_linear_*)
};

namespace gr {

constexpr int kPlanUnit = 1024;      // slots of given experts that a workgroup puts in order
constexpr size_t kPartFloats = size_t(16) << 20;
constexpr int kClipBlocks = 1024;    // workgroups of a launch over gradients
constexpr int kClipTensors = 96;     // gradients that one launch takes: their table is passed by value, 3 KB of the 4 that arguments may be
constexpr size_t kClipParts = size_t(kClipBlocks) * ((GR_MAX_GRADIENTS + kClipTensors - 1) / kClipTensors);

typedef __bf16 bf16;
typedef _Float16 f16;

// Calls `f` with a value of the type that `dtype` names.
template <typename F>
int by_type(int dtype, F f)
{
    return dtype == GR_F32 ? f(float{}) : dtype == GR_BF16 ? f(bf16{}) : f(f16{});
}

inline bool type_ok(int dtype) { return dtype == GR_F32 || dtype == GR_BF16 || dtype == GR_F16; }
inline size_t size_of(int dtype) { return dtype == GR_F32 ? 4 : 2; }
inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
constexpr int64_t kMostBlocks = UINT32_MAX / 256;      // workgroups of 256 that a launch may have
inline int launched() { return hipGetLastError() == hipSuccess ? GR_OK : GR_ERR_HIP; }

// The 16 bytes that one access moves, as elements.
template <typename T>
struct Chunk {
    static constexpr int n = 16 / sizeof(T);
    typedef T Vec __attribute__((ext_vector_type(16 / sizeof(T))));
};

constexpr int kRouteBlock = 256, kLaneExperts = 16;      // threads of a workgroup of the choice; scores of a row that a lane holds

// log2 of the lanes that share a row's scores
inline int team_log(int n_expert)
{
    int lg = 0;
    while ((kLaneExperts << lg) < n_expert) ++lg;
    return lg;
}

// Most units of slots of a call: the choice's workgroups, or units of given experts.
inline size_t plan_units(int n_expert, int64_t rows, int64_t slots)
{
    const int64_t of_rows = kRouteBlock >> team_log(n_expert), a = (rows + of_rows - 1) / of_rows, b = (slots + kPlanUnit - 1) / kPlanUnit;
    return (size_t)(a > b ? a : b);
}

// N neighbouring elements at any address of an element: one access where the hardware has one of that size, aligned or not.
template <typename T, int N>
struct Elements {
    T v[N];
    __device__ __forceinline__ static Elements load(const T* at)
    {
        Elements e;
        __builtin_memcpy(&e, at, sizeof e);
        return e;
    }
    __device__ __forceinline__ void store(T* at) const { __builtin_memcpy(at, this, sizeof *this); }
};

struct RouteIn {
    const void* logits;
    const float* bias;
    int64_t rows;
    int n_expert, top_k, scoring, n_group, kept, renorm;
    float scale;
};

// off, slot, pos: null, or the order of the slots as well
int launch_route(gr_experts* h, const RouteIn& in, int dtype, float* weight, int* expert, int* off, int* slot, int* pos, hipStream_t s);
int launch_route_backward(const RouteIn& in, int dtype, const int* expert, const float* dweight, void* dlogits, hipStream_t s);
int launch_plan(gr_experts* h, int64_t slots, const int* expert, int* off, int* slot, int* pos, hipStream_t s);
int launch_combine(int64_t rows, int top_k, int width, int dtype, const float* weight, const int* pos, const void* y, void* out,
                   hipStream_t s);
int launch_combine_backward(int64_t rows, int top_k, int width, int dtype, const float* weight, const int* slot, const void* y,
                            const void* dout, void* dy, float* dweight, hipStream_t s);

struct LinearIn {
    const int *off, *slot;     // null: one matrix; rows are positions
    const void *x, *w, *bias, *y, *dy;
    int64_t n_pos;
    int n_expert, n_in, n_out, top_k, relu;
};
int launch_linear(gr_experts* h, const LinearIn& in, int dtype, void* out_y, hipStream_t s);
int launch_linear_backward(gr_experts* h, const LinearIn& in, int dtype, void* dz, void* dx, void* dw, void* db, hipStream_t s);
int launch_clip(gr_experts* h, int n, const void* const* grad, void* const* out, const int64_t* count, const int* dtype,
                float max_norm, float* norm, hipStream_t s);

}  // namespace gr
