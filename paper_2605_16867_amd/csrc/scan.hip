// A gated recurrence along sequences of tokens, forward and backward (gfx950).
//
//   f = sigmoid(gate), i = sigmoid(-gate);  h_t = f_t h_{t-1} + i_t x_t
//   D_t = dy_t + c_{t+1}, c_t = f_t D_t;  dx_t = i_t D_t, dgate_t = f_t i_t D_t (h_{t-1} - x_t)
#include "tokens.h"

namespace gr {
namespace {

constexpr int kBlock = 256;

struct Gate {
    float keep, take;      // sigmoid(gate), sigmoid(-gate)
};

// Both from exp(-|gate|) =: e, as 1 / (1 + e) and e / (1 + e): neither is a difference, so both have all their digits however far the gate is from 0.
// The exponent's rounding, |gate| log2(e) * 2^-24, is made good where results are in single precision.  (A gate that is no number stays one.)
template <typename T>
__device__ __forceinline__ Gate gate_of(float g)
{
    constexpr float kLog2e = 1.44269504089f, kLog2eRest = 1.92596299e-8f, kLn2 = 0.693147181f;
    float a = fabsf(g);
    a = a > 88.0f ? 88.0f : a;      // (behind that e is no whole number of single precision, and 0 is as good)
    const float p = a * -kLog2e;
    float e = __builtin_amdgcn_exp2f(p);
    if (sizeof(T) == 4) e = fmaf(e, fmaf(a, -kLog2eRest, fmaf(a, -kLog2e, -p)) * kLn2, e);
    const float near = __builtin_amdgcn_rcpf(1.0f + e), far = e * near;
    return g >= 0 ? Gate{near, far} : Gate{far, near};
}

struct Range {
    int64_t from, to;
};

__device__ __forceinline__ Range range_of(const ScanIn& in, int64_t s)
{
    if (!in.off) return {s, s + 1};
    int64_t from = in.off[s], to = in.off[s + 1];
    from = from < 0 ? 0 : from > in.n ? in.n : from;
    to = to < from ? from : to > in.n ? in.n : to;
    return {from, to};
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_scan(ScanIn in, T* y, float* last)
{
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x, s = i / in.width;
    if (s >= in.n_seq) return;
    const int c = (int)(i - s * in.width);
    const T *const gate = static_cast<const T*>(in.gate) + c, *const x = static_cast<const T*>(in.x) + c;
    float h = in.h0 ? in.h0[i] : 0.0f;
    const Range r = range_of(in, s);
    for (int64_t t = r.from; t < r.to; ++t) {
        const Gate g = gate_of<T>((float)gate[t * in.gate_stride]);
        h = fmaf(g.keep, h, g.take * (float)x[t * in.x_stride]);
        if (y) y[t * in.width + c] = (T)h;
    }
    if (last) last[i] = h;
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_scan_back(ScanIn in, T* dgate, T* dx, float* dh0)
{
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x, s = i / in.width;
    if (s >= in.n_seq) return;
    const int c = (int)(i - s * in.width);
    const T *const gate = static_cast<const T*>(in.gate) + c, *const x = static_cast<const T*>(in.x) + c, *const y = static_cast<const T*>(in.y) + c,
        *const dy = static_cast<const T*>(in.dy) + c;
    float carry = in.dh ? in.dh[i] : 0.0f;
    const float h0 = in.h0 ? in.h0[i] : 0.0f;
    const Range r = range_of(in, s);
    for (int64_t t = r.to - 1; t >= r.from; --t) {
        const Gate g = gate_of<T>((float)gate[t * in.gate_stride]);
        const float d = carry + (in.dy ? (float)dy[t * in.width] : 0.0f), v = (float)x[t * in.x_stride];
        const float before = t > r.from ? (float)y[(t - 1) * in.width] : h0;
        dx[t * in.dx_stride + c] = (T)(d * g.take);
        dgate[t * in.dgate_stride + c] = (T)(d * g.take * g.keep * (before - v));
        carry = d * g.keep;
    }
    if (dh0) dh0[i] = carry;
}

}  // namespace

int launch_scan(gr_tokens*, const ScanIn& in, int dtype, void* y, float* last, hipStream_t s)
{
    const int64_t blocks = (in.n_seq * in.width + kBlock - 1) / kBlock;
    if (blocks > kMostBlocks) return GR_ERR_TOO_LARGE;
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        k_scan<T><<<(unsigned)blocks, kBlock, 0, s>>>(in, static_cast<T*>(y), last);
        return launched();
    });
}

int launch_scan_backward(gr_tokens*, const ScanIn& in, int dtype, void* dgate, void* dx, float* dh0, hipStream_t s)
{
    const int64_t blocks = (in.n_seq * in.width + kBlock - 1) / kBlock;
    if (blocks > kMostBlocks) return GR_ERR_TOO_LARGE;
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        k_scan_back<T><<<(unsigned)blocks, kBlock, 0, s>>>(in, static_cast<T*>(dgate), static_cast<T*>(dx), dh0);
        return launched();
    });
}

}  // namespace gr
