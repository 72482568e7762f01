// Host entry points of the operators that read a request's tokens: the workspace handle and the argument checks.
#include <cmath>
#include <initializer_list>
#include <memory>
#include <new>

#include "tokens.h"

using namespace gr;

namespace {

template <typename T>
bool dev_alloc(T** p, size_t n)
{
    if (hipMalloc(reinterpret_cast<void**>(p), (n ? n : 1) * sizeof(T)) == hipSuccess) return true;
    (void)hipGetLastError();      // (returned as GR_ERR_NOMEM: left behind, it would be the next launch's)
    return false;
}

// Tokens and widths within what the handle was created for.
int sizes(const gr_tokens* h, int64_t n_tokens, int32_t width, int32_t dtype)
{
    if (!h || n_tokens < 0 || width < 1 || !type_ok(dtype)) return GR_ERR_INVALID_ARG;
    return n_tokens > h->max_tokens || width > h->max_width ? GR_ERR_TOO_LARGE : GR_OK;
}

int embed_ok(const gr_tokens* h, int64_t n_tokens, int32_t n_vocab, int32_t width, int32_t dtype, float scale)
{
    if (const int rc = sizes(h, n_tokens, width, dtype)) return rc;
    if (n_vocab < 1 || !std::isfinite(scale)) return GR_ERR_INVALID_ARG;
    return n_vocab > h->max_vocab ? GR_ERR_TOO_LARGE : GR_OK;
}

constexpr int64_t kMostSequences = int64_t(1) << 30;

int scan_ok(const gr_tokens* h, int64_t n_tokens, int64_t n_seq, int32_t width, int32_t dtype, const int32_t* off)
{
    if (const int rc = sizes(h, n_tokens, width, dtype)) return rc;
    if (n_seq < 0 || (!off && n_seq != n_tokens)) return GR_ERR_INVALID_ARG;
    return n_seq > kMostSequences ? GR_ERR_TOO_LARGE : GR_OK;
}

int strides(std::initializer_list<int64_t> all, int32_t width)
{
    for (const int64_t v : all) {
        if (v < width) return GR_ERR_INVALID_ARG;
        if (v > GR_MAX_STRIDE) return GR_ERR_TOO_LARGE;
    }
    return GR_OK;
}

}  // namespace

extern "C" {

int gr_tokens_create(gr_tokens** out, int64_t max_tokens, int32_t max_vocab, int32_t max_width)
{
    if (!out) return GR_ERR_INVALID_ARG;
    *out = nullptr;
    if (max_tokens < 0 || max_vocab < 1 || max_width < 1) return GR_ERR_INVALID_ARG;
    if (max_tokens > (int64_t(1) << 30) || max_vocab > GR_MAX_VOCAB || max_width > GR_MAX_WIDTH) return GR_ERR_TOO_LARGE;
    gr_tokens* h = new (std::nothrow) gr_tokens;
    if (!h) return GR_ERR_NOMEM;
    h->max_tokens = max_tokens;
    h->max_vocab = max_vocab;
    h->max_width = max_width;
    h->n_words = scan_words(max_tokens, max_width);
    h->n_parts = embed_parts(max_tokens, max_vocab, max_width);
    h->counters = scan_counters(max_width);
    const size_t n_control = (size_t)(h->counters + 1) * kScanLine;
    std::unique_ptr<uint64_t[]> first(new (std::nothrow) uint64_t[n_control]());      // (the first call is number 1)
    for (int i = 0; first && i < h->counters; ++i) first[(i + 1) * kScanLine] = uint64_t(1) << 32;
    if (!first || !dev_alloc(&h->words, h->n_words) || hipMemset(h->words, 0, h->n_words * sizeof(uint64_t)) != hipSuccess ||
        !dev_alloc(&h->control, n_control) || hipMemcpy(h->control, first.get(), n_control * sizeof(uint64_t), hipMemcpyHostToDevice) != hipSuccess ||
        !dev_alloc(&h->parts, h->n_parts) || !dev_alloc(&h->ended, (size_t)embed_pieces(max_tokens, max_vocab)) || !dev_alloc(&h->order, 2 * (size_t)max_tokens) || !dev_alloc(&h->digits, (size_t)(sort_units(max_tokens) + 1) * kDigits + 1)) {
        gr_tokens_destroy(h);
        return GR_ERR_NOMEM;
    }
    *out = h;
    return GR_OK;
}

int gr_tokens_destroy(gr_tokens* h)
{
    if (!h) return GR_OK;
    (void)hipDeviceSynchronize();
    int rc = GR_OK;
    for (void* p : {(void*)h->order, (void*)h->digits, (void*)h->parts, (void*)h->ended, (void*)h->words, (void*)h->control})
        if (p && hipFree(p) != hipSuccess) rc = GR_ERR_HIP;
    delete h;
    return rc;
}

int gr_token_embed(gr_tokens* h, int64_t n_tokens, int32_t n_vocab, int32_t width, int32_t dtype, const int32_t* token,
                   const void* table, float scale, void* out, void* hip_stream)
{
    if (const int rc = embed_ok(h, n_tokens, n_vocab, width, dtype, scale)) return rc;
    if (n_tokens == 0) return GR_OK;
    if (!token || !table || !out) return GR_ERR_INVALID_ARG;
    return launch_embed(n_tokens, n_vocab, width, dtype, token, table, scale, out, static_cast<hipStream_t>(hip_stream));
}

int gr_token_embed_backward(gr_tokens* h, int64_t n_tokens, int32_t n_vocab, int32_t width, int32_t dtype, const int32_t* token,
                            const void* dout, float scale, void* out_dtable, void* hip_stream)
{
    if (const int rc = embed_ok(h, n_tokens, n_vocab, width, dtype, scale)) return rc;
    // (with no tokens the gradient is still written: 0)
    if (!out_dtable || (n_tokens > 0 && (!token || !dout))) return GR_ERR_INVALID_ARG;
    return launch_embed_backward(h, n_tokens, n_vocab, width, dtype, token, dout, scale, out_dtable, static_cast<hipStream_t>(hip_stream));
}

int gr_gated_scan(gr_tokens* h, int64_t n_tokens, int64_t n_seq, int32_t width, int32_t dtype, const int32_t* off,
                  const void* gate, int64_t gate_stride, const void* x, int64_t x_stride, const float* h0, void* out_y, float* out_h,
                  void* hip_stream)
{
    if (const int rc = scan_ok(h, n_tokens, n_seq, width, dtype, off)) return rc;
    if (const int rc = strides({gate_stride, x_stride}, width)) return rc;
    if (off && out_h && out_h == h0) return GR_ERR_INVALID_ARG;
    if (n_seq == 0 || (!out_y && !out_h) || (n_tokens == 0 && !out_h)) return GR_OK;
    if (n_tokens > 0 && (!gate || !x)) return GR_ERR_INVALID_ARG;
    ScanIn in{};
    in.off = off; in.gate = gate; in.x = x; in.h0 = h0; in.n = n_tokens; in.n_seq = n_seq; in.width = width;
    in.gate_stride = gate_stride; in.x_stride = x_stride;
    return launch_scan(h, in, dtype, out_y, out_h, static_cast<hipStream_t>(hip_stream));
}

int gr_gated_scan_backward(gr_tokens* h, int64_t n_tokens, int64_t n_seq, int32_t width, int32_t dtype, const int32_t* off,
                           const void* gate, int64_t gate_stride, const void* x, int64_t x_stride, const void* y, const float* h0,
                           const void* dy, const float* dh, void* out_dgate, int64_t dgate_stride, void* out_dx, int64_t dx_stride,
                           float* out_dh0, void* hip_stream)
{
    if (const int rc = scan_ok(h, n_tokens, n_seq, width, dtype, off)) return rc;
    if (const int rc = strides({gate_stride, x_stride, dgate_stride, dx_stride}, width)) return rc;
    if (off && out_dh0 && out_dh0 == dh) return GR_ERR_INVALID_ARG;
    if (n_seq == 0 || (n_tokens == 0 && !out_dh0)) return GR_OK;
    if (n_tokens > 0 && (!gate || !x || !y || !out_dgate || !out_dx)) return GR_ERR_INVALID_ARG;
    ScanIn in{};
    in.off = off; in.gate = gate; in.x = x; in.y = y; in.dy = dy; in.h0 = h0; in.dh = dh; in.n = n_tokens; in.n_seq = n_seq; in.width = width;
    in.gate_stride = gate_stride; in.x_stride = x_stride; in.dgate_stride = dgate_stride; in.dx_stride = dx_stride;
    return launch_scan_backward(h, in, dtype, out_dgate, out_dx, out_dh0, static_cast<hipStream_t>(hip_stream));
}

int gr_dropout(gr_tokens* h, int64_t n, int32_t dtype, const void* x, const void* residual, double rate, uint64_t seed,
               uint64_t offset, const uint64_t* offset_add, void* out, void* hip_stream)
{
    if (!h || n < 0 || !type_ok(dtype) || !(rate >= 0 && rate < 1)) return GR_ERR_INVALID_ARG;
    const int limit = (int)std::nearbyint(rate * 65536);
    if (limit > 65535) return GR_ERR_INVALID_ARG;
    if (n > (int64_t(1) << 40)) return GR_ERR_TOO_LARGE;
    if (n == 0) return GR_OK;
    if (!x || !out) return GR_ERR_INVALID_ARG;
    return launch_dropout({x, residual, offset_add, n, seed, offset, limit}, dtype, out, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
