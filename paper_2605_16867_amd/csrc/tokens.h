// Internal declarations shared by the source files of the operators that read a request's tokens
// (embed.hip, scan.hip, dropout.hip).  The public interface and the mathematics are in goodroute.h.
#pragma once

#include "experts.h"

struct gr_tokens {
    int64_t max_tokens = 0;
    int max_vocab = 0, max_width = 0;
    int2* order = nullptr;     // [2][max_tokens] tokens and where they stood, before and after a pass of the sort (see embed.hip)
    float* parts = nullptr;    // [n_parts] parts of long sums (see embed.hip)
    int64_t n_parts = 0;
    int2* ended = nullptr;     // [embed_pieces] rows that pieces share
    uint64_t* words = nullptr;      // [n_words] what workgroups of a recurrence tell each other (see scan.hip)
    size_t n_words = 0;
    uint64_t* control = nullptr;      // its counters
    int counters = 0;
    int* digits = nullptr;     // [kDigits][units] tokens of each digit in each unit, then those before; behind them those of all units
};

namespace gr {

// A call whose arrays are more than half of the device's last-level cache (256 MB) goes past it: what it reads and writes once would only push itself
// out.  With 6 to 40 times that: the recurrence of 262 144 x 1 024 in bfloat16 379 us for 406, backward 692 for 722, dropout of 2^28 elements 257 for
// 272, the gradient of 524 288 rows of 1 024 285 for 300; with 33 MB that the last kernel may have left there, 34 us for 30 (16 000 rows of 512).
inline bool past_cache(int64_t bytes) { return bytes > int64_t(128) << 20; }

// N neighbouring elements at any address of one, past the cache or not.
template <bool kPast, typename T, int N>
__device__ __forceinline__ Elements<T, N> load_of(const T* at)
{
    typedef T Vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    Elements<T, N> e;
    if (kPast) {
        const Vec v = __builtin_nontemporal_load(reinterpret_cast<const Vec*>(at));
        __builtin_memcpy(&e, &v, sizeof e);
    } else e = Elements<T, N>::load(at);
    return e;
}

template <bool kPast, typename T, int N>
__device__ __forceinline__ void store_of(T* at, const Elements<T, N>& e)
{
    typedef T Vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    if (kPast) {
        Vec v;
        __builtin_memcpy(&v, &e, sizeof e);
        __builtin_nontemporal_store(v, reinterpret_cast<Vec*>(at));
    } else e.store(at);
}

constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;      // of a pass of the sort
constexpr int kSortUnit = 2048;                               // tokens that a workgroup puts in order
inline int64_t sort_units(int64_t n) { return (n + kSortUnit - 1) / kSortUnit; }

constexpr int kPieceItems = 1024;                             // of a piece of the sums, at most
int64_t embed_pieces(int64_t n, int vocab);
int64_t embed_parts(int64_t n, int vocab, int width);
int launch_embed(int64_t n, int vocab, int width, int dtype, const int* token, const void* table, float scale, void* out, hipStream_t s);
int launch_embed_backward(gr_tokens* h, int64_t n, int vocab, int width, int dtype, const int* token, const void* dout, float scale,
                          void* dtable, hipStream_t s);

struct ScanIn {
    const int* off;      // null: every token is a sequence
    const void *gate, *x, *y, *dy;
    const float *h0, *dh;
    int64_t n, n_seq, gate_stride, x_stride, dgate_stride, dx_stride;
    int width;
};
constexpr int kScanChannels = 4, kScanLanesLog = 5;      // channels that a lane takes of a row; log2 of lanes that share one
constexpr int kScanLine = 16;                                           // words from one counter to the next
int scan_counters(int width);
size_t scan_words(int64_t n, int width);
int launch_scan(gr_tokens* h, const ScanIn& in, int dtype, void* y, float* last, hipStream_t s);
int launch_scan_backward(gr_tokens* h, const ScanIn& in, int dtype, void* dgate, void* dx, float* dh0, hipStream_t s);

struct DropoutIn {
    const void *x, *residual;
    const uint64_t* offset_add;
    int64_t n;
    uint64_t seed, offset;
    int limit;      // of 65 536 elements so many are dropped
};
int launch_dropout(const DropoutIn& in, int dtype, void* out, hipStream_t s);

}  // namespace gr
