// Dropout whose mask is never stored (gfx950).
//
//   out_i = residual_i + (u_i < limit ? 0 : x_i * 65536 / (65536 - limit)),  u_i 16 random bits
//
// Random bits are Philox 4x32 with ten rounds, a counter-based generator (Salmon, Moraes, Dror, Shaw 2011): four words of a counter and two of a key
// give four random words, so any block of bits is there without those before it, forward and backward alike.  16 bits an element make a block
// eight elements, 16 bytes of a 16-bit type; rates are multiples of 2^-16, as the scale is.
//
// Bound by memory: 2^28 elements in bfloat16 with a residual 1.6 GB, 254 us, 6.3 TB/s.  A block of bits is twenty products of 32 bits and forty other
// operations for its eight elements; with all else 141 vector instructions a thread, busy for 47 % of the time.
#include "tokens.h"

namespace gr {
namespace {

constexpr int kBlock = 256, kPer = 8;      // threads of a workgroup; elements of a block of random bits

struct Words {
    uint32_t w[4];
};

__device__ __forceinline__ Words philox(uint64_t counter, uint64_t offset, uint64_t seed)
{
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p = (uint64_t)0xD2511F53u * c0, q = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)q;
        c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// Product and sum are rounded to single precision together, then once to the type.
template <typename T>
__device__ __forceinline__ T kept(float x, uint32_t bits, uint32_t limit, float scale, float residual, bool add)
{
    if (bits < limit) return (T)(add ? residual : 0.0f);
    return (T)(add ? fmaf(x, scale, residual) : x * scale);
}

template <typename T, bool kPast>
__global__ __launch_bounds__(kBlock) void k_dropout(DropoutIn in, float scale, T* out)
{
    typedef Elements<T, kPer> Of;
    const T *const x = static_cast<const T*>(in.x), *const residual = static_cast<const T*>(in.residual);
    const uint64_t offset = in.offset + (in.offset_add ? *in.offset_add : 0);
    const int64_t blocks = (in.n + kPer - 1) / kPer;
    for (int64_t b = (int64_t)blockIdx.x * kBlock + threadIdx.x; b < blocks; b += (int64_t)gridDim.x * kBlock) {
        const Words r = philox((uint64_t)b, offset, in.seed);
        const int64_t at = b * kPer;
        if (at + kPer <= in.n) {
            const Of v = load_of<kPast, T, kPer>(x + at);
            Of o, add{};
            if (residual) add = load_of<kPast, T, kPer>(residual + at);
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                o.v[j] = kept<T>((float)v.v[j], r.w[j / 2] >> (j % 2 * 16) & 0xFFFF, in.limit, scale, (float)add.v[j], residual != nullptr);
            store_of<kPast>(out + at, o);
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (at + j < in.n)
                    out[at + j] = kept<T>((float)x[at + j], r.w[j / 2] >> (j % 2 * 16) & 0xFFFF, in.limit, scale,
                                          residual ? (float)residual[at + j] : 0.0f, residual != nullptr);
        }
    }
}

}  // namespace

int launch_dropout(const DropoutIn& in, int dtype, void* out, hipStream_t s)
{
    const int64_t blocks = (in.n + (int64_t)kPer * kBlock - 1) / (kPer * kBlock);
    const float scale = 65536.0f / (float)(65536 - in.limit);
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const unsigned grid = (unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks);
        if (past_cache(in.n * (int64_t)sizeof(T) * (in.residual ? 3 : 2))) k_dropout<T, true><<<grid, kBlock, 0, s>>>(in, scale, static_cast<T*>(out));
        else k_dropout<T, false><<<grid, kBlock, 0, s>>>(in, scale, static_cast<T*>(out));
        return launched();
    });
}

}  // namespace gr
