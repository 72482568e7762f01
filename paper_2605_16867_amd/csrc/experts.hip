// The choice of experts, the order of their slots, and the weighted sum of their results (gfx950).
#include "experts.h"

namespace gr {
namespace {

constexpr int kBlock = 256;
constexpr int kWave = 64;
constexpr int kLaneExperts = 16;     // scores of a row that one lane holds

// ---- choice ------------------------------------------------------------------------------------
//
// A score and its expert are one number of 64 bits: a score in single precision leaves 29 bits of a double's mantissa
// free, and the lowest nine take the expert, so that of two equal scores the lower index is the larger number.
// The largest top_k of a list are then found with minima and maxima alone.
constexpr double kNoExpert = -1.0e300;      // below every score

__device__ __forceinline__ double key_of(float c, int e, bool masked)
{
    if (masked || c == -__builtin_inff()) return kNoExpert;
    double d = (double)(c + 0.0f);            // (-0 counts as 0)
    if (!(c == c)) d = -1.0e200;
    if (c == __builtin_inff()) d = 1.0e200;
    const int64_t b = __double_as_longlong(d);
    return __longlong_as_double((b & ~int64_t(511)) | (b < 0 ? e : 511 - e));
}

__device__ __forceinline__ int expert_of(double key)
{
    const int64_t b = __double_as_longlong(key);
    return key < -1.0e299 ? -1 : (int)(b & 511) ^ (b < 0 ? 0 : 511);
}

__device__ __forceinline__ float larger(float a, float b) { return __builtin_fmaxf(a, b); }

// over the 2^lg lanes of a row's team
__device__ __forceinline__ float team_max(float v, int lg)
{
    for (int m = 1; m < (1 << lg); m *= 2) v = larger(v, __shfl_xor(v, m));
    return v;
}

__device__ __forceinline__ float team_sum(float v, int lg)
{
    for (int m = 1; m < (1 << lg); m *= 2) v += __shfl_xor(v, m);
    return v;
}

// What turns a row's logits into its scores: softmax is exp(x - shift) * inv, sigmoid needs neither.
struct Softmax {
    float shift, inv;
};

template <int V>
__device__ __forceinline__ Softmax softmax_of(const float (&x)[V], int lg)
{
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < V; ++i) m = larger(m, x[i]);
    m = team_max(m, lg);
    if (m == -__builtin_inff()) return {0.0f, 0.0f};       // (nothing but masked experts)
    float sum = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) sum += expf(x[i] - m);
    return {m, 1.0f / team_sum(sum, lg)};
}

template <bool kSigmoid>
__device__ __forceinline__ float score_of(float x, Softmax sm)
{
    if (kSigmoid) return 1.0f / (1.0f + expf(-x));
    return expf(x - sm.shift) * sm.inv;
}

// A lane's share of a row: experts first .. first + V - 1; -inf where there is none.
template <typename T, int V>
__device__ __forceinline__ void load_row(float (&x)[V], const T* row, int first, int n_expert, bool whole)
{
    if (whole) {
        typedef typename Chunk<T>::Vec Vec;
        constexpr int n = Chunk<T>::n;
        if (first < n_expert) {
#pragma unroll
            for (int i = 0; i < V / n; ++i) {
                const Vec v = reinterpret_cast<const Vec*>(row + first)[i];
#pragma unroll
                for (int j = 0; j < n; ++j) x[i * n + j] = (float)v[j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = -__builtin_inff();
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = first + i < n_expert ? (float)row[first + i] : -__builtin_inff();
}

struct RouteArgs {
    RouteIn in;
    float* weight;
    int* expert;
    int lg;          // log2 of the lanes per row
    int whole;       // rows are whole chunks of a lane, 16 bytes aligned
};

template <typename T, int K, bool kSigmoid, bool kGroups>
__global__ __launch_bounds__(kBlock) void k_route(RouteArgs a)
{
    constexpr int V = kLaneExperts;
    const int lg = a.lg, team = 1 << lg, lane = threadIdx.x & (team - 1);
    const int64_t row = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> lg;
    const bool there = row < a.in.rows;
    const int E = a.in.n_expert, first = lane * V;
    const T* const at = static_cast<const T*>(a.in.logits) + (there ? row : 0) * E;

    float x[V];
    load_row<T, V>(x, at, first, E, a.whole);
    Softmax sm{};
    if (!kSigmoid) sm = softmax_of<V>(x, lg);

    float c[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const bool masked = x[i] == -__builtin_inff();
        c[i] = masked ? x[i] : score_of<kSigmoid>(x[i], sm) + (a.in.bias ? a.in.bias[first + i] : 0.0f);
    }

    uint32_t kept = ~0u;
    if constexpr (kGroups) {
        // the groups' two largest, by lanes of the team in turn; each group's rank by counting the better ones
        __shared__ float all[kBlock * V];
        __shared__ double group[kBlock * V];       // (of each team the first n_group: a group has at least one expert)
        float* const mine = all + (threadIdx.x >> lg) * (team * V);
        double* const g_mine = group + (threadIdx.x >> lg) * (team * V);
#pragma unroll
        for (int i = 0; i < V; ++i) mine[first + i] = c[i];
        __syncthreads();
        const int n = E / a.in.n_group;
        for (int g = lane; g < a.in.n_group; g += team) {
            double b0 = kNoExpert, b1 = kNoExpert;
            for (int i = 0; i < n; ++i) {
                const float v = mine[g * n + i];
                const double k = key_of(v, 0, false);
                b1 = fmax(b1, fmin(b0, k));
                b0 = fmax(b0, k);
            }
            // (the keys hold the scores but for the index bits, which are the same in all)
            const auto value = [](double k) { return k == kNoExpert ? 0.0f : k < -1.0e199 ? __builtin_nanf("") : (float)k; };
            float sum = value(b0) + value(b1);
            if (b0 == kNoExpert) sum = -__builtin_inff();
            g_mine[g] = key_of(sum, g, false);
        }
        __syncthreads();
        kept = 0;
        for (int g = lane; g < a.in.n_group; g += team) {
            int better = 0;
            for (int i = 0; i < a.in.n_group; ++i) better += g_mine[i] > g_mine[g];
            if (better < a.in.kept) kept |= 1u << g;
        }
        for (int m = 1; m < team; m *= 2) kept |= __shfl_xor(kept, m);
    }

    double best[K];
#pragma unroll
    for (int j = 0; j < K; ++j) best[j] = kNoExpert;
    int in_group = 0, group_no = 0, group_size = E;
    if constexpr (kGroups) {
        group_size = E / a.in.n_group;
        group_no = first / group_size;
        in_group = first - group_no * group_size;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        double k = key_of(c[i], first + i, false);
        if constexpr (kGroups) {
            if (!(kept >> (group_no & 31) & 1)) k = kNoExpert;
            if (++in_group == group_size) { in_group = 0; ++group_no; }
        }
#pragma unroll
        for (int j = 0; j < (i + 1 < K ? i + 1 : K); ++j) {
            const double up = fmax(best[j], k);
            k = fmin(best[j], k);
            best[j] = up;
        }
    }
    // lanes' lists, each in order, become the team's: the larger of one list's j-th and the other's j-th from the end are
    // the K largest of both
    for (int m = 1; m < team; m *= 2) {
        double other[K];
#pragma unroll
        for (int j = 0; j < K; ++j) other[j] = __shfl_xor(best[K - 1 - j], m);
#pragma unroll
        for (int j = 0; j < K; ++j) best[j] = fmax(best[j], other[j]);
#pragma unroll
        for (int d = K / 2; d > 0; d /= 2)
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (!(j & d)) {
                    const double hi = fmax(best[j], best[j + d]), lo = fmin(best[j], best[j + d]);
                    best[j] = hi;
                    best[j + d] = lo;
                }
    }
    float s[K], sum = 0;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        s[j] = 0;
        if (j < a.in.top_k && (j & (team - 1)) == lane) {
            const int e = expert_of(best[j]);
            if (e >= 0) s[j] = score_of<kSigmoid>((float)at[e], sm);
            sum += s[j];
        }
    }
    float by = a.in.scale;
    if (a.in.renorm) {
        sum = team_sum(sum, lg);
        by = sum == 0 ? 0.0f : a.in.scale / sum;
    }
    if (!there) return;
#pragma unroll
    for (int j = 0; j < K; ++j)
        if (j < a.in.top_k && (j & (team - 1)) == lane) {
            a.weight[row * a.in.top_k + j] = s[j] * by;
            a.expert[row * a.in.top_k + j] = expert_of(best[j]);
        }
}

struct RouteBackArgs {
    RouteIn in;
    const int* expert;
    const float* dweight;
    void* dlogits;
    int lg, whole;
};

template <typename T, bool kSigmoid>
__global__ __launch_bounds__(kBlock) void k_route_back(RouteBackArgs a)
{
    constexpr int V = kLaneExperts;
    const int lg = a.lg, team = 1 << lg, lane = threadIdx.x & (team - 1);
    const int64_t row = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> lg;
    const bool there = row < a.in.rows;
    const int E = a.in.n_expert, first = lane * V, k = a.in.top_k;
    const int64_t r = there ? row : 0;
    const T* const at = static_cast<const T*>(a.in.logits) + r * E;
    float x[V];
    load_row<T, V>(x, at, first, E, a.whole);
    Softmax sm{};
    if (!kSigmoid) sm = softmax_of<V>(x, lg);
    float s[V], u[V];
    bool chosen[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        s[i] = x[i] == -__builtin_inff() ? 0.0f : score_of<kSigmoid>(x[i], sm);
        u[i] = 0;
        chosen[i] = false;
    }
    for (int j = 0; j < k; ++j) {
        const int e = a.expert[r * k + j] - first;
        const float d = a.dweight[r * k + j];
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (e == i && first + i < E) { u[i] = d * a.in.scale; chosen[i] = true; }
    }
    // sum of u over the shares, and of the chosen scores
    float dot = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (chosen[i]) { dot += u[i] * s[i]; sum += s[i]; }
    dot = team_sum(dot, lg);
    float inv = 1;
    if (a.in.renorm) {
        sum = team_sum(sum, lg);
        inv = sum == 0 ? 0.0f : 1.0f / sum;
        dot *= inv;
    }
    if (!there) return;
    float d[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (a.in.renorm) d[i] = chosen[i] ? s[i] * inv * (u[i] - dot) * (kSigmoid ? 1 - s[i] : 1.0f) : 0.0f;
        else if (kSigmoid) d[i] = chosen[i] ? s[i] * (1 - s[i]) * u[i] : 0.0f;
        else d[i] = s[i] * (u[i] - dot);
    }
    T* const out = static_cast<T*>(a.dlogits) + row * E;
    if (a.whole) {
        typedef typename Chunk<T>::Vec Vec;
        constexpr int n = Chunk<T>::n;
        if (first < E) {
#pragma unroll
            for (int i = 0; i < V / n; ++i) {
                Vec v;
#pragma unroll
                for (int j = 0; j < n; ++j) v[j] = (T)d[i * n + j];
                reinterpret_cast<Vec*>(out + first)[i] = v;
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (first + i < E) out[first + i] = (T)d[i];
}

// Lanes per row: each holds kLaneExperts scores.
int team_log(int n_expert)
{
    int lg = 0;
    while ((kLaneExperts << lg) < n_expert) ++lg;
    return lg;
}

template <typename T>
bool whole_rows(const void* a, const void* b, int n_expert)
{
    return n_expert % kLaneExperts == 0 && aligned16(a) && aligned16(b);
}

template <typename T, int K>
void route_by_form(const RouteArgs& a, hipStream_t s)
{
    const int64_t blocks = ((a.in.rows << a.lg) + kBlock - 1) / kBlock;
    const bool groups = a.in.kept < a.in.n_group;
    if (a.in.scoring == GR_SCORE_SIGMOID)
        groups ? k_route<T, K, true, true><<<blocks, kBlock, 0, s>>>(a) : k_route<T, K, true, false><<<blocks, kBlock, 0, s>>>(a);
    else
        groups ? k_route<T, K, false, true><<<blocks, kBlock, 0, s>>>(a) : k_route<T, K, false, false><<<blocks, kBlock, 0, s>>>(a);
}

// ---- order -------------------------------------------------------------------------------------
//
// A counting sort by expert that keeps the order of slots: how many slots of each expert every unit of slots holds, the sums
// of those over the units before, and every slot to its place.  Slots without an expert are those of expert E.

__device__ __forceinline__ int bin_of(int e, int n_expert) { return (unsigned)e < (unsigned)n_expert ? e : n_expert; }

__global__ __launch_bounds__(kWave) void k_plan_count(const int* expert, int64_t slots, int n_expert, int* counts)
{
    __shared__ int cnt[GR_MAX_EXPERTS + 1];
    for (int e = threadIdx.x; e <= n_expert; e += kWave) cnt[e] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * kPlanUnit;
    for (int i = threadIdx.x; i < kPlanUnit; i += kWave)
        if (from + i < slots) atomicAdd(&cnt[bin_of(expert[from + i], n_expert)], 1);
    __syncthreads();
    for (int e = threadIdx.x; e <= n_expert; e += kWave) counts[(int64_t)blockIdx.x * (n_expert + 1) + e] = cnt[e];
}

// One workgroup per expert: its counts become the sums over the units before.
__global__ __launch_bounds__(kBlock) void k_plan_scan(int* counts, int units, int n_expert, int* totals)
{
    __shared__ int wave_sum[kBlock / kWave];
    const int e = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int before = 0;
    for (int u0 = 0; u0 < units; u0 += kBlock) {
        const int u = u0 + threadIdx.x;
        int* const at = counts + (int64_t)u * (n_expert + 1) + e;
        const int own = u < units ? *at : 0;
        int v = own;
        for (int d = 1; d < kWave; d *= 2) {
            const int o = __shfl_up(v, d);
            if (lane >= d) v += o;
        }
        if (lane == kWave - 1) wave_sum[wave] = v;
        __syncthreads();
        int base = before, all = 0;
        for (int w = 0; w < kBlock / kWave; ++w) {
            if (w < wave) base += wave_sum[w];
            all += wave_sum[w];
        }
        if (u < units) *at = base + v - own;
        before += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) totals[e] = before;
}

__global__ __launch_bounds__(kWave) void k_plan_place(const int* expert, int64_t slots, int n_expert, const int* counts,
                                                      const int* totals, int* off, int* slot, int* pos)
{
    __shared__ int next[GR_MAX_EXPERTS + 1];
    const int lane = threadIdx.x;
    int before = 0;
    for (int e0 = 0; e0 <= n_expert; e0 += kWave) {
        const int e = e0 + lane, own = e <= n_expert ? totals[e] : 0;
        int v = own;
        for (int d = 1; d < kWave; d *= 2) {
            const int o = __shfl_up(v, d);
            if (lane >= d) v += o;
        }
        if (e <= n_expert) {
            const int at = before + v - own;
            next[e] = at + counts[(int64_t)blockIdx.x * (n_expert + 1) + e];
            if (blockIdx.x == 0) off[e] = at;
        }
        before += __shfl(v, kWave - 1);
    }
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * kPlanUnit;
    int bits = 0;
    while ((n_expert >> bits) > 0) ++bits;
    for (int i = 0; i < kPlanUnit; i += kWave) {
        const int64_t s = from + i + lane;
        const bool there = s < slots;
        const int e = there ? bin_of(expert[s], n_expert) : 0;
        unsigned long long alike = __ballot(there);
        for (int b = 0; b < bits; ++b) {
            const unsigned long long with = __ballot(e >> b & 1);
            alike &= e >> b & 1 ? with : ~with;
        }
        const int rank = __popcll(alike & ((1ull << lane) - 1));
        int at = 0;
        if (there) at = next[e];
        __syncthreads();
        if (there) {
            if (rank == 0) next[e] = at + __popcll(alike);
            slot[at + rank] = e < n_expert ? (int)s : -1 - (int)s;
            pos[s] = e < n_expert ? at + rank : -1;
        }
        __syncthreads();
    }
}

__global__ void k_no_slots(int* off, int n_expert)
{
    for (int e = threadIdx.x; e <= n_expert; e += blockDim.x) off[e] = 0;
}

// ---- weighted sum ------------------------------------------------------------------------------
//
// Bound by memory: every result is read once, every sum written once.  A thread takes 16 bytes of a row's width (one element where
// rows are not whole 16 bytes).

template <typename T, int N>
struct Piece {
    typedef T Vec __attribute__((ext_vector_type(N)));
};
template <typename T>
struct Piece<T, 1> {
    struct Vec {
        T v;
        __device__ T& operator[](int) { return v; }
        __device__ T operator[](int) const { return v; }
    };
};

struct CombineArgs {
    const float* weight;
    const int* pos;      // or slot, backward
    const void *y, *dout;
    void *out, *dy;
    float* dweight;
    int64_t rows, slots;
    int top_k, width, pieces, lg;
};

template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_combine(CombineArgs a)
{
    typedef typename Piece<T, N>::Vec Vec;
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x, row = i / a.pieces;
    if (row >= a.rows) return;
    const int c = (int)(i - row * a.pieces) * N;
    float sum[N] = {};
    for (int j = 0; j < a.top_k; ++j) {
        const int p = a.pos[row * a.top_k + j];
        if (p < 0 || p >= a.slots) continue;
        const float w = a.weight ? a.weight[row * a.top_k + j] : 1.0f;
        const Vec v = *reinterpret_cast<const Vec*>(static_cast<const T*>(a.y) + (int64_t)p * a.width + c);
#pragma unroll
        for (int n = 0; n < N; ++n) sum[n] = fmaf(w, (float)v[n], sum[n]);
    }
    Vec o;
#pragma unroll
    for (int n = 0; n < N; ++n) o[n] = (T)sum[n];
    *reinterpret_cast<Vec*>(static_cast<T*>(a.out) + row * a.width + c) = o;
}

// A team of 2^lg lanes takes a position.
template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_combine_back(CombineArgs a)
{
    typedef typename Piece<T, N>::Vec Vec;
    const int lane = threadIdx.x & ((1 << a.lg) - 1);
    const int64_t p = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> a.lg;
    if (p >= a.slots) return;             // (whole teams)
    const int given = a.pos[p];
    int64_t s = given < 0 ? -1 - (int64_t)given : given;
    const bool kept = given >= 0 && s < a.slots;
    if (s >= a.slots) s = a.slots - 1;
    const int64_t row = s / a.top_k;
    const float w = a.weight ? a.weight[s] : 1.0f;
    float dot = 0;
    for (int c = lane * N; c < a.width; c += N << a.lg) {
        Vec o;
        if (kept) {
            const Vec d = *reinterpret_cast<const Vec*>(static_cast<const T*>(a.dout) + row * a.width + c);
            if (a.dweight) {
                const Vec y = *reinterpret_cast<const Vec*>(static_cast<const T*>(a.y) + p * a.width + c);
#pragma unroll
                for (int n = 0; n < N; ++n) dot = fmaf((float)d[n], (float)y[n], dot);
            }
#pragma unroll
            for (int n = 0; n < N; ++n) o[n] = (T)(w * (float)d[n]);
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n) o[n] = (T)0.0f;
        }
        if (a.dy) *reinterpret_cast<Vec*>(static_cast<T*>(a.dy) + p * a.width + c) = o;
    }
    if (!a.dweight) return;
    dot = team_sum(dot, a.lg);
    if (lane == 0) a.dweight[s] = dot;
}

template <typename T>
bool by_chunk(int width, const void* a, const void* b, const void* c)
{
    return width % Chunk<T>::n == 0 && aligned16(a) && aligned16(b) && aligned16(c);
}

}  // namespace

int launch_route(const RouteIn& in, int dtype, float* weight, int* expert, hipStream_t s)
{
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const RouteArgs a{in, weight, expert, team_log(in.n_expert), whole_rows<T>(in.logits, nullptr, in.n_expert)};
        in.top_k <= 2 ? route_by_form<T, 2>(a, s) : in.top_k <= 8 ? route_by_form<T, 8>(a, s) : route_by_form<T, 16>(a, s);
        return launched();
    });
}

int launch_route_backward(const RouteIn& in, int dtype, const int* expert, const float* dweight, void* dlogits, hipStream_t s)
{
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const RouteBackArgs a{in, expert, dweight, dlogits, team_log(in.n_expert), whole_rows<T>(in.logits, dlogits, in.n_expert)};
        const int64_t blocks = ((in.rows << a.lg) + kBlock - 1) / kBlock;
        if (in.scoring == GR_SCORE_SIGMOID) k_route_back<T, true><<<blocks, kBlock, 0, s>>>(a);
        else k_route_back<T, false><<<blocks, kBlock, 0, s>>>(a);
        return launched();
    });
}

int launch_plan(gr_experts* h, int64_t slots, const int* expert, int* off, int* slot, int* pos, hipStream_t s)
{
    const int E = h->n_expert, units = (int)((slots + kPlanUnit - 1) / kPlanUnit);
    if (units == 0) {
        k_no_slots<<<1, kBlock, 0, s>>>(off, E);
        return launched();
    }
    k_plan_count<<<units, kWave, 0, s>>>(expert, slots, E, h->counts);
    k_plan_scan<<<E + 1, kBlock, 0, s>>>(h->counts, units, E, h->totals);
    k_plan_place<<<units, kWave, 0, s>>>(expert, slots, E, h->counts, h->totals, off, slot, pos);
    return launched();
}

int launch_combine(int64_t rows, int top_k, int width, int dtype, const float* weight, const int* pos, const void* y, void* out,
                   hipStream_t s)
{
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        CombineArgs a{};
        a.weight = weight; a.pos = pos; a.y = y; a.out = out;
        a.rows = rows; a.slots = rows * top_k; a.top_k = top_k; a.width = width;
        const bool chunks = by_chunk<T>(width, y, out, nullptr);
        a.pieces = chunks ? width / Chunk<T>::n : width;
        const int64_t blocks = (rows * a.pieces + kBlock - 1) / kBlock;
        if (chunks) k_combine<T, Chunk<T>::n><<<blocks, kBlock, 0, s>>>(a);
        else k_combine<T, 1><<<blocks, kBlock, 0, s>>>(a);
        return launched();
    });
}

int launch_combine_backward(int64_t rows, int top_k, int width, int dtype, const float* weight, const int* slot, const void* y,
                            const void* dout, void* dy, float* dweight, hipStream_t s)
{
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        CombineArgs a{};
        a.weight = weight; a.pos = slot; a.y = y; a.dout = dout; a.dy = dy; a.dweight = dweight;
        a.rows = rows; a.slots = rows * top_k; a.top_k = top_k; a.width = width;
        const bool chunks = by_chunk<T>(width, y, dout, dy);
        const int pieces = chunks ? width / Chunk<T>::n : width;
        while ((1 << a.lg) < pieces && a.lg < 6) ++a.lg;
        const int64_t blocks = ((a.slots << a.lg) + kBlock - 1) / kBlock;
        if (chunks) k_combine_back<T, Chunk<T>::n><<<blocks, kBlock, 0, s>>>(a);
        else k_combine_back<T, 1><<<blocks, kBlock, 0, s>>>(a);
        return launched();
    });
}

}  // namespace gr
