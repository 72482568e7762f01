// The choice of experts, the order of their slots, and the weighted sum of their results (gfx950).
#include <type_traits>

#include "experts.h"

namespace gr {
namespace {

constexpr int kBlock = kRouteBlock;
constexpr int kWave = 64;
constexpr int kPlanWaves = kBlock / kWave;
constexpr int kScanBlock = 1024;
// Batches of rows of a workgroup of the choice: one, and two or four where that leaves four workgroups to each compute unit, so that there are
// fewer counts to add up and longer runs to place.  Always one / this: 131 072 rows of 64 experts, eight of them, 41.5 / 35.7 us, 524 288 of nine,
// two, 34.6 / 29.5; from one workgroup to a unit on, 34.4 and 29.2, but 32 768 of nine 13.3 / 12.2.
constexpr int kEnoughUnits = 1024;
// Units of slots whose counts every workgroup adds up by itself; more have a launch for it.  The launch always / this / never: 2 units 12.4 / 9.6
// / 9.6 us, 32 12.3 / 10.3 / 10.0, 128 12.4 / 12.2 / 12.5, 512 14.3 / 15.2 / 21.6, 1 024 (131 072 rows of 64 experts) 36 / 36 / 72.
constexpr int kFewUnits = 128;

// ---- within a team of lanes ----------------------------------------------------------------------
//
// 2^lg neighbouring lanes share a row.  Step m exchanges between halves of 2m lanes whose lanes all hold the same already, so which lane of the
// other half is asked does not matter: within 16 lanes the register file's own permutations do.

template <int kStep>
__device__ __forceinline__ int other_half(int v)
{
    if constexpr (kStep == 1) return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true);        // quad_perm 1 0 3 2
    if constexpr (kStep == 2) return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true);        // quad_perm 2 3 0 1
    if constexpr (kStep == 4) return __builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, true);       // row_half_mirror
    if constexpr (kStep == 8) return __builtin_amdgcn_mov_dpp(v, 0x140, 0xF, 0xF, true);       // row_mirror
    return __shfl_xor(v, kStep);
}
template <int kStep>
__device__ __forceinline__ float other_half(float v) { return __int_as_float(other_half<kStep>(__float_as_int(v))); }
template <int kStep>
__device__ __forceinline__ double other_half(double v)
{
    return __hiloint2double(other_half<kStep>(__double2hiint(v)), other_half<kStep>(__double2loint(v)));
}

// `join` (a value, the other half's) at every step
template <typename V, typename F>
__device__ __forceinline__ V over_team(V v, int lg, F join)
{
    if (lg > 0) v = join(v, other_half<1>(v));
    if (lg > 1) v = join(v, other_half<2>(v));
    if (lg > 2) v = join(v, other_half<4>(v));
    if (lg > 3) v = join(v, other_half<8>(v));
    if (lg > 4) v = join(v, other_half<16>(v));
    if (lg > 5) v = join(v, other_half<32>(v));
    return v;
}

__device__ __forceinline__ float team_max(float v, int lg)
{
    return over_team(v, lg, [](float a, float b) { return __builtin_fmaxf(a, b); });
}
__device__ __forceinline__ float team_sum(float v, int lg)
{
    return over_team(v, lg, [](float a, float b) { return a + b; });
}

// ---- choice ------------------------------------------------------------------------------------
//
// A score and its expert are one number of 64 bits: a score in single precision leaves 29 bits of a double's mantissa
// free, and the lowest nine take the expert, so that of two equal scores the lower index is the larger number.
// The largest top_k of a list are then found with minima and maxima alone: a lane sorts eight of its scores by a network and merges them, half
// against half, with what it has; then lanes merge theirs.
//
// Bound by vector instructions: 262 144 rows of 64 experts in bfloat16, eight of them, take 31 us, where reading the 33.5 MB is 7.  A batch of 16
// rows is about 900 of a wave (a third of them exponentials, half scores, keys and the choice), and they keep the units two thirds busy at four
// waves a unit.  Keys of 32 bits would be cheaper, but cannot hold a score whole and its expert.  Lanes share a row by 16 scores each: 16 are four
// loads of 16 bytes in single precision, and a list that stays in registers.  Asking for a batch's rows during the one before took longer (48.7 /
// 45.7 with the places).
//
// Scores are computed and leave in single precision whatever the type of the logits.
constexpr int kNoExpert = (int)0xFE37E43C;      // upper half of a number below every score's (-1e300)

__device__ __forceinline__ double key_of(float c, int e)      // (c is not -0: a score is not)
{
    const double d = (double)__builtin_amdgcn_fmed3f(c, -3.4028235e38f, 3.4028235e38f);      // (what is no number is the least score)
    const int hi = __double2hiint(d), lo = __double2loint(d) | ((511 - e) ^ (hi >> 31 & 511));
    return __hiloint2double(c == -__builtin_inff() ? kNoExpert : hi, lo);
}

__device__ __forceinline__ int expert_of(double key)
{
    const int hi = __double2hiint(key);
    return hi == kNoExpert ? -1 : 511 - ((__double2loint(key) ^ hi >> 31) & 511);      // (every score's is larger)
}

// (fmax and fmin would first quiet what might be a signalling not-a-number; keys are numbers)
__device__ __forceinline__ double key_max(double a, double b)
{
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ double key_min(double a, double b)
{
    double r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// The larger first.
__device__ __forceinline__ void in_order(double& a, double& b)
{
    const double up = key_max(a, b);
    b = key_min(a, b);
    a = up;
}

// Lists of N in order, by odd-even merges: 19 exchanges for 8, 63 for 16, where insertion takes 28 and 120.
template <int N>
__device__ __forceinline__ void sort_list(double* v)
{
#pragma unroll
    for (int p = 1; p < N; p *= 2)
#pragma unroll
        for (int k = p; k >= 1; k /= 2)
#pragma unroll
            for (int i = k % p; i + k < N; ++i)
                if ((i - k % p) / k % 2 == 0 && i / (2 * p) == (i + k) / (2 * p)) in_order(v[i], v[i + k]);
}

// The N largest of two lists in order, in order: the larger of one's j-th and the other's j-th from the end are those, falling and
// rising once; `other`(j) gives the other's.
template <int N, typename F>
__device__ __forceinline__ void join_lists(double* v, F other)
{
    double of[N];
#pragma unroll
    for (int j = 0; j < N; ++j) of[j] = other(N - 1 - j);
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = key_max(v[j], of[j]);
#pragma unroll
    for (int d = N / 2; d > 0; d /= 2)
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (!(j & d)) in_order(v[j], v[j + d]);
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
    for (int i = 0; i < V; ++i) m = __builtin_fmaxf(m, x[i]);
    m = team_max(m, lg);
    if (m == -__builtin_inff()) m = 0;       // (nothing but masked experts, whose scores are 0 whatever this is)
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

// Chosen scores that add up to less than this (a bias chose them, or all of a row's sigmoids are small) are divided by their sum another way: in
// single precision they may have lost their digits, and the reciprocal of their sum may be past its range.  So far down a sigmoid is an exponential to within 2^-30, and so is
// a softmax but for a factor: shares are those of exp(x - the largest chosen x).  (A sum of 0 gives no shares.)
constexpr float kFaint = 0x1p-30f;

// Which expert is number i of a lane's share of a row: neighbouring lanes of a team take neighbouring 16 bytes.
struct Share {
    int lg, lane, n_expert;

    template <int kChunk>
    __device__ __forceinline__ int operator()(int i) const
    {
        return ((i / kChunk << lg) + lane) * kChunk + i % kChunk;
    }
};

// A lane's share of a row; -inf where there is no expert.
template <typename T, int V>
__device__ __forceinline__ void load_row(float (&x)[V], const T* row, const Share& of)
{
    constexpr int n = Chunk<T>::n;
    Elements<T, n> v[V / n];
    if (of.n_expert == V << of.lg) {      // (all lanes have 16: nothing to ask for between the loads)
#pragma unroll
        for (int i = 0; i < V / n; ++i) v[i] = Elements<T, n>::load(row + of.template operator()<n>(i * n));
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (float)v[i / n].v[i % n];
        return;
    }
#pragma unroll
    for (int i = 0; i < V / n; ++i) {
        const int e = of.template operator()<n>(i * n);
        if (e + n <= of.n_expert) v[i] = Elements<T, n>::load(row + e);
        else
#pragma unroll
            for (int j = 0; j < n; ++j) v[i].v[j] = row[e + j < of.n_expert ? e + j : 0];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = of.template operator()<n>(i) < of.n_expert ? (float)v[i / n].v[i % n] : -__builtin_inff();
}

// The order of slots (see below), as far as a workgroup has a part in it.
struct PlanArgs {
    const int* expert;
    int* counts;      // [n_expert + 1][units]
    int *off, *slot, *pos;
    int64_t slots;
    int n_expert, units, per_unit;      // slots of a unit, of the last one fewer
    int summed;                         // counts are those of the units before, the last column's successor those of all
};

__device__ __forceinline__ int bin_of(int e, int n_expert) { return (unsigned)e < (unsigned)n_expert ? e : n_expert; }

template <typename F>
__device__ void place_unit(const PlanArgs& a, int unit, int (*hist)[GR_MAX_EXPERTS + 1], F expert_at);

struct RouteArgs {
    RouteIn in;
    float* weight;
    int* expert;
    int lg;          // log2 of the lanes per row
    uint32_t group_mul;      // 2^20 / experts of a group, rounded up
    PlanArgs plan;   // units 0: no order is asked for
};

template <typename T, int K, bool kSigmoid, bool kGroups>
__global__ __launch_bounds__(kBlock) void k_route(RouteArgs a)
{
    constexpr int V = kLaneExperts, n = Chunk<T>::n;
    const int lg = a.lg, team = 1 << lg, lane = threadIdx.x & (team - 1), rows = kBlock >> lg;
    const int E = a.in.n_expert, k = a.in.top_k;
    __shared__ int hist[kPlanWaves][GR_MAX_EXPERTS + 1];
    // scores of the team's row, by expert, and then weights of the wave's rows, by choice; the workgroup's choices
    __shared__ __attribute__((aligned(16))) float scores[kBlock * V];
    __shared__ int ids[kBlock * (kGroups ? V : K)];      // (or, before they are known, what the groups are scored by)
    float* const mine = scores + (threadIdx.x - lane) * V;
    const int batches = a.plan.units > 0 ? a.plan.per_unit / (rows * k) : 1;
    if (a.plan.units > 1) {
        for (int e = threadIdx.x; e <= E; e += kBlock) hist[0][e] = 0;
        __syncthreads();
    }
    float b[V] = {};
    if (a.in.bias) {
        const Share of{lg, lane, E};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = of.template operator()<n>(i);
            b[i] = a.in.bias[e < E ? e : 0];
        }
    }
    for (int batch = 0; batch < batches; ++batch) {
        // The lane's number, anew: what is made of it is not kept from batch to batch, which took registers for a third of the waves.
        int now = lane;
        asm volatile("" : "+v"(now));
        const Share of{lg, now, E};
        const int64_t row = ((int64_t)blockIdx.x * batches + batch) * rows + (threadIdx.x >> lg);
        const bool there = row < a.in.rows;
        const T* const at = static_cast<const T*>(a.in.logits) + (there ? row : 0) * E;
        float x[V], c[V];
        load_row<T, V>(x, at, of);
        Softmax sm{};
        if (!kSigmoid) sm = softmax_of<V>(x, lg);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float s = score_of<kSigmoid>(x[i], sm);
            c[i] = x[i] == -__builtin_inff() ? x[i] : s + b[i];
            x[i] = s;
        }
        if (a.in.bias)
#pragma unroll
            for (int i = 0; i < V; ++i) mine[of.template operator()<n>(i)] = x[i];

        uint32_t kept = ~0u;
        if constexpr (kGroups) {
            // the groups' two largest, by lanes of the team in turn; each group's rank by counting the better ones
            __shared__ double group[kBlock * V];       // (of each team the first n_group: a group has at least one expert)
            float* const c_mine = reinterpret_cast<float*>(ids) + (threadIdx.x >> lg) * (team * V);
            double* const g_mine = group + (threadIdx.x >> lg) * (team * V);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) c_mine[of.template operator()<n>(i)] = c[i];
            __syncthreads();
            const int size = E / a.in.n_group;
            for (int g = lane; g < a.in.n_group; g += team) {
                // (what is no number counts as the least score meanwhile)
                constexpr float kNone = -__builtin_inff(), kLeast = -3.4028235e38f;
                float b0 = kNone, b1 = kNone;
#pragma unroll 4
                for (int i = 0; i < size; ++i) {
                    const float v = c_mine[g * size + i], w = v == v ? v : kLeast;
                    b1 = __builtin_fmaxf(b1, __builtin_fminf(b0, w));
                    b0 = __builtin_fmaxf(b0, w);
                }
                const auto value = [](float v) { return v == kNone ? 0.0f : v == kLeast ? __builtin_nanf("") : v; };
                g_mine[g] = key_of(b0 == kNone ? kNone : value(b0) + value(b1), g);
            }
            __syncthreads();
            kept = 0;
            for (int g = lane; g < a.in.n_group; g += team) {
                int better = 0;
                for (int i = 0; i < a.in.n_group; ++i) better += g_mine[i] > g_mine[g];
                if (better < a.in.kept) kept |= 1u << g;
            }
            kept = (uint32_t)over_team((int)kept, lg, [](int p, int q) { return p | q; });
        }

        // the lane's K best of its own, in order, then the team's
        double keys[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = of.template operator()<n>(i);
            keys[i] = key_of(c[i], e);
            if constexpr (kGroups) keys[i] = kept >> ((uint32_t)e * a.group_mul >> 20 & 31) & 1 ? keys[i] : __hiloint2double(kNoExpert, 0);
        }
#pragma unroll
        for (int i = 0; i < V; i += K) sort_list<K>(keys + i);
#pragma unroll
        for (int m = K; m < V; m *= 2)
#pragma unroll
            for (int i = 0; i < V; i += 2 * m) join_lists<K>(keys + i, [&](int j) { return keys[i + m + j]; });
        double* const best = keys;
        if (lg > 0) join_lists<K>(best, [&](int j) { return other_half<1>(best[j]); });
        if (lg > 1) join_lists<K>(best, [&](int j) { return other_half<2>(best[j]); });
        if (lg > 2) join_lists<K>(best, [&](int j) { return other_half<4>(best[j]); });
        if (lg > 3) join_lists<K>(best, [&](int j) { return other_half<8>(best[j]); });
        if (lg > 4) join_lists<K>(best, [&](int j) { return other_half<16>(best[j]); });
        // their scores: c itself without a bias
        float s[K], sum = 0;
        int id[K];
#pragma unroll
        for (int j = 0; j < K; ++j) id[j] = j < k ? expert_of(best[j]) : -1;
        if (a.in.bias) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // (a team is of one wave)
#pragma unroll
            for (int j = 0; j < K; ++j) s[j] = mine[id[j] < 0 ? 0 : id[j]];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        } else {
#pragma unroll
            for (int j = 0; j < K; ++j)      // (the least score: no number)
                s[j] = __double2hiint(best[j]) == (int)0xC7EFFFFF ? __builtin_nanf("") : (float)best[j];
        }
#pragma unroll
        for (int j = 0; j < K; ++j) {
            s[j] = id[j] >= 0 ? s[j] : 0.0f;
            sum += s[j];
        }
        if (a.in.renorm) {
            if (sum > 0 && sum < kFaint) {
                float most = -__builtin_inff();
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    s[j] = id[j] >= 0 ? (float)at[id[j]] : -__builtin_inff();
                    most = __builtin_fmaxf(most, s[j]);
                }
                sum = 0;
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    s[j] = expf(s[j] - most);
                    sum += s[j];
                }
            }
            const float inv = sum == 0 ? 0.0f : 1.0f / sum;
#pragma unroll
            for (int j = 0; j < K; ++j) s[j] *= inv;
        }
        // out through shared memory, one after the other
        const int wave = threadIdx.x / kWave, at_wave = (wave * kWave >> lg) * k, own = ((threadIdx.x & (kWave - 1)) >> lg) * k;
        float* const weights = scores + wave * kWave * V;
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (j < k && (j & (team - 1)) == lane) {
                weights[own + j] = s[j] * a.in.scale;
                ids[at_wave + own + j] = id[j];
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int64_t first = ((int64_t)blockIdx.x * batches + batch) * rows * k + at_wave, left = a.in.rows * k - first;
        const int count = (kWave >> lg) * k < left ? (kWave >> lg) * k : (int)left;
        for (int i = threadIdx.x & (kWave - 1); i < count; i += kWave) {
            const int e = ids[at_wave + i];
            a.weight[first + i] = weights[i];
            a.expert[first + i] = e;
            if (a.plan.units > 1) atomicAdd(&hist[0][bin_of(e, E)], 1);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    // how many of its slots each expert has; a workgroup alone puts them in order as well
    if (a.plan.units == 0) return;
    __syncthreads();
    if (a.plan.units > 1) {
        for (int e = threadIdx.x; e <= E; e += kBlock) a.plan.counts[(int64_t)e * a.plan.units + blockIdx.x] = hist[0][e];
        return;
    }
    place_unit(a.plan, 0, hist, [&](int i) { return ids[i]; });
}

struct RouteBackArgs {
    RouteIn in;
    const int* expert;
    const float* dweight;
    void* dlogits;
    int lg;
};

// With s the scores, c the chosen, g = scale * dweight there and 0 elsewhere, the gradient by a logit is
//   softmax                s_i (g_i - sum g s)
//   softmax, renormalised  for chosen i: s_i / S (g_i - sum g s / S), S = the sum of s over c; 0 elsewhere (the other shares cancel)
//   sigmoid                the same two with another factor 1 - s_i, without the sum where nothing is renormalised
// Scores are computed again from the logits: reading them back would be as many bytes more.  Bound by memory and a launch: 65 536 rows of 64 in
// single precision, 38 MB with the choices, 10.9 us (3.5 TB/s).  What is chosen goes by expert through shared memory, as a mark and a gradient
// each.
template <typename T, bool kSigmoid>
__global__ __launch_bounds__(kBlock) void k_route_back(RouteBackArgs a)
{
    constexpr int V = kLaneExperts, n = Chunk<T>::n;
    __shared__ __attribute__((aligned(16))) float given[kBlock * V];      // by expert, where there is one
    __shared__ uint32_t marks[kBlock];                                    // 16 experts each
    const int lg = a.lg, team = 1 << lg, lane = threadIdx.x & (team - 1), mine = threadIdx.x - lane;
    const int64_t row = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> lg;
    const bool there = row < a.in.rows;
    const int E = a.in.n_expert, k = a.in.top_k;
    const int64_t r = there ? row : 0;
    const Share of{lg, lane, E};
    const T* const at = static_cast<const T*>(a.in.logits) + r * E;
    marks[threadIdx.x] = 0;
    float x[V];
    load_row<T, V>(x, at, of);
    __syncthreads();
    for (int j = lane; j < k; j += team) {
        const int e = a.expert[r * k + j];
        if ((unsigned)e < (unsigned)E) {
            given[mine * V + e] = a.dweight[r * k + j] * a.in.scale;
            atomicOr(&marks[mine + e / 16], 1u << e % 16);
        }
    }
    Softmax sm{};
    if (!kSigmoid) sm = softmax_of<V>(x, lg);
    float s[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = x[i] == -__builtin_inff() ? 0.0f : score_of<kSigmoid>(x[i], sm);
    float rest[V];      // 1 - s, which a sigmoid's derivative by its logit is s times; near 1 the difference would have no digits
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float e = kSigmoid ? expf(-x[i]) : 0.0f;
        rest[i] = !kSigmoid ? 1.0f : e > 1 ? 1 - s[i] : e * s[i];
    }
    __syncthreads();
    // sum of u over the shares, and of the chosen scores
    float u[V], dot = 0, sum = 0;
    uint32_t chosen = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = of.template operator()<n>(i);      // (below team * V)
        const bool is = marks[mine + e / 16] >> e % 16 & 1;
        const float g = given[mine * V + e];
        u[i] = is ? g : 0.0f;
        chosen |= (uint32_t)is << i;
        dot += is ? g * s[i] : 0.0f;
        sum += is ? s[i] : 0.0f;
    }
    dot = team_sum(dot, lg);
    float inv = 1;
    if (a.in.renorm) {
        sum = team_sum(sum, lg);
        if (sum > 0 && sum < kFaint) {      // (of the whole team)
            float most = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < V; ++i) most = chosen >> i & 1 ? __builtin_fmaxf(most, x[i]) : most;
            most = team_max(most, lg);
            dot = sum = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[i] = chosen >> i & 1 ? expf(x[i] - most) : 0.0f;
                dot += u[i] * s[i];
                sum += s[i];
            }
            dot = team_sum(dot, lg);
            sum = team_sum(sum, lg);
        }
        inv = sum == 0 ? 0.0f : 1.0f / sum;
        dot *= inv;
    }
    if (!there) return;
    float d[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const bool is = chosen >> i & 1;
        if (a.in.renorm) d[i] = is ? s[i] * inv * (u[i] - dot) * rest[i] : 0.0f;
        else if (kSigmoid) d[i] = is ? s[i] * rest[i] * u[i] : 0.0f;
        else d[i] = s[i] * (u[i] - dot);
    }
    T* const out = static_cast<T*>(a.dlogits) + row * E;
#pragma unroll
    for (int i = 0; i < V; i += n) {
        const int e = of.template operator()<n>(i);
        Elements<T, n> v;
#pragma unroll
        for (int j = 0; j < n; ++j) v.v[j] = (T)d[i + j];
        if (e + n <= E) v.store(out + e);
        else
#pragma unroll
            for (int j = 0; j < n - 1; ++j)
                if (e + j < E) out[e + j] = v.v[j];
    }
}

template <typename T, int K>
void route_by_form(const RouteArgs& a, hipStream_t s)
{
    const int64_t blocks = a.plan.units > 0 ? a.plan.units : ((a.in.rows << a.lg) + kBlock - 1) / kBlock;
    const bool groups = a.in.kept < a.in.n_group;
    if (a.in.scoring == GR_SCORE_SIGMOID)
        groups ? k_route<T, K, true, true><<<blocks, kBlock, 0, s>>>(a) : k_route<T, K, true, false><<<blocks, kBlock, 0, s>>>(a);
    else
        groups ? k_route<T, K, false, true><<<blocks, kBlock, 0, s>>>(a) : k_route<T, K, false, false><<<blocks, kBlock, 0, s>>>(a);
}

// ---- order -------------------------------------------------------------------------------------
//
// A counting sort by expert that keeps the order of slots: how many slots of each expert every unit of slots holds, the sums of those over the
// units before, and every slot to its place.  Slots without an expert are those of expert E.  No atomics on memory: the order is the same every
// time.  Bound by the scattered writes of `slot` and the latency of the three steps: 2.1 million slots of 64 experts 11.6 us for the places (25
// MB, 2.2 TB/s) and 4.9 for the sums, where the choice has done the counting; 131 072 rows of 64, eight each, by itself 15.7 us. Units of 1 024
// given slots: of 512 / 1 024 / 4 096 16 384 x 2 of nine 7.1 / 7.4 / 13.6, 131 072 x 8 of 256 30 / 23 / 25.

__global__ __launch_bounds__(kBlock) void k_plan_count(PlanArgs a)
{
    __shared__ int cnt[GR_MAX_EXPERTS + 1];
    for (int e = threadIdx.x; e <= a.n_expert; e += kBlock) cnt[e] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * a.per_unit;
    for (int i = threadIdx.x; i < a.per_unit; i += kBlock)
        if (from + i < a.slots) atomicAdd(&cnt[bin_of(a.expert[from + i], a.n_expert)], 1);
    __syncthreads();
    for (int e = threadIdx.x; e <= a.n_expert; e += kBlock) a.counts[(int64_t)e * a.units + blockIdx.x] = cnt[e];
}

// One workgroup per expert: its counts become the sums over the units before; the sum of all goes behind them all.
__global__ __launch_bounds__(kScanBlock) void k_plan_sum(PlanArgs a)
{
    __shared__ int wave_sum[kScanBlock / kWave];
    const int e = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int* const at = a.counts + (int64_t)e * a.units;
    int before = 0;
    for (int u0 = 0; u0 < a.units; u0 += kScanBlock) {
        const int u = u0 + threadIdx.x, own = u < a.units ? at[u] : 0;
        int v = own;
        for (int d = 1; d < kWave; d *= 2) {
            const int o = __shfl_up(v, d);
            if (lane >= d) v += o;
        }
        if (lane == kWave - 1) wave_sum[wave] = v;
        __syncthreads();
        int base = before, all = 0;
        for (int w = 0; w < kScanBlock / kWave; ++w) {
            if (w < wave) base += wave_sum[w];
            all += wave_sum[w];
        }
        if (u < a.units) at[u] = base + v - own;
        before += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) a.counts[(int64_t)(a.n_expert + 1) * a.units + e] = before;
}

// A unit's slots to their places, by four waves: each counts its own part, then puts it in order 64 slots at a time.  `expert_at`(i): of the
// unit's slot i.
template <typename F>
__device__ void place_unit(const PlanArgs& a, int unit, int (*hist)[GR_MAX_EXPERTS + 1], F expert_at)
{
    __shared__ int wave_sum[kPlanWaves], carry;
    const int E = a.n_expert, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t from = (int64_t)unit * a.per_unit;
    const int n = a.slots - from < a.per_unit ? (int)(a.slots - from) : a.per_unit;
    const int part = (n + kPlanWaves * kWave - 1) / (kPlanWaves * kWave) * kWave, begin = wave * part, end = begin + part < n ? begin + part : n;
    for (int i = threadIdx.x; i < kPlanWaves * (E + 1); i += kBlock) hist[i / (E + 1)][i % (E + 1)] = 0;
    if (threadIdx.x == 0) carry = 0;
    __syncthreads();
    // (several slots of a lane asked for at a time)
    constexpr int kHeld = 8;
    int held[kHeld];
    const auto hold = [&](int i0) {
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const int i = i0 + h * kWave + lane;
            held[h] = expert_at(i < end ? i : begin);
        }
    };
    for (int i0 = begin; i0 < end; i0 += kHeld * kWave) {
        hold(i0);
#pragma unroll
        for (int h = 0; h < kHeld; ++h)
            if (i0 + h * kWave + lane < end) atomicAdd(&hist[wave][bin_of(held[h], E)], 1);
    }
    __syncthreads();
    // where each expert's slots of this unit go: behind all of the experts before, those of the units before, those of the waves before
    for (int e0 = 0; e0 <= E; e0 += kBlock) {
        const int e = e0 + threadIdx.x;
        int mine = 0, all = 0, own[kPlanWaves] = {};
        if (e <= E) {
            for (int w = 0; w < kPlanWaves; ++w) own[w] = hist[w][e];
            if (a.units == 1) {
                for (int w = 0; w < kPlanWaves; ++w) all += own[w];
            } else if (a.summed) {
                mine = a.counts[(int64_t)e * a.units + unit];
                all = a.counts[(int64_t)(E + 1) * a.units + e];
            } else {
#pragma unroll 8
                for (int u = 0; u < a.units; ++u) {
                    const int c = a.counts[e * a.units + u];
                    mine += u < unit ? c : 0;
                    all += c;
                }
            }
        }
        int v = all;
        for (int d = 1; d < kWave; d *= 2) {
            const int o = __shfl_up(v, d);
            if (lane >= d) v += o;
        }
        if (lane == kWave - 1) wave_sum[wave] = v;
        __syncthreads();
        int at = carry + v - all, sum = 0;
        for (int w = 0; w < kPlanWaves; ++w) {
            if (w < wave) at += wave_sum[w];
            sum += wave_sum[w];
        }
        if (e <= E) {
            if (unit == 0) a.off[e] = at;
            at += mine;
            for (int w = 0; w < kPlanWaves; ++w) {
                hist[w][e] = at;
                at += own[w];
            }
        }
        __syncthreads();
        if (threadIdx.x == 0) carry += sum;
        __syncthreads();
    }
    int bits = 0;
    while ((E >> bits) > 0) ++bits;
    for (int i0 = begin; i0 < end; i0 += kHeld * kWave) {
        if (end - begin > kHeld * kWave) hold(i0);
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const int i = i0 + h * kWave + lane;
            if (i0 + h * kWave >= end) break;
            const bool there = i < end;
            const int e = there ? bin_of(held[h], E) : 0;
            unsigned long long alike = __ballot(there);
            for (int b = 0; b < bits; ++b) {
                const unsigned long long with = __ballot(e >> b & 1);
                alike &= e >> b & 1 ? with : ~with;
            }
            if (there) {
                const int rank = __popcll(alike & ((1ull << lane) - 1)), at = hist[wave][e] + rank;
                const int64_t s = from + i;
                a.slot[at] = e < E ? (int)s : -1 - (int)s;
                a.pos[s] = e < E ? at : -1;
            }
            // (a wave's reads come before its later writes)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (there && (alike >> lane) == 1) hist[wave][e] += __popcll(alike);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
}

__global__ __launch_bounds__(kBlock) void k_plan_place(PlanArgs a)
{
    __shared__ int hist[kPlanWaves][GR_MAX_EXPERTS + 1];
    const int64_t from = (int64_t)blockIdx.x * a.per_unit;
    place_unit(a, blockIdx.x, hist, [&](int i) { return a.expert[from + i]; });
}

__global__ void k_no_slots(int* off, int n_expert)
{
    for (int e = threadIdx.x; e <= n_expert; e += blockDim.x) off[e] = 0;
}

// behind the counts
int finish_plan(PlanArgs a, hipStream_t s)
{
    if (a.units > kFewUnits) {
        k_plan_sum<<<a.n_expert + 1, kScanBlock, 0, s>>>(a);
        a.summed = 1;
    }
    k_plan_place<<<a.units, kBlock, 0, s>>>(a);
    return launched();
}

// ---- weighted sum ------------------------------------------------------------------------------
//
//   out[r] = sum over j of weight[r, j] * y[pos[r, j]];  dy[p] = weight * dout[row],  dweight = dout[row] . y[p]
//
// Bound by memory: every result is read once, every sum written once.  65 536 rows, two results each of 1 024 in float16 (403 MB): 77 us, 5.2
// TB/s; rows of nine single numbers, backward, 4.6 us.  Sums are in single precision in the order of j and rounded once; a weight is single
// precision whatever the type.  A thread takes 16 bytes of a row's width, at any address; where a row is no whole number of those the last ones
// reach back into the ones before, and both come to the same values.

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
    typedef Elements<T, N> Of;
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x, row = i / a.pieces;
    if (row >= a.rows) return;
    int c = (int)(i - row * a.pieces) * N;
    if (c + N > a.width) c = a.width - N;
    float sum[N] = {};
    for (int j = 0; j < a.top_k; ++j) {
        const int p = a.pos[row * a.top_k + j];
        if (p < 0 || p >= a.slots) continue;
        const float w = a.weight ? a.weight[row * a.top_k + j] : 1.0f;
        const Of v = Of::load(static_cast<const T*>(a.y) + (int64_t)p * a.width + c);
#pragma unroll
        for (int n = 0; n < N; ++n) sum[n] = fmaf(w, (float)v.v[n], sum[n]);
    }
    Of o;
#pragma unroll
    for (int n = 0; n < N; ++n) o.v[n] = (T)sum[n];
    o.store(static_cast<T*>(a.out) + row * a.width + c);
}

// A team of 2^lg lanes takes a position: dy needs its weight and dweight a sum over its width, so both come from one pass over y and dout.  20 000
// x 9 of 512 in bfloat16 (391 MB) 89 us, 4.4 TB/s.
template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_combine_back(CombineArgs a)
{
    typedef Elements<T, N> Of;
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
    for (int at = lane * N; at < a.width; at += N << a.lg) {
        const int c = at + N > a.width ? a.width - N : at, again = at - c;      // columns that the lane before has as well: not added twice
        Of o;
        if (kept) {
            const Of d = Of::load(static_cast<const T*>(a.dout) + row * a.width + c);
            if (a.dweight) {
                const Of y = Of::load(static_cast<const T*>(a.y) + p * a.width + c);
#pragma unroll
                for (int n = 0; n < N; ++n) dot = n >= again ? fmaf((float)d.v[n], (float)y.v[n], dot) : dot;
            }
#pragma unroll
            for (int n = 0; n < N; ++n) o.v[n] = (T)(w * (float)d.v[n]);
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n) o.v[n] = (T)0.0f;
        }
        if (a.dy) o.store(static_cast<T*>(a.dy) + p * a.width + c);
    }
    if (!a.dweight) return;
    dot = team_sum(dot, a.lg);
    if (lane == 0) a.dweight[s] = dot;
}

}  // namespace

int launch_route(gr_experts* h, const RouteIn& in, int dtype, float* weight, int* expert, int* off, int* slot, int* pos, hipStream_t s)
{
    if (in.rows > ((kMostBlocks - 1) * kBlock >> team_log(in.n_expert))) return GR_ERR_TOO_LARGE;
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const int size = in.n_expert / in.n_group;
        RouteArgs a{in, weight, expert, team_log(in.n_expert), (uint32_t)(((1 << 20) + size - 1) / size), {}};
        if (off) {
            // a unit of slots is what a workgroup chooses: more than one batch of rows where that leaves enough workgroups
            int rows = kBlock >> a.lg;
            const int64_t batches = (in.rows + rows - 1) / rows;
            if (batches >= 4 * kEnoughUnits) rows *= 4;
            else if (batches >= 2 * kEnoughUnits) rows *= 2;
            a.plan = {expert, h->counts, off, slot, pos, in.rows * in.top_k, in.n_expert, (int)((in.rows + rows - 1) / rows), rows * in.top_k, 0};
        }
        in.top_k <= 2 ? route_by_form<T, 2>(a, s) : in.top_k <= 8 ? route_by_form<T, 8>(a, s) : route_by_form<T, 16>(a, s);
        return a.plan.units > 1 ? finish_plan(a.plan, s) : launched();
    });
}

int launch_route_backward(const RouteIn& in, int dtype, const int* expert, const float* dweight, void* dlogits, hipStream_t s)
{
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const RouteBackArgs a{in, expert, dweight, dlogits, team_log(in.n_expert)};
        const int64_t blocks = ((in.rows << a.lg) + kBlock - 1) / kBlock;
        if (blocks > kMostBlocks) return (int)GR_ERR_TOO_LARGE;
        if (in.scoring == GR_SCORE_SIGMOID) k_route_back<T, true><<<blocks, kBlock, 0, s>>>(a);
        else k_route_back<T, false><<<blocks, kBlock, 0, s>>>(a);
        return launched();
    });
}

int launch_plan(gr_experts* h, int64_t slots, const int* expert, int* off, int* slot, int* pos, hipStream_t s)
{
    const int E = h->n_expert;
    if (slots == 0) {
        k_no_slots<<<1, kBlock, 0, s>>>(off, E);
        return launched();
    }
    const PlanArgs a{expert, h->counts, off, slot, pos, slots, E, (int)((slots + kPlanUnit - 1) / kPlanUnit), kPlanUnit, 0};
    if (a.units > 1) k_plan_count<<<a.units, kBlock, 0, s>>>(a);
    return finish_plan(a, s);
}

int launch_combine(int64_t rows, int top_k, int width, int dtype, const float* weight, const int* pos, const void* y, void* out,
                   hipStream_t s)
{
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        CombineArgs a{};
        a.weight = weight; a.pos = pos; a.y = y; a.out = out;
        a.rows = rows; a.slots = rows * top_k; a.top_k = top_k; a.width = width;
        const bool chunks = width >= Chunk<T>::n;
        a.pieces = chunks ? (width + Chunk<T>::n - 1) / Chunk<T>::n : width;
        const int64_t blocks = (rows * a.pieces + kBlock - 1) / kBlock;
        if (blocks > kMostBlocks) return (int)GR_ERR_TOO_LARGE;
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
        const bool chunks = width >= Chunk<T>::n;
        const int pieces = chunks ? (width + Chunk<T>::n - 1) / Chunk<T>::n : width;
        while ((1 << a.lg) < pieces && a.lg < 6) ++a.lg;
        const int64_t blocks = ((a.slots << a.lg) + kBlock - 1) / kBlock;
        if (blocks > kMostBlocks) return (int)GR_ERR_TOO_LARGE;
        if (chunks) k_combine_back<T, Chunk<T>::n><<<blocks, kBlock, 0, s>>>(a);
        else k_combine_back<T, 1><<<blocks, kBlock, 0, s>>>(a);
        return launched();
    });
}

}  // namespace gr
