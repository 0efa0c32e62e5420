// The router of a mixture of experts: each token's k largest logits, their softmax, and the stable sort of the (token, choice) pairs by
// expert that the grouped products take their rows from; and the gated sum of the experts' outputs behind them.
//
// The sort is a counting sort in two launches.  Tokens are cut into at most kRouteBlocks runs.  The first launch picks the experts, 16 lanes
// a token, and counts each run's pairs of every expert.  The second adds up, for each run, the pairs that precede it -- those of smaller
// experts and those of earlier runs -- and places its own in order.  Only whole numbers are added, so no order of workgroups or atomics
// changes a result.  Small batches take both steps in one launch.  (12288 tokens, 2 of 64 experts: 3.6 and 5.6 us; the
// second reads the counts of all runs in every workgroup, 16 MB from the L2s.)
#include <float.h>

#include "q8_grouped_device.h"

namespace q8 {

constexpr int kRouteBlocks = Q8_ROUTE_BLOCKS, kRouteThreads = 1024, kRouteWaves = kRouteThreads / 64, kRouteExperts = Q8_ROUTE_MAX_EXPERTS;
constexpr int kRouteSinglePairs = 512;  // of a batch that one workgroup takes

// Unsigned order of floats: -inf < ... < -0 < +0 < ... < +inf.  NaN counts as -inf.  +0 and -0 are the same logit.
__device__ __forceinline__ unsigned logit_key(float f)
{
    if (f != f) f = -__builtin_inff();
    const unsigned u = __float_as_uint(__fadd_rn(f, 0.0f));
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of_key(unsigned k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }

// A logit and its index as one number: 2^52 + 2^10 key + 1023 - index, an exact double, so that the larger of two is one instruction and of equal logits the
// lower index is the larger number.  0 is below all of them.
constexpr int kIndexBits = 10;
static_assert(kRouteExperts <= 1 << kIndexBits, "an index has ten bits");
__device__ __forceinline__ double candidate(float logit, int index, bool there)
{
    const unsigned key = logit_key(logit), mask = 0u - (unsigned)there;  // 0 where there is no such logit
    return __hiloint2double((int)((0x43300000u | key >> (32 - kIndexBits)) & mask), (int)((key << kIndexBits | (unsigned)((1 << kIndexBits) - 1 - index)) & mask));
}
__device__ __forceinline__ float logit_of(double c)
{
    return logit_of_key((unsigned)__double2hiint(c) << (32 - kIndexBits) | (unsigned)__double2loint(c) >> kIndexBits);
}
__device__ __forceinline__ int index_of(double c) { return (1 << kIndexBits) - 1 - (__double2loint(c) & ((1 << kIndexBits) - 1)); }

// Over the 16 lanes of a row, the same value in every lane.
template <int kCtrl>
__device__ __forceinline__ int ror(int v)
{
    return __builtin_amdgcn_update_dpp(0, v, 0x120 + kCtrl, 0xf, 0xf, true);
}
template <int kCtrl>
__device__ __forceinline__ double max_ror(double v)
{
    return __builtin_fmax(v, __hiloint2double(ror<kCtrl>(__double2hiint(v)), ror<kCtrl>(__double2loint(v))));
}
__device__ __forceinline__ double row_max(double v) { return max_ror<1>(max_ror<2>(max_ror<4>(max_ror<8>(v)))); }
template <int kCtrl>
__device__ __forceinline__ float add_ror(float v)
{
    return v + __int_as_float(ror<kCtrl>(__float_as_int(v)));
}
__device__ __forceinline__ float row_sum(float v) { return add_ror<1>(add_ror<2>(add_ror<4>(add_ror<8>(v)))); }

__device__ __forceinline__ void exchange(double& a, double& b)
{
    const double large = __builtin_fmax(a, b);
    b = __builtin_fmin(a, b);
    a = large;
}
// c[0 .. n) from "falling, then rising" to falling.
template <int n>
__device__ __forceinline__ void merge_falling(double* c)
{
#pragma unroll
    for (int d = n / 2; d > 0; d /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i)
            if (!(i & d)) exchange(c[i], c[i + d]);
}
// c[0 .. n) in falling order: halves sorted, the largest of the one against the smallest of the other, and either side merged.
template <int n>
__device__ __forceinline__ void sort_falling(double* c)
{
    if constexpr (n > 1) {
        sort_falling<n / 2>(c);
        sort_falling<n / 2>(c + n / 2);
#pragma unroll
        for (int i = 0; i < n / 2; ++i) exchange(c[i], c[n - 1 - i]);
        merge_falling<n / 2>(c);
        merge_falling<n / 2>(c + n / 2);
    }
}

// The k experts of a token by 16 lanes, four tokens a wave.  Lane r of them takes the logits r, r + 16, ... , kPer of them, as falling lists of four; or, beyond 16 of them,
// in batches of 16 of which it keeps the largest 16, one list, and k is no more.  Every round takes the largest head of all lists and moves its list on.
// Minima and maxima of doubles issue at half rate, so lists are short (64 tokens, 8 of 256 experts, one workgroup: a list of 16 11.6 us, lists of four 9.5, all logits
// searched in every round 14.0).
template <int kPer>
__device__ __forceinline__ void choose(const float* __restrict__ logits, int n_experts, int k, int& expert, float& gate)
{
    constexpr int kHeld = kPer < 16 ? kPer : 16, kList = kPer > kHeld ? kHeld : 4;
    const int r = threadIdx.x & 15, row = threadIdx.x & 48;
    double held[kHeld];
#pragma unroll 1
    for (int b = 0; b < kPer; b += kHeld) {
        float raw[kHeld];
        double c[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) raw[i] = logits[min((b + i) * 16 + r, n_experts - 1)];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) asm volatile("" : "+v"(raw[i]));  // all under way before the first is looked at, and no branch around any
#pragma unroll
        for (int i = 0; i < kHeld; ++i) c[i] = candidate(raw[i], (b + i) * 16 + r, (b + i) * 16 + r < n_experts);
#pragma unroll
        for (int i = 0; i < kHeld; i += kList) sort_falling<kList>(c + i);
#pragma unroll
        for (int i = 0; i < kHeld; ++i) held[i] = b ? __builtin_fmax(held[i], c[kHeld - 1 - i]) : c[i];
        if (kPer > kHeld && b) merge_falling<kHeld>(held);
    }
    double chosen = 0.0;
    for (int j = 0; j < k; ++j) {
        double best = held[0];
#pragma unroll
        for (int i = kList; i < kHeld; i += kList) best = __builtin_fmax(best, held[i]);
        const double top = row_max(best);
#pragma unroll
        for (int h = 0; h < kHeld; h += kList) {
            const bool taken = __double2loint(held[h]) == __double2loint(top);  // the index is in the low word
#pragma unroll
            for (int i = 0; i < kList; ++i) {
                const double here = held[h + i], next = i + 1 < kList ? held[h + i + 1] : 0.0;
                held[h + i] = taken ? next : here;
            }
        }
        if (r == j) chosen = top;
    }
    // softmax over the chosen: against the largest, infinities taken as the largest finite number, nothing for -inf
    expert = index_of(chosen);
    const float l = logit_of(chosen);
    const float finite = __builtin_fminf(__builtin_fmaxf(l, -FLT_MAX), FLT_MAX);
    const float p = r < k && l != -__builtin_inff() ? expf(finite - __shfl(finite, row)) : 0.0f;
    const float sum = row_sum(p);
    gate = sum > 0.0f ? __fdiv_rn(p, sum) : 0.0f;
}

// Tokens [t0, t1): experts and gates out, the pairs of each expert counted into hist (LDS, cleared), the experts also to `here` (LDS) if that is given.
template <int kPer>
__device__ __forceinline__ void choose_run(const float* __restrict__ logits, int64_t t0, int64_t t1, int n_experts, int k, int32_t* __restrict__ experts,
                                           float* __restrict__ gates, int* hist, int* here)
{
    const int tokens = (int)blockDim.x / 16;
    const int r = threadIdx.x & 15;
    for (int64_t t = t0 + threadIdx.x / 16; t - (threadIdx.x & 63) / 16 < t1; t += tokens) {  // a wave's lanes stay together: the reductions are a row's
        int e;
        float g;
        choose<kPer>(logits + min(t, t1 - 1) * n_experts, n_experts, k, e, g);
        if (t < t1 && r < k) {
            experts[t * k + r] = e;
            gates[t * k + r] = g;
            atomicAdd(hist + e, 1);
            if (here) here[(t - t0) * k + r] = e;
        }
    }
}

// How the pairs [i0, i1) of a run are placed in order.  Each wave takes a contiguous part in steps of 64, so that within an expert earlier waves
// come first.
struct Part {
    int64_t w0, w1;  // this wave's pairs
    int waves;       // waves that have any
};
__device__ __forceinline__ Part part_of_wave(int64_t i0, int64_t i1)
{
    const int64_t per = ((i1 - i0 + kRouteWaves - 1) / kRouteWaves + 63) / 64 * 64;
    const int64_t w0 = min(i0 + (int64_t)(threadIdx.x >> 6) * per, i1);
    return Part{w0, min(w0 + per, i1), per ? (int)((i1 - i0 + per - 1) / per) : 0};
}

// base[e] (LDS): the place of the run's first pair of expert e.  count (LDS): waves x n_experts, cleared.  expert_at(i): the expert of pair i; first: that of
// this lane's first pair, asked for ahead.
template <class F>
__device__ __forceinline__ void place_run(F expert_at, int first, Part q, int n_experts, int k, const int* base, int* count, int32_t* __restrict__ rows, int32_t* __restrict__ slots)
{
    const int lane = threadIdx.x & 63;
    int* next = count + (threadIdx.x >> 6) * n_experts;
    for (int64_t i = q.w0 + lane; i < q.w1; i += 64) atomicAdd(next + (i - lane == q.w0 ? first : expert_at(i)), 1);
    __syncthreads();
    for (int e = threadIdx.x; e < n_experts; e += kRouteThreads) {
        int at = base[e];
#pragma unroll 4
        for (int w = 0; w < q.waves; ++w) {
            const int n = count[w * n_experts + e];
            count[w * n_experts + e] = at;
            at += n;
        }
    }
    __syncthreads();
    for (int64_t c = q.w0; c < q.w1; c += 64) {
        const int64_t i = c + lane;
        const bool live = i < q.w1;
        const int e = !live ? 0 : c == q.w0 ? first : expert_at(i);
        unsigned long long same = __ballot(live);  // lanes with this lane's expert
        for (int b = 1; b < n_experts; b <<= 1) {
            const unsigned long long set = __ballot(live && (e & b));
            same &= (e & b) ? set : ~set;
        }
        const int rank = __builtin_popcountll(same & ((1ull << lane) - 1));
        if (live) {
            const int at = next[e] + rank;
            rows[at] = (int32_t)((uint32_t)i / (uint32_t)k);
            slots[i] = at;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // all lanes have read before the first of each expert moves its place on
        __builtin_amdgcn_wave_barrier();
        if (live && rank == 0) next[e] += __builtin_popcountll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// base[e] += the sum of total[0 .. e), for up to kRouteThreads experts; scratch: LDS for kRouteWaves integers.
__device__ __forceinline__ void add_smaller_experts(int n_experts, const int* total, int* base, int* scratch)
{
    const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
    const unsigned n = e < n_experts ? (unsigned)total[e] : 0u, upto = wave_scan_most(n, 0x7fffffffu);
    if (n_experts > 64) {
        if (lane == 63) scratch[wave] = (int)upto;
        __syncthreads();
    }
    int before = (int)(upto - n);
    for (int w = 0; w < (e < n_experts ? wave : 0); ++w) before += scratch[w];
    if (e < n_experts) base[e] += before;
    __syncthreads();
}

struct RouteArgs {
    const float* logits;
    int64_t T, run;  // tokens of a run
    int n_experts, k, runs;
    int32_t* experts;
    float* gates;
    int32_t *group_rows, *rows, *slots, *work;
};

template <int kPer>
__global__ __launch_bounds__(kRouteThreads) void route_choose_kernel(RouteArgs a)
{
    __shared__ int hist[kRouteExperts];
    for (int e = threadIdx.x; e < a.n_experts; e += (int)blockDim.x) hist[e] = 0;
    __syncthreads();
    const int64_t t0 = blockIdx.x * a.run, t1 = min(t0 + a.run, a.T);
    choose_run<kPer>(a.logits, t0, t1, a.n_experts, a.k, a.experts, a.gates, hist, nullptr);
    __syncthreads();
    for (int e = threadIdx.x; e < a.n_experts; e += (int)blockDim.x) a.work[blockIdx.x * a.n_experts + e] = hist[e];
}

__global__ __launch_bounds__(kRouteThreads) void route_place_kernel(RouteArgs a)
{
    __shared__ int base[kRouteExperts], total[kRouteExperts], scratch[kRouteWaves];
    __shared__ int count[kRouteWaves * kRouteExperts];
    const int64_t t0 = blockIdx.x * a.run, t1 = min(t0 + a.run, a.T);
    const Part q = part_of_wave(t0 * a.k, t1 * a.k);
    const int64_t i = q.w0 + (threadIdx.x & 63);
    const int first = i < q.w1 ? a.experts[i] : 0;
    for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) base[e] = total[e] = 0;
    for (int e = threadIdx.x; e < q.waves * a.n_experts; e += kRouteThreads) count[e] = 0;
    // The counts of all runs: a thread adds up one expert in every parts-th run, and the parts meet in LDS.
    const int parts = kRouteThreads / a.n_experts, part = threadIdx.x / a.n_experts, mine = threadIdx.x - part * a.n_experts;
    int all = 0, before = 0;
    if (part < parts) {
#pragma unroll 8
        for (int run = part; run < a.runs; run += parts) {
            const int n = a.work[run * a.n_experts + mine];
            all += n;
            before += run < (int)blockIdx.x ? n : 0;
        }
    }
    __syncthreads();
    if (all) atomicAdd(total + mine, all);
    if (before) atomicAdd(base + mine, before);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) a.group_rows[e] = total[e];
    add_smaller_experts(a.n_experts, total, base, scratch);
    place_run([&](int64_t at) { return a.experts[at]; }, first, q, a.n_experts, a.k, base, count, a.rows, a.slots);
}

// Both steps of a batch of one run, the experts kept in LDS.
template <int kPer>
__global__ __launch_bounds__(kRouteThreads) void route_single_kernel(RouteArgs a)
{
    __shared__ int hist[kRouteExperts], base[kRouteExperts], scratch[kRouteWaves], here[kRouteSinglePairs];
    __shared__ int count[kRouteWaves * kRouteExperts];
    const Part q = part_of_wave(0, a.T * a.k);
    for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) hist[e] = base[e] = 0;
    for (int e = threadIdx.x; e < q.waves * a.n_experts; e += kRouteThreads) count[e] = 0;
    __syncthreads();
    choose_run<kPer>(a.logits, 0, a.T, a.n_experts, a.k, a.experts, a.gates, hist, here);
    __syncthreads();
    for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) a.group_rows[e] = hist[e];
    add_smaller_experts(a.n_experts, hist, base, scratch);
    const int64_t i = q.w0 + (threadIdx.x & 63);
    place_run([&](int64_t at) { return here[at]; }, i < q.w1 ? here[i] : 0, q, a.n_experts, a.k, base, count, a.rows, a.slots);
}

template <int kPer>
static int launch(RouteArgs a, hipStream_t st)
{
    // One launch of one workgroup while it has little to search (one launch and two: 128 tokens, 2 of 64 experts 5.9 and 7.1 us; 32 tokens, 8 of 256 7.0 and 8.3, 64
    // tokens 9.6 and 8.6; 128 tokens, 8 of 64 8.8 and 7.2).  Else short runs, of many units, and shorter ones where a token takes long (1024 tokens, 8 of 256 experts,
    // runs of 16 tokens 10.0 us, of 32 10.6, of 64 13.6; 512 tokens, 2 of 64 7.3, 7.2 and 7.0).
    if (a.T <= 128 && a.T * a.k <= kRouteSinglePairs && a.T * kPer * (a.k > 4 ? a.k : 4) <= 4096) {
        a.run = a.T;
        hipLaunchKernelGGL(route_single_kernel<kPer>, dim3(1), dim3(kRouteThreads), 0, st, a);
        return hipGetLastError() == hipSuccess ? 0 : 1;
    }
    const int64_t least = kPer < 16 ? 32 : 16, most = (a.T + kRouteBlocks - 1) / kRouteBlocks;
    a.run = most > least ? most : least;
    a.runs = (int)((a.T + a.run - 1) / a.run);
    const int threads = (int)(a.run * 16 < kRouteThreads ? (a.run * 16 + 63) / 64 * 64 : kRouteThreads);
    hipLaunchKernelGGL(route_choose_kernel<kPer>, dim3((unsigned)a.runs), dim3((unsigned)threads), 0, st, a);
    if (hipGetLastError() != hipSuccess) return 1;
    hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)a.runs), dim3(kRouteThreads), 0, st, a);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

int launch_route(const float* logits, int64_t T, int n_experts, int k, int32_t* experts, float* gates, int32_t* group_rows, int32_t* rows, int32_t* slots,
                 int32_t* work, hipStream_t st)
{
    const RouteArgs a{logits, T, 0, n_experts, k, 0, experts, gates, group_rows, rows, slots, work};
    if (n_experts <= 64) return launch<4>(a, st);
    if (n_experts <= 128) return launch<8>(a, st);
    if (n_experts <= 256) return launch<16>(a, st);
    return launch<kRouteExperts / 16>(a, st);
}

// out[t,:] = sum over j, in order, of gates[t,j] y[slots[t,j],:], in fp32 with one rounding to the output type; a slot outside y adds
// nothing.  Bound by memory: k rows read, one written, 16 bytes a thread at whatever address a row starts, single elements behind a row's
// last whole 16 bytes.  Threads run through out as one run of vectors; the token is a 32-bit division behind the workgroup's own.  Two rows are
// in flight a thread, and the store passes the caches by (12288 x 2 rows of 1024 bf16: 18.6 us without that, 15.0 with; 13.2 with slots and gates read
// without a branch).
typedef unsigned v4u_any __attribute__((ext_vector_type(4), aligned(2)));  // 16 bytes wherever an element may start
template <bool kBf16>
struct CombineVector {
    static constexpr int kElems = kBf16 ? 8 : 4;
    float v[kElems];
    __device__ __forceinline__ void load(const void* y, int64_t at, int left)
    {
        v4u_any w = {0, 0, 0, 0};
        if (left >= kElems) {
            w = *reinterpret_cast<const v4u_any*>(static_cast<const char*>(y) + at * (kBf16 ? 2 : 4));
        } else {
#pragma unroll
            for (int i = 0; i < kElems; ++i)
                if (i < left) {
                    if constexpr (kBf16)
                        w[i / 2] |= (unsigned)static_cast<const unsigned short*>(y)[at + i] << (16 * (i % 2));
                    else
                        w[i] = static_cast<const unsigned*>(y)[at + i];
                }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (kBf16)
                v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            else
                v[i] = __uint_as_float(w[i]);
        }
    }
    __device__ __forceinline__ void store(void* out, int64_t at, int left) const
    {
        if (left >= kElems) {
            v4u_any w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = kBf16 ? f32_to_bf16x2(v[2 * i % kElems], v[(2 * i + 1) % kElems]) : __float_as_uint(v[i]);
            __builtin_nontemporal_store(w, reinterpret_cast<v4u_any*>(static_cast<char*>(out) + at * (kBf16 ? 2 : 4)));
        } else {
#pragma unroll
            for (int i = 0; i < kElems; ++i)
                if (i < left) {
                    if constexpr (kBf16)
                        static_cast<unsigned short*>(out)[at + i] = f32_to_bf16(v[i]);
                    else
                        static_cast<float*>(out)[at + i] = v[i];
                }
        }
    }
};
constexpr int kCombineThreads = 64;
// kWhole: rows are whole vectors.
template <bool kBf16, bool kWhole>
__global__ __launch_bounds__(kCombineThreads) void combine_kernel(const void* __restrict__ y, int64_t R, const int32_t* __restrict__ slots,
                                                                  const float* __restrict__ gates, int64_t T, int k, int64_t N, unsigned per_row, void* __restrict__ out)
{
    using Vector = CombineVector<kBf16>;
    constexpr int kFlight = 2;
    const int64_t first = (int64_t)blockIdx.x * kCombineThreads, t0 = first / per_row;
    const unsigned in = (unsigned)(first - t0 * per_row) + threadIdx.x;  // vectors from the first token's row on
    const unsigned dt = in / per_row;
    const int64_t t = t0 + dt, n = (int64_t)(in - dt * per_row) * Vector::kElems;
    if (t >= T) return;
    const int left = kWhole ? Vector::kElems : (int)min(N - n, (int64_t)Vector::kElems);
    Vector sum;
#pragma unroll
    for (int e = 0; e < Vector::kElems; ++e) sum.v[e] = 0.0f;
    for (int j0 = 0; j0 < k; j0 += kFlight) {
        Vector row[kFlight];
        float g[kFlight];
        int s[kFlight];
        bool there[kFlight];
#pragma unroll
        for (int j = 0; j < kFlight; ++j) {  // slots and gates without a branch, so that none waits for another
            const int64_t at = t * k + min(j0 + j, k - 1);
            s[j] = slots[at];
            g[j] = gates[at];
            there[j] = j0 + j < k && s[j] >= 0 && s[j] < R;
        }
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (there[j]) row[j].load(y, (int64_t)s[j] * N + n, left);
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (there[j]) {
#pragma unroll
                for (int e = 0; e < Vector::kElems; ++e) sum.v[e] = __builtin_fmaf(g[j], row[j].v[e], sum.v[e]);
            }
    }
    sum.store(out, t * N + n, left);
}

int launch_combine(const void* y, int64_t R, const int32_t* slots, const float* gates, int64_t T, int k, int64_t N, void* out, bool bf16, hipStream_t st)
{
    const int64_t elems = bf16 ? 8 : 4, per_row = (N + elems - 1) / elems, blocks = (T * per_row + kCombineThreads - 1) / kCombineThreads;
    if (per_row >= (int64_t)1 << 31 || blocks * kCombineThreads >= (int64_t)1 << 32) return 1;  // a launch is limited to 2^32 threads
    const dim3 grid((unsigned)blocks), block(kCombineThreads);
#define Q8_COMBINE(B, W) hipLaunchKernelGGL((combine_kernel<B, W>), grid, block, 0, st, y, R, slots, gates, T, k, N, (unsigned)per_row, out)
    if (N % elems == 0) {
        if (bf16)
            Q8_COMBINE(true, true);
        else
            Q8_COMBINE(false, true);
    } else if (bf16) {
        Q8_COMBINE(true, false);
    } else {
        Q8_COMBINE(false, false);
    }
#undef Q8_COMBINE
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

}  // namespace q8
