// The router of a mixture of experts: each token's k largest logits, their softmax, and the stable sort of the (token, choice) pairs by
// expert that the grouped products take their rows from; and the gated sum of the experts' outputs behind them.
//
// The sort is a counting sort in two launches.  Tokens are cut into at most kBlocks runs.  The first launch picks the experts, one wave
// a token, and counts each run's pairs of every expert.  The second adds up, for each run, the pairs that precede it -- those of smaller
// experts and those of earlier runs -- and places its own in order.  Only whole numbers are added, so no order of workgroups or atomics
// changes a result.  Batches of one run take both steps in one launch.
#include <float.h>

#include "q8_device.h"
#include "q8_launch.h"
#include "q8_mx4_device.h"
#include "q8.h"

namespace q8 {

constexpr int kRouteBlocks = Q8_ROUTE_BLOCKS, kRouteThreads = 1024, kRouteWaves = kRouteThreads / 64, kRouteExperts = Q8_ROUTE_MAX_EXPERTS;

// Unsigned order of floats: -inf < ... < -0 < +0 < ... < +inf.  NaN counts as -inf.  +0 and -0 are the same logit.
__device__ __forceinline__ unsigned logit_key(float f)
{
    if (f != f) f = -__builtin_inff();
    const unsigned u = __float_as_uint(__fadd_rn(f, 0.0f));
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of_key(unsigned k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }

// The k experts of one token by a wave: lane l holds the logits l*kPer .. l*kPer + kPer - 1, so that the lowest lane of a tie holds
// the lowest index.  Every round takes the largest key left over (0 is below all of them).  Lane j returns choice j.
template <int kPer>
__device__ __forceinline__ void choose(const float* __restrict__ logits, int n_experts, int k, int& expert, float& gate)
{
    const int lane = threadIdx.x & 63;
    unsigned key[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = lane * kPer + i;
        key[i] = e < n_experts ? logit_key(logits[e]) : 0u;
    }
    unsigned chosen = 0;
    expert = 0;
    for (int j = 0; j < k; ++j) {
        unsigned best = key[0];
#pragma unroll
        for (int i = 1; i < kPer; ++i) best = max(best, key[i]);
        const unsigned top = wave_max_u32(best);
        const int owner = __builtin_ctzll(__ballot(best == top));
        int at = 0;
#pragma unroll
        for (int i = kPer - 1; i >= 0; --i) at = key[i] == top ? i : at;
        const int which = __builtin_amdgcn_readlane(at, owner);
        if (lane == owner) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) key[i] = i == which ? 0u : key[i];
        }
        if (lane == j) chosen = top, expert = owner * kPer + which;
    }
    // softmax over the chosen: against the largest, infinities taken as the largest finite number, nothing for -inf
    const float l = logit_of_key(chosen);
    const float finite = __builtin_fminf(__builtin_fmaxf(l, -FLT_MAX), FLT_MAX);
    const float most = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(finite), 0));
    const float p = lane < k && l != -__builtin_inff() ? expf(finite - most) : 0.0f;
    float sum = 0.0f;
    for (int j = 0; j < k; ++j) sum += __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(p), j));
    gate = sum > 0.0f ? __fdiv_rn(p, sum) : 0.0f;
}

// Tokens [t0, t1): experts and gates out, the pairs of each expert counted into hist (LDS, cleared).
template <int kPer>
__device__ __forceinline__ void choose_run(const float* __restrict__ logits, int64_t t0, int64_t t1, int n_experts, int k, int32_t* __restrict__ experts,
                                           float* __restrict__ gates, int* hist)
{
    const int lane = threadIdx.x & 63;
    for (int64_t t = t0 + (threadIdx.x >> 6); t < t1; t += kRouteWaves) {
        int e;
        float g;
        choose<kPer>(logits + t * n_experts, n_experts, k, e, g);
        if (lane < k) {
            experts[t * k + lane] = e;
            gates[t * k + lane] = g;
            atomicAdd(hist + e, 1);
        }
    }
}

// Places the pairs [i0, i1) of a run in order.  base[e] (LDS): the place of the run's first pair of expert e.  count: LDS for kRouteWaves x n_experts.
// Each wave takes a contiguous part, so that within an expert earlier waves come first.
__device__ __forceinline__ void place_run(const int32_t* __restrict__ experts, int64_t i0, int64_t i1, int n_experts, int k, const int* base, int* count,
                                          int32_t* __restrict__ rows, int32_t* __restrict__ slots)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t per = ((i1 - i0 + kRouteWaves - 1) / kRouteWaves + 63) / 64 * 64;  // whole steps of 64
    const int64_t w0 = min(i0 + wave * per, i1), w1 = min(w0 + per, i1);
    for (int e = threadIdx.x; e < kRouteWaves * n_experts; e += kRouteThreads) count[e] = 0;
    __syncthreads();
    for (int64_t i = w0 + lane; i < w1; i += 64) atomicAdd(count + wave * n_experts + experts[i], 1);
    __syncthreads();
    for (int e = threadIdx.x; e < n_experts; e += kRouteThreads) {
        int at = base[e];
        for (int w = 0; w < kRouteWaves; ++w) {
            const int n = count[w * n_experts + e];
            count[w * n_experts + e] = at;
            at += n;
        }
    }
    __syncthreads();
    int* next = count + wave * n_experts;
    for (int64_t c = w0; c < w1; c += 64) {
        const int64_t i = c + lane;
        const bool live = i < w1;
        const int e = live ? experts[i] : 0;
        unsigned long long same = __ballot(live);  // lanes with this lane's expert
        for (int b = 1; b < n_experts; b <<= 1) {
            const unsigned long long set = __ballot(live && (e & b));
            same &= (e & b) ? set : ~set;
        }
        const int rank = __builtin_popcountll(same & ((1ull << lane) - 1));
        if (live) {
            const int at = next[e] + rank;
            rows[at] = (int32_t)(i / k);
            slots[i] = at;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // all lanes have read before the first of each expert moves its place on
        __builtin_amdgcn_wave_barrier();
        if (live && rank == 0) next[e] += __builtin_popcountll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// base[e] += the sum of total[0 .. e), for up to kRouteThreads experts; scratch: LDS for kRouteWaves ints.
__device__ __forceinline__ void add_smaller_experts(int n_experts, const int* total, int* base, int* scratch)
{
    const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
    const int n = e < n_experts ? total[e] : 0;
    int upto = n;
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(upto, d);
        upto += lane >= d ? o : 0;
    }
    if (lane == 63) scratch[wave] = upto;
    __syncthreads();
    int before = upto - n;
    for (int w = 0; w < wave; ++w) before += scratch[w];
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
    for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) hist[e] = 0;
    __syncthreads();
    const int64_t t0 = blockIdx.x * a.run, t1 = min(t0 + a.run, a.T);
    choose_run<kPer>(a.logits, t0, t1, a.n_experts, a.k, a.experts, a.gates, hist);
    __syncthreads();
    for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) a.work[blockIdx.x * a.n_experts + e] = hist[e];
}

__global__ __launch_bounds__(kRouteThreads) void route_place_kernel(RouteArgs a)
{
    __shared__ int base[kRouteExperts], total[kRouteExperts], scratch[kRouteWaves];
    __shared__ int count[kRouteWaves * kRouteExperts];
    for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) base[e] = total[e] = 0;
    __syncthreads();
    // the counts of all runs, each thread those of one expert in some of the runs
    for (int i = threadIdx.x; i < a.runs * a.n_experts; i += kRouteThreads) {
        const int run = i / a.n_experts, e = i - run * a.n_experts, n = a.work[i];
        atomicAdd(total + e, n);
        if (run < (int)blockIdx.x) atomicAdd(base + e, n);
    }
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) a.group_rows[e] = total[e];
    add_smaller_experts(a.n_experts, total, base, scratch);
    const int64_t t0 = blockIdx.x * a.run, t1 = min(t0 + a.run, a.T);
    place_run(a.experts, t0 * a.k, t1 * a.k, a.n_experts, a.k, base, count, a.rows, a.slots);
}

// Both steps of a batch of one run.
template <int kPer>
__global__ __launch_bounds__(kRouteThreads) void route_single_kernel(RouteArgs a)
{
    __shared__ int hist[kRouteExperts], base[kRouteExperts], scratch[kRouteWaves];
    __shared__ int count[kRouteWaves * kRouteExperts];
    for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) hist[e] = base[e] = 0;
    __syncthreads();
    choose_run<kPer>(a.logits, 0, a.T, a.n_experts, a.k, a.experts, a.gates, hist);
    __threadfence_block();
    __syncthreads();
    for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) a.group_rows[e] = hist[e];
    add_smaller_experts(a.n_experts, hist, base, scratch);
    place_run(a.experts, 0, a.T * a.k, a.n_experts, a.k, base, count, a.rows, a.slots);
}

template <int kPer>
static int launch(RouteArgs a, hipStream_t st)
{
    if (a.runs == 1) {
        hipLaunchKernelGGL(route_single_kernel<kPer>, dim3(1), dim3(kRouteThreads), 0, st, a);
        return hipGetLastError() == hipSuccess ? 0 : 1;
    }
    hipLaunchKernelGGL(route_choose_kernel<kPer>, dim3((unsigned)a.runs), dim3(kRouteThreads), 0, st, a);
    if (hipGetLastError() != hipSuccess) return 1;
    hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)a.runs), dim3(kRouteThreads), 0, st, a);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

int launch_route(const float* logits, int64_t T, int n_experts, int k, int32_t* experts, float* gates, int32_t* group_rows, int32_t* rows, int32_t* slots,
                 int32_t* work, hipStream_t st)
{
    constexpr int64_t kLeast = 64;  // tokens of a run
    const int64_t most = (T + kRouteBlocks - 1) / kRouteBlocks, run = most > kLeast ? most : kLeast;
    const RouteArgs a{logits, T, run, n_experts, k, T ? (int)((T + run - 1) / run) : 1, experts, gates, group_rows, rows, slots, work};
    if (n_experts <= 64) return launch<1>(a, st);
    if (n_experts <= 128) return launch<2>(a, st);
    if (n_experts <= 256) return launch<4>(a, st);
    return launch<kRouteExperts / 64>(a, st);
}

// out[t,:] = sum over j, in order, of gates[t,j] y[slots[t,j],:], in fp32 with one rounding to the output type; a slot outside y adds
// nothing.  Bound by memory: k rows read, one written, 16 bytes a thread.
template <bool kBf16, bool kVec>
__global__ __launch_bounds__(256) void combine_kernel(const void* __restrict__ y, int64_t R, const int32_t* __restrict__ slots, const float* __restrict__ gates,
                                                      int64_t T, int k, int64_t N, int64_t per_row, void* __restrict__ out)
{
    constexpr int kElems = kVec ? (kBf16 ? 8 : 4) : 1;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= T * per_row) return;
    const int64_t t = i / per_row, n = (i - t * per_row) * kElems;
    float sum[kElems];
#pragma unroll
    for (int e = 0; e < kElems; ++e) sum[e] = 0.0f;
    for (int j = 0; j < k; ++j) {
        const int s = slots[t * k + j];
        if (s < 0 || s >= R) continue;
        const float g = gates[t * k + j];
        const int64_t at = (int64_t)s * N + n;
        if constexpr (kVec) {
            typedef unsigned v4u __attribute__((ext_vector_type(4)));
            const v4u v = *reinterpret_cast<const v4u*>(static_cast<const char*>(y) + at * (kBf16 ? 2 : 4));
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if constexpr (kBf16) {
                    sum[2 * w] = __builtin_fmaf(g, __uint_as_float(v[w] << 16), sum[2 * w]);
                    sum[2 * w + 1] = __builtin_fmaf(g, __uint_as_float(v[w] & 0xffff0000u), sum[2 * w + 1]);
                } else {
                    sum[w] = __builtin_fmaf(g, __uint_as_float(v[w]), sum[w]);
                }
            }
        } else if constexpr (kBf16) {
            sum[0] = __builtin_fmaf(g, bf16_to_f32(static_cast<const unsigned short*>(y)[at]), sum[0]);
        } else {
            sum[0] = __builtin_fmaf(g, static_cast<const float*>(y)[at], sum[0]);
        }
    }
#pragma unroll
    for (int e = 0; e < kElems; ++e) {
        if constexpr (kBf16)
            static_cast<unsigned short*>(out)[t * N + n + e] = f32_to_bf16(sum[e]);
        else
            static_cast<float*>(out)[t * N + n + e] = sum[e];
    }
}

int launch_combine(const void* y, int64_t R, const int32_t* slots, const float* gates, int64_t T, int k, int64_t N, void* out, bool bf16, hipStream_t st)
{
    const int64_t elems = bf16 ? 8 : 4;
    const bool vec = N % elems == 0 && (reinterpret_cast<uintptr_t>(y) | reinterpret_cast<uintptr_t>(out)) % 16 == 0;
    const int64_t per_row = vec ? N / elems : N, blocks = (T * per_row + 255) / 256;
    if (blocks >= (int64_t)1 << 24) return 1;  // a launch is limited to 2^32 threads
    const dim3 grid((unsigned)blocks), block(256);
#define Q8_COMBINE(B, V) hipLaunchKernelGGL((combine_kernel<B, V>), grid, block, 0, st, y, R, slots, gates, T, k, N, per_row, out)
    if (bf16 && vec)
        Q8_COMBINE(true, true);
    else if (bf16)
        Q8_COMBINE(true, false);
    else if (vec)
        Q8_COMBINE(false, true);
    else
        Q8_COMBINE(false, false);
#undef Q8_COMBINE
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

}  // namespace q8
