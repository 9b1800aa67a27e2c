// graft_token_counts: how often each token of the vocabulary occurs in a sequence, the numbers that penalties go by.
//
// Whole rows are counted in LDS: a workgroup has a slice of a sequence's vocabulary, reads the whole context and counts what
// falls into its slice, so that a row needs no clearing pass, no atomics in memory and one launch.  Additions to rows that
// are there (a round's few tokens) are atomics in memory: sums and ORs of whole numbers, whose order does not show.
// Bound by two trips to memory and, for long contexts, by the pass over them: 16 contexts of up to 16K, 151936 tokens, 6.4 us in a graph, one context
// of a small vocabulary 3.5.  Slices of 4096: 6.9 and 3.4, of 16384 with 1024 threads 6.2 and 3.9 (a context of 300, 32 sequences: 7.1, 6.8 against 6.3).
#include "common.h"

namespace graft {

constexpr int TC_THREADS = 512;
constexpr int TC_AHEAD = 8;                      // 16-byte loads of the context in flight per thread
constexpr int TC_SLICE = 8192;                   // counters of a workgroup, 32 KB of LDS
constexpr int32_t TC_PROMPT = INT32_MIN;         // the bit of tokens that the prompt holds
typedef int32_t int4u __attribute__((ext_vector_type(4), aligned(4)));

struct ContextRange { int32_t from, to; bool ok; };
__device__ __forceinline__ ContextRange context_range(const int32_t* len, const int32_t* start, int b, int32_t L_max) {
    const int32_t n = len[b], s = start ? start[b] : 0;
    return {s, n, n >= 0 && n <= L_max && s >= 0 && s <= n};
}

__global__ __launch_bounds__(TC_THREADS) void token_counts_kernel(const int32_t* __restrict__ ctx, const int32_t* __restrict__ ctx_len,
                                                                  const int32_t* __restrict__ prompt_len, int32_t L_max, int32_t V, int32_t per,
                                                                  int32_t* __restrict__ counts, int32_t* __restrict__ status) {
    __shared__ __attribute__((aligned(16))) int32_t n_of[TC_SLICE];
    const int b = blockIdx.y, tid = threadIdx.x;
    const ContextRange r = context_range(ctx_len, nullptr, b, L_max);
    const int32_t prompt = prompt_len ? prompt_len[b] : 0, to = r.ok ? r.to : 0;
    const int32_t v0 = blockIdx.x * per, rest = V - v0, size = rest < 0 ? 0 : rest < per ? rest : per;
    const int32_t* row = ctx + static_cast<size_t>(b) * L_max;
    for (int32_t v = 4 * tid; v < size; v += 4 * TC_THREADS) *reinterpret_cast<int4*>(n_of + v) = int4{0, 0, 0, 0};
    __syncthreads();
    auto take = [&](int32_t tok, int32_t t) __attribute__((always_inline)) {
        const uint32_t at = static_cast<uint32_t>(tok) - static_cast<uint32_t>(v0);
        if (at >= static_cast<uint32_t>(size)) return;            // (tokens outside [0,V) are in no slice)
        if (t < prompt) atomicOr(&n_of[at], TC_PROMPT);
        else atomicAdd(&n_of[at], 1);
    };
    const int32_t quads = to / 4;
    for (int32_t q0 = tid; q0 < quads; q0 += TC_AHEAD * TC_THREADS) {
        int4u x[TC_AHEAD];
#pragma unroll
        for (int u = 0; u < TC_AHEAD; ++u) {
            const int32_t q = q0 + u * TC_THREADS;
            x[u] = q < quads ? *reinterpret_cast<const int4u*>(row + 4 * static_cast<size_t>(q)) : int4u{-1, -1, -1, -1};
        }
#pragma unroll
        for (int u = 0; u < TC_AHEAD; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) take(x[u][k], 4 * (q0 + u * TC_THREADS) + k);
    }
    if (tid < to - 4 * quads) take(row[4 * quads + tid], 4 * quads + tid);
    __syncthreads();
    int32_t* out = counts + static_cast<size_t>(b) * V + v0;
    const int32_t full = size & ~3;
    for (int32_t v = 4 * tid; v < full; v += 4 * TC_THREADS) {
        const int4 x = *reinterpret_cast<const int4*>(n_of + v);
        *reinterpret_cast<int4u*>(out + v) = int4u{x.x, x.y, x.z, x.w};
    }
    if (tid < size - full) out[full + tid] = n_of[full + tid];
    if (blockIdx.x == 0 && tid == 0) status[b] = r.ok ? 0 : GRAFT_STATUS_BAD_LENGTH;
}

__global__ __launch_bounds__(TC_THREADS) void token_counts_add_kernel(const int32_t* __restrict__ ctx, const int32_t* __restrict__ ctx_len,
                                                                      const int32_t* __restrict__ prompt_len, const int32_t* __restrict__ start,
                                                                      int32_t L_max, int32_t V, int32_t* __restrict__ counts,
                                                                      int32_t* __restrict__ status) {
    const int b = blockIdx.y;
    const ContextRange r = context_range(ctx_len, start, b, L_max);
    const int32_t prompt = prompt_len ? prompt_len[b] : 0;
    const int32_t* row = ctx + static_cast<size_t>(b) * L_max;
    int32_t* out = counts + static_cast<size_t>(b) * V;
    if (r.ok)
        for (int64_t t = static_cast<int64_t>(r.from) + blockIdx.x * TC_THREADS + threadIdx.x; t < r.to; t += gridDim.x * TC_THREADS) {
            const int32_t tok = row[t];
            if (static_cast<uint32_t>(tok) >= static_cast<uint32_t>(V)) continue;
            if (t < prompt) atomicOr(out + tok, TC_PROMPT);
            else atomicAdd(out + tok, 1);
        }
    if (blockIdx.x == 0 && threadIdx.x == 0) status[b] = r.ok ? 0 : GRAFT_STATUS_BAD_LENGTH;
}

}  // namespace graft

extern "C" int32_t graft_token_counts(const int32_t* ctx, const int32_t* ctx_len, const int32_t* prompt_len, const int32_t* start, int32_t B,
                                      int32_t L_max, int32_t V, int32_t* counts, int32_t* status, void* stream) {
    using namespace graft;
    if (!ctx || !ctx_len || !counts || !status) return GRAFT_ERR_NULL;
    if (B < 1 || B > 65535 || L_max < 1 || L_max >= (1 << 30) || V < 1 || V >= (1 << 30)) return GRAFT_ERR_SHAPE;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (start) {
        const int32_t groups = (L_max + TC_THREADS - 1) / TC_THREADS;
        hipLaunchKernelGGL(token_counts_add_kernel, dim3(groups < 16 ? groups : 16, B), dim3(TC_THREADS), 0, s, ctx, ctx_len, prompt_len, start, L_max, V,
                           counts, status);
    } else {
        const int32_t slices = (V - 1) / TC_SLICE + 1, per = ((V - 1) / slices + 4) & ~3;          // (whole groups of four; the last slice is smaller)
        hipLaunchKernelGGL(token_counts_kernel, dim3(slices, B), dim3(TC_THREADS), 0, s, ctx, ctx_len, prompt_len, L_max, V, per, counts, status);
    }
    return check_launch();
}
