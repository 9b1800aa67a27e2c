// graft_logits_adjust: a request's rules on the logits of its tree's nodes, and the greedy token that they leave.
//
// One pass over the logits.  A row is cut into chunks of 16-byte groups as the scans of the logits in graft_accept are; a workgroup
// requests its whole chunk, with the counts, biases and mask words of the same tokens, before it looks at any of it.  Counts are kept
// per sequence; what a node's path adds to them is a handful of tokens, which each thread compares with its own.  The
// chunks' maxima are folded by a second kernel.
#include "common.h"

namespace graft {

constexpr int LA_THREADS = 512;
constexpr int LA_QUADS = 4;                      // 16-byte loads of logits in flight per thread
constexpr int LA_WAVES = LA_THREADS / 64;
constexpr int LA_MAX_CHUNKS = 64;                // one lane each in the fold
typedef int32_t int4u __attribute__((ext_vector_type(4), aligned(4)));      // groups that need not be aligned
typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));

struct AdjustParams {
    const float* logits;
    const int32_t* n_nodes;
    const int32_t* tokens;
    const u64* mask;
    const int32_t* counts;
    const float *repetition, *frequency, *presence, *bias;
    const uint32_t* allow;
    const int32_t* allow_index;
    float* out;
    int32_t* target_ids;
    int32_t* status;
    u64* partial;            // [rows][chunks] keys
    int64_t bias_stride;     // 0: one row of biases for all sequences
    int32_t K_max, V, W, n_allow, chunks, per;
};

// Larger numbers have larger keys, of equal numbers the one of the smaller index; 0 is below every number above -inf.
__device__ __forceinline__ u64 key_of(float v, int32_t i) {
    if (!(v > -INFINITY)) return 0;
    const uint32_t bits = __float_as_uint(v + 0.0f);               // -0 is +0
    const uint32_t up = bits ^ (static_cast<uint32_t>(static_cast<int32_t>(bits) >> 31) | 0x80000000u);
    return (static_cast<u64>(up) << 32) | ~static_cast<uint32_t>(i);
}
__device__ __forceinline__ int32_t id_of(u64 key) { return key ? static_cast<int32_t>(~static_cast<uint32_t>(key)) : -1; }

struct Rules { float repetition, frequency, presence; };
// A logit under the rules; each operation rounded to fp32 by itself.
__device__ __forceinline__ float adjusted(float x, int32_t count, int32_t on_path, const Rules& r) {
#pragma clang fp contract(off)
    const uint32_t later = static_cast<uint32_t>(count & INT32_MAX) + static_cast<uint32_t>(on_path);
    if (later > 0 || count < 0) x = x > 0.f ? x / r.repetition : x * r.repetition;
    if (later > 0) {
        const float f = static_cast<float>(later) * r.frequency;
        x = x - f;
        x = x - r.presence;
    }
    return x;
}

template <bool PENALTIES, bool ONCE>
__global__ __launch_bounds__(LA_THREADS) void logits_adjust_kernel(const int32_t* __restrict__ n_nodes, AdjustParams p) {
#pragma clang fp contract(off)
    __shared__ int32_t path[GRAFT_MAX_NODES];    // tokens of the row's path that lie in this chunk
    __shared__ int32_t n_path[2];
    __shared__ u64 best_of[LA_WAVES];
    __shared__ int32_t faults;
    const int chunk = blockIdx.x, i = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t n = n_nodes[b];
    const bool n_ok = n >= 1 && n <= p.K_max;
    const size_t row = static_cast<size_t>(b) * p.K_max + i;
    if (chunk == 0 && i == 0) {
        if (tid == 0) faults = n_ok ? 0 : GRAFT_STATUS_BAD_TREE;
        __syncthreads();
        if (p.allow && n_ok && tid < n) {
            const int32_t at = p.allow_index[row + tid];
            if (at < -1 || at >= p.n_allow) atomicOr(&faults, GRAFT_STATUS_BAD_LENGTH);
        }
        __syncthreads();
        if (tid == 0) p.status[b] = faults;
    }
    if (!n_ok || i >= n) {
        if (tid == 0 && p.partial) p.partial[row * p.chunks + chunk] = 0;
        return;
    }
    const float* logits = p.logits + row * p.V;
    const RowChunk c = row_chunk(logits, p.V, chunk, p.chunks, p.per);
    // what this chunk covers: groups q0 .. q1 and, in the first and the last one, the row's edges
    const int32_t first = chunk == 0 ? 0 : c.head + 4 * c.q0, behind = chunk == p.chunks - 1 ? p.V : c.head + 4 * c.q1;
    Rules rules{1.f, 0.f, 0.f};
    int32_t on_path = 0;
    const int32_t* counts = nullptr;
    if constexpr (PENALTIES) {
        if (p.repetition) rules.repetition = p.repetition[b];
        if (p.frequency) rules.frequency = p.frequency[b];
        if (p.presence) rules.presence = p.presence[b];
        counts = p.counts ? p.counts + static_cast<size_t>(b) * p.V : nullptr;
        if (p.mask) {                            // (uniform)
            bool mine = false;
            int32_t tok = -1;
            if (tid < GRAFT_MAX_NODES && tid > 0 && tid < n) {
                tok = p.tokens[static_cast<size_t>(b) * p.K_max + tid];
                mine = ((p.mask[row * GRAFT_MASK_WORDS + (tid >> 6)] >> (tid & 63)) & 1) && tok >= first && tok < behind;
            }
            const u64 vote = __builtin_amdgcn_ballot_w64(mine);
            if (wave < 2 && lane == 0) n_path[wave] = __popcll(vote);
            __syncthreads();
            const int32_t below = wave == 1 ? n_path[0] : 0;
            if (mine) path[below + __popcll(vote & ((1ull << lane) - 1))] = tok;
            on_path = n_path[0] + n_path[1];
            __syncthreads();
        }
    }
    const float* bias = p.bias ? p.bias + static_cast<size_t>(b) * p.bias_stride : nullptr;
    const uint32_t* allow = nullptr;
    bool nothing = false;
    if (p.allow) {
        const int32_t at = p.allow_index[row];
        nothing = at < -1 || at >= p.n_allow;
        allow = at == -1 || nothing ? nullptr : p.allow + static_cast<size_t>(at) * p.W;
    }
    float* out = p.out ? p.out + row * p.V : nullptr;
    auto times = [&](int32_t e) __attribute__((always_inline)) {
        int32_t k = 0;
        for (int32_t j = 0; j < on_path; ++j) k += path[j] == e ? 1 : 0;
        return k;
    };
    u64 edge_key = 0;
    if (tid < c.edge) {                          // at most three elements in front of the groups and three behind
        const int32_t e = c.edge_at(tid);
        float x = logits[e];
        if constexpr (PENALTIES) x = adjusted(x, counts ? counts[e] : 0, times(e), rules);
        if (bias) x = x + bias[e];
        if (nothing || (allow && !((allow[e >> 5] >> (e & 31)) & 1))) x = -INFINITY;
        if (out) out[e] = x;
        edge_key = key_of(x, e);
    }
    float bv = -INFINITY;                        // of this thread's groups, whose indices rise
    int32_t bi = 0;
    for (int32_t s0 = c.q0; s0 < c.q1; s0 += LA_QUADS * LA_THREADS) {
        float4 x[LA_QUADS];
        int4u n_of[LA_QUADS];
        float4u add[LA_QUADS];
        uint32_t may[LA_QUADS];
#pragma unroll
        for (int u = 0; u < LA_QUADS; ++u) {
            const int32_t q = s0 + tid + u * LA_THREADS, e = c.head + 4 * q;
            const bool there = q < c.q1;
            x[u] = there ? load_logits<ONCE>(c.quad + q) : float4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            n_of[u] = int4u{0, 0, 0, 0};
            add[u] = float4u{0.f, 0.f, 0.f, 0.f};
            may[u] = nothing ? 0u : 15u;
            if (there) {
                if constexpr (PENALTIES) if (counts) n_of[u] = *reinterpret_cast<const int4u*>(counts + e);
                if (bias) add[u] = *reinterpret_cast<const float4u*>(bias + e);
                if (allow) {
                    uint32_t w = allow[e >> 5] >> (e & 31);
                    if ((e & 31) > 28) w |= allow[(e >> 5) + 1] << (32 - (e & 31));
                    may[u] = w;
                }
            }
        }
        u64 hit = 0;                             // this thread's elements that are tokens of the path
        for (int32_t j = 0; j < on_path; ++j) {
            const int32_t d = path[j] - (c.head + 4 * s0);
            if (d >= 0 && ((d >> 2) & (LA_THREADS - 1)) == tid && (d >> 2) < LA_QUADS * LA_THREADS)
                hit |= 1ull << (4 * ((d >> 2) / LA_THREADS) + (d & 3));
        }
#pragma unroll
        for (int u = 0; u < LA_QUADS; ++u) {
            const int32_t q = s0 + tid + u * LA_THREADS, e = c.head + 4 * q;
            float y[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (PENALTIES) y[k] = adjusted(y[k], n_of[u][k], (hit >> (4 * u + k)) & 1 ? times(e + k) : 0, rules);
                if (bias) y[k] = y[k] + add[u][k];
                y[k] = (may[u] >> k) & 1 ? y[k] : -INFINITY;
            }
            if (q < c.q1) {
                if (out) *reinterpret_cast<float4u*>(out + e) = float4u{y[0], y[1], y[2], y[3]};
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (y[k] > bv) { bv = y[k]; bi = e + k; }
            }
        }
    }
    if (!p.target_ids) return;
    const u64 groups_key = key_of(bv, bi), key = wave_max_u64(groups_key > edge_key ? groups_key : edge_key);
    if (lane == 0) best_of[wave] = key;
    __syncthreads();
    if (tid == 0) {
        u64 best = best_of[0];
#pragma unroll
        for (int w = 1; w < LA_WAVES; ++w) best = best_of[w] > best ? best_of[w] : best;
        p.partial[row * p.chunks + chunk] = best;
    }
}

// One wavefront a row: the best of its chunks.
__global__ __launch_bounds__(256) void adjust_fold_kernel(const u64* __restrict__ partial, int32_t chunks, int32_t rows, int32_t* __restrict__ target_ids) {
    const int32_t row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (row >= rows) return;
    const u64 best = wave_max_u64(lane < chunks ? partial[static_cast<size_t>(row) * chunks + lane] : 0);
    if (lane == 0) target_ids[row] = id_of(best);
}

struct AdjustCut { int32_t chunks, per; };
static AdjustCut adjust_cut(int64_t rows, int32_t V) {
    const int32_t quads = V / 4, whole = LA_QUADS * LA_THREADS;
    int64_t chunks = (quads + whole - 1) / whole;
    const int64_t fill = (ROW_FILL + rows - 1) / rows, most = (quads + 127) / 128;
    if (chunks < fill) chunks = fill < most ? fill : most;
    if (chunks > LA_MAX_CHUNKS) chunks = LA_MAX_CHUNKS;
    if (chunks < 1) chunks = 1;
    return {static_cast<int32_t>(chunks), static_cast<int32_t>((quads + chunks - 1) / chunks)};
}

}  // namespace graft

extern "C" size_t graft_logits_adjust_workspace_bytes(int32_t B, int32_t K_max, int32_t V) {
    if (B < 1 || K_max < 1 || V < 1) return 0;
    const int64_t rows = static_cast<int64_t>(B) * K_max;
    return static_cast<size_t>(rows) * graft::adjust_cut(rows, V).chunks * sizeof(graft::u64);
}

extern "C" int32_t graft_logits_adjust(const float* logits, const int32_t* n_nodes, const int32_t* tokens, const uint64_t* mask, int32_t B,
                                       int32_t K_max, int32_t V, const int32_t* counts, const float* repetition, const float* frequency,
                                       const float* presence, const float* bias, int32_t bias_rows, const uint32_t* allow, int32_t n_allow,
                                       const int32_t* allow_index, float* out, int32_t* target_ids, int32_t* status, void* workspace,
                                       size_t workspace_bytes, void* stream) {
    using namespace graft;
    if (!logits || !n_nodes || !status || (!out && !target_ids) || (!tokens) != (!mask) || (!allow) != (!allow_index)) return GRAFT_ERR_NULL;
    if (B < 1 || B > 65535 || K_max < 1 || K_max > GRAFT_MAX_NODES || V < 1 || (bias && bias_rows != 1 && bias_rows != B) || (allow && n_allow < 1))
        return GRAFT_ERR_SHAPE;
    const int64_t rows = static_cast<int64_t>(B) * K_max;
    if (out && out != logits) {
        const size_t a = reinterpret_cast<size_t>(out), l = reinterpret_cast<size_t>(logits), size = static_cast<size_t>(rows) * V * sizeof(float);
        if (a < l + size && l < a + size) return GRAFT_ERR_SHAPE;
    }
    if (target_ids && (!workspace || workspace_bytes < graft_logits_adjust_workspace_bytes(B, K_max, V))) return GRAFT_ERR_WORKSPACE;
    if (reinterpret_cast<size_t>(workspace) & 7) return GRAFT_ERR_WORKSPACE;
    const AdjustCut cut = adjust_cut(rows, V);
    const AdjustParams p{logits, n_nodes, tokens, reinterpret_cast<const u64*>(mask), counts, repetition, frequency, presence, bias, allow, allow_index,
                         out, target_ids, status, target_ids ? static_cast<u64*>(workspace) : nullptr, bias && bias_rows > 1 ? static_cast<int64_t>(V) : 0,
                         K_max, V, (V - 1) / 32 + 1, n_allow, cut.chunks, cut.per};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid(cut.chunks, K_max, B);
    const bool penalties = repetition || frequency || presence, once = read_once(rows, V);
    if (penalties) hipLaunchKernelGGL((once ? logits_adjust_kernel<true, true> : logits_adjust_kernel<true, false>), grid, dim3(LA_THREADS), 0, s, n_nodes, p);
    else hipLaunchKernelGGL((once ? logits_adjust_kernel<false, true> : logits_adjust_kernel<false, false>), grid, dim3(LA_THREADS), 0, s, n_nodes, p);
    int32_t rc = check_launch();
    if (rc != GRAFT_OK || !target_ids) return rc;
    hipLaunchKernelGGL(adjust_fold_kernel, dim3(static_cast<uint32_t>((rows + 3) / 4)), dim3(256), 0, s, p.partial, cut.chunks, static_cast<int32_t>(rows),
                       target_ids);
    return check_launch();
}
