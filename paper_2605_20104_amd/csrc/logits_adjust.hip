// graft_logits_adjust: a request's rules on the logits of its tree's nodes, and the greedy token that they leave.
//
// One pass over the logits.  Counts and biases belong to a sequence, not to a node: a workgroup takes a block of the vocabulary's columns
// for several of a sequence's rows, makes of counts and biases what every row needs of them (which tokens have been seen, what to
// subtract, what to add) and keeps that in LDS, each thread its own columns, while the rows pass, the next one's logits on their way.  What a node's path adds
// to its history is a handful of tokens, found by comparing and done over for the threads that have them.  Columns are the same for
// all rows, whatever a row's address: loads of 16 bytes need not be aligned.
//
#include <type_traits>

#include "common.h"

namespace graft {

constexpr int LA_THREADS = 256, LA_QUADS = 2;    // 2048 columns a block
// Rows of a workgroup: as many as leave LA_FILL workgroups, up to LA_ROWS.  Its columns' set-up (a trip to memory, two barriers) is worth
// several rows: us a call in a graph, everything on, 8 x 48 rows of 151936 written with up to 1, 2, 4, 8 and 16 rows: 111, 90.2, 88.7, 87.7, 91.9;
// ids only: 94.4, 77.3, 68.2, 67.4, 72.6.  Smaller calls have fewer by the rule; ids only, with LA_FILL 2048 (one row), 1024 (two), 512 (four) and
// 256 (eight): 3 x up to 40 rows of 50257 12.4, 12.1, 14.8, 21.3; 64 rows of 128256 18.0, 16.2, 17.2, 20.1.  LA_QUADS 1 and 4: the first
// call 92.2 and 92.6, the 3 x 40 rows 13.4 and 14.6.
constexpr int LA_ROWS = 8;
constexpr int64_t LA_FILL = 1024;
typedef int32_t int4u __attribute__((ext_vector_type(4), aligned(4)));      // groups of four columns
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
    u64* partial;            // [rows][blocks * wavefronts] keys
    int64_t bias_stride;     // 0: one row of biases for all sequences
    int32_t K_max, V, W, n_allow, rows_per;
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
// A logit under the penalties; each operation rounded to fp32 by itself.
__device__ __forceinline__ float penalised(float x, int32_t count, int32_t on_path, const Rules& r) {
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
// x / d for d from 2^-20 to 2^20 and x from 2^-90 to 2^100, y = 1 / d: a quotient within a step of the exact one, corrected by its
// remainder, is the rounded quotient (P. Markstein, IBM Journal of Research and Development 34, 1990); the product x y may be two
// steps off, and is corrected twice.  Five instructions for twelve; 4e8 quotients compared with a division's, on the host.
__device__ __forceinline__ float quotient(float x, float d, float y) {
    float q = x * y;
    q = __builtin_fmaf(__builtin_fmaf(-q, d, x), y, q);
    return __builtin_fmaf(__builtin_fmaf(-q, d, x), y, q);
}

// A value that is computed whether or not a later choice takes it: choices between sums become selects, not branches.
__device__ __forceinline__ float apart(float x) {
    asm volatile("" : "+v"(x));
    return x;
}

// THREADS x QUADS groups of four columns a block.  WHOLE: a workgroup goes over all blocks of one row; otherwise over rows_per rows of one.
template <bool PENALTIES, bool ONCE, int QUADS>
__global__ __launch_bounds__(LA_THREADS) void logits_adjust_kernel(const int32_t* __restrict__ n_nodes, AdjustParams p) {
#pragma clang fp contract(off)
    constexpr int THREADS = LA_THREADS, WAVES = THREADS / 64;
    __shared__ int32_t near_token[GRAFT_MAX_NODES], near_node[GRAFT_MAX_NODES];     // nodes below the root whose tokens lie in this block
    __shared__ float4 columns[3 * QUADS * THREADS];                                // what to subtract, to add, and the counts
    __shared__ int32_t n_near[2];
    __shared__ int32_t faults;
    const int b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int i0 = blockIdx.y * p.rows_per, block = blockIdx.x;
    const int32_t n = n_nodes[b];
    const bool n_ok = n >= 1 && n <= p.K_max;
    const size_t row0 = static_cast<size_t>(b) * p.K_max;
    if (blockIdx.x == 0 && blockIdx.y == 0) {
        if (tid == 0) faults = n_ok ? 0 : GRAFT_STATUS_BAD_TREE;
        __syncthreads();
        if (p.allow && n_ok && tid < n) {
            const int32_t at = p.allow_index[row0 + tid];
            if (at < -1 || at >= p.n_allow) atomicOr(&faults, GRAFT_STATUS_BAD_LENGTH);
        }
        __syncthreads();
        if (tid == 0) p.status[b] = faults;
    }
    const int i_end = i0 + p.rows_per < p.K_max ? i0 + p.rows_per : p.K_max, i1 = n_ok ? (n < i_end ? n : i_end) : i0;
    // rows that are not there
    if (p.target_ids)
        for (int i = (i1 > i0 ? i1 : i0) + wave; i < i_end; i += WAVES) {
            if (lane < WAVES) p.partial[((row0 + i) * gridDim.x + block) * WAVES + lane] = 0;
        }
    if (i1 <= i0) return;
    Rules rules{1.f, 0.f, 0.f};
    const int32_t* counts = nullptr;
    float inverse = 1.f;
    bool divide = false;                         // repetitions that quotient() does not take
    if constexpr (PENALTIES) {
        if (p.repetition) rules.repetition = p.repetition[b];
        if (p.frequency) rules.frequency = p.frequency[b];
        if (p.presence) rules.presence = p.presence[b];
        counts = p.counts ? p.counts + static_cast<size_t>(b) * p.V : nullptr;
        inverse = 1.f / rules.repetition;
        divide = !(rules.repetition >= 0x1p-20f && rules.repetition <= 0x1p20f);
    }
    const float* bias = p.bias ? p.bias + static_cast<size_t>(b) * p.bias_stride : nullptr;
    int32_t token = -1;                          // thread j: the token of node j below the root
    if (PENALTIES && p.mask && tid > 0 && tid < n) token = p.tokens[row0 + tid];
    // lane j: the grammar's state and the path of row i0 + j (one trip to memory for all rows)
    int32_t state_of = -1;
    u64 path_of[2] = {0, 0};
    if (lane < i1 - i0) {
        if (p.allow) state_of = p.allow_index[row0 + i0 + lane];
        if (PENALTIES && p.mask) {
            path_of[0] = p.mask[(row0 + i0 + lane) * GRAFT_MASK_WORDS];
            path_of[1] = p.mask[(row0 + i0 + lane) * GRAFT_MASK_WORDS + 1];
        }
    }
    auto path_word = [&](int i, int h) __attribute__((always_inline)) {
        const int lo = __builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(path_of[h])), i - i0);
        const int hi = __builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(path_of[h] >> 32)), i - i0);
        return (static_cast<u64>(static_cast<uint32_t>(hi)) << 32) | static_cast<uint32_t>(lo);
    };
    {
        const int32_t first = block * (4 * THREADS * QUADS), e0 = first + 4 * tid;            // group u of the thread: e0 + 4 THREADS u
        const int32_t full = p.V & ~3;           // columns behind it are the last group's, one by one
        int32_t near = 0, tok_of[2] = {-1, -1}, node_of[2] = {0, 0};
        auto find_near = [&]() __attribute__((always_inline)) {
            bool mine = token >= first && token < p.V && token - first < 4 * THREADS * QUADS;
            const u64 vote = __builtin_amdgcn_ballot_w64(mine);
            if (wave < 2 && lane == 0) n_near[wave] = __popcll(vote);
            __syncthreads();
            if (mine) {
                const int at = (wave == 1 ? n_near[0] : 0) + __popcll(vote & ((1ull << lane) - 1));
                near_token[at] = token;
                near_node[at] = tid;
            }
            __syncthreads();
            near = n_near[0] + n_near[1];
            // lane j has the j-th and the 64 + j-th
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool there = lane + 64 * h < near;
                tok_of[h] = there ? near_token[lane + 64 * h] : -1;
                node_of[h] = there ? near_node[lane + 64 * h] : 0;
            }
        };
        auto pass = [&](auto inside_) __attribute__((always_inline)) {       // INSIDE: all of the block's columns are whole groups
        constexpr bool INSIDE = decltype(inside_)::value;
        auto load4 = [&](const float* from, int32_t e, float fill, auto once_) __attribute__((always_inline)) {
            float4u x = {fill, fill, fill, fill};
            if (INSIDE || e < full) {
                if constexpr (decltype(once_)::value) x = __builtin_nontemporal_load(reinterpret_cast<const float4u*>(from + e));
                else x = *reinterpret_cast<const float4u*>(from + e);
            } else if (e < p.V) {
                x[0] = from[e];
                if (e + 1 < p.V) x[1] = from[e + 1];
                if (e + 2 < p.V) x[2] = from[e + 2];
            }
            return x;
        };
        const int32_t w_last = p.W - 1;
        struct Row { float4u x[QUADS]; uint32_t may[QUADS]; };
        auto load_row = [&](int i) __attribute__((always_inline)) {
            Row r;
            const float* logits = p.logits + (row0 + i) * p.V;
#pragma unroll
            for (int u = 0; u < QUADS; ++u) r.x[u] = load4(logits, e0 + 4 * THREADS * u, -INFINITY, std::bool_constant<ONCE>{});
            if (p.allow) {                       // (words as they are: what is done to them now would be waited for)
                const int32_t at = __builtin_amdgcn_readlane(state_of, i - i0);
                const uint32_t* allow = p.allow + static_cast<size_t>(at < 0 || at >= p.n_allow ? 0 : at) * p.W;
#pragma unroll
                for (int u = 0; u < QUADS; ++u) {
                    const int32_t w = (e0 + 4 * THREADS * u) >> 5;
                    r.may[u] = allow[INSIDE || w < w_last ? w : w_last];
                }
            }
            return r;
        };
        Row next = load_row(i0);
        // ---- what the block's columns are to every row: lane masks in scalar registers, what to subtract and to add in LDS (each
        //      thread's own columns, which nobody else reads)
        bool seen[QUADS][4], later[QUADS][4];
        float4* const mine4 = columns + tid;
        int4u c[QUADS];
        float4u add[QUADS];
#pragma unroll
        for (int u = 0; u < QUADS; ++u) {
            const int32_t e = e0 + 4 * THREADS * u;
            c[u] = int4u{0, 0, 0, 0};
            if (PENALTIES && counts) {
                if (INSIDE || e < full) c[u] = *reinterpret_cast<const int4u*>(counts + e);
                else if (e < p.V) {
                    c[u][0] = counts[e];
                    if (e + 1 < p.V) c[u][1] = counts[e + 1];
                    if (e + 2 < p.V) c[u][2] = counts[e + 2];
                }
            }
            if (bias) add[u] = load4(bias, e, 0.f, std::false_type{});
        }
        if constexpr (PENALTIES) if (p.mask) find_near();         // (uniform)
#pragma unroll
        for (int u = 0; u < QUADS; ++u) {
            if constexpr (PENALTIES) {
                float minus[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int32_t gen = c[u][k] & INT32_MAX;
                    seen[u][k] = c[u][k] != 0;
                    later[u][k] = gen != 0;
                    minus[k] = gen != 0 ? static_cast<float>(gen) * rules.frequency : 0.f;
                }
                mine4[3 * u * THREADS] = float4{minus[0], minus[1], minus[2], minus[3]};
                *reinterpret_cast<int4*>(mine4 + (3 * u + 2) * THREADS) = int4{c[u][0], c[u][1], c[u][2], c[u][3]};
            }
            if (bias) mine4[(3 * u + 1) * THREADS] = float4{add[u][0], add[u][1], add[u][2], add[u][3]};
        }
        for (int i = i0; i < i1; ++i) {
            const Row r = next;
            if (i + 1 < i1) next = load_row(i + 1);
            uint32_t hit = 0;                    // columns of this thread that are tokens of the row's path
            u64 on_path[2] = {0, 0};             // which of the lanes' tokens are
            if constexpr (PENALTIES) if (near > 0) {                                          // (uniform)
                const u64 m[2] = {path_word(i, 0), path_word(i, 1)};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    on_path[h] = __builtin_amdgcn_ballot_w64(tok_of[h] >= 0 && (((node_of[h] < 64 ? m[0] : m[1]) >> (node_of[h] & 63)) & 1));
                    for (u64 left = on_path[h]; left != 0; left &= left - 1) {
                        const int d = __builtin_amdgcn_readlane(tok_of[h], __builtin_ctzll(left)) - first, g = d >> 2;
                        if ((g & (THREADS - 1)) == tid) hit |= 1u << (4 * (g / THREADS) + (d & 3));
                    }
                }
            }
            float y[QUADS][4], least = 1.f, most = 1.f;       // of the numbers that are divided
#pragma unroll
            for (int u = 0; u < QUADS; ++u) {
                float4 minus = {0.f, 0.f, 0.f, 0.f};
                if constexpr (PENALTIES) minus = mine4[3 * u * THREADS];
                const float m4[4] = {minus.x, minus.y, minus.z, minus.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float x = r.x[u][k];
                    if constexpr (PENALTIES) {
                        const bool up = x > 0.f;
                        const float divided = (up & seen[u][k]) ? x : 1.f, less = apart(quotient(x, rules.repetition, inverse)), more = apart(x * rules.repetition);
                        least = __builtin_fminf(least, divided);
                        most = __builtin_fmaxf(most, divided);
                        const float scaled = up ? less : more;
                        x = seen[u][k] ? scaled : x;
                        x = x - m4[k];
                        const float present = apart(x - rules.presence);
                        x = later[u][k] ? present : x;
                    }
                    y[u][k] = x;
                }
            }
            if constexpr (PENALTIES) {
                const uint32_t again = least < 0x1p-90f || most > 0x1p100f || divide ? (1u << 4 * QUADS) - 1 : hit;
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(again != 0) != 0, 0)) {
                    for (int w = 0; w < 4 * QUADS; ++w) {
                        if (!((again >> w) & 1)) continue;
                        const int32_t e = e0 + 4 * THREADS * (w >> 2) + (w & 3);
                        int32_t times = 0;
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            for (u64 left = on_path[h]; left != 0; left &= left - 1) times += __builtin_amdgcn_readlane(tok_of[h], __builtin_ctzll(left)) == e ? 1 : 0;
                        float x = 0.f;
#pragma unroll
                        for (int z = 0; z < 4 * QUADS; ++z) x = z == w ? r.x[z / 4][z % 4] : x;
                        x = penalised(x, reinterpret_cast<const int32_t*>(mine4 + (3 * (w >> 2) + 2) * THREADS)[w & 3], times, rules);
#pragma unroll
                        for (int z = 0; z < 4 * QUADS; ++z) y[z / 4][z % 4] = z == w ? x : y[z / 4][z % 4];
                    }
                }
            }
            float* out = p.out ? p.out + (row0 + i) * p.V : nullptr;
            float top = -INFINITY;
            uint32_t keep = ~0u, all = 0u;       // of the grammar's words, and what is added: a row without a state allows everything
            if (p.allow) {
                const int32_t at = __builtin_amdgcn_readlane(state_of, i - i0);
                keep = at < -1 || at >= p.n_allow ? 0u : ~0u;
                all = at == -1 ? ~0u : 0u;
            }
#pragma unroll
            for (int u = 0; u < QUADS; ++u) {
                const int32_t e = e0 + 4 * THREADS * u;
                if (bias) {
                    const float4 x = mine4[(3 * u + 1) * THREADS];
                    y[u][0] = y[u][0] + x.x;
                    y[u][1] = y[u][1] + x.y;
                    y[u][2] = y[u][2] + x.z;
                    y[u][3] = y[u][3] + x.w;
                }
                if (p.allow) {
                    const uint32_t may = ((r.may[u] & keep) | all) >> (e & 31);
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[u][k] = (may >> k) & 1 ? y[u][k] : -INFINITY;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) top = __builtin_fmaxf(top, y[u][k]);      // (passes over NaN; columns that are not there are -infinity)
                if (out) {
                    if (INSIDE || e < full) *reinterpret_cast<float4u*>(out + e) = float4u{y[u][0], y[u][1], y[u][2], y[u][3]};
                    else if (e < p.V) {
                        out[e] = y[u][0];
                        if (e + 1 < p.V) out[e + 1] = y[u][1];
                        if (e + 2 < p.V) out[e + 2] = y[u][2];
                    }
                }
            }
            if (p.target_ids) {
                // the wavefront's maximum, then its first column, looked for by the lanes that have it
                const float best = wave_max_f32(top);
                int32_t at = INT32_MAX;
                if (top == best) {
#pragma unroll
                    for (int z = 4 * QUADS - 1; z >= 0; --z) at = y[z / 4][z % 4] == best ? e0 + 4 * THREADS * (z / 4) + z % 4 : at;
                }
                const u64 having = __builtin_amdgcn_ballot_w64(top == best);
                if ((having & (having - 1)) == 0) at = __builtin_amdgcn_readlane(at, __builtin_ctzll(having));
                else at = static_cast<int32_t>(~wave_max_u32(~static_cast<uint32_t>(at)));
                if (lane == 0) p.partial[((row0 + i) * gridDim.x + block) * WAVES + wave] = key_of(best, at);
            }
        }
        };
        if (full - first >= 4 * THREADS * QUADS) pass(std::true_type{});
        else pass(std::false_type{});
    }
}

// One wavefront a row: the best of its parts.
__global__ __launch_bounds__(256) void adjust_fold_kernel(const u64* __restrict__ partial, int32_t parts, int32_t rows, int32_t* __restrict__ target_ids) {
    const int32_t row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (row >= rows) return;
    u64 best = 0;
    for (int32_t j = lane; j < parts; j += 64) {
        const u64 x = partial[static_cast<size_t>(row) * parts + j];
        best = x > best ? x : best;
    }
    best = wave_max_key(best);
    if (lane == 0) target_ids[row] = id_of(best);
}

// Columns of a block, rows of a workgroup.
struct AdjustPlan { int32_t quads, blocks, rows_per; };
static AdjustPlan adjust_plan(int32_t B, int32_t K_max, int32_t V) {
    const int64_t rows = static_cast<int64_t>(B) * K_max;
    auto blocks = [&](int32_t quads) { return (V - 1) / (4 * LA_THREADS * quads) + 1; };
    AdjustPlan a{LA_QUADS, blocks(LA_QUADS), 1};
    if (a.blocks * rows < LA_FILL) a = {1, blocks(1), 1};         // few: smaller blocks
    while (a.rows_per < LA_ROWS && 2 * a.rows_per <= K_max && a.blocks * rows / (2 * a.rows_per) >= LA_FILL) a.rows_per *= 2;
    return a;
}

}  // namespace graft

extern "C" size_t graft_logits_adjust_workspace_bytes(int32_t B, int32_t K_max, int32_t V) {
    if (B < 1 || K_max < 1 || V < 1 || V >= (1 << 30)) return 0;
    const int64_t rows = static_cast<int64_t>(B) * K_max;
    const graft::AdjustPlan a = graft::adjust_plan(B, K_max, V);
    return static_cast<size_t>(rows) * a.blocks * (graft::LA_THREADS / 64) * sizeof(graft::u64);
}

extern "C" int32_t graft_logits_adjust(const float* logits, const int32_t* n_nodes, const int32_t* tokens, const uint64_t* mask, int32_t B,
                                       int32_t K_max, int32_t V, const int32_t* counts, const float* repetition, const float* frequency,
                                       const float* presence, const float* bias, int32_t bias_rows, const uint32_t* allow, int32_t n_allow,
                                       const int32_t* allow_index, float* out, int32_t* target_ids, int32_t* status, void* workspace,
                                       size_t workspace_bytes, void* stream) {
    using namespace graft;
    if (!logits || !n_nodes || !status || (!out && !target_ids) || (!tokens) != (!mask) || (!allow) != (!allow_index)) return GRAFT_ERR_NULL;
    if (B < 1 || B > 65535 || K_max < 1 || K_max > GRAFT_MAX_NODES || V < 1 || V >= (1 << 30) || (bias && bias_rows != 1 && bias_rows != B) || (allow && n_allow < 1))
        return GRAFT_ERR_SHAPE;
    const int64_t rows = static_cast<int64_t>(B) * K_max;
    if (out && out != logits) {
        const size_t a = reinterpret_cast<size_t>(out), l = reinterpret_cast<size_t>(logits), size = static_cast<size_t>(rows) * V * sizeof(float);
        if (a < l + size && l < a + size) return GRAFT_ERR_SHAPE;
    }
    const AdjustPlan a = adjust_plan(B, K_max, V);
    if (target_ids && (!workspace || workspace_bytes < graft_logits_adjust_workspace_bytes(B, K_max, V))) return GRAFT_ERR_WORKSPACE;
    if (reinterpret_cast<size_t>(workspace) & 7) return GRAFT_ERR_WORKSPACE;
    const AdjustParams p{logits, n_nodes, tokens, reinterpret_cast<const u64*>(mask), counts, repetition, frequency, presence, bias, allow, allow_index,
                         out, target_ids, status, target_ids ? static_cast<u64*>(workspace) : nullptr,
                         bias && bias_rows > 1 ? static_cast<int64_t>(V) : 0, K_max, V, (V - 1) / 32 + 1, n_allow, a.rows_per};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool penalties = repetition || frequency || presence, once = read_once(rows, V);
    const dim3 grid(a.blocks, (K_max + a.rows_per - 1) / a.rows_per, B);
    auto launch = [&](auto quads) {
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(LA_THREADS), 0, s, n_nodes, p); };
        if (penalties) { if (once) go(logits_adjust_kernel<true, true, quads>); else go(logits_adjust_kernel<true, false, quads>); }
        else if (once) go(logits_adjust_kernel<false, true, quads>);
        else go(logits_adjust_kernel<false, false, quads>);
    };
    using std::integral_constant;
    if (a.quads == 1) launch(integral_constant<int, 1>{});
    else launch(integral_constant<int, LA_QUADS>{});
    int32_t rc = check_launch();
    if (rc != GRAFT_OK || !p.partial) return rc;
    hipLaunchKernelGGL(adjust_fold_kernel, dim3(static_cast<uint32_t>((rows + 3) / 4)), dim3(256), 0, s, p.partial, a.blocks * (LA_THREADS / 64),
                       static_cast<int32_t>(rows), target_ids);
    return check_launch();
}
