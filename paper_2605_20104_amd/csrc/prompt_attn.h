// What the parts of graft_prompt_attn share: prompt_attn.hip (plan, merge, entry point) and the kernels:
// prompt_attn_bf16.hip, prompt_attn_f32.hip, and for few rows prompt_attn_few.hip, prompt_attn_few_f32.hip.
#pragma once
#include "attn_mfma.h"

namespace graft {

constexpr int PA_MAX_SPLITS = 32;

struct PromptParams {
    const void* q;
    const void* k;
    const void* v;
    void* out;
    const int32_t* block_table;
    const int32_t* prefix_len;
    const int32_t* n_nodes;
    float* ws_o;            // partial rows of the splits, [B * Hkv][splits][R][D]
    float* ws_ml;           // their reference (log2 units) and sum, [B * Hkv][splits][R][2]
    int64_t page_stride, token_stride, head_stride;
    int32_t max_pages, B, T, Hq, Hkv, G, R, n_splits, n_row_tiles;      // R = T G rows of a KV head: row r is head r % G of token r / G
    int32_t window;         // INT32_MAX: none
    uint32_t g_magic;       // div_any(r, g_magic, g_shift) = r / G
    int32_t g_shift;
    uint32_t q_sign;        // a negative scale is a positive one with queries of the other sign (hidden scores are -inf, and stay it)
    float scale_log2e;      // scores in log2 units are x * scale_log2e, or
    float cap_in, cap_log2e;    // cap_log2e tanh(x * scale / cap), cap_in = 2 scale log2(e) / cap
};

// Lengths of a sequence; n = 0 where they do not fit (its rows are zeros).
struct PromptLengths { int P, n; };
__device__ __forceinline__ PromptLengths prompt_lengths(const PromptParams& p, int P, int n) {
    const bool ok = P >= 0 && n >= 0 && n <= p.T && static_cast<int64_t>(P) + n <= static_cast<int64_t>(p.max_pages) * GRAFT_PAGE_SIZE;
    return {ok ? P : 0, ok ? n : 0};
}

// Tokens i0 .. i1 of a row tile that are there (i1 < i0: none), and the stages of STAGE tokens that they see.
struct PromptRange { int i0, i1, st0, st1; };
template <int STAGE>
__device__ __forceinline__ PromptRange prompt_range(const PromptParams& p, PromptLengths len, int r0, int tile_rows) {
    PromptRange t;
    t.i0 = div_any(r0, p.g_magic, p.g_shift);
    const int last = r0 + tile_rows - 1;
    t.i1 = div_any(last < p.R ? last : p.R - 1, p.g_magic, p.g_shift);
    t.i1 = t.i1 < len.n ? t.i1 : len.n - 1;
    const int first = len.P + t.i0 >= p.window ? len.P + t.i0 - p.window + 1 : 0;
    t.st0 = first / STAGE;
    t.st1 = t.i1 < t.i0 ? t.st0 : (len.P + t.i1) / STAGE + 1;
    return t;
}

// Workgroups, one for each (sequence, KV head, split) = unit and row tile, are dealt to the 8 XCDs as xcd_work_item deals them: all
// row tiles of a unit on one XCD, those of what is left over one by one.  The last tiles, which see most keys, come first, of all
// of an XCD's units before the next ones of any: unit by unit, the last units' long tiles started when everything else was done (four ragged prompts of
// 2049, 8 KV heads: 114 -> 108 us).
struct PromptItem { int unit, row_tile; };                         // unit < 0: padding of the grid
inline unsigned prompt_grid(const PromptParams& p) { return xcd_grid(static_cast<int64_t>(p.B) * p.Hkv * p.n_splits, p.n_row_tiles); }
__device__ __forceinline__ PromptItem prompt_item(const PromptParams& p) {
    const int n_units = p.B * p.Hkv * p.n_splits, xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, each = n_units >> 3, whole = each * p.n_row_tiles;
    const bool left = slot >= whole;
    const int s = left ? (slot - whole) * 8 + xcd : slot, among = left ? n_units & 7 : each;
    if (among == 0) return {-1, 0};
    const int rank = s / among, u = s - rank * among, unit = left ? (n_units & ~7) + u : u * 8 + xcd;
    return {rank < p.n_row_tiles ? unit : -1, p.n_row_tiles - 1 - rank};
}

// y of the capped scores in log2 units: cap log2(e) tanh(x scale / cap), as 1 - 2 / (1 + e^2z).  Off by a few 2^-24 of the cap.
__device__ __forceinline__ float capped(float x, float cap_in, float cap_log2e) {
    const float e = __builtin_amdgcn_exp2f(x * cap_in);
    return __builtin_fmaf(-2.f * cap_log2e, __builtin_amdgcn_rcpf(1.f + e), cap_log2e);
}
// The same for fp32 attention: small arguments, where the difference above keeps few bits, by tanh's odd polynomial (up to |z| = 0.45
// the terms to z^13 of its series are within 2^-25 of it; the argument is 2 z log2(e)).
__device__ __forceinline__ float capped_f32(float x, float cap_in, float cap_log2e) {
    const float u = x * cap_in, z = u * 0.34657359028f, w = z * z;
    float s = __builtin_fmaf(w, 21844.f / 6081075.f, -1382.f / 155925.f);
    s = __builtin_fmaf(w, s, 62.f / 2835.f);
    s = __builtin_fmaf(w, s, -17.f / 315.f);
    s = __builtin_fmaf(w, s, 2.f / 15.f);
    s = __builtin_fmaf(w, s, -1.f / 3.f);
    s = __builtin_fmaf(w * z, s, z);
    const float far = __builtin_fmaf(-2.f * cap_log2e, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(u)), cap_log2e);
    return __builtin_fabsf(z) < 0.45f ? s * cap_log2e : far;
}

constexpr int PA_BF16_ROWS = 256, PA_F32_ROWS = 128, PA_FEW_ROWS = 32;             // rows of a tile
int32_t launch_prompt_f32(const PromptParams& p, int32_t D, bool cap, hipStream_t s);
int32_t launch_prompt_bf16(const PromptParams& p, int32_t D, bool cap, hipStream_t s);
int32_t launch_prompt_few_f32(const PromptParams& p, int32_t D, bool cap, int32_t tile_rows, hipStream_t s);
int32_t launch_prompt_few(const PromptParams& p, int32_t D, bool cap, int32_t tile_rows, hipStream_t s);     // tiles of 32 or 64 rows, bf16

}  // namespace graft
