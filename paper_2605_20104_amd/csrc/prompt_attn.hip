// graft_prompt_attn: plan, merge of the keys' splits, entry point.  The kernels: prompt_attn_bf16.hip, prompt_attn_f32.hip, prompt_attn_few.hip,
// prompt_attn_few_f32.hip.
#include <cmath>

#include "prompt_attn.h"

namespace graft {

// Few row tiles leave compute units without work: their keys are cut into splits, whose unnormalised rows go through memory in fp32
// and are joined by their references and sums.
// A wavefront a row: lane s has split s's reference and sum, then every lane its D / 64 elements of all splits' rows, eight in flight.
// Bound by the Infinity Cache and its own launch: 4.6 to 5.7 us for 1024 rows, 20.5 for 1024 tokens of 40 heads (D = 128, 3 splits: 63 MB read).
static_assert(PA_MAX_SPLITS <= 64, "a lane each");
template <int DPP_CTRL> __device__ __forceinline__ float add_dpp(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), DPP_CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float wave_sum_f32(float v) {
    v = add_dpp<0xB1>(v);
    v = add_dpp<0x4E>(v);
    v = add_dpp<0x141>(v);
    v = add_dpp<0x140>(v);
    unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    u = __float_as_uint(__uint_as_float(a[0]) + __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
template <int D, class T>
__global__ __launch_bounds__(256) void prompt_merge_kernel(const int32_t* n_nodes, const int32_t* prefix_len, PromptParams p) {
    constexpr int EACH = D / 64, AHEAD = 8;
    typedef float part_t __attribute__((ext_vector_type(EACH)));
    const int lane = threadIdx.x & 63, per = (p.R + 3) / 4, bg = blockIdx.x / per;
    const int r = __builtin_amdgcn_readfirstlane((blockIdx.x - bg * per) * 4 + (threadIdx.x >> 6)), b = bg / p.Hkv, g = bg - b * p.Hkv;
    if (r >= p.R) return;
    const size_t part = static_cast<size_t>(bg) * p.n_splits * p.R + r;
    const float* from = p.ws_o + part * D + EACH * lane;
    const size_t step = static_cast<size_t>(p.R) * D;
    const float2 ml = lane < p.n_splits ? reinterpret_cast<const float2*>(p.ws_ml)[part + static_cast<size_t>(lane) * p.R] : float2{0.f, 0.f};
    part_t o[AHEAD];
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) o[s] = *reinterpret_cast<const part_t*>(from + (s < p.n_splits ? s : 0) * step);
    const PromptLengths len = prompt_lengths(p, scalar_load(prefix_len, b), scalar_load(n_nodes, b));
    const int i = div_any(r, p.g_magic, p.g_shift);
    // (a sum of zero: the split saw nothing; NaN passes)
    const float m = wave_max_f32(lane < p.n_splits && ml.y != 0.f ? ml.x : -INFINITY), f = ml.y != 0.f ? __builtin_amdgcn_exp2f(ml.x - m) : 0.f;
    const float total = wave_sum_f32(ml.y * f);
    const u64 some = __builtin_amdgcn_ballot_w64(ml.y != 0.f);      // (not by f: 0 times an infinity is not 0)
    part_t sum = part_t(0.f);
    for (int s0 = 0; s0 < p.n_splits; s0 += AHEAD) {
        if (s0 > 0) {
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) o[s] = *reinterpret_cast<const part_t*>(from + (s0 + s < p.n_splits ? s0 + s : 0) * step);
        }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
            if (s0 + s < p.n_splits) {
                const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), s0 + s));
                if ((some >> (s0 + s)) & 1) sum += o[s] * w;                      // (uniform)
            }
    }
    const float inv = total != 0.f ? 1.f / total : 0.f;
    if (i < len.n) sum *= inv;
    else sum = part_t(0.f);
    const size_t to = ((static_cast<size_t>(b) * p.T + i) * p.Hq + g * p.G + (r - i * p.G)) * D + EACH * lane;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<part_t*>(static_cast<float*>(p.out) + to) = sum;
    else if constexpr (EACH == 2) *reinterpret_cast<unsigned*>(static_cast<unsigned short*>(p.out) + to) = pack_bf16(sum[0], sum[1]);
    else static_cast<unsigned short*>(p.out)[to] = static_cast<unsigned short>(pack_bf16(sum[0], 0.f));
}

// A kernel and its splits, by an estimate of what a launch takes: rounds of the compute units (`per_cu` workgroups each) times a tile's
// share of the keys, stage by stage, and its set-up; a stage takes what the matrix cores take, or memory for all that run at once; splits
// add a launch and the partial rows' way through memory.  The host knows the table's capacity, not the lengths: where there are several
// sequences, half of the estimate is for ones that fill it, half for ragged ones, three quarters of it in the mean, whose workgroups end one by one.
// Measured with the splits given (us, 32 heads on 8, D = 128; rows of a tile, splits): 1 token behind 2000: 32 rows, 1: 21, 4: 14.0, 8:
// 12.1, 16: 12.5; behind 65536: 8: 67, 16: 48.1, 32: 51.1; 32 ragged sequences' tokens behind 16384: 1: 305, 4: 278, 8: 282; 32 tokens behind
// 32768: 64 rows, 16: 43.6, 256 rows, 32: 50.8; 64 behind 2048: 64 rows, 6: 20.7, 256 rows, 8: 29.6; 48 behind 32768: 64 rows, 8: 65.6, 256 rows,
// 32: 55.4; 256 behind 2048: 1: 65, 6: 37.7, 12: 56.7; 1024 behind 32768, 40 heads: 1: 719, 3: 621, 4: 679.
// fp32, 16 rows: 1 behind 65536: 16: 132, 20: 111, 24: 100, 32: 103; 8 tokens behind 16000: 1: 463, 2: 243, 3: 183, 5: 248, 8: 185.
// Partial rows may take what the Infinity Cache holds, 256 MiB.  Past that a split gains the end of a last round where the table is full, and
// costs most where it is not (us, D = 128, without a split / with two, from an empty cache / in a full table): 4500 tokens of 64 heads, 131072 in the
// table: 353 / 565, 16530 / 15360; 9000 of 32, 65536: 610 / 800, 7950 / 7430.  (So a merge, with 64 lanes a row, always fits a launch.)
// Within it a table that is wide and empty still costs: 1100 tokens of 32 heads in 7 splits from an empty cache 101 us where the table has 131072
// tokens, behind 130000 2060.  A table as wide as what a sequence holds is planned for what it holds.
constexpr int64_t PA_SPLIT_BYTES = 1 << 28;
struct PromptKernel { int32_t rows, stage, per_cu; double stage_us, setup_us; };      // rows of a tile, keys of a stage
struct PromptPlan { int32_t tile_rows, n_row_tiles, n_splits; size_t o_bytes, bytes; };
static PromptPlan prompt_plan(int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_pages, int32_t dtype, int32_t window) {
    const bool f32 = dtype == GRAFT_F32, wide = D == 128;
    const int32_t G = Hq / Hkv;
    const int64_t R = static_cast<int64_t>(T) * G, units = static_cast<int64_t>(B) * Hkv, cus = device_compute_units();
    const PromptKernel bf16_kernels[] = {{PA_FEW_ROWS, 128, 1, wide ? 1.3 : 0.8, 5.0}, {2 * PA_FEW_ROWS, 128, 1, wide ? 2.0 : 1.2, 5.0},
                                         {PA_BF16_ROWS, 64, wide ? 1 : 2, wide ? 1.8 : 2.0, 5.0}};
    const PromptKernel f32_kernels[] = {{PA_FEW_ROWS / 2, 128, 1, wide ? 3.6 : 1.75, 5.0}, {PA_FEW_ROWS, 128, 1, wide ? 5.0 : 2.5, 5.0},
                                        {PA_F32_ROWS, 32, 2, wide ? 7.6 : 3.8, 5.0}};
    PromptPlan best{0, 0, 0, 0, 0};
    double cost = 0.0;
    auto look = [&](const PromptKernel& kernel) {
        const int64_t tiles = (R + kernel.rows - 1) / kernel.rows, places = cus * kernel.per_cu;
        int64_t keys = static_cast<int64_t>(max_pages) * GRAFT_PAGE_SIZE;
        const int64_t reach = static_cast<int64_t>(window) + kernel.rows / G + 1;
        if (window > 0 && reach < keys) keys = reach;
        const int64_t stages = (keys + kernel.stage - 1) / kernel.stage;
        const double stage_bytes = 2.0 * kernel.stage * D * (f32 ? 4 : 2);
        for (int64_t s = 1; s <= PA_MAX_SPLITS && s <= stages && tiles * units * s < (1 << 23); ++s) {
            if (s > 1 && R * units * s * (D + 2) * 4 > PA_SPLIT_BYTES) break;
            const double jobs = static_cast<double>(tiles * units * s), at_once = jobs < places ? jobs : places;
            const double memory_us = at_once / tiles * stage_bytes / 5.6e6;       // (the tiles of a unit share what they read)
            const double per = static_cast<double>((stages + s - 1) / s) * (memory_us > kernel.stage_us ? memory_us : kernel.stage_us) + kernel.setup_us;
            const double even = std::ceil(jobs / places) * per, last = 0.75 * jobs / places * per + 0.5 * per, ragged = last > per ? last : per;
            double now = B > 1 ? 0.5 * (even + ragged) : even;
            if (s > 1) now += 3.0 + static_cast<double>(R * units * s) * D * 4 * 2 / 4e6;
            if (best.n_splits == 0 || now < cost) {
                cost = now;
                best = {kernel.rows, static_cast<int32_t>(tiles), static_cast<int32_t>(s), 0, 0};
            }
        }
    };
    if (f32) {
        if (R <= PA_FEW_ROWS / 2) look(f32_kernels[0]);
        else if (R <= PA_FEW_ROWS) look(f32_kernels[1]);
        else look(f32_kernels[2]);
    } else if (R <= PA_FEW_ROWS) look(bf16_kernels[0]);
    else {
        if (R <= 2 * PA_BF16_ROWS) look(bf16_kernels[1]);
        look(bf16_kernels[2]);
    }
    if (best.n_splits > 1) {
        const size_t rows = static_cast<size_t>(R) * units * best.n_splits;
        best.o_bytes = rows * D * sizeof(float);
        best.bytes = best.o_bytes + rows * 2 * sizeof(float);
    }
    return best;
}

static bool prompt_sizes_ok(int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_pages, int32_t window) {
    return B >= 1 && B <= 65535 && T >= 1 && T <= (1 << 22) && Hkv >= 1 && Hq >= 1 && Hq % Hkv == 0 && Hq / Hkv <= 16 && (D == 64 || D == 128) &&
           max_pages >= 1 && max_pages <= 262144 && window >= 0 && static_cast<int64_t>(B) * Hkv <= (1 << 18) &&
           static_cast<int64_t>(B) * Hkv * ((static_cast<int64_t>(T) * (Hq / Hkv) + 127) / 128) < (1 << 23);     // (lanes of a launch)
}

}  // namespace graft

extern "C" size_t graft_prompt_attn_workspace_bytes(int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_pages, int32_t window,
                                                    int32_t dtype) {
    if ((dtype != GRAFT_F32 && dtype != GRAFT_BF16) || !graft::prompt_sizes_ok(B, T, Hq, Hkv, D, max_pages, window)) return 0;
    return graft::prompt_plan(B, T, Hq, Hkv, D, max_pages, dtype, window).bytes;
}

extern "C" int32_t graft_prompt_attn(const void* q, const void* k_cache, const void* v_cache, int64_t page_stride, int64_t token_stride,
                                     int64_t head_stride, const int32_t* block_table, int32_t max_pages, const int32_t* prefix_len,
                                     const int32_t* n_nodes, int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t page_size, float scale,
                                     float softcap, int32_t window, int32_t dtype, void* out, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace graft;
    if (!q || !k_cache || !v_cache || !block_table || !prefix_len || !n_nodes || !out) return GRAFT_ERR_NULL;
    if (dtype != GRAFT_F32 && dtype != GRAFT_BF16) return GRAFT_ERR_DTYPE;
    if (!prompt_sizes_ok(B, T, Hq, Hkv, D, max_pages, window) || page_size != GRAFT_PAGE_SIZE || page_stride < 1 || token_stride < D || head_stride < D ||
        token_stride >= (1 << 26) || page_stride % 8 != 0 || token_stride % 8 != 0 || head_stride % 8 != 0)
        return GRAFT_ERR_SHAPE;
    const float log2e = 1.44269504088896340736f, in = scale * log2e, cap_in = softcap > 0.f ? 2.f * scale * log2e / softcap : 0.f;
    if (!std::isfinite(in) || !(softcap >= 0.f && softcap <= 1024.f) || !std::isfinite(cap_in)) return GRAFT_ERR_SHAPE;
    if ((reinterpret_cast<size_t>(q) | reinterpret_cast<size_t>(k_cache) | reinterpret_cast<size_t>(v_cache) | reinterpret_cast<size_t>(out)) & 15)
        return GRAFT_ERR_SHAPE;
    if (out != q) {
        const size_t a = reinterpret_cast<size_t>(out), x = reinterpret_cast<size_t>(q), size = static_cast<size_t>(B) * T * Hq * D * (dtype == GRAFT_F32 ? 4 : 2);
        if (a < x + size && x < a + size) return GRAFT_ERR_SHAPE;
    }
    const PromptPlan plan = prompt_plan(B, T, Hq, Hkv, D, max_pages, dtype, window);
    if (plan.bytes > 0 && (!workspace || workspace_bytes < plan.bytes || (reinterpret_cast<size_t>(workspace) & 15))) return GRAFT_ERR_WORKSPACE;
    const int32_t G = Hq / Hkv;
    const Magic by_g = magic_any(static_cast<uint32_t>(G));
    // Hidden scores are -inf, which a scale of zero behind them would make NaN.  A cap of 1 without a cap's scale makes the same zeros of what
    // is seen (and NaN where 0 times the product is none), in front of what hides.  (A product with log2(e) is zero for a scale of zero only.)
    const bool flat = in == 0.f && softcap == 0.f, cap = softcap > 0.f || flat;
    float* const ws = static_cast<float*>(workspace);
    const PromptParams p{q, k_cache, v_cache, out, block_table, prefix_len, n_nodes, ws, plan.bytes ? ws + plan.o_bytes / sizeof(float) : nullptr, page_stride,
                         token_stride, head_stride, max_pages, B, T, Hq, Hkv, G, T * G, plan.n_splits, plan.n_row_tiles,
                         window > 0 ? window : INT32_MAX, by_g.m, by_g.shift,
                         !std::signbit(scale) ? 0u : dtype == GRAFT_F32 ? 0x80000000u : 0x80008000u, std::fabs(in), std::fabs(cap_in), (flat ? 1.f : softcap) * log2e};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int32_t rc = plan.tile_rows <= PA_FEW_ROWS && dtype == GRAFT_F32 ? launch_prompt_few_f32(p, D, cap, plan.tile_rows, s)
                     : dtype == GRAFT_F32 ? launch_prompt_f32(p, D, cap, s)
                     : plan.tile_rows < PA_BF16_ROWS ? launch_prompt_few(p, D, cap, plan.tile_rows, s) : launch_prompt_bf16(p, D, cap, s);
    if (rc != GRAFT_OK || plan.n_splits == 1) return rc;
    auto merge = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>((p.R + 3) / 4) * B * Hkv), dim3(256), 0, s, n_nodes, prefix_len, p); };
    if (dtype == GRAFT_F32) { if (D == 128) merge(prompt_merge_kernel<128, float>); else merge(prompt_merge_kernel<64, float>); }
    else if (D == 128) merge(prompt_merge_kernel<128, unsigned short>);
    else merge(prompt_merge_kernel<64, unsigned short>);
    return check_launch();
}
