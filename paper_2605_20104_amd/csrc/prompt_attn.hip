// graft_prompt_attn: plan, merge of the keys' splits, entry point.  The kernels: prompt_attn_bf16.hip, prompt_attn_f32.hip.
#include <cmath>

#include "prompt_attn.h"

namespace graft {

// Few row tiles leave compute units without work: their keys are cut into splits, whose unnormalised rows go through memory in fp32
// and are joined by their references and sums.
template <int D, class T>
__global__ __launch_bounds__(256) void prompt_merge_kernel(const int32_t* n_nodes, const int32_t* prefix_len, PromptParams p) {
    constexpr int LANES = D / 4, ROWS = 256 / LANES;               // lanes a row, four elements each
    const int lane = threadIdx.x % LANES, per = (p.R + ROWS - 1) / ROWS, bg = blockIdx.x / per,
              r = (blockIdx.x - bg * per) * ROWS + threadIdx.x / LANES, b = bg / p.Hkv, g = bg - b * p.Hkv;
    if (r >= p.R) return;
    const PromptLengths len = prompt_lengths(p, scalar_load(prefix_len, b), scalar_load(n_nodes, b));
    const int i = div_any(r, p.g_magic, p.g_shift);
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
    if (i < len.n) {
        const size_t part = static_cast<size_t>(bg) * p.n_splits * p.R + r;
        const float2* ml = reinterpret_cast<const float2*>(p.ws_ml);
        float m = -INFINITY;
        for (int s = 0; s < p.n_splits; ++s) {
            const float2 x = ml[part + static_cast<size_t>(s) * p.R];
            m = __builtin_fmaxf(m, x.y != 0.f ? x.x : -INFINITY);   // (a sum of zero: nothing seen; NaN passes)
        }
        for (int s = 0; s < p.n_splits; ++s) {
            const size_t at = part + static_cast<size_t>(s) * p.R;
            const float2 x = ml[at];
            const floatx4 o = *reinterpret_cast<const floatx4*>(p.ws_o + at * D + 4 * lane);
            const float f = x.y != 0.f ? __builtin_amdgcn_exp2f(x.x - m) : 0.f;
            total += x.y * f;
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] += x.y != 0.f ? o[j] * f : 0.f;
        }
        const float inv = total != 0.f ? 1.f / total : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] *= inv;
    }
    const size_t to = ((static_cast<size_t>(b) * p.T + i) * p.Hq + g * p.G + (r - i * p.G)) * D + 4 * lane;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uintx2*>(static_cast<unsigned short*>(p.out) + to) = uintx2{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
    else *reinterpret_cast<floatx4*>(static_cast<float*>(p.out) + to) = sum;
}

struct PromptPlan { int32_t tile_rows, n_row_tiles, n_splits; size_t o_bytes, bytes; };
#ifndef PA_FEW
#define PA_FEW 64
#endif
// A kernel and its splits, by what a launch takes: rounds of the compute units times a tile's share of the keys and its set-up, and for splits
// a launch and the partial rows' way through memory.  The host knows the table's capacity, not the lengths: half of the cost is
// that of sequences that fill it, half that of ragged ones, three quarters of it in the mean, whose workgroups end one by one.
static PromptPlan prompt_plan(int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_pages, int32_t dtype, int32_t window) {
    const bool f32 = dtype == GRAFT_F32;
    const int32_t G = Hq / Hkv;
    const int64_t R = static_cast<int64_t>(T) * G, units = static_cast<int64_t>(B) * Hkv, cus = device_compute_units();
    struct Kernel { int32_t rows, stage, per_cu; double stage_us, setup_us; };
    const Kernel kernel = f32 ? Kernel{PA_F32_ROWS, 32, 2, D == 128 ? 8.0 : 4.0, 3.0}
                        : R <= 32 ? Kernel{32, 128, 1, D == 128 ? 2.7 : 1.4, 4.0}
                        : R <= PA_FEW ? Kernel{64, 128, 1, D == 128 ? 2.7 : 1.5, 4.0} : Kernel{PA_BF16_ROWS, 64, D == 128 ? 1 : 2, D == 128 ? 1.2 : 1.4, 4.0};
    const int64_t tiles = (R + kernel.rows - 1) / kernel.rows, places = cus * kernel.per_cu;
    int64_t keys = static_cast<int64_t>(max_pages) * GRAFT_PAGE_SIZE;
    const int64_t reach = static_cast<int64_t>(window) + kernel.rows / G + 1;
    if (window > 0 && reach < keys) keys = reach;
    const int64_t stages = (keys + kernel.stage - 1) / kernel.stage;
    PromptPlan best{kernel.rows, static_cast<int32_t>(tiles), 1, 0, 0};
    double cost = -1.0;
    for (int64_t s = 1; s <= PA_MAX_SPLITS && s <= stages && tiles * units * s < (1 << 23); ++s) {
        const double jobs = static_cast<double>(tiles * units * s), per = static_cast<double>((stages + s - 1) / s) * kernel.stage_us + kernel.setup_us;
        const double even = std::ceil(jobs / places) * per, last = 0.75 * jobs / places * per + 0.5 * per, ragged = last > per ? last : per;
        double now = 0.5 * (even + ragged);
        if (s > 1) now += 4.0 + static_cast<double>(R * units * s) * D * 4 * 2 / 4e6;
        if (cost < 0 || now < cost) { cost = now; best.n_splits = static_cast<int32_t>(s); }
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
    float* const ws = static_cast<float*>(workspace);
    const PromptParams p{q, k_cache, v_cache, out, block_table, prefix_len, n_nodes, ws, plan.bytes ? ws + plan.o_bytes / sizeof(float) : nullptr, page_stride,
                         token_stride, head_stride, max_pages, B, T, Hq, Hkv, G, T * G, plan.n_splits, plan.n_row_tiles,
                         window > 0 ? window : INT32_MAX, by_g.m, by_g.shift,
                         !std::signbit(scale) ? 0u : dtype == GRAFT_F32 ? 0x80000000u : 0x80008000u, std::fabs(in), std::fabs(cap_in), softcap * log2e};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool cap = softcap > 0.f;
    const int32_t rc = dtype == GRAFT_F32 ? launch_prompt_f32(p, D, cap, s)
                     : plan.tile_rows < PA_BF16_ROWS ? launch_prompt_few(p, D, cap, plan.tile_rows, s) : launch_prompt_bf16(p, D, cap, s);
    if (rc != GRAFT_OK || plan.n_splits == 1) return rc;
    auto merge = [&](auto kernel, int rows) { hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>((p.R + rows - 1) / rows) * B * Hkv), dim3(256), 0, s, n_nodes, prefix_len, p); };
    if (dtype == GRAFT_F32) { if (D == 128) merge(prompt_merge_kernel<128, float>, 8); else merge(prompt_merge_kernel<64, float>, 16); }
    else if (D == 128) merge(prompt_merge_kernel<128, unsigned short>, 8);
    else merge(prompt_merge_kernel<64, unsigned short>, 16);
    return check_launch();
}
