// graft_prompt_attn, fp32, few rows (up to 32 of a KV head: single tokens, short pieces): the wavefronts take 32 tokens each in turn and join
// their rows through LDS at the end, as in prompt_attn_few.hip; products as in prompt_attn_f32.hip.
//
// Keys and values go from memory to registers as the products want them, values during the first product of their step, the next
// step's keys during the second: lane (half, l32) reads dims 8 c + 4 half + 0..3 of key l32, and dim 32 e + l32 of the values of tokens 8 (x / 4) + 4 half + x % 4.
// Bound by memory where there is much of it (8 sequences, 4 tokens of 32 heads behind 8000, D = 64: 61 us with the merge, 4.3 TB/s), else by the
// way through a wavefront's steps: one token behind 255 takes 10.6 us.  Eight wavefronts a workgroup: 11.5, 62; four it is.
#include "prompt_attn.h"

namespace graft {

constexpr int PV_STEP = 32;
constexpr float PV_RISE = 8.f, PV_FRESH = 3e38f;      // as in prompt_attn_bf16.hip

__device__ __forceinline__ float pv_sum(float v) {
    const unsigned u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float pv_max(float v) {
    const unsigned u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ bool pv_no_number(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

template <int D, bool CAP>
__global__ __launch_bounds__(AT_THREADS, 1) void prompt_few_f32_kernel(const int32_t* n_nodes, const int32_t* prefix_len, PromptParams p) {
    constexpr int DE = D / 32, DC = D / 8;
    __shared__ __attribute__((aligned(16))) float rows[AT_WAVES][PV_STEP * D];     // values that are no numbers, then what is joined
    __shared__ float2 stat[AT_WAVES][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const PromptItem item = prompt_item(p);
    if (item.unit < 0) return;
    const int bg = item.unit / p.n_splits, split = item.unit - bg * p.n_splits, b = bg / p.Hkv, g = bg - b * p.Hkv;
    const PromptLengths len = prompt_lengths(p, scalar_load(prefix_len, b), scalar_load(n_nodes, b));
    const int r_tile = item.row_tile * PA_FEW_ROWS;
    const PromptRange t = prompt_range<PV_STEP>(p, len, r_tile, PA_FEW_ROWS);
    const int spt = (t.st1 - t.st0 + p.n_splits - 1) / p.n_splits, st0 = t.st0 + split * spt, st1 = st0 + spt < t.st1 ? st0 + spt : t.st1;

    const int r = r_tile + l32, i = div_any(r, p.g_magic, p.g_shift), lim = len.P + i;
    const bool live = r < p.R && i < len.n;
    const size_t row = (static_cast<size_t>(b) * p.T + i) * p.Hq + g * p.G + (r - i * p.G);
    const int s_first = st0 + wave, last_tok = len.P + len.n - 1;
    struct Pages { int64_t at[2]; };
    auto pages_of = [&](int s) __attribute__((always_inline)) {        // offsets of the KV head in the step's two pages
        const int top = last_tok >> 4;
        const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_pages;
        Pages x;
#pragma unroll
        for (int j = 0; j < 2; ++j) x.at[j] = static_cast<int64_t>(scalar_load(table, 2 * s + j < top ? 2 * s + j : top)) * p.page_stride + g * p.head_stride;
        return x;
    };
    floatx4 key[DC];
    auto load_keys = [&](int s, const Pages& pg) __attribute__((always_inline)) {      // (tokens behind the last: the last one, which is not seen there)
        const int left = last_tok - s * PV_STEP, at = l32 < left ? l32 : left;
        const float* k = static_cast<const float*>(p.k) + (at >= 16 ? pg.at[1] : pg.at[0]) + (at & 15) * p.token_stride + 4 * half;
#pragma unroll
        for (int c = 0; c < DC; ++c) key[c] = *reinterpret_cast<const floatx4*>(k + 8 * c);
    };
    // Values through descriptors that end with the sequence's last token: zeros behind it, and one address register for all rows.
    float val[16][DE];
    const unsigned ts4 = static_cast<unsigned>(p.token_stride) * 4u, v_lane = 4u * half * ts4 + 4u * l32;
    auto load_values = [&](int s, const Pages& pg) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int rows = last_tok - s * PV_STEP - 16 * (j >> 3);
            const unsigned bytes = rows >= 0 ? static_cast<unsigned>(rows < 15 ? rows : 15) * ts4 + 4 * D : 0u;
            const auto from = merge_buffer(static_cast<const float*>(p.v) + pg.at[j >> 3], bytes);
#pragma unroll
            for (int e = 0; e < DE; ++e)
                val[j][e] = __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, static_cast<int>(v_lane + 128u * e), static_cast<int>((8u * ((j >> 2) & 1) + (j & 3)) * ts4), 0));
        }
    };
    floatx4 q[DC];
    floatx16 o[DE];
    float l = 0.f, negm = PV_FRESH;
#pragma unroll
    for (int e = 0; e < DE; ++e) o[e] = floatx16{};
    if (s_first < st1) {
        Pages pg = pages_of(s_first);
        load_keys(s_first, pg);
        const float* from = static_cast<const float*>(p.q) + row * D + 4 * half;
#pragma unroll
        for (int c = 0; c < DC; ++c) {
            q[c] = floatx4{0.f, 0.f, 0.f, 0.f};
            if (live) q[c] = __builtin_bit_cast(floatx4, *reinterpret_cast<const uintx4*>(from + 8 * c) ^ p.q_sign);
        }
        const float c = CAP ? 1.f : p.scale_log2e;
        const int low = len.P + t.i1 - p.window, high = len.P + t.i0 + 1;       // tokens behind `low` and in front of `high` are seen by all rows
        for (int s = s_first; s < st1; s += AT_WAVES) {
            load_values(s, pg);
            __builtin_amdgcn_sched_barrier(0);
            const int t0 = s * PV_STEP;
            const bool plain = t0 > low && t0 + PV_STEP <= high;
            floatx16 x = floatx16{};
#pragma unroll
            for (int d = 0; d < DC; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) x = __builtin_amdgcn_mfma_f32_32x32x2f32(key[d][j], q[d][j], x, 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (!plain) {
                bool odd = false;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
#pragma unroll
                    for (int e = 0; e < DE; ++e) odd |= pv_no_number(val[j][e]);
                }
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) != 0, 0)) {
                    // values that are not numbers: added to the rows that see them, zeros from here on (0 times them would reach the others)
                    float* const vs = rows[wave];
#pragma unroll
                    for (int j = 0; j < 16; ++j)
#pragma unroll
                        for (int e = 0; e < DE; ++e) {
                            const bool bad = pv_no_number(val[j][e]);
                            vs[(8 * (j >> 2) + 4 * half + (j & 3)) * D + 32 * e + l32] = bad ? val[j][e] : 0.f;
                            val[j][e] = bad ? 0.f : val[j][e];
                        }
                    wavefront_lds_order();
                    for (int tok = 0; tok < PV_STEP; ++tok) {
                        const bool sees = static_cast<unsigned>(lim - (t0 + tok)) < static_cast<unsigned>(p.window);
#pragma unroll
                        for (int e = 0; e < DE; ++e)
#pragma unroll
                            for (int x = 0; x < 16; ++x) {
                                const float y = vs[tok * D + 32 * e + 8 * (x >> 2) + 4 * half + (x & 3)];
                                o[e][x] += sees ? y : 0.f;
                            }
                    }
                    wavefront_lds_order();
                }
            }
            if constexpr (CAP) {
#pragma unroll
                for (int j = 0; j < 16; ++j) x[j] = capped_f32(x[j], p.cap_in, p.cap_log2e);
            }
            if (!plain) {
                const int rel = lim - t0 - 4 * half;
#pragma unroll
                for (int j = 0; j < 16; ++j) x[j] = static_cast<unsigned>(rel - (8 * (j >> 2) + (j & 3))) < static_cast<unsigned>(p.window) ? x[j] : -INFINITY;
            }
            float top = __builtin_fmaf(x[0], c, negm);
#pragma unroll
            for (int j = 1; j < 16; ++j) top = __builtin_fmaxf(top, __builtin_fmaf(x[j], c, negm));
            const bool rise = pv_max(top) > PV_RISE;
            if (__builtin_amdgcn_ballot_w64(rise) != 0) {
                float mm = x[0] * c;
#pragma unroll
                for (int j = 1; j < 16; ++j) mm = __builtin_fmaxf(mm, x[j] * c);
                // (a first reference scales nothing: rows have nothing yet, or what keeping apart has added)
                const float m = rise ? -pv_max(mm) : negm, f = rise && negm != PV_FRESH ? __builtin_amdgcn_exp2f(m - negm) : 1.f;
                negm = m;
                l *= f;
#pragma unroll
                for (int e = 0; e < DE; ++e)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[e][j] *= f;
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                x[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], c, negm));
                l += x[j];
            }
            __builtin_amdgcn_sched_barrier(0);
            if (s + AT_WAVES < st1) {
                pg = pages_of(s + AT_WAVES);
                load_keys(s + AT_WAVES, pg);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < 16; ++j)
#pragma unroll
                for (int e = 0; e < DE; ++e) o[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(val[j][e], x[j], o[e], 0, 0, 0);
        }
    }
    // ---- join: wavefront e finishes dims 32 e ..
    l = pv_sum(l);
    if (half == 0) stat[wave][l32] = float2{-negm, l};
#pragma unroll
    for (int e = 0; e < DE; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<floatx4*>(&rows[wave][(e * 4 + j) * 256 + lane * 4]) = floatx4{o[e][4 * j], o[e][4 * j + 1], o[e][4 * j + 2], o[e][4 * j + 3]};
    __syncthreads();
    if (wave >= DE || r >= p.R) return;
    float2 st[AT_WAVES];
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < AT_WAVES; ++w) {
        st[w] = stat[w][l32];
        m = __builtin_fmaxf(m, st[w].y != 0.f ? st[w].x : -INFINITY);
    }
    float f[AT_WAVES], total = 0.f;
#pragma unroll
    for (int w = 0; w < AT_WAVES; ++w) {
        f[w] = st[w].y != 0.f ? __builtin_amdgcn_exp2f(st[w].x - m) : 0.f;
        total += st[w].y * f[w];
    }
    const float inv = p.n_splits > 1 ? 1.f : live && total != 0.f ? 1.f / total : 0.f;
    const size_t part = (static_cast<size_t>(bg) * p.n_splits + split) * p.R + r;
    float* const to = (p.n_splits > 1 ? p.ws_o + part * D : static_cast<float*>(p.out) + row * D) + 32 * wave + 4 * half;
    if (p.n_splits > 1 && !live) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < AT_WAVES; ++w) {
            const floatx4 y = *reinterpret_cast<const floatx4*>(&rows[w][(wave * 4 + j) * 256 + lane * 4]);
#pragma unroll
            for (int z = 0; z < 4; ++z) sum[z] += st[w].y != 0.f ? y[z] * f[w] : 0.f;
        }
        for (int z = 0; z < 4; ++z) sum[z] = live ? sum[z] * inv : 0.f;
        *reinterpret_cast<floatx4*>(to + 8 * j) = sum;
    }
    if (p.n_splits > 1 && half == 0 && wave == 0) *reinterpret_cast<float2*>(p.ws_ml + 2 * part) = float2{m, total};
}

int32_t launch_prompt_few_f32(const PromptParams& p, int32_t D, bool cap, hipStream_t s) {
    const dim3 grid(prompt_grid(p));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(AT_THREADS), 0, s, p.n_nodes, p.prefix_len, p); };
    if (D == 128) { if (cap) launch(prompt_few_f32_kernel<128, true>); else launch(prompt_few_f32_kernel<128, false>); }
    else if (cap) launch(prompt_few_f32_kernel<64, true>);
    else launch(prompt_few_f32_kernel<64, false>);
    return check_launch();
}

}  // namespace graft
