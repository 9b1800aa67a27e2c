// graft_prompt_attn, fp32, few rows (up to 32 of a KV head: single tokens, short pieces): the wavefronts take 32 tokens each in turn and join
// their rows through LDS at the end, as in prompt_attn_few.hip; products as in prompt_attn_f32.hip.
// With up to 16 rows (single tokens always) tiles of 16 x 16 and v_mfma_f32_16x16x4: half the matrix cycles and half the registers.
//
// Keys and values go from memory to registers as the products want them, values during the first product of their step, the next
// step's keys during the second: of G = 2 or 4 groups of lanes, lane (group, lr) reads dims 4 G c + 4 group + 0..3 of key lr, and
// dim ROWS e + lr of the values of tokens 4 G (x / 4) + 4 group + x % 4.
//
// Bound by memory where there is much of it, else by the way through a wavefront's steps.  16 rows against 32 for the same calls, us in a graph: one
// token behind 255, 2 KV heads, D = 64: 7.5, 10.5; 32 sequences' tokens behind 2000, 8 KV heads, D = 64: 43, 50 (6.1 TB/s); one behind 65536,
// D = 128: 101, 121; 8 behind 16000: 187, 211.  Two workgroups a compute unit: 32 tokens behind 4096 in three splits 195, one 203.  Eight
// wavefronts a workgroup with 32 rows, D = 64: 11.5 for 10.6 behind 255.
#include <type_traits>

#include "prompt_attn.h"

namespace graft {

constexpr int PV_STEP = 32;
constexpr float PV_RISE = 8.f, PV_FRESH = 3e38f;      // as in prompt_attn_bf16.hip

// Over the lanes of a row (ROWS apart).
template <int ROWS, class F> __device__ __forceinline__ float pv_fold(float v, F&& f) {
    unsigned u = __float_as_uint(v);
    if constexpr (ROWS == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        u = __float_as_uint(f(__uint_as_float(r[0]), __uint_as_float(r[1])));
    }
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int ROWS> __device__ __forceinline__ float pv_sum(float v) { return pv_fold<ROWS>(v, [](float a, float b) { return a + b; }); }
template <int ROWS> __device__ __forceinline__ float pv_max(float v) { return pv_fold<ROWS>(v, [](float a, float b) { return __builtin_fmaxf(a, b); }); }
__device__ __forceinline__ floatx16 pv_mfma(float a, float b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
__device__ __forceinline__ floatx4 pv_mfma(float a, float b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
__device__ __forceinline__ bool pv_no_number(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

template <int D, int ROWS, bool CAP>
__global__ __launch_bounds__(AT_THREADS, ROWS == 16 ? 2 : 1) void prompt_few_f32_kernel(const int32_t* n_nodes, const int32_t* prefix_len, PromptParams p) {
    // lane: row (or token, or dim) lr of ROWS, one of GROUPS groups; element y of a tile of ROWS x ROWS is 4 GROUPS (y / 4) + 4 group + y % 4
    using Tile = std::conditional_t<ROWS == 32, floatx16, floatx4>;
    constexpr int DE = D / ROWS, GROUPS = 64 / ROWS, NE = ROWS / GROUPS, TB = PV_STEP / ROWS, DC = D / (4 * GROUPS), NV = TB * NE;
    __shared__ __attribute__((aligned(16))) float rows[AT_WAVES][PV_STEP * D];     // values that are no numbers, then what is joined
    __shared__ float2 stat[AT_WAVES][ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane % ROWS, group = lane / ROWS;
    const PromptItem item = prompt_item(p);
    if (item.unit < 0) return;
    const int bg = item.unit / p.n_splits, split = item.unit - bg * p.n_splits, b = bg / p.Hkv, g = bg - b * p.Hkv;
    const PromptLengths len = prompt_lengths(p, scalar_load(prefix_len, b), scalar_load(n_nodes, b));
    const int r_tile = item.row_tile * ROWS;
    const PromptRange t = prompt_range<PV_STEP>(p, len, r_tile, ROWS);
    const int spt = (t.st1 - t.st0 + p.n_splits - 1) / p.n_splits, st0 = t.st0 + split * spt, st1 = st0 + spt < t.st1 ? st0 + spt : t.st1;

    const int r = r_tile + lr, i = div_any(r, p.g_magic, p.g_shift), lim = len.P + i;
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
    floatx4 key[TB][DC];
    auto load_keys = [&](int s, const Pages& pg) __attribute__((always_inline)) {      // (tokens behind the last: the last one, which is not seen there)
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) {
            const int left = last_tok - s * PV_STEP, at = ROWS * tb + lr < left ? ROWS * tb + lr : left;
            const float* k = static_cast<const float*>(p.k) + (at >= 16 ? pg.at[1] : pg.at[0]) + (at & 15) * p.token_stride + 4 * group;
#pragma unroll
            for (int c = 0; c < DC; ++c) key[tb][c] = *reinterpret_cast<const floatx4*>(k + 4 * GROUPS * c);
        }
    };
    // Values through descriptors that end with the sequence's last token: zeros behind it, and one address register for all rows.
    float val[NV][DE];
    const unsigned ts4 = static_cast<unsigned>(p.token_stride) * 4u, v_lane = 4u * group * ts4 + 4u * lr;
    auto load_values = [&](int s, const Pages& pg) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int at = 4 * GROUPS * (j >> 2) + (j & 3), rows = last_tok - s * PV_STEP - (at & ~15);
            const unsigned bytes = rows >= 0 ? static_cast<unsigned>(rows < 15 ? rows : 15) * ts4 + 4 * D : 0u;
            const auto from = merge_buffer(static_cast<const float*>(p.v) + pg.at[at >> 4], bytes);
#pragma unroll
            for (int e = 0; e < DE; ++e)
                val[j][e] = __int_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, static_cast<int>(v_lane + 4u * ROWS * e), static_cast<int>((at & 15) * ts4), 0));
        }
    };
    floatx4 q[DC];
    Tile o[DE];
    float l = 0.f, negm = PV_FRESH;
#pragma unroll
    for (int e = 0; e < DE; ++e) o[e] = Tile{};
    if (s_first < st1) {
        Pages pg = pages_of(s_first);
        load_keys(s_first, pg);
        const float* from = static_cast<const float*>(p.q) + row * D + 4 * group;
#pragma unroll
        for (int c = 0; c < DC; ++c) {
            q[c] = floatx4{0.f, 0.f, 0.f, 0.f};
            if (live) q[c] = __builtin_bit_cast(floatx4, *reinterpret_cast<const uintx4*>(from + 4 * GROUPS * c) ^ p.q_sign);
        }
        const float c = CAP ? 1.f : p.scale_log2e;
        const int low = len.P + t.i1 - p.window, high = len.P + t.i0 + 1;       // tokens behind `low` and in front of `high` are seen by all rows
        for (int s = s_first; s < st1; s += AT_WAVES) {
            load_values(s, pg);
            __builtin_amdgcn_sched_barrier(0);
            const int t0 = s * PV_STEP;
            const bool plain = t0 > low && t0 + PV_STEP <= high;
            float x[NV];
            {
                Tile scores[TB];
#pragma unroll
                for (int tb = 0; tb < TB; ++tb) scores[tb] = Tile{};
#pragma unroll
                for (int d = 0; d < DC; ++d)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int tb = 0; tb < TB; ++tb) scores[tb] = pv_mfma(key[tb][d][j], q[d][j], scores[tb]);
#pragma unroll
                for (int j = 0; j < NV; ++j) x[j] = scores[j / NE][j % NE];
            }
            __builtin_amdgcn_sched_barrier(0);
            if (!plain) {
                bool odd = false;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
#pragma unroll
                    for (int e = 0; e < DE; ++e) odd |= pv_no_number(val[j][e]);
                }
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) != 0, 0)) {
                    // values that are not numbers: added to the rows that see them, zeros from here on (0 times them would reach the others)
                    float* const vs = rows[wave];
#pragma unroll
                    for (int j = 0; j < NV; ++j)
#pragma unroll
                        for (int e = 0; e < DE; ++e) {
                            const bool bad = pv_no_number(val[j][e]);
                            vs[(4 * GROUPS * (j >> 2) + 4 * group + (j & 3)) * D + ROWS * e + lr] = bad ? val[j][e] : 0.f;
                            val[j][e] = bad ? 0.f : val[j][e];
                        }
                    wavefront_lds_order();
                    for (int tok = 0; tok < PV_STEP; ++tok) {
                        const bool sees = static_cast<unsigned>(lim - (t0 + tok)) < static_cast<unsigned>(p.window);
#pragma unroll
                        for (int e = 0; e < DE; ++e)
#pragma unroll
                            for (int z = 0; z < NE; ++z) {
                                const float y = vs[tok * D + ROWS * e + 4 * GROUPS * (z >> 2) + 4 * group + (z & 3)];
                                o[e][z] += sees ? y : 0.f;
                            }
                    }
                    wavefront_lds_order();
                }
            }
            if constexpr (CAP) {
#pragma unroll
                for (int j = 0; j < NV; ++j) x[j] = capped_f32(x[j], p.cap_in, p.cap_log2e);
            }
            if (!plain) {
                const int rel = lim - t0 - 4 * group;
#pragma unroll
                for (int j = 0; j < NV; ++j) x[j] = static_cast<unsigned>(rel - (4 * GROUPS * (j >> 2) + (j & 3))) < static_cast<unsigned>(p.window) ? x[j] : -INFINITY;
            }
            float top = __builtin_fmaf(x[0], c, negm);
#pragma unroll
            for (int j = 1; j < NV; ++j) top = __builtin_fmaxf(top, __builtin_fmaf(x[j], c, negm));
            const bool rise = pv_max<ROWS>(top) > PV_RISE;
            if (__builtin_amdgcn_ballot_w64(rise) != 0) {
                float mm = x[0] * c;
#pragma unroll
                for (int j = 1; j < NV; ++j) mm = __builtin_fmaxf(mm, x[j] * c);
                // (a first reference scales nothing: rows have nothing yet, or what keeping apart has added)
                const float m = rise ? -pv_max<ROWS>(mm) : negm, f = rise && negm != PV_FRESH ? __builtin_amdgcn_exp2f(m - negm) : 1.f;
                negm = m;
                l *= f;
#pragma unroll
                for (int e = 0; e < DE; ++e)
#pragma unroll
                    for (int j = 0; j < NE; ++j) o[e][j] *= f;
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
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
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < DE; ++e) o[e] = pv_mfma(val[j][e], x[j], o[e]);
        }
    }
    // ---- join: each wavefront its dims, ROWS at a time
    l = pv_sum<ROWS>(l);
    if (group == 0) stat[wave][lr] = float2{-negm, l};
#pragma unroll
    for (int e = 0; e < DE; ++e)
#pragma unroll
        for (int j = 0; j < NE / 4; ++j)
            *reinterpret_cast<floatx4*>(&rows[wave][(e * (NE / 4) + j) * 256 + lane * 4]) = floatx4{o[e][4 * j], o[e][4 * j + 1], o[e][4 * j + 2], o[e][4 * j + 3]};
    __syncthreads();
    if (wave >= DE || r >= p.R) return;
    float2 st[AT_WAVES];
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < AT_WAVES; ++w) {
        st[w] = stat[w][lr];
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
    float* const to = (p.n_splits > 1 ? p.ws_o + part * D : static_cast<float*>(p.out) + row * D) + 4 * group;
    if (p.n_splits > 1 && !live) return;
    for (int e = wave; e < DE; e += AT_WAVES)
#pragma unroll
        for (int j = 0; j < NE / 4; ++j) {
            floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < AT_WAVES; ++w) {
                const floatx4 y = *reinterpret_cast<const floatx4*>(&rows[w][(e * (NE / 4) + j) * 256 + lane * 4]);
#pragma unroll
                for (int z = 0; z < 4; ++z) sum[z] += st[w].y != 0.f ? y[z] * f[w] : 0.f;
            }
            for (int z = 0; z < 4; ++z) sum[z] = live ? sum[z] * inv : 0.f;
            *reinterpret_cast<floatx4*>(to + ROWS * e + 4 * GROUPS * j) = sum;
        }
    if (p.n_splits > 1 && group == 0 && wave == 0) *reinterpret_cast<float2*>(p.ws_ml + 2 * part) = float2{m, total};
}

int32_t launch_prompt_few_f32(const PromptParams& p, int32_t D, bool cap, int32_t tile_rows, hipStream_t s) {
    const dim3 grid(prompt_grid(p));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(AT_THREADS), 0, s, p.n_nodes, p.prefix_len, p); };
    auto pick = [&](auto d, auto rows) {
        if (cap) launch(prompt_few_f32_kernel<d, rows, true>);
        else launch(prompt_few_f32_kernel<d, rows, false>);
    };
    using std::integral_constant;
    using Half = integral_constant<int, PA_FEW_ROWS / 2>;
    using Whole = integral_constant<int, PA_FEW_ROWS>;
    if (D == 128) { if (tile_rows < PA_FEW_ROWS) pick(integral_constant<int, 128>{}, Half{}); else pick(integral_constant<int, 128>{}, Whole{}); }
    else if (tile_rows < PA_FEW_ROWS) pick(integral_constant<int, 64>{}, Half{});
    else pick(integral_constant<int, 64>{}, Whole{});
    return check_launch();
}

}  // namespace graft
