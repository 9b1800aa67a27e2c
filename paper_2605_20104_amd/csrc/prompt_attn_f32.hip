// graft_prompt_attn, fp32: storage, products, softmax and sums.
//
// Four wavefronts with 32 rows each share stages of 32 tokens in an LDS ring of two; two workgroups a compute unit, so that one
// multiplies while the other takes exponentials.  Products are v_mfma_f32_32x32x2: S^T = K Q^T in any order of the dims, so a
// lane reads 16 bytes of a key (dims 8 c + 4 half + 0..3) for four of them; lane (half, l32) of the result has row l32 and the tokens
// 8 (v / 4) + 4 half + v % 4, and register v is the B operand of the second product as it lies, with value rows of those two tokens.
// Bound by the matrix cores: 128 MFMAs of 64 cycles for 32 x 32 scores with D = 128, 0.5 K cycles of other instructions beside them.
// They are busy in 89 % of the cycles; 41 GFLOP in 357 us with the merge of 16 us (115 TFLOP/s; a library product of 8192^3 reaches 153).
#include "prompt_attn.h"

namespace graft {

constexpr int PF_STAGE = 32, PF_NBUF = 2;
constexpr float PF_RISE = 8.f, PF_FRESH = 3e38f;      // as in the bf16 kernel

__device__ __forceinline__ float pf_sum(float v) {
    const unsigned u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float pf_max(float v) {
    const unsigned u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ bool no_number(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

template <int D, bool CAP>
__global__ __launch_bounds__(AT_THREADS, 2) void prompt_attn_f32_kernel(const int32_t* n_nodes, const int32_t* prefix_len, PromptParams p) {
    constexpr int RB = 4 * D, DE = D / 32, DC = D / 8, TILE_ROWS = 128, HALF_BYTES = PF_STAGE * RB, STAGE_BYTES = 2 * HALF_BYTES;
    constexpr int LANES = RB / 16, ROWS = 64 / LANES, LOADS = 16 / ROWS;      // lanes a row, rows an instruction, instructions a page
    __shared__ __attribute__((aligned(1024))) unsigned char kv[PF_NBUF][STAGE_BYTES];
    __shared__ int32_t vote[AT_WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const PromptItem item = prompt_item(p);
    if (item.unit < 0) return;
    const int bg = item.unit / p.n_splits, split = item.unit - bg * p.n_splits, b = bg / p.Hkv, g = bg - b * p.Hkv;
    const PromptLengths len = prompt_lengths(p, scalar_load(prefix_len, b), scalar_load(n_nodes, b));
    const int r_tile = item.row_tile * TILE_ROWS;
    const PromptRange t = prompt_range<PF_STAGE>(p, len, r_tile, TILE_ROWS);
    const int spt = (t.st1 - t.st0 + p.n_splits - 1) / p.n_splits, st0 = t.st0 + split * spt, st1 = st0 + spt < t.st1 ? st0 + spt : t.st1;
    const int n_st = st1 - st0;
    const unsigned kv_base = __builtin_amdgcn_readfirstlane(lds_address(&kv[0][0]));

    const int r = r_tile + wave * 32 + l32, i = div_any(r, p.g_magic, p.g_shift), lim = len.P + i;
    const bool live = r < p.R && i < len.n;
    const size_t row = (static_cast<size_t>(b) * p.T + i) * p.Hq + g * p.G + (r - i * p.G);
    floatx4 q[DC];
    {
        const float* from = static_cast<const float*>(p.q) + row * D + 4 * half;
#pragma unroll
        for (int c = 0; c < DC; ++c) {
            q[c] = floatx4{0.f, 0.f, 0.f, 0.f};
            if (live) q[c] = __builtin_bit_cast(floatx4, *reinterpret_cast<const uintx4*>(from + 8 * c) ^ p.q_sign);
        }
    }
    floatx16 o[DE];
#pragma unroll
    for (int e = 0; e < DE; ++e) o[e] = floatx16{};
    float l = 0.f, negm = PF_FRESH;
    if (n_st > 0) {
        const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_pages;
        const int last_tok = len.P + len.n - 1, last_pg = last_tok >> 4;
        const unsigned ts4 = static_cast<unsigned>(p.token_stride) * 4u;
        const int kind = wave & 1, my_page = wave >> 1, lr = lane / LANES, lc = lane % LANES;       // keys or values of one of the stage's two pages
        const u64 head = reinterpret_cast<u64>(kind ? p.v : p.k) + static_cast<u64>(g * p.head_stride) * 4;
        auto move_page = [&](int k) __attribute__((always_inline)) {
            const int pg = (st0 + k) * 2 + my_page, rows = last_tok - pg * GRAFT_PAGE_SIZE;         // the last token's row in the page
            const unsigned bytes = rows >= 0 && k < n_st ? static_cast<unsigned>(rows < 15 ? rows : 15) * ts4 + RB : 0u;
            const u64 at = head + static_cast<u64>(static_cast<unsigned>(scalar_load(table, pg < last_pg ? pg : last_pg))) * static_cast<u64>(p.page_stride * 4);
            const uintx4 d = {static_cast<unsigned>(at), static_cast<unsigned>(at >> 32), bytes, BUFFER_WORD3};
            const unsigned lds = kv_base + (k & 1) * STAGE_BYTES + kind * HALF_BYTES + my_page * (16 * RB);
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int rr = ROWS * j + lr;
                // keys: 16-byte chunk c of row r at c ^ (r & 15); values: 128-byte segment at s ^ (r / 4) % 2
                const int chunk = kind ? lc ^ (((rr >> 2) & 1) << 3) : lc ^ (rr & 15);
                buffer_to_lds_b128(d, static_cast<unsigned>(rr) * ts4 + chunk * 16, lds + j * 1024);
            }
        };
        move_page(0);
        const float c = CAP ? 1.f : p.scale_log2e;
        const int low = len.P + t.i1 - p.window, high = len.P + t.i0 + 1;       // tokens behind `low` and in front of `high` are seen by all rows
        for (int k = 0; k < n_st; ++k) {
            GRAFT_WAIT_VMCNT(0);
            lds_barrier();                       // stage k is there; nobody reads stage k - 1 any more
            if (k + 1 < n_st) move_page(k + 1);
            const int t0 = (st0 + k) * PF_STAGE;
            const bool plain = t0 > low && t0 + PF_STAGE <= high;
            unsigned char* const ks = &kv[k & 1][0];
            unsigned char* const vs = ks + HALF_BYTES;
            if (!plain) {
                // values that are not numbers: added to the rows that see them, zeros from here on (0 times them would reach the others)
                bool odd = false;
                for (int x = tid; x < HALF_BYTES / 16; x += AT_THREADS) {
                    const floatx4 y = reinterpret_cast<const floatx4*>(vs)[x];
#pragma unroll
                    for (int j = 0; j < 4; ++j) odd |= no_number(y[j]);
                }
                if (__builtin_amdgcn_ballot_w64(odd) != 0) odd = true;
                if (lane == 0) vote[wave] = odd;
                lds_barrier();
                if (__builtin_expect((vote[0] | vote[1] | vote[2] | vote[3]) != 0, 0)) {
                    for (int tok = 0; tok < PF_STAGE; ++tok) {
                        const bool sees = static_cast<unsigned>(lim - (t0 + tok)) < static_cast<unsigned>(p.window);
#pragma unroll
                        for (int e = 0; e < DE; ++e)
#pragma unroll
                            for (int x = 0; x < 16; ++x) {
                                const float y = *reinterpret_cast<const float*>(vs + tok * RB + ((e ^ ((tok >> 2) & 1)) << 7) + 4 * (8 * (x >> 2) + 4 * half + (x & 3)));
                                o[e][x] += sees && no_number(y) ? y : 0.f;
                            }
                    }
                    lds_barrier();
                    for (int x = tid; x < HALF_BYTES / 4; x += AT_THREADS) {
                        float* const y = reinterpret_cast<float*>(vs) + x;
                        if (no_number(*y)) *y = 0.f;
                    }
                    lds_barrier();
                }
            }
            floatx16 s = floatx16{};
#pragma unroll
            for (int d = 0; d < DC; ++d) {
                const floatx4 key = *reinterpret_cast<const floatx4*>(ks + l32 * RB + (((2 * d + half) ^ (l32 & 15)) << 4));
#pragma unroll
                for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(key[j], q[d][j], s, 0, 0, 0);
            }
            if constexpr (CAP) {
#pragma unroll
                for (int x = 0; x < 16; ++x) s[x] = capped_f32(s[x], p.cap_in, p.cap_log2e);
            }
            if (!plain) {
                const int rel = lim - t0 - 4 * half;
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    s[x] = static_cast<unsigned>(rel - (8 * (x >> 2) + (x & 3))) < static_cast<unsigned>(p.window) ? s[x] : -INFINITY;
            }
            float top = __builtin_fmaf(s[0], c, negm);
#pragma unroll
            for (int x = 1; x < 16; ++x) top = __builtin_fmaxf(top, __builtin_fmaf(s[x], c, negm));
            const bool rise = pf_max(top) > PF_RISE;
            if (__builtin_amdgcn_ballot_w64(rise) != 0) {
                float mm = s[0] * c;
#pragma unroll
                for (int x = 1; x < 16; ++x) mm = __builtin_fmaxf(mm, s[x] * c);
                // (a first reference scales nothing: rows have nothing yet, or what keeping apart has added)
                const float now = rise ? -pf_max(mm) : negm, f = rise && negm != PF_FRESH ? __builtin_amdgcn_exp2f(now - negm) : 1.f;
                negm = now;
                l *= f;
#pragma unroll
                for (int e = 0; e < DE; ++e)
#pragma unroll
                    for (int x = 0; x < 16; ++x) o[e][x] *= f;
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                s[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x], c, negm));
                l += s[x];
            }
#pragma unroll
            for (int x = 0; x < 16; ++x)
#pragma unroll
                for (int e = 0; e < DE; ++e) {
                    const int tok = 8 * (x >> 2) + 4 * half + (x & 3);
                    o[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(vs + tok * RB + ((e ^ half) << 7) + 4 * l32), s[x], o[e], 0, 0, 0);
                }
        }
    }
    l = pf_sum(l);
    if (r >= p.R) return;
    if (p.n_splits == 1) {
        const float inv = live && l != 0.f ? 1.f / l : 0.f;
        float* out = static_cast<float*>(p.out) + row * D + 4 * half;
#pragma unroll
        for (int e = 0; e < DE; ++e)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                floatx4 x = {o[e][4 * j] * inv, o[e][4 * j + 1] * inv, o[e][4 * j + 2] * inv, o[e][4 * j + 3] * inv};
                if (!live) x = floatx4{0.f, 0.f, 0.f, 0.f};
                *reinterpret_cast<floatx4*>(out + 32 * e + 8 * j) = x;
            }
    } else if (live) {
        const size_t part = (static_cast<size_t>(bg) * p.n_splits + split) * p.R + r;
        float* to = p.ws_o + part * D + 4 * half;
#pragma unroll
        for (int e = 0; e < DE; ++e)
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<floatx4*>(to + 32 * e + 8 * j) = floatx4{o[e][4 * j], o[e][4 * j + 1], o[e][4 * j + 2], o[e][4 * j + 3]};
        if (half == 0) *reinterpret_cast<float2*>(p.ws_ml + 2 * part) = float2{-negm, l};
    }
}

int32_t launch_prompt_f32(const PromptParams& p, int32_t D, bool cap, hipStream_t s) {
    const dim3 grid(prompt_grid(p));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(AT_THREADS), 0, s, p.n_nodes, p.prefix_len, p); };
    if (D == 128) { if (cap) launch(prompt_attn_f32_kernel<128, true>); else launch(prompt_attn_f32_kernel<128, false>); }
    else if (cap) launch(prompt_attn_f32_kernel<64, true>);
    else launch(prompt_attn_f32_kernel<64, false>);
    return check_launch();
}

}  // namespace graft
