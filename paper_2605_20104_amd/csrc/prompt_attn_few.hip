// graft_prompt_attn, bf16, few rows (tiles of 32 or 64 rows of a KV head: single tokens, short pieces): bound by the way of keys and values from
// memory.
//
// All of a sequence and KV head's rows are one tile, NB blocks of 32 rows that every wavefront has; the wavefronts take 32 tokens each in
// turn, from memory straight to two LDS buffers of their own (no barrier in the loop), and join their rows through LDS at the
// end.  Products, masks and softmax as in prompt_attn_bf16.hip, one step after the other: 16 NB MFMAs and some 250 NB other
// instructions for the 16 KB (D = 128) that a wavefront waits for.  32 ragged sequences' tokens behind up to 16384 (1.63 GB): 290 us, 5.6 TB/s.
#include "prompt_attn.h"

namespace graft {

constexpr int PW_STEP = 32;                      // tokens of a wavefront's step
constexpr float PW_RISE = 8.f, PW_FRESH = 3e38f;      // as in prompt_attn_bf16.hip

template <int D> __device__ __forceinline__ int pw_key_swizzle(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
template <int D> __device__ __forceinline__ int pw_value_swizzle(int r) { return D == 128 ? (r & 3) << 1 : ((r >> 1) & 1) << 1; }
__device__ __forceinline__ float pw_sum(float v) {
    const unsigned u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float pw_max(float v) {
    const unsigned u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int D, int NB, bool CAP>
__global__ __launch_bounds__(AT_THREADS, 1) void prompt_few_kernel(const int32_t* n_nodes, const int32_t* prefix_len, PromptParams p) {
    constexpr int RB = 2 * D, DK = D / 16, DE = D / 32, HALF_BYTES = PW_STEP * RB, STEP_BYTES = 2 * HALF_BYTES, LOADS = STEP_BYTES / 1024;
    constexpr int LANES = RB / 16, ROWS = 64 / LANES;              // lanes a row, rows an instruction
    __shared__ __attribute__((aligned(1024))) unsigned char kv[AT_WAVES][2][STEP_BYTES];
    __shared__ float2 stat[AT_WAVES][NB * 32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, l32 = lane & 31, half = lane >> 5;
    const PromptItem item = prompt_item(p);
    if (item.unit < 0) return;
    const int bg = item.unit / p.n_splits, split = item.unit - bg * p.n_splits, b = bg / p.Hkv, g = bg - b * p.Hkv;
    const PromptLengths len = prompt_lengths(p, scalar_load(prefix_len, b), scalar_load(n_nodes, b));
    const int r_tile = item.row_tile * (NB * 32);
    const PromptRange t = prompt_range<PW_STEP>(p, len, r_tile, NB * 32);
    const int spt = (t.st1 - t.st0 + p.n_splits - 1) / p.n_splits, st0 = t.st0 + split * spt, st1 = st0 + spt < t.st1 ? st0 + spt : t.st1;
    const unsigned base = __builtin_amdgcn_readfirstlane(lds_address(&kv[wave][0][0]));

    floatx16 o[NB][DE];
    float l[NB], negm[NB];
    int lim[NB];
    bool live[NB];
    bf16x8 q[NB][DK];
#pragma unroll
    for (int rb = 0; rb < NB; ++rb) {
        const int r = r_tile + rb * 32 + l32, i = div_any(r, p.g_magic, p.g_shift);
        live[rb] = r < p.R && i < len.n;
        lim[rb] = len.P + i;
        l[rb] = 0.f;
        negm[rb] = PW_FRESH;
        const unsigned short* from = static_cast<const unsigned short*>(p.q) + ((static_cast<int64_t>(b) * p.T + i) * p.Hq + g * p.G + (r - i * p.G)) * D + 8 * half;
#pragma unroll
        for (int d = 0; d < DK; ++d) {
            uintx4 x = {0u, 0u, 0u, 0u};
            if (live[rb]) x = *reinterpret_cast<const uintx4*>(from + 16 * d) ^ p.q_sign;
            q[rb][d] = __builtin_bit_cast(bf16x8, x);
        }
#pragma unroll
        for (int e = 0; e < DE; ++e) o[rb][e] = floatx16{};
    }
    if (st0 < st1) {
        const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_pages;
        const int last_tok = len.P + len.n - 1, last_pg = last_tok >> 4;
        const unsigned ts2 = static_cast<unsigned>(p.token_stride) * 2u;
        const int lr = lane / LANES, lc = lane % LANES;
        const u64 k_head = reinterpret_cast<u64>(p.k) + static_cast<u64>(g * p.head_stride) * 2, v_head = reinterpret_cast<u64>(p.v) + static_cast<u64>(g * p.head_stride) * 2;
        // step s of this wavefront (tokens 32 s ..), through buffer descriptors that end with the sequence's last token: zeros behind it
        auto load_pages = [&](int s0) __attribute__((always_inline)) {        // lane 2 i + j: page j of step s0 + AT_WAVES i
            const int pg = 2 * (s0 + AT_WAVES * (lane >> 1)) + (lane & 1);
            int32_t x = table[pg < last_pg ? pg : last_pg];
            asm volatile("" : "+v"(x));
            return x;
        };
        auto move = [&](int s, int pages, int at, int buffer) __attribute__((always_inline)) {
#pragma unroll
            for (int pg = 0; pg < 2; ++pg) {
                const u64 off = static_cast<u64>(static_cast<unsigned>(__builtin_amdgcn_readlane(pages, 2 * at + pg))) * static_cast<u64>(p.page_stride * 2);
                const int rows = last_tok - s * PW_STEP - 16 * pg;
                const unsigned bytes = rows >= 0 ? static_cast<unsigned>(rows < 15 ? rows : 15) * ts2 + RB : 0u;
                const u64 ka = k_head + off, va = v_head + off;
                const uintx4 dk = {static_cast<unsigned>(ka), static_cast<unsigned>(ka >> 32), bytes, BUFFER_WORD3}, dv = {static_cast<unsigned>(va), static_cast<unsigned>(va >> 32), bytes, BUFFER_WORD3};
                const unsigned lds = base + buffer * STEP_BYTES + pg * (16 * RB);
#pragma unroll
                for (int j = 0; j < 16 / ROWS; ++j) {
                    const int r = ROWS * j + lr;
                    buffer_to_lds_b128(dk, static_cast<unsigned>(r) * ts2 + (lc ^ pw_key_swizzle<D>(r)) * 16, lds + j * 1024);
                    buffer_to_lds_b128(dv, static_cast<unsigned>(r) * ts2 + ((((lc >> 1) ^ pw_value_swizzle<D>(r)) << 1) | (lc & 1)) * 16, lds + HALF_BYTES + j * 1024);
                }
            }
        };
        const int s_first = st0 + wave;
        int32_t pages = s_first < st1 ? load_pages(s_first) : 0;
        if (s_first < st1) move(s_first, pages, 0, 0);
        const float c = CAP ? 1.f : p.scale_log2e;
        const unsigned k_lane = l32 * RB + ((half ^ pw_key_swizzle<D>(l32)) << 4);
        const int v_row = 4 * half + (l16 >> 2);
        const unsigned v_lane = HALF_BYTES + v_row * RB + (((l32 >> 4) ^ pw_value_swizzle<D>(v_row)) << 5) + 8 * (l16 & 3);
        const int low = len.P + t.i1 - p.window, high = len.P + t.i0 + 1;       // tokens behind `low` and in front of `high` are seen by all rows
        int k = 0;
        for (int s = s_first; s < st1; s += AT_WAVES, ++k) {
            const unsigned at = base + (k & 1) * STEP_BYTES;
            if (s + AT_WAVES < st1) {
                if (((k + 1) & 31) == 0) pages = load_pages(s + AT_WAVES);
                move(s + AT_WAVES, pages, (k + 1) & 31, (k + 1) & 1);
                GRAFT_WAIT_VMCNT(LOADS);
            } else GRAFT_WAIT_VMCNT(0);
            asm volatile("" ::: "memory");
            const int t0 = s * PW_STEP;
            const bool plain = t0 > low && t0 + PW_STEP <= high;
            unsigned char* const vs = &kv[wave][k & 1][HALF_BYTES];
            if (!plain) {
                // values that are not numbers: added to the rows that see them, zeros from here on (0 times them would reach the others)
                bool odd = false;
#pragma unroll
                for (int x = 0; x < HALF_BYTES / 1024; ++x) {
                    const uintx4 y = reinterpret_cast<const uintx4*>(vs)[x * 64 + lane];
#pragma unroll
                    for (int j = 0; j < 4; ++j) odd |= (y[j] & 0x7f80u) == 0x7f80u || (y[j] & 0x7f800000u) == 0x7f800000u;
                }
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) != 0, 0)) {
                    for (int tok = 0; tok < PW_STEP; ++tok)
#pragma unroll
                        for (int rb = 0; rb < NB; ++rb) {
                            const bool sees = static_cast<unsigned>(lim[rb] - (t0 + tok)) < static_cast<unsigned>(p.window);
#pragma unroll
                            for (int e = 0; e < DE; ++e)
#pragma unroll
                                for (int x = 0; x < 16; ++x) {
                                    const int dim = 32 * e + 8 * (x >> 2) + 4 * half + (x & 3);
                                    const unsigned short bits = *reinterpret_cast<const unsigned short*>(vs + tok * RB + (((dim >> 4) ^ pw_value_swizzle<D>(tok)) << 5) + 2 * (dim & 15));
                                    o[rb][e][x] += sees && (bits & 0x7f80) == 0x7f80 ? __uint_as_float(static_cast<unsigned>(bits) << 16) : 0.f;
                                }
                        }
                    wavefront_lds_order();
#pragma unroll
                    for (int x = 0; x < HALF_BYTES / 1024; ++x) {
                        uintx4* const y = reinterpret_cast<uintx4*>(vs) + x * 64 + lane;
                        uintx4 z = *y;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if ((z[j] & 0x7f80u) == 0x7f80u) z[j] &= 0xffff0000u;
                            if ((z[j] & 0x7f800000u) == 0x7f800000u) z[j] &= 0xffffu;
                        }
                        *y = z;
                    }
                    wavefront_lds_order();
                }
            }
            bf16x8 key[DK], val[DK];
#pragma unroll
            for (int d = 0; d < DK; ++d) key[d] = *reinterpret_cast<const bf16x8 __attribute__((address_space(3)))*>(static_cast<size_t>((at + k_lane) ^ (static_cast<unsigned>(d) << 5)));
#pragma unroll
            for (int n = 0; n < DK; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const short4_t r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4_t __attribute__((address_space(3)))*)(static_cast<size_t>(
                        ((at + v_lane) ^ (static_cast<unsigned>(n % DE) << 6)) + (16 * (n / DE) + 8 * h) * RB)));
                    const bf16x4 r4 = __builtin_bit_cast(bf16x4, r);
#pragma unroll
                    for (int j = 0; j < 4; ++j) val[n][4 * h + j] = r4[j];
                }
#pragma unroll
            for (int rb = 0; rb < NB; ++rb) {
                floatx16 x = floatx16{};
#pragma unroll
                for (int d = 0; d < DK; ++d) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key[d], q[rb][d], x, 0, 0, 0);
                if constexpr (CAP) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[j] = capped(x[j], p.cap_in, p.cap_log2e);
                }
                if (!plain) {
                    const int rel = lim[rb] - t0 - 4 * half;
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        x[j] = static_cast<unsigned>(rel - (8 * (j >> 2) + (j & 3))) < static_cast<unsigned>(p.window) ? x[j] : -INFINITY;
                }
                float top = __builtin_fmaf(x[0], c, negm[rb]);
#pragma unroll
                for (int j = 1; j < 16; ++j) top = __builtin_fmaxf(top, __builtin_fmaf(x[j], c, negm[rb]));
                const bool rise = pw_max(top) > PW_RISE;
                if (__builtin_amdgcn_ballot_w64(rise) != 0) {
                    float mm = x[0] * c;
#pragma unroll
                    for (int j = 1; j < 16; ++j) mm = __builtin_fmaxf(mm, x[j] * c);
                    // (a first reference scales nothing: rows have nothing yet, or what keeping apart has added)
                    const float now = rise ? -pw_max(mm) : negm[rb], f = rise && negm[rb] != PW_FRESH ? __builtin_amdgcn_exp2f(now - negm[rb]) : 1.f;
                    negm[rb] = now;
                    l[rb] *= f;
#pragma unroll
                    for (int e = 0; e < DE; ++e)
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[rb][e][j] *= f;
                }
                uintx4 w[2];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[2 * j], c, negm[rb])), e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[2 * j + 1], c, negm[rb]));
                    l[rb] += e0;
                    l[rb] += e1;
                    w[j >> 2][j & 3] = pack_bf16(e0, e1);
                }
#pragma unroll
                for (int n = 0; n < DK; ++n)
                    o[rb][n % DE] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(val[n], __builtin_bit_cast(bf16x8, w[n / DE]), o[rb][n % DE], 0, 0, 0);
            }
            // the next step's transfers may take this buffer once everything has been read from it
            __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0)
            asm volatile("" ::: "memory");
        }
    }
    // ---- join: wavefront w finishes dims 32 w .. (D = 64: the first two) of every block
    GRAFT_WAIT_VMCNT(0);
    __syncthreads();                             // nobody waits for keys any more: their buffers take the rows
    float* const mine = reinterpret_cast<float*>(&kv[0][0][0]) + wave * (NB * DE * 1024);
#pragma unroll
    for (int rb = 0; rb < NB; ++rb) {
        l[rb] = pw_sum(l[rb]);
        if (half == 0) stat[wave][rb * 32 + l32] = float2{-negm[rb], l[rb]};
#pragma unroll
        for (int e = 0; e < DE; ++e)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<floatx4*>(mine + (rb * DE + e) * 1024 + j * 256 + lane * 4) = floatx4{o[rb][e][4 * j], o[rb][e][4 * j + 1], o[rb][e][4 * j + 2], o[rb][e][4 * j + 3]};
    }
    __syncthreads();
    for (int job = wave; job < NB * DE; job += AT_WAVES) {
        const int rb = job / DE, e = job % DE, r = r_tile + rb * 32 + l32, i = div_any(r, p.g_magic, p.g_shift);
        if (r >= p.R) continue;
        const bool there = i < len.n;
        float2 s[AT_WAVES];
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < AT_WAVES; ++w) {
            s[w] = stat[w][rb * 32 + l32];
            m = __builtin_fmaxf(m, s[w].y != 0.f ? s[w].x : -INFINITY);
        }
        float f[AT_WAVES], total = 0.f;
#pragma unroll
        for (int w = 0; w < AT_WAVES; ++w) {
            f[w] = s[w].y != 0.f ? __builtin_amdgcn_exp2f(s[w].x - m) : 0.f;
            total += s[w].y * f[w];
        }
        floatx4 sum[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            sum[j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < AT_WAVES; ++w) {
                const floatx4 x = *reinterpret_cast<const floatx4*>(reinterpret_cast<const float*>(&kv[0][0][0]) + w * (NB * DE * 1024) + job * 1024 + j * 256 + lane * 4);
#pragma unroll
                for (int y = 0; y < 4; ++y) sum[j][y] += s[w].y != 0.f ? x[y] * f[w] : 0.f;
            }
        }
        if (p.n_splits == 1) {
            const float inv = there && total != 0.f ? 1.f / total : 0.f;
            unsigned short* out = static_cast<unsigned short*>(p.out) + ((static_cast<int64_t>(b) * p.T + i) * p.Hq + g * p.G + (r - i * p.G)) * D + 32 * e + 4 * half;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uintx2 x = {pack_bf16(sum[j][0] * inv, sum[j][1] * inv), pack_bf16(sum[j][2] * inv, sum[j][3] * inv)};
                if (!there) x = uintx2{0u, 0u};
                *reinterpret_cast<uintx2*>(out + 8 * j) = x;
            }
        } else if (there) {
            const size_t part = (static_cast<size_t>(bg) * p.n_splits + split) * p.R + r;
            float* to = p.ws_o + part * D + 32 * e + 4 * half;
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<floatx4*>(to + 8 * j) = sum[j];
            if (half == 0 && e == 0) *reinterpret_cast<float2*>(p.ws_ml + 2 * part) = float2{m, total};
        }
    }
}

int32_t launch_prompt_few(const PromptParams& p, int32_t D, bool cap, int32_t tile_rows, hipStream_t s) {
    const dim3 grid(prompt_grid(p));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(AT_THREADS), 0, s, p.n_nodes, p.prefix_len, p); };
    auto pick = [&](auto d, auto nb) {
        if (cap) launch(prompt_few_kernel<d, nb, true>);
        else launch(prompt_few_kernel<d, nb, false>);
    };
    using std::integral_constant;
    using One = integral_constant<int, 1>;
    using Two = integral_constant<int, 2>;
    if (D == 128) { if (tile_rows == 32) pick(integral_constant<int, 128>{}, One{}); else pick(integral_constant<int, 128>{}, Two{}); }
    else if (tile_rows == 32) pick(integral_constant<int, 64>{}, One{});
    else pick(integral_constant<int, 64>{}, Two{});
    return check_launch();
}

}  // namespace graft
