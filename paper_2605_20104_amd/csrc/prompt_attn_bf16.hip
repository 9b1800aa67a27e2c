// graft_prompt_attn: causal attention of a piece of a prompt over the paged cache (bf16).
//
// A wavefront has NB blocks of 32 rows (a row: one token and one of the G query heads that share a KV head), four wavefronts a
// tile of 128 NB rows, which goes over the keys once: stages of 64 tokens from memory straight to an LDS ring of four.  A unit is
// (32 tokens, row block); in phase u the matrix cores multiply S^T = K Q^T of unit u and O^T += V^T P^T of unit u - 2 in turn while
// the vector ALUs turn the scores of unit u - 1 into probabilities, a slot of the source for each MFMA.  Lane (half, l32) of a score
// tile has row l32 and the tokens 8 (v / 4) + 4 half + v % 4, which are the B operand of the second product as they lie; its A operand
// comes from the LDS transpose read in that order.
//
// Softmax: one pass.  A row's scores are taken relative to a reference, its first maximum; the reference moves when a score
// passes it by 8 (log2 units), so accumulated rows are rescaled hardly ever.  Inside the sequence it is looked at once a stage: what a
// stage adds in between has probabilities of up to 2^24 (past that the tile is done again, every unit checked), everything else of up
// to 2^8.  So sums stay below (2^22 tokens 2^8 + 64 2^24) = 2^31 times the largest value.  Scores, references and sums are fp32;
// probabilities are rounded to bf16 for the second product, results once at the end.
//
// Bound by the energy of its MFMAs and by issue slots: a stage of 64 tokens and 256 rows (D = 128) takes about 3390 cycles, 2056 of them the MFMAs',
// at some 1.9 GHz.  1024 tokens of 40 heads behind 32768: 698 GFLOP, 621 us with the merge (1.12 PFLOP/s, where a library product of 8192^3 reaches 1.24);
// a prompt of 4096 tokens, 32 heads: 141 us (0.98, half of the tiles' ends are masked).  D = 64 and caps have as many exponentials
// for half the products, or two more instructions of that kind a score: 107 us for 84 GFLOP, 180 us for 134.  Matrix cores and vector
// instructions, which one wavefront a SIMD issues, hardly run beside each other: busy in 48 and 41 % of the cycles of the prompt of 4096, in 40
// and 69 % with D = 64 (two wavefronts a SIMD), 36 and 57 % with a cap.
#include "prompt_attn.h"

namespace graft {

constexpr int PA_STAGE = 64, PA_SUB = 32, PA_NBUF = 4;
constexpr float PA_RISE = 8.f;                  // log2 units by which scores may pass their row's reference
constexpr float PA_DAMAGE = 24.f;             // ... and must not, where they are checked late
constexpr float PA_FRESH = 3e38f;               // minus the reference of a row that has seen nothing

template <int D_, int NB_> struct PromptShape {
    static constexpr int D = D_, NB = NB_, RB = 2 * D;             // bytes of a row of keys
    static constexpr int DK = D / 16, DE = D / 32;                 // MFMAs of a unit's scores (and of its output), 32-dim tiles
    static constexpr int SLOTS = 2 * DK, UNITS = 2 * NB;           // of a phase, of a stage
    static constexpr int TILE_ROWS = 4 * NB * 32;
    static constexpr int STAGE_BYTES = 2 * PA_STAGE * RB;          // keys, then values
    static constexpr int LOADS = STAGE_BYTES / 4096;               // transfers of a wavefront and stage
    static constexpr int wrap(int u) { return (u + 2 * UNITS) % UNITS; }
    static constexpr int block(int u) { return wrap(u) % NB; }
    static constexpr bool last_of_sub(int u) { return block(u) == NB - 1; }
    static constexpr int o(int b, int e) { return 16 * (b * DE + e); }
    static constexpr int q(int b, int d) { return 16 * NB * DE + 4 * (b * DK + d); }
    static constexpr int ACC = 16 * NB * DE + 4 * NB * DK;
};

template <class S> struct PromptState {
    floatx16 s[S::NB];
    uintx4 p[S::NB][2];
    bf16x8 k[S::DK], v[S::DK];
    float l[S::NB], negm[S::NB];
    float late[S::NB];                          // the largest score past its reference, of units whose check is still to come
    int lim[S::NB];                             // the last token that the lane's row sees
    bool damaged;
};

// ---- layout of a stage.  Keys: 16-byte chunk c of row r at c ^ key_swizzle(r); values: 32-byte segment at s ^ value_swizzle(r).
// Reads of an operand then touch every bank once: with rows of 256 bytes 16 neighbouring rows, with 128 two of them share a line.
template <int D> __device__ __forceinline__ int key_swizzle(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
template <int D> __device__ __forceinline__ int value_swizzle(int r) { return D == 128 ? (r & 3) << 1 : ((r >> 1) & 1) << 1; }

__device__ __forceinline__ bf16x8 lds_bf16x8(unsigned at) { return *reinterpret_cast<const bf16x8 __attribute__((address_space(3)))*>(static_cast<size_t>(at)); }
template <class S> __device__ __forceinline__ bf16x8 read_keys(unsigned base, int d) { return lds_bf16x8(base ^ (static_cast<unsigned>(d) << 5)); }
// operand n = DE kk + e: dims 32 e .., tokens 16 kk + 8 c + 4 half + 0..3
template <class S> __device__ __forceinline__ bf16x8 read_values(unsigned base, int n) {
    bf16x8 v;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const short4_t r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4_t __attribute__((address_space(3)))*)(static_cast<size_t>(
            (base ^ (static_cast<unsigned>(n % S::DE) << 6)) + (16 * (n / S::DE) + 8 * c) * S::RB)));
        const bf16x4 r4 = __builtin_bit_cast(bf16x4, r);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * c + j] = r4[j];
    }
    return v;
}

// AccVGPRs, placed by hand (left to the compiler, whole accumulators are moved about and registers go to scratch memory): O^T of row
// block b, dims 32 e ..: a[S::o(b, e) ..]; queries of block b, dim step d: a[S::q(b, d) ..].  The compiler does not know that the
// statements below are MFMAs: whoever reads their results, or writes their operands, keeps the distance that the build checks.
__device__ __forceinline__ void reserve_registers_128() {
    asm volatile("" ::: GRAFT_ACC_BLOCK_0);
    asm volatile("" ::: GRAFT_ACC_BLOCK_1);
    asm volatile("" ::: GRAFT_ACC_BLOCK_2);
    asm volatile("" ::: GRAFT_ACC_BLOCK_3);
}
__device__ __forceinline__ void reserve_registers_64() {
    asm volatile("" ::: GRAFT_ACC_BLOCK_0);
    asm volatile("" ::: GRAFT_ACC_BLOCK_1);
}
template <class S> __device__ __forceinline__ void reserve_registers() {
    static_assert(S::ACC <= (S::D == 128 ? 192 : 96));
    if constexpr (S::D == 128) reserve_registers_128();
    else reserve_registers_64();
}
template <int QR, bool FIRST> __device__ __forceinline__ void mfma_scores(floatx16& s, const bf16x8& k) {
    if constexpr (FIRST) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, a[%2:%3], 0" : "=&v"(s) : "v"(k), "n"(QR), "n"(QR + 3));
    else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, a[%2:%3], %0" : "+v"(s) : "v"(k), "n"(QR), "n"(QR + 3));
}
template <int OR> __device__ __forceinline__ void mfma_output(const bf16x8& v, const uintx4& p) {
    asm volatile("v_mfma_f32_32x32x16_bf16 a[%0:%1], %2, %3, a[%0:%1]" : : "n"(OR), "n"(OR + 15), "v"(v), "v"(p));
}
template <int R> __device__ __forceinline__ void acc_add(float a) {
    float t;
    asm volatile("v_accvgpr_read_b32 %0, a[%1]\n\ts_nop 1\n\tv_add_f32 %0, %0, %2\n\ts_nop 1\n\tv_accvgpr_write_b32 a[%1], %0" : "=&v"(t) : "n"(R), "v"(a));
}
__device__ __forceinline__ void settle_scores(floatx16& s) { asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s)); }

template <class T> __device__ __forceinline__ T in_place(T x) {    // computed where it stands in the source
    asm volatile("" : : "v"(x));
    return x;
}
__device__ __forceinline__ float halves_sum(float v) {
    const unsigned u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float halves_max(float v) {
    const unsigned u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Scores to log2 units: c x, or with a cap c = cap log2(e) times tanh(x in / 2 log2(e)).
struct ToLog2 { float c, in; };

// Behind the probabilities of block B's unit, now and then.  Its scores have passed their rows' references (or are the first):
// new references, what is accumulated scaled down, the probabilities again.  Units without a check of their own: probabilities of up
// to 2^PA_DAMAGE are accumulated as they are; past that they, and sums and products with them, may not be numbers any more.
// RAW: scores whose cap is still to come.
template <class S, int B, bool RAW> __device__ __forceinline__ void raise_reference(PromptState<S>& w, ToLog2 to, float l_before) {
    auto score = [&](int x) __attribute__((always_inline)) { return RAW ? capped(w.s[B][x], to.in, to.c) : w.s[B][x] * to.c; };
    GRAFT_MFMA_SETTLE();
    static_for<0, S::NB>([&](auto b_) {
        GRAFT_CONST(b, b_);
        const float late = halves_max(w.late[b]);
        w.damaged = w.damaged || __builtin_amdgcn_ballot_w64(late > PA_DAMAGE) != 0;
        float negm = w.negm[b], l = b == B ? l_before : w.l[b];
        if (late > PA_RISE) negm -= late;
        if constexpr (b == B) {
            float mm = score(0);
#pragma unroll
            for (int x = 1; x < 16; ++x) mm = __builtin_fmaxf(mm, score(x));
            mm = halves_max(mm);
            if (mm + negm > PA_RISE) negm = -mm;
        }
        // (a first reference scales nothing: rows have nothing yet, or what keeping apart has added)
        const float f = negm < w.negm[b] && w.negm[b] != PA_FRESH ? __builtin_amdgcn_exp2f(negm - w.negm[b]) : 1.f;
        w.negm[b] = negm;
        w.late[b] = -INFINITY;
        l *= f;
        static_for<0, 16 * S::DE>([&](auto x_) {
            GRAFT_CONST(x, x_);
            acc_scale<S::o(b, 0) + x>(f);
        });
        if constexpr (b == B) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p0 = __builtin_amdgcn_exp2f(RAW ? score(2 * j) + negm : __builtin_fmaf(w.s[b][2 * j], to.c, negm));
                const float p1 = __builtin_amdgcn_exp2f(RAW ? score(2 * j + 1) + negm : __builtin_fmaf(w.s[b][2 * j + 1], to.c, negm));
                l += p0;
                l += p1;
                w.p[b][j >> 2][j & 3] = pack_bf16(p0, p1);
            }
        }
        w.l[b] = l;
    });
    GRAFT_MFMA_SETTLE();
}

// One phase: scores of unit J, probabilities of unit J - 1 (RAW: their cap on the way), products of unit J - 2.  CHECK: with the check of
// the references.
template <class S, int J, bool QK, bool SM, bool PV, bool CHECK, bool RAW, class Extra>
__device__ __forceinline__ void prompt_phase(PromptState<S>& w, ToLog2 to, unsigned k_next, unsigned v_next, Extra&& extra) {
    constexpr int QB = S::block(J), SB = S::block(J - 1), PB = S::block(J - 2), PER = 16 / S::SLOTS;
    constexpr bool K_RELOAD = QK && S::last_of_sub(J), V_RELOAD = QK && S::last_of_sub(J - 2);      // for the next 32 tokens
    float t[16], y[16], e[16], top = -INFINITY;
    reserve_registers<S>();
    if constexpr (!QK) asm volatile("s_nop 1");
    const float l_before = w.l[SB], base = RAW ? w.negm[SB] + to.c : w.negm[SB];
    // Element x, in slots of their own where a cap makes it a chain: the exponential of tanh, its reciprocal, then the rest.
    auto first = [&](auto x_) __attribute__((always_inline)) {
        GRAFT_CONST(x, x_);
        t[x] = in_place(__builtin_amdgcn_exp2f(w.s[SB][x] * to.in));
    };
    auto second = [&](auto x_) __attribute__((always_inline)) {
        GRAFT_CONST(x, x_);
        t[x] = in_place(__builtin_amdgcn_rcpf(1.f + t[x]));
    };
    auto last = [&](auto x_) __attribute__((always_inline)) {
        GRAFT_CONST(x, x_);
        y[x] = RAW ? __builtin_fmaf(-2.f * to.c, t[x], base) : __builtin_fmaf(w.s[SB][x], to.c, base);
        e[x] = in_place(__builtin_amdgcn_exp2f(y[x]));
        if constexpr (x % 2 == 1) top = in_place(__builtin_fmaxf(__builtin_fmaxf(top, y[x - 1]), y[x]));
        if constexpr (x >= 1) w.l[SB] = in_place(w.l[SB] + e[x - 1]);
        if constexpr (x >= 2 && x % 2 == 0) w.p[SB][(x - 2) >> 3][((x - 2) >> 1) & 3] = in_place(pack_bf16(e[x - 2], e[x - 1]));
    };
    static_for<0, S::SLOTS>([&](auto i_) {
        GRAFT_CONST(i, i_);
        constexpr int h = i >> 1;
        if constexpr (i % 2 == 0) {
            if constexpr (QK) mfma_scores<S::q(QB, h), i == 0>(w.s[QB], w.k[h]);
        } else {
            if constexpr (PV) mfma_output<S::o(PB, h % S::DE)>(w.v[h], w.p[PB][h / S::DE]);
        }
        if constexpr (SM) {                      // (the scores have settled by slot 1)
            constexpr int to1 = i == 0 ? 0 : PER * (i + 1), from1 = i < 2 ? 0 : PER * i;
            constexpr int to2 = i < 2 ? 0 : PER * i, from2 = i < 3 ? 0 : PER * (i - 1), to3 = i < 3 ? 0 : PER * (i - 1), from3 = i < 4 ? 0 : PER * (i - 2);
            if constexpr (RAW) {
                static_for<from1, to1>(first);
                static_for<from2, to2>(second);
                static_for<from3, to3>(last);
            } else static_for<from1, to1>(last);
        }
        if constexpr (K_RELOAD && i % 2 == 1) w.k[h] = read_keys<S>(k_next, h);
        if constexpr (V_RELOAD && i % 2 == 0 && i >= 2) w.v[h - 1] = read_values<S>(v_next, h - 1);
        extra(i_);
        __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (SM && RAW) {
        static_for<16 - PER, 16>(second);
        static_for<16 - 2 * PER, 16>(last);
    }
    if constexpr (SM) {
        w.p[SB][1][3] = in_place(pack_bf16(e[14], e[15]));
        w.l[SB] = in_place(w.l[SB] + e[15]);
    }
    if constexpr (V_RELOAD) w.v[S::DK - 1] = read_values<S>(v_next, S::DK - 1);
    if constexpr (SM && !CHECK) w.late[SB] = in_place(__builtin_fmaxf(w.late[SB], top));
    if constexpr (SM && CHECK) {
#pragma unroll
        for (int b = 0; b < S::NB; ++b) top = __builtin_fmaxf(top, w.late[b]);
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(top > PA_RISE) != 0, 0)) raise_reference<S, SB, RAW>(w, to, l_before);
    }
    __builtin_amdgcn_sched_barrier(0);
}

// What the rows of block B do not see of the 32 tokens from t on becomes -inf.
template <class S, int B> __device__ __forceinline__ void hide(PromptState<S>& w, int t, int half, int window) {
    settle_scores(w.s[B]);
    const int rel = w.lim[B] - t - 4 * half;
#pragma unroll
    for (int x = 0; x < 16; ++x)
        w.s[B][x] = static_cast<unsigned>(rel - (8 * (x >> 2) + (x & 3))) < static_cast<unsigned>(window) ? w.s[B][x] : -INFINITY;
}

template <int D, int NB, bool CAP>
__global__ __launch_bounds__(AT_THREADS, 1) void prompt_attn_kernel(const int32_t* n_nodes, const int32_t* prefix_len, PromptParams p) {
    using S = PromptShape<D, NB>;
    constexpr int UNITS = S::UNITS, RB = S::RB;
    __shared__ __attribute__((aligned(1024))) unsigned char kv[PA_NBUF][S::STAGE_BYTES];
    __shared__ int32_t vote[AT_WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, l32 = lane & 31, half = lane >> 5;
    const PromptItem item = prompt_item(p);
    if (item.unit < 0) return;
    const int bg = item.unit / p.n_splits, split = item.unit - bg * p.n_splits, b = bg / p.Hkv, g = bg - b * p.Hkv;
    const PromptLengths len = prompt_lengths(p, scalar_load(prefix_len, b), scalar_load(n_nodes, b));
    const int r_tile = item.row_tile * S::TILE_ROWS;
    const PromptRange t = prompt_range<PA_STAGE>(p, len, r_tile, S::TILE_ROWS);
    const int spt = (t.st1 - t.st0 + p.n_splits - 1) / p.n_splits, st0 = t.st0 + split * spt, st1 = st0 + spt < t.st1 ? st0 + spt : t.st1;
    const int n_st = st1 - st0;                                    // (may be negative)
    const unsigned kv_base = __builtin_amdgcn_readfirstlane(lds_address(&kv[0][0]));

    PromptState<S> w;
    int row_of[NB];                                                // the lane's row, and whether it is there
    bool live[NB];
    uintx4 qd[NB][S::DK];
#pragma unroll
    for (int rb = 0; rb < NB; ++rb) {
        const int r = r_tile + (wave * NB + rb) * 32 + l32, i = div_any(r, p.g_magic, p.g_shift);
        row_of[rb] = r;
        live[rb] = r < p.R && i < len.n;
        w.lim[rb] = len.P + (live[rb] ? i : t.i1);                // (rows that are not there see what others see)
        const unsigned short* q = static_cast<const unsigned short*>(p.q) +
            ((static_cast<int64_t>(b) * p.T + i) * p.Hq + g * p.G + (r - i * p.G)) * D + 8 * half;
#pragma unroll
        for (int d = 0; d < S::DK; ++d) {
            qd[rb][d] = uintx4{0u, 0u, 0u, 0u};
            if (live[rb]) qd[rb][d] = *reinterpret_cast<const uintx4*>(q + 16 * d) ^ p.q_sign;
        }
    }
    reserve_registers<S>();
    auto clear_rows = [&]() __attribute__((always_inline)) {
        static_for<0, 16 * NB * S::DE>([&](auto x_) {
            GRAFT_CONST(x, x_);
            acc_set<x>(0.f);
        });
#pragma unroll
        for (int rb = 0; rb < NB; ++rb) {
            w.l[rb] = 0.f;
            w.negm[rb] = PA_FRESH;
            w.late[rb] = -INFINITY;
            w.p[rb][0] = w.p[rb][1] = uintx4{0u, 0u, 0u, 0u};
        }
        w.damaged = false;
    };
    clear_rows();
    static_for<0, NB>([&](auto rb_) {
        GRAFT_CONST(rb, rb_);
        static_for<0, 4 * S::DK>([&](auto x_) {
            GRAFT_CONST(x, x_);
            acc_set_bits<S::q(rb, 0) + x>(qd[rb][x / 4][x % 4]);
        });
    });
    if (n_st > 0) {
        // ---- transfers: a wavefront moves one page a stage, through a buffer descriptor that ends with the sequence's last token (with
        //      nothing, past the last page): what lies behind it arrives as zeros.
        const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_pages;
        const int last_tok = len.P + len.n - 1, last_pg = last_tok >> 4;
        const unsigned ts2 = static_cast<unsigned>(p.token_stride) * 2u;
        constexpr int LANES = RB / 16, ROWS = 64 / LANES;          // lanes a row, rows an instruction
        const int lr = lane / LANES, lc = lane % LANES;
        const u64 k_head = reinterpret_cast<u64>(p.k) + static_cast<u64>(g * p.head_stride) * 2, v_head = reinterpret_cast<u64>(p.v) + static_cast<u64>(g * p.head_stride) * 2;
        auto page_index = [&](int k) __attribute__((always_inline)) {
            const int pg = (st0 + k) * (PA_STAGE / GRAFT_PAGE_SIZE) + wave;
            return pg < last_pg ? pg : last_pg;
        };
        auto load_table = [&](int k0) __attribute__((always_inline)) {        // lane i: the page of stage k0 + i
            int32_t x = table[page_index(k0 + lane)];
            asm volatile("" : "+v"(x));          // (waited for here, not where it is used, behind transfers)
            return x;
        };
        int32_t pages = 0;
        struct PageOf { uintx4 k, v; unsigned lds; };
        auto page_of = [&](int k) __attribute__((always_inline)) {
            PageOf d;
            const u64 off = static_cast<u64>(static_cast<unsigned>(__builtin_amdgcn_readlane(pages, k & 63))) * static_cast<u64>(p.page_stride * 2);
            const u64 ka = k_head + off, va = v_head + off;
            const int rows = last_tok - (st0 + k) * PA_STAGE - 16 * wave;          // the last token's row in the page
            const bool some = rows >= 0 && k < n_st;
            const unsigned bytes = some ? static_cast<unsigned>(rows < 15 ? rows : 15) * ts2 + RB : 0u;
            d.k = uintx4{static_cast<unsigned>(ka), static_cast<unsigned>(ka >> 32), bytes, BUFFER_WORD3};
            d.v = uintx4{static_cast<unsigned>(va), static_cast<unsigned>(va >> 32), bytes, BUFFER_WORD3};
            d.lds = kv_base + (k & (PA_NBUF - 1)) * S::STAGE_BYTES + wave * (16 * RB);
            return d;
        };
        auto move = [&](const PageOf& d, int n) __attribute__((always_inline)) {    // instruction n of LOADS
            const int j = n >> 1, r = ROWS * j + lr;
            const unsigned chunk = n & 1 ? (((lc >> 1) ^ value_swizzle<D>(r)) << 1) | (lc & 1) : lc ^ key_swizzle<D>(r);
            buffer_to_lds_b128(n & 1 ? d.v : d.k, static_cast<unsigned>(r) * ts2 + chunk * 16, d.lds + (n & 1) * PA_STAGE * RB + j * 1024);
        };
        auto move_page = [&](int k) __attribute__((always_inline)) {
            const PageOf d = page_of(k);
#pragma unroll
            for (int n = 0; n < S::LOADS; ++n) move(d, n);
        };
        // every stage is LOADS instructions of a wavefront, whatever they move
        auto arrive = [&](auto newer_) __attribute__((always_inline)) {     // all but the newest stages are there, for everybody
            GRAFT_CONST(newer, newer_);
            GRAFT_WAIT_VMCNT(newer * S::LOADS);
            lds_barrier();
        };
        // lane parts of the operand addresses inside 32 tokens
        constexpr unsigned V_OFF = PA_STAGE * RB, SUB = PA_SUB * RB;
        const int v_row = 4 * half + (l16 >> 2);
        const unsigned k_lane = kv_base + l32 * RB + ((half ^ key_swizzle<D>(l32)) << 4);
        const unsigned v_lane = kv_base + V_OFF + v_row * RB + (((l32 >> 4) ^ value_swizzle<D>(v_row)) << 5) + 8 * (l16 & 3);
        auto sub_base = [&](int k, int sub) __attribute__((always_inline)) { return static_cast<unsigned>((k & (PA_NBUF - 1)) * S::STAGE_BYTES) + sub * SUB; };

        const ToLog2 done = {CAP ? 1.f : p.scale_log2e, 0.f}, raw = {p.cap_log2e, p.cap_in};
        auto cap_scores = [&](floatx16& x) __attribute__((always_inline)) {
            settle_scores(x);
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] = capped(x[j], p.cap_in, p.cap_log2e);
        };

        // Values that are not numbers, in a stage that not every row sees whole: 0 times them would reach rows that do not.
        // They are added to the rows that see them here, and become zeros.
        auto keep_apart = [&](int k) __attribute__((always_inline)) {
            unsigned char* const vs = &kv[k & (PA_NBUF - 1)][V_OFF];
            bool odd = false;
#pragma unroll
            for (int x = 0; x < PA_STAGE * RB / 16 / AT_THREADS; ++x) {
                const uintx4 y = reinterpret_cast<const uintx4*>(vs)[x * AT_THREADS + tid];
#pragma unroll
                for (int j = 0; j < 4; ++j) odd |= (y[j] & 0x7f80u) == 0x7f80u || (y[j] & 0x7f800000u) == 0x7f800000u;
            }
            if (__builtin_amdgcn_ballot_w64(odd) != 0) odd = true;
            if (lane == 0) vote[wave] = odd;
            lds_barrier();
            if (__builtin_expect((vote[0] | vote[1] | vote[2] | vote[3]) == 0, 1)) return;
            GRAFT_MFMA_SETTLE();
            for (int tok = 0; tok < PA_STAGE; ++tok) {
                const int at = (st0 + k) * PA_STAGE + tok;
                static_for<0, NB>([&](auto rb_) {
                    GRAFT_CONST(rb, rb_);
                    const bool sees = static_cast<unsigned>(w.lim[rb] - at) < static_cast<unsigned>(p.window);
                    static_for<0, S::DE>([&](auto e_) {
                        GRAFT_CONST(e, e_);
                        static_for<0, 16>([&](auto x_) {
                            GRAFT_CONST(x, x_);
                            const int dim = 32 * e + 8 * (x >> 2) + 4 * half + (x & 3), seg = dim >> 4;
                            const unsigned short bits = *reinterpret_cast<const unsigned short*>(vs + tok * RB + ((seg ^ value_swizzle<D>(tok)) << 5) + 2 * (dim & 15));
                            const bool add = sees && (bits & 0x7f80) == 0x7f80;
                            acc_add<S::o(rb, e) + x>(add ? __uint_as_float(static_cast<unsigned>(bits) << 16) : 0.f);
                        });
                    });
                });
            }
            lds_barrier();
#pragma unroll
            for (int x = 0; x < PA_STAGE * RB / 16 / AT_THREADS; ++x) {
                uintx4* const y = reinterpret_cast<uintx4*>(vs) + x * AT_THREADS + tid;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    unsigned z = (*y)[j];
                    if ((z & 0x7f80u) == 0x7f80u) z &= 0xffff0000u;
                    if ((z & 0x7f800000u) == 0x7f800000u) z &= 0xffffu;
                    (*y)[j] = z;
                }
            }
            lds_barrier();
        };

        // Caps: in a PLAIN stage on the way to the probabilities, a phase behind the scores (RAW_BEFORE: those of the stage before wait for
        // theirs); elsewhere at once, since what is hidden has to stay so.
        auto stage = [&](int k, auto plain_, auto raw_before_) __attribute__((always_inline)) {
            constexpr bool PLAIN = decltype(plain_)::value, RAW_BEFORE = decltype(raw_before_)::value;
            PageOf next;
            arrive(std::integral_constant<int, 1>{});              // stage k + 1 is there; nobody reads stage k - 1 any more
            if constexpr (!PLAIN) keep_apart(k);
            static_for<0, UNITS>([&](auto j_) {
                GRAFT_CONST(J, j_);
                constexpr int QB = S::block(J);
                const unsigned k_next = k_lane + (J == UNITS - 1 ? sub_base(k + 1, 0) : sub_base(k, 1));
                const unsigned v_next = v_lane + (S::wrap(J - 2) == UNITS - 1 ? sub_base(k, 0) : sub_base(k, 1));
                constexpr bool RAW = CAP && (J == 0 ? RAW_BEFORE : PLAIN);
                prompt_phase<S, J, true, true, true, !PLAIN || J == 0, RAW>(w, RAW ? raw : done, k_next, v_next, [&](auto i_) __attribute__((always_inline)) {
                    GRAFT_CONST(i, i_);
                    constexpr int at = S::SLOTS * J + i, SPACE = S::SLOTS * UNITS / S::LOADS / 2;
                    if constexpr (at == 0) next = page_of(k + 3);
                    if constexpr (at > 0 && at % SPACE == 0 && at / SPACE <= S::LOADS) move(next, at / SPACE - 1);
                });
                if constexpr (CAP && !PLAIN) cap_scores(w.s[QB]);
                if constexpr (!PLAIN) hide<S, QB>(w, (st0 + k) * PA_STAGE + (J / NB) * PA_SUB, half, p.window);
            });
        };
        // Stages that every row of the tile sees whole, behind one (the split's first, or the last with a row's first token) that is checked
        // as it goes, so that every row has its reference: plain_from .. plain_to.
        const int first = len.P + t.i1 - p.window + 1, whole = first < 0 ? 1 : first / PA_STAGE + 1 - st0;
        const int plain_from = whole < 1 ? 1 : whole;
        int plain_to = (len.P + t.i0 + 1) / PA_STAGE - st0;
        plain_to = plain_to < n_st ? plain_to : n_st;
        const auto next_pages = [&](int k) __attribute__((always_inline)) { if (((k + 3) & 63) == 0) pages = load_table(k + 3); };
        for (int attempt = 0;; ++attempt) {
            pages = load_table(0);
            move_page(0);
            move_page(1);
            move_page(2);
            arrive(std::integral_constant<int, 2>{});
#pragma unroll
            for (int d = 0; d < S::DK; ++d) {
                w.k[d] = read_keys<S>(k_lane + sub_base(0, 0), d);
                w.v[d] = __builtin_bit_cast(bf16x8, uintx4{0u, 0u, 0u, 0u});
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) w.s[S::block(UNITS - 1)][x] = -INFINITY;
            for (int k = 0; k < n_st;) {         // (loops of their own: the registers stay where they are from stage to stage)
                const int masked_to = k < plain_from ? (plain_from < n_st ? plain_from : n_st) : (k < plain_to ? k : n_st);
                while (k < masked_to) {
                    stage(k, std::false_type{}, std::false_type{});
                    next_pages(++k);
                }
                if (CAP && k < plain_to) {
                    stage(k, std::true_type{}, std::false_type{});
                    next_pages(++k);
                }
                while (k < plain_to) {
                    stage(k, std::true_type{}, std::bool_constant<CAP>{});
                    next_pages(++k);
                }
                if (CAP && k > plain_from && k == plain_to) cap_scores(w.s[S::block(UNITS - 1)]);
            }
            const auto nothing = [](auto) {};
            prompt_phase<S, 0, false, true, true, true, false>(w, done, 0u, 0u, nothing);
            prompt_phase<S, 1, false, false, true, false, false>(w, done, 0u, 0u, nothing);
            GRAFT_MFMA_SETTLE();
            GRAFT_WAIT_VMCNT(0);                 // (transfers of stages that are not there)
            lds_barrier();
            if (lane == 0) vote[wave] = w.damaged;
            lds_barrier();
            if (__builtin_expect(attempt > 0 || (vote[0] | vote[1] | vote[2] | vote[3]) == 0, 1)) break;
            plain_to = 0;                        // once more, every unit checked
            clear_rows();
            GRAFT_MFMA_SETTLE();
        }
    }
    // ---- results: dims 32 e + 8 j + 4 half + 0..3 of row l32 in a[o(rb, e) + 4 j ..]
    static_for<0, NB>([&](auto rb_) {
        GRAFT_CONST(rb, rb_);
        const float l = halves_sum(w.l[rb]);
        const int r = row_of[rb];
        float o[S::DE * 16];
        static_for<0, S::DE * 16>([&](auto x_) {
            GRAFT_CONST(x, x_);
            o[x] = acc_get<S::o(rb, 0) + x>();
        });
        if (r >= p.R) return;
        if (p.n_splits == 1) {
            const int i = div_any(r, p.g_magic, p.g_shift);
            const float inv = live[rb] && l != 0.f ? 1.f / l : 0.f;
            unsigned short* out = static_cast<unsigned short*>(p.out) + ((static_cast<int64_t>(b) * p.T + i) * p.Hq + g * p.G + (r - i * p.G)) * D + 4 * half;
#pragma unroll
            for (int j = 0; j < 4 * S::DE; ++j) {
                uintx2 x = {pack_bf16(o[4 * j] * inv, o[4 * j + 1] * inv), pack_bf16(o[4 * j + 2] * inv, o[4 * j + 3] * inv)};
                if (!live[rb]) x = uintx2{0u, 0u};
                *reinterpret_cast<uintx2*>(out + 8 * j) = x;
            }
        } else if (live[rb]) {
            const size_t part = (static_cast<size_t>(bg) * p.n_splits + split) * p.R + r;
            float* to = p.ws_o + part * D + 4 * half;
#pragma unroll
            for (int j = 0; j < 4 * S::DE; ++j) *reinterpret_cast<floatx4*>(to + 8 * j) = floatx4{o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]};
            if (half == 0) *reinterpret_cast<float2*>(p.ws_ml + 2 * part) = float2{-w.negm[rb], l};
        }
    });
}

int32_t launch_prompt_bf16(const PromptParams& p, int32_t D, bool cap, hipStream_t s) {
    const dim3 grid(prompt_grid(p));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(AT_THREADS), 0, s, p.n_nodes, p.prefix_len, p); };
    auto pick = [&](auto d, auto nb) {
        if (cap) launch(prompt_attn_kernel<d, nb, true>);
        else launch(prompt_attn_kernel<d, nb, false>);
    };
    using std::integral_constant;
    if (D == 128) pick(integral_constant<int, 128>{}, integral_constant<int, 2>{});
    else pick(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    return check_launch();
}

}  // namespace graft
