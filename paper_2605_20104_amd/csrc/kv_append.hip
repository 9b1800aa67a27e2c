// graft_kv_append, graft_kv_append_mx: new tokens' queries and keys are turned by their positions, keys and values go to their slots of
// the paged cache, as they are or as 4-bit elements.
//
// A pair (a, b) of a row becomes (a cos - b sin, b cos + a sin), products and sum each rounded to float32 (no fused multiply-add:
// which 4-bit element a number becomes does not depend on how a compiler contracts), and once more where the row is stored.
//
// Bound by memory: every element is read once and written once.  A lane has 8 elements of a row, 16 lanes (8 with D = 64) a row, whatever
// the pairing: where partners are R / 2 apart a lane loads its partner's 16 bytes too, from a line that its own request brings to
// the cache (four lanes of a block of 32 stay neighbours, so a block's largest magnitude takes two lane exchanges).  A lane has the
// cosines and sines of one token in registers, and loads up to HELD rows before it waits for any.
// With few tokens the lanes of a workgroup share one token's rows, and as long as there are compute units to spare several workgroups do (64 + 2 x 4
// heads, us: 1 or 48 tokens 5.4 -> 4.2; 384 tokens, with two each, 7.1 -> 7.5).  With so many tokens that three of four compute units get a workgroup all the same, a
// wavefront's groups of lanes have a token each and its steps are the rows: what it writes to the cache is next to each other, also where elements of tokens are interleaved.
// (32 + 2 x 8 bf16 heads of 128, us: 512 tokens 6.9 shared and 7.8 not, 1024 tokens 11.5 and 9.0, 16382 tokens 128 and 90.)  The groups are of one
// sequence: where fewer than half of them would have a token, tokens stay shared.  (Shared and not, us: 1024 x 1 10.0 and 15.0, 4096 x 1 32.6 and 47.7, 2048 x 2
// 32.5 and 27.8; of heads of 64, which have eight groups, 2048 x 1 10.8 and 24.4, 2730 x 3 32.0 and 35.2, 2048 x 4 31.9 and 28.5.)  Stores do not push
// what is read out of the caches: the prompt 87.  A wait for loads is one for the stores in front of them too, so there 12 rows (8 of float32) are held
// and not 4: 84.  411 MB in 84 us are 4.9 TB/s.  Fewer rows a workgroup (in more of them) take longer, and so do two batches of rows in turn.
// Of 64 + 2 x 4 heads, where tokens are shared, four of five steps are held: keys and values are such a second batch (384 tokens 8.2).
// A sequence's first workgroup looks at all positions before it asks for its own rows: a third trip to memory for a single token, and of prompts of one
// head 2 to 4 % (8192 tokens 14.1 without given positions and 14.4 with, 65536 96 and 100).
#include "mx.h"

namespace graft {

constexpr int KA_THREADS = 256;

struct AppendParams {
    const void *q, *k, *v;
    void *q_out, *k_cache, *v_cache;
    const float* cos_sin;
    const int32_t *block_table, *prefix_len, *n_nodes, *pos;
    int32_t* status;
    int64_t q_stride, k_stride, v_stride;                     // elements from token to token
    int64_t page_stride, token_stride, head_stride;           // elements; bytes in the 4-bit cache
    int32_t n_pos, R, max_pages, T, Hq, Hkv;
};

typedef unsigned Quad4 __attribute__((ext_vector_type(4)));

// Eight elements of a row, as loaded and as numbers.
template <bool F32> struct Eight {
    Quad4 raw[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void* base, int64_t at) {
        const Quad4* p = reinterpret_cast<const Quad4*>(static_cast<const char*>(base) + at * (F32 ? 4 : 2));
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) raw[i] = p[i];
    }
    __device__ __forceinline__ void store(void* base, int64_t at) const {
        Quad4* p = reinterpret_cast<Quad4*>(static_cast<char*>(base) + at * (F32 ? 4 : 2));
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) __builtin_nontemporal_store(raw[i], p + i);
    }
    __device__ __forceinline__ float get(int j) const {
        if constexpr (F32) return __uint_as_float(raw[j / 4][j % 4]);
        else return __uint_as_float((j & 1) ? raw[0][j / 2] & 0xFFFF0000u : raw[0][j / 2] << 16);
    }
    __device__ __forceinline__ void set(const float* x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (F32) {
                raw[0][i] = __float_as_uint(x[i]);
                raw[1][i] = __float_as_uint(x[4 + i]);
            } else {
                typedef __bf16 Two __attribute__((ext_vector_type(2)));
                const Two t = {static_cast<__bf16>(x[2 * i]), static_cast<__bf16>(x[2 * i + 1])};
                raw[0][i] = __builtin_bit_cast(unsigned, t);
            }
        }
    }
};

// a cos -+ b sin as three roundings
__device__ __forceinline__ float turn(float a, float c, float b, float s) {
#pragma clang fp contract(off)
    const float x = a * c, y = b * s;
    return x + y;
}

// A row's 8 elements of a lane into the 4-bit cache.  Four lanes (a quad) have a block of 32.
template <int D> __device__ __forceinline__ void store_mx(unsigned char* run, bool values, int token, int lane, const float* x) {
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const unsigned u = __float_as_uint(x[j]) & 0x7FFFFFFFu;
        top = u > top ? u : top;
    }
    top = max_dpp_u32<0xB1>(top);
    top = max_dpp_u32<0x4E>(top);
    const unsigned byte = mx_scale_byte(top);
    const float scale = mx_scale(byte);
    unsigned four = 0;
    four = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(four, x[0], x[1], scale, 0);
    four = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(four, x[2], x[3], scale, 1);
    four = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(four, x[4], x[5], scale, 2);
    four = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(four, x[6], x[7], scale, 3);
    if (byte == MX_NAN) four = 0;
    if (D == 128 || !values) *reinterpret_cast<unsigned*>(run + mx_part_at<D>(values, token, lane * 8 / (D / 16))) = four;
    else {
        *reinterpret_cast<unsigned short*>(run + mx_part_at<D>(true, token, lane * 2)) = static_cast<unsigned short>(four);
        *reinterpret_cast<unsigned short*>(run + mx_part_at<D>(true, token, lane * 2 + 1)) = static_cast<unsigned short>(four >> 16);
    }
    if ((lane & 3) == 0) run[mx_scale_at<D>(token, lane >> 2)] = static_cast<unsigned char>(byte);
}

// (the arguments of the first trip to memory stand first: they arrive in registers)
template <int D, bool F32, bool MX, bool INTERLEAVED, bool SHARE>
__global__ __launch_bounds__(KA_THREADS) void kv_append_kernel(const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ n_nodes,
                                                               const int32_t* __restrict__ pos, int32_t T, AppendParams p) {
    constexpr int LANES = D / 8, ROWS = 64 / LANES, HELD = SHARE ? (F32 ? 2 : 4) : (F32 ? 8 : 12), WAVES = KA_THREADS / 64;
    const int b = blockIdx.y, lane64 = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = SHARE ? blockIdx.x : blockIdx.x * ROWS + lane64 / LANES;     // this lane's token
    const int64_t token0 = static_cast<int64_t>(b) * T, token = token0 + i;
    // (the position of a padding token too: one trip to memory for all three)
    const int32_t P = prefix_len[b], n = n_nodes[b], given = pos ? pos[i < T ? token : token0] : 0;
    const bool bad = P < 0 || n < 0 || n > T || static_cast<int64_t>(P) + n > static_cast<int64_t>(p.max_pages) * GRAFT_PAGE_SIZE;
    auto turned = [&](int32_t at) { return p.R == 0 || (at >= 0 && at < p.n_pos); };
    if (blockIdx.x == 0 && blockIdx.z == 0) {      // a sequence's first workgroup looks at all of its positions
        __shared__ int32_t wrong[WAVES];
        bool off = false;
        if (!bad) for (int32_t j = threadIdx.x; j < n; j += KA_THREADS) off = off || !turned(pos ? pos[token0 + j] : P + j);
        const bool any = __builtin_amdgcn_ballot_w64(off) != 0;
        if (lane64 == 0) wrong[wave] = any;
        __syncthreads();
        if (threadIdx.x == 0) {
            int32_t st = bad;
            for (int w = 0; w < WAVES; ++w) st |= wrong[w];
            p.status[b] = st ? GRAFT_STATUS_BAD_LENGTH : 0;
        }
    }
    if (bad || i >= n) return;
    const int32_t at = pos ? given : P + i, slot = P + i;
    if (!turned(at)) return;
    const int64_t page = p.block_table[static_cast<int64_t>(b) * p.max_pages + slot / GRAFT_PAGE_SIZE];
    const int in_page = slot & (GRAFT_PAGE_SIZE - 1);

    const int lane = threadIdx.x % LANES, row = SHARE ? (blockIdx.z * WAVES + wave) * ROWS + lane64 / LANES : wave, step = SHARE ? gridDim.z * WAVES * ROWS : WAVES, d = lane * 8, half = p.R / 2;
    const bool rotates = d < p.R, second = !INTERLEAVED && d >= half;
    const int partner = second ? -half : half;     // (elements to the pair's other one)
    const int rows = p.Hq + 2 * p.Hkv;
    constexpr int ANGLES = INTERLEAVED ? 4 : 8;
    float c[ANGLES], s[ANGLES];
    if (rotates) {
        const float* angle = p.cos_sin + static_cast<int64_t>(at) * p.R + (INTERLEAVED ? d / 2 : second ? d - half : d);
#pragma unroll
        for (int j = 0; j < ANGLES; ++j) {
            c[j] = angle[j];
            s[j] = second || INTERLEAVED ? angle[half + j] : -angle[half + j];
        }
    }
    for (int r0 = row; r0 < rows; r0 += HELD * step) {
        Eight<F32> held[HELD], others[HELD];
#pragma unroll
        for (int u = 0; u < HELD; ++u) {           // all that is read, before any of it is waited for
            const int r = r0 + u * step;
            if (r >= rows) break;
            const bool is_q = r < p.Hq, is_v = r >= p.Hq + p.Hkv;
            const void* src = is_q ? p.q : is_v ? p.v : p.k;
            const int64_t from = token * (is_q ? p.q_stride : is_v ? p.v_stride : p.k_stride) + static_cast<int64_t>(is_q ? r : is_v ? r - p.Hq - p.Hkv : r - p.Hq) * D + d;
            held[u].load(src, from);
            if (!INTERLEAVED && !is_v && rotates) others[u].load(src, from + partner);
        }
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            const int r = r0 + u * step;
            if (r >= rows) break;
            const bool is_q = r < p.Hq, is_v = r >= p.Hq + p.Hkv;
            const int h = is_q ? r : is_v ? r - p.Hq - p.Hkv : r - p.Hq;
            Eight<F32>& own = held[u];
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = own.get(j);
            if (!is_v && rotates) {
                if constexpr (INTERLEAVED) {
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const float a = x[j], o = x[j + 1];
                        x[j] = turn(a, c[j / 2], o, -s[j / 2]);
                        x[j + 1] = turn(o, c[j / 2], a, s[j / 2]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = turn(x[j], c[j], others[u].get(j), s[j]);
                }
                own.set(x);
            }
            if constexpr (MX) {
                if (!is_q) {                       // (the lanes of a block are together: some of them may not have rotated, but none has left)
                    unsigned char* cache = static_cast<unsigned char*>(is_v ? p.v_cache : p.k_cache);
                    store_mx<D>(cache + page * p.page_stride + h * p.head_stride, is_v, in_page, lane, x);
                    continue;
                }
            }
            if (is_q) own.store(p.q_out, (token * p.Hq + h) * D + d);
            else own.store(is_v ? p.v_cache : p.k_cache, page * p.page_stride + in_page * p.token_stride + h * p.head_stride + d);
        }
    }
}

static bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
    const size_t x = reinterpret_cast<size_t>(a), y = reinterpret_cast<size_t>(b);
    return x < y + static_cast<size_t>(b_bytes) && y < x + static_cast<size_t>(a_bytes);
}

static int32_t kv_append(AppendParams& p, int32_t B, int32_t D, int32_t interleaved, int32_t dtype, bool mx, void* stream) {
    if (!p.k || !p.v || !p.k_cache || !p.v_cache || !p.block_table || !p.prefix_len || !p.n_nodes || !p.status) return GRAFT_ERR_NULL;
    if ((p.Hq > 0 && (!p.q || !p.q_out)) || (p.R > 0 && !p.cos_sin)) return GRAFT_ERR_NULL;
    if (dtype != GRAFT_F32 && dtype != GRAFT_BF16) return GRAFT_ERR_DTYPE;
    const int64_t align = dtype == GRAFT_F32 ? 4 : 8;          // 16-byte loads
    if (B < 1 || B > 65535 || p.T < 1 || p.Hq < 0 || p.Hq > 65535 || p.Hkv < 1 || p.Hkv > 65535 || (D != 64 && D != 128) || p.max_pages < 1 ||
        p.max_pages > 262144 || p.R < 0 || p.R > D || p.R % 16 != 0 || (p.R > 0 && p.n_pos < 1) || (interleaved != 0 && interleaved != 1) ||
        p.k_stride < static_cast<int64_t>(p.Hkv) * D || p.v_stride < static_cast<int64_t>(p.Hkv) * D || p.k_stride % align != 0 ||
        p.v_stride % align != 0 || (p.Hq > 0 && (p.q_stride < static_cast<int64_t>(p.Hq) * D || p.q_stride % align != 0)))
        return GRAFT_ERR_SHAPE;
    const int own = 64 / (D / 8);                              // tokens of a workgroup that does not share one with others
    if ((static_cast<int64_t>(p.T) + own - 1) / own >= (1ll << 32) / KA_THREADS) return GRAFT_ERR_SHAPE;         // (lanes of a launch)
    if (mx) {
        if (p.page_stride < mx_run_bytes(D) || p.head_stride < mx_run_bytes(D) || p.page_stride % 16 != 0 || p.head_stride % 16 != 0) return GRAFT_ERR_SHAPE;
    } else if (p.page_stride < 1 || p.token_stride < D || p.head_stride < D || p.page_stride % align != 0 || p.token_stride % align != 0 ||
               p.head_stride % align != 0) return GRAFT_ERR_SHAPE;
    size_t at = reinterpret_cast<size_t>(p.k) | reinterpret_cast<size_t>(p.v) | reinterpret_cast<size_t>(p.k_cache) | reinterpret_cast<size_t>(p.v_cache);
    if (p.Hq > 0) at |= reinterpret_cast<size_t>(p.q) | reinterpret_cast<size_t>(p.q_out);
    if (at & 15) return GRAFT_ERR_SHAPE;
    // A row of q is read and written by one wavefront, so q_out may be q; any other overlap would read what was written.
    const int64_t es = dtype == GRAFT_F32 ? 4 : 2, tokens = static_cast<int64_t>(B) * p.T;
    if (p.Hq > 0) {
        const bool in_place = p.q_out == p.q && p.q_stride == static_cast<int64_t>(p.Hq) * D;
        const int64_t out = tokens * p.Hq * D * es;
        auto spans = [&](int64_t stride, int64_t row) { return ((tokens - 1) * stride + row) * es; };
        if ((!in_place && overlap(p.q_out, out, p.q, spans(p.q_stride, static_cast<int64_t>(p.Hq) * D))) ||
            overlap(p.q_out, out, p.k, spans(p.k_stride, static_cast<int64_t>(p.Hkv) * D)) ||
            overlap(p.q_out, out, p.v, spans(p.v_stride, static_cast<int64_t>(p.Hkv) * D)))
            return GRAFT_ERR_SHAPE;
    }
    const int64_t cus = device_compute_units();
    const int per = tokens < 3 * own * cus / 4 || 2 * p.T < own ? 1 : own;                     // tokens of a workgroup, all of one sequence
    const bool share = per == 1;
    // Few tokens' rows go to several workgroups each, as long as there are compute units without one.
    const int64_t steps = (p.Hq + 2 * p.Hkv + KA_THREADS / (D / 8) - 1) / (KA_THREADS / (D / 8)), room = cus / tokens;
    const dim3 grid((p.T + per - 1) / per, B, !share || room < 2 ? 1 : room < steps ? room : steps);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(KA_THREADS), 0, static_cast<hipStream_t>(stream), p.prefix_len, p.n_nodes, p.pos, p.T, p);
    };
    auto pick = [&](auto d, auto f32, auto m) {
        if (interleaved) { if (share) launch(kv_append_kernel<d, f32, m, true, true>); else launch(kv_append_kernel<d, f32, m, true, false>); }
        else if (share) launch(kv_append_kernel<d, f32, m, false, true>);
        else launch(kv_append_kernel<d, f32, m, false, false>);
    };
    auto typed = [&](auto d) {
        using std::false_type;
        using std::true_type;
        if (dtype == GRAFT_F32) { if (mx) pick(d, true_type{}, true_type{}); else pick(d, true_type{}, false_type{}); }
        else if (mx) pick(d, false_type{}, true_type{});
        else pick(d, false_type{}, false_type{});
    };
    if (D == 64) typed(std::integral_constant<int, 64>{});
    else typed(std::integral_constant<int, 128>{});
    return check_launch();
}

}  // namespace graft

extern "C" int32_t graft_kv_append(const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                   const float* cos_sin, int32_t n_pos, int32_t rot_dim, int32_t interleaved, const int32_t* pos,
                                   void* k_cache, void* v_cache, int64_t page_stride, int64_t token_stride, int64_t head_stride,
                                   const int32_t* block_table, int32_t max_pages, const int32_t* prefix_len, const int32_t* n_nodes,
                                   int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t page_size, int32_t dtype,
                                   void* q_out, int32_t* status, void* stream) {
    if (page_size != GRAFT_PAGE_SIZE) return GRAFT_ERR_SHAPE;
    graft::AppendParams p{q, k, v, q_out, k_cache, v_cache, cos_sin, block_table, prefix_len, n_nodes, pos, status, q_stride, k_stride, v_stride,
                          page_stride, token_stride, head_stride, n_pos, rot_dim, max_pages, T, Hq, Hkv};
    return graft::kv_append(p, B, D, interleaved, dtype, false, stream);
}

extern "C" int32_t graft_kv_append_mx(const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                      const float* cos_sin, int32_t n_pos, int32_t rot_dim, int32_t interleaved, const int32_t* pos,
                                      void* k_cache, void* v_cache, int64_t page_stride, int64_t head_stride,
                                      const int32_t* block_table, int32_t max_pages, const int32_t* prefix_len, const int32_t* n_nodes,
                                      int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t page_size, int32_t dtype,
                                      void* q_out, int32_t* status, void* stream) {
    if (page_size != GRAFT_PAGE_SIZE) return GRAFT_ERR_SHAPE;
    graft::AppendParams p{q, k, v, q_out, k_cache, v_cache, cos_sin, block_table, prefix_len, n_nodes, pos, status, q_stride, k_stride, v_stride,
                          page_stride, 0, head_stride, n_pos, rot_dim, max_pages, T, Hq, Hkv};
    return graft::kv_append(p, B, D, interleaved, dtype, true, stream);
}
