// graft_tree_attn_mx: tree-masked attention over a cache of 4-bit elements (mx.h).
//
// For a row (node and query head) and its tokens t: x_t = scale q.k_t, or c tanh(x_t / c) with a cap c; out = sum p_t v_t / sum p_t,
// p_t = exp(x_t - m), in one pass over the keys with a running maximum m (kept where it is until a score exceeds it by 2^8:
// probabilities and sums are the same floating-point numbers up to a power of two).
//
// Scores: 4-bit keys enter the matrix cores as they are in memory (v_mfma_scale_f32_16x16x128_f8f6f4, 16 tokens x 16 rows x 128
// elements).  At the rate of 4 and 6 bits, twice that of 8, a query takes three e2m3 numbers of 6 bits: its block of 32 elements is scaled to
// (3.75, 7.5], the second holds what the first leaves, times 2^4, the third the rest, times 2^9.  Up to 2^-14 of the block's largest
// element is left out, less than the rounding of probabilities below makes of a score.  48 cycles, as bf16 operands take 64, and no
// conversion of keys.
// Values: scales are per token, the matrix cores' per 32 summands, so values are converted to bfloat16 (exact: one bit of mantissa and a
// power of two), probabilities are rounded to bfloat16 (2^-9 each, the choice of the kernels over bfloat16 caches), sums are float32.
// Scores come out of the matrix cores as D[token][row]: lane l has row l % 16, tokens 4 (l / 16) .. + 4 of each page; that is the layout in
// which the second product takes probabilities (with 8 tokens a lane, 4 from each of two pages), so nothing crosses lanes.
#include "mx.h"

namespace graft {

typedef int Int8 __attribute__((ext_vector_type(8)));
typedef unsigned UInt6 __attribute__((ext_vector_type(6)));
typedef unsigned UInt4 __attribute__((ext_vector_type(4)));
typedef unsigned UInt2 __attribute__((ext_vector_type(2)));
typedef float Float4 __attribute__((ext_vector_type(4)));
typedef float Float16 __attribute__((ext_vector_type(16)));
typedef float Float32 __attribute__((ext_vector_type(32)));
typedef __bf16 Bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 Bf8 __attribute__((ext_vector_type(8)));

constexpr int TM_WAVES = 4, TM_THREADS = 64 * TM_WAVES;
constexpr float TM_LOW = -3.402823466e38f;         // no score yet: below or equal to every finite score
constexpr float TM_SLACK = 8.0f;                   // powers of two by which a score may exceed the running maximum

struct AttnMxParams {
    const unsigned short* q;
    const unsigned char *k_cache, *v_cache;
    const int32_t *block_table, *pos;
    const u64* mask;
    unsigned short* out;
    float *partial, *stat;                         // [B,Hkv,S,rows] x D and x 2, where keys are split over workgroups
    int64_t page_stride, head_stride;              // bytes
    float factor, cap_in, cap_out;                 // of a raw score: to powers of two; with a cap 2 log2(e) / c, and c log2(e)
    int32_t sign;                                  // of the scale
    int32_t K, Hkv, G, max_pages, window, splits, row_tiles, items;
};

// One row's 32 elements of a lane in three parts of 6 bits, and the parts' scale bytes.
struct Query {
    UInt6 part[3];
    int bytes;
};
__device__ __forceinline__ Query split_query(const float* x) {
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const unsigned u = __float_as_uint(x[j]) & 0x7FFFFFFFu;
        top = u > top ? u : top;
    }
    int byte = static_cast<int>((top + 0x0FFFFFu) >> 23) - 2;      // (largest element within (3.75, 7.5] of it)
    byte = byte < 12 ? 12 : byte > 252 ? 252 : byte;
    Query q;
    float rest[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) rest[j] = x[j];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const float scale = mx_scale(byte - (i == 0 ? 0 : i == 1 ? 4 : 9));
        Float16 even, odd;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            even[j] = rest[2 * j];
            odd[j] = rest[2 * j + 1];
        }
        // These two conversions take several cycles and write their first results before they read their last operands, which the
        // compiler does not know: it placed the scale in a register of the result, and the third part of a query came out wrong.
        // The statements behind them keep the operands' registers in use until the results are there.
        q.part[i] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, scale);
        asm volatile("" : "+v"(q.part[i]) : "v"(even), "v"(odd), "v"(scale));
        if (i < 2) {
            Float32 held = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(q.part[i], scale);
            asm volatile("" : "+v"(held) : "v"(q.part[i]), "v"(scale));
#pragma unroll
            for (int j = 0; j < 32; ++j) rest[j] -= held[j];
        }
    }
    q.bytes = byte | (byte - 4) << 8 | (byte - 9) << 16;
    if (top >= 0x7F800000u) q.bytes = 0xFFFFFF;                    // an infinity or NaN makes NaN of the row's scores
    return q;
}

// Keys and values of NP pages as they are in memory, this lane's 16 bytes (values: 8 with D = 64) and scale bytes.
template <int D, int NP> struct Pages {
    using V = std::conditional_t<D == 128, UInt4, UInt2>;
    UInt4 k[NP];
    V v[NP];
    unsigned k_scale[NP], v_scale[NP];
};

template <int D, int MB, int NP, bool CAP>
__global__ __launch_bounds__(TM_THREADS, 2) void tree_attn_mx_kernel(const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ n_nodes,
                                                                     AttnMxParams p) {
    constexpr int TILES = D / 16, BLOCKS = D / 32;                 // tiles of the output; scale blocks of a row
    __shared__ float exchange[TM_WAVES * D / 16 * 4 * 64];
    __shared__ float stats[TM_WAVES][MB][16][2];
    // Workgroups that read the same keys for other rows run next to each other on the same XCD (ids 8 apart).
    const int id = blockIdx.x, item = id / (8 * p.row_tiles) * 8 + (id & 7), row_tile = (id >> 3) % p.row_tiles;
    if (item >= p.items) return;
    const int split = item % p.splits, g = item / p.splits % p.Hkv, b = item / p.splits / p.Hkv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row16 = lane & 15, quad = lane >> 4;
    int P = prefix_len[b], n = n_nodes[b];
    if (P < 0 || n < 0 || n > p.K || static_cast<int64_t>(P) + n > static_cast<int64_t>(p.max_pages) * GRAFT_PAGE_SIZE) n = 0;
    const int rows = n * p.G, all_rows = p.K * p.G, row0 = row_tile * 16 * MB, L = P + n;
    const int64_t out_b = static_cast<int64_t>(b) * p.K * p.Hkv * p.G * D;
    auto out_at = [&](int row) {
        const int node = row / p.G;
        return out_b + (static_cast<int64_t>(node) * p.Hkv * p.G + g * p.G + (row - node * p.G)) * D;
    };
    if (row0 >= rows) {                                            // uniform: padding nodes only
        if (p.splits == 1)
            for (int i = threadIdx.x; i < 16 * MB * (D / 8); i += TM_THREADS) {
                const int row = row0 + i / (D / 8);
                if (row < all_rows) *reinterpret_cast<UInt4*>(p.out + out_at(row) + i % (D / 8) * 8) = UInt4{0, 0, 0, 0};
            }
        return;
    }

    // queries
    Query query[MB];
    int node[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int row = row0 + mb * 16 + row16;
        node[mb] = row < rows ? row / p.G : 0;
        float x[32];
        const bool there = row < rows && quad < BLOCKS;
        const UInt4* src = reinterpret_cast<const UInt4*>(p.q + (there ? out_at(row) + quad * 32 : 0));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const UInt4 u = src[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[i * 8 + j * 2] = there ? __uint_as_float(u[j] << 16) * p.sign : 0.0f;
                x[i * 8 + j * 2 + 1] = there ? __uint_as_float(u[j] & 0xFFFF0000u) * p.sign : 0.0f;
            }
        }
        query[mb] = split_query(x);
    }

    // the pages that some node sees, and from which token on every node sees all of the prefix
    const int32_t* pos = p.pos ? p.pos + static_cast<int64_t>(b) * p.K : nullptr;
    int first_page = 0, all_see = 0;
    if (p.window > 0) {
        int low = 0x7FFFFFFF, high = -0x7FFFFFFF;
        for (int i = lane; i < n; i += 64) {
            const int at = pos ? pos[i] : P + i;
            low = at < low ? at : low;
            high = at > high ? at : high;
        }
#pragma unroll
        for (int s = 32; s > 0; s >>= 1) {
            const int l2 = __shfl_xor(low, s), h2 = __shfl_xor(high, s);
            low = l2 < low ? l2 : low;
            high = h2 > high ? h2 : high;
        }
        const int64_t from = static_cast<int64_t>(low) - p.window + 1, all = static_cast<int64_t>(high) - p.window + 1;
        const int64_t from_in = from < 0 ? 0 : from > P ? P : from;
        first_page = __builtin_amdgcn_readfirstlane(static_cast<int>(from_in) / GRAFT_PAGE_SIZE);
        all_see = __builtin_amdgcn_readfirstlane(static_cast<int>(all < 0 ? 0 : all > P ? P : all));
    }
    const int end_page = (L + GRAFT_PAGE_SIZE - 1) / GRAFT_PAGE_SIZE;
    const int tiles = (end_page - first_page + NP - 1) / NP;
    const int tile_end = static_cast<int>(static_cast<int64_t>(tiles) * (split + 1) / p.splits);
    int tile = static_cast<int>(static_cast<int64_t>(tiles) * split / p.splits) + wave;

    const int32_t* table = p.block_table + static_cast<int64_t>(b) * p.max_pages;
    const unsigned char *k_head = p.k_cache + g * p.head_stride, *v_head = p.v_cache + g * p.head_stride;
    const int k_block = quad & (BLOCKS - 1);                       // (D = 64: lanes past the row's end have zeros of the query)
    const int k_at = row16 * (D / 2) + k_block * 16, ks_at = mx_scale_at<D>(row16, k_block);
    const int v_at = lane * (D / 8), vs_at = mx_scale_at<D>(quad * 4, row16 * TILES / 32);
    using Held = Pages<D, NP>;
    auto load = [&](int t) {
        Held h;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int at = first_page + t * NP + i;
            const int64_t page = static_cast<int64_t>(table[at < end_page ? at : end_page - 1]) * p.page_stride;
            const unsigned char *k = k_head + page, *v = v_head + page;
            h.k[i] = *reinterpret_cast<const UInt4*>(k + k_at);
            h.k_scale[i] = k[ks_at];
            h.v[i] = *reinterpret_cast<const typename Held::V*>(v + v_at);
            h.v_scale[i] = *reinterpret_cast<const unsigned*>(v + vs_at);
        }
        return h;
    };

    Float4 acc[MB][TILES];
    float top[MB], sum[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        top[mb] = TM_LOW;
        sum[mb] = 0.0f;
#pragma unroll
        for (int m = 0; m < TILES; ++m) acc[mb][m] = Float4{0, 0, 0, 0};
    }

    auto step = [&](int t, Held& h) {
        const int first = (first_page + t * NP) * GRAFT_PAGE_SIZE;
        const bool masked = first + NP * GRAFT_PAGE_SIZE > P || first < all_see;
        unsigned no_number = 0;                                    // bit 4 i + r: a value of token 4 quad + r of page i is none
        if (masked) {
            // Values of tokens behind the last one and values that are no numbers become small ones, which a probability of 0
            // takes out; rows that see one of the latter get NaN as its score.
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int at = first_page + t * NP + i, token = first + i * GRAFT_PAGE_SIZE + quad * 4;
                const unsigned char* v = v_head + static_cast<int64_t>(table[at < end_page ? at : end_page - 1]) * p.page_stride;
                unsigned any = 0;
#pragma unroll
                for (int c = 0; c < BLOCKS; ++c) {
                    const unsigned s4 = *reinterpret_cast<const unsigned*>(v + mx_scale_at<D>(quad * 4, c));
#pragma unroll
                    for (int r = 0; r < 4; ++r) any |= ((s4 >> (8 * r)) & 255u) == MX_NAN ? 1u << r : 0u;
                }
                no_number |= any << (4 * i);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (token + r >= L || (any >> r & 1)) h.v_scale[i] = (h.v_scale[i] & ~(255u << (8 * r))) | 2u << (8 * r);
            }
        }
        Bf8 prob[MB][NP / 2];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            Float4 s[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const Int8 key = {static_cast<int>(h.k[i][0]), static_cast<int>(h.k[i][1]), static_cast<int>(h.k[i][2]), static_cast<int>(h.k[i][3]), 0, 0, 0, 0};
                auto part = [&](int j) {
                    const UInt6 u = query[mb].part[j];
                    return Int8{static_cast<int>(u[0]), static_cast<int>(u[1]), static_cast<int>(u[2]), static_cast<int>(u[3]),
                                static_cast<int>(u[4]), static_cast<int>(u[5]), 0, 0};
                };
                s[i] = Float4{0, 0, 0, 0};
                s[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(key, part(2), s[i], 4, 2, 0, h.k_scale[i], 2, query[mb].bytes);
                s[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(key, part(1), s[i], 4, 2, 0, h.k_scale[i], 1, query[mb].bytes);
                s[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(key, part(0), s[i], 4, 2, 0, h.k_scale[i], 0, query[mb].bytes);
            }
            if constexpr (CAP) {
#pragma unroll
                for (int i = 0; i < NP; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        s[i][r] = __builtin_fmaf(__builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[i][r] * p.cap_in) + 1.0f), -2.0f * p.cap_out, p.cap_out);
            }
            if (masked) {
                u64 word[2] = {~0ull, ~0ull};
                if (p.mask) {
                    const u64* w = p.mask + (static_cast<int64_t>(b) * p.K + node[mb]) * GRAFT_MASK_WORDS;
                    word[0] = w[0];
                    word[1] = w[1];
                }
                const int at = p.window > 0 ? pos ? pos[node[mb]] : P + node[mb] : 0;
#pragma unroll
                for (int i = 0; i < NP; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int token = first + i * GRAFT_PAGE_SIZE + quad * 4 + r, j = token - P;
                        bool sees = token < P;
                        if (token >= P && j < n) sees = p.mask ? (word[j >> 6] >> (j & 63)) & 1 : j <= node[mb];
                        if (p.window > 0 && sees) {
                            const int64_t place = token < P ? token : pos ? pos[j] : token;
                            sees = at - place < p.window;
                        }
                        s[i][r] = !sees ? -__builtin_inff() : (no_number >> (4 * i + r) & 1) ? __builtin_nanf("") : s[i][r];
                    }
            }
            float most = s[0][0];
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) most = __builtin_fmaxf(most, s[i][r]);
            if constexpr (!CAP) most *= p.factor;
            most = rows_max_f32(most);
            if (__builtin_amdgcn_ballot_w64(most > top[mb] + TM_SLACK) != 0) {
                const float now = __builtin_fmaxf(most, top[mb]), shrink = __builtin_amdgcn_exp2f(top[mb] - now);
                top[mb] = now;
                sum[mb] *= shrink;
#pragma unroll
                for (int m = 0; m < TILES; ++m) acc[mb][m] *= shrink;
            }
            float x[NP][4];
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[i][r] = __builtin_amdgcn_exp2f(CAP ? s[i][r] - top[mb] : __builtin_fmaf(s[i][r], p.factor, -top[mb]));
                    sum[mb] += x[i][r];
                }
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) prob[mb][i / 2][(i & 1) * 4 + r] = static_cast<__bf16>(x[i][r]);
        }
        // values: two neighbouring tiles come out of a conversion, four tokens each of two pages make an operand
#pragma unroll
        for (int i2 = 0; i2 < NP / 2; ++i2) {
            float scale[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) scale[i][r] = mx_scale((h.v_scale[2 * i2 + i] >> (8 * r)) & 255u);
            auto tiles_of = [&](auto pair) {
                constexpr int M = decltype(pair)::value;
                unsigned lo[4], hi[4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    unsigned c[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if constexpr (D == 128) c[r] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(h.v[2 * i2 + i][r], scale[i][r], M));
                        else if (r & 1) c[r] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(h.v[2 * i2 + i][r / 2], scale[i][r], 2 + M));
                        else c[r] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(h.v[2 * i2 + i][r / 2], scale[i][r], M));
                    }
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        lo[2 * i + r] = __builtin_amdgcn_perm(c[2 * r + 1], c[2 * r], 0x05040100);
                        hi[2 * i + r] = __builtin_amdgcn_perm(c[2 * r + 1], c[2 * r], 0x07060302);
                    }
                }
                const Bf8 even = __builtin_bit_cast(Bf8, UInt4{lo[0], lo[1], lo[2], lo[3]}), odd = __builtin_bit_cast(Bf8, UInt4{hi[0], hi[1], hi[2], hi[3]});
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                    acc[mb][2 * M] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, prob[mb][i2], acc[mb][2 * M], 0, 0, 0);
                    acc[mb][2 * M + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, prob[mb][i2], acc[mb][2 * M + 1], 0, 0, 0);
                }
            };
            tiles_of(std::integral_constant<int, 0>{});
            tiles_of(std::integral_constant<int, 1>{});
            if constexpr (TILES > 4) {
                tiles_of(std::integral_constant<int, 2>{});
                tiles_of(std::integral_constant<int, 3>{});
            }
        }
    };

    if (tile < tile_end) {
        Held here = load(tile);
        for (; tile < tile_end; tile += TM_WAVES) {
            const int next = tile + TM_WAVES;
            Held ahead = load(next < tile_end ? next : tile);
            step(tile, here);
            here = ahead;
        }
    }

    // The wavefronts' sums are brought to the rows' common maximum and added: wavefront w takes the elements whose place in
    // their tile is 4 quad + w, D / 16 neighbours in the row.
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        float s = sum[mb];
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (quad == 0) {
            stats[wave][mb][row16][0] = top[mb];
            stats[wave][mb][row16][1] = s;
        }
    }
    __syncthreads();
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        float most = TM_LOW, total = 0.0f;
#pragma unroll
        for (int w = 0; w < TM_WAVES; ++w) most = __builtin_fmaxf(most, stats[w][mb][row16][0]);
#pragma unroll
        for (int w = 0; w < TM_WAVES; ++w) total += stats[w][mb][row16][1] * __builtin_amdgcn_exp2f(stats[w][mb][row16][0] - most);
        const float shrink = __builtin_amdgcn_exp2f(top[mb] - most);
        if (mb > 0) __syncthreads();
#pragma unroll
        for (int m = 0; m < TILES; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) exchange[((wave * TILES + m) * 4 + r) * 64 + lane] = acc[mb][m][r] * shrink;
        __syncthreads();
        float o[TILES];
#pragma unroll
        for (int m = 0; m < TILES; ++m) {
            o[m] = 0.0f;
#pragma unroll
            for (int w = 0; w < TM_WAVES; ++w) o[m] += exchange[((w * TILES + m) * 4 + wave) * 64 + lane];
        }
        const int row = row0 + mb * 16 + row16, d = (quad * 4 + wave) * TILES;
        if (row >= all_rows) continue;
        if (p.splits == 1) {
            const float inv = total == 0.0f || row >= rows ? 0.0f : 1.0f / total;
            unsigned packed[TILES / 2];
#pragma unroll
            for (int m = 0; m < TILES; m += 2) {
                const Bf2 two = {static_cast<__bf16>(row < rows ? o[m] * inv : 0.0f), static_cast<__bf16>(row < rows ? o[m + 1] * inv : 0.0f)};
                packed[m / 2] = __builtin_bit_cast(unsigned, two);
            }
            if constexpr (D == 128) *reinterpret_cast<UInt4*>(p.out + out_at(row) + d) = UInt4{packed[0], packed[1], packed[2], packed[3]};
            else *reinterpret_cast<UInt2*>(p.out + out_at(row) + d) = UInt2{packed[0], packed[1]};
        } else if (row < rows) {
            const int64_t at = static_cast<int64_t>(item) * all_rows + row;
            Float4* dst = reinterpret_cast<Float4*>(p.partial + at * D + d);
#pragma unroll
            for (int m = 0; m < TILES / 4; ++m) dst[m] = Float4{o[4 * m], o[4 * m + 1], o[4 * m + 2], o[4 * m + 3]};
            if (wave == 0 && quad == 0) *reinterpret_cast<float2*>(p.stat + at * 2) = float2{most, total};
        }
    }
}

// The splits' sums of a row, 8 elements a lane.
template <int D>
__global__ __launch_bounds__(TM_THREADS) void tree_attn_mx_merge_kernel(const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ n_nodes,
                                                                        AttnMxParams p) {
    constexpr int LANES = D / 8;
    const int b = blockIdx.z, g = blockIdx.y, row = blockIdx.x * (TM_THREADS / LANES) + threadIdx.x / LANES, d = threadIdx.x % LANES * 8;
    const int all_rows = p.K * p.G;
    if (row >= all_rows) return;
    const int P = prefix_len[b];
    int n = n_nodes[b];
    if (P < 0 || n < 0 || n > p.K || static_cast<int64_t>(P) + n > static_cast<int64_t>(p.max_pages) * GRAFT_PAGE_SIZE) n = 0;
    float o[8] = {0, 0, 0, 0, 0, 0, 0, 0}, total = 0.0f;
    if (row < n * p.G) {
        const int64_t base = static_cast<int64_t>(b * p.Hkv + g) * p.splits * all_rows + row;
        float most = TM_LOW;
        for (int s = 0; s < p.splits; ++s) most = __builtin_fmaxf(most, p.stat[(base + static_cast<int64_t>(s) * all_rows) * 2]);
        for (int s = 0; s < p.splits; ++s) {
            const int64_t at = base + static_cast<int64_t>(s) * all_rows;
            const float2 st = *reinterpret_cast<const float2*>(p.stat + at * 2);
            const Float4 *src = reinterpret_cast<const Float4*>(p.partial + at * D + d), x = src[0], y = src[1];
            const float w = __builtin_amdgcn_exp2f(st.x - most);
            total += st.y * w;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                o[j] += x[j] * w;
                o[4 + j] += y[j] * w;
            }
        }
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const int node = row / p.G;
    unsigned packed[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const Bf2 two = {static_cast<__bf16>(o[2 * j] * inv), static_cast<__bf16>(o[2 * j + 1] * inv)};
        packed[j] = __builtin_bit_cast(unsigned, two);
    }
    const int64_t at = ((static_cast<int64_t>(b) * p.K + node) * p.Hkv * p.G + g * p.G + (row - node * p.G)) * D + d;
    *reinterpret_cast<UInt4*>(p.out + at) = UInt4{packed[0], packed[1], packed[2], packed[3]};
}

// ---- plan --------------------------------------------------------------------------------------------------------------------------
struct AttnMxPlan { int row_blocks, row_tiles, splits; };

static int compute_units() {
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) {
        (void)hipGetLastError();                   // (no device: sizes are asked for all the same)
        return 256;
    }
    return n;
}

static AttnMxPlan plan_attn_mx(int32_t B, int32_t K, int32_t Hq, int32_t Hkv, int32_t max_pages) {
    const int rows = K * (Hq / Hkv);
    AttnMxPlan best{1, (rows + 15) / 16, 1};
    if (rows > 16) best = {2, (rows + 31) / 32, 1};
    const int64_t groups = static_cast<int64_t>(B) * Hkv * best.row_tiles;
    // two workgroups a compute unit; a split has at least two tiles of four pages for each wavefront
    const int64_t fill = 2 * compute_units(), most = (max_pages + 31) / 32;
    int64_t s = groups >= fill ? 1 : fill / groups;
    if (s > most) s = most;
    if (s > 64) s = 64;
    if (s < 1) s = 1;
    best.splits = static_cast<int>(s);
    return best;
}

static bool bad_attn_mx_shape(int32_t B, int32_t K, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_pages) {
    return B < 1 || B > 65535 || K < 1 || K > GRAFT_MAX_NODES || Hkv < 1 || Hkv > 65535 || Hq < Hkv || Hq % Hkv != 0 || Hq / Hkv > 16 ||
           (D != 64 && D != 128) || max_pages < 1 || max_pages > 262144 || static_cast<int64_t>(B) * Hkv > (1 << 22);
}

static size_t attn_mx_bytes(const AttnMxPlan& plan, int32_t B, int32_t K, int32_t Hq, int32_t D) {
    return plan.splits == 1 ? 0 : static_cast<size_t>(B) * K * Hq * plan.splits * (D + 2) * 4;
}

}  // namespace graft

extern "C" size_t graft_tree_attn_mx_workspace_bytes(int32_t B, int32_t K_max, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_pages) {
    using namespace graft;
    if (bad_attn_mx_shape(B, K_max, Hq, Hkv, D, max_pages)) return 0;
    return attn_mx_bytes(plan_attn_mx(B, K_max, Hq, Hkv, max_pages), B, K_max, Hq, D);
}

extern "C" int32_t graft_tree_attn_mx(const void* q, const void* k_cache, const void* v_cache, int64_t page_stride, int64_t head_stride,
                                      const int32_t* block_table, int32_t max_pages, const int32_t* prefix_len, const int32_t* n_nodes,
                                      const uint64_t* mask, const int32_t* pos, int32_t B, int32_t K_max, int32_t Hq, int32_t Hkv, int32_t D,
                                      int32_t page_size, float scale, float softcap, int32_t window, void* out, void* workspace,
                                      size_t workspace_bytes, void* stream) {
    using namespace graft;
    if (!q || !k_cache || !v_cache || !block_table || !prefix_len || !n_nodes || !out) return GRAFT_ERR_NULL;
    if (window > 0 && mask && !pos) return GRAFT_ERR_NULL;
    if (page_size != GRAFT_PAGE_SIZE || bad_attn_mx_shape(B, K_max, Hq, Hkv, D, max_pages) || page_stride < mx_run_bytes(D) ||
        head_stride < mx_run_bytes(D) || page_stride % 16 != 0 || head_stride % 16 != 0 || window < 0)
        return GRAFT_ERR_SHAPE;
    if (!(scale - scale == 0.0f) || !(softcap - softcap == 0.0f) || softcap < 0.0f) return GRAFT_ERR_SHAPE;
    if ((reinterpret_cast<size_t>(q) | reinterpret_cast<size_t>(k_cache) | reinterpret_cast<size_t>(v_cache) | reinterpret_cast<size_t>(out)) & 15)
        return GRAFT_ERR_SHAPE;
    const AttnMxPlan plan = plan_attn_mx(B, K_max, Hq, Hkv, max_pages);
    const size_t need = attn_mx_bytes(plan, B, K_max, Hq, D);
    if (need > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<size_t>(workspace) & 15))) return GRAFT_ERR_WORKSPACE;
    constexpr float LOG2E = 1.44269504088896340736f;
    AttnMxParams p{};
    p.q = static_cast<const unsigned short*>(q);
    p.k_cache = static_cast<const unsigned char*>(k_cache);
    p.v_cache = static_cast<const unsigned char*>(v_cache);
    p.block_table = block_table;
    p.pos = pos;
    p.mask = reinterpret_cast<const u64*>(mask);
    p.out = static_cast<unsigned short*>(out);
    p.partial = static_cast<float*>(workspace);
    p.stat = p.partial + static_cast<size_t>(B) * K_max * Hq * plan.splits * D;
    p.page_stride = page_stride;
    p.head_stride = head_stride;
    const float size = scale < 0.0f ? -scale : scale;
    p.sign = scale > 0.0f ? 1 : scale < 0.0f ? -1 : 0;             // (the running maximum is one of raw scores: their factor is positive)
    p.factor = p.sign == 0 ? 1.0f : size * LOG2E;
    if (softcap > 0.0f) {
        p.cap_in = 2.0f * LOG2E * size / softcap;
        p.cap_out = softcap * LOG2E;
    }
    p.K = K_max; p.Hkv = Hkv; p.G = Hq / Hkv; p.max_pages = max_pages; p.window = window; p.splits = plan.splits; p.row_tiles = plan.row_tiles;
    p.items = B * Hkv * plan.splits;
    const int64_t blocks = (static_cast<int64_t>(p.items) + 7) / 8 * 8 * plan.row_tiles;
    if (blocks > 0x7FFFFFFF) return GRAFT_ERR_SHAPE;
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(TM_THREADS), 0, static_cast<hipStream_t>(stream), prefix_len, n_nodes, p);
    };
    auto sized = [&](auto d) {
        constexpr int DIM = decltype(d)::value;
        if (softcap > 0.0f) { if (plan.row_blocks == 1) launch(tree_attn_mx_kernel<DIM, 1, 4, true>); else launch(tree_attn_mx_kernel<DIM, 2, 4, true>); }
        else if (plan.row_blocks == 1) launch(tree_attn_mx_kernel<DIM, 1, 4, false>);
        else launch(tree_attn_mx_kernel<DIM, 2, 4, false>);
    };
    if (D == 128) sized(std::integral_constant<int, 128>{});
    else sized(std::integral_constant<int, 64>{});
    const int32_t rc = check_launch();
    if (rc != GRAFT_OK || plan.splits == 1) return rc;
    const int per = TM_THREADS / (D / 8);
    const dim3 grid((K_max * p.G + per - 1) / per, Hkv, B);
    if (D == 128) hipLaunchKernelGGL(tree_attn_mx_merge_kernel<128>, grid, dim3(TM_THREADS), 0, static_cast<hipStream_t>(stream), prefix_len, n_nodes, p);
    else hipLaunchKernelGGL(tree_attn_mx_merge_kernel<64>, grid, dim3(TM_THREADS), 0, static_cast<hipStream_t>(stream), prefix_len, n_nodes, p);
    return check_launch();
}
