// graft_tree_attn_mx: tree-masked attention over a cache of 4-bit elements (mx.h).
//
// For a row (node and query head) and its tokens t: x_t = scale q.k_t, or c tanh(x_t / c) with a cap c; out = sum p_t v_t / sum p_t,
// p_t = exp(x_t - m), in one pass over the keys with a running maximum m.
//
// Scores: 4-bit keys enter the matrix cores as they are in memory (v_mfma_scale_f32_16x16x128_f8f6f4, 16 tokens x 16 rows x 128
// elements).  At the rate of 4 and 6 bits, twice that of 8, a query takes three e2m3 numbers of 6 bits: its block of 32 elements is scaled to
// (3.75, 7.5], the second holds what the first leaves, times 2^4, the third the rest, times 2^9.  Up to 2^-14 of the block's largest
// element is left out, less than the rounding of probabilities below makes of a score.  48 cycles, as bf16 operands take 64, and no
// conversion of keys.
// Values: scales are per token, the matrix cores' per 32 summands, so values are converted to bfloat16 (exact: one bit of mantissa and a
// power of two), probabilities are rounded to bfloat16 (2^-8 of each, the choice of the kernels over bfloat16 caches), sums are float32.
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
constexpr int TM_MAX_SPLITS = 64;
constexpr int64_t TM_CACHED = 208ll << 20;         // bytes that the Infinity Cache keeps between launches
constexpr float TM_LOW = -3.402823466e38f;         // no score yet: below or equal to every finite score
constexpr float TM_MOST = 4096.0f;                 // sum of a lane's probabilities of a tile from which on the maximum is raised

struct AttnMxParams {
    const unsigned short* q;
    const unsigned char *k_cache, *v_cache;
    const int32_t* pos;
    const u64* mask;
    unsigned short* out;
    float *partial, *stat;                         // [B,Hkv,S,rows] x D and x 2, where keys are split over workgroups
    int64_t head_stride;                           // bytes
    unsigned page_stride;
    float factor, cap;                             // of queries, so that scores are powers of two, or with a cap c 2 x / c is one; c log2(e)
    unsigned per_group;                            // rows to nodes: 2^16 / G, rounded up
    int32_t K, Hkv, G, max_pages, window, splits, row_tiles, waves, items;       // (waves: of a workgroup, that have rows)
};

// One row's 32 elements of a lane in three parts of 6 bits, and the parts' scale bytes.
struct Query {
    UInt6 part[3];
    int bytes;
};
__device__ __forceinline__ Query split_query(const UInt4 (&raw)[4], float factor) {        // 32 elements of bfloat16, times the factor
    typedef unsigned short Short2 __attribute__((ext_vector_type(2)));
    Short2 most = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(Short2, raw[i][j] & 0x7FFF7FFFu));
    const unsigned top = __float_as_uint(__uint_as_float(static_cast<unsigned>(most[0] > most[1] ? most[0] : most[1]) << 16) * factor) & 0x7FFFFFFFu;
    int byte = static_cast<int>((top + 0x0FFFFFu) >> 23) - 2;      // (largest element within (3.75, 7.5] of it)
    byte = byte < 12 ? 12 : byte > 252 ? 252 : byte;
    Query q;
    Float16 even, odd;                             // elements 2 j, 2 j + 1
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        even[j] = __uint_as_float(raw[j / 4][j % 4] << 16) * factor;
        odd[j] = __uint_as_float(raw[j / 4][j % 4] & 0xFFFF0000u) * factor;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        float scale = mx_scale(byte - (i == 0 ? 0 : i == 1 ? 4 : 9));
        // These two conversions take several cycles and write their first results before they read their last operands, which the
        // compiler does not know: it placed the scale in a register of the result, and the third part of a query came out wrong.
        // The statements behind them keep the operands' registers in use until the results are there; the build looks whether they are.
        q.part[i] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, scale);
        asm volatile("" : "+v"(q.part[i]) : "v"(even), "v"(odd), "v"(scale));
        if (i < 2) {
            Float32 held = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(q.part[i], scale);
            asm volatile("" : "+v"(held) : "v"(q.part[i]), "v"(scale));
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                even[j] -= held[2 * j];
                odd[j] -= held[2 * j + 1];
            }
        }
    }
    q.bytes = byte | (byte - 4) << 8 | (byte - 9) << 16;
    if (top >= 0x7F800000u) q.bytes = 0xFFFFFF;                    // an infinity or NaN makes NaN of the row's scores
    return q;
}

// What a workgroup knows of its sequence.
struct Sequence {
    int P, n, L, rows, all_rows;                   // prefix, nodes, their sum; rows (node, head of the group) that are there, and slots
    int first_page, end_page, all_see;             // pages that some node sees; the first token from which on every node sees all of the prefix
    bool deep;                                     // some node does not see an ancestor any more
    const int32_t *table, *pos;
    const u64* mask;
    int64_t out;                                   // element of the sequence's first row
};

__device__ __forceinline__ Sequence sequence_of(int b, int P, int n, const int32_t* block_table, const AttnMxParams& p, int D) {
    Sequence q;
    if (P < 0 || n < 0 || n > p.K || static_cast<int64_t>(P) + n > static_cast<int64_t>(p.max_pages) * GRAFT_PAGE_SIZE) n = 0;
    q.P = P;
    q.n = n;
    q.L = P + n;
    q.rows = n * p.G;
    q.all_rows = p.K * p.G;
    q.table = block_table + static_cast<int64_t>(b) * p.max_pages;
    q.pos = p.pos ? p.pos + static_cast<int64_t>(b) * p.K : nullptr;
    q.mask = p.mask ? p.mask + static_cast<int64_t>(b) * p.K * GRAFT_MASK_WORDS : nullptr;
    q.out = static_cast<int64_t>(b) * p.K * p.Hkv * p.G * D;
    q.first_page = 0;
    q.all_see = 0;
    q.deep = false;
    q.end_page = (q.L + GRAFT_PAGE_SIZE - 1) / GRAFT_PAGE_SIZE;
    return q;
}

// With a window: the pages in front of every node's are left out.
__device__ __forceinline__ void look_back(Sequence& q, int window, int lane) {
    int low = 0x7FFFFFFF, high = -0x7FFFFFFF;
    for (int i = lane; i < q.n; i += 64) {
        const int at = q.pos ? q.pos[i] : q.P + i;
        low = at < low ? at : low;
        high = at > high ? at : high;
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
        const int l2 = __shfl_xor(low, s), h2 = __shfl_xor(high, s);
        low = l2 < low ? l2 : low;
        high = h2 > high ? h2 : high;
    }
    const int64_t from = static_cast<int64_t>(low) - window + 1, all = static_cast<int64_t>(high) - window + 1;
    q.first_page = __builtin_amdgcn_readfirstlane(static_cast<int>(from < 0 ? 0 : from > q.P ? q.P : from) / GRAFT_PAGE_SIZE);
    q.all_see = __builtin_amdgcn_readfirstlane(static_cast<int>(all < 0 ? 0 : all > q.P ? q.P : all));
    q.deep = __builtin_amdgcn_readfirstlane(static_cast<int64_t>(high) - low >= window) != 0;
}

// row / G: rows are fewer than 2^11 and G is 16 at most, so the product is less than 1 / 32 above the quotient's 1 / G steps.
static_assert(GRAFT_MAX_NODES * 16 <= 2048, "the division of rows by heads");
__device__ __forceinline__ int node_of(const AttnMxParams& p, int row) { return static_cast<int>((static_cast<unsigned>(row) * p.per_group) >> 16); }

// Element of a row of KV head g in q and out.
__device__ __forceinline__ int64_t row_at(const Sequence& q, const AttnMxParams& p, int g, int row, int D) {
    const int node = node_of(p, row);
    return q.out + (static_cast<int64_t>(node) * p.Hkv * p.G + g * p.G + (row - node * p.G)) * D;
}

// A split's units (tiles or stages of `tokens` tokens): those in front of `whole` and from `whole_end` on (where windows begin, and at the tree) are not
// seen whole by every node.  They are taken from `whole` on, around the end to the first ones: sums over keys have no order, and so one
// loop without masks and one with them see to all.
struct Units {
    int first, count, whole, whole_end;            // first unit of all; the rest counted from it
    __device__ __forceinline__ Units(const Sequence& q, int tokens, int split, int splits) {
        const int per = tokens / GRAFT_PAGE_SIZE, units = (q.end_page - q.first_page + per - 1) / per, base = q.first_page * GRAFT_PAGE_SIZE;
        // (2^18 units, 2^8 splits at most)
        first = static_cast<int>(static_cast<unsigned>(units) * static_cast<unsigned>(split) / static_cast<unsigned>(splits));
        count = static_cast<int>(static_cast<unsigned>(units) * static_cast<unsigned>(split + 1) / static_cast<unsigned>(splits)) - first;
        whole = min(max((max(q.all_see - base, 0) + tokens - 1) / tokens - first, 0), count);
        whole_end = max(min(max(q.P - base, 0) / tokens - first, count), whole);
    }
    __device__ __forceinline__ int end() const { return whole + count; }
    __device__ __forceinline__ int unit(int i) const { return i < count ? i : i - count; }
};

// The page numbers of the units: lane j of `here` has that of page 64 block + j (counted from the first unit's), of `next` that of the block behind it,
// on its way since the last change of blocks.  A number is read across lanes, without a trip to memory in front of the
// loads that it addresses.
struct PageIds {
    const int32_t* table;
    int last, lane, block, here, next;             // the last page there is; pages past it are taken for it
    __device__ __forceinline__ PageIds(const Sequence& q, int first_page, int lane_) : table(q.table + first_page), last(q.end_page - 1 - first_page), lane(lane_), block(0) {
        here = load(0);
        next = load(1);
    }
    __device__ __forceinline__ int load(int b) const { return table[min(64 * b + lane, last)]; }
    __device__ __forceinline__ void seek(int page) {                // uniform
        const int b = page >> 6;
        if (b == block) return;
        here = b == block + 1 ? next : load(b);
        next = load(b + 1);
        block = b;
    }
    __device__ __forceinline__ u64 offset(int page, unsigned stride) const {
        return static_cast<u64>(static_cast<unsigned>(__builtin_amdgcn_readlane(here, page & 63))) * stride;
    }
};

// Zeros for a tile of rows of padding nodes.
__device__ __forceinline__ void zero_rows(const Sequence& q, const AttnMxParams& p, int g, int row0, int count, int D) {
    for (int i = threadIdx.x; i < count * (D / 8); i += blockDim.x) {
        const int row = row0 + i / (D / 8);
        if (row < q.all_rows) *reinterpret_cast<UInt4*>(p.out + row_at(q, p, g, row, D) + i % (D / 8) * 8) = UInt4{0, 0, 0, 0};
    }
}

// 32 elements of a row's query from `from` on; zeros past the row's end.  Rows that are not there get padding's or some row's, so that the load need
// not wait for the sequence's length: what comes of it stays in their column of the products, and they have no vote in to_probabilities.
template <int D> __device__ __forceinline__ Query load_query(const Sequence& q, const AttnMxParams& p, int g, int row, int from) {
    const bool there = from < D;
    const UInt4* src = reinterpret_cast<const UInt4*>(p.q + row_at(q, p, g, row < q.all_rows ? row : 0, D) + (there ? from : 0));
    UInt4 raw[4];
    const unsigned keep = there ? ~0u : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = src[i] & keep;
    return split_query(raw, p.factor);
}

// Where a lane's bytes of a run are.
template <int D> struct LaneAt {
    unsigned k, k_scale, v, v_scale;
    __device__ __forceinline__ explicit LaneAt(int lane) {
        const int row16 = lane & 15, quad = lane >> 4, block = quad & (D / 32 - 1);   // (D = 64: lanes past the row's end have zeros of the query)
        k = row16 * (D / 2) + block * 16;
        k_scale = mx_scale_at<D>(row16, block);
        v = lane * (D / 8);
        v_scale = mx_scale_at<D>(quad * 4, row16 * (D / 16) / 32);
    }
};

// A run as a buffer: one base for all lanes, 32 bits of offset in each, and nothing outside it is read.
template <int D> __device__ __forceinline__ __amdgpu_buffer_rsrc_t run_of(const unsigned char* base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, mx_run_bytes(D), 0x00020000);
}

// A lane's bytes of a page's values.
template <int D> struct ValuePage {
    using V = std::conditional_t<D == 128, UInt4, UInt2>;
    V four;
    unsigned scale;
    template <int AUX = 0> __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t run, unsigned at, unsigned scale_at) {
        if constexpr (D == 128) four = __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(run, at, 0, AUX));
        else four = __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b64(run, at, 0, AUX));
        scale = __builtin_amdgcn_raw_buffer_load_b32(run, scale_at, 0, AUX);
    }
    // Values of tokens behind the last one and values that are, or may be, infinite or no numbers become small ones, which a probability of 0 takes out.
    __device__ __forceinline__ void keep_numbers(int first_token, int L) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (first_token + r >= L || ((scale >> (8 * r)) & 255u) >= MX_TOO_LARGE) scale = (scale & ~(255u << (8 * r))) | 2u << (8 * r);
    }
};

// Bit r: the value of token 4 quad + r of a page is, or may be, infinite or no number in any of its blocks, which the 16 lanes of a quad hold between them.
__device__ __forceinline__ unsigned no_numbers(unsigned scale, int quad) {
    unsigned any = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const u64 lanes = __builtin_amdgcn_ballot_w64(((scale >> (8 * r)) & 255u) >= MX_TOO_LARGE);
        any |= (lanes >> (16 * quad) & 0xFFFFull) != 0 ? 1u << r : 0u;
    }
    return any;
}

// Adds one part's products to the raw scores of 16 tokens and 16 rows; the keys' scale is byte BYTE of `scale`.
template <int BYTE, int PART> __device__ __forceinline__ Float4 add_scores(UInt4 key, unsigned scale, const Query& q, Float4 s) {
    const UInt6 u = q.part[PART];
    const Int8 a = {static_cast<int>(key[0]), static_cast<int>(key[1]), static_cast<int>(key[2]), static_cast<int>(key[3]), 0, 0, 0, 0};
    const Int8 b = {static_cast<int>(u[0]), static_cast<int>(u[1]), static_cast<int>(u[2]), static_cast<int>(u[3]), static_cast<int>(u[4]), static_cast<int>(u[5]), 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, s, 4, 2, BYTE, scale, PART, q.bytes);
}
// The scores of four pages, less the rows' maxima so far (`start`), the small parts of the queries first; pages in turn, so that no product
// waits for the one in front.  The keys' scales: a register for each page, or a byte of one.
__device__ __forceinline__ void scores(const UInt4 (&key)[4], const unsigned (&scale)[4], const Query& q, float start, Float4 (&s)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = add_scores<0, 2>(key[i], scale[i], q, Float4{start, start, start, start});
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = add_scores<0, 1>(key[i], scale[i], q, s[i]);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = add_scores<0, 0>(key[i], scale[i], q, s[i]);
}
template <int PART> __device__ __forceinline__ void scores_of_part(const UInt4 (&key)[4], unsigned scales, const Query& q, Float4 (&s)[4]) {
    s[0] = add_scores<0, PART>(key[0], scales, q, s[0]);
    s[1] = add_scores<1, PART>(key[1], scales, q, s[1]);
    s[2] = add_scores<2, PART>(key[2], scales, q, s[2]);
    s[3] = add_scores<3, PART>(key[3], scales, q, s[3]);
}
__device__ __forceinline__ void scores(const UInt4 (&key)[4], unsigned scales, const Query& q, float start, Float4 (&s)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = Float4{start, start, start, start};
    scores_of_part<2>(key, scales, q, s);
    scores_of_part<1>(key, scales, q, s);
    scores_of_part<0>(key, scales, q, s);
}

// What a row sees: tree slots (those past the last node taken out), and prefix tokens behind `last`.
struct Sight {
    unsigned word[2 * GRAFT_MASK_WORDS];
    int last;
};
__device__ __forceinline__ u64 low_bits(int count) { return count >= 64 ? ~0ull : count <= 0 ? 0ull : (1ull << count) - 1; }
__device__ __forceinline__ Sight sight_of(const Sequence& q, int window, int node, int lane) {
    u64 word[GRAFT_MASK_WORDS] = {low_bits(node + 1), low_bits(node + 1 - 64)};            // (a chain)
    if (q.mask) {
        word[0] = q.mask[node * GRAFT_MASK_WORDS];
        word[1] = q.mask[node * GRAFT_MASK_WORDS + 1];
    }
    word[0] &= low_bits(q.n);
    word[1] &= low_bits(q.n - 64);
    Sight x;
    x.last = -1;
    if (window > 0) {                              // uniform
        const int64_t last = (q.pos ? q.pos[node] : q.P + node) - static_cast<int64_t>(window);
        x.last = static_cast<int>(last < -1 ? -1 : last > q.P ? q.P : last);
        if (q.deep) {
            const int at[2] = {q.pos ? q.pos[min(lane, q.n - 1)] : q.P + lane, q.pos ? q.pos[min(lane + 64, q.n - 1)] : q.P + lane + 64};
            for (int j = 0; j < q.n; ++j) {
                const int place = __builtin_amdgcn_readlane(j < 64 ? at[0] : at[1], j & 63);
                const u64 bit = place > last ? 0ull : 1ull << (j & 63);
                if (j < 64) word[0] &= ~bit;
                else word[1] &= ~bit;
            }
        }
    }
    x.word[0] = static_cast<unsigned>(word[0]);
    x.word[1] = static_cast<unsigned>(word[0] >> 32);
    x.word[2] = static_cast<unsigned>(word[1]);
    x.word[3] = static_cast<unsigned>(word[1] >> 32);
    return x;
}

// Which of 64 tokens from `token` on a row sees, the first in bit 0.
__device__ __forceinline__ u64 seen(const Sequence& q, const Sight& sight, int token) {
    const int j = token - q.P, k = j >> 5;         // (the slot of the first token, and its word: negative in the prefix)
    unsigned w[3] = {0, 0, 0};                     // words k, k + 1, k + 2; none outside the four
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int m = 0; m < 4; ++m) w[i] = k + i == m ? sight.word[m] : w[i];
    const u64 slots = __builtin_amdgcn_alignbit(w[1], w[0], j & 31) | static_cast<u64>(__builtin_amdgcn_alignbit(w[2], w[1], j & 31)) << 32;
    return slots | (low_bits(-j) & ~low_bits(sight.last + 1 - token));
}

// Where a tile of four pages from token `first` on is not seen whole by every node: what this lane's row does not see becomes -inf, what it sees and
// has a value that is no number becomes NaN (no_number: bit 4 i + r).
__device__ __forceinline__ void mask_scores(Float4 (&s)[4], const Sequence& q, const Sight& sight, int first, int quad, unsigned no_number) {
    const u64 see = seen(q, sight, first + quad * 4);
    if (__builtin_amdgcn_ballot_w64(no_number != 0) != 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[i][r] = (no_number >> (4 * i + r) & 1) ? __builtin_nanf("") : s[i][r];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[i][r] = (static_cast<unsigned>(see >> (32 * (i / 2))) >> (16 * (i & 1) + r) & 1) ? s[i][r] : -__builtin_inff();
}

// With a cap c the products are y = 2 log2(e) x / c: c tanh(x / c) = c - 2 c / (2^y + 1), in powers of two, less the row's maximum so far.  The two
// terms cancel for scores that are small next to the cap: up to 2^-20 c is left as an error, which bounds the cap.
template <int NP> __device__ __forceinline__ void cap_scores(Float4 (&s)[NP], float cap, float start) {
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            s[i][r] = __builtin_fmaf(__builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[i][r]) + 1.0f), -2.0f * cap, cap) + start;
}

// Sums are brought to another maximum by 2^x, x <= 0.  They may be well above 1, and below 2^-126 that factor is 0 though the product with them is a
// number: there it is taken in two halves, the second one behind a branch (two halves for all: a tree over 2048 tokens 14.5 -> 15.0 us).
struct Shrink {
    float by;
    bool twice;
    __device__ __forceinline__ explicit Shrink(float x) : twice(x < -100.0f) { by = __builtin_amdgcn_exp2f(twice ? 0.5f * x : x); }
    template <int TILES> __device__ __forceinline__ void apply(Float4 (&acc)[TILES]) const {
#pragma unroll
        for (int m = 0; m < TILES; ++m) acc[m] *= by;
        if (__builtin_amdgcn_ballot_w64(twice) == 0) return;
        const float again = twice ? by : 1.0f;
#pragma unroll
        for (int m = 0; m < TILES; ++m) acc[m] *= again;
    }
    __device__ __forceinline__ float of(float sum) const { return sum * by * (twice ? by : 1.0f); }
};

// A row block's softmax: the maximum `top` that scores are taken less of (TM_LOW as long as the row has seen nothing; common to its four
// lanes), this lane's part `sum` of the row's sum, and the weighted sum of values.
template <int TILES> struct Softmax {
    float top, sum;
    Float4 acc[TILES];
    __device__ __forceinline__ void clear() {
        top = TM_LOW;
        sum = 0.0f;
#pragma unroll
        for (int m = 0; m < TILES; ++m) acc[m] = Float4{0, 0, 0, 0};
    }
    __device__ __forceinline__ float start() const { return top == TM_LOW ? 0.0f : -top; }
    // A new maximum, of what the row has seen and these scores, for rows that vote for it; all else stays as it is, to the bit.
    template <int NP> __device__ __forceinline__ void raise(Float4 (&s)[NP], bool vote) {
        float most = __builtin_fmaxf(s[0][0], s[0][1]);
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int r = i == 0 ? 2 : 0; r < 4; r += 2) most = __builtin_fmaxf(__builtin_fmaxf(most, s[i][r]), s[i][r + 1]);
        most = rows_max_f32(most);
        const bool fresh = top == TM_LOW;
        float up = fresh ? most : __builtin_fmaxf(most, 0.0f);
        if (!vote || up == -__builtin_inff()) up = 0.0f;           // (nothing seen yet, and nothing here)
        else top = (fresh ? 0.0f : top) + up;
        const Shrink shrink(fresh ? 0.0f : -up);
        sum = shrink.of(sum);
        shrink.apply(acc);
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[i][r] -= up;
    }
};
template <int NP> __device__ __forceinline__ float powers(const Float4 (&s)[NP], Float4 (&x)[NP]) {        // and their sum
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            x[i][r] = __builtin_amdgcn_exp2f(s[i][r]);
            sum[r & 1] += x[i][r];
        }
    return sum[0] + sum[1];
}
template <int NP> __device__ __forceinline__ void to_operand(const Float4 (&x)[NP], Bf8 (&prob)[NP / 2]) {
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) prob[i / 2][(i & 1) * 4 + r] = static_cast<__bf16>(x[i][r]);
}
// Scores to probabilities.  A row's maximum is left as it is as long as it has one and the probabilities add up to less than TM_MOST in each of its
// lanes: they and their sums are floating-point numbers, the same up to a power of two.  (So the common case takes no
// maximum: an exponential, half a conversion and an addition a score.)  A power of two that is no whole one moves where probabilities are
// rounded, so a row's four lanes decide for that row alone, and rows that are not there (`live`: a bit for each lane whose row is) not at all:
// a result depends on its row's query and on what the row sees.
template <int MB, int NP, int TILES>
__device__ __forceinline__ void to_probabilities(Float4 (&s)[MB][NP], Softmax<TILES> (&soft)[MB], const u64 (&live)[MB], Bf8 (&prob)[MB][NP / 2]) {
    Float4 x[MB][NP];
    float sum[MB];
    u64 over[MB], any = 0;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        sum[mb] = powers<NP>(s[mb], x[mb]);
        over[mb] = __builtin_amdgcn_ballot_w64(soft[mb].top == TM_LOW || sum[mb] > TM_MOST) & live[mb];
        any |= over[mb];
    }
    if (any != 0) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const u64 half = over[mb] | over[mb] >> 32, votes = (half | half >> 16) & 0xFFFF;
            soft[mb].raise(s[mb], __builtin_amdgcn_inverse_ballot_w64(votes * 0x0001000100010001ull));     // (the row's, in each of its lanes)
            sum[mb] = powers<NP>(s[mb], x[mb]);
        }
    }
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        soft[mb].sum += sum[mb];
        to_operand<NP>(x[mb], prob[mb]);
    }
}

// Part PAIR of a page's values as halves of operands (4 of their 8 tokens a lane): elements 2 PAIR and 2 PAIR + 1 of the lane's part of its tokens.
template <int D, int PAIR> __device__ __forceinline__ void value_pair(const ValuePage<D>& v, const float (&scale)[4], UInt2 (&two)[2]) {
    unsigned c[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if constexpr (D == 128) c[r] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v.four[r], scale[r], PAIR));
        else if (r & 1) c[r] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v.four[r / 2], scale[r], 2 + PAIR));
        else c[r] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v.four[r / 2], scale[r], PAIR));
    }
    two[0] = UInt2{__builtin_amdgcn_perm(c[1], c[0], 0x05040100), __builtin_amdgcn_perm(c[3], c[2], 0x05040100)};
    two[1] = UInt2{__builtin_amdgcn_perm(c[1], c[0], 0x07060302), __builtin_amdgcn_perm(c[3], c[2], 0x07060302)};
}
template <int D> __device__ __forceinline__ void value_scales(const ValuePage<D>& v, float (&scale)[4]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) scale[r] = mx_scale((v.scale >> (8 * r)) & 255u);
}

template <class F, int... I> __device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F&& f) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F> __device__ __forceinline__ void each(F&& f) { each_of(std::make_integer_sequence<int, N>{}, f); }

// All of them: `put` gets element 0, 1, ..
template <int D, class Put> __device__ __forceinline__ void value_operands(const ValuePage<D>& v, Put&& put) {
    float scale[4];
    value_scales<D>(v, scale);
    each<D / 32>([&](auto pair) {
        UInt2 two[2];
        value_pair<D, decltype(pair)::value>(v, scale, two);
        put(2 * decltype(pair)::value, two[0]);
        put(2 * decltype(pair)::value + 1, two[1]);
    });
}

// N neighbouring elements of a row from `d` on: the result, or with the keys split the sums.
template <int D, int N>
__device__ __forceinline__ void store_part(const Sequence& q, const AttnMxParams& p, int64_t out_at, int64_t item, int row, int d, const float (&o)[N], float total) {
    if (row >= q.all_rows) return;
    if (p.splits == 1) {
        const bool there = row < q.rows;
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        unsigned packed[N / 2];
#pragma unroll
        for (int m = 0; m < N; m += 2) {
            const Bf2 two = {static_cast<__bf16>(there ? o[m] * inv : 0.0f), static_cast<__bf16>(there ? o[m + 1] * inv : 0.0f)};
            packed[m / 2] = __builtin_bit_cast(unsigned, two);
        }
        unsigned short* out = p.out + out_at + d;
        if constexpr (N % 8 == 0) {
#pragma unroll
            for (int m = 0; m < N / 8; ++m) reinterpret_cast<UInt4*>(out)[m] = UInt4{packed[4 * m], packed[4 * m + 1], packed[4 * m + 2], packed[4 * m + 3]};
        } else *reinterpret_cast<UInt2*>(out) = UInt2{packed[0], packed[1]};
    } else if (row < q.rows) {
        Float4* dst = reinterpret_cast<Float4*>(p.partial + (item * q.all_rows + row) * D + d);
#pragma unroll
        for (int m = 0; m < N / 4; ++m) dst[m] = Float4{o[4 * m], o[4 * m + 1], o[4 * m + 2], o[4 * m + 3]};
    }
}
__device__ __forceinline__ void store_stat(const Sequence& q, const AttnMxParams& p, int64_t item, int row, float top, float total) {
    if (p.splits > 1 && row < q.rows) *reinterpret_cast<float2*>(p.stat + (item * q.all_rows + row) * 2) = float2{top, total};
}

// A workgroup's place: ids 8 apart are on one XCD, and those that read the same keys for other rows follow each other there.
struct Place { int item, row_tile, split, g, b; };
__device__ __forceinline__ Place place_of(const AttnMxParams& p) {
    const unsigned item = blockIdx.y * 8 + (blockIdx.x & 7), head = item / static_cast<unsigned>(p.splits), b = head / static_cast<unsigned>(p.Hkv);
    return {static_cast<int>(item), static_cast<int>(blockIdx.x >> 3), static_cast<int>(item - head * p.splits), static_cast<int>(head - b * p.Hkv), static_cast<int>(b)};
}

// ---- few rows: the wavefronts of a workgroup share the rows and deal the keys out among themselves ----------------------------------
// With one block of rows bound by the cache's bytes: 32 sequences of up to 16384 tokens, 8 heads of 128, 434 MB in 82 us, 5.3 TB/s (all 16384 tokens long:
// 5.7, and as much with one or two more tiles in flight; a plain read of long pieces reaches 6.3).  With two by the issue of instructions,
// and where keys are few by the trips to memory in front of the first tile (3 us) and the joining of sums (2 us).  Every wavefront
// streams pages of its own, 16 bytes a lane and page of keys and of values, the next four pages in flight while four are worked on; no barrier until the
// end.  The next tile's loads come behind this one's scores, with masks behind its probabilities, when registers are free: no scratch memory.
template <int D, int MB, bool CAP, bool STREAM>
__global__ __launch_bounds__(TM_THREADS, 2) void tree_attn_mx_kernel(const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ n_nodes,
                                                                     const int32_t* __restrict__ block_table, AttnMxParams p) {
    constexpr int TILES = D / 16, NP = 4, AUX = STREAM ? 2 : 0;    // tiles of the output; pages of a tile of keys; (2: nontemporal)
    __shared__ float exchange[TM_WAVES * TILES * 4 * 64];
    __shared__ float stats[TM_WAVES][MB][16][2];
    __shared__ Sight sights[TM_WAVES][MB][16];
    const Place at = place_of(p);
    if (at.item >= p.items) return;
    const int g = at.g, b = at.b, row0 = at.row_tile * 16 * MB;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row16 = lane & 15, quad = lane >> 4;
    Sequence q = sequence_of(b, prefix_len[b], n_nodes[b], block_table, p, D);
    if (row0 >= q.rows) {                          // uniform
        if (p.splits == 1) zero_rows(q, p, g, row0, 16 * MB, D);
        return;
    }
    Query query[MB];
    int node[MB];
    u64 live[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int row = row0 + mb * 16 + row16;
        node[mb] = row < q.rows ? node_of(p, row) : 0;
        live[mb] = __builtin_amdgcn_ballot_w64(row < q.rows);
        query[mb] = load_query<D>(q, p, g, row, quad * 32);
    }
    if (p.window > 0) look_back(q, p.window, lane);
    const Units units(q, NP * GRAFT_PAGE_SIZE, at.split * TM_WAVES + wave, p.splits * TM_WAVES);   // (a piece of the keys for each wavefront)
    const int page0 = q.first_page + units.first * NP;
    const unsigned char *k_head = p.k_cache + g * p.head_stride, *v_head = p.v_cache + g * p.head_stride;
    const LaneAt<D> lane_at(lane);
    struct Held {
        UInt4 k[NP];
        unsigned k_scale[NP];
        ValuePage<D> v[NP];
    };
    auto load = [&](PageIds& ids, int i0) {
        Held h;
        const int page = units.unit(i0) * NP;
        ids.seek(page);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const u64 run = ids.offset(page + i, p.page_stride);
            const __amdgpu_buffer_rsrc_t k = run_of<D>(k_head + run);
            h.k[i] = __builtin_bit_cast(UInt4, __builtin_amdgcn_raw_buffer_load_b128(k, lane_at.k, 0, AUX));
            h.k_scale[i] = __builtin_amdgcn_raw_buffer_load_b8(k, lane_at.k_scale, 0, AUX);
            h.v[i].template load<AUX>(run_of<D>(v_head + run), lane_at.v, lane_at.v_scale);
        }
        return h;
    };

    Softmax<TILES> soft[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) soft[mb].clear();
    auto step = [&](PageIds& ids, int i0, Held& h, auto masks) {   // and h becomes the next tile
        constexpr bool MASKS = decltype(masks)::value;
        const int first = (page0 + units.unit(i0) * NP) * GRAFT_PAGE_SIZE;
        unsigned no_number = 0;
        if constexpr (MASKS) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                no_number |= no_numbers(h.v[i].scale, quad) << (4 * i);
                h.v[i].keep_numbers(first + i * GRAFT_PAGE_SIZE + quad * 4, q.L);
            }
        }
        Bf8 prob[MB][NP / 2];
        Float4 s[MB][NP];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) scores(h.k, h.k_scale, query[mb], CAP ? 0.0f : soft[mb].start(), s[mb]);
        Held ahead;                                // (from here on: this tile's keys have left their registers, with masks its scores too)
        if constexpr (!MASKS) ahead = load(ids, i0 + 1);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            if constexpr (CAP) cap_scores<NP>(s[mb], p.cap, soft[mb].start());
            if constexpr (MASKS) mask_scores(s[mb], q, sights[wave][mb][row16], first, quad, no_number);
        }
        to_probabilities<MB, NP, TILES>(s, soft, live, prob);
        if constexpr (MASKS) ahead = load(ids, i0 + 1);
#pragma unroll
        for (int i = 0; i < NP / 2; ++i) {
            UInt2 low[TILES];
            value_operands<D>(h.v[2 * i], [&](int m, UInt2 v) { low[m] = v; });
            value_operands<D>(h.v[2 * i + 1], [&](int m, UInt2 v) {
                const Bf8 both = __builtin_bit_cast(Bf8, UInt4{low[m][0], low[m][1], v[0], v[1]});
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) soft[mb].acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(both, prob[mb][i], soft[mb].acc[m], 0, 0, 0);
            });
        }
        h = ahead;
    };
    if (units.count > 0) {
        PageIds ids(q, page0, lane);
        int i = units.whole;
        Held here = load(ids, i);
        if (units.whole_end < units.end()) {       // (now: their trip to memory is that of the first keys)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                const Sight x = sight_of(q, p.window, node[mb], lane);
                if (quad == 0) sights[wave][mb][row16] = x;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");        // (the other lanes of the wavefront read it)
            __builtin_amdgcn_wave_barrier();
        }
        auto loop = [&](int end, auto masks) {
#pragma nounroll
            for (; i < end; ++i) {
                step(ids, i, here, masks);
            }
        };
        loop(units.whole_end, std::false_type{});
        loop(units.end(), std::true_type{});
    }

    // The wavefronts' sums are brought to the rows' common maximum and added: wavefront w takes the elements whose place in
    // their tile is 4 quad + w, D / 16 neighbours in the row.
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        float s = soft[mb].sum;
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (quad == 0) {
            stats[wave][mb][row16][0] = soft[mb].top;
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
        for (int w = 0; w < TM_WAVES; ++w) total += Shrink(stats[w][mb][row16][0] - most).of(stats[w][mb][row16][1]);
        Shrink(soft[mb].top - most).apply(soft[mb].acc);
        if (mb > 0) __syncthreads();
#pragma unroll
        for (int m = 0; m < TILES; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) exchange[((wave * TILES + m) * 4 + r) * 64 + lane] = soft[mb].acc[m][r];
        __syncthreads();
        float o[TILES];
#pragma unroll
        for (int m = 0; m < TILES; ++m) {
            o[m] = 0.0f;
#pragma unroll
            for (int w = 0; w < TM_WAVES; ++w) o[m] += exchange[((w * TILES + m) * 4 + wave) * 64 + lane];
        }
        const int row = row0 + mb * 16 + row16;
        store_part<D, TILES>(q, p, row_at(q, p, g, row, D), at.item, row, (quad * 4 + wave) * TILES, o, total);
        if (wave == 0 && quad == 0) store_stat(q, p, at.item, row, most, total);
    }
}

// ---- more rows: the wavefronts of a workgroup have 16 rows each and share keys and values -----------------------------------------------
// Bound by the matrix cores and the vector units together: 64 tokens x 16 rows are 28 matrix instructions of 16 cycles, and with a wavefront's share of
// what is done for all 67 vector instructions and 16 exponentials; a matrix instruction takes 8 cycles (bfloat16) or 12 (4 and 6 bits) of the vector
// units' issue, so four wavefronts need 2800 cycles of it for 1790 of the matrix cores.  A stage takes 3500.
// One wavefront waits for its own products and exponentials in turn, so others have to have work meanwhile: hence 16 rows and 128 registers a
// wavefront, four wavefronts a SIMD, and nothing of the hot loop in scratch, whose reloads would wait for the loads from memory in front of them.
// Converting 64 tokens' values is 164 vector instructions: four of the eight wavefronts convert a page each into LDS, the others bring a page's
// keys, and all of them take keys and values from there.  Two stages' buffers, one barrier a
// stage: while one is read the next is written, from registers that were loaded a stage ago.
// 96 nodes x 32 heads over 8 KV heads, 4 sequences, prefix 65536: 358 us, 1.14 PFLOP/s for both products, where a large bfloat16 matrix product
// reaches 1.3 to 1.4 on the same card.  Two row blocks a wavefront, or 32 x 32 products with their order laid down by hand, which halve the
// matrix instructions' share of the issue, take 362 and 372 us, and longer where there are few stages.
constexpr int TR_WAVES = 8, TR_PAGES = 4;          // wavefronts; pages of a stage

// A barrier that waits for a wavefront's LDS operations alone: loads from memory stay on their way.
__device__ __forceinline__ void workgroup_lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int D, bool CAP>
__global__ __launch_bounds__(64 * TR_WAVES, 4) void tree_attn_mx_rows_kernel(const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ n_nodes,
                                                                             const int32_t* __restrict__ block_table, AttnMxParams p) {
    constexpr int TILES = D / 16, NP = TR_PAGES;
    __shared__ UInt4 values[2][NP / 2][TILES][64];
    __shared__ UInt4 keys[2][NP][64];
    __shared__ unsigned key_scales[2][64];                         // a byte for each page
    __shared__ unsigned short none[2][NP][4];                      // no_numbers of a stage's pages, by quad
    __shared__ Sight sights[TR_WAVES][16];
    const Place at = place_of(p);
    if (at.item >= p.items) return;
    const int g = at.g, b = at.b;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row16 = lane & 15, quad = lane >> 4;
    const int tile_row0 = at.row_tile * 16 * p.waves, row0 = tile_row0 + wave * 16, row = row0 + row16;
    Sequence q = sequence_of(b, prefix_len[b], n_nodes[b], block_table, p, D);
    if (tile_row0 >= q.rows) {                     // uniform
        if (p.splits == 1) zero_rows(q, p, g, tile_row0, 16 * p.waves, D);
        return;
    }
    const int node = row < q.rows ? node_of(p, row) : 0;
    const u64 live[1] = {__builtin_amdgcn_ballot_w64(row < q.rows)};
    const Query query = load_query<D>(q, p, g, row, quad * 32);
    if (p.window > 0) look_back(q, p.window, lane);
    const Units units(q, NP * GRAFT_PAGE_SIZE, at.split, p.splits);
    const int page0 = q.first_page + units.first * NP;

    const unsigned char *k_head = p.k_cache + g * p.head_stride, *v_head = p.v_cache + g * p.head_stride;
    const LaneAt<D> lane_at(lane);
    // What this wavefront brings of a stage: the first four a page's values each, the others a page's keys; a wavefront without rows does no more.
    const bool has_rows = wave < p.waves && row0 < q.rows, converts = wave < NP;
    const int page_of = wave % NP;
    const unsigned char* head = converts ? v_head : k_head;
    const unsigned lane_run = converts ? lane_at.v : lane_at.k, lane_scale = converts ? lane_at.v_scale : lane_at.k_scale & ~3u;
    UInt4 raw;                                     // (of values with D = 64 the first half)
    unsigned raw_scale;
    auto fetch = [&](PageIds& ids, int i0) {
        const int page = units.unit(i0) * NP;
        ids.seek(page);
        const __amdgpu_buffer_rsrc_t run = run_of<D>(head + ids.offset(page + page_of, p.page_stride));
        raw = __builtin_bit_cast(UInt4, __builtin_amdgcn_raw_buffer_load_b128(run, lane_run, 0, 0));
        raw_scale = __builtin_amdgcn_raw_buffer_load_b32(run, lane_scale, 0, 0);
    };
    auto bring = [&](int i0) {
        const int buf = i0 & 1;
        if (converts) {
            ValuePage<D> page;
            if constexpr (D == 128) page.four = raw;
            else page.four = UInt2{raw[0], raw[1]};
            page.scale = raw_scale;
            if (i0 >= units.whole_end) {
                const unsigned any = no_numbers(page.scale, quad);
                if (row16 == 0) none[buf][wave][quad] = static_cast<unsigned short>(any);
                page.keep_numbers((page0 + units.unit(i0) * NP + wave) * GRAFT_PAGE_SIZE + quad * 4, q.L);
            }
            value_operands<D>(page, [&](int m, UInt2 v) { reinterpret_cast<UInt2*>(&values[buf][wave >> 1][m][lane])[wave & 1] = v; });
        } else {
            keys[buf][page_of][lane] = raw;
            reinterpret_cast<unsigned char*>(&key_scales[buf][lane])[page_of] = static_cast<unsigned char>(raw_scale >> (8 * (lane_at.k_scale & 3)));
        }
    };

    Softmax<TILES> soft[1];
    soft[0].clear();
    auto stage = [&](PageIds& ids, int i0, auto masks) {
        constexpr bool MASKS = decltype(masks)::value;
        const int buf = i0 & 1;
        Float4 s[1][NP];
        if (has_rows) {
            UInt4 key[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) key[i] = keys[buf][i][lane];
            scores(key, key_scales[buf][lane], query, CAP ? 0.0f : soft[0].start(), s[0]);
        }
        // (while the matrix cores have these: the next stage's buffer, whose readers have passed the last barrier; behind the last stage nobody
        // reads what comes there)
        bring(i0 + 1);
        fetch(ids, i0 + 2);
        if (has_rows) {
            constexpr bool AHEAD = !MASKS && !CAP;  // values on their way from LDS three products ahead (masks and the cap leave no registers for it)
            UInt4 three[3];
            auto value = [&](int n) { return values[buf][n / TILES][n % TILES][lane]; };
            if constexpr (AHEAD) {
#pragma unroll
                for (int n = 0; n < 3; ++n) three[n] = value(n);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (CAP) cap_scores<NP>(s[0], p.cap, soft[0].start());
            if constexpr (MASKS) {
                unsigned no_number = 0;
#pragma unroll
                for (int i = 0; i < NP; ++i) no_number |= static_cast<unsigned>(none[buf][i][quad]) << (4 * i);
                mask_scores(s[0], q, sights[wave][row16], (page0 + units.unit(i0) * NP) * GRAFT_PAGE_SIZE, quad, no_number);
            }
            Bf8 prob[1][NP / 2];
            to_probabilities<1, NP, TILES>(s, soft, live, prob);
            if constexpr (AHEAD) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < NP / 2 * TILES; ++n) {
                const UInt4 v = !AHEAD ? value(n) : three[n % 3];
                soft[0].acc[n % TILES] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf8, v), prob[0][n / TILES], soft[0].acc[n % TILES], 0, 0, 0);
                if constexpr (AHEAD) {
                    if (n + 3 < NP / 2 * TILES) three[n % 3] = value(n + 3);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        workgroup_lds_barrier();
    };
    if (units.count > 0) {                         // uniform over the workgroup
        PageIds ids(q, page0, lane);
        int i = units.whole;
        fetch(ids, i);
        if (units.whole_end < units.end()) {       // (now: its trip to memory is that of the first keys)
            const Sight x = sight_of(q, p.window, node, lane);
            if (quad == 0) sights[wave][row16] = x;
        }
        bring(i);
        fetch(ids, i + 1);
        workgroup_lds_barrier();
#pragma nounroll
        for (; i < units.whole_end; ++i) stage(ids, i, std::false_type{});
#pragma nounroll
        for (; i < units.end(); ++i) stage(ids, i, std::true_type{});
    }
    if (wave >= p.waves) return;                   // (its rows are the next tile's)
    float total = soft[0].sum;
    total += __shfl_xor(total, 16);
    total += __shfl_xor(total, 32);
    const int64_t out_at = row_at(q, p, g, row, D);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float o[TILES];
#pragma unroll
        for (int m = 0; m < TILES; ++m) o[m] = soft[0].acc[m][r];
        store_part<D, TILES>(q, p, out_at, at.item, row, (quad * 4 + r) * TILES, o, total);
    }
    if (quad == 0) store_stat(q, p, at.item, row, soft[0].top, total);
}

// The splits' sums of a row, 8 elements a lane, bound by its launch and a trip to memory (4 to 5 us), or with many rows by the 4 D bytes of every row and split
// (31 MB 7.5 us): each lane has the weights of every LANES-th split, and eight splits' sums are on their way at a time.
template <int D>
__global__ __launch_bounds__(TM_THREADS) void tree_attn_mx_merge_kernel(const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ n_nodes,
                                                                        const float* __restrict__ partial, const float* __restrict__ stat,
                                                                        AttnMxParams p) {
    constexpr int LANES = D / 8, HELD = TM_MAX_SPLITS / LANES, BATCH = 8;
    const int b = blockIdx.z, g = blockIdx.y, row = blockIdx.x * (TM_THREADS / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES, d = lane * 8;
    const int64_t all_rows = p.K * p.G, base = static_cast<int64_t>(b * p.Hkv + g) * p.splits * all_rows + min(row, static_cast<int>(all_rows) - 1);
    // What rows that are not there have in the workspace is loaded too, and not used: one trip to memory for lengths, statistics and the first sums.
    Float4 x[BATCH], y[BATCH];
    auto load = [&](int s0) {
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            const Float4* src = reinterpret_cast<const Float4*>(partial + (base + min(s0 + j, p.splits - 1) * all_rows) * D + d);
            x[j] = src[0];
            y[j] = src[1];
        }
    };
    float2 st[HELD];
#pragma unroll
    for (int h = 0; h < HELD; ++h) st[h] = *reinterpret_cast<const float2*>(stat + (base + min(lane + h * LANES, p.splits - 1) * all_rows) * 2);
    load(0);
    const Sequence q = sequence_of(b, prefix_len[b], n_nodes[b], nullptr, p, D);
    float weight[HELD], again[HELD], total = 0.0f, most = TM_LOW;
    bool twice = false;
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        if (lane + h * LANES >= p.splits) st[h] = float2{TM_LOW, 0.0f};
        most = __builtin_fmaxf(most, st[h].x);
    }
#pragma unroll
    for (int s = LANES / 2; s > 0; s >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, s));
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        const Shrink shrink(st[h].x - most);
        weight[h] = shrink.by;
        again[h] = shrink.twice ? shrink.by : 1.0f;
        twice = twice || (shrink.twice && st[h].y != 0.0f);
        total += shrink.of(st[h].y);
    }
    twice = __builtin_amdgcn_ballot_w64(twice) != 0;
#pragma unroll
    for (int s = LANES / 2; s > 0; s >>= 1) total += __shfl_xor(total, s);
    float o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int h = 0; h < HELD; ++h)
        for (int s0 = h * LANES; s0 < min(p.splits, (h + 1) * LANES); s0 += BATCH) {
            if (s0 > 0) load(s0);
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const float w = __shfl(weight[h], s0 - h * LANES + j, LANES);
                if (s0 + j >= p.splits) continue;
                if (twice) {
                    const float w2 = __shfl(again[h], s0 - h * LANES + j, LANES);
                    x[j] *= w2;
                    y[j] *= w2;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    o[k] += x[j][k] * w;
                    o[4 + k] += y[j][k] * w;
                }
            }
        }
    if (row >= q.all_rows) return;
    const bool there = row < q.rows;
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    unsigned packed[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const Bf2 two = {static_cast<__bf16>(there ? o[2 * j] * inv : 0.0f), static_cast<__bf16>(there ? o[2 * j + 1] * inv : 0.0f)};
        packed[j] = __builtin_bit_cast(unsigned, two);
    }
    *reinterpret_cast<UInt4*>(p.out + row_at(q, p, g, row, D) + d) = UInt4{packed[0], packed[1], packed[2], packed[3]};
}

// ---- plan --------------------------------------------------------------------------------------------------------------------------
struct AttnMxPlan {
    int row_blocks;                                // of 16 rows for each wavefront of the kernel for few rows, 0: the kernel for more
    int waves, row_tiles, splits;                  // of a workgroup, that have rows; tiles of a head's rows; splits of the keys
};

// The kernel for few rows in tiles of 32 rows, unless a head has more than TM_MANY and its tiles alone give every compute unit a workgroup: with work
// for all, the kernel for more rows converts values for 128 rows at once (with as few workgroups as that takes and rows dealt out
// evenly); with less, it splits keys further and has more to join.  The border is where most shapes gain; one just above it loses 3 % (16 x 64 below).
// Few / more, us, D = 128, B x K x Hq over Hkv at a prefix:
//   4 x 96 x 32/8 at 65536  461 / 354     32 x 64 x 32/8 at 4096  149 / 129    16 x 128 x 32/8 at 8192  266 / 229    4 x 64 x 32/8 at 65536  266 / 248
//   16 x 48 x 32/8 at 8192  113 / 124     16 x 64 x 32/8 at 8192  139 / 143    1 x 128 x 40/8 at 4096    27 / 36     1 x 40 x 32/8 at 2048   15 / 18
constexpr int TM_MANY = 192;
static AttnMxPlan plan_attn_mx(int32_t B, int32_t K, int32_t Hq, int32_t Hkv, int64_t pages) {          // (that a sequence's nodes may see)
    const int rows = K * (Hq / Hkv), blocks = (rows + 15) / 16;
    AttnMxPlan plan{blocks > 1 ? 2 : 1, TM_WAVES, (blocks + 1) / 2, 1};
    if (rows > TM_MANY && static_cast<int64_t>(B) * Hkv * plan.row_tiles >= device_compute_units()) {
        plan.row_blocks = 0;
        plan.row_tiles = (blocks + TR_WAVES - 1) / TR_WAVES;
        plan.waves = (blocks + plan.row_tiles - 1) / plan.row_tiles;
    }
    const int64_t groups = static_cast<int64_t>(B) * Hkv * plan.row_tiles;
    // Two workgroups a compute unit: as many as are at work at a time (with four, us: single tokens of 32 sequences 114 -> 117, of 8 28 -> 35,
    // 64 x 40 rows at 32768 65 -> 72).  A split has at least two tiles of four pages for each wavefront where the table is full (with one: 64 rows of 8 heads at 256 tokens
    // 10.2 -> 12.2, at 2048 14.3 -> 14.6, at 8192 20.7 -> 22.9; with four: at 2048 19.0 -> 19.8).  Lengths are not known here: in a table of 2048 pages, one token of 2
    // heads over 255 tokens takes 12.9 and not 5.9, 40 nodes of 8 over 2048 17.8 and not 14.7.
    const int64_t fill = 2 * device_compute_units(), most = (pages + 31) / 32;
    int64_t s = groups >= fill ? 1 : fill / groups;
    if (s > most) s = most;
    if (s > TM_MAX_SPLITS) s = TM_MAX_SPLITS;
    if (s < 1) s = 1;
    plan.splits = static_cast<int>(s);
    return plan;
}

static bool bad_attn_mx_shape(int32_t B, int32_t K, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_pages) {
    return B < 1 || B > 65535 || K < 1 || K > GRAFT_MAX_NODES || Hkv < 1 || Hkv > 65535 || Hq < Hkv || Hq % Hkv != 0 || Hq / Hkv > 16 ||
           (D != 64 && D != 128) || max_pages < 1 || max_pages > 262144 || static_cast<int64_t>(B) * Hkv > (1 << 18);                      // (items in the grid's second dimension)
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
        head_stride < mx_run_bytes(D) || page_stride > 0xFFFFFFFFll || page_stride % 16 != 0 || head_stride % 16 != 0 || window < 0)
        return GRAFT_ERR_SHAPE;
    constexpr float LOG2E = 1.44269504088896340736f;
    const float factor = softcap > 0.0f ? 2.0f * LOG2E * scale / softcap : scale * LOG2E;
    if (!(factor - factor == 0.0f) || !(softcap >= 0.0f && softcap <= 1024.0f)) return GRAFT_ERR_SHAPE;
    if ((reinterpret_cast<size_t>(q) | reinterpret_cast<size_t>(k_cache) | reinterpret_cast<size_t>(v_cache) | reinterpret_cast<size_t>(out)) & 15)
        return GRAFT_ERR_SHAPE;
    // With a window the keys are split by the pages that it leaves of the table's (nodes' positions are at most K_max apart, or more is left out of
    // the plan, not of the sums): never into more pieces than without, for which the workspace was asked for.  (One token, 8 heads, a
    // table of 4064 pages, us: a window of 4096 17.6 by the table and 11.3 by the window, of 128 17.3 and 7.0; 40 nodes, of 1024 17.2 and 14.4.)
    const int64_t windowed = window / GRAFT_PAGE_SIZE + K_max / GRAFT_PAGE_SIZE + 3, pages = window > 0 && windowed < max_pages ? windowed : max_pages;
    const AttnMxPlan plan = plan_attn_mx(B, K_max, Hq, Hkv, pages);
    const size_t need = attn_mx_bytes(plan, B, K_max, Hq, D);
    if (need > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<size_t>(workspace) & 15))) return GRAFT_ERR_WORKSPACE;
    AttnMxParams p{};
    p.q = static_cast<const unsigned short*>(q);
    p.k_cache = static_cast<const unsigned char*>(k_cache);
    p.v_cache = static_cast<const unsigned char*>(v_cache);
    p.pos = pos;
    p.mask = reinterpret_cast<const u64*>(mask);
    p.out = static_cast<unsigned short*>(out);
    p.partial = static_cast<float*>(workspace);
    p.stat = p.partial + static_cast<size_t>(B) * K_max * Hq * plan.splits * D;
    p.page_stride = static_cast<unsigned>(page_stride);
    p.head_stride = head_stride;
    p.factor = factor;
    p.cap = softcap * LOG2E;
    p.per_group = (65536 + Hq / Hkv - 1) / (Hq / Hkv);
    p.K = K_max; p.Hkv = Hkv; p.G = Hq / Hkv; p.max_pages = max_pages; p.window = window; p.splits = plan.splits; p.row_tiles = plan.row_tiles; p.waves = plan.waves;
    p.items = B * Hkv * plan.splits;
    // One tile of rows reads every page once: from more than the Infinity Cache holds on, of the pages that there is room for and that windows leave,
    // loads are nontemporal (us: single tokens of 32 sequences of 16384, 571 MB, 114 -> 106; of 64 of 4096, 286 MB, 47 -> 46; of 8 of 8192,
    // 71 MB, they would be 19 -> 21).
    const bool stream_cache = plan.row_blocks != 0 && plan.row_tiles == 1 && 2 * pages * B * Hkv * mx_run_bytes(D) > TM_CACHED;
    const dim3 blocks(8 * plan.row_tiles, (p.items + 7) / 8);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, blocks, dim3(plan.row_blocks == 0 ? 64 * TR_WAVES : TM_THREADS), 0, static_cast<hipStream_t>(stream), prefix_len, n_nodes, block_table, p);
    };
    auto sized = [&](auto d) {
        constexpr int DIM = decltype(d)::value;
        auto capped = [&](auto cap) {
            constexpr bool CAP = decltype(cap)::value;
            if (plan.row_blocks == 0) launch(tree_attn_mx_rows_kernel<DIM, CAP>);
            else if (plan.row_blocks == 1 && stream_cache) launch(tree_attn_mx_kernel<DIM, 1, CAP, true>);
            else if (plan.row_blocks == 1) launch(tree_attn_mx_kernel<DIM, 1, CAP, false>);
            else if (stream_cache) launch(tree_attn_mx_kernel<DIM, 2, CAP, true>);
            else launch(tree_attn_mx_kernel<DIM, 2, CAP, false>);
        };
        if (softcap > 0.0f) capped(std::true_type{});
        else capped(std::false_type{});
    };
    if (D == 128) sized(std::integral_constant<int, 128>{});
    else sized(std::integral_constant<int, 64>{});
    const int32_t rc = check_launch();
    if (rc != GRAFT_OK || plan.splits == 1) return rc;
    const int per = TM_THREADS / (D / 8);
    const dim3 grid((K_max * p.G + per - 1) / per, Hkv, B);
    if (D == 128) hipLaunchKernelGGL(tree_attn_mx_merge_kernel<128>, grid, dim3(TM_THREADS), 0, static_cast<hipStream_t>(stream), prefix_len, n_nodes, p.partial, p.stat, p);
    else hipLaunchKernelGGL(tree_attn_mx_merge_kernel<64>, grid, dim3(TM_THREADS), 0, static_cast<hipStream_t>(stream), prefix_len, n_nodes, p.partial, p.stat, p);
    return check_launch();
}
