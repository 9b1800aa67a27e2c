// graft_kv_gather_mx: rows of the 4-bit cache as numbers; graft_kv_compact_mx: its update after acceptance.
#include "mx.h"

namespace graft {

// ---- rows as numbers ---------------------------------------------------------------------------------------------------------------
// One lane makes 8 numbers of 4 bytes and a scale: bound by what it writes (16388 tokens of 8 heads of 128 to bfloat16, 18 MB in and 67 out:
// 18.8 us, 4.5 TB/s).  Lanes follow the output, so stores are whole lines; a token's keys of a head are 8 D / 16 bytes in a row, its values
// pieces of 4 (2 with D = 64) bytes whose neighbours other rows of the launch read.  Stores do not push what is read out of the caches (an append
// of those tokens and this 98.8 -> 93.0 us).
constexpr int KG_THREADS = 256;

struct GatherParams {
    const unsigned char *k_cache, *v_cache;
    void *k_out, *v_out;
    int32_t* status;
    int64_t layer_stride, page_stride, head_stride;            // bytes
    int32_t T, Hkv;
};

template <int D, bool F32>
__global__ __launch_bounds__(KG_THREADS) void kv_gather_mx_kernel(const int32_t* __restrict__ start, const int32_t* __restrict__ count,
                                                                  const int32_t* __restrict__ block_table, int32_t max_pages, GatherParams p) {
    constexpr int LANES = D / 8;
    const int b = blockIdx.y, layer = blockIdx.z;
    const int32_t first = start ? start[b] : 0, n = count[b];
    const bool bad = first < 0 || n < 0 || n > p.T || static_cast<int64_t>(first) + n > static_cast<int64_t>(max_pages) * GRAFT_PAGE_SIZE;
    if (blockIdx.x == 0 && layer == 0 && threadIdx.x == 0) p.status[b] = bad ? GRAFT_STATUS_BAD_LENGTH : 0;
    const unsigned at = blockIdx.x * KG_THREADS + threadIdx.x, per_token = p.Hkv * LANES;       // (a launch has fewer than 2^32 lanes a sequence)
    if (at >= static_cast<int64_t>(p.T) * per_token) return;
    const int t = at / per_token, rest = at - t * per_token;
    const int g = rest / LANES, lane = rest % LANES;
    unsigned k4 = 0, v4 = 0, ks = 0, vs = 0;
    if (!bad && t < n) {
        const int32_t token = first + t, in_page = token & (GRAFT_PAGE_SIZE - 1);
        const int64_t page = block_table[static_cast<int64_t>(b) * max_pages + token / GRAFT_PAGE_SIZE];
        const int64_t run = layer * p.layer_stride + page * p.page_stride + g * p.head_stride;
        const unsigned char *k = p.k_cache + run, *v = p.v_cache + run;
        k4 = *reinterpret_cast<const unsigned*>(k + mx_part_at<D>(false, in_page, lane * 8 / (D / 16)));
        if constexpr (D == 128) v4 = *reinterpret_cast<const unsigned*>(v + mx_part_at<D>(true, in_page, lane));
        else v4 = *reinterpret_cast<const unsigned short*>(v + mx_part_at<D>(true, in_page, lane * 2)) |
                  static_cast<unsigned>(*reinterpret_cast<const unsigned short*>(v + mx_part_at<D>(true, in_page, lane * 2 + 1))) << 16;
        ks = k[mx_scale_at<D>(in_page, lane >> 2)];
        vs = v[mx_scale_at<D>(in_page, lane >> 2)];
    }
    const int64_t out = (static_cast<int64_t>(layer) * gridDim.y + b) * p.T * per_token + at;
    typedef unsigned Quad4 __attribute__((ext_vector_type(4)));
    auto put = [&](void* base, unsigned four, unsigned byte) {
        const float scale = mx_scale(byte);        // (0 for rows that are not there: their elements are 0)
        if constexpr (F32) {
            typedef float Two __attribute__((ext_vector_type(2)));
            const Two a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(four, scale, 0), c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(four, scale, 1),
                      d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(four, scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(four, scale, 3);
            typedef float Float4 __attribute__((ext_vector_type(4)));
            Float4* o = static_cast<Float4*>(base) + 2 * out;
            __builtin_nontemporal_store(Float4{a[0], a[1], c[0], c[1]}, o);
            __builtin_nontemporal_store(Float4{d[0], d[1], e[0], e[1]}, o + 1);
        } else {
            const Quad4 x = {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(four, scale, 0)),
                             __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(four, scale, 1)),
                             __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(four, scale, 2)),
                             __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(four, scale, 3))};
            __builtin_nontemporal_store(x, static_cast<Quad4*>(base) + out);
        }
    };
    put(p.k_out, k4, ks);
    put(p.v_out, v4, vs);
}

// ---- update after acceptance -------------------------------------------------------------------------------------------------------
// As with whole elements (kv_compact.hip): few rows, a chain of dependent trips (lengths and path, page table, rows), every
// wavefront for itself.  A lane has one part of a token's row of one side and head (4 bytes, 2 with D = 64; the parts of a
// row lie 16 bytes apart in the values) and, where the part's number is below D / 32, one of the row's scale bytes; it walks the path
// in order, MC_BATCH rows in flight (us with the rows read back, 4 / 8 / 16 in flight: 4 rows of 32 layers x 8 heads 5.4 / 5.5 / 6.1, 12 rows 7.3 / 7.2 /
// 6.8, up to 9 rows of 16 sequences x 94 layers x 4 heads 18.7 / 19.1 / 19.1).  In place: no lane touches another's bytes, and the path
// increases strictly, so a row's destination P + k never is a later row's source.
// Bound by lines: a row's values lie in 16 pieces over 256 bytes and its scales in 4 over 64, which move whole both ways.
constexpr int MC_THREADS = 256, MC_BATCH = 4;
static_assert(64 % MC_BATCH == 0 && GRAFT_MAX_NODES <= 128, "a batch stays within one register of the lanes' rows");

struct CompactMxParams {
    unsigned char *k, *v;
    int32_t *new_prefix_len, *status;
    int64_t layer_stride, page_stride, head_stride;            // bytes
    int32_t Hkv;
};

template <int D>
__global__ __launch_bounds__(MC_THREADS) void kv_compact_mx_kernel(const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ accept_len,
                                                                   const int32_t* __restrict__ path, const int32_t* __restrict__ block_table,
                                                                   int32_t depth_cap, int32_t K_max, int32_t max_pages, CompactMxParams p) {
    using Unit = std::conditional_t<D == 128, unsigned, unsigned short>;
    const int b = blockIdx.z, layer = blockIdx.y, lane = threadIdx.x & 63;
    const int32_t* path_b = path + static_cast<int64_t>(b) * (depth_cap + 1);
    const int32_t P = __builtin_amdgcn_readfirstlane(prefix_len[b]), a = __builtin_amdgcn_readfirstlane(accept_len[b]);
    const int32_t first = path_b[0];
    int32_t node[2], above[2];                     // path[k] and path[k - 1] of this lane's rows k
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int32_t k = lane + 1 + 64 * h;
        node[h] = path_b[k < depth_cap ? k : depth_cap];
        above[h] = path_b[k - 1 < depth_cap ? k - 1 : depth_cap];
    }
    bool bad = first != 0, outside = false;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const bool used = lane + 1 + 64 * h <= a;
        bad = bad || (used && (node[h] <= above[h] || node[h] >= K_max));
        outside = outside || (used && static_cast<int64_t>(P) + node[h] >= static_cast<int64_t>(max_pages) * GRAFT_PAGE_SIZE);
    }
    int32_t st = 0;
    if (P < 0 || a < 0 || a > depth_cap) st = GRAFT_STATUS_BAD_LENGTH;
    else if (__builtin_amdgcn_ballot_w64(bad) != 0) st = GRAFT_STATUS_BAD_TREE;
    else if (__builtin_amdgcn_ballot_w64(outside) != 0) st = GRAFT_STATUS_BAD_LENGTH;
    if (layer == 0 && blockIdx.x == 0 && threadIdx.x == 0) {
        p.status[b] = st;
        p.new_prefix_len[b] = st == 0 ? P + a + 1 : P;
    }
    if (st != 0 || a == 0) return;                 // uniform

    // each row's page (its byte offset) and place in the page, source and destination
    const int32_t* table = block_table + static_cast<int64_t>(b) * max_pages;
    u64 src[2], dst[2];
    int src_at[2], dst_at[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int32_t k = lane + 1 + 64 * h;
        const int32_t from = k <= a ? P + node[h] : 0, to = k <= a ? P + k : 0;
        src[h] = static_cast<u64>(static_cast<int64_t>(table[from / GRAFT_PAGE_SIZE]) * p.page_stride);
        dst[h] = static_cast<u64>(static_cast<int64_t>(table[to / GRAFT_PAGE_SIZE]) * p.page_stride);
        src_at[h] = from & (GRAFT_PAGE_SIZE - 1);
        dst_at[h] = to & (GRAFT_PAGE_SIZE - 1);
    }
    // 32 lanes a head: 16 parts of its keys, 16 of its values.  All lanes stay (their rows are read across lanes); those behind the
    // last head load its rows and store nothing.
    const int column = blockIdx.x * blockDim.x + threadIdx.x;
    const bool live = column < p.Hkv * 32;
    const int g = live ? column >> 5 : p.Hkv - 1, part = column & 15, block = part < D / 32 ? part : 0;
    const bool values = column & 16, scales = live && part < D / 32;
    unsigned char* base = (values ? p.v : p.k) + layer * p.layer_stride + g * p.head_stride;
    auto of_lane = [](u64 v, int l) {
        return (static_cast<u64>(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(v >> 32), l))) << 32) |
               static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(v), l));
    };
    for (int k0 = 0; k0 < a; k0 += MC_BATCH) {     // row k of the path is number k - 1 here
        const int half = k0 >> 6;
        Unit unit[MC_BATCH];
        unsigned char scale[MC_BATCH];
#pragma unroll
        for (int j = 0; j < MC_BATCH; ++j) {       // (no branch around a load; behind the end the last row is read again)
            const int l = (k0 + j < a ? k0 + j : a - 1) & 63;
            const unsigned char* page = base + of_lane(half ? src[1] : src[0], l);
            const int t = __builtin_amdgcn_readlane(half ? src_at[1] : src_at[0], l);
            unit[j] = *reinterpret_cast<const Unit*>(page + mx_part_at<D>(values, t, part));
            scale[j] = page[mx_scale_at<D>(t, block)];
        }
#pragma unroll
        for (int j = 0; j < MC_BATCH; ++j) {
            const int l = (k0 + j) & 63;
            unsigned char* page = base + of_lane(half ? dst[1] : dst[0], l);
            const int t = __builtin_amdgcn_readlane(half ? dst_at[1] : dst_at[0], l);
            if (k0 + j < a) {
                if (live) *reinterpret_cast<Unit*>(page + mx_part_at<D>(values, t, part)) = unit[j];
                if (scales) page[mx_scale_at<D>(t, block)] = scale[j];
            }
        }
    }
}

static bool bad_mx_strides(int64_t page_stride, int64_t head_stride, int64_t layer_stride, int32_t n_layers, int32_t D) {
    return page_stride < mx_run_bytes(D) || head_stride < mx_run_bytes(D) || page_stride % 16 != 0 || head_stride % 16 != 0 || layer_stride < 0 ||
           (n_layers > 1 && layer_stride < 1) || layer_stride % 16 != 0;
}

}  // namespace graft

extern "C" int32_t graft_kv_gather_mx(const void* k_cache, const void* v_cache, int64_t layer_stride, int32_t n_layers, int64_t page_stride,
                                      int64_t head_stride, const int32_t* block_table, int32_t max_pages, const int32_t* start,
                                      const int32_t* count, int32_t B, int32_t T, int32_t Hkv, int32_t D, int32_t dtype, void* k_out,
                                      void* v_out, int32_t* status, void* stream) {
    using namespace graft;
    if (!k_cache || !v_cache || !block_table || !count || !k_out || !v_out || !status) return GRAFT_ERR_NULL;
    if (dtype != GRAFT_F32 && dtype != GRAFT_BF16) return GRAFT_ERR_DTYPE;
    if (B < 1 || B > 65535 || n_layers < 1 || n_layers > 65535 || T < 1 || Hkv < 1 || Hkv > 65535 || (D != 64 && D != 128) || max_pages < 1 ||
        max_pages > 262144 || bad_mx_strides(page_stride, head_stride, layer_stride, n_layers, D))
        return GRAFT_ERR_SHAPE;
    if ((reinterpret_cast<size_t>(k_cache) | reinterpret_cast<size_t>(v_cache) | reinterpret_cast<size_t>(k_out) | reinterpret_cast<size_t>(v_out)) & 15)
        return GRAFT_ERR_SHAPE;
    const int64_t blocks = (static_cast<int64_t>(T) * Hkv * (D / 8) + KG_THREADS - 1) / KG_THREADS;
    if (blocks >= (1ll << 32) / KG_THREADS) return GRAFT_ERR_SHAPE;
    const GatherParams p{static_cast<const unsigned char*>(k_cache), static_cast<const unsigned char*>(v_cache), k_out, v_out, status,
                         layer_stride, page_stride, head_stride, T, Hkv};
    const dim3 grid(static_cast<unsigned>(blocks), B, n_layers);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(KG_THREADS), 0, static_cast<hipStream_t>(stream), start, count, block_table, max_pages, p);
    };
    if (D == 128) { if (dtype == GRAFT_F32) launch(kv_gather_mx_kernel<128, true>); else launch(kv_gather_mx_kernel<128, false>); }
    else if (dtype == GRAFT_F32) launch(kv_gather_mx_kernel<64, true>);
    else launch(kv_gather_mx_kernel<64, false>);
    return check_launch();
}

extern "C" int32_t graft_kv_compact_mx(void* k_cache, void* v_cache, int64_t layer_stride, int32_t n_layers, int64_t page_stride,
                                       int64_t head_stride, const int32_t* block_table, int32_t max_pages, const int32_t* prefix_len,
                                       const int32_t* path, const int32_t* accept_len, int32_t B, int32_t depth_cap, int32_t K_max, int32_t Hkv,
                                       int32_t D, int32_t* new_prefix_len, int32_t* status, void* stream) {
    using namespace graft;
    if (!k_cache || !v_cache || !block_table || !prefix_len || !path || !accept_len || !new_prefix_len || !status) return GRAFT_ERR_NULL;
    if (B < 1 || B > 65535 || n_layers < 1 || n_layers > 65535 || depth_cap < 0 || depth_cap >= GRAFT_MAX_NODES || K_max < 1 ||
        K_max > GRAFT_MAX_NODES || Hkv < 1 || Hkv > 65535 || (D != 64 && D != 128) || max_pages < 1 || max_pages > 262144 ||
        bad_mx_strides(page_stride, head_stride, layer_stride, n_layers, D))
        return GRAFT_ERR_SHAPE;
    if ((reinterpret_cast<size_t>(k_cache) | reinterpret_cast<size_t>(v_cache)) & 15) return GRAFT_ERR_SHAPE;
    // Every workgroup of a sequence reads prefix_len[b] and accept_len[b] when it starts and one of them writes new_prefix_len[b].
    if ((new_prefix_len < prefix_len + B && prefix_len < new_prefix_len + B) || (new_prefix_len < accept_len + B && accept_len < new_prefix_len + B))
        return GRAFT_ERR_SHAPE;
    const CompactMxParams p{static_cast<unsigned char*>(k_cache), static_cast<unsigned char*>(v_cache), new_prefix_len, status, layer_stride,
                            page_stride, head_stride, Hkv};
    const int columns = Hkv * 32, waves = (columns + 63) / 64;                 // per layer and sequence
    const int threads = 64 * waves < MC_THREADS ? 64 * waves : MC_THREADS;
    const dim3 grid((columns + threads - 1) / threads, n_layers, B);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, static_cast<hipStream_t>(stream), prefix_len, accept_len, path, block_table, depth_cap,
                           K_max, max_pages, p);
    };
    if (D == 128) launch(kv_compact_mx_kernel<128>);
    else launch(kv_compact_mx_kernel<64>);
    return check_launch();
}
