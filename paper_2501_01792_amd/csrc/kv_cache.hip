// Rows of the paged K/V cache (16 bits, int8, e4m3): written, and quantised as they are written, by hk_kv_store; read back by
// hk_kv_load.  Both only move bytes: DH / 8 lanes take a row, 8 elements (16 bytes in 16 bits) each, K and V together; the
// largest magnitude of a row is found among its lanes, as the integer that its bits are, so that infinities and NaN order
// above every finite value.
//
// Memory bounds both.  Alone, over 814 MB (32 requests x 32 heads x 1024 tokens): written 4.7 TB/s (int8) and 5.0 (e4m3), 5.6 in 16
// bits; read back 5.6, 5.5 and 5.5.  A copy of 1 GiB reaches 5.2, a fill 6.8: what a mixture of reads and writes reaches lies
// between, by its shares.  Prompts of 8 requests of 1024 to 2048 tokens, 8 heads of 128, bf16 to e4m3 and back again 31 us, 136 MB.
// Rows leave non-temporal (147 us without, for 122, where 32 requests x 32 heads of 512 to 1024 tokens are read back).  What the
// quantisation costs is kept small: the quotients take two multiply-adds each where a division takes ten instructions (prompts
// written at 3.7 TB/s with it, 4.7 without).  Small calls are a launch (3.4 us) and the host's 6.
#include "hk_internal.h"
#include "kv_format.h"

#include <type_traits>

namespace hk {
namespace {

using namespace kvfmt;
constexpr int kThreads = 256;

// Where token t of a request goes: KV block (>= 0), ~ACT block (< 0) of the table's row; false: nowhere.
__device__ __forceinline__ bool block_of(const KvCacheView &c, int r, int t, int *e)
{
    if (t < 0 || (t >> c.blk_log2) >= c.max_blocks) return false;
    *e = c.block_table[(int64_t)r * c.max_blocks + (t >> c.blk_log2)];
    return *e >= 0 ? *e < c.P_kv : ~*e < c.P_act;
}

template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }

template <int FMT, int DT>
__device__ __forceinline__ void put8(void *pool, float *scales, int64_t row, int DH, int c, u32x4_t raw)
{
    typedef typename Elem<DT>::V8 vec8_t;
    if constexpr (FMT == k16) {
        __builtin_nontemporal_store(raw, reinterpret_cast<u32x4_t *>(static_cast<uint16_t *>(pool) + row * DH + 8 * c));
    } else {
        // the largest magnitude, two at a time, then among the row's lanes (8 or 16 neighbours: moves on the vector ALU)
        typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
        u16x2_t two = {0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) two = __builtin_elementwise_max(two, __builtin_bit_cast(u16x2_t, raw[j] & 0x7fff7fffu));
        uint32_t top = max((uint32_t)two[0], (uint32_t)two[1]);
        top = max(top, moved<0xb1>(top));                  // lane ^ 1
        top = max(top, moved<0x4e>(top));                  // lane ^ 2
        top = max(top, moved<0x141>(top));                 // lane ^ 7
        if (DH == 128) top = max(top, moved<0x128>(top));  // lane ^ 8
        const bool finite = top < (DT == 1 ? 0x7f80u : 0x7c00u);
        const float most_x = (float)__builtin_bit_cast(typename Elem<DT>::T, (uint16_t)top);
        float scale = most_x / most<FMT>();
        scale = scale < kLeastScale ? kLeastScale : scale;
        const vec8_t v = __builtin_bit_cast(vec8_t, raw);
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = finite ? (float)v[j] : 0.f;
        scale = finite ? scale : 1.f;
        const u32x2_t code = encode8<FMT>(x, scale, 1.f / scale);
        __builtin_nontemporal_store(code, reinterpret_cast<u32x2_t *>(static_cast<uint8_t *>(pool) + row * DH + 8 * c));
        if (c == 0) scales[row] = finite ? scale : __builtin_nanf("");
    }
}

// tt_log2: 2^tt_log2 tokens of a head are neighbours in the launch, so that their codes and scales, which are neighbours in a
// block, leave together.
template <int DH, int DT, int FMT>
__global__ __launch_bounds__(kThreads) void kv_store_kernel(KvStoreArgs a, int tt_log2, int groups, int64_t rows)
{
    constexpr int LPR = DH / 8;
    const int64_t id = (int64_t)blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
    if (id >= rows) return;                                // whole rows
    const int c = threadIdx.x % LPR;
    const uint32_t rest = (uint32_t)(id >> tt_log2);
    const int h = rest % (uint32_t)a.c.Hkv;
    const uint32_t rg = rest / (uint32_t)a.c.Hkv;
    const int r = rg / (uint32_t)groups;
    const int i = (int)(rg % (uint32_t)groups << tt_log2) + (int)(id & ((1 << tt_log2) - 1));
    int n = a.n_new ? a.n_new[r] : a.T;
    n = n < a.T ? n : a.T;
    if (i >= n) return;
    const int src = a.pick ? a.pick[(int64_t)r * a.T + i] : i;
    const int t = a.c.seq_len[r] - n + i;
    int e;
    if (src < 0 || src >= a.T || !block_of(a.c, r, t, &e)) return;
    const int64_t from = ((int64_t)r * a.T + src) * a.c.Hkv + h;
    const int blk = 1 << a.c.blk_log2, at = t & (blk - 1);
    if (e < 0) {                                           // an ACT block: this head's part of the layer input (d = Hkv * DH)
        if (!a.x) return;
        const u32x4_t v = *reinterpret_cast<const u32x4_t *>(static_cast<const uint16_t *>(a.x) + from * DH + 8 * c);
        *reinterpret_cast<u32x4_t *>(static_cast<uint16_t *>(a.act_pool) + (((int64_t)~e << a.c.blk_log2) + at) * a.d + h * DH + 8 * c) = v;
        return;
    }
    const u32x4_t kv = *reinterpret_cast<const u32x4_t *>(static_cast<const uint16_t *>(a.k) + from * DH + 8 * c);
    const u32x4_t vv = *reinterpret_cast<const u32x4_t *>(static_cast<const uint16_t *>(a.v) + from * DH + 8 * c);
    const int64_t row = (((int64_t)e * a.c.Hkv + h) << a.c.blk_log2) + at;
    put8<FMT, DT>(a.c.K_pool, a.c.K_scale, row, DH, c, kv);
    put8<FMT, DT>(a.c.V_pool, a.c.V_scale, row, DH, c, vv);
}

template <int FMT, int DT>
__device__ __forceinline__ u32x4_t widen8(u32x2_t code, float scale)
{
    typedef typename Elem<DT>::V8 vec8_t;
    vec8_t v;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        float x[4];
        decode4<FMT>(code[w], x);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * w + j] = (typename Elem<DT>::T)(x[j] * scale);
    }
    return __builtin_bit_cast(u32x4_t, v);
}

constexpr int kLoadRows = 2;                               // rows of K and of V that a thread has on the way

template <int DH, int DT, int FMT>
__global__ __launch_bounds__(kThreads) void kv_load_kernel(KvLoadArgs a, int tiles)
{
    constexpr int LPR = DH / 8, RPB = kThreads / LPR;
    const int pair = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int r = pair / a.c.Hkv, h = pair % a.c.Hkv, c = threadIdx.x % LPR;
    const int64_t len = a.c.seq_len[r];
    int64_t from[kLoadRows];
    int to[kLoadRows];
#pragma unroll
    for (int u = 0; u < kLoadRows; ++u) {
        const int i = (tile * kLoadRows + u) * RPB + threadIdx.x / LPR;
        const int64_t t = (int64_t)a.tok_off + i;
        int e = -1;
        to[u] = i < a.L_cap && t < len && t <= 0x7fffffff && block_of(a.c, r, (int)t, &e) && e >= 0 ? i : -1;
        from[u] = to[u] < 0 ? 0 : (((int64_t)e * a.c.Hkv + h) << a.c.blk_log2) + (t & ((1 << a.c.blk_log2) - 1));
    }
    if constexpr (FMT == k16) {
        u32x4_t k[kLoadRows], v[kLoadRows];
#pragma unroll
        for (int u = 0; u < kLoadRows; ++u)
            if (to[u] >= 0) {
                k[u] = *reinterpret_cast<const u32x4_t *>(static_cast<const uint16_t *>(a.c.K_pool) + from[u] * DH + 8 * c);
                v[u] = *reinterpret_cast<const u32x4_t *>(static_cast<const uint16_t *>(a.c.V_pool) + from[u] * DH + 8 * c);
            }
#pragma unroll
        for (int u = 0; u < kLoadRows; ++u)
            if (to[u] >= 0) {
                const int64_t at = ((int64_t)pair * a.L_cap + to[u]) * DH + 8 * c;
                __builtin_nontemporal_store(k[u], reinterpret_cast<u32x4_t *>(static_cast<uint16_t *>(a.K_out) + at));
                __builtin_nontemporal_store(v[u], reinterpret_cast<u32x4_t *>(static_cast<uint16_t *>(a.V_out) + at));
            }
    } else {
        u32x2_t k[kLoadRows], v[kLoadRows];
        float ks[kLoadRows], vs[kLoadRows];
#pragma unroll
        for (int u = 0; u < kLoadRows; ++u)
            if (to[u] >= 0) {
                k[u] = *reinterpret_cast<const u32x2_t *>(static_cast<const uint8_t *>(a.c.K_pool) + from[u] * DH + 8 * c);
                v[u] = *reinterpret_cast<const u32x2_t *>(static_cast<const uint8_t *>(a.c.V_pool) + from[u] * DH + 8 * c);
                ks[u] = a.c.K_scale[from[u]];
                vs[u] = a.c.V_scale[from[u]];
            }
#pragma unroll
        for (int u = 0; u < kLoadRows; ++u)
            if (to[u] >= 0) {
                const int64_t at = ((int64_t)pair * a.L_cap + to[u]) * DH + 8 * c;
                __builtin_nontemporal_store(widen8<FMT, DT>(k[u], ks[u]), reinterpret_cast<u32x4_t *>(static_cast<uint16_t *>(a.K_out) + at));
                __builtin_nontemporal_store(widen8<FMT, DT>(v[u], vs[u]), reinterpret_cast<u32x4_t *>(static_cast<uint16_t *>(a.V_out) + at));
            }
    }
}

template <int DH, int DT, int FMT>
hipError_t store_as(const KvStoreArgs &a, hipStream_t s)
{
    int tt = 0;
    while (tt < 4 && (2 << tt) <= a.T) ++tt;
    const int groups = (a.T + (1 << tt) - 1) >> tt;
    const int64_t rows = (int64_t)a.B * groups * a.c.Hkv << tt;
    constexpr int per = kThreads / (DH / 8);
    hipLaunchKernelGGL((kv_store_kernel<DH, DT, FMT>), dim3((unsigned)((rows + per - 1) / per)), dim3(kThreads), 0, s, a, tt, groups, rows);
    return hipGetLastError();
}
template <int DH, int DT, int FMT>
hipError_t load_as(const KvLoadArgs &a, hipStream_t s)
{
    constexpr int per = kThreads / (DH / 8) * kLoadRows;
    const int tiles = (a.L_cap + per - 1) / per;
    hipLaunchKernelGGL((kv_load_kernel<DH, DT, FMT>), dim3((unsigned)((int64_t)a.B * a.c.Hkv * tiles)), dim3(kThreads), 0, s, a, tiles);
    return hipGetLastError();
}

template <int DH, int DT, typename Args>
hipError_t by_format(const Args &a, hipStream_t s)
{
    if constexpr (std::is_same<Args, KvStoreArgs>::value) {
        return a.format == k16 ? store_as<DH, DT, k16>(a, s) : a.format == kInt8 ? store_as<DH, DT, kInt8>(a, s) : store_as<DH, DT, kE4m3>(a, s);
    } else {
        return a.format == k16 ? load_as<DH, DT, k16>(a, s) : a.format == kInt8 ? load_as<DH, DT, kInt8>(a, s) : load_as<DH, DT, kE4m3>(a, s);
    }
}
template <typename Args>
hipError_t by_shape(const Args &a, hipStream_t s)
{
    if (a.head_dim == 128) return a.dtype == 1 ? by_format<128, 1>(a, s) : by_format<128, 0>(a, s);
    if (a.head_dim == 64) return a.dtype == 1 ? by_format<64, 1>(a, s) : by_format<64, 0>(a, s);
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_kv_store(const KvStoreArgs &a, hipStream_t s) { return a.B <= 0 || a.T <= 0 ? hipSuccess : by_shape(a, s); }
hipError_t launch_kv_load(const KvLoadArgs &a, hipStream_t s) { return a.B <= 0 || a.L_cap <= 0 ? hipSuccess : by_shape(a, s); }

}  // namespace hk
