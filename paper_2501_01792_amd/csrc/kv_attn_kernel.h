// Attention of a tree of drafted tokens (or of one query token) over the paged K/V cache, in 16 bits, int8 or e4m3.
//
// For row (node i, query head h) of a request, hk = h / g its K/V head:
//     t_j = scale q . k_j log2(e),   out = sum_j 2^(t_j - m) v_j / sum_j 2^(t_j - m)
// over the request's cached tokens and the nodes that node i sees; one pass over K and V with a running m (the usual rescaling
// of the sums where it grows), everything after the products in fp32.
//
// One wavefront takes 32 tokens at a time and all 16 MT rows of its tile; K and V are read once for all of them.
//   scores   S^T = K Q^T with mfma 16x16x32: lane (g4 = lane / 16, r16 = lane % 16) holds tokens 4 g4 .. 4 g4 + 3 of each 16 of
//            query row r16.  The reduction index may be permuted, so a lane reads K in whole 16-byte pieces.
//   weights  the four tokens a lane holds of both 16s are the 8 reduction elements of its lane group in
//   sum      out^T = V^T P^T, so P goes from one product to the other without leaving its lane.  A lane reads DH / 16 elements of
//            each of those 8 tokens and turns the block with byte permutes; row a of product i is element a DH / 16 + i.
//   8 bits   the scales are constants of a token: K's multiplies the score.  V's goes into the weight: with vs = mant 2^e,
//            2^(t + e - m) mant <= 1 for the running maximum m of t + e, so the weight keeps fp16's 11 bits whatever the
//            scales are, and the denominator takes 2^(t + e - m) 2^-e, in fp32.  A bf16 query is brought to fp16 by a power of
//            two of its row.
// A workgroup's 4 wavefronts take the 32-token tiles of a piece in turn and join at the end in LDS.  A piece that is its
// request's only one writes the output; the others leave (m, l, o) for the merge.
#pragma once
#include "hk_internal.h"
#include "kv_format.h"
#include "kv_split.h"

namespace hk {
namespace kvattn {

using namespace kvfmt;
constexpr int kThreads = 64 * kWaves;
constexpr float kLog2e = 1.4426950408889634f;

struct Params {
    KvCacheView c;
    const void *K_regen, *V_regen, *q, *k, *v;
    const int64_t *mask;
    const int32_t *n_nodes;
    void *out;
    float *partial;                                        // [slots, DH] sums, then [slots] (m, l)
    int64_t slots;
    int B, T, H, mask_stride, g, row_groups, extra;
    float scale_log2e;
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ int length_of(const KvCacheView &c, int r)
{
    const int64_t room = (int64_t)c.max_blocks << c.blk_log2;
    const int len = c.seq_len[r];
    return len < 0 ? 0 : len < room ? len : (int)room;
}

// Piece length for the lengths that the device holds (wavefront-uniform; every lane calls it).
__device__ __forceinline__ int64_t piece_length(const Params &p, int lane)
{
    if (p.extra <= 0) return piece_tokens(0, 0);
    int64_t sum = 0;
    for (int r = lane; r < p.B; r += 64) sum += length_of(p.c, r);
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    return piece_tokens(sum, p.extra);
}

// Piece x of the line of all requests' pieces -> request r, piece c of n; false: there are fewer.
__device__ __forceinline__ bool locate(const Params &p, int64_t C, int x, int lane, int &r, int &c, int &n)
{
    int before = 0;
    for (int r0 = 0; r0 < p.B; r0 += 64) {
        const int own = r0 + lane < p.B ? pieces_of(length_of(p.c, r0 + lane), C) : 0;
        int upto = own;
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(upto, off, 64);
            if (lane >= off) upto += o;
        }
        const uint64_t in = __ballot(before + upto > x);
        if (in) {
            const int at = __builtin_ctzll(in);
            n = __builtin_amdgcn_readlane(own, at);
            c = x - (before + __builtin_amdgcn_readlane(upto, at) - n);
            r = r0 + at;
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// First piece of request r, and how many it has.
__device__ __forceinline__ int first_piece(const Params &p, int64_t C, int r, int lane, int &n)
{
    int before = 0;
    for (int i = lane; i < r; i += 64) before += pieces_of(length_of(p.c, i), C);
    for (int off = 32; off > 0; off >>= 1) before += __shfl_xor(before, off, 64);
    n = pieces_of(length_of(p.c, r), C);
    return before;
}

__device__ __forceinline__ int nodes_of(const Params &p, int r)
{
    const int n = p.n_nodes ? p.n_nodes[r] : p.T;
    return n < 0 ? 0 : n < p.T ? n : p.T;
}
// Nodes that node i of request r sees, of the `nodes` that there are.
__device__ __forceinline__ uint64_t seen_by(const Params &p, int r, int i, int nodes)
{
    if (!p.k) return 0;
    const uint64_t have = nodes >= 64 ? ~0ull : (1ull << nodes) - 1;
    const uint64_t m = p.mask ? (uint64_t)p.mask[(int64_t)r * p.mask_stride + i] : (2ull << i) - 1;   // i = 63: all
    return m & have;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const void *base, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uintptr_t>(base);
    const uint64_t lo = (uint32_t)uniform((int)(uint32_t)at), hi = (uint32_t)uniform((int)(uint32_t)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(hi << 32 | lo), 0, uniform((int)bytes), 0x00020000);
}
// N bytes (4, 8, 16) at `off`, in the low words of the result.
template <int N>
__device__ __forceinline__ u32x4_t fetch(__amdgpu_buffer_rsrc_t rs, int off)
{
    if constexpr (N == 16) return __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0));
    else if constexpr (N == 8) {
        const u32x2_t v = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0));
        return u32x4_t{v[0], v[1], 0, 0};
    } else {
        return u32x4_t{(uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, 0), 0, 0, 0};
    }
}

template <int DH, int DT, int FMT, int MT>
struct Wave {
    typedef typename Elem<DT>::T elem_t;
    typedef typename Elem<DT>::V8 vec8_t;
    static constexpr int MDT = FMT == k16 ? DT : 0;        // type of the products over the cache
    typedef typename Elem<MDT>::V8 mvec8_t;
    static constexpr int KK = DH / 32, NI = DH / 16;

    mvec8_t qf[MT][KK];
    float qfac[MT];                                        // what the scores of a row are taken times
    float m[MT], l[MT];
    float4_t o[MT][NI];
    const elem_t *qrow[MT];                                // the query row of this lane's column
    uint64_t seen[MT];                                     // nodes that it sees
    int g4, r16;

    // Reduction elements of product kk that this lane holds: 8 from here on.
    __device__ __forceinline__ int k_elem(int kk) const
    {
        return FMT == k16 ? kk * 32 + g4 * 8 : (kk >> 1) * 64 + g4 * 16 + (kk & 1) * 8;
    }

    __device__ __forceinline__ void start(float scale_log2e)
    {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            vec8_t raw[KK];
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) raw[kk] = *reinterpret_cast<const vec8_t *>(qrow[mt] + k_elem(kk));
            float fac = 1.f;
            if constexpr (DT != MDT) {                     // bf16 -> fp16: the row's largest element between 1/2 and 1
                float top = 0.f;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = fmaxf(top, __builtin_fabsf((float)raw[kk][j]));
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const int ex = top > 0.f && top < INFINITY ? __builtin_amdgcn_frexp_expf(top) : 0;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                    for (int j = 0; j < 8; ++j) qf[mt][kk][j] = (_Float16)__builtin_amdgcn_ldexpf((float)raw[kk][j], -ex);
                fac = __builtin_amdgcn_ldexpf(1.f, ex);
            } else {
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) qf[mt][kk] = raw[kk];
            }
            qfac[mt] = fac * scale_log2e;
            m[mt] = -INFINITY;
            l[mt] = 0.f;
#pragma unroll
            for (int i = 0; i < NI; ++i) o[mt][i] = float4_t{0.f, 0.f, 0.f, 0.f};
        }
    }

    // Folds the scores t (log2 domain, -inf where masked) of row tile mt into (m, l, o) and returns 2^(t - m).
    __device__ __forceinline__ void softmax(int mt, float (&t)[2][4])
    {
        float top = t[0][0];
#pragma unroll
        for (int u = 1; u < 8; ++u) top = fmaxf(top, t[u >> 2][u & 3]);
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m_new = fmaxf(m[mt], top);
        const float ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m[mt] - ref);
        m[mt] = m_new;
        l[mt] *= alpha;
#pragma unroll
        for (int i = 0; i < NI; ++i) o[mt][i] *= alpha;
#pragma unroll
        for (int u = 0; u < 8; ++u) t[u >> 2][u & 3] = __builtin_amdgcn_exp2f(t[u >> 2][u & 3] - ref);
    }

    // V^T of 32 tokens: raw[s] is what this lane read of token slot s (16-bit elements) -> the NI operands.
    static __device__ __forceinline__ void turn16(const u32x4_t (&raw)[8], u32x4_t (&vt)[NI])
    {
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int s = 0; s < 4; ++s)
                vt[i][s] = __builtin_amdgcn_perm(raw[2 * s + 1][i >> 1], raw[2 * s][i >> 1], i & 1 ? 0x07060302u : 0x05040100u);
    }
    // The same from 8-bit codes, as fp16.
    static __device__ __forceinline__ void turn8(const u32x4_t (&raw)[8], u32x4_t (&vt)[NI])
    {
#pragma unroll
        for (int w = 0; w < NI / 4; ++w)
#pragma unroll
            for (int q = 0; q < 2; ++q) {                  // token slots 4 q .. 4 q + 3, elements 4 w .. 4 w + 3
                const uint32_t a = biased<FMT>(raw[4 * q][w]), b = biased<FMT>(raw[4 * q + 1][w]);
                const uint32_t c = biased<FMT>(raw[4 * q + 2][w]), d = biased<FMT>(raw[4 * q + 3][w]);
                const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
                const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
                const uint32_t e[4] = {__builtin_amdgcn_perm(cd0, ab0, 0x05040100u), __builtin_amdgcn_perm(cd0, ab0, 0x07060302u),
                                       __builtin_amdgcn_perm(cd1, ab1, 0x05040100u), __builtin_amdgcn_perm(cd1, ab1, 0x07060302u)};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    vt[4 * w + j][2 * q] = __builtin_bit_cast(uint32_t, pair_f16<FMT, false>(e[j]));
                    vt[4 * w + j][2 * q + 1] = __builtin_bit_cast(uint32_t, pair_f16<FMT, true>(e[j]));
                }
            }
    }

    // 32 cached tokens: rows n[j] of 16 at block offset base[j] (in rows of the pool), all wavefront-uniform.
    struct Tokens {
        const void *K[2], *V[2];                           // the 16 rows
        const float *ks[2], *vs[2];
        int n[2];
    };
    __device__ __forceinline__ void cached(const Tokens &tk)
    {
        constexpr int EB = FMT == k16 ? 2 : 1, RB = DH * EB;          // bytes of an element, of a row
        constexpr int VB = NI * EB;                                    // bytes of a token that a lane reads of V
        float t[MT][2][4], ks[2][4], mant[2][4];
        int e[2][4];
        u32x4_t vraw[8];
        mvec8_t kf[2][KK];
        __amdgpu_buffer_rsrc_t vrs[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const __amdgpu_buffer_rsrc_t krs = rows_at(tk.K[j], tk.n[j] * RB);
            vrs[j] = rows_at(tk.V[j], tk.n[j] * RB);
            if constexpr (FMT == k16) {
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
                    kf[j][kk] = __builtin_bit_cast(mvec8_t, fetch<16>(krs, r16 * RB + k_elem(kk) * EB));
            } else {
#pragma unroll
                for (int kp = 0; kp < KK / 2; ++kp) {
                    u32x4_t raw = fetch<16>(krs, r16 * RB + k_elem(2 * kp));
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t b = biased<FMT>(raw[w]);
                        const half2_t lo = pair_f16<FMT, false>(b), hi = pair_f16<FMT, true>(b);
                        mvec8_t &f = kf[j][2 * kp + (w >> 1)];
                        const int at = 4 * (w & 1);
                        f[at] = lo[0]; f[at + 1] = lo[1]; f[at + 2] = hi[0]; f[at + 3] = hi[1];
                    }
                }
            }
        }
#pragma unroll
        for (int s = 0; s < 8; ++s) vraw[s] = fetch<VB>(vrs[s >> 2], (4 * g4 + (s & 3)) * RB + r16 * VB);
        if constexpr (FMT != k16) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4_t a = __builtin_bit_cast(float4_t, fetch<16>(rows_at(tk.ks[j], 64), g4 * 16));
                const float4_t b = __builtin_bit_cast(float4_t, fetch<16>(rows_at(tk.vs[j], 64), g4 * 16));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ks[j][i] = a[i];
                    const float v = b[i] < kLeastScale ? kLeastScale : b[i];
                    const bool in = 4 * g4 + i < tk.n[j];
                    mant[j][i] = in ? __builtin_amdgcn_frexp_mantf(v) : 0.f;
                    e[j][i] = in ? __builtin_amdgcn_frexp_expf(v) : 0;
                }
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) s = Elem<MDT>::mfma_16x16x32(kf[j][kk], qf[mt][kk], s);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = s[i] * qfac[mt];
                    if constexpr (FMT != k16) v = __builtin_fmaf(v, ks[j][i], (float)e[j][i]);
                    t[mt][j][i] = 4 * g4 + i < tk.n[j] ? v : -INFINITY;
                }
            }
        u32x4_t vt[NI];
        if constexpr (FMT == k16) turn16(vraw, vt);
        else turn8(vraw, vt);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            softmax(mt, t[mt]);
            mvec8_t pf;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float w = t[mt][u >> 2][u & 3];
                if constexpr (FMT == k16) {
                    l[mt] += w;
                    pf[u] = (typename Elem<MDT>::T)w;
                } else {
                    l[mt] += __builtin_amdgcn_ldexpf(w, -e[u >> 2][u & 3]);
                    pf[u] = (_Float16)(w * mant[u >> 2][u & 3]);
                }
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) o[mt][i] = Elem<MDT>::mfma_16x16x32(__builtin_bit_cast(mvec8_t, vt[i]), pf, o[mt][i]);
        }
    }

    // 32 nodes from node `first` on: K, V point at the first one's row, rows are `pitch` bytes apart, n of them exist.
    __device__ __forceinline__ void drafted(const elem_t *K, const elem_t *V, int pitch, int first, int n)
    {
        float t[MT][2][4];
        vec8_t kf[2][KK];
        u32x4_t vraw[8], vt[NI];
        const uint32_t bytes = n > 0 ? (uint32_t)(n - 1) * pitch + DH * 2 : 0;
        const __amdgpu_buffer_rsrc_t krs = rows_at(K, bytes), vrs = rows_at(V, bytes);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
                kf[j][kk] = __builtin_bit_cast(vec8_t, fetch<16>(krs, (16 * j + r16) * pitch + (kk * 32 + g4 * 8) * 2));
#pragma unroll
        for (int s = 0; s < 8; ++s) vraw[s] = fetch<NI * 2>(vrs, (16 * (s >> 2) + 4 * g4 + (s & 3)) * pitch + r16 * NI * 2);
        // A weight of zero does not take an infinity or a NaN out of the product: such elements are zeros there and reach
        // the rows that see them on their own.
        bool wild = false;
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
            for (int w = 0; w < NI / 2; ++w) {
                constexpr uint32_t ex = DT == 1 ? 0x7f80u : 0x7c00u;
                const bool lo = (vraw[s][w] & ex) == ex, hi = (vraw[s][w] >> 16 & ex) == ex;
                wild = wild || lo || hi;
                vraw[s][w] = (lo ? 0u : vraw[s][w] & 0xffffu) | (hi ? 0u : vraw[s][w] & 0xffff0000u);
            }
        const bool any_wild = __ballot(wild) != 0;
        turn16(vraw, vt);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const float sc = qscale;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
                    s = Elem<DT>::mfma_16x16x32(kf[j][kk], *reinterpret_cast<const vec8_t *>(qrow[mt] + kk * 32 + g4 * 8), s);
#pragma unroll
                for (int i = 0; i < 4; ++i) t[mt][j][i] = (seen[mt] >> (first + 16 * j + 4 * g4 + i)) & 1 ? s[i] * sc : -INFINITY;
            }
            softmax(mt, t[mt]);
            vec8_t pf;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                l[mt] += t[mt][u >> 2][u & 3];
                pf[u] = (elem_t)t[mt][u >> 2][u & 3];
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) o[mt][i] = Elem<DT>::mfma_16x16x32(__builtin_bit_cast(vec8_t, vt[i]), pf, o[mt][i]);
            if (any_wild) add_wild(V, pitch, first, n, mt, t[mt]);
        }
    }
    // The infinities and NaN of V, node by node; t: the weights of this lane's row and tokens.
    __device__ __forceinline__ void add_wild(const elem_t *V, int pitch, int first, int n, int mt, const float (&t)[2][4])
    {
        for (int j = 0; j < n && j < kTileTokens; ++j) {
            float w = 0.f;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float x = __shfl(t[u >> 2][u & 3], (j >> 2 & 3) * 16 + r16, 64);
                w = (j & 16) == (u & 4) << 2 && (j & 3) == (u & 3) ? x : w;
            }
            if (!(seen[mt] >> (first + j) & 1)) continue;
            const elem_t *row = reinterpret_cast<const elem_t *>(reinterpret_cast<const char *>(V) + (int64_t)j * pitch);
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = (float)row[(4 * g4 + e) * NI + i];
                    if (!(__builtin_fabsf(v) < INFINITY)) o[mt][i][e] += w * v;
                }
        }
    }
    float qscale;                                          // scale * log2(e)
};

template <int DH, int DT, int FMT, int MT>
__global__ __launch_bounds__(kThreads) void kv_attn_kernel(Params p)
{
    typedef Wave<DH, DT, FMT, MT> wave_t;
    typedef typename wave_t::elem_t elem_t;
    constexpr int NI = wave_t::NI;
    __shared__ float join_ml[kWaves][MT * 16][2];
    __shared__ float4_t join_o[MT * NI * 64];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int rg = blockIdx.x % p.row_groups, xh = blockIdx.x / p.row_groups;
    const int h = xh % p.c.Hkv, x = xh / p.c.Hkv;
    const int64_t C = piece_length(p, lane);
    int r = x, piece = 0, pieces = 1;
    if (p.extra > 0 && !locate(p, C, x, lane, r, piece, pieces)) return;
    r = uniform(r);
    piece = uniform(piece);
    pieces = uniform(pieces);
    const int nodes = uniform(nodes_of(p, r));
    const int first_row = rg * MT * 16;
    if (first_row >= nodes * p.g) return;                  // rows of nodes that there are not
    const int len = uniform(length_of(p.c, r));
    const int t_begin = piece == 0 ? 0 : (int)(piece * C), t_end = piece + 1 < pieces ? (int)(t_begin + C) : len;

    wave_t w;
    w.g4 = lane >> 4;
    w.r16 = lane & 15;
    w.qscale = p.scale_log2e;
    bool some[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        int row = first_row + mt * 16 + w.r16;
        row = row < nodes * p.g ? row : nodes * p.g - 1;   // works on the last row, stores nothing
        const int node = row / p.g;
        w.qrow[mt] = static_cast<const elem_t *>(p.q) + (((int64_t)r * p.T + node) * p.H + h * p.g + row % p.g) * DH;
        w.seen[mt] = seen_by(p, r, node, nodes);
        some[mt] = len > 0 || w.seen[mt] != 0;
    }
    w.start(p.scale_log2e);

    const int32_t *tab = p.c.block_table + (int64_t)r * p.c.max_blocks;
    const int blk = 1 << p.c.blk_log2;
    constexpr int RB = DH * (FMT == k16 ? 2 : 1);
    int turn = t_begin / kTileTokens;                      // pieces begin at whole rounds: wavefront 0 takes the first tile
    for (int tb = t_begin + wave * kTileTokens; tb < t_end; tb += kStep) {
        typename wave_t::Tokens tk;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int t = tb + 16 * j < t_end ? tb + 16 * j : tb;      // its table entry exists
            const int here = t_end - (tb + 16 * j);
            tk.n[j] = here < 0 ? 0 : here < 16 ? here : 16;
            int e = uniform(tab[t >> p.c.blk_log2]);
            bool act = FMT == k16 && e < 0;
            int pb = e < 0 ? ~e : e;
            if constexpr (FMT == k16) {
                if ((act ? p.c.P_act : p.c.P_kv) <= 0) { act = !act; pb = 0; }       // a corrupt table cannot leave
            }
            const int P = act ? p.c.P_act : p.c.P_kv;                                // the pools
            pb = pb < P ? pb : P - 1;
            const int64_t row = (((int64_t)pb * p.c.Hkv + h) << p.c.blk_log2) + (t & (blk - 1));
            tk.K[j] = static_cast<const char *>(act ? p.K_regen : p.c.K_pool) + row * RB;
            tk.V[j] = static_cast<const char *>(act ? p.V_regen : p.c.V_pool) + row * RB;
            if constexpr (FMT != k16) {
                tk.ks[j] = p.c.K_scale + row;
                tk.vs[j] = p.c.V_scale + row;
            }
        }
        w.cached(tk);
    }
    if (p.k && piece + 1 == pieces) {
        turn = (t_end - t_begin + kTileTokens - 1) / kTileTokens;
        const int pitch = p.c.Hkv * DH * 2;
        for (int d = 0; d * kTileTokens < nodes; ++d) {
            if ((turn + d) % kWaves != wave) continue;
            const int64_t at = (((int64_t)r * p.T + d * kTileTokens) * p.c.Hkv + h) * DH;
            const int n = nodes - d * kTileTokens;
            w.drafted(static_cast<const elem_t *>(p.k) + at, static_cast<const elem_t *>(p.v) + at, pitch, d * kTileTokens,
                      n < kTileTokens ? n : kTileTokens);
        }
    }

    // The wavefronts' results about their common maximum, added in the order of the wavefronts.
    float ref[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        w.l[mt] += __shfl_xor(w.l[mt], 16, 64);
        w.l[mt] += __shfl_xor(w.l[mt], 32, 64);
        if (w.g4 == 0) {
            join_ml[wave][mt * 16 + w.r16][0] = w.m[mt];
            join_ml[wave][mt * 16 + w.r16][1] = w.l[mt];
        }
    }
    __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        float top = -INFINITY;
#pragma unroll
        for (int q = 0; q < kWaves; ++q) top = fmaxf(top, join_ml[q][mt * 16 + w.r16][0]);
        ref[mt] = top == -INFINITY ? 0.f : top;
        const float mine = __builtin_amdgcn_exp2f(w.m[mt] - ref[mt]);
#pragma unroll
        for (int i = 0; i < NI; ++i) w.o[mt][i] *= mine;
        float l = 0.f;
#pragma unroll
        for (int q = 0; q < kWaves; ++q) l += join_ml[q][mt * 16 + w.r16][1] * __builtin_amdgcn_exp2f(join_ml[q][mt * 16 + w.r16][0] - ref[mt]);
        w.l[mt] = l;
        w.m[mt] = top;
    }
    for (int q = 1; q < kWaves; ++q) {
        if (wave == q) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < NI; ++i) join_o[(mt * NI + i) * 64 + lane] = w.o[mt][i];
        }
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < NI; ++i) w.o[mt][i] += join_o[(mt * NI + i) * 64 + lane];
        }
        __syncthreads();
    }
    if (wave != 0) return;

#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = first_row + mt * 16 + w.r16;
        if (row >= nodes * p.g) continue;
        if (pieces == 1) {
            elem_t *dst = static_cast<elem_t *>(p.out) + (w.qrow[mt] - static_cast<const elem_t *>(p.q));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                typedef elem_t vec_t __attribute__((ext_vector_type(NI)));
                vec_t v;
#pragma unroll
                for (int i = 0; i < NI; ++i) v[i] = some[mt] ? (elem_t)(w.o[mt][i][e] / w.l[mt]) : (elem_t)0.f;
                *reinterpret_cast<vec_t *>(dst + (4 * w.g4 + e) * NI) = v;
            }
        } else {
            const int64_t slot = ((int64_t)x * p.c.Hkv + h) * ((int64_t)p.T * p.g) + row;
            float *dst = p.partial + slot * DH;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < NI; i += 4)
                    *reinterpret_cast<float4_t *>(dst + (4 * w.g4 + e) * NI + i) =
                        float4_t{w.o[mt][i][e], w.o[mt][i + 1][e], w.o[mt][i + 2][e], w.o[mt][i + 3][e]};
            if (w.g4 == 0) *reinterpret_cast<float2 *>(p.partial + p.slots * DH + 2 * slot) = make_float2(w.m[mt], w.l[mt]);
        }
    }
}

template <int DH, int DT, int FMT>
hipError_t launch_as(const Params &p, const Plan &pl, hipStream_t s)
{
    const dim3 grid((unsigned)pl.groups), block(kThreads);
    if (pl.tiles == 1) hipLaunchKernelGGL((kv_attn_kernel<DH, DT, FMT, 1>), grid, block, 0, s, p);
    else if (pl.tiles == 2) hipLaunchKernelGGL((kv_attn_kernel<DH, DT, FMT, 2>), grid, block, 0, s, p);
    else if (pl.tiles == 3) hipLaunchKernelGGL((kv_attn_kernel<DH, DT, FMT, 3>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((kv_attn_kernel<DH, DT, FMT, 4>), grid, block, 0, s, p);
    return hipGetLastError();
}

template <int FMT>
hipError_t launch_format(const Params &p, const Plan &pl, int head_dim, int dtype, hipStream_t s)
{
    if (head_dim == 128) return dtype == 1 ? launch_as<128, 1, FMT>(p, pl, s) : launch_as<128, 0, FMT>(p, pl, s);
    return dtype == 1 ? launch_as<64, 1, FMT>(p, pl, s) : launch_as<64, 0, FMT>(p, pl, s);
}

// One translation unit each.
hipError_t launch_16(const Params &p, const Plan &pl, int head_dim, int dtype, hipStream_t s);
hipError_t launch_int8(const Params &p, const Plan &pl, int head_dim, int dtype, hipStream_t s);
hipError_t launch_e4m3(const Params &p, const Plan &pl, int head_dim, int dtype, hipStream_t s);

}  // namespace kvattn
}  // namespace hk
