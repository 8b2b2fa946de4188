// Attention of a tree of drafted tokens (or of one query token) over the paged K/V cache, in 16 bits, int8 or e4m3.
//
// For row (node i, query head h) of a request, hk = h / g its K/V head:
//     t_j = scale q . k_j log2(e),   out = sum_j 2^(t_j - m) v_j / sum_j 2^(t_j - m)
// over the request's cached tokens and the nodes that node i sees; one pass over K and V with a running m (the usual rescaling
// of the sums where it grows), everything after the products in fp32.
//
// One wavefront takes 32 tokens at a time and 16 MT query rows.
//   scores   S^T = K Q^T with mfma 16x16x32: lane (g4 = lane / 16, r16 = lane % 16) holds tokens 4 g4 .. 4 g4 + 3 of each 16 of
//            query row r16.  The reduction index may be permuted, so a lane reads K in whole 16-byte pieces.
//   weights  the four tokens a lane holds of both 16s are the 8 reduction elements of its lane group in
//   sum      out^T = V^T P^T, so P goes from one product to the other without leaving its lane.  A lane reads DH / 16 elements of
//            each of those 8 tokens and turns the block with byte permutes; row a of product i is element a DH / 16 + i.
//   8 bits   the scales are constants of a token: K's multiplies the score.  V's goes into the weight: with vs = mant 2^e,
//            2^(t + e - m) mant <= 1 for the running maximum m of t + e, so the weight keeps fp16's 11 bits whatever the
//            scales are, and the denominator takes 2^(t + e - m) 2^-e, in fp32.  Scales reach from 2^-100 (a row of zeros) to
//            2^121, so that weight may be nothing in fp32 where the denominator's part is not: tiles with scales that far apart
//            take count_far(), and factors between running maxima are kept from vanishing (times_power).  A bf16 query is brought to
//            fp16 by a power of two of its row.
// Up to 32 rows (kv_attn_kernel): a workgroup's 4 wavefronts take the 32-token tiles of a piece in turn, rows of K and V go from
// memory to registers, and they join at the end in LDS.  More rows: kv_attn_rows.h.  A piece that is its request's only one
// writes the output; the others leave (m, l, o) for the merge.
//
// What bounds the streaming form is memory: 64 requests of up to 4096 tokens, 72 heads of 128, e4m3, bf16 (3.8 GB): 607 us, 6.27
// TB/s; 16 bits, 8 query heads on each of 8 K/V heads, 4 requests of 16384 to 32768 tokens (375 MB): 69 us, 5.4 TB/s; int8, 32
// requests x 32 heads of 512 to 1024 tokens (211 MB): 43 us, 4.9 TB/s, the longest requests' last rounds with ever fewer of them
// on the chip.  So a wavefront keeps a whole tile on its way while it takes one in: the loop asks for the next rows as registers
// fall free, the table entry of the one after by a scalar load, and nothing in it waits for more than it uses (1064 us for the
// first of these before).  Rows that one workgroup reads are loaded non-temporal: caches of several layers leave nothing of them
// for the next step (85 to 78 us for a second one, 48 to 42 for the third; rows that the last-level cache still holds, the same
// 211 MB read over and over, would take 36).
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
    float *partial;                                        // [slots, DH] sums, [slots] (m, l), what the merge has to know
    int64_t slots;
    int B, T, H, mask_stride, g, extra, groups;            // groups: workgroups of the launch
    float scale_log2e;
};

// The kernels in a cache's format; a translation unit each.
hipError_t launch_16(const Params &p, const Plan &pl, int head_dim, int dtype, hipStream_t s);
hipError_t launch_int8(const Params &p, const Plan &pl, int head_dim, int dtype, hipStream_t s);
hipError_t launch_e4m3(const Params &p, const Plan &pl, int head_dim, int dtype, hipStream_t s);

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Element i (wavefront-uniform) of an array that no kernel of the call writes, by a scalar load: counted apart from the loads
// of K and V, so that waiting for it waits for nothing else.
__device__ __forceinline__ int scalar_at(const int32_t *a, int64_t i)
{
    typedef const __attribute__((address_space(4))) int32_t *const_ptr_t;
    return ((const_ptr_t)(uintptr_t)a)[i];
}

// r may differ from lane to lane.
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

// What a workgroup works on.
struct Place {
    int h, x;                                              // K/V head, piece of the line of all pieces
    int r, piece, pieces, nodes, len, t_begin, t_end;      // request, its pieces, nodes, tokens; the piece's (the part's) tokens
    bool last;                                             // the request's last piece, which takes the nodes, too
};
// false: there is nothing to do.
__device__ __forceinline__ bool place(const Params &p, int lane, Place &a)
{
    const int xh = blockIdx.x;
    a.h = xh % p.c.Hkv;
    a.x = xh / p.c.Hkv;
    a.r = a.x;
    a.piece = 0;
    a.pieces = 1;
    int64_t C = 0;
    if (p.extra > 0) {
        C = piece_length(p, lane);
        int r, piece, pieces;
        if (!locate(p, C, a.x, lane, r, piece, pieces)) return false;
        a.r = uniform(r);
        a.piece = uniform(piece);
        a.pieces = uniform(pieces);
    }
    a.nodes = uniform(nodes_of(p, a.r));
    a.len = uniform(length_of(p.c, a.r));
    a.t_begin = uniform((int)(a.piece * C));
    a.last = a.piece + 1 == a.pieces;
    a.t_end = uniform(a.last ? a.len : (int)(a.t_begin + C));
    return true;
}
// First piece of a request and how many it has, for the merge.
__device__ __forceinline__ int2 *piece_notes(const Params &p, int DH) { return reinterpret_cast<int2 *>(p.partial + p.slots * (DH + 2)); }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const void *base, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uintptr_t>(base);
    const uint64_t lo = (uint32_t)uniform((int)(uint32_t)at), hi = (uint32_t)uniform((int)(uint32_t)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(hi << 32 | lo), 0, uniform((int)bytes), 0x00020000);
}
// N bytes (4, 8, 16) at `off`.  Whole vectors, so that what a loop carries stays in the registers that the load fills.
template <int N>
struct WordsOf;
template <>
struct WordsOf<4> { typedef uint32_t type; };
template <>
struct WordsOf<8> { typedef u32x2_t type; };
template <>
struct WordsOf<16> { typedef u32x4_t type; };
template <int N>
using Words = typename WordsOf<N>::type;
__device__ __forceinline__ uint32_t word(uint32_t v, int) { return v; }
__device__ __forceinline__ uint32_t word(u32x2_t v, int i) { return v[i]; }
__device__ __forceinline__ uint32_t word(u32x4_t v, int i) { return v[i]; }
constexpr int kStreamed = 2;                               // cache policy of rows that one workgroup reads: non-temporal
template <int N, int AUX = 0>
__device__ __forceinline__ Words<N> fetch(__amdgpu_buffer_rsrc_t rs, int off)
{
    if constexpr (N == 16) return __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, AUX));
    else if constexpr (N == 8) return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, AUX));
    else return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, AUX);
}

// The largest over the four lane groups of a row.
__device__ __forceinline__ float max_over_groups(float v)
{
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    u2 s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    uint32_t a = s[0], b = s[1];
    v = fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
    s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    a = s[0];
    b = s[1];
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// 2^d below fp32's normal numbers, which the exponential gives as 0, is 2^-126 times 2^(d + 126).
constexpr float kLeastPower = -126.f;
__device__ __forceinline__ bool is_far(float d) { return d < kLeastPower && d > -INFINITY; }
__device__ __forceinline__ float times_power(float v, float d)
{
    const bool far = d < kLeastPower;
    return v * __builtin_amdgcn_exp2f(far ? d - kLeastPower : d) * (far ? 0x1p-126f : 1.f);
}

// The scales of a tile, one a lane (`sc`: K's in lanes 0 .. 31, V's in the others), as its scores and weights take them: [0, 32)
// K's times the softmax scale, [32, 64) log2 of V's, [96, 128) the reciprocals of V's.  Tokens that do not exist (n0, n1 of the two
// 16s do): 0 s - inf, and no part of the denominator.  Returns whether a scale of V lies outside [kNearLow, kNearHigh]: among
// scales within it a weight below fp32's numbers belongs to a token 62 binary orders below another one.
constexpr float kNearLow = 0x1p-48f, kNearHigh = 0x1p16f;
constexpr int kScales = 4 * kTileTokens;
__device__ __forceinline__ const float *scale_at(const float *ks0, const float *ks1, const float *vs0, const float *vs1, int lane)
{
    const uintptr_t k0 = reinterpret_cast<uintptr_t>(ks0), k1 = reinterpret_cast<uintptr_t>(ks1);
    const uintptr_t v0 = reinterpret_cast<uintptr_t>(vs0), v1 = reinterpret_cast<uintptr_t>(vs1);
    const uintptr_t a = lane & 16 ? k1 : k0, b = lane & 16 ? v1 : v0;
    return reinterpret_cast<const float *>(lane < 32 ? a : b) + (lane & 15);
}
__device__ __forceinline__ uint32_t put_scales(float *to, float sc, int n0, int n1, int lane, float scale)
{
    const int tok = lane & 31;
    const bool in = (tok & 15) < (tok < 16 ? n0 : n1);
    const float v = sc < kLeastScale ? kLeastScale : sc;
    const float lv = in ? __builtin_amdgcn_logf(v) : -INFINITY, kq = in ? sc * scale : 0.f;
    to[lane] = lane < 32 ? kq : lv;
    to[64 + lane] = in ? __builtin_amdgcn_rcpf(v) : 0.f;
    // (the bits of positive floats order as they do; V's are those of the upper half of the wavefront)
    constexpr uint32_t low = __builtin_bit_cast(uint32_t, kNearLow), high = __builtin_bit_cast(uint32_t, kNearHigh);
    return (uint32_t)(__ballot(in && __builtin_bit_cast(uint32_t, v) - low > high - low) >> 32);
}

// Waits until at most N of this wavefront's loads are on their way.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    static_assert(N <= 63, "vmcnt counts to 63");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0F70);
}

// How far the running maximum may lag behind, in the log2 domain: weights stay below 2^kLag, far inside fp16, and most tiles move
// no sums.  0 instead: 16 requests of up to 8192 tokens, 512 rows on a K/V head 376 us for 354.
constexpr float kLag = 8.f;

template <int DH, int DT, int FMT, int MT>
struct Wave {
    typedef typename Elem<DT>::T elem_t;
    typedef typename Elem<DT>::V8 vec8_t;
    static constexpr int MDT = FMT == k16 ? DT : 0;        // type of the products over the cache
    typedef typename Elem<MDT>::V8 mvec8_t;
    static constexpr int KK = DH / 32, NI = DH / 16;
    static constexpr bool kOwnQ = DT == MDT;               // the products over the nodes take the same queries
    static constexpr int EB = FMT == k16 ? 2 : 1, RB = DH * EB;       // bytes of an element, of a row
    static constexpr int VB = NI * EB;                     // bytes of a token that a lane reads of V
    static constexpr int KR = FMT == k16 ? KK : KK / 2;    // 16-byte pieces of a token that a lane reads of K
    static constexpr int kTileLoads = 2 * KR + (FMT == k16 ? 0 : 1) + 8;

    mvec8_t qf[MT][KK];
    float qfac[MT];                                        // the power of two that a row's query was divided by
    float m[MT], l[MT];
    float4_t o[MT][NI];
    const elem_t *qrow[MT];                                // the query row of this lane's column
    uint64_t seen[MT];                                     // nodes that it sees
    float scale;                                           // scale * log2(e)
    int g4, r16, some;                                     // some: bit mt: the row sees something
    uint32_t wide;                                         // 8 bits, not 0: scales of V far apart have been met (wavefront-uniform)

    // Reduction elements of product kk that this lane holds: 8 from here on.
    __device__ __forceinline__ int k_elem(int kk) const
    {
        return FMT == k16 ? kk * 32 + g4 * 8 : (kk >> 1) * 64 + g4 * 16 + (kk & 1) * 8;
    }

    // The query rows of this lane's columns, from `first_row` on (rows that there are not: the last one, which is not stored).
    __device__ __forceinline__ void rows(const Params &p, const Place &at, int first_row, int lane, bool tree)
    {
        g4 = lane >> 4;
        r16 = lane & 15;
        scale = p.scale_log2e;
        some = 0;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            int row = first_row + mt * 16 + r16;
            row = row < at.nodes * p.g ? row : at.nodes * p.g - 1;
            const int node = row / p.g;
            qrow[mt] = static_cast<const elem_t *>(p.q) + (((int64_t)at.r * p.T + node) * p.H + at.h * p.g + row % p.g) * DH;
            seen[mt] = tree ? seen_by(p, at.r, node, at.nodes) : 0;
            some |= (at.len > 0 || seen[mt] != 0) << mt;
        }
    }

    // The same for the products over the nodes, and the query's operand there.
    __device__ __forceinline__ int node_elem(int kk) const { return kOwnQ ? k_elem(kk) : kk * 32 + g4 * 8; }
    __device__ __forceinline__ vec8_t node_query(int mt, int kk) const
    {
        if constexpr (kOwnQ) return __builtin_bit_cast(vec8_t, qf[mt][kk]);
        else return *reinterpret_cast<const vec8_t *>(qrow[mt] + node_elem(kk));
    }

    // The queries are asked for before the first rows of K and V: a wait for the latter is then one for the former, too.
    __device__ __forceinline__ void ask_q()
    {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) qf[mt][kk] = *reinterpret_cast<const mvec8_t *>(qrow[mt] + k_elem(kk));
    }
    // The queries as the products over the cache take them.
    __device__ __forceinline__ void start()
    {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            qfac[mt] = 1.f;
            if constexpr (DT != MDT) {                     // bf16 -> fp16: the row's largest element between 1/2 and 1
                vec8_t raw[KK];
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) raw[kk] = __builtin_bit_cast(vec8_t, qf[mt][kk]);
                float top = 0.f;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = fmaxf(top, __builtin_fabsf((float)raw[kk][j]));
                top = max_over_groups(top);
                const int ex = top > 0.f && top < INFINITY ? __builtin_amdgcn_frexp_expf(top) : 0;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                    for (int j = 0; j < 8; ++j) qf[mt][kk][j] = (_Float16)__builtin_amdgcn_ldexpf((float)raw[kk][j], -ex);
                qfac[mt] = __builtin_amdgcn_ldexpf(1.f, ex);
            }
        }
    }
    __device__ __forceinline__ void clear()
    {
        wide = 0;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            m[mt] = -INFINITY;
            l[mt] = 0.f;
#pragma unroll
            for (int i = 0; i < NI; ++i) o[mt][i] = float4_t{0.f, 0.f, 0.f, 0.f};
        }
    }

    // Moves the running maxima where a row's largest score, top[mt] (this lane's part of it), has left them behind by more than
    // kLag; ref: what scores are taken about (0 while the row has seen nothing: every weight is 2^-inf).
    __device__ __forceinline__ void follow(float (&top)[MT], float (&ref)[MT])
    {
        bool behind[MT], any = false;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            top[mt] = max_over_groups(top[mt]);
            behind[mt] = top[mt] > m[mt] + kLag;
            any = any || behind[mt];
        }
        if (__ballot(any)) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const float d = m[mt] - top[mt], alpha = behind[mt] ? __builtin_amdgcn_exp2f(d) : 1.f;
                const float before = l[mt];
                l[mt] *= alpha;
                if constexpr (FMT != k16) {                // m holds V's scale, l does not
                    const bool far = behind[mt] && is_far(d);
                    if (__builtin_expect(__ballot(far) != 0, 0)) l[mt] = far ? times_power(before, d) : l[mt];
                }
                m[mt] = behind[mt] ? top[mt] : m[mt];
#pragma unroll
                for (int i = 0; i < NI; ++i) o[mt][i] *= alpha;
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) ref[mt] = m[mt] == -INFINITY ? 0.f : m[mt];
    }

    // Scores t: -inf where there is no token; 16 bits: before the scale; 8 bits: with the scale and log2(vs), inv = 1 / vs.
    __device__ __forceinline__ void references(const float4_t (&t)[MT][2], float (&ref)[MT])
    {
        float top[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            top[mt] = t[mt][0][0];
#pragma unroll
            for (int u = 1; u < 8; ++u) top[mt] = fmaxf(top[mt], t[mt][u >> 2][u & 3]);
            if constexpr (FMT == k16) top[mt] *= scale;
        }
        follow(top, ref);
    }
    // 8 bits, scales of V far apart: the part in the denominator of weights that are below fp32's numbers, which are then nothing.
    __device__ __forceinline__ void count_far(float4_t (&t)[MT][2], const float4_t (&inv)[2], const float (&ref)[MT])
    {
        bool any = false;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float low = t[mt][0][0];
#pragma unroll
            for (int u = 1; u < 8; ++u) low = fminf(low, t[mt][u >> 2][u & 3]);
            any = any || low - ref[mt] < kLeastPower;
        }
        if (__ballot(any) == 0) return;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float d = t[mt][u >> 2][u & 3] - ref[mt];
                const bool far = d < kLeastPower;
                l[mt] += far ? __builtin_amdgcn_exp2f(d - kLeastPower) * inv[u >> 2][u & 3] * 0x1p-126f : 0.f;
                t[mt][u >> 2][u & 3] = far ? -INFINITY : t[mt][u >> 2][u & 3];
                __builtin_amdgcn_sched_barrier(0);         // one by one: no registers for what is rare
            }
    }
    // The weights as the product with V takes them, and their part in the denominator.
    __device__ __forceinline__ void weigh(int mt, const float4_t (&t)[2], const float4_t (&inv)[2], float ref, mvec8_t &pf)
    {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float x = t[u >> 2][u & 3];
            const float w = __builtin_amdgcn_exp2f(FMT == k16 ? __builtin_fmaf(x, scale, -ref) : x - ref);
            l[mt] = FMT == k16 ? l[mt] + w : __builtin_fmaf(w, inv[u >> 2][u & 3], l[mt]);
            pf[u] = (typename Elem<MDT>::T)w;
        }
    }
    // The same for the scores (before the scale) of the 32 nodes from `first` on, of which the rows see some; t becomes the weights.
    __device__ __forceinline__ void weigh_nodes(float4_t (&t)[MT][2], int first, vec8_t (&pf)[MT])
    {
        float top[MT], ref[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            top[mt] = -INFINITY;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float x = t[mt][u >> 2][u & 3] * scale;
                t[mt][u >> 2][u & 3] = seen[mt] >> (first + 16 * (u >> 2) + 4 * g4 + (u & 3)) & 1 ? x : -INFINITY;
                top[mt] = fmaxf(top[mt], t[mt][u >> 2][u & 3]);
            }
        }
        follow(top, ref);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float d = t[mt][u >> 2][u & 3] - ref[mt];
                float w = __builtin_amdgcn_exp2f(d);
                if constexpr (FMT != k16) {
                    if (__builtin_expect(wide != 0, 0)) {  // the maximum may hold a scale of V up to 2^121
                        w = times_power(1.f, d);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                t[mt][u >> 2][u & 3] = w;
                l[mt] += w;
                pf[mt][u] = (elem_t)w;
            }
    }
    // The lane groups' parts of the denominators.
    __device__ __forceinline__ void sum_denominators()
    {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            l[mt] += __shfl_xor(l[mt], 16, 64);
            l[mt] += __shfl_xor(l[mt], 32, 64);
        }
    }
    // The rows' results: to the output (`whole`: all tokens of theirs), or as a part's, row i in slot slot0 + i.
    __device__ __forceinline__ void store(const Params &p, const Place &at, int first_row, bool whole, int64_t slot0) const
    {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int row = first_row + mt * 16 + r16;
            if (row >= at.nodes * p.g) continue;
            if (whole) {
                elem_t *dst = static_cast<elem_t *>(p.out) + (qrow[mt] - static_cast<const elem_t *>(p.q));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    typedef elem_t vec_t __attribute__((ext_vector_type(NI)));
                    vec_t v;
#pragma unroll
                    for (int i = 0; i < NI; ++i) v[i] = some >> mt & 1 ? (elem_t)(o[mt][i][e] / l[mt]) : (elem_t)0.f;
                    *reinterpret_cast<vec_t *>(dst + (4 * g4 + e) * NI) = v;
                }
            } else {
                const int64_t slot = slot0 + row;
                float *dst = p.partial + slot * DH;
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int i = 0; i < NI; i += 4)
                        *reinterpret_cast<float4_t *>(dst + (4 * g4 + e) * NI + i) =
                            float4_t{o[mt][i][e], o[mt][i + 1][e], o[mt][i + 2][e], o[mt][i + 3][e]};
                if (g4 == 0) *reinterpret_cast<float2 *>(p.partial + p.slots * DH + 2 * slot) = make_float2(m[mt], l[mt]);
            }
        }
    }

    // V^T of 32 tokens, of which this lane read raw[s] of token slot s: the operands of the elements in word w, two of 16 bits
    // (as they are) or four codes (as fp16).
    template <typename W>
    static __device__ __forceinline__ void turn16(const W (&raw)[8], int w, u32x4_t (&vt)[2])
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int s = 0; s < 4; ++s) vt[i][s] = __builtin_amdgcn_perm(word(raw[2 * s + 1], w), word(raw[2 * s], w), i ? 0x07060302u : 0x05040100u);
    }
    template <typename W>
    static __device__ __forceinline__ void turn8(const W (&raw)[8], int w, u32x4_t (&vt)[4])
    {
#pragma unroll
        for (int q = 0; q < 2; ++q) {                      // token slots 4 q .. 4 q + 3
            const uint32_t a = biased<FMT>(word(raw[4 * q], w)), b = biased<FMT>(word(raw[4 * q + 1], w));
            const uint32_t c = biased<FMT>(word(raw[4 * q + 2], w)), d = biased<FMT>(word(raw[4 * q + 3], w));
            const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
            const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
            const uint32_t e[4] = {__builtin_amdgcn_perm(cd0, ab0, 0x05040100u), __builtin_amdgcn_perm(cd0, ab0, 0x07060302u),
                                   __builtin_amdgcn_perm(cd1, ab1, 0x05040100u), __builtin_amdgcn_perm(cd1, ab1, 0x07060302u)};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                vt[j][2 * q] = __builtin_bit_cast(uint32_t, pair_f16<FMT, false>(e[j]));
                vt[j][2 * q + 1] = __builtin_bit_cast(uint32_t, pair_f16<FMT, true>(e[j]));
            }
        }
    }

    // ---- 32 cached tokens, two 16s of which n[j] exist: where they are (wavefront-uniform) and what is on its way of them.
    struct Tokens {
        const void *K[2], *V[2];
        const float *ks[2], *vs[2];
        int n[2];
    };
    Words<16> kraw[2][KR];
    Words<VB> vraw[8];
    float sc;                                              // a scale (8 bits), see put_scales
    float *scales;                                         // LDS of the wavefront

    __device__ __forceinline__ void ask_k(const Tokens &tk)
    {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const __amdgpu_buffer_rsrc_t rs = rows_at(tk.K[j], tk.n[j] * RB);
#pragma unroll
            for (int i = 0; i < KR; ++i) kraw[j][i] = fetch<16, kStreamed>(rs, r16 * RB + k_elem(FMT == k16 ? i : 2 * i) * EB);
        }
        if constexpr (FMT != k16) sc = *scale_at(tk.ks[0], tk.ks[1], tk.vs[0], tk.vs[1], 16 * g4 + r16);
    }
    __device__ __forceinline__ void ask_v(const Tokens &tk)
    {
        const __amdgpu_buffer_rsrc_t rs[2] = {rows_at(tk.V[0], tk.n[0] * RB), rows_at(tk.V[1], tk.n[1] * RB)};
#pragma unroll
        for (int s = 0; s < 8; ++s) vraw[s] = fetch<VB, kStreamed>(rs[s >> 2], (4 * g4 + (s & 3)) * RB + r16 * VB);
    }
    // Takes the tokens in; n as they were asked for.  `next` is asked for as registers fall free.
    __device__ __forceinline__ void take(const int (&n)[2], const Tokens &next)
    {
        float4_t t[MT][2], inv[2];
        if constexpr (FMT != k16) wide |= put_scales(scales, sc, n[0], n[1], 16 * g4 + r16, scale);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            mvec8_t kf[KK];
#pragma unroll
            for (int i = 0; i < KR; ++i) {
                if constexpr (FMT == k16) {
                    kf[i] = __builtin_bit_cast(mvec8_t, kraw[j][i]);
                } else {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t b = biased<FMT>(kraw[j][i][w]);
                        const half2_t lo = pair_f16<FMT, false>(b), hi = pair_f16<FMT, true>(b);
                        mvec8_t &f = kf[2 * i + (w >> 1)];
                        const int at = 4 * (w & 1);
                        f[at] = lo[0]; f[at + 1] = lo[1]; f[at + 2] = hi[0]; f[at + 3] = hi[1];
                    }
                }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                t[mt][j] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) t[mt][j] = Elem<MDT>::mfma_16x16x32(kf[kk], qf[mt][kk], t[mt][j]);
            }
        }
        if constexpr (FMT != k16) {                        // t = score * scale log2(e) + log2(vs), and the denominator's factor 1 / vs
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4_t kq = *reinterpret_cast<const float4_t *>(scales + 16 * j + 4 * g4);
                const float4_t lv = *reinterpret_cast<const float4_t *>(scales + 32 + 16 * j + 4 * g4);
                inv[j] = *reinterpret_cast<const float4_t *>(scales + 96 + 16 * j + 4 * g4);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) t[mt][j][i] = __builtin_fmaf(DT != MDT ? t[mt][j][i] * qfac[mt] : t[mt][j][i], kq[i], lv[i]);
            }
        } else if (n[0] + n[1] < kTileTokens) {            // tokens that do not exist
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) t[mt][j][i] = 4 * g4 + i < n[j] ? t[mt][j][i] : -INFINITY;
        }
        ask_k(next);
        __builtin_amdgcn_sched_barrier(0);
        mvec8_t pf[MT];
        float ref[MT];
        references(t, ref);
        if constexpr (FMT != k16) {
            if (__builtin_expect(wide != 0, 0)) count_far(t, inv, ref);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) weigh(mt, t[mt], inv, ref[mt], pf[mt]);
        constexpr int G = FMT == k16 ? 2 : 4;
#pragma unroll
        for (int w = 0; w < NI / G; ++w) {
            u32x4_t vt[G];
            if constexpr (FMT == k16) turn16(vraw, w, vt);
            else turn8(vraw, w, vt);
            if (w == NI / G - 1) {
                // vraw has been read before it is asked for again: else the compiler keeps both, and the loop copies, that is
                // waits for, what has just been asked for
#pragma unroll
                for (int i = 0; i < G; ++i) asm volatile("" : "+v"(vt[i])::"memory");
                ask_v(next);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < G; ++i)
                    o[mt][G * w + i] = Elem<MDT>::mfma_16x16x32(__builtin_bit_cast(mvec8_t, vt[i]), pf[mt], o[mt][G * w + i]);
        }
    }

    // ---- 32 nodes from node `first` on: K, V point at the first one's row, rows are `pitch` bytes apart, n of them exist.
    __device__ __forceinline__ void drafted(const elem_t *K, const elem_t *V, int pitch, int first, int n)
    {
        const uint32_t bytes = n > 0 ? (uint32_t)(n - 1) * pitch + DH * 2 : 0;
        const __amdgpu_buffer_rsrc_t krs = rows_at(K, bytes), vrs = rows_at(V, bytes);
        Words<16> kraw[2][KK];
        Words<NI * 2> raw[8];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) kraw[j][kk] = fetch<16>(krs, (16 * j + r16) * pitch + node_elem(kk) * 2);
#pragma unroll
        for (int s = 0; s < 8; ++s) raw[s] = fetch<NI * 2>(vrs, (16 * (s >> 2) + 4 * g4 + (s & 3)) * pitch + r16 * NI * 2);
        float4_t t[MT][2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                t[mt][j] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
                    t[mt][j] = Elem<DT>::mfma_16x16x32(__builtin_bit_cast(vec8_t, kraw[j][kk]), node_query(mt, kk), t[mt][j]);
            }
        // A weight of zero does not take an infinity or a NaN out of the product: such elements are zeros there and reach
        // the rows that see them on their own.
        constexpr uint32_t ex = DT == 1 ? 0x7f80u : 0x7c00u;
        uint32_t wild = 0;
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
            for (int w = 0; w < NI / 2; ++w) {
                const uint32_t x = word(raw[s], w);
                wild |= ((x & ex) + (ex & -ex) & 0x8000u) | ((x >> 16 & ex) + (ex & -ex) & 0x8000u);   // an exponent of ones carries
            }
        const bool any_wild = __ballot(wild != 0) != 0;
        if (any_wild) {
#pragma unroll
            for (int s = 0; s < 8; ++s)
#pragma unroll
                for (int w = 0; w < NI / 2; ++w) {
                    const uint32_t x = word(raw[s], w);
                    raw[s][w] = ((x & ex) == ex ? 0u : x & 0xffffu) | ((x >> 16 & ex) == ex ? 0u : x & 0xffff0000u);
                    __builtin_amdgcn_sched_barrier(0);
                }
        }
        vec8_t pf[MT];
        weigh_nodes(t, first, pf);
#pragma unroll
        for (int w = 0; w < NI / 2; ++w) {
            u32x4_t vt[2];
            turn16(raw, w, vt);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    o[mt][2 * w + i] = Elem<DT>::mfma_16x16x32(__builtin_bit_cast(vec8_t, vt[i]), pf[mt], o[mt][2 * w + i]);
        }
        if constexpr (FMT != k16) lift();
        if (any_wild) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) add_wild(V, pitch, first, n, mt, t[mt]);
        }
    }
    // The nodes came first, and the rows of the cache, whose scores hold log2 of their scales of V, may all lie far below the
    // nodes' maximum where V is small: their weights would be below fp16's numbers.  So the maximum goes down as far as the sums
    // have room for; rows of the cache that still lie below it are less than 2^-90 of the sums.
    __device__ __forceinline__ void lift()
    {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float top = l[mt];
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, __builtin_fabsf(o[mt][i][e]));
            top = max_over_groups(top);
            const int ex = top > 0.f ? __builtin_amdgcn_frexp_expf(top) : 100, up = ex < 100 ? 100 - ex : 0;
            m[mt] -= (float)up;
            l[mt] = __builtin_amdgcn_ldexpf(l[mt], up);
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[mt][i][e] = __builtin_amdgcn_ldexpf(o[mt][i][e], up);
        }
    }
    // The infinities and NaN of V, node by node; t: the weights of this lane's row and tokens.
    __device__ __forceinline__ void add_wild(const elem_t *V, int pitch, int first, int n, int mt, const float4_t (&t)[2])
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
                    __builtin_amdgcn_sched_barrier(0);     // one by one: this path is for its results, not for its speed
                }
        }
    }
};

// Table entries of the two 16s of the tile at token t; 16s that do not exist: the last one's that does (t_end > 0).
__device__ __forceinline__ void entries_of(const int32_t *__restrict__ tab, int t, int t_end, int blk_log2, int (&e)[2])
{
    const int last = t_end - 1;
    e[0] = scalar_at(tab, (t < last ? t : last) >> blk_log2);
    e[1] = scalar_at(tab, (t + 16 < last ? t + 16 : last) >> blk_log2);
}

// Where the tile's rows are.  Also for a tile behind the last: it has no rows, and a load of it reads nothing (the scales: those
// of a block that exists).  Loops ask for it like for any other; a branch around the loads would have every pass copy, and so
// wait for, what is on its way.
template <typename wave_t, int FMT>
__device__ __forceinline__ void tokens_at(const Params &p, int h, int t0, int t_end, const int (&ent)[2], typename wave_t::Tokens &tk)
{
    const int blk = 1 << p.c.blk_log2;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int t = t0 + 16 * j, here = t_end - t;
        tk.n[j] = here < 0 ? 0 : here < 16 ? here : 16;
        const int e = uniform(ent[j]);
        bool act = FMT == k16 && e < 0;
        int pb = e < 0 ? ~e : e;
        if constexpr (FMT == k16) {
            if ((act ? p.c.P_act : p.c.P_kv) <= 0) { act = !act; pb = 0; }       // a corrupt table cannot leave
        }
        const int P = act ? p.c.P_act : p.c.P_kv;                                // the pools
        pb = pb < P ? pb : P - 1;
        const int64_t row = (((int64_t)pb * p.c.Hkv + h) << p.c.blk_log2) + (t & (blk - 1));
        tk.K[j] = static_cast<const char *>(act ? p.K_regen : p.c.K_pool) + row * wave_t::RB;
        tk.V[j] = static_cast<const char *>(act ? p.V_regen : p.c.V_pool) + row * wave_t::RB;
        if constexpr (FMT != k16) {
            tk.ks[j] = p.c.K_scale + row;
            tk.vs[j] = p.c.V_scale + row;
        }
    }
}

// Workgroups a compute unit that the registers are held to: resident_pieces(), or the third one that fp16 rows leave room for at
// dh = 64 and two tiles (167 registers; the compiler's own choice is 177, which ends at two).
constexpr int held_to(int DH, int DT, bool codes, int MT, bool tree) { return DH == 64 && MT == 2 && DT == 0 ? 3 : resident_pieces(DH, MT, codes, tree); }

template <int DH, int DT, int FMT, int MT, bool TREE>
__global__ __launch_bounds__(kThreads, held_to(DH, DT, FMT != k16, MT, TREE)) void kv_attn_kernel(Params p)
{
    typedef Wave<DH, DT, FMT, MT> wave_t;
    typedef typename wave_t::elem_t elem_t;
    constexpr int NI = wave_t::NI;
    __shared__ float join_ml[kWaves][MT * 16][2];
    __shared__ float4_t join_o[kWaves][MT * NI * 64];
    __shared__ __align__(16) float scales[FMT == k16 ? 1 : kWaves][FMT == k16 ? 4 : kScales];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    Place at;
    int ent[2] = {0, 0};
    if (p.extra <= 0 && p.c.max_blocks > 0) {
        // The first tile's table entries, asked for together with the length that says whether they count.
        const int32_t *tab = p.c.block_table + (int64_t)(blockIdx.x / p.c.Hkv) * p.c.max_blocks;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int b = (wave * kTileTokens + 16 * j) >> p.c.blk_log2;
            ent[j] = scalar_at(tab, b < p.c.max_blocks ? b : p.c.max_blocks - 1);
        }
    }
    if (!place(p, lane, at)) return;
    if (p.slots > 0 && at.piece == 0 && at.h == 0 && threadIdx.x == 0) piece_notes(p, DH)[at.r] = make_int2(at.x, at.pieces);
    if (at.nodes <= 0) return;                             // no rows
    wave_t w;
    w.rows(p, at, 0, lane, TREE);
    w.scales = scales[FMT == k16 ? 0 : wave];
    w.clear();
    w.ask_q();
    if (TREE && p.k && at.last) {                          // the nodes, by the wavefronts that have the fewest tiles
        const int pitch = p.c.Hkv * DH * 2;
        for (int d = 0; d * kTileTokens < at.nodes; ++d) {
            if (kWaves - 1 - d != wave) continue;
            const int64_t from = (((int64_t)at.r * p.T + d * kTileTokens) * p.c.Hkv + at.h) * DH;
            const int n = at.nodes - d * kTileTokens;
            w.drafted(static_cast<const elem_t *>(p.k) + from, static_cast<const elem_t *>(p.v) + from, pitch, d * kTileTokens,
                      n < kTileTokens ? n : kTileTokens);
        }
    }
    const int32_t *tab = p.c.block_table + (int64_t)at.r * p.c.max_blocks;
    const int t_end = at.t_end;
    int tb = at.t_begin + wave * kTileTokens;              // pieces begin at whole rounds: wavefront 0 takes the first tile
    if (tb < t_end) {
        typename wave_t::Tokens tk;
        if (p.extra > 0) entries_of(tab, tb, t_end, p.c.blk_log2, ent);
        tokens_at<wave_t, FMT>(p, at.h, tb, t_end, ent, tk);
        w.ask_k(tk);
        w.ask_v(tk);
        entries_of(tab, tb + kStep, t_end, p.c.blk_log2, ent);
        w.start();
        // Said once, in front of the loop: the queries are there.  Else every pass would wait for all that is on its way.
        wait_loads<wave_t::kTileLoads>();
        do {
            const int n[2] = {tk.n[0], tk.n[1]};
            tokens_at<wave_t, FMT>(p, at.h, tb + kStep, t_end, ent, tk);
            entries_of(tab, tb + 2 * kStep, t_end, p.c.blk_log2, ent);
            w.take(n, tk);
            tb += kStep;
        } while (tb < t_end);
    }

    // The wavefronts' results about their common maximum, added in the order of the wavefronts; each stores a part of the row.
    w.sum_denominators();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        if (w.g4 == 0) {
            join_ml[wave][mt * 16 + w.r16][0] = w.m[mt];
            join_ml[wave][mt * 16 + w.r16][1] = w.l[mt];
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) join_o[wave][(mt * NI + i) * 64 + lane] = w.o[mt][i];
    }
    __syncthreads();
    constexpr int NQ = NI / kWaves;                        // products whose results this wavefront joins
    const int64_t slot0 = ((int64_t)at.x * p.c.Hkv + at.h) * ((int64_t)p.T * p.g);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int row = mt * 16 + w.r16;
        if (row >= at.nodes * p.g) continue;
        float top = -INFINITY, l = 0.f, f[kWaves];
#pragma unroll
        for (int q = 0; q < kWaves; ++q) top = fmaxf(top, join_ml[q][row][0]);
        const float ref = top == -INFINITY ? 0.f : top;
        bool far = false;
#pragma unroll
        for (int q = 0; q < kWaves; ++q) {
            const float d = join_ml[q][row][0] - ref;
            f[q] = __builtin_amdgcn_exp2f(d);
            l = __builtin_fmaf(join_ml[q][row][1], f[q], l);
            far = far || is_far(d);
        }
        if constexpr (FMT != k16) {
            if (__builtin_expect(__ballot(far) != 0, 0)) { // as in follow()
                l = 0.f;
#pragma unroll
                for (int q = 0; q < kWaves; ++q) l += times_power(join_ml[q][row][1], join_ml[q][row][0] - ref);
            }
        }
        float4_t sum[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            sum[i] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < kWaves; ++q) sum[i] += join_o[q][(mt * NI + wave * NQ + i) * 64 + lane] * f[q];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int elem = (4 * w.g4 + e) * NI + wave * NQ;
            if (at.pieces == 1) {
                elem_t *dst = static_cast<elem_t *>(p.out) + (w.qrow[mt] - static_cast<const elem_t *>(p.q)) + elem;
                typedef elem_t vec_t __attribute__((ext_vector_type(NQ)));
                vec_t v;
#pragma unroll
                for (int i = 0; i < NQ; ++i) v[i] = w.some >> mt & 1 ? (elem_t)(sum[i][e] / l) : (elem_t)0.f;
                *reinterpret_cast<vec_t *>(dst) = v;
            } else {
                typedef float fvec_t __attribute__((ext_vector_type(NQ)));
                fvec_t v;
#pragma unroll
                for (int i = 0; i < NQ; ++i) v[i] = sum[i][e];
                *reinterpret_cast<fvec_t *>(p.partial + (slot0 + row) * DH + elem) = v;
            }
        }
        if (at.pieces > 1 && wave == 0 && w.g4 == 0)
            *reinterpret_cast<float2 *>(p.partial + p.slots * DH + 2 * (slot0 + row)) = make_float2(top, l);
    }
}

}  // namespace kvattn
}  // namespace hk
