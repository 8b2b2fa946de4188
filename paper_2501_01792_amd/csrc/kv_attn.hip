// Attention over the paged K/V cache: the launch of its kernels (kv_attn_kernel.h, kv_attn_rows.h) in the cache's format, and
// the merges of what they leave of requests whose tokens were cut.
#include "kv_attn_kernel.h"
#include "kv_attn_rows.h"

namespace hk {
namespace kvattn {
namespace {

constexpr int kMergeBatch = 8;

// Joins the pieces of a row: one wavefront each, DH / 64 elements a lane.  A few KB a row, bound by one way to memory: the
// loads of kMergeBatch pieces are on their way together (one request of 2000 tokens, 32 rows of 16 pieces: 4 us, which is what a launch and two ways to memory take).
template <int DH, int DT>
__global__ __launch_bounds__(256) void kv_merge_kernel(Params p)
{
    typedef typename Elem<DT>::T elem_t;
    constexpr int E = DH / 64;
    const int lane = threadIdx.x & 63;
    const int R = p.T * p.g;
    const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (id >= (int64_t)p.B * p.c.Hkv * R) return;
    const int row = uniform((int)(id % R)), h = uniform((int)(id / R % p.c.Hkv)), r = uniform((int)(id / R / p.c.Hkv));
    const int2 note = piece_notes(p, DH)[r];
    const int nodes = nodes_of(p, r), x0 = uniform(note.x), n = uniform(note.y);
    if (n == 1 || row >= nodes * p.g) return;              // its only piece has written it, or there is none
    const int64_t slot0 = ((int64_t)x0 * p.c.Hkv + h) * R + row, step = (int64_t)p.c.Hkv * R;
    const float *ml = p.partial + p.slots * DH;
    float top = -INFINITY;
    for (int i = lane; i < n; i += 64) top = fmaxf(top, ml[2 * (slot0 + i * step)]);
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    const float ref = top == -INFINITY ? 0.f : top;
    float l = 0.f, o[E] = {};
    for (int i0 = 0; i0 < n; i0 += 64) {
        float w = 0.f, lw = 0.f;
        if (i0 + lane < n) {
            const float2 v = *reinterpret_cast<const float2 *>(ml + 2 * (slot0 + (i0 + lane) * step));
            w = __builtin_amdgcn_exp2f(v.x - ref);
            lw = w * v.y;
            // over 8 bits the maxima hold scales of V, the denominators do not
            if (__builtin_expect(is_far(v.x - ref), 0)) lw = times_power(v.y, v.x - ref);
        }
        for (int off = 32; off > 0; off >>= 1) lw += __shfl_xor(lw, off, 64);
        l += lw;
        const int upto = n - i0 < 64 ? n - i0 : 64;
        for (int i = 0; i < upto; i += kMergeBatch) {      // every load of a batch on its way before the first use
            float v[kMergeBatch][E], wi[kMergeBatch];
#pragma unroll
            for (int b = 0; b < kMergeBatch; ++b) {
                const int at = i + b < upto ? i + b : i;   // a piece that fills the batch: read, not used
                wi[b] = __shfl(w, i + b, 64);
                const float *src = p.partial + (slot0 + (i0 + at) * step) * DH + lane * E;
#pragma unroll
                for (int e = 0; e < E; ++e) v[b][e] = src[e];
            }
#pragma unroll
            for (int b = 0; b < kMergeBatch; ++b)
                if (i + b < upto) {
#pragma unroll
                    for (int e = 0; e < E; ++e) o[e] = __builtin_fmaf(wi[b], v[b][e], o[e]);
                }
        }
    }
    // n > 1: the request has tokens, so every row of it sees some
    elem_t *dst = static_cast<elem_t *>(p.out) + (((int64_t)r * p.T + row / p.g) * p.H + h * p.g + row % p.g) * DH + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) dst[e] = (elem_t)(o[e] / l);
}

// Joins the parts of a unit that more than one range of kv_attn_rows.h holds: kMergeRows rows of the unit whose second part
// lies in range w.  A row is DH / 4 lanes, four elements each.  It is bound by the way to memory: the parts come two and then four
// at a time, and 16 rows a workgroup spread a unit of many parts (a long request) over more of them.  The whole call, int8, 8 K/V
// heads: one request of 4000 tokens and 256 rows a head 48 us (32 rows a workgroup, one part at a time: 52), 64 rows over 1000
// tokens 21.8 (24.3).  Eight at a time cost occupancy where units have few parts: 16 requests of 2000 tokens 79 for 75.
constexpr int kMergeRows = 16, kMergeThreads = 256;

template <int DH, int DT>
__global__ __launch_bounds__(kMergeThreads) void kv_rows_merge_kernel(Params p, int held)
{
    typedef typename Elem<DT>::T elem_t;
    typedef elem_t vec4_t __attribute__((ext_vector_type(4)));
    constexpr int LPR = DH / 4, RPB = kMergeThreads / LPR, kDeep = kMergeRows / RPB;
    const int blocks = held / kMergeRows, wg = blockIdx.x / blocks + 1, block = blockIdx.x % blocks;
    const int4 note = reinterpret_cast<const int4 *>(p.partial + p.slots * (DH + 2))[wg];
    const int r = uniform(note.x), h = uniform(note.y), row0 = uniform(note.z) + block * kMergeRows, n_parts = uniform(note.w);
    if (n_parts == 0) return;                              // no unit whose second part begins this range
    const int len = length_of(p.c, r), nodes = nodes_of(p, r), rows = nodes * p.g;
    if (row0 >= rows) return;
    const float *ml = p.partial + p.slots * DH;
    const int c = threadIdx.x % LPR, mine = threadIdx.x / LPR;
    float m[kDeep], l[kDeep];
    float4_t o[kDeep];
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
        m[u] = -INFINITY;
        l[u] = 0.f;
        o[u] = float4_t{0.f, 0.f, 0.f, 0.f};
    }
    const int last = wg + n_parts - 2;                     // the range of the last part
    auto join = [&](auto count, int x0) {                  // parts of ranges x0 .. x0 + count - 1, all on their way at once
        constexpr int N = decltype(count)::value;
        float2 v[N][kDeep];
        float4_t s[N][kDeep];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            // the first part is that of range wg - 1, which begins the unit; the others do not
            const int x = x0 + i;
            const int64_t slot = (int64_t)(2 * x + (x == wg - 1)) * held + block * kMergeRows + mine;
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {              // also rows that there are not: what their slots hold is not used
                v[i][u] = *reinterpret_cast<const float2 *>(ml + 2 * (slot + u * RPB));
                s[i][u] = *reinterpret_cast<const float4_t *>(p.partial + (slot + u * RPB) * DH + 4 * c);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                const float top = fmaxf(m[u], v[i][u].x), ref = top == -INFINITY ? 0.f : top;
                const float f = __builtin_amdgcn_exp2f(m[u] - ref), g = __builtin_amdgcn_exp2f(v[i][u].x - ref);
                // over 8 bits the maxima hold scales of V, the denominators do not
                const float d = fminf(m[u] - ref, v[i][u].x - ref), before = l[u];
                l[u] = l[u] * f + v[i][u].y * g;
                if (__builtin_expect(is_far(d), 0)) l[u] = m[u] < top ? v[i][u].y + times_power(before, d) : before + times_power(v[i][u].y, d);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[u][e] = o[u][e] * f + s[i][u][e] * g;
                m[u] = top;
            }
    };
    join(std::integral_constant<int, 2>(), wg - 1);        // two parts at least
    int x = wg + 1;
    for (; x + 3 <= last; x += 4) join(std::integral_constant<int, 4>(), x);
    for (; x <= last; ++x) join(std::integral_constant<int, 1>(), x);
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
        const int row = row0 + mine + u * RPB, node = row / p.g;
        if (row >= rows) continue;
        const bool some = len > 0 || seen_by(p, r, node, nodes) != 0;
        vec4_t out;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = some ? (elem_t)(o[u][e] / l[u]) : (elem_t)0.f;
        elem_t *dst = static_cast<elem_t *>(p.out) + (((int64_t)r * p.T + node) * p.H + h * p.g + row % p.g) * DH + 4 * c;
        *reinterpret_cast<vec4_t *>(dst) = out;
    }
}

template <int DH, int DT>
hipError_t launch_merge(const Params &p, const Plan &pl, hipStream_t s)
{
    if (pl.shared) {
        const int held = 16 * kWaves * pl.tiles;
        hipLaunchKernelGGL((kv_rows_merge_kernel<DH, DT>), dim3((unsigned)((pl.groups - 1) * (held / kMergeRows))), dim3(kMergeThreads), 0, s, p, held);
    } else {
        const int64_t rows = (int64_t)p.B * p.c.Hkv * pl.rows;
        hipLaunchKernelGGL((kv_merge_kernel<DH, DT>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace
}  // namespace kvattn

size_t kv_attn_partial_floats(int64_t B, int T, int H, int Hkv, int head_dim, bool codes, int64_t total_tokens, int64_t room, int splits)
{
    return (size_t)kvattn::plan(B, T, H, Hkv, head_dim, codes, total_tokens, room, splits).partial_floats;
}
bool kv_attn_launchable(int64_t B, int T, int H, int Hkv, int head_dim, bool codes, int64_t total_tokens, int64_t room, int splits)
{
    const kvattn::Plan pl = kvattn::plan(B, T, H, Hkv, head_dim, codes, total_tokens, room, splits);
    // the launches of both forms and of their merges
    if (pl.shared) return pl.groups * (16 * kvattn::kWaves * pl.tiles / kvattn::kMergeRows) <= kvattn::kMostGroups;
    return pl.groups <= kvattn::kMostGroups && B * Hkv * pl.rows <= 4 * kvattn::kMostGroups;
}

hipError_t launch_kv_attn(const KvAttnArgs &a, hipStream_t s)
{
    using namespace kvattn;
    if (a.B <= 0) return hipSuccess;
    const Plan pl = plan(a.B, a.T, a.H, a.c.Hkv, a.head_dim, a.format != kvfmt::k16, a.total_tokens, (int64_t)a.c.max_blocks << a.c.blk_log2, a.splits);
    Params p;
    p.c = a.c;
    p.K_regen = a.K_regen; p.V_regen = a.V_regen; p.q = a.q; p.k = a.k; p.v = a.v;
    p.mask = a.mask; p.n_nodes = a.n_nodes; p.out = a.out; p.partial = a.partial;
    p.slots = pl.slots;
    p.B = a.B; p.T = a.T; p.H = a.H; p.mask_stride = a.mask_stride; p.g = a.H / a.c.Hkv;
    p.extra = (int)pl.extra; p.groups = (int)pl.groups;
    p.scale_log2e = a.scale * kLog2e;
    const hipError_t e = a.format == kvfmt::k16     ? launch_16(p, pl, a.head_dim, a.dtype, s)
                         : a.format == kvfmt::kInt8 ? launch_int8(p, pl, a.head_dim, a.dtype, s)
                                                    : launch_e4m3(p, pl, a.head_dim, a.dtype, s);
    if (e != hipSuccess || pl.slots <= 0) return e;
    if (a.head_dim == 128) return a.dtype == 1 ? launch_merge<128, 1>(p, pl, s) : launch_merge<128, 0>(p, pl, s);
    return a.dtype == 1 ? launch_merge<64, 1>(p, pl, s) : launch_merge<64, 0>(p, pl, s);
}

}  // namespace hk
