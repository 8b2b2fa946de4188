// The form of kv_attn_kernel.h for many query rows (trees, shared K/V heads): the 4 wavefronts of a workgroup take 16 MT rows
// each and share every tile of 32 tokens through LDS.
//
// There the products are no longer what costs: a weight takes some ten vector instructions and an exponential, and making operands
// of the rows of K and V (widening codes, turning V) as many as 16 to 32 query rows do.  So a wavefront makes a quarter of a
// tile's operands and stores them in LDS in the order in which the matrix instructions read them, a lane's 16 bytes beside
// its neighbour's; every wavefront reads them all.  Two buffers and one barrier a tile: while a tile is taken in, the next one's
// operands are stored, and the rows of the two behind that are on their way from memory.
// The wavefronts never join: each has all tokens of its rows.  How the work is cut into ranges is in kv_split.h.
//
// 16 requests of 4096 to 8192 tokens, 64 nodes, 8 query heads on each of 8 K/V heads of 128, int8, bf16: 1.6e11 products and sums
// in 314 us, 0.51 PFLOP/s (481 us with workgroups of equal requests instead of ranges, 850 with every wavefront making its own
// operands).  No unit is full (counters, of the time that the wavefronts are there, two a SIMD, which is all that the registers, o
// alone 64, leave room for): a SIMD's vector ALU works 62 %, its matrix core 28 %, and of a wavefront's time 46 % issues
// an instruction, 29 % has one ready that waits for its turn, 24 % waits for a barrier, LDS or memory.
// 33 nodes of 40 heads, e4m3, 7 requests of 383 to 1148 tokens: 36 us, some 14 tiles a workgroup; wavefronts wait 47 % of their
// time, at the beginning (lengths, table, queries, first rows: four ways to memory) above all, and the merge takes 7.  Where a
// request has few of the T nodes, wavefronts whose rows do not exist only make operands.
#pragma once
#include "kv_attn_kernel.h"

#include <type_traits>

namespace hk {
namespace kvattn {

// A tile's rows, two 16s of which n0 and n1 exist: where they are (wavefront-uniform), `pitch` bytes apart.
struct Rows {
    const void *K0, *K1, *V0, *V1;
    const float *ks0, *ks1, *vs0, *vs1;
    int n0, n1, pitch;
};

template <int DH>
struct Operands {
    u32x4_t k[2 * (DH / 32)][64];                          // [16s of tokens x products][lane]
    u32x4_t v[DH / 16][64];
    float scales[kScales];                                 // see put_scales
    int wild;                                              // V of a tile of nodes holds infinities or NaN
};

// A wavefront's part of a tile, from memory to LDS; F: the format of the rows.
template <int DH, int F>
struct Part {
    static constexpr bool kCodes = F != k16;
    static constexpr int EB = kCodes ? 1 : 2, RB = DH * EB, KK = DH / 32, NI = DH / 16, VB = NI * EB;
    static constexpr int KP = kCodes ? 2 : 1;              // products that a 16-byte piece of K feeds
    static constexpr int NK = kCodes || DH == 64 ? 1 : 2;  // pieces of K, token slots of V (of the 8 a lane has) of a wavefront
    static constexpr int NV = !kCodes && DH == 128 ? 8 : 4;
    static constexpr bool kSplit = kCodes && DH == 64;     // two wavefronts take K, the others V
    static constexpr int kLoads = (kSplit ? NK : NK + NV) + (kCodes ? 1 : 0);     // at least so many loads of a wavefront
    Words<16> kraw[NK];
    uint32_t vraw[NV];
    float sc;

    // K: pieces of 16s j; V: word `word` of a lane's elements, token slots from 4 q on.
    static __device__ __forceinline__ int k_sixteen(int wave) { return kSplit ? wave & 1 : wave >> 1; }
    static __device__ __forceinline__ int k_piece(int wave, int i) { return kSplit ? 0 : NK * (wave & 1) + i; }
    static __device__ __forceinline__ int v_word(int wave) { return kSplit ? 0 : NV == 8 ? wave : wave & 1; }
    static __device__ __forceinline__ int v_quad(int wave) { return kSplit ? wave & 1 : NV == 8 ? 0 : wave >> 1; }

    // codes_order: 16-bit rows whose products take queries that are laid out for codes.
    template <bool codes_order = kCodes>
    __device__ __forceinline__ void ask(const Rows &r, int wave, int lane)
    {
        const int g4 = lane >> 4, r16 = lane & 15;
        if (!kSplit || wave < 2) {
            const int j = k_sixteen(wave);
            const __amdgpu_buffer_rsrc_t rs = rows_at(j ? r.K1 : r.K0, bytes(r, j));
#pragma unroll
            for (int i = 0; i < NK; ++i) {
                const int kk = k_piece(wave, i);
                kraw[i] = fetch<16>(rs, r16 * r.pitch + (codes_order && !kCodes ? (kk >> 1) * 128 + g4 * 32 + (kk & 1) * 16 : kk * 64 + g4 * 16));
            }
        }
        if (!kSplit || wave >= 2) {
#pragma unroll
            for (int half = 0; half < NV / 4; ++half) {
                const int q = NV == 8 ? half : v_quad(wave);
                const __amdgpu_buffer_rsrc_t rs = rows_at(q ? r.V1 : r.V0, bytes(r, q));
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    vraw[4 * half + s] = fetch<4>(rs, (4 * g4 + s) * r.pitch + r16 * VB + v_word(wave) * 4);
            }
        }
        if constexpr (kCodes) {                            // a scale a lane: those of K in lanes 0 .. 31, of V in the others
            sc = *scale_at(r.ks0, r.ks1, r.vs0, r.vs1, lane);
        }
    }
    static __device__ __forceinline__ uint32_t bytes(const Rows &r, int j)
    {
        const int n = j ? r.n1 : r.n0;
        return n > 0 ? (uint32_t)(n - 1) * r.pitch + RB : 0;
    }

    // n0, n1: as the rows were asked for.  Returns what put_scales does.
    __device__ __forceinline__ uint32_t put(Operands<DH> &to, int n0, int n1, int wave, int lane, float scale) const
    {
        if (!kSplit || wave < 2) {
            const int j = k_sixteen(wave);
#pragma unroll
            for (int i = 0; i < NK; ++i) {
                const int at = j * KK + KP * k_piece(wave, i);
                if constexpr (kCodes) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        u32x4_t f;
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            const uint32_t b = biased<F>(kraw[i][2 * half + w]);
                            f[2 * w] = __builtin_bit_cast(uint32_t, pair_f16<F, false>(b));
                            f[2 * w + 1] = __builtin_bit_cast(uint32_t, pair_f16<F, true>(b));
                        }
                        to.k[at + half][lane] = f;
                    }
                } else {
                    to.k[at][lane] = __builtin_bit_cast(u32x4_t, kraw[i]);
                }
            }
        }
        if (!kSplit || wave >= 2) {
            const int word = v_word(wave);
            if constexpr (kCodes) {
                const uint32_t a = biased<F>(vraw[0]), b = biased<F>(vraw[1]), c = biased<F>(vraw[2]), d = biased<F>(vraw[3]);
                const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
                const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
                const uint32_t e[4] = {__builtin_amdgcn_perm(cd0, ab0, 0x05040100u), __builtin_amdgcn_perm(cd0, ab0, 0x07060302u),
                                       __builtin_amdgcn_perm(cd1, ab1, 0x05040100u), __builtin_amdgcn_perm(cd1, ab1, 0x07060302u)};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    reinterpret_cast<u32x2_t *>(&to.v[4 * word + i][lane])[v_quad(wave)] =
                        u32x2_t{__builtin_bit_cast(uint32_t, pair_f16<F, false>(e[i])), __builtin_bit_cast(uint32_t, pair_f16<F, true>(e[i]))};
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t f[NV / 2];
#pragma unroll
                    for (int s = 0; s < NV / 2; ++s) f[s] = __builtin_amdgcn_perm(vraw[2 * s + 1], vraw[2 * s], i ? 0x07060302u : 0x05040100u);
                    if constexpr (NV == 8) to.v[2 * word + i][lane] = u32x4_t{f[0], f[1], f[2], f[3]};
                    else reinterpret_cast<u32x2_t *>(&to.v[2 * word + i][lane])[v_quad(wave)] = u32x2_t{f[0], f[1]};
                }
            }
        }
        if constexpr (kCodes) {
            // every wavefront stores the same: a branch would part the products from what runs under them
            return put_scales(to.scales, sc, n0, n1, lane, scale);
        }
        return 0;
    }
    // Infinities and NaN of V become zeros (16-bit rows); whether there were any.
    template <int DT>
    __device__ __forceinline__ bool tame()
    {
        constexpr uint32_t ex = DT == 1 ? 0x7f80u : 0x7c00u;
        bool wild = false;
#pragma unroll
        for (int s = 0; s < NV; ++s) {
            const uint32_t x = vraw[s];
            const bool lo = (x & ex) == ex, hi = (x >> 16 & ex) == ex;
            wild = wild || lo || hi;
            vraw[s] = (lo ? 0u : x & 0xffffu) | (hi ? 0u : x & 0xffff0000u);
        }
        return __ballot(wild) != 0;
    }
};

// Every wavefront's stores to LDS are there, and its reads have come back; loads from memory stay on their way.
__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The tiles of a request's units on the line, and what the units are.
struct Request {
    int len, nodes, tiles, groups;
    int64_t line;
};
__device__ __forceinline__ Request request(const Params &p, int r, int held)
{
    Request q;
    q.len = length_of(p.c, r);
    q.nodes = nodes_of(p, r);
    q.tiles = unit_tiles(q.len, q.nodes, p.k != nullptr);
    q.groups = unit_groups(q.nodes, p.g, held);
    q.line = (int64_t)q.tiles * q.groups * p.c.Hkv;
    return q;
}
__device__ __forceinline__ int64_t line_total(const Params &p, int lane, int held)
{
    int64_t sum = 0;
    for (int r = lane; r < p.B; r += 64) sum += request(p, r, held).line;
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    return (int64_t)(uint32_t)uniform((int)(uint32_t)sum) | (int64_t)uniform((int)(sum >> 32)) << 32;
}
// The request that holds position x of the line (x < total), and where its tiles begin.
__device__ __forceinline__ int request_at(const Params &p, int64_t x, int lane, int held, int64_t &begin)
{
    int64_t before = 0;
    for (int r0 = 0; r0 < p.B; r0 += 64) {
        const int64_t own = r0 + lane < p.B ? request(p, r0 + lane, held).line : 0;
        int64_t upto = own;
        for (int off = 1; off < 64; off <<= 1) {
            const int64_t o = __shfl_up(upto, off, 64);
            if (lane >= off) upto += o;
        }
        const uint64_t in = __ballot(before + upto > x);
        if (in) {
            const int at = uniform(__builtin_ctzll(in));
            begin = before + __shfl(upto - own, at, 64);
            begin = (int64_t)(uint32_t)uniform((int)(uint32_t)begin) | (int64_t)uniform((int)(begin >> 32)) << 32;
            return r0 + at;
        }
        before += __shfl(upto, 63, 64);
    }
    begin = 0;
    return 0;
}

template <int DH, int DT, int FMT, int MT>
__global__ __launch_bounds__(kThreads, resident(DH, MT)) void kv_rows_kernel(Params p)
{
    typedef Wave<DH, DT, FMT, MT> wave_t;
    typedef typename wave_t::elem_t elem_t;
    typedef typename wave_t::vec8_t vec8_t;
    typedef typename wave_t::mvec8_t mvec8_t;
    constexpr int NI = wave_t::NI, KK = wave_t::KK, MDT = wave_t::MDT, kHeld = kWaves * MT * 16;
    __shared__ Operands<DH> ops[2];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int64_t total = line_total(p, lane, kHeld);
    const int used = ranges_used(total, p.groups);
    // Workgroups go to the 8 XCDs in turn: neighbours on the line, which read the same rows, on one of them.
    const int b = blockIdx.x, wg = p.groups % 8 == 0 ? (b & 7) * (p.groups / 8) + (b >> 3) : b;
    if (p.slots > 0 && threadIdx.x == 0) reinterpret_cast<int4 *>(p.partial + p.slots * (DH + 2))[wg] = int4{0, 0, 0, 0};
    if (wg >= used || total <= 0) return;
    int64_t pos = ranges::range_begin(wg, total, used);
    const int64_t end = ranges::range_begin(wg + 1, total, used);
    int64_t begin;
    Place at;
    at.r = request_at(p, pos, lane, kHeld, begin);
    while (pos < end) {
        const Request rq = request(p, at.r, kHeld);
        if (pos >= begin + rq.line) {
            begin += rq.line;
            ++at.r;
            continue;
        }
        // the part of a unit that this is: tiles [first, first + n) of rq.tiles
        const int unit = (int)ranges::quot(pos - begin, rq.tiles);
        const int first = (int)(pos - begin - (int64_t)unit * rq.tiles);
        const int n = rq.tiles - first < end - pos ? rq.tiles - first : (int)(end - pos);
        at.h = unit / rq.groups;
        at.nodes = rq.nodes;
        at.len = rq.len;
        const int of_tokens = (rq.len + kTileTokens - 1) / kTileTokens;
        at.t_begin = first < of_tokens ? first * kTileTokens : rq.len;
        at.t_end = first + n < of_tokens ? (first + n) * kTileTokens : rq.len;
        const int node_begin = (first > of_tokens ? first - of_tokens : 0) * kTileTokens;
        const int node_end = p.k && first + n > of_tokens ? (first + n - of_tokens) * kTileTokens : 0;
        const int group_first = unit % rq.groups * kHeld, first_row = group_first + wave * MT * 16;
        if (first > 0 && threadIdx.x == 0 && pos - first >= ranges::range_begin(wg - 1, total, used))
            // for the merge, at the unit's second part: request, head, first row, number of parts
            reinterpret_cast<int4 *>(p.partial + p.slots * (DH + 2))[wg] =
                int4{at.r, at.h, group_first, ranges::owner(pos - first + rq.tiles - 1, total, used) - wg + 2};
        pos += n;

        wave_t w;
        w.rows(p, at, first_row, lane, true);
        w.clear();
        w.ask_q();
        const int32_t *tab = p.c.block_table + (int64_t)at.r * p.c.max_blocks;
        // Rows are asked for three tiles ahead (two wait in registers, in turn), their table entries four.
        Part<DH, FMT> part[2];
        int ent[2], t_ask = at.t_begin;
        auto ask = [&](Part<DH, FMT> &to, const int (&e)[2]) {
            typename wave_t::Tokens tk;
            tokens_at<wave_t, FMT>(p, at.h, t_ask, at.t_end, e, tk);
            t_ask += kTileTokens;
            Rows r = {tk.K[0], tk.K[1], tk.V[0], tk.V[1], nullptr, nullptr, nullptr, nullptr, tk.n[0], tk.n[1], wave_t::RB};
            if constexpr (FMT != k16) { r.ks0 = tk.ks[0]; r.ks1 = tk.ks[1]; r.vs0 = tk.vs[0]; r.vs1 = tk.vs[1]; }
            to.ask(r, wave, lane);
        };
        auto put = [&](const Part<DH, FMT> &from, int t, Operands<DH> &to) {
            const int here = at.t_end - t;
            const uint32_t far = from.put(to, here < 16 ? here : 16, here < 16 ? 0 : here < 32 ? here - 16 : 16, wave, lane, w.scale);
            if constexpr (FMT != k16) w.wide |= far;
        };
        // One tile: its successor's operands are made from `next`, which then waits for the tile two behind that.  A wavefront
        // whose rows do not exist only makes operands.
        const bool mine = first_row < at.nodes * p.g;
        auto tile = [&](auto has_rows, int tb, const Operands<DH> &op, Operands<DH> &op_next, Part<DH, FMT> &next) __attribute__((always_inline)) {
            if constexpr (!decltype(has_rows)::value) {
                put(next, tb + kTileTokens, op_next);
            } else {
                // Operands are asked of LDS well ahead: K's before the next tile's are made, V's before the weights.
                mvec8_t kf[2 * KK], vf[NI];
                float4_t kq[2], lv[2], inv[2];
#pragma unroll
                for (int i = 0; i < 2 * KK; ++i) kf[i] = __builtin_bit_cast(mvec8_t, op.k[i][lane]);
                if constexpr (FMT != k16) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        kq[j] = *reinterpret_cast<const float4_t *>(op.scales + 16 * j + 4 * w.g4);
                        lv[j] = *reinterpret_cast<const float4_t *>(op.scales + 32 + 16 * j + 4 * w.g4);
                        inv[j] = *reinterpret_cast<const float4_t *>(op.scales + 96 + 16 * j + 4 * w.g4);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                put(next, tb + kTileTokens, op_next);              // behind the last tile: what nobody reads
                float4_t t[MT][2];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) t[mt][j] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) t[mt][j] = Elem<MDT>::mfma_16x16x32(kf[j * KK + kk], w.qf[mt][kk], t[mt][j]);
#pragma unroll
                for (int i = 0; i < NI; ++i) vf[i] = __builtin_bit_cast(mvec8_t, op.v[i][lane]);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (FMT != k16) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                t[mt][j][i] = __builtin_fmaf(DT != MDT ? t[mt][j][i] * w.qfac[mt] : t[mt][j][i], kq[j][i], lv[j][i]);
                } else if (at.t_end - tb < kTileTokens) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) t[mt][j][i] = tb + 16 * j + 4 * w.g4 + i < at.t_end ? t[mt][j][i] : -INFINITY;
                }
                mvec8_t pf[MT];
                float ref[MT];
                w.references(t, ref);
                if constexpr (FMT != k16) {
                    if (__builtin_expect(w.wide != 0, 0)) w.count_far(t, inv, ref);
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {                  // one tile's products run under the next one's weights
                    w.weigh(mt, t[mt], inv, ref[mt], pf[mt]);
#pragma unroll
                    for (int i = 0; i < NI; ++i) w.o[mt][i] = Elem<MDT>::mfma_16x16x32(vf[i], pf[mt], w.o[mt][i]);
                }
            }
            ask(next, ent);
            entries_of(tab, t_ask, at.t_end, p.c.blk_log2, ent);
            meet();                                            // the next tile is there, and this one's buffer is free
        };
        if (at.t_begin < at.t_end) {
            int ent0[2], ent1[2];
            entries_of(tab, t_ask, at.t_end, p.c.blk_log2, ent0);
            entries_of(tab, t_ask + kTileTokens, at.t_end, p.c.blk_log2, ent1);
            entries_of(tab, t_ask + 2 * kTileTokens, at.t_end, p.c.blk_log2, ent);
            ask(part[0], ent0);
            ask(part[1], ent1);
            w.start();
            put(part[0], at.t_begin, ops[0]);
            // Said once, in front of the loop: the queries are there.  Else every tile would wait for all that is on its way.
            wait_loads<Part<DH, FMT>::kLoads>();
            ask(part[0], ent);
            entries_of(tab, t_ask, at.t_end, p.c.blk_log2, ent);
            meet();
            auto tiles = [&](auto has_rows) __attribute__((always_inline)) {
                int tb = at.t_begin;
                do {
                    tile(has_rows, tb, ops[0], ops[1], part[1]);
                    if (tb + kTileTokens < at.t_end) tile(has_rows, tb + kTileTokens, ops[1], ops[0], part[0]);
                    tb += 2 * kTileTokens;
                } while (tb < at.t_end);
            };
            if (mine) tiles(std::true_type());
            else tiles(std::false_type());
        } else {
            w.start();
        }

        if (node_begin < node_end && node_begin < at.nodes) {
            // the nodes' tiles, two at most, both asked for at once
            const int pitch = p.c.Hkv * DH * 2;
            Part<DH, k16> nodes[2];
            Rows r[2];
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const int node = node_begin + d * kTileTokens, upto = at.nodes < node_end ? at.nodes : node_end;
                const int64_t from = (((int64_t)at.r * p.T + node) * p.c.Hkv + at.h) * DH;
                const elem_t *K = static_cast<const elem_t *>(p.k) + from, *V = static_cast<const elem_t *>(p.v) + from;
                const int here = upto - node;
                r[d] = {K, reinterpret_cast<const char *>(K) + 16 * pitch, V, reinterpret_cast<const char *>(V) + 16 * pitch,
                        nullptr, nullptr, nullptr, nullptr, here < 0 ? 0 : here < 16 ? here : 16,
                        here < 16 ? 0 : here < 32 ? here - 16 : 16, pitch};
                nodes[d].template ask<FMT != k16 && wave_t::kOwnQ>(r[d], wave, lane);
            }
            if (threadIdx.x < 2) ops[threadIdx.x].wild = 0;
            meet();
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                if (r[d].n0 <= 0) break;
                if (nodes[d].template tame<DT>() && lane == 0) ops[d].wild = 1;
                nodes[d].put(ops[d], r[d].n0, r[d].n1, wave, lane, 0.f);
                meet();
                const Operands<DH> &op = ops[d];
                float4_t t[MT][2];
                vec8_t pf[MT];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        t[mt][j] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int kk = 0; kk < KK; ++kk)
                            t[mt][j] = Elem<DT>::mfma_16x16x32(__builtin_bit_cast(vec8_t, op.k[j * KK + kk][lane]), w.node_query(mt, kk), t[mt][j]);
                    }
                const int node = node_begin + d * kTileTokens;
                w.weigh_nodes(t, node, pf);
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const vec8_t vf = __builtin_bit_cast(vec8_t, op.v[i][lane]);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) w.o[mt][i] = Elem<DT>::mfma_16x16x32(vf, pf[mt], w.o[mt][i]);
                }
                if (uniform(op.wild)) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                        w.add_wild(static_cast<const elem_t *>(r[d].V0), pitch, node, r[d].n0 + r[d].n1, mt, t[mt]);
                }
            }
            meet();                                        // the operands have been read: the range's next unit may store its own
        }
        w.sum_denominators();
        // a range has one part that does not begin its unit at most, and one that begins a unit and does not end it
        w.store(p, at, first_row, n == rq.tiles, (int64_t)(2 * wg + (first == 0)) * kHeld - group_first);
    }
}

}  // namespace kvattn
}  // namespace hk
