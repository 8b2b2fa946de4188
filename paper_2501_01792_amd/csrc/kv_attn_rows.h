// The form of kv_attn_kernel.h for many query rows (trees, shared K/V heads): the 4 wavefronts of a workgroup take 16 MT rows
// each and share every tile of 32 tokens through LDS.
//
// There the vector ALU is the bound: a weight costs some ten instructions and an exponential, and making operands of the
// rows of K and V (widening codes, turning V) costs as much as 16 to 32 query rows do.  So a wavefront makes a quarter of a
// tile's operands and stores them in LDS in the order in which the matrix instructions read them, a lane's 16 bytes beside
// its neighbour's; every wavefront reads them all.  Two buffers and one barrier a tile: while a tile is taken in, the next one's
// operands are stored, and its successor's rows are on their way from memory.
// The wavefronts never join: each has all tokens of its rows.
#pragma once
#include "kv_attn_kernel.h"

namespace hk {
namespace kvattn {

// A tile's rows, two 16s of which n[j] exist: where they are (wavefront-uniform), `pitch` bytes apart.
struct Rows {
    const void *K[2], *V[2];
    const float *ks[2], *vs[2];
    int n[2], pitch;
};

template <int DH>
struct Operands {
    u32x4_t k[2 * (DH / 32)][64];                          // [16s of tokens x products][lane]
    u32x4_t v[DH / 16][64];
    float kq[kTileTokens], lv[kTileTokens], inv[kTileTokens];
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
    Words<16> kraw[NK];
    uint32_t vraw[NV];
    float sc;

    // K: pieces of 16s j; V: word `word` of a lane's elements, token slots from 4 q on.
    static __device__ __forceinline__ int k_sixteen(int wave) { return kSplit ? wave & 1 : wave >> 1; }
    static __device__ __forceinline__ int k_piece(int wave, int i) { return kSplit ? 0 : NK * (wave & 1) + i; }
    static __device__ __forceinline__ int v_word(int wave) { return kSplit ? 0 : NV == 8 ? wave : wave & 1; }
    static __device__ __forceinline__ int v_quad(int wave) { return kSplit ? wave & 1 : NV == 8 ? 0 : wave >> 1; }

    __device__ __forceinline__ void ask(const Rows &r, int wave, int lane)
    {
        const int g4 = lane >> 4, r16 = lane & 15;
        if (!kSplit || wave < 2) {
            const int j = k_sixteen(wave);
            const __amdgpu_buffer_rsrc_t rs = rows_at(j ? r.K[1] : r.K[0], bytes(r, j));
#pragma unroll
            for (int i = 0; i < NK; ++i) kraw[i] = fetch<16>(rs, r16 * r.pitch + k_piece(wave, i) * 64 + g4 * 16);
        }
        if (!kSplit || wave >= 2) {
#pragma unroll
            for (int half = 0; half < NV / 4; ++half) {
                const int q = NV == 8 ? half : v_quad(wave);
                const __amdgpu_buffer_rsrc_t rs = rows_at(q ? r.V[1] : r.V[0], bytes(r, q));
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    vraw[4 * half + s] = fetch<4>(rs, (4 * g4 + s) * r.pitch + r16 * VB + v_word(wave) * 4).w[0];
            }
        }
        if constexpr (kCodes) {
            if (wave == 3) {                               // a scale a lane: those of K in lanes 0 .. 31, of V in the others
                const uintptr_t k0 = reinterpret_cast<uintptr_t>(r.ks[0]), k1 = reinterpret_cast<uintptr_t>(r.ks[1]);
                const uintptr_t v0 = reinterpret_cast<uintptr_t>(r.vs[0]), v1 = reinterpret_cast<uintptr_t>(r.vs[1]);
                const uintptr_t a = lane & 16 ? k1 : k0, b = lane & 16 ? v1 : v0;
                sc = reinterpret_cast<const float *>(lane < 32 ? a : b)[r16];
            }
        }
    }
    static __device__ __forceinline__ uint32_t bytes(const Rows &r, int j)
    {
        const int n = j ? r.n[1] : r.n[0];
        return n > 0 ? (uint32_t)(n - 1) * r.pitch + RB : 0;
    }

    // n: as the rows were asked for.
    __device__ __forceinline__ void put(Operands<DH> &to, const int (&n)[2], int wave, int lane, float scale) const
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
                            const uint32_t b = biased<F>(kraw[i].w[2 * half + w]);
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
            if (wave == 3) {                               // a token that does not exist: 0 s - inf, and no part of the denominator
                const int tok = lane & 31;
                const bool in = (tok & 15) < (tok < 16 ? n[0] : n[1]);
                const float v = sc < kLeastScale ? kLeastScale : sc;
                if (lane < 32) {
                    to.kq[tok] = in ? sc * scale : 0.f;
                } else {
                    to.lv[tok] = in ? __builtin_amdgcn_logf(v) : -INFINITY;
                    to.inv[tok] = in ? __builtin_amdgcn_rcpf(v) : 0.f;
                }
            }
        }
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

template <int DH, int DT, int FMT, int MT>
__global__ __launch_bounds__(kThreads, 2) void kv_rows_kernel(Params p)
{
    typedef Wave<DH, DT, FMT, MT> wave_t;
    typedef typename wave_t::elem_t elem_t;
    typedef typename wave_t::vec8_t vec8_t;
    typedef typename wave_t::mvec8_t mvec8_t;
    constexpr int NI = wave_t::NI, KK = wave_t::KK, MDT = wave_t::MDT;
    __shared__ Operands<DH> ops[2];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    Place at;
    if (!place(p, lane, at)) return;
    const int group_rows = kWaves * MT * 16, group_first = at.rg * group_rows;
    if (group_first >= at.nodes * p.g) return;             // rows of nodes that there are not
    const int first_row = group_first + wave * MT * 16;
    wave_t w;
    w.rows(p, at, first_row, lane, true);
    w.start();

    const int32_t *tab = p.c.block_table + (int64_t)at.r * p.c.max_blocks;
    auto rows_of = [&](int t0, Rows &r) {
        int ent[2];
        entries_of(tab, t0, at.t_end, p.c.blk_log2, ent);
        typename wave_t::Tokens tk;
        tokens_at<wave_t, FMT>(p, at.h, t0, at.t_end, ent, tk);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            r.K[j] = tk.K[j]; r.V[j] = tk.V[j]; r.n[j] = tk.n[j];
            if constexpr (FMT != k16) { r.ks[j] = tk.ks[j]; r.vs[j] = tk.vs[j]; }
        }
        r.pitch = wave_t::RB;
    };

    Part<DH, FMT> part;
    Rows ahead;                                            // of the tile whose rows are on their way
    int tb = at.t_begin, cur = 0;
    int n_cur[2] = {0, 0};
    if (tb < at.t_end) {
        rows_of(tb, ahead);
        part.ask(ahead, wave, lane);
        n_cur[0] = ahead.n[0];
        n_cur[1] = ahead.n[1];
        part.put(ops[0], ahead.n, wave, lane, w.scale);
        if (tb + kTileTokens < at.t_end) {
            rows_of(tb + kTileTokens, ahead);
            part.ask(ahead, wave, lane);
        }
        meet();
    }
    for (; tb < at.t_end; tb += kTileTokens) {
        const bool more = tb + kTileTokens < at.t_end;
        int n_next[2] = {0, 0};
        if (more) {
            n_next[0] = ahead.n[0];
            n_next[1] = ahead.n[1];
            part.put(ops[cur ^ 1], ahead.n, wave, lane, w.scale);
            if (tb + 2 * kTileTokens < at.t_end) {
                rows_of(tb + 2 * kTileTokens, ahead);
                part.ask(ahead, wave, lane);
            }
        }
        const Operands<DH> &op = ops[cur];
        float4_t t[MT][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) t[mt][j] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const mvec8_t kf = __builtin_bit_cast(mvec8_t, op.k[j * KK + kk][lane]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) t[mt][j] = Elem<MDT>::mfma_16x16x32(kf, w.qf[mt][kk], t[mt][j]);
            }
        }
        float4_t inv[2];
        if constexpr (FMT != k16) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4_t kq = *reinterpret_cast<const float4_t *>(op.kq + 16 * j + 4 * w.g4);
                const float4_t lv = *reinterpret_cast<const float4_t *>(op.lv + 16 * j + 4 * w.g4);
                inv[j] = *reinterpret_cast<const float4_t *>(op.inv + 16 * j + 4 * w.g4);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) t[mt][j][i] = __builtin_fmaf(DT != MDT ? t[mt][j][i] * w.qfac[mt] : t[mt][j][i], kq[i], lv[i]);
            }
        } else if (n_cur[0] + n_cur[1] < kTileTokens) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) t[mt][j][i] = 4 * w.g4 + i < n_cur[j] ? t[mt][j][i] : -INFINITY;
        }
        mvec8_t pf[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) w.weigh(mt, t[mt], inv, pf[mt]);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const mvec8_t vf = __builtin_bit_cast(mvec8_t, op.v[i][lane]);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) w.o[mt][i] = Elem<MDT>::mfma_16x16x32(vf, pf[mt], w.o[mt][i]);
        }
        n_cur[0] = n_next[0];
        n_cur[1] = n_next[1];
        cur ^= 1;
        meet();                                            // the next tile is there, and this one's buffer is free
    }

    if (p.k && at.last) {
        const int pitch = p.c.Hkv * DH * 2;
        for (int first = 0; first < at.nodes; first += kTileTokens) {
            const int64_t from = (((int64_t)at.r * p.T + first) * p.c.Hkv + at.h) * DH;
            const elem_t *K = static_cast<const elem_t *>(p.k) + from, *V = static_cast<const elem_t *>(p.v) + from;
            const int n = at.nodes - first < kTileTokens ? at.nodes - first : kTileTokens;
            Rows r;
            r.K[0] = K; r.V[0] = V;
            r.K[1] = reinterpret_cast<const char *>(K) + 16 * pitch;
            r.V[1] = reinterpret_cast<const char *>(V) + 16 * pitch;
            r.n[0] = n < 16 ? n : 16;
            r.n[1] = n < 16 ? 0 : n - 16;
            r.pitch = pitch;
            Part<DH, k16> nodes;
            nodes.ask(r, wave, lane);
            if (threadIdx.x == 0) ops[cur].wild = 0;
            meet();
            if (nodes.template tame<DT>() && lane == 0) ops[cur].wild = 1;
            nodes.put(ops[cur], r.n, wave, lane, 0.f);
            meet();
            const Operands<DH> &op = ops[cur];
            float4_t t[MT][2];
            vec8_t pf[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    t[mt][j] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk)
                        t[mt][j] = Elem<DT>::mfma_16x16x32(__builtin_bit_cast(vec8_t, op.k[j * KK + kk][lane]),
                                                           *reinterpret_cast<const vec8_t *>(w.qrow[mt] + kk * 32 + w.g4 * 8), t[mt][j]);
                }
                w.weigh_nodes(mt, t[mt], first, pf[mt]);
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const vec8_t vf = __builtin_bit_cast(vec8_t, op.v[i][lane]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) w.o[mt][i] = Elem<DT>::mfma_16x16x32(vf, pf[mt], w.o[mt][i]);
            }
            if (uniform(op.wild)) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) w.add_wild(V, pitch, first, n, mt, t[mt]);
            }
            meet();
        }
    }
    w.sum_denominators();
    w.store(p, at, first_row);
}

}  // namespace kvattn
}  // namespace hk
