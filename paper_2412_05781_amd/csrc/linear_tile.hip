// The matrix kernel of the transformer-block operators for operands that can be fetched 16 bytes at a time: global -> LDS transfers without a
// detour through registers, a ring of stages of 128 bytes of reduction elements (64, fp32: 32), four to eight waves that own 32x32 MFMA tiles.
//
// A stage of an operand that runs along the reduction is BI rows of 128 bytes, of one across it 64 (fp32: 32) rows of BI elements; both are filled by transfers of
// 1 KB whose lanes fetch from swizzled places, so that the fragment reads (ds_read_b128, or the transposing ds_read_b64_tr_b16) find every bank
// once.  Rows behind the edge are fetched from the last row inside (their sums are not stored), reduction elements behind the end from 16 zero bytes.
#include "linear_tile.h"

namespace wino {

namespace {

__device__ __attribute__((aligned(16))) const unsigned char zero16[16] = {};

// lanes 32-63 of a against lanes 0-31 of b
__device__ __forceinline__ void swap_halves(float& a, float& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}
// sum over the sixteen lanes of a row, in all of them
__device__ __forceinline__ float sum_over_16(float v) {
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x128, 0xf, 0xf, false));    // row_ror:8
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x124, 0xf, 0xf, false));
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x122, 0xf, 0xf, false));
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x121, 0xf, 0xf, false));
    return v;
}

// eight neighbouring elements of a row
template <typename E> struct Eight { uint4 w[sizeof(E) / 2]; };
template <typename E> __device__ __forceinline__ Eight<E> load8(const E* p) {
    Eight<E> f;
#pragma unroll
    for (int i = 0; i < (int)sizeof(E) / 2; ++i) f.w[i] = reinterpret_cast<const uint4*>(p)[i];
    return f;
}
template <typename E> __device__ __forceinline__ void unpack8(const Eight<E>& e, float* v) {
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) { v[4 * i] = __uint_as_float(e.w[i].x); v[4 * i + 1] = __uint_as_float(e.w[i].y); v[4 * i + 2] = __uint_as_float(e.w[i].z); v[4 * i + 3] = __uint_as_float(e.w[i].w); }
    } else {
        const uint4& f = e.w[0];
        v[0] = lo16<E>(f.x); v[1] = hi16<E>(f.x); v[2] = lo16<E>(f.y); v[3] = hi16<E>(f.y);
        v[4] = lo16<E>(f.z); v[5] = hi16<E>(f.z); v[6] = lo16<E>(f.w); v[7] = hi16<E>(f.w);
    }
}
template <typename E> __device__ __forceinline__ void store8(E* p, const float* v) {
    if constexpr (sizeof(E) == 4) {
        reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_pair<E>(v[0], v[1]), pack_pair<E>(v[2], v[3]), pack_pair<E>(v[4], v[5]), pack_pair<E>(v[6], v[7]));
    }
}

// Epilogue of one wave's tile.  acc[i][j]: rows n of 32-row block i (GLU: block i of the up rows, FP / 2 + i of the gate rows), columns m of block j.
// What a block reads besides its sums is requested for all of its columns before the first is used, from clamped places; only stores are guarded.
template <typename E, int EP, int ACT, int FP, int FQ, int WP, int WQ>
__device__ __forceinline__ void finish_tile(const GemmShape& g, const Epilogue& e, float16_t (&acc)[FP][FQ], int n0, long long m0, int wp, int wq, long long sum_row, long long top_at, int lane, int split) {
    constexpr bool GLU = EP == EP_GLU || EP == EP_DGLU, SUMS = EP == EP_DLINEAR || EP == EP_DGLU;
    constexpr int NI = GLU ? FP / 2 : FP;
    const int half = lane >> 5;
    E* out = static_cast<E*>(e.out);
    const E* extra = static_cast<const E*>(e.extra);
    const bool has_bias = EP != EP_STORE && e.bias, has_extra = SUMS || (EP == EP_LINEAR && extra);
    constexpr bool F16 = std::is_same_v<E, __half>;
    const float factor = store_factor<E, SUMS>(e);
    float top = 0.f;
    long long mrow[FQ];
    bool m_on[FQ];
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
        const long long m = m0 + (j * WQ + wq) * 32 + (lane & 31);
        m_on[j] = m < g.M;
        mrow[j] = m_on[j] ? m : g.M - 1;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        int n[2];
        bool n_on[2];
        float bias[2][8] = {}, bias2[2][8] = {};
        Eight<E> ex[2][FQ] = {};
#pragma unroll
        for (int qp = 0; qp < 2; ++qp) {
            // after the exchange of halves a lane holds n .. n + 7 of its row; N is a multiple of 8 here
            const int c = n0 + (i * WP + wp) * 32 + 16 * qp + 8 * half;
            n_on[qp] = c < g.N;
            n[qp] = n_on[qp] ? c : g.N - 8;
            if (has_bias) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    bias[qp][k] = e.bias[n[qp] + k];
                    if constexpr (GLU) bias2[qp][k] = e.bias[g.N + n[qp] + k];
                }
            }
            if (has_extra) {
#pragma unroll
                for (int j = 0; j < FQ; ++j) ex[qp][j] = load8<E>(extra + mrow[j] * e.ld_extra + n[qp]);
            }
        }
#pragma unroll
        for (int qp = 0; qp < 2; ++qp) {
            float sum[8] = {}, sum2[8] = {};
#pragma unroll
            for (int j = 0; j < FQ; ++j) {
                float s[8], s2[8], a[8], b[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    s[k] = acc[i][j][8 * qp + k];
                    s[k + 4] = acc[i][j][8 * qp + 4 + k];
                    swap_halves(s[k], s[k + 4]);
                    if constexpr (GLU) {
                        s2[k] = acc[NI + i][j][8 * qp + k];
                        s2[k + 4] = acc[NI + i][j][8 * qp + 4 + k];
                        swap_halves(s2[k], s2[k + 4]);
                    }
                }
                const bool on = n_on[qp] && m_on[j];
                if (EP == EP_STORE && e.part) {            // uniform: one of several ranges
                    float* p = e.part + ((long long)split * g.M + mrow[j]) * g.N + n[qp];
                    if (on) {
                        *reinterpret_cast<float4*>(p) = make_float4(s[0], s[1], s[2], s[3]);
                        *reinterpret_cast<float4*>(p + 4) = make_float4(s[4], s[5], s[6], s[7]);
                    }
                    continue;
                }
                float r[8];
                unpack8<E>(ex[qp][j], r);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if constexpr (EP == EP_STORE) a[k] = F16 ? s[k] * factor : s[k];
                    else if constexpr (EP == EP_LINEAR) a[k] = act_only<E, ACT>(s[k] + bias[qp][k]) + r[k];
                    else if constexpr (EP == EP_GLU) a[k] = (s[k] + bias[qp][k]) * act_only<E, ACT>(s2[k] + bias2[qp][k]);
                    else {
                        float v, d;
                        if constexpr (EP == EP_DLINEAR) {
                            act_both<E, ACT>(s[k] + bias[qp][k], v, d);
                            a[k] = r[k] * d;
                        } else {
                            act_both<E, ACT>(s2[k] + bias2[qp][k], v, d);
                            a[k] = r[k] * v;
                            b[k] = r[k] * (s[k] + bias[qp][k]) * d;
                            sum2[k] += on ? b[k] : 0.f;
                            if constexpr (F16) {
                                top = larger_finite(top, on ? b[k] : 0.f);
                                b[k] *= factor;
                            }
                        }
                        sum[k] += on ? a[k] : 0.f;
                        if constexpr (F16) {
                            top = larger_finite(top, on ? a[k] : 0.f);
                            a[k] *= factor;
                        }
                    }
                }
                if (on) {
                    E* at = out + mrow[j] * e.ld_out + n[qp];
                    store8<E>(at, a);
                    if constexpr (EP == EP_DGLU) store8<E>(at + g.N, b);
                }
            }
            if constexpr (SUMS) {
                const int width = EP == EP_DGLU ? 2 * g.N : g.N;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    sum[k] = sum_over_16(sum[k]);
                    sum[k] += __shfl_xor(sum[k], 16);
                    if constexpr (EP == EP_DGLU) {
                        sum2[k] = sum_over_16(sum2[k]);
                        sum2[k] += __shfl_xor(sum2[k], 16);
                    }
                }
                if ((lane & 31) == 0 && n_on[qp]) {
                    float* to = e.sums + sum_row * width + n[qp];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        to[k] = sum[k];
                        if constexpr (EP == EP_DGLU) to[g.N + k] = sum2[k];
                    }
                }
            }
        }
    }
    if constexpr (SUMS && F16) store_top(e, top_at, top, lane);
}

// ---- fragments under explicit control: the reads are issued from inline assembly, waited for by count, and tied to the wait by pin ----------------
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
template <int OFF> __device__ __forceinline__ void lds_read_across_async(u32x2_t& dst, uint32_t addr) {
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(OFF));
}
__device__ __forceinline__ void pin2(u32x2_t& v) { asm volatile("" : "+v"(v)); }

// The fragments of F blocks of 32 rows (block i at tile row (i * W + w) * 32) for one MFMA step, and the addresses they are read from.
template <typename E, bool ACROSS, int BI, int F, int W> struct Fragments;
template <typename E, int BI, int F, int W> struct Fragments<E, false, BI, F, W> {
    static constexpr int READS = F;
    struct Place { uint32_t base; };
    u32x4_t f[F];
    static __device__ __forceinline__ Place place(uint32_t tile, int w, int lane) {
        const int row = w * 32 + (lane & 31);
        return Place{tile + (uint32_t)row * 128u + (uint32_t)(((lane >> 5) ^ ((row >> 1) & 7)) << 4)};       // 32 W rows further: the same swizzle
    }
    template <int KS> __device__ __forceinline__ void read(const Place& p, uint32_t slot) {
        const uint32_t at = (p.base ^ (uint32_t)(KS << 5)) + slot;
        static_for<F>([&](auto ic) { constexpr int i = decltype(ic)::value; lds_read16_async<i * W * 32 * 128>(f[i], at); });
    }
    __device__ __forceinline__ void pin_all() {
#pragma unroll
        for (int i = 0; i < F; ++i) pin(f[i]);
    }
    __device__ __forceinline__ u32x4_t get(int i) const { return f[i]; }
};
template <int OFF> __device__ __forceinline__ void lds_read4_async(uint32_t& dst, uint32_t addr) {
    asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(OFF));
}
template <int BI, int F, int W> struct Fragments<float, true, BI, F, W> {
    static constexpr int READS = 4 * F;
    struct Place { uint32_t base[F]; };
    uint32_t f[F][4];
    static __device__ __forceinline__ Place place(uint32_t tile, int w, int lane) {
        Place p;
        const int row = 4 * (lane >> 5);                                                         // three rows further, or eight: the same swizzle
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const int col = (i * W + w) * 32 + (lane & 31);
            p.base[i] = tile + (uint32_t)(row * (BI * 4) + (((col >> 2) ^ swz_across<float, BI>(row)) << 4) + ((col & 3) << 2));
        }
        return p;
    }
    template <int KS> __device__ __forceinline__ void read(const Place& p, uint32_t slot) {
        static_for<F>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            const uint32_t at = p.base[i] + slot;
            static_for<4>([&](auto jc) { constexpr int j = decltype(jc)::value; lds_read4_async<(KS * 8 + j) * BI * 4>(f[i][j], at); });
        });
    }
    __device__ __forceinline__ void pin_all() {
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(f[i][j]));
    }
    __device__ __forceinline__ u32x4_t get(int i) const { return u32x4_t{f[i][0], f[i][1], f[i][2], f[i][3]}; }
};
template <typename E, int BI, int F, int W> struct Fragments<E, true, BI, F, W> {
    static constexpr int READS = 2 * F;
    struct Place { uint32_t base[F]; };
    u32x2_t f[F][2];
    static __device__ __forceinline__ Place place(uint32_t tile, int w, int lane) {
        Place p;
        const int row = 8 * (lane >> 5) + ((lane & 15) >> 2);                                              // rows 4 and 16 further: the same swizzle
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const int col = (i * W + w) * 32 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
            p.base[i] = tile + (uint32_t)(row * (BI * 2) + (((col >> 3) ^ swz_across<E, BI>(row)) << 4) + ((col & 4) << 1));
        }
        return p;
    }
    template <int KS> __device__ __forceinline__ void read(const Place& p, uint32_t slot) {
        static_for<F>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            const uint32_t at = p.base[i] + slot;
            lds_read_across_async<KS * 16 * BI * 2>(f[i][0], at);
            lds_read_across_async<KS * 16 * BI * 2 + 4 * BI * 2>(f[i][1], at);
        });
    }
    __device__ __forceinline__ void pin_all() {
#pragma unroll
        for (int i = 0; i < F; ++i) { pin2(f[i][0]); pin2(f[i][1]); }
    }
    __device__ __forceinline__ u32x4_t get(int i) const { return __builtin_shufflevector(f[i][0], f[i][1], 0, 1, 2, 3); }
};

// BP rows of P x BQ rows of Q per workgroup of WP x WQ waves, ring of NST stages.
template <typename E, int EP, bool PA, bool QA, int BP, int BQ, int WP, int WQ, int NST>
__device__ __forceinline__ void gemm_tile(const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int tiles_p, int tiles_q, int nsplit, int logical, unsigned char* lds) {
    constexpr bool GLU = EP == EP_GLU || EP == EP_DGLU;
    constexpr int ES = (int)sizeof(E), V = 16 / ES, KEL = 128 / ES;              // elements per chunk, reduction elements per stage
    constexpr int NW = WP * WQ, FP = BP / (32 * WP), FQ = BQ / (32 * WQ);
    constexpr int P_BYTES = BP * 128, STAGE = (BP + BQ) * 128;
    constexpr int LP = BP / 8 / NW, LQ = BQ / 8 / NW;      // 1 KB transfers per wave and stage
    constexpr int BN = GLU ? BP / 2 : BP;
    // MFMA steps whose fragments are requested together: a group's MFMAs have to last as long as the next group's reads
    constexpr int KH = FP * FQ >= 8 ? 1 : 2, NG = 4 / KH;
    static_assert(BP % (8 * NW) == 0 && BQ % (8 * NW) == 0, "whole transfers");
    const int split = logical / (tiles_p * tiles_q), in = logical - split * (tiles_p * tiles_q);
    // Eight tiles of Q against each tile of P in turn: the 32 to 64 workgroups that an XCD runs at a time then share tiles of both operands in its L2.
    constexpr int GROUP = 8;
    const int group = in / (GROUP * tiles_p), left_q = tiles_q - group * GROUP, gq = left_q < GROUP ? left_q : GROUP, rest = in - group * (GROUP * tiles_p);
    const int bp = rest / gq, bq = group * GROUP + rest - bp * gq;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wq = wave / WP;
    const int n0 = bp * BN;
    const long long m0 = (long long)bq * BQ;
    const int nk = (g.K + KEL - 1) / KEL;
    const int kt0 = (int)((long long)split * nk / nsplit), kt1 = (int)((long long)(split + 1) * nk / nsplit), stages = kt1 - kt0;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte_t*)lds;

    // Where transfer i of this wave fetches: a wave-uniform base that moves with the stage and a byte offset per lane.
    const unsigned char* sp = static_cast<const unsigned char*>(P.p) + (PA ? (long long)kt0 * KEL * P.ld + n0 : (long long)n0 * P.ld + (long long)kt0 * KEL) * ES;
    const unsigned char* sq = static_cast<const unsigned char*>(Q.p) + (QA ? (long long)kt0 * KEL * Q.ld + m0 : m0 * Q.ld + (long long)kt0 * KEL) * ES;
    uint32_t op[LP], oq[LQ];
    int kp[LP], kq[LQ];                                    // first reduction element of the lane's chunk within a stage
#pragma unroll
    for (int i = 0; i < LP; ++i) {
        const int t = wave + NW * i;
        if constexpr (!PA) {
            const int row = t * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
            int r = row;                                   // row of P, relative to n0
            if (GLU && row >= BP / 2) { r = row - BP / 2; r = (n0 + r < g.N ? r : g.N - 1 - n0) + g.N; }
            else r = n0 + r < g.N ? r : g.N - 1 - n0;
            op[i] = (uint32_t)r * (uint32_t)(P.ld * ES) + (uint32_t)chunk * 16u;
            kp[i] = chunk * V;
        } else {
            constexpr int CPR = BP / V, RPT = 64 / CPR;
            const int row = t * RPT + lane / CPR, chunk = (lane % CPR) ^ swz_across<E, BP>(row);
            const int c = n0 + chunk * V < g.N ? chunk * V : g.N - V - n0;
            op[i] = (uint32_t)row * (uint32_t)(P.ld * ES) + (uint32_t)(c * ES);
            kp[i] = row;
        }
    }
#pragma unroll
    for (int i = 0; i < LQ; ++i) {
        const int t = wave + NW * i;
        if constexpr (!QA) {
            const int row = t * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
            const int r = m0 + row < g.M ? row : (int)(g.M - 1 - m0);
            oq[i] = (uint32_t)r * (uint32_t)(Q.ld * ES) + (uint32_t)chunk * 16u;
            kq[i] = chunk * V;
        } else {
            constexpr int CPR = BQ / V, RPT = 64 / CPR;
            const int row = t * RPT + lane / CPR, chunk = (lane % CPR) ^ swz_across<E, BQ>(row);
            const int c = m0 + chunk * V < g.M ? chunk * V : (int)(g.M - V - m0);
            oq[i] = (uint32_t)row * (uint32_t)(Q.ld * ES) + (uint32_t)(c * ES);
            kq[i] = row;
        }
    }
    const long long step_p = PA ? KEL * P.ld * ES : 128, step_q = QA ? KEL * Q.ld * ES : 128;
    int next = kt0;                                        // next stage to fetch
    auto issue = [&](int slot) {
        const uint32_t dst = lds0 + (uint32_t)slot * STAGE + (uint32_t)wave * 1024u;
        const int left = g.K - next * KEL;                  // reduction elements from this stage on
        if (left >= KEL) {
#pragma unroll
            for (int i = 0; i < LP; ++i) dma_load_1k_s(sp, op[i], dst + (uint32_t)(NW * i) * 1024u);
#pragma unroll
            for (int i = 0; i < LQ; ++i) dma_load_1k_s(sq, oq[i], dst + P_BYTES + (uint32_t)(NW * i) * 1024u);
        } else {                                           // K is a multiple of a chunk where one runs along it
#pragma unroll
            for (int i = 0; i < LP; ++i) dma_load_1k_v(kp[i] < left ? sp + op[i] : zero16, dst + (uint32_t)(NW * i) * 1024u);
#pragma unroll
            for (int i = 0; i < LQ; ++i) dma_load_1k_v(kq[i] < left ? sq + oq[i] : zero16, dst + P_BYTES + (uint32_t)(NW * i) * 1024u);
        }
        sp += step_p;
        sq += step_q;
        ++next;
    };

    float16_t acc[FP][FQ] = {};
    using FragP = Fragments<E, PA, BP, FP, WP>;
    using FragQ = Fragments<E, QA, BQ, FQ, WQ>;
    FragP fp[2][KH];
    FragQ fq[2][KH];
    const typename FragP::Place place_p = FragP::place(lds0, wp, lane);
    const typename FragQ::Place place_q = FragQ::place(lds0 + P_BYTES, wq, lane);
    constexpr int READS = KH * (FragP::READS + FragQ::READS);
    auto read_group = [&](uint32_t at, auto gc) {           // MFMA steps gc * KH .. of the stage at byte `at` of the ring
        constexpr int gr = decltype(gc)::value;
        static_for<KH>([&](auto kc) {
            constexpr int k = decltype(kc)::value;
            fq[gr & 1][k].template read<gr * KH + k>(place_q, at);
            fp[gr & 1][k].template read<gr * KH + k>(place_p, at);
        });
    };
    auto await_group = [&](auto bufc, auto newerc) {
        lds_wait<(decltype(newerc)::value < 15 ? decltype(newerc)::value : 15)>();
#pragma unroll
        for (int k = 0; k < KH; ++k) { fp[decltype(bufc)::value][k].pin_all(); fq[decltype(bufc)::value][k].pin_all(); }
    };
    auto mma_group = [&](auto bufc) {
#pragma unroll
        for (int k = 0; k < KH; ++k)
#pragma unroll
            for (int i = 0; i < FP; ++i)
#pragma unroll
                for (int j = 0; j < FQ; ++j) Mma<E>::run(fp[decltype(bufc)::value][k].get(i), fq[decltype(bufc)::value][k].get(j), acc[i][j]);
    };
    using Newer = std::integral_constant<int, READS>;
    using None = std::integral_constant<int, 0>;

    // fill the ring, wait for the first stage, request its first fragments
#pragma unroll
    for (int s = 0; s < NST; ++s)
        if (s < stages) issue(s);
    if (stages >= NST) wait_vmcnt<(NST - 1) * (LP + LQ)>();
    else wait_vmcnt<0>();
    __syncthreads();
    read_group(0, std::integral_constant<int, 0>());
    int slot = 0;
    for (int s = 0; s < stages; ++s) {
        const uint32_t at = (uint32_t)slot * STAGE;
        const int next_slot = slot + 1 == NST ? 0 : slot + 1;
        static_for<NG - 1>([&](auto gc) {
            constexpr int gr = decltype(gc)::value;
            read_group(at, std::integral_constant<int, gr + 1>());
            await_group(std::integral_constant<int, (gr & 1)>(), Newer());
            __builtin_amdgcn_sched_barrier(0);
            mma_group(std::integral_constant<int, (gr & 1)>());
            __builtin_amdgcn_sched_barrier(0);
        });
        using Last = std::integral_constant<int, ((NG - 1) & 1)>;
        await_group(Last(), None());                       // this wave has read all of stage s
        if (s + 1 < stages) {
            // stage s + 1 has landed once no more transfers are outstanding than were issued after it
            if (s + NST <= stages) wait_vmcnt<(NST - 2) * (LP + LQ)>();
            else wait_vmcnt<0>();
            __syncthreads();                               // ... for every wave, and every wave has read all of stage s
            if (s + NST < stages) issue(slot);             // stage s + NST, into the slot that stage s used
            read_group((uint32_t)next_slot * STAGE, std::integral_constant<int, 0>());
        }
        __builtin_amdgcn_sched_barrier(0);
        mma_group(Last());
        __builtin_amdgcn_sched_barrier(0);
        slot = next_slot;
    }

    const long long sum_row = (long long)bq * WQ + wq, top_at = ((long long)bq * tiles_p + bp) * NW + wave;
    if constexpr (EP == EP_STORE) {
        finish_tile<E, EP, ACT_NONE, FP, FQ, WP, WQ>(g, e, acc, n0, m0, wp, wq, sum_row, top_at, lane, split);
    } else {
        switch (e.act) {                                   // uniform
            case ACT_NONE:
                if constexpr (EP != EP_DLINEAR) finish_tile<E, EP, ACT_NONE, FP, FQ, WP, WQ>(g, e, acc, n0, m0, wp, wq, sum_row, top_at, lane, split);
                break;                                     // (dz is dy as it stands)
            case ACT_SILU: finish_tile<E, EP, ACT_SILU, FP, FQ, WP, WQ>(g, e, acc, n0, m0, wp, wq, sum_row, top_at, lane, split); break;
            case ACT_GELU: finish_tile<E, EP, ACT_GELU, FP, FQ, WP, WQ>(g, e, acc, n0, m0, wp, wq, sum_row, top_at, lane, split); break;
            default: finish_tile<E, EP, ACT_GELU_TANH, FP, FQ, WP, WQ>(g, e, acc, n0, m0, wp, wq, sum_row, top_at, lane, split); break;
        }
    }
}

template <typename E, int EP, bool PA, bool QA, int BP, int BQ, int WP, int WQ, int NST>
__global__ void __launch_bounds__(WP * WQ * 64) gemm_tile_kernel(Operand P, Operand Q, GemmShape g, Epilogue e, int tiles_p, int tiles_q, int total, int per_xcd, int nsplit) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int logical = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if (logical >= total) return;                          // uniform per workgroup, before any barrier
    if ((EP == EP_DLINEAR || EP == EP_DGLU) && store_factor<E, true>(e) == 0.f) return;
    gemm_tile<E, EP, PA, QA, BP, BQ, WP, WQ, NST>(P, Q, g, e, tiles_p, tiles_q, nsplit, logical, lds);
}

// Two products in one launch, dz w (P across, Q along) and dz^T x (both across): either alone has few tiles and long reductions, together they fill the
// chip.  XCD by XCD the first one's tiles, then the second one's.  The bias gradient, where it is asked for, is summed by workgroups of its own in
// front of them (616 x 2048 x 1280: 5.6 us as a launch before; 4096 x 640 x 2 x 2560: 5.1 us after).
struct PairPart { Operand P, Q; GemmShape g; Epilogue e; int tiles_p, tiles_q, total, per_xcd, nsplit; };
template <typename E, int BP, int BQ, int WP, int WQ, int NST>
__global__ void __launch_bounds__(WP * WQ * 64) gemm_pair_kernel(PairPart a, PairPart b, ColumnSums c, bool vec, int sum_blocks, int sum_per_xcd) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int xcd = blockIdx.x % 8, at = (int)(blockIdx.x / 8) - sum_per_xcd;
    if (at < 0) {
        const int id = blockIdx.x, range = id / sum_blocks;
        if (range >= c.ranges) return;
        if (c.f32) column_sums<float, WP * WQ>(c, vec, id - range * sum_blocks, range, c.ranges, reinterpret_cast<float*>(lds));
        else column_sums<E, WP * WQ>(c, vec, id - range * sum_blocks, range, c.ranges, reinterpret_cast<float*>(lds));
    } else if (at < a.per_xcd) {
        const int logical = xcd * a.per_xcd + at;
        if (logical < a.total) gemm_tile<E, EP_STORE, true, false, BP, BQ, WP, WQ, NST>(a.P, a.Q, a.g, a.e, a.tiles_p, a.tiles_q, a.nsplit, logical, lds);
    } else {
        const int logical = xcd * b.per_xcd + at - a.per_xcd;
        if (logical < b.total) gemm_tile<E, EP_STORE, true, true, BP, BQ, WP, WQ, NST>(b.P, b.Q, b.g, b.e, b.tiles_p, b.tiles_q, b.nsplit, logical, lds);
    }
}

template <typename E, int EP, bool PA, bool QA, int BP, int BQ, int WP, int WQ, int NST>
hipError_t launch_cfg(const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, hipStream_t s, Filled* filled) {
    constexpr bool GLU = EP == EP_GLU || EP == EP_DGLU;
    constexpr int bn = GLU ? BP / 2 : BP, bytes = (BP + BQ) * 128 * NST;
    static_assert(bytes <= 160 * 1024, "LDS budget");
    const long long tp = (g.N + bn - 1) / bn, tq = ((long long)g.M + BQ - 1) / BQ, total = tp * tq * nsplit;
    if (total > 0x3fffffffLL) return hipErrorInvalidValue;
    const int per_xcd = (int)((total + 7) / 8);
    if (filled) *filled = Filled{(int)tq * WQ, tp * tq * (WP * WQ)};
    auto kern = gemm_tile_kernel<E, EP, PA, QA, BP, BQ, WP, WQ, NST>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(kern, dim3((unsigned)(per_xcd * 8)), dim3(WP * WQ * 64), bytes, s, P, Q, g, e, (int)tp, (int)tq, (int)total, per_xcd, nsplit);
    return hipGetLastError();
}

// Which block.  Measured on 44 products of a block's sizes, us (4096^3 / 4096 x 640 x 5120 / 4096 x 2560 x 640 / 512 x 5120 x 1280, M x K x N):
// 256x256 116 / 41 / 56 / 104, 128x128 with two stages 129 / 34 / 30 / 55, with three 160 / 40 / 23 / 42, 64x64 - / 46 / 26 / 23.  A large block
// moves the fewest bytes through LDS per flop, but has to fill the chip, and with one workgroup per compute unit its epilogue overlaps with nothing:
// worth it for long reductions only.  128x128 runs two workgroups per unit where there are enough; where there is about one, a third stage pays.
template <typename E, int EP, bool PA, bool QA> hipError_t launch_shape(const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, hipStream_t s, Filled* filled) {
    constexpr bool GLU = EP == EP_GLU || EP == EP_DGLU;
    const long long width = GLU ? 2LL * g.N : g.N, t256 = ((width + 255) / 256) * ((g.M + 255) / 256) * nsplit, t128 = ((width + 127) / 128) * ((g.M + 127) / 128) * nsplit;
    const int depth = g.K / nsplit;
    if constexpr (sizeof(E) == 4) {
        // bound by its MFMAs: the large block only where its tiles fill the units evenly (4096^3 144 TFLOP/s of the library's 151)
        if (t128 >= 768) return launch_cfg<E, EP, PA, QA, 128, 128, 2, 2, 2>(P, Q, g, e, nsplit, s, filled);
        if constexpr (GLU) return launch_cfg<E, EP, PA, QA, 128, 64, 2, 2, 2>(P, Q, g, e, nsplit, s, filled);
        else if (depth < 512) return launch_cfg<E, EP, PA, QA, 64, 64, 2, 2, 2>(P, Q, g, e, nsplit, s, filled);
        else return launch_cfg<E, EP, PA, QA, 64, 64, 2, 2, 3>(P, Q, g, e, nsplit, s, filled);
    } else {
    if (depth >= 1536 && t256 >= 224) return launch_cfg<E, EP, PA, QA, 256, 256, 2, 4, 2>(P, Q, g, e, nsplit, s, filled);
    if (t128 >= 320) return launch_cfg<E, EP, PA, QA, 128, 128, 2, 4, 2>(P, Q, g, e, nsplit, s, filled);
    if (t128 >= 130 && depth >= 1024) return launch_cfg<E, EP, PA, QA, 128, 128, 2, 4, 3>(P, Q, g, e, nsplit, s, filled);
    if constexpr (GLU) return launch_cfg<E, EP, PA, QA, 128, 64, 2, 2, 3>(P, Q, g, e, nsplit, s, filled);       // u and g in one wave: 64 rows of P each
    else return launch_cfg<E, EP, PA, QA, 64, 64, 2, 2, 3>(P, Q, g, e, nsplit, s, filled);
    }
}

template <typename E, int EP> hipError_t launch_layout(bool pa, bool qa, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, hipStream_t s, Filled* filled) {
    if constexpr (EP == EP_STORE) {
        if (pa && qa) return launch_shape<E, EP, true, true>(P, Q, g, e, nsplit, s, filled);
        if (pa) return launch_shape<E, EP, true, false>(P, Q, g, e, nsplit, s, filled);
    }
    return launch_shape<E, EP, false, false>(P, Q, g, e, nsplit, s, filled);
}

template <typename E> hipError_t launch_ep(int ep, bool pa, bool qa, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, hipStream_t s, Filled* filled) {
    switch (ep) {
        case EP_STORE:
        case EP_PART: return launch_layout<E, EP_STORE>(pa, qa, P, Q, g, e, nsplit, s, filled);      // (told apart by e.part)
        case EP_LINEAR: return launch_layout<E, EP_LINEAR>(pa, qa, P, Q, g, e, nsplit, s, filled);
        case EP_DLINEAR: return launch_layout<E, EP_DLINEAR>(pa, qa, P, Q, g, e, nsplit, s, filled);
        case EP_GLU: return launch_layout<E, EP_GLU>(pa, qa, P, Q, g, e, nsplit, s, filled);
        case EP_DGLU: return launch_layout<E, EP_DGLU>(pa, qa, P, Q, g, e, nsplit, s, filled);
        default: return hipErrorInvalidValue;
    }
}

template <typename E, int BP, int BQ, int WP, int WQ, int NST> hipError_t launch_pair(PairPart a, PairPart b, const ColumnSums& c, hipStream_t s) {
    constexpr int bytes = (BP + BQ) * 128 * NST;
    static_assert(bytes <= 160 * 1024, "LDS budget");
    for (PairPart* p : {&a, &b}) {
        const long long tp = (p->g.N + BP - 1) / BP, tq = ((long long)p->g.M + BQ - 1) / BQ, total = tp * tq * p->nsplit;
        if (total > 0x1fffffffLL) return hipErrorInvalidValue;
        p->tiles_p = (int)tp; p->tiles_q = (int)tq; p->total = (int)total; p->per_xcd = (int)((total + 7) / 8);
    }
    auto kern = gemm_pair_kernel<E, BP, BQ, WP, WQ, NST>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (attr != hipSuccess) return attr;
    const int sum_blocks = c.out ? (c.N + 63) / 64 : 0, sum_per_xcd = (sum_blocks * c.ranges + 7) / 8;
    const Operand x{c.x, c.ld};
    const bool vec = c.f32 ? vec_rows<float>(x) : vec_rows<E>(x);
    hipLaunchKernelGGL(kern, dim3((unsigned)((sum_per_xcd + a.per_xcd + b.per_xcd) * 8)), dim3(WP * WQ * 64), bytes, s, a, b, c, vec, sum_blocks, sum_per_xcd);
    return hipGetLastError();
}

long long tiles128(const GemmShape& g) { return (((long long)g.N + 127) / 128) * (((long long)g.M + 127) / 128); }

}  // namespace

hipError_t launch_tile_pair(const Product& a, const Product& b, const ColumnSums& c, int dt, hipStream_t s) {
    const PairPart pa{a.P, a.Q, a.g, a.e, 0, 0, 0, 0, a.nsplit}, pb{b.P, b.Q, b.g, b.e, 0, 0, 0, 0, b.nsplit};
    const long long t128 = tiles128(a.g) * a.nsplit + tiles128(b.g) * b.nsplit;
    return with_dtype(dt, [&](auto* tag) -> hipError_t {
        using E = std::remove_pointer_t<decltype(tag)>;
        if constexpr (sizeof(E) == 4) return t128 >= 768 ? launch_pair<E, 128, 128, 2, 2, 2>(pa, pb, c, s) : launch_pair<E, 64, 64, 2, 2, 3>(pa, pb, c, s);
        else return t128 >= 256 ? launch_pair<E, 128, 128, 2, 4, 2>(pa, pb, c, s) : launch_pair<E, 64, 64, 2, 2, 3>(pa, pb, c, s);
    });
}

bool tile_gemm_ok(int ep, bool pa, bool qa, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int dt) {
    const long long es = two_byte(dt) ? 2 : 4;
    if (es == 2 ? !(vec_rows<__half>(P) && vec_rows<__half>(Q)) : !(vec_rows<float>(P) && vec_rows<float>(Q))) return false;
    const bool glu = ep == EP_GLU || ep == EP_DGLU;
    const int v = es == 2 ? 8 : 4;
    if (g.N % 8 || (qa && g.M % v) || (!(pa && qa) && g.K % v)) return false;       // chunks of 16 bytes are whole; out is written in eights
    // a lane's offset within a workgroup's rows is 32 bits wide
    const long long span_p = pa ? 64 : glu ? (long long)g.N + 256 : 256, span_q = qa ? 64 : 256;
    if (P.ld * es * span_p >= (1LL << 31) || Q.ld * es * span_q >= (1LL << 31)) return false;
    if (ep == EP_PART) return true;
    uintptr_t bits = reinterpret_cast<uintptr_t>(e.out) | (uintptr_t)(e.ld_out * es);
    if (e.extra) bits |= reinterpret_cast<uintptr_t>(e.extra) | (uintptr_t)(e.ld_extra * es);
    return (bits & 15) == 0;
}

hipError_t launch_tile_gemm(int ep, bool pa, bool qa, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, int dt, hipStream_t s, Filled* filled) {
    return with_dtype(dt, [&](auto* tag) -> hipError_t { return launch_ep<std::remove_pointer_t<decltype(tag)>>(ep, pa, qa, P, Q, g, e, nsplit, s, filled); });
}

}  // namespace wino
