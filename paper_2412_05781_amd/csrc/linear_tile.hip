// The matrix kernel of the transformer-block operators for two-byte types whose operands can be fetched 16 bytes at a time: global -> LDS transfers
// without a detour through registers, a ring of stages of 64 reduction elements, eight or four waves that own 32x32 MFMA tiles.
//
// A stage of an operand that runs along the reduction is BI rows of 128 bytes, of one across it 64 rows of BI elements; both are filled by transfers of
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
template <typename E> __device__ __forceinline__ void load8(const E* p, float* v) {
    const uint4 f = *reinterpret_cast<const uint4*>(p);
    v[0] = lo16<E>(f.x); v[1] = hi16<E>(f.x); v[2] = lo16<E>(f.y); v[3] = hi16<E>(f.y);
    v[4] = lo16<E>(f.z); v[5] = hi16<E>(f.z); v[6] = lo16<E>(f.w); v[7] = hi16<E>(f.w);
}
template <typename E> __device__ __forceinline__ void store8(E* p, const float* v) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2<E>(v[0], v[1]), pack2<E>(v[2], v[3]), pack2<E>(v[4], v[5]), pack2<E>(v[6], v[7]));
}

// Epilogue of one wave's tile.  acc[i][j]: rows n of 32-row block i (GLU: block i of the up rows, FP / 2 + i of the gate rows), columns m of block j.
template <typename E, int EP, int ACT, int FP, int FQ, int WP, int WQ>
__device__ __forceinline__ void finish_tile(const GemmShape& g, const Epilogue& e, float16_t (&acc)[FP][FQ], int n0, long long m0, int wp, int wq, long long sum_row, int lane, int split) {
    constexpr bool GLU = EP == EP_GLU || EP == EP_DGLU, SUMS = EP == EP_DLINEAR || EP == EP_DGLU;
    constexpr int NI = GLU ? FP / 2 : FP;
    const int half = lane >> 5;
    E* out = static_cast<E*>(e.out);
    const E* extra = static_cast<const E*>(e.extra);
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int qp = 0; qp < 2; ++qp) {
            // after the exchange of halves a lane holds n .. n + 7 of its row
            const int n = n0 + (i * WP + wp) * 32 + 16 * qp + 8 * half;
            const bool n_on = n < g.N;                     // N is a multiple of 8 here
            float bias[8] = {}, bias2[8] = {}, sum[8] = {}, sum2[8] = {};
            if constexpr (EP != EP_STORE && EP != EP_PART) {
                if (e.bias && n_on) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) bias[k] = e.bias[n + k];
                    if constexpr (GLU) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) bias2[k] = e.bias[g.N + n + k];
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < FQ; ++j) {
                const long long m = m0 + (j * WQ + wq) * 32 + (lane & 31);
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
                if (!(n_on && m < g.M)) continue;
                if constexpr (EP == EP_PART) {
                    float* p = e.part + ((long long)split * g.M + m) * g.N + n;
                    *reinterpret_cast<float4*>(p) = make_float4(s[0], s[1], s[2], s[3]);
                    *reinterpret_cast<float4*>(p + 4) = make_float4(s[4], s[5], s[6], s[7]);
                } else if constexpr (EP == EP_STORE) {
                    store8<E>(out + m * e.ld_out + n, s);
                } else if constexpr (EP == EP_LINEAR) {
                    float r[8] = {};
                    if (extra) load8<E>(extra + m * e.ld_extra + n, r);
#pragma unroll
                    for (int k = 0; k < 8; ++k) a[k] = act_only<E, ACT>(s[k] + bias[k]) + r[k];
                    store8<E>(out + m * e.ld_out + n, a);
                } else if constexpr (EP == EP_GLU) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) a[k] = (s[k] + bias[k]) * act_only<E, ACT>(s2[k] + bias2[k]);
                    store8<E>(out + m * e.ld_out + n, a);
                } else {
                    float r[8];
                    load8<E>(extra + m * e.ld_extra + n, r);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        float v, d;
                        if constexpr (EP == EP_DLINEAR) {
                            act_both<E, ACT>(s[k] + bias[k], v, d);
                            a[k] = r[k] * d;
                        } else {
                            act_both<E, ACT>(s2[k] + bias2[k], v, d);
                            a[k] = r[k] * v;
                            b[k] = r[k] * (s[k] + bias[k]) * d;
                            sum2[k] += b[k];
                        }
                        sum[k] += a[k];
                    }
                    store8<E>(out + m * e.ld_out + n, a);
                    if constexpr (EP == EP_DGLU) store8<E>(out + m * e.ld_out + g.N + n, b);
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
                if ((lane & 31) == 0 && n_on) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        e.sums[sum_row * width + n + k] = sum[k];
                        if constexpr (EP == EP_DGLU) e.sums[sum_row * width + g.N + n + k] = sum2[k];
                    }
                }
            }
        }
}

// BP rows of P x BQ rows of Q per workgroup of WP x WQ waves, ring of NST stages.
template <typename E, int EP, bool PA, bool QA, int BP, int BQ, int WP, int WQ, int NST>
__global__ void __launch_bounds__(WP * WQ * 64) gemm_tile_kernel(Operand P, Operand Q, GemmShape g, Epilogue e, int tiles_p, int tiles_q, int total, int per_xcd, int nsplit) {
    constexpr bool GLU = EP == EP_GLU || EP == EP_DGLU;
    constexpr int NW = WP * WQ, FP = BP / (32 * WP), FQ = BQ / (32 * WQ);
    constexpr int P_BYTES = BP * 128, STAGE = (BP + BQ) * 128;
    constexpr int LP = BP / 8 / NW, LQ = BQ / 8 / NW;      // 1 KB transfers per wave and stage
    constexpr int BN = GLU ? BP / 2 : BP;
    static_assert(BP % (8 * NW) == 0 && BQ % (8 * NW) == 0, "whole transfers");
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];

    const int logical = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if (logical >= total) return;                          // uniform per workgroup, before any barrier
    const int split = logical / (tiles_p * tiles_q), in = logical - split * (tiles_p * tiles_q);
    const int bq = in / tiles_p, bp = in - bq * tiles_p;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wq = wave / WP;
    const int n0 = bp * BN;
    const long long m0 = (long long)bq * BQ;
    const int nk = (g.K + 63) / 64;
    const int kt0 = (int)((long long)split * nk / nsplit), kt1 = (int)((long long)(split + 1) * nk / nsplit), stages = kt1 - kt0;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte_t*)lds;

    // Where transfer i of this wave fetches: a wave-uniform base that moves with the stage and a byte offset per lane.
    const unsigned char* sp = static_cast<const unsigned char*>(P.p) + (PA ? ((long long)kt0 * 64 * P.ld + n0) * 2 : ((long long)n0 * P.ld + (long long)kt0 * 64) * 2);
    const unsigned char* sq = static_cast<const unsigned char*>(Q.p) + (QA ? ((long long)kt0 * 64 * Q.ld + m0) * 2 : (m0 * Q.ld + (long long)kt0 * 64) * 2);
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
            op[i] = (uint32_t)r * (uint32_t)(P.ld * 2) + (uint32_t)chunk * 16u;
            kp[i] = chunk * 8;
        } else {
            constexpr int CPR = BP / 8, RPT = 64 / CPR;
            const int row = t * RPT + lane / CPR, chunk = (lane % CPR) ^ swz_across<E, BP>(row);
            const int c = n0 + chunk * 8 < g.N ? chunk * 8 : g.N - 8 - n0;
            op[i] = (uint32_t)row * (uint32_t)(P.ld * 2) + (uint32_t)(c * 2);
            kp[i] = row;
        }
    }
#pragma unroll
    for (int i = 0; i < LQ; ++i) {
        const int t = wave + NW * i;
        if constexpr (!QA) {
            const int row = t * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
            const int r = m0 + row < g.M ? row : (int)(g.M - 1 - m0);
            oq[i] = (uint32_t)r * (uint32_t)(Q.ld * 2) + (uint32_t)chunk * 16u;
            kq[i] = chunk * 8;
        } else {
            constexpr int CPR = BQ / 8, RPT = 64 / CPR;
            const int row = t * RPT + lane / CPR, chunk = (lane % CPR) ^ swz_across<E, BQ>(row);
            const int c = m0 + chunk * 8 < g.M ? chunk * 8 : (int)(g.M - 8 - m0);
            oq[i] = (uint32_t)row * (uint32_t)(Q.ld * 2) + (uint32_t)(c * 2);
            kq[i] = row;
        }
    }
    const long long step_p = PA ? 64 * P.ld * 2 : 128, step_q = QA ? 64 * Q.ld * 2 : 128;
    int next = kt0;                                        // next stage to fetch
    auto issue = [&](int slot) {
        const uint32_t dst = lds0 + (uint32_t)slot * STAGE + (uint32_t)wave * 1024u;
        const int left = g.K - next * 64;                  // reduction elements from this stage on
        if (left >= 64) {
#pragma unroll
            for (int i = 0; i < LP; ++i) dma_load_1k_s(sp, op[i], dst + (uint32_t)(NW * i) * 1024u);
#pragma unroll
            for (int i = 0; i < LQ; ++i) dma_load_1k_s(sq, oq[i], dst + P_BYTES + (uint32_t)(NW * i) * 1024u);
        } else {                                           // K is a multiple of 8 where a chunk runs along it
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
#pragma unroll
    for (int s = 0; s < NST - 1; ++s)
        if (s < stages) issue(s);
    int slot = 0;
    for (int s = 0; s < stages; ++s) {
        // stage s has landed once no more transfers are outstanding than were issued after it
        if (s + NST - 1 <= stages) wait_vmcnt<(NST - 2) * (LP + LQ)>();
        else wait_vmcnt<0>();
        __syncthreads();                                   // ... for every wave, and every wave has read stage s - 1
        if (s + NST - 1 < stages) issue(slot == 0 ? NST - 1 : slot - 1);
        const unsigned char* tp = lds + slot * STAGE;
        const unsigned char* tq = tp + P_BYTES;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            u32x4_t fp[FP], fq[FQ];
#pragma unroll
            for (int j = 0; j < FQ; ++j) fq[j] = read_fragment<E, QA, BQ>(tq, (j * WQ + wq) * 32, ks, lane);
#pragma unroll
            for (int i = 0; i < FP; ++i) fp[i] = read_fragment<E, PA, BP>(tp, (i * WP + wp) * 32, ks, lane);
#pragma unroll
            for (int i = 0; i < FP; ++i)
#pragma unroll
                for (int j = 0; j < FQ; ++j) Mma<E>::run(fp[i], fq[j], acc[i][j]);
        }
        slot = slot + 1 == NST ? 0 : slot + 1;
    }

    const long long sum_row = (long long)bq * WQ + wq;
    if constexpr (EP == EP_STORE || EP == EP_PART) {
        finish_tile<E, EP, ACT_NONE, FP, FQ, WP, WQ>(g, e, acc, n0, m0, wp, wq, sum_row, lane, split);
    } else {
        switch (e.act) {                                   // uniform
            case ACT_NONE: finish_tile<E, EP, ACT_NONE, FP, FQ, WP, WQ>(g, e, acc, n0, m0, wp, wq, sum_row, lane, split); break;
            case ACT_SILU: finish_tile<E, EP, ACT_SILU, FP, FQ, WP, WQ>(g, e, acc, n0, m0, wp, wq, sum_row, lane, split); break;
            case ACT_GELU: finish_tile<E, EP, ACT_GELU, FP, FQ, WP, WQ>(g, e, acc, n0, m0, wp, wq, sum_row, lane, split); break;
            default: finish_tile<E, EP, ACT_GELU_TANH, FP, FQ, WP, WQ>(g, e, acc, n0, m0, wp, wq, sum_row, lane, split); break;
        }
    }
}

template <typename E, int EP, bool PA, bool QA, int BP, int BQ, int WP, int WQ, int NST>
hipError_t launch_cfg(const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, hipStream_t s, int* sum_rows) {
    constexpr bool GLU = EP == EP_GLU || EP == EP_DGLU;
    constexpr int bn = GLU ? BP / 2 : BP, bytes = (BP + BQ) * 128 * NST;
    static_assert(bytes <= 160 * 1024, "LDS budget");
    const long long tp = (g.N + bn - 1) / bn, tq = ((long long)g.M + BQ - 1) / BQ, total = tp * tq * nsplit;
    if (total > 0x3fffffffLL) return hipErrorInvalidValue;
    const int per_xcd = (int)((total + 7) / 8);
    if (sum_rows) *sum_rows = (int)tq * WQ;
    auto kern = gemm_tile_kernel<E, EP, PA, QA, BP, BQ, WP, WQ, NST>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(kern, dim3((unsigned)(per_xcd * 8)), dim3(WP * WQ * 64), bytes, s, P, Q, g, e, (int)tp, (int)tq, (int)total, per_xcd, nsplit);
    return hipGetLastError();
}

template <typename E, int EP, bool PA, bool QA> hipError_t launch_shape(const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, hipStream_t s, int* sum_rows) {
    constexpr bool GLU = EP == EP_GLU || EP == EP_DGLU;
    const long long width = GLU ? 2LL * g.N : g.N, big = ((width + 255) / 256) * ((g.M + 255) / 256) * nsplit;
    if (big >= 224) return launch_cfg<E, EP, PA, QA, 256, 256, 2, 4, 2>(P, Q, g, e, nsplit, s, sum_rows);
    return launch_cfg<E, EP, PA, QA, 128, 128, 2, 2, 2>(P, Q, g, e, nsplit, s, sum_rows);
}

template <typename E, int EP> hipError_t launch_layout(bool pa, bool qa, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, hipStream_t s, int* sum_rows) {
    if constexpr (EP == EP_STORE || EP == EP_PART) {
        if (pa && qa) return launch_shape<E, EP, true, true>(P, Q, g, e, nsplit, s, sum_rows);
        if (pa) return launch_shape<E, EP, true, false>(P, Q, g, e, nsplit, s, sum_rows);
    }
    return launch_shape<E, EP, false, false>(P, Q, g, e, nsplit, s, sum_rows);
}

template <typename E> hipError_t launch_ep(int ep, bool pa, bool qa, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, hipStream_t s, int* sum_rows) {
    switch (ep) {
        case EP_STORE: return launch_layout<E, EP_STORE>(pa, qa, P, Q, g, e, nsplit, s, sum_rows);
        case EP_PART: return launch_layout<E, EP_PART>(pa, qa, P, Q, g, e, nsplit, s, sum_rows);
        case EP_LINEAR: return launch_layout<E, EP_LINEAR>(pa, qa, P, Q, g, e, nsplit, s, sum_rows);
        case EP_DLINEAR: return launch_layout<E, EP_DLINEAR>(pa, qa, P, Q, g, e, nsplit, s, sum_rows);
        case EP_GLU: return launch_layout<E, EP_GLU>(pa, qa, P, Q, g, e, nsplit, s, sum_rows);
        case EP_DGLU: return launch_layout<E, EP_DGLU>(pa, qa, P, Q, g, e, nsplit, s, sum_rows);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

bool tile_gemm_ok(int ep, bool pa, bool qa, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int dt) {
    if (!two_byte(dt) || !vec_rows<__half>(P) || !vec_rows<__half>(Q)) return false;
    const bool glu = ep == EP_GLU || ep == EP_DGLU;
    if (g.N % 8 || (qa && g.M % 8) || (!(pa && qa) && g.K % 8)) return false;       // chunks of 16 bytes are whole; out's rows as well
    // a lane's offset within a workgroup's rows is 32 bits wide
    const long long span_p = pa ? 64 : glu ? (long long)g.N + 256 : 256, span_q = qa ? 64 : 256;
    if (P.ld * 2 * span_p >= (1LL << 31) || Q.ld * 2 * span_q >= (1LL << 31)) return false;
    if (ep == EP_PART) return true;
    uintptr_t bits = reinterpret_cast<uintptr_t>(e.out) | (uintptr_t)(e.ld_out * 2);
    if (e.extra) bits |= reinterpret_cast<uintptr_t>(e.extra) | (uintptr_t)(e.ld_extra * 2);
    return (bits & 15) == 0;
}

hipError_t launch_tile_gemm(int ep, bool pa, bool qa, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, int dt, hipStream_t s, int* sum_rows) {
    return dt == DT_F16 ? launch_ep<__half>(ep, pa, qa, P, Q, g, e, nsplit, s, sum_rows) : launch_ep<bf16_t>(ep, pa, qa, P, Q, g, e, nsplit, s, sum_rows);
}

}  // namespace wino
