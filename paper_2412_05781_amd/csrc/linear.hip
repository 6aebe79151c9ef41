// Matrix products of a transformer block with what follows them in the epilogue:
//   out[m][n] = sum_k Q(m,k) P(n,k)
// with either operand stored along k or across it, so that one kernel serves x W^T, dz W and dz^T x.
//
// MFMA tiles hold n in their rows and m in their columns: a lane then owns four neighbouring n of one row m per four accumulator registers
// and stores them together.  For the gated block a tile holds as many rows of the up weights as of the gate weights, dealt to the waves such that
// a lane owns u and g of the same (m, n).
#include "linear_tile.h"

namespace wino {

namespace {

// four columns n0.. of row m, from the sums of one lane; returns in c (and c2: the gate half) what the column sums take
// f: the power of two that what is stored takes (EP_STORE, EP_DLINEAR, EP_DGLU)
template <typename E, int EP, int ACT>
__device__ __forceinline__ void finish4(const GemmShape& g, const Epilogue& e, long long m, int n0, const float* s, const float* s2, float* c, float* c2, float f) {
    const int n = g.N - n0;
    float a[4];
    if constexpr (EP == EP_STORE) {
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = s[i] * f;
        store4<E>(static_cast<E*>(e.out) + m * e.ld_out + n0, n, a);
    } else if constexpr (EP == EP_LINEAR) {
        float r[4] = {0.f, 0.f, 0.f, 0.f};
        if (e.extra) load4<E>(static_cast<const E*>(e.extra) + m * e.ld_extra + n0, n, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float b = e.bias && i < n ? e.bias[n0 + i] : 0.f;
            a[i] = act_only<E, ACT>(s[i] + b) + r[i];
        }
        store4<E>(static_cast<E*>(e.out) + m * e.ld_out + n0, n, a);
    } else if constexpr (EP == EP_DLINEAR) {
        float r[4];
        load4<E>(static_cast<const E*>(e.extra) + m * e.ld_extra + n0, n, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float b = e.bias && i < n ? e.bias[n0 + i] : 0.f;
            float v, d;
            act_both<E, ACT>(s[i] + b, v, d);
            c[i] = i < n ? r[i] * d : 0.f;
            a[i] = c[i] * f;
        }
        store4<E>(static_cast<E*>(e.out) + m * e.ld_out + n0, n, a);
    } else if constexpr (EP == EP_GLU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float bu = e.bias && i < n ? e.bias[n0 + i] : 0.f, bg = e.bias && i < n ? e.bias[g.N + n0 + i] : 0.f;
            a[i] = (s[i] + bu) * act_only<E, ACT>(s2[i] + bg);
        }
        store4<E>(static_cast<E*>(e.out) + m * e.ld_out + n0, n, a);
    } else if constexpr (EP == EP_DGLU) {
        float r[4];
        load4<E>(static_cast<const E*>(e.extra) + m * e.ld_extra + n0, n, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float bu = e.bias && i < n ? e.bias[n0 + i] : 0.f, bg = e.bias && i < n ? e.bias[g.N + n0 + i] : 0.f;
            float v, d;
            act_both<E, ACT>(s2[i] + bg, v, d);
            c[i] = i < n ? r[i] * v : 0.f;
            c2[i] = i < n ? r[i] * (s[i] + bu) * d : 0.f;
            a[i] = c[i] * f;
        }
        store4<E>(static_cast<E*>(e.out) + m * e.ld_out + n0, n, a);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = c2[i] * f;
        store4<E>(static_cast<E*>(e.out) + m * e.ld_out + g.N + n0, n, a);
    }
}

__device__ __forceinline__ float sum_over_32(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// ---- the kernel for every shape: operands go through registers, at any alignment, element by element at the edge -------------------
constexpr int kBP = 128, kBQ = 64;       // tile: 128 rows of P x 64 rows of Q, four waves, 64 x 32 each

template <typename E, int EP, int ACT, bool PA, bool QA>
__global__ void __launch_bounds__(256) gemm_any_kernel(Operand P, Operand Q, GemmShape g, Epilogue e, int tiles_p, int tiles_q, int total, int per_xcd,
                                                       int nsplit) {
    constexpr bool GLU = EP == EP_GLU || EP == EP_DGLU;
    constexpr int BK = 128 / (int)sizeof(E), V = 16 / (int)sizeof(E);
    constexpr int P_CHUNKS = kBP * 8 / 256, Q_CHUNKS = kBQ * 8 / 256;
    __shared__ __attribute__((aligned(16))) unsigned char lds[(kBP + kBQ) * 128];
    unsigned char* tp = lds;
    unsigned char* tq = lds + kBP * 128;

    const int logical = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if (logical >= total) return;                          // uniform per workgroup, before any barrier
    constexpr bool SUMS = EP == EP_DLINEAR || EP == EP_DGLU;
    const float factor = store_factor<E, SUMS>(e);
    if (SUMS && factor == 0.f) return;                     // nothing to do again
    const int split = logical / (tiles_p * tiles_q), in = logical - split * (tiles_p * tiles_q);
    const int bq = in / tiles_p, bp = in - bq * tiles_p;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wp = wave & 1, wq = wave >> 1;
    constexpr int BN = GLU ? kBP / 2 : kBP;                // columns of out per tile
    const int n0 = bp * BN;
    const long long m0 = (long long)bq * kBQ;
    const int nk = (g.K + BK - 1) / BK;
    const int k_begin = (int)((long long)split * nk / nsplit), k_end = (int)((long long)(split + 1) * nk / nsplit);

    const E* pp = static_cast<const E*>(P.p);
    const E* qp = static_cast<const E*>(Q.p);
    // row r of the P tile is row p_row(r) of P, if r stands for an n inside the matrix
    auto p_row = [&](int r) { return GLU && r >= kBP / 2 ? g.N + n0 + r - kBP / 2 : n0 + r; };
    auto p_left = [&](int r) { const int n = n0 + (GLU && r >= kBP / 2 ? r - kBP / 2 : r); return g.N - n; };      // <= 0: outside
    u32x4_t rp[P_CHUNKS], rq[Q_CHUNKS];
    const u32x4_t zero = {0, 0, 0, 0};
    auto fetch = [&](int kt) {
        const int k0 = kt * BK;
#pragma unroll
        for (int i = 0; i < P_CHUNKS; ++i) {
            const int id = tid + 256 * i;
            if constexpr (!PA) {
                const int r = id >> 3, k = k0 + (id & 7) * V, n = p_left(r) > 0 ? g.K - k : 0;
                const E* at = pp + (long long)p_row(r) * P.ld + k;
                rp[i] = n <= 0 ? zero : load_part<E>(at, n);
            } else {
                constexpr int CPR = kBP / V;
                const int k = k0 + id / CPR, r = (id % CPR) * V, n = k < g.K ? p_left(r) : 0;
                const E* at = pp + (long long)k * P.ld + p_row(r);
                rp[i] = n <= 0 ? zero : load_part<E>(at, n);
            }
        }
#pragma unroll
        for (int i = 0; i < Q_CHUNKS; ++i) {
            const int id = tid + 256 * i;
            if constexpr (!QA) {
                const int k = k0 + (id & 7) * V;
                const long long m = m0 + (id >> 3);
                const int n = m < g.M ? g.K - k : 0;
                const E* at = qp + m * Q.ld + k;
                rq[i] = n <= 0 ? zero : load_part<E>(at, n);
            } else {
                constexpr int CPR = kBQ / V;
                const int k = k0 + id / CPR;
                const long long m = m0 + (id % CPR) * V;
                const long long left = k < g.K ? g.M - m : 0;
                const int n = left > V ? V : (int)left;
                const E* at = qp + (long long)k * Q.ld + m;
                rq[i] = n <= 0 ? zero : load_part<E>(at, n);
            }
        }
    };
    auto put = [&]() {
#pragma unroll
        for (int i = 0; i < P_CHUNKS; ++i) {
            const int id = tid + 256 * i;
            if constexpr (!PA) { const int r = id >> 3; *reinterpret_cast<u32x4_t*>(tp + r * 128 + (((id & 7) ^ ((r >> 1) & 7)) << 4)) = rp[i]; }
            else { constexpr int CPR = kBP / V; const int r = id / CPR; *reinterpret_cast<u32x4_t*>(tp + r * (kBP * (int)sizeof(E)) + (((id % CPR) ^ swz_across<E, kBP>(r)) << 4)) = rp[i]; }
        }
#pragma unroll
        for (int i = 0; i < Q_CHUNKS; ++i) {
            const int id = tid + 256 * i;
            if constexpr (!QA) { const int r = id >> 3; *reinterpret_cast<u32x4_t*>(tq + r * 128 + (((id & 7) ^ ((r >> 1) & 7)) << 4)) = rq[i]; }
            else {
                constexpr int CPR = kBQ / V;
                const int r = id / CPR;
                *reinterpret_cast<u32x4_t*>(tq + r * (kBQ * (int)sizeof(E)) + (((id % CPR) ^ swz_across<E, kBQ>(r)) << 4)) = rq[i];
            }
        }
    };

    float16_t acc[2] = {};
    if (k_begin < k_end) fetch(k_begin);
    for (int kt = k_begin; kt < k_end; ++kt) {
        __syncthreads();                                   // the tile has been read
        put();
        __syncthreads();
        if (kt + 1 < k_end) fetch(kt + 1);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const u32x4_t fq = read_fragment<E, QA, kBQ>(tq, wq * 32, ks, lane);
#pragma unroll
            for (int i = 0; i < 2; ++i) Mma<E>::run(read_fragment<E, PA, kBP>(tp, i * 64 + wp * 32, ks, lane), fq, acc[i]);
        }
    }

    // register r of lane l holds row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32 of a 32x32 tile
    const long long m = m0 + wq * 32 + (lane & 31);
    const int half = lane >> 5;
    if constexpr (EP == EP_PART) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int n = n0 + i * 64 + wp * 32 + 8 * (r / 4) + 4 * half + r % 4;
                if (m < g.M && n < g.N) e.part[((long long)split * g.M + m) * g.N + n] = acc[i][r];
            }
        return;
    }
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < (GLU ? 1 : 2); ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = n0 + i * 64 + wp * 32 + 8 * q + 4 * half;
            float s[4], s2[4], c[4] = {}, c2[4] = {};
#pragma unroll
            for (int j = 0; j < 4; ++j) { s[j] = acc[i][4 * q + j]; s2[j] = acc[1][4 * q + j]; }
            if (m < g.M && n < g.N) finish4<E, EP, ACT>(g, e, m, n, s, s2, c, c2, factor);
            if constexpr (SUMS) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    top = larger_finite(top, c[j]);
                    if constexpr (EP == EP_DGLU) top = larger_finite(top, c2[j]);
                }
                const long long row = (long long)bq * 2 + wq;
                const int width = EP == EP_DGLU ? 2 * g.N : g.N;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float t = sum_over_32(c[j]);
                    if ((lane & 31) == 0 && n + j < g.N) e.sums[row * width + n + j] = t;
                    if constexpr (EP == EP_DGLU) {
                        const float t2 = sum_over_32(c2[j]);
                        if ((lane & 31) == 0 && n + j < g.N) e.sums[row * width + g.N + n + j] = t2;
                    }
                }
            }
        }
    if constexpr (SUMS && std::is_same_v<E, __half>) store_top(e, ((long long)bq * tiles_p + bp) * 4 + wave, top, lane);
}

template <typename E, int EP, int ACT, bool PA, bool QA>
hipError_t launch_any(const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, hipStream_t s) {
    constexpr bool GLU = EP == EP_GLU || EP == EP_DGLU;
    const int bn = GLU ? kBP / 2 : kBP;
    const long long tp = (g.N + bn - 1) / bn, tq = ((long long)g.M + kBQ - 1) / kBQ, total = tp * tq * nsplit;
    if (total > 0x3fffffffLL) return hipErrorInvalidValue;
    const int per_xcd = (int)((total + 7) / 8);
    hipLaunchKernelGGL((gemm_any_kernel<E, EP, ACT, PA, QA>), dim3((unsigned)(per_xcd * 8)), dim3(256), 0, s, P, Q, g, e, (int)tp, (int)tq, (int)total, per_xcd,
                       nsplit);
    return hipGetLastError();
}

template <typename E, int EP> hipError_t with_act(const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, hipStream_t s) {
    switch (e.act) {
        case ACT_NONE:
            if constexpr (EP == EP_DLINEAR) return hipErrorInvalidValue;         // dz is dy as it stands
            else return launch_any<E, EP, ACT_NONE, false, false>(P, Q, g, e, 1, s);
        case ACT_SILU: return launch_any<E, EP, ACT_SILU, false, false>(P, Q, g, e, 1, s);
        case ACT_GELU: return launch_any<E, EP, ACT_GELU, false, false>(P, Q, g, e, 1, s);
        case ACT_GELU_TANH: return launch_any<E, EP, ACT_GELU_TANH, false, false>(P, Q, g, e, 1, s);
        default: return hipErrorInvalidValue;
    }
}

template <typename E, int EP> hipError_t with_layout(bool pa, bool qa, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, hipStream_t s) {
    if constexpr (EP == EP_PART)
        if (!pa && !qa) return launch_any<E, EP, ACT_NONE, false, false>(P, Q, g, e, nsplit, s);
    if (pa && !qa) return launch_any<E, EP, ACT_NONE, true, false>(P, Q, g, e, nsplit, s);
    if (pa && qa) return launch_any<E, EP, ACT_NONE, true, true>(P, Q, g, e, nsplit, s);
    return hipErrorInvalidValue;
}

// ---- joining ranges, column sums ------------------------------------------------------------------------------------------------------
template <typename E, int ACT> __global__ void __launch_bounds__(256) join_kernel(const float* part, int nsplit, GemmShape g, Epilogue e, bool linear) {
    const long long quads = (g.N + 3) / 4, id = (long long)blockIdx.x * 256 + threadIdx.x;
    if (id >= quads * g.M) return;
    const float factor = store_factor<E, false>(e);
    const long long m = id / quads;
    const int n0 = (int)(id - m * quads) * 4;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    const size_t step = (size_t)g.M * g.N;
    const float* p = part + (size_t)m * g.N + n0;
    if (g.N % 4 == 0) {
#pragma unroll 4
        for (int r = 0; r < nsplit; ++r) {
            const float4 v = *reinterpret_cast<const float4*>(p + (size_t)r * step);
            s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
        }
    } else {
        for (int r = 0; r < nsplit; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < g.N) s[i] += p[(size_t)r * step + i];
    }
    if (linear) finish4<E, EP_LINEAR, ACT>(g, e, m, n0, s, s, nullptr, nullptr, factor);
    else finish4<E, EP_STORE, ACT>(g, e, m, n0, s, s, nullptr, nullptr, factor);
}

// 64 columns per workgroup, sixteen waves that take every sixteenth row
__global__ void __launch_bounds__(1024) sum_rows_kernel(const float* part, int rows, int cols, float* out) {
    const int l = threadIdx.x & 63, c = blockIdx.x * 64 + l, w = threadIdx.x >> 6;
    __shared__ float t[16][64];
    float a = 0.f;
    if (c < cols)
#pragma unroll 4
        for (int r = w; r < rows; r += 16) a += part[(size_t)r * cols + c];
    t[w][l] = a;
    __syncthreads();
    if (w == 0 && c < cols) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v += t[i][l];
        out[c] = v;
    }
}

// Up to 65504 there is nothing to do, and from 1 on what lies a factor of 2^14 below the largest still has all its bits.  Otherwise the largest goes to 2^14 .. 2^15.
__global__ void __launch_bounds__(1024) power_kernel(const float* tops, long long n, int* power) {
    __shared__ float t[16];
    float v = 0.f;
    for (long long i = threadIdx.x; i < n; i += 1024) v = fmaxf(v, tops[i]);
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) t[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) v = fmaxf(v, t[i]);
    const int p = 15 - __builtin_amdgcn_frexp_expf(v);
    *power = v == 0.f || (v >= 1.f && v <= 65504.f) ? 0 : p < 100 ? p : 100;
}

template <typename E> __global__ void __launch_bounds__(256) column_sums_kernel(ColumnSums c, bool vec) {
    __shared__ float t[4 * 64];
    column_sums<E, 4>(c, vec, blockIdx.x, blockIdx.y, gridDim.y, t);
}

}  // namespace

bool gemm_dims_ok(long long M, long long N, long long K) {
    const long long most = 1LL << 30, elements = 1LL << 40;
    return M >= 1 && N >= 1 && K >= 1 && M <= most && N <= most / 4 && K <= most / 4 && M * N <= elements && M * K <= elements && N * K <= elements &&
           ((M + kBQ - 1) / kBQ) * ((N + kBP / 2 - 1) / (kBP / 2)) <= (1LL << 24) - 8;      // a launch has less than 2^32 threads: 256 per tile
}

// one row of sums per 32 rows, per 64 rows twice, per 128 rows twice or four times, or per 256 rows four times
int gemm_most_sum_rows(int M) { return (M + 63) / 64 * 2 + 4; }

// four for a tile of 64 x 64 or more, eight for one of twice that or more
long long gemm_most_tops(int M, int N) { return 4 * (((long long)M + 63) / 64 + 1) * (((long long)N + 63) / 64 + 1); }

// How many ranges a reduction is cut into: the number with the least time by this count.  A stage of a 64x64 tile takes a workgroup 0.29 us where it waits
// for its operands (two-byte types, up to 768 workgroups side by side: 512 x 5120 x 1280, 160 tiles, 23 us) and 0.49 us of a compute unit's MFMAs for
// fp32, where what counts is how evenly the tiles fill the units (2028 x 2560 x 640, 320 tiles: one range 88 us, four 70).  A join is 5 us and the
// ranges' sums written and read.  Two-byte products with enough tiles of 128x128 are not cut at all.  The ranges together may reach a larger block (launch_shape), which is
// only faster.  us, one range / as counted / as counted in 64x64 (M x K x N, fp16): 90 x 5120 x 320 22.5 / 9.0 / 9.0, 256 x 2560 x 1280 13.2 / 12.3 / 12.0, 512 x 10240 x 1280
// 42.6 / 27.8 / 34.8, 1000 x 5120 x 1280 32.0 / 30.2 / 32.8; odd 90 x 2563 x 320 41.6 / 18.7, 1000 x 5123 x 1280 85.8 / 58.9; fp32 2028 x 2560 x 320 52.0 / 38.5.
// The gated product is not cut: few tiles of it wait 6 us per 1000 of the reduction (64 x 5120 x 2 x 1280 33 us).
int gemm_ranges(int M, int N, int K, int dt) {
    auto tiles = [&](int n, int m) { return (((long long)N + n - 1) / n) * (((long long)M + m - 1) / m); };
    const bool f32 = dt == DT_F32;
    if (!f32 && tiles(128, 128) >= 130) return 1;
    const long long t64 = tiles(64, 64);
    const int stages = (K + (f32 ? 31 : 63)) / (f32 ? 32 : 64);
    int best = 1;
    double least = 0.;
    for (int n = 1; n <= 16 && (n == 1 || stages / n >= 8); ++n) {
        const double wide = (double)(t64 * n) / 768.;
        const double us = (f32 ? 0.49 * (double)((t64 * n + 255) / 256) : 0.29 * (wide > 1. ? wide : 1.)) * ((stages + n - 1) / n) +
                          (n == 1 ? 0. : 5. + (double)n * M * N * 8. / 4e6);
        if (n == 1 || us < least) { best = n; least = us; }
    }
    return best;
}

hipError_t launch_gemm(int ep, bool p_trans, bool q_trans, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, int dt, hipStream_t s,
                       Filled* filled) {
    if (tile_gemm_ok(ep, p_trans, q_trans, P, Q, g, e, dt)) return launch_tile_gemm(ep, p_trans, q_trans, P, Q, g, e, nsplit, dt, s, filled);
    if (filled) {
        const int bn = ep == EP_DGLU ? kBP / 2 : kBP;
        filled->sum_rows = (g.M + kBQ - 1) / kBQ * 2;
        filled->tops = 4LL * ((g.M + kBQ - 1) / kBQ) * ((g.N + bn - 1) / bn);
    }
    return with_dtype(dt, [&](auto* tag) -> hipError_t {
        using E = std::remove_pointer_t<decltype(tag)>;
        switch (ep) {
            case EP_STORE: return with_layout<E, EP_STORE>(p_trans, q_trans, P, Q, g, e, 1, s);
            case EP_PART: return with_layout<E, EP_PART>(p_trans, q_trans, P, Q, g, e, nsplit, s);
            case EP_LINEAR: return with_act<E, EP_LINEAR>(P, Q, g, e, s);
            case EP_DLINEAR: return with_act<E, EP_DLINEAR>(P, Q, g, e, s);
            case EP_GLU: return with_act<E, EP_GLU>(P, Q, g, e, s);
            case EP_DGLU: return with_act<E, EP_DGLU>(P, Q, g, e, s);
            default: return hipErrorInvalidValue;
        }
    });
}

hipError_t launch_gemm_pair(const Product& a, const Product& b, const ColumnSums& c, int dt, hipStream_t s) {
    const int ea = a.e.part ? EP_PART : EP_STORE, eb = b.e.part ? EP_PART : EP_STORE;
    if (tile_gemm_ok(ea, true, false, a.P, a.Q, a.g, a.e, dt) && tile_gemm_ok(eb, true, true, b.P, b.Q, b.g, b.e, dt)) return launch_tile_pair(a, b, c, dt, s);
    hipError_t rc = c.out ? launch_column_sums(c, dt, s) : hipSuccess;
    if (rc == hipSuccess) rc = launch_gemm(ea, true, false, a.P, a.Q, a.g, a.e, a.nsplit, dt, s);
    return rc != hipSuccess ? rc : launch_gemm(eb, true, true, b.P, b.Q, b.g, b.e, b.nsplit, dt, s);
}

hipError_t launch_join(const float* part, int nsplit, const GemmShape& g, const Epilogue& e, int dt, hipStream_t s) {
    const long long blocks = ((long long)((g.N + 3) / 4) * g.M + 255) / 256;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    return with_dtype(dt, [&](auto* tag) -> hipError_t {
        using E = std::remove_pointer_t<decltype(tag)>;
        const bool linear = e.bias || e.extra || e.act != ACT_NONE;
        const dim3 grid((unsigned)blocks);
        switch (e.act) {
            case ACT_NONE: hipLaunchKernelGGL((join_kernel<E, ACT_NONE>), grid, dim3(256), 0, s, part, nsplit, g, e, linear); break;
            case ACT_SILU: hipLaunchKernelGGL((join_kernel<E, ACT_SILU>), grid, dim3(256), 0, s, part, nsplit, g, e, linear); break;
            case ACT_GELU: hipLaunchKernelGGL((join_kernel<E, ACT_GELU>), grid, dim3(256), 0, s, part, nsplit, g, e, linear); break;
            default: hipLaunchKernelGGL((join_kernel<E, ACT_GELU_TANH>), grid, dim3(256), 0, s, part, nsplit, g, e, linear); break;
        }
        return hipGetLastError();
    });
}

hipError_t launch_sum_rows(const float* part, int rows, int cols, float* out, hipStream_t s) {
    hipLaunchKernelGGL(sum_rows_kernel, dim3((unsigned)((cols + 63) / 64)), dim3(1024), 0, s, part, rows, cols, out);
    return hipGetLastError();
}

hipError_t launch_power(const float* tops, long long n, int* power, hipStream_t s) {
    hipLaunchKernelGGL(power_kernel, dim3(1), dim3(1024), 0, s, tops, n, power);
    return hipGetLastError();
}

int column_sum_rows(int M) { return M <= 1024 ? 1 : M < 256 * 64 ? M / 256 : 64; }

hipError_t launch_column_sums(const ColumnSums& c, int dt, hipStream_t s) {
    if (c.f32) return launch_sum_rows(static_cast<const float*>(c.x), c.M, c.N, c.out, s);
    return with_dtype(dt, [&](auto* tag) -> hipError_t {
        using E = std::remove_pointer_t<decltype(tag)>;
        hipLaunchKernelGGL((column_sums_kernel<E>), dim3((unsigned)((c.N + 63) / 64), (unsigned)c.ranges), dim3(256), 0, s, c, vec_rows<E>(Operand{c.x, c.ld}));
        return hipGetLastError();
    });
}

}  // namespace wino
