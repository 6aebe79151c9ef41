// Products with at most 64 rows of x (single tokens, time embeddings): a stream of the weights.
//
// A workgroup owns 16 columns of the result (gated: 16 of u and the same 16 of g) and all rows; its eight waves take the reduction in turn, 32 elements (fp32: 16)
// a step, as 16x16 MFMAs with the weights' rows in the tile's rows, both operands straight from memory: a load of the wave covers 64 neighbouring
// bytes of 16 weight rows.  The waves' sums meet in LDS, one thread finishes one value.  No workspace, no second kernel.
#include "linear_tile.h"

namespace wino {

namespace {

constexpr int kWaves = 8, kCols = 16;

template <typename E> __device__ __forceinline__ void mma16(const u32x4_t& a, const u32x4_t& b, f32x4_t& c) {
    if constexpr (sizeof(E) == 2) Mma16<E>::run(a, b, c);
    else {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
    }
}

// MT tiles of 16 rows of x
template <typename E, bool GLU, int MT>
__global__ void __launch_bounds__(kWaves * 64) gemm_few_kernel(Operand P, Operand Q, GemmShape g, Epilogue e) {
    constexpr int V = 16 / (int)sizeof(E), NW = GLU ? 2 : 1, U = MT * NW > 4 ? 2 : 4, TILES = MT * NW, ROW = 20;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n0 = blockIdx.x * kCols, idx = lane & 15, quarter = lane >> 4;
    const int steps = (g.K + 4 * V - 1) / (4 * V);
    const E* wrow[NW];
    const E* xrow[MT];
    bool w_on = n0 + idx < g.N, x_on[MT];
#pragma unroll
    for (int h = 0; h < NW; ++h) wrow[h] = static_cast<const E*>(P.p) + (long long)(h * g.N + (w_on ? n0 + idx : 0)) * P.ld;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        x_on[t] = t * 16 + idx < g.M;
        xrow[t] = static_cast<const E*>(Q.p) + (long long)(x_on[t] ? t * 16 + idx : 0) * Q.ld;
    }
    f32x4_t acc[MT][NW] = {};
    auto load = [&](const E* row, int k, bool on) {
        const u32x4_t zero = {0, 0, 0, 0};
        const int left = on ? g.K - k : 0;
        if (left <= 0) return zero;
        return load_part<E>(row + k, left);
    };
    // rows behind the edge repeat row 0: their sums are not stored
    const int full = g.K / (4 * V);                        // steps that need no guard
    int s = wave;
    for (; s + kWaves * (U - 1) < full; s += kWaves * U) {
        u32x4_t fw[U][NW], fx[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = (s + kWaves * u) * 4 * V + quarter * V;
#pragma unroll
            for (int h = 0; h < NW; ++h) fw[u][h] = load_part<E>(wrow[h] + k, V);
#pragma unroll
            for (int t = 0; t < MT; ++t) fx[u][t] = load_part<E>(xrow[t] + k, V);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int h = 0; h < NW; ++h) mma16<E>(fw[u][h], fx[u][t], acc[t][h]);
    }
    for (; s < steps; s += kWaves) {
        const int k = s * 4 * V + quarter * V;
        u32x4_t fw[NW], fx[MT];
#pragma unroll
        for (int h = 0; h < NW; ++h) fw[h] = load(wrow[h], k, w_on);
#pragma unroll
        for (int t = 0; t < MT; ++t) fx[t] = load(xrow[t], k, x_on[t]);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int h = 0; h < NW; ++h) mma16<E>(fw[h], fx[t], acc[t][h]);
    }
    // register r of lane l holds column 4 (l / 16) + r of row l % 16
    float* mine = reinterpret_cast<float*>(lds) + wave * (TILES * 16 * ROW);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int h = 0; h < NW; ++h) *reinterpret_cast<f32x4_t*>(mine + ((t * NW + h) * 16 + idx) * ROW + 4 * quarter) = acc[t][h];
    __syncthreads();
    for (int id = threadIdx.x; id < MT * 256; id += kWaves * 64) {
        const int m = id >> 4, c = id & 15, n = n0 + c;
        if (m >= g.M || n >= g.N) continue;
        float v[NW] = {};
#pragma unroll
        for (int h = 0; h < NW; ++h) {
            const float* at = reinterpret_cast<const float*>(lds) + (((m >> 4) * NW + h) * 16 + (m & 15)) * ROW + c;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) v[h] += at[w * (TILES * 16 * ROW)];
            if (e.bias) v[h] += e.bias[h * g.N + n];
        }
        const float z = v[NW - 1];
        float a;
        switch (e.act) {                                   // uniform
            case ACT_NONE: a = z; break;
            case ACT_SILU: a = act_only<E, ACT_SILU>(z); break;
            case ACT_GELU: a = act_only<E, ACT_GELU>(z); break;
            default: a = act_only<E, ACT_GELU_TANH>(z); break;
        }
        if constexpr (GLU) a *= v[0];
        else if (e.extra) a += to_f32<E>(static_cast<const E*>(e.extra)[m * e.ld_extra + n]);
        static_cast<E*>(e.out)[m * e.ld_out + n] = from_f32<E>(a);
    }
}

template <typename E, bool GLU, int MT> hipError_t launch_few(const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, hipStream_t s) {
    constexpr int bytes = kWaves * MT * (GLU ? 2 : 1) * 16 * 20 * 4;
    static_assert(bytes <= 160 * 1024, "LDS budget");
    auto kern = gemm_few_kernel<E, GLU, MT>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(kern, dim3((unsigned)((g.N + kCols - 1) / kCols)), dim3(kWaves * 64), bytes, s, P, Q, g, e);
    return hipGetLastError();
}

template <typename E, bool GLU> hipError_t launch_rows(const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, hipStream_t s) {
    if (g.M <= 16) return launch_few<E, GLU, 1>(P, Q, g, e, s);
    if (g.M <= 32) return launch_few<E, GLU, 2>(P, Q, g, e, s);
    return launch_few<E, GLU, 4>(P, Q, g, e, s);
}

}  // namespace

// The kernel's time grows with the rows and the reduction, and from 2560 columns on with those; the tiles' hardly does, but they have fewer workgroups, and for the
// gated product no ranges of the reduction.  us, this kernel / tiles (N x K, fp16): 1 row 320 x 1280 3.9 / 8.9, 1280 x 5120 8.7 / 9.1; 16 rows 640 x 2560 6.9 / 7.8, 1280 x
// 5120 12.2 / 9.6; 32 rows 1280 x 1280 6.0 / 8.6, 640 x 2560 9.2 / 7.9, 5120 x 1280 10.0 / 9.4; 64 rows 320 x 320 4.5 / 5.1, 1280 x 1280 8.5 / 8.7, 1280 x 5120 25.3 / 11.1;
// fp32 32 rows 1280 x 1280 9.5 / 11.6, 64 rows 15.1 / 12.0; odd reductions 64 rows 320 x 1283 19.2 / 26.4, 1280 x 5123 67 / 21.5, fp32 32 rows 1280 x 5123 28.7 / 30.0.
// Gated: 64 rows 1280 x 1280 10.2 / 11.2, 1280 x 5120 30.4 / 33.0, 5120 x 1280 17.6 / 11.9 (17 rows 10.6 / 11.7), fp32 5120 x 1280 40.4 / 49.1.
bool few_gemm_ok(bool glu, int M, int N, int K, int dt, bool tiles) {
    if (M > 64) return false;
    const bool f32 = dt == DT_F32;
    if (glu) return (long long)M * N <= (f32 ? 400000 : 164000);
    const double work = (double)M * K * (N > 2560 ? N / 2560. : 1.);
    return work <= (f32 ? (tiles ? 40960. : 163840.) : (tiles ? 65536. : 82400.));
}

hipError_t launch_few_gemm(bool glu, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int dt, hipStream_t s) {
    return with_dtype(dt, [&](auto* tag) -> hipError_t {
        using E = std::remove_pointer_t<decltype(tag)>;
        return glu ? launch_rows<E, true>(P, Q, g, e, s) : launch_rows<E, false>(P, Q, g, e, s);
    });
}

}  // namespace wino
