// Pieces shared by the matrix kernels of the transformer-block operators: LDS tiles and the MFMA fragments read from them, row accesses.
#pragma once
#include "block_act.h"
#include "wino_mma.h"

namespace wino {

// ---- LDS tiles ------------------------------------------------------------------------------------------------------------------------
// Operand along k: rows of 128 bytes, chunk c of row r at c ^ ((r >> 1) & 7).  Operand across k: one row of BI elements per k, chunk c of row r at
// c ^ swz(r), such that the four rows that a transposing read takes (two-byte types) or the two rows that the halves of a wave take (fp32) lie
// in different banks.
template <typename E, int BI> __device__ __forceinline__ int swz_across(int r) {
    if constexpr (sizeof(E) == 4) return ((r >> 2) & 1) << 3;
    return BI == 64 ? ((r >> 1) & 1) << 2 : (r & 3) << 2;           // 64 elements: neighbouring rows lie 128 bytes apart already
}

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// the 16 bytes that lane `lane` gives to one 32x32 MFMA step: index i0 + lane % 32, reduction elements of step ks
template <typename E, bool ACROSS, int BI> __device__ __forceinline__ u32x4_t read_fragment(const unsigned char* tile, int i0, int ks, int lane) {
    const int half = lane >> 5;
    if constexpr (!ACROSS) {
        const int row = i0 + (lane & 31), chunk = (2 * ks + half) ^ ((row >> 1) & 7);
        return *reinterpret_cast<const u32x4_t*>(tile + row * 128 + chunk * 16);
    } else if constexpr (sizeof(E) == 2) {
        // four rows k x 16 columns per 16 lanes and read; lane i of the 16 gets column i
        const int col = i0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
        u32x4_t f;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int row = 16 * ks + 8 * half + 4 * t + ((lane & 15) >> 2);
            const unsigned char* at = tile + row * (BI * 2) + (((col >> 3) ^ swz_across<E, BI>(row)) << 4) + ((col & 4) << 1);
            const s16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)at);
            const uint2 w = __builtin_bit_cast(uint2, v);
            f[2 * t] = w.x;
            f[2 * t + 1] = w.y;
        }
        return f;
    } else {
        const int col = i0 + (lane & 31);
        u32x4_t f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = 8 * ks + 4 * half + j;
            f[j] = *reinterpret_cast<const uint32_t*>(tile + row * (BI * 4) + (((col >> 2) ^ swz_across<E, BI>(row)) << 4) + ((col & 3) << 2));
        }
        return f;
    }
}

// n elements (up to 16 bytes) from p, the rest zero.  Whole chunks are one load at any alignment of the elements.
template <typename E> __device__ __forceinline__ u32x4_t load_part(const E* p, int n) {
    u32x4_t f = {0, 0, 0, 0};
    constexpr int V = 16 / (int)sizeof(E);
    if (n >= V) {
        __builtin_memcpy(&f, p, 16);
        return f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (i < n) {
            if constexpr (sizeof(E) == 4) f[i] = *reinterpret_cast<const uint32_t*>(p + i);
            else f[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p + i) << (16 * (i & 1));
        }
    }
    return f;
}

// four neighbouring elements of a row, one access at any alignment of the elements
template <typename E> __device__ __forceinline__ void load4(const E* p, int n, float* v) {
    if (n >= 4) {
        if constexpr (sizeof(E) == 4) {
            __builtin_memcpy(v, p, 16);
        } else {
            uint2 f;
            __builtin_memcpy(&f, p, 8);
            v[0] = lo16<E>(f.x); v[1] = hi16<E>(f.x); v[2] = lo16<E>(f.y); v[3] = hi16<E>(f.y);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? to_f32<E>(p[i]) : 0.f;
}
template <typename E> __device__ __forceinline__ void store4(E* p, int n, const float* v) {
    if (n >= 4) {
        if constexpr (sizeof(E) == 4) {
            __builtin_memcpy(p, v, 16);
        } else {
            const uint2 f = make_uint2(pack_pair<E>(v[0], v[1]), pack_pair<E>(v[2], v[3]));
            __builtin_memcpy(p, &f, 8);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < n) p[i] = from_f32<E>(v[i]);
}

// ---- fp16's range, for the gradients of the pre-activations -----------------------------------------------------------------------------
// They are stored in between two products, where a factor can be far from one (a scaled loss, or none) and the results still fit.  The first launch finds their
// largest; only where that is below 1 or beyond 65504 are they formed again, times a power of two that the products take back.  The two launches more, a sum
// of the largest and one that ends at once, cost 4 to 7 us: 4096 x 640 x 2560 gated 115 to 123, 616 x 2048 x 1280 linear 27.6 to 32.6.
__device__ __forceinline__ float larger_finite(float top, float v) { return fabsf(v) < INFINITY ? fmaxf(top, fabsf(v)) : top; }
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ void store_top(const Epilogue& e, long long at, float top, int lane) {
    if (!e.tops) return;                                   // uniform
    top = wave_max(top);
    if (lane == 0) e.tops[at] = top;
}
// what a stored value is multiplied by; INTO: the gradients themselves, 0 where they stand already
template <typename E, bool INTO> __device__ __forceinline__ float store_factor(const Epilogue& e) {
    if constexpr (std::is_same_v<E, __half>) {
        if (e.power) {
            const int p = *e.power;
            return INTO ? (p ? __builtin_amdgcn_ldexpf(1.f, p) : 0.f) : __builtin_amdgcn_ldexpf(1.f, -p);
        }
    }
    return 1.f;
}

template <typename E> inline bool vec_rows(const Operand& o) {
    return ((reinterpret_cast<uintptr_t>(o.p) | (uintptr_t)(o.ld * (long long)sizeof(E))) & 15u) == 0;
}

// the launch of a call that tile_gemm_ok lets through
hipError_t launch_tile_gemm(int ep, bool pa, bool qa, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit, int dt, hipStream_t s, Filled* filled);

// two products in one launch: a with P across and Q along the reduction, b with both across; and the column sums, where c.out is set
hipError_t launch_tile_pair(const Product& a, const Product& b, const ColumnSums& c, int dt, hipStream_t s);

// Column sums of 64 columns x one of `ranges` ranges of rows by a workgroup of NW waves; eight lanes a row, eight rows a wave at a time.  t: 64 NW floats in LDS.
template <typename E, int NW> __device__ __forceinline__ void column_sums(const ColumnSums& c, bool vec, int block, int range, int ranges, float* t) {
    const E* x = static_cast<const E*>(c.x);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c0 = block * 64 + (lane & 7) * 8, left = c.N - c0;
    const long long r0 = (long long)range * c.M / ranges, r1 = (long long)(range + 1) * c.M / ranges;
    float a[8] = {};
    if (vec && left >= 8) {
#pragma unroll 4
        for (long long r = r0 + w * 8 + (lane >> 3); r < r1; r += 8 * NW) {
            const E* p = x + r * c.ld + c0;
            if constexpr (sizeof(E) == 4) {
                const float4 u = reinterpret_cast<const float4*>(p)[0], v = reinterpret_cast<const float4*>(p)[1];
                a[0] += u.x; a[1] += u.y; a[2] += u.z; a[3] += u.w; a[4] += v.x; a[5] += v.y; a[6] += v.z; a[7] += v.w;
            } else {
                const uint4 u = *reinterpret_cast<const uint4*>(p);
                a[0] += lo16<E>(u.x); a[1] += hi16<E>(u.x); a[2] += lo16<E>(u.y); a[3] += hi16<E>(u.y);
                a[4] += lo16<E>(u.z); a[5] += hi16<E>(u.z); a[6] += lo16<E>(u.w); a[7] += hi16<E>(u.w);
            }
        }
    } else {
        for (long long r = r0 + w * 8 + (lane >> 3); r < r1; r += 8 * NW)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) a[i] += to_f32<E>(x[r * c.ld + c0 + i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int d = 8; d < 64; d <<= 1) a[i] += __shfl_xor(a[i], d);
        if (lane < 8) t[w * 64 + lane * 8 + i] = a[i];
    }
    __syncthreads();
    const int col = block * 64 + threadIdx.x;
    if (threadIdx.x < 64 && col < c.N) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) v += t[i * 64 + threadIdx.x];
        c.out[(size_t)range * c.N + col] = v;
    }
}

}  // namespace wino
