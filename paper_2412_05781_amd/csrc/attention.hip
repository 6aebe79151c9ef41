// Attention to keys and values of another length: o = softmax(scale q k^T) v over the valid keys of a row of the batch, one pass over the keys with
// the running maximum and sum of the softmax.
#include "attention_tile.h"

namespace wino {

namespace {

// Part of a row's result over one range of the keys: o normalised, and the base-2 logarithm of its sum.
struct AttnParts { float* o; float* lse2; };

template <typename E, int DP> __global__ void __launch_bounds__(256) attention_kernel(AttnArgs a, AttnParts parts, int row_tiles, int nsplit, int total, int per_xcd) {
    using T = AttnTile<E, DP>;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    unsigned char* tk = lds;
    unsigned char* tv = lds + T::BYTES;
    const int logical = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if (logical >= total) return;
    const int per_head = row_tiles * nsplit, bh = logical / per_head, in = logical - bh * per_head, split = in / row_tiles, tile = in - split * row_tiles;
    const int b = bh / a.Hkv, hk = bh - b * a.Hkv, G = a.H / a.Hkv;
    const AttnRows rows{a.Sq, G * a.Sq};
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int r = tile * 128 + wave * 32 + (lane & 31);
    const bool row_on = r < rows.R;

    u32x4_t fq[T::KS];
    {
        const unsigned char* qrow = row_on ? rows.at(a.q, G, b, hk, r, T::ES) : nullptr;
#pragma unroll
        for (int ks = 0; ks < T::KS; ++ks) fq[ks] = load_channels<E>(qrow, (2 * ks + half) * T::V, row_on ? a.D : 0);
    }
    const unsigned char* kbase = static_cast<const unsigned char*>(a.k.p) + ((long long)b * a.k.b + (long long)hk * a.k.h) * T::ES;
    const unsigned char* vbase = static_cast<const unsigned char*>(a.v.p) + ((long long)b * a.v.b + (long long)hk * a.v.h) * T::ES;
    const int len = key_count(a, b), tiles = (len + T::ROWS - 1) / T::ROWS;
    const int t0 = (int)((long long)split * tiles / nsplit), t1 = (int)((long long)(split + 1) * tiles / nsplit);

    u32x4_t lk[T::LOADS], lv[T::LOADS];
    auto fetch = [&](int t, unsigned long long on) {
#pragma unroll
        for (int i = 0; i < T::LOADS; ++i) {
            const int id = tid + 256 * i, row = id / T::CPR, c = (id - row * T::CPR) * T::V;
            const bool ok = row < T::ROWS && ((on >> (row & 63)) & 1);
            const long long key = (long long)t * T::ROWS + row;
            lk[i] = load_channels<E>(kbase + key * a.k.s * T::ES, c, ok ? a.D : 0);
            lv[i] = load_channels<E>(vbase + key * a.v.s * T::ES, c, ok ? a.D : 0);
        }
    };
    float16_t acc[T::NV] = {};
    float m = -INFINITY, l = 0.f;
    const float c2 = a.scale * kLog2e;
    unsigned long long next_on = t0 < t1 ? valid_keys(a, b, t0 * T::ROWS, len) : 0;
    if (t0 < t1) fetch(t0, next_on);
    for (int t = t0; t < t1; ++t) {
        const unsigned long long on = next_on;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < T::LOADS; ++i) {
            const int id = tid + 256 * i, row = id / T::CPR;
            if (row < T::ROWS) {
                const int at = T::at(row, id - row * T::CPR);
                *reinterpret_cast<u32x4_t*>(tk + at) = lk[i];
                *reinterpret_cast<u32x4_t*>(tv + at) = lv[i];
            }
        }
        __syncthreads();
        if (t + 1 < t1) {
            next_on = valid_keys(a, b, (t + 1) * T::ROWS, len);
            fetch(t + 1, next_on);
        }
        if (on == 0) continue;                             // uniform: every wave has the same keys
        float16_t s[2] = {};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int ks = 0; ks < T::KS; ++ks) Mma<E>::run(T::along(tk, 32 * i, ks, lane), fq[ks], s[i]);
        if (on != ~0ull) {
            const unsigned long long mine = on >> (4 * half);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < 16; ++q)
                    if (!((mine >> (32 * i + 8 * (q / 4) + q % 4)) & 1)) s[i][q] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int q = 1; q < 32; ++q) top = fmaxf(top, s[q / 16][q % 16]);
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m, top * c2), base = m_new == -INFINITY ? 0.f : m_new, alpha = __builtin_amdgcn_exp2f(m - base);
        m = m_new;
        float sum = 0.f;
#pragma unroll
        for (int q = 0; q < 32; ++q) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[q / 16][q % 16], c2, -base));
            s[q / 16][q % 16] = p;
            sum += p;
        }
        l = fmaf(l, alpha, sum);
#pragma unroll
        for (int d = 0; d < T::NV; ++d)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[d][q] *= alpha;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int st = 0; st < T::ST; ++st) {
                const u32x4_t w = T::weights(s[i], st);
#pragma unroll
                for (int d = 0; d < T::NV; ++d) Mma<E>::run(T::across(tv, 32 * i, st, d, lane), w, acc[d]);
            }
    }
    l += __shfl_xor(l, 32);
    if (!row_on) return;
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;           // a NaN stays one
    const float lse2 = l == 0.f ? -INFINITY : m + log2f(l);
    const long long row = (long long)bh * rows.R + r;
    if (nsplit > 1) {
        const long long all = (long long)a.B * a.Hkv * rows.R, at = (long long)split * all + row;
        if (half == 0) parts.lse2[at] = lse2;
        float* o = parts.o + at * a.D;
#pragma unroll
        for (int d = 0; d < T::NV; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = d * 32 + 8 * q + 4 * half;
                if (c < a.D) *reinterpret_cast<float4*>(o + c) = make_float4(acc[d][4 * q] * inv, acc[d][4 * q + 1] * inv, acc[d][4 * q + 2] * inv, acc[d][4 * q + 3] * inv);
            }
        return;
    }
    if (a.lse && half == 0) a.lse[row] = lse2 * kLn2;
    unsigned char* orow = const_cast<unsigned char*>(rows.at(a.o, G, b, hk, r, T::ES));
#pragma unroll
    for (int d = 0; d < T::NV; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float v[4] = {acc[d][4 * q] * inv, acc[d][4 * q + 1] * inv, acc[d][4 * q + 2] * inv, acc[d][4 * q + 3] * inv};
            store_channels<E>(orow, d * 32 + 8 * q + 4 * half, a.D, v);
        }
}

// one wave per row: the ranges' results, weighted by their sums
template <typename E> __global__ void __launch_bounds__(256) attention_join_kernel(AttnArgs a, AttnParts parts, int nsplit, long long all) {
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= all) return;
    const int lane = threadIdx.x & 63, G = a.H / a.Hkv;
    const AttnRows rows{a.Sq, G * a.Sq};
    float m = -INFINITY;
    for (int i = 0; i < nsplit; ++i) m = fmaxf(m, parts.lse2[i * all + row]);
    const float base = m == -INFINITY ? 0.f : m;
    float total = 0.f;
    for (int i = 0; i < nsplit; ++i) total += __builtin_amdgcn_exp2f(parts.lse2[i * all + row] - base);
    const float inv = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
    const int bh = (int)(row / rows.R), r = (int)(row - (long long)bh * rows.R), b = bh / a.Hkv, hk = bh - b * a.Hkv;
    E* o = reinterpret_cast<E*>(const_cast<unsigned char*>(rows.at(a.o, G, b, hk, r, (int)sizeof(E))));
    for (int c = lane; c < a.D; c += 64) {
        float v = 0.f;
        for (int i = 0; i < nsplit; ++i) v = fmaf(__builtin_amdgcn_exp2f(parts.lse2[i * all + row] - base) * inv, parts.o[(i * all + row) * a.D + c], v);
        o[c] = from_f32<E>(v);
    }
    if (a.lse && lane == 0) a.lse[row] = total == 0.f ? -INFINITY : (m + log2f(total)) * kLn2;
}

// Ranges of the keys, where the rows alone leave compute units idle: up to two workgroups a unit, at least four tiles a range.
int attention_ranges(int B, int Sq, int Skv, int H, int Hkv) {
    const long long blocks = (long long)B * Hkv * (((long long)(H / Hkv) * Sq + 127) / 128);
    const int tiles = (Skv + 63) / 64;
    long long n = 512 / blocks;
    if (n > tiles / 4) n = tiles / 4;
    if (n > 64) n = 64;
    return n < 2 ? 1 : (int)n;
}

}  // namespace

size_t attention_ws_bytes(int B, int Sq, int Skv, int H, int Hkv, int D, int) {
    const int n = attention_ranges(B, Sq, Skv, H, Hkv);
    return n == 1 ? 0 : (size_t)n * B * H * Sq * ((size_t)D + 1) * sizeof(float);
}

hipError_t launch_attention(const AttnArgs& a, int dt, hipStream_t s) {
    const int R = a.H / a.Hkv * a.Sq, nsplit = attention_ranges(a.B, a.Sq, a.Skv, a.H, a.Hkv), row_tiles = (R + 127) / 128;
    const long long all = (long long)a.B * a.Hkv * R, total = (long long)a.B * a.Hkv * row_tiles * nsplit;
    if (total > 0x3fffffffLL || (all + 3) / 4 > 0x7fffffffLL) return hipErrorInvalidValue;
    const int per_xcd = (int)((total + 7) / 8);
    AttnParts parts{nullptr, nullptr};
    if (nsplit > 1) { parts.o = a.ws; parts.lse2 = a.ws + (size_t)nsplit * all * a.D; }
    return with_dtype(dt, [&](auto* tag) -> hipError_t {
        using E = std::remove_pointer_t<decltype(tag)>;
        const hipError_t rc = with_channels(a.D, [&](auto dp) -> hipError_t {
            constexpr int DP = decltype(dp)::value;
            if constexpr (sizeof(E) == 4 && DP > 10) return hipErrorInvalidValue;
            else {
                using T = AttnTile<E, DP>;
                auto kern = attention_kernel<E, DP>;
                constexpr int bytes = 2 * T::BYTES;
                static_assert(bytes <= 160 * 1024, "LDS budget");
                static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
                if (attr != hipSuccess) return attr;
                hipLaunchKernelGGL(kern, dim3((unsigned)(per_xcd * 8)), dim3(256), bytes, s, a, parts, row_tiles, nsplit, (int)total, per_xcd);
                return hipGetLastError();
            }
        });
        if (rc != hipSuccess || nsplit == 1) return rc;
        hipLaunchKernelGGL((attention_join_kernel<E>), dim3((unsigned)((all + 3) / 4)), dim3(256), 0, s, a, parts, nsplit, all);
        return hipGetLastError();
    });
}

}  // namespace wino
