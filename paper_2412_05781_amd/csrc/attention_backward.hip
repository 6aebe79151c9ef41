// Gradients of attention.  With p = exp(s - lse) from the forward pass and D_i = do_i . o_i:
//   dv = p^T do,  ds = p (do v^T - D),  dq = scale ds k,  dk = scale ds^T q.
// Scores are made again, never stored.  Two kernels, both without atomics, so that results do not depend on the order of the workgroups: one owns
// 128 query rows and streams the keys (dq), one owns 128 keys and streams the query rows of their head (dk, dv; over ranges of the rows, joined in
// order, where there are few keys).
#include "attention_tile.h"

namespace wino {

namespace {

struct BackwardParts {
    float* delta;                    // [B][Hkv][R]
    float* dk;                       // [nsplit][B][Hkv][Skv][D], both null with one range
    float* dv;
};

// D_i = do_i . o_i, sixteen lanes a row
template <typename E> __global__ void __launch_bounds__(256) attention_delta_kernel(AttnArgs a, float* delta, long long all) {
    const long long row = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int lane = threadIdx.x & 15, G = a.H / a.Hkv;
    if (row >= all) return;                                // whole groups of sixteen lanes leave together
    const AttnRows rows{a.Sq, G * a.Sq};
    const int bh = (int)(row / rows.R), r = (int)(row - (long long)bh * rows.R), b = bh / a.Hkv, hk = bh - b * a.Hkv;
    const unsigned char* o = rows.at(a.o, G, b, hk, r, (int)sizeof(E));
    const unsigned char* d = rows.at(a.dout, G, b, hk, r, (int)sizeof(E));
    constexpr int V = 16 / (int)sizeof(E);
    float t = 0.f;
    for (int c = lane * V; c < a.D; c += 16 * V) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(o + c * (int)sizeof(E)), y = *reinterpret_cast<const u32x4_t*>(d + c * (int)sizeof(E));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(E) == 4) t = fmaf(__uint_as_float(x[i]), __uint_as_float(y[i]), t);
            else { t = fmaf(lo16<E>(x[i]), lo16<E>(y[i]), t); t = fmaf(hi16<E>(x[i]), hi16<E>(y[i]), t); }
        }
    }
#pragma unroll
    for (int k = 8; k; k >>= 1) t += __shfl_xor(t, k, 16);
    if (lane == 0) delta[row] = t;
}

template <typename E, int DP> __global__ void __launch_bounds__(256) attention_dq_kernel(AttnArgs a, const float* delta, int row_tiles, int total, int per_xcd) {
    using T = AttnTile<E, DP>;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    unsigned char* tk = lds;
    unsigned char* tv = lds + T::BYTES;
    const int logical = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if (logical >= total) return;
    const int bh = logical / row_tiles, tile = logical - bh * row_tiles, b = bh / a.Hkv, hk = bh - b * a.Hkv, G = a.H / a.Hkv;
    const AttnRows rows{a.Sq, G * a.Sq};
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int r = tile * 128 + wave * 32 + (lane & 31);
    const bool row_on = r < rows.R;
    u32x4_t fq[T::KS], fo[T::KS];
    {
        const unsigned char* qrow = row_on ? rows.at(a.q, G, b, hk, r, T::ES) : nullptr;
        const unsigned char* orow = row_on ? rows.at(a.dout, G, b, hk, r, T::ES) : nullptr;
#pragma unroll
        for (int ks = 0; ks < T::KS; ++ks) {
            fq[ks] = load_channels<E>(qrow, (2 * ks + half) * T::V, row_on ? a.D : 0);
            fo[ks] = load_channels<E>(orow, (2 * ks + half) * T::V, row_on ? a.D : 0);
        }
    }
    const long long row = (long long)bh * rows.R + r;
    const float lse2 = row_on ? a.lse[row] * kLog2e : 0.f, dlt = row_on ? delta[row] : 0.f;
    const unsigned char* kbase = static_cast<const unsigned char*>(a.k.p) + ((long long)b * a.k.b + (long long)hk * a.k.h) * T::ES;
    const unsigned char* vbase = static_cast<const unsigned char*>(a.v.p) + ((long long)b * a.v.b + (long long)hk * a.v.h) * T::ES;
    const int len = key_count(a, b), tiles = (len + T::ROWS - 1) / T::ROWS;
    float16_t acc[T::NV] = {};
    const float c2 = a.scale * kLog2e;
    for (int t = 0; t < tiles; ++t) {
        const unsigned long long on = valid_keys(a, b, t * T::ROWS, len);
        if (on == 0) continue;                             // uniform
        __syncthreads();
#pragma unroll
        for (int i = 0; i < T::LOADS; ++i) {
            const int id = tid + 256 * i, kr = id / T::CPR, ch = id - kr * T::CPR;
            if (kr < T::ROWS) {
                const bool ok = (on >> kr) & 1;
                const long long key = (long long)t * T::ROWS + kr;
                *reinterpret_cast<u32x4_t*>(tk + T::at(kr, ch)) = load_channels<E>(kbase + key * a.k.s * T::ES, ch * T::V, ok ? a.D : 0);
                *reinterpret_cast<u32x4_t*>(tv + T::at(kr, ch)) = load_channels<E>(vbase + key * a.v.s * T::ES, ch * T::V, ok ? a.D : 0);
            }
        }
        __syncthreads();
        const unsigned long long mine = on >> (4 * half);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float16_t s = {}, dp = {};
#pragma unroll
            for (int ks = 0; ks < T::KS; ++ks) {
                Mma<E>::run(T::along(tk, 32 * i, ks, lane), fq[ks], s);
                Mma<E>::run(T::along(tv, 32 * i, ks, lane), fo[ks], dp);
            }
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const bool ok = (mine >> (32 * i + 8 * (q / 4) + q % 4)) & 1;
                const float p = __builtin_amdgcn_exp2f(fmaf(s[q], c2, -lse2));
                s[q] = ok ? p * (dp[q] - dlt) : 0.f;
            }
#pragma unroll
            for (int st = 0; st < T::ST; ++st) {
                const u32x4_t w = T::weights(s, st);
#pragma unroll
                for (int d = 0; d < T::NV; ++d) Mma<E>::run(T::across(tk, 32 * i, st, d, lane), w, acc[d]);
            }
        }
    }
    if (!row_on) return;
    unsigned char* out = const_cast<unsigned char*>(rows.at(a.dq, G, b, hk, r, T::ES));
#pragma unroll
    for (int d = 0; d < T::NV; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float v[4] = {acc[d][4 * q] * a.scale, acc[d][4 * q + 1] * a.scale, acc[d][4 * q + 2] * a.scale, acc[d][4 * q + 3] * a.scale};
            store_channels<E>(out, d * 32 + 8 * q + 4 * half, a.D, v);
        }
}

template <typename E, int DP> __global__ void __launch_bounds__(256) attention_dkv_kernel(AttnArgs a, BackwardParts parts, int key_tiles, int nsplit, int total, int per_xcd) {
    using T = AttnTile<E, DP>;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    unsigned char* tq = lds;
    unsigned char* to = lds + T::BYTES;
    float* tl = reinterpret_cast<float*>(lds + 2 * T::BYTES);          // lse and delta of the tile's rows
    float* td = tl + T::ROWS;
    const int logical = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if (logical >= total) return;
    const int per_head = key_tiles * nsplit, bh = logical / per_head, in = logical - bh * per_head, split = in / key_tiles, tile = in - split * key_tiles;
    const int b = bh / a.Hkv, hk = bh - b * a.Hkv, G = a.H / a.Hkv;
    const AttnRows rows{a.Sq, G * a.Sq};
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int len = key_count(a, b), key = tile * 128 + wave * 32 + (lane & 31);
    const bool in_range = key < a.Skv, key_on = key < len && (!a.key_mask || a.key_mask[(long long)b * a.Skv + key] != 0);
    float16_t adk[T::NV] = {}, adv[T::NV] = {};
    // a tile of keys that no query may look at has nothing to sum (uniform over the workgroup)
    if (__syncthreads_or(key_on)) {
        u32x4_t fk[T::KS], fv[T::KS];
        {
            const unsigned char* krow = static_cast<const unsigned char*>(a.k.p) + ((long long)b * a.k.b + (long long)hk * a.k.h + (long long)(key_on ? key : 0) * a.k.s) * T::ES;
            const unsigned char* vrow = static_cast<const unsigned char*>(a.v.p) + ((long long)b * a.v.b + (long long)hk * a.v.h + (long long)(key_on ? key : 0) * a.v.s) * T::ES;
#pragma unroll
            for (int ks = 0; ks < T::KS; ++ks) {
                fk[ks] = load_channels<E>(krow, (2 * ks + half) * T::V, key_on ? a.D : 0);
                fv[ks] = load_channels<E>(vrow, (2 * ks + half) * T::V, key_on ? a.D : 0);
            }
        }
        const int tiles = (rows.R + T::ROWS - 1) / T::ROWS;
        const int t0 = (int)((long long)split * tiles / nsplit), t1 = (int)((long long)(split + 1) * tiles / nsplit);
        const float c2 = a.scale * kLog2e;
        for (int t = t0; t < t1; ++t) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < T::LOADS; ++i) {
                const int id = tid + 256 * i, qr = id / T::CPR, ch = id - qr * T::CPR;
                if (qr < T::ROWS) {
                    const int r = t * T::ROWS + qr;
                    const bool ok = r < rows.R;
                    *reinterpret_cast<u32x4_t*>(tq + T::at(qr, ch)) = load_channels<E>(ok ? rows.at(a.q, G, b, hk, r, T::ES) : nullptr, ch * T::V, ok ? a.D : 0);
                    *reinterpret_cast<u32x4_t*>(to + T::at(qr, ch)) = load_channels<E>(ok ? rows.at(a.dout, G, b, hk, r, T::ES) : nullptr, ch * T::V, ok ? a.D : 0);
                }
            }
            if (tid < T::ROWS) {
                const int r = t * T::ROWS + tid;
                const bool ok = r < rows.R;
                tl[tid] = ok ? a.lse[(long long)bh * rows.R + r] * kLog2e : INFINITY;      // a row behind the last: p = 0
                td[tid] = ok ? parts.delta[(long long)bh * rows.R + r] : 0.f;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float16_t s = {}, dp = {};
#pragma unroll
                for (int ks = 0; ks < T::KS; ++ks) {
                    Mma<E>::run(T::along(tq, 32 * i, ks, lane), fk[ks], s);
                    Mma<E>::run(T::along(to, 32 * i, ks, lane), fv[ks], dp);
                }
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const int qr = 32 * i + 8 * (q / 4) + 4 * half + q % 4;
                    const float p = key_on ? __builtin_amdgcn_exp2f(fmaf(s[q], c2, -tl[qr])) : 0.f;
                    s[q] = p;
                    dp[q] = key_on ? p * (dp[q] - td[qr]) : 0.f;
                }
#pragma unroll
                for (int st = 0; st < T::ST; ++st) {
                    const u32x4_t wp = T::weights(s, st), wd = T::weights(dp, st);
#pragma unroll
                    for (int d = 0; d < T::NV; ++d) {
                        Mma<E>::run(T::across(to, 32 * i, st, d, lane), wp, adv[d]);
                        Mma<E>::run(T::across(tq, 32 * i, st, d, lane), wd, adk[d]);
                    }
                }
            }
        }
    }
    if (!in_range) return;
    if (nsplit > 1) {
        const long long at = (((long long)split * a.B * a.Hkv + bh) * a.Skv + key) * a.D;
#pragma unroll
        for (int d = 0; d < T::NV; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = d * 32 + 8 * q + 4 * half;
                if (c < a.D) {
                    *reinterpret_cast<float4*>(parts.dk + at + c) = make_float4(adk[d][4 * q], adk[d][4 * q + 1], adk[d][4 * q + 2], adk[d][4 * q + 3]);
                    *reinterpret_cast<float4*>(parts.dv + at + c) = make_float4(adv[d][4 * q], adv[d][4 * q + 1], adv[d][4 * q + 2], adv[d][4 * q + 3]);
                }
            }
        return;
    }
    unsigned char* dk = static_cast<unsigned char*>(const_cast<void*>(a.dk.p)) + ((long long)b * a.dk.b + (long long)hk * a.dk.h + (long long)key * a.dk.s) * T::ES;
    unsigned char* dv = static_cast<unsigned char*>(const_cast<void*>(a.dv.p)) + ((long long)b * a.dv.b + (long long)hk * a.dv.h + (long long)key * a.dv.s) * T::ES;
#pragma unroll
    for (int d = 0; d < T::NV; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = d * 32 + 8 * q + 4 * half;
            const float x[4] = {adk[d][4 * q] * a.scale, adk[d][4 * q + 1] * a.scale, adk[d][4 * q + 2] * a.scale, adk[d][4 * q + 3] * a.scale};
            const float y[4] = {adv[d][4 * q], adv[d][4 * q + 1], adv[d][4 * q + 2], adv[d][4 * q + 3]};
            store_channels<E>(dk, c, a.D, x);
            store_channels<E>(dv, c, a.D, y);
        }
}

// the ranges' sums, four channels a thread
template <typename E> __global__ void __launch_bounds__(256) attention_dkv_join_kernel(AttnArgs a, BackwardParts parts, int nsplit) {
    const long long quads = a.D / 4, each = (long long)a.B * a.Hkv * a.Skv * quads, id = (long long)blockIdx.x * 256 + threadIdx.x;
    if (id >= each) return;
    const long long row = id / quads;
    const int c = (int)(id - row * quads) * 4;
    const long long bh = row / a.Skv;
    const int key = (int)(row - bh * a.Skv), b = (int)(bh / a.Hkv), hk = (int)(bh - (long long)b * a.Hkv);
    float x[4] = {}, y[4] = {};
    for (int i = 0; i < nsplit; ++i) {
        const long long at = (i * (each / quads) + row) * a.D + c;
        const float4 u = *reinterpret_cast<const float4*>(parts.dk + at), v = *reinterpret_cast<const float4*>(parts.dv + at);
        x[0] += u.x; x[1] += u.y; x[2] += u.z; x[3] += u.w;
        y[0] += v.x; y[1] += v.y; y[2] += v.z; y[3] += v.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= a.scale;
    constexpr int ES = (int)sizeof(E);
    store_channels<E>(static_cast<unsigned char*>(const_cast<void*>(a.dk.p)) + ((long long)b * a.dk.b + (long long)hk * a.dk.h + (long long)key * a.dk.s) * ES, c, a.D, x);
    store_channels<E>(static_cast<unsigned char*>(const_cast<void*>(a.dv.p)) + ((long long)b * a.dv.b + (long long)hk * a.dv.h + (long long)key * a.dv.s) * ES, c, a.D, y);
}

// Ranges of the query rows, where the keys alone leave compute units idle: about two workgroups a unit, at least four tiles of rows a range.
int backward_ranges(int B, int Sq, int Skv, int H, int Hkv) {
    const long long blocks = (long long)B * Hkv * (((long long)Skv + 127) / 128);
    const long long tiles = ((long long)(H / Hkv) * Sq + 63) / 64;
    long long n = 512 / blocks;
    if (n > tiles / 4) n = tiles / 4;
    if (n > 16) n = 16;
    return n < 2 ? 1 : (int)n;
}
size_t align_floats(size_t n) { return (n + 63) / 64 * 64; }

}  // namespace

size_t attention_backward_ws_bytes(int B, int Sq, int Skv, int H, int Hkv, int D, int) {
    const int n = backward_ranges(B, Sq, Skv, H, Hkv);
    return (align_floats((size_t)B * H * Sq) + (n == 1 ? 0 : 2 * (size_t)n * B * Hkv * Skv * D)) * sizeof(float);
}

hipError_t launch_attention_backward(const AttnArgs& a, int dt, hipStream_t s) {
    const int R = a.H / a.Hkv * a.Sq, nsplit = backward_ranges(a.B, a.Sq, a.Skv, a.H, a.Hkv);
    const int row_tiles = (R + 127) / 128, key_tiles = (a.Skv + 127) / 128;
    const long long all = (long long)a.B * a.Hkv * R, qt = (long long)a.B * a.Hkv * row_tiles, kt = (long long)a.B * a.Hkv * key_tiles * nsplit;
    const long long joins = ((long long)a.B * a.Hkv * a.Skv * (a.D / 4) + 255) / 256;
    if (qt > 0x3fffffffLL || kt > 0x3fffffffLL || (all + 15) / 16 > 0x7fffffffLL || joins > 0x7fffffffLL) return hipErrorInvalidValue;
    BackwardParts parts{a.ws, nullptr, nullptr};
    if (nsplit > 1) {
        parts.dk = a.ws + align_floats((size_t)all);
        parts.dv = parts.dk + (size_t)nsplit * a.B * a.Hkv * a.Skv * a.D;
    }
    return with_dtype(dt, [&](auto* tag) -> hipError_t {
        using E = std::remove_pointer_t<decltype(tag)>;
        hipLaunchKernelGGL((attention_delta_kernel<E>), dim3((unsigned)((all + 15) / 16)), dim3(256), 0, s, a, parts.delta, all);
        hipError_t rc = hipGetLastError();
        if (rc != hipSuccess) return rc;
        rc = with_channels(a.D, [&](auto dp) -> hipError_t {
            constexpr int DP = decltype(dp)::value;
            if constexpr (sizeof(E) == 4 && DP > 10) return hipErrorInvalidValue;
            else {
                using T = AttnTile<E, DP>;
                constexpr int bytes = 2 * T::BYTES + 2 * T::ROWS * (int)sizeof(float);
                static_assert(bytes <= 160 * 1024, "LDS budget");
                auto kq = attention_dq_kernel<E, DP>;
                auto kk = attention_dkv_kernel<E, DP>;
                static const hipError_t attr_q = hipFuncSetAttribute(reinterpret_cast<const void*>(kq), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
                static const hipError_t attr_k = hipFuncSetAttribute(reinterpret_cast<const void*>(kk), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
                if (attr_q != hipSuccess || attr_k != hipSuccess) return hipErrorInvalidValue;
                const int pq = (int)((qt + 7) / 8), pk = (int)((kt + 7) / 8);
                hipLaunchKernelGGL(kq, dim3((unsigned)(pq * 8)), dim3(256), bytes, s, a, (const float*)parts.delta, row_tiles, (int)qt, pq);
                hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
                hipLaunchKernelGGL(kk, dim3((unsigned)(pk * 8)), dim3(256), bytes, s, a, parts, key_tiles, nsplit, (int)kt, pk);
                return hipGetLastError();
            }
        });
        if (rc != hipSuccess || nsplit == 1) return rc;
        hipLaunchKernelGGL((attention_dkv_join_kernel<E>), dim3((unsigned)joins), dim3(256), 0, s, a, parts, nsplit);
        return hipGetLastError();
    });
}

}  // namespace wino
