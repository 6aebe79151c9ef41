// Attention to keys and values of another length: o = softmax(scale q k^T) v over the valid keys of a row of the batch, one pass over the keys with
// the running maximum and sum of the softmax.
#include "attention_tile.h"

namespace wino {

namespace {

// Part of a row's result over one range of the keys: o normalised, and the base-2 logarithm of its sum.
struct AttnParts { float* o; float* lse2; };

// Running state of a wave's 32 rows, one per lane and half: the maximum is not followed exactly.  Weights are taken relative to `base`, a multiple of the
// scores in base 2 that lags behind the true maximum by up to 8: weights stay below 256, far from every type's end, and the sums are rescaled once
// in many tiles instead of in each.  The result does not depend on base but for rounding.
template <typename E, int DP> struct AttnState {
    using T = AttnTile<E, DP>;
    float16_t acc[T::NV] = {};
    float base = -INFINITY, l = 0.f;

    // takes the scores of 32 * SUBS streamed keys (raw; valid keys in the bits of `on`, uniform over the wave) into account for the base
    template <int SUBS> __device__ __forceinline__ void settle(float16_t (&s)[SUBS], unsigned long long on, int half, float c2) {
        if (on != (SUBS == 2 ? ~0ull : 0xffffffffull)) {
            asm volatile("" ::: "memory");                 // keeps this a branch: as selects it costs every tile as much as the exponentials
            const unsigned long long mine = on >> (4 * half);
#pragma unroll
            for (int q = 0; q < 16 * SUBS; ++q)
                if (!((mine >> (32 * (q / 16) + 8 * ((q % 16) / 4) + q % 4)) & 1)) s[q / 16][q % 16] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int q = 1; q < 16 * SUBS; ++q) top = fmaxf(top, s[q / 16][q % 16]);
        top *= c2;
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > base + 8.f)) {                     // rows without a key so far: base is -infinity
            const float next = fmaxf(top, base), f = base == next ? 1.f : __builtin_amdgcn_exp2f(base - next);
            base = next;
            l *= f;
#pragma unroll
            for (int d = 0; d < T::NV; ++d)
#pragma unroll
                for (int q = 0; q < 16; ++q) acc[d][q] *= f;
        }
    }
    __device__ __forceinline__ float shift() const { return base == -INFINITY ? 0.f : base; }
    // scores to weights
    __device__ __forceinline__ void weigh(float16_t& s, float c2, float sh) {
        float sum = 0.f;
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[q], c2, -sh));
            s[q] = p;
            sum += p;
        }
        l += sum;
    }
    // base-2 logarithm of the row's sum and the factor that its channels take
    __device__ __forceinline__ void finish(float& lse2, float& inv) {
        l += __shfl_xor(l, 32);
        inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;      // a NaN stays one
        lse2 = l == 0.f ? -INFINITY : base + log2f(l);
    }
};

// One row's channels: to the output, or with several ranges to the parts.
template <typename E, int DP>
__device__ __forceinline__ void store_row(const AttnArgs& a, const AttnParts& parts, const AttnRows& rows, int G, int b, int hk, int r, int split, int nsplit, int half,
                                          const AttnState<E, DP>& st, float inv, float lse2) {
    using T = AttnTile<E, DP>;
    const long long row = ((long long)b * a.Hkv + hk) * rows.R + r;
    if (nsplit > 1) {
        const long long at = (long long)split * a.B * a.Hkv * rows.R + row;
        if (half == 0) parts.lse2[at] = lse2;
        float* o = parts.o + at * a.D;
#pragma unroll
        for (int d = 0; d < T::NV; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = d * 32 + 8 * q + 4 * half;
                if (c < a.D) *reinterpret_cast<float4*>(o + c) = make_float4(st.acc[d][4 * q] * inv, st.acc[d][4 * q + 1] * inv, st.acc[d][4 * q + 2] * inv, st.acc[d][4 * q + 3] * inv);
            }
        return;
    }
    if (a.lse && half == 0) a.lse[row] = lse2 * kLn2;
    unsigned char* orow = const_cast<unsigned char*>(rows.at(a.o, G, b, hk, r, T::ES));
#pragma unroll
    for (int d = 0; d < T::NV; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float v[4] = {st.acc[d][4 * q] * inv, st.acc[d][4 * q + 1] * inv, st.acc[d][4 * q + 2] * inv, st.acc[d][4 * q + 3] * inv};
            store_channels<E>(orow, d * 32 + 8 * q + 4 * half, a.D, v);
        }
}

// 128 query rows per workgroup, 32 per wave; keys and values pass through LDS in tiles of 64 while the next tile is on its way in registers.
// Two waves a SIMD at least, as long as their registers suffice (up to 64 channels the compiler needs 105 to 145 and leaves room for three); wide heads give up the
// tile on its way for that.  What bounds it, at 2 x 10 x 4096 x 4096 x 64 (128 us): 640 workgroups are two or three a unit, 1.75 waves a SIMD on the mean; the vector unit
// is busy 48 % of the time (180 instructions a 64x32 tile beside its 16 MFMAs), the MFMAs 27 %, LDS 21 %.
template <typename E, int DP> constexpr int attention_waves() { return DP <= (sizeof(E) == 2 ? 10 : 5) ? 2 : 1; }
template <typename E, int DP> constexpr int attention_few_waves() { return DP <= 4 ? 2 : 1; }
template <typename E, int DP> constexpr bool attention_ahead() { return sizeof(E) == 2 && DP <= 8; }
template <typename E, int DP> __global__ void __launch_bounds__(256, (attention_waves<E, DP>()))
attention_kernel(AttnArgs a, AttnParts parts, int row_tiles, int nsplit, int total, int per_xcd) {
    using T = AttnTile<E, DP>;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int logical = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if (logical >= total) return;
    const int per_head = row_tiles * nsplit, slot = logical / per_head, in = logical - slot * per_head, split = in / row_tiles, tile = in - split * row_tiles;
    const int bh = deal_heads(slot, a.B * a.Hkv);
    const int b = bh / a.Hkv, hk = bh - b * a.Hkv, G = a.H / a.Hkv;
    const AttnRows rows{a.Sq, G * a.Sq};
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const typename T::Places places(lane);
    const int r = tile * 128 + wave * 32 + (lane & 31);
    const bool row_on = r < rows.R;

    u32x4_t fq[T::KS];                                     // first: under way while lengths and masks are looked at
    {
        const unsigned char* qrow = row_on ? rows.at(a.q, G, b, hk, r, T::ES) : nullptr;
#pragma unroll
        for (int ks = 0; ks < T::KS; ++ks) fq[ks] = load_channels<E>(qrow, (2 * ks + half) * T::V, row_on ? a.D : 0);
    }
    const unsigned char* kbase = static_cast<const unsigned char*>(a.k.p) + ((long long)b * a.k.b + (long long)hk * a.k.h) * T::ES;
    const unsigned char* vbase = static_cast<const unsigned char*>(a.v.p) + ((long long)b * a.v.b + (long long)hk * a.v.h) * T::ES;
    KeyMask mask(a, b);
    if (nsplit == 1) mask.request(0);
    const int len = key_count(a, b), tiles = (len + T::ROWS - 1) / T::ROWS;
    const int t0 = (int)((long long)split * tiles / nsplit), t1 = (int)((long long)(split + 1) * tiles / nsplit);
    using Stream = AttnStream<E, DP>;
    const typename Stream::Map map(tid, a.D);
    Stream sk(map, kbase, t0 * T::ROWS, a.k.s), sv(map, vbase, t0 * T::ROWS, a.v.s);
    AttnState<E, DP> st;
    const float c2 = a.scale * kLog2e;
    if (nsplit > 1) mask.request(t0 * T::ROWS);
    auto valid = [&](int t) {                              // and the next tile's mask on its way
        const unsigned long long on = mask.bits(t * T::ROWS, len);
        mask.request((t + 1) * T::ROWS);
        return on;
    };
    auto step = [&](const unsigned char* tk, const unsigned char* tv, unsigned long long on) {
        float16_t s[2] = {};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int ks = 0; ks < T::KS; ++ks) Mma<E>::run(T::along(tk, 32 * i, ks, places), fq[ks], s[i]);
        st.template settle<2>(s, on, half, c2);
        const float sh = st.shift();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            st.weigh(s[i], c2, sh);
#pragma unroll
            for (int k = 0; k < T::ST; ++k) {
                const u32x4_t w = T::weights(s[i], k);
#pragma unroll
                for (int d = 0; d < T::NV; ++d) Mma<E>::run(T::across(tv, 32 * i, k, d, places), w, st.acc[d]);
            }
        }
    };
    if constexpr (attention_ahead<E, DP>()) {
        // two buffers in turn, one barrier a tile
        unsigned long long on = valid(t0);
        if (t0 < t1) {
            sk.fetch(map, on);
            sv.fetch(map, on);
        }
        for (int t = t0; t < t1; ++t) {
            unsigned char* tk = lds + ((t - t0) & 1) * 2 * T::BYTES;
            unsigned char* tv = tk + T::BYTES;
            sk.put(map, tk);
            sv.put(map, tv);
            __syncthreads();
            const unsigned long long cur = on;
            if (t + 1 < t1) {
                on = valid(t + 1);
                sk.fetch(map, on);
                sv.fetch(map, on);
            }
            if (cur) step(tk, tv, cur);                    // uniform: every wave has the same keys
        }
    } else {
        unsigned char* tk = lds;
        unsigned char* tv = lds + T::BYTES;
        for (int t = t0; t < t1; ++t) {
            const unsigned long long on = valid(t);
            sk.fetch(map, on);
            sv.fetch(map, on);
            __syncthreads();
            sk.put(map, tk);
            sv.put(map, tv);
            __syncthreads();
            if (on) step(tk, tv, on);
        }
    }
    float lse2, inv;
    st.finish(lse2, inv);
    if (row_on) store_row<E, DP>(a, parts, rows, G, b, hk, r, split, nsplit, half, st, inv, lse2);
}

// At most 32 query rows a key head (one token of each query head that shares it, say): the four waves of a workgroup take different keys for the same
// rows and are joined in LDS.  Bound by reading keys and values: each wave streams tiles of its own through LDS of its own, without a barrier in the loop,
// with the next tile in flight (128 KB a compute unit at 128 channels).  8 x 15000 keys of 8 x 128 channels, bf16: 3.8 TB/s on those that are valid.  One wave a SIMD from
// 80 channels on; above 96 the registers spill all the same, 36 bytes a lane at 128 channels, 60 at 160, 172 at 256.
template <typename E, int DP> struct AttnFew {
    using T = AttnTile<E, DP>;
    static constexpr int SUBS = T::ES == 2 && DP <= 10 ? 2 : 1, KEYS = 32 * SUBS;
    static constexpr int WAVE_BYTES = 2 * KEYS * T::STRIDE;    // keys, values
    static constexpr int RPI = 64 / T::CPR;                    // rows that one load of the wave covers; the last lanes may have none
    static constexpr int LOADS = (KEYS + RPI - 1) / RPI;
    static constexpr int ROW = T::NV * 32 + 3;                 // floats per row and wave that are joined: channels, base, sum; odd
    static constexpr int BYTES = 4 * (WAVE_BYTES > 32 * ROW * 4 ? WAVE_BYTES : 32 * ROW * 4);
};
template <typename E, int DP> __global__ void __launch_bounds__(256, (attention_few_waves<E, DP>()))
attention_few_kernel(AttnArgs a, AttnParts parts, int nsplit) {
    using T = AttnTile<E, DP>;
    using F = AttnFew<E, DP>;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int bh = blockIdx.x / nsplit, split = blockIdx.x - bh * nsplit;       // no two workgroups read the same keys: no order among the XCDs
    const int b = bh / a.Hkv, hk = bh - b * a.Hkv, G = a.H / a.Hkv;
    const AttnRows rows{a.Sq, G * a.Sq};
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const typename T::Places places(lane);
    const int r = lane & 31;
    const bool row_on = r < rows.R;
    unsigned char* tk = lds + wave * F::WAVE_BYTES;
    unsigned char* tv = tk + F::KEYS * T::STRIDE;

    const unsigned char* kbase = static_cast<const unsigned char*>(a.k.p) + ((long long)b * a.k.b + (long long)hk * a.k.h) * T::ES;
    const unsigned char* vbase = static_cast<const unsigned char*>(a.v.p) + ((long long)b * a.v.b + (long long)hk * a.v.h) * T::ES;
    const int len = key_count(a, b), tiles = (len + F::KEYS - 1) / F::KEYS, part = split * 4 + wave;
    const int t0 = (int)((long long)part * tiles / (nsplit * 4)), t1 = (int)((long long)(part + 1) * tiles / (nsplit * 4));
    // this lane's chunk of each load: a 32-bit offset behind a wave-uniform place (the launcher checks the strides for that)
    const int lrow = lane / T::CPR, chunk = lane - lrow * T::CPR;
    const bool lane_on = lrow < F::RPI && chunk * T::V < a.D, whole = a.D == DP * 16 && 64 % T::CPR == 0;
    const uint32_t koff = (uint32_t)(lrow * a.k.s * T::ES) + chunk * 16, voff = (uint32_t)(lrow * a.v.s * T::ES) + chunk * 16;
    u32x4_t fq[T::KS], lk[F::LOADS], lv[F::LOADS];
    const u32x4_t zero = {0, 0, 0, 0};
    constexpr unsigned long long ALL = F::SUBS == 2 ? ~0ull : 0xffffffffull;
    KeyMask keys(a, b);
    keys.request(t0 * F::KEYS);
    auto mask = [&](int t) {                               // and the next tile's on its way
        const unsigned long long on = keys.bits(t * F::KEYS, len) & ALL;
        keys.request((t + 1) * F::KEYS);
        return on;
    };
    auto fetch = [&](int t, unsigned long long on) {
        const unsigned char* kt = kbase + (long long)t * F::KEYS * a.k.s * T::ES;
        const unsigned char* vt = vbase + (long long)t * F::KEYS * a.v.s * T::ES;
        const long long kstep = F::RPI * a.k.s * T::ES, vstep = F::RPI * a.v.s * T::ES;
        if (whole && on == ALL) {
#pragma unroll
            for (int i = 0; i < F::LOADS; ++i) lk[i] = *reinterpret_cast<const u32x4_t*>(kt + i * kstep + koff);
#pragma unroll
            for (int i = 0; i < F::LOADS; ++i) lv[i] = *reinterpret_cast<const u32x4_t*>(vt + i * vstep + voff);
        } else {
#pragma unroll
            for (int i = 0; i < F::LOADS; ++i) {
                const int row = i * F::RPI + lrow;
                const bool ok = lane_on && row < F::KEYS && ((on >> (row & 63)) & 1);
                lk[i] = ok ? *reinterpret_cast<const u32x4_t*>(kt + i * kstep + koff) : zero;
                lv[i] = ok ? *reinterpret_cast<const u32x4_t*>(vt + i * vstep + voff) : zero;
            }
        }
    };
    auto put = [&] {
#pragma unroll
        for (int i = 0; i < F::LOADS; ++i) {
            const int row = i * F::RPI + lrow, at = T::at(row, chunk);
            if (64 % T::CPR == 0 || (lrow < F::RPI && row < F::KEYS)) {
                *reinterpret_cast<u32x4_t*>(tk + at) = lk[i];
                *reinterpret_cast<u32x4_t*>(tv + at) = lv[i];
            }
        }
    };
    unsigned long long on = t0 < t1 ? mask(t0) : 0;
    if (t0 < t1) fetch(t0, on);
    {
        const unsigned char* qrow = row_on ? rows.at(a.q, G, b, hk, r, T::ES) : nullptr;
#pragma unroll
        for (int ks = 0; ks < T::KS; ++ks) fq[ks] = load_channels<E>(qrow, (2 * ks + half) * T::V, row_on ? a.D : 0);
    }
    AttnState<E, DP> st;
    const float c2 = a.scale * kLog2e;
    for (int t = t0; t < t1; ++t) {
        const unsigned long long cur = on;
        __builtin_amdgcn_wave_barrier();                   // a tile in LDS is written and read by this wave alone, in order
        put();
        __builtin_amdgcn_wave_barrier();
        if (t + 1 < t1) {
            on = mask(t + 1);
            fetch(t + 1, on);
        }
        if (cur == 0) continue;                            // uniform over the wave
        float16_t s[F::SUBS] = {};
#pragma unroll
        for (int i = 0; i < F::SUBS; ++i)
#pragma unroll
            for (int ks = 0; ks < T::KS; ++ks) Mma<E>::run(T::along(tk, 32 * i, ks, places), fq[ks], s[i]);
        st.template settle<F::SUBS>(s, cur, half, c2);
        const float sh = st.shift();
#pragma unroll
        for (int i = 0; i < F::SUBS; ++i) {
            st.weigh(s[i], c2, sh);
#pragma unroll
            for (int k = 0; k < T::ST; ++k) {
                const u32x4_t w = T::weights(s[i], k);
#pragma unroll
                for (int d = 0; d < T::NV; ++d) Mma<E>::run(T::across(tv, 32 * i, k, d, places), w, st.acc[d]);
            }
        }
    }
    // join the four waves: each leaves base, sum and channels; wave 0 adds them up in order
    st.l += __shfl_xor(st.l, 32);
    __syncthreads();
    float* mine = reinterpret_cast<float*>(lds) + (wave * 32 + r) * F::ROW;
    if (row_on) {
#pragma unroll
        for (int d = 0; d < T::NV; ++d)
#pragma unroll
            for (int q = 0; q < 16; ++q) mine[d * 32 + 8 * (q / 4) + 4 * half + q % 4] = st.acc[d][q];
        if (half == 0) { mine[T::NV * 32] = st.base; mine[T::NV * 32 + 1] = st.l; }
    }
    __syncthreads();
    if (wave != 0 || !row_on) return;
    const float* all = reinterpret_cast<const float*>(lds) + r * F::ROW;
    constexpr int STEP = 32 * F::ROW;
    float base = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) base = fmaxf(base, all[w * STEP + T::NV * 32]);
    const float shift = base == -INFINITY ? 0.f : base;
    float l = 0.f, f[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        f[w] = __builtin_amdgcn_exp2f(all[w * STEP + T::NV * 32] - shift);
        l = fmaf(all[w * STEP + T::NV * 32 + 1], f[w], l);
    }
#pragma unroll
    for (int d = 0; d < T::NV; ++d)
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int c = d * 32 + 8 * (q / 4) + 4 * half + q % 4;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) v = fmaf(all[w * STEP + c], f[w], v);
            st.acc[d][q] = v;
        }
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l, lse2 = l == 0.f ? -INFINITY : base + log2f(l);
    store_row<E, DP>(a, parts, rows, G, b, hk, r, split, nsplit, half, st, inv, lse2);
}

// one workgroup per row: the ranges' results, weighted by their sums (lane i has range i's; there are at most 64).  What it reads was written by other
// XCDs a moment ago and is 2 us away: wave w takes ranges w, w + 4, ..., and everything is requested before the first weight is known.
template <typename E> __global__ void __launch_bounds__(256) attention_join_kernel(AttnArgs a, AttnParts parts, int nsplit, long long all) {
    const long long row = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), G = a.H / a.Hkv;
    const AttnRows rows{a.Sq, G * a.Sq};
    __shared__ float sums[4][256];
    const float lse2 = lane < nsplit ? parts.lse2[lane * all + row] : -INFINITY;
    float v[4] = {}, first[4][4];
    const float* base = parts.o + row * a.D;
    const long long step = all * a.D;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) first[i][c] = wave + 4 * i < nsplit && lane + 64 * c < a.D ? base[(wave + 4 * i) * step + lane + 64 * c] : 0.f;
    float m = lse2;
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    float w = __builtin_amdgcn_exp2f(lse2 - (m == -INFINITY ? 0.f : m)), total = w;
#pragma unroll
    for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
    w *= total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
    auto weight = [&](int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), i)); };
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (wave + 4 * i < nsplit) {
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = fmaf(weight(wave + 4 * i), first[i][c], v[c]);
        }
    for (int i = wave + 16; i < nsplit; i += 4)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (lane + 64 * c < a.D) v[c] = fmaf(weight(i), base[i * step + lane + 64 * c], v[c]);
#pragma unroll
    for (int c = 0; c < 4; ++c) sums[wave][lane + 64 * c] = v[c];
    __syncthreads();
    const int bh = (int)(row / rows.R), r = (int)(row - (long long)bh * rows.R), b = bh / a.Hkv, hk = bh - b * a.Hkv, c = threadIdx.x;
    E* o = reinterpret_cast<E*>(const_cast<unsigned char*>(rows.at(a.o, G, b, hk, r, (int)sizeof(E))));
    if (c < a.D) o[c] = from_f32<E>((sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]));
    if (a.lse && threadIdx.x == 0) a.lse[row] = total == 0.f ? -INFINITY : (m + log2f(total)) * kLn2;
}

// Whether the rows of a key head fit one wave's tile.
bool few_rows(int Sq, int H, int Hkv) { return (long long)(H / Hkv) * Sq <= 32; }

// Ranges of the keys, where the rows alone leave compute units idle.  Few rows: about four workgroups a unit, because lengths that differ leave some of
// them short, and at least 128 keys a wave.  Otherwise the number with the least time by this count: 1 us a tile of keys for up to two workgroups
// a unit (fp32: its MFMAs, 0.06 us a channel); a join is 5 us and the parts written and read (16 heads x 1024 x 1024 x 80 in fp16, 128 workgroups: one
// range 31, four 45 us).
int attention_ranges(int B, int Sq, int Skv, int H, int Hkv, int D, int dt) {
    if (few_rows(Sq, H, Hkv)) {
        long long n = 1024 / ((long long)B * Hkv);
        if (n > Skv / 512) n = Skv / 512;
        if (n > 64) n = 64;
        return n < 2 ? 1 : (int)n;
    }
    const long long blocks = (long long)B * Hkv * (((long long)(H / Hkv) * Sq + 127) / 128);
    const int tiles = (Skv + 63) / 64;
    int best = 1;
    double least = 0.;
    for (int n = 1; n <= 64 && (n == 1 || tiles / n >= 4); ++n) {
        const double wide = (double)(blocks * n) / 512.;
        const double us = (dt == DT_F32 ? 1. + 0.06 * D : 1.) * (double)((tiles + n - 1) / n) * (wide > 1. ? wide : 1.) + (n == 1 ? 0. : 5. + (double)n * B * H * Sq * D * 8. / 4e6);
        if (n == 1 || us < least) { best = n; least = us; }
    }
    return best;
}

}  // namespace

size_t attention_ws_bytes(int B, int Sq, int Skv, int H, int Hkv, int D, int dt) {
    const int n = attention_ranges(B, Sq, Skv, H, Hkv, D, dt);
    return n == 1 ? 0 : (size_t)n * B * H * Sq * ((size_t)D + 1) * sizeof(float);
}

hipError_t launch_attention(const AttnArgs& a, int dt, hipStream_t s) {
    const int R = a.H / a.Hkv * a.Sq, nsplit = attention_ranges(a.B, a.Sq, a.Skv, a.H, a.Hkv, a.D, dt), row_tiles = (R + 127) / 128;
    const long long all = (long long)a.B * a.Hkv * R, total = (long long)a.B * a.Hkv * row_tiles * nsplit;
    if (total > 0x3fffffffLL || all > 0x7fffffffLL) return hipErrorInvalidValue;
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
                if constexpr (AttnFew<E, DP>::BYTES <= 160 * 1024) {           // fp32 with more than 128 channels does not fit
                    // (offsets within a load of the few-rows kernel are 32 bits wide)
                    if (few_rows(a.Sq, a.H, a.Hkv) && (a.k.s | a.v.s) < (1LL << 24)) {
                        auto kern = attention_few_kernel<E, DP>;
                        constexpr int bytes = AttnFew<E, DP>::BYTES;
                        static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
                        if (attr != hipSuccess) return attr;
                        hipLaunchKernelGGL(kern, dim3((unsigned)(a.B * a.Hkv * nsplit)), dim3(256), bytes, s, a, parts, nsplit);
                        return hipGetLastError();
                    }
                }
                auto kern = attention_kernel<E, DP>;
                constexpr int bytes = (attention_ahead<E, DP>() ? 4 : 2) * T::BYTES;
                static_assert(bytes <= 160 * 1024, "LDS budget");
                static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
                if (attr != hipSuccess) return attr;
                hipLaunchKernelGGL(kern, dim3((unsigned)(per_xcd * 8)), dim3(256), bytes, s, a, parts, row_tiles, nsplit, (int)total, per_xcd);
                return hipGetLastError();
            }
        });
        if (rc != hipSuccess || nsplit == 1) return rc;
        hipLaunchKernelGGL((attention_join_kernel<E>), dim3((unsigned)all), dim3(256), 0, s, a, parts, nsplit, all);
        return hipGetLastError();
    });
}

}  // namespace wino
