// Gradients of attention.  With p = exp(s - lse) from the forward pass and D_i = do_i . o_i:
//   dv = p^T do,  ds = p (do v^T - D),  dq = scale ds k,  dk = scale ds^T q.
// Scores are made again, never stored.  Two kernels, both without atomics, so that results do not depend on the order of the workgroups: one owns
// query rows and streams the keys (dq, and D for the other), one owns keys and streams the query rows of their head (dk, dv; over ranges of the rows,
// joined in order, where there are few keys).  In either a wave owns 32 rows or keys: a workgroup 128 (WIDE), or 64 where those would be too few
// workgroups, with two waves for each 32 that take one half of every streamed tile each; the halves are added in LDS at the end.
#include "attention_tile.h"

namespace wino {

namespace {

struct BackwardParts {
    float* delta;                    // [B][Hkv][R]
    float* dk;                       // [nsplit][B][Hkv][Skv][D], both null with one range
    float* dv;
};

// Two waves a SIMD as long as their registers suffice.
template <typename E, int DP> constexpr int dq_waves() { return DP <= (sizeof(E) == 2 ? 5 : 4) ? 2 : 1; }
template <typename E, int DP> constexpr int backward_waves() { return DP <= (sizeof(E) == 2 ? 6 : 4) ? 2 : 1; }
// Two-byte types keep two tiles in LDS and one on its way, except where its registers and addresses cost more than it hides: us with / without, for
// 2 x 8 x 1024 x 1024 x D in bf16 (128: 2 x 8 x 2048 x 2048): D 96 57 / 58, 128 187 / 173, 160 94 / 99, 256 366 / 153 (648 bytes a lane spilled; without it 148 to 312 are
// still).  fp32's tiles are too large for it.
template <typename E, int DP> constexpr bool backward_ahead() { return sizeof(E) == 2 && (DP <= 6 || DP == 10); }

// fp16 ends at 65504 and loses bits below 6e-5, and the gradients of the scores may lie beyond either where the results do not.  They become an operand times
// f = 2^e, with an e of its own for each column of the product (a query row, or a key; one per lane, the same in both halves), and the accumulated sums carry
// that factor too.  e falls when a value passes 2^15, to where the column's largest so far is between 2^7 and 2^8: once or twice a column.  The first e cannot take
// a value out of fp32: |ds| < 2^42, by fp16's own range.  Softmax weights are at most 1 and take a fixed 2^12, with which 2^-26 is still a normal number.
// Heads of more than 160 channels have no registers left for the branch: they find the largest value in a pass of its own and keep one e (2 x 8 x 1024 x 1024 x
// 256: 234 us; 465 with the branch, which spills).  us without / with factors: 4 x 10 x 1024 x 154 x 64 33.6 / 34.8, 4 x 8 x 1024 x 1024 x 80 73 / 77 (20 to 44
// bytes a lane spilled), 2 x 10 x 4096 x 4096 x 64 451 / 476, 2 x 8 x 2048 x 2048 x 128 171 / 180, 2 x 8 x 1024 x 1024 x 256 152 / 234.
template <typename E> constexpr bool short_range() { return std::is_same_v<E, __half>; }
template <typename E, int DP> constexpr bool two_passes() { return short_range<E>() && DP > 10; }
constexpr int kWeightPower = 12;
struct ColumnPower {
    int e = 60;
    float f = 0x1p60f;
    float top = 0.f;                                       // of a pass that looks only
    __device__ __forceinline__ void look(const float16_t& ds) {
#pragma unroll
        for (int q = 0; q < 16; ++q) top = fmaxf(top, fabsf(ds[q]));
    }
    __device__ __forceinline__ void decide() {
        e += 14 - __builtin_amdgcn_frexp_expf(fmaxf(top, __shfl_xor(top, 32)));
        f = __builtin_amdgcn_ldexpf(1.f, e);
    }
    // ds: 16 values with the factor; `sums` the N accumulators that have it, `more` another sum.  Called by whole waves; `on` false: the column does not count
    template <int N, int M> __device__ __forceinline__ void settle(float16_t& ds, float16_t (&sums)[M], float& more, bool on) {
        float top = 0.f;
#pragma unroll
        for (int q = 0; q < 16; ++q) top = fmaxf(top, fabsf(ds[q]));
        if (__builtin_expect(__any(on && top > 32768.f), 0)) {
            top = fmaxf(top, __shfl_xor(top, 32));
            const int down = on && top > 32768.f ? 8 - __builtin_amdgcn_frexp_expf(top) : 0;        // (infinity stays what it is)
            const float by = __builtin_amdgcn_ldexpf(1.f, down);
            e += down;
            f *= by;
            more *= by;
#pragma unroll
            for (int q = 0; q < 16; ++q) ds[q] *= by;
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int q = 0; q < 16; ++q) sums[d][q] *= by;
        }
    }
    __device__ __forceinline__ float inverse() const { return __builtin_amdgcn_ldexpf(1.f, -e); }
};

// accumulators times their factors, `first` for the first half of them; with two waves for the same rows (!WIDE) those of waves 2 and 3 are added to those of waves 0
// and 1, through LDS; called by the whole workgroup
template <bool WIDE, int N> __device__ __forceinline__ void add_halves(float16_t (&acc)[N], float first, float second, unsigned char* lds, int wave, int lane) {
    if constexpr (WIDE) {
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[d][q] *= 2 * d < N ? first : second;
        return;
    }
    float* t = reinterpret_cast<float*>(lds) + (wave & 1) * (N * 1024) + lane;
    __syncthreads();
    if (wave >= 2) {
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int q = 0; q < 16; ++q) t[(d * 16 + q) * 64] = acc[d][q] * (2 * d < N ? first : second);
    }
    __syncthreads();
    if (wave < 2) {
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[d][q] = fmaf(acc[d][q], 2 * d < N ? first : second, t[(d * 16 + q) * 64]);
    }
}

// Query rows: dq, and D_i for the other kernel.
//
// D_i = do_i . o_i from the stored o carries o's rounding, which reaches every ds of the row with the same sign.  But the ds of a row add up to zero, so
// what they do add up to, r, is that error: D_i + r is right to fp32, and dq less r times the weighted mean of the keys as well.  The mean costs one more
// product with operands that are there already (4 x 8 x 1024 x 1024 x 80: 35 -> 43 us); the error of dq against 64 bits falls from 1.50 to 1.41 times that of
// one rounding, which is the rounding of ds and that of dq.
template <typename E, int DP, bool WIDE> __global__ void __launch_bounds__(256, (dq_waves<E, DP>()))
attention_dq_kernel(AttnArgs a, float* delta, int row_tiles, int total, int per_xcd) {
    using T = AttnTile<E, DP>;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int logical = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if (logical >= total) return;
    const int slot = logical / row_tiles, tile = logical - slot * row_tiles, bh = deal_heads(slot, a.B * a.Hkv), b = bh / a.Hkv, hk = bh - b * a.Hkv, G = a.H / a.Hkv;
    const AttnRows rows{a.Sq, G * a.Sq};
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, sub = WIDE ? 0 : wave >> 1;
    const typename T::Places places(lane);
    const int r = tile * (WIDE ? 128 : 64) + (WIDE ? wave : wave & 1) * 32 + (lane & 31);
    const bool row_on = r < rows.R;
    const unsigned char* kbase = static_cast<const unsigned char*>(a.k.p) + ((long long)b * a.k.b + (long long)hk * a.k.h) * T::ES;
    const unsigned char* vbase = static_cast<const unsigned char*>(a.v.p) + ((long long)b * a.v.b + (long long)hk * a.v.h) * T::ES;
    KeyMask mask(a, b);
    mask.request(0);
    const int len = key_count(a, b), tiles = (len + T::ROWS - 1) / T::ROWS;
    using Stream = AttnStream<E, DP>;
    const typename Stream::Map map(tid, a.D);
    Stream sk(map, kbase, 0, a.k.s), sv(map, vbase, 0, a.v.s);
    constexpr bool AHEAD = backward_ahead<E, DP>();
    unsigned long long on = mask.bits(0, len);
    mask.request(T::ROWS);
    if (AHEAD && tiles) {
        sk.fetch(map, on);
        sv.fetch(map, on);
    }
    u32x4_t fq[T::KS], fo[T::KS];
    const long long row = (long long)bh * rows.R + r;
    float dlt = 0.f;
    {
        const unsigned char* qrow = row_on ? rows.at(a.q, G, b, hk, r, T::ES) : nullptr;
        const unsigned char* grow = row_on ? rows.at(a.dout, G, b, hk, r, T::ES) : nullptr;
        const unsigned char* orow = row_on ? rows.at(a.o, G, b, hk, r, T::ES) : nullptr;
#pragma unroll
        for (int ks = 0; ks < T::KS; ++ks) {
            const int c = (2 * ks + half) * T::V, D = row_on ? a.D : 0;
            fq[ks] = load_channels<E>(qrow, c, D);
            fo[ks] = load_channels<E>(grow, c, D);
            const u32x4_t x = load_channels<E>(orow, c, D);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (T::ES == 4) dlt = fmaf(__uint_as_float(x[i]), __uint_as_float(fo[ks][i]), dlt);
                else { dlt = fmaf(lo16<E>(x[i]), lo16<E>(fo[ks][i]), dlt); dlt = fmaf(hi16<E>(x[i]), hi16<E>(fo[ks][i]), dlt); }
            }
        }
        dlt += __shfl_xor(dlt, 32);
    }
    const float lse2 = row_on ? a.lse[row] * kLog2e : 0.f;
    constexpr bool MEAN = T::ES == 2;                      // fp32: o is not rounded
    constexpr int NA = MEAN ? 2 * T::NV : T::NV;           // dq, then the mean of the keys
    float16_t acc[NA] = {};
    float rest = 0.f;
    [[maybe_unused]] ColumnPower power;
    const float c2 = a.scale * kLog2e;
    constexpr bool TWICE = two_passes<E, DP>();
    static_assert(!(TWICE && AHEAD), "the first pass leaves no tile on its way");
    auto stream = [&](auto look) {                         // all tiles; look: for the largest gradient of a score only
        for (int t = 0; t < tiles; ++t) {
            unsigned char* tk = lds + (AHEAD ? (t & 1) * 2 * T::BYTES : 0);
            unsigned char* tv = tk + T::BYTES;
            if (!AHEAD) {
                sk.fetch(map, on);
                sv.fetch(map, on);
                __syncthreads();
            }
            sk.put(map, tk);
            sv.put(map, tv);
            __syncthreads();
            const unsigned long long now = on;
            if (t + 1 < tiles) {
                on = mask.bits((t + 1) * T::ROWS, len);
                mask.request((t + 2) * T::ROWS);
                if (AHEAD) {
                    sk.fetch(map, on);
                    sv.fetch(map, on);
                }
            }
#pragma unroll 1
            for (int h = sub; h < (WIDE ? 2 : sub + 1); ++h) {
                const uint32_t cur = (uint32_t)(now >> (32 * h));
                if (cur == 0) continue;                        // uniform over the wave
                float16_t s = {}, dp = {};
#pragma unroll
                for (int ks = 0; ks < T::KS; ++ks) {
                    Mma<E>::run(T::along(tk, 32 * h, ks, places), fq[ks], s);
                    Mma<E>::run(T::along(tv, 32 * h, ks, places), fo[ks], dp);
                }
#pragma unroll
                for (int q = 0; q < 16; ++q) s[q] = __builtin_amdgcn_exp2f(fmaf(s[q], c2, -lse2));
                if (cur != 0xffffffffu) {
                    asm volatile("" ::: "memory");             // a branch
                    const uint32_t mine = cur >> (4 * half);
#pragma unroll
                    for (int q = 0; q < 16; ++q)
                        if (!((mine >> (8 * (q / 4) + q % 4)) & 1)) s[q] = 0.f;
                }
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    if constexpr (short_range<E>()) dp[q] = s[q] * fmaf(dp[q], power.f, -dlt * power.f);
                    else dp[q] = s[q] * (dp[q] - dlt);
                    if constexpr (MEAN && !look) rest += dp[q];
                }
                if constexpr (look) {
                    power.look(dp);
                    continue;
                }
                // (with a branch for the factors: the mean's products run beside it)
                constexpr bool SETTLE = short_range<E>() && !TWICE;
                u32x4_t keys[T::ST][T::NV];
                if constexpr (SETTLE) {
#pragma unroll
                    for (int st = 0; st < T::ST; ++st) {
                        const u32x4_t wp = T::weights(s, st);
#pragma unroll
                        for (int d = 0; d < T::NV; ++d) {
                            keys[st][d] = T::across(tk, 32 * h, st, d, places);
                            Mma<E>::run(keys[st][d], wp, acc[T::NV + d]);
                        }
                    }
                    power.settle<T::NV>(dp, acc, rest, true);
                }
#pragma unroll
                for (int st = 0; st < T::ST; ++st) {
                    const u32x4_t w = T::weights(dp, st), wp = MEAN ? T::weights(s, st) : w;
#pragma unroll
                    for (int d = 0; d < T::NV; ++d) {
                        if constexpr (!SETTLE) keys[st][d] = T::across(tk, 32 * h, st, d, places);
                        Mma<E>::run(keys[st][d], w, acc[d]);
                        if constexpr (MEAN && !SETTLE) Mma<E>::run(keys[st][d], wp, acc[T::NV + d]);
                    }
                }
            }
        }
    };
    if constexpr (TWICE) {
        stream(std::true_type());
        power.decide();
        sk.jump(-tiles * sk.step);
        sv.jump(-tiles * sv.step);
        mask.request(0);
        on = mask.bits(0, len);
        mask.request(T::ROWS);
    }
    stream(std::false_type());
    const float back = short_range<E>() ? power.inverse() : 1.f;
    rest *= back;
    add_halves<WIDE>(acc, back, 1.f, lds, wave, lane);
    if constexpr (MEAN) {
        rest += __shfl_xor(rest, 32);
        if constexpr (!WIDE) {
            float* t = reinterpret_cast<float*>(lds) + (wave & 1) * 64 + lane;
            __syncthreads();
            if (sub) *t = rest;
            __syncthreads();
            if (!sub) rest += *t;
        }
#pragma unroll
        for (int d = 0; d < T::NV; ++d)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[d][q] = fmaf(-rest, acc[T::NV + d][q], acc[d][q]);
    }
    if (sub || !row_on) return;
    if (half == 0) delta[row] = dlt + rest;
    unsigned char* out = const_cast<unsigned char*>(rows.at(a.dq, G, b, hk, r, T::ES));
#pragma unroll
    for (int d = 0; d < T::NV; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float v[4] = {acc[d][4 * q] * a.scale, acc[d][4 * q + 1] * a.scale, acc[d][4 * q + 2] * a.scale, acc[d][4 * q + 3] * a.scale};
            store_channels<E>(out, d * 32 + 8 * q + 4 * half, a.D, v);
        }
}

// Keys: dk and dv over one range of the query rows.  Tiles hold rows of one query head each.
template <typename E, int DP, bool WIDE> __global__ void __launch_bounds__(256, (backward_waves<E, DP>()))
attention_dkv_kernel(AttnArgs a, BackwardParts parts, int key_tiles, int nsplit, int total, int per_xcd) {
    using T = AttnTile<E, DP>;
    constexpr bool AHEAD = backward_ahead<E, DP>();
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    float* stats = reinterpret_cast<float*>(lds + (AHEAD ? 4 : 2) * T::BYTES);        // per buffer: -lse (base 2) and D of the tile's rows
    const int logical = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if (logical >= total) return;
    const int per_head = key_tiles * nsplit, slot = logical / per_head, in = logical - slot * per_head, split = in / key_tiles, tile = in - split * key_tiles;
    const int bh = deal_heads(slot, a.B * a.Hkv);
    const int b = bh / a.Hkv, hk = bh - b * a.Hkv, G = a.H / a.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, sub = WIDE ? 0 : wave >> 1;
    const typename T::Places places(lane);
    const int len = key_count(a, b), key = tile * (WIDE ? 128 : 64) + (WIDE ? wave : wave & 1) * 32 + (lane & 31);
    const bool in_range = key < a.Skv, key_on = key < len && (!a.key_mask || a.key_mask[(long long)b * a.Skv + key] != 0);
    // acc: dk, then dv.  What a lane whose key is not valid sums stays in its own column and is dropped at the end.
    float16_t acc[2 * T::NV] = {};
    // a tile of keys that no query may look at has nothing to sum (uniform over the workgroup)
    if (__syncthreads_or(key_on)) {
        const int head_tiles = (a.Sq + T::ROWS - 1) / T::ROWS, tiles = G * head_tiles;
        const int t0 = (int)((long long)split * tiles / nsplit), t1 = (int)((long long)(split + 1) * tiles / nsplit);
        const int g0 = t0 / head_tiles, ht0 = t0 - g0 * head_tiles;
        int g = g0, ht = ht0;                                                        // head and tile of the next fetch
        using Stream = AttnStream<E, DP>;
        const typename Stream::Map map(tid, a.D);
        const unsigned char* qbase = static_cast<const unsigned char*>(a.q.p) + ((long long)b * a.q.b + (long long)(hk * G + g) * a.q.h) * T::ES;
        const unsigned char* obase = static_cast<const unsigned char*>(a.dout.p) + ((long long)b * a.dout.b + (long long)(hk * G + g) * a.dout.h) * T::ES;
        Stream sq(map, qbase, (long long)ht * T::ROWS, a.q.s), so(map, obase, (long long)ht * T::ROWS, a.dout.s);
        float nlse = 0.f, dlt = 0.f;
        constexpr float lift = short_range<E>() ? kWeightPower : 0.f;                // weights times 2^lift, and with them the gradients of the scores
        [[maybe_unused]] ColumnPower power;
        auto fetch = [&] {
            const int left = a.Sq - ht * T::ROWS;
            const unsigned long long on = left >= T::ROWS ? ~0ull : (1ull << left) - 1;
            sq.fetch(map, on);
            so.fetch(map, on);
            if (tid < T::ROWS) {
                const long long at = ((long long)bh * G + g) * a.Sq + ht * T::ROWS + tid;
                nlse = tid < left ? fmaf(-a.lse[at], kLog2e, lift) : -INFINITY;         // a row behind the last: p = 0
                dlt = tid < left ? parts.delta[at] : 0.f;
            }
            if (++ht == head_tiles) {
                ht = 0;
                ++g;
                sq.jump(a.q.h * T::ES - head_tiles * sq.step);
                so.jump(a.dout.h * T::ES - head_tiles * so.step);
            }
        };
        if (AHEAD && t0 < t1) fetch();
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
        const float c2 = a.scale * kLog2e;
        constexpr bool TWICE = two_passes<E, DP>();
        static_assert(!(TWICE && AHEAD), "the first pass leaves no tile on its way");
        auto stream = [&](auto look) {                     // as above
            for (int t = t0; t < t1; ++t) {
                const int buffer = AHEAD ? (t - t0) & 1 : 0;
                unsigned char* tq = lds + buffer * 2 * T::BYTES;
                unsigned char* to = tq + T::BYTES;
                float* tl = stats + buffer * 2 * T::ROWS;
                float* td = tl + T::ROWS;
                if (!AHEAD) {
                    fetch();
                    __syncthreads();
                }
                sq.put(map, tq);
                so.put(map, to);
                if (tid < T::ROWS) { tl[tid] = nlse; td[tid] = dlt; }
                __syncthreads();
                if (AHEAD && t + 1 < t1) fetch();
#pragma unroll 1
                for (int h = sub; h < (WIDE ? 2 : sub + 1); ++h) {
                    float16_t s = {}, dp = {};
#pragma unroll
                    for (int ks = 0; ks < T::KS; ++ks) {
                        Mma<E>::run(T::along(tq, 32 * h, ks, places), fk[ks], s);
                        Mma<E>::run(T::along(to, 32 * h, ks, places), fv[ks], dp);
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float4 nl = *reinterpret_cast<const float4*>(tl + 32 * h + 8 * q + 4 * half), dl = *reinterpret_cast<const float4*>(td + 32 * h + 8 * q + 4 * half);
                        const float n4[4] = {nl.x, nl.y, nl.z, nl.w}, d4[4] = {dl.x, dl.y, dl.z, dl.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float p = __builtin_amdgcn_exp2f(fmaf(s[4 * q + j], c2, n4[j]));
                            s[4 * q + j] = p;
                            dp[4 * q + j] = (short_range<E>() ? p * power.f : p) * (dp[4 * q + j] - d4[j]);
                        }
                    }
                    if constexpr (look) {
                        power.look(dp);
                        continue;
                    }
                    constexpr bool SETTLE = short_range<E>() && !TWICE;                  // as above, with dv's products
                    if constexpr (SETTLE) {
#pragma unroll
                        for (int st = 0; st < T::ST; ++st) {
                            const u32x4_t wp = T::weights(s, st);
#pragma unroll
                            for (int d = 0; d < T::NV; ++d) Mma<E>::run(T::across(to, 32 * h, st, d, places), wp, acc[T::NV + d]);
                        }
                        float none = 0.f;
                        power.settle<T::NV>(dp, acc, none, key_on);
                    }
#pragma unroll
                    for (int st = 0; st < T::ST; ++st) {
                        const u32x4_t wp = T::weights(s, st), wd = T::weights(dp, st);
#pragma unroll
                        for (int d = 0; d < T::NV; ++d) {
                            if constexpr (!SETTLE) Mma<E>::run(T::across(to, 32 * h, st, d, places), wp, acc[T::NV + d]);
                            Mma<E>::run(T::across(tq, 32 * h, st, d, places), wd, acc[d]);
                        }
                    }
                }
            }
        };
        if constexpr (TWICE) {
            stream(std::true_type());
            power.decide();
            sq.jump((ht0 - ht) * sq.step + (long long)(g0 - g) * a.q.h * T::ES);
            so.jump((ht0 - ht) * so.step + (long long)(g0 - g) * a.dout.h * T::ES);
            g = g0;
            ht = ht0;
        }
        stream(std::false_type());
        constexpr float drop = short_range<E>() ? 1.f / (1 << kWeightPower) : 1.f;
        add_halves<WIDE>(acc, short_range<E>() ? power.inverse() * drop : 1.f, drop, lds, wave, lane);
    }
    if (sub || !in_range) return;
    if (!key_on) {
#pragma unroll
        for (int d = 0; d < 2 * T::NV; ++d)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[d][q] = 0.f;
    }
    if (nsplit > 1) {
        const long long at = (((long long)split * a.B * a.Hkv + bh) * a.Skv + key) * a.D;
#pragma unroll
        for (int d = 0; d < T::NV; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = d * 32 + 8 * q + 4 * half;
                if (c < a.D) {
                    *reinterpret_cast<float4*>(parts.dk + at + c) = make_float4(acc[d][4 * q], acc[d][4 * q + 1], acc[d][4 * q + 2], acc[d][4 * q + 3]);
                    *reinterpret_cast<float4*>(parts.dv + at + c) =
                        make_float4(acc[T::NV + d][4 * q], acc[T::NV + d][4 * q + 1], acc[T::NV + d][4 * q + 2], acc[T::NV + d][4 * q + 3]);
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
            const float x[4] = {acc[d][4 * q] * a.scale, acc[d][4 * q + 1] * a.scale, acc[d][4 * q + 2] * a.scale, acc[d][4 * q + 3] * a.scale};
            const float y[4] = {acc[T::NV + d][4 * q], acc[T::NV + d][4 * q + 1], acc[T::NV + d][4 * q + 2], acc[T::NV + d][4 * q + 3]};
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

// Ranges of the query rows, where the keys alone leave compute units idle: the number with the least time by this count, 1.3 us a tile of rows for up to
// two workgroups a unit (fp32: its MFMAs, 0.06 us a channel more); a join is 5 us and the parts written and read.
int backward_ranges(int B, int Sq, int Skv, int H, int Hkv, int D, int dt) {
    const long long blocks = (long long)B * Hkv * (((long long)Skv + 63) / 64);
    const long long tiles = (long long)(H / Hkv) * ((Sq + 63) / 64);
    int best = 1;
    double least = 0.;
    for (int n = 1; n <= 16 && (n == 1 || tiles / n >= 4); ++n) {
        const double wide = (double)(blocks * n) / 512.;
        const double us = (dt == DT_F32 ? 1.3 + 0.06 * D : 1.3) * (double)((tiles + n - 1) / n) * (wide > 1. ? wide : 1.) + (n == 1 ? 0. : 5. + (double)n * B * Hkv * Skv * D * 16. / 4e6);
        if (n == 1 || us < least) { best = n; least = us; }
    }
    return best;
}
// Whether workgroups own 128 rows, 32 a wave, rather than 64.  Tiles then pass through LDS half as often and no halves are added, but a workgroup has twice
// the work, which takes it 1.75 times as long (fp32, bound by its MFMAs, 1.95): taken where that beats the rounds in which the chip runs twice as many
// workgroups of 64.  us of both kernels with 64 / 128 (B x H x Sq x Skv x D, bf16): 1 x 10 x 4096 x 4096 x 64 280 / 250, 4 x 16 x 1024 x 1024 x 80 140 / 118,
// 2 x 8 x 2048 x 2048 x 128 263 / 171, 4 x 8 x 1024 x 1024 x 80 71 / 83, 2 x 8 x 1024 x 1024 x 160 85 / 118; 4 x 10 x 1024 x 154 x 64 38.8 / 38.0, and 35.3 by the rule, which asks
// for each of them; fp32 4 x 8 x 1024 x 1024 x 80 396 / 355, 2 x 8 x 1024 x 1024 x 160 366 / 457.
bool own_wide(long long heads, int rows, int waves, bool f32) {
    const long long slots = 256 * waves, narrow = heads * (((long long)rows + 63) / 64), wide = heads * (((long long)rows + 127) / 128);
    return (double)((narrow + slots - 1) / slots) > (f32 ? 1.95 : 1.75) * (double)((wide + slots - 1) / slots);
}
template <typename E, int DP, bool WIDE> hipError_t launch_dq(const AttnArgs& a, float* delta, hipStream_t s) {
    using T = AttnTile<E, DP>;
    constexpr int tiles = (backward_ahead<E, DP>() ? 2 : 1) * 2 * T::BYTES, halves = WIDE ? 0 : 2 * 1024 * (T::ES == 2 ? 2 : 1) * T::NV * 4, bytes = tiles > halves ? tiles : halves;
    static_assert(bytes <= 160 * 1024, "LDS budget");
    constexpr int own = WIDE ? 128 : 64;
    const int row_tiles = (a.H / a.Hkv * a.Sq + own - 1) / own;
    const long long total = (long long)a.B * a.Hkv * row_tiles;
    if (total > 0xfffff0LL) return hipErrorInvalidValue;
    auto kern = attention_dq_kernel<E, DP, WIDE>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (attr != hipSuccess) return attr;
    const int per_xcd = (int)((total + 7) / 8);
    hipLaunchKernelGGL(kern, dim3((unsigned)(per_xcd * 8)), dim3(256), bytes, s, a, delta, row_tiles, (int)total, per_xcd);
    return hipGetLastError();
}
template <typename E, int DP, bool WIDE> hipError_t launch_dkv(const AttnArgs& a, const BackwardParts& parts, int nsplit, hipStream_t s) {
    using T = AttnTile<E, DP>;
    constexpr int tiles = (backward_ahead<E, DP>() ? 2 : 1) * (2 * T::BYTES + 2 * T::ROWS * 4), halves = WIDE ? 0 : 4 * 1024 * T::NV * 4, bytes = tiles > halves ? tiles : halves;
    static_assert(bytes <= 160 * 1024, "LDS budget");
    constexpr int own = WIDE ? 128 : 64;
    const int key_tiles = (a.Skv + own - 1) / own;
    const long long total = (long long)a.B * a.Hkv * key_tiles * nsplit;
    if (total > 0xfffff0LL) return hipErrorInvalidValue;
    auto kern = attention_dkv_kernel<E, DP, WIDE>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (attr != hipSuccess) return attr;
    const int per_xcd = (int)((total + 7) / 8);
    hipLaunchKernelGGL(kern, dim3((unsigned)(per_xcd * 8)), dim3(256), bytes, s, a, parts, key_tiles, nsplit, (int)total, per_xcd);
    return hipGetLastError();
}
size_t align_floats(size_t n) { return (n + 63) / 64 * 64; }

}  // namespace

size_t attention_backward_ws_bytes(int B, int Sq, int Skv, int H, int Hkv, int D, int dt) {
    const int n = backward_ranges(B, Sq, Skv, H, Hkv, D, dt);
    return (align_floats((size_t)B * H * Sq) + (n == 1 ? 0 : 2 * (size_t)n * B * Hkv * Skv * D)) * sizeof(float);
}

hipError_t launch_attention_backward(const AttnArgs& a, int dt, hipStream_t s) {
    const int nsplit = backward_ranges(a.B, a.Sq, a.Skv, a.H, a.Hkv, a.D, dt);
    const long long all = (long long)a.B * a.H * a.Sq, joins = ((long long)a.B * a.Hkv * a.Skv * (a.D / 4) + 255) / 256;
    if (nsplit > 1 && joins > 0xffffffLL) return hipErrorInvalidValue;
    BackwardParts parts{a.ws, nullptr, nullptr};
    if (nsplit > 1) {
        parts.dk = a.ws + align_floats((size_t)all);
        parts.dv = parts.dk + (size_t)nsplit * a.B * a.Hkv * a.Skv * a.D;
    }
    return with_dtype(dt, [&](auto* tag) -> hipError_t {
        using E = std::remove_pointer_t<decltype(tag)>;
        const hipError_t rc = with_channels(a.D, [&](auto dp) -> hipError_t {
            constexpr int DP = decltype(dp)::value;
            if constexpr (sizeof(E) == 4 && DP > 10) return hipErrorInvalidValue;
            else {
                const bool wide_q = own_wide((long long)a.B * a.Hkv, a.H / a.Hkv * a.Sq, dq_waves<E, DP>(), sizeof(E) == 4);
                const bool wide_k = own_wide((long long)a.B * a.Hkv * nsplit, a.Skv, backward_waves<E, DP>(), sizeof(E) == 4);
                const hipError_t e = wide_q ? launch_dq<E, DP, true>(a, parts.delta, s) : launch_dq<E, DP, false>(a, parts.delta, s);
                if (e != hipSuccess) return e;
                return wide_k ? launch_dkv<E, DP, true>(a, parts, nsplit, s) : launch_dkv<E, DP, false>(a, parts, nsplit, s);
            }
        });
        if (rc != hipSuccess || nsplit == 1) return rc;
        hipLaunchKernelGGL((attention_dkv_join_kernel<E>), dim3((unsigned)joins), dim3(256), 0, s, a, parts, nsplit);
        return hipGetLastError();
    });
}

}  // namespace wino
