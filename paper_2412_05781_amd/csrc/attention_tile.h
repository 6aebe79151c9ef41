// LDS tiles of the attention kernels: rows of one head's channels, read along the row (scores: the reduction runs over channels) and across the
// rows (products with the weights: the reduction runs over rows).
//
// 32x32 MFMA accumulators hold, in register r of lane l, row 8 (r / 4) + 4 (l / 32) + r % 4 and column l % 32.  Scores are formed with the streamed
// rows in the accumulator's rows and the wave's own 32 rows in its columns, one per lane.  The weights of a lane are then, register by register, an
// operand of the next product as they stand, if the other operand takes the streamed rows in the same order: element j of half h of step t is row
// 16 t + 8 (j / 4) + 4 h + j % 4 for two-byte types, 8 t + 4 h + j for fp32.  Nothing is exchanged between lanes or passed through LDS.
#pragma once
#include "block_act.h"
#include "wino_mma.h"

namespace wino {

typedef short attn_s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) attn_s16x4_t attn_lds_s16x4_t;

// DP: channels / 16, rounded up
template <typename E, int DP> struct AttnTile {
    static constexpr int ES = (int)sizeof(E);
    static constexpr int NV = (DP + 1) / 2;                     // 32-channel blocks
    static constexpr int KS = ES == 2 ? DP : 2 * DP;            // MFMA steps over the channels
    static constexpr int CPR = 2 * KS;                          // 16-byte chunks of a row that a score reads
    static constexpr int V = 16 / ES;                           // elements per chunk
    static constexpr int ST = ES == 2 ? 2 : 4;                  // MFMA steps over 32 streamed rows
    static constexpr int ROWS = 64;                             // streamed rows per tile
    // Two-byte types: an odd multiple of 64 bytes, and the low bits of the chunk flipped by (row / 4) % 4: sixteen rows read at one chunk and four rows
    // read at 64 neighbouring bytes both touch every bank once.  fp32: an odd number of chunks.
    static constexpr int STRIDE = ES == 2 ? 64 * (NV | 1) : NV * 128 + 16;
    static constexpr int BYTES = ROWS * STRIDE;
    static constexpr int LOADS = (ROWS * CPR + 255) / 256;      // chunks per thread and tile

    static __device__ __forceinline__ int at(int row, int chunk) {
        return row * STRIDE + ((ES == 2 ? chunk ^ ((row >> 2) & 3) : chunk) << 4);
    }
    // Where a lane reads.  Rows start at multiples of 32 (two-byte types: or 16), which leave the flipped bits alone, so that a read is one of four places per
    // lane and a constant: row lane % 32 along the channels (two-byte types: even and odd steps), or its rows and channel across.
    struct Places {
        int along[2], across[2];
        __device__ __forceinline__ explicit Places(int lane) {
            const int half = lane >> 5, row = lane & 31;
            along[0] = at(row, half);
            along[1] = at(row, 2 + half);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if constexpr (ES == 2) {                       // four rows x 16 channels per 16 lanes and read; lane i of the 16 gets channel i
                    const int col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
                    across[k] = at(8 * k + 4 * half + ((lane & 15) >> 2), col >> 3) + ((col & 4) << 1);
                } else {
                    across[k] = at(4 * half, row >> 2) + ((row & 3) << 2);
                }
            }
        }
    };
    // row row0 + lane % 32, channels of step ks
    static __device__ __forceinline__ u32x4_t along(const unsigned char* t, int row0, int ks, const Places& p) {
        const int place = ES == 2 ? p.along[ks & 1] + (ks >> 1) * 64 : p.along[0] + ks * 32;
        return *reinterpret_cast<const u32x4_t*>(t + row0 * STRIDE + place);
    }
    // channel 32 dt + lane % 32, rows of step st from row0
    static __device__ __forceinline__ u32x4_t across(const unsigned char* t, int row0, int st, int dt, const Places& p) {
        u32x4_t f;
        if constexpr (ES == 2) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const attn_s16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((attn_lds_s16x4_t*)(t + (row0 + 16 * st) * STRIDE + p.across[k] + dt * 64));
                const uint2 w = __builtin_bit_cast(uint2, v);
                f[2 * k] = w.x;
                f[2 * k + 1] = w.y;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = *reinterpret_cast<const uint32_t*>(t + (row0 + 8 * st + j) * STRIDE + p.across[0] + dt * 128);
        }
        return f;
    }
    // Step st of 32 weights in accumulator order, rounded to the storage type: a matrix instruction takes both operands in one type.  Of the error of o against 64 bits
    // (bf16, 4096 keys) 1.7e-3 is its own rounding and 1.5e-3 this one, 2.3e-3 together; the sum that divides is of the weights before it.
    static __device__ __forceinline__ u32x4_t weights(const float16_t& p, int st) {
        u32x4_t f;
        if constexpr (ES == 2) {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = pack_pair<E>(p[8 * st + 2 * j], p[8 * st + 2 * j + 1]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = __float_as_uint(p[4 * st + j]);
        }
        return f;
    }
};

// A thread's share (of 256) of the tiles of 64 rows that a workgroup streams: chunks of 16 bytes, on their way in registers until they are put into LDS.
template <typename E, int DP> struct AttnStream {
    using T = AttnTile<E, DP>;
    static constexpr int N = T::LOADS;
    static constexpr bool EVEN = T::ROWS * T::CPR % 256 == 0;   // every thread has N chunks
    struct Map {                                                // where the chunks lie, the same for every tensor
        int row[N], at[N], byte[N];
        bool on[N];                                             // holds channels at all (a head's last chunk, and threads behind the tile's end, may not)
        bool whole;                                             // uniform: all do
        __device__ __forceinline__ Map(int tid, int D) {
            whole = EVEN && D == DP * 16;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int id = tid + 256 * i, r = id / T::CPR, chunk = id - r * T::CPR;
                on[i] = r < T::ROWS && chunk * T::V < D;
                row[i] = r & 63;
                byte[i] = chunk * 16;
                at[i] = r < T::ROWS ? T::at(r, chunk) : -1;
            }
        }
    };
    u32x4_t f[N];
    const unsigned char* p[N];
    long long step;
    // rows from `first` on of a tensor with `stride` elements between rows
    __device__ __forceinline__ AttnStream(const Map& m, const unsigned char* base, long long first, long long stride) {
        step = (long long)T::ROWS * stride * T::ES;
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = base + (first + m.row[i]) * stride * T::ES + m.byte[i];
    }
    // the next tile; rows whose bit is clear are zero and not read
    __device__ __forceinline__ void fetch(const Map& m, unsigned long long rows) {
        const u32x4_t zero = {0, 0, 0, 0};
        if (m.whole && rows == ~0ull) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = *reinterpret_cast<const u32x4_t*>(p[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = m.on[i] && ((rows >> m.row[i]) & 1) ? *reinterpret_cast<const u32x4_t*>(p[i]) : zero;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] += step;
    }
    __device__ __forceinline__ void jump(long long bytes) {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] += bytes;
    }
    __device__ __forceinline__ void put(const Map& m, unsigned char* tile) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (EVEN || m.at[i] >= 0) *reinterpret_cast<u32x4_t*>(tile + m.at[i]) = f[i];
    }
};

// The rows that a key head's queries are dealt with as: r = g * Sq + s for query head hk * G + g, so that heads which share keys share a tile.
struct AttnRows {
    int Sq, R;                       // R = G * Sq
    __device__ __forceinline__ const unsigned char* at(const AttnTensor& t, int G, int b, int hk, int r, int es) const {
        const int g = r / Sq, s = r - g * Sq;
        return static_cast<const unsigned char*>(t.p) + ((long long)b * t.b + (long long)s * t.s + (long long)(hk * G + g) * t.h) * es;
    }
};

// 16 bytes at channel c of a row, zero behind the head's D channels (D is a multiple of 8)
template <typename E> __device__ __forceinline__ u32x4_t load_channels(const unsigned char* row, int c, int D) {
    const u32x4_t zero = {0, 0, 0, 0};
    return c < D ? *reinterpret_cast<const u32x4_t*>(row + c * (int)sizeof(E)) : zero;
}

// four channels of one row
template <typename E> __device__ __forceinline__ void store_channels(unsigned char* row, int c, int D, const float* v) {
    if (c >= D) return;
    if constexpr (sizeof(E) == 4) *reinterpret_cast<float4*>(row + c * 4) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2*>(row + c * 2) = make_uint2(pack_pair<E>(v[0], v[1]), pack_pair<E>(v[2], v[3]));
}

// Valid keys among 64, one bit each: below the row's length and not masked.  A tile's mask is requested a tile before its bits are asked for, so that
// the loads of keys and values do not wait for it (and the first one not for the length).  Called by whole waves.
struct KeyMask {
    const unsigned char* mask;       // null: every key
    int Skv;
    uint32_t raw = 1;
    __device__ __forceinline__ KeyMask(const AttnArgs& a, int b) : mask(a.key_mask ? a.key_mask + (long long)b * a.Skv : nullptr), Skv(a.Skv) {}
    __device__ __forceinline__ void request(int key0) {
        const int key = key0 + (int)(threadIdx.x & 63);
        if (mask) raw = key < Skv ? mask[key] : 0;
    }
    // of the tile requested last
    __device__ __forceinline__ unsigned long long bits(int key0, int len) const { return __ballot(key0 + (int)(threadIdx.x & 63) < len && raw); }
};
__device__ __forceinline__ int key_count(const AttnArgs& a, int b) {
    if (!a.kv_len) return a.Skv;
    const int n = a.kv_len[b];
    return n < 0 ? 0 : n < a.Skv ? n : a.Skv;
}

// Each XCD runs a contiguous range of the workgroups' order, whole heads after one another, so that a head's streamed rows stay in one L2.  Lengths differ
// between the batch's rows, not between heads: where the heads divide evenly, neighbours go to different XCDs.
__device__ __forceinline__ int deal_heads(int bh, int heads) {
    return heads % 8 ? bh : (bh % (heads / 8)) * 8 + bh / (heads / 8);
}

constexpr float kLog2e = 1.44269504f, kLn2 = 0.69314718f;

// channels / 16 as a compile-time number
template <typename F> hipError_t with_channels(int D, F&& f) {
    const int n = (D + 15) / 16;
    if (n <= 2) return f(std::integral_constant<int, 2>());
    if (n == 3) return f(std::integral_constant<int, 3>());
    if (n == 4) return f(std::integral_constant<int, 4>());
    if (n == 5) return f(std::integral_constant<int, 5>());
    if (n == 6) return f(std::integral_constant<int, 6>());
    if (n <= 8) return f(std::integral_constant<int, 8>());
    if (n <= 10) return f(std::integral_constant<int, 10>());
    return f(std::integral_constant<int, 16>());
}

}  // namespace wino
