// Declarations shared by the sources of the transformer-block operators: matrix products with an epilogue (linear.hip), the gated
// feed-forward block (the same products, two weight blocks per tile) and attention (attention.hip, attention_backward.hip).
#pragma once
#include "wino_internal.h"

namespace wino {

// Values of wino_act.
enum { ACT_NONE = 0, ACT_SILU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3 };

// out[m][n] = sum_k Q(m,k) P(n,k).  An operand is stored with its reduction index contiguous, element (i,k) at p[i*ld + k], or
// transposed, element (i,k) at p[k*ld + i].
struct Operand {
    const void* p;
    long long ld;
};

// What becomes of the sums of a tile.
enum {
    EP_STORE = 0,      // out = sum
    EP_LINEAR = 1,     // out = act(sum + bias) + extra                     (extra: residual, may be null)
    EP_DLINEAR = 2,    // out = extra * act'(sum + bias)                    (extra: dy);       column sums of out to `sums`
    EP_GLU = 3,        // out = u * act(g)                                  u, g: rows n and N + n of P
    EP_DGLU = 4,       // out[n] = extra * act(g), out[N+n] = extra * u * act'(g)  (extra: dh); column sums of out to `sums`
    EP_PART = 5        // fp32 sums of one range of the reduction to `part`
};

struct Epilogue {
    const float* bias = nullptr;     // [N], EP_GLU / EP_DGLU [2N]; may be null
    const void* extra = nullptr;     // [M][N] in the storage type
    long long ld_extra = 0;
    void* out = nullptr;
    long long ld_out = 0;
    float* sums = nullptr;           // [sum_rows][width of out]
    float* part = nullptr;           // [nsplit][M][N]
    float* tops = nullptr;           // EP_DLINEAR / EP_DGLU in fp16: the largest finite magnitude of out (before its rounding), by wave; may be null
    const int* power = nullptr;      // EP_DLINEAR / EP_DGLU in fp16: out is formed again times 2^*power, or left alone where that is 0.  EP_STORE and joins: result
                                     // times 2^-*power.  May be null
    int act = ACT_NONE;
};

// how many rows of sums and how many tops a launch with EP_DLINEAR / EP_DGLU fills
struct Filled { int sum_rows; long long tops; };

// M rows and N columns of out (EP_GLU / EP_DGLU: N gate pairs, P has 2N rows), reduction length K.
struct GemmShape { int M, N, K; };

// A product with its ranges: e.part set where there are several.
struct Product { Operand P, Q; GemmShape g; Epilogue e; int nsplit; };

bool gemm_dims_ok(long long M, long long N, long long K);
// whether the kernel for operands that can be fetched 16 bytes at a time (linear_tile.hip) takes a call
bool tile_gemm_ok(int ep, bool p_trans, bool q_trans, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int dt);
// rows of Epilogue::sums and number of Epilogue::tops that a launch with EP_DLINEAR / EP_DGLU may fill; launch_gemm says how many it did (may be null)
int gemm_most_sum_rows(int M);
long long gemm_most_tops(int M, int N);
// ranges the reduction of a plain product (EP_STORE, EP_LINEAR) is cut into
int gemm_ranges(int M, int N, int K, int dt);
hipError_t launch_gemm(int ep, bool p_trans, bool q_trans, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int nsplit,
                       int dt, hipStream_t s, Filled* filled = nullptr);
// Sums over the rows of x[M][N], in `ranges` ranges: out[range][n].  out null: not asked for.  f32: x is fp32 whatever the call's type, in one range.
struct ColumnSums { const void* x; long long ld; int M, N; float* out; int ranges; bool f32; };
// a = dz w (P across, Q along the reduction) and b = dz^T x (both across), with EP_STORE or ranges; and the column sums c
hipError_t launch_gemm_pair(const Product& a, const Product& b, const ColumnSums& c, int dt, hipStream_t s);
// x W^T with EP_LINEAR or (glu) EP_GLU for few rows, one kernel, no workspace.  Whether it is taken; tiles: whether the kernel for aligned operands is the other choice
// (true never takes it where false does not)
bool few_gemm_ok(bool glu, int M, int N, int K, int dt, bool tiles);
hipError_t launch_few_gemm(bool glu, const Operand& P, const Operand& Q, const GemmShape& g, const Epilogue& e, int dt, hipStream_t s);
// out = act(sum over ranges + bias) + extra
hipError_t launch_join(const float* part, int nsplit, const GemmShape& g, const Epilogue& e, int dt, hipStream_t s);
// out[c] = sum over rows of part[row][c]
hipError_t launch_sum_rows(const float* part, int rows, int cols, float* out, hipStream_t s);
// the power of two for an fp16 tensor whose largest finite magnitude is the largest of `tops`: 0 where it fits and keeps its bits as it is
hipError_t launch_power(const float* tops, long long n, int* power, hipStream_t s);
int column_sum_rows(int M);
hipError_t launch_column_sums(const ColumnSums& c, int dt, hipStream_t s);

// One call of the attention operators; strides in elements, the last dimension contiguous.
struct AttnTensor { const void* p; long long b, s, h; };
struct AttnArgs {
    int B, Sq, Skv, H, Hkv, D;
    float scale;
    AttnTensor q, k, v, o, dout;
    AttnTensor dq, dk, dv;
    float* lse;                      // [B][H][Sq], natural logarithm; may be null in the forward pass
    const int* kv_len;               // [B] or null
    const unsigned char* key_mask;   // [B][Skv] or null
    float* ws;
};
size_t attention_ws_bytes(int B, int Sq, int Skv, int H, int Hkv, int D, int dt);
size_t attention_backward_ws_bytes(int B, int Sq, int Skv, int H, int Hkv, int D, int dt);
hipError_t launch_attention(const AttnArgs& a, int dt, hipStream_t s);
hipError_t launch_attention_backward(const AttnArgs& a, int dt, hipStream_t s);

}  // namespace wino
