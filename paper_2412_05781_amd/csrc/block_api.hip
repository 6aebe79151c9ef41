// C-ABI boundary of the transformer-block operators: argument validation on the host, workspace carving, and the chains of launches.
// Nothing here computes.
#include "../../include/wino.h"
#include "block_internal.h"

#include <math.h>

using namespace wino;

namespace {

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
inline bool at16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool at4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool is_dtype(int d) { return d == WINO_F32 || d == WINO_F16 || d == WINO_BF16; }
inline bool is_act(int a) { return a >= WINO_ACT_NONE && a <= WINO_ACT_GELU_TANH; }
inline size_t bytes_of(int d) { return d == WINO_F32 ? 4 : 2; }

// bytes from the first to behind the last element of `rows` rows of `cols`
inline size_t extent(long long rows, long long ld, long long cols, size_t es) { return ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * es; }
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && x < y + nb && y < x + na;
}
inline bool ld_ok(long long ld, long long cols) { return ld >= cols && ld <= (1LL << 36); }

// product out[M][N] = Q P^T in one launch or as ranges that are joined; `scratch` holds the ranges' sums
size_t product_bytes(int M, int N, int K, int dt) {
    const int n = gemm_ranges(M, N, K, dt);
    return n == 1 ? 0 : up256((size_t)n * M * N * sizeof(float));
}
hipError_t product(int ep, bool pt, bool qt, const Operand& P, const Operand& Q, const GemmShape& g, Epilogue e, void* scratch, int dt, hipStream_t s) {
    const int n = gemm_ranges(g.M, g.N, g.K, dt);
    if (n == 1) return launch_gemm(ep, pt, qt, P, Q, g, e, 1, dt, s);
    e.part = static_cast<float*>(scratch);
    const hipError_t rc = launch_gemm(EP_PART, pt, qt, P, Q, g, e, n, dt, s);
    return rc != hipSuccess ? rc : launch_join(e.part, n, g, e, dt, s);
}

// workspace of a backward pass over W output columns (`halves` of them a column of dy): dz, the column sums, the ranges' sums; fp16: the largest of dz by wave and their power
struct BackwardSpace { size_t dz, sums, parts, tops, total; long long ld; Filled filled; };
BackwardSpace backward_space(int M, int W, int K, int dt, bool stored, int halves) {
    BackwardSpace b;
    b.ld = ((long long)W + 7) / 8 * 8;
    b.dz = stored ? up256((size_t)M * b.ld * bytes_of(dt)) : 0;
    b.filled = Filled{stored ? gemm_most_sum_rows(M) : column_sum_rows(M), stored && dt == WINO_F16 ? gemm_most_tops(M, W / halves) : 0};
    b.sums = up256((size_t)b.filled.sum_rows * W * sizeof(float));
    b.parts = product_bytes(M, K, W, dt) + product_bytes(W, K, M, dt);
    b.tops = b.filled.tops ? 256 + up256((size_t)b.filled.tops * sizeof(float)) : 0;
    b.total = b.dz + b.sums + b.parts + b.tops;
    return b;
}

// dx = dz w and dw = dz^T x, in one launch where both are asked for; and the column sums of dz
int run_products(const void* x, long long ldx, const void* w, const void* dz, long long lddz, void* dx, long long lddx, void* dw, const ColumnSums& c, const int* power,
                 int M, int W, int K, void* scratch, int dt, hipStream_t s) {
    Product a{Operand{w, K}, Operand{dz, lddz}, GemmShape{M, K, W}, Epilogue(), gemm_ranges(M, K, W, dt)};
    Product b{Operand{x, ldx}, Operand{dz, lddz}, GemmShape{W, K, M}, Epilogue(), gemm_ranges(W, K, M, dt)};
    a.e.out = dx; a.e.ld_out = lddx;
    b.e.out = dw; b.e.ld_out = K;
    a.e.power = b.e.power = power;
    if ((!dx || !dw) && c.out && launch_column_sums(c, dt, s) != hipSuccess) return WINO_ERR_HIP;
    if (!dx && !dw) return WINO_OK;
    if (!dw) return product(EP_STORE, true, false, a.P, a.Q, a.g, a.e, scratch, dt, s) == hipSuccess ? WINO_OK : WINO_ERR_HIP;
    if (!dx) return product(EP_STORE, true, true, b.P, b.Q, b.g, b.e, scratch, dt, s) == hipSuccess ? WINO_OK : WINO_ERR_HIP;
    unsigned char* base = static_cast<unsigned char*>(scratch);
    if (a.nsplit > 1) a.e.part = reinterpret_cast<float*>(base);
    if (b.nsplit > 1) b.e.part = reinterpret_cast<float*>(base + product_bytes(M, K, W, dt));
    if (launch_gemm_pair(a, b, c, dt, s) != hipSuccess) return WINO_ERR_HIP;
    for (const Product* p : {&a, &b})
        if (p->nsplit > 1 && launch_join(p->e.part, p->nsplit, p->g, p->e, dt, s) != hipSuccess) return WINO_ERR_HIP;
    return WINO_OK;
}

bool product_dims_ok(int M, int N, int K, int halves) {
    if (M < 1 || N < 1 || K < 1 || N > (1 << 26)) return false;
    const long long W = (long long)N * halves;
    return gemm_dims_ok(M, W, K) && gemm_dims_ok(M, K, W) && gemm_dims_ok(W, K, M);
}

// One call for both backward passes: `halves` rows of w per output column.  dz is stored in the type of dy, because it is an operand of the two products after it and a matrix
// instruction takes both operands in one type; a rounding more than its own in dx and dw (bf16, 4096 x 640 x 2560: error against 64 bits 2.3e-3 where one rounding is 1.7e-3).
int products_backward(const void* x, const void* w, const float* bias, const void* dy, void* dx, void* dw, float* dbias, int M, int N, int K, long long ldx,
                      long long lddy, long long lddx, int dt, int act, int halves, void* workspace, size_t workspace_bytes, void* stream) {
    if (!x || !w || !dy || (!dx && !dw && !dbias)) return WINO_ERR_NULL;
    if (!is_dtype(dt)) return WINO_ERR_DTYPE;
    if (!is_act(act)) return WINO_ERR_VARIANT;
    if (!product_dims_ok(M, N, K, halves) || !ld_ok(ldx, K) || !ld_ok(lddy, N) || (dx && !ld_ok(lddx, K))) return WINO_ERR_DIM;
    if (!at16(x) || !at16(w) || !at16(dy) || !at16(dx) || !at16(dw) || !at4(bias) || !at4(dbias)) return WINO_ERR_ALIGN;
    const int W = N * halves;
    const size_t es = bytes_of(dt);
    const struct { const void* p; size_t n; } in[4] = {{x, extent(M, ldx, K, es)}, {w, (size_t)W * K * es}, {dy, extent(M, lddy, N, es)}, {bias, (size_t)W * 4}},
                                              out[3] = {{dx, dx ? extent(M, lddx, K, es) : 0}, {dw, (size_t)W * K * es}, {dbias, (size_t)W * 4}};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 4; ++j) if (overlap(out[i].p, out[i].n, in[j].p, in[j].n)) return WINO_ERR_ALIAS;
        for (int j = 0; j < i; ++j) if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return WINO_ERR_ALIAS;
    }
    const bool stored = halves == 2 || act != WINO_ACT_NONE;
    BackwardSpace b = backward_space(M, W, K, dt, stored, halves);
    if (!workspace || workspace_bytes < b.total) return WINO_ERR_WORKSPACE;
    if (!at16(workspace)) return WINO_ERR_ALIGN;
    for (const auto& t : in) if (overlap(workspace, b.total, t.p, t.n)) return WINO_ERR_ALIAS;
    for (const auto& t : out) if (overlap(workspace, b.total, t.p, t.n)) return WINO_ERR_ALIAS;
    hipStream_t s = static_cast<hipStream_t>(stream);
    unsigned char* base = static_cast<unsigned char*>(workspace);
    float* sums = reinterpret_cast<float*>(base + b.dz);
    const void* dz = dy;
    long long lddz = lddy;
    ColumnSums c{dy, lddy, M, N, nullptr, b.filled.sum_rows, false};
    int* power = nullptr;
    if (stored) {
        Epilogue e;
        e.bias = bias; e.extra = dy; e.ld_extra = lddy; e.out = base; e.ld_out = b.ld; e.sums = sums; e.act = act;
        const int ep = halves == 2 ? EP_DGLU : EP_DLINEAR;
        if (b.tops && (dx || dw)) {
            power = reinterpret_cast<int*>(base + b.dz + b.sums + b.parts);
            e.tops = reinterpret_cast<float*>(power) + 64;
        }
        if (launch_gemm(ep, false, false, Operand{w, K}, Operand{x, ldx}, GemmShape{M, N, K}, e, 1, dt, s, &b.filled) != hipSuccess) return WINO_ERR_HIP;
        if (power) {
            if (launch_power(e.tops, b.filled.tops, power, s) != hipSuccess) return WINO_ERR_HIP;
            e.tops = nullptr; e.power = power;
            if (launch_gemm(ep, false, false, Operand{w, K}, Operand{x, ldx}, GemmShape{M, N, K}, e, 1, dt, s) != hipSuccess) return WINO_ERR_HIP;
        }
        dz = base; lddz = b.ld;
        if (dbias) c = ColumnSums{sums, W, b.filled.sum_rows, W, dbias, 1, true};
    } else if (dbias) {
        c.out = b.filled.sum_rows == 1 ? dbias : sums;
    }
    const int rc = run_products(x, ldx, w, dz, lddz, dx, lddx, dw, c, power, M, W, K, base + b.dz + b.sums, dt, s);
    if (rc != WINO_OK || !dbias || c.out == dbias) return rc;
    return launch_sum_rows(sums, b.filled.sum_rows, W, dbias, s) == hipSuccess ? WINO_OK : WINO_ERR_HIP;
}

// ---- attention ------------------------------------------------------------------------------------------------------------------------
bool attention_dims_ok(int B, int Sq, int Skv, int H, int Hkv, int D, int dt) {
    if (B < 1 || Sq < 1 || Skv < 1 || H < 1 || Hkv < 1 || H % Hkv || D < 8 || D % 8 || D > (dt == WINO_F32 ? 160 : 256)) return false;
    // (a launch has less than 2^32 threads: 2^24 workgroups of 256, one per 64 or more rows of a head)
    const long long most = 1LL << 29, elements = 1LL << 40;
    return (long long)H * Sq <= most && Skv <= most && (long long)B * Hkv <= (1LL << 22) && (long long)B * H * Sq <= most && (long long)B * H * Sq * D <= elements &&
           (long long)B * Hkv * Skv <= most && (long long)B * Hkv * Skv * D <= elements;
}
int tensor_status(const wino_tensor& t, size_t es, bool out, int B, int S, int H) {
    if (!t.data) return WINO_ERR_NULL;
    const long long st[3] = {t.stride_b, t.stride_s, t.stride_h};
    const int n[3] = {B, S, H};
    for (int i = 0; i < 3; ++i) {
        if (n[i] == 1) continue;                           // a stride that is not used
        if (st[i] < 0 || st[i] > (1LL << 36) || (out && st[i] == 0)) return WINO_ERR_DIM;
        if (((size_t)st[i] * es) & 15u) return WINO_ERR_ALIGN;
    }
    return at16(t.data) ? WINO_OK : WINO_ERR_ALIGN;
}
size_t tensor_extent(const wino_tensor& t, size_t es, int B, int S, int H, int D) {
    return ((size_t)(B > 1 ? (B - 1) * t.stride_b : 0) + (size_t)(S > 1 ? (S - 1) * t.stride_s : 0) + (size_t)(H > 1 ? (H - 1) * t.stride_h : 0) + (size_t)D) * es;
}

// A tensor as a lattice of runs of D elements, the widest stride first; dimensions of one position have none.
struct Lattice { long long stride[3]; int n[3]; int dims; };
// Of one tensor, or of two that lie among each other: false where they do not have the same strides.
bool lattices(const wino_tensor& x, const int (&nx)[3], const wino_tensor& y, const int (&ny)[3], Lattice& a, Lattice& b) {
    const long long sx[3] = {x.stride_b, x.stride_s, x.stride_h}, sy[3] = {y.stride_b, y.stride_s, y.stride_h};
    a.dims = b.dims = 0;
    for (int i = 0; i < 3; ++i) {
        if (nx[i] == 1 && ny[i] == 1) continue;
        if (nx[i] > 1 && ny[i] > 1 && sx[i] != sy[i]) return false;
        const long long st = nx[i] > 1 ? sx[i] : sy[i];
        int at = a.dims++;
        b.dims = a.dims;
        for (; at > 0 && a.stride[at - 1] < st; --at) { a.stride[at] = a.stride[at - 1]; a.n[at] = a.n[at - 1]; b.n[at] = b.n[at - 1]; }
        a.stride[at] = st; a.n[at] = nx[i]; b.n[at] = ny[i];
    }
    for (int i = 0; i < 3; ++i) b.stride[i] = a.stride[i];
    return true;
}
// each stride spans what the narrower ones reach
bool nested(const Lattice& a, int D) {
    long long reach = D;
    for (int i = a.dims - 1; i >= 0; --i) {
        if (a.stride[i] < reach) return false;
        reach += (a.n[i] - 1) * a.stride[i];
    }
    return true;
}
// whether a position of a and one of b meet, with b `d` elements behind a; both nested, so that a level's difference is one of the two nearest d
bool meet(const Lattice& a, const Lattice& b, int level, long long d, int D) {
    if (level == a.dims) return d > -D && d < D;
    const long long st = a.stride[level], least = -(long long)(b.n[level] - 1), most = a.n[level] - 1;
    const long long down = (d >= 0 ? d : d - st + 1) / st;
    for (long long i = down; i <= down + 1; ++i)
        if (i >= least && i <= most && meet(a, b, level + 1, d - i * st, D)) return true;
    return false;
}
// Gradients may share a packed buffer: tensors of the same strides whose positions lie between each other's.
bool gradients_meet(const wino_tensor& x, const int (&nx)[3], const wino_tensor& y, const int (&ny)[3], int D, size_t es) {
    Lattice a, b;
    if (!lattices(x, nx, y, ny, a, b) || !nested(a, D) || !nested(b, D)) return true;
    const long long bytes = (long long)(reinterpret_cast<uintptr_t>(y.data) - reinterpret_cast<uintptr_t>(x.data));
    return meet(a, b, 0, bytes / (long long)es, D);        // (addresses are multiples of 16)
}

AttnTensor inner(const wino_tensor& t) { return AttnTensor{t.data, t.stride_b, t.stride_s, t.stride_h}; }

int attention_status(const wino_attention_args* a, bool backward, const void* workspace, size_t workspace_bytes) {
    if (!a) return WINO_ERR_NULL;
    if (!is_dtype(a->dtype)) return WINO_ERR_DTYPE;
    if (!attention_dims_ok(a->B, a->Sq, a->Skv, a->H, a->Hkv, a->D, a->dtype) || !(a->scale > 0.f) || !isfinite(a->scale)) return WINO_ERR_DIM;
    const size_t es = bytes_of(a->dtype);
    struct Item { const wino_tensor* t; bool out, key; };
    const Item fwd[4] = {{&a->q, false, false}, {&a->k, false, true}, {&a->v, false, true}, {&a->o, true, false}};
    const Item bwd[8] = {{&a->q, false, false}, {&a->k, false, true}, {&a->v, false, true}, {&a->o, false, false},
                         {&a->d_o, false, false}, {&a->dq, true, false}, {&a->dk, true, true}, {&a->dv, true, true}};
    const Item* items = backward ? bwd : fwd;
    const int n = backward ? 8 : 4;
    for (int i = 0; i < n; ++i) {
        const int rc = tensor_status(*items[i].t, es, items[i].out, a->B, items[i].key ? a->Skv : a->Sq, items[i].key ? a->Hkv : a->H);
        if (rc != WINO_OK) return rc;
    }
    auto count = [&](const Item& x, int (&c)[3]) { c[0] = a->B; c[1] = x.key ? a->Skv : a->Sq; c[2] = x.key ? a->Hkv : a->H; };
    for (int i = 0; i < n; ++i) {
        if (!items[i].out) continue;
        int c[3];
        Lattice l, same;
        count(items[i], c);
        if (!lattices(*items[i].t, c, *items[i].t, c, l, same) || !nested(l, a->D)) return WINO_ERR_DIM;
    }
    if (backward && !a->lse) return WINO_ERR_NULL;
    if (!at4(a->lse) || !at4(a->kv_len)) return WINO_ERR_ALIGN;
    auto size = [&](const Item& x) { return tensor_extent(*x.t, es, a->B, x.key ? a->Skv : a->Sq, x.key ? a->Hkv : a->H, a->D); };
    for (int i = 0; i < n; ++i) {
        if (!items[i].out) continue;
        const void* p = items[i].t->data;
        const size_t np = size(items[i]);
        for (int j = 0; j < n; ++j) {
            if (j == i) continue;
            if (!overlap(p, np, items[j].t->data, size(items[j]))) continue;
            if (!items[j].out) return WINO_ERR_ALIAS;
            int ci[3], cj[3];
            count(items[i], ci);
            count(items[j], cj);
            if (gradients_meet(*items[i].t, ci, *items[j].t, cj, a->D, es)) return WINO_ERR_ALIAS;
        }
        if (overlap(p, np, a->lse, (size_t)a->B * a->H * a->Sq * 4) || overlap(p, np, a->kv_len, (size_t)a->B * 4) ||
            overlap(p, np, a->key_mask, (size_t)a->B * a->Skv))
            return WINO_ERR_ALIAS;
    }
    if (!backward && a->lse) {                             // an output there
        const size_t n_lse = (size_t)a->B * a->H * a->Sq * 4;
        for (int i = 0; i < 3; ++i) if (overlap(a->lse, n_lse, items[i].t->data, size(items[i]))) return WINO_ERR_ALIAS;
        if (overlap(a->lse, n_lse, a->kv_len, (size_t)a->B * 4) || overlap(a->lse, n_lse, a->key_mask, (size_t)a->B * a->Skv)) return WINO_ERR_ALIAS;
    }
    const size_t need = backward ? attention_backward_ws_bytes(a->B, a->Sq, a->Skv, a->H, a->Hkv, a->D, a->dtype) : attention_ws_bytes(a->B, a->Sq, a->Skv, a->H, a->Hkv, a->D, a->dtype);
    if (!need) return WINO_OK;
    if (!workspace || workspace_bytes < need) return WINO_ERR_WORKSPACE;
    if (!at16(workspace)) return WINO_ERR_ALIGN;
    for (int i = 0; i < n; ++i) if (overlap(workspace, need, items[i].t->data, size(items[i]))) return WINO_ERR_ALIAS;
    if (overlap(workspace, need, a->lse, (size_t)a->B * a->H * a->Sq * 4) || overlap(workspace, need, a->kv_len, (size_t)a->B * 4) ||
        overlap(workspace, need, a->key_mask, (size_t)a->B * a->Skv))
        return WINO_ERR_ALIAS;
    return WINO_OK;
}

AttnArgs attention_args(const wino_attention_args* a, void* workspace) {
    AttnArgs r{};
    r.B = a->B; r.Sq = a->Sq; r.Skv = a->Skv; r.H = a->H; r.Hkv = a->Hkv; r.D = a->D; r.scale = a->scale;
    r.q = inner(a->q); r.k = inner(a->k); r.v = inner(a->v); r.o = inner(a->o); r.dout = inner(a->d_o);
    r.dq = inner(a->dq); r.dk = inner(a->dk); r.dv = inner(a->dv);
    r.lse = a->lse; r.kv_len = a->kv_len; r.key_mask = a->key_mask;
    r.ws = static_cast<float*>(workspace);
    return r;
}

}  // namespace

extern "C" {

size_t wino_linear_workspace_bytes(int M, int N, int K, int dtype, int act) {
    if (!is_dtype(dtype) || !is_act(act) || !product_dims_ok(M, N, K, 1)) return 0;
    return few_gemm_ok(false, M, N, K, dtype, true) ? 0 : product_bytes(M, N, K, dtype);
}

int wino_linear(const void* x, const void* w, const float* bias, const void* residual, void* y, int M, int N, int K, long long ldx, long long ldr,
                long long ldy, int dtype, int act, void* workspace, size_t workspace_bytes, void* stream) {
    if (!x || !w || !y) return WINO_ERR_NULL;
    if (!is_dtype(dtype)) return WINO_ERR_DTYPE;
    if (!is_act(act)) return WINO_ERR_VARIANT;
    if (!product_dims_ok(M, N, K, 1) || !ld_ok(ldx, K) || !ld_ok(ldy, N) || (residual && !ld_ok(ldr, N))) return WINO_ERR_DIM;
    if (!at16(x) || !at16(w) || !at16(y) || !at16(residual) || !at4(bias)) return WINO_ERR_ALIGN;
    const size_t es = bytes_of(dtype), ny = extent(M, ldy, N, es);
    if (overlap(y, ny, x, extent(M, ldx, K, es)) || overlap(y, ny, w, (size_t)N * K * es) || overlap(y, ny, bias, (size_t)N * 4)) return WINO_ERR_ALIAS;
    if (residual && !(residual == y && ldr == ldy) && overlap(y, ny, residual, extent(M, ldr, N, es))) return WINO_ERR_ALIAS;
    Epilogue e;
    e.bias = bias; e.extra = residual; e.ld_extra = ldr; e.out = y; e.ld_out = ldy; e.act = act;
    const Operand P{w, K}, Q{x, ldx};
    const GemmShape g{M, N, K};
    const bool few = few_gemm_ok(false, M, N, K, dtype, tile_gemm_ok(EP_LINEAR, false, false, P, Q, g, e, dtype));
    const size_t need = few ? 0 : product_bytes(M, N, K, dtype);
    if (need && (!workspace || workspace_bytes < need)) return WINO_ERR_WORKSPACE;
    if (need) {
        if (!at16(workspace)) return WINO_ERR_ALIGN;
        if (overlap(workspace, need, y, ny) || overlap(workspace, need, x, extent(M, ldx, K, es)) || overlap(workspace, need, w, (size_t)N * K * es) ||
            overlap(workspace, need, bias, (size_t)N * 4) || overlap(workspace, need, residual, extent(M, ldr, N, es)))
            return WINO_ERR_ALIAS;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t rc = few ? launch_few_gemm(false, P, Q, g, e, dtype, s) : product(EP_LINEAR, false, false, P, Q, g, e, workspace, dtype, s);
    return rc == hipSuccess ? WINO_OK : WINO_ERR_HIP;
}

size_t wino_linear_backward_workspace_bytes(int M, int N, int K, int dtype, int act) {
    if (!is_dtype(dtype) || !is_act(act) || !product_dims_ok(M, N, K, 1)) return 0;
    return backward_space(M, N, K, dtype, act != WINO_ACT_NONE, 1).total;
}

int wino_linear_backward(const void* x, const void* w, const float* bias, const void* dy, void* dx, void* dw, float* dbias, int M, int N, int K, long long ldx,
                         long long lddy, long long lddx, int dtype, int act, void* workspace, size_t workspace_bytes, void* stream) {
    return products_backward(x, w, bias, dy, dx, dw, dbias, M, N, K, ldx, lddy, lddx, dtype, act, 1, workspace, workspace_bytes, stream);
}

size_t wino_glu_workspace_bytes(int, int, int, int, int) { return 0; }

int wino_glu(const void* x, const void* w, const float* bias, void* h, int M, int N, int K, long long ldx, long long ldh, int dtype, int act,
             void* workspace, size_t workspace_bytes, void* stream) {
    (void)workspace; (void)workspace_bytes;
    if (!x || !w || !h) return WINO_ERR_NULL;
    if (!is_dtype(dtype)) return WINO_ERR_DTYPE;
    if (!is_act(act)) return WINO_ERR_VARIANT;
    if (!product_dims_ok(M, N, K, 2) || !ld_ok(ldx, K) || !ld_ok(ldh, N)) return WINO_ERR_DIM;
    if (!at16(x) || !at16(w) || !at16(h) || !at4(bias)) return WINO_ERR_ALIGN;
    const size_t es = bytes_of(dtype), nh = extent(M, ldh, N, es);
    if (overlap(h, nh, x, extent(M, ldx, K, es)) || overlap(h, nh, w, 2 * (size_t)N * K * es) || overlap(h, nh, bias, 2 * (size_t)N * 4)) return WINO_ERR_ALIAS;
    Epilogue e;
    e.bias = bias; e.out = h; e.ld_out = ldh; e.act = act;
    const Operand P{w, K}, Q{x, ldx};
    const GemmShape g{M, N, K};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t rc = few_gemm_ok(true, M, N, K, dtype, false) ? launch_few_gemm(true, P, Q, g, e, dtype, s) : launch_gemm(EP_GLU, false, false, P, Q, g, e, 1, dtype, s);
    return rc == hipSuccess ? WINO_OK : WINO_ERR_HIP;
}

size_t wino_glu_backward_workspace_bytes(int M, int N, int K, int dtype, int act) {
    if (!is_dtype(dtype) || !is_act(act) || !product_dims_ok(M, N, K, 2)) return 0;
    return backward_space(M, 2 * N, K, dtype, true, 2).total;
}

int wino_glu_backward(const void* x, const void* w, const float* bias, const void* dh, void* dx, void* dw, float* dbias, int M, int N, int K, long long ldx,
                      long long lddh, long long lddx, int dtype, int act, void* workspace, size_t workspace_bytes, void* stream) {
    return products_backward(x, w, bias, dh, dx, dw, dbias, M, N, K, ldx, lddh, lddx, dtype, act, 2, workspace, workspace_bytes, stream);
}

size_t wino_attention_workspace_bytes(int B, int Sq, int Skv, int H, int Hkv, int D, int dtype) {
    if (!is_dtype(dtype) || !attention_dims_ok(B, Sq, Skv, H, Hkv, D, dtype)) return 0;
    return attention_ws_bytes(B, Sq, Skv, H, Hkv, D, dtype);
}

int wino_attention(const wino_attention_args* a, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = attention_status(a, false, workspace, workspace_bytes);
    if (rc != WINO_OK) return rc;
    return launch_attention(attention_args(a, workspace), a->dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? WINO_OK : WINO_ERR_HIP;
}

size_t wino_attention_backward_workspace_bytes(int B, int Sq, int Skv, int H, int Hkv, int D, int dtype) {
    if (!is_dtype(dtype) || !attention_dims_ok(B, Sq, Skv, H, Hkv, D, dtype)) return 0;
    return attention_backward_ws_bytes(B, Sq, Skv, H, Hkv, D, dtype);
}

int wino_attention_backward(const wino_attention_args* a, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = attention_status(a, true, workspace, workspace_bytes);
    if (rc != WINO_OK) return rc;
    return launch_attention_backward(attention_args(a, workspace), a->dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? WINO_OK : WINO_ERR_HIP;
}

}  // extern "C"
