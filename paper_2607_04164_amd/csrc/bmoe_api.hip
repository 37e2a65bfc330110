// Host side of the C ABI: argument checks (host only, before anything is
// enqueued), workspace sizing, status strings and the four entry points.
#include <limits.h>
#include <math.h>

#include "bmoe_common.h"

namespace {

using namespace bmoe;

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

inline int elem_bytes(int dtype) { return dtype == BMOE_BF16 ? 2 : 4; }

// whether an output of n bytes shares memory with an input of m bytes
inline bool shares(const void* out, size_t n, const void* in, size_t m) {
    return out && in && (uintptr_t)out < (uintptr_t)in + m && (uintptr_t)in < (uintptr_t)out + n;
}

bmoe_status norm_check(int32_t dtype, int32_t T, int32_t d, float eps) {
    if (dtype != BMOE_F32 && dtype != BMOE_BF16) return BMOE_ERR_UNSUPPORTED;
    if (T < 0 || d < 8 || d % 8 != 0 || d > BMOE_NORM_MAX_D) return BMOE_ERR_SHAPE;
    if (!(eps >= 1e-12f && eps <= 1.f)) return BMOE_ERR_SHAPE;
    return BMOE_OK;
}

inline bool w4_group_ok(int32_t group) { return group == 32 || group == 64 || group == 128; }

// One grouped product with 4-bit weights [n_seg, N, K] (w1: the second matrix of a gated one, or nullptr)
bmoe_status w4_check(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t N, int32_t K, const int32_t* offsets,
                     const int32_t* a_rows, int32_t a_count, const void* a, const bmoe_w4* w0, const bmoe_w4* w1,
                     const void* c) {
    if (dtype != BMOE_BF16) return BMOE_ERR_UNSUPPORTED;
    if (n_seg < 1 || n_seg > BMOE_MAX_EXPERTS || rows_cap < 0) return BMOE_ERR_SHAPE;
    if (N < 8 || N % 8 != 0 || N > (1 << 20) || K < 8 || K % 8 != 0 || K > (1 << 20)) return BMOE_ERR_SHAPE;
    if (rows_cap == 0) return BMOE_OK;
    if (!offsets || !a || !w0 || !c) return BMOE_ERR_NULL;
    if (a_rows && a_count < 1) return BMOE_ERR_SHAPE;
    for (const bmoe_w4* w : {w0, w1}) {
        if (!w) continue;
        if (!w->codes || !w->scales) return BMOE_ERR_NULL;
        if (!w4_group_ok(w->group) || w->group != w0->group || (w->zeros != nullptr) != (w0->zeros != nullptr))
            return BMOE_ERR_UNSUPPORTED;
        if (!aligned16(w->codes) || ((uintptr_t)w->scales & 1u)) return BMOE_ERR_ALIGN;
    }
    if (!aligned16(a) || !aligned16(c)) return BMOE_ERR_ALIGN;
    return BMOE_OK;
}

constexpr int32_t kW8MaxRows = 1 << 30;

inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }
// rows of K values in 8 bits: the codes, then the scales
inline size_t w8_codes_bytes(int64_t rows, int K) { return up256((size_t)rows * w8_pitch(K)); }
inline size_t w8_rows_bytes(int64_t rows, int K) { return w8_codes_bytes(rows, K) + up256((size_t)rows * 4); }

// One grouped product in 8 bits (w1: the second matrix of a gated one, or nullptr). a, a8: its input, one of them.
bmoe_status w8_check(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t N, int32_t K, const int32_t* offsets,
                     const int32_t* a_rows, int32_t a_count, const void* a, const bmoe_w8* a8, const bmoe_w8* w0,
                     const bmoe_w8* w1, const void* c) {
    if (dtype != BMOE_BF16) return BMOE_ERR_UNSUPPORTED;
    if (n_seg < 1 || n_seg > BMOE_MAX_EXPERTS || rows_cap < 0 || rows_cap > kW8MaxRows) return BMOE_ERR_SHAPE;
    if (N < 8 || N % 8 != 0 || N > (1 << 20) || K < 8 || K % 8 != 0 || K > BMOE_W8_MAX_K) return BMOE_ERR_SHAPE;
    if (rows_cap == 0) return BMOE_OK;
    if (!offsets || (!a && !a8) || !w0 || !c) return BMOE_ERR_NULL;
    if (a && a8) return BMOE_ERR_UNSUPPORTED;
    // (the copies address a gathered source with 32-bit byte offsets)
    if (a_rows && (a_count < 1 || a_count > kW8MaxRows || a_count * w8_pitch(K) >= ((int64_t)1 << 32)))
        return BMOE_ERR_SHAPE;
    for (const bmoe_w8* w : {a8, w0, w1}) {
        if (!w) continue;
        if (!w->codes || !w->scales) return BMOE_ERR_NULL;
        if (!aligned16(w->codes) || !aligned16(w->scales)) return BMOE_ERR_ALIGN;
    }
    if (!aligned16(a) || !aligned16(c)) return BMOE_ERR_ALIGN;
    const size_t out = (size_t)rows_cap * N * 2;
    const int64_t rows = a_rows ? a_count : rows_cap;
    if (a8 ? shares(c, out, a8->codes, (size_t)rows * w8_pitch(K)) || shares(c, out, a8->scales, (size_t)rows * 4)
           : shares(c, out, a, (size_t)rows * K * 2))
        return BMOE_ERR_UNSUPPORTED;
    return BMOE_OK;
}

// a [rows, K] rounded into the workspace
hipError_t w8_rounded(const void* a, int64_t rows, int K, void* ws, bmoe_w8& out, hipStream_t s,
                      const int32_t* offsets = nullptr, int n_seg = 0) {
    int8_t* codes = (int8_t*)ws;
    float* scales = (float*)(codes + w8_codes_bytes(rows, K));
    out = bmoe_w8{codes, scales};
    W8QuantizeArgs q{a, codes, scales, rows, K, BMOE_BF16};
    q.offsets = offsets;
    q.n_seg = n_seg;
    return launch_w8_quantize(q, s);
}

// The products of a checked call (w_down: the second one, from h)
struct W8Call {
    int32_t n_seg, rows_cap, d, d_ff;
    const int32_t* offsets;
    const int32_t* a_rows;
    int32_t a_count;
    const void* a;
    const bmoe_w8 *a8, *w_gate, *w_up, *w_down;
    void *h, *y, *ws;
    size_t ws_bytes;
    hipStream_t s;
};

bmoe_status w8_run(const W8Call& c) {
    const int64_t rows = c.a_rows ? c.a_count : c.rows_cap;
    const size_t need = bmoe_w8_workspace_bytes(c.a8 ? 0 : (int32_t)rows, c.d, c.rows_cap, c.w_down ? c.d_ff : 0, 0);
    if (need > 0 && !c.ws) return BMOE_ERR_WORKSPACE;
    if (c.ws_bytes < need) return BMOE_ERR_WORKSPACE;
    if ((uintptr_t)c.ws & 255u) return BMOE_ERR_ALIGN;
    char* ws = (char*)c.ws;
    const bool split = c.ws && c.ws_bytes - need >= ffn_workspace_bytes();
    W8GemmArgs g{c.offsets, c.a_rows, c.a_count, {}, *c.w_gate, c.w_up ? *c.w_up : bmoe_w8{nullptr, nullptr}, c.h,
                 split ? ws + need : nullptr, split ? c.ws_bytes - need : 0, c.n_seg, c.rows_cap, c.d_ff, c.d};
    // x (or a8) times g's weights
    auto product = [&](const void* x, int64_t x_rows, const bmoe_w8* a8, const int32_t* offsets) {
        if (!a8 && w8_few_fits(g)) return launch_w8_few(g, x, c.s);
        hipError_t e = hipSuccess;
        if (a8) g.a = *a8;
        else e = w8_rounded(x, x_rows, g.K, ws, g.a, c.s, offsets, c.n_seg);
        return e == hipSuccess ? launch_w8_gemm(g, c.s) : e;
    };
    hipError_t e = product(c.a, rows, c.a8, nullptr);
    if (e != hipSuccess || !c.w_down) return e == hipSuccess ? BMOE_OK : BMOE_ERR_HIP;
    g.a_rows = nullptr;
    g.a_count = 0;
    g.w0 = *c.w_down;
    g.w1 = bmoe_w8{nullptr, nullptr};
    g.c = c.y;
    g.N = c.d;
    g.K = c.d_ff;
    // (the rounded rows of h in the place of a's, which the product before has read; only rows of segments are there)
    e = product(c.h, c.rows_cap, nullptr, c.offsets);
    return e == hipSuccess ? BMOE_OK : BMOE_ERR_HIP;
}

inline bmoe_status hip_status(hipError_t e) { return e == hipSuccess ? BMOE_OK : BMOE_ERR_HIP; }

}  // namespace

extern "C" {

int32_t bmoe_version(void) { return 10000; }

const char* bmoe_status_str(bmoe_status s) {
    switch (s) {
        case BMOE_OK: return "ok";
        case BMOE_ERR_NULL: return "a required pointer is NULL";
        case BMOE_ERR_SHAPE: return "a size is out of range";
        case BMOE_ERR_ALIGN: return "a tensor pointer is not 16-byte aligned";
        case BMOE_ERR_MAP: return "an expert-to-group map entry is outside [0, G)";
        case BMOE_ERR_UNSUPPORTED: return "unsupported dtype or mode";
        case BMOE_ERR_WORKSPACE: return "workspace missing or too small";
        case BMOE_ERR_HIP: return "HIP runtime error at launch";
    }
    return "unknown status";
}

bmoe_status bmoe_validate(const bmoe_desc* d) {
    if (!d) return BMOE_ERR_NULL;
    if (d->dtype != BMOE_F32 && d->dtype != BMOE_BF16) return BMOE_ERR_UNSUPPORTED;
    if (d->T < 0 || d->E < 1 || d->E > BMOE_MAX_EXPERTS) return BMOE_ERR_SHAPE;
    if (d->top_k < 1 || d->top_k > d->E || d->top_k > BMOE_MAX_TOPK) return BMOE_ERR_SHAPE;
    if (d->G < 1 || d->G > d->E) return BMOE_ERR_SHAPE;
    if (d->d < 8 || d->d % 8 != 0 || d->d_ff < 8 || d->d_ff % 8 != 0) return BMOE_ERR_SHAPE;
    if (d->d_ff_shared < 0 || d->d_ff_shared % 8 != 0) return BMOE_ERR_SHAPE;
    if (d->norm_topk != 0 && d->norm_topk != 1) return BMOE_ERR_SHAPE;
    // row indices (T*k) and element offsets within a row fit 32-bit ints
    if ((int64_t)d->T * d->top_k > INT_MAX / 2) return BMOE_ERR_SHAPE;
    if (d->d > (1 << 20) || d->d_ff > (1 << 20) || d->d_ff_shared > (1 << 20)) return BMOE_ERR_SHAPE;
    return BMOE_OK;
}

bmoe_status bmoe_validate_map(const int32_t* e2g, int32_t E, int32_t G) {
    if (!e2g) return BMOE_ERR_NULL;
    if (E < 1 || E > BMOE_MAX_EXPERTS || G < 1 || G > E) return BMOE_ERR_SHAPE;
    for (int e = 0; e < E; ++e)
        if (e2g[e] < 0 || e2g[e] >= G) return BMOE_ERR_MAP;
    return BMOE_OK;
}

size_t bmoe_workspace_bytes(const bmoe_desc* d, int32_t stage) {
    if (bmoe_validate(d) != BMOE_OK) return 0;
    if (stage == BMOE_STAGE_DISPATCH) return dispatch_ws_bytes(d->T, d->G);
    if (stage == BMOE_STAGE_FFN && d->dtype == BMOE_BF16) return ffn_workspace_bytes();
    if (stage == BMOE_STAGE_DOWN_COMBINE) return down_combine_ws_bytes(d->T, d->d);
    if (stage == BMOE_STAGE_FEW && d->T <= BMOE_FEW_MAX_TOKENS)
        return few_ws_bytes(d->T, d->E, d->top_k, d->d, d->d_ff, d->d_ff_shared);
    return 0;
}

bmoe_status brownout_moe_route(const bmoe_desc* d, const void* x, const void* w_router,
                               const float* bias, const float* logits_in, const int32_t* e2g,
                               int32_t* topk_idx, float* topk_w, int32_t* slot_group, float* slot_gate,
                               float* logits_out, void* stream) {
    bmoe_status st = bmoe_validate(d);
    if (st != BMOE_OK) return st;
    if (d->T == 0) return BMOE_OK;
    if (!e2g || !topk_idx || !topk_w || !slot_group || !slot_gate) return BMOE_ERR_NULL;
    if (!logits_in && (!x || !w_router)) return BMOE_ERR_NULL;
    if (!logits_in && (!aligned16(x) || !aligned16(w_router))) return BMOE_ERR_ALIGN;
    RouteArgs a{x, w_router, bias, logits_in, e2g, topk_idx, topk_w, slot_group, slot_gate, logits_out,
                d->T, d->d, d->E, d->top_k, d->G, d->norm_topk, d->dtype};
    return hip_status(launch_route(a, (hipStream_t)stream));
}

bmoe_status brownout_moe_dispatch(const bmoe_desc* d, const int32_t* slot_group, const void* x,
                                  int32_t* counts, int32_t* offsets, int32_t* perm_token,
                                  int32_t* slot_row, void* x_perm, void* ws, size_t ws_bytes,
                                  void* stream) {
    bmoe_status st = bmoe_validate(d);
    if (st != BMOE_OK) return st;
    if (d->T == 0) return BMOE_OK;
    // x_perm NULL: the permutation only (x is then not read and may be NULL)
    if (!slot_group || !counts || !offsets || !perm_token || !slot_row || (x_perm && !x))
        return BMOE_ERR_NULL;
    if (x_perm && (!aligned16(x) || !aligned16(x_perm))) return BMOE_ERR_ALIGN;
    if (!ws || ws_bytes < dispatch_ws_bytes(d->T, d->G)) return BMOE_ERR_WORKSPACE;
    if (((uintptr_t)ws & 255u) != 0) return BMOE_ERR_ALIGN;
    DispatchArgs a{slot_group, x, counts, offsets, perm_token, slot_row, x_perm, ws,
                   d->T, d->d, d->top_k, d->G, elem_bytes(d->dtype)};
    return hip_status(launch_dispatch(a, (hipStream_t)stream));
}

bmoe_status brownout_moe_dispatch_noalloc(const bmoe_desc* d, const int32_t* slot_group, const void* x,
                                          int32_t* counts, int32_t* offsets, int32_t* perm_token,
                                          int32_t* slot_row, void* x_perm, void* stream) {
    bmoe_status st = bmoe_validate(d);
    if (st != BMOE_OK) return st;
    if (d->T == 0) return BMOE_OK;
    if (!slot_group || !counts || !offsets || !perm_token || !slot_row || (x_perm && !x))
        return BMOE_ERR_NULL;
    if (x_perm && (!aligned16(x) || !aligned16(x_perm))) return BMOE_ERR_ALIGN;
    if (dispatch_ws_bytes(d->T, d->G) > (size_t)BMOE_DISPATCH_SCRATCH_BYTES) return BMOE_ERR_WORKSPACE;
    DispatchArgs a{slot_group, x, counts, offsets, perm_token, slot_row, x_perm, nullptr,
                   d->T, d->d, d->top_k, d->G, elem_bytes(d->dtype)};
    return hip_status(launch_dispatch_noalloc(a, (hipStream_t)stream));
}

}  // extern "C"

namespace {

// a_rows != nullptr: the gate/up GEMM reads row r of its A operand from
// a[a_rows[r]], a holding a_count rows
bmoe_status ffn_common(int part, int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                       const int32_t* offsets, const void* a, const void* w_gate, const void* w_up,
                       const void* w_down, void* h, void* y, void* ws, size_t ws_bytes, void* stream,
                       const int32_t* a_rows = nullptr, int32_t a_count = 0, int32_t split_min_idle = -1) {
    if (dtype != BMOE_F32 && dtype != BMOE_BF16) return BMOE_ERR_UNSUPPORTED;
    if (n_seg < 1 || n_seg > BMOE_MAX_EXPERTS || rows_cap < 0) return BMOE_ERR_SHAPE;
    if (d < 8 || d % 8 != 0 || d_ff < 8 || d_ff % 8 != 0) return BMOE_ERR_SHAPE;
    if (d > (1 << 20) || d_ff > (1 << 20)) return BMOE_ERR_SHAPE;
    if ((int64_t)rows_cap * (d > d_ff ? d : d_ff) > ((int64_t)1 << 40)) return BMOE_ERR_SHAPE;
    if (rows_cap == 0) return BMOE_OK;
    const bool up = part != 2, down = part != 1;
    if (!offsets || !h) return BMOE_ERR_NULL;
    if (up && (!a || !w_gate || !w_up)) return BMOE_ERR_NULL;
    if (down && (!w_down || !y)) return BMOE_ERR_NULL;
    if (!aligned16(h)) return BMOE_ERR_ALIGN;
    if (up && (!aligned16(a) || !aligned16(w_gate) || !aligned16(w_up))) return BMOE_ERR_ALIGN;
    if (down && (!aligned16(w_down) || !aligned16(y))) return BMOE_ERR_ALIGN;
    if (ws && ((uintptr_t)ws & 255u)) return BMOE_ERR_ALIGN;
    if (dtype != BMOE_BF16) ws = nullptr;  // the fp32 kernels take no workspace
    if (ws && ws_bytes < ffn_workspace_bytes()) return BMOE_ERR_WORKSPACE;
    if (split_min_idle < -1 || split_min_idle > (1 << 20)) return BMOE_ERR_SHAPE;
    FfnArgs args{offsets, a, w_gate, w_up, w_down, h, y, ws, ws_bytes, n_seg, rows_cap, d, d_ff, dtype};
    args.split_min_idle = split_min_idle;
    if (a_rows) {
        // the copy kernels address a gathered source with 32-bit byte offsets
        if (a_count < 1 || (int64_t)a_count * d * elem_bytes(dtype) >= ((int64_t)1 << 32)) return BMOE_ERR_SHAPE;
        args.a_rows = a_rows;
        args.a_count = a_count;
    }
    return hip_status(launch_ffn(args, (hipStream_t)stream, part));
}

}  // namespace

extern "C" {

bmoe_status brownout_moe_ffn(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                             const int32_t* offsets, const void* a, const void* w_gate,
                             const void* w_up, const void* w_down, void* h, void* y, void* workspace,
                             size_t workspace_bytes, void* stream) {
    return ffn_common(0, dtype, n_seg, rows_cap, d, d_ff, offsets, a, w_gate, w_up, w_down, h, y, workspace,
                      workspace_bytes, stream);
}

bmoe_status brownout_moe_ffn_ex(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                                const int32_t* offsets, const void* a, const void* w_gate, const void* w_up,
                                const void* w_down, void* h, void* y, void* workspace, size_t workspace_bytes,
                                int32_t split_min_idle, void* stream) {
    return ffn_common(0, dtype, n_seg, rows_cap, d, d_ff, offsets, a, w_gate, w_up, w_down, h, y, workspace,
                      workspace_bytes, stream, nullptr, 0, split_min_idle);
}

bmoe_status brownout_moe_ffn_gather(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                                    const int32_t* offsets, const int32_t* a_rows, int32_t a_count,
                                    const void* a, const void* w_gate, const void* w_up, const void* w_down,
                                    void* h, void* y, void* workspace, size_t workspace_bytes, void* stream) {
    if (rows_cap > 0 && !a_rows) return BMOE_ERR_NULL;
    return ffn_common(0, dtype, n_seg, rows_cap, d, d_ff, offsets, a, w_gate, w_up, w_down, h, y, workspace,
                      workspace_bytes, stream, a_rows, a_count);
}

bmoe_status brownout_moe_ffn_gate_up_gather(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d,
                                            int32_t d_ff, const int32_t* offsets, const int32_t* a_rows,
                                            int32_t a_count, const void* a, const void* w_gate, const void* w_up,
                                            void* h, void* workspace, size_t workspace_bytes, void* stream) {
    if (rows_cap > 0 && !a_rows) return BMOE_ERR_NULL;
    return ffn_common(1, dtype, n_seg, rows_cap, d, d_ff, offsets, a, w_gate, w_up, nullptr, h, nullptr,
                      workspace, workspace_bytes, stream, a_rows, a_count);
}

bmoe_status brownout_moe_ffn_gate_up(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d,
                                     int32_t d_ff, const int32_t* offsets, const void* a,
                                     const void* w_gate, const void* w_up, void* h, void* workspace,
                                     size_t workspace_bytes, void* stream) {
    return ffn_common(1, dtype, n_seg, rows_cap, d, d_ff, offsets, a, w_gate, w_up, nullptr, h, nullptr,
                      workspace, workspace_bytes, stream);
}

bmoe_status brownout_moe_ffn_down(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                                  const int32_t* offsets, const void* h, const void* w_down, void* y,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    // h is only read by the down GEMM
    return ffn_common(2, dtype, n_seg, rows_cap, d, d_ff, offsets, nullptr, nullptr, nullptr, w_down,
                      const_cast<void*>(h), y, workspace, workspace_bytes, stream);
}

bmoe_status brownout_moe_ffn_down_combine(const bmoe_desc* d, const int32_t* offsets, const void* h,
                                          const void* w_down, void* y, const int32_t* perm_token,
                                          const int32_t* slot_row, const float* slot_gate, const void* y_shared,
                                          void* out, void* workspace, size_t workspace_bytes, void* stream) {
    bmoe_status st = bmoe_validate(d);
    if (st != BMOE_OK) return st;
    if (d->T == 0) return BMOE_OK;
    if (!offsets || !h || !w_down || !y || !perm_token || !slot_row || !slot_gate || !out) return BMOE_ERR_NULL;
    if (!aligned16(h) || !aligned16(w_down) || !aligned16(y) || !aligned16(out) ||
        (y_shared && !aligned16(y_shared)))
        return BMOE_ERR_ALIGN;
    const int32_t rows_cap = d->T * d->top_k;
    if ((int64_t)rows_cap * (d->d > d->d_ff ? d->d : d->d_ff) > ((int64_t)1 << 40)) return BMOE_ERR_SHAPE;
    if (!workspace || workspace_bytes < down_combine_ws_bytes(d->T, d->d)) return BMOE_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 255u) return BMOE_ERR_ALIGN;
    FfnArgs args{offsets, nullptr, nullptr, nullptr, w_down, const_cast<void*>(h), y, nullptr, 0,
                 d->G, rows_cap, d->d, d->d_ff, d->dtype};
    args.fold.perm_token = perm_token;
    args.fold.slot_row = slot_row;
    args.fold.slot_gate = slot_gate;
    args.fold.y_shared = (const uint16_t*)y_shared;
    args.fold.out = (uint16_t*)out;
    args.fold.cnt = (int32_t*)workspace;
    args.fold.k = d->top_k;
    if (ffn_can_fold(args)) return hip_status(launch_ffn(args, (hipStream_t)stream, 2));
    // other shapes: the down projection, then the combine kernel
    args.fold = FoldArgs{};
    hipError_t e = launch_ffn(args, (hipStream_t)stream, 2);
    if (e != hipSuccess) return BMOE_ERR_HIP;
    CombineArgs c{slot_row, slot_gate, y, y_shared, out, d->T, d->top_k, d->d, elem_bytes(d->dtype),
                  (int64_t)rows_cap};
    return hip_status(launch_combine(c, (hipStream_t)stream));
}

bmoe_status brownout_moe_united_init(int32_t dtype, int32_t E, int32_t G, int32_t d, int32_t d_ff,
                                     const int32_t* e2g, const void* w_gate_e, const void* w_up_e,
                                     const void* w_down_e, void* w_gate_u, void* w_up_u, void* w_down_u,
                                     void* stream) {
    if (dtype != BMOE_F32 && dtype != BMOE_BF16) return BMOE_ERR_UNSUPPORTED;
    if (E < 1 || E > BMOE_MAX_EXPERTS || G < 1 || G > BMOE_MAX_EXPERTS) return BMOE_ERR_SHAPE;
    if (d < 8 || d % 8 != 0 || d_ff < 8 || d_ff % 8 != 0 || d > (1 << 20) || d_ff > (1 << 20))
        return BMOE_ERR_SHAPE;
    if (!e2g || !w_gate_e || !w_up_e || !w_down_e || !w_gate_u || !w_up_u || !w_down_u) return BMOE_ERR_NULL;
    for (const void* p : {w_gate_e, w_up_e, w_down_e, (const void*)w_gate_u, (const void*)w_up_u,
                          (const void*)w_down_u})
        if (!aligned16(p)) return BMOE_ERR_ALIGN;
    bmoe::UnitedInitArgs a{e2g, {w_gate_e, w_up_e, w_down_e}, {w_gate_u, w_up_u, w_down_u}, E, G, d, d_ff, dtype};
    return hip_status(bmoe::launch_united_init(a, (hipStream_t)stream));
}

bmoe_status brownout_moe_distill_mse(int32_t dtype, int32_t E, int32_t G, int32_t T, int32_t d,
                                     const int32_t* e2g, const float* w_freq, const void* y_expert,
                                     const void* y_united, double* mse, double* mse_total, void* workspace,
                                     size_t workspace_bytes, void* stream) {
    if (dtype != BMOE_F32 && dtype != BMOE_BF16) return BMOE_ERR_UNSUPPORTED;
    if (E < 1 || E > BMOE_MAX_EXPERTS || G < 1 || G > BMOE_MAX_EXPERTS || T < 0) return BMOE_ERR_SHAPE;
    if (d < 8 || d % 8 != 0 || d > (1 << 20)) return BMOE_ERR_SHAPE;
    if (T == 0) return BMOE_OK;
    const int nb = bmoe::distill_ws_blocks(G, T);
    // the partial kernel counts a workgroup's chunks in 32 bits
    if ((((int64_t)T + nb - 1) / nb + 1) * (d / (dtype == BMOE_BF16 ? 8 : 4)) >= ((int64_t)1 << 31))
        return BMOE_ERR_SHAPE;
    if (!e2g || !w_freq || !y_expert || !y_united || !mse) return BMOE_ERR_NULL;
    if (!aligned16(y_expert) || !aligned16(y_united) || ((uintptr_t)mse & 7u) || ((uintptr_t)mse_total & 7u))
        return BMOE_ERR_ALIGN;
    if (!workspace || workspace_bytes < bmoe::distill_ws_bytes(G, T)) return BMOE_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 7u) return BMOE_ERR_ALIGN;
    bmoe::DistillArgs a{e2g, w_freq, y_expert, y_united, mse, mse_total, workspace, E, G, T, d, dtype};
    return hip_status(bmoe::launch_distill_mse(a, (hipStream_t)stream));
}

bmoe_status brownout_moe_combine(const bmoe_desc* d, const int32_t* slot_row, const float* slot_gate,
                                 const void* y_perm, const void* y_shared, void* out, void* stream) {
    bmoe_status st = bmoe_validate(d);
    if (st != BMOE_OK) return st;
    if (d->T == 0) return BMOE_OK;
    if (!slot_row || !slot_gate || !y_perm || !out) return BMOE_ERR_NULL;
    if (!aligned16(y_perm) || !aligned16(out) || (y_shared && !aligned16(y_shared))) return BMOE_ERR_ALIGN;
    CombineArgs a{slot_row, slot_gate, y_perm, y_shared, out, d->T, d->top_k, d->d, elem_bytes(d->dtype),
                  (int64_t)d->T * d->top_k};
    return hip_status(launch_combine(a, (hipStream_t)stream));
}

bmoe_status brownout_moe_pre_norm(int32_t dtype, int32_t T, int32_t d, float eps, const void* x, const void* w,
                                  void* out, void* stream) {
    bmoe_status st = norm_check(dtype, T, d, eps);
    if (st != BMOE_OK || T == 0) return st;
    if (!x || !out) return BMOE_ERR_NULL;
    if (!aligned16(x) || !aligned16(out) || !aligned16(w)) return BMOE_ERR_ALIGN;
    const size_t row = (size_t)d * elem_bytes(dtype), all = (size_t)T * row;
    // (a row is read before it is written, but no other row, nor the weights once there are more)
    if ((out != x && shares(out, all, x, all)) || ((out != w || T > 1) && shares(out, all, w, row)))
        return BMOE_ERR_UNSUPPORTED;
    return hip_status(bmoe::launch_pre_norm(bmoe::PreNormArgs{x, w, out, T, d, dtype, eps}, (hipStream_t)stream));
}

bmoe_status brownout_moe_post_norm(int32_t dtype, int32_t T, int32_t d, float eps, int32_t norm_y, float res_scale,
                                   int32_t gate_mode, const void* y, const void* x, const void* w_post,
                                   const void* gate, void* r, const void* w_next, void* a, void* stream) {
    bmoe_status st = norm_check(dtype, T, d, eps);
    if (st != BMOE_OK) return st;
    if (gate_mode < BMOE_GATE_NONE || gate_mode > BMOE_GATE_FULL || (norm_y != 0 && norm_y != 1))
        return BMOE_ERR_UNSUPPORTED;
    if (!isfinite(res_scale)) return BMOE_ERR_SHAPE;
    if (T == 0) return BMOE_OK;
    if (!y || !x || !r || (gate_mode != BMOE_GATE_NONE && !gate)) return BMOE_ERR_NULL;
    // what would not be read is not taken
    if ((gate_mode == BMOE_GATE_NONE && gate) || (!norm_y && w_post) || (!a && w_next))
        return BMOE_ERR_UNSUPPORTED;
    for (const void* p : {y, x, w_post, (const void*)r, w_next, (const void*)a})
        if (!aligned16(p)) return BMOE_ERR_ALIGN;
    if (gate && ((uintptr_t)gate & (gate_mode == BMOE_GATE_TOKEN ? 3u : 15u))) return BMOE_ERR_ALIGN;
    const size_t row = (size_t)d * elem_bytes(dtype), all = (size_t)T * row;
    const size_t gates = gate_mode == BMOE_GATE_FULL ? all : gate_mode == BMOE_GATE_CHANNEL ? row : (size_t)T * 4;
    if (shares(r, all, a, all)) return BMOE_ERR_UNSUPPORTED;
    for (const void* out : {(const void*)r, (const void*)a}) {
        if ((out != y && shares(out, all, y, all)) || (out != x && shares(out, all, x, all)) ||
            (!(out == gate && gate_mode == BMOE_GATE_FULL) && shares(out, all, gate, gates)) ||
            shares(out, all, w_post, row) || shares(out, all, w_next, row))
            return BMOE_ERR_UNSUPPORTED;
    }
    return hip_status(bmoe::launch_post_norm(
        bmoe::PostNormArgs{y, x, w_post, gate, w_next, r, a, T, d, dtype, norm_y, gate_mode, eps, res_scale},
        (hipStream_t)stream));
}

bmoe_status brownout_moe_w4_quantize(int32_t dtype, int32_t n, int32_t N, int32_t K, int32_t group, const void* w,
                                     uint8_t* codes, void* scales, uint8_t* zeros, void* stream) {
    if (dtype != BMOE_F32 && dtype != BMOE_BF16) return BMOE_ERR_UNSUPPORTED;
    if (!w4_group_ok(group)) return BMOE_ERR_UNSUPPORTED;
    if (n < 1 || n > BMOE_MAX_EXPERTS || N < 1 || N > (1 << 20) || K < 8 || K % 8 != 0 || K > (1 << 20))
        return BMOE_ERR_SHAPE;
    if (!w || !codes || !scales) return BMOE_ERR_NULL;
    if (!aligned16(w) || !aligned16(codes) || ((uintptr_t)scales & 1u)) return BMOE_ERR_ALIGN;
    return hip_status(bmoe::launch_w4_quantize(
        bmoe::W4QuantizeArgs{w, codes, scales, zeros, n, N, K, group, dtype}, (hipStream_t)stream));
}

bmoe_status brownout_moe_w4_matmul(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t N, int32_t K,
                                   const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                   const bmoe_w4* w, void* y, void* stream) {
    bmoe_status st = w4_check(dtype, n_seg, rows_cap, N, K, offsets, a_rows, a_count, a, w, nullptr, y);
    if (st != BMOE_OK || rows_cap == 0) return st;
    // (other workgroups still read a)
    if (shares(y, (size_t)rows_cap * N * 2, a, (size_t)(a_rows ? a_count : rows_cap) * K * 2)) return BMOE_ERR_UNSUPPORTED;
    return hip_status(bmoe::launch_w4_gemm(
        bmoe::W4GemmArgs{offsets, a_rows, a_count, a, w, nullptr, y, n_seg, rows_cap, N, K}, (hipStream_t)stream));
}

bmoe_status brownout_moe_w4_gate_up(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                                    const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                    const bmoe_w4* w_gate, const bmoe_w4* w_up, void* h, void* stream) {
    if (rows_cap > 0 && !w_up) return BMOE_ERR_NULL;
    bmoe_status st = w4_check(dtype, n_seg, rows_cap, d_ff, d, offsets, a_rows, a_count, a, w_gate, w_up, h);
    if (st != BMOE_OK || rows_cap == 0) return st;
    if (shares(h, (size_t)rows_cap * d_ff * 2, a, (size_t)(a_rows ? a_count : rows_cap) * d * 2)) return BMOE_ERR_UNSUPPORTED;
    return hip_status(bmoe::launch_w4_gemm(
        bmoe::W4GemmArgs{offsets, a_rows, a_count, a, w_gate, w_up, h, n_seg, rows_cap, d_ff, d},
        (hipStream_t)stream));
}

bmoe_status brownout_moe_w4_ffn(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                                const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                const bmoe_w4* w_gate, const bmoe_w4* w_up, const bmoe_w4* w_down, void* h, void* y,
                                void* stream) {
    if (rows_cap > 0 && !w_up) return BMOE_ERR_NULL;
    bmoe_status st = w4_check(dtype, n_seg, rows_cap, d_ff, d, offsets, a_rows, a_count, a, w_gate, w_up, h);
    if (st == BMOE_OK) st = w4_check(dtype, n_seg, rows_cap, d, d_ff, offsets, nullptr, 0, h, w_down, nullptr, y);
    if (st != BMOE_OK || rows_cap == 0) return st;
    const size_t h_bytes = (size_t)rows_cap * d_ff * 2;  // (y may be a: it is read before)
    if (shares(h, h_bytes, a, (size_t)(a_rows ? a_count : rows_cap) * d * 2) || shares(y, (size_t)rows_cap * d * 2, h, h_bytes))
        return BMOE_ERR_UNSUPPORTED;
    const hipError_t e = bmoe::launch_w4_gemm(
        bmoe::W4GemmArgs{offsets, a_rows, a_count, a, w_gate, w_up, h, n_seg, rows_cap, d_ff, d}, (hipStream_t)stream);
    if (e != hipSuccess) return BMOE_ERR_HIP;
    return hip_status(bmoe::launch_w4_gemm(
        bmoe::W4GemmArgs{offsets, nullptr, 0, h, w_down, nullptr, y, n_seg, rows_cap, d, d_ff}, (hipStream_t)stream));
}

bmoe_status brownout_moe_w8_quantize(int32_t dtype, int32_t rows, int32_t K, const void* x, int8_t* codes,
                                     float* scales, void* stream) {
    if (dtype != BMOE_F32 && dtype != BMOE_BF16) return BMOE_ERR_UNSUPPORTED;
    if (rows < 0 || rows > kW8MaxRows || K < 8 || K % 8 != 0 || K > BMOE_W8_MAX_K) return BMOE_ERR_SHAPE;
    if (rows == 0) return BMOE_OK;
    if (!x || !codes || !scales) return BMOE_ERR_NULL;
    if (!aligned16(x) || !aligned16(codes) || !aligned16(scales)) return BMOE_ERR_ALIGN;
    const size_t in = (size_t)rows * K * elem_bytes(dtype), out = (size_t)rows * w8_pitch(K);
    if (shares(codes, out, x, in) || shares(scales, (size_t)rows * 4, x, in) ||
        shares(scales, (size_t)rows * 4, codes, out))
        return BMOE_ERR_UNSUPPORTED;
    return hip_status(bmoe::launch_w8_quantize(bmoe::W8QuantizeArgs{x, codes, scales, rows, K, dtype},
                                               (hipStream_t)stream));
}

size_t bmoe_w8_workspace_bytes(int32_t a_count, int32_t K, int32_t rows_cap, int32_t d_ff, int32_t split) {
    if (a_count < 0 || a_count > kW8MaxRows || rows_cap < 0 || rows_cap > kW8MaxRows || K < 8 || K > BMOE_W8_MAX_K ||
        d_ff < 0 || d_ff > BMOE_W8_MAX_K)
        return 0;
    const size_t a = a_count ? w8_rows_bytes(a_count, K) : 0, h = d_ff && rows_cap ? w8_rows_bytes(rows_cap, d_ff) : 0;
    return (a > h ? a : h) + (split ? ffn_workspace_bytes() : 0);
}

bmoe_status brownout_moe_w8_matmul(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t N, int32_t K,
                                   const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                   const bmoe_w8* a8, const bmoe_w8* w, void* y, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    const bmoe_status st = w8_check(dtype, n_seg, rows_cap, N, K, offsets, a_rows, a_count, a, a8, w, nullptr, y);
    if (st != BMOE_OK || rows_cap == 0) return st;
    return w8_run(W8Call{n_seg, rows_cap, K, N, offsets, a_rows, a_count, a, a8, w, nullptr, nullptr, y, nullptr,
                         workspace, workspace_bytes, (hipStream_t)stream});
}

bmoe_status brownout_moe_w8_gate_up(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                                    const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                    const bmoe_w8* a8, const bmoe_w8* w_gate, const bmoe_w8* w_up, void* h,
                                    void* workspace, size_t workspace_bytes, void* stream) {
    if (rows_cap > 0 && !w_up) return BMOE_ERR_NULL;
    const bmoe_status st = w8_check(dtype, n_seg, rows_cap, d_ff, d, offsets, a_rows, a_count, a, a8, w_gate, w_up, h);
    if (st != BMOE_OK || rows_cap == 0) return st;
    return w8_run(W8Call{n_seg, rows_cap, d, d_ff, offsets, a_rows, a_count, a, a8, w_gate, w_up, nullptr, h, nullptr,
                         workspace, workspace_bytes, (hipStream_t)stream});
}

bmoe_status brownout_moe_w8_ffn(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                                const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                const bmoe_w8* a8, const bmoe_w8* w_gate, const bmoe_w8* w_up, const bmoe_w8* w_down,
                                void* h, void* y, void* workspace, size_t workspace_bytes, void* stream) {
    if (rows_cap > 0 && (!w_up || !w_down)) return BMOE_ERR_NULL;
    bmoe_status st = w8_check(dtype, n_seg, rows_cap, d_ff, d, offsets, a_rows, a_count, a, a8, w_gate, w_up, h);
    // (the down product's input is h)
    if (st == BMOE_OK) st = w8_check(dtype, n_seg, rows_cap, d, d_ff, offsets, nullptr, 0, h, nullptr, w_down, nullptr, y);
    if (st != BMOE_OK || rows_cap == 0) return st;
    return w8_run(W8Call{n_seg, rows_cap, d, d_ff, offsets, a_rows, a_count, a, a8, w_gate, w_up, w_down, h, y,
                         workspace, workspace_bytes, (hipStream_t)stream});
}

size_t bmoe_balance_workspace_bytes(int32_t T, int32_t E) {
    return T < 1 || E < 1 || E > BMOE_MAX_EXPERTS ? 0 : balance_ws_bytes(T, E);
}

}  // extern "C"

namespace {
bmoe_status balance_check(int32_t T, int32_t E, int32_t k, int32_t G, const int32_t* e2g) {
    if (T < 0 || E < 1 || E > BMOE_MAX_EXPERTS || k < 1 || k > BMOE_MAX_TOPK || G < 1 || G > BMOE_MAX_EXPERTS)
        return BMOE_ERR_SHAPE;
    if ((int64_t)T * k > INT_MAX / 2 || (!e2g && G != E)) return BMOE_ERR_SHAPE;
    return BMOE_OK;
}
inline bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
}  // namespace

extern "C" {

bmoe_status brownout_moe_balance(int32_t T, int32_t E, int32_t k, int32_t G, const float* logits,
                                 const int32_t* topk_idx, const uint8_t* valid, const int32_t* e2g, float* losses,
                                 int32_t* counts, float* prob, void* workspace, size_t workspace_bytes, void* stream) {
    const bmoe_status st = balance_check(T, E, k, G, e2g);
    if (st != BMOE_OK || T == 0) return st;
    if (!logits || !topk_idx || !losses || !counts || !prob) return BMOE_ERR_NULL;
    for (const void* p : {(const void*)logits, (const void*)topk_idx, (const void*)e2g, (const void*)losses,
                          (const void*)counts, (const void*)prob})
        if (!aligned4(p)) return BMOE_ERR_ALIGN;
    const size_t need = balance_ws_bytes(T, E), sizes[3] = {8, 4 * (size_t)E + 4, 4 * (size_t)E};
    if (need > 0 && (!workspace || workspace_bytes < need)) return BMOE_ERR_WORKSPACE;
    if (need > 0 && ((uintptr_t)workspace & 7u)) return BMOE_ERR_ALIGN;
    const void* outs[3] = {losses, counts, prob};
    for (int i = 0; i < 3; ++i) {  // (other workgroups still read the inputs)
        if (shares(outs[i], sizes[i], logits, (size_t)T * E * 4) || shares(outs[i], sizes[i], topk_idx, (size_t)T * k * 4) ||
            shares(outs[i], sizes[i], valid, (size_t)T) || shares(outs[i], sizes[i], e2g, (size_t)E * 4))
            return BMOE_ERR_UNSUPPORTED;
        for (int j = 0; j < i; ++j)
            if (shares(outs[i], sizes[i], outs[j], sizes[j])) return BMOE_ERR_UNSUPPORTED;
    }
    return hip_status(bmoe::launch_balance(
        bmoe::BalanceArgs{logits, topk_idx, valid, e2g, losses, counts, prob, workspace, T, E, k, G}, (hipStream_t)stream));
}

bmoe_status brownout_moe_balance_grad(int32_t T, int32_t E, int32_t k, int32_t G, const float* logits,
                                      const uint8_t* valid, const int32_t* e2g, const int32_t* counts,
                                      const float* d_losses, float* d_logits, void* stream) {
    const bmoe_status st = balance_check(T, E, k, G, e2g);
    if (st != BMOE_OK || T == 0) return st;
    if (!logits || !counts || !d_losses || !d_logits) return BMOE_ERR_NULL;
    for (const void* p : {(const void*)logits, (const void*)e2g, (const void*)counts, (const void*)d_losses,
                          (const void*)d_logits})
        if (!aligned4(p)) return BMOE_ERR_ALIGN;
    const size_t all = (size_t)T * E * 4;
    if ((d_logits != logits && shares(d_logits, all, logits, all)) || shares(d_logits, all, valid, (size_t)T) ||
        shares(d_logits, all, e2g, (size_t)E * 4) || shares(d_logits, all, counts, (size_t)E * 4 + 4) ||
        shares(d_logits, all, d_losses, 8))
        return BMOE_ERR_UNSUPPORTED;
    return hip_status(bmoe::launch_balance_grad(
        bmoe::BalanceGradArgs{logits, valid, e2g, counts, d_losses, d_logits, T, E, k, G}, (hipStream_t)stream));
}

bmoe_status brownout_moe_few(const bmoe_desc* d, const bmoe_few_weights* w, const void* x, int32_t* topk_idx,
                             float* topk_w, int32_t* slot_group, float* slot_gate, void* out, void* workspace,
                             size_t workspace_bytes, void* stream) {
    bmoe_status st = bmoe_validate(d);
    if (st != BMOE_OK) return st;
    if (!w) return BMOE_ERR_NULL;
    if (d->T > BMOE_FEW_MAX_TOKENS) return BMOE_ERR_SHAPE;
    if (w->group != 0 && (!w4_group_ok(w->group) || d->dtype != BMOE_BF16)) return BMOE_ERR_UNSUPPORTED;
    if (d->T == 0) return BMOE_OK;
    if (!w->w_router || !w->e2g || !x || !topk_idx || !topk_w || !slot_group || !slot_gate || !out) return BMOE_ERR_NULL;
    if (!aligned16(x) || !aligned16(w->w_router) || !aligned16(out)) return BMOE_ERR_ALIGN;
    const bmoe_matrix* m[6] = {&w->gate, &w->up, &w->down, &w->gate_sh, &w->up_sh, &w->down_sh};
    const int used = d->d_ff_shared > 0 ? 6 : 3;
    for (int i = 0; i < used; ++i) {
        if (!m[i]->w || (w->group != 0 && !m[i]->scales)) return BMOE_ERR_NULL;
        if (!aligned16(m[i]->w) || ((uintptr_t)m[i]->scales & 1u)) return BMOE_ERR_ALIGN;
        if (w->group == 0 ? (m[i]->scales || m[i]->zeros) : ((m[i]->zeros != nullptr) != (m[0]->zeros != nullptr)))
            return BMOE_ERR_UNSUPPORTED;
    }
    if (!workspace || workspace_bytes < few_ws_bytes(d->T, d->E, d->top_k, d->d, d->d_ff, d->d_ff_shared)) return BMOE_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 255u) return BMOE_ERR_ALIGN;
    bmoe::FewArgs a{*w, x, topk_idx, topk_w, slot_group, slot_gate, out, workspace,
                    d->T, d->d, d->E, d->top_k, d->G, d->d_ff, d->d_ff_shared, d->norm_topk, d->dtype};
    return hip_status(bmoe::launch_few(a, (hipStream_t)stream));
}

}  // extern "C"
