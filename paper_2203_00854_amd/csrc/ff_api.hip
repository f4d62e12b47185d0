// C ABI entry points of libff: argument checking, workspace carving, the chunk loop.
// All arithmetic of the path runs in the kernels of the other translation units.
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <initializer_list>
#include <mutex>
#include <vector>

#include "ff_common.h"

namespace ff {

// ---- launch timer: HIP events around kernel launches, on the launch stream -------------
static bool g_prof_on = false;
static std::mutex g_prof_mu;
struct ProfRec { int kind; hipEvent_t a, b; };
static std::vector<ProfRec> g_prof;
static std::vector<hipEvent_t> g_prof_pool;
static const char* kKindNames[KK_COUNT] = {"k_prep", "pair bias pass", "k_gemm<PROJ>", "k_attn_rows",
                                           "k_gemm<OUT>", "k_layernorm", "generic family", "probe: mfma loop",
                                           "probe: copy", "k_tm_prep", "k_tm_proj", "k_tm_mul", "k_tm_out",
                                           "k_gca_kv", "k_gca_softmax", "k_gca_out",
                                           "k_bwd_stats", "k_bwd_dq", "k_bwd_dkv", "k_bwd_dbias", "probe: vector loop",
                                           "k_proj_attn", "k_bwd_rows", "k_bwd_prepare", "k_bwd_dbias_reduce", "k_ln_forward",
                                           "k_ln_backward", "k_ln_join", "k_grad_norm", "k_adamw", "k_moments", "k_tr_pack", "k_tr_hidden", "k_tr_out",
                                           "k_tr_grad", "k_tr_weights", "k_tr_join", "k_tr_rows", "k_muon_momentum", "k_ns_start", "k_ns_gram", "k_ns_poly", "k_ns_apply", "k_ns_small"};

static hipEvent_t prof_event() {
    if (!g_prof_pool.empty()) {
        hipEvent_t e = g_prof_pool.back();
        g_prof_pool.pop_back();
        return e;
    }
    hipEvent_t e = nullptr;
    if (hipEventCreate(&e) != hipSuccess) return nullptr;
    return e;
}

void prof_begin(int kind, hipStream_t st) {
    if (!g_prof_on) return;
    std::lock_guard<std::mutex> lk(g_prof_mu);
    if (g_prof.size() >= (1u << 18)) return;
    ProfRec r{kind, prof_event(), prof_event()};
    if (!r.a || !r.b) return;
    (void)hipEventRecord(r.a, st);
    g_prof.push_back(r);
}

void prof_end(int kind, hipStream_t st) {
    if (!g_prof_on) return;
    std::lock_guard<std::mutex> lk(g_prof_mu);
    for (size_t i = g_prof.size(); i-- > 0;)
        if (g_prof[i].kind == kind) {
            (void)hipEventRecord(g_prof[i].b, st);
            return;
        }
}

static thread_local char g_err[512] = "";
static thread_local const char* g_last_path = "";     // kernel family of this thread's last attention call

ff_status fail(ff_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return st;
}

ff_status check_launch(const char* what) {
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FF_EHIP, "%s: %s", what, hipGetErrorString(e));
    return FF_OK;
}

static ff_status make_problem(const ff_attn_desc* d, Problem* p) {
    if (!d) return fail(FF_EINVAL, "desc is NULL");
    if (d->mode < FF_MSA_ROW || d->mode > FF_TRI_END) return fail(FF_EINVAL, "bad mode %d", d->mode);
    if (d->dtype != FF_F32 && d->dtype != FF_BF16) return fail(FF_EINVAL, "bad dtype %d", d->dtype);
    if (d->n_a < 1 || d->n_b < 1 || d->c < 1 || d->heads < 1 || d->head_dim < 1)
        return fail(FF_EINVAL, "non-positive size (n_a=%d n_b=%d c=%d heads=%d head_dim=%d)", d->n_a, d->n_b,
                    d->c, d->heads, d->head_dim);
    if (d->mode == FF_MSA_ROW && d->c_z < 1) return fail(FF_EINVAL, "row mode needs c_z >= 1 (got %d)", d->c_z);
    if ((d->mode == FF_TRI_START || d->mode == FF_TRI_END) && d->n_a != d->n_b)
        return fail(FF_EINVAL, "triangle modes need n_a == n_b (got %d, %d)", d->n_a, d->n_b);
    if (!(d->ln_eps >= 0.f)) return fail(FF_EINVAL, "ln_eps must be >= 0");
    if (d->head_dim > 128) return fail(FF_EUNSUPPORTED, "head_dim %d > 128", d->head_dim);
    if (d->c > 8192 || (d->mode == FF_MSA_ROW && d->c_z > 8192))
        return fail(FF_EUNSUPPORTED, "c or c_z > 8192");
    if ((int64_t)d->heads * d->head_dim > 16384) return fail(FF_EUNSUPPORTED, "heads*head_dim > 16384");
    p->mode = d->mode;
    p->dtype = d->dtype;
    p->n_a = d->n_a;
    p->n_b = d->n_b;
    p->c = d->c;
    p->c_z = d->mode == FF_MSA_ROW ? d->c_z : 0;
    p->H = d->heads;
    p->d = d->head_dim;
    p->Hd = d->heads * d->head_dim;
    p->eps = d->ln_eps;
    const bool along_b = (d->mode == FF_MSA_ROW || d->mode == FF_TRI_START);
    p->R = along_b ? d->n_a : d->n_b;
    p->L = along_b ? d->n_b : d->n_a;
    p->sr = along_b ? d->n_b : 1;
    p->sl = along_b ? 1 : d->n_b;
    p->has_bias = d->mode != FF_MSA_COL;
    return FF_OK;
}

// Both families need at most max(mfma, generic) bytes; the size reported to the caller is that
// maximum so that the family can still be chosen per call (the matrix-core kernels use 16-byte
// accesses and are only taken when every pointer is 16-byte aligned).
static size_t carve(const Problem& p, int chunk, Workspace* ws, void* base, bool fast) {
    return fast ? mfma_workspace(p, chunk, ws, base) : generic_workspace(p, chunk, ws, base);
}
static size_t workspace_need(const Problem& p, int chunk) {
    Workspace tmp;
    size_t a = generic_workspace(p, chunk, &tmp, nullptr);
    if (mfma_supported(p)) {
        size_t b = mfma_workspace(p, chunk, &tmp, nullptr);
        if (b > a) a = b;
    }
    return a;
}
static bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
static bool overlaps(const void* a, size_t an, const void* b, size_t bn) {
    return (uintptr_t)a < (uintptr_t)b + bn && (uintptr_t)b < (uintptr_t)a + an;
}

static ff_status run(const ff_attn_desc* desc, const ff_attn_weights* w, const void* x, const void* z,
                     const float* mask, void* out, void* wsp, size_t ws_bytes, void* stream_, int chunk_rows,
                     bool chunked, bool residual = false) {
    Problem p;
    ff_status st = make_problem(desc, &p);
    if (st != FF_OK) return st;
    if (chunked && chunk_rows < 1) return fail(FF_EINVAL, "chunk_rows must be >= 1 (got %d)", chunk_rows);
    if (!w) return fail(FF_EINVAL, "weights is NULL");
    if (!x || !out) return fail(FF_EINVAL, "x or out is NULL");
    if (!w->ln_g || !w->ln_b || !w->w_q || !w->w_k || !w->w_v || !w->w_g || !w->b_g || !w->w_o || !w->b_o)
        return fail(FF_EINVAL, "a required weight pointer is NULL");
    if (p.mode == FF_MSA_ROW) {
        if (!z) return fail(FF_EINVAL, "row mode needs z");
        if (!w->lnz_g || !w->lnz_b || !w->w_b) return fail(FF_EINVAL, "row mode needs lnz_g, lnz_b and w_b");
    } else {
        if (z) return fail(FF_EINVAL, "z must be NULL outside row mode");
        if (p.has_bias && !w->w_b) return fail(FF_EINVAL, "triangle modes need w_b");
    }
    const size_t esz = p.dtype == FF_F32 ? 4 : 2;
    const size_t x_bytes = (size_t)p.n_a * p.n_b * p.c * esz;
    const size_t z_bytes = (size_t)p.n_b * p.n_b * p.c_z * esz;
    // (the residual update may replace x in place: every kernel has read x, or the part of it that a
    // chunk needs, before the output projection of that chunk stores, and an element of the
    // residual is read by the very lane that stores it)
    if ((overlaps(out, x_bytes, x, x_bytes) && !(residual && out == x)) || (z && overlaps(out, x_bytes, z, z_bytes)))
        return fail(FF_EINVAL, residual ? "out must be x itself or not overlap x, and must not overlap z"
                                        : "out must not overlap x or z");
    int chunk = chunked ? (chunk_rows < p.R ? chunk_rows : p.R) : p.R;
    const size_t need = workspace_need(p, chunk);
    if (!wsp) return fail(FF_EINVAL, "workspace is NULL (%zu bytes needed)", need);
    if (((uintptr_t)wsp & 255u) != 0) return fail(FF_EINVAL, "workspace must be 256-byte aligned");
    if (ws_bytes < need) return fail(FF_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", ws_bytes, need);
    if (overlaps(out, x_bytes, wsp, need)) return fail(FF_EINVAL, "out must not overlap the workspace");

    hipStream_t stream = (hipStream_t)stream_;
    bool fast = mfma_supported(p) && mfma_chunk_ok(p, chunk) && aligned16(x) && aligned16(out) && aligned16(z);
    const void* wp[] = {w->ln_g, w->ln_b, w->lnz_g, w->lnz_b, w->w_q, w->w_k, w->w_v, w->w_b, w->w_g, w->b_g, w->w_o, w->b_o};
    for (const void* q : wp) fast = fast && aligned16(q);
    Workspace ws;
    carve(p, chunk, &ws, wsp, fast);
    g_last_path = fast ? "mfma_bf16" : "generic";
    if (fast) {
        st = mfma_prepare(p, *w, x, z, ws, stream);
    } else {
        st = generic_prepare(p, *w, x, z, ws, stream);
    }
    if (st != FF_OK) return st;
    for (int r0 = 0; r0 < p.R; r0 += chunk) {
        int rows = p.R - r0 < chunk ? p.R - r0 : chunk;
        if (fast) {
            st = mfma_chunk(p, *w, x, mask, residual ? x : nullptr, out, ws, r0, rows, stream);
        } else {
            Timed t(KK_GENERIC, stream);
            st = generic_chunk(p, *w, x, z, mask, residual ? x : nullptr, out, ws, r0, rows, stream);
        }
        if (st != FF_OK) return st;
    }
    return FF_OK;
}

// ---- device memory of the library's own, for callers that cannot hand over a workspace -------
// ff_gated_attention_static runs the chunked path with this array as its workspace.  Every GPU the
// library runs on holds its own copy until the process ends.  In host code the array's name is only
// a handle for hipGetSymbolAddress: the device address is looked up once per device (with that
// device current) and used everywhere after that.
constexpr size_t kScratchBytes = (size_t)48 << 20;
static __device__ __align__(256) __attribute__((used)) unsigned char scratch[kScratchBytes];

constexpr int kMaxDevices = 64;
static std::mutex g_scratch_mu;
static void* g_scratch_ptr[kMaxDevices] = {};

static ff_status scratch_of_current_device(void** out) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail(FF_EHIP, "hipGetDevice: %s", hipGetErrorString(e));
    if (dev < 0 || dev >= kMaxDevices) return fail(FF_EUNSUPPORTED, "device index %d beyond %d", dev, kMaxDevices - 1);
    std::lock_guard<std::mutex> lk(g_scratch_mu);
    if (!g_scratch_ptr[dev]) {
        void* ptr = nullptr;
        e = hipGetSymbolAddress((void**)&ptr, HIP_SYMBOL(scratch));
        if (e != hipSuccess || !ptr)
            return fail(FF_EHIP, "hipGetSymbolAddress(scratch) on device %d: %s", dev, hipGetErrorString(e));
        g_scratch_ptr[dev] = ptr;
    }
    *out = g_scratch_ptr[dev];
    return FF_OK;
}

// largest chunk (batch rows per launch sequence) whose workspace fits `limit` bytes; 0 if not even one row does
static int largest_chunk_within(const Problem& p, size_t limit) {
    if (workspace_need(p, 1) > limit) return 0;
    int lo = 1, hi = p.R;                      // workspace_need grows with the chunk
    while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (workspace_need(p, mid) <= limit) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

}  // namespace ff

using namespace ff;

extern "C" {

ff_status ff_layernorm(const void* x, const void* gamma, const void* beta, void* y, int64_t rows, int32_t c,
                       float eps, int32_t dt, void* hip_stream) {
    if (dt != FF_F32 && dt != FF_BF16) return fail(FF_EINVAL, "bad dtype %d", dt);
    if (rows < 0 || c < 1 || c > 8192) return fail(FF_EINVAL, "bad size rows=%lld c=%d", (long long)rows, c);
    if (!(eps >= 0.f)) return fail(FF_EINVAL, "eps must be >= 0");
    if (rows == 0) return FF_OK;
    if (!x || !gamma || !beta || !y) return fail(FF_EINVAL, "NULL pointer");
    Timed t(KK_LAYERNORM, (hipStream_t)hip_stream);
    return layernorm_launch(x, gamma, beta, y, rows, c, eps, dt, (hipStream_t)hip_stream);
}

static ff_status check_trimul(const ff_trimul_desc* d) {
    if (!d) return fail(FF_EINVAL, "desc is NULL");
    if (d->dtype != FF_F32 && d->dtype != FF_BF16) return fail(FF_EINVAL, "bad dtype %d", d->dtype);
    if (d->n < 1 || d->c_z < 1 || d->c < 1) return fail(FF_EINVAL, "non-positive size (n=%d c_z=%d c=%d)", d->n, d->c_z, d->c);
    if (d->incoming != 0 && d->incoming != 1) return fail(FF_EINVAL, "incoming must be 0 or 1 (got %d)", d->incoming);
    if (!(d->ln_eps >= 0.f)) return fail(FF_EINVAL, "ln_eps must be >= 0");
    if (d->n > 16384) return fail(FF_EUNSUPPORTED, "n %d > 16384", d->n);
    if (!trimul_supported(d->dtype, d->c_z, d->c))
        return fail(FF_EUNSUPPORTED, "triangle multiplication: bfloat16 only, c_z and c multiples of 32 up to 128 "
                                     "(got dtype %d, c_z %d, c %d)", d->dtype, d->c_z, d->c);
    return FF_OK;
}

size_t ff_triangle_multiplication_workspace_bytes(const ff_trimul_desc* desc) {
    if (check_trimul(desc) != FF_OK) return 0;
    return trimul_workspace(desc->n, desc->c_z, desc->c);
}

ff_status ff_triangle_multiplication(const ff_trimul_desc* desc, const ff_trimul_weights* w, const void* z,
                                     const float* mask, void* out, int32_t residual, void* ws, size_t ws_bytes,
                                     void* hip_stream) {
    ff_status st = check_trimul(desc);
    if (st != FF_OK) return st;
    if (residual != 0 && residual != 1) return fail(FF_EINVAL, "residual must be 0 or 1 (got %d)", residual);
    if (!w || !z || !out) return fail(FF_EINVAL, "weights, z or out is NULL");
    const void* wp[] = {w->ln_g, w->ln_b, w->w_ap, w->b_ap, w->w_ag, w->b_ag, w->w_bp, w->b_bp, w->w_bg, w->b_bg,
                        w->w_g, w->b_g, w->lno_g, w->lno_b, w->w_o, w->b_o};
    for (const void* q : wp)
        if (!q) return fail(FF_EINVAL, "a weight pointer is NULL");
    if (!aligned16(z) || !aligned16(out)) return fail(FF_EINVAL, "z and out must be 16-byte aligned");
    const size_t z_bytes = (size_t)desc->n * desc->n * desc->c_z * 2;
    if (overlaps(out, z_bytes, z, z_bytes) && !(residual && out == z))
        return fail(FF_EINVAL, residual ? "out must be z itself or not overlap z" : "out must not overlap z");
    const size_t need = trimul_workspace(desc->n, desc->c_z, desc->c);
    if (!ws) return fail(FF_EINVAL, "workspace is NULL (%zu bytes needed)", need);
    if (((uintptr_t)ws & 255u) != 0) return fail(FF_EINVAL, "workspace must be 256-byte aligned");
    if (ws_bytes < need) return fail(FF_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", ws_bytes, need);
    if (overlaps(out, z_bytes, ws, need) || overlaps(z, z_bytes, ws, need))
        return fail(FF_EINVAL, "z and out must not overlap the workspace");
    return trimul_run(*desc, *w, z, mask, residual != 0, out, ws, (hipStream_t)hip_stream);
}

static ff_status check_global(const ff_global_desc* d) {
    if (!d) return fail(FF_EINVAL, "desc is NULL");
    if (d->dtype != FF_F32 && d->dtype != FF_BF16) return fail(FF_EINVAL, "bad dtype %d", d->dtype);
    if (d->n_seq < 1 || d->n_res < 1 || d->c < 1 || d->heads < 1 || d->head_dim < 1)
        return fail(FF_EINVAL, "non-positive size (n_seq=%d n_res=%d c=%d heads=%d head_dim=%d)", d->n_seq, d->n_res, d->c,
                    d->heads, d->head_dim);
    if (!(d->ln_eps >= 0.f)) return fail(FF_EINVAL, "ln_eps must be >= 0");
    if ((int64_t)d->n_seq * d->n_res > ((int64_t)1 << 31) - 1) return fail(FF_EUNSUPPORTED, "more than 2^31 tokens");
    if (!global_supported(*d))
        return fail(FF_EUNSUPPORTED, "global column attention: bfloat16 only, c a multiple of 32 up to 128, head_dim 8 or 16, "
                                     "heads*head_dim 32, 64 or 128 (got dtype %d, c %d, heads %d, head_dim %d)",
                    d->dtype, d->c, d->heads, d->head_dim);
    return FF_OK;
}

size_t ff_global_column_attention_workspace_bytes(const ff_global_desc* desc) {
    if (check_global(desc) != FF_OK) return 0;
    return global_workspace(*desc);
}

ff_status ff_global_column_attention(const ff_global_desc* desc, const ff_global_weights* w, const void* m,
                                     const float* mask, void* out, void* ws, size_t ws_bytes, void* hip_stream) {
    ff_status st = check_global(desc);
    if (st != FF_OK) return st;
    if (!w || !m || !out) return fail(FF_EINVAL, "weights, m or out is NULL");
    const void* wp[] = {w->ln_g, w->ln_b, w->w_q, w->w_k, w->w_v, w->w_g, w->b_g, w->w_o, w->b_o};
    for (const void* q : wp)
        if (!q) return fail(FF_EINVAL, "a weight pointer is NULL");
    if (!aligned16(m) || !aligned16(out)) return fail(FF_EINVAL, "m and out must be 16-byte aligned");
    const size_t m_bytes = (size_t)desc->n_seq * desc->n_res * desc->c * 2;
    if (overlaps(out, m_bytes, m, m_bytes)) return fail(FF_EINVAL, "out must not overlap m");
    const size_t need = global_workspace(*desc);
    if (!ws) return fail(FF_EINVAL, "workspace is NULL (%zu bytes needed)", need);
    if (((uintptr_t)ws & 255u) != 0) return fail(FF_EINVAL, "workspace must be 256-byte aligned");
    if (ws_bytes < need) return fail(FF_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", ws_bytes, need);
    if (overlaps(out, m_bytes, ws, need) || overlaps(m, m_bytes, ws, need))
        return fail(FF_EINVAL, "m and out must not overlap the workspace");
    return global_run(*desc, *w, m, mask, out, ws, (hipStream_t)hip_stream);
}

static ff_status check_core(const ff_core_desc* d) {
    if (!d) return fail(FF_EINVAL, "desc is NULL");
    if (d->dtype != FF_F32 && d->dtype != FF_BF16) return fail(FF_EINVAL, "bad dtype %d", d->dtype);
    if (d->rows < 1 || d->heads < 1 || d->length < 1 || d->head_dim < 1)
        return fail(FF_EINVAL, "non-positive size (rows=%d heads=%d length=%d head_dim=%d)", d->rows, d->heads, d->length, d->head_dim);
    if (d->length > 16384) return fail(FF_EUNSUPPORTED, "length %d > 16384", d->length);
    const int64_t tiles = (int64_t)d->rows * d->heads * ((d->length + 31) / 32);
    const int64_t btiles = (int64_t)d->heads * ((d->length + 31) / 32) * ((d->length + 31) / 32);
    if (tiles > ((int64_t)1 << 30) || btiles > ((int64_t)1 << 30)) return fail(FF_EUNSUPPORTED, "too many tiles for one launch");
    if (!core_backward_supported(*d))
        return fail(FF_EUNSUPPORTED, "attention core backward: bfloat16 only, head_dim 8, 16 or 32 (got dtype %d, head_dim %d)",
                    d->dtype, d->head_dim);
    return FF_OK;
}

size_t ff_attention_core_backward_workspace_bytes(const ff_core_desc* desc) {
    if (check_core(desc) != FF_OK) return 0;
    return core_backward_workspace(*desc);
}

ff_status ff_attention_core_backward(const ff_core_desc* desc, const void* q, const void* k, const void* v, const void* g,
                                     const float* bias, const float* mask, const void* dout, void* dq, void* dk, void* dv,
                                     void* dg, float* dbias, void* ws, size_t ws_bytes, void* hip_stream) {
    ff_status st = check_core(desc);
    if (st != FF_OK) return st;
    if (!q || !k || !v || !g || !dout || !dq || !dk || !dv || !dg) return fail(FF_EINVAL, "a required tensor pointer is NULL");
    if ((bias == nullptr) != (dbias == nullptr)) return fail(FF_EINVAL, "dbias must be given exactly when bias is");
    if (!aligned16(bias) || !aligned16(dbias)) return fail(FF_EINVAL, "bias and dbias must be 16-byte aligned");
    const void* ptrs[] = {q, k, v, g, dout, dq, dk, dv, dg};
    for (const void* t : ptrs)
        if (!aligned16(t)) return fail(FF_EINVAL, "tensor pointers must be 16-byte aligned");
    const size_t n_bytes = (size_t)desc->rows * desc->heads * desc->length * desc->head_dim * 2;
    const void* ins[] = {q, k, v, g, dout};
    void* outs[] = {dq, dk, dv, dg};
    for (void* o : outs) {
        for (const void* in : ins)
            if (overlaps(o, n_bytes, in, n_bytes)) return fail(FF_EINVAL, "a gradient tensor overlaps an input");
        for (void* o2 : outs)
            if (o != o2 && overlaps(o, n_bytes, o2, n_bytes)) return fail(FF_EINVAL, "gradient tensors overlap each other");
    }
    const size_t need = core_backward_workspace(*desc);
    if (!ws) return fail(FF_EINVAL, "workspace is NULL (%zu bytes needed)", need);
    if (((uintptr_t)ws & 255u) != 0) return fail(FF_EINVAL, "workspace must be 256-byte aligned");
    if (ws_bytes < need) return fail(FF_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", ws_bytes, need);
    return core_backward_run(*desc, q, k, v, g, bias, mask, dout, dq, dk, dv, dg, dbias, ws, (hipStream_t)hip_stream);
}

// ---- layer norm in training
static ff_status check_norm(const ff_norm_desc* d) {
    if (!d) return fail(FF_EINVAL, "desc is NULL");
    if (d->dtype != FF_F32 && d->dtype != FF_BF16) return fail(FF_EINVAL, "bad dtype %d", d->dtype);
    if (d->rows < 0 || d->c < 1 || d->c > 8192 || d->rows > (int64_t)1 << 40)
        return fail(FF_EINVAL, "bad size rows=%lld c=%d", (long long)d->rows, d->c);
    if (!(d->ln_eps >= 0.f)) return fail(FF_EINVAL, "ln_eps must be >= 0");
    return FF_OK;
}
static bool aligned_to(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) == 0; }

ff_status ff_layernorm_forward(const ff_norm_desc* desc, const void* x, const void* residual, const void* gamma, const void* beta,
                               void* sum, void* y, float* mean, float* rstd, void* hip_stream) {
    ff_status st = check_norm(desc);
    if (st != FF_OK) return st;
    if ((residual == nullptr) != (sum == nullptr)) return fail(FF_EINVAL, "sum must be given exactly when residual is");
    if ((mean == nullptr) != (rstd == nullptr)) return fail(FF_EINVAL, "mean and rstd must be given together");
    if (desc->rows == 0) return FF_OK;
    if (!x || !gamma || !beta || !y) return fail(FF_EINVAL, "NULL pointer");
    const size_t esz = desc->dtype == FF_F32 ? 4 : 2, n = (size_t)desc->rows * desc->c * esz;
    const void* ptrs[] = {x, residual, gamma, beta, sum, y};
    for (const void* p : ptrs)
        if (!aligned_to(p, esz)) return fail(FF_EINVAL, "a pointer is not aligned to its type");
    if (!aligned_to(mean, 4) || !aligned_to(rstd, 4)) return fail(FF_EINVAL, "mean and rstd must be 4-byte aligned");
    if (overlaps(y, n, x, n) || (residual && (overlaps(y, n, residual, n) || overlaps(y, n, sum, n))))
        return fail(FF_EINVAL, "y must not overlap x, residual or sum");
    if (sum && ((sum != x && overlaps(sum, n, x, n)) || (sum != residual && overlaps(sum, n, residual, n))))
        return fail(FF_EINVAL, "sum must be x itself, residual itself, or overlap neither");
    const size_t cb = desc->c * esz, rb = (size_t)desc->rows * 4;
    for (const void* w : {gamma, beta})
        if (overlaps(y, n, w, cb) || (sum && overlaps(sum, n, w, cb)) || (mean && (overlaps(mean, rb, w, cb) || overlaps(rstd, rb, w, cb))))
            return fail(FF_EINVAL, "an output overlaps gamma or beta");
    if (mean) {
        if (overlaps(mean, rb, rstd, rb)) return fail(FF_EINVAL, "mean and rstd overlap");
        for (const void* t : {x, residual, (const void*)sum, (const void*)y})
            if (t && (overlaps(mean, rb, t, n) || overlaps(rstd, rb, t, n))) return fail(FF_EINVAL, "mean or rstd overlaps a tensor");
    }
    return layernorm_forward_run(*desc, x, residual, gamma, beta, sum, y, mean, rstd, (hipStream_t)hip_stream);
}

size_t ff_layernorm_backward_workspace_bytes(const ff_norm_desc* desc) {
    if (check_norm(desc) != FF_OK) return 0;
    return layernorm_backward_workspace(*desc);
}

ff_status ff_layernorm_backward(const ff_norm_desc* desc, const void* s, const void* gamma, const float* mean, const float* rstd,
                                const void* dy, const void* dsum, void* dx, float* dgamma, float* dbeta, int32_t accumulate,
                                void* ws, size_t ws_bytes, void* hip_stream) {
    ff_status st = check_norm(desc);
    if (st != FF_OK) return st;
    if ((mean == nullptr) != (rstd == nullptr)) return fail(FF_EINVAL, "mean and rstd must be given together");
    if (accumulate != 0 && accumulate != 1) return fail(FF_EINVAL, "accumulate must be 0 or 1 (got %d)", accumulate);
    if (!gamma || !dgamma || !dbeta || (desc->rows > 0 && (!s || !dy || !dx))) return fail(FF_EINVAL, "NULL pointer");
    const size_t esz = desc->dtype == FF_F32 ? 4 : 2, n = (size_t)desc->rows * desc->c * esz;
    const void* ptrs[] = {s, gamma, dy, dsum, dx};
    for (const void* p : ptrs)
        if (!aligned_to(p, esz)) return fail(FF_EINVAL, "a pointer is not aligned to its type");
    const float* floats[] = {mean, rstd, dgamma, dbeta};
    for (const float* p : floats)
        if (!aligned_to(p, 4)) return fail(FF_EINVAL, "mean, rstd, dgamma and dbeta must be 4-byte aligned");
    if (overlaps(dx, n, s, n)) return fail(FF_EINVAL, "dx must not overlap s");
    if ((dx != dy && overlaps(dx, n, dy, n)) || (dsum && dx != dsum && overlaps(dx, n, dsum, n)))
        return fail(FF_EINVAL, "dx must be dy itself, dsum itself, or overlap neither");
    const size_t need = layernorm_backward_workspace(*desc), cb = (size_t)desc->c * 4;
    if (overlaps(dgamma, cb, dbeta, cb)) return fail(FF_EINVAL, "dgamma and dbeta overlap");
    const size_t wb = desc->c * esz, rb = (size_t)desc->rows * 4;
    for (const void* o : {(const void*)dgamma, (const void*)dbeta}) {
        for (const void* t : {s, dy, dsum, (const void*)dx})
            if (t && overlaps(o, cb, t, n)) return fail(FF_EINVAL, "dgamma or dbeta overlaps a tensor");
        if (overlaps(o, cb, gamma, wb) || (mean && (overlaps(o, cb, mean, rb) || overlaps(o, cb, rstd, rb))) || (ws && overlaps(o, cb, ws, need)))
            return fail(FF_EINVAL, "dgamma or dbeta overlaps an input or the workspace");
    }
    if (overlaps(dx, n, gamma, wb) || (mean && (overlaps(dx, n, mean, rb) || overlaps(dx, n, rstd, rb))))
        return fail(FF_EINVAL, "dx overlaps gamma, mean or rstd");
    for (const void* t : {s, dy, dsum, (const void*)dx})
        if (t && ws && overlaps(ws, need, t, n)) return fail(FF_EINVAL, "the workspace overlaps a tensor");
    if (ws && (overlaps(ws, need, gamma, wb) || (mean && (overlaps(ws, need, mean, rb) || overlaps(ws, need, rstd, rb)))))
        return fail(FF_EINVAL, "the workspace overlaps gamma, mean or rstd");
    if (!ws) return fail(FF_EINVAL, "workspace is NULL (%zu bytes needed)", need);
    if (((uintptr_t)ws & 255u) != 0) return fail(FF_EINVAL, "workspace must be 256-byte aligned");
    if (ws_bytes < need) return fail(FF_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", ws_bytes, need);
    return layernorm_backward_run(*desc, s, gamma, mean, rstd, dy, dsum, dx, dgamma, dbeta, accumulate != 0, ws, (hipStream_t)hip_stream);
}

// ---- the optimiser
static ff_status check_adamw(const ff_adamw_desc* d) {
    if (!d) return fail(FF_EINVAL, "desc is NULL");
    if (d->param_dtype != FF_F32 && d->param_dtype != FF_BF16) return fail(FF_EINVAL, "bad param_dtype %d", d->param_dtype);
    if (d->grad_dtype != FF_F32 && d->grad_dtype != FF_BF16) return fail(FF_EINVAL, "bad grad_dtype %d", d->grad_dtype);
    if (d->state_bits != 0 && d->state_bits != 8 && d->state_bits != 32) return fail(FF_EINVAL, "state_bits must be 0, 8 or 32 (got %d)", d->state_bits);
    if (d->n_tensors < 0) return fail(FF_EINVAL, "n_tensors must be >= 0 (got %d)", d->n_tensors);
    return FF_OK;
}

static ff_status check_tensors(const ff_adamw_desc* d, const ff_adamw_tensor* ts) {
    ff_status st = check_adamw(d);
    if (st != FF_OK) return st;
    if (d->n_tensors > 0 && !ts) return fail(FF_EINVAL, "tensors is NULL");
    int64_t total = 0;
    for (int i = 0; i < d->n_tensors; ++i) {
        const ff_adamw_tensor& t = ts[i];
        if (t.numel < 0 || t.numel > (int64_t)1 << 40 || (total += t.numel) > (int64_t)1 << 40)
            return fail(FF_EINVAL, "tensor %d: bad numel %lld", i, (long long)t.numel);
        if (t.numel == 0) continue;
        if (!t.g || !aligned_to(t.g, d->grad_dtype == FF_F32 ? 4 : 2)) return fail(FF_EINVAL, "tensor %d: g is NULL or misaligned", i);
        if (d->state_bits == 0) continue;
        if (!t.p || !t.m || !t.v) return fail(FF_EINVAL, "tensor %d: p, m or v is NULL", i);
        if (!aligned_to(t.p, d->param_dtype == FF_F32 ? 4 : 2)) return fail(FF_EINVAL, "tensor %d: p is misaligned", i);
        if (t.master && (d->param_dtype != FF_BF16 || !aligned_to(t.master, 4)))
            return fail(FF_EINVAL, "tensor %d: master belongs to bfloat16 parameters and is 4-byte aligned", i);
        if (d->state_bits == 32 && (!aligned_to(t.m, 4) || !aligned_to(t.v, 4))) return fail(FF_EINVAL, "tensor %d: m or v is misaligned", i);
        if ((d->state_bits == 8) != (t.m_exp != nullptr) || (d->state_bits == 8) != (t.v_exp != nullptr))
            return fail(FF_EINVAL, "tensor %d: m_exp and v_exp belong to 8-bit states", i);
        if (!(t.weight_decay >= 0.f) || t.weight_decay > 1e30f) return fail(FF_EINVAL, "tensor %d: weight_decay must be finite and >= 0", i);
    }
    return FF_OK;
}

static ff_status check_plan(const ff_adamw_desc* d, const void* plan, size_t bytes) {
    ff_status st = check_adamw(d);
    if (st != FF_OK) return st;
    if (!plan) return fail(FF_EINVAL, "plan is NULL");
    if (!aligned16(plan)) return fail(FF_EINVAL, "plan must be 16-byte aligned");
    if (!adamw_plan_whole(bytes)) return fail(FF_EINVAL, "no plan has %zu bytes", bytes);
    return FF_OK;
}

size_t ff_adamw_plan_bytes(const ff_adamw_desc* desc, const ff_adamw_tensor* tensors) {
    if (check_tensors(desc, tensors) != FF_OK) return 0;
    const size_t bytes = adamw_plan_size(*desc, tensors);
    if (!adamw_plan_whole(bytes)) {
        fail(FF_EUNSUPPORTED, "the tensors need more pieces than one launch has blocks");
        return 0;
    }
    return bytes;
}

ff_status ff_adamw_plan(const ff_adamw_desc* desc, const ff_adamw_tensor* tensors, void* plan, size_t plan_bytes) {
    ff_status st = check_tensors(desc, tensors);
    if (st != FF_OK) return st;
    const size_t need = adamw_plan_size(*desc, tensors);
    if (!adamw_plan_whole(need)) return fail(FF_EUNSUPPORTED, "the tensors need more pieces than one launch has blocks");
    if (!plan || !aligned_to(plan, 8)) return fail(FF_EINVAL, "plan is NULL or misaligned");
    if (plan_bytes != need) return fail(FF_EWORKSPACE, "the plan has %zu bytes, %zu given", need, plan_bytes);
    const int overlaps = adamw_overlaps(*desc, tensors);
    if (overlaps < 0) return fail(FF_EINVAL, "no host memory for %d tensors", desc->n_tensors);
    if (overlaps) return fail(FF_EINVAL, "a tensor that the step writes overlaps another one of the plan");
    adamw_plan_fill(*desc, tensors, plan);
    return FF_OK;
}

size_t ff_grad_norm_workspace_bytes(void) { return grad_norm_workspace(); }

ff_status ff_grad_norm(const ff_adamw_desc* desc, const void* plan, size_t plan_bytes, float* norm, void* ws, size_t ws_bytes,
                       void* hip_stream) {
    ff_status st = check_plan(desc, plan, plan_bytes);
    if (st != FF_OK) return st;
    if (!norm || !aligned_to(norm, 4)) return fail(FF_EINVAL, "norm is NULL or misaligned");
    if (!ws) return fail(FF_EINVAL, "workspace is NULL (%zu bytes needed)", grad_norm_workspace());
    if (((uintptr_t)ws & 255u) != 0) return fail(FF_EINVAL, "workspace must be 256-byte aligned");
    if (ws_bytes < grad_norm_workspace())
        return fail(FF_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", ws_bytes, grad_norm_workspace());
    if (overlaps(norm, 4, ws, grad_norm_workspace())) return fail(FF_EINVAL, "norm overlaps the workspace");
    if (overlaps(norm, 4, plan, plan_bytes) || overlaps(ws, grad_norm_workspace(), plan, plan_bytes))
        return fail(FF_EINVAL, "norm or the workspace overlaps the plan");
    return grad_norm_run(*desc, plan, plan_bytes, norm, ws, (hipStream_t)hip_stream);
}

ff_status ff_adamw_step(const ff_adamw_desc* desc, const void* plan, size_t plan_bytes, const ff_adamw_hyper* h, const float* norm,
                        void* hip_stream) {
    ff_status st = check_plan(desc, plan, plan_bytes);
    if (st != FF_OK) return st;
    if (desc->state_bits == 0) return fail(FF_EINVAL, "a plan of gradients alone has nothing to step");
    if (!h) return fail(FF_EINVAL, "hyper is NULL");
    if (!(h->lr >= 0.) || h->lr > 1e30 || !(h->eps >= 0.) || h->eps > 1e30) return fail(FF_EINVAL, "lr and eps must be finite and >= 0");
    if (!(h->beta1 >= 0.) || !(h->beta1 < 1.) || !(h->beta2 >= 0.) || !(h->beta2 < 1.)) return fail(FF_EINVAL, "beta1 and beta2 must be in [0, 1)");
    if (h->step < 1) return fail(FF_EINVAL, "step must be >= 1 (got %lld)", (long long)h->step);
    if (norm && (!(h->max_norm > 0.) || h->max_norm > 1e30)) return fail(FF_EINVAL, "max_norm must be finite and > 0");
    if (!aligned_to(norm, 4)) return fail(FF_EINVAL, "norm is misaligned");
    return adamw_step_run(*desc, plan, plan_bytes, *h, norm, (hipStream_t)hip_stream);
}

ff_status ff_adamw_moments(const ff_adamw_desc* desc, const void* plan, size_t plan_bytes, float* m_out, float* v_out, void* hip_stream) {
    ff_status st = check_plan(desc, plan, plan_bytes);
    if (st != FF_OK) return st;
    if (desc->state_bits == 0) return fail(FF_EINVAL, "a plan of gradients alone has no moments");
    if (!aligned_to(m_out, 4) || !aligned_to(v_out, 4)) return fail(FF_EINVAL, "m_out or v_out is misaligned");
    if (!m_out && !v_out) return FF_OK;
    const size_t least = adamw_least_values(*desc, plan_bytes) * 4;
    if (m_out && v_out && overlaps(m_out, least, v_out, least)) return fail(FF_EINVAL, "m_out and v_out overlap");
    if ((m_out && overlaps(m_out, least, plan, plan_bytes)) || (v_out && overlaps(v_out, least, plan, plan_bytes)))
        return fail(FF_EINVAL, "m_out or v_out overlaps the plan");
    return adamw_moments_run(*desc, plan, plan_bytes, m_out, v_out, (hipStream_t)hip_stream);
}

// ---- the gated transition
static ff_status check_transition(const ff_transition_desc* d) {
    if (!d) return fail(FF_EINVAL, "desc is NULL");
    if (d->dtype != FF_F32 && d->dtype != FF_BF16) return fail(FF_EINVAL, "bad dtype %d", d->dtype);
    if (d->act != FF_SILU && d->act != FF_GELU && d->act != FF_SIGMOID) return fail(FF_EINVAL, "bad act %d", d->act);
    if (d->c < 1 || d->c > 8192) return fail(FF_EINVAL, "c must be in 1 .. 8192 (got %d)", d->c);
    if (d->f < 1 || d->f > 32768) return fail(FF_EINVAL, "f must be in 1 .. 32768 (got %d)", d->f);
    if (d->rows < 0 || d->rows > (int64_t)1 << 40 || d->rows * d->c > (int64_t)1 << 40) return fail(FF_EINVAL, "bad number of rows %lld", (long long)d->rows);
    return FF_OK;
}
static ff_status check_ws(const void* ws, size_t given, size_t need) {
    if (!ws) return fail(FF_EINVAL, "workspace is NULL (%zu bytes needed)", need);
    if (((uintptr_t)ws & 255u) != 0) return fail(FF_EINVAL, "workspace must be 256-byte aligned");
    if (given < need) return fail(FF_EWORKSPACE, "workspace too small: %zu bytes given, %zu needed", given, need);
    return FF_OK;
}
namespace {
struct Span {
    const void* p;
    size_t n;
    const char* name;
};
}  // namespace
// outputs overlap neither each other nor an input, but for the one that may be that input itself
static ff_status check_spans(const Span* out, int n_out, const Span* in, int n_in, const void* same_out = nullptr, const void* same_in = nullptr) {
    for (int i = 0; i < n_out; ++i) {
        if (!out[i].p || !out[i].n) continue;
        for (int j = 0; j < i; ++j)
            if (out[j].p && overlaps(out[i].p, out[i].n, out[j].p, out[j].n)) return fail(FF_EINVAL, "%s overlaps %s", out[i].name, out[j].name);
        for (int j = 0; j < n_in; ++j)
            if (in[j].p && in[j].n && !(out[i].p == same_out && in[j].p == same_in && same_out == same_in) && overlaps(out[i].p, out[i].n, in[j].p, in[j].n))
                return fail(FF_EINVAL, "%s overlaps %s", out[i].name, in[j].name);
    }
    return FF_OK;
}

size_t ff_gated_transition_forward_workspace_bytes(const ff_transition_desc* desc) {
    return check_transition(desc) == FF_OK ? transition_forward_workspace(*desc) : 0;
}
size_t ff_gated_transition_backward_workspace_bytes(const ff_transition_desc* desc) {
    return check_transition(desc) == FF_OK ? transition_backward_workspace(*desc) : 0;
}

ff_status ff_gated_transition_forward(const ff_transition_desc* desc, const void* x, const void* w_a, const void* w_b, const void* w_o, const void* residual,
                                      const float* mask, void* y, void* ws, size_t ws_bytes, void* hip_stream) {
    ff_status st = check_transition(desc);
    if (st != FF_OK) return st;
    if (desc->rows == 0) return FF_OK;
    if (!x || !w_a || !w_b || !w_o || !y) return fail(FF_EINVAL, "NULL pointer");
    const size_t esz = desc->dtype == FF_F32 ? 4 : 2, n = (size_t)desc->rows * desc->c * esz, wn = (size_t)desc->c * desc->f * esz;
    for (const void* p : {x, w_a, w_b, w_o, residual, (const void*)y})
        if (!aligned_to(p, esz)) return fail(FF_EINVAL, "a pointer is not aligned to its type");
    if (!aligned_to(mask, 4)) return fail(FF_EINVAL, "mask must be 4-byte aligned");
    const size_t need = transition_forward_workspace(*desc);
    if ((st = check_ws(ws, ws_bytes, need)) != FF_OK) return st;
    const Span in[] = {{x, n, "x"}, {w_a, wn, "w_a"}, {w_b, wn, "w_b"}, {w_o, wn, "w_o"}, {mask, (size_t)desc->rows * 4, "mask"}};
    const Span out[] = {{y, n, "y"}, {ws, need, "the workspace"}}, kept[] = {{residual, n, "residual"}};
    if ((st = check_spans(out, 2, in, 5)) != FF_OK) return st;
    if ((st = check_spans(out, 2, kept, 1, y, residual)) != FF_OK) return st;
    return transition_forward_run(*desc, x, w_a, w_b, w_o, residual, mask, y, ws, (hipStream_t)hip_stream);
}

ff_status ff_gated_transition_backward(const ff_transition_desc* desc, const void* x, const void* w_a, const void* w_b, const void* w_o, const void* dy,
                                       const float* mask, void* dx, void* dw_a, void* dw_b, void* dw_o, int32_t grad_dtype, int32_t accumulate, void* ws,
                                       size_t ws_bytes, void* hip_stream) {
    ff_status st = check_transition(desc);
    if (st != FF_OK) return st;
    if (grad_dtype != FF_F32 && grad_dtype != FF_BF16) return fail(FF_EINVAL, "bad grad_dtype %d", grad_dtype);
    if (accumulate != 0 && accumulate != 1) return fail(FF_EINVAL, "accumulate must be 0 or 1 (got %d)", accumulate);
    if (!w_a || !w_b || !w_o || !dw_a || !dw_b || !dw_o || (desc->rows > 0 && (!x || !dy || !dx))) return fail(FF_EINVAL, "NULL pointer");
    const size_t esz = desc->dtype == FF_F32 ? 4 : 2, gsz = grad_dtype == FF_F32 ? 4 : 2, n = (size_t)desc->rows * desc->c * esz,
                 wn = (size_t)desc->c * desc->f * esz, gn = (size_t)desc->c * desc->f * gsz;
    for (const void* p : {x, w_a, w_b, w_o, dy, (const void*)dx})
        if (!aligned_to(p, esz)) return fail(FF_EINVAL, "a pointer is not aligned to its type");
    for (const void* p : {dw_a, dw_b, dw_o})
        if (!aligned_to(p, gsz)) return fail(FF_EINVAL, "a gradient is not aligned to its type");
    if (!aligned_to(mask, 4)) return fail(FF_EINVAL, "mask must be 4-byte aligned");
    const size_t need = transition_backward_workspace(*desc);
    if ((st = check_ws(ws, ws_bytes, need)) != FF_OK) return st;
    const Span in[] = {{x, n, "x"}, {w_a, wn, "w_a"}, {w_b, wn, "w_b"}, {w_o, wn, "w_o"}, {dy, n, "dy"}, {mask, (size_t)desc->rows * 4, "mask"}};
    const Span out[] = {{dx, n, "dx"}, {dw_a, gn, "dw_a"}, {dw_b, gn, "dw_b"}, {dw_o, gn, "dw_o"}, {ws, need, "the workspace"}};
    if ((st = check_spans(out, 5, in, 6)) != FF_OK) return st;
    return transition_backward_run(*desc, x, w_a, w_b, w_o, dy, mask, dx, dw_a, dw_b, dw_o, grad_dtype, accumulate != 0, ws, (hipStream_t)hip_stream);
}

// ---- orthogonalising, the optimiser of matrices
static bool is_finite(double v) { return v - v == 0.; }
static ff_status check_polynomial(double a, double b, double c, double eps, int steps) {
    if (!is_finite((float)a) || !is_finite((float)b) || !is_finite((float)c)) return fail(FF_EINVAL, "a, b and c must be finite");
    if (!(eps >= 0.) || !is_finite(eps)) return fail(FF_EINVAL, "eps must be finite and >= 0");
    if (steps < 1 || steps > 64) return fail(FF_EINVAL, "steps must be in 1 .. 64 (got %d)", steps);
    return FF_OK;
}
static ff_status check_orthogonalise(const ff_orthogonalise_desc* d) {
    if (!d) return fail(FF_EINVAL, "desc is NULL");
    if (d->dtype != FF_F32 && d->dtype != FF_BF16) return fail(FF_EINVAL, "bad dtype %d", d->dtype);
    if (d->rows < 1 || d->rows > 32768 || d->cols < 1 || d->cols > 32768) return fail(FF_EINVAL, "rows and cols must be in 1 .. 32768 (got %d, %d)", d->rows, d->cols);
    if (d->count < 0 || (int64_t)d->count * d->rows * d->cols > (int64_t)1 << 36) return fail(FF_EINVAL, "bad number of matrices %d", d->count);
    return check_polynomial(d->a, d->b, d->c, d->eps, d->steps);
}
size_t ff_orthogonalise_workspace_bytes(const ff_orthogonalise_desc* desc) {
    return check_orthogonalise(desc) == FF_OK ? orthogonalise_workspace(*desc) : 0;
}
ff_status ff_orthogonalise(const ff_orthogonalise_desc* desc, const void* x, void* out, void* ws, size_t ws_bytes, void* hip_stream) {
    ff_status st = check_orthogonalise(desc);
    if (st != FF_OK) return st;
    if (desc->count == 0) return FF_OK;
    if (!x || !out) return fail(FF_EINVAL, "NULL pointer");
    const size_t esz = desc->dtype == FF_F32 ? 4 : 2, n = (size_t)desc->count * desc->rows * desc->cols * esz;
    if (!aligned_to(x, esz) || !aligned_to(out, esz)) return fail(FF_EINVAL, "a pointer is not aligned to its type");
    const size_t need = orthogonalise_workspace(*desc);
    if ((st = check_ws(ws, ws_bytes, need)) != FF_OK) return st;
    const Span in[] = {{x, n, "x"}}, outs[] = {{out, n, "out"}, {ws, need, "the workspace"}};
    if ((st = check_spans(outs, 2, in, 1, out, x)) != FF_OK) return st;
    return orthogonalise_run(*desc, x, out, ws, (hipStream_t)hip_stream);
}

static ff_status check_muon(const ff_muon_desc* d) {
    if (!d) return fail(FF_EINVAL, "desc is NULL");
    if (d->param_dtype != FF_F32 && d->param_dtype != FF_BF16) return fail(FF_EINVAL, "bad param_dtype %d", d->param_dtype);
    if (d->grad_dtype != FF_F32 && d->grad_dtype != FF_BF16) return fail(FF_EINVAL, "bad grad_dtype %d", d->grad_dtype);
    if (d->n_tensors < 0) return fail(FF_EINVAL, "n_tensors must be >= 0 (got %d)", d->n_tensors);
    return FF_OK;
}
static ff_status check_matrices(const ff_muon_desc* d, const ff_muon_tensor* ts) {
    ff_status st = check_muon(d);
    if (st != FF_OK) return st;
    if (d->n_tensors > 0 && !ts) return fail(FF_EINVAL, "tensors is NULL");
    int64_t total = 0;
    for (int i = 0; i < d->n_tensors; ++i) {
        const ff_muon_tensor& t = ts[i];
        if (t.rows < 0 || t.cols < 0 || t.rows > 32768 || t.cols > 32768) return fail(FF_EINVAL, "tensor %d: rows and cols must be in 0 .. 32768 (got %d, %d)", i, t.rows, t.cols);
        if (t.rows == 0 || t.cols == 0) continue;
        if ((total += (int64_t)t.rows * t.cols) > (int64_t)1 << 40) return fail(FF_EINVAL, "too many values");
        if (!t.p || !t.g || !t.m) return fail(FF_EINVAL, "tensor %d: p, g or m is NULL", i);
        if (!aligned_to(t.p, d->param_dtype == FF_F32 ? 4 : 2) || !aligned_to(t.g, d->grad_dtype == FF_F32 ? 4 : 2) || !aligned_to(t.m, 4))
            return fail(FF_EINVAL, "tensor %d: p, g or m is misaligned", i);
        if (t.master && (d->param_dtype != FF_BF16 || !aligned_to(t.master, 4)))
            return fail(FF_EINVAL, "tensor %d: master belongs to bfloat16 parameters and is 4-byte aligned", i);
        if (!(t.weight_decay >= 0.f) || t.weight_decay > 1e30f) return fail(FF_EINVAL, "tensor %d: weight_decay must be finite and >= 0", i);
    }
    return FF_OK;
}
size_t ff_muon_plan_bytes(const ff_muon_desc* desc, const ff_muon_tensor* tensors) {
    if (check_matrices(desc, tensors) != FF_OK) return 0;
    const size_t bytes = muon_plan_size(*desc, tensors);
    if (!bytes) fail(FF_EINVAL, "no host memory for %d matrices, or too many of them", desc->n_tensors);
    return bytes;
}
ff_status ff_muon_plan(const ff_muon_desc* desc, const ff_muon_tensor* tensors, void* plan, size_t plan_bytes) {
    ff_status st = check_matrices(desc, tensors);
    if (st != FF_OK) return st;
    const size_t need = muon_plan_size(*desc, tensors);
    if (!need) return fail(FF_EINVAL, "no host memory for %d matrices, or too many of them", desc->n_tensors);
    if (!plan || !aligned_to(plan, 8)) return fail(FF_EINVAL, "plan is NULL or misaligned");
    if (plan_bytes != need) return fail(FF_EWORKSPACE, "the plan has %zu bytes, %zu given", need, plan_bytes);
    const int found = muon_plan_fill(*desc, tensors, plan);
    if (found < 0) return fail(FF_EINVAL, "no host memory for %d matrices", desc->n_tensors);
    if (found) return fail(FF_EINVAL, "a tensor that the step writes overlaps another one of the plan");
    return FF_OK;
}
static ff_status check_muon_plan(const ff_muon_desc* desc, const void* plan_host, size_t plan_bytes) {
    ff_status st = check_muon(desc);
    if (st != FF_OK) return st;
    if (!plan_host || !aligned_to(plan_host, 8)) return fail(FF_EINVAL, "plan_host is NULL or misaligned");
    if (!muon_plan_whole(*desc, plan_host, plan_bytes)) return fail(FF_EINVAL, "this is no plan of this descriptor");
    return FF_OK;
}
size_t ff_muon_workspace_bytes(const ff_muon_desc* desc, const void* plan_host, size_t plan_bytes) {
    return check_muon_plan(desc, plan_host, plan_bytes) == FF_OK ? muon_workspace(plan_host) : 0;
}
ff_status ff_muon_step(const ff_muon_desc* desc, const void* plan_host, const void* plan, size_t plan_bytes, const ff_muon_hyper* h, const float* norm, void* ws,
                       size_t ws_bytes, void* hip_stream) {
    ff_status st = check_muon_plan(desc, plan_host, plan_bytes);
    if (st != FF_OK) return st;
    if (!plan || !aligned16(plan)) return fail(FF_EINVAL, "plan is NULL or not 16-byte aligned");
    if (!h) return fail(FF_EINVAL, "hyper is NULL");
    if (!(h->lr >= 0.) || h->lr > 1e30) return fail(FF_EINVAL, "lr must be finite and >= 0");
    if (!(h->beta >= 0.) || !(h->beta < 1.)) return fail(FF_EINVAL, "beta must be in [0, 1)");
    if (h->nesterov != 0 && h->nesterov != 1) return fail(FF_EINVAL, "nesterov must be 0 or 1 (got %d)", h->nesterov);
    if (h->scale != FF_MUON_SPECTRAL && h->scale != FF_MUON_RMS) return fail(FF_EINVAL, "bad scale %d", h->scale);
    if ((st = check_polynomial(h->a, h->b, h->c, h->eps, h->steps)) != FF_OK) return st;
    if (norm && (!(h->max_norm > 0.) || h->max_norm > 1e30)) return fail(FF_EINVAL, "max_norm must be finite and > 0");
    if (!aligned_to(norm, 4)) return fail(FF_EINVAL, "norm is misaligned");
    const size_t need = muon_workspace(plan_host);
    if ((st = check_ws(ws, ws_bytes, need)) != FF_OK) return st;
    const Span in[] = {{plan, plan_bytes, "the plan"}, {norm, 4, "norm"}}, out[] = {{ws, need, "the workspace"}};
    if ((st = check_spans(out, 1, in, 2)) != FF_OK) return st;
    return muon_step_run(*desc, plan_host, plan, *h, norm, ws, (hipStream_t)hip_stream);
}

size_t ff_attention_workspace_bytes(const ff_attn_desc* desc, int32_t chunk_rows) {
    Problem p;
    if (make_problem(desc, &p) != FF_OK) return 0;
    if (chunk_rows < 0) {
        fail(FF_EINVAL, "chunk_rows must be >= 0");
        return 0;
    }
    int chunk = (chunk_rows == 0 || chunk_rows > p.R) ? p.R : chunk_rows;
    return workspace_need(p, chunk);
}

ff_status ff_gated_attention(const ff_attn_desc* desc, const ff_attn_weights* w, const void* x, const void* z,
                             const float* mask, void* out, void* ws, size_t ws_bytes, void* hip_stream) {
    return run(desc, w, x, z, mask, out, ws, ws_bytes, hip_stream, 0, false);
}

ff_status ff_attention_chunked(const ff_attn_desc* desc, const ff_attn_weights* w, const void* x, const void* z,
                               const float* mask, void* out, void* ws, size_t ws_bytes, void* hip_stream,
                               int32_t chunk_rows) {
    return run(desc, w, x, z, mask, out, ws, ws_bytes, hip_stream, chunk_rows, true);
}

ff_status ff_gated_attention_residual(const ff_attn_desc* desc, const ff_attn_weights* w, const void* x,
                                      const void* z, const float* mask, void* out, void* ws, size_t ws_bytes,
                                      void* hip_stream, int32_t chunk_rows) {
    if (chunk_rows < 0) return fail(FF_EINVAL, "chunk_rows must be >= 0 (got %d)", chunk_rows);
    return run(desc, w, x, z, mask, out, ws, ws_bytes, hip_stream, chunk_rows, chunk_rows > 0, true);
}

ff_status ff_gated_attention_static(const ff_attn_desc* desc, const ff_attn_weights* w, const void* x, const void* z,
                                    const float* mask, void* out, void* hip_stream) {
    Problem p;
    ff_status st = make_problem(desc, &p);
    if (st != FF_OK) return st;
    const int chunk = largest_chunk_within(p, kScratchBytes);
    if (chunk < 1)
        return fail(FF_EWORKSPACE, "shape too large for the static scratch: one batch row needs %zu bytes, %zu available",
                    workspace_need(p, 1), kScratchBytes);
    void* ptr = nullptr;
    st = scratch_of_current_device(&ptr);
    if (st != FF_OK) return st;
    return run(desc, w, x, z, mask, out, ptr, kScratchBytes, hip_stream, chunk, true);
}

size_t ff_static_scratch_bytes(void) { return kScratchBytes; }

const char* ff_attention_path(const ff_attn_desc* desc) {
    Problem p;
    if (make_problem(desc, &p) != FF_OK) return nullptr;
    return mfma_supported(p) ? "mfma_bf16" : "generic";
}

const char* ff_attention_last_path(void) { return g_last_path; }

void ff_profile_enable(int32_t on) {
    std::lock_guard<std::mutex> lk(g_prof_mu);
    for (auto& r : g_prof) {
        g_prof_pool.push_back(r.a);
        g_prof_pool.push_back(r.b);
    }
    g_prof.clear();
    g_prof_on = on != 0;
}

int32_t ff_profile_kinds(void) { return KK_COUNT; }

const char* ff_profile_name(int32_t kind) { return (kind >= 0 && kind < KK_COUNT) ? kKindNames[kind] : nullptr; }

ff_status ff_profile_collect(double* total_ms, int64_t* launches) {
    if (!total_ms || !launches) return fail(FF_EINVAL, "NULL pointer");
    std::lock_guard<std::mutex> lk(g_prof_mu);
    for (int i = 0; i < KK_COUNT; ++i) {
        total_ms[i] = 0.0;
        launches[i] = 0;
    }
    ff_status st = FF_OK;
    for (auto& r : g_prof) {
        float ms = 0.f;
        if (hipEventSynchronize(r.b) != hipSuccess || hipEventElapsedTime(&ms, r.a, r.b) != hipSuccess)
            st = fail(FF_EHIP, "launch timer: event read failed");
        else {
            total_ms[r.kind] += ms;
            launches[r.kind] += 1;
        }
        g_prof_pool.push_back(r.a);
        g_prof_pool.push_back(r.b);
    }
    g_prof.clear();
    return st;
}

const char* ff_last_error(void) { return g_err; }

const char* ff_version(void) { return "libff 0.1 (gfx950)"; }

}  // extern "C"
