// C ABI of the layer operators: the lf_ops handle, argument checks, dispatch to the kernels.
#include <math.h>
#include <new>
#include <string.h>

#include "lf_ops_internal.h"

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

constexpr int MAX_TOKENS = 1 << 30;      // row counters of the kernels are ints with room for a grid stride

// Collects the findings of one call; the order of precedence is the header's.
struct checker {
    const bool empty;                    // no tokens: matrices over tokens may be NULL, nothing reads them
    bool null_ = false, invalid = false, misaligned = false;
    explicit checker(int n_tokens) : empty(n_tokens == 0) { ok(n_tokens >= 0 && n_tokens <= MAX_TOKENS); }
    void matrix(const void* p) { if (!empty) require(p); }
    void require(const void* p) { if (!p) null_ = true; else if (!aligned16(p)) misaligned = true; }
    void optional(const void* p) { if (p && !aligned16(p)) misaligned = true; }
    void both(const void* q, const void* s) { if (!empty && (q == nullptr) != (s == nullptr)) null_ = true; optional(q); }
    void bytes(const void* p) { if (!empty && !p) null_ = true; }       // scale bytes: any alignment
    void ok(bool c) { if (!c) invalid = true; }
    void type(int t) { ok(t == LF_F32 || t == LF_BF16 || t == LF_F16); }
    void type16(int t) { ok(t == LF_BF16 || t == LF_F16); }
    void act(int a) { ok(a >= LF_ACT_SIGMOID && a <= LF_ACT_GELU); }
    void width(int n) { ok(n >= 8 && n <= LF_OPS_MAX_WIDTH && (n & 7) == 0); }
    // the stride of a matrix's rows; 0 = contiguous
    void ld(long long l, int n, int dtype) { ok(l == 0 || (l >= n && l % (dtype == LF_F32 ? 4 : 8) == 0 && l < (1ll << 36))); }
    int result() const { return null_ ? LF_ENULL : invalid ? LF_EINVAL : misaligned ? LF_EALIGN : LF_OK; }
};

// The handle's device, current while an entry point runs.
struct on_device {
    int before = -1;
    cudaError_t error;
    explicit on_device(const lf_ops* o)
    {
        int now = -1;
        error = cudaGetDevice(&now);
        if (error == cudaSuccess && now != o->device && (error = cudaSetDevice(o->device)) == cudaSuccess) before = now;
    }
    ~on_device() { if (before >= 0) cudaSetDevice(before); }
};
#define LF_OPS_DEVICE(o) const on_device on_device__(o); LF_OPS_TRY(o, on_device__.error)

inline long long ld_or(long long l, int n) { return l ? l : n; }

}  // namespace

extern "C" {

long long lf_ops_workspace(long long tokens, long long n_in)
{
    if (tokens < 0 || n_in < 0 || tokens > MAX_TOKENS || n_in > LF_OPS_MAX_WIDTH) return LF_EINVAL;      // (also: the product fits)
    return (long long)LF_OPS_FIXED_BYTES + ((tokens * n_in * 2 + 255) / 256) * 256;
}

int lf_ops_create(lf_ops** out, long long workspace_bytes)
{
    if (!out) return LF_ENULL;
    *out = nullptr;
    if (workspace_bytes < (long long)LF_OPS_FIXED_BYTES) return LF_EINVAL;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return LF_ECUDA; }
    cudaDeviceProp prop;
    if (cudaGetDeviceProperties(&prop, dev) != cudaSuccess) { cudaGetLastError(); return LF_ECUDA; }
    lf_ops* o = new (std::nothrow) lf_ops;
    if (!o) return LF_ENOMEM;
    memset(o, 0, sizeof(*o));
    o->device = dev;
    o->sm_count = prop.multiProcessorCount;
    o->wait_budget_us = 2000000;
    o->ws_bytes = (size_t)workspace_bytes;
    bool ok = cudaMalloc(&o->ws, o->ws_bytes) == cudaSuccess;
    ok = ok && cudaMalloc(&o->status_dev, sizeof(unsigned)) == cudaSuccess;
    ok = ok && cudaMalloc(&o->counters, LF_OPS_COUNTERS * sizeof(unsigned)) == cudaSuccess;
    ok = ok && cudaMemset(o->counters, 0, LF_OPS_COUNTERS * sizeof(unsigned)) == cudaSuccess;
    ok = ok && cudaMallocHost(&o->status_host, sizeof(unsigned)) == cudaSuccess;
    ok = ok && cudaMemset(o->status_dev, 0, sizeof(unsigned)) == cudaSuccess;
    // (the memsets are only queued, on a stream that the handle's own need not wait for)
    ok = ok && cudaStreamSynchronize(nullptr) == cudaSuccess;
    ok = ok && lf_product_tc_init(o) == LF_OK && lf_linear_stream_init() == LF_OK && lf_rows_init() == LF_OK;
    if (!ok) {
        const cudaError_t e = cudaGetLastError();
        lf_ops_destroy(o);
        return e == cudaErrorMemoryAllocation ? LF_ENOMEM : LF_ECUDA;
    }
    *o->status_host = 0;
    o->stats.sm_count = o->sm_count;
    o->stats.device = dev;
    o->stats.workspace_bytes = workspace_bytes;
    *out = o;
    return LF_OK;
}

int lf_ops_set_stream(lf_ops* o, void* cuda_stream)
{
    if (!o) return LF_ENULL;
    o->stream = (cudaStream_t)cuda_stream;
    return LF_OK;
}

int lf_ops_set_option(lf_ops* o, int key, long long value)
{
    if (!o) return LF_ENULL;
    switch (key) {
        case LF_OPT_WAIT_BUDGET_US:
            if (value < 1 || value > 60000000LL) return LF_EINVAL;
            o->wait_budget_us = value;
            return LF_OK;
        case LF_OPT_WITHHOLD:
            if (value != 0 && value != 1) return LF_EINVAL;
            o->withhold = (int)value;
            return LF_OK;
        default: return LF_EINVAL;
    }
}

int lf_ops_get_stats(lf_ops* o, lf_ops_stats* out)
{
    if (!o || !out) return LF_ENULL;
    *out = o->stats;
    return LF_OK;
}

int lf_ops_last_cuda_error(const lf_ops* o) { return o ? o->last_cuda_error : 0; }

int lf_ops_sync(lf_ops* o)
{
    if (!o) return LF_ENULL;
    LF_OPS_DEVICE(o);
    LF_OPS_TRY(o, cudaMemcpyAsync(o->status_host, o->status_dev, sizeof(unsigned), cudaMemcpyDeviceToHost, o->stream));
    LF_OPS_TRY(o, cudaStreamSynchronize(o->stream));
    o->stats.device_status = *o->status_host;
    if (*o->status_host != 0) {
        LF_OPS_TRY(o, cudaMemsetAsync(o->status_dev, 0, sizeof(unsigned), o->stream));   // the next call starts clean
        return LF_ETIMEOUT;
    }
    return LF_OK;
}

int lf_ops_destroy(lf_ops* o)
{
    if (!o) return LF_ENULL;
    const on_device there(o);
    cudaStreamSynchronize(o->stream);
    if (o->ws) cudaFree(o->ws);
    if (o->counters) cudaFree(o->counters);
    if (o->status_dev) cudaFree(o->status_dev);
    if (o->status_host) cudaFreeHost(o->status_host);
    delete o;
    return LF_OK;
}

int lf_linear(lf_ops* o, const lf_linear_args* a)
{
    if (!o || !a) return LF_ENULL;
    checker c(a->tokens);
    c.type16(a->dtype); c.act(a->act); c.width(a->n_in); c.width(a->n_out);
    c.matrix(a->x); c.require(a->w); c.matrix(a->y); c.optional(a->bias); c.optional(a->residual); c.both(a->q, a->s);
    c.ld(a->ld_x, a->n_in, a->dtype); c.ld(a->ld_residual, a->n_out, a->dtype); c.ld(a->ld_y, a->n_out, a->dtype);
    if (const int rc = c.result()) return rc;
    LF_OPS_DEVICE(o);
    o->stats.launches = 0;
    if (a->tokens == 0) return LF_OK;
    lf_product p = {};
    p.prod = LF_PROD_FORWARD; p.dtype = p.out_dtype = a->dtype; p.act = a->act;
    p.M = a->tokens; p.N = a->n_out; p.K = a->n_in;
    p.a = a->x; p.ld_a = ld_or(a->ld_x, a->n_in);
    p.b = a->w; p.ld_b = a->n_in;
    p.d = a->y; p.ld_d = ld_or(a->ld_y, a->n_out);
    p.bias = a->bias;
    p.add = a->residual; p.ld_add = ld_or(a->ld_residual, a->n_out);
    p.q = a->q; p.s = a->s;
    if (a->tokens <= LF_STREAM_MAX_TOKENS) {
        LF_OPS_TRY(o, lfk_linear_stream(p, o->sm_count, o->stream));
        o->stats.splits = 1;
        o->stats.form = LF_FORM_STREAM;
        o->stats.launches = 1;
        return LF_OK;
    }
    return lf_product_tc(o, p);
}

int lf_linear_grad_x(lf_ops* o, const lf_linear_grad_x_args* a)
{
    if (!o || !a) return LF_ENULL;
    checker c(a->tokens);
    c.type16(a->dtype); c.act(a->act); c.width(a->n_in); c.width(a->n_out);
    c.matrix(a->dz); c.require(a->w); c.matrix(a->dx); c.optional(a->add); c.both(a->q, a->s);
    c.ok(a->q || c.empty || a->act == LF_ACT_NONE);   // sigma' needs the pre-activation
    c.ld(a->ld_dz, a->n_out, a->dtype); c.ld(a->ld_add, a->n_in, a->dtype); c.ld(a->ld_dx, a->n_in, a->dtype);
    if (const int rc = c.result()) return rc;
    LF_OPS_DEVICE(o);
    o->stats.launches = 0;
    if (a->tokens == 0) return LF_OK;
    lf_product p = {};
    p.prod = LF_PROD_GRAD_X; p.dtype = p.out_dtype = a->dtype; p.act = a->act;
    p.M = a->tokens; p.N = a->n_in; p.K = a->n_out;
    p.a = a->dz; p.ld_a = ld_or(a->ld_dz, a->n_out);
    p.b = a->w; p.ld_b = a->n_in;
    p.d = a->dx; p.ld_d = ld_or(a->ld_dx, a->n_in);
    p.add = a->add; p.ld_add = ld_or(a->ld_add, a->n_in);
    if (a->act != LF_ACT_NONE) { p.q = const_cast<unsigned char*>(a->q); p.s = const_cast<unsigned char*>(a->s); }
    return lf_product_tc(o, p);
}

int lf_linear_grad_w(lf_ops* o, const lf_linear_grad_w_args* a)
{
    if (!o || !a) return LF_ENULL;
    checker c(a->tokens);
    c.type16(a->dtype); c.ok(a->gw_dtype == LF_F32 || a->gw_dtype == a->dtype); c.act(a->act);
    c.width(a->n_in); c.width(a->n_out);
    c.matrix(a->dz); c.require(a->gw); c.optional(a->gb); c.optional(a->x); c.both(a->q, a->s);
    if (!a->x) c.matrix(a->q);
    c.ok(!(a->x && a->q));                        // one form of the layer's input
    c.ok(!a->x || a->act == LF_ACT_NONE);         // x is already an activation
    c.ld(a->ld_dz, a->n_out, a->dtype); c.ld(a->ld_x, a->n_in, a->dtype);
    if (const int rc = c.result()) return rc;
    LF_OPS_DEVICE(o);
    o->stats.launches = 0;
    const size_t gw_bytes = (size_t)a->n_out * a->n_in * (a->gw_dtype == LF_F32 ? 4 : 2);
    if (a->tokens == 0) {
        LF_OPS_TRY(o, cudaMemsetAsync(a->gw, 0, gw_bytes, o->stream));
        if (a->gb) LF_OPS_TRY(o, cudaMemsetAsync(a->gb, 0, (size_t)a->n_out * sizeof(float), o->stream));
        return LF_OK;
    }
    const void* x = a->x;
    long long ld_x = ld_or(a->ld_x, a->n_in);
    if (a->q) {
        if (LF_OPS_FIXED_BYTES + (size_t)a->tokens * a->n_in * 2 > o->ws_bytes) return LF_ECAPACITY;
        void* to = o->ws + LF_OPS_FIXED_BYTES;
        x = to; ld_x = a->n_in;
    }
    if (a->q || a->gb) {
        LF_OPS_TRY(o, lfk_grad_w_prepare(*a, ld_or(a->ld_dz, a->n_out), o->ws + LF_OPS_FIXED_BYTES, reinterpret_cast<float*>(o->ws), o->counters,
                                         o->sm_count, o->stream));
        o->stats.launches += 1;
    }
    lf_product p = {};
    p.prod = LF_PROD_GRAD_W; p.dtype = a->dtype; p.out_dtype = a->gw_dtype; p.act = LF_ACT_NONE;
    p.M = a->n_out; p.N = a->n_in; p.K = a->tokens;
    p.a = a->dz; p.ld_a = ld_or(a->ld_dz, a->n_out);
    p.b = x; p.ld_b = ld_x;
    p.d = a->gw; p.ld_d = a->n_in;
    return lf_product_tc(o, p);
}

int lf_rms_norm(lf_ops* o, const lf_rms_norm_args* args)
{
    if (!o || !args) return LF_ENULL;
    lf_rms_norm_args a = *args;
    checker c(a.tokens);
    c.type(a.dtype); c.width(a.n); c.ok(a.n <= LF_OPS_MAX_NORM); c.ok(a.eps >= 0.f && isfinite(a.eps));
    c.matrix(a.x); c.require(a.gain); c.optional(a.residual); c.optional(a.h); c.optional(a.y); c.both(a.q, a.s);
    if (!a.y) c.matrix(a.q);
    c.ld(a.ld_x, a.n, a.dtype); c.ld(a.ld_residual, a.n, a.dtype); c.ld(a.ld_h, a.n, a.dtype); c.ld(a.ld_y, a.n, a.dtype);
    if (const int rc = c.result()) return rc;
    LF_OPS_DEVICE(o);
    o->stats.launches = 0;
    if (a.tokens == 0) return LF_OK;
    a.ld_x = ld_or(a.ld_x, a.n); a.ld_residual = ld_or(a.ld_residual, a.n); a.ld_h = ld_or(a.ld_h, a.n); a.ld_y = ld_or(a.ld_y, a.n);
    LF_OPS_TRY(o, lfk_rms_norm(a, o->sm_count, o->stream));
    o->stats.launches = 1;
    return LF_OK;
}

int lf_rms_norm_backward(lf_ops* o, const lf_rms_norm_backward_args* args)
{
    if (!o || !args) return LF_ENULL;
    lf_rms_norm_backward_args a = *args;
    checker c(a.tokens);
    c.type(a.dtype); c.width(a.n); c.ok(a.n <= LF_OPS_MAX_NORM); c.ok(a.eps >= 0.f && isfinite(a.eps));
    c.matrix(a.dy); c.matrix(a.h); c.require(a.gain); c.matrix(a.dh); c.optional(a.dres); c.optional(a.dgain);
    c.ld(a.ld_dy, a.n, a.dtype); c.ld(a.ld_h, a.n, a.dtype); c.ld(a.ld_dres, a.n, a.dtype); c.ld(a.ld_dh, a.n, a.dtype);
    if (const int rc = c.result()) return rc;
    LF_OPS_DEVICE(o);
    o->stats.launches = 0;
    if (a.tokens == 0) {
        if (a.dgain) LF_OPS_TRY(o, cudaMemsetAsync(a.dgain, 0, (size_t)a.n * sizeof(float), o->stream));
        return LF_OK;
    }
    a.ld_dy = ld_or(a.ld_dy, a.n); a.ld_h = ld_or(a.ld_h, a.n); a.ld_dres = ld_or(a.ld_dres, a.n); a.ld_dh = ld_or(a.ld_dh, a.n);
    LF_OPS_TRY(o, lfk_rms_norm_backward(a, reinterpret_cast<float*>(o->ws), o->sm_count, o->stream, &o->stats.launches));
    return LF_OK;
}

int lf_pack8(lf_ops* o, int dtype, int tokens, int n, const void* x, long long ld_x, unsigned char* q, unsigned char* s)
{
    if (!o) return LF_ENULL;
    checker c(tokens);
    c.type(dtype); c.width(n); c.matrix(x); c.matrix(q); c.bytes(s);
    c.ld(ld_x, n, dtype);
    if (const int rc = c.result()) return rc;
    LF_OPS_DEVICE(o);
    o->stats.launches = 0;
    if (tokens == 0) return LF_OK;
    LF_OPS_TRY(o, lfk_pack8(dtype, tokens, n, x, ld_or(ld_x, n), q, s, o->sm_count, o->stream));
    o->stats.launches = 1;
    return LF_OK;
}

int lf_unpack8(lf_ops* o, int dtype, int act, int tokens, int n, const unsigned char* q, const unsigned char* s, void* x,
               long long ld_x)
{
    if (!o) return LF_ENULL;
    checker c(tokens);
    c.type(dtype); c.act(act); c.width(n); c.matrix(x); c.matrix(q); c.bytes(s);
    c.ld(ld_x, n, dtype);
    if (const int rc = c.result()) return rc;
    LF_OPS_DEVICE(o);
    o->stats.launches = 0;
    if (tokens == 0) return LF_OK;
    LF_OPS_TRY(o, lfk_unpack8(dtype, act, tokens, n, q, s, x, ld_or(ld_x, n), o->sm_count, o->stream));
    o->stats.launches = 1;
    return LF_OK;
}

int lf_act_backward(lf_ops* o, int dtype, int act, int tokens, int n, const void* dy, long long ld_dy, const unsigned char* q,
                    const unsigned char* s, void* dz, long long ld_dz)
{
    if (!o) return LF_ENULL;
    checker c(tokens);
    c.type(dtype); c.act(act); c.width(n); c.matrix(dy); c.matrix(q); c.matrix(dz); c.bytes(s);
    c.ld(ld_dy, n, dtype); c.ld(ld_dz, n, dtype);
    if (const int rc = c.result()) return rc;
    LF_OPS_DEVICE(o);
    o->stats.launches = 0;
    if (tokens == 0) return LF_OK;
    LF_OPS_TRY(o, lfk_act_backward(dtype, act, tokens, n, dy, ld_or(ld_dy, n), q, s, dz, ld_or(ld_dz, n), o->sm_count, o->stream));
    o->stats.launches = 1;
    return LF_OK;
}

}  // extern "C"
