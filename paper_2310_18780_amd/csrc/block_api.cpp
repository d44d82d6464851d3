// C ABI of the selective block (declared in include/lh.h): layer norm, the short
// causal convolution and the selective scan.  As in the other entry points every
// check runs on the host before anything is enqueued.
#include "lh_check.hpp"
#include "lh_internal.hpp"
#include "norm.hpp"
#include "selective.hpp"
#include "short_conv.hpp"

using namespace lh::check;

namespace {

size_t esize(lh_dtype t) { return t == LH_BF16 ? 2 : 4; }

lh_status check_at_least(const char* name, int64_t v, int64_t least)
{
    if (v < least)
        return fail(LH_ERR_INVALID_ARG, "%s = %lld must be >= %lld", name, (long long)v,
                    (long long)least);
    return LH_OK;
}

// n = a b c ... must stay small enough for byte offsets.
template <typename... I>
lh_status check_product(const char* what, I... v)
{
    int64_t n = 16;
    for (int64_t i : {int64_t(v)...})
        if (!mul_ok(n, i > 0 ? i : 1, &n))
            return fail(LH_ERR_INVALID_ARG, "sizes overflow (%s)", what);
    return LH_OK;
}

// One launch holds fewer than 2^32 threads.
lh_status check_threads(int64_t threads)
{
    if (threads >= (INT64_C(1) << 32))
        return fail(LH_ERR_INVALID_ARG, "sizes need %lld threads, a launch holds fewer than 2^32",
                    (long long)threads);
    return LH_OK;
}

// `rows` rows of `width` elements, `ld` apart.
Buf row_buf(const char* name, const void* p, int64_t rows, int64_t width, int64_t ld, size_t es)
{
    return buf(name, p, p && rows > 0 ? es * (size_t(rows - 1) * ld + width) : 0);
}

lh_status check_ld(const char* name, int64_t ld, int64_t width, int64_t rows)
{
    if (ld < width)
        return fail(LH_ERR_INVALID_ARG, "%s = %lld must be >= the row's %lld elements", name,
                    (long long)ld, (long long)width);
    return check_product(name, rows, ld);
}

lh_status check_workspace(const Buf& b, size_t have)
{
    const size_t need = b.hi - b.lo;
    if (need == 0) return LH_OK;
    if (!b.lo) return fail(LH_ERR_WORKSPACE, "workspace is NULL but %zu bytes are needed", need);
    if (have < need)
        return fail(LH_ERR_WORKSPACE, "workspace has %zu bytes, %zu are needed", have, need);
    return check_align(b, 256);
}

// Every buffer of a call: alignments, no output over another buffer, all accessible.
// An output that may be the same buffer as an input names it in `same`.
struct Arg {
    Buf b;
    size_t align;
    const void* same[2] = {nullptr, nullptr};
};

template <size_t I, size_t O>
lh_status check_buffers(const Arg (&ins)[I], const Arg (&outs)[O])
{
    lh_status s;
    for (const Arg& a : ins)
        if ((s = check_align(a.b, a.align))) return s;
    for (const Arg& a : outs)
        if ((s = check_align(a.b, a.align))) return s;
    for (const Arg& o : outs) {
        for (const Arg& i : ins) {
            const uintptr_t lo = i.b.lo;
            const bool same = lo == o.b.lo && i.b.hi == o.b.hi &&
                              (lo == reinterpret_cast<uintptr_t>(o.same[0]) ||
                               lo == reinterpret_cast<uintptr_t>(o.same[1]));
            if (!same && overlaps(o.b, i.b))
                return fail(LH_ERR_OVERLAP, "%s overlaps %s", o.b.name, i.b.name);
        }
        for (const Arg& p : outs)
            if (&p != &o && overlaps(o.b, p.b))
                return fail(LH_ERR_OVERLAP, "%s overlaps %s", o.b.name, p.b.name);
    }
    int dev = 0;
    if ((s = check_device(&dev)) != LH_OK) return s;
    // the allocations found accessible in this call: a framework's tensors share them
    Buf seen[I + O] = {};
    size_t n = 0;
    auto accessible = [&](const Buf& b) {
        for (size_t i = 0; i < n; ++i)
            if (b.lo >= seen[i].lo && b.hi <= seen[i].hi) return LH_OK;
        Buf found{"", 0, 0};
        const lh_status r = check_accessible(b, dev, &found);
        if (found.hi > found.lo) seen[n++] = found;
        return r;
    };
    for (const Arg& a : ins)
        if ((s = accessible(a.b)) != LH_OK) return s;
    for (const Arg& a : outs)
        if ((s = accessible(a.b)) != LH_OK) return s;
    return LH_OK;
}

lh_status check_norm_sizes(int64_t rows, int64_t D)
{
    lh_status s;
    if ((s = check_at_least("rows", rows, 0)) || (s = check_at_least("D", D, 1)) ||
        (s = check_product("rows, D", rows, D)))
        return s;
    return check_threads(2 * 32 * D + 1024);  // column sums
}

lh_status check_conv_sizes(int64_t B, int64_t T, int64_t D, int64_t K)
{
    lh_status s;
    if ((s = check_at_least("B", B, 1)) || (s = check_at_least("T", T, 0)) ||
        (s = check_at_least("D", D, 1)))
        return s;
    if (K < 1 || K > LH_SHORT_CONV_MAX_TAPS)
        return fail(LH_ERR_INVALID_ARG, "K = %lld must be in [1, %d]", (long long)K,
                    LH_SHORT_CONV_MAX_TAPS);
    if ((s = check_product("B, T, D, K", B, T, D, K))) return s;
    return check_threads(lh::short_conv_threads(B, T, D, K));
}

enum class Form { kPrompt, kStep, kGradient };

lh_status check_selective_sizes(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G, Form form)
{
    lh_status s;
    if ((s = check_at_least("B", B, 1)) || (s = check_at_least("T", T, 0)) ||
        (s = check_at_least("D", D, 1)) || (s = check_at_least("G", G, 1)))
        return s;
    if (N < 1 || N > LH_SELECTIVE_MAX_STATES)
        return fail(LH_ERR_INVALID_ARG, "N = %lld must be in [1, %d]", (long long)N,
                    LH_SELECTIVE_MAX_STATES);
    if (D % G != 0 || G > D)
        return fail(LH_ERR_INVALID_ARG, "D = %lld must be a multiple of G = %lld", (long long)D,
                    (long long)G);
    // (the gradient's partial sums take G N floats per tile and token)
    if ((s = check_product("B, T, D, N", B, T, D, N)) || (s = check_product("G", G, INT64_C(1) << 30)))
        return s;
    return check_threads(form == Form::kStep     ? lh::selective_step_threads(B, D, int(N))
                         : form == Form::kPrompt ? lh::selective_threads(B, T, D, int(N), int(G))
                                                 : lh::selective_grad_threads(B, T, D, int(N), int(G)));
}

// The struct's pointers and sizes.
lh_status check_selective(const lh_selective_inputs* in, Form form)
{
    lh_status s;
    if (!in) return fail(LH_ERR_INVALID_ARG, "inputs must not be NULL");
    if ((s = check_selective_sizes(in->B, in->T, in->D, in->N, in->G, form))) return s;
    if (form == Form::kStep && (in->T != 1 || in->lengths))
        return fail(LH_ERR_INVALID_ARG, "a step needs T = 1 and no lengths");
    if ((s = check_dtype(in->io_dtype))) return s;
    if (!in->A) return fail(LH_ERR_INVALID_ARG, "A must not be NULL");
    if (in->T > 0 && (!in->dt || !in->u || !in->Bm || !in->Cm))
        return fail(LH_ERR_INVALID_ARG, "dt, u, Bm and Cm must not be NULL when T > 0");
    const int64_t rows = in->B * in->T, w = in->G * in->N;
    if ((s = check_ld("ld_dt", in->ld_dt, in->D, rows)) || (s = check_ld("ld_u", in->ld_u, in->D, rows)) ||
        (in->z && (s = check_ld("ld_z", in->ld_z, in->D, rows))) ||
        (s = check_ld("ld_B", in->ld_B, w, rows)) || (s = check_ld("ld_C", in->ld_C, w, rows)))
        return s;
    // (a prompt addresses the rows of a tile in 32 bits)
    if (form != Form::kPrompt) return LH_OK;
    for (const int64_t ld : {in->ld_dt, in->ld_u, in->z ? in->ld_z : 0, in->ld_B, in->ld_C})
        if (ld >= (INT64_C(1) << 26))
            return fail(LH_ERR_INVALID_ARG, "rows must be less than 2^26 elements apart, got %lld",
                        (long long)ld);
    return LH_OK;
}

lh::Selective selective_args(const lh_selective_inputs& in)
{
    lh::Selective s;
    s.dt = in.dt, s.u = in.u, s.z = in.z, s.Bm = in.Bm, s.Cm = in.Cm;
    s.ld_dt = in.ld_dt, s.ld_u = in.ld_u, s.ld_z = in.ld_z, s.ld_b = in.ld_B, s.ld_c = in.ld_C;
    s.A = in.A, s.dt_bias = in.dt_bias, s.h0 = in.h0, s.lengths = in.lengths;
    s.B = in.B, s.T = in.T, s.D = in.D, s.N = int(in.N), s.G = int(in.G);
    s.bf16_io = in.io_dtype == LH_BF16;
    return s;
}

// The input buffers of the struct, in a fixed order.
void selective_bufs(const lh_selective_inputs& in, Arg (&a)[9])
{
    const size_t es = esize(in.io_dtype);
    const int64_t rows = in.B * in.T, w = in.G * in.N;
    a[0] = {buf("A", in.A, 4 * size_t(in.D) * in.N), 4};
    a[1] = {buf("dt_bias", in.dt_bias, in.dt_bias ? 4 * size_t(in.D) : 0), 4};
    a[2] = {buf("h0", in.h0, in.h0 ? 4 * size_t(in.D) : 0), 4};
    a[3] = {buf("lengths", in.lengths, in.lengths ? 4 * size_t(in.B) : 0), 4};
    a[4] = {row_buf("dt", in.dt, rows, in.D, in.ld_dt, es), es};
    a[5] = {row_buf("u", in.u, rows, in.D, in.ld_u, es), es};
    a[6] = {row_buf("z", in.z, rows, in.D, in.ld_z, es), es};
    a[7] = {row_buf("Bm", in.Bm, rows, w, in.ld_B, es), es};
    a[8] = {row_buf("Cm", in.Cm, rows, w, in.ld_C, es), es};
}

}  // namespace

extern "C" {

lh_status lh_layer_norm(const void* x, const void* residual, const float* w, const float* b,
                        int64_t rows, int64_t D, float eps, lh_dtype io_dtype, void* y,
                        void* total, float* mean, float* rstd, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_norm_sizes(rows, D)) || (s = check_dtype(io_dtype))) return s;
    if (!w || (rows > 0 && (!x || !y)))
        return fail(LH_ERR_INVALID_ARG, "x, w and y must not be NULL");
    if (total && !residual)
        return fail(LH_ERR_INVALID_ARG, "total is the sum of x and residual, which is NULL");
    if (!(eps >= 0.f)) return fail(LH_ERR_INVALID_ARG, "eps = %g must be >= 0", double(eps));
    const size_t es = esize(io_dtype), n = es * size_t(rows) * D;
    const Arg ins[] = {{buf("x", x, n), es},
                       {buf("residual", residual, residual ? n : 0), es},
                       {buf("w", w, 4 * size_t(D)), 4},
                       {buf("b", b, b ? 4 * size_t(D) : 0), 4}};
    const Arg outs[] = {{buf("y", y, n), es},
                        {buf("total", total, total ? n : 0), es, {x, residual}},
                        {buf("mean", mean, mean ? 4 * size_t(rows) : 0), 4},
                        {buf("rstd", rstd, rstd ? 4 * size_t(rows) : 0), 4}};
    if ((s = check_buffers(ins, outs))) return s;
    if (rows == 0) return LH_OK;
    return from_hip(lh::launch_norm(x, residual, w, b, y, total, mean, rstd, io_dtype == LH_BF16,
                                    rows, D, eps, static_cast<hipStream_t>(stream)),
                    "layer norm launch");
}

size_t lh_layer_norm_backward_workspace_bytes(int64_t rows, int64_t D)
{
    if (check_norm_sizes(rows, D) != LH_OK) return (size_t)-1;
    return lh::norm_grad_workspace_bytes(rows, D);
}

lh_status lh_layer_norm_backward(const void* dy, const void* x, const float* w, const float* mean,
                                 const float* rstd, const void* dtotal, int64_t rows, int64_t D,
                                 lh_dtype io_dtype, void* dx, float* dw, float* db,
                                 void* workspace, size_t workspace_bytes, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_norm_sizes(rows, D)) || (s = check_dtype(io_dtype))) return s;
    if (!w || !dw || (rows > 0 && (!dy || !x || !mean || !rstd || !dx)))
        return fail(LH_ERR_INVALID_ARG, "dy, x, w, mean, rstd, dx and dw must not be NULL");
    const size_t es = esize(io_dtype), n = es * size_t(rows) * D;
    const Buf ws = buf("workspace", workspace, lh::norm_grad_workspace_bytes(rows, D));
    if ((s = check_workspace(ws, workspace_bytes))) return s;
    const Arg ins[] = {{buf("dy", dy, n), es},
                       {buf("x", x, n), es},
                       {buf("w", w, 4 * size_t(D)), 4},
                       {buf("mean", mean, 4 * size_t(rows)), 4},
                       {buf("rstd", rstd, 4 * size_t(rows)), 4},
                       {buf("dtotal", dtotal, dtotal ? n : 0), es}};
    const Arg outs[] = {{buf("dx", dx, n), es, {dtotal, nullptr}},
                        {buf("dw", dw, 4 * size_t(D)), 4},
                        {buf("db", db, db ? 4 * size_t(D) : 0), 4},
                        {ws, 1}};
    if ((s = check_buffers(ins, outs))) return s;
    return from_hip(lh::launch_norm_grad(dy, x, w, mean, rstd, dtotal, dx, dw, db,
                                         io_dtype == LH_BF16, rows, D, workspace,
                                         static_cast<hipStream_t>(stream)),
                    "layer norm gradient launch");
}

lh_status lh_short_conv_prefill(const void* x, int64_t ld_x, const float* w, const float* bias,
                                const int32_t* lengths, int64_t B, int64_t T, int64_t D, int64_t K,
                                lh_dtype io_dtype, int silu, int resume, void* state, void* y,
                                void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_conv_sizes(B, T, D, K)) || (s = check_dtype(io_dtype)) ||
        (s = check_ld("ld_x", ld_x, D, B * T)))
        return s;
    if (!w || (K > 1 && !state) || (T > 0 && (!x || !y)))
        return fail(LH_ERR_INVALID_ARG, "x, w, state and y must not be NULL");
    const size_t es = esize(io_dtype);
    const Arg ins[] = {{row_buf("x", x, B * T, D, ld_x, es), es},
                       {buf("w", w, 4 * size_t(D) * K), 4},
                       {buf("bias", bias, bias ? 4 * size_t(D) : 0), 4},
                       {buf("lengths", lengths, lengths ? 4 * size_t(B) : 0), 4}};
    const Arg outs[] = {{buf("state", state, es * size_t(B) * (K - 1) * D), es},
                        {buf("y", y, es * size_t(B) * T * D), es}};
    if ((s = check_buffers(ins, outs))) return s;
    return from_hip(lh::launch_short_conv(x, ld_x, w, bias, lengths, state, resume != 0, y,
                                          io_dtype == LH_BF16, silu != 0, B, T, D, K,
                                          static_cast<hipStream_t>(stream)),
                    "short convolution launch");
}

lh_status lh_short_conv_step(const void* x_t, int64_t ld_x, const float* w, const float* bias,
                             int64_t B, int64_t D, int64_t K, lh_dtype io_dtype, int silu,
                             void* state, void* y_t, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_conv_sizes(B, 1, D, K)) || (s = check_dtype(io_dtype)) ||
        (s = check_ld("ld_x", ld_x, D, B)))
        return s;
    if (!x_t || !w || (K > 1 && !state) || !y_t)
        return fail(LH_ERR_INVALID_ARG, "x_t, w, state and y_t must not be NULL");
    const size_t es = esize(io_dtype);
    const Arg ins[] = {{row_buf("x_t", x_t, B, D, ld_x, es), es},
                       {buf("w", w, 4 * size_t(D) * K), 4},
                       {buf("bias", bias, bias ? 4 * size_t(D) : 0), 4}};
    const Arg outs[] = {{buf("state", state, es * size_t(B) * (K - 1) * D), es},
                        {buf("y_t", y_t, es * size_t(B) * D), es}};
    if ((s = check_buffers(ins, outs))) return s;
    return from_hip(lh::launch_short_conv_step(x_t, ld_x, w, bias, state, y_t,
                                               io_dtype == LH_BF16, silu != 0, B, D, K,
                                               static_cast<hipStream_t>(stream)),
                    "short convolution step launch");
}

size_t lh_short_conv_backward_workspace_bytes(int64_t B, int64_t T, int64_t D, int64_t K)
{
    if (check_conv_sizes(B, T, D, K) != LH_OK) return (size_t)-1;
    return lh::short_conv_grad_workspace_bytes(B, T, D, K);
}

lh_status lh_short_conv_backward(const void* dy, const void* x, int64_t ld_x, const float* w,
                                 const float* bias, const int32_t* lengths, int64_t B, int64_t T,
                                 int64_t D, int64_t K, lh_dtype io_dtype, int silu, void* dx,
                                 float* dw, float* dbias, void* workspace, size_t workspace_bytes,
                                 void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_conv_sizes(B, T, D, K)) || (s = check_dtype(io_dtype)) ||
        (s = check_ld("ld_x", ld_x, D, B * T)))
        return s;
    if (!w || !dw || (T > 0 && (!dy || !x || !dx)))
        return fail(LH_ERR_INVALID_ARG, "dy, x, w, dx and dw must not be NULL");
    const size_t es = esize(io_dtype), n = es * size_t(B) * T * D;
    const Buf ws = buf("workspace", workspace, lh::short_conv_grad_workspace_bytes(B, T, D, K));
    if ((s = check_workspace(ws, workspace_bytes))) return s;
    const Arg ins[] = {{buf("dy", dy, n), es},
                       {row_buf("x", x, B * T, D, ld_x, es), es},
                       {buf("w", w, 4 * size_t(D) * K), 4},
                       {buf("bias", bias, bias ? 4 * size_t(D) : 0), 4},
                       {buf("lengths", lengths, lengths ? 4 * size_t(B) : 0), 4}};
    const Arg outs[] = {{buf("dx", dx, n), es},
                        {buf("dw", dw, 4 * size_t(D) * K), 4},
                        {buf("dbias", dbias, dbias ? 4 * size_t(D) : 0), 4},
                        {ws, 1}};
    if ((s = check_buffers(ins, outs))) return s;
    return from_hip(lh::launch_short_conv_grad(dy, x, ld_x, w, bias, lengths, dx, dw, dbias,
                                               io_dtype == LH_BF16, silu != 0, B, T, D, K,
                                               workspace, static_cast<hipStream_t>(stream)),
                    "short convolution gradient launch");
}

size_t lh_selective_workspace_bytes(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G)
{
    if (check_selective_sizes(B, T, D, N, G, Form::kPrompt) != LH_OK) return (size_t)-1;
    return lh::selective_plan(B, T, D, int(N), int(G)).ws_bytes;
}

lh_status lh_selective_prefill(const lh_selective_inputs* in, int resume, float* state, void* y,
                               void* workspace, size_t workspace_bytes, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_selective(in, Form::kPrompt))) return s;
    if (!state || (in->T > 0 && !y))
        return fail(LH_ERR_INVALID_ARG, "state and y must not be NULL");
    const size_t es = esize(in->io_dtype);
    const Buf ws = buf("workspace", workspace,
                       lh::selective_plan(in->B, in->T, in->D, int(in->N), int(in->G)).ws_bytes);
    if ((s = check_workspace(ws, workspace_bytes))) return s;
    Arg ins[9];
    selective_bufs(*in, ins);
    const Arg outs[] = {{buf("state", state, 4 * size_t(in->B) * in->D * in->N), 4},
                        {buf("y", y, es * size_t(in->B) * in->T * in->D), es},
                        {ws, 1}};
    if ((s = check_buffers(ins, outs))) return s;
    return from_hip(lh::launch_selective(selective_args(*in), state, resume != 0, y, workspace,
                                         static_cast<hipStream_t>(stream)),
                    "selective scan launch");
}

lh_status lh_selective_step(const lh_selective_inputs* in, float* state, void* y_t, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_selective(in, Form::kStep))) return s;
    if (!state || !y_t) return fail(LH_ERR_INVALID_ARG, "state and y_t must not be NULL");
    const size_t es = esize(in->io_dtype);
    Arg ins[9];
    selective_bufs(*in, ins);
    const Arg outs[] = {{buf("state", state, 4 * size_t(in->B) * in->D * in->N), 4},
                        {buf("y_t", y_t, es * size_t(in->B) * in->D), es}};
    if ((s = check_buffers(ins, outs))) return s;
    return from_hip(lh::launch_selective_step(selective_args(*in), state, y_t,
                                              static_cast<hipStream_t>(stream)),
                    "selective step launch");
}

size_t lh_selective_backward_workspace_bytes(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G)
{
    if (check_selective_sizes(B, T, D, N, G, Form::kGradient) != LH_OK) return (size_t)-1;
    return lh::selective_grad_workspace_bytes(B, T, D, int(N), int(G));
}

lh_status lh_selective_backward(const lh_selective_inputs* in, const lh_selective_grads* g,
                                void* workspace, size_t workspace_bytes, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_selective(in, Form::kGradient))) return s;
    if (!g || !g->dA) return fail(LH_ERR_INVALID_ARG, "gradients and dA must not be NULL");
    if (in->T > 0 && (!g->dy || !g->ddt || !g->du || !g->dBm || !g->dCm))
        return fail(LH_ERR_INVALID_ARG, "dy, ddt, du, dBm and dCm must not be NULL when T > 0");
    if (in->T > 0 && !in->z != !g->dz)
        return fail(LH_ERR_INVALID_ARG, "dz and z must both be given or both be NULL");
    if ((g->dh0 && !in->h0) || (g->ddt_bias && !in->dt_bias))
        return fail(LH_ERR_INVALID_ARG, "dh0 and ddt_bias need h0 and dt_bias");
    const size_t es = esize(in->io_dtype);
    const size_t n = es * size_t(in->B) * in->T * in->D, r = es * size_t(in->B) * in->T * in->G * in->N;
    const Buf ws = buf("workspace", workspace,
                       lh::selective_grad_workspace_bytes(in->B, in->T, in->D, int(in->N), int(in->G)));
    if ((s = check_workspace(ws, workspace_bytes))) return s;
    Arg a[9], ins[10];
    selective_bufs(*in, a);
    for (int i = 0; i < 9; ++i) ins[i] = a[i];
    ins[9] = {buf("dy", g->dy, n), es};
    const Arg outs[] = {{buf("ddt", g->ddt, n), es},
                        {buf("du", g->du, n), es},
                        {buf("dz", g->dz, g->dz ? n : 0), es},
                        {buf("dBm", g->dBm, r), es},
                        {buf("dCm", g->dCm, r), es},
                        {buf("dA", g->dA, 4 * size_t(in->D) * in->N), 4},
                        {buf("dh0", g->dh0, g->dh0 ? 4 * size_t(in->D) : 0), 4},
                        {buf("ddt_bias", g->ddt_bias, g->ddt_bias ? 4 * size_t(in->D) : 0), 4},
                        {ws, 1}};
    if ((s = check_buffers(ins, outs))) return s;
    lh::SelectiveGrads d;
    d.dy = g->dy, d.ddt = g->ddt, d.du = g->du, d.dz = g->dz, d.dBm = g->dBm, d.dCm = g->dCm;
    d.dA = g->dA, d.dh0 = g->dh0, d.ddt_bias = g->ddt_bias;
    return from_hip(lh::launch_selective_grad(selective_args(*in), d, workspace,
                                              static_cast<hipStream_t>(stream)),
                    "selective gradient launch");
}

}  // extern "C"
