// C ABI of the gated recurrence, the embedding, the distillation of logits and the
// verification of drafts (declared in include/lh.h).  As in the other entry points every
// check runs on the host before anything is enqueued.
#include "call_check.hpp"
#include "distill_logits.hpp"
#include "embed.hpp"
#include "gated.hpp"
#include "lh_internal.hpp"
#include "verify.hpp"

using namespace lh::check;

namespace {

enum class Form { kPrompt, kStep, kGradient };

lh_status check_gated_sizes(int64_t B, int64_t T, int64_t D, Form form)
{
    lh_status s;
    if ((s = check_at_least("B", B, 1)) || (s = check_at_least("T", T, 0)) ||
        (s = check_at_least("D", D, 1)) || (s = check_product("B, T, D", B, T, D)))
        return s;
    // (the tiles of all chunks must be countable, too)
    if ((s = check_product("B, D", B, D, INT64_C(1) << 20))) return s;
    return check_threads(form == Form::kStep     ? lh::gated_step_threads(B, D)
                         : form == Form::kPrompt ? lh::gated_threads(B, T, D)
                                                 : lh::gated_grad_threads(B, T, D));
}

// The struct's pointers and sizes.
lh_status check_gated(const lh_gated_inputs* in, Form form)
{
    lh_status s;
    if (!in) return fail(LH_ERR_INVALID_ARG, "inputs must not be NULL");
    if ((s = check_gated_sizes(in->B, in->T, in->D, form))) return s;
    if (form == Form::kStep && (in->T != 1 || in->lengths))
        return fail(LH_ERR_INVALID_ARG, "a step needs T = 1 and no lengths");
    if ((s = check_dtype(in->io_dtype))) return s;
    if (!in->rate) return fail(LH_ERR_INVALID_ARG, "rate must not be NULL");
    if (in->T > 0 && (!in->r || !in->i || !in->u))
        return fail(LH_ERR_INVALID_ARG, "r, i and u must not be NULL when T > 0");
    const int64_t rows = in->B * in->T;
    if ((s = check_ld("ld_r", in->ld_r, in->D, rows)) || (s = check_ld("ld_i", in->ld_i, in->D, rows)) ||
        (s = check_ld("ld_u", in->ld_u, in->D, rows)) || (in->z && (s = check_ld("ld_z", in->ld_z, in->D, rows))))
        return s;
    // (a run's rows are addressed in 32 bits)
    if (form == Form::kStep) return LH_OK;
    for (const int64_t ld : {in->ld_r, in->ld_i, in->ld_u, in->z ? in->ld_z : 0})
        if (ld >= (INT64_C(1) << 26))
            return fail(LH_ERR_INVALID_ARG, "rows must be less than 2^26 elements apart, got %lld", (long long)ld);
    return LH_OK;
}

lh::Gated gated_args(const lh_gated_inputs& in)
{
    lh::Gated g;
    g.r = in.r, g.i = in.i, g.u = in.u, g.z = in.z;
    g.ld_r = in.ld_r, g.ld_i = in.ld_i, g.ld_u = in.ld_u, g.ld_z = in.ld_z;
    g.rate = in.rate, g.r_bias = in.r_bias, g.i_bias = in.i_bias, g.lengths = in.lengths;
    g.B = in.B, g.T = in.T, g.D = in.D;
    g.bf16_io = in.io_dtype == LH_BF16;
    return g;
}

// The input buffers of the struct, in a fixed order.
constexpr int kGatedBufs = 8;
void gated_bufs(const lh_gated_inputs& in, Arg* a)
{
    const size_t es = esize(in.io_dtype), w = 4 * size_t(in.D);
    const int64_t rows = in.B * in.T;
    a[0] = {buf("rate", in.rate, w), 4};
    a[1] = {buf("r_bias", in.r_bias, in.r_bias ? w : 0), 4};
    a[2] = {buf("i_bias", in.i_bias, in.i_bias ? w : 0), 4};
    a[3] = {buf("lengths", in.lengths, in.lengths ? 4 * size_t(in.B) : 0), 4};
    a[4] = {row_buf("r", in.r, rows, in.D, in.ld_r, es), es};
    a[5] = {row_buf("i", in.i, rows, in.D, in.ld_i, es), es};
    a[6] = {row_buf("u", in.u, rows, in.D, in.ld_u, es), es};
    a[7] = {row_buf("z", in.z, rows, in.D, in.ld_z, es), es};
}

size_t marks_bytes(const lh_gated_inputs& in)
{
    return 4 * size_t(in.B) * ((in.T + LH_GATED_MARK - 1) / LH_GATED_MARK) * in.D;
}

lh_status check_below_2_31(const char* name, int64_t v)
{
    if (v >= (INT64_C(1) << 31))
        return fail(LH_ERR_INVALID_ARG, "%s = %lld must be less than 2^31", name, (long long)v);
    return LH_OK;
}

lh_status check_embed_sizes(int64_t n, int64_t V, int64_t D)
{
    lh_status s;
    if ((s = check_at_least("n", n, 0)) || (s = check_at_least("V", V, 1)) || (s = check_at_least("D", D, 1)) ||
        (s = check_below_2_31("n", n)) || (s = check_below_2_31("V", V)) ||
        (s = check_product("n, D", n, D, 8)) || (s = check_product("V, D", V, D)))
        return s;
    return LH_OK;
}

lh_status check_embed_grad_sizes(int64_t n, int64_t V, int64_t D)
{
    const lh_status s = check_embed_sizes(n, V, D);
    return s ? s : check_threads(lh::embed_grad_threads(n, V, D));
}

lh_status check_distill_sizes(int64_t rows, int64_t V, int64_t K)
{
    lh_status s;
    if ((s = check_at_least("rows", rows, 0)) || (s = check_at_least("V", V, 1)) || (s = check_below_2_31("V", V)))
        return s;
    if (K < 1 || K > LH_DISTILL_MAX_TOP)
        return fail(LH_ERR_INVALID_ARG, "K = %lld must be in [1, %d]", (long long)K, LH_DISTILL_MAX_TOP);
    if ((s = check_product("rows, V, K", rows, V, K))) return s;
    return rows < (INT64_C(1) << 22) ? LH_OK : check_threads(rows * 1024);  // (a workgroup to a row)
}

// What both distillation calls take; ins gets 4 buffers.
lh_status check_distill(const void* logits, int64_t ld, const float* values, const int32_t* ids,
                        const float* scale, int64_t rows, int64_t V, int64_t K, lh_dtype io_dtype, float tau,
                        const void* dlogits, int64_t ld_d, Arg* ins)
{
    lh_status s;
    if ((s = check_distill_sizes(rows, V, K)) || (s = check_dtype(io_dtype)) ||
        (s = check_ld("ld_logits", ld, V, rows)) || (dlogits && (s = check_ld("ld_dlogits", ld_d, V, rows))))
        return s;
    // (its square and its reciprocal are normal numbers)
    if (!(tau >= 0x1p-60f && tau <= 0x1p60f))
        return fail(LH_ERR_INVALID_ARG, "tau = %g must be in [2^-60, 2^60]", double(tau));
    if (rows > 0 && (!logits || !values || !ids))
        return fail(LH_ERR_INVALID_ARG, "logits, values and ids must not be NULL");
    const size_t es = esize(io_dtype);
    ins[0] = {row_buf("logits", logits, rows, V, ld, es), es};
    ins[1] = {buf("values", values, 4 * size_t(rows) * K), 4};
    ins[2] = {buf("ids", ids, 4 * size_t(rows) * K), 4};
    ins[3] = {buf("scale", scale, scale ? 4 * size_t(rows) : 0), 4};
    return LH_OK;
}

lh::DistillLogits distill_args(const void* logits, int64_t ld, const float* values, const int32_t* ids,
                               const float* scale, int64_t rows, int64_t V, int64_t K, lh_dtype io_dtype, float tau,
                               void* dlogits, int64_t ld_d)
{
    lh::DistillLogits d;
    d.logits = logits, d.ld = ld, d.values = values, d.ids = ids, d.scale = scale;
    d.rows = rows, d.V = V, d.K = int(K), d.tau = tau, d.bf16_io = io_dtype == LH_BF16;
    d.dlogits = dlogits, d.ld_d = ld_d;
    return d;
}

lh_status check_verify_sizes(int64_t B, int64_t K, int64_t V)
{
    lh_status s;
    if ((s = check_at_least("B", B, 1)) || (s = check_at_least("V", V, 1)) || (s = check_below_2_31("V", V)))
        return s;
    if (K < 1 || K > LH_VERIFY_MAX_DRAFT)
        return fail(LH_ERR_INVALID_ARG, "K = %lld must be in [1, %d]", (long long)K, LH_VERIFY_MAX_DRAFT);
    if ((s = check_product("B, K, V", B, K + 1, V))) return s;
    return check_threads(lh::verify_threads(B, V));
}

}  // namespace

extern "C" {

size_t lh_gated_workspace_bytes(int64_t B, int64_t T, int64_t D)
{
    if (check_gated_sizes(B, T, D, Form::kPrompt) != LH_OK) return (size_t)-1;
    return lh::gated_plan(B, T, D).ws_bytes;
}

lh_status lh_gated_prefill(const lh_gated_inputs* in, int resume, float* state, void* y, float* marks,
                           void* workspace, size_t workspace_bytes, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_gated(in, Form::kPrompt))) return s;
    if (!state || (in->T > 0 && !y))
        return fail(LH_ERR_INVALID_ARG, "state and y must not be NULL");
    const size_t es = esize(in->io_dtype);
    const Buf ws = buf("workspace", workspace, lh::gated_plan(in->B, in->T, in->D).ws_bytes);
    if ((s = check_workspace(ws, workspace_bytes))) return s;
    Arg ins[kGatedBufs];
    gated_bufs(*in, ins);
    const Arg outs[] = {{buf("state", state, 4 * size_t(in->B) * in->D), 4},
                        {buf("y", y, es * size_t(in->B) * in->T * in->D), es},
                        {buf("marks", marks, marks ? marks_bytes(*in) : 0), 4},
                        {ws, 1}};
    if ((s = check_buffers(ins, outs))) return s;
    return from_hip(lh::launch_gated(gated_args(*in), state, resume != 0, y, marks, workspace,
                                     static_cast<hipStream_t>(stream)),
                    "gated recurrence launch");
}

lh_status lh_gated_step(const lh_gated_inputs* in, float* state, void* y_t, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_gated(in, Form::kStep))) return s;
    if (!state || !y_t) return fail(LH_ERR_INVALID_ARG, "state and y_t must not be NULL");
    Arg ins[kGatedBufs];
    gated_bufs(*in, ins);
    const size_t es = esize(in->io_dtype);
    const Arg outs[] = {{buf("state", state, 4 * size_t(in->B) * in->D), 4},
                        {buf("y_t", y_t, es * size_t(in->B) * in->D), es}};
    if ((s = check_buffers(ins, outs))) return s;
    return from_hip(lh::launch_gated_step(gated_args(*in), state, y_t, static_cast<hipStream_t>(stream)),
                    "gated step launch");
}

size_t lh_gated_backward_workspace_bytes(int64_t B, int64_t T, int64_t D)
{
    if (check_gated_sizes(B, T, D, Form::kGradient) != LH_OK) return (size_t)-1;
    return lh::gated_grad_plan(B, T, D).ws_bytes;
}

lh_status lh_gated_backward(const lh_gated_inputs* in, const lh_gated_grads* g, void* workspace,
                            size_t workspace_bytes, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_gated(in, Form::kGradient))) return s;
    if (!g || !g->drate) return fail(LH_ERR_INVALID_ARG, "gradients and drate must not be NULL");
    if (in->T > 0 && (!g->dy || !g->marks || !g->dr || !g->di || !g->du))
        return fail(LH_ERR_INVALID_ARG, "dy, marks, dr, di and du must not be NULL when T > 0");
    if (in->T > 0 && !in->z != !g->dz)
        return fail(LH_ERR_INVALID_ARG, "dz and z must both be given or both be NULL");
    if ((g->dr_bias && !in->r_bias) || (g->di_bias && !in->i_bias))
        return fail(LH_ERR_INVALID_ARG, "dr_bias and di_bias need r_bias and i_bias");
    const size_t es = esize(in->io_dtype), n = es * size_t(in->B) * in->T * in->D;
    const size_t w = 4 * size_t(in->D), st = w * in->B;
    const Buf ws = buf("workspace", workspace, lh::gated_grad_plan(in->B, in->T, in->D).ws_bytes);
    if ((s = check_workspace(ws, workspace_bytes))) return s;
    Arg ins[kGatedBufs + 3];
    gated_bufs(*in, ins);
    ins[kGatedBufs] = {buf("dy", g->dy, n), es};
    ins[kGatedBufs + 1] = {buf("marks", g->marks, marks_bytes(*in)), 4};
    ins[kGatedBufs + 2] = {buf("dlast", g->dlast, g->dlast ? st : 0), 4};
    const Arg outs[] = {{buf("dr", g->dr, n), es},
                        {buf("di", g->di, n), es},
                        {buf("du", g->du, n), es},
                        {buf("dz", g->dz, g->dz ? n : 0), es},
                        {buf("drate", g->drate, w), 4},
                        {buf("dr_bias", g->dr_bias, g->dr_bias ? w : 0), 4},
                        {buf("di_bias", g->di_bias, g->di_bias ? w : 0), 4},
                        {buf("dfirst", g->dfirst, g->dfirst ? st : 0), 4},
                        {ws, 1}};
    if ((s = check_buffers(ins, outs))) return s;
    lh::GatedGrads d;
    d.dy = g->dy, d.marks = g->marks, d.dlast = g->dlast, d.dr = g->dr, d.di = g->di, d.du = g->du, d.dz = g->dz;
    d.drate = g->drate, d.dr_bias = g->dr_bias, d.di_bias = g->di_bias, d.dfirst = g->dfirst;
    return from_hip(lh::launch_gated_grad(gated_args(*in), d, workspace, static_cast<hipStream_t>(stream)),
                    "gated gradient launch");
}

lh_status lh_embed(const void* W, const int32_t* ids, int64_t n, int64_t V, int64_t D, lh_dtype table_dtype,
                   lh_dtype io_dtype, float scale, void* y, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_embed_sizes(n, V, D)) || (s = check_dtype(table_dtype)) || (s = check_dtype(io_dtype))) return s;
    if (!W || (n > 0 && (!ids || !y))) return fail(LH_ERR_INVALID_ARG, "W, ids and y must not be NULL");
    const size_t et = esize(table_dtype), es = esize(io_dtype);
    const Arg ins[] = {{buf("W", W, et * size_t(V) * D), et}, {buf("ids", ids, 4 * size_t(n)), 4}};
    const Arg outs[] = {{buf("y", y, es * size_t(n) * D), es}};
    if ((s = check_buffers(ins, outs))) return s;
    if (n == 0) return LH_OK;
    return from_hip(lh::launch_embed(W, ids, n, V, D, table_dtype == LH_BF16, io_dtype == LH_BF16, scale, y,
                                     static_cast<hipStream_t>(stream)),
                    "embedding launch");
}

size_t lh_embed_backward_workspace_bytes(int64_t n, int64_t V, int64_t D)
{
    if (check_embed_grad_sizes(n, V, D) != LH_OK) return (size_t)-1;
    return lh::embed_grad_plan(n, V, D).ws_bytes;
}

lh_status lh_embed_backward(const void* dy, const int32_t* ids, int64_t n, int64_t V, int64_t D, lh_dtype io_dtype,
                            float scale, int accumulate, float* dW, void* workspace, size_t workspace_bytes,
                            void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_embed_grad_sizes(n, V, D)) || (s = check_dtype(io_dtype))) return s;
    if (!dW || (n > 0 && (!dy || !ids))) return fail(LH_ERR_INVALID_ARG, "dy, ids and dW must not be NULL");
    const size_t es = esize(io_dtype);
    const Buf ws = buf("workspace", workspace, lh::embed_grad_plan(n, V, D).ws_bytes);
    if ((s = check_workspace(ws, workspace_bytes))) return s;
    const Arg ins[] = {{buf("dy", dy, es * size_t(n) * D), es}, {buf("ids", ids, 4 * size_t(n)), 4}};
    const Arg outs[] = {{buf("dW", dW, 4 * size_t(V) * D), 4}, {ws, 1}};
    if ((s = check_buffers(ins, outs))) return s;
    return from_hip(lh::launch_embed_grad(dy, ids, n, V, D, io_dtype == LH_BF16, scale, accumulate != 0, dW, workspace,
                                          static_cast<hipStream_t>(stream)),
                    "embedding gradient launch");
}

size_t lh_distill_logits_workspace_bytes(int64_t rows, int64_t V, int64_t K)
{
    if (check_distill_sizes(rows, V, K) != LH_OK) return (size_t)-1;
    return 0;  // (the boundary has it all the same, for rows that a later form may split)
}

lh_status lh_distill_logits(const void* logits, int64_t ld_logits, const float* values, const int32_t* ids,
                            const float* scale, int64_t rows, int64_t V, int64_t K, lh_dtype io_dtype, float tau,
                            float* loss, float* lse, void* dlogits, int64_t ld_dlogits, void* workspace,
                            size_t workspace_bytes, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    Arg ins[4];
    if ((s = check_distill(logits, ld_logits, values, ids, scale, rows, V, K, io_dtype, tau, dlogits, ld_dlogits, ins)))
        return s;
    if (rows > 0 && !loss) return fail(LH_ERR_INVALID_ARG, "loss must not be NULL");
    (void)workspace, (void)workspace_bytes;  // (none is needed)
    const size_t es = esize(io_dtype);
    const Arg outs[] = {{buf("loss", loss, 4 * size_t(rows)), 4},
                        {buf("lse", lse, lse ? 4 * size_t(rows) : 0), 4},
                        {row_buf("dlogits", dlogits, rows, V, ld_dlogits, es), es,
                         {ld_dlogits == ld_logits ? logits : nullptr, nullptr}}};
    if ((s = check_buffers(ins, outs))) return s;
    return from_hip(lh::launch_distill_logits(distill_args(logits, ld_logits, values, ids, scale, rows, V, K, io_dtype,
                                                           tau, dlogits, ld_dlogits),
                                              loss, lse, static_cast<hipStream_t>(stream)),
                    "distillation launch");
}

lh_status lh_distill_logits_backward(const float* dloss, const void* logits, int64_t ld_logits, const float* values,
                                     const int32_t* ids, const float* scale, const float* lse, int64_t rows, int64_t V,
                                     int64_t K, lh_dtype io_dtype, float tau, void* dlogits, int64_t ld_dlogits,
                                     void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    Arg ins[6];
    if ((s = check_distill(logits, ld_logits, values, ids, scale, rows, V, K, io_dtype, tau, dlogits, ld_dlogits, ins)))
        return s;
    if (rows > 0 && (!dloss || !lse || !dlogits))
        return fail(LH_ERR_INVALID_ARG, "dloss, lse and dlogits must not be NULL");
    ins[4] = {buf("dloss", dloss, 4 * size_t(rows)), 4};
    ins[5] = {buf("lse", lse, 4 * size_t(rows)), 4};
    const size_t es = esize(io_dtype);
    const Arg outs[] = {{row_buf("dlogits", dlogits, rows, V, ld_dlogits, es), es,
                         {ld_dlogits == ld_logits ? logits : nullptr, nullptr}}};
    if ((s = check_buffers(ins, outs))) return s;
    return from_hip(lh::launch_distill_logits_grad(distill_args(logits, ld_logits, values, ids, scale, rows, V, K,
                                                                io_dtype, tau, dlogits, ld_dlogits),
                                                   dloss, lse, static_cast<hipStream_t>(stream)),
                    "distillation gradient launch");
}

size_t lh_verify_draft_workspace_bytes(int64_t B, int64_t K, int64_t V)
{
    if (check_verify_sizes(B, K, V) != LH_OK) return (size_t)-1;
    return lh::verify_workspace_bytes(B, K, V);
}

lh_status lh_verify_draft(const int32_t* drafted, const int32_t* lengths, const void* draft_p, int64_t ld_draft,
                          const void* target_p, int64_t ld_target, const float* u, const float* u_last, int64_t B,
                          int64_t K, int64_t V, lh_dtype io_dtype, int32_t* accepted, int32_t* tokens, void* workspace,
                          size_t workspace_bytes, void* stream)
{
    g_last_error[0] = '\0';
    lh_status s;
    if ((s = check_verify_sizes(B, K, V)) || (s = check_dtype(io_dtype)) ||
        (draft_p && (s = check_ld("ld_draft", ld_draft, V, B * K))) ||
        (s = check_ld("ld_target", ld_target, V, B * (K + 1))))
        return s;
    if (!drafted || !target_p || !u || !u_last || !accepted || !tokens)
        return fail(LH_ERR_INVALID_ARG, "drafted, target_p, u, u_last, accepted and tokens must not be NULL");
    const size_t es = esize(io_dtype), rows = size_t(B) * K;
    const Buf ws = buf("workspace", workspace, lh::verify_workspace_bytes(B, K, V));
    if ((s = check_workspace(ws, workspace_bytes))) return s;
    const Arg ins[] = {{buf("drafted", drafted, 4 * rows), 4},
                       {buf("lengths", lengths, lengths ? 4 * size_t(B) : 0), 4},
                       {row_buf("draft_p", draft_p, B * K, V, ld_draft, es), es},
                       {row_buf("target_p", target_p, B * (K + 1), V, ld_target, es), es},
                       {buf("u", u, 4 * rows), 4},
                       {buf("u_last", u_last, 4 * size_t(B)), 4}};
    const Arg outs[] = {{buf("accepted", accepted, 4 * size_t(B)), 4},
                        {buf("tokens", tokens, 4 * (rows + B)), 4},
                        {ws, 1}};
    if ((s = check_buffers(ins, outs))) return s;
    lh::Verify v;
    v.drafted = drafted, v.lengths = lengths, v.draft_p = draft_p, v.target_p = target_p;
    v.ld_draft = ld_draft, v.ld_target = ld_target, v.u = u, v.u_last = u_last;
    v.B = B, v.K = K, v.V = V, v.bf16_io = io_dtype == LH_BF16, v.accepted = accepted, v.tokens = tokens;
    return from_hip(lh::launch_verify(v, workspace, static_cast<hipStream_t>(stream)), "verification launch");
}

}  // extern "C"
