// C-ABI entry points of the operators of a language model's head: argument checks, then one launch wrapper each.
#include "checks.h"

using namespace hadfl;
using namespace hadfl::checks;

namespace {

std::string check_norm(const hadfl_norm* d)
{
    if (!d) return "norm is null";
    if (!(d->eps >= 0.f) || d->eps > 1e30f) return "eps must be a number, at least 0";
    return first({check_sizes(d->n_replicas, d->n_rows, d->bf16), check_cols("n_features", d->n_features)});
}
std::string check_pack(const hadfl_pack* d)
{
    if (!d) return "pack is null";
    return first({check_sizes(d->n_replicas, d->n_rows, d->bf16), check_cols("n_features", d->n_features)});
}
std::string check_dense(const hadfl_dense* d)
{
    if (!d) return "dense is null";
    return first({check_sizes(d->n_replicas, d->n_rows, d->bf16), check_cols("n_in", d->n_in), check_cols("n_out", d->n_out)});
}
std::string check_loss(const hadfl_loss* d)
{
    if (!d) return "shape is null";
    return first({check_sizes(d->n_replicas, d->n_rows, d->bf16), check_cols("n_features", d->n_features),
                  check_cols("n_classes", d->n_classes, kMaxClasses)});
}

hadfl_status loss_common(const hadfl_loss* d, bool grad, const hadfl_rows* x, const hadfl_rows* w, const hadfl_rows* bias,
                         const int32_t* labels, float* loss, float* row_loss, const hadfl_rows* dx, const hadfl_rows* dw,
                         const hadfl_rows* db, void* work, void* stream)
{
    std::string text = check_loss(d);
    if (!text.empty()) return bad(text);
    const int n = d->n_replicas, rows = d->n_rows, f = d->n_features, v = d->n_classes;
    text = first({check_rows("x", x, n, rows, f, d->bf16, false), check_rows("w", w, n, f, v, d->bf16, false),
                  bias ? check_rows("bias", bias, n, 1, v, 0, false, true) : "",
                  rows ? check_work("labels", labels, 4) : "", check_work("loss", loss, 4),
                  row_loss ? check_work("row_loss", row_loss, 4) : "",
                  dx ? check_rows("dx", dx, n, rows, f, d->bf16, true) : "", dw ? check_rows("dw", dw, n, f, v, d->bf16, true) : "",
                  db ? check_rows("db", db, n, 1, v, 0, true, true) : "", check_work("work", work, 256)});
    if (!text.empty()) return bad(text);
    head::LossArgs a{n, rows, f, v, d->bf16, head::rows_of(x), head::rows_of(w), head::rows_of(bias), head::rows_of(dx),
                     head::rows_of(dw), head::rows_of(db), labels, loss, row_loss, grad, work};
    return done(head::launch_loss(a, (hipStream_t)stream), "class loss");
}

}  // namespace

hadfl_status hadfl_norm_workspace(const hadfl_norm* norm, size_t* bytes)
{
    return guarded([&]() -> hadfl_status {
    const std::string text = first({check_norm(norm), bytes ? "" : "bytes is null"});
    if (!text.empty()) return bad(text);
    *bytes = head::norm_work_bytes(norm->n_replicas, norm->n_rows, norm->n_features);
    return HADFL_OK;
    });
}

hadfl_status hadfl_norm_forward(const hadfl_norm* norm, const hadfl_rows* x, const hadfl_rows* gamma, const hadfl_rows* beta,
                                const hadfl_rows* y, float* mean, float* rstd, void* stream)
{
    return guarded([&]() -> hadfl_status {
    std::string text = check_norm(norm);
    if (!text.empty()) return bad(text);
    const int n = norm->n_replicas, rows = norm->n_rows, f = norm->n_features;
    text = first({check_rows("x", x, n, rows, f, norm->bf16, false), check_rows("gamma", gamma, n, 1, f, 0, false, true),
                  check_rows("beta", beta, n, 1, f, 0, false, true), check_rows("y", y, n, rows, f, norm->bf16, true),
                  (mean == nullptr) != (rstd == nullptr) ? "mean and rstd must both be given or both be null" : "",
                  mean ? check_work("mean", mean, 4) : "", rstd ? check_work("rstd", rstd, 4) : ""});
    if (!text.empty()) return bad(text);
    head::NormArgs a{};
    a.n = n; a.rows = rows; a.cols = f; a.bf16 = norm->bf16; a.eps = norm->eps;
    a.x = head::rows_of(x); a.gamma = head::rows_of(gamma); a.beta = head::rows_of(beta); a.y = head::rows_of(y);
    a.mean = mean; a.rstd = rstd;
    return done(head::launch_norm_forward(a, (hipStream_t)stream), "layer norm");
    });
}

hadfl_status hadfl_norm_backward(const hadfl_norm* norm, const hadfl_rows* dy, const hadfl_rows* x, const void* packed,
                                 const hadfl_rows* gamma, const float* mean, const float* rstd, const hadfl_rows* dx,
                                 const hadfl_rows* dgamma, const hadfl_rows* dbeta, void* work, void* stream)
{
    return guarded([&]() -> hadfl_status {
    std::string text = check_norm(norm);
    if (!text.empty()) return bad(text);
    const int n = norm->n_replicas, rows = norm->n_rows, f = norm->n_features;
    text = first({check_rows("dy", dy, n, rows, f, norm->bf16, false),
                  rows == 0 ? "" : packed ? check_work("packed", packed, 256) : check_rows("x", x, n, rows, f, norm->bf16, false),
                  check_rows("gamma", gamma, n, 1, f, 0, false, true),
                  rows ? check_work("mean", mean, 4) : "", rows ? check_work("rstd", rstd, 4) : "",
                  check_rows("dx", dx, n, rows, f, norm->bf16, true), check_rows("dgamma", dgamma, n, 1, f, 0, true, true),
                  check_rows("dbeta", dbeta, n, 1, f, 0, true, true), check_work("work", work, 256)});
    if (!text.empty()) return bad(text);
    head::NormArgs a{};
    a.n = n; a.rows = rows; a.cols = f; a.bf16 = norm->bf16; a.eps = norm->eps;
    a.x = head::rows_of(packed ? nullptr : x); a.gamma = head::rows_of(gamma); a.dy = head::rows_of(dy);
    a.dx = head::rows_of(dx); a.dgamma = head::rows_of(dgamma); a.dbeta = head::rows_of(dbeta);
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
    a.work = (float*)work;
    if (packed) a.kept = head::packed_of(packed, (long long)n * rows, f);
    return done(head::launch_norm_backward(a, (hipStream_t)stream), "layer norm's gradient");
    });
}

hadfl_status hadfl_packed_bytes(const hadfl_pack* pack, size_t* bytes)
{
    return guarded([&]() -> hadfl_status {
    const std::string text = first({check_pack(pack), bytes ? "" : "bytes is null"});
    if (!text.empty()) return bad(text);
    *bytes = std::max<size_t>(256, head::packed_bytes((long long)pack->n_replicas * pack->n_rows, pack->n_features));
    return HADFL_OK;
    });
}

hadfl_status hadfl_pack_rows(const hadfl_pack* pack, const hadfl_rows* x, void* packed, void* stream)
{
    return guarded([&]() -> hadfl_status {
    std::string text = check_pack(pack);
    if (!text.empty()) return bad(text);
    text = first({check_rows("x", x, pack->n_replicas, pack->n_rows, pack->n_features, pack->bf16, false), check_work("packed", packed, 256)});
    if (!text.empty()) return bad(text);
    return done(head::launch_pack(pack->n_replicas, pack->n_rows, pack->n_features, pack->bf16, head::rows_of(x), packed,
                                  (hipStream_t)stream), "packing rows");
    });
}

hadfl_status hadfl_unpack_rows(const hadfl_pack* pack, const void* packed, const hadfl_rows* out, void* stream)
{
    return guarded([&]() -> hadfl_status {
    std::string text = check_pack(pack);
    if (!text.empty()) return bad(text);
    text = first({check_work("packed", packed, 256), check_rows("out", out, pack->n_replicas, pack->n_rows, pack->n_features, pack->bf16, true)});
    if (!text.empty()) return bad(text);
    return done(head::launch_unpack(pack->n_replicas, pack->n_rows, pack->n_features, pack->bf16, packed, head::rows_of(out),
                                    (hipStream_t)stream), "unpacking rows");
    });
}

hadfl_status hadfl_dense_workspace(const hadfl_dense* dense, size_t* bytes)
{
    return guarded([&]() -> hadfl_status {
    const std::string text = first({check_dense(dense), bytes ? "" : "bytes is null"});
    if (!text.empty()) return bad(text);
    *bytes = std::max<size_t>(256, head::dense_work_bytes(dense->n_replicas, dense->n_rows, dense->n_in, dense->n_out, dense->bf16));
    return HADFL_OK;
    });
}

hadfl_status hadfl_dense_grad_packed(const hadfl_dense* dense, const void* packed, const hadfl_rows* dy, const hadfl_rows* dw,
                                     const hadfl_rows* db, void* work, void* stream)
{
    return guarded([&]() -> hadfl_status {
    std::string text = check_dense(dense);
    if (!text.empty()) return bad(text);
    const int n = dense->n_replicas, rows = dense->n_rows;
    text = first({rows ? check_work("packed", packed, 256) : "", check_rows("dy", dy, n, rows, dense->n_out, dense->bf16, false),
                  check_rows("dw", dw, n, dense->n_in, dense->n_out, 0, true),
                  db ? check_rows("db", db, n, 1, dense->n_out, 0, true, true) : "", check_work("work", work, 256)});
    if (!text.empty()) return bad(text);
    head::DenseArgs a{n, rows, dense->n_in, dense->n_out, dense->bf16, head::packed_of(packed, (long long)n * rows, dense->n_in),
                      head::rows_of(dy), head::rows_of(dw), head::rows_of(db), work};
    return done(head::launch_dense_grad(a, (hipStream_t)stream), "dense layer's gradient");
    });
}

hadfl_status hadfl_loss_workspace(const hadfl_loss* shape, int32_t grad, size_t* bytes)
{
    return guarded([&]() -> hadfl_status {
    const std::string text = first({check_loss(shape), bytes ? "" : "bytes is null"});
    if (!text.empty()) return bad(text);
    *bytes = std::max<size_t>(256, head::loss_work_bytes(shape->n_replicas, shape->n_rows, shape->n_features, shape->n_classes,
                                                         shape->bf16, grad != 0));
    return HADFL_OK;
    });
}

hadfl_status hadfl_loss_forward(const hadfl_loss* shape, const hadfl_rows* x, const hadfl_rows* w, const hadfl_rows* bias,
                                const int32_t* labels, float* loss, float* row_loss, void* work, void* stream)
{
    return guarded([&]() -> hadfl_status {
    return loss_common(shape, false, x, w, bias, labels, loss, row_loss, nullptr, nullptr, nullptr, work, stream);
    });
}

hadfl_status hadfl_loss_grad(const hadfl_loss* shape, const hadfl_rows* x, const hadfl_rows* w, const hadfl_rows* bias,
                             const int32_t* labels, float* loss, float* row_loss, const hadfl_rows* dx, const hadfl_rows* dw,
                             const hadfl_rows* db, void* work, void* stream)
{
    return guarded([&]() -> hadfl_status {
    return loss_common(shape, true, x, w, bias, labels, loss, row_loss, dx, dw, db, work, stream);
    });
}
