// C-ABI entry points of the operators of a next-word model's layers and answers: argument checks, then one launch wrapper each.
#include "checks.h"
#include "layer.h"

using namespace hadfl;
using namespace hadfl::checks;

namespace {

std::string check_drop(float p) { return p >= 0.f && p < 1.f ? "" : "the probability of dropping must be in [0, 1)"; }
std::string check_draw(const hadfl_draw* d, float p)
{
    if (layer::drop_limit(p) == 0) return "";
    if (!d) return "draw is null";
    return (uintptr_t)d->counter & 7 ? "draw: counter must be 8-byte aligned" : "";
}
std::string check_layer(const hadfl_layer* d)
{
    if (!d) return "layer is null";
    return first({check_sizes(d->n_replicas, d->n_rows, d->bf16), check_cols("n_in", d->n_in), check_cols("n_out", d->n_out),
                  d->activation < HADFL_ACT_NONE || d->activation > HADFL_ACT_SILU ? "activation is none that there is" : "", check_drop(d->drop)});
}
std::string check_dropout(const hadfl_dropout* d)
{
    if (!d) return "dropout is null";
    return first({check_sizes(d->n_replicas, d->n_rows, d->bf16), check_cols("n_features", d->n_features), check_drop(d->p)});
}
std::string check_scores(const hadfl_scores* d)
{
    if (!d) return "scores is null";
    return first({check_sizes(d->n_replicas, d->n_rows, d->bf16), check_cols("n_classes", d->n_classes, kMaxClasses),
                  d->n_tokens < 0 || d->n_tokens > 64 ? "n_tokens must be in [0, 64]" : "",
                  d->n_top < 0 || d->n_top > 32 || d->n_top > d->n_classes ? "n_top must be in [0, 32] and at most n_classes" : ""});
}
std::string check_given(const char* name, const void* p, bool wanted) { return wanted ? check_work(name, p, 4) : ""; }

layer::LayerArgs layer_args(const hadfl_layer* d, const hadfl_draw* draw, void* work)
{
    layer::LayerArgs a{};
    a.n = d->n_replicas; a.rows = d->n_rows; a.in = d->n_in; a.out = d->n_out; a.bf16 = d->bf16; a.act = d->activation;
    a.draws = layer::draws_of(draw, d->drop);
    a.work = work;
    return a;
}

}  // namespace

hadfl_status hadfl_layer_workspace(const hadfl_layer* layer, int32_t grad, size_t* bytes)
{
    return guarded([&]() -> hadfl_status {
    const std::string text = first({check_layer(layer), bytes ? "" : "bytes is null"});
    if (!text.empty()) return bad(text);
    *bytes = std::max<size_t>(256, layer::layer_work_bytes(layer->n_replicas, layer->n_rows, layer->n_in, layer->n_out, layer->bf16, layer->activation, layer->drop, grad != 0));
    return HADFL_OK;
    });
}

hadfl_status hadfl_layer_forward(const hadfl_layer* layer, const hadfl_rows* x, const hadfl_rows* w, const hadfl_rows* bias, const hadfl_rows* residual,
                                 const hadfl_draw* draw, const hadfl_rows* pre, const hadfl_rows* y, void* work, void* stream)
{
    return guarded([&]() -> hadfl_status {
    std::string text = check_layer(layer);
    if (!text.empty()) return bad(text);
    const int n = layer->n_replicas, rows = layer->n_rows, in = layer->n_in, out = layer->n_out, bf16 = layer->bf16;
    text = first({check_rows("x", x, n, rows, in, bf16, false), check_rows("w", w, n, in, out, bf16, false),
                  bias ? check_rows("bias", bias, n, 1, out, 0, false, true) : "", residual ? check_rows("residual", residual, n, rows, out, bf16, false) : "",
                  check_draw(draw, layer->drop), pre ? check_rows("pre", pre, n, rows, out, bf16, true) : "", check_rows("y", y, n, rows, out, bf16, true),
                  check_work("work", work, 256)});
    if (!text.empty()) return bad(text);
    layer::LayerArgs a = layer_args(layer, draw, work);
    a.x = head::rows_of(x); a.w = head::rows_of(w); a.bias = head::rows_of(bias); a.residual = head::rows_of(residual);
    a.pre = head::rows_of(pre); a.y = head::rows_of(y);
    return done(layer::launch_layer_forward(a, (hipStream_t)stream), "dense layer");
    });
}

hadfl_status hadfl_layer_backward(const hadfl_layer* layer, const hadfl_rows* dy, const hadfl_rows* pre, const hadfl_rows* x, const void* packed,
                                  const hadfl_rows* w, const hadfl_draw* draw, const hadfl_rows* dx, const hadfl_rows* dw, const hadfl_rows* db,
                                  void* work, void* stream)
{
    return guarded([&]() -> hadfl_status {
    std::string text = check_layer(layer);
    if (!text.empty()) return bad(text);
    const int n = layer->n_replicas, rows = layer->n_rows, in = layer->n_in, out = layer->n_out, bf16 = layer->bf16;
    text = first({check_rows("dy", dy, n, rows, out, bf16, false), layer->activation != HADFL_ACT_NONE ? check_rows("pre", pre, n, rows, out, bf16, false) : "",
                  !dw || rows == 0 ? "" : packed ? check_work("packed", packed, 256) : check_rows("x", x, n, rows, in, bf16, false),
                  dx ? check_rows("w", w, n, in, out, bf16, false) : "", check_draw(draw, layer->drop),
                  dx ? check_rows("dx", dx, n, rows, in, bf16, true) : "", dw ? check_rows("dw", dw, n, in, out, bf16, true) : "",
                  db ? check_rows("db", db, n, 1, out, 0, true, true) : "", check_work("work", work, 256)});
    if (!text.empty()) return bad(text);
    layer::LayerArgs a = layer_args(layer, draw, work);
    a.dy = head::rows_of(dy); a.pre = head::rows_of(pre); a.x = head::rows_of(packed ? nullptr : x); a.w = head::rows_of(w);
    a.dx = head::rows_of(dx); a.dw = head::rows_of(dw); a.db = head::rows_of(db);
    if (packed) a.packed = head::packed_of(packed, (long long)n * rows, in);
    return done(layer::launch_layer_backward(a, (hipStream_t)stream), "dense layer's gradient");
    });
}

hadfl_status hadfl_dropout_rows(const hadfl_dropout* dropout, const hadfl_rows* x, const hadfl_rows* residual, const hadfl_draw* draw, const hadfl_rows* y,
                                void* stream)
{
    return guarded([&]() -> hadfl_status {
    std::string text = check_dropout(dropout);
    if (!text.empty()) return bad(text);
    const int n = dropout->n_replicas, rows = dropout->n_rows, f = dropout->n_features, bf16 = dropout->bf16;
    text = first({check_rows("x", x, n, rows, f, bf16, false), residual ? check_rows("residual", residual, n, rows, f, bf16, false) : "",
                  check_draw(draw, dropout->p), check_rows("y", y, n, rows, f, bf16, true)});
    if (!text.empty()) return bad(text);
    return done(layer::launch_dropout(n, rows, f, bf16, head::rows_of(x), head::rows_of(residual), head::rows_of(y), layer::draws_of(draw, dropout->p),
                                      (hipStream_t)stream), "dropout");
    });
}

hadfl_status hadfl_scores_workspace(const hadfl_scores* scores, size_t* bytes)
{
    return guarded([&]() -> hadfl_status {
    const std::string text = first({check_scores(scores), bytes ? "" : "bytes is null"});
    if (!text.empty()) return bad(text);
    *bytes = std::max<size_t>(256, layer::score_work_bytes(scores->n_replicas, scores->n_rows, scores->n_classes, scores->n_top, scores->bf16));
    return HADFL_OK;
    });
}

hadfl_status hadfl_scores_forward(const hadfl_scores* scores, const hadfl_rows* logits, const int32_t* tokens, float* logp, float* entropy, float* stats,
                                  int32_t* top, float* top_logp, void* work, void* stream)
{
    return guarded([&]() -> hadfl_status {
    std::string text = check_scores(scores);
    if (!text.empty()) return bad(text);
    const int n = scores->n_replicas, rows = scores->n_rows;
    text = first({check_rows("logits", logits, n, rows, scores->n_classes, scores->bf16, false), check_given("tokens", tokens, rows && scores->n_tokens),
                  check_given("logp", logp, rows && scores->n_tokens), check_given("entropy", entropy, entropy), check_given("stats", stats, stats),
                  check_given("top", top, rows && scores->n_top), check_given("top_logp", top_logp, rows && scores->n_top), check_work("work", work, 256)});
    if (!text.empty()) return bad(text);
    layer::ScoreArgs a{};
    a.n = n; a.rows = rows; a.classes = scores->n_classes; a.n_tokens = scores->n_tokens; a.n_top = scores->n_top; a.bf16 = scores->bf16;
    a.logits = head::rows_of(logits); a.tokens = tokens; a.logp = logp; a.entropy = entropy; a.stats = stats; a.top = top; a.top_logp = top_logp;
    a.work = work;
    return done(layer::launch_scores_forward(a, (hipStream_t)stream), "token scores");
    });
}

hadfl_status hadfl_scores_backward(const hadfl_scores* scores, const hadfl_rows* logits, const int32_t* tokens, const float* stats, const float* dlogp,
                                   const float* dentropy, const hadfl_rows* dlogits, void* stream)
{
    return guarded([&]() -> hadfl_status {
    std::string text = check_scores(scores);
    if (!text.empty()) return bad(text);
    const int n = scores->n_replicas, rows = scores->n_rows;
    text = first({check_rows("logits", logits, n, rows, scores->n_classes, scores->bf16, false), check_given("tokens", tokens, rows && scores->n_tokens),
                  check_given("stats", stats, rows), check_given("dlogp", dlogp, rows && scores->n_tokens), check_given("dentropy", dentropy, dentropy),
                  check_rows("dlogits", dlogits, n, rows, scores->n_classes, scores->bf16, true)});
    if (!text.empty()) return bad(text);
    layer::ScoreArgs a{};
    a.n = n; a.rows = rows; a.classes = scores->n_classes; a.n_tokens = scores->n_tokens; a.bf16 = scores->bf16;
    a.logits = head::rows_of(logits); a.tokens = tokens; a.stats = const_cast<float*>(stats); a.dlogp = dlogp; a.dentropy = dentropy;
    a.dlogits = head::rows_of(dlogits);
    return done(layer::launch_scores_backward(a, (hipStream_t)stream), "token scores' gradient");
    });
}
