// C ABI of the token operators: checks of arguments in front of the kernels.  Nothing here allocates,
// waits or keeps anything, and nothing throws.
#include "tokens.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>

namespace {

constexpr int64_t kMost32 = 0x7fffffff;
constexpr size_t kAlignment = 256;

int refuse(int code, const char *format, ...)
{
    char text[256];
    va_list ap;
    va_start(ap, format);
    vsnprintf(text, sizeof text, format, ap);
    va_end(ap);
    return cbk::set_error(code, text);
}

int launched(hipError_t e, const char *what)
{
    return e == hipSuccess ? CBINFER_OK : refuse(CBINFER_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

bool known(int dtype) { return dtype == CBINFER_F32 || dtype == CBINFER_BF16; }
bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
// A pointer that has to be there, at its element's alignment.
bool placed(const void *p, size_t to) { return p && aligned(p, to); }
size_t element(int dtype) { return dtype == CBINFER_F32 ? 4 : 2; }

int check_workspace(const char *what, const void *workspace, size_t bytes, size_t needed)
{
    if (needed == 0) return CBINFER_OK;
    if (!placed(workspace, kAlignment)) return refuse(CBINFER_EINVAL, "%s: workspace must be given, 256-byte aligned", what);
    if (bytes < needed) return refuse(CBINFER_ENOMEM, "%s: workspace of %zu bytes, %zu are needed", what, bytes, needed);
    return CBINFER_OK;
}

int check(const cbinfer_log_probs_args *a)
{
    const char *w = "log_probs";
    if (!a) return refuse(CBINFER_EINVAL, "%s: arguments are NULL", w);
    if (!known(a->dtype)) return refuse(CBINFER_EINVAL, "%s: dtype must be CBINFER_F32 or CBINFER_BF16", w);
    if (a->outer < 0 || a->inner < 0 || a->outer > kMost32 || a->inner > kMost32 || a->outer * a->inner > kMost32)
        return refuse(CBINFER_EINVAL, "%s: outer and inner must be >= 0 and their product below 2^31", w);
    if (a->classes < 1 || a->classes > kMost32) return refuse(CBINFER_EINVAL, "%s: classes must be 1 .. 2^31-1", w);
    if (a->top < 0 || a->top > 64 || a->top > a->classes)
        return refuse(CBINFER_EINVAL, "%s: top must be 0 .. 64 and at most the number of classes", w);
    return CBINFER_OK;
}

int check(const cbinfer_linear_attention_args *a)
{
    const char *w = "linear_attention";
    if (!a) return refuse(CBINFER_EINVAL, "%s: arguments are NULL", w);
    if (!known(a->dtype)) return refuse(CBINFER_EINVAL, "%s: dtype must be CBINFER_F32 or CBINFER_BF16", w);
    if (a->streams < 0 || a->tokens < 0 || a->heads < 0 || a->kv_heads < 0)
        return refuse(CBINFER_EINVAL, "%s: sizes must be >= 0", w);
    if (a->heads > 0 && (a->kv_heads < 1 || a->heads % a->kv_heads))
        return refuse(CBINFER_EINVAL, "%s: heads (%d) must be a multiple of kv_heads (%d)", w, a->heads, a->kv_heads);
    if (a->key_size < 1 || a->key_size > 256 || a->value_size < 1 || a->value_size > 256)
        return refuse(CBINFER_EUNSUPPORTED, "%s: key and value sizes must be 1 .. 256 (got %d and %d)", w, a->key_size,
                      a->value_size);
    if ((int64_t)a->streams * a->heads > (1 << 18))
        return refuse(CBINFER_EUNSUPPORTED, "%s: streams times heads must be at most 2^18", w);
    if (a->tokens > (1 << 28)) return refuse(CBINFER_EUNSUPPORTED, "%s: tokens must be at most 2^28", w);
    if (!std::isfinite(a->scale)) return refuse(CBINFER_EINVAL, "%s: scale must be finite", w);
    return CBINFER_OK;
}

int check(const cbinfer_quantised_product_args *a)
{
    const char *w = "quantised_product";
    if (!a) return refuse(CBINFER_EINVAL, "%s: arguments are NULL", w);
    if (!known(a->dtype)) return refuse(CBINFER_EINVAL, "%s: dtype must be CBINFER_F32 or CBINFER_BF16", w);
    if (cbinfer_packed_weights_bytes(a->rows, a->cols, a->group) == 0) return CBINFER_EINVAL;
    if (a->tokens < 0 || a->tokens > (1 << 19)) return refuse(CBINFER_EUNSUPPORTED, "%s: tokens must be 0 .. 2^19", w);
    return CBINFER_OK;
}

} // namespace

extern "C" {

size_t cbinfer_log_probs_workspace_bytes(const cbinfer_log_probs_args *a)
{
    if (check(a) != CBINFER_OK) return 0;
    return cbk::log_probs_workspace(*a);
}

int cbinfer_log_probs(const cbinfer_log_probs_args *a, void *stream)
{
    const char *w = "log_probs";
    if (int rc = check(a)) return rc;
    if (a->labels && a->label_bytes != 4 && a->label_bytes != 8)
        return refuse(CBINFER_EINVAL, "%s: label_bytes must be 4 or 8", w);
    if (a->label && !a->labels) return refuse(CBINFER_EINVAL, "%s: label log probabilities without labels", w);
    if (a->outer * a->inner == 0) return CBINFER_OK;
    if (!placed(a->scores, element(a->dtype))) return refuse(CBINFER_EINVAL, "%s: scores must be given, aligned to their element", w);
    if (a->labels && !aligned(a->labels, a->label_bytes)) return refuse(CBINFER_EINVAL, "%s: labels must be aligned to their element", w);
    if (!aligned(a->label, 4) || !aligned(a->entropy, 4)) return refuse(CBINFER_EINVAL, "%s: outputs must be aligned to their element", w);
    if (a->top && (!placed(a->top_values, 4) || !placed(a->top_index, 4)))
        return refuse(CBINFER_EINVAL, "%s: top_values and top_index must be given, aligned to their element", w);
    if (!a->label && !a->entropy && !a->top) return refuse(CBINFER_EINVAL, "%s: no output asked for", w);
    if (int rc = check_workspace(w, a->workspace, a->workspace_bytes, cbk::log_probs_workspace(*a))) return rc;
    return launched(cbk::log_probs(static_cast<hipStream_t>(stream), *a), w);
}

size_t cbinfer_linear_attention_workspace_bytes(const cbinfer_linear_attention_args *a)
{
    if (check(a) != CBINFER_OK) return 0;
    return cbk::linear_attention_workspace(*a);
}

int cbinfer_linear_attention(const cbinfer_linear_attention_args *a, void *stream)
{
    const char *w = "linear_attention";
    if (int rc = check(a)) return rc;
    if (a->streams == 0 || a->heads == 0 || a->tokens == 0) return CBINFER_OK;
    const size_t e = element(a->dtype);
    if (!placed(a->q, e) || !placed(a->k, e) || !placed(a->v, e) || !placed(a->o, e))
        return refuse(CBINFER_EINVAL, "%s: q, k, v and o must be given, aligned to their element", w);
    if (!placed(a->state, 4) || !placed(a->decay, 4))
        return refuse(CBINFER_EINVAL, "%s: state and decay must be given, aligned to their element", w);
    if (!aligned(a->lengths, 4)) return refuse(CBINFER_EINVAL, "%s: lengths must be aligned to their element", w);
    if (int rc = check_workspace(w, a->workspace, a->workspace_bytes, cbk::linear_attention_workspace(*a))) return rc;
    return launched(cbk::linear_attention(static_cast<hipStream_t>(stream), *a), w);
}

int cbinfer_quantise_weights(const void *weights, int32_t dtype, int64_t rows, int64_t cols, int64_t row_stride, int32_t group,
                             uint8_t *codes, uint16_t *scales, void *stream)
{
    const char *w = "quantise_weights";
    if (!known(dtype)) return refuse(CBINFER_EINVAL, "%s: dtype must be CBINFER_F32 or CBINFER_BF16", w);
    if (cbinfer_packed_weights_bytes(rows, cols, group) == 0) return CBINFER_EINVAL;
    if (!placed(weights, element(dtype)) || !codes || !placed(scales, 2))
        return refuse(CBINFER_EINVAL, "%s: weights, codes and scales must be given, aligned to their element", w);
    return launched(cbk::quantise_weights(static_cast<hipStream_t>(stream), weights, dtype, rows, cols, row_stride, group, codes,
                                          scales), w);
}

size_t cbinfer_packed_weights_bytes(int64_t rows, int64_t cols, int32_t group)
{
    // threads of a launch are counted in 32 bits
    if (rows < 1 || cols < 1 || rows > (1 << 26) || cols > (1 << 25) || rows * cols > (int64_t)1 << 32) {
        refuse(CBINFER_EINVAL, "4-bit weights: rows and cols must be 1 .. 2^26 and 1 .. 2^25, together at most 2^32");
        return 0;
    }
    if (group != 32 && group != 64 && group != 128) {
        refuse(CBINFER_EINVAL, "4-bit weights: a group must be 32, 64 or 128 weights (got %d)", group);
        return 0;
    }
    return cbk::packed_weights_bytes(rows, cols, group);
}

int cbinfer_pack_weights(const uint8_t *codes, const uint16_t *scales, int64_t rows, int64_t cols, int32_t group, void *packed,
                         void *stream)
{
    const char *w = "pack_weights";
    if (cbinfer_packed_weights_bytes(rows, cols, group) == 0) return CBINFER_EINVAL;
    if (!codes || !placed(scales, 2) || !placed(packed, kAlignment))
        return refuse(CBINFER_EINVAL, "%s: codes, scales and packed must be given, scales at 2 bytes, packed at 256", w);
    return launched(cbk::pack_weights(static_cast<hipStream_t>(stream), codes, scales, rows, cols, group, packed), w);
}

size_t cbinfer_quantised_product_workspace_bytes(const cbinfer_quantised_product_args *a)
{
    if (check(a) != CBINFER_OK) return 0;
    return cbk::quantised_product_workspace(*a);
}

int cbinfer_quantised_product(const cbinfer_quantised_product_args *a, void *stream)
{
    const char *w = "quantised_product";
    if (int rc = check(a)) return rc;
    if (a->tokens == 0) return CBINFER_OK;
    const size_t e = element(a->dtype);
    if (!placed(a->x, e) || !placed(a->y, e)) return refuse(CBINFER_EINVAL, "%s: x and y must be given, aligned to their element", w);
    if (!placed(a->packed, kAlignment)) return refuse(CBINFER_EINVAL, "%s: packed weights must be given, 256-byte aligned", w);
    if (!aligned(a->bias, 4)) return refuse(CBINFER_EINVAL, "%s: bias must be aligned to its element", w);
    if (int rc = check_workspace(w, a->workspace, a->workspace_bytes, cbk::quantised_product_workspace(*a))) return rc;
    return launched(cbk::quantised_product(static_cast<hipStream_t>(stream), *a), w);
}

int cbinfer_gated_norm(const cbinfer_gated_norm_args *a, void *stream)
{
    const char *w = "gated_norm";
    if (!a) return refuse(CBINFER_EINVAL, "%s: arguments are NULL", w);
    if (!known(a->dtype)) return refuse(CBINFER_EINVAL, "%s: dtype must be CBINFER_F32 or CBINFER_BF16", w);
    if (a->sum_dtype != CBINFER_F32 && a->sum_dtype != a->dtype)
        return refuse(CBINFER_EINVAL, "%s: sum_dtype must be CBINFER_F32 or dtype", w);
    if (a->rows < 0 || a->rows > kMost32) return refuse(CBINFER_EINVAL, "%s: rows must be 0 .. 2^31-1", w);
    if (a->size < 1) return refuse(CBINFER_EINVAL, "%s: size must be >= 1", w);
    if (a->size > 16384) return refuse(CBINFER_EUNSUPPORTED, "%s: rows of more than 16384 values", w);
    if (a->group < 0 || (a->group && a->size % a->group)) return refuse(CBINFER_EINVAL, "%s: group must divide size", w);
    if (a->gate_kind < CBINFER_GATE_NONE || a->gate_kind > CBINFER_GATE_SIGMOID)
        return refuse(CBINFER_EINVAL, "%s: unknown gate_kind", w);
    if ((a->gate_kind != CBINFER_GATE_NONE) != (a->gate != nullptr) && a->rows)
        return refuse(CBINFER_EINVAL, "%s: gate and gate_kind go together", w);
    if (!std::isfinite(a->scale) || !(a->eps >= 0.0f) || !std::isfinite(a->eps))
        return refuse(CBINFER_EINVAL, "%s: scale must be finite, eps finite and >= 0", w);
    if (a->rows == 0) return CBINFER_OK;
    const size_t e = element(a->dtype), s = element(a->sum_dtype);
    if (!placed(a->x, e)) return refuse(CBINFER_EINVAL, "%s: x must be given, aligned to its element", w);
    if (!a->h && !a->y) return refuse(CBINFER_EINVAL, "%s: no output asked for", w);
    if ((a->y != nullptr) != (a->next_weight != nullptr)) return refuse(CBINFER_EINVAL, "%s: y and next_weight go together", w);
    if (!aligned(a->gate, e) || !aligned(a->y, e) || !aligned(a->residual, s) || !aligned(a->h, s) || !aligned(a->weight, 4) ||
        !aligned(a->channel_scale, 4) || !aligned(a->next_weight, 4))
        return refuse(CBINFER_EINVAL, "%s: every tensor must be aligned to its element", w);
    return launched(cbk::gated_norm(static_cast<hipStream_t>(stream), *a), w);
}

} // extern "C"
