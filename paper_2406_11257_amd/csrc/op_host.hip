// Entry points of the operators on reconstructed weights: argument checks and the choice of kernels.
#include <hip/hip_runtime.h>

#include "../../include/excp.h"
#include "excp_ops.h"

namespace {

static_assert(EXCP_TOP_MAX == EXCP_MAX_TOP, "");

bool elem_size(int type, u64 &size) {
    switch (type) {
        case EXCP_TYPE_F32: size = 4; return true;
        case EXCP_TYPE_F16: case EXCP_TYPE_BF16: size = 2; return true;
        default: return false;
    }
}
bool dims_ok(u64 a, u64 b, u64 c = 0) { return a <= EXCP_MAX_DIM && b <= EXCP_MAX_DIM && c <= EXCP_MAX_DIM; }
bool aligned(const void *p, u64 to) { return p && ((uintptr_t)p & (to - 1)) == 0; }
// a matrix that is there: element aligned, rows that do not overlap, offsets that 64 bits hold
bool matrix_ok(const void *p, int type, u64 cols, u64 ld) {
    u64 size;
    return elem_size(type, size) && aligned(p, size) && ld >= cols && ld <= 1ull << 32;
}
bool coded_ok(const void *codes, const void *scales) { return aligned(codes, 16) && aligned(scales, 4); }
u32 groups_of(u64 cols) { return (u32)((cols + EXCP_MX_GROUP - 1) / EXCP_MX_GROUP); }

// The context's device made current; EXCP_E_HIP where that fails or the context takes no more work.
int enter(const excp_ctx *c, OpsContext &o) {
    o = excp_ops_context(c);
    int now = -1;
    if (o.broken || hipGetDevice(&now) != hipSuccess || (now != o.device && hipSetDevice(o.device) != hipSuccess)) return EXCP_E_HIP;
    return EXCP_OK;
}
int launched() { return hipGetLastError() == hipSuccess ? EXCP_OK : EXCP_E_HIP; }

}  // namespace

extern "C" {

uint64_t excp_mx_code_bytes(uint64_t rows, uint64_t cols) { return dims_ok(rows, cols) ? rows * 64 * groups_of(cols) : 0; }
uint64_t excp_mx_scale_bytes(uint64_t rows, uint64_t cols) { return dims_ok(rows, cols) ? rows * 4 * groups_of(cols) : 0; }

int excp_mx_quantize(excp_ctx *c, const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ld, void *codes,
                     void *scales, void *codes_t, void *scales_t) {
    u64 size;
    if (!c || !elem_size(type, size) || !dims_ok(rows, cols) || !codes != !scales || !codes_t != !scales_t) return EXCP_E_ARG;
    if (!codes && !codes_t && rows && cols) return EXCP_E_ARG;
    if (rows == 0 || cols == 0) return EXCP_OK;
    if (!matrix_ok(x, type, cols, ld) || (codes && !coded_ok(codes, scales)) || (codes_t && !coded_ok(codes_t, scales_t)))
        return EXCP_E_ARG;
    OpsContext o;
    if (int rc = enter(c, o)) return rc;
    launch_mx_quantize({{x, ld, (u32)rows, (u32)cols, type}, (unsigned char *)codes, (unsigned char *)scales,
                        (unsigned char *)codes_t, (unsigned char *)scales_t}, o.cus, o.stream);
    return launched();
}

int excp_mx_dequantize(excp_ctx *c, const void *codes, const void *scales, uint64_t rows, uint64_t cols, void *x, int type,
                       uint64_t ld) {
    u64 size;
    if (!c || !elem_size(type, size) || !dims_ok(rows, cols)) return EXCP_E_ARG;
    if (rows == 0 || cols == 0) return EXCP_OK;
    if (!matrix_ok(x, type, cols, ld) || !coded_ok(codes, scales)) return EXCP_E_ARG;
    OpsContext o;
    if (int rc = enter(c, o)) return rc;
    launch_mx_dequantize({(const unsigned char *)codes, (const unsigned char *)scales, x, ld, (u32)rows, (u32)cols, type},
                         o.cus, o.stream);
    return launched();
}

int excp_mx_matmul(excp_ctx *c, const void *a_codes, const void *a_scales, const void *b_codes, const void *b_scales,
                   uint64_t m, uint64_t n, uint64_t k, void *y, int type, uint64_t ld) {
    u64 size;
    if (!c || !elem_size(type, size) || !dims_ok(m, n, k) || k > EXCP_MX_MAX_K) return EXCP_E_ARG;
    if (m == 0 || n == 0) return EXCP_OK;
    if (!matrix_ok(y, type, n, ld) || (k && (!coded_ok(a_codes, a_scales) || !coded_ok(b_codes, b_scales)))) return EXCP_E_ARG;
    OpsContext o;
    if (int rc = enter(c, o)) return rc;
    MxProduct p = {(const unsigned char *)a_codes, (const unsigned char *)a_scales, (const unsigned char *)b_codes,
                   (const unsigned char *)b_scales, {}, y, ld, (u32)m, (u32)n, groups_of(k), type};
    launch_mx_product(p, o.cus, o.stream);
    return launched();
}

int excp_mx_linear(excp_ctx *c, const void *x, int x_type, uint64_t ldx, const void *w_codes, const void *w_scales, uint64_t m,
                   uint64_t n, uint64_t k, void *y, int y_type, uint64_t ldy, void *x_codes, void *x_scales) {
    u64 size;
    if (!c || !elem_size(x_type, size) || !elem_size(y_type, size) || !dims_ok(m, n, k) || k > EXCP_MX_MAX_K || !x_codes != !x_scales) return EXCP_E_ARG;
    if (m == 0 || n == 0) return EXCP_OK;
    if (!matrix_ok(y, y_type, n, ldy)) return EXCP_E_ARG;
    if (k && (!matrix_ok(x, x_type, k, ldx) || !coded_ok(w_codes, w_scales))) return EXCP_E_ARG;
    if (k && (x_codes ? !coded_ok(x_codes, x_scales) : m > EXCP_MX_FEW_ROWS)) return EXCP_E_ARG;
    OpsContext o;
    if (int rc = enter(c, o)) return rc;
    MxProduct p = {(const unsigned char *)x_codes, (const unsigned char *)x_scales, (const unsigned char *)w_codes,
                   (const unsigned char *)w_scales, {x, ldx, (u32)m, (u32)k, x_type}, y, ldy, (u32)m, (u32)n, groups_of(k), y_type};
    if (m <= EXCP_MX_FEW_ROWS) {
        // which way they go, and so the order of their sums, is the same whether the caller has given room or not
        const u64 codes = excp_mx_code_bytes(m, k);
        if (codes + excp_mx_scale_bytes(m, k) > sizeof(RowPart) * EXCP_ROW_PARTS || !mx_quantized_first(p, o.cus)) {
            launch_mx_few_rows(p, o.cus, o.stream);
            return launched();
        }
        if (!x_codes) {
            p.a_codes = (const unsigned char *)o.parts;
            p.a_scales = p.a_codes + codes;
        }
    }
    if (k) launch_mx_quantize({p.x, (unsigned char *)p.a_codes, (unsigned char *)p.a_scales, nullptr, nullptr}, o.cus, o.stream);
    launch_mx_product(p, o.cus, o.stream);
    return launched();
}

int excp_token_logprobs(excp_ctx *c, const void *logits, int type, uint64_t rows, uint64_t vocab, uint64_t ld,
                        const int64_t *targets, int ntop, float *logprob, float *entropy, float *lse, float *top_logprob,
                        int64_t *top_ids) {
    u64 size;
    if (!c || !elem_size(type, size) || !dims_ok(rows, vocab) || ntop < 0 || ntop > EXCP_MAX_TOP) return EXCP_E_ARG;
    if (rows == 0) return EXCP_OK;
    if (vocab && !matrix_ok(logits, type, vocab, ld)) return EXCP_E_ARG;
    if ((logprob && !aligned(targets, 8)) || (logprob && !aligned(logprob, 4)) || (entropy && !aligned(entropy, 4)) ||
        (lse && !aligned(lse, 4)) || (top_logprob && !aligned(top_logprob, 4)) || (top_ids && !aligned(top_ids, 8)))
        return EXCP_E_ARG;
    OpsContext o;
    if (int rc = enter(c, o)) return rc;
    const bool top = ntop && (top_logprob || top_ids);
    launch_row_scores({logits, ld, (u32)rows, (u32)vocab, type, top ? ntop : 0, (const long long *)targets, logprob, entropy, lse,
                       top_logprob, (long long *)top_ids}, o);
    return launched();
}

int excp_token_logprobs_backward(excp_ctx *c, const void *logits, int type, uint64_t rows, uint64_t vocab, uint64_t ld,
                                 const int64_t *targets, const float *lse, const float *entropy, const int64_t *top_ids, int ntop,
                                 const float *g_logprob, const float *g_entropy, const float *g_top, void *dlogits, uint64_t ldd) {
    u64 size;
    if (!c || !elem_size(type, size) || !dims_ok(rows, vocab) || ntop < 0 || ntop > EXCP_MAX_TOP) return EXCP_E_ARG;
    if (rows == 0 || vocab == 0) return EXCP_OK;
    if (!matrix_ok(logits, type, vocab, ld) || !matrix_ok(dlogits, type, vocab, ldd) || (logits == dlogits && ld != ldd)) return EXCP_E_ARG;
    if (!aligned(lse, 4) || (g_logprob && (!aligned(g_logprob, 4) || !aligned(targets, 8))) ||
        (g_entropy && (!aligned(g_entropy, 4) || !aligned(entropy, 4))))
        return EXCP_E_ARG;
    if (ntop == 0) g_top = nullptr;
    if (g_top && (!aligned(g_top, 4) || !aligned(top_ids, 8))) return EXCP_E_ARG;
    OpsContext o;
    if (int rc = enter(c, o)) return rc;
    launch_row_gradient({logits, dlogits, ld, ldd, (u32)rows, (u32)vocab, type, g_top ? ntop : 0, (const long long *)targets,
                         (const long long *)top_ids, lse, entropy, g_logprob, g_entropy, g_top}, o.cus, o.stream);
    return launched();
}

}  // extern "C"
