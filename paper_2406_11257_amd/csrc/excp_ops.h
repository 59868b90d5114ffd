// What the operators on reconstructed weights (4-bit microscaled products, token log probabilities) share:
// the launchers that op_host.hip calls, element types, and loads of rows that may start anywhere.
#pragma once
#include "excp_device.h"

struct excp_ctx;

#define EXCP_TOP_MAX 64u           // alternatives of a row (EXCP_MAX_TOP of the C ABI)
#define EXCP_ROW_PARTS 1024u       // parts of rows that a call may have
// What one workgroup found in its part of a row of logits (see k_logprobs.hip).
struct RowPart { float max, sum, weighted, pad; u64 key[EXCP_TOP_MAX]; };

// What an operator needs of a context.
struct OpsContext {
    int device;
    hipStream_t stream;
    u32 cus;               // compute units
    RowPart *parts;        // EXCP_ROW_PARTS records of rows that several workgroups share; or room for a few rows' codes
    u32 *tickets;          // as many counters, zero between calls
    bool broken;
};
OpsContext excp_ops_context(const excp_ctx *c);   // (excp_host.hip)

enum ElemType { ET_F32 = 0, ET_F16 = 1, ET_BF16 = 2 };

#define EXCP_MX_BLOCK 32u          // elements under one scale
#define EXCP_MX_GROUP 128u         // elements to which rows are padded: 64 B of codes, 4 B of scales

// rows x cols matrix, element (i, j) at p + (i * ld + j) elements
struct Matrix { const void *p; u64 ld; u32 rows, cols; int type; };

struct MxQuantize { Matrix x; unsigned char *codes, *scales, *codes_t, *scales_t; };
struct MxDequantize { const unsigned char *codes, *scales; void *x; u64 ld; u32 rows, cols; int type; };
// y (m x n) = A B^T over `groups` groups of 128 elements; x, where it is given, is A before its quantisation
struct MxProduct {
    const unsigned char *a_codes, *a_scales, *b_codes, *b_scales;
    Matrix x;
    void *y;
    u64 ld;
    u32 m, n, groups;
    int type;
};

struct RowScores {
    const void *logits;
    u64 ld;
    u32 rows, vocab;
    int type, ntop;
    const long long *targets;
    float *logprob, *entropy, *lse, *top_logprob;
    long long *top_ids;
};
struct RowGradient {
    const void *logits;
    void *d;
    u64 ld, ldd;
    u32 rows, vocab;
    int type, ntop;
    const long long *targets, *top_ids;
    const float *lse, *entropy, *g_logprob, *g_entropy, *g_top;
};

void launch_mx_quantize(const MxQuantize &q, u32 cus, hipStream_t s);
void launch_mx_dequantize(const MxDequantize &d, u32 cus, hipStream_t s);
void launch_mx_product(const MxProduct &p, u32 cus, hipStream_t s);
void launch_mx_few_rows(const MxProduct &p, u32 cus, hipStream_t s);
bool mx_quantized_first(const MxProduct &p, u32 cus);   // whether a few rows of x are better quantised in a launch of their own
void launch_row_scores(const RowScores &r, const OpsContext &c);
void launch_row_gradient(const RowGradient &r, u32 cus, hipStream_t s);

// Calls f with a tag of the element type: `f(float())`, `f(_Float16())`, `f(__bf16())`.
template <class F>
inline void with_type(int type, F f) {
    if (type == ET_F32) f(float());
    else if (type == ET_F16) f((_Float16)0);
    else f((__bf16)0);
}
