/*
 * dynlp_train.h — C ABI of libdynlp: training and asking a student of propagated labels on one AMD MI355X.
 *
 * dynlp_get_labels gives the vertices of the graph their class distributions.  A student learns them, so that items that
 * are not in the graph have labels too.  An item is a list of tokens with weights (TF-IDF, for a text); its row is the
 * weighted sum of the tokens' rows in a table; a head with one row per class turns that into a class distribution:
 *   dynlp_embed        rows of items (or of single tokens) from the table
 *   dynlp_head_labels  class distributions and hard labels, in the form of dynlp_get_labels
 *   dynlp_head_loss    cross entropy against soft rows (what dynlp_get_labels returns) or hard labels, with its gradients
 *   dynlp_embed_grad   gradient of the table
 *   dynlp_adamw_step   one AdamW step over many tensors, states in 32 or 8 bits
 *
 * Conventions (those of dynlp.h, and where they differ)
 *   - Array arguments are DEVICE pointers on the calling thread's current device.  Structs and scalars are host memory.
 *   - Calls only ENQUEUE work on dynlp_call.stream (a hipStream_t; NULL = the default stream) and return; inputs must stay as
 *     they are, and outputs may be read, in stream order.  Nothing is allocated, copied or waited for, so that calls may be
 *     captured in a HIP graph (host scalars such as lr and step are captured as they stand).
 *   - Scratch memory is the caller's: dynlp_call.workspace, of the size that the *_workspace function of the call gives for the same
 *     sizes, aligned to 256 bytes, not shared with calls that may run at the same time.
 *   - Outputs overlap neither inputs, workspace nor each other, but for what a call says that it updates in place.  Rows of two matrices may
 *     take turns in one array.  (Checked: the matrices of a call.)
 *   - A call refuses what it can see (DYNLP_ERR_INVALID_ARG, nothing enqueued; dynlp_last_error(NULL) says what, on the same
 *     thread).  Values on the device are not waited for: every id and offset is checked where it is used, and what is out
 *     of range is left out as described below; nothing outside the arrays is read or written.
 *   - Sums, softmax statistics and the states' arithmetic are held in 32 bits whatever the types; results are rounded once.
 *     No result depends on timing: the same inputs give the same bits.
 *   - No C++ exception crosses this boundary.  Calls hold no state; any thread may make them.
 */
#ifndef DYNLP_TRAIN_H
#define DYNLP_TRAIN_H

#include "dynlp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of the elements of an array. */
typedef enum dynlp_type { DYNLP_FLOAT32 = 0, DYNLP_BFLOAT16 = 1, DYNLP_FLOAT16 = 2 } dynlp_type;

/* A matrix in row-major order: element (i, j) is data[i * stride + j].  stride >= dim, and any (no alignment beyond the
 * element's own is needed; 16 bytes are faster).  rows < 2^31 - 1, 1 <= dim <= 2^28. */
typedef struct dynlp_matrix {
    void* data;
    int64_t rows;
    int64_t stride; /* elements from one row to the next */
    int32_t dim;    /* elements of a row */
    int32_t type;   /* dynlp_type */
} dynlp_matrix;

/* Where and with what scratch memory a call runs. */
typedef struct dynlp_call {
    void* stream;
    void* workspace;
    int64_t workspace_bytes;
} dynlp_call;

/*
 * Tokens of items.  Item b has the tokens offsets[b] .. offsets[b + 1] - 1; with offsets NULL every token is an item of its
 * own (items == count).
 *   ids      count ids, int32 or (ids_are_64) int64.  A negative id is padding: it contributes nothing.  So does an id that
 *            is not below the table's rows, and it is counted in *rejected.
 *   offsets  items + 1 offsets that do not decrease, from 0 to count (tokens outside offsets[0] .. offsets[items] belong to no
 *            item; offsets that decrease give no defined result, but nothing outside the arrays is touched)
 *   weights  count weights, or NULL for 1.  The weight of a token that contributes nothing is not looked at.
 *   scale    factor of every item
 *   rejected one int32 that grows by the number of rejected ids of the whole list, those that are in no item among them, or NULL
 * count and items are below 2^31.
 */
typedef struct dynlp_tokens {
    int64_t count;
    int64_t items;
    const void* ids;
    const int64_t* offsets;
    const float* weights;
    int32_t* rejected;
    float scale;
    int32_t ids_are_64;
} dynlp_tokens;

/*
 * out[b] = scale * sum over the tokens i of item b of weights[i] * table[ids[i]]; nothing but zeros for an item without tokens.
 * table and out have the same type and dim; out->rows == tokens->items.
 */
dynlp_status dynlp_embed(const dynlp_matrix* table, const dynlp_tokens* tokens, const dynlp_matrix* out, const dynlp_call* call);
int64_t dynlp_embed_workspace(int64_t count, int64_t items, int32_t dim);

/*
 * The table's gradient, dense: out[v] = scale * sum over the tokens i with ids[i] == v of weights[i] * grad[item of i]; rows
 * of ids that do not occur are zeros.  grad->rows == tokens->items; out is float32 or of grad's type.  The tokens are sorted
 * by id, and those of one id are added in the order they are listed in, in pieces whose bounds depend on the sizes alone.
 */
dynlp_status dynlp_embed_grad(const dynlp_matrix* grad, const dynlp_tokens* tokens, const dynlp_matrix* out, const dynlp_call* call);
int64_t dynlp_embed_grad_workspace(int64_t count, int64_t items, int32_t dim, int64_t table_rows);

/*
 * The head's answers: z = h W^T + bias, soft = softmax(z) (float32, rows x classes, no padding; or NULL), hard = argmax with the
 * lowest class winning ties (int32; or NULL), as dynlp_get_labels gives them.
 *   h       rows x dim; weight: classes x dim, of h's type, 1 .. DYNLP_MAX_CLASSES classes; bias: classes float32, or NULL
 * A class whose logit is -infinity has probability 0; a row with no other logit is 1/C everywhere, hard label 0.  A logit that is
 * not a number makes the row's soft labels so; for the hard label it counts as -infinity.
 */
dynlp_status dynlp_head_labels(const dynlp_matrix* h, const dynlp_matrix* weight, const float* bias, float* soft, int32_t* hard,
                               const dynlp_call* call);

/*
 * Loss of the head against targets and its gradients:
 *   loss[n] = r[n] * sum_c q[n][c] * (logsumexp(z[n]) - z[n][c])          (a class with q = 0 adds nothing, whatever its logit)
 *   dz = grad_scale * r[n] * (S[n] * softmax(z[n]) - q[n]),  S[n] = sum_c q[n][c]
 *   dh = dz W,  dweight = dz^T h,  dbias = sum_n dz[n]
 *   soft        targets q: rows x classes float32 (need not sum to one), or NULL and then
 *   hard        classes, int32: q is one-hot.  A negative class leaves the row out; so does one that is not below classes,
 *               and it is counted in *rejected (int32, or NULL)
 *   row_weight  r, float32, or NULL for 1.  A row with weight 0 is left out: loss 0, dh 0, nothing in the other gradients, whatever
 *               its h and target hold
 *   loss        rows float32; dh: rows x dim, of h's type; dweight: classes x dim float32, no padding; dbias: classes float32.
 *               Each of the four may be NULL (a matrix with data NULL, for dh).  Where dweight is, dh may be h itself: same data and stride.
 * A row whose logits are all -infinity is left out.
 */
typedef struct dynlp_targets {
    const float* soft;
    const int32_t* hard;
    const float* row_weight;
    int32_t* rejected;
    float grad_scale;
} dynlp_targets;
dynlp_status dynlp_head_loss(const dynlp_matrix* h, const dynlp_matrix* weight, const float* bias, const dynlp_targets* targets,
                             float* loss, const dynlp_matrix* dh, float* dweight, float* dbias, const dynlp_call* call);
int64_t dynlp_head_loss_workspace(int64_t rows, int32_t dim, int32_t classes, int32_t type);

/*
 * One step of AdamW with decoupled weight decay over `count` tensors:
 *   g' = *grad_scale * grad (1 without it);  m = beta1 m + (1 - beta1) g';  v = beta2 v + (1 - beta2) g'^2
 *   param = param (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps);  copy = param, rounded
 * States in 32 bits: m and v, float32, n each.  States in 8 bits: m and r = sqrt(v) as 8-bit floats of 4 exponent and 3 mantissa
 * bits (OCP e4m3, no infinities) times a power of two for each block of DYNLP_STATE_BLOCK elements, chosen so that the block's
 * largest value lies in 128 .. 256 of the format.  The arithmetic is that of 32 bits; only what is kept is rounded, up or down at
 * random (a running mean that is rounded to nearest in 8 bits stands still once its steps are smaller than half a unit), from 16 bits
 * that are a function of seed, step, the tensor's place in the list and the element's place in the tensor alone.
 * An r that is not zero is never rounded to zero.  A block whose largest value is below 2^-119 is kept as zero, one
 * with a value that is not finite as not-a-number from then on.
 */
#define DYNLP_STATE_BLOCK 256
typedef struct dynlp_adamw_tensor {
    int64_t n;
    void* param;         /* n of param_type, read and written */
    const void* grad;    /* n of grad_type */
    void* m;             /* n float32, or n 8-bit codes */
    void* v;             /* n float32, or n 8-bit codes of r */
    float* m_scale;      /* 8 bits: ceil(n / DYNLP_STATE_BLOCK) float32 */
    float* v_scale;
    void* copy;          /* n of copy_type, written, or NULL */
    float weight_decay;
    int32_t param_type, grad_type, copy_type; /* dynlp_type */
} dynlp_adamw_tensor;
typedef struct dynlp_adamw_options {
    double lr, beta1, beta2, eps; /* lr >= 0, 0 <= beta < 1, eps > 0; eps, lr / (1 - beta1^step) and lr weight_decay finite, and eps > 0, in 32 bits */
    int64_t step;                 /* 1 for the first step */
    const float* grad_scale;      /* one float32 on the device, or NULL */
    uint32_t seed;
    int32_t state_bits;           /* 32 or 8 */
} dynlp_adamw_options;
dynlp_status dynlp_adamw_step(int32_t count, const dynlp_adamw_tensor* tensors, const dynlp_adamw_options* options,
                              const dynlp_call* call);

#ifdef __cplusplus
}
#endif
#endif /* DYNLP_TRAIN_H */
