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
 * How sure labels are, and what a student learns from the best classes of a teacher alone; heads of any number of classes:
 *   dynlp_row_scores   log probabilities of given classes, entropy and first classes of rows of logits or of propagated labels
 *   dynlp_head_scores  the same of the head's answers
 *   dynlp_head_distill divergence of the head from a teacher's first classes, with its gradients
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
 * What rows of one value per class say, without the distribution itself: with p = softmax(x), or (probabilities) x / sum of x, as propagated labels are,
 *   log_given[n][k] = log p[classes[n][k]];  a negative class is padding and gives 0, so does one that is not below the row's classes, and it is counted in *rejected
 *   entropy[n]      = - sum over c of p[c] log p[c], 0 where p is 0
 *   top_classes[n]  = the `top` first classes by their values, of equal ones the lowest, from the first on;  log_top[n] = their log p
 * classes: rows x given int32; outputs rows x given and rows x top without padding; entropy, top_classes and log_top may each be NULL.
 * 0 <= given <= DYNLP_MAX_GIVEN, 0 <= top <= DYNLP_MAX_TOP and the classes there are.
 * A logit of -infinity (a probability of 0) has log p = -infinity; a row of nothing else is 1/C everywhere.  A value that is not a number
 * makes log p and entropy of its row so, as does +infinity; for the order it counts as -infinity.  Probabilities are not negative.
 * The order is that of the values, also where log p is the same.  Rows of probabilities may have any sum, also one that 32 bits do not hold.
 */
#define DYNLP_MAX_TOP 128
#define DYNLP_MAX_GIVEN (1 << 20)
#define DYNLP_MAX_WIDE_CLASSES (1 << 22) /* of the heads below */
#define DYNLP_MAX_WIDE_DIM (1 << 16)
typedef struct dynlp_scores {
    int32_t given, top;
    const int32_t* classes;
    float* log_given;
    float* entropy;
    int32_t* top_classes;
    float* log_top;
    int32_t* rejected; /* one int32 that grows, or NULL */
} dynlp_scores;
dynlp_status dynlp_row_scores(const dynlp_matrix* x, int32_t probabilities, const dynlp_scores* scores, const dynlp_call* call);
int64_t dynlp_row_scores_workspace(int64_t rows, int32_t classes, int32_t top);

/*
 * The same of the head's logits z = h W^T + bias, which are not kept: h, weight and bias as in dynlp_head_labels, but of up to DYNLP_MAX_WIDE_CLASSES classes and
 * DYNLP_MAX_WIDE_DIM elements of a row.  A class whose bias is -infinity has that logit whatever h holds.  The logits of float32 heads of more than 64 classes are made
 * from three 16-bit terms of each value, which hold all of it, but where up to 16 rows are scored: there an infinite element of h or weight makes infinite logits, as it does in
 * other heads, and otherwise makes the logits it meets not a number (products that 32 bits do not hold may).
 */
dynlp_status dynlp_head_scores(const dynlp_matrix* h, const dynlp_matrix* weight, const float* bias, const dynlp_scores* scores, const dynlp_call* call);
int64_t dynlp_head_scores_workspace(int64_t rows, int32_t dim, int32_t classes, int32_t type);

/*
 * Learning from a teacher of which each row keeps some classes with their logits (log probabilities do as well: a constant of the row does not matter).
 * q = softmax(logits / temperature) over a row's list, 0 for classes that are not in it; p = softmax(z / temperature) over all classes of the head:
 *   loss[n] = r[n] temperature^2 sum over c of q[n][c] (log q[n][c] - log p[n][c])
 *   dz = grad_scale r[n] temperature (p[n] - q[n]);  dh = dz W,  dweight = dz^T h,  dbias = sum_n dz[n]
 *   classes, logits  rows x kept, 1 <= kept <= DYNLP_MAX_TOP.  A negative class is no entry, nor is one that is not below the head's classes, which is counted in
 *                    *rejected (int32, or NULL).  A class that is named several times has the sum of its probabilities.  One class alone
 *                    is a hard label, and the loss its cross entropy.
 *   row_weight       r, float32, or NULL for 1.  A row with weight 0 is left out (loss 0, dh 0, nothing in the other gradients, whatever h and its list hold), and so is
 *                    one without an entry whose logit is more than -infinity, and one whose own logits are all -infinity.
 *   loss             rows float32; dh: rows x dim, of h's type; dweight: classes x dim, float32 or of h's type; dbias: classes float32.  Each of the four may be NULL (a
 *                    matrix with data NULL, too).
 * An entry's logit that is not a number, or +infinity, makes its row's loss and dz so, of all classes.  Heads as in dynlp_head_scores.
 * Up to 64 classes, and in float32 heads, the gradients are made from all 24 bits of dz.  Of larger heads in 16 bits, dh and a dweight in 16 bits are made from dz
 * rounded to h's type, with up to 256 rows, or 2^31 rows times dim times classes, to two such terms; a dweight in float32 is made from all of it (float16: 22 bits).  In
 * float16 what lies below 2^-39 of a row's r is left out of its dh, and what lies below 2^-39 of the largest r of dweight.
 */
typedef struct dynlp_teacher {
    const int32_t* classes;
    const float* logits;
    const float* row_weight;
    int32_t* rejected;
    int32_t kept;
    float temperature; /* > 0; it, its square and log2(e) over it finite in 32 bits, as is grad_scale times it */
    float grad_scale;
} dynlp_teacher;
dynlp_status dynlp_head_distill(const dynlp_matrix* h, const dynlp_matrix* weight, const float* bias, const dynlp_teacher* teacher, float* loss,
                                const dynlp_matrix* dh, const dynlp_matrix* dweight, float* dbias, const dynlp_call* call);
/* grad_type: of dweight (h's where there is none), or -1 where the loss alone is asked for. */
int64_t dynlp_head_distill_workspace(int64_t rows, int32_t dim, int32_t classes, int32_t kept, int32_t type, int32_t grad_type);

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
