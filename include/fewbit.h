/*
 * fewbit.h -- C ABI of the Few-Bit Backward hot path for NVIDIA B200 (sm_100a).
 *
 * The method (arXiv 2202.00441): a pointwise activation f keeps, for its
 * backward pass, not the input x but only the index of the interval of a
 * piecewise-constant approximation q of f' that x falls into (Eq. 2), i.e.
 * `bits` = log2(K) bits per element.  Backward multiplies grad_out by the
 * level of that interval instead of f'(x) (Listing 1).  The intervals and
 * levels minimise the L2 error of Eq. 3 and are found once, offline, by the
 * dynamic programme of Eq. 7-9.
 *
 * Conventions that hold for every call
 *   - plain C types only; every pointer is commented HOST or DEVICE;
 *   - the library never throws, never calls exit(), never synchronises the
 *     device in the DEVICE-pointer calls and never allocates device memory;
 *     the only allocation is the host-side table object;
 *   - the caller owns every buffer; a table is immutable after creation and
 *     may be used from many threads and streams at once;
 *   - every function that can fail returns a fewbit_status.
 *
 * Table layout: K = 2^bits levels lev[0..K-1] and K-1 interior boundaries
 * s[0..K-2] (non-decreasing), both binary32.  The code of x is
 *     code(x) = #{ j : s[j] < x }        (strict, compared in binary32)
 * so interval i is (s[i-1], s[i]], anything below s[0] has code 0, anything
 * above s[K-2] has code K-1, and NaN has code 0.
 *
 * Saved-tensor layout ("packed"): one flat bit stream, element e occupies
 * bits [e*bits, e*bits + bits), least significant bit first, stored in
 * little-endian 32-bit words.  32 consecutive elements always fill exactly
 * `bits` words.  Unused high bits of the last word are written as zero.
 */
#ifndef FEWBIT_H_
#define FEWBIT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(_WIN32)
#define FEWBIT_API
#else
#define FEWBIT_API __attribute__((visibility("default")))
#endif

typedef struct fewbit_table fewbit_table;

/* Activations f (Sec. 2; the rows of Table 1 plus ELU and LeakyReLU). */
typedef enum fewbit_act {
    FEWBIT_GELU = 0,       /* x * Phi(x), the erf form                       */
    FEWBIT_SILU = 1,       /* x * sigmoid(x)  (Swish)                        */
    FEWBIT_SIGMOID = 2,    /* 1 / (1 + exp(-x))                              */
    FEWBIT_TANH = 3,
    FEWBIT_ELU = 4,        /* x > 0 ? x : exp(x) - 1        (alpha = 1)      */
    FEWBIT_SOFTPLUS = 5,   /* log(1 + exp(x))               (beta = 1)       */
    FEWBIT_LEAKY_RELU = 6, /* x > 0 ? x : 0.01 x                             */
    FEWBIT_RELU = 7,       /* max(x, 0); exact with 1 bit (Sec. 2)           */
    FEWBIT_SELU = 8        /* 1.0507 (x > 0 ? x : 1.6733 (exp(x) - 1))       */
} fewbit_act;
#define FEWBIT_NUM_ACTS 9

typedef enum fewbit_dtype {
    FEWBIT_F32 = 0,        /* IEEE binary32                                  */
    FEWBIT_BF16 = 1,       /* bfloat16                                       */
    FEWBIT_F16 = 2         /* IEEE binary16                                  */
} fewbit_dtype;

typedef enum fewbit_status {
    FEWBIT_OK = 0,
    FEWBIT_ERR_INVALID_ARG = 1,   /* NULL pointer, bits outside 1..4, bad enum, unsorted table */
    FEWBIT_ERR_UNSUPPORTED = 2,   /* valid request this build cannot serve                      */
    FEWBIT_ERR_ALIGNMENT = 3,     /* a buffer breaks the alignment rule of the call             */
    FEWBIT_ERR_CUDA = 4,          /* a CUDA call failed; see fewbit_last_cuda_error()           */
    FEWBIT_ERR_ALLOC = 5,         /* host allocation failed / workspace too small               */
    FEWBIT_ERR_TOO_LARGE = 6      /* n exceeds the fixed capacity of an allocation-free call    */
} fewbit_status;

/* ------------------------------------------------------------------------- */
/* Tables (Eq. 2: parameters s and y; solved by Eq. 7-9, levels by Eq. 4)     */
/* ------------------------------------------------------------------------- */

/*
 * Optimal `bits`-bit table for `act`: the dynamic programme of Eq. 7 over a
 * uniform grid of 4096 cells on [-8, 8] with the uniform weight of Eq. 10
 * (A = -8, B = 8), prefix integrals as in Eq. 8-9, levels by Eq. 4.  Runs on
 * the CPU (a fraction of a second; results are cached per activation).
 * Returns a HOST handle, or NULL when act/bits are invalid or memory is
 * exhausted.  Release with fewbit_table_destroy().
 */
FEWBIT_API fewbit_table *fewbit_table_create(fewbit_act act, int bits);

/*
 * Same solver with explicit range [A, B] and number of grid cells
 * (2^bits <= n_cells <= 65536).  *out (HOST) receives the handle.
 */
FEWBIT_API fewbit_status fewbit_table_create_ex(fewbit_act act, int bits, double A, double B,
                                                int n_cells, fewbit_table **out);

/*
 * Table from caller-supplied parameters (Listing 1's globally stored s, y):
 * s = 2^bits - 1 boundaries, lev = 2^bits levels, both HOST binary32 arrays,
 * copied.  s must be non-decreasing and free of NaN, else
 * FEWBIT_ERR_INVALID_ARG.
 */
FEWBIT_API fewbit_status fewbit_table_from_arrays(fewbit_act act, int bits, const float *s,
                                                  const float *lev, fewbit_table **out);

/*
 * Folded table for an activation whose derivative is even (caption of Fig. 3:
 * for such an f only the non-negative half-axis needs intervals, which is
 * worth one more bit):
 * 2^bits pieces on [0, B], found by the same dynamic programme on a grid of
 * n_cells cells; the code of x is then #{ j : s[j] < |x| }.  Defined for
 * FEWBIT_SIGMOID and FEWBIT_TANH, otherwise FEWBIT_ERR_UNSUPPORTED.  The
 * objective reported by fewbit_table_get is the error over [-B, B] (twice the
 * half-axis value).  fewbit_fwd / fewbit_bwd take such a table like any other.
 * Suggested: B = 8, n_cells = 2048 (the grid step of the default tables).
 */
FEWBIT_API fewbit_status fewbit_table_create_folded(fewbit_act act, int bits, double B, int n_cells,
                                                    fewbit_table **out);

/*
 * The solver with every choice the paper leaves open (Sec. 3):
 *   A, B           support of the weight w of Eq. 3 (folded: A must be 0);
 *   n_cells        grid of the dynamic programme (Eq. 7);
 *   weight         FEWBIT_WEIGHT_UNIFORM: w = 1 on [A,B] (Eq. 10);
 *                  FEWBIT_WEIGHT_NORMAL: w = standard normal density on [A,B];
 *   finetune_iters 0: boundaries stay on the grid; > 0: at most that many
 *                  gradient steps on the boundaries by Eq. 5, started from the
 *                  DP result (boundaries then leave the grid; a few dozen
 *                  steps reach 2 f'(s_i) = y_i + y_{i-1} to ~1e-7);
 *   folded         as fewbit_table_create_folded.
 * The struct is read during the call only.
 */
#define FEWBIT_WEIGHT_UNIFORM 0
#define FEWBIT_WEIGHT_NORMAL 1
typedef struct fewbit_solver_options {
    double A, B;
    int n_cells;
    int weight;
    int finetune_iters;
    int folded;
} fewbit_solver_options;
FEWBIT_API fewbit_status fewbit_table_create_opt(fewbit_act act, int bits, const fewbit_solver_options *opt,
                                                 fewbit_table **out);

/* fewbit_table_from_arrays with the folded flag (folded != 0: s are boundaries of |x|). */
FEWBIT_API fewbit_status fewbit_table_from_arrays_ex(fewbit_act act, int bits, const float *s,
                                                     const float *lev, int folded, fewbit_table **out);

/* 1 if the table is folded, else 0 (also for NULL). */
FEWBIT_API int fewbit_table_is_folded(const fewbit_table *table);

/* Frees a table; NULL is accepted. */
FEWBIT_API void fewbit_table_destroy(fewbit_table *table);

/*
 * Reads a table back.  Any output pointer (all HOST) may be NULL.
 * s_out needs room for 2^bits - 1 floats, lev_out for 2^bits floats.
 * *objective is the value of Eq. 3 reached by the solver (NaN for a table
 * made by fewbit_table_from_arrays).
 */
FEWBIT_API fewbit_status fewbit_table_get(const fewbit_table *table, int *act, int *bits,
                                          float *s_out, float *lev_out, double *objective);

/* Bytes of the saved tensor for n elements: 4 * ceil(n * bits / 32); 0 if bits is invalid. */
FEWBIT_API size_t fewbit_packed_bytes(size_t n, int bits);

/* ------------------------------------------------------------------------- */
/* Hot path on DEVICE buffers (Listing 1)                                     */
/* ------------------------------------------------------------------------- */

/*
 * Forward half, one kernel launch on `stream` (a cudaStream_t passed as
 * void*; NULL = the legacy default stream), asynchronous:
 *     y[e]      = f(x[e])                 exact activation, rounded to dtype
 *     code[e]   = #{ j : s[j] < x[e] }    Eq. 2 / the sorted search of Listing 1
 *     packed    = the codes as a `bits`-bit stream (layout above)
 * x, y: DEVICE, n elements of `dtype`, 16-byte aligned; y == x (exact alias)
 * is allowed, any other overlap is undefined.  packed: DEVICE,
 * fewbit_packed_bytes(n, bits) bytes, 4-byte aligned; nothing beyond those
 * bytes is written.  n == 0 returns FEWBIT_OK without a launch.
 * (Alignment beyond the rule only widens the accesses: binary32 buffers that
 * are all 32-byte aligned move 256 bits per lane instead of 2 x 128, packed
 * words that are 8-byte (2 bits) or 16-byte (4 bits) aligned are stored as one
 * vector.  Any view of a tensor that starts on a multiple of 32 elements
 * therefore satisfies the rule for x, y and packed at once.)
 * Errors: FEWBIT_ERR_INVALID_ARG (NULL table or buffer, bad dtype),
 * FEWBIT_ERR_ALIGNMENT, FEWBIT_ERR_CUDA (launch failed).
 * The interval search has several equivalent kernel variants (binary search,
 * two-at-a-time bfloat16 search, shared-memory code table) chosen from the
 * activation, bits, dtype and n by measured thresholds; all give identical
 * codes.  The code-table variants (3-4 bits, from a few waves of resident warps
 * on, earlier the costlier f is) distribute their work through a set of
 * counters in a
 * file-scope device array (16 sets per device; nothing is allocated, but the
 * first such call on a device creates up to 16 CUDA events, and each call
 * records one after its kernel).  While `stream` is being captured,
 * or when all sets are in use by other streams, the kernel falls back to a
 * static partition: same results, ~10 % slower.  Small tensors (fewer 1024-
 * element blocks than resident warps) are processed a 256-element tile per
 * warp, which puts four times as many warps to work.  The choices can be overridden
 * for testing and tuning with fewbit_set_option (below); the library reads no
 * environment variable.
 * Both device kernels are launched with programmatic stream serialization:
 * their CTAs may be scheduled while the previous kernel of `stream` drains,
 * and wait there for its completion before they touch memory, so stream order
 * holds as usual (FEWBIT_OPT_PDL = 0 launches them the ordinary way).
 */
FEWBIT_API fewbit_status fewbit_fwd(const fewbit_table *table, const void *x, void *y,
                                    uint32_t *packed, size_t n, fewbit_dtype dtype, void *stream);

/*
 * Forward half with a bias in front of the activation (an extension; Listing 1
 * starts at the activation's input): for x of shape rows x cols, row-major,
 *   z[r][c] = x[r][c] + bias[c]     the exact sum, rounded once to `dtype`,
 *   y = f(z),  code = #{ j : s_j < z }   exactly as fewbit_fwd would on z.
 * The backward half needs nothing new: grad_in = fewbit_bwd(packed, grad_out)
 * is the gradient with respect to x, and its column sums are the gradient with
 * respect to the bias.
 *
 * x, y: DEVICE, rows * cols elements; bias: DEVICE, cols elements of `dtype`,
 * 16-byte aligned like x and y; packed: DEVICE, fewbit_packed_bytes(rows * cols,
 * bits) bytes, 4-byte aligned.  y may alias x exactly.  cols must be a multiple
 * of 8 below 2^32 (a lane's 8 consecutive elements then never straddle a row
 * end) and the table must not be a folded one, else FEWBIT_ERR_UNSUPPORTED;
 * rows * cols == 0 is a no-op.  Asynchronous on `stream`, allocates nothing; same kernel
 * variants and launch rules as fewbit_fwd.
 * Errors: INVALID_ARG (NULL, bad dtype, rows * cols overflows), UNSUPPORTED,
 * ALIGNMENT, CUDA.
 */
FEWBIT_API fewbit_status fewbit_fwd_bias(const fewbit_table *table, const void *x, const void *bias,
                                         void *y, uint32_t *packed, size_t rows, size_t cols,
                                         fewbit_dtype dtype, void *stream);

/*
 * Backward half, one kernel launch on `stream`, asynchronous:
 *     grad_in[e] = round_dtype( (float)grad_out[e] * lev[code[e]] )
 * (Eq. 1 with f' replaced by q of Eq. 2; one binary32 multiply, one rounding).
 * packed: DEVICE, as written by fewbit_fwd with a table of the same `bits`,
 * 4-byte aligned.  grad_out, grad_in: DEVICE, n elements of `dtype`,
 * 16-byte aligned; grad_in == grad_out allowed.  Errors as fewbit_fwd.
 */
FEWBIT_API fewbit_status fewbit_bwd(const fewbit_table *table, const uint32_t *packed,
                                    const void *grad_out, void *grad_in, size_t n,
                                    fewbit_dtype dtype, void *stream);

/* ------------------------------------------------------------------------- */
/* Operators next to the activation in a transformer's training step          */
/*                                                                            */
/* The activations keep 1-4 bits per element; what else a training step keeps */
/* is attention's probabilities, the copies around the head norm and the      */
/* rotation, and the optimizer's moments.  The entry points below recompute   */
/* the first, fuse the second and hold the third in 8 bits.  (The paper has   */
/* no counterpart for any of them.)  Same conventions as above: asynchronous  */
/* on `stream`, no allocation, no synchronisation, a status for every error   */
/* that the host can see.                                                     */
/* ------------------------------------------------------------------------- */

/*
 * A DEVICE tensor of heads: element (b, i, h, e) of a (batch, length, heads,
 * head_dim) tensor lies at data[b * batch_stride + i * row_stride +
 * h * head_stride + e].  Strides count elements and may be anything that
 * keeps every head inside the caller's buffer (a view of a fused projection,
 * a transposed layout); the elements of one head are contiguous.
 */
typedef struct fewbit_heads {
    void *data;
    int64_t batch_stride, row_stride, head_stride;
} fewbit_heads;

/*
 * RMS norm of every query and key head, then the position rotation, in one
 * pass.  For a head x of head_dim = D elements at position p:
 *     u[e] = x[e] * rsqrt(mean(x^2) + eps) * weight[e]           in binary32
 *     (y[a], y[b]) = (u[a] c - u[b] s, u[a] s + u[b] c)          for each rotated pair j,
 * with c = cos[p * rotary_dim/2 + j], s = sin[...], and pair j being
 * (j, j + rotary_dim/2), or (2j, 2j+1) when `interleaved`; elements from
 * rotary_dim on are not rotated.  y is rounded once to `dtype`.
 *
 *   batch, length   tokens (batch * length < 2^31)
 *   heads, kv_heads query and key heads, up to 2^15 (0 allowed: that tensor is not touched)
 *   head_dim        even, 2 .. 256;   rotary_dim  even, 0 .. head_dim
 *   positions       DEVICE, batch * length int32 (positions_are_64bit: int64),
 *                   or NULL: token i of a sequence has position i
 *   table_rows      rows of cos and sin (DEVICE, binary32, contiguous).  A
 *                   position outside [0, table_rows) makes its token's heads
 *                   NaN; nothing outside the tables is read.  Without
 *                   `positions`, table_rows >= length is required.
 *   q_weight, k_weight  DEVICE, head_dim binary32 values, or NULL for ones.
 * The struct is HOST memory, read during the call only.
 * Buffers need the alignment of their element type; 16-byte aligned heads (and
 * pairs that keep whole 16-byte pieces together) move in wider pieces.
 */
typedef struct fewbit_qk_shape {
    int64_t batch, length;
    int heads, kv_heads, head_dim, rotary_dim, interleaved;
    const void *positions;
    int positions_are_64bit;
    int64_t table_rows;
    const float *cos, *sin;
    const float *q_weight, *k_weight;
    float eps;
    fewbit_dtype dtype;
} fewbit_qk_shape;

/*
 * q, k -> q_out, k_out; one launch.  An output may alias its input exactly.
 * Errors: INVALID_ARG (NULL, sizes, eps < 0 or NaN), UNSUPPORTED (head_dim > 256),
 * TOO_LARGE, ALIGNMENT, CUDA.
 */
FEWBIT_API fewbit_status fewbit_qk_norm_rope_fwd(const fewbit_qk_shape *shape, const fewbit_heads *q, const fewbit_heads *k,
                                                 const fewbit_heads *q_out, const fewbit_heads *k_out, void *stream);

/* Bytes of `workspace` for the backward pass with weight gradients; 0 without a device or for a bad shape. */
FEWBIT_API size_t fewbit_qk_norm_rope_workspace_bytes(const fewbit_qk_shape *shape);

/*
 * Gradients of fewbit_qk_norm_rope_fwd: (grad_q_out, grad_k_out) and the
 * forward pass's inputs q, k -> grad_q, grad_k (may alias grad_*_out exactly),
 * and the weights' gradients, head_dim binary32 values each (NULL: not wanted).
 * The norm's factor is recomputed.  With weight gradients: `workspace` (DEVICE,
 * 16-byte aligned, fewbit_qk_norm_rope_workspace_bytes long), and a second
 * launch that adds up the partial sums in a fixed order (the same inputs give
 * the same bits).  Errors as above, ALLOC (workspace too small).
 */
FEWBIT_API fewbit_status fewbit_qk_norm_rope_bwd(const fewbit_qk_shape *shape, const fewbit_heads *grad_q_out,
                                                 const fewbit_heads *grad_k_out, const fewbit_heads *q, const fewbit_heads *k,
                                                 const fewbit_heads *grad_q, const fewbit_heads *grad_k,
                                                 float *grad_q_weight, float *grad_k_weight,
                                                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * Attention, out = softmax(scale * q k^T + mask) v for each head, and its
 * gradients.  The probabilities are never stored: the forward pass keeps the
 * logarithm of each row's sum (lse, binary32, natural logarithm), from which
 * the backward pass recomputes them.
 *
 *   dtype           FEWBIT_BF16 or FEWBIT_F16 (products with binary32 sums on
 *                   the tensor cores; the probabilities and their gradients
 *                   are rounded to `dtype` as operands of the second products)
 *   heads, kv_heads query head h reads key head h / (heads / kv_heads); without query heads
 *                   a call reads and writes nothing
 *   head_dim        a multiple of 8, 8 .. 128
 *   causal          row i of a sequence sees keys j <= i + k_len - q_len (the
 *                   last row sees every key)
 *   q_offsets, k_offsets   NULL: `batch` sequences of q_len rows and k_len keys.
 *                   Otherwise DEVICE int32 arrays of batch + 1 non-decreasing
 *                   values: sequence b is rows [q_offsets[b], q_offsets[b+1])
 *                   of q and keys [k_offsets[b], k_offsets[b+1]) of k and v,
 *                   in tensors of q_rows and k_rows rows (batch_stride is not
 *                   used); q_len and k_len are then upper bounds of the
 *                   sequences' lengths.  Offsets are clamped to [0, q_rows] /
 *                   [0, k_rows], lengths to [0, q_len] / [0, k_len].  Rows in
 *                   front of the first and behind the last sequence, and those
 *                   of a sequence past its clamped length, belong to none: they
 *                   get zeros (lse: -inf).
 *   scale           finite, > 0
 * lse: (batch, heads, q_len), or (heads, q_rows) for packed sequences.
 * A row that sees no key has out = 0, lse = -inf and zero gradients.
 * Pointers must be 16-byte aligned, strides multiples of 8 elements (of
 * dimensions longer than 1).  Keys past the end of a sequence are not part of
 * any sum, whatever the memory there holds.  A non-finite value inside a
 * sequence's k or v can spread to rows that the causal mask hides it from.
 * The backward pass recomputes a row's probabilities from its lse, whose rounding to
 * 32 bits they feel: by about |lse| 2^-23 of themselves.  (Biased scores: see there.)
 */
typedef struct fewbit_attention_shape {
    int batch, heads, kv_heads, head_dim;
    int64_t q_len, k_len;
    int64_t q_rows, k_rows;
    const int32_t *q_offsets, *k_offsets;
    int causal;
    float scale;
    fewbit_dtype dtype;
} fewbit_attention_shape;

/* Errors: INVALID_ARG, UNSUPPORTED (head_dim, dtype), TOO_LARGE, ALIGNMENT, CUDA. */
FEWBIT_API fewbit_status fewbit_attention_fwd(const fewbit_attention_shape *shape, const fewbit_heads *q, const fewbit_heads *k,
                                              const fewbit_heads *v, const fewbit_heads *out, float *lse, void *stream);

/* Bytes of `workspace` for the backward pass (1 KB for each 128 rows of each head); 0 for a bad shape. */
FEWBIT_API size_t fewbit_attention_workspace_bytes(const fewbit_attention_shape *shape);

/*
 * (grad_out; q, k, v, out, lse of the forward pass) -> grad_q, grad_k, grad_v,
 * every element of every sequence written.  The gradients of a key head that
 * several query heads share are summed in binary32, in a fixed order: the same
 * inputs give the same bits.  Two launches.  workspace: DEVICE, 16-byte aligned.
 */
FEWBIT_API fewbit_status fewbit_attention_bwd(const fewbit_attention_shape *shape, const fewbit_heads *grad_out,
                                              const fewbit_heads *q, const fewbit_heads *k, const fewbit_heads *v,
                                              const fewbit_heads *out, const float *lse,
                                              const fewbit_heads *grad_q, const fewbit_heads *grad_k, const fewbit_heads *grad_v,
                                              void *workspace, size_t workspace_bytes, void *stream);

/*
 * What comes between attention's products and its softmax.  With the distance
 *     d = j - i - (k_len - q_len)
 * of key j from row i (both counted within their sequence; the last row and
 * the last key are level), the score of a visible key is
 *     z = scale q.k;   cap > 0: z = cap tanh(z / cap);
 *     z -= slopes[h] |d|;   z += distance_bias[h][clamp(d, -R, R) + R]
 * (each where given), and row i of a sequence sees key j if
 *     not causal, or d <= 0, or j < prefix_lens[b];   and
 *     q_documents[i] == k_documents[j]     (where given)
 *
 *   cap             0: none; else 2^-60 .. 2^60
 *   slopes          DEVICE, a binary32 value for each query head, or NULL.  A score that
 *                   they bring below -2.3e38 is held as that, or hides its key.
 *   distance_bias   DEVICE, heads x (2 R + 1) binary32 values, R = max_distance,
 *                   1 .. FEWBIT_MAX_DISTANCE, or NULL; up to 65535 heads.  -inf hides the key; so does a
 *                   finite value below -2.3e38 (the scores are held in units of ln 2).
 *                   Scores are rounded to 32 bits: with a bias of -1e9 nothing else is left of
 *                   one.  Rows whose lse is beyond +-2839, by biases or slopes, take the
 *                   backward pass much longer (some 15 times).
 *   prefix_lens     DEVICE, int32 for each sequence, or NULL; causal attention only
 *   q_documents, k_documents  DEVICE int32 (batch, q_len) and (batch, k_len),
 *                   contiguous, or (q_rows) and (k_rows) for packed sequences;
 *                   both or neither.  Any numbers; where they do not fall along a
 *                   sequence, tiles that no document of theirs shares are skipped.
 * The struct is HOST memory, read during the call only; buffers are 4-byte aligned.  What is said about rows that see nothing and about
 * non-finite values in fewbit_attention_shape holds for every key that a mask hides.
 */
#define FEWBIT_MAX_DISTANCE 4096
typedef struct fewbit_attention_scores {
    float cap;
    const float *slopes;
    const float *distance_bias;
    int max_distance;
    const int32_t *prefix_lens;
    const int32_t *q_documents, *k_documents;
} fewbit_attention_scores;

/* fewbit_attention_fwd with these scores (NULL: the plain ones).  Errors as there. */
FEWBIT_API fewbit_status fewbit_attention_scores_fwd(const fewbit_attention_shape *shape, const fewbit_attention_scores *scores, const fewbit_heads *q,
                                                     const fewbit_heads *k, const fewbit_heads *v, const fewbit_heads *out, float *lse, void *stream);

/*
 * Bytes of `workspace` for the backward pass; 0 for a bad shape.  bias_gradient: with the gradient of distance_bias, which
 * takes 4 KB for each pair of a row tile and a key tile (128 x 128) within max_distance of each other, and each head
 * (4 or so such pairs for a key tile with a max_distance of 128), and 512 bytes for each row tile and head.
 */
FEWBIT_API size_t fewbit_attention_scores_workspace_bytes(const fewbit_attention_shape *shape, const fewbit_attention_scores *scores, int bias_gradient);

/*
 * fewbit_attention_bwd with these scores.  grad_distance_bias: heads x (2 R + 1) binary32 values, or NULL: the gradients of the
 * scores, summed over the batch, the rows and the keys of each distance in a fixed order (one launch more).
 */
FEWBIT_API fewbit_status fewbit_attention_scores_bwd(const fewbit_attention_shape *shape, const fewbit_attention_scores *scores, const fewbit_heads *grad_out,
                                                     const fewbit_heads *q, const fewbit_heads *k, const fewbit_heads *v, const fewbit_heads *out,
                                                     const float *lse, const fewbit_heads *grad_q, const fewbit_heads *grad_k,
                                                     const fewbit_heads *grad_v, float *grad_distance_bias, void *workspace,
                                                     size_t workspace_bytes, void *stream);

/*
 * A learned bias of relative positions by buckets (Raffel et al., Exploring the limits of transfer learning, 2020), spread
 * over the distances d = -R .. R for fewbit_attention_scores: distance_bias[h][d + R] = table[bucket(d)][h].  With
 * B = buckets (half of them if bidirectional), n = |d| if bidirectional, else max(-d, 0), and m = B / 2 rounded down:
 *     n < m:  bucket = n
 *     else    bucket = min(B - 1, m + floor(log(n / m) / log(R / m) * (B - m)))     with the floor of the exact value
 * and B is added for d > 0 if bidirectional.
 *   table           DEVICE, buckets x heads elements of `dtype`, contiguous
 *   buckets         2 .. 1024, bidirectional: even, from 4
 *   max_distance    R: larger than m, up to FEWBIT_MAX_DISTANCE
 * Errors: INVALID_ARG, TOO_LARGE (heads above 65535), ALIGNMENT, CUDA.
 */
FEWBIT_API fewbit_status fewbit_relative_bias_fwd(const void *table, int buckets, int heads, int max_distance, int bidirectional,
                                                  fewbit_dtype dtype, float *distance_bias, void *stream);

/* grad_table[b][h] (of `dtype`) = the sum of grad_distance_bias[h] over the distances of bucket b, in a fixed order. */
FEWBIT_API fewbit_status fewbit_relative_bias_bwd(const float *grad_distance_bias, int buckets, int heads, int max_distance, int bidirectional,
                                                  fewbit_dtype dtype, void *grad_table, void *stream);

/*
 * Diagnostic: *count (HOST) receives how often a wait inside the attention kernels gave up on the current
 * device since the library was loaded (each wait is limited to two seconds; the results that such a launch could
 * not finish are NaN).  Always 0 unless the device or the program is broken.  Synchronises the device.
 */
FEWBIT_API fewbit_status fewbit_attention_timeout_count(uint64_t *count);

/*
 * One AdamW step over many tensors.  For every element, in binary32:
 *     g  = grad * grad_scale
 *     m  = beta1 m + (1 - beta1) g
 *     v  = beta2 v + (1 - beta2) g^2
 *     p  = p (1 - lr weight_decay) - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)
 * With a master copy, p is read from and written to `master` (binary32) and
 * `param` receives it rounded to `dtype`; without one, `param` is read.
 *
 * Moments of 8 bits (state_bits = 8): a tensor is cut into blocks of 256
 * consecutive elements.  exp_avg holds m and exp_avg_sq holds sqrt(v), both as
 * float8 codes (e4m3: sign, 4 bits of exponent, 3 of mantissa; 448 is the
 * largest), one byte an element, with one binary32 scale a block: value =
 * code * scale, scale = (largest magnitude of the block) / 448.  The new values
 * are rounded stochastically: up with the probability of what is cut off, so
 * that a moment that changes by less than a step still changes on average.
 * Each product and sum of the moments is rounded to binary32 by itself, so the
 * codes follow from the inputs and the seed alone.
 * The 16 + 16 random bits of an element are a hash of `seed` and of its place
 * in the call (tensors in order, each taking a whole number of blocks):
 * place * 0x9E3779B1 + seed is what is hashed, so seeds that differ by a small
 * multiple of that constant give the same bits a few places apart.  Give every
 * step a seed of its own that is no count but a hash of one.  A positive second moment never becomes zero.  A
 * block with a non-finite value gets a NaN scale: it reads back as NaN.  A
 * block whose largest magnitude is below 2^-126 reads back as zero.
 * Moments of 32 bits: exp_avg = m, exp_avg_sq = v, binary32; no scales.
 *
 * tensors: HOST array of `count` descriptions of DEVICE buffers; grads: HOST
 * array of `count` DEVICE pointers (n elements of `dtype` each).  Both are read
 * during the call only.  Any n, zero included.  Buffers need the alignment of
 * their element type; tensors whose binary32 buffers are 32-byte aligned, 16-bit
 * ones 16-byte and codes 8-byte move in wider pieces.  The tensors of
 * a call must not overlap.  One launch for up to 400 tensors.
 * grad_scale_device: DEVICE binary32 value that multiplies every gradient (1 /
 * the loss scale, a clipping factor), or NULL.
 */
#define FEWBIT_ADAMW_BLOCK 256
typedef struct fewbit_adamw_tensor {
    void *param;
    void *exp_avg, *exp_avg_sq;
    float *exp_avg_scale, *exp_avg_sq_scale;   /* state_bits 8: ceil(n / 256) values each; else NULL */
    float *master;                             /* NULL: none */
    uint64_t n;
} fewbit_adamw_tensor;

typedef struct fewbit_adamw_options {
    double lr, beta1, beta2, eps, weight_decay;
    int64_t step;                              /* 1 for the first step */
    const float *grad_scale_device;
    uint32_t seed;
    int state_bits;                            /* 8 or 32 */
    fewbit_dtype dtype;                        /* of param and grad */
} fewbit_adamw_options;

/*
 * Errors: INVALID_ARG (NULL, step < 1, a beta outside [0, 1), eps < 0, lr or weight_decay
 * negative or not finite, some tensors with a master copy and some without,
 * a master copy with FEWBIT_F32), TOO_LARGE (a tensor of more than 2^38 elements), ALIGNMENT, CUDA.
 */
FEWBIT_API fewbit_status fewbit_adamw_step(const fewbit_adamw_tensor *tensors, const void *const *grads, int count,
                                           const fewbit_adamw_options *options, void *stream);

/*
 * Dropout whose mask is drawn from a counter wherever it is needed and never
 * stored.  Element e (counted over the whole tensor) takes word e % 4 of the
 * Philox4x32-10 block (Salmon et al., 2011) of the counter
 * (e / 4 mod 2^32, e / 2^34, place, 0) under the key (seed mod 2^32, seed / 2^32);
 * it is kept where that word is at least round(p * 2^32), and multiplied by
 * 1 / (1 - p).
 *   p            0 <= p < 1; 0: nothing is drawn
 *   seed         of the step;  seed_device  DEVICE (8-byte aligned) or NULL: one
 *                value that is added to it, so that a captured graph draws anew
 *                each time.  The backward pass needs the forward pass's values.
 *   place        tells one use of a seed from another (a layer's number)
 */
typedef struct fewbit_dropout_options {
    double p;
    uint64_t seed;
    const int64_t *seed_device;
    uint32_t place;
} fewbit_dropout_options;

/*
 * y = residual + dropout(x), in binary32, rounded once.  x, residual (NULL:
 * none), y: DEVICE, n elements of `dtype`, aligned to the element type (16-byte
 * aligned ones move in wider pieces); y may alias x or residual exactly.
 * Errors: INVALID_ARG, TOO_LARGE, ALIGNMENT, CUDA.
 */
FEWBIT_API fewbit_status fewbit_dropout_fwd(const void *x, const void *residual, void *y, size_t n, fewbit_dtype dtype,
                                            const fewbit_dropout_options *options, void *stream);

/* grad_in = grad_out where x was kept, times 1 / (1 - p); else 0.  (The residual's gradient is grad_out.) */
FEWBIT_API fewbit_status fewbit_dropout_bwd(const void *grad_out, void *grad_in, size_t n, fewbit_dtype dtype,
                                            const fewbit_dropout_options *options, void *stream);

/*
 * A branch's addition to the residual stream and the RMS norm of the sum:
 *     h = residual + dropout(x),   y = h / sqrt(mean(h^2) + eps) * weight
 * for each row of `width` elements, in binary32; h is rounded when it is stored,
 * the norm takes it as it was.
 *   rows, width   of contiguous tensors; width up to 16384
 *   weight        DEVICE, width binary32 values, or NULL for ones
 *   dropout       of x; an element's number is row * width + column
 * The struct is HOST memory, read during the call only.
 */
typedef struct fewbit_norm_shape {
    int64_t rows, width;
    const float *weight;
    float eps;
    fewbit_dtype dtype;
    fewbit_dropout_options dropout;
} fewbit_norm_shape;

/*
 * residual: NULL for none.  h: NULL if it is not wanted.  y_bits 0: y has `dtype`
 * and y_scale is NULL.  y_bits 8: y holds e4m3 codes (one byte each), y_scale
 * one binary32 value a row: y = code * scale, scale = (largest magnitude of the
 * row) / 448, codes rounded to nearest; a row with a non-finite value gets a NaN
 * scale, one whose largest magnitude is below 2^-117 reads back as zero.
 * An output may alias an input of the same type exactly.  One launch.
 * Errors: INVALID_ARG (NULL, sizes, eps < 0 or NaN, p), UNSUPPORTED (width),
 * TOO_LARGE (rows above 2^31 - 1), ALIGNMENT, CUDA.
 */
FEWBIT_API fewbit_status fewbit_add_rms_norm_fwd(const fewbit_norm_shape *shape, const void *x, const void *residual, void *h, void *y,
                                                 float *y_scale, int y_bits, void *stream);

/* Bytes of `workspace` for the backward pass with a weight gradient; 0 without a device or for a bad shape. */
FEWBIT_API size_t fewbit_add_rms_norm_workspace_bytes(const fewbit_norm_shape *shape);

/*
 * Gradients of fewbit_add_rms_norm_fwd from grad_y, the gradient grad_h that
 * reaches h from elsewhere (NULL: none) and h as it was stored:
 * grad_residual (the sum's) and grad_x (the same through the dropout), either
 * may be NULL; grad_weight: width binary32 values, or NULL.  With it:
 * `workspace` (DEVICE, 16-byte aligned), and a second launch that adds up the
 * partial sums in a fixed order.  (The rounding of 8-bit results has no gradient
 * of its own: grad_y passes it as it is.)  An output may alias an input exactly.
 * Errors as above, ALLOC (workspace too small).
 */
FEWBIT_API fewbit_status fewbit_add_rms_norm_bwd(const fewbit_norm_shape *shape, const void *grad_y, const void *grad_h, const void *h,
                                                 void *grad_x, void *grad_residual, float *grad_weight, void *workspace,
                                                 size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------- */
/* Hot path on HOST buffers                                                   */
/* ------------------------------------------------------------------------- */

/*
 * Device bytes fewbit_fwd_host / fewbit_bwd_host need in `workspace` to
 * stream `chunk_elems` elements per pipeline stage (rounded up to a multiple
 * of 1024 elements; the pipeline has 3 stages).
 */
FEWBIT_API size_t fewbit_host_workspace_bytes(size_t chunk_elems, fewbit_dtype dtype, int bits);

/*
 * Forward half on HOST buffers: x_host -> (y_host, packed_host), same
 * results as fewbit_fwd.  The tensor is cut into chunks; each chunk is copied
 * to `workspace` (DEVICE, caller-owned, 256-byte aligned, `workspace_bytes`
 * long), run through the forward kernel and copied back, with the copies of
 * neighbouring chunks overlapping the kernel on three internal streams (created
 * by the first call on a device and kept for later calls; concurrent calls get
 * triples of their own).  Blocks until the results are in host memory.  Page-locked host buffers are
 * needed for the copies to overlap; pageable ones work, slower.
 * FEWBIT_ERR_ALLOC if the workspace cannot hold one 1024-element chunk.
 * Calls on the same device that overlap in time must use disjoint workspaces.
 */
FEWBIT_API fewbit_status fewbit_fwd_host(const fewbit_table *table, const void *x_host,
                                         void *y_host, uint32_t *packed_host, size_t n,
                                         fewbit_dtype dtype, void *workspace,
                                         size_t workspace_bytes);

/* Backward half on HOST buffers: (packed_host, grad_out_host) -> grad_in_host; see fewbit_fwd_host. */
FEWBIT_API fewbit_status fewbit_bwd_host(const fewbit_table *table, const uint32_t *packed_host,
                                         const void *grad_out_host, void *grad_in_host, size_t n,
                                         fewbit_dtype dtype, void *workspace,
                                         size_t workspace_bytes);

/*
 * Forward half on HOST buffers WITHOUT any device allocation -- not even one
 * made by the caller.  (The paper has no counterpart: this is a packaging
 * variant of fewbit_fwd_host, same kernel, same results.)
 *
 * Who needs it: code that must not, or cannot, call cudaMalloc at the point
 * where it wants the forward pass -- a plug-in running inside a host
 * application whose memory pool already owns the whole device, a process held
 * to a fixed device-memory budget, or a latency-sensitive loop that cannot
 * afford the device-wide synchronisation an allocation may imply.  For them
 * the staging area that fewbit_fwd_host expects as `workspace` is a fixed
 * array inside the library image: FEWBIT_STATIC_MAX_ELEMS elements of room
 * (about 2.1 MiB of device memory), held by every GPU on which the library is
 * loaded until the process exits.
 *
 * x_host, y_host, packed_host: HOST buffers as in fewbit_fwd_host.  `stream`:
 * the copies and the kernel are enqueued on it and it is synchronised before
 * the call returns.  n > fewbit_static_max_elements() is rejected with
 * FEWBIT_ERR_TOO_LARGE (split the tensor on a multiple of 1024 elements and
 * call once per piece, or use fewbit_fwd_host).  The call makes no
 * cudaMalloc / cudaFree and, with the default options, creates no stream or
 * event (at this capacity the kernel variants that lease work counters are
 * never the size-based choice).
 *
 * The first call on each device looks up the device address of the array
 * (cudaGetSymbolAddress, with that device current); make that first call
 * outside of any stream capture.  Under CUDA's lazy module loading that same
 * first call is what loads the part of the library holding the array, i.e. it
 * is the moment the ~2.1 MiB are taken from the device: a caller whose pool
 * later claims all device memory should make one (small) call at start-up,
 * before the pool does, or run with CUDA_MODULE_LOADING=EAGER.  The address is
 * cached per device for the life of the process; it does not survive a
 * cudaDeviceReset.  All calls on a device share the one array:
 * it still holds the previous call's data (harmless -- every byte that is
 * read is written first, so nothing needs clearing), and two calls whose GPU
 * work overlaps in time, from different threads or streams, race on it.
 * Serialise them.
 */
#define FEWBIT_STATIC_MAX_ELEMS 262144
FEWBIT_API size_t fewbit_static_max_elements(void);
FEWBIT_API fewbit_status fewbit_fwd_host_static(const fewbit_table *table, const void *x_host,
                                                void *y_host, uint32_t *packed_host, size_t n,
                                                fewbit_dtype dtype, void *stream);

/* ------------------------------------------------------------------------- */
/* Options and diagnostics                                                    */
/* ------------------------------------------------------------------------- */

/*
 * Process-wide switches for testing and tuning (the paper has no counterpart;
 * every setting gives the same results, only the kernel variant or the launch
 * geometry changes).  Stored in atomics: may be set from any thread at any
 * time and apply to the launches that follow.
 *   FEWBIT_OPT_FWD_TABLE    0 size-based choice (default), 1 the shared-memory
 *                           code-table variant whenever the table has one,
 *                           2 never;
 *   FEWBIT_OPT_FWD_QUEUE    0 lease work counters when possible (default),
 *                           1 always the static partition;
 *   FEWBIT_OPT_FWD_ITERS    0 size-based (default), 1..64 warp-blocks per warp;
 *   FEWBIT_OPT_FWD_WARPS    0 default, 1..16 warps per CTA of the variants
 *                           without a code table (values beyond what the kernel
 *                           is compiled for are ignored);
 *   FEWBIT_OPT_PDL          1 programmatic dependent launch (default), 0 off;
 *   FEWBIT_OPT_COUNT_TAILS  1: every warp that runs the forward kernel's
 *                           ragged-tail path adds one to a device counter read
 *                           by fewbit_tail_warp_count (default 0: no counting);
 *   FEWBIT_OPT_FWD_TILE     0 by size (default): small tensors are processed a
 *                           256-element tile per warp instead of a 1024-element
 *                           block, 1 always (variants without a code table),
 *                           2 never.
 * fewbit_set_option returns FEWBIT_ERR_INVALID_ARG for an unknown option or a
 * value outside its range; fewbit_get_option returns -1 for an unknown option.
 */
typedef enum fewbit_option {
    FEWBIT_OPT_FWD_TABLE = 0,
    FEWBIT_OPT_FWD_QUEUE = 1,
    FEWBIT_OPT_FWD_ITERS = 2,
    FEWBIT_OPT_FWD_WARPS = 3,
    FEWBIT_OPT_PDL = 4,
    FEWBIT_OPT_COUNT_TAILS = 5,
    FEWBIT_OPT_FWD_TILE = 6
} fewbit_option;
FEWBIT_API fewbit_status fewbit_set_option(fewbit_option option, int value);
FEWBIT_API int fewbit_get_option(fewbit_option option);

/*
 * Diagnostic: *count (HOST) receives how many warps have run the ragged-tail
 * path of the forward kernel on the current device while FEWBIT_OPT_COUNT_TAILS
 * was 1 (exactly one per launch whose n is not a multiple of 1024 -- of 256 for
 * a launch in tile mode); reset != 0
 * clears the counter afterwards.  Synchronises the device.
 */
FEWBIT_API fewbit_status fewbit_tail_warp_count(uint64_t *count, int reset);

/* Static, never NULL. */
FEWBIT_API const char *fewbit_status_string(fewbit_status status);

/* The cudaError_t (as int) behind the calling thread's last FEWBIT_ERR_CUDA; 0 if none. */
FEWBIT_API int fewbit_last_cuda_error(void);

/* Kernels launched by this library in this process so far (all threads). */
FEWBIT_API uint64_t fewbit_launch_count(void);

/*
 * Accuracy scan of the binary32 evaluation of an activation (the arithmetic fewbit_fwd uses for
 * FEWBIT_F32) against the same function evaluated in binary64 and rounded once, for the `count`
 * input bit patterns first_pattern, first_pattern + 1, ... (first_pattern + count <= 2^32; the
 * whole range takes a few seconds).  Non-finite inputs are skipped.  The paper has no counterpart:
 * this is a self-check of the library's arithmetic (Sec. 2 only names the functions).
 *
 * result_device: DEVICE pointer to 5 uint64 words, 8-byte aligned, owned by the caller; the call
 * clears them on `stream`, then the kernel fills them:
 *   [0], [1], [2]  inputs whose result is 0, 1, 2 ulp from the rounded binary64 value;
 *   [3]            inputs further away (a NaN on one side only counts here);
 *   [4]            (largest distance, capped at 2^31 - 1) << 32 | an input pattern that has it.
 * Asynchronous on `stream`; read the words after synchronising.
 * Errors: INVALID_ARG (bad enum, NULL, range beyond 2^32), ALIGNMENT, CUDA.
 */
FEWBIT_API fewbit_status fewbit_f32_activation_scan(fewbit_act act, uint64_t first_pattern,
                                                    uint64_t count, uint64_t *result_device,
                                                    void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FEWBIT_H_ */
