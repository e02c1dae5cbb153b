/*
 * dash.h -- C ABI of libdash: garbling and evaluating arithmetic garbled circuits over CRT
 * residues on one AMD MI355X (gfx950), after "Dash" (arXiv 2302.06361).
 *
 * The four scheme algorithms of the paper (Sec. Garbled Circuits: Gb, En, Ev, De) map to
 *   Gb : dash_input_labels + dash_garble_layer per layer      En : dash_encode
 *   Ev : dash_eval_layer per layer                            De : dash_decode
 *
 * Conventions that hold for every entry point
 *   - "device" pointers are HIP device memory on the context's GPU, owned by the caller;
 *     "host" pointers are ordinary host memory.  The library owns only the dash_ctx.
 *   - Calls enqueue work on the given hipStream_t (passed as void*, NULL = default stream) and
 *     return without synchronising; no call allocates or frees device memory except
 *     dash_ctx_create / dash_ctx_destroy.
 *   - Return value: 0 = DASH_OK, negative = error (dash_strerror).  Nothing is launched when an
 *     argument check fails.  A forged output label is data (valid[] of dash_decode), not an error.
 *
 * LabelTensor layout (the paper's LabelTensor, Sec. LabelTensors, re-laid out for 64-wide
 * wavefronts): one tensor per CRT residue; the lambda digits of a label (one byte each, values
 * in [0, p)) are cut into chunks of 16 digits and the tensor is stored chunk-major,
 *      digit j of element e  at  data + (j / 16) * chunk_stride + 16 * e + (j % 16),
 * so consecutive elements of one chunk are consecutive 16-byte words (one dwordx4 per lane,
 * fully coalesced) and, inside a batch element, consecutive features are consecutive words (the
 * K-contiguous operand of the int8 MFMA contraction).  Digits past lambda in the last chunk are
 * zero.  Elements are ordered [batch][y][x][channel].
 *
 * Ciphertext tables (Sec. Arithmetic Garbled Circuits, projection gates: p ciphertexts per gate,
 * ordered by the colour = digit 0 of the input label): a batch of E gates Z_p -> Z_q is one
 * segment [gate][row 0..p-1][pitch_q] with pitch_q = 4 * ceil(lambda_q / 4) bytes, pad bytes
 * zero.  A layer's table buffer is the concatenation of its segments in slot order; segment s
 * starts at E * (bytes per element of the segments before s).
 */
#ifndef DASH_H
#define DASH_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DASH_MAX_PRIMES 16
#define DASH_MAX_DIGITS 16

enum {
    DASH_OK = 0,
    DASH_EINVAL = -1,       /* bad argument (NULL, out of range, inconsistent shapes) */
    DASH_ESIZE = -2,        /* a size exceeds what the kernels support */
    DASH_EHIP = -3,         /* a HIP runtime call failed */
    DASH_EUNSUPPORTED = -4  /* valid request that this build does not implement */
};

/* Label length rule (Sec. LabelTensors, figure caption).  CEIL: smallest lambda with
 * m^lambda >= 2^128 (at least 128 bits per label).  FLOOR: largest lambda with m^lambda <= 2^128
 * (the caption's floor(128 / log2 m): the label packs into one 128-bit block). */
enum { DASH_LAMBDA_CEIL = 0, DASH_LAMBDA_FLOOR = 1 };

enum {
    DASH_DENSE = 1,    /* out[j] = sum_i W[j][i] * in[i] (+ bias[j])           free gates  */
    DASH_CONV2D = 2,   /* 2-d convolution, zero padding, square stride          free gates  */
    DASH_SUMPOOL = 3,  /* 2x2 sum, stride 2                                     free gates  */
    DASH_RELU = 4,     /* a * sgn_{0,1}(a): sign gadget + mixed-modulus half gates           */
    DASH_SCALE = 5,    /* CRT scaling by 2, `repeat` times                                  */
    DASH_SIGN = 6,     /* sgn_{-1,1}(a)                                                     */
    DASH_PROJ = 7,     /* n independent unary gates Z_p -> Z_q with per-gate function tables */
    DASH_EXPERTS = 8,  /* out[r][j] = sum_i W_e(r)[j][i] * in[r / top_k][i] (+ bias_e(r)[j])  free gates  */
    DASH_COMBINE = 9   /* out[t][v] = sum_j gate[t][j] * in[t * top_k + j][v]           free gates  */
};

/* Weights of an EXPERTS layer: signed bytes, 4-bit floats with a shared power of two for every 32, or 8-bit floats with an integer
 * scale for every block of 128 x 128. */
enum { DASH_W8 = 0, DASH_MX4 = 1, DASH_F8 = 8 };
/* Types of the weights that dash_mx4_quantise and dash_f8_quantise read, and of the logits that dash_choose reads. */
enum { DASH_F32 = 0, DASH_BF16 = 1, DASH_F16 = 2 };

typedef struct dash_ctx dash_ctx;

/* One LabelTensor per CRT residue (see the layout above). */
typedef struct {
    void *data[DASH_MAX_PRIMES];            /* device */
    int64_t chunk_stride[DASH_MAX_PRIMES];  /* bytes between chunks, >= 16 * n_elem, multiple of 16 */
    int64_t n_elem;
} dash_labels;

/* The rows of an EXPERTS layer sorted by expert: written by dash_route, read by every layer call of the same rows. */
typedef struct {
    void *data;             /* device, dash_route_bytes bytes, 16-byte aligned */
    const dash_ctx *ctx;    /* the context it was made with */
    int64_t n;              /* rows */
    int32_t n_experts;
} dash_routing;

/* One layer call.  Fields not used by `kind` are ignored. */
typedef struct {
    int32_t kind;
    int32_t layer_id;   /* 0..65535, enters every hash tweak and PRG counter of the layer */
    int64_t elem_base;  /* index, inside the whole layer, of this call's element 0: a layer may be
                           processed in several calls over disjoint element ranges (batch chunks) */
    int64_t n_elem;     /* RELU / SCALE / SIGN / PROJ: values (gates) in this call;
                           DENSE / CONV2D / SUMPOOL: batch elements in this call;
                           EXPERTS: rows (batch elements * top_k); COMBINE: batch elements of the output */
    /* DENSE, EXPERTS (in_c = K inputs, out_c = M outputs), CONV2D, SUMPOOL (in_h, in_w, in_c), COMBINE (in_c values) */
    int32_t in_h, in_w, in_c, out_c, kh, kw, stride, pad;
    const void *weights;  /* device, written by dash_weights_prepare; EXPERTS: dash_weights8_prepare, dash_mx4_quantise, dash_f8_quantise, dash_f8_prepare */
    const int32_t *bias;  /* device int32 [out_c] (EXPERTS: [n_experts][out_c]) or NULL: added as bias * (constant-one wire) */
    /* Each kind reads its own names.  EXPERTS and COMBINE share places with SCALE and PROJ: the size of the descriptor and the places of
       its fields stay as they were (arrays of it are passed by programs compiled before there were expert layers). */
    union {
        int32_t repeat;         /* SCALE */
        int32_t top_k;          /* EXPERTS, COMBINE: rows per batch element, >= 1 (COMBINE: at most 1024) */
    };
    /* PROJ: input tensor in->data[p_index], output tensor out->data[q_index] */
    union {
        int32_t p_index;
        int32_t n_experts;      /* EXPERTS: matrices in `weights`, >= 1 */
    };
    union {
        int32_t q_index;
        int32_t weight_format;  /* EXPERTS: DASH_W8, DASH_MX4 or DASH_F8 */
    };
    union {
        const uint8_t *phi;           /* PROJ: device, function tables, phi[g * phi_stride + a] in [0, q) */
        const dash_routing *routing;  /* EXPERTS: host pointer; NULL with n_experts = 1: every row takes the one matrix (a dense layer) */
        const int32_t *gates;         /* COMBINE: device int32 [n_elem][top_k], public */
    };
    int64_t phi_stride;   /* PROJ: p (one table per gate) or 0 (one table for all gates) */
} dash_layer;

/* Create a context on GPU `hip_device`: the CRT base (distinct primes, primes[0] must be 2 for
 * SCALE, every prime <= 127, product of the primes below 2^62), the label lengths, the 16-byte seed of
 * the counter-based PRG that replaces the paper's hardware RNG (Sec. Implementation) and the
 * mixed-radix digits d_1..d_n of the sign gadget (Appendix, Approximated Garbled Sign; d_1 most
 * significant and even, k * d_j <= 255; NULL = built-in set with prod(d) >= k * P, which makes the
 * sign exact).
 * Label lengths (Sec. LabelTensors): lambda_rule gives the length of every modulus; `lambda`, if not
 * NULL, is a host array of k entries that overrides it for the CRT primes (lambda[i] digits for
 * primes[i], 1..128; the accumulation moduli of the sign gadget keep the rule).
 * Draws the offset label R_m of every modulus in use (colour digit forced to 1) and the
 * constant-one wire of every prime.  Allocates a few hundred KB of device memory.  Tuning variables of
 * the environment (DASH_BANKED_MIN_LANES, DASH_DIGITS_BANKED_MIN_LANES, DASH_GARBLE_FEW_ROWS, DASH_FUSED_MIN_ELEMS_GARBLE,
 * DASH_FUSED_MIN_ELEMS_EVAL, DASH_WIDE_MAX_LANES, DASH_SUM_IN_LAUNCH, DASH_QUAD_MAX_LANES, DASH_GEMM_TILE, DASH_EXPERTS_TILE, DASH_LINEAR_FORM,
 * DASH_PACK_RUN_LOG2, DASH_ACT_EVAL, DASH_ACT_SHALLOW_MIN_ELEMS, DASH_ACT_DEEP_MIN_ELEMS) are read here, once per context, and nowhere else.
 * Naming one of the four that belong to the evaluator's path by step (DASH_FUSED_MIN_ELEMS_EVAL, DASH_WIDE_MAX_LANES,
 * DASH_SUM_IN_LAUNCH, DASH_QUAD_MAX_LANES), with any value, takes that path instead of the one launch per ReLU or scaling
 * layer, unless DASH_ACT_EVAL=1.
 * Errors: DASH_EINVAL (NULL, non-prime or repeated modulus, bad digits or lambda), DASH_ESIZE (product
 * of the primes too large), DASH_EUNSUPPORTED (no digit set found), DASH_EHIP. */
int dash_ctx_create(dash_ctx **out, const uint16_t *primes, int k, int lambda_rule, const uint16_t *lambda,
                    const uint8_t seed[16], const uint16_t *sign_digits, int n_digits, int hip_device);
void dash_ctx_destroy(dash_ctx *ctx);

/* Label length of modulus m (2..255) under the context's rule; 0 if m is out of range. */
int dash_lambda(const dash_ctx *ctx, int m);
/* Copy to host memory: the offset label R_m (lambda_m bytes) of a modulus the context uses;
 * the constant-one wire of prime i (which = 0 zero label, 1 active label).  Synchronous. */
int dash_ctx_offset(const dash_ctx *ctx, int m, uint8_t *host_out);
int dash_ctx_one(const dash_ctx *ctx, int i, int which, uint8_t *host_out);
/* Mixed-radix digits in use: writes d_1..d_n to host_digits (DASH_MAX_DIGITS entries), returns n. */
int dash_ctx_digits(const dash_ctx *ctx, uint16_t *host_digits);

/* Sizes of one layer call: output elements (values, or batch elements for the linear kinds:
 * then *out_elems is values per batch element, of an EXPERTS layer values per row), bytes of ciphertext tables, bytes of scratch.  The scratch of a
 * SCALE layer does not depend on its repetitions and grows with its values: one buffer serves smaller layers. */
int dash_layer_sizes(const dash_ctx *ctx, const dash_layer *layer, int64_t *out_elems, size_t *table_bytes,
                     size_t *scratch_bytes);

/* Weights of a linear layer are public constants (Sec. Arithmetic Garbled Circuits,
 * multiplication by a public constant): reduce them once per prime into the int8 operand layout
 * of the contraction kernels.  w: device int32 [out_c][K] (K = kh*kw*in_c, order [ky][kx][ci]). */
size_t dash_weights_bytes(const dash_ctx *ctx, int out_c, int K);
int dash_weights_prepare(dash_ctx *ctx, const int32_t *w, int out_c, int K, void *prepared, void *hip_stream);

/* Layers whose matrix depends on the row (EXPERTS).  Which expert serves a row is public: a garbled circuit is fixed before its
 * inputs are known, so rows are routed by what is known then (the client, the task, a position), never by a label.
 *
 * Sums are held in 31 bits: in_c times 256 (p - 1) for DASH_W8 and DASH_F8, (p - 1)^2 for DASH_MX4, has to stay below 2^31 for the largest prime p,
 * else DASH_ESIZE; so for more than 2^31 - 256 outputs.
 *
 * Prepared weights of an EXPERTS layer: n_experts matrices [out_c][K] one after the other, 16-byte aligned, independent of the
 * primes.  A matrix is cut into tiles of 32 rows x 64 columns, row tiles outermost, zeros past out_c and K.
 *   DASH_W8   2048 bytes a tile: weight (r, c) at 64 r + 16 ((c / 16) ^ f(r)) + c % 16, f(r) = (r / 2) % 4 ^ (r / 8) % 2
 *   DASH_MX4  1088 bytes a tile: the codes of (r, c) in byte 32 r + c % 32, low four bits where c < 32, else high; then the shifts, of (r, c) in byte 1024 + 2 r + c / 32.  A code is an e2m1 float: bit 3 the sign, bits 0..2
 *             the magnitude 0, 1/2, 1, 3/2, 2, 3, 4, 6; the weight that enters the layer is the integer 2 * e2m1 * 2^shift.
 *   DASH_F8   tiles as DASH_W8's with codes in place of the weights; behind a matrix's tiles the scales, int32 [ceil(out_c / 128)][ceil(K / 128)],
 *             padded to a multiple of 16 bytes.  A code is an e4m3 float: bit 7 the sign, bits 3..6 the exponent e, bits 0..2 the mantissa m,
 *             (1 + m/8) 2^(e - 7), or m 2^-9 where e = 0; 0x7f and 0xff, not a number, are stored as 0.  The weight that enters the layer is the
 *             integer 512 * e4m3 * scale.  The product of the primes has to hold the sums of these: 458752 * scale at least for one of the largest code
 *             (8 primes from 2 on, 9699690, up to a scale of 21; 12 primes, 7.4e12). */
size_t dash_expert_weights_bytes(int format, int n_experts, int out_c, int K);
/* DASH_W8.  w: device int8, element (e, j, i) at w[e * expert_stride + j * row_stride + i] (row_stride >= K, expert_stride
 * >= 0). */
int dash_weights8_prepare(dash_ctx *ctx, const int8_t *w, int64_t row_stride, int64_t expert_stride, int n_experts, int out_c,
                          int K, void *prepared, void *hip_stream);
/* DASH_MX4, quantised on the device.  w: device, `dtype` elements, strides in elements as above.  Of 32 consecutive weights of a
 * row (fewer at its end) with largest magnitude a, the shared exponent is E = floor(log2 a) - 2, brought into
 * [base, base + max_shift] (-126 <= base <= 125, 0 <= max_shift <= 255; never above 125); each weight becomes the e2m1 value nearest
 * to w / 2^E, ties to the even code, magnitudes past 6 the 6.  The stored shift is E - base: the layer multiplies by integers in
 * units of 2^(base - 1), at most 12 * 2^max_shift of them, which is what the product of the primes has to hold beside the
 * activations.  A NaN counts as 0, an infinity as the largest float32.  values: device, contiguous [n_experts][out_c][K] of
 * `dtype`, or NULL: the weights that the codes stand for, e2m1 * 2^E (float16 rounds those outside its range). */
int dash_mx4_quantise(dash_ctx *ctx, const void *w, int dtype, int64_t row_stride, int64_t expert_stride, int n_experts, int out_c,
                      int K, int base, int max_shift, void *prepared, void *values, void *hip_stream);
/* DASH_F8, quantised on the device.  w, dtype, strides, values as for dash_mx4_quantise.  The weights of a block of 128 rows by 128 columns
 * (fewer at the ends) with largest magnitude a get the scale S = ceil(a / (448 * 2^base)), brought into [1, max_scale] (-64 <= base <= 64, 1 <=
 * max_scale <= 32767); each weight becomes the e4m3 value nearest to w / (S 2^base), ties to the even code, magnitudes past 448 the 448.  The
 * layer multiplies by integers in units of 2^(base - 9), at most 229376 * max_scale of them.  (From base = ceil(log2(largest magnitude /
 * (448 * max_scale))) on no weight is clipped; a larger base makes the integers smaller, and weights below 2^(base - 6) are then steps of 2^(base - 9).)  A NaN counts as 0, an infinity as the
 * largest float32; no sign on a zero.  values: e4m3 * S * 2^base, rounded once to `dtype`. */
int dash_f8_quantise(dash_ctx *ctx, const void *w, int dtype, int64_t row_stride, int64_t expert_stride, int n_experts, int out_c,
                     int K, int base, int max_scale, void *prepared, void *values, void *hip_stream);
/* DASH_F8 from codes and scales that exist already.  codes: device, e4m3 bytes, strides as above; scales: device int32, contiguous
 * [n_experts][ceil(out_c / 128)][ceil(K / 128)], any values.  Codes that are not a number count as 0. */
int dash_f8_prepare(dash_ctx *ctx, const uint8_t *codes, int64_t row_stride, int64_t expert_stride, const int32_t *scales, int n_experts,
                    int out_c, int K, void *prepared, void *hip_stream);
/* Experts and gates from a router's logits, public values as everything that a circuit is routed by. */
enum { DASH_SOFTMAX = 0, DASH_SIGMOID = 1 };
enum { DASH_GROUP_MAX = 0, DASH_GROUP_PAIR = 1 };
#define DASH_MAX_ROUTED 1024    /* experts */
#define DASH_MAX_TOP_K 32
typedef struct {
    int32_t n_experts, top_k;
    int32_t score;                      /* DASH_SOFTMAX (over the experts of a row) or DASH_SIGMOID */
    int32_t n_groups, top_groups;       /* equal groups of neighbouring experts (at most 64), and how many of them experts are chosen from */
    int32_t group_score;                /* a group counts as its largest choice value, or the sum of its two largest (DASH_GROUP_PAIR) */
    int32_t renormalise;                /* != 0: weights are divided by the sum of a row's chosen scores */
    int32_t gate_bits;                  /* 0..30; scale * 2^gate_bits at most 2^30 */
    float scale;                        /* > 0 */
    const float *bias;                  /* device [n_experts] or NULL: added to the scores for the choice, not in the weights */
} dash_router;
/* logits: device, n rows of n_experts `dtype` elements (DASH_F32, DASH_BF16, DASH_F16), row_stride (>= n_experts) elements apart.  Of every row: scores s = softmax(l)
 * or sigmoid(l); choice values c = s + bias, without a bias the order of l (groups of DASH_GROUP_PAIR: sums of s); the top_groups groups
 * with the largest value; of their experts the top_k with the largest c, in descending order.  Ties go to the lower number.  Weights w =
 * scale * s (renormalise: / sum of the chosen s, zero if that is zero), gates = w * 2^gate_bits to the nearest integer, ties to the even
 * (of the quotient itself, not of its rounding: k equal scores get gates of scale * 2^gate_bits / k).  Scores, sums, choice values and weights are held in 64 bits.
 * A logit that is not a number counts as -infinity, infinity as the largest float32.  Experts whose logit is -infinity, or whose choice value is -infinity or no number, are
 * never chosen; groups without any other are not either.  A score below e^-690 (softmax: of the row's largest) is zero.  valid: device, a byte for every row, 0: no expert is chosen (NULL: all rows are valid).  What is missing of
 * top_k: expert -1, weight and gate 0.
 * experts, gates, weights: device [n][top_k]; gates and weights may be NULL.  experts is what dash_route takes (rows n * top_k), gates what COMBINE does.
 * DASH_ESIZE: more than DASH_MAX_ROUTED experts, DASH_MAX_TOP_K of them chosen or 64 groups. */
int dash_choose(dash_ctx *ctx, const dash_router *router, const void *logits, int dtype, int64_t row_stride, int64_t n, const uint8_t *valid,
                int32_t *experts, int32_t *gates, float *weights, void *hip_stream);
/* Sorts rows by expert: experts: device int32 [n], the expert of every row in [0, n_experts); any other number: no expert, the
 * row's outputs are all-zero labels on both sides (the value 0, no bias).  Fills *routing, which the caller keeps (with `data`) as long as layers refer
 * to it; one routing serves garbler and evaluator, and every layer over the same rows.  `experts` may be changed once the stream
 * has passed the call.  dash_route_bytes is 0 for sizes that dash_route refuses (n times the 16-digit chunks of all primes and 64 more
 * below 2^31, n_experts below 2^24 - 1). */
size_t dash_route_bytes(const dash_ctx *ctx, int64_t n, int n_experts);
int dash_route(dash_ctx *ctx, const int32_t *experts, int64_t n, int n_experts, void *data, dash_routing *routing,
               void *hip_stream);

/* Gb, one layer: from the zero labels of the layer's input wires produce the zero labels of its
 * output wires and (RELU, SCALE, SIGN, PROJ) its ciphertext tables.  Fresh zero labels come from
 * the PRG, addressed by (layer_id, slot, element).  tables / scratch: device, sizes from
 * dash_layer_sizes (may be NULL when the size is 0).  For RELU, SCALE and SIGN out_zero may be the same bundle as in_zero
 * (in place; likewise out_act and in_act of dash_eval_layer); bundles that overlap only in part are not supported.
 * Large garbling launches raise the issue priority of their waves until they are about to end (inside the kernel; stream priorities are not
 * touched): work on other streams beside them takes up to a tenth longer, and the garbling ends sooner. */
int dash_garble_layer(dash_ctx *ctx, const dash_layer *layer, const dash_labels *in_zero, dash_labels *out_zero,
                      void *tables, void *scratch, void *hip_stream);
/* Ev, one layer: from the active labels of the input wires and the tables produce the active
 * labels of the output wires. */
int dash_eval_layer(dash_ctx *ctx, const dash_layer *layer, const dash_labels *in_act, const void *tables,
                    dash_labels *out_act, void *scratch, void *hip_stream);

/* n independent layer calls in one (Sec. LabelTensors: gates of the same kind are processed together as tensors): the
 * result is that of dash_garble_layer (dash_eval_layer) on (layers[i], in[i], out[i], tables[i], scratch[i]) for
 * i = 0 .. n-1, and no call of the list may read what another one writes.  The library may serve several calls with
 * one kernel launch: PROJ calls with the same layer_id share launches, when garbling those with the same output modulus, up to
 * 16 a launch (the 144 (p, q) groups of a mixed batch of independent gates take 12 gate launches instead of 144), when evaluating
 * over the primes up to 37 those of any moduli, up to 64 a launch (3 instead of 144), unless an output modulus has gates enough
 * for launches of its own; other kinds are run in turn.  layers, in, out: host arrays of n entries; tables, scratch: host arrays of n device pointers (an entry
 * may be NULL where dash_layer_sizes gives 0; scratch itself may be NULL if no call needs scratch).  If the list holds
 * PROJ calls only, nothing is launched when the argument check of any call fails; otherwise the calls before the
 * failing one have been enqueued. */
int dash_garble_layers(dash_ctx *ctx, int n, const dash_layer *layers, const dash_labels *in_zero, dash_labels *out_zero,
                       void *const *tables, void *const *scratch, void *hip_stream);
int dash_eval_layers(dash_ctx *ctx, int n, const dash_layer *layers, const dash_labels *in_act, const void *const *tables,
                     dash_labels *out_act, void *const *scratch, void *hip_stream);

/* For callers that cannot allocate device memory (code under HIP graph capture, serving loops with a fixed memory
 * budget, harnesses that forbid hipMalloc): dash_eval_layer with the scratch buffer taken from a fixed array of
 * DASH_NOALLOC_SCRATCH_BYTES that lives inside the library (one copy per GPU, held until the process ends; its
 * device address is resolved once per GPU by dash_ctx_create).  Same arguments, results and errors as
 * dash_eval_layer otherwise; inputs, tables and outputs are still the caller's.  Returns DASH_ESIZE, and launches
 * nothing, when the layer call needs more scratch than the array holds (dash_layer_sizes reports the need; split
 * the layer into several calls over element ranges then).  The call allocates and frees nothing and does not
 * synchronise.  Every kernel writes the scratch wires it reads, so nothing has to be cleared between calls, but all
 * calls on one GPU share the one array: two calls that may overlap in time on the same GPU (different streams,
 * different contexts) race; order them. */
#define DASH_NOALLOC_SCRATCH_BYTES (32u << 20)
int dash_eval_layer_noalloc(dash_ctx *ctx, const dash_layer *layer, const dash_labels *in_act, const void *tables,
                            dash_labels *out_act, void *hip_stream);

/* e: zero labels of the circuit-input wires first_wire .. first_wire + n - 1, every residue, into elements 0 .. n - 1
 * of `zero` (n <= zero->n_elem, else DASH_EINVAL). */
int dash_input_labels(dash_ctx *ctx, int64_t first_wire, int64_t n, dash_labels *zero, void *hip_stream);
/* En: out = zero + (value mod p) * R_p (Sec. Quantization and Encoding: Encode(x) = x mod P).
 * values: device int64 [n].  A residue whose data pointer is NULL in both bundles is skipped (bundles that carry
 * a single residue, as the inputs of PROJ gates do); NULL in only one of them is DASH_EINVAL. */
int dash_encode(dash_ctx *ctx, const int64_t *values, int64_t n, const dash_labels *zero, dash_labels *out,
                void *hip_stream);
/* De: per element, the residue a_i with act = zero + a_i * R_p on every digit, CRT-reconstructed and
 * mapped to signed (upper half of Z_P negative).  values: device int64 [n]; valid: device u8 [n],
 * 0 where some residue's label is not a valid label of its wire (then values = 0). */
int dash_decode(dash_ctx *ctx, const dash_labels *act, const dash_labels *zero, int64_t n, int64_t *values,
                uint8_t *valid, void *hip_stream);

/* The 128-bit wire format of labels (Sec. Evaluation, online communication: every label is compressed
 * to 128 bits for transfer; Sec. Implementation: compress(l) = (...(l_n p + l_{n-1}) p + ...) p + l_1).
 * packed: device, 16-byte aligned, [k residues][n][16 bytes], each entry the little-endian 128-bit
 * integer sum_j l_j p^j of the label of element e (elements 0 .. n-1 of the LabelTensor), residue i.
 * 16 bytes per label instead of 16 * ceil(lambda / 16).  unpack is the inverse (base-p digits, least
 * significant first, digits past lambda zero).  Lossless only if p^lambda <= 2^128 for every residue,
 * i.e. for contexts created with the floor rule of the LabelTensor figure; otherwise both calls
 * return DASH_EUNSUPPORTED and touch nothing.  Asynchronous on the stream, no allocation. */
int dash_labels_pack(dash_ctx *ctx, const dash_labels *labels, int64_t n, void *packed, void *hip_stream);
int dash_labels_unpack(dash_ctx *ctx, const void *packed, int64_t n, dash_labels *labels, void *hip_stream);

/* The packed storage format of a layer's ciphertext tables, for keeping garbled layers and for shipping them from the
 * garbling device to the inference device (Sec. System-level Architecture, offline phase).  A ciphertext is an
 * encrypted label, a vector in Z_q^lambda, and is compressed exactly like a label (Sec. Implementation, compress;
 * Sec. Evaluation: labels travel as 128 bits): row r of a segment becomes the little-endian 128-bit integer
 * sum_j row[j] q^j, 16 bytes instead of pitch_q = 4 ceil(lambda_q / 4); the one-digit rows of a half gate become one
 * byte each.  Packed layout: the layer's segments in the same order, segment [gate][row][16] (one-digit segments
 * [gate][row][1], padded to a multiple of 16 bytes).  `layer` is the descriptor the tables were garbled with (kind,
 * n_elem, repeat, p_index / q_index).  Lossless only if q^lambda_q <= 2^128 for every output modulus of the layer,
 * i.e. for contexts with the floor rule; otherwise dash_tables_packed_bytes returns 0 and the two calls return
 * DASH_EUNSUPPORTED and touch nothing.  The garbling and evaluating kernels work on the unpacked format: unpack before
 * dash_eval_layer.  tables: device, 4-byte aligned; packed: device, 16-byte aligned, dash_tables_packed_bytes bytes.
 * Asynchronous on the stream, no allocation.  (Garbled row reduction, which would drop one row per gate, is not part
 * of the scheme: Sec. Arithmetic Garbled Circuits, projection gates, leaves it out.) */
size_t dash_tables_packed_bytes(const dash_ctx *ctx, const dash_layer *layer);
int dash_tables_pack(dash_ctx *ctx, const dash_layer *layer, const void *tables, void *packed, void *hip_stream);
int dash_tables_unpack(dash_ctx *ctx, const dash_layer *layer, const void *packed, void *tables, void *hip_stream);

const char *dash_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* DASH_H */
