/*
 * ssnet.h - C ABI of the MI355X (gfx950) library for the per-party arithmetic
 * of Shamir-secret-sharing neural-network inference.
 *
 * All n parties of a (k = t+1, n) threshold scheme are simulated as the
 * leading (batch) dimension of every share tensor on one GPU; no data leaves
 * the device inside a call.  The field is F_p with p = 2^61 - 1; a field
 * element is a uint64_t in [0, p-1] (canonical: the value p never appears).
 *
 * The field is fixed when the library is compiled.  The same sources built
 * with -DSS_FIELD_P45 give a second library with this same ABI over the prime
 * of Sec. VII-A, p = 2^45 - 55 (16-bit operands, 13 bits of accumulation room):
 * field elements have 6 int8 limbs instead of 8, so limb tiles and limb planes
 * are three quarters the size (ask ssnet_packed_weight_bytes /
 * ssnet_conv_planes_bytes of the library in use) and a product costs 36 int8
 * multiply-adds instead of 64.  Wherever a comment below says 2^61 - 1, "61
 * bits" or "eight limbs", read the library's own prime (ssnet_field_prime) and
 * limb count.  Preconditions stated against p/2 scale with it: over the
 * 45-bit prime truncation needs |x| + 2^32 <= (p-1)/2 and the ReLU mask
 * |x| * 2^28 < p/2, i.e. |x| < 2^16, the paper's 16-bit budget (Sec. VII-B).
 *
 * Conventions for every entry point below
 *   - `d_` pointers are DEVICE pointers owned by the caller (8-byte aligned;
 *     16-byte aligned buffers take the faster vector path).  The library never
 *     allocates, frees or keeps them, except the workspace handed over with
 *     ssnet_set_workspace, which it uses until replaced or the context dies.
 *   - Share tensors are party-major: shares[i*count + e] is the share of
 *     element e held by the party with ID i+1 (IDs are 1..n, Sec. IV-A).
 *   - Work is enqueued on the HIP stream given at creation; calls do not
 *     synchronise.  Inputs and outputs must not alias unless stated.
 *   - Inputs must be canonical (< p); outputs always are.
 *   - Return value: SSNET_OK (0) or a negative SSNET_E* code; nothing throws.
 *   - A launch holds less than 2^32 threads of one or two elements each.  Longer
 *     tensors are taken by ssnet_truncate(_div), ssnet_reduce_truncate_direct and
 *     the product calls; the other element-wise calls return SSNET_EHIP for them
 *     before any launch.
 *   - Randomness: every random polynomial coefficient is a pure function of
 *     (seed, domain, stream_id, party, coefficient index, element index) by the
 *     counter-based generator documented with ssnet_rng_key / ssnet_rng_draw,
 *     so equal arguments give equal bits.  Use a fresh stream_id per call.
 */
#ifndef SSNET_H
#define SSNET_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SSNET_OK 0
#define SSNET_EINVAL (-1)     /* null pointer, bad n/t/f/degree/shape                 */
#define SSNET_EPRIME (-2)     /* p is not the prime this library was built for         */
#define SSNET_ESHARES (-3)    /* fewer than degree+1 parties given to reconstruct      */
#define SSNET_EID (-4)        /* party id outside [1, n] or repeated                   */
#define SSNET_EWORKSPACE (-5) /* workspace missing or too small for this call          */
#define SSNET_EHIP (-6)       /* a HIP call failed; see ssnet_last_hip_error           */
#define SSNET_ESCRATCH (-7)   /* count beyond the fixed scratch of ssnet_degree_reduce_static */

#define SSNET_MAX_PARTIES 8   /* n <= 8                                                */
#define SSNET_MAX_T 3         /* t <= 3 (n >= 2t+1)                                    */
#define SSNET_MAX_K 16383     /* contraction length of linear/conv (int32 exactness)   */

#define SSNET_P61 0x1FFFFFFFFFFFFFFFULL /* 2^61 - 1                                    */
#define SSNET_P45 0x1FFFFFFFFFC9ULL     /* 2^45 - 55 (Sec. VII-A)                      */

/* The prime this library was built for: SSNET_P61 or SSNET_P45. */
uint64_t ssnet_field_prime(void);

typedef struct ssnet_ctx ssnet_ctx;

/* Context: parameters of the scheme plus host-computed constant tables
 * (Lagrange multipliers of Eq. 2 for IDs 1..k, the factors of the reduction
 * matrix R = B^-1 P B of Eq. 3).  Requires n >= 2t+1 (Sec. III-B), 1 <= t <=
 * SSNET_MAX_T, n <= SSNET_MAX_PARTIES, p == ssnet_field_prime(), 1 <= f <= 31.
 * `hip_stream` is a hipStream_t (NULL = the default stream).  Host-only work:
 * creating a context does not touch the GPU. */
int ssnet_create(ssnet_ctx **out, int n, int t, uint64_t p, int f, uint64_t seed, void *hip_stream);
int ssnet_destroy(ssnet_ctx *ctx);

/* Scratch memory for the inter-party messages of ssnet_degree_reduce /
 * ssnet_truncate on `count` elements, and for the int8 limb tiles and split
 * partial sums of ssnet_linear_mod / ssnet_conv_mod.  Sizes are in bytes; a
 * workspace of the maximum over the calls that will be made serves all of them.
 * The first SSNET_WS_HEADER_BYTES of a workspace are reserved; the messages of
 * ssnet_degree_reduce ([2t+1][k][count] then [k][n][count]) and of
 * ssnet_truncate ([k][count] then [n][count]) start right behind that header.
 * 16-byte aligned. */
#define SSNET_WS_HEADER_BYTES 65536
size_t ssnet_workspace_bytes_stream(const ssnet_ctx *ctx, size_t count);
size_t ssnet_workspace_bytes_linear(const ssnet_ctx *ctx, int M, int K, int N);
size_t ssnet_workspace_bytes_conv(const ssnet_ctx *ctx, int B, int C, int H, int W, int Co, int kh, int kw,
                                  int stride, int pad);
int ssnet_set_workspace(ssnet_ctx *ctx, void *d_workspace, size_t bytes);

/* GEN (Eq. 1): for each element e draw a_1..a_degree uniformly from F_p
 * (domain SHARE) and write share_i[e] = a0 + a1 i + ... + a_d i^d mod p for
 * i = 1..n.  d_secret [count] -> d_shares [n][count].  0 <= degree <= 2t. */
int ssnet_share(ssnet_ctx *ctx, const uint64_t *d_secret, size_t count, int degree, uint64_t stream_id,
                uint64_t *d_shares);

/* REC (Eq. 2): secret[e] = sum_{i in ids} lambda_i * shares[i-1][e] mod p with
 * lambda_i = prod_{j != i} j / (j - i).  `party_ids` is a HOST array of m
 * distinct IDs in [1, n]; m >= degree+1 else SSNET_ESHARES (degree = t or 2t).
 * d_shares [n][count] (only the m named planes are read) -> d_secret [count]. */
int ssnet_reconstruct(ssnet_ctx *ctx, const uint64_t *d_shares, size_t count, const int *party_ids, int m,
                      int degree, uint64_t *d_secret);

/* SSS-Linear step 1, dense (Sec. VI-A): every party multiplies its own share
 * matrices, y_i = x_i * w_i mod p.  d_x [n][M][K], d_w [n][K][N] -> d_y
 * [n][M][N], all row-major.  The result is a degree-2t sharing.
 * K <= SSNET_MAX_K.  Needs a workspace (ssnet_workspace_bytes_linear). */
int ssnet_linear_mod(ssnet_ctx *ctx, const uint64_t *d_x, const uint64_t *d_w, int M, int K, int N,
                     uint64_t *d_y);

/* SSS-Linear step 1, convolution (Sec. VI-A): per party, cross-correlation
 * (no kernel flip) with zero padding, mod p.  d_x [n][B][C][H][W], d_w
 * [n][Co][C][kh][kw] -> d_y [n][B][Co][Ho][Wo], Ho = (H+2*pad-kh)/stride+1.
 * C*kh*kw <= SSNET_MAX_K.  Needs a workspace (ssnet_workspace_bytes_conv). */
int ssnet_conv_mod(ssnet_ctx *ctx, const uint64_t *d_x, const uint64_t *d_w, int B, int C, int H, int W,
                   int Co, int kh, int kw, int stride, int pad, uint64_t *d_y);

/* Weights are fixed across inferences (Sec. II-B: preprocessing is done once
 * for a sequence of inferences), so their int8 limb tiles can be prepared
 * once: ssnet_pack_weights_* writes them to caller memory of
 * ssnet_packed_weight_bytes(rows, K) * n bytes, and the *_packed variants of
 * the two layer calls take that buffer in place of d_w.  rows = N (dense) or
 * Co (conv), K = contraction length.  Results are bit-identical. */
size_t ssnet_packed_weight_bytes(int rows, int K);
int ssnet_pack_weights_linear(ssnet_ctx *ctx, const uint64_t *d_w /*[n][K][N]*/, int K, int N, void *d_packed);
int ssnet_pack_weights_conv(ssnet_ctx *ctx, const uint64_t *d_w /*[n][Co][C][kh][kw]*/, int Co, int CKK,
                            void *d_packed);
int ssnet_linear_mod_packed(ssnet_ctx *ctx, const uint64_t *d_x, const void *d_w_packed, int M, int K, int N,
                            uint64_t *d_y);
int ssnet_conv_mod_packed(ssnet_ctx *ctx, const uint64_t *d_x, const void *d_w_packed, int B, int C, int H,
                          int W, int Co, int kh, int kw, int stride, int pad, uint64_t *d_y);

/* The input of a dense layer or of a 1x1, stride 1, unpadded convolution can be
 * shared and brought into limb tiles in one launch, and the layer then run on
 * the tiles alone:
 *   ssnet_share_packed: GEN (Eq. 1, degree t, domain SHARE) of d_secret
 *     [B][K][HW] -> d_shares [n][B][K][HW], the very values ssnet_share writes
 *     for the same stream_id, plus their tiles d_packed (n *
 *     ssnet_packed_weight_bytes(B*HW, K) bytes, 16-byte aligned).  Dense input
 *     [M][K]: B = M, HW = 1.  Conv input [B][C][H][W]: K = C, HW = H*W.
 *   ssnet_linear_mod_prepacked / ssnet_conv1x1_mod_prepacked: SSS-Linear step 1
 *     (Sec. VI-A) as ssnet_linear_mod_packed / ssnet_conv_mod_packed (kh = kw =
 *     stride = 1, pad = 0) compute it, bit-identical, from those tiles.  They
 *     need the workspace of the corresponding ssnet_workspace_bytes_* call. */
int ssnet_share_packed(ssnet_ctx *ctx, const uint64_t *d_secret, int B, int K, int HW, uint64_t stream_id,
                       uint64_t *d_shares, void *d_packed);
int ssnet_linear_mod_prepacked(ssnet_ctx *ctx, const void *d_x_packed, const void *d_w_packed, int M, int K, int N,
                               uint64_t *d_y);
int ssnet_conv1x1_mod_prepacked(ssnet_ctx *ctx, const void *d_x_packed, const void *d_w_packed, int B, int C, int HW,
                                int Co, uint64_t *d_y);

/* Convolution without a materialised im2col matrix (SSS-Linear step 1, Sec.
 * VI-A, for kh x kw kernels with C a multiple of 64): the input is kept as
 * int8 limb planes, per party [limb 0..7][channel block of 16][b][h][w][16] plus a
 * 256-byte pad (ssnet_conv_planes_bytes(B, C, H, W) bytes per party, n parties
 * back to back, 16-byte aligned; 0 for an unsupported shape), from which the
 * product kernel gathers the 16 channels of one tap of one output pixel as 16
 * consecutive bytes; the weights are packed with contraction index (tap,
 * channel).
 *   ssnet_share_planes: GEN (Eq. 1, degree t, domain SHARE) of d_secret
 *     [B][C][H][W] -> d_shares [n][B][C][H][W] (the values of ssnet_share for
 *     the same stream_id) and their planes, in one launch.
 *   ssnet_split_planes: planes of existing shares d_x [n][B][C][H][W].
 *   ssnet_pack_weights_conv_taps: d_w [n][Co][C][kh][kw] -> tiles of
 *     ssnet_packed_weight_bytes(Co, C*kh*kw) bytes per party.
 *   ssnet_conv_mod_planes: d_y [n][B][Co][Ho][Wo], bit-identical to
 *     ssnet_conv_mod on the same shares; workspace as ssnet_workspace_bytes_conv. */
size_t ssnet_conv_planes_bytes(int B, int C, int H, int W);
int ssnet_share_planes(ssnet_ctx *ctx, const uint64_t *d_secret, int B, int C, int H, int W, uint64_t stream_id,
                       uint64_t *d_shares, void *d_planes);
int ssnet_split_planes(ssnet_ctx *ctx, const uint64_t *d_x, int B, int C, int H, int W, void *d_planes);
int ssnet_pack_weights_conv_taps(ssnet_ctx *ctx, const uint64_t *d_w, int Co, int C, int kh, int kw, void *d_packed);
int ssnet_conv_mod_planes(ssnet_ctx *ctx, const void *d_planes, const void *d_w_packed, int B, int C, int H, int W,
                          int Co, int kh, int kw, int stride, int pad, uint64_t *d_y);

/* SSS-Linear step 1 (Sec. VI-A) with the product shares left inside the
 * workspace for the reduction that follows (steps 2 and 3): the layers of a
 * batch-1 network are small, a product kernel then has fewer output tiles than
 * the chip has compute units and splits the contraction over them, and in this
 * form it does not gather the pieces: every workgroup stores what it has, as
 * planes, and the reduction adds them while it reads.  A tile of the product that
 * was cut is the sum mod p of its places in all planes; one that a single
 * workgroup computed lies in the first plane alone, and its places in the further
 * ones may hold anything: they are neither written nor read.  Nothing is exchanged
 * or waited for inside the product kernel.
 *   ssnet_*_product_*: same operands, shapes and checks as ssnet_linear_mod_prepacked,
 *     ssnet_conv1x1_mod_prepacked and ssnet_conv_mod_planes, but no d_y: the
 *     product (count = M*N, resp. B*Co*Ho*Wo elements per party) becomes the
 *     context's pending product, kept in the last ssnet_product_bytes_* bytes of
 *     the workspace until the next ssnet_*_product_* or ssnet_set_workspace call.
 *   Consuming it: ssnet_degree_reduce, ssnet_degree_reduce_truncate(_div,
 *     _reconstruct), ssnet_reduce_truncate_direct and ssnet_reduce_truncate_relu
 *     take d_c = NULL for "the pending product" (count, resp. B*C*HW, must equal
 *     its element count, else SSNET_EINVAL; SSNET_EINVAL too if there is none).
 *     Results, messages and random draws are those of the same call on the d_y
 *     that the corresponding ssnet_*_mod_* call writes.  The call's messages
 *     start behind the workspace header as always, so the workspace must hold
 *     ssnet_workspace_bytes_stream(count) (ssnet_workspace_bytes_layer_tail for
 *     ssnet_reduce_truncate_relu) plus ssnet_product_bytes_*(...) bytes, else
 *     SSNET_EWORKSPACE. */
size_t ssnet_product_bytes_linear(const ssnet_ctx *ctx, int M, int K, int N);
size_t ssnet_product_bytes_conv(const ssnet_ctx *ctx, int B, int C, int H, int W, int Co, int kh, int kw, int stride,
                                int pad);
int ssnet_linear_product_prepacked(ssnet_ctx *ctx, const void *d_x_packed, const void *d_w_packed, int M, int K, int N);
int ssnet_conv1x1_product_prepacked(ssnet_ctx *ctx, const void *d_x_packed, const void *d_w_packed, int B, int C, int HW,
                                    int Co);
int ssnet_conv_product_planes(ssnet_ctx *ctx, const void *d_planes, const void *d_w_packed, int B, int C, int H, int W,
                              int Co, int kh, int kw, int stride, int pad);

/* RED by resharing (Sec. IV-B, the three protocol steps with the matrix of
 * Eq. 3) followed by RERAND (Sec. IV-C), all n parties:
 *   1. parties 1..2t+1: GEN(c_i, k, k) towards parties 1..k   (domain RESHARE, party i)
 *   2. parties 1..k: received row vector times R               -> one value per party 1..n
 *   3. parties 1..n: REC of the k values received, then add the party's share
 *      of a fresh degree-t sharing of zero                     (domain ZERO)
 * d_c [n][count] (degree 2t) -> d_out [n][count] (degree t).  The messages of
 * steps 1 and 2 are materialised in the workspace ([2t+1][k][count] and
 * [k][n][count]).  d_out may alias d_c.  d_c = NULL: the pending product. */
int ssnet_degree_reduce(ssnet_ctx *ctx, const uint64_t *d_c, size_t count, uint64_t stream_id, uint64_t *d_out);

/* ssnet_degree_reduce for callers that cannot allocate device memory or hand a
 * workspace over: code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc.  Same arguments, same random draws, same d_out and the
 * same two message arrays as ssnet_degree_reduce, but the messages go to a fixed
 * array of SSNET_STATIC_SCRATCH_BYTES inside the library's device image (each
 * GPU the library runs on holds it until the process ends) instead of the
 * workspace; no workspace is needed and the call allocates and frees nothing.
 * Limit: (2t+1)(t+1) + (t+1)n message words per element must fit, i.e. count <=
 * SSNET_STATIC_SCRATCH_BYTES / 8 / ((2t+1)(t+1) + (t+1)n) (34952 elements for
 * n = 5, t = 2), else SSNET_ESCRATCH and nothing is launched.  Every call on a
 * GPU uses that GPU's one array (nothing in it needs clearing: a launch writes
 * each message before it is read), so calls that overlap on one GPU, from any
 * context or stream, race on it; calls on one stream are ordered and safe.
 * The device current at the call must be the one the context's stream is on.
 * d_out may alias d_c. */
#define SSNET_STATIC_SCRATCH_BYTES (8u << 20)
int ssnet_degree_reduce_static(ssnet_ctx *ctx, const uint64_t *d_c, size_t count, uint64_t stream_id,
                               uint64_t *d_out);

/* SSS-Truncation (Sec. VI-B) by r = 2^f: shares of floor(x / 2^f), x read as a
 * signed value in [-(p-1)/2, (p-1)/2].
 *   1. parties 1..k add their share of alpha = e*2^f, e uniform in [1, 2^(32-f)]
 *      (Sec. VII-B; domains MASK_E, MASK_ALPHA)
 *   2. the elite party reconstructs x+alpha, shifts right by f (arithmetic) and
 *      re-shares the result                                    (domain TRUNC_GEN)
 *   3. all n parties add their share of alpha~ = -e             (domain MASK_ALPHAT)
 * d_x [n][count] (degree t; planes 1..k are read) -> d_out [n][count].
 * Requires |x| + 2^32 <= (p-1)/2.  Messages go through the workspace.
 * d_out may alias d_x. */
int ssnet_truncate(ssnet_ctx *ctx, const uint64_t *d_x, size_t count, uint64_t stream_id, uint64_t *d_out);

/* SSS-Truncation followed by the rounding division that average pooling moves
 * into it (Sec. VI-C, extra step for AvgPooling; App. C): shares of
 * [floor(x / 2^f) / kdiv], kdiv = kh*kw of the pooling kernel that follows, so
 * that the pooling itself is a sum.  The mask becomes alpha = e*2^f*kdiv with
 * e uniform in [1, floor(2^(32-f) / kdiv)] (the smaller sample space of
 * Sec. VII-B, so that alpha stays in (0, 2^32]; the draw is that of
 * ssnet_truncate, reduced modulo the range instead of masked); [.] rounds to
 * the nearest integer, a remainder of ceil(kdiv/2) or more going up, on the
 * signed value.  1 <= kdiv <= min(SSNET_MAX_KDIV, 2^(32-f)), else
 * SSNET_EINVAL; kdiv = 1 is ssnet_truncate.  Requires |x| + 2^32 <= (p-1)/2,
 * as ssnet_truncate does.  Everything else as ssnet_truncate. */
#define SSNET_MAX_KDIV 4096
int ssnet_truncate_div(ssnet_ctx *ctx, const uint64_t *d_x, size_t count, int kdiv, uint64_t stream_id,
                       uint64_t *d_out);

/* SSS-Linear's reduction followed at once by SSS-Truncation (the default layer
 * order Linear - Truncation of Sec. VII-A): the result, every message and every
 * random draw are those of ssnet_degree_reduce(stream_id) followed by
 * ssnet_truncate(stream_id), in one launch.  Workspace behind the header:
 * [2t+1][k][count], [k][n][count] (reduction), then [k][count], [n][count]
 * (truncation).  d_out may alias d_c. */
int ssnet_degree_reduce_truncate(ssnet_ctx *ctx, const uint64_t *d_c, size_t count, uint64_t stream_id,
                                 uint64_t *d_out);

/* ssnet_degree_reduce(stream_id) followed by ssnet_truncate_div(kdiv, stream_id)
 * in one launch; workspace as for ssnet_degree_reduce_truncate. */
int ssnet_degree_reduce_truncate_div(ssnet_ctx *ctx, const uint64_t *d_c, size_t count, int kdiv, uint64_t stream_id,
                                     uint64_t *d_out);

/* The same launch followed, per element, by REC (Eq. 2) of the truncated shares
 * of the parties party_ids[0..m) (distinct IDs in 1..n, m >= t+1): d_out
 * [n][count] is what ssnet_degree_reduce_truncate writes, d_secret [count] what
 * ssnet_reconstruct(d_out, party_ids, m, degree t) would then return.  The
 * layer-by-layer harness uses it where a layer's result is opened at once.
 * Errors as for the two calls; d_out may alias d_c, d_secret may not alias
 * either. */
int ssnet_degree_reduce_truncate_reconstruct(ssnet_ctx *ctx, const uint64_t *d_c, size_t count, uint64_t stream_id,
                                             uint64_t *d_out, const int *party_ids, int m, uint64_t *d_secret);

/* The outputs of ssnet_degree_reduce_truncate(_reconstruct) without the protocol:
 * they do not depend on the reshare and zero randomness (the elite party of the
 * truncation sees x + alpha, x being the secret of the incoming degree-2t
 * sharing), so with all parties on one device they follow from REC of the 2t+1
 * incoming shares and truncation steps 2 and 3.  d_out (and d_secret, if not
 * NULL) hold the very residues the protocol entry points write for the same
 * stream_id; no message is formed and no workspace is used.  This is a
 * simulation shortcut, reported beside the protocol path, never in its place.
 * d_out may alias d_c. */
int ssnet_reduce_truncate_direct(ssnet_ctx *ctx, const uint64_t *d_c, size_t count, uint64_t stream_id,
                                 uint64_t *d_out, const int *party_ids, int m, uint64_t *d_secret);

/* SSS-NonLinear with ReLU (Sec. VI-C), on shares that were truncated before
 * (order Linear - Truncation - NonLinear, Sec. VII-A).
 *   ssnet_nonlinear_masks: what the trusted source prepares ahead of the
 *     inference (Sec. VII-B): per element a mask beta, uniform in
 *     [1, 2^SSNET_BETA_BITS] (domain MASK_BETA), its inverse in F_p, and a
 *     degree-t sharing of each (domains BETA_GEN, BETAINV_GEN) -> d_beta,
 *     d_betainv [n][count].
 *   ssnet_relu: 1. parties 1..2t+1 multiply their share of x by their share of
 *     beta; 2. the elite party reconstructs x*beta from the 2t+1 products and
 *     applies max(., 0) to the signed value in the clear; 3. every party
 *     multiplies that plain value by its share of beta^-1.  d_x, d_beta,
 *     d_betainv, d_out [n][count]; d_out is a degree-t sharing of max(x, 0).
 *     Requires |x| * 2^SSNET_BETA_BITS < p/2, i.e. |x| < 2^32.  The 2t+1
 *     products and the plain value go through the workspace ([2t+1][count] then
 *     [count] behind the header; ssnet_workspace_bytes_stream(count) covers
 *     it).  d_out may alias d_x. */
#define SSNET_BETA_BITS 28
int ssnet_nonlinear_masks(ssnet_ctx *ctx, size_t count, uint64_t stream_id, uint64_t *d_beta, uint64_t *d_betainv);
int ssnet_relu(ssnet_ctx *ctx, const uint64_t *d_x, const uint64_t *d_beta, const uint64_t *d_betainv, size_t count,
               uint64_t *d_out);

/* SSS-NonLinear with ReLU followed by pooling (Sec. VI-C).  A tensor is `planes`
 * images of H x W (planes = batch * channels, [n][planes][H][W]); the pooling
 * kernel is kh x kw, moved by (sh, sw) over the image padded by ph / pw zeros
 * on each side, Ho = (H + 2*ph - kh) / sh + 1 = ssnet_pool_out_size(H, kh, sh,
 * ph) (0 for sizes that do not fit), Wo likewise.  Accepted: ph < kh, pw < kw,
 * kh <= H + 2*ph, kw <= W + 2*pw, H, W <= 2^15, kh*kw <= SSNET_MAX_KDIV.
 *   ssnet_pool_masks: the trusted source's masks.  beta is equal inside one
 *     pooling kernel: where the kernels partition the image (stride = kernel, no
 *     padding) one beta per kernel position, drawn at counter (plane*Ho + oh)*Wo
 *     + ow (elements beyond the last full kernel join the last one); where they
 *     overlap, one beta per plane, drawn at counter = plane (shared kernels link
 *     every element of a plane to every other).  The sharing coefficients are
 *     drawn per element.  d_beta [n][planes*H*W]; d_betainv [n][planes*Ho*Wo]
 *     shares beta^-1 of the pooled element's kernel.  Domains as
 *     ssnet_nonlinear_masks.
 *   ssnet_relu_pool: 1. parties 1..2t+1 multiply their shares of x and beta;
 *     2. the elite party reconstructs x*beta elementwise, applies max(., 0), and
 *     pools in the clear: mode SSNET_POOL_MAX the maximum, SSNET_POOL_SUM the sum
 *     over the kernel's elements inside the image (the division of an average is
 *     done before, by ssnet_truncate_div with kdiv = kh*kw); 3. every party
 *     multiplies the pooled plain value by its share of beta^-1.  d_out
 *     [n][planes*Ho*Wo] is a degree-t sharing of the pooled max(x, 0).
 *     Requires kh*kw * |x| * 2^SSNET_BETA_BITS < p/2 for the sum, |x| < 2^32 for
 *     the maximum.  Workspace behind the header: the products [2t+1][planes*H*W],
 *     the rectified plain values [planes*H*W], the pooled plain values
 *     [planes*Ho*Wo]; ssnet_workspace_bytes_stream(max of the two counts) covers
 *     it.  d_out must not overlap d_x (SSNET_EINVAL).  It may lie in the memory
 *     of d_beta, which is used up by the call, and may be d_betainv itself
 *     (Ho*Wo being equal); it must not overlap d_betainv in any other way. */
#define SSNET_POOL_MAX 0
#define SSNET_POOL_SUM 1
int ssnet_pool_out_size(int H, int k, int s, int pad);
int ssnet_pool_masks(ssnet_ctx *ctx, size_t planes, int H, int W, int kh, int kw, int sh, int sw, int ph, int pw,
                     uint64_t stream_id, uint64_t *d_beta, uint64_t *d_betainv);
int ssnet_relu_pool(ssnet_ctx *ctx, const uint64_t *d_x, const uint64_t *d_beta, const uint64_t *d_betainv,
                    size_t planes, int H, int W, int kh, int kw, int sh, int sw, int ph, int pw, int mode,
                    uint64_t *d_out);

/* The tail of a convolution layer in the default order Linear - Truncation -
 * NonLinear (Sec. VII-A) in one launch: ssnet_degree_reduce_truncate(stream_id)
 * of the product shares d_c [n][B][C][HW], then ssnet_relu with the masks
 * d_beta, d_betainv [n][B][C][HW]; d_out [n][B][C][HW] holds the residues these
 * two calls give, and d_planes, if not NULL, the same values as
 * limb planes for the next ssnet_conv_mod_planes (C a multiple of 64 then).
 * Messages behind the workspace header: those of the reduction and truncation,
 * then the 2t+1 masked products and the plain value of the ReLU, as planes of
 * P = ssnet_layer_tail_message_plane(B, C, HW) positions each
 * ([2t+1][k][P], [k][n][P], [k][P], [n][P], [2t+1][P], [P]).  For the schemes
 * (3,1) and (5,2), which run as one kernel, a plane is ordered by that kernel's
 * threads, blocks of 16 pixels x 16 channels: element (b, c, hw), pix = b*HW+hw,
 * sits at ((c/16) * ceil(B*HW/16) + pix/16) * 256 + (c%16/4) * 64 + (c%4) * 16 +
 * pix%16, and P counts the padded blocks; for other schemes P = B*C*HW in
 * element order.  ssnet_workspace_bytes_layer_tail gives the bytes needed.
 * d_out may alias d_c.  d_planes may lie in the memory of d_c (if d_out does
 * not), d_beta or d_betainv, which are used up by the call. */
size_t ssnet_layer_tail_message_plane(const ssnet_ctx *ctx, int B, int C, int HW);
size_t ssnet_workspace_bytes_layer_tail(const ssnet_ctx *ctx, int B, int C, int HW);
int ssnet_reduce_truncate_relu(ssnet_ctx *ctx, const uint64_t *d_c, int B, int C, int HW, uint64_t stream_id,
                               const uint64_t *d_beta, const uint64_t *d_betainv, uint64_t *d_out, void *d_planes);

/* The outputs of ssnet_reduce_truncate_relu without the protocol, for all
 * parties on one device (the companion of ssnet_reduce_truncate_direct for the
 * order Linear - Truncation - NonLinear of Sec. VII-A): d_out and, if not NULL,
 * d_planes hold the very residues the protocol entry point writes for any
 * stream_id, because they do not depend on the reshare, zero and truncation
 * randomness: the elite party of SSS-NonLinear (Sec. VI-C) sees floor(x / 2^f) *
 * beta, x being the secret of the incoming degree-2t sharing, and every party's
 * result is max(., 0) times its share of beta^-1.  One pass, no message, no
 * workspace (beyond a pending product, d_c = NULL).  A simulation shortcut,
 * reported beside the protocol path, never in its place.  Any scheme; shapes,
 * masks and planes as for ssnet_reduce_truncate_relu.  d_out may alias d_c;
 * d_planes has memory of its own. */
int ssnet_reduce_truncate_relu_direct(ssnet_ctx *ctx, const uint64_t *d_c, int B, int C, int HW, const uint64_t *d_beta,
                                      const uint64_t *d_betainv, uint64_t *d_out, void *d_planes);

/* ---- transformer blocks: rotary positions, a paged cache, attention ----
 *
 * The dense layers of a block are those above; what follows is what lies between
 * them.  Everything stays on shares: degree-t shares at scale 2^f come in (of
 * queries, keys and values, as ssnet_degree_reduce_truncate leaves them), and
 * the attention's result is a degree-2t sharing like that of a dense layer.
 * d_x of the calls below is [n][tokens][ld]: the heads of a token, heads *
 * head_dim consecutive elements, start every `ld` >= heads * head_dim elements,
 * so that queries, keys and values may be parts of one product; tokens * heads *
 * head_dim < SSNET_MAX_HEADS_COUNT.
 *
 * Rotary positions.  Pair j < rot/2 of the first `rot` elements of every head
 * is turned by the angle of its token: with (c, s) = table[pos[token]][j],
 *   (x_a, x_b) -> (x_a c - x_b s, x_b c + x_a s),
 * (a, b) = (2j, 2j+1) if interleaved, else (j, j + rot/2); elements from `rot`
 * on pass through.  d_table [positions][rot/2][2] holds round(2^f cos),
 * round(2^f sin), whatever the angles are (scaled for a longer context, say);
 * entries are public and may be any int32.  d_pos [tokens]: rows of the table
 * (a row outside of it counts as the nearest one).  2 <= rot <= head_dim, even.
 * The turned elements have 2f fraction bits and are truncated in the same
 * launch: results, messages and draws are those of ssnet_truncate(stream_id) on
 * the tensor [tokens][heads][rot] of turned elements.  Requires |x_a c| + |x_b s|
 * + 2^32 <= (p-1)/2.  Workspace: ssnet_workspace_bytes_stream(tokens * heads *
 * rot).
 *   ssnet_rotary_truncate: d_out [n][tokens][heads][head_dim]; it may be d_x
 *     itself if ld = heads * head_dim, and must not overlap it otherwise. */
#define SSNET_MAX_HEADS_COUNT (1L << 30)
typedef struct ssnet_rotary {
    const int32_t *d_table;
    const int32_t *d_pos;
    int positions, rot, interleaved;
} ssnet_rotary;
int ssnet_rotary_truncate(ssnet_ctx *ctx, const uint64_t *d_x, size_t ld, int tokens, int heads, int head_dim,
                          const ssnet_rotary *rotary, uint64_t stream_id, uint64_t *d_out);

/* A paged cache of keys and values.  A page has `page_size` places for one token
 * each (a multiple of 16); place number page * page_size + i is the token's
 * slot.  The cache holds the balanced digits to the base 256 of every share (8
 * per element, 6 over the 45-bit prime), in cells of 16 places, ready for the
 * int8 products:
 *   d_keys   [pages][n][heads][page_size/16][digit][head_dim/16][16 places][16 elements] int8
 *   d_values [pages][n][heads][page_size/16][digit][head_dim][16 places] int8
 * (ssnet_cache_page_bytes bytes per page each, 16-byte aligned, memory of the
 * caller's; what unused places hold does not matter).  head_dim is a multiple
 * of 16 up to SSNET_MAX_HEAD_DIM; pages * page_size < 2^31.
 *   ssnet_cache_append: keys d_k and values d_v of `tokens` new tokens (token
 *     strides ld_k, ld_v) go to the places d_slots [tokens], all different; a
 *     token whose slot is negative or beyond the cache is left out.  rotary, if
 *     not NULL, turns and truncates the keys on the way as ssnet_rotary_truncate
 *     does (same messages, draws and workspace, heads being the cache's); keys
 *     and values are at scale 2^f. */
#define SSNET_MAX_HEAD_DIM 256
typedef struct ssnet_paged_cache {
    void *d_keys, *d_values;
    int pages, page_size, heads, head_dim;
} ssnet_paged_cache;
size_t ssnet_cache_page_bytes(const ssnet_ctx *ctx, int page_size, int heads, int head_dim);
int ssnet_cache_append(ssnet_ctx *ctx, const ssnet_paged_cache *cache, const uint64_t *d_k, size_t ld_k, const uint64_t *d_v, size_t ld_v,
                       int tokens, const int64_t *d_slots, const ssnet_rotary *rotary, uint64_t stream_id);

/* Attention of new tokens over the paged cache.  `tokens` query tokens belong to
 * `sequences` sequences: those of sequence b are d_start[b] .. d_start[b+1] - 1
 * (d_start[0] = 0, d_start[sequences] = tokens, none or more each).  Its context
 * is the d_length[b] <= max_length tokens whose keys and values lie in the places
 * of the pages d_table[b][0], d_table[b][1], ... in order; the query tokens are
 * the last of them.  causal != 0: query token i of c sees the first d_length[b]
 * - c + i + 1 keys, otherwise all; a row that sees nothing gives zero.  heads
 * query heads, a multiple of the cache's; query head h reads head h / (heads /
 * cache heads).  The arrays lie on the device; entries of d_table beyond a
 * sequence's context are not used.
 *
 * Per row (token, head), row index r = token * heads + head, keys j:
 *   1. parties i = 1..2t+1: S_i[j] = q_i . k_i[j] mod p (degree 2t, 2f fraction
 *      bits) plus their share of a mask, uniform in F_p and the same for all keys
 *      of the row (domain ROW_MASK, counter r).  It is shared afresh with degree 2t
 *      for every key: the shares of parties 1..2t are uniform (domain ROWMASK_GEN,
 *      party i, counter r 2^32 + j), that of party 2t+1 is the one with which all of
 *      them open to the mask.  So the messages of a key are uniform but for the
 *      sum they open to.  Of keys that the row does not see none are sent;
 *   2. the elite party reconstructs s[j] + mask, takes the softmax of the row,
 *      which no constant added to it changes, and shares the weights with degree
 *      t (domain WEIGHT_GEN, counter r 2^32 + j).  Of keys that the row does not
 *      see every party's share is 0;
 *   3. all parties: O_i = sum_j P_i[j] v_i[j] mod p.
 * So the elite party learns the differences of a row's scores, that is the
 * weights, as it learns the ratios inside a pooling kernel under a mask that is
 * equal there.  Beyond these differences t parties learn nothing of scores,
 * queries, keys or values.  The differences of more than head_dim rows over as
 * many keys give the queries and the differences of keys up to a linear map that
 * is common to them: where that is too much, weights must not be opened.
 * The softmax is defined in whole numbers: with d the distance of a score from
 * the largest of its row (signed, 2f fraction bits) and h = min(2f, 24),
 *   u = (min(d >> (2f - h), 2^37) * scale) >> (h + 8)  (octaves, 16 fraction bits),
 *   w = E(u mod 2^16) >> (u >> 16), 0 from 31 octaves on,  E(r) ~ 2^30 2^(-r/2^16):
 *     e = 1077640, then for c = 10033292, 59494488, 257928559, 744260865, 2^30:
 *     e = c - ((e r) >> 16)   (off by 2.2e-7 of the weight at most),
 *   W = sum of w, z = max(0, bits of W - 32), R = floor(2^62 / (W >> z)),
 *   P = (((w R) >> 16) + 2^(45 - weight_bits + z)) >> (46 - weight_bits + z),
 * P being 2^weight_bits times the weight.  scale = round(2^24 log2(e) factor), the
 * factor of the scores (1 / sqrt(head_dim)); 2^16 <= scale < 2^26; 8 <=
 * weight_bits <= 30; max_length <= SSNET_MAX_CONTEXT.  Requires differences of
 * scores below p/2.  d_out [n][tokens][heads][head_dim]: a degree-2t sharing with
 * f + weight_bits fraction bits (as with every product, RED and truncation follow;
 * with weight_bits = 2f two truncations).  A weight below 2^-(weight_bits+1) is 0
 * and nothing makes up for it: weight_bits has to grow with the context.  Weights of
 * scores of unit variance sum to 1 within 0.3 % over up to 2^(weight_bits-2) keys, to
 * 0.994 over twice and 0.94 over four times as many.
 * Workspace: ssnet_workspace_bytes_attention for `tokens` tokens has room for the
 * messages of the whole call; a smaller one serves if it has room for one token's,
 * and the tokens are then taken in several runs with the same result.  Messages
 * behind the header: [2t+1][rows][max_length rounded up to 64] masked scores (of the
 * last run; the places of keys that a row does not see are left as they were). */
#define SSNET_MAX_CONTEXT (1 << 20)
typedef struct ssnet_sequences {
    const int32_t *d_start, *d_table, *d_length;
    int sequences, tokens, max_pages, max_length;
} ssnet_sequences;
size_t ssnet_workspace_bytes_attention(const ssnet_ctx *ctx, const ssnet_paged_cache *cache, int sequences, int tokens, int heads,
                                       int max_length);
int ssnet_paged_attention(ssnet_ctx *ctx, const ssnet_paged_cache *cache, const ssnet_sequences *seqs, const uint64_t *d_q, size_t ld_q,
                          int heads, uint32_t scale, int weight_bits, int causal, uint64_t stream_id, uint64_t *d_out);

/* Low-rank adapters of many requests beside a projection that they share.  An
 * adapter changes a dense layer W [K][N] by A B, A [K][rank], B [rank][N] (any
 * factor of theirs belongs into B).  A set holds `adapters` of them, all of one
 * K, N and rank, as the digits that the products need:
 *   d_down, d_up: ssnet_adapter_down_bytes / ssnet_adapter_up_bytes for each, one
 *     after the other, 16-byte aligned, memory of the caller's;
 *   ssnet_pack_adapter: shares d_a [n][K][rank], d_b [n][rank][N] (degree t, scale
 *     2^f) go to place `index`, in place of what it held; rank may be less than
 *     the set's.  Places that nothing was packed into hold no adapter: zeroed
 *     memory stands for one that changes nothing.
 * K <= SSNET_MAX_K, N <= 2^20.
 *   ssnet_adapters_mod: `tokens` tokens belong to `requests` requests, those of
 *     request b are d_start[b] .. d_start[b+1] - 1 (d_start[0] = 0,
 *     d_start[requests] = tokens, none or more each) and take adapter d_adapter[b];
 *     a number outside the set is none.  Tokens in front of d_start[0] or behind
 *     d_start[requests], in a batch that is larger, belong to no request: their y
 *     stays as it is, and step 2 takes zeros for them.  Per token:
 *       1. parties i = 1..2t+1: Z_i = x_i A_i mod p (degree 2t, 2f fraction bits);
 *       2. degree reduction and truncation of Z, messages and draws as in
 *          ssnet_degree_reduce_truncate with count = tokens * rank -> z;
 *       3. all parties: y_i = base_i + z_i B_i mod p,
 *     a degree-2t sharing with 2f fraction bits as the shared projection's product
 *     d_base [n][tokens][N] is, so RED and truncation of both follow once.  Of a
 *     token without an adapter y = base.  d_base may be d_y, or NULL for 0.
 *     d_x [n][tokens][K], d_base and d_y [n][tokens][N] may be parts of longer
 *     rows: element j of a token is number (party * tokens + token) * ld + j.
 *     d_y overlaps neither d_x nor, unless it is the same, d_base.  The range of z
 *     is that of the truncation.  Who takes which adapter is known to all parties. */
#define SSNET_MAX_RANK 128
typedef struct ssnet_adapters {
    void *d_down, *d_up;
    int adapters, K, rank, N;
} ssnet_adapters;
typedef struct ssnet_requests {
    const int32_t *d_start, *d_adapter;
    int requests, tokens;
} ssnet_requests;
size_t ssnet_adapter_down_bytes(const ssnet_ctx *ctx, int K, int rank);
size_t ssnet_adapter_up_bytes(const ssnet_ctx *ctx, int rank, int N);
int ssnet_pack_adapter(ssnet_ctx *ctx, const ssnet_adapters *set, int index, const uint64_t *d_a, const uint64_t *d_b, int rank);
size_t ssnet_workspace_bytes_adapters(const ssnet_ctx *ctx, const ssnet_adapters *set, int requests, int tokens);
int ssnet_adapters_mod(ssnet_ctx *ctx, const ssnet_adapters *set, const ssnet_requests *requests, const uint64_t *d_x, size_t ld_x, const uint64_t *d_base,
                       size_t ld_base, uint64_t stream_id, uint64_t *d_y, size_t ld_y);

/* The next token of every row, drawn from the softmax of its logits: REC from the
 * parties party_ids (as in ssnet_reconstruct, degree t) for whoever receives the
 * result, and the draw in one call; nothing but the logits is opened.  d_logits
 * [n][rows][vocab], possibly part of longer rows (element j of a row is number
 * (party * rows + row) * ld + j), at scale 2^f.  d_params [rows][4] (16-byte
 * aligned): scale, top_k, top_p, min_p of each row; d_random [rows]: uniform
 * numbers below 2^62 (higher bits are ignored); d_allowed [rows][ld_allowed], if
 * not NULL: bit j % 32 of word j / 32 is 1 for tokens that may be drawn.  In whole
 * numbers, per row, over the allowed tokens:
 *   h = min(f, 16); L = the logit in units of 2^-h (floor), limited to +-(2^31 - 1);
 *   d = the largest L of the row - L;
 *   u = (d * scale) >> (h + 8)  (octaves, 16 fraction bits), scale = round(2^24
 *     log2(e) / temperature), taken as 2^14 where it is less;
 *   w = floor(2^30 2^-u), as in ssnet_paged_attention (0 from 31 octaves on);
 *   order: by d, equal ones by their number.
 *   top_k > 0: the first top_k stay.  scale <= 0: the first alone.
 *   top_p < 2^30: of these the fewest first ones stay whose weights sum to at least
 *     max(1, ceil(top_p * sum of all of these / 2^30)) (a negative top_p is 0).
 *   Of these stay those with w >= max(1, min(min_p, 2^30)): min_p is 2^30 times a part
 *     of the largest weight.
 * S = the sum of what stays.  d_tokens: the first token, by number, up to and
 * with which the weights sum to more than floor(random * S / 2^62); d_shown: its
 * probability floor((2^30 w + S / 2) / S).  A row that allows nothing: -1, 0.
 * vocab <= SSNET_MAX_VOCAB.  Needs ssnet_workspace_bytes_sample (that of more rows
 * will do too). */
#define SSNET_MAX_VOCAB (1 << 20)
typedef struct ssnet_sampling {
    const int32_t *d_params;
    const int64_t *d_random;
    const uint32_t *d_allowed;
    size_t ld_allowed;
} ssnet_sampling;
size_t ssnet_workspace_bytes_sample(const ssnet_ctx *ctx, int rows, int vocab);
int ssnet_sample(ssnet_ctx *ctx, const uint64_t *d_logits, size_t ld, int rows, int vocab, const int *party_ids, int m, const ssnet_sampling *how,
                 int64_t *d_tokens, int32_t *d_shown);

/* Host-side generator, exposed so that its bits can be checked without a GPU.
 * key = absorb(seed, domain, stream_id, party, j) with h <- mix64((h ^ word) +
 * 0x9E3779B97F4A7C15) from h = 0, mix64 being the SplitMix64 output function;
 * draw(key, e) = mix64(key + (e+1) * 0x9E3779B97F4A7C15); the field element is
 * draw >> 3, with the single value p mapped to 0. */
#define SSNET_DOM_SHARE 1
#define SSNET_DOM_RESHARE 2
#define SSNET_DOM_ZERO 3
#define SSNET_DOM_MASK_E 4
#define SSNET_DOM_MASK_ALPHA 5
#define SSNET_DOM_MASK_ALPHAT 6
#define SSNET_DOM_TRUNC_GEN 7
#define SSNET_DOM_MASK_BETA 8
#define SSNET_DOM_BETA_GEN 9
#define SSNET_DOM_BETAINV_GEN 10
#define SSNET_DOM_ROW_MASK 11
#define SSNET_DOM_ROWMASK_GEN 12
#define SSNET_DOM_WEIGHT_GEN 13
uint64_t ssnet_rng_key(uint64_t seed, uint64_t domain, uint64_t stream_id, uint64_t party, uint64_t j);
uint64_t ssnet_rng_draw(uint64_t key, uint64_t e);
uint64_t ssnet_rng_field(uint64_t key, uint64_t e);

/* Host-side constant tables of a context, for inspection: Lagrange multipliers
 * of an ID set (Eq. 2) into out[m]; the reduction matrix R (Eq. 3, row-vector
 * convention c' = c R) as [2t+1][n] row-major into out. */
int ssnet_host_lagrange(const ssnet_ctx *ctx, const int *party_ids, int m, uint64_t *out);
int ssnet_host_reduction_matrix(const ssnet_ctx *ctx, uint64_t *out);

/* Live kernel timing.  Between ssnet_profile_begin and ssnet_profile_end every
 * entry point brackets the kernels of each class below with a pair of HIP
 * events recorded on the context's stream.  ssnet_profile_end waits for those
 * events and writes, per class, the summed elapsed milliseconds and the number
 * of bracketed spans into two HOST arrays of SSNET_PROF_CLASSES entries.  A
 * span is what one entry-point call launches of that class: one kernel, two
 * where a call is documented as two launches.  An event recorded in front of a
 * launch is stamped when the queue reaches it, so a span contains the few
 * microseconds between that and the kernel's first wave.  Class
 * SSNET_PROF_GEMM_KERNEL has none of that: after ssnet_profile_begin_kernels
 * (instead of ssnet_profile_begin) it holds, for every product kernel (the
 * kernels of class SSNET_PROF_GEMM without the pass that adds planes up), the
 * time between the kernel's own start and end on the GPU, which is what a
 * profiler's kernel trace reports as its duration; the launches that take these
 * time stamps are slower to enqueue, so the bracketed spans of the same pass
 * are wider than after ssnet_profile_begin.  ssnet_linear_mod packs both of its
 * operands in one launch, which is a span of SSNET_PROF_PACK_X; a product small
 * enough to read its input as field elements (by shape, in ssnet_linear_mod(_packed)
 * and ssnet_conv_mod(_packed)) packs its weights alone, SSNET_PROF_PACK_W, if at all.
 * Not for use under stream capture. */
#define SSNET_PROF_SHARE 0
#define SSNET_PROF_RECONSTRUCT 1
#define SSNET_PROF_PACK_W 2
#define SSNET_PROF_PACK_X 3
#define SSNET_PROF_GEMM 4
#define SSNET_PROF_DEGREE_REDUCE 5
#define SSNET_PROF_TRUNCATE 6
#define SSNET_PROF_NONLINEAR 7
#define SSNET_PROF_GEMM_KERNEL 8
#define SSNET_PROF_CLASSES 9
int ssnet_profile_begin(ssnet_ctx *ctx);
int ssnet_profile_begin_kernels(ssnet_ctx *ctx);
int ssnet_profile_end(ssnet_ctx *ctx, double *ms_by_class, uint64_t *spans_by_class);

/* Measured ceilings of the machine, for roofline reports beside the published
 * peaks (bench support, not part of the share arithmetic; each call runs its
 * kernel reps + 1 times on the stream and waits for it):
 *   ssnet_probe_planes: `planes` copies of the `bytes` at d_src to d_dst
 *     (planes * bytes large), 16 bytes per lane, streaming stores: planes = 1 is
 *     a device copy, planes = n the traffic pattern of GEN (Eq. 1).  Result:
 *     moved gigabytes, (1 + planes) * bytes per run, per second.
 *   ssnet_probe_mfma_int8: a register-resident loop of v_mfma_i32_16x16x64_i8, two
 *     waves per SIMD with the operand and accumulator registers of the product
 *     kernel, on operand bytes from the generator (random_operands != 0: the clock
 *     this part holds under MFMA load depends on the data) or on constants.
 *     Result: int8 tera-operations per second.  d_sink: 4 device bytes. */
int ssnet_probe_planes(void *hip_stream, void *d_dst, const void *d_src, size_t bytes, int planes, int reps,
                       double *gb_per_s);
int ssnet_probe_mfma_int8(void *hip_stream, void *d_sink, int random_operands, int reps, double *tera_ops_per_s);

const char *ssnet_strerror(int code);
int ssnet_last_hip_error(const ssnet_ctx *ctx); /* hipError_t of the last failed HIP call, 0 if none */

#ifdef __cplusplus
}
#endif
#endif /* SSNET_H */
