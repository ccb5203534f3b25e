/*
 * sph.h -- C ABI of the SPHQuant decode path on MI355X (gfx950).
 *
 * SPHQuant (spherical weight-only quantisation) stores every 8-element weight vector w of a
 * matrix row, cut along the input dimension, as
 *   - 8 sign bits s            (Sec. 3.1, Eq. 3: s = sign(w), kept exactly),
 *   - a D-bit direction index z into a codebook of 2^D non-negative unit 8-D directions c_k
 *                              (Sec. 3.1, Eq. 5; K_dir = 7B - 8 bits for target width B),
 *   - a V-bit radius level q, dequantised per group of 128 weights (16 vectors) of one row as
 *     r^ = min_G + q * step_G  (Sec. 3.1, Eq. 7; "group minima and scales", App. A),
 * and rebuilds it as w^ = r^ * s (.) c_z (Eq. 4). The library's hot path multiplies the rebuilt
 * matrix with fp16 activations and accumulates in fp32 (Sec. 3.4 and App. D: fused decode in
 * registers, no dequantised weights ever written to memory).
 *
 * Conventions shared by every entry point:
 *  - W is n x k (n = d_out rows, k = d_in columns). k must be a multiple of 128 with
 *    128 <= k <= 2^20, 1 <= n <= 2^24, and ceil(n/16) * k/8 < 2^31.
 *  - Logical codes are row-major: signs/dir/q are [n][k/8] (k/vec_dim for the 4-D and 16-D
 *    formats), group params are [n][k/128]. Sign bit j of a vector belongs to element 8v+j
 *    (least significant bit first); a set bit means the element is negative.
 *  - fp16 values (group params, codebook, activations) are passed as IEEE binary16 bit patterns.
 *  - The caller owns every buffer. The library never allocates device memory; it allocates
 *    host staging memory inside sph_pack_weights only, and frees it on return.
 *  - Device pointers must be device-accessible HIP allocations of the current device, 16-byte
 *    aligned. Compute calls are asynchronous on the given stream; argument errors are detected
 *    on the host before any HIP call and reported through sph_status. Nothing throws or aborts
 *    across this ABI.
 */
#ifndef SPH_H
#define SPH_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SPH_OK = 0,
  SPH_ERR_NULL = 1,               /* a required pointer is NULL                                 */
  SPH_ERR_SHAPE = 2,              /* n < 1, k not a positive multiple of 128, m out of range,   */
                                  /* leading dimension too small, or misaligned pointer         */
  SPH_ERR_UNSUPPORTED_FORMAT = 3, /* (vec_dim, dir_bits, radius_bits, group_size) not built in  */
  SPH_ERR_CODE_RANGE = 4,         /* a direction index >= 2^D or a radius level >= 2^V          */
  SPH_ERR_BAD_VALUE = 5,          /* codebook entry non-finite, negative or above 2; offset     */
                                  /* non-finite; step non-finite or negative                    */
  SPH_ERR_BUFFER_TOO_SMALL = 6,   /* device buffer smaller than sph_packed_bytes                */
  SPH_ERR_HIP = 7,                /* a HIP runtime call or kernel launch failed                 */
  SPH_ERR_BAD_DESCRIPTOR = 8      /* the sph_weights descriptor is not one this library filled  */
} sph_status;

typedef enum { SPH_F16 = 0, SPH_F32 = 1 } sph_dtype;

/* The representation (Sec. 3.1-3.2). Built-in (dir_bits, radius_bits) pairs with vec_dim 8 and
 * group_size 128:
 *   (6, 4)  W2: 8 sign + 6 direction + 4 radius bits, the packed W2 format of Sec. 3.4 / App. D
 *   (13, 3) W3: K_dir = 7*3 - 8 = 13 with 3 radius bits (3.00 bits/weight payload, App. B)
 *   (4, 4)  16-bit vectors: 8 sign + 4 direction + 4 radius bits
 *   (6, 2)  16-bit vectors: 8 sign + 6 direction + 2 radius bits (2.00 bits/weight payload)
 *   (8, 8)  24-bit vectors: 8 sign + 8 direction + 8 radius bits
 *   (13, 4) W3 with 4 radius bits (3.125 bits/weight payload, the W3 row of Tab. 1)
 *   (6, 3), (7, 2), (8, 2)  further splits of the W2 budget from the bit-allocation study of
 *           Tab. 4 (8 sign bits + D direction + V radius bits)
 * and the other vector sizes of Tab. 7 (group_size 128): vec_dim 4 with (2, 3) (4 sign + 2 direction
 * + 3 radius bits) and vec_dim 16 with (14, 6) (16 sign + 14 direction + 6 radius bits); for vec_dim
 * 16 the sign array holds one uint16 per vector.                                               */
typedef struct {
  int32_t vec_dim;      /* 8, or 4 / 16 with the pairs above */
  int32_t dir_bits;     /* D           */
  int32_t radius_bits;  /* V           */
  int32_t group_size;   /* must be 128 */
} sph_format;

/* A packed matrix on the device. Filled by sph_pack_weights; a plain host-side value that may be
 * copied. Points into the caller-owned device buffer; off[] and layout_version are private. */
typedef struct {
  sph_format fmt;
  int64_t n, k;
  void* d_base;
  size_t bytes;
  uint64_t off[8];
  uint32_t layout_version;
  uint32_t magic;
} sph_weights;

/* Bytes of device memory sph_pack_weights needs for an n x k matrix in format *fmt. The figure
 * covers the packed codes (rows padded to a multiple of 16), the fp16 group parameters, the
 * codebook and the lookup tables derived from it. */
sph_status sph_packed_bytes(const sph_format* fmt, int64_t n, int64_t k, size_t* bytes);

/* Validate the logical codes of an n x k matrix (Sec. 3.1, Eq. 3-7), pack them into the library's
 * device layout and copy them into d_buf (d_buf_bytes >= sph_packed_bytes). Inputs are host
 * arrays: signs uint8[n][k/8], dir_idx uint16[n][k/8] (< 2^D), radius_code uint8[n][k/8]
 * (< 2^V), group_min / group_step uint16[n][k/128] (fp16 bits: min finite, step finite and
 * >= 0), codebook uint16[2^D][vec_dim] (fp16 bits, in [0, 2]: coordinates of non-negative unit
 * directions, Sec. 3.1, with room for rounding). Synchronous: returns after the
 * copy on `stream` has completed, so the host arrays may be freed. On success *out describes
 * the packed matrix. */
sph_status sph_pack_weights(const sph_format* fmt, int64_t n, int64_t k, const uint8_t* signs,
                            const uint16_t* dir_idx, const uint8_t* radius_code,
                            const uint16_t* group_min, const uint16_t* group_step,
                            const uint16_t* codebook, void* d_buf, size_t d_buf_bytes,
                            void* stream, sph_weights* out);

/* y = W^ x for one fp16 activation vector (batch 1): the fused dequantise-and-multiply GEMV of
 * Sec. 3.4 / App. D. d_x: device fp16[k]; d_y: device [n] of y_dtype (fp32 accumulation, then
 * rounded to fp16 when y_dtype is SPH_F16). d_ws/ws_bytes: device workspace of at least
 * sph_workspace_bytes(w, 1) bytes (see there; may be NULL when that is 0). The split-K sums are
 * combined in a fixed order, so repeated calls give bitwise identical results.
 * Asynchronous on `stream`. */
sph_status sph_gemv(const sph_weights* w, const void* d_x, void* d_y, sph_dtype y_dtype,
                    void* d_ws, size_t ws_bytes, void* stream);

/* Y = X W^T for 1 <= m <= 32 activation rows: d_x is device fp16[m][ldx] (ldx >= k), d_y is
 * device [m][ldy] of y_dtype (ldy >= n). Every batch size forms exact products of fp16 numbers
 * and rounds only fp32 sums: batch 1, and batch 2 for formats with at most 8 direction bits, on the
 * vector ALUs (signed direction times activations, then times the fp32 radius); batches 3..8 on
 * 4x4x4 MFMA blocks, one vector per block, each block's sum times the fp32 radius; batches 9..32
 * on 16x16x32 MFMA tiles with Eq. 7 factored over each 128-weight group, offset * sum <t, x> +
 * step * sum q <t, x>, where t (the signed direction) and q * t (split exactly into two fp16
 * numbers) are the operands (9..16 inside the step plan; 17..32, and 9..16 on matrices of about
 * 10^8 weights or more, in the prefill kernel of sph_gemm with 16 or 32 activation rows staged in
 * LDS). Asynchronous on `stream`. */
sph_status sph_gemm_small(const sph_weights* w, const void* d_x, int64_t m, int64_t ldx, void* d_y,
                          int64_t ldy, sph_dtype y_dtype, void* d_ws, size_t ws_bytes,
                          void* stream);

/* Y = X W^T for any batch 1 <= m <= 65536 (prefill and large batches): m <= 32 is sph_gemm_small;
 * larger batches run on the matrix cores (16x16x32 fp16 MFMA, fp32 accumulation) with the
 * factored exact-product arithmetic of sph_gemm_small's batches above 8, each weight's operands
 * rebuilt once per 64-row slice of X and per 128-column chunk of K; or, on large shapes, with the
 * radius applied first and radius times direction split into two fp16 operands (23 bits), rebuilt
 * once per 128-row slice, where the rounding error is no larger: that needs group offsets of 0 or of
 * at least 2^-12 of the group's largest radius, and neither zero offsets nor zero steps in more than 3
 * groups of 16 (found by sph_pack_weights and kept in the
 * descriptor), and enough columns. Same argument rules as sph_gemm_small. When the
 * grid would not cover the chip, K is split and fp32 partial outputs go through the workspace
 * (sph_workspace_bytes(w, m); for m > 32 it needs no zero-fill) and are added in a fixed order,
 * so repeated calls give bitwise identical results. Asynchronous on `stream`. */
sph_status sph_gemm(const sph_weights* w, const void* d_x, int64_t m, int64_t ldx, void* d_y, int64_t ldy,
                    sph_dtype y_dtype, void* d_ws, size_t ws_bytes, void* stream);

/* sph_gemm_small without a caller workspace, for callers that cannot allocate device memory (code
 * under HIP graph capture, tight serving loops, harnesses that forbid allocation). Same arguments,
 * arithmetic, results (bitwise) and errors as sph_gemm_small, with d_ws/ws_bytes replaced by a
 * fixed array of SPH_NOALLOC_SCRATCH_BYTES in device memory that the library's code object holds
 * (one per GPU it runs on, kept until the process ends). A call whose sph_workspace_bytes exceeds
 * that size returns SPH_ERR_BUFFER_TOO_SMALL before any HIP call. The first call on a device looks
 * up the array's address and clears it with a kernel on `stream`; every call leaves it zero-filled
 * again. Every call on one GPU shares that GPU's array: calls that may overlap on one GPU (other
 * streams, other threads) race and must not be made. Allocates nothing, on the host or the device.
 * Asynchronous on `stream`. */
#define SPH_NOALLOC_SCRATCH_BYTES (16u << 20)
sph_status sph_gemm_small_noalloc(const sph_weights* w, const void* d_x, int64_t m, int64_t ldx, void* d_y,
                                  int64_t ldy, sph_dtype y_dtype, void* stream);

/* Device workspace needed by sph_gemv (m = 1), sph_gemm_small or sph_gemm for this matrix and
 * batch (1 <= m <= 65536) on the current device (0 when the call needs none; d_ws may then be
 * NULL). For m <= 16 it holds the partial sums of 16-row tiles whose K range is split between
 * workgroups: 64-bit words (fp32 sum and a valid flag), one per value of a tile over two
 * workgroups, one per workgroup and value of a tile over more, and one 32-bit arrival counter per
 * tile; where the prefill kernel runs (m above 16, and 9..16 on large matrices: see
 * sph_gemm_small) it holds fp32 partial outputs of a K split (a large batch with less workspace than
 * this reports, but enough for the three-operand kernel, runs on that). It must be 256-byte
 * aligned and zero-filled before its first use, and every call leaves it zero-filled again (above
 * m = 32 it needs no initial contents, but is still left zero-filled). Calls that may run
 * concurrently must not share one. No call waits for another workgroup to make progress, so calls
 * on other streams may occupy any part of the GPU meanwhile. */
sph_status sph_workspace_bytes(const sph_weights* w, int64_t m, size_t* bytes);

/* Read the packed matrix back as logical codes, on the device, with the same bit extraction the
 * compute kernels use: d_signs uint8[n][k/vec_dim] (uint16 for vec_dim 16), d_dir_idx
 * uint16[n][k/vec_dim], d_radius_code uint8[n][k/vec_dim] are caller-owned DEVICE arrays, written
 * asynchronously on `stream`; the caller copies them to the host and synchronizes. (A host-array,
 * synchronous form would need device staging memory, and the library never allocates device
 * memory; the Python binding does the copy.) For the table-lookup formats the sign bits and the
 * direction are recovered from the two lookup indices each row uses; a mismatch between the
 * direction seen through the low and the high table is reported by setting the direction to
 * 0xFFFF. Intended for bit-exactness tests. */
sph_status sph_unpack(const sph_weights* w, uint8_t* d_signs, uint16_t* d_dir_idx,
                      uint8_t* d_radius_code, void* stream);

/* Spherical quantisation of a dense matrix on the device (Sec. 3.1: Eq. 3 decomposition into signs,
 * radius and unit direction, Eq. 5 nearest direction by cosine, Eq. 6 least-squares radius
 * <|w|, c_z>, Eq. 7 per-group offset min_G, step (max_G - min_G)/(2^V - 1) and level
 * q = clip(round((r~ - min_G)/step_G), 0, 2^V - 1) with the offset and step as stored in fp16).
 * d_w: device fp32[n][ldw] (ldw >= k, ldw % 4 == 0, 16-byte aligned); d_codebook: device
 * fp16 bits [2^D][8]. Outputs are caller-owned device arrays in the layout sph_pack_weights reads:
 * d_signs uint8[n][k/8], d_dir_idx uint16[n][k/8], d_radius_code uint8[n][k/8],
 * d_group_min / d_group_step fp16 bits [n][k/128]. Arithmetic is fp64. Decisions: a coordinate is
 * negative when w < 0 (so -0 is positive); among equal cosines the lowest index wins; a radius of
 * zero divides by 1e-12 instead; rounding is to nearest, ties to even, for the level and for the
 * fp16 offset and step; a zero step gives level 0. The codebook is not validated here (a
 * non-finite or negative entry gives unspecified codes; sph_pack_weights rejects it later), and
 * non-finite weights give unspecified codes. Offsets or steps beyond the fp16 range become
 * infinite, which sph_pack_weights rejects. Asynchronous on `stream`; the result does not depend
 * on the launch or on earlier calls. */
sph_status sph_encode(const sph_format* fmt, int64_t n, int64_t k, const float* d_w, int64_t ldw,
                      const uint16_t* d_codebook, uint8_t* d_signs, uint16_t* d_dir_idx,
                      uint8_t* d_radius_code, uint16_t* d_group_min, uint16_t* d_group_step,
                      void* stream);

/* Device workspace needed by sph_kmeans_codebook for an n x k matrix and n_samples samples
 * (1 <= n_samples <= 2^24): 8 bytes per 8-D vector of the matrix (running sum of squared radii),
 * 76 bytes per sample (direction, assignment, objective part), 12 bytes per sample and codebook
 * split of the assignment (splits x samples stays below about 2^20 + n_samples), 64 bytes per
 * codebook entry (the fp64 centre), and 192 bytes per codebook entry and sample chunk (about
 * 128 / ceil(2^D / 512) chunks, fewer when samples are few) for the counts, the list of samples by
 * centre and the centres' fp16 words (which take less than that), plus alignment. */
sph_status sph_kmeans_workspace_bytes(const sph_format* fmt, int64_t n, int64_t k, int64_t n_samples,
                                      size_t* bytes);

/* Radius-weighted spherical k-means codebook of a matrix (Sec. 3.1; Sec. 4.1 uses 65,536 samples
 * and 20 iterations). The matrix's 8-D vectors are decomposed as in sph_encode; sample j draws the
 * first vector (in row-major order) whose running sum of r^2 exceeds d_u[j] * (total r^2), so
 * vectors are drawn with replacement with probability r^2 / sum r^2; d_u is device fp64[n_samples]
 * of uniforms in [0, 1), drawn by the caller. Starting from the centres d_init (device fp16 bits
 * [2^D][8]), each of `iters` iterations assigns every sampled unit direction to its nearest centre
 * by cosine (lowest index among equals) and moves each centre to the normalised sum of its
 * directions; a centre without directions stays. d_codebook (device fp16 bits [2^D][8]) receives
 * the final centres rounded to nearest fp16. d_objective (device fp64[iters + 1], or NULL) receives
 * the summed cosine of each iteration's assignment and, last, of the final centres.
 * d_sample_idx (device int64[n_samples], or NULL) receives the drawn vector indices (row * k/8 +
 * vector). d_ws: workspace of sph_kmeans_workspace_bytes, 256-byte aligned, no initial contents;
 * concurrent calls must not share one. iters is 0..10000. fp64 arithmetic; every sum runs in a
 * fixed order, so repeated calls give bitwise identical results. Asynchronous on `stream`. */
sph_status sph_kmeans_codebook(const sph_format* fmt, int64_t n, int64_t k, const float* d_w, int64_t ldw,
                               const double* d_u, int64_t n_samples, int32_t iters,
                               const uint16_t* d_init, uint16_t* d_codebook, double* d_objective,
                               int64_t* d_sample_idx, void* d_ws, size_t ws_bytes, void* stream);

/* ---- Fine-tuning side (Sec. 3.3; App. A steps 6-10). fp32 device arrays unless stated. ---- */

/* Angular codebook (Sec. 3.3, Eq. 9-10): for each of the 2^D entries, seven angle logits phi
 * (d_phi fp32[2^D][7]) give theta_j = eps + (pi/2 - 2 eps) sigmoid(phi_j) and the positive unit
 * direction c_1 = cos t_1, c_i = (prod_{j<i} sin t_j) cos t_i (2 <= i <= 7), c_8 = prod_j sin t_j,
 * written to d_codebook fp32[2^D][8]. 1 <= dir_bits <= 13, 0 <= eps < 0.25. Asynchronous. */
sph_status sph_angular_codebook(int32_t dir_bits, const float* d_phi, float eps, float* d_codebook, void* stream);

/* Gradient of a loss through sph_angular_codebook: d_grad_codebook fp32[2^D][8] (dL/dc) gives
 * d_grad_phi fp32[2^D][7] (dL/dphi), from the closed-form derivatives of Eq. 9 and Eq. 10. */
sph_status sph_angular_codebook_backward(int32_t dir_bits, const float* d_phi, float eps,
                                         const float* d_grad_codebook, float* d_grad_phi, void* stream);

/* Inverse of Eq. 9-10 (initialises the angle logits from a codebook, App. A step 7):
 * theta_i = atan2(||c_{i+1..8}||, c_i), t = (theta - eps)/(pi/2 - 2 eps) clamped to
 * [1e-6, 1 - 1e-6], phi = log t - log(1 - t). d_codebook fp32[2^D][8] of non-negative unit
 * directions; d_phi fp32[2^D][7]. */
sph_status sph_angular_logits(int32_t dir_bits, const float* d_codebook, float eps, float* d_phi, void* stream);

/* Host-only, synchronous: the vectors grouped by direction index, for the codebook gradient
 * of sph_fake_quant_backward. dir_idx: host uint16[count] (< 2^D); perm: host int32[count]
 * receives the vector indices sorted by direction, stably (ascending index within a
 * direction); offsets: host int64[2^D + 1], direction z owns perm[offsets[z] .. offsets[z+1]).
 * 1 <= count < 2^31. SPH_ERR_CODE_RANGE for an index >= 2^D. */
sph_status sph_direction_groups(int32_t dir_bits, int64_t count, const uint16_t* dir_idx, int32_t* perm,
                                int64_t* offsets);

/* Radius parameters from a dense matrix (App. A steps 6-7): rho_i = log(exp(r~_i) - 1), the
 * inverse of softplus, of Eq. 6's radius r~_i = <|w_i|, c_{z_i}> floored at 1e-6. d_w fp32[n][ldw]
 * (ldw >= k, ldw % 4 == 0, 16-byte aligned), d_dir_idx uint16[n][k/8], d_codebook fp32[2^D][8]
 * (16-byte aligned), d_rho fp32[n][k/8]. */
sph_status sph_fake_quant_init_rho(const sph_format* fmt, int64_t n, int64_t k, const float* d_w, int64_t ldw,
                                   const uint16_t* d_dir_idx, const float* d_codebook, float* d_rho, void* stream);

/* The pseudo-quantised weight of a linear module (Sec. 3.3; App. A step 8): r = softplus(rho),
 * group-wise V-bit fake quantisation with Eq. 7's offset min_G and step (max_G - min_G)/(2^V - 1),
 * both rounded to fp16 as the finalised codes store them, q = clip(round((r - min_G)/step_G),
 * 0, 2^V - 1) half to even (0 for a zero step), r^ = min_G + q step_G, and w^_i = r^_i s_i (.)
 * c_{z_i} written to d_w_hat fp32[n][ldw] (ldw >= k, ldw % 4 == 0, 16-byte aligned). The radius,
 * offset, step and level are computed in fp64. d_rho fp32[n][k/8]; d_signs, d_dir_idx as in
 * sph_pack_weights; d_codebook fp32[2^D][8] (e.g. from sph_angular_codebook), not validated.
 * Optional outputs (NULL to skip): d_r_hat fp32[n][k/8] (needed by the backward), and together
 * d_radius_code uint8[n][k/8], d_group_min, d_group_step fp16 bits [n][k/128] -- the finalised
 * codes of App. A step 10. Asynchronous; results do not depend on the launch. */
sph_status sph_fake_quant_forward(const sph_format* fmt, int64_t n, int64_t k, const float* d_rho,
                                  const uint8_t* d_signs, const uint16_t* d_dir_idx, const float* d_codebook,
                                  float* d_w_hat, int64_t ldw, float* d_r_hat, uint8_t* d_radius_code,
                                  uint16_t* d_group_min, uint16_t* d_group_step, void* stream);

/* Device workspace of sph_fake_quant_backward for a 2^D-entry codebook (needs no zero-fill). */
sph_status sph_fake_quant_backward_workspace_bytes(int32_t dir_bits, size_t* bytes);

/* Gradients through sph_fake_quant_forward with the straight-through estimator (the rounding of
 * the radius is taken as the identity): given d_grad_w fp32[n][ldg] (dL/dW^; ldg >= k,
 * ldg % 4 == 0, 16-byte aligned), writes d_grad_rho fp32[n][k/8] with
 * dL/drho_i = sigmoid(rho_i) sum_j dL/dw^_ij s_ij c_{z_i,j}, and d_grad_codebook fp32[2^D][8]
 * with dL/dc_z = sum over vectors i of direction z of r^_i s_i (.) dL/dw^_i. d_r_hat is the
 * forward's r^; d_perm int32[n*k/8] and d_offsets int64[2^D + 1] are device copies of
 * sph_direction_groups for the same d_dir_idx (not validated). d_grad_rho may be d_rho or d_r_hat, and
 * d_grad_codebook may be d_codebook. Sums run in an order fixed by the sizes, so repeated calls give bitwise identical
 * results (a centre with a gradient that is not finite excepted, whose sum is not finite). d_ws:
 * sph_fake_quant_backward_workspace_bytes bytes, 16-byte aligned; d_grad_rho serves as more of it
 * before it is written. Asynchronous. */
sph_status sph_fake_quant_backward(const sph_format* fmt, int64_t n, int64_t k, const float* d_rho,
                                   const uint8_t* d_signs, const uint16_t* d_dir_idx, const float* d_codebook,
                                   const float* d_r_hat, const float* d_grad_w, int64_t ldg, const int32_t* d_perm,
                                   const int64_t* d_offsets, float* d_grad_rho, float* d_grad_codebook, void* d_ws,
                                   size_t ws_bytes, void* stream);

/* ---- Between the linear layers of a decoder block: rotary positions, the paged key-value cache and the
 * attention that reads it. Activations are fp16 as the GEMMs take and give them (fp32 where stated). A
 * "row" is one token's vector of one head: head_dim consecutive elements, 16-byte aligned. Token and
 * head strides are in elements and keep that alignment (multiples of 8 for fp16, of 4 for fp32), so q, k
 * and v may be column ranges of the fused product's output. Token counts are 0..2^26 (SPH_ERR_SHAPE for more, and where a
 * call would need 2^32 threads of eight channels each); calls on no tokens do nothing. Values that only the device holds (positions, slots, lengths, pages) cannot be refused by the
 * host; each call says what it does with wrong ones, and none reads or writes outside its arrays. ---- */

/* Rotary positions: the first rot_dim channels of a row turn by position-dependent angles, the others
 * stay. d_table: device fp32[max_pos][rot_dim/2][2] of (cos, sin) for every position and pair (e.g. from
 * sph_rope_table), 16-byte aligned. flags: SPH_ROPE_INTERLEAVED pairs channels (2i, 2i+1), otherwise pair i
 * is (i, i + rot_dim/2); SPH_ROPE_INVERSE turns back (sin -> -sin), which is also the gradient, since a
 * rotation's transpose is its inverse and the table's common factor stays. */
#define SPH_ROPE_INTERLEAVED 1
#define SPH_ROPE_INVERSE 2
typedef struct {
  const float* d_table;
  int64_t max_pos;      /* 1..2^31-1 */
  int32_t rot_dim;      /* a positive multiple of 16, at most head_dim */
  int32_t flags;
} sph_rope_desc;

/* Fill a table: (cos, sin)(p * inv_freq[i]) * magnitude for 0 <= p < max_pos, computed in fp64 and rounded
 * once. inv_freq: HOST double[rot_dim/2] (read before the call returns), rot_dim a multiple of 16 up to 512.
 * SPH_ERR_BAD_VALUE for a frequency or magnitude that is not finite. Asynchronous. */
sph_status sph_rope_table(int32_t rot_dim, int64_t max_pos, const double* inv_freq, double magnitude, float* d_table,
                          void* stream);

/* y = rotated x: rows of `heads` heads (1..65535) of head_dim channels (a multiple of 16, at most 512) for each token, fp16 or
 * fp32 (dtype), computed in fp32 and rounded once. d_pos: device int32[tokens]; a token whose position is
 * outside 0..max_pos-1 gets NaN in the rotated channels. d_y may be d_x with the same strides.
 * Asynchronous. */
sph_status sph_rope(const sph_rope_desc* rope, sph_dtype dtype, int64_t tokens, int32_t heads, int32_t head_dim,
                    const void* d_x, int64_t x_token_stride, int64_t x_head_stride, const int32_t* d_pos, void* d_y,
                    int64_t y_token_stride, int64_t y_head_stride, void* stream);

/* sph_rope with positions along several axes, as images and videos have them: pair i of a row turns by the angles that the table has for
 * the token's position along axis d_axes[i] (device uint8[rot_dim/2], 8-byte aligned). n_axes: 1..16; d_pos: device int32[n_axes], each
 * axis's `tokens` positions pos_stride (0 and more) elements behind the last one's. The table's frequencies are per pair, so axes may share
 * one spectrum or have one each. A pair whose position is outside the table, or whose axis is n_axes or more, gets NaN. With one
 * axis, or positions that agree along all of them, results are sph_rope's, bit for bit. */
sph_status sph_rope_axes(const sph_rope_desc* rope, const uint8_t* d_axes, int32_t n_axes, int64_t pos_stride, sph_dtype dtype,
                         int64_t tokens, int32_t heads, int32_t head_dim, const void* d_x, int64_t x_token_stride, int64_t x_head_stride,
                         const int32_t* d_pos, void* d_y, int64_t y_token_stride, int64_t y_head_stride, void* stream);

/* A key-value cache in pages of page_size tokens: a plain host-side value that describes caller-owned
 * device arrays. Slot s is token s % page_size of page s / page_size. With 16 bits a row of d_k / d_v is
 * head_dim fp16 numbers. With 8 or 4 bits it is head_dim codes (bytes; at 4 bits the 32-bit word w of a row
 * holds channel 8w + 2i at bit 4i and channel 8w + 2i + 1 at bit 16 + 4i), and d_k_par / d_v_par hold an fp16
 * pair (offset, step) for every 32 channels. A code q stands for the fp16 number nearest to
 * offset + q * step; sph_kv_read and sph_attention see exactly these numbers. Strides are in bytes and
 * common to keys and values: code strides multiples of 16, parameter strides multiples of 4; d_k and d_v 16-byte, parameter
 * arrays 4-byte aligned. */
typedef struct {
  int32_t bits;         /* 16, 8 or 4 */
  int32_t kv_heads;     /* 1..1024 */
  int32_t head_dim;     /* 64, 96, 128, 192 or 256 */
  int32_t page_size;    /* tokens a page: a power of two, at most 65536 */
  int64_t n_pages;      /* n_pages * page_size < 2^31 */
  void *d_k, *d_v;
  int64_t page_stride, head_stride, token_stride;
  void *d_k_par, *d_v_par;            /* NULL with 16 bits */
  int64_t par_page_stride, par_head_stride, par_token_stride;
} sph_kv_cache;

/* Write one key row and one value row per token and kv head into the slots d_slots (device int32[tokens]).
 * rope, if not NULL, rotates the keys on the way, and the queries d_q -> d_q_out (q_heads rows a token; both
 * NULL and q_heads 0 for none; without rope no queries are taken) in the same launch. d_k, d_v, d_q: device rows of dtype (fp16 or
 * fp32); d_q_out: fp16 rows, may be an fp16 d_q with the same strides. Quantising, per row and 32 channels of the
 * fp32 (rotated) values x: offset = fp16(min x), step = fp16((max x - offset)/(2^bits - 1)) (by the fp32 reciprocal; the next smaller number if
 * offset + (2^bits - 1) step would pass 65504),
 * q = clip(round((x - offset)/step), 0, 2^bits - 1), half to even, 0 for a step of 0; 32 channels with an entry that is not finite (or
 * too large for fp16) all read back as NaN. A slot outside the pool (such as -1 for padding) writes nothing; a position outside the
 * table rotates to NaN. Two tokens of one call must not share a slot. Asynchronous. */
sph_status sph_kv_append(const sph_kv_cache* cache, const sph_rope_desc* rope, sph_dtype dtype, int64_t tokens,
                         const void* d_k, int64_t k_token_stride, int64_t k_head_stride, const void* d_v,
                         int64_t v_token_stride, int64_t v_head_stride, const int32_t* d_slots, int32_t q_heads,
                         const void* d_q, int64_t q_token_stride, int64_t q_head_stride, void* d_q_out,
                         int64_t qo_token_stride, int64_t qo_head_stride, const int32_t* d_pos, void* stream);

/* sph_kv_append with positions along several axes: d_axes, n_axes, pos_stride and d_pos as in sph_rope_axes; rope must not be NULL. */
sph_status sph_kv_append_axes(const sph_kv_cache* cache, const sph_rope_desc* rope, const uint8_t* d_axes, int32_t n_axes,
                              int64_t pos_stride, sph_dtype dtype, int64_t tokens, const void* d_k, int64_t k_token_stride,
                              int64_t k_head_stride, const void* d_v, int64_t v_token_stride, int64_t v_head_stride,
                              const int32_t* d_slots, int32_t q_heads, const void* d_q, int64_t q_token_stride, int64_t q_head_stride,
                              void* d_q_out, int64_t qo_token_stride, int64_t qo_head_stride, const int32_t* d_pos, void* stream);

/* Read tokens back: d_k_out and d_v_out (device fp16[tokens][kv_heads][head_dim], contiguous) receive the
 * rows of the slots d_slots (device int32[tokens], any order, repeats allowed). A slot outside the pool reads as zeros. Asynchronous. */
sph_status sph_kv_read(const sph_kv_cache* cache, int64_t tokens, const int32_t* d_slots, void* d_k_out, void* d_v_out,
                       void* stream);

/* Attention of new tokens over a paged cache that already holds their keys and values (sph_kv_append
 * first): sequence b has d_seq_lens[b] tokens (0..max_len), of which the last n_b are new and ask. Token j of the
 * sequence is slot d_pages[b * pages_stride + j / page_size] * page_size + j % page_size. The query at
 * position p sees the tokens j <= p, and with window > 0 only j > p - window; o = sum_j softmax_j(scale
 * q.k_j) v_j, with query head h reading kv head h / (q_heads / kv_heads). A query that sees nothing,
 * or whose every score is -inf, gets zeros. Scores, the softmax's maximum and sum and the output are held in fp32; the weights
 * exp(s - max) are rounded to fp16 for the matrix cores, lifted so that those down to 2^-25 of the largest keep 11 bits and none
 * is off by more than 2^-36 of it.
 *
 * d_q, d_o: device fp16 rows [tokens][q_heads]. d_q_start: device int32[batch + 1], ascending from 0 to
 * `tokens`: sequence b's queries are tokens d_q_start[b]..d_q_start[b+1]-1, at most max_q of them; or NULL with
 * max_q = 1 and tokens = batch: one each. d_seq_lens: device int32[batch]; d_pages: device int32[batch][pages_stride], at least
 * ceil(max_len / page_size) entries each, of which only those below the sequence's length are read. max_len (0..2^30): the
 * host's bound of the lengths; the launch is planned for it. batch is 0..65536 and max_q 1..2^24; SPH_ERR_SHAPE, from the workspace
 * query too, where batch * kv_heads * ceil(max_q * group / 128) passes a launch's 2^24 workgroups. With up to 32 rows (max_q * group; 16 above 128
 * channels) a kv head and up to 512 sequences, keys are shared out by the lengths that the device holds; more sequences are a workgroup each
 * and kv head, however long, and more rows are shared out by max_q and max_len, which are therefore better close to the truth. d_lse: device fp32[tokens][q_heads], natural
 * logarithm of sum_j exp(scale q.k_j) (-inf where nothing is seen), or NULL. scale must be finite. d_ws: at
 * least sph_attention_workspace_bytes, 256-byte aligned, no initial contents; concurrent calls must not share one.
 * Keys and values that no query sees are never used, whatever they hold. Queries of a sequence whose length is outside 0..max_len, whose start and count are
 * outside their range, or that see a page outside the pool get NaN. Where d_q_start descends, several sequences may claim a token, which then gets
 * anything. Every sum runs in an order fixed by the
 * arguments, so repeated calls give bitwise identical results. Asynchronous. */
sph_status sph_attention(const sph_kv_cache* cache, int64_t batch, int64_t tokens, int32_t q_heads, const void* d_q,
                         int64_t q_token_stride, int64_t q_head_stride, const int32_t* d_q_start, int64_t max_q,
                         const int32_t* d_pages, int64_t pages_stride, const int32_t* d_seq_lens, int64_t max_len,
                         int64_t window, float scale, void* d_o, int64_t o_token_stride, int64_t o_head_stride,
                         float* d_lse, void* d_ws, size_t ws_bytes, void* stream);

/* Device workspace of sph_attention with these arguments on the current device (0 when it needs none): partial
 * outputs where a sequence's length is split between workgroups. */
sph_status sph_attention_workspace_bytes(const sph_kv_cache* cache, int64_t batch, int64_t tokens, int32_t q_heads,
                                         int64_t max_q, int64_t max_len, int64_t window, size_t* bytes);

/* sph_attention of sequences that share long prefixes (system prompts, documents, prompts with several answers), each prefix read once for all
 * of them. A sequence's own tokens are d_pages, d_seq_lens (own tokens, with the new ones, 0..max_len), q, o, d_q_start, max_q, scale and d_lse as in sph_attention
 * without a window; prefix g has d_prefix_lens[g] tokens (0..max_prefix) in d_prefix_pages[g * prefix_stride ..] (device int32[prefixes][prefix_stride],
 * rows of at least ceil(max_prefix / page_size)) and comes before the own tokens of sequences d_first[g]..d_first[g+1]-1: device
 * int32[prefixes + 1], ascending, prefixes 1..65536; sequences before d_first[0] or from the last on have none. Every query sees the
 * whole prefix, and its own tokens up to its position. d_first may be NULL with one prefix, of all sequences. max_group (1..65536; at least batch where d_first is
 * NULL): the host's bound of sequences behind a prefix, for which the launch is planned as for max_prefix, max_len and max_q: better close to the truth. Prefixes and own tokens
 * are pages of the same cache, and a page may be in any number of rows.
 * A sequence whose own values are wrong (see sph_attention), or whose prefix has a length outside 0..max_prefix, more tokens behind it than
 * max_group * max_q or a page outside the pool, gets NaN, and so does every sequence of a call whose d_first descends anywhere. Precision, empty rows and values that no row sees: as in sph_attention; repeated
 * calls give bitwise identical results. d_ws: at least sph_attention_shared_workspace_bytes, 256-byte aligned, no
 * initial contents; concurrent calls must not share one. Asynchronous. */
sph_status sph_attention_shared(const sph_kv_cache* cache, int64_t prefixes, const int32_t* d_first, int64_t max_group,
                                const int32_t* d_prefix_pages, int64_t prefix_stride, const int32_t* d_prefix_lens, int64_t max_prefix,
                                int64_t batch, int64_t tokens, int32_t q_heads, const void* d_q, int64_t q_token_stride,
                                int64_t q_head_stride, const int32_t* d_q_start, int64_t max_q, const int32_t* d_pages,
                                int64_t pages_stride, const int32_t* d_seq_lens, int64_t max_len, float scale, void* d_o,
                                int64_t o_token_stride, int64_t o_head_stride, float* d_lse, void* d_ws, size_t ws_bytes, void* stream);

/* Device workspace of sph_attention_shared with these arguments on the current device: the parts of every row, up to 32 rows (16 above 128 channels) a
 * sequence of as many as max_q of every sequence has, otherwise of `tokens`. SPH_ERR_SHAPE, from the call too, where batch * max_q * q_heads
 * passes 2^26 - 1 (with more than 20 parts a row 32 / head_dim of that), or the workgroups of prefixes and own tokens 2^24 - 1. */
sph_status sph_attention_shared_workspace_bytes(const sph_kv_cache* cache, int64_t prefixes, int64_t max_group, int64_t max_prefix,
                                                int64_t batch, int64_t tokens, int32_t q_heads, int64_t max_q, int64_t max_len,
                                                size_t* bytes);

/* How much attention every cached token got: for each token j of a sequence, the sum over the new tokens and query heads that see it of
 * exp(scale q.k_j - lse), their softmax's weight for it, added to what it got before (d_before). Arguments as in sph_attention (whose d_q, d_q_start, d_pages,
 * d_seq_lens, window and scale give the same weights); d_lse: device fp32[tokens][q_heads] as sph_attention writes it, -inf for rows that
 * see nothing. d_sums, d_before: device fp32 rows of max_len numbers and more for each sequence and kv head (heads = kv_heads), over its group
 * of query heads, or one row for each sequence (heads = 1), over all; strides in elements. d_before: NULL for zeros, or d_sums with the same strides, or rows
 * that do not overlap it. Entries from a sequence's length on, up to max_len, become 0 whatever they were, so that tokens added later start there.
 * Keys that no row sees are never used, whatever they hold. A sequence whose length, start or count is outside its range gets NaN, a token of a page outside
 * the pool that some row sees, too. Sums are held in fp32, in an order fixed by the arguments: repeated calls give bitwise
 * identical results. d_ws: at least sph_attention_weights_workspace_bytes, 256-byte aligned, no initial contents; concurrent calls must not share one.
 * SPH_ERR_SHAPE also where a launch would pass 2^24 workgroups: up to 32 new rows a kv head, one for every sequence, kv head and 128 to 512 tokens of max_len (by the
 * bytes of a token's key; with one sum for all heads one for every sequence and 16 to 64 tokens), otherwise for every sequence, kv head and 128 or 256. Asynchronous. */
sph_status sph_attention_weights(const sph_kv_cache* cache, int64_t batch, int64_t tokens, int32_t q_heads, const void* d_q,
                                 int64_t q_token_stride, int64_t q_head_stride, const int32_t* d_q_start, int64_t max_q,
                                 const int32_t* d_pages, int64_t pages_stride, const int32_t* d_seq_lens, int64_t max_len, int64_t window,
                                 float scale, const float* d_lse, int32_t heads, const float* d_before, int64_t before_seq_stride,
                                 int64_t before_head_stride, float* d_sums, int64_t sums_seq_stride, int64_t sums_head_stride, void* d_ws,
                                 size_t ws_bytes, void* stream);

/* Device workspace of sph_attention_weights with these arguments (0 when it needs none): sums of several heads, or of some of the rows, where they are joined. */
sph_status sph_attention_weights_workspace_bytes(const sph_kv_cache* cache, int64_t batch, int64_t tokens, int32_t q_heads, int32_t heads,
                                                 int64_t max_q, int64_t max_len, int64_t window, size_t* bytes);

/* Shrink sequences to `keep` tokens (1..2^30): the first `first` and the last `recent` of them (together at most keep) and, of the
 * others, those with the largest sums, equal ones by the lower index, NaN above all numbers. Kept tokens stay in order: the i-th becomes token
 * i. Sequences of `keep` tokens or fewer keep all. d_sums: device fp32, a sum for every token of a sequence (rows of at least max_len;
 * strides in elements), for each kv head (heads = kv_heads), whose tokens are then chosen and moved by themselves, or one for
 * all (heads = 1). Such sums are sph_attention_weights' results.
 *
 * d_pages, pages_stride, d_seq_lens, max_len: as in sph_attention (batch 0..65536). d_to_pages: device int32[batch][to_stride], the
 * pages that receive the tokens, at least ceil(min(keep, max_len) / page_size) of each row. Either d_pages itself (and to_stride equal to
 * pages_stride): tokens move within their pages, which no other sequence may hold from the first evicted token on; or other pages, none of
 * them in d_pages or twice among the first that receive tokens, and then d_pages' are only read (they may be shared). Keys stay rotated as they were.
 *
 * d_new_lens: device int32[batch], min(length, keep); may be d_seq_lens. d_new_sums: device fp32 rows of new_width (min(keep, max_len)..2^30), apart from each
 * other: the kept tokens' sums, then zeros; may be d_sums with the same strides, otherwise must not overlap it. d_kept: device int32[batch][heads][keep],
 * which tokens were kept, in order, then -1 (keep above max_len evicts nothing, as max_len does with first and recent 0, whose rows are shorter). A sequence whose length is outside 0..max_len stays as it is, with NaN for its
 * new sums and -1 for kept. A token of a page outside the pool is NaN in its new place; nothing is written to such a page.
 * Results do not depend on the launch. SPH_ERR_SHAPE also where batch * heads passes 2^22 - 1, or a launch 2^32 threads. Asynchronous. */
sph_status sph_kv_evict(const sph_kv_cache* cache, int64_t batch, const int32_t* d_pages, int64_t pages_stride, const int32_t* d_seq_lens,
                        int64_t max_len, const float* d_sums, int32_t heads, int64_t sums_seq_stride, int64_t sums_head_stride,
                        int64_t keep, int64_t recent, int64_t first, const int32_t* d_to_pages, int64_t to_stride, int32_t* d_new_lens,
                        float* d_new_sums, int64_t new_width, int64_t new_seq_stride, int64_t new_head_stride, int32_t* d_kept,
                        void* stream);

/* Whether (dir_bits, radius_bits) is one of the built-in formats: 1 yes, 0 no. */
int sph_format_supported(const sph_format* fmt);

/* Static, human-readable name of a status code. */
const char* sph_status_str(sph_status s);

#ifdef __cplusplus
}
#endif

#endif /* SPH_H */
