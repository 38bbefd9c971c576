/*
 * torq.h -- C ABI of the B200 (sm_100a) hot path of TORQ's rotated-MXFP4 linear layer.
 *
 * The path is the paper's online inference procedure (Algorithm 3): a token's d features are
 * viewed as d/32 blocks of 32 (step 1), multiplied by the inter-block rotation (step 2) and by
 * the intra-block rotation of each block (step 3), quantized per block to MXFP4 (step 4, Eq. 1)
 * and handed to the next linear layer whose weights already carry the inverse rotation and are
 * themselves MXFP4 (step 5, option B "weight fusion").
 *
 * Conventions for every entry point
 *   - All data pointers are DEVICE pointers owned by the caller; the library allocates nothing
 *     and keeps no reference after the call returns.  `stream` is a cudaStream_t passed as
 *     void* (NULL = the legacy default stream).  Calls only enqueue work; they never synchronise.
 *   - Tokens are rows (row-vector convention): Z = X . R_inter, then per block Z_b . R_intra[b].
 *   - bf16 = bfloat16, u8 = unsigned byte.  Matrices are row-major, densely packed.
 *   - MXFP4 codes: 4 bits per element = sign<<3 | e2m1 magnitude index over
 *     {0, 0.5, 1, 1.5, 2, 3, 4, 6}; two codes per byte, the even element in the low nibble.
 *   - Scales: one E8M0 byte per (row, 32-element block), byte = e + 127 with
 *     e = clamp(floor(log2 amax) - 2, -127, 127) (amax == 0 -> byte 0), stored in the tiled
 *     layout the block-scaled tensor-core instruction reads (see torq_scale_offset).  A scale
 *     buffer always has torq_scales_bytes(rows, k) bytes: rows are padded to a multiple of 128
 *     and K-blocks to a multiple of 4.  Producers in this library write 0x00 (2^-127) into the
 *     padding rows; consumers never let padding reach a stored output.
 *   - Rotations and weights (R_inter, R_intra, Wq, Wn, W8 and their scales) are constants of the layer.  The tensor-core
 *     kernels (rotations, GEMMs, products) may start reading them while kernels launched before on the same stream are
 *     still running (everything else waits for these), so whatever writes them must have COMPLETED before.  Put between
 *     producing them and the first call a stream or device synchronisation, a wait for an event of the other stream that
 *     they were produced on, or a kernel that keeps its neighbours apart: any that is launched without programmatic
 *     stream serialization (torch's, this library's quantizers and weight-side helpers) or torq_add_rmsnorm*.  The
 *     rotations, the GEMMs and the products themselves do not count: one of them may run beside both the kernel before
 *     it and the kernel behind it.
 *   - Return value: TORQ_OK or a host-detected error; nothing is launched on error.  Conditions
 *     only the device can see (a bounded wait that ran out) are latched in an error word read by
 *     torq_last_device_error(); a kernel that hits one stops issuing work, drains and returns --
 *     it never traps.  Non-finite inputs are outside the contract (results unspecified, no hang).
 */
#ifndef TORQ_H_
#define TORQ_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  TORQ_OK = 0,
  TORQ_ERR_NULL = 1,       /* a required pointer is NULL */
  TORQ_ERR_SHAPE = 2,      /* a size violates the stated divisibility / range rules */
  TORQ_ERR_ALIGN = 3,      /* a pointer is not 16-byte aligned */
  TORQ_ERR_ARCH = 4,       /* current device is not compute capability 10.x */
  TORQ_ERR_LAUNCH = 5,     /* CUDA reported an error while encoding descriptors or launching */
  TORQ_ERR_TIMEOUT = 6,    /* (device error word) a bounded wait inside a kernel ran out */
  TORQ_ERR_WORKSPACE = 7,  /* workspace missing or smaller than torq_workspace_bytes() */
  TORQ_ERR_PAGE = 8        /* (device error word) a page number or a length of a key/value cache is out of range */
} torq_status;

typedef enum { TORQ_F32 = 0, TORQ_BF16 = 1 } torq_dtype;

/* Algorithm 3 steps 1-4 (rotation as in Section 5: R = inter then intra; quantizer Eq. 1).
 *   X         [M, d]        bf16
 *   R_inter   [d, d]        bf16, y[m,j] = sum_i x[m,i] R_inter[i,j]; NULL = identity
 *   R_intra   [d/32,32,32]  bf16, z[m,32b+j] = sum_i y[m,32b+i] R_intra[b][i][j]; NULL = identity
 *   out_codes [M, d/2]      u8
 *   out_scales              torq_scales_bytes(M, d) bytes, tiled layout
 * Requires M >= 1, d >= 32, d % 32 == 0, 16-byte aligned pointers.  Accumulation is fp32
 * (inter: tensor cores with exact bf16 products; intra: fp32 FMAs in index order).
 * When R_inter is NULL the call runs the quantize-only kernel (plus the intra step if given). */
torq_status torq_rotate_quantize(const void* X, const void* R_inter, const void* R_intra,
                                 int64_t M, int64_t d, void* out_codes, void* out_scales,
                                 void* stream);

/* Algorithm 3 steps 1-4 with the rotation in the paper's own structure (Section 5; App. A.7 counts
 * B^2 + K^2 parameters and O(B^2 K) + O(B K^2) work per token): ONE inter-block matrix R_B that
 * mixes the B = d/32 blocks of a token, the same for each of the 32 positions, and ONE intra-block
 * matrix shared by all blocks.  Per token, with X the token's [B, 32] reshape:
 *   Y = R_B X        y[32 b' + k] = sum_b  R_B[b'][b] x[32 b + k]
 *   Z = Y R_intra    z[32 b' + j] = sum_k  y[32 b' + k] R_intra[k][j]
 * then Eq. 1 as in torq_rotate_quantize (same output layouts).  Equivalent to torq_rotate_quantize
 * with R_inter = kron(R_B^T, I_32) and R_intra repeated for every block, at 2 d (B + 32) instead of
 * 2 d^2 flop per token.
 *   X [M, d] bf16;  R_B [d/32, d/32] bf16 (required);  R_intra [32, 32] bf16 or NULL = identity
 * Requires d % 256 == 0, 16-byte aligned pointers.  fp32 accumulation: step 2 on the tensor cores
 * with exact bf16 products, step 3 on the tensor cores as well, with y split exactly into three
 * bf16 terms against the bf16 R_intra.  R_B is a constant of the layer like R_inter (see the
 * conventions above). */
torq_status torq_rotate_quantize_structured(const void* X, const void* R_B, const void* R_intra,
                                            int64_t M, int64_t d, void* out_codes, void* out_scales,
                                            void* stream);

/* Algorithm 3 steps 1-5 with the structured rotation: torq_rotate_quantize_structured into
 * `workspace` (codes [M, d/2], then 256-byte aligned the tiled scales; >= M*d/2 rounded up to 256
 * plus torq_scales_bytes(M, d) bytes, 256-byte aligned), then torq_mxfp4_gemm against weights that
 * were rotated with the same R_B and R_intra offline.  dbg_codes / dbg_scales as in
 * torq_rotated_linear.  Requires d % 256 == 0 and N % 8 == 0. */
torq_status torq_rotated_linear_structured(const void* X, const void* R_B, const void* R_intra,
                                           const void* Wq, const void* Ws, int64_t M, int64_t d,
                                           int64_t N, void* Y, torq_dtype y_dtype, void* workspace,
                                           size_t workspace_bytes, void* dbg_codes, void* dbg_scales,
                                           void* stream);

/* Algorithm 3 step 5 (option B): Y[m,n] = sum_k a^[m,k] w^[n,k], a^/w^ the dequantized MXFP4
 * values (codeword x 2^e), fp32 accumulation on the block-scaled FP4 tensor cores.
 *   Aq [M, K/2] u8, As scales of A (tiled, torq_scales_bytes(M, K))
 *   Wq [N, K/2] u8 (the fused weight W' stored with K contiguous), Ws (tiled, (N, K))
 *   Y  [M, N] row-major of y_dtype
 * Requires M,N >= 1, K % 128 == 0, N % 8 == 0, 16-byte aligned pointers. */
torq_status torq_mxfp4_gemm(const void* Aq, const void* As, const void* Wq, const void* Ws,
                            int64_t M, int64_t N, int64_t K, void* Y, torq_dtype y_dtype,
                            void* stream);

/* Algorithm 3 steps 1-5 in one call: rotate, quantize, multiply.  The quantized activations live
 * in `workspace` (>= torq_workspace_bytes(M, d, N) bytes, 256-byte aligned), laid out as codes
 * [M, d/2] followed (256-byte aligned) by the tiled scales; pass dbg_codes / dbg_scales non-NULL
 * to also receive copies of them.  Up to 256 tokens the rotation is one kernel that splits its
 * contraction over thread-block clusters and adds the partial sums on chip, in a fixed order.
 * The rotation is one launch, the same kernels as torq_rotate_quantize; beyond two waves of 256 x 256
 * tiles with d > 4096 a last wave of a few tiles is a launch of its own.  The workspace size includes room
 * that no kernel uses any more (it once held partial sums).
 * Requires d % 128 == 0 and N % 8 == 0. */
torq_status torq_rotated_linear(const void* X, const void* R_inter, const void* R_intra,
                                const void* Wq, const void* Ws, int64_t M, int64_t d, int64_t N,
                                void* Y, torq_dtype y_dtype, void* workspace,
                                size_t workspace_bytes, void* dbg_codes, void* dbg_scales,
                                void* stream);

/* The whole layer for callers that must not allocate device memory.  (No counterpart in the
 * paper: this exists for the library's users, not for the method.)
 *
 * torq_rotated_linear needs a scratch buffer for the quantized activations, and normally the
 * caller allocates it.  Some callers cannot: a plug-in or custom operator that an inference
 * engine hands nothing but input and output pointers; a serving process whose whole device
 * budget was given to a KV-cache pool at start-up, where a late cudaMalloc fails or evicts;
 * a latency-critical decode loop, where the implicit device-wide synchronisation of
 * cudaMalloc / cudaFree is not acceptable.  For them this entry point keeps the scratch in a
 * fixed array of TORQ_STATIC_WORKSPACE_BYTES that is part of the library image: every device
 * that loads the library holds those bytes from load until the process exits, used or not.
 * The call itself allocates nothing and frees nothing, on the host or the device, and neither
 * does anything it calls.
 *
 * Same arguments, layouts and results as torq_rotated_linear without its workspace and debug
 * parameters.  A problem whose quantized activations (M * d / 2 code bytes rounded up to 256,
 * plus torq_scales_bytes(M, d)) exceed TORQ_STATIC_WORKSPACE_BYTES is refused with
 * TORQ_ERR_WORKSPACE before anything is launched (for example M = 2048, d = 14336 fits;
 * M = 8192, d = 5120 does not).
 *
 * First call on each device: the library looks up the array's device address (and, if no other
 * entry point ran before, performs the one-time per-device set-up every entry point shares).
 * Make that first call during start-up, outside any stream capture.
 *
 * All calls on a device share the one array, and it keeps whatever the previous call left.
 * Nothing in it has to start at zero: the rotation step rewrites every code and scale byte the
 * multiplication step reads before it reads them, so stale contents are never observed.  But two
 * calls that can overlap on the GPU (different streams, or different host threads without
 * ordering between them) write the same bytes and race; run them in one stream or order them
 * with events.  Calls on different devices do not interact. */
#define TORQ_STATIC_WORKSPACE_BYTES (16u << 20)
torq_status torq_rotated_linear_static(const void* X, const void* R_inter, const void* R_intra,
                                       const void* Wq, const void* Ws, int64_t M, int64_t d,
                                       int64_t N, void* Y, torq_dtype y_dtype, void* stream);

/* Eq. 1 alone: quantize Z [M, d] (fp32 or bf16) to MXFP4.  On fp32 input the result is defined
 * bit for bit (round to nearest even on the e2m1 grid, saturation to +-6, sign bit kept). */
torq_status torq_quantize_mxfp4(const void* Z, torq_dtype z_dtype, int64_t M, int64_t d,
                                void* out_codes, void* out_scales, void* stream);

/* Scale-factor layout (not in the paper; fixed by the FP4 tensor-core instruction): 512-byte tiles
 * of 128 rows x 4 K-blocks, tiles ordered row-tile major; inside a tile
 *   byte = (row % 32) * 16 + ((row % 128) / 32) * 4 + (kblock % 4).
 * Host-side pure functions. */
size_t torq_scales_bytes(int64_t rows, int64_t k);
size_t torq_scale_offset(int64_t row, int64_t kblock, int64_t k);
size_t torq_workspace_bytes(int64_t M, int64_t d, int64_t N);

/* Re-tile a plain [rows, k/32] scale matrix into the layout above (padding bytes := 0x00). */
torq_status torq_swizzle_scales(const void* linear_scales, int64_t rows, int64_t k, void* out,
                                void* stream);

/* Offline helper for the weight side of step 5 (W' = R~^T W, R~ = R_inter . blockdiag(R_intra)):
 * writes R~ [d, d] as fp32 computed in fp32 from the bf16 inputs.  d % 32 == 0. */
torq_status torq_merge_rotations(const void* R_inter, const void* R_intra, int64_t d,
                                 void* R_merged_f32, void* stream);

/* The same merged matrix rounded once (nearest even) to bfloat16: the operand of the one-GEMM form
 * of the rotation, torq_rotate_quantize(X, R_merged, NULL), which Section 5 writes as
 * R = R_inter (x) R_intra.  That form is a different quantized operator from the two-level one (the
 * rounding of R~ to bfloat16 moves about one code in a thousand). */
torq_status torq_merge_rotations_bf16(const void* R_inter, const void* R_intra, int64_t d,
                                      void* R_merged_bf16, void* stream);

/* Algorithm 3 step 5, option B ("weight fusion"), the offline weight side: W' = R~^T W with
 * R~ = R_inter . blockdiag(R_intra), stored as [N, d] (K = d contiguous), then quantized along K
 * (Section 6.1: weights and activations are both quantized).
 *   W        [d, N] float32 row-major (out = x W)
 *   R_inter  [d, d] bf16 (required), R_intra [d/32, 32, 32] bf16 or NULL = identity
 *   Wq [N, d/2] u8, Ws torq_scales_bytes(N, d) bytes: the operands torq_mxfp4_gemm takes
 *   workspace: torq_prepare_weights_workspace_bytes(d, N) bytes (10 N d, rounded up), 256-byte aligned
 * Row n of W' is (W^T[n, :] R_inter) R_intra per block, i.e. steps 2-3 applied to the rows of W^T:
 * W^T is split exactly into three bfloat16 terms and the rotation kernels contract all of them against
 * R_inter in one fp32 accumulation on the tensor cores (every product exact); the intra-block step
 * is fp32 FMAs; the result is quantized by the kernel behind torq_quantize_mxfp4.  d % 64 == 0.
 * Three launches (split, rotation, quantizer).  Not on the inference path. */
size_t torq_prepare_weights_workspace_bytes(int64_t d, int64_t N);
torq_status torq_prepare_weights(const void* W, const void* R_inter, const void* R_intra, int64_t d,
                                 int64_t N, void* Wq, void* Ws, void* workspace, size_t workspace_bytes,
                                 void* stream);

/* ---- NVFP4 variant (the paper's format study, Section 6 "Generalizability to Other Formats") -----
 * The same layer with NVFP4 operands: e2m1 codes as above, blocks of 16 along K, one FP8 E4M3
 * scale byte per (row, block) and one float32 scale per tensor; x^ = codeword * e4m3(byte) *
 * tensor_scale.  The paper names the format and reports accuracies only; the arithmetic below is
 * the library's definition (each step one IEEE float32 operation, round to nearest even):
 *   c = 1 / (6 tensor_scale);  byte = E4M3(amax_block * c), saturating at 448;
 *   r = 1 / (e4m3(byte) * tensor_scale), or 0 when byte == 0;  code = e2m1(z * r), saturating at
 *   6, sign of z kept.
 * The tensor scale is an input (calibrated beforehand; amax(tensor) / (6 * 448) uses the whole
 * E4M3 range) and must be positive and finite.  Scale bytes use the tiled layout of
 * torq_scale_offset with 16-element blocks: a buffer has torq_nvfp4_scales_bytes(rows, k) bytes,
 * the byte of (row, block c) sits at torq_scale_offset(row, c, 2 * k); padding bytes are 0x00
 * (E4M3 zero).  The intra-block rotation acts inside a quantization block, so it is [d/16, 16, 16]
 * here; the rotation kernels take it in 32-wide block-diagonal form, made once by
 * torq_expand_intra16. */
size_t torq_nvfp4_scales_bytes(int64_t rows, int64_t k);
size_t torq_nvfp4_workspace_bytes(int64_t M, int64_t d, int64_t N);

/* R_intra16 [d/16, 16, 16] bf16 -> R_intra32 [d/32, 32, 32] bf16: blocks 2b and 2b+1 on the diagonal of
 * block b, zeros elsewhere.  d % 32 == 0. */
torq_status torq_expand_intra16(const void* R_intra16, int64_t d, void* R_intra32, void* stream);

/* torq_prepare_weights in NVFP4 (R_intra32 as for torq_rotate_quantize_nvfp4).  The tensor scale is
 * max |W'| / (6 * 448) (one float32 division), found by a reduction on the device and written to
 * *tensor_scale (HOST pointer): this call therefore synchronises `stream` once, between the
 * rotation and the quantization.  An all-zero W' has no scale: TORQ_ERR_SHAPE.
 * Ws: torq_nvfp4_scales_bytes(N, d) bytes. */
torq_status torq_prepare_weights_nvfp4(const void* W, const void* R_inter, const void* R_intra32, int64_t d,
                                       int64_t N, void* Wq, void* Ws, float* tensor_scale, void* workspace,
                                       size_t workspace_bytes, void* stream);

/* Quantize Z [M, d] (fp32 or bf16) to NVFP4; d % 16 == 0.  Bit-exact by the definition above. */
torq_status torq_quantize_nvfp4(const void* Z, torq_dtype z_dtype, int64_t M, int64_t d,
                                float tensor_scale, void* out_codes, void* out_scales, void* stream);

/* Algorithm 3 steps 1-4 with the NVFP4 quantizer.  X [M, d] bf16; R_inter [d, d] bf16 (required);
 * R_intra32 [d/32, 32, 32] bf16 or NULL = identity; d % 32 == 0.  Outputs as torq_quantize_nvfp4. */
torq_status torq_rotate_quantize_nvfp4(const void* X, const void* R_inter, const void* R_intra32,
                                       int64_t M, int64_t d, float tensor_scale, void* out_codes,
                                       void* out_scales, void* stream);

/* torq_rotate_quantize_structured with the NVFP4 quantizer at its end: the rotation in the paper's own
 * structure (R_B across blocks, one shared R_intra [32, 32] -- for a 16-wide intra rotation its two
 * 16 x 16 blocks on the diagonal -- or NULL) and 16-element blocks with E4M3 scales.  d % 256 == 0. */
torq_status torq_rotate_quantize_structured_nvfp4(const void* X, const void* R_B, const void* R_intra,
                                                  int64_t M, int64_t d, float tensor_scale,
                                                  void* out_codes, void* out_scales, void* stream);

/* Algorithm 3 step 5 on NVFP4 operands: Y[m,n] = a_tensor_scale * w_tensor_scale *
 * sum_k (code * e4m3 scale)_a[m,k] (code * e4m3 scale)_w[n,k], fp32 accumulation on the tensor
 * cores (kind::mxf4nvf4, 16-element blocks).  Shapes and layouts as torq_mxfp4_gemm with
 * 16-element blocks: K % 128 == 0, N % 8 == 0. */
torq_status torq_nvfp4_gemm(const void* Aq, const void* As, float a_tensor_scale, const void* Wq,
                            const void* Ws, float w_tensor_scale, int64_t M, int64_t N, int64_t K,
                            void* Y, torq_dtype y_dtype, void* stream);

/* Steps 1-5 in NVFP4: torq_rotate_quantize_nvfp4 into `workspace` (at least
 * torq_nvfp4_workspace_bytes(M, d, N) bytes, 256-byte aligned), then torq_nvfp4_gemm.  Launches
 * as in torq_rotated_linear.  d % 128 == 0, N % 8 == 0. */
torq_status torq_rotated_linear_nvfp4(const void* X, const void* R_inter, const void* R_intra32,
                                      float x_tensor_scale, const void* Wq, const void* Ws,
                                      float w_tensor_scale, int64_t M, int64_t d, int64_t N, void* Y,
                                      torq_dtype y_dtype, void* workspace, size_t workspace_bytes,
                                      void* dbg_codes, void* dbg_scales, void* stream);

/* ---- MXINT4 variant (the paper's format study, Section 6 "Generalizability to Other Formats") ----
 * The same layer with integer elements: blocks of 32 along K, one E8M0 scale byte per block by
 * the same rule and in the same tiled layout as MXFP4 (torq_scales_bytes / torq_scale_offset),
 * elements q = clamp(rint(z / 2^e), -7, 7) (rint = round half to even; z / 2^e is exact, so the
 * quantizer is bit-exact by definition); decoding x^ = q * 2^e.
 * Two forms of the codes:
 *   stored form   [rows, k/2] bytes: two's-complement nibbles, even element in the low nibble;
 *   operand form  [rows, k]   bytes: the FP8 E4M3 byte whose value is q (a zero may carry a sign
 *                 bit).  The tensor cores of this GPU have no 4-bit integer path; the GEMM runs
 *                 as tcgen05.mma kind::mxf8f6f4 on E4M3 operands with the E8M0 block scales.
 *                 Integer products and their power-of-two scales are exact in it; accumulation
 *                 is fp32.
 * The rotation entry points write the operand form directly.  All pointers device, 16-byte
 * aligned; errors as elsewhere in this header.  The paper has no worked example of this format. */
size_t torq_mxint4_workspace_bytes(int64_t M, int64_t d, int64_t N);

/* torq_prepare_weights in MXINT4: Wn [N, d/2] stored form and / or W8 [N, d] operand form (either
 * may be NULL, not both), Ws torq_scales_bytes(N, d) bytes. */
torq_status torq_prepare_weights_mxint4(const void* W, const void* R_inter, const void* R_intra, int64_t d,
                                        int64_t N, void* Wn, void* W8, void* Ws, void* workspace,
                                        size_t workspace_bytes, void* stream);

/* Quantize Z [M, d] (fp32 or bf16), d % 32 == 0.  packed != 0: stored form, out_codes [M, d/2];
 * packed == 0: operand form, out_codes [M, d].  out_scales: torq_scales_bytes(M, d) bytes. */
torq_status torq_quantize_mxint4(const void* Z, torq_dtype z_dtype, int64_t M, int64_t d, int packed,
                                 void* out_codes, void* out_scales, void* stream);

/* Stored form [rows, k/2] -> operand form [rows, k] (nibble -8 becomes the E4M3 byte of -8). */
torq_status torq_mxint4_expand(const void* packed, int64_t rows, int64_t k, void* out_bytes, void* stream);

/* Algorithm 3 steps 1-4 with the MXINT4 quantizer.  X [M, d] bf16; R_inter [d, d] bf16 (required);
 * R_intra [d/32, 32, 32] bf16 or NULL = identity; d % 32 == 0.  out_bytes [M, d] operand form. */
torq_status torq_rotate_quantize_mxint4(const void* X, const void* R_inter, const void* R_intra, int64_t M,
                                        int64_t d, void* out_bytes, void* out_scales, void* stream);

/* torq_rotate_quantize_structured with the MXINT4 quantizer at its end (R_B [d/32, d/32] bf16, one
 * shared R_intra [32, 32] bf16 or NULL; d % 256 == 0).  out_bytes [M, d] operand form. */
torq_status torq_rotate_quantize_structured_mxint4(const void* X, const void* R_B, const void* R_intra,
                                                   int64_t M, int64_t d, void* out_bytes, void* out_scales,
                                                   void* stream);

/* Algorithm 3 step 5 on MXINT4 operands: Y[m,n] = sum_k a^[m,k] w^[n,k].  A8 [M, K], W8 [N, K]
 * operand form; As, Ws tiled E8M0 scales; K % 128 == 0, N % 8 == 0; Y [M, N] fp32 or bf16. */
torq_status torq_mxint4_gemm(const void* A8, const void* As, const void* W8, const void* Ws, int64_t M,
                             int64_t N, int64_t K, void* Y, torq_dtype y_dtype, void* stream);

/* Steps 1-5 in MXINT4: torq_rotate_quantize_mxint4 into `workspace` (at least
 * torq_mxint4_workspace_bytes(M, d, N) bytes, 256-byte aligned), then torq_mxint4_gemm.  Launches
 * as in torq_rotated_linear.  dbg_bytes
 * [M, d] / dbg_scales, when not NULL, receive copies of the quantized activations.
 * d % 128 == 0, N % 8 == 0. */
torq_status torq_rotated_linear_mxint4(const void* X, const void* R_inter, const void* R_intra, const void* W8,
                                       const void* Ws, int64_t M, int64_t d, int64_t N, void* Y,
                                       torq_dtype y_dtype, void* workspace, size_t workspace_bytes,
                                       void* dbg_bytes, void* dbg_scales, void* stream);

/* ---- operators around the layer (no counterpart in the paper: what a transformer block does next to its 4-bit products) ----
 * Root-mean-square norm with the residual's addition:
 *   h = x + r (float32);  y = h / sqrt(mean_d(h^2) + eps) * w (float32)
 *   X [M, d] of x_dtype; residual [M, d] of r_dtype or NULL (h = x); residual_out [M, d] of r_dtype gets h, rounded once; it may be
 *   `residual` itself, or X where the types agree, and is NULL exactly where residual is; weight [d] bf16; eps >= 0.
 * The norm is taken of h before it is rounded.  torq_add_rmsnorm: out [M, d] bf16, rounded once: the X of the rotation and
 * matvec entry points.  torq_add_rmsnorm_mxfp8: out_bytes [M, d] FP8 E4M3 and out_scales, torq_scales_bytes(M, d) bytes in the tiled
 * layout, one E8M0 byte per 32 elements: byte = e + 127, e = clamp(floor(log2 amax) - 8, -127, 127) (amax == 0 -> byte 0), codes
 * E4M3(y / 2^e) to nearest even, saturating at 448, padding bytes 0x00: the A operand that torq_mxint4_gemm and
 * torq_mxint4_gated_gemm take (any E4M3 bytes with E8M0 scales are).  The squares of a row must sum to less than float32's largest value.
 * Squares below 2^-126 lose bits: a row whose mean square and eps are as small as that is not normalised (zeros with eps = 0: not a number).
 * 32 <= d <= 16384, d % 32 == 0.  One launch.  Apart from residual_out the outputs overlap nothing. */
torq_status torq_add_rmsnorm(const void* X, torq_dtype x_dtype, const void* residual, void* residual_out, torq_dtype r_dtype,
                             const void* weight, float eps, int64_t M, int64_t d, void* out, void* stream);
torq_status torq_add_rmsnorm_mxfp8(const void* X, torq_dtype x_dtype, const void* residual, void* residual_out, torq_dtype r_dtype,
                                   const void* weight, float eps, int64_t M, int64_t d, void* out_bytes, void* out_scales,
                                   void* stream);

/* Products of few tokens with 4-bit weights and activations that stay in bfloat16 (weights that were quantized without a rotation, or
 * activations that were rotated before): Y[m,n] = sum_k x[m,k] w^[n,k], w^ the dequantized weights.
 *   X [M, K] bf16;  Wq [N, K/2], Ws: the weight operands of torq_mxfp4_gemm / torq_nvfp4_gemm; MXINT4: Wn [N, K/2] in the STORED form
 *   (half the bytes of the operand form torq_mxint4_gemm takes), nibble -8 included;  Y [M, N] of y_dtype
 *   workspace: torq_matvec_workspace_bytes(M, N, K) bytes, 256-byte aligned; NULL where that is 0 (up to 4 tokens, unless a CTA's range of K
 *   is long)
 * Products exact, sums float32.  The tensor cores do not take bfloat16 beside 4-bit weights, so x is split exactly into eight 3-bit digits,
 * each an FP4 operand, after it has been rounded to a multiple of 2^-21 of the power of two at or below the largest magnitude of its block of
 * 32 (NVFP4: 16, and a block's counts as 2^-17 of the largest in the token at least): elements down to 2^-14 of the block's largest keep all
 * their bits, nothing is off by more than 2^-22 of it (which is more than a float32 sum loses where the large element meets a weight of zero:
 * 2^-6 beside one of 2^16).  What is smaller than 2^-106 counts as zero in part or whole; MXINT4: a token with a magnitude of 2^126 or more
 * is not a number.  The digits' magnitudes add up to at most three times (MXINT4: nine times) those of the products they stand for: sums
 * of magnitudes that come as near as that to float32's largest may overflow.
 * Weights are read from HBM once, for 8 to 32 tokens at a time, the others finding them in the L2: made for decoding, any M <= 2^18 is served.  K % 128 == 0, K <= 65536, N % 8 == 0.  One launch without a workspace, else two; two calls that may overlap need a workspace
 * each.  Y and the workspace overlap no operand and not each other, here and in the entry points below. */
size_t torq_matvec_workspace_bytes(int64_t M, int64_t N, int64_t K);
torq_status torq_mxfp4_matvec(const void* X, const void* Wq, const void* Ws, int64_t M, int64_t N, int64_t K, void* Y, torq_dtype y_dtype,
                              void* workspace, size_t workspace_bytes, void* stream);
torq_status torq_nvfp4_matvec(const void* X, const void* Wq, const void* Ws, float w_tensor_scale, int64_t M, int64_t N, int64_t K, void* Y,
                              torq_dtype y_dtype, void* workspace, size_t workspace_bytes, void* stream);
torq_status torq_mxint4_matvec(const void* X, const void* Wn, const void* Ws, int64_t M, int64_t N, int64_t K, void* Y, torq_dtype y_dtype,
                               void* workspace, size_t workspace_bytes, void* stream);

/* The gated pair of projections of a feed-forward block, in one call:
 *   Y[m,n] = silu(g) u,  g = sum_k x[m,k] w^[n,k],  u = sum_k x[m,k] w^[N+n,k],  silu(g) = g / (1 + exp(-g)), float32 up to Y
 * (a gate below -87.3, whose silu lies between -1.1e-36 and 0, counts as zero).
 * Both projections are one weight matrix of 2 N rows, gate rows first (Wq [2N, K/2], Ws of 2 N rows); Y [M, N] of y_dtype.
 * Otherwise as the products above.  N % 128 == 0. */
torq_status torq_mxfp4_gated_matvec(const void* X, const void* Wq, const void* Ws, int64_t M, int64_t N, int64_t K, void* Y,
                                    torq_dtype y_dtype, void* workspace, size_t workspace_bytes, void* stream);
torq_status torq_nvfp4_gated_matvec(const void* X, const void* Wq, const void* Ws, float w_tensor_scale, int64_t M, int64_t N, int64_t K,
                                    void* Y, torq_dtype y_dtype, void* workspace, size_t workspace_bytes, void* stream);
torq_status torq_mxint4_gated_matvec(const void* X, const void* Wn, const void* Ws, int64_t M, int64_t N, int64_t K, void* Y,
                                     torq_dtype y_dtype, void* workspace, size_t workspace_bytes, void* stream);

/* The same on quantized activations, the activation and the product in the epilogue of the block-scaled GEMM (M rows, from
 * decoding to prefill): operands as torq_mxfp4_gemm, torq_nvfp4_gemm and torq_mxint4_gemm take them, weights of 2 N rows, gate
 * rows first; Y [M, N].  The A operand of the MXINT4 form may be any E4M3 bytes with E8M0 scales, torq_add_rmsnorm_mxfp8's among
 * them.  N % 128 == 0, K % 128 == 0.  One launch. */
torq_status torq_mxfp4_gated_gemm(const void* Aq, const void* As, const void* Wq, const void* Ws, int64_t M, int64_t N, int64_t K, void* Y,
                                  torq_dtype y_dtype, void* stream);
torq_status torq_nvfp4_gated_gemm(const void* Aq, const void* As, float a_tensor_scale, const void* Wq, const void* Ws, float w_tensor_scale,
                                  int64_t M, int64_t N, int64_t K, void* Y, torq_dtype y_dtype, void* stream);
torq_status torq_mxint4_gated_gemm(const void* A8, const void* As, const void* W8, const void* Ws, int64_t M, int64_t N, int64_t K, void* Y,
                                   torq_dtype y_dtype, void* stream);

/* ---- calibration of the inter-block rotation (Section 5.1; offline, not on the inference path) ----
 * Covariance across the blocks of a token, pooled over the T calibration tokens and the 32
 * positions of a block (block means taken as zero, as Section 5.1 assumes):
 *   Sigma[b, b'] = (1 / (32 T)) sum_t sum_k x[t, 32 b + k] x[t, 32 b' + k]
 * X [T, d] bf16, Sigma_f64 [d/32, d/32] float64 (written whole); d % 32 == 0.  float64 accumulation. */
torq_status torq_block_covariance(const void* X, int64_t T, int64_t d, void* Sigma_f64, void* stream);

/* Algorithm 1 (Givens rotations for variance equalisation): an orthogonal Q with
 * diag(Q Sigma Q^T) = (tr Sigma / B) 1 up to the absolute threshold eps -- the matrix R_B that
 * torq_rotate_quantize_structured applies across the blocks of a token.  Departures from the
 * listing, which cannot reach its own stated output as printed: the rotation angle is the one that
 * sets sigma_ii to the target exactly (the printed angle zeroes sigma_ij instead and spreads the two
 * variances); the pair is (largest deviation, smallest deviation), ties to the lowest index; the
 * matrix returned is the transpose of the listing's accumulated product, so that the output line
 * holds as written.  At most B - 1 rotations.
 *   Sigma_f64 [B, B] float64: in Sigma, out Q Sigma Q^T;  Q_f64 [B, B] float64;
 *   Q_bf16 [B, B] bf16 or NULL (Q rounded through float32);  n_rotations: device int32 or NULL.
 * One CTA; float64, one rounding per operation (no fused multiply-add), so the result is defined
 * bit for bit.  1 <= B <= 32768, eps >= 0. */
torq_status torq_givens_equalize(void* Sigma_f64, int64_t B, double eps, void* Q_f64, void* Q_bf16,
                                 void* n_rotations, void* stream);

/* Measurement tool (no counterpart in the paper): runs `groups` groups of four block-scaled FP4
 * tensor-core instructions (256 x 256 x 64 each, the GEMM's own instruction) per CTA pair on operands
 * that already sit in shared memory, with no loads and no epilogue, times them with CUDA events on
 * `stream`, synchronises, and writes the rate in TFLOP/s to *tflops (host pointer).  This is the
 * issue-bound peak of the FP4 tensor pipe on the device at hand: the denominator for the GEMM's
 * roofline fraction where no vendor-measured FP4 peak exists.  Includes the kernel's launch, so use
 * groups >= 20000 (about a millisecond). */
torq_status torq_probe_fp4_peak(int groups, double* tflops, void* stream);

/* Self-test of the bounded device waits (no counterpart in the paper).  Every wait inside the
 * tensor-core kernels gives up after 2 s, latches TORQ_ERR_TIMEOUT, lets the kernel's other warps
 * drain and returns; a healthy run never takes that path.  This call runs it on purpose in a
 * one-CTA kernel whose two barriers nothing ever arrives on: one warp's wait runs out after
 * `limit_ns` (1 us .. 100 ms) and latches the error word with wait-site id 7, the other warp's wait
 * (2 s limit) must leave through the CTA's abort flag.  Nothing faults or hangs: the waits give up
 * by design, and the context stays usable.
 *   result_u64x3: three device uint64: [0] = 1 if the first wait gave up by itself, [1] = 1 if the
 *   second left through the abort flag, [2] = nanoseconds the second one waited.
 * Afterwards torq_last_device_error() returns TORQ_ERR_TIMEOUT | 7 << 8 (and clears the word). */
torq_status torq_selftest_wait_timeout(uint64_t limit_ns, void* result_u64x3, void* stream);

const char* torq_status_string(torq_status s);

/* Synchronises `stream`, then returns and clears the device error word of the current device:
 * 0, or TORQ_ERR_TIMEOUT in the low byte with the id of the wait that gave up in bits 8..15, or TORQ_ERR_PAGE. */
int torq_last_device_error(void* stream);

/* Host helper (no device work): the list of output tiles that the CTA-pair kernels (more than
 * 48 rows) walk for a [rows x cols] output on `pairs` CTA pairs (74 on a 148-SM part), in the order
 * in which they are dealt round robin: tile i goes to pair i % pairs.  Tiles are 256 rows high and
 * 256 columns wide; where that leaves the last wave partly empty and cols is a multiple of 256,
 * some row tiles are covered by fewer 256-column tiles followed by 192-column ones (three wide
 * tiles traded for four narrow ones), chosen so that the longest pair finishes earliest.
 * torq_rotate_quantize (cols = d) and its format variants use this list where these kernels serve a
 * call, except that a rotation with d > 4096 whose last wave would hold a few 256-column tiles
 * leaves those to another kernel (see torq_rotated_linear).  Of a GEMM (cols = N) these are the
 * tiles; torq_gemm_tile_list has them in its order.
 *   out: host array of 3 * cap int32, or NULL; receives (row_tile, first_column, width) per tile.
 * Returns the number of tiles (also when it exceeds cap; only cap triples are written), or -1 for
 * rows < 1, cols < 1 or pairs < 1. */
int64_t torq_pair_tile_list(int64_t rows, int64_t cols, int32_t pairs, int32_t* out, int64_t cap);

/* The same for torq_mxfp4_gemm and its format variants on an [M x N] output with weights whose rows
 * are `w_row_bytes` long (K / 2; MXINT4: K): the tiles of torq_pair_tile_list(M, N), with the row
 * tiles taken in groups of sixteen instead of eight where N is 10240 or more and the weights are 16
 * MiB or more, or 8192 and 32 MiB.  Same results; -1 also for w_row_bytes < 1. */
int64_t torq_gemm_tile_list(int64_t M, int64_t N, int64_t w_row_bytes, int32_t pairs, int32_t* out, int64_t cap);

/* Number of kernels this library has launched since load (all devices, all streams). */
int64_t torq_launch_count(void);

/* ---- a key/value cache in 4 bits --------------------------------------------------------------------------------------------------------
 * The cache of an attention layer lies in pages of page_tokens tokens (a power of two from 16 to 1024) that all sequences share; table[b][i] is
 * the page of the tokens i page_tokens ... of sequence b.  A page holds, for one key/value head after the other,
 *   key codes [page_tokens][D/2] | key scale bytes [page_tokens][D/B] | value codes [page_tokens][D/2] | value scale bytes [page_tokens][D/B]
 * with D = head_dim (64, 128 or 256), B = 32 (MXFP4, MXINT4) or 16 (NVFP4): codes and scale bytes by the rules of torq_quantize_*, MXINT4 in its
 * stored form, scale bytes row by row.  NVFP4 caches have a float32 tensor scale for the keys and one for the values.
 * lengths[b] counts the tokens of sequence b, the new ones included.  The new tokens of a call are rows of one batch: rows starts[b] to
 * starts[b+1] - 1 are the last ones of sequence b (0 <= starts[0], ascending, starts[batch] <= tokens); starts == NULL: one row per sequence,
 * tokens == batch.  A row that no sequence has, or more new rows than a length, is a row without a place: nothing is stored for it, and its
 * results are zeros (lse: minus infinity).  table, lengths, starts are int32 and 4-byte aligned, and are read on the device: one captured call
 * serves every step.  A page number that a call needs and that lies outside [0, num_pages), or a length that the table has no room for, latches
 * TORQ_ERR_PAGE in the device error word; nothing is read or written there, and the results of that sequence are unspecified.
 * Entries of table behind a sequence's length and what pages hold there are never looked at, so they may hold anything.  A length below zero counts as none.
 * Sequences may have pages in common (a prompt that they share), but no two of them slots that append writes, nor any page in a call of weights, which writes
 * all of a sequence's.
 * Sizes: batch <= 65536, kv_heads <= 1024, table_width page_tokens <= 2^30, tokens <= 2^24; append and read: tokens kv_heads head_dim / 4 < 2^31; attention and
 * weights: heads <= 65536, tokens heads < 2^31.  Tensor scales above 0 and up to 3e38. */
typedef struct {
  void* pages;               /* [num_pages][kv_heads][torq_kv_page_bytes()], 16-byte aligned */
  const int32_t* table;      /* [batch][table_width] */
  const int32_t* lengths;    /* [batch] */
  int64_t num_pages, page_tokens, kv_heads, head_dim, batch, table_width;
  float k_tensor_scale, v_tensor_scale;   /* NVFP4; the others do not look at them */
} torq_kv_cache;

/* Bytes of one head's page; scale_block: 32, NVFP4 16.  0 for sizes that make none. */
size_t torq_kv_page_bytes(int64_t scale_block, int64_t page_tokens, int64_t head_dim);

/* New keys and values, quantized into their slots.  K, V [tokens][kv_heads][D] of `dtype`, rows k_stride and v_stride elements apart (columns of
 * a fused projection; 16-byte aligned, strides a multiple of 16 bytes).  Everything else in the pages stays as it is.  One launch. */
torq_status torq_mxfp4_kv_append(const torq_kv_cache* cache, const void* K, const void* V, torq_dtype dtype, int64_t k_stride, int64_t v_stride,
                                 const int32_t* starts, int64_t tokens, void* stream);
torq_status torq_nvfp4_kv_append(const torq_kv_cache* cache, const void* K, const void* V, torq_dtype dtype, int64_t k_stride, int64_t v_stride,
                                 const int32_t* starts, int64_t tokens, void* stream);
torq_status torq_mxint4_kv_append(const torq_kv_cache* cache, const void* K, const void* V, torq_dtype dtype, int64_t k_stride, int64_t v_stride,
                                  const int32_t* starts, int64_t tokens, void* stream);

/* The values that the same slots stand for, K and V [tokens][kv_heads][D] dense, float32 or rounded once to bfloat16 (exact but for NVFP4).
 * With starts the sums of all lengths this is the whole cache.  One launch. */
torq_status torq_mxfp4_kv_read(const torq_kv_cache* cache, const int32_t* starts, int64_t tokens, void* K, void* V, torq_dtype dtype, void* stream);
torq_status torq_nvfp4_kv_read(const torq_kv_cache* cache, const int32_t* starts, int64_t tokens, void* K, void* V, torq_dtype dtype, void* stream);
torq_status torq_mxint4_kv_read(const torq_kv_cache* cache, const int32_t* starts, int64_t tokens, void* K, void* V, torq_dtype dtype, void* stream);

/* How a query at place p of its sequence (its last new row is at length - 1) scores and sees the token at place j:
 *   x_j = cap(scale q k_j) - slopes[head] |p - j|,   cap(x) = softcap tanh(x / softcap), or x where softcap is 0
 *   p - window < j (window > 0),   j <= max(p, prefix[b] - 1),   first[row] <= j < length
 * slopes [heads] float32, prefix [batch] and first [tokens] int32, each or all NULL: no bias by distance, causal, from the beginning.
 * 0 < scale <= 1e30, 0 <= softcap <= 1e30, window >= 0. */
typedef struct {
  float scale, softcap;
  const float* slopes;
  int64_t window;
  const int32_t* prefix;
  const int32_t* first;
} torq_kv_scoring;

/* Attention of the new rows over the cache (append them first):  out = sum_j exp(x_j - lse) v_j,  lse = log sum_j exp(x_j), the sums over what
 * a row sees; zeros and minus infinity for a row that sees nothing.
 *   Q [tokens][heads][D] bf16, rows q_stride elements apart; heads % kv_heads == 0, query heads h G ... h G + G - 1 share key/value head h
 *   out [tokens][heads][D] bf16;  lse [tokens][heads] float32, natural logarithm, or NULL
 *   workspace: torq_kv_attention_workspace_bytes() bytes, 256-byte aligned; two calls that may overlap need one each
 * Scores, sums and the running maximum are float32: scores may be of any size there, with the relative error of float32, as long as scale times a row's largest
 * element times the largest key that it meets is below 2^110.  Q is held as float16 relative to a row's largest element: all bits of what is down to 2^-21 of it,
 * and nothing is off by more than 2^-39 (rows whose largest is below 2^-112: of 2^-112).  A weight is float16 when it meets the values: 11 bits, but off by 2^-35 of
 * the row's largest so far where that is more.  MXFP4, MXINT4: scale byte 0 counts as zero, and further
 *   few rows (tokens / batch, whole, times heads / kv_heads below 64): values' scales below 2^-26 of the largest so far that the same 32 features have among the
 *   tokens that any of the 8 or 16 rows worked on together sees; keys' scales below 2^-190 of the largest of the same 32 tokens
 *   many rows: scales below 2^-35 of the largest of the same 128 tokens, keys' and values' apart; a weight times the largest scale of its 128 tokens is off by
 *   2^-35 of the row's largest such product so far, instead of the weights alone
 * Tokens that no row of a sequence sees may hold anything.  Two launches.  Outputs overlap no operand. */
size_t torq_kv_attention_workspace_bytes(int64_t tokens, int64_t batch, int64_t heads, int64_t kv_heads, int64_t head_dim);
torq_status torq_mxfp4_kv_attention(const torq_kv_cache* cache, const torq_kv_scoring* scoring, const void* Q, int64_t q_stride, int64_t heads,
                                    const int32_t* starts, int64_t tokens, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream);
torq_status torq_nvfp4_kv_attention(const torq_kv_cache* cache, const torq_kv_scoring* scoring, const void* Q, int64_t q_stride, int64_t heads,
                                    const int32_t* starts, int64_t tokens, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream);
torq_status torq_mxint4_kv_attention(const torq_kv_cache* cache, const torq_kv_scoring* scoring, const void* Q, int64_t q_stride, int64_t heads,
                                     const int32_t* starts, int64_t tokens, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* The account of the cache: what attention gave to each cached token, summed over the new rows and the query heads that share its head.
 *   weights_out[page][h][slot] = (weights[page][h][slot] of a token that is not new, else 0) + sum over rows and heads of exp(x_j - lse)
 * weights, weights_out [num_pages][kv_heads][page_tokens] float32 (16-byte aligned; they may be the same); only slots of the sequences' tokens are
 * written.  Q, scoring and starts as the attention call had them, lse [tokens][heads] what it gave.  The order of the sums is fixed.  One launch.
 * No two sequences of a call have a page in common: what its slots get would be one's sum or the other's or both.  For sequences that share pages make one call
 * after the other, each with its rows, its row of table and its length, in place: every slot then has the sum over all of them.
 * An exponent x_j - lse is off by what float32 keeps of a score and of lse, 2^-20 of the larger: where scores are beyond some thousands, so is the account. */
torq_status torq_mxfp4_kv_weights(const torq_kv_cache* cache, const torq_kv_scoring* scoring, const void* Q, int64_t q_stride, int64_t heads,
                                  const int32_t* starts, int64_t tokens, const float* lse, const float* weights, float* weights_out, void* stream);
torq_status torq_nvfp4_kv_weights(const torq_kv_cache* cache, const torq_kv_scoring* scoring, const void* Q, int64_t q_stride, int64_t heads,
                                  const int32_t* starts, int64_t tokens, const float* lse, const float* weights, float* weights_out, void* stream);
torq_status torq_mxint4_kv_weights(const torq_kv_cache* cache, const torq_kv_scoring* scoring, const void* Q, int64_t q_stride, int64_t heads,
                                   const int32_t* starts, int64_t tokens, const float* lse, const float* weights, float* weights_out, void* stream);

/* Eviction by account: of each sequence and key/value head the `recent` newest tokens and, of the others, those with the largest weights stay, `keep`
 * in all (equal weights, zeros of either sign among them: the lower place stays; a sequence of at most `keep` tokens stays whole).  Codes, scale bytes and weights of what stays
 * are copied, in their order, to the pages of new_table [batch][new_width], which are no pages of the sequences and no page twice.  Places count anew there: a
 * bias by distance or a window then counts what is left.
 *   new_lengths [batch] int32 = min(length, keep);  kept [batch][kv_heads][keep] int32: the places of what stayed, -1 behind them
 * 1 <= keep <= 2^30, 0 <= recent <= keep, new_width <= 2^26, new_width page_tokens >= min(keep, table_width page_tokens); batch kv_heads <= 65535.  Weights that are no numbers are outside the contract.
 * Two launches. */
torq_status torq_mxfp4_kv_evict(const torq_kv_cache* cache, float* weights, const int32_t* new_table, int64_t new_width, int64_t keep, int64_t recent,
                                int32_t* new_lengths, int32_t* kept, void* stream);
torq_status torq_nvfp4_kv_evict(const torq_kv_cache* cache, float* weights, const int32_t* new_table, int64_t new_width, int64_t keep, int64_t recent,
                                int32_t* new_lengths, int32_t* kept, void* stream);
torq_status torq_mxint4_kv_evict(const torq_kv_cache* cache, float* weights, const int32_t* new_table, int64_t new_width, int64_t keep, int64_t recent,
                                 int32_t* new_lengths, int32_t* kept, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TORQ_H_ */
