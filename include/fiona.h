/*
 * fiona.h -- C ABI of the MI355X (gfx950) hybrid weighted sum.
 *
 * The operation (Fiona, Sec. 4.2 "Exact Compilation of Routed Linear
 * Operators", Eq. (routed-example) and Eq. (shared-example)): a routed linear
 * layer computes every packed output ciphertext y_j from already prepared
 * (rotated) input ciphertexts A_i as
 *
 *     y_j = sum over raw terms (i, pi) of  pt_pi (*) A_i              (one PMult each)
 *         + sum over signed-sum uses (s, sigma, c) of  c * sigma * U_s
 *     U_s = sum over members (i, h) of  h * A_i,   h in {-1, 0, +1}   (Add / Sub / skip)
 *
 * where (*) is the slot-wise product, c is the reconstruction factor of the
 * group (applied once to the group's signed sum: "Grouping Reconstruction
 * Operations"), a signed sum U_s may be shared by several outputs, also with
 * all signs reversed (sigma = -1: "Sharing Signed Sums"), and the signed and
 * raw results of an output are added before any rescale ("Combining the
 * Signed and Raw Routes").  The library evaluates this exactly in every RNS
 * limb: ciphertexts are in the negacyclic NTT domain, where a PMult is an
 * element-wise product mod q_l and a constant factor c is a scalar product.
 * Rotation, key switching, rescale, encoding and bootstrapping are not part
 * of it.
 *
 * Data layout ("limb-major"), all uint64 residues:
 *   ciphertext i, polynomial p (0 = c0, 1 = c1), limb l, coefficient k is
 *   element ((i * 2 + p) * L + l) * N + k of a ciphertext array;
 *   plaintext pi, limb l, coefficient k is element (pi * L + l) * N + k.
 *
 * Every function returns FIONA_OK (0) or a negative fiona_status and never
 * throws or aborts.  All objects are created and destroyed by the caller.
 */
#ifndef FIONA_H
#define FIONA_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum fiona_status {
  FIONA_OK = 0,
  FIONA_ERR_ARG = -1,          /* null pointer, zero or inconsistent size */
  FIONA_ERR_PLAN = -2,         /* layer description inconsistent (index out of range, bad CSR) */
  FIONA_ERR_UNSUPPORTED = -3,  /* N, L or a modulus outside the supported range */
  FIONA_ERR_ALIGN = -4,        /* a device pointer is not 8-byte aligned (rotation keys: 16-byte; the key
                                  holder's operators: their elements' size) */
  FIONA_ERR_ALIAS = -5,        /* the output buffer overlaps an input buffer */
  FIONA_ERR_HIP = -6,          /* a HIP runtime call failed (device allocation, copy, launch) */
  FIONA_ERR_NOMEM = -7,        /* host allocation failed */
  FIONA_ERR_NODEVICE = -8,     /* the plan was created host-only and has no device image */
  FIONA_ERR_PRECONDITION = -9, /* an input breaks a precondition (checked only where documented) */
  FIONA_ERR_BOUNDS = -10       /* a replayed access falls outside its buffer (fiona_check_ntt_offsets) */
} fiona_status;

/* Limits checked by fiona_ctx_create. */
#define FIONA_MAX_N (1u << 20)
#define FIONA_MAX_L 64u
#define FIONA_MODULUS_BITS 50      /* every modulus satisfies 2^20 < q < 2^50 */
#define FIONA_SCALE_BITS 20        /* every integer scale c satisfies c < 2^20 */
#define FIONA_MAX_MEMBERS 48u      /* longer ternary groups are split into exact sub-sums */
#define FIONA_MAX_INPUTS 159u      /* input ciphertexts of one pass: a 64-coefficient tile of every
                                      input (16 B each) plus one zero row fill the 160 KiB LDS; a layer
                                      with more inputs runs in passes over input ranges */
#define FIONA_MAX_LAYER_INPUTS 65536u   /* input ciphertexts per layer */

typedef struct fiona_ctx fiona_ctx;
typedef struct fiona_plan fiona_plan;

/*
 * fiona_ctx_create: RNS parameters of the ciphertexts.
 *   N       coefficients per limb, 1 <= N <= FIONA_MAX_N (any N; CKKS uses a
 *           power of two, and the kernel handles a partial last tile);
 *   L       number of RNS limbs, 1 <= L <= FIONA_MAX_L;
 *   moduli  host array of L moduli, each 2^20 < q_l < 2^50 (so that every
 *           integer scale, < 2^20, is a canonical residue).  The element-wise
 *           path does not need them to be NTT-friendly primes; CKKS callers
 *           pass primes q = 1 (mod 2N).
 * Host-only: no device memory is touched.  On success *out owns a context
 * that fiona_ctx_destroy frees.  Errors: FIONA_ERR_ARG (null), FIONA_ERR_UNSUPPORTED.
 */
int fiona_ctx_create(uint32_t N, uint32_t L, const uint64_t *moduli, fiona_ctx **out);
void fiona_ctx_destroy(fiona_ctx *ctx);

/* Plan flags. */
#define FIONA_PLAN_NO_SHARING 1u   /* evaluate every group's signed sum on its own (no reuse) */
#define FIONA_PLAN_HOST_ONLY 2u    /* build and check the plan on the host; upload nothing */
#define FIONA_PLAN_NO_LDS_SUMS 4u  /* never keep shared signed sums resident in LDS */
#define FIONA_PLAN_NO_PARTIAL_SHARING 8u   /* share only whole signed sums, no common sub-sums */
#define FIONA_PLAN_PER_CONTRIBUTION 16u    /* no grouping: a scalar product per nonzero signed term
                                              (the first compilation of Sec. 6.2; implies NO_SHARING) */
#define FIONA_PLAN_NO_OUTPUT_BURSTS 32u    /* store each output as soon as it is finished instead of
                                              buffering a round of outputs in LDS and writing them together
                                              (the default when outputs are at least 2.5% of the bytes) */
#define FIONA_PLAN_CHECK_INPUTS 64u        /* a checking plan: it keeps the layer's signs, and every
                                              fiona_hybrid_linear call checks its inputs' preconditions on the
                                              host first (synchronously; see fiona_plan_check_inputs) */

/*
 * One routed layer, in the raw per-(output, term) form the offline compiler
 * emits (paper Sec. 2.2 "Execution Plan": fixed before any query).  Host
 * arrays, all read during fiona_plan_create only (the caller keeps ownership).
 *
 * Raw route, per output CSR:
 *   pm_off[n_out+1]        terms of output j are pm_off[j] .. pm_off[j+1]-1
 *   pm_input[n_pm]         input ciphertext of each raw term (< n_in)
 *   pm_pt[n_pm]            plaintext of each raw term (< n_pt)
 * Signed route, per output CSR over groups, per group CSR over members:
 *   grp_off[n_out+1]       groups of output j are grp_off[j] .. grp_off[j+1]-1
 *   grp_mem_off[n_group+1] members of group g are grp_mem_off[g] .. grp_mem_off[g+1]-1
 *   mem_input[n_member]    input ciphertext of each member (< n_in)
 *   mem_sign[n_member]     sign h in {-1, 0, +1} of each member: the same
 *                          values the caller later passes as ternary_groups
 *   grp_scale[n_group]     index into the scales array of each group (< n_scale)
 * n_group and n_member are grp_off[n_out] and grp_mem_off[n_group].
 * Plaintext table layout:
 *   pt_pitch               words from one plaintext to the next in pt_diags:
 *                          0 means L*N (packed rows), otherwise at least L*N
 *                          (FIONA_ERR_ARG if less).  Words between rows are
 *                          never read.  fiona_pt_pitch_hint gives a padded
 *                          pitch that spreads the rows over the HBM banks.
 */
typedef struct fiona_layer_desc {
  uint32_t n_in, n_out, n_pt, n_scale;
  const uint32_t *pm_off;
  const uint32_t *pm_input;
  const uint32_t *pm_pt;
  const uint32_t *grp_off;
  const uint32_t *grp_mem_off;
  const uint32_t *mem_input;
  const int8_t *mem_sign;
  const uint32_t *grp_scale;
  uint32_t flags;
  uint64_t pt_pitch;
} fiona_layer_desc;

/*
 * fiona_pt_pitch_hint: a plaintext pitch for fiona_layer_desc.pt_pitch (in
 * words) that keeps the rows streamed together by one launch off the same
 * HBM banks: L*N rounded up to a multiple of 64 words, plus 128 words.  With
 * packed rows (pitch L*N, a multiple of 2 MiB at N = 2^16) every plaintext's
 * slice of a tile lands at the same bank offset; the padding spreads them.
 * Returns 0 for a null ctx.
 */
uint64_t fiona_pt_pitch_hint(const fiona_ctx *ctx);

/*
 * fiona_plan_create: compile one layer for the GPU.
 *   - checks every index of desc (FIONA_ERR_PLAN on any inconsistency);
 *   - drops members whose sign is 0 and groups with no nonzero member: they
 *     contribute nothing (Sec. 3 Obs. 2, the skip; Sec. 4.2 "contributes nothing");
 *   - splits groups of more than FIONA_MAX_MEMBERS members into sub-sums with
 *     the same scale (exact, since c*(U1 + U2) = c*U1 + c*U2);
 *   - unless FIONA_PLAN_NO_SHARING, finds signed sums that are equal or
 *     exactly opposite (same inputs, same or all reversed signs) across the
 *     layer and computes each once (Sec. 4.2 "Sharing Signed Sums"); sums
 *     used more than once are kept resident in LDS per position tile;
 *   - unless FIONA_PLAN_NO_SHARING or FIONA_PLAN_NO_PARTIAL_SHARING, also
 *     shares signed terms common to several sums that only partly overlap
 *     (Sec. 4.2, the candidate search with its estimate k*m - m - k of the
 *     Add/Sub saved by a common term of m members reused k times): the most
 *     reused common pair (two inputs, or inputs and earlier common terms,
 *     with fixed relative sign) is taken while the estimate is positive,
 *     the reuse pays for forming it once per tile and LDS rows are left.
 *     Each common term is formed once per position tile and then enters
 *     every sum that contains it as a single member;
 *   - uploads the compiled metadata to the current HIP device (synchronous)
 *     unless FIONA_PLAN_HOST_ONLY.
 *   - a layer with more than FIONA_MAX_INPUTS inputs is compiled as passes
 *     over consecutive input ranges of at most 128 inputs each: a pass takes
 *     the raw terms and the group members whose input falls in its range (a
 *     group spanning several ranges becomes one sub-sum per range with the
 *     group's scale, exact since c*(U1 + U2) = c*U1 + c*U2); the first pass
 *     stores the outputs and each later pass adds its sums to them mod q_l,
 *     so the outputs are read and written once more per extra pass; a range
 *     that no term reads gets no pass;
 * The plan keeps a reference to ctx (which must outlive it).  Errors:
 * FIONA_ERR_ARG (also a pt_pitch below L*N), FIONA_ERR_PLAN, FIONA_ERR_UNSUPPORTED
 * (more than FIONA_MAX_LAYER_INPUTS inputs, or a plaintext table beyond 2^48 bytes), FIONA_ERR_NOMEM, FIONA_ERR_HIP.
 * The plan owns a small device
 * workspace (the members of its signed sums, reordered by sign on every call),
 * so one plan must not be used by two streams at the same time.
 */
int fiona_plan_create(const fiona_ctx *ctx, const fiona_layer_desc *desc, fiona_plan **out);
void fiona_plan_destroy(fiona_plan *plan);

/* Operation counts of a compiled plan (per position and polynomial, as the
 * paper counts CKKS operations per ciphertext in Sec. 4.2 and Sec. 6.2). */
typedef struct fiona_plan_stats_t {
  uint64_t ct_terms;               /* all (output, term) pairs, sign-0 members included */
  uint64_t n_pmult;                /* raw terms: one PMult each */
  uint64_t n_member;               /* signed terms (members), sign 0 included */
  uint64_t n_member_nonzero;       /* signed terms with h != 0 */
  uint64_t n_use;                  /* (output, signed sum) uses: one scalar product each */
  uint64_t n_sum_distinct;         /* distinct signed sums after sharing */
  uint64_t n_sum_resident;         /* shared sums kept in LDS, computed once per tile */
  uint64_t pmult_per_contribution; /* PMults if every signed term were applied on its own */
  uint64_t pmult_grouped;          /* PMults after grouping: raw terms + uses */
  uint64_t addsub_unshared;        /* Add/Sub to form every use's signed sum on its own */
  uint64_t addsub_shared;          /* Add/Sub with each distinct sum formed once */
  uint64_t addsub_partial;         /* Add/Sub after also sharing common partial sums:
                                      distinct sums plus the common terms themselves */
  uint32_t tile;                   /* coefficients per workgroup */
  uint32_t waves;                  /* wavefronts per workgroup */
  uint32_t lds_bytes;              /* LDS per workgroup */
  uint32_t grid;                   /* workgroups per launch */
  uint32_t split_outputs;          /* outputs split into segments over several wavefronts */
  uint32_t segment_slots;          /* LDS rows holding the segments' partial residues */
  uint32_t n_partial;              /* common partial sums, each formed once per tile in LDS */
  uint32_t partial_levels;         /* longest chain of common terms built from common terms */
  uint32_t output_rounds;          /* rounds of outputs per tile, each ending in one burst of stores */
  uint32_t output_buffer_rows;     /* LDS rows (outputs) buffered per round; 0 = stored directly */
  uint32_t input_passes;           /* launches (input ranges) per call: 1 up to FIONA_MAX_INPUTS inputs;
                                      with several, the counts above add up over the passes (a group
                                      split over passes counts one use per pass) and the launch shape is
                                      the widest pass's */
} fiona_plan_stats_t;

int fiona_plan_stats(const fiona_plan *plan, fiona_plan_stats_t *out);

/*
 * fiona_plan_check_inputs: the preconditions of fiona_hybrid_linear that a
 * checking plan (FIONA_PLAN_CHECK_INPUTS) enforces, tested on host copies of
 * the call's arrays (Sec. 2.2: the plan is fixed offline from the weights,
 * so the signs a call passes must be the signs the plan was compiled from):
 *   signs   host, [n_member] int8: must equal the layer description's mem_sign
 *   scales  host, [n_scale] uint64: each < 2^20
 *   in      host or NULL, [n_in][2][L][N] uint64: each < 2^50
 *   pt      host or NULL, [n_pt] rows at the plan's pitch: each word of a
 *           row's first L*N < 2^50
 * Returns FIONA_OK, FIONA_ERR_PRECONDITION (the first failing check), or
 * FIONA_ERR_ARG (a null plan or array with a nonzero size, or a plan made
 * without FIONA_PLAN_CHECK_INPUTS, which keeps no signs).  Host only; works
 * with a host-only plan.
 * A checking plan's fiona_hybrid_linear copies ternary_groups, scales,
 * in_cts and pt_diags back to the host (on its stream, then waits for it),
 * runs this check, and returns FIONA_ERR_PRECONDITION without launching
 * anything if it fails.  It is a debugging aid: it allocates host memory
 * and is as slow as copying every input.
 */
int fiona_plan_check_inputs(const fiona_plan *plan, const int8_t *signs, const uint64_t *scales, const uint64_t *in,
                            const uint64_t *pt);

/*
 * fiona_hybrid_linear: evaluate the layer (the hot path).
 *   in_cts          device, [n_in][2][L][N] uint64, every value < 2^50
 *                   (CKKS residues are < q_l)
 *   pt_diags        device, n_pt plaintexts of [L][N] uint64 NTT-domain
 *                   residues < 2^50, plaintext p starting at word p * pitch
 *                   (pitch = the plan's pt_pitch, L*N by default)
 *   ternary_groups  device, [n_member] int8 signs in {-1, 0, +1}, in the
 *                   member order of the layer description; must equal the
 *                   mem_sign the plan was created with (members that were 0
 *                   then are skipped; the others are read here)
 *   scales          device, [n_scale] uint64 integer reconstruction factors,
 *                   each < 2^20
 *   out_cts         device, [n_out][2][L][N] uint64, overwritten with
 *                   canonical residues in [0, q_l); must not overlap any input
 *   stream          HIP stream the work is queued on (0 = legacy default)
 * Asynchronous: returns once the kernel is queued; the buffers must stay
 * valid and unchanged until the stream reaches it.  Allocates nothing, and
 * issues kernel launches only (no memset or copy; a checking plan excepted),
 * so a call can be captured in a HIP graph.
 * Results are exact (bit-identical to evaluating every term on its own mod q_l).
 * Input ranges and signs above are preconditions, checked only by a checking
 * plan (FIONA_PLAN_CHECK_INPUTS).  Device pointers need 8-byte alignment
 * (every access is an 8-byte word).  Errors (nothing is launched):
 * FIONA_ERR_ARG (null pointer with a nonzero size), FIONA_ERR_ALIGN,
 * FIONA_ERR_ALIAS, FIONA_ERR_NODEVICE, FIONA_ERR_PRECONDITION (checking plans),
 * FIONA_ERR_HIP (launch, or a checking plan's copies).
 */
int fiona_hybrid_linear(const fiona_plan *plan, const uint64_t *in_cts, const uint64_t *pt_diags,
                        const int8_t *ternary_groups, const uint64_t *scales, uint64_t *out_cts,
                        hipStream_t stream);

/*
 * fiona_hybrid_linear_static: fiona_hybrid_linear for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  Same arguments, results and errors.
 * The per-call word blocks (the signed sums' member rows and the uses'
 * scales, written by the sign-packing kernel on every call) go to a
 * library-owned static device array of 4 MiB per device instead of the
 * plan's workspace; the array's address is looked up on the first call on a
 * device and kept until the process ends.  Allocates nothing (neither device
 * nor host memory).  Every call on one device shares its array and leaves its
 * blocks there; each call writes every block it reads before reading it, so
 * nothing needs clearing, but calls that overlap on one device (two streams,
 * or two host threads) race and must be serialized by the caller.
 * Errors, besides fiona_hybrid_linear's: FIONA_ERR_UNSUPPORTED if the plan's
 * word blocks exceed 4 MiB (more than 16384 common terms, resident sums and
 * uses); FIONA_ERR_ARG for a checking plan (FIONA_PLAN_CHECK_INPUTS), whose
 * check copies into host memory.
 */
int fiona_hybrid_linear_static(const fiona_plan *plan, const uint64_t *in_cts, const uint64_t *pt_diags,
                               const int8_t *ternary_groups, const uint64_t *scales, uint64_t *out_cts,
                               hipStream_t stream);

/*
 * Rescale epilogue: divide ciphertexts by the last modulus q_t = q_{L-1} of the
 * chain, with rounding, and drop that limb (CKKS rescaling, paper Sec. 2
 * "Levels and Bootstrapping").  Sec. 4.2 "Combining the Signed and Raw
 * Routes" rescales an output once, after its routes are summed: this is the
 * call that follows fiona_hybrid_linear.  Per coefficient, with C the integer
 * of the L residues: C' = round(C / q_t), kept as residues of the first L-1
 * moduli.
 *
 * NTT convention of every limb (input and output): a_hat_k = sum_n a_n
 * psi_l^((2k+1) n) mod q_l, k in natural order, psi_l a primitive 2N-th root
 * of unity mod q_l.
 *
 * fiona_rescaler_create: the NTT twiddle tables of every limb (device) and a
 * workspace: none up to N = 2^13, else about
 * 2 * c * N * 8 * (1 + (L - 1) (1 + 16 / sqrt(N))) bytes, c = max_ct or the
 * ciphertexts whose intermediates fill 256 MiB if those are fewer (a call over
 * more takes them in chunks).
 *   psi     host [L] roots psi_l, or NULL for the default: psi_l =
 *           x^((q_l - 1) / 2N) for the smallest x >= 2 with psi_l^N = -1
 * Requires N a power of two in [2^8, 2^17], L >= 2, every q_l = 1 mod 2N and
 * max_ct <= 32767.
 * The rescaler keeps a reference to ctx (which must outlive it).  Errors:
 * FIONA_ERR_ARG, FIONA_ERR_UNSUPPORTED (N, L, a modulus or a root),
 * FIONA_ERR_NOMEM, FIONA_ERR_HIP.
 */
typedef struct fiona_rescaler fiona_rescaler;
int fiona_rescaler_create(const fiona_ctx *ctx, const uint64_t *psi, uint32_t max_ct, fiona_rescaler **out);
void fiona_rescaler_destroy(fiona_rescaler *rescaler);

/*
 * fiona_rescale: out = in / q_t with rounding, per ciphertext and polynomial.
 *   in_cts   device, [n_ct][2][L][N] uint64 canonical residues (NTT domain)
 *   out_cts  device, [n_ct][2][L-1][N] uint64, overwritten with canonical
 *            residues; must not overlap in_cts
 *   n_ct     at most the max_ct of the rescaler
 * Asynchronous on stream; allocates nothing, and issues kernel launches only
 * (no memset or copy), so a call can be captured in a HIP graph.  The
 * rescaler's workspace is shared by its calls: one rescaler must not be used
 * by two streams at the same time.  Errors (nothing is launched):
 * FIONA_ERR_ARG, FIONA_ERR_ALIGN, FIONA_ERR_ALIAS, FIONA_ERR_HIP.
 */
int fiona_rescale(const fiona_rescaler *rescaler, const uint64_t *in_cts, uint32_t n_ct, uint64_t *out_cts,
                  hipStream_t stream);

/*
 * Hoisted baby-step rotations: the step that produces fiona_hybrid_linear's
 * input ciphertexts.  A layer's inputs A_i are the packed input rotated by
 * the packing layout's baby steps (paper Sec. 2 "Homomorphic Operations": Rot
 * cyclically shifts the slots; Sec. 4.2: the A_i are prepared according to
 * the packing layout).  Rot by r slots is the automorphism sigma_g:
 * a(X) -> a(X^g), g = 5^r mod 2N (slot j of a message is its value at
 * zeta^(5^j), zeta = exp(i pi / N)), on both polynomials, followed by a key
 * switch of the second polynomial from sigma_g(s) back to s.  Key switching
 * decomposes c1 by RNS limb (digit j = the coefficients of c1 mod q_j, as
 * integers in [0, q_j)), multiplies digit j by key polynomial pair j over the
 * data moduli and one special prime P, sums, and divides by P with rounding:
 *     Rot(c0, c1) = (sigma(c0) + v_0, v_1),
 *     v_p = round(sum_j sigma(D_j) ksk[j][p] / P)    (coefficient-wise).
 * The digits are formed once per call and shared by all its rotations
 * (hoisting); the automorphism acts on the integer digits.  NTT convention:
 * as for the rescaler, for every modulus including P.
 *
 * fiona_rotator_create: NTT tables of q_0 .. q_{L-1} and P, and a workspace
 * for up to max_rot rotations per call (max_rot <= 256): about
 * 8 N (L + 1) (L + 2 max_rot) bytes, and from N = 2^13 on
 * 8 N (2 L + c + (1 + 16 / sqrt(N)) L max(L + 1, c)) more, c = 2 max_rot or the
 * vectors whose L intermediates fill 416 MiB if those are fewer (a call over
 * more divides by P in chunks).
 *   special_prime  P with 2^20 < P < 2^50, P = 1 mod 2N, unequal to every q_l
 *   psi            host [L + 1] roots (the data moduli, then P) or NULL for
 *                  the defaults of fiona_rescaler_create
 * Requires N a power of two in [2^8, 2^17], L + 1 <= FIONA_MAX_L and
 * max_rot <= 256.  Keeps a reference to ctx.  Errors: FIONA_ERR_ARG, FIONA_ERR_UNSUPPORTED,
 * FIONA_ERR_NOMEM, FIONA_ERR_HIP.
 *
 * Keys.  A rotation's key holds, for digit j < L and polynomial p in {0, 1},
 * one polynomial over the L + 1 moduli, NTT domain: [L][2][L + 1][N] uint64
 * canonical residues, modulus index L being P (fiona_rotation_key_words
 * words).  In its natural order, sum_j D_j ksk[j][0] + (sum_j D_j ksk[j][1]) s
 * = P D sigma_g(s) + small for a key that switches sigma_g(s) to s.
 * fiona_hoisted_rotate reads keys in the library's layout: each row of N
 * words permuted by the rotation's slot map and stored transposed (N = N1 N2
 * as in the NTT passes), written by fiona_rotation_key_layout from a key in
 * natural order (once per key).
 *
 * fiona_rotation_key_layout: key_out = the library layout of key (both device,
 *   fiona_rotation_key_words words, not overlapping) for Galois element
 *   galois (odd, < 2N).  Asynchronous on stream; allocates nothing.
 *
 * fiona_hoisted_rotate: n_rot rotations of one ciphertext.
 *   ct       device, [2][L][N] canonical residues (NTT domain)
 *   galois   host, [n_rot] Galois elements (odd, < 2N; 5^r mod 2N rotates by r)
 *   keys     device, [n_rot] keys in the library layout, key r for galois[r];
 *            16-byte aligned (read 16 bytes per lane)
 *   out_cts  device, [n_rot][2][L][N], overwritten with canonical residues;
 *            must not overlap ct or keys
 *   n_rot    at most the rotator's max_rot
 * Asynchronous on stream; allocates nothing, and issues kernel launches only
 * (the Galois elements travel by value in the launch arguments), so a call
 * can be captured in a HIP graph.  The workspace is shared by the rotator's
 * calls: one rotator must not be used by two streams at the same
 * time.  Results are exact: bit-identical to the definition above computed
 * in integers.  Errors (nothing is launched): FIONA_ERR_ARG, FIONA_ERR_ALIGN,
 * FIONA_ERR_ALIAS, FIONA_ERR_HIP.
 */
typedef struct fiona_rotator fiona_rotator;
int fiona_rotator_create(const fiona_ctx *ctx, uint64_t special_prime, const uint64_t *psi, uint32_t max_rot,
                         fiona_rotator **out);
void fiona_rotator_destroy(fiona_rotator *rotator);
uint64_t fiona_rotation_key_words(const fiona_rotator *rotator);
int fiona_rotation_key_layout(const fiona_rotator *rotator, uint32_t galois, const uint64_t *key,
                              uint64_t *key_out, hipStream_t stream);
int fiona_hoisted_rotate(const fiona_rotator *rotator, const uint64_t *ct, uint32_t n_rot, const uint32_t *galois,
                         const uint64_t *keys, uint64_t *out_cts, hipStream_t stream);

/* ------------------------------------------------------------------------
 * The key holder's operators.
 *
 * Between two encrypted projections of a transformer stand steps that residues
 * have no exact form for (a softmax, its maximum, a division).  A program that
 * runs them at the key holder has the decrypted rows of a projection on its
 * own GPU: it adds its private adapters' part to them (fiona_adapter_linear),
 * appends the keys and values to its cache (fiona_kv_append), attends
 * (fiona_paged_attention) and encrypts the result for the next projection.
 * The adapters are trained there too (fiona_adapter_backward).
 *
 * Elements are IEEE binary32, binary16 or bfloat16.  Whatever the type, every
 * product is summed in 32 bits, softmax statistics are held in 32 bits, and a
 * result is rounded to its type once.  Two intermediate values are multiplied in
 * fewer bits where the type has 16: fiona_paged_attention's softmax weights, in the
 * type itself (half a unit of each weight; their sum is not rounded), and the
 * adapters' h and g, as two bfloat16 parts (2^-16 of the value).  Every launch goes
 * to the current device.  Strides count elements; the last axis
 * of every array is contiguous.  Device pointers need the alignment of their
 * elements; where pointers and strides are multiples of 16 bytes and rows are
 * multiples of 8 elements the kernels read and write 16 bytes per lane.
 * ------------------------------------------------------------------------ */
typedef enum fiona_type { FIONA_F32 = 0, FIONA_F16 = 1, FIONA_BF16 = 2 } fiona_type;

#define FIONA_MAX_HEAD_DIM 256u
#define FIONA_MAX_RANK 128u

/*
 * A paged cache: key (and value) row `head` of the token in place `at` of page
 * `page` starts at element page * k_page + at * k_token + head * k_head of k.
 * Rows of different (page, place, head) must not overlap, nor k with v.
 */
typedef struct fiona_kv_cache {
  uint32_t type;       /* fiona_type of both arrays */
  uint32_t n_pages, page_size, n_kv, head_dim;   /* head_dim <= FIONA_MAX_HEAD_DIM; n_pages * page_size < 2^31 */
  void *k, *v;         /* device */
  uint64_t k_page, k_token, k_head;
  uint64_t v_page, v_token, v_head;
} fiona_kv_cache;

/*
 * fiona_kv_append: rotate the new tokens' keys (and queries) by their
 * positions and write keys and values into the cache.
 *
 * Pair i < rot_dim / 2 of a row, elements (i, i + rot_dim / 2), or
 * (2 i, 2 i + 1) with interleaved, becomes
 *     (a cos[p][i] - b sin[p][i],  a sin[p][i] + b cos[p][i])
 * at the token's position p; elements from rot_dim on are copied.
 *   rows_type   fiona_type of k, v and q
 *   k, v        device, [n_tok][n_kv][head_dim]
 *   q, q_out    device, [n_tok][n_head][head_dim], or NULL with n_head 0;
 *               q_out has the cache's type; it may be q itself (same type and strides)
 *   slots       device, [n_tok]: page * page_size + place of each token; a token
 *               whose slot lies outside the cache is not written (padding: -1).
 *               Slots of one call are distinct, or which token is kept is unspecified
 *   positions   device, [n_tok], with rot_dim > 0
 *   cos, sin    device, [n_pos][rot_dim / 2] (not read with n_pos 0); a token whose
 *               position lies outside [0, n_pos) gets NaN in its rotated elements
 * Asynchronous on stream; one kernel launch, allocates nothing.  Errors
 * (nothing is launched): FIONA_ERR_ARG, FIONA_ERR_UNSUPPORTED (a type or size
 * outside its range), FIONA_ERR_ALIGN, FIONA_ERR_ALIAS (an output overlaps an
 * input or another output; cache rows that overlap each other), FIONA_ERR_HIP.
 */
typedef struct fiona_append_args {
  uint32_t n_tok, n_head, rows_type, rot_dim, n_pos, interleaved;
  const void *k, *v, *q;
  void *q_out;
  uint64_t k_tok, k_head, v_tok, v_head, q_tok, q_head, q_out_tok, q_out_head;
  const int64_t *slots;
  const int32_t *positions;
  const float *cos, *sin;
} fiona_append_args;

int fiona_kv_append(const fiona_kv_cache *cache, const fiona_append_args *args, hipStream_t stream);

/*
 * fiona_attention_create: the workspace of fiona_paged_attention (the parts of
 * a long cache's softmax that are joined), for up to max_seq sequences of up
 * to max_length tokens.  n_head is a multiple of n_kv: query head h reads key
 * head h / (n_head / n_kv).  Errors: FIONA_ERR_ARG, FIONA_ERR_UNSUPPORTED
 * (a type or size outside its range), FIONA_ERR_NOMEM, FIONA_ERR_HIP.
 */
typedef struct fiona_attention_desc {
  uint32_t type, n_head, n_kv, head_dim, page_size, max_seq, max_length;
} fiona_attention_desc;

typedef struct fiona_attention fiona_attention;
int fiona_attention_create(const fiona_attention_desc *desc, fiona_attention **out);
void fiona_attention_destroy(fiona_attention *att);

/*
 * fiona_paged_attention: one new token of each sequence attends to its cache.
 * With n the sequence's length (the new token included), first = n - window
 * (0 without a window, or below it), and key j in page page_table[j / page_size]
 * at place j mod page_size,
 *     s_j = scale q . k_j,  or softcap tanh(s_j / softcap) with a softcap
 *           (its error is relative to s_j, whatever the softcap),
 *     out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),   first <= j < n
 *     lse = m + log sum_j exp(s_j - m),                    m = max_j s_j.
 *   n_seq       at most the handle's max_seq
 *   q, out      device, [n_seq][n_head][head_dim], of the handle's type
 *   lse         device, [n_seq][n_head] float32, or NULL
 *   page_table  device, [n_seq] rows of table_width entries, table_stride
 *               apart (0: one row for all).  A key whose entry lies outside
 *               [0, n_pages) is left out, as if it were masked
 *   lengths     device, [n_seq]; clamped to [0, min(max_length,
 *               table_width * page_size)]
 *   scale > 0; window 0: none; softcap 0: none, else > 0
 * A sequence with no key, or none whose score is above -inf, gets out = 0 and
 * lse = -inf.  Cache places past a
 * sequence's length are never used, whatever they hold.
 * Asynchronous on stream; one or two kernel launches, allocates nothing.  The
 * workspace is shared by the handle's calls: one handle must not be used by
 * two streams at the same time.  Errors (nothing is launched): FIONA_ERR_ARG
 * (also a cache that does not match the handle), FIONA_ERR_UNSUPPORTED,
 * FIONA_ERR_ALIGN, FIONA_ERR_ALIAS, FIONA_ERR_HIP.
 */
typedef struct fiona_attention_args {
  uint32_t n_seq, table_width, window;
  float scale, softcap;
  const void *q;
  void *out;
  float *lse;
  uint64_t q_seq, q_head, out_seq, out_head, table_stride;
  const int32_t *page_table;
  const int32_t *lengths;
} fiona_attention_args;

int fiona_paged_attention(const fiona_attention *att, const fiona_kv_cache *cache, const fiona_attention_args *args,
                          hipStream_t stream);

/*
 * Low-rank adapters of many requests beside a shared projection.  Token t has
 * adapter a = ids[t] (any order; an id outside [0, n_adapter): none) of rank
 * r = ranks[a] (clamped to [0, max_rank]; NULL: max_rank) and scaling
 * c = scaling[a] (NULL: 1):
 *     h_t = A_a x_t,   y_t = base_t + c B_a h_t.
 *
 * fiona_adapters_create: the workspace of calls of up to max_tokens tokens.
 * Errors: FIONA_ERR_ARG, FIONA_ERR_UNSUPPORTED (a type, a rank over
 * FIONA_MAX_RANK, a size outside its range), FIONA_ERR_NOMEM, FIONA_ERR_HIP.
 *
 * fiona_adapter_linear:
 *   x     device, [n_tok][d_in]            A  device, [n_adapter][max_rank][d_in]
 *   base  device, [n_tok][d_out], or NULL  B  device, [n_adapter][d_out][max_rank]
 *         (zero); it may be y itself       y  device, [n_tok][d_out]
 * Rows of A and columns of B from the adapter's rank on are not used.  A token
 * without an adapter gets y_t = base_t.
 *
 * fiona_adapter_backward: from dy, the gradient of y,
 *     g_t = c B_a^T dy_t,   dx_t = dx_base_t + A_a^T g_t,
 *     dA_a = sum over its tokens of g_t x_t^T,   dB_a = c sum dy_t h_t^T
 * dx_base may be NULL (zero) or dx itself (the gradient through the shared
 * projection); dA and dB are overwritten whole, with zeros for adapters no
 * token has and from an adapter's rank on.  The gradient of base is dy.
 * Sums run in a fixed order: the same call gives the same bits.
 * Rows of other tokens never reach a token's outputs, whatever they hold; a
 * token's own infinities reach them (and its adapter's gradients) as infinities
 * or NaN.
 *
 * Both: asynchronous on stream, kernel launches only, allocate nothing.  The
 * workspace is shared by the handle's calls: one handle must not be used by
 * two streams at the same time.  Errors (nothing is launched): FIONA_ERR_ARG,
 * FIONA_ERR_UNSUPPORTED (rows more than 2^24 elements apart), FIONA_ERR_ALIGN,
 * FIONA_ERR_ALIAS, FIONA_ERR_HIP.
 */
#define FIONA_ADAPTERS_FORWARD_ONLY 1u   /* no workspace for fiona_adapter_backward (FIONA_ERR_ARG on such a handle) */

typedef struct fiona_adapters_desc {
  uint32_t type, n_adapter, max_rank, d_in, d_out, max_tokens, flags;
} fiona_adapters_desc;

typedef struct fiona_adapter_args {
  uint32_t n_tok;
  const void *x, *A, *B;
  const int32_t *ids;
  const int32_t *ranks;    /* [n_adapter] or NULL */
  const float *scaling;    /* [n_adapter] or NULL */
  uint64_t x_row;
  /* fiona_adapter_linear */
  const void *base;
  void *y;
  uint64_t base_row, y_row;
  /* fiona_adapter_backward */
  const void *dy, *dx_base;
  void *dx, *dA, *dB;
  uint64_t dy_row, dx_base_row, dx_row;
} fiona_adapter_args;

typedef struct fiona_adapters fiona_adapters;
int fiona_adapters_create(const fiona_adapters_desc *desc, fiona_adapters **out);
void fiona_adapters_destroy(fiona_adapters *adapters);
int fiona_adapter_linear(const fiona_adapters *adapters, const fiona_adapter_args *args, hipStream_t stream);
int fiona_adapter_backward(const fiona_adapters *adapters, const fiona_adapter_args *args, hipStream_t stream);

/* ------------------------------------------------------------------------
 * The key holder's training step: a norm between projections, losses on the
 * logits with their gradients, and the optimiser that applies fiona_adapter_backward's.
 * Types, rounding, strides, alignment and streams as above: 32-bit sums and
 * statistics, one rounding of each result, sums in a fixed order.
 * ------------------------------------------------------------------------ */
#define FIONA_MAX_NORM_WIDTH 32768u
#define FIONA_MAX_NORM_ROWS (1u << 22)

/*
 * fiona_layer_norm: with s_t = x_t, or x_t + residual_t rounded to the type,
 *     mean = sum s / width,  rstd = 1 / sqrt(sum (s - mean)^2 / width + eps),
 *     y_t = weight (s_t - mean) rstd + bias
 *   type, weight_type  fiona_type of the rows, and of weight and bias (the rows' type or FIONA_F32)
 *   x, residual   device, [n][width]; residual NULL: none
 *   weight, bias  device, [width], or NULL (one, zero)
 *   y, total      device, [n][width]; total receives s, or is NULL.  y or total may be x or residual
 *                 itself (same pointer and stride), but not both the same
 *   mean, rstd    device, [n] float32, or NULL
 *   eps > 0; width at most FIONA_MAX_NORM_WIDTH, n at most FIONA_MAX_NORM_ROWS
 * Asynchronous on stream; one kernel launch, allocates nothing.  Errors
 * (nothing is launched): FIONA_ERR_ARG, FIONA_ERR_UNSUPPORTED, FIONA_ERR_ALIGN,
 * FIONA_ERR_ALIAS, FIONA_ERR_HIP.
 */
typedef struct fiona_norm_args {
  uint32_t n, width, type, weight_type;
  float eps;
  const void *x, *residual, *weight, *bias;
  void *y, *total;
  float *mean, *rstd;
  uint64_t x_row, residual_row, y_row, total_row;
} fiona_norm_args;

int fiona_layer_norm(const fiona_norm_args *args, hipStream_t stream);

/*
 * fiona_layer_norm_backward: from dy, the gradient of y, with xh = (x - mean) rstd
 * (x: what was normalised, s above) and u = weight dy,
 *     dx_t = dx_base_t + rstd (u - sum u / width - xh sum (u xh) / width)
 *     dweight = sum over the rows of dy xh,   dbias = sum of dy
 *   dy, x, dx_base, dx  device, [n][width]; dx_base NULL: zero (else the gradient that
 *                       reaches s by other ways); dx may be dx_base, dy or x itself
 *   mean, rstd          device, [n] float32, as fiona_layer_norm wrote them
 *   weight              device, [width], or NULL (one)
 *   dweight, dbias      device, [width], of the weight's type, overwritten (zeros with n 0);
 *                       NULL: not wanted
 * fiona_norm_create: the workspace (the parts of dweight and dbias) for up to
 * max_rows rows.  Asynchronous on stream; at most three kernel launches, allocates nothing.
 * The workspace is shared by the handle's calls: one handle must not be used by
 * two streams, or in two graphs that run, at the same time.  Errors: as above, and
 * FIONA_ERR_NOMEM from fiona_norm_create.
 */
typedef struct fiona_norm_desc {
  uint32_t type, weight_type, width, max_rows;
} fiona_norm_desc;

typedef struct fiona_norm_backward_args {
  uint32_t n;
  const void *dy, *x, *weight;
  const float *mean, *rstd;
  const void *dx_base;
  void *dx, *dweight, *dbias;
  uint64_t dy_row, x_row, dx_base_row, dx_row;
} fiona_norm_backward_args;

typedef struct fiona_norm fiona_norm;
int fiona_norm_create(const fiona_norm_desc *desc, fiona_norm **out);
void fiona_norm_destroy(fiona_norm *norm);
int fiona_layer_norm_backward(const fiona_norm *norm, const fiona_norm_backward_args *args, hipStream_t stream);

/*
 * Losses on tokens' logits z, [n_tok][vocab], and the gradient with respect to
 * them.  A token's log-probability is
 *     l_t = z_t[targets[t]] - log sum_j exp(z_t[j]);
 * a target outside [0, vocab) says that the token does not count (a prompt,
 * padding): its logits are never used, whatever they hold, and its row of dlogits
 * is zero.  A loss whose derivative with respect to l_t is g_t has
 *     dlogits_t = g_t (onehot(targets[t]) - softmax(z_t)),
 * zero where g_t is.  dlogits may be NULL (no gradient) or logits itself (same
 * pointer and stride).
 *
 * fiona_token_loss_create: the workspace of calls of up to max_tokens tokens and
 * max_pairs pairs (0: none) of vocab logits.  Limits: vocab, max_tokens and
 * max_pairs at most 2^21.
 *
 * fiona_preference_loss: sequence s has tokens offsets[s] to offsets[s + 1] - 1;
 * sequence 2 p is the preferred one of pair p, 2 p + 1 the other.  With L_s the sum
 * of its tokens' log-probabilities and R_s = reference[s], the same of another model,
 *     h = beta ((L_{2p} - R_{2p}) - (L_{2p+1} - R_{2p+1})),
 *     loss_p = -w_p ((1 - label_smoothing) log sigmoid(h) + label_smoothing log sigmoid(-h))
 * with w_p = weights[p], or 1 / n_pair without; logps receives L.
 *   targets, offsets  device, [n_tok] and [2 n_pair + 1] (clamped to [0, n_tok]; not decreasing, or
 *                     the gradients of tokens in several sequences are one of theirs);
 *                     tokens of no sequence do not count
 *   reference, logps  device, [2 n_pair]
 *   loss, weights     device, [n_pair]; weights NULL: 1 / n_pair
 *   beta > 0, label_smoothing in [0, 1)
 * A pair of weight zero has no loss and no gradient, whatever its logits.
 *
 * fiona_policy_loss: with the ratio r = exp(l_t - old_t) to the policy that sampled
 * the token, its advantage A and d = reference_t - l_t,
 *     loss_t = w_t (-min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl (exp(d) - d - 1))
 * with w_t = weights[t], or 1 / n_tok without; logps receives l.  Tokens that do not
 * count get loss and logps 0.
 *   old, advantages, loss, logps   device, [n_tok]
 *   reference   device, [n_tok]; not read (NULL) with kl 0
 *   weights     device, [n_tok], or NULL
 *   clip_low in [0, 1], clip_high >= 0, kl >= 0
 * Where the ratio stands at an end of the clip the free product's derivative is taken.  A token of weight
 * zero has no loss and no gradient, whatever its logits.
 *
 * Both: asynchronous on stream, kernel launches only, allocate nothing.  The
 * workspace is shared by the handle's calls: one handle must not be used by two
 * streams, or in two graphs that run, at the same time.  Errors (nothing is launched): FIONA_ERR_ARG,
 * FIONA_ERR_UNSUPPORTED, FIONA_ERR_ALIGN, FIONA_ERR_ALIAS, FIONA_ERR_HIP.
 */
typedef struct fiona_token_loss_desc {
  uint32_t type, vocab, max_tokens, max_pairs;
} fiona_token_loss_desc;

typedef struct fiona_preference_args {
  uint32_t n_tok, n_pair;
  float beta, label_smoothing;
  const void *logits;
  void *dlogits;
  uint64_t logits_row, dlogits_row;
  const int32_t *targets, *offsets;
  const float *reference, *weights;
  float *loss, *logps;
} fiona_preference_args;

typedef struct fiona_policy_args {
  uint32_t n_tok;
  float clip_low, clip_high, kl;
  const void *logits;
  void *dlogits;
  uint64_t logits_row, dlogits_row;
  const int32_t *targets;
  const float *old, *advantages, *reference, *weights;
  float *loss, *logps;
} fiona_policy_args;

typedef struct fiona_token_loss fiona_token_loss;
int fiona_token_loss_create(const fiona_token_loss_desc *desc, fiona_token_loss **out);
void fiona_token_loss_destroy(fiona_token_loss *loss);
int fiona_preference_loss(const fiona_token_loss *loss, const fiona_preference_args *args, hipStream_t stream);
int fiona_policy_loss(const fiona_token_loss *loss, const fiona_policy_args *args, hipStream_t stream);

/*
 * fiona_adamw_step: one step over all tensors of a handle, each of n contiguous
 * elements.  With g the gradient (times *grad_scale), t = *step and lr = *lr,
 *     m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
 *     p = p - lr weight_decay p - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps),
 * p rounded once a step (so that a decay far below 2^-24 p a step is applied in the mean)
 *   param, grad  device, of the desc's type; param is written
 *   master       device, float32, or NULL.  With it p is the master, and param its value rounded;
 *                without, what a step changes by less than half a unit of a 16-bit param is lost
 *   m, v         device: float32 (state_bits 32), or (8) e4m3 values c of blocks of
 *                FIONA_ADAMW_BLOCK elements, counted from the tensor's first, that stand
 *                for m = c m_scale and sqrt(v) = c v_scale of their block
 *   m_scale, v_scale  device, float32, one to a block (a last short one as well); NULL with 32 bits
 *   weight_decay  at least zero, finite in 32 bits
 *   lr, step, grad_scale  device, one float32, int32 (from 1 on; less counts as 1) and float32 (NULL:
 *                1): read when the step runs, so that a captured one follows them
 * 8-bit states: the new m and v, from operations in 32 bits each rounded by itself, are used, then rounded to one of the two
 * neighbouring values, up with the probability that keeps their mean (rounded to
 * nearest, beta2 v would stay v for ever); sqrt(v) > 0 is never rounded to zero.  A
 * block's scale is its largest magnitude / 448 (zero, as its values, below 2^-100; of v below 2^-126 less
 * than the root is taken).  The dither of
 * element i is 16 bits for m (low) and 16 for v (high) of mix(i ^ mix(step 0x9E3779B1 + seed)) in
 * 32-bit arithmetic, i counting from the first tensor on, every tensor from a multiple of the block;
 *     mix(x): x ^= x >> 16; x *= 0xA3D8B167; x ^= x >> 15; x *= 0xC94F6E2B; x ^= x >> 16.
 * A gradient that is no number makes its element's states and parameter so.  With 8 bits one whose square
 * passes float32's range does the same to v and the parameter, and an infinite one to m of its block.
 *
 * fiona_adamw_create keeps the tensors' addresses, not the tensors: they have to
 * live, where they are, as long as the handle is used.  What is written must not
 * overlap anything else of any tensor (FIONA_ERR_ALIAS).  Limit: fewer than 2^24 pieces
 * of 1024 elements, a tensor's last one counted whole (FIONA_ERR_UNSUPPORTED).
 * fiona_adamw_step: asynchronous on stream; one kernel launch, allocates nothing.
 * Errors: FIONA_ERR_ARG, FIONA_ERR_UNSUPPORTED, FIONA_ERR_ALIGN, FIONA_ERR_ALIAS,
 * FIONA_ERR_NOMEM, FIONA_ERR_HIP.
 */
#define FIONA_ADAMW_BLOCK 256u

typedef struct fiona_adamw_tensor {
  void *param;
  const void *grad;
  float *master;
  void *m, *v;
  float *m_scale, *v_scale;
  uint64_t n;
  double weight_decay;
} fiona_adamw_tensor;

typedef struct fiona_adamw_desc {
  uint32_t type, state_bits, n_tensor, seed;
  double beta1, beta2, eps;              /* betas in [0, 1), eps a normal float32 > 0 */
  const fiona_adamw_tensor *tensors;     /* host, [n_tensor] */
} fiona_adamw_desc;

typedef struct fiona_adamw fiona_adamw;
int fiona_adamw_create(const fiona_adamw_desc *desc, fiona_adamw **out);
void fiona_adamw_destroy(fiona_adamw *opt);
int fiona_adamw_step(const fiona_adamw *opt, const float *lr, const int32_t *step, const float *grad_scale,
                     hipStream_t stream);

/*
 * Measurement helper (not part of the weighted sum): the register-only rate
 * of the raw route's arithmetic, against which the hybrid kernel's
 * multiply-add rate is compared.
 *
 * fiona_mac_microbench: launches blocks workgroups of 256 threads; every
 *   thread multiplies chunks * 56 plaintext words held in registers into both
 *   polynomials' exact accumulators, as the hybrid kernel does for one raw
 *   term at one position (four 32x32->64 multiply-adds per polynomial, a
 *   carry step every 56 words), reads no memory, and writes one word to
 *   sink[thread] (device, blocks * 256 words, caller-owned; the values mean
 *   nothing).  Asynchronous on stream; allocates nothing.  Errors:
 *   FIONA_ERR_ARG (blocks or chunks 0, sink NULL), FIONA_ERR_HIP.
 * fiona_mac_microbench_words: the plaintext words one such launch multiplies
 *   (blocks * 256 * chunks * 56).
 */
int fiona_mac_microbench(uint32_t blocks, uint32_t chunks, uint64_t *sink, hipStream_t stream);
uint64_t fiona_mac_microbench_words(uint32_t blocks, uint32_t chunks);

/*
 * Measurement helpers (not part of the weighted sum): the HBM bandwidth of a
 * plain contiguous read, of a plain copy and of a plain write, the ceilings
 * the kernels' rates are set against.  Grid-stride loops over 16-byte words
 * on blocks workgroups of 256 threads, nontemporal accesses.
 * fiona_stream_read: reads words (even) uint64 words of src (device, 16-byte
 *   aligned) and writes one word per workgroup to sink (device, blocks words).
 * fiona_stream_copy: dst[i] = src[i] for words (even) words (device, 16-byte
 *   aligned, not overlapping).
 * fiona_stream_write: writes words (even) words of dst (device, 16-byte
 *   aligned) with a pattern of the slot index; reads nothing.
 * Asynchronous on stream; allocate nothing.  Errors: FIONA_ERR_ARG,
 * FIONA_ERR_ALIGN, FIONA_ERR_ALIAS (copy), FIONA_ERR_HIP.
 */
int fiona_stream_read(const uint64_t *src, uint64_t words, uint32_t blocks, uint64_t *sink, hipStream_t stream);
int fiona_stream_copy(const uint64_t *src, uint64_t *dst, uint64_t words, uint32_t blocks, hipStream_t stream);
int fiona_stream_write(uint64_t *dst, uint64_t words, uint32_t blocks, hipStream_t stream);

/*
 * Checking helper (no device needed): replays the memory accesses of one
 * rescale (op 0) or one hoisted-rotation call (op 1) on the host.  The
 * rescaler (capacity = max_ct) or rotator (capacity = max_rot) is laid out
 * at fake device addresses, the call's launches are recorded instead of
 * issued, and every global access of every workgroup and thread of every NTT
 * pass and launch of whole transforms is recomputed with the kernels' own
 * offset arithmetic, as are the whole transforms' LDS words; the inner product
 * and the transpose are checked by the byte ranges they touch.
 *   moduli      host, L moduli (op 0) or L data moduli then the special
 *               prime (op 1), each = 1 mod 2N
 *   n_call      ciphertexts (op 0) or rotations (op 1) of the call; the
 *               rotations use Galois elements 5^r, then 2N - 1 and 1
 *   out_shrink  the caller's output buffer is taken to be this many bytes
 *               short (0 for the real size; a positive value checks that
 *               the checker finds the overrun)
 *   msg         host, msg_len bytes: the first violation, or ""
 * Returns FIONA_OK if every access lies inside the buffer that holds its
 * descriptor's base, below 2^32 bytes from it, with every descriptor's end
 * pointer at that buffer's end; FIONA_ERR_BOUNDS otherwise; the errors of
 * fiona_rescaler_create / fiona_rotator_create for bad parameters.
 */
int fiona_check_ntt_offsets(uint32_t op, uint32_t N, uint32_t L, const uint64_t *moduli, uint32_t capacity,
                            uint32_t n_call, uint64_t out_shrink, char *msg, size_t msg_len);

/* Static string naming a status code. */
const char *fiona_status_string(int status);

#ifdef __cplusplus
}
#endif

#endif /* FIONA_H */
