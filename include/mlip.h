/*
 * mlip.h - C ABI of the MI355X (gfx950) small-footprint MLIP library.
 *
 * The library evaluates the per-atom energy, forces and virial of the
 * machine-learning interatomic potential of arXiv 2608.16329 (Section 3.1,
 * Eqs. 1-10): for every atom it gathers the neighbours inside the cutoff,
 * builds the species-conditioned radial features (Eq. 2) and the
 * irreducible-harmonic angular features (Eq. 3, Section 3.3), contracts them
 * to the equivariant moment P_i (Eq. 4) and invariant descriptor G_i (Eq. 5),
 * runs the energy head (Eq. 6) and back-propagates analytically to partial
 * forces (Eqs. 7-10).  The MLIP receives coordinates from the MD code and
 * returns energies and forces (Section 2.1, "MLIP Inference").
 *
 * Conventions shared by every call:
 *   - "_dev" pointers are device memory on the context's device (for
 *     example PyTorch-ROCm tensors), contiguous, row-major; "_host" pointers
 *     are host memory.  The caller owns every buffer it passes; the library
 *     never frees or retains caller memory beyond the call, except that
 *     mlip_compute reads the species array given to the last
 *     mlip_build_neighbors from the library's own copy.
 *   - Atom arrays are in the caller's order.  Positions are float64 [n][3]
 *     in Angstrom, species are int32 [n], forces float64 [n][3] in eV/A,
 *     energies float64 [n] in eV, virials float64 [n][9] in eV (row-major
 *     3x3).
 *   - Work is enqueued on the HIP stream given to mlip_create and the call
 *     returns without waiting, unless stated otherwise.
 *   - Every call returns a status; nothing throws or aborts across the ABI.
 *     On failure mlip_last_error(ctx) describes the cause.
 *   - A context is not thread-safe; use one context per host thread.
 *   - Every buffer crossing the ABI is float64 or int32.  The arithmetic of
 *     the network is set by mlip_hparams.precision: 64 evaluates everything
 *     in float64 (Section 4.1); 32 is the reduced-precision mode the paper
 *     evaluates beside it (Sections 3.4 and 4.4), here with the network, the
 *     angular features, the moment/adjoint contractions and the pair
 *     geometry after the minimum-image difference in float32, and that
 *     difference and all force, virial and energy accumulation in float64.
 *     The matrix products of the radial encoder take one of two forms, chosen
 *     in mlip_create by the weights alone:
 *       - sums of 8-bit integer products, exact, of the weights and values
 *         rounded to 56-bit (precision 64) or 32-bit (32) integers with one
 *         scale per weight row and per pair, rounded to the type at the end.
 *         They err by a part of (largest weight of the row) x (largest value
 *         of the pair), below 128 x 2^-53 or 128 x 2^-29 of it;
 *       - products and sums of the type, which err by a part of the sum of the
 *         absolute terms.
 *     The first is taken where at 64 distances up to the cutoff no product of
 *     maxima exceeds the sum of the absolute terms (precision 32: 32 times
 *     that sum), which is where its outputs are as accurate as the second's:
 *     ordinary weights stay below 0.6 times, one hidden unit some ten times
 *     larger than the others and used with as much smaller weights does not.
 *     The first is faster, by a fifth in float64 and a third in float32.
 */
#ifndef MLIP_H
#define MLIP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct mlip_ctx mlip_ctx;

typedef enum {
  MLIP_OK = 0,
  MLIP_E_ARG = -1,      /* NULL pointer, bad size, unsupported hyper-parameter */
  MLIP_E_OOM = -2,      /* device allocation failed                            */
  MLIP_E_HIP = -3,      /* HIP runtime error                                   */
  MLIP_E_BOX = -4,      /* non-positive box edge, or cutoff+skin > min(L)/2    */
  MLIP_E_NBR_CAP = -5,  /* a neighbour row is longer than the kernel can hold  */
  MLIP_E_STATE = -6,    /* call out of order (compute before build_neighbors)  */
  MLIP_E_TYPE = -7      /* species outside [0, n_species) or non-finite input  */
} mlip_status;

/*
 * Hyper-parameters (Section 3.2 species conditioning, Section 3.3 angular
 * basis, Section 4.1 architecture).  Defaults of the paper: k = 32,
 * lmax = 3, irreducible basis, pair-conditioned encoder, species-conditioned
 * head, encoder 3 hidden layers of width 128, head 4 hidden layers of width
 * 64, cutoff 6 A.
 */
typedef struct {
  int32_t n_species;   /* C >= 1 (the GPU path supports C <= 16)                  */
  double  cutoff;      /* r_c in A                                               */
  double  skin;        /* Verlet skin in A; neighbour lists use r_c + skin       */
  int32_t k;           /* radial feature width (GPU path: 16, 32 or 64)          */
  int32_t lmax;        /* maximum angular order (GPU path: 0..5 irreducible,
                          0..3 Cartesian; the Cartesian basis needs k = 32)      */
  int32_t angular;     /* 0 irreducible harmonic basis, d = (lmax+1)^2;
                          1 Cartesian monomials, d = (lmax+1)(lmax+2)(lmax+3)/6,
                          descriptor metric l!/(a!b!c!) (Section 3.3)            */
  int32_t enc_cond;    /* encoder tables: 2 per (s_i,s_j), 1 per s_j, 0 one      */
  int32_t reg_cond;    /* head tables: 1 per s_i, 0 one                          */
  int32_t enc_width;   /* encoder hidden width (GPU path: 128)                   */
  int32_t enc_hidden;  /* encoder hidden layers (GPU path: 1..8)                 */
  int32_t reg_width;   /* head hidden width (GPU path: 64)                       */
  int32_t reg_hidden;  /* head hidden layers (GPU path: 1..8)                    */
  int32_t precision;   /* 64 (float64) or 32 (float32 network, see above)         */
} mlip_hparams;

/* Statistics of the context (mlip_get_stats). */
typedef struct {
  int64_t n_atoms;          /* atoms of the last neighbour build                 */
  int64_t n_listed_pairs;   /* directed pairs within cutoff + skin              */
  int64_t n_active_pairs;   /* directed pairs within cutoff at the last compute */
  int32_t max_row;          /* longest neighbour row                             */
  int32_t tile_atoms;       /* centre atoms per work-group tile                  */
  int64_t n_tiles;          /* tiles of the fused kernel                         */
  int32_t n_blocks;         /* resident work-groups of the fused kernel          */
  int32_t n_cells;          /* cells of the neighbour grid                       */
  int64_t n_builds;         /* neighbour builds so far                           */
  size_t  device_bytes;     /* device memory held by the context                 */
  int32_t list_entry_bytes; /* bytes per neighbour-list entry: 2 (coded), 4      */
} mlip_stats;

/*
 * Number of float64 values in the packed weight blob for these
 * hyper-parameters; 0 if the hyper-parameters are invalid.
 *
 * Blob layout (row-major, matrices [out][in], W = enc_width, R = reg_width):
 *   encoder tables, tau = s_i*C + s_j (enc_cond 2), s_j (1) or 0 (0), each
 *     w0[W] b0[W], then for t = 1..enc_hidden-1: W_t[W][W] b_t[W],
 *     then W_out[k][W] b_out[k]
 *   head tables, rho = s_i (reg_cond 1) or 0, each
 *     A0[R][(lmax+1)*k] c0[R], then for t = 1..reg_hidden-1: A_t[R][R] c_t[R],
 *     then a_out[R] c_out[1]
 * Encoder: h = silu(w0 r + b0); h += silu(W_t h + b_t); g = fc(r) (W_out h +
 * b_out) with fc(r) = (1 + cos(pi r / r_c)) / 2 (Eq. 2).  Head: y =
 * silu(A0 x + c0); y += silu(A_t y + c_t); E_i = a_out . y + c_out (Eq. 6)
 * with x = vec(G_i) in l-major order (index l*k + c).
 */
size_t mlip_weight_count(const mlip_hparams* hp);

/*
 * Create a context on the current HIP device.  Copies and repacks the
 * weights (weights_host, n_weights float64 values, layout above) into device
 * memory, rounded to float32 when precision is 32 (encoder matrices on integer
 * products: to integers of 56 or 32 bits), and builds the angular projection
 * tables.  hip_stream is a
 * hipStream_t (NULL = default stream); all later work is enqueued on it.
 * Errors: MLIP_E_ARG (bad hparams, unsupported on the GPU path, n_weights
 * mismatch, NULL pointers), MLIP_E_OOM, MLIP_E_HIP.  On error *out is NULL
 * and mlip_last_error(NULL) says why.
 */
mlip_status mlip_create(const mlip_hparams* hp, const double* weights_host, size_t n_weights,
                        void* hip_stream, mlip_ctx** out);

/*
 * Build the neighbour list (Section 3.1: N(i) = atoms within the cutoff;
 * here within cutoff + skin so the list stays valid while atoms move less
 * than skin/2).  Definition (exact, reproducible bit for bit): coordinates
 * wrapped into [0, L) by w = fmod(x, L), +L if negative, -L if >= L; pair
 * vector dx = w_j - w_i folded once by -L if dx > L/2 or +L if dx < -L/2;
 * d2 = (dx*dx + dy*dy) + dz*dz without fused multiply-add; j != i is listed
 * iff d2 < (cutoff + skin)^2.  Rows are grouped by neighbour species.
 * Entries take 2 bytes each (the neighbour's place among the cells scanned
 * around the centre's cell, its species and its place in that cell's
 * species bucket) when every (species, cell) bucket of the cell grid holds at
 * most 2^(11 - ceil(log2 C)) atoms, 4 bytes (its index) otherwise or when
 * mlip_set_list_format asks for indices; mlip_get_stats reports which.
 *   n_atoms   number of atoms (>= 0, < 2^31).  0 records an empty system
 *             (the pointers may then be NULL): later calls succeed and
 *             produce nothing, totals and kinetic energy 0
 *   pos_dev   float64 [n_atoms][3], any real values (wrapped internally)
 *   types_dev int32 [n_atoms], species in [0, n_species); copied
 *   box_host  float64 [3], orthorhombic periodic box edges L_x, L_y, L_z
 * Synchronises the stream (the list length sizes the allocation).
 * Errors: MLIP_E_ARG, MLIP_E_BOX, MLIP_E_TYPE (bad species or non-finite
 * position), MLIP_E_NBR_CAP (a row longer than 2048), MLIP_E_OOM, MLIP_E_HIP.
 */
mlip_status mlip_build_neighbors(mlip_ctx* ctx, int64_t n_atoms, const double* pos_dev,
                                 const int32_t* types_dev, const double box_host[3]);

/*
 * Evaluate energies, forces and virial at pos_dev (float64 [n][3], same n as
 * the last build; atoms must have moved less than skin/2 since then) in one
 * fused pass per atom tile (Eqs. 1-10) that keeps every intermediate on chip
 * except the per-pair radial features, which stay in a fixed-size
 * per-work-group workspace.  Outputs are overwritten:
 *   energy_dev  float64 [n] per-atom E_i, or NULL
 *   forces_dev  float64 [n][3] F_i = -dE/dr_i (required)
 *   virial_dev  float64 [n][9] per-atom w_i = -sum_j r_ij (x) f_ij with
 *               r_ij = r_j - r_i, f_ij = dE_i/dr_ij (row-major), or NULL
 *   totals_host float64 [10] = (E, W[0..8]) summed over atoms, or NULL; when
 *               non-NULL the call synchronises the stream.
 * Errors: MLIP_E_ARG, MLIP_E_STATE (no build), MLIP_E_HIP.
 */
mlip_status mlip_compute(mlip_ctx* ctx, const double* pos_dev, double* energy_dev,
                         double* forces_dev, double* virial_dev, double* totals_host);

/*
 * mlip_compute without device allocation, for callers that cannot allocate:
 * code under HIP graph capture, tight serving loops, hosts that forbid
 * hipMalloc after set-up.  Same arguments, evaluation and outputs as
 * mlip_compute in the single-kernel configurations (MLIP_FUSION_CACHED,
 * MLIP_FUSION_RECOMPUTE).  The fused kernel's per-work-group workspace, the
 * block totals and the active-pair counter go to a fixed scratch array of
 * MLIP_STATIC_SCRATCH_BYTES built into the library, one per device, which
 * that device holds from the first call on it until the process ends; no
 * allocating routine is called.
 *
 * Every call on one device shares that device's scratch and leaves its
 * contents there (the totals and the counter are cleared at the start of a
 * call, the workspace is written before it is read): calls that overlap on
 * one device, from any context or stream, race and give wrong results.
 * Serialise them.  The context's device must be current.
 *
 * Errors: those of mlip_compute; MLIP_E_ARG when the configuration is
 * MLIP_FUSION_PARTIAL or MLIP_FUSION_UNFUSED (they keep per-atom
 * intermediates the library allocates) or when the workspace of the current
 * neighbour list (resident work-groups x per-work-group slot) exceeds the
 * scratch (mlip_last_error gives both sizes); MLIP_E_HIP when the scratch
 * cannot be resolved on the current device.
 */
#define MLIP_STATIC_SCRATCH_BYTES (256u * 1024u * 1024u)
mlip_status mlip_compute_noalloc(mlip_ctx* ctx, const double* pos_dev, double* energy_dev,
                                 double* forces_dev, double* virial_dev, double* totals_host);

/*
 * Copy the neighbour list to the host in caller order: offsets_host int64
 * [n+1], idx_host int32 [offsets[n]] (use mlip_get_stats().n_listed_pairs to
 * size it).  Entries of a row are grouped by neighbour species.  Synchronises.
 */
mlip_status mlip_get_neighbors(mlip_ctx* ctx, int64_t* offsets_host, int32_t* idx_host);

/*
 * Copy the neighbour rows of selected atoms to the host (for checks of the
 * list at sizes where the whole list is too large to copy; the rows are the
 * same as those of mlip_get_neighbors).
 *   atoms_host  int64 [n_rows], caller indices in [0, n), any order, repeats
 *               allowed
 *   counts_host int64 [n_rows], receives the length of each row
 *   idx_host    int32 [cap], receives the rows back to back in the order of
 *               atoms_host (caller indices, grouped by neighbour species)
 * Errors: MLIP_E_ARG (NULL pointer, index outside [0, n), or the rows do not
 * fit in cap entries: counts_host is filled even then), MLIP_E_STATE (no
 * build), MLIP_E_HIP.  Synchronises the stream.
 */
mlip_status mlip_get_neighbor_rows(mlip_ctx* ctx, const int64_t* atoms_host, int64_t n_rows, int64_t* counts_host,
                                   int32_t* idx_host, int64_t cap);

/*
 * Fusion configuration of mlip_compute (Section 3.4, Table "Configurable
 * fusion"); all four give the same results up to rounding.
 *   MLIP_FUSION_CACHED     one kernel: pass 1 keeps the encoder output and its
 *                          radial derivative per pair in a fixed-size
 *                          per-work-group workspace until pass 2 (default)
 *   MLIP_FUSION_RECOMPUTE  one kernel: pass 2 recomputes the encoder (the
 *                          paper's mega-fusion); no workspace traffic, twice
 *                          the encoder work
 *   MLIP_FUSION_PARTIAL    three kernels (Eqs. 1-5; Eq. 6; Eqs. 7-10, the
 *                          paper's partial fusion): G_i and then dE/dG_i go
 *                          through HBM, (l_max+1) k values per atom, which the
 *                          context allocates at the next mlip_compute
 *   MLIP_FUSION_UNFUSED    ten kernels, one per equation of Eqs. 1-10 (the
 *                          table's "before fusion" row): every intermediate
 *                          goes through HBM, per listed neighbour-list entry
 *                          the pair vector and distance, g_rad and dg_rad/dr,
 *                          g_ang and its Jacobian, and the U and V rows
 *                          (4 float64 + 176 values at k = 32), per atom P_i,
 *                          W_i and G_i / dE/dG_i (1152 values at k = 32,
 *                          l_max = 3); allocated at the next mlip_compute
 *                          (MLIP_E_OOM if they do not fit)
 * Values are float64 or float32 as set by mlip_hparams.precision.
 */
typedef enum {
  MLIP_FUSION_CACHED = 0,
  MLIP_FUSION_RECOMPUTE = 1,
  MLIP_FUSION_PARTIAL = 2,
  MLIP_FUSION_UNFUSED = 3
} mlip_fusion;

/*
 * Select the fusion configuration for later mlip_compute calls.  The
 * configurations other than MLIP_FUSION_CACHED exist for k = 32 with the
 * irreducible basis and l_max <= 3.  Synchronises the stream, releases the
 * buffers of a configuration that is left and, after a neighbour build,
 * allocates the per-work-group workspace of the cached and three-kernel
 * configurations (MLIP_E_OOM if it does not fit); the recompute and unfused
 * configurations hold none.
 * Errors: MLIP_E_ARG (unknown value, or a non-default one with other
 * hyper-parameters), MLIP_E_OOM, MLIP_E_HIP.
 */
mlip_status mlip_set_fusion(mlip_ctx* ctx, int32_t fusion);

/*
 * How the cached single kernel adds -f_ij to F_j (Section 3.1: the forces are
 * the scatter-sum of the partial forces), for measuring the two designs
 * against each other; both give the same forces up to rounding order.
 *   MLIP_SCATTER_ATOMIC  one float64 atomic add to HBM per pair and
 *                        component (default)
 *   MLIP_SCATTER_TILE    contributions summed per distinct neighbour of a
 *                        tile in an LDS table, then one atomic add per
 *                        neighbour and component
 * Applies to MLIP_FUSION_CACHED at k = 32 with the irreducible basis and
 * l_max <= 3 (the other configurations scatter by atomics).  Errors:
 * MLIP_E_ARG (unknown value, or MLIP_SCATTER_TILE with other
 * hyper-parameters).
 */
typedef enum { MLIP_SCATTER_ATOMIC = 0, MLIP_SCATTER_TILE = 1 } mlip_scatter;
mlip_status mlip_set_scatter(mlip_ctx* ctx, int32_t scatter);

/*
 * Encoding of the neighbour list's entries from the next mlip_build_neighbors
 * on: MLIP_LIST_AUTO (default) codes entries in 2 bytes whenever the cell
 * grid's buckets allow it, MLIP_LIST_INDEX always stores 4-byte indices.
 * Both give the same neighbour sets and results.  Errors: MLIP_E_ARG.
 */
typedef enum { MLIP_LIST_AUTO = 0, MLIP_LIST_INDEX = 1 } mlip_list_format;
mlip_status mlip_set_list_format(mlip_ctx* ctx, int32_t format);

/*
 * The descriptors of the current positions, for heads outside the library's
 * fused evaluation (mlip_heads): rows_dev float32 [n][(lmax+1) k], x = vec(G_i)
 * in l-major order (Eq. 5) rounded to float32, in the caller's order of atoms.
 * pos_dev as in mlip_compute.
 * mlip_forces_from_descriptors is the other end: forces_dev float64 [n][3] and,
 * unless NULL, virial_dev float64 [n][9], as mlip_compute writes them, of
 * energies whose gradient in the descriptors is drows_dev, float32
 * [n][(lmax+1) k] (Eqs. 7-10): the encoder and the geometry are differentiated
 * here, the head was by the caller.
 * Both are the outer kernels of the three-kernel configuration and need it
 * (mlip_set_fusion(MLIP_FUSION_PARTIAL)).
 * Errors: MLIP_E_ARG, MLIP_E_STATE (no build, another configuration),
 * MLIP_E_OOM, MLIP_E_HIP.
 */
mlip_status mlip_descriptors(mlip_ctx* ctx, const double* pos_dev, float* rows_dev);
mlip_status mlip_forces_from_descriptors(mlip_ctx* ctx, const double* pos_dev, const float* drows_dev,
                                         double* forces_dev, double* virial_dev);

/* Device memory held by the context, in bytes. */
mlip_status mlip_memory_bytes(const mlip_ctx* ctx, size_t* bytes);

/* Fill *stats (synchronises to read the active-pair counter). */
mlip_status mlip_get_stats(mlip_ctx* ctx, mlip_stats* stats);

/*
 * Text of the last error on this context (never NULL; "" when none).  With
 * ctx NULL: why the last mlip_create on the calling thread failed ("" if it
 * succeeded).
 */
const char* mlip_last_error(const mlip_ctx* ctx);

/* Release the context and its device memory (NULL is ignored). */
void mlip_destroy(mlip_ctx* ctx);

/*
 * Molecular-dynamics driver helpers (velocity Verlet in metal units: A, fs,
 * amu, eV; acceleration = F/m * 9.648533212e-3).  They are not part of the
 * potential; the paper runs its MLIP inside LAMMPS with a 1 fs step
 * (Section 4.1).  They use the species of the last neighbour build.
 */

/* Per-species masses in amu, masses_host float64 [n_species] (> 0). */
mlip_status mlip_md_set_masses(mlip_ctx* ctx, const double* masses_host);

/*
 * First half of a step: vel += dt/2 * a(F); pos += dt * vel.  If
 * max_disp2_host is non-NULL the largest squared displacement is written
 * there (synchronises): against ref_dev (float64 [n][3]) when it is non-NULL,
 * otherwise against the positions of the last neighbour build (minimum image,
 * no extra memory).
 */
mlip_status mlip_md_first_half(mlip_ctx* ctx, double* pos_dev, double* vel_dev,
                               const double* forces_dev, double dt, const double* ref_dev,
                               double* max_disp2_host);

/* Second half of a step: vel += dt/2 * a(F). */
mlip_status mlip_md_second_half(mlip_ctx* ctx, double* vel_dev, const double* forces_dev, double dt);

/* Kinetic energy sum_i m_i |v_i|^2 / 2 in eV into *ke_host (synchronises). */
mlip_status mlip_md_kinetic(mlip_ctx* ctx, const double* vel_dev, double* ke_host);

/*
 * Learning operators: what the tables of the potential are learned with.
 * Training is outside the paper's runtime (its models are fitted to energies
 * and forces beforehand); these calls are the parts of a training step that
 * run per atom or per weight, and the heads they train can be chosen by the
 * environment of an atom instead of by its species alone (Section 3.2).
 *
 * A mlip_learn context holds the stream, the workspace and the error text of
 * the calls made with it.  Work is enqueued on its stream; buffers are the
 * caller's, as above.  The context's device must be current (MLIP_E_ARG).  A
 * call may enlarge the workspace (hipMalloc, and a wait for the stream where an
 * older one is freed) the first time it meets a size; later calls of that size
 * or smaller allocate nothing, and may be recorded in a HIP graph (a call that
 * would have to enlarge it while its stream is recorded is refused,
 * MLIP_E_STATE).  A graph keeps to the workspace it was recorded with, which
 * stays allocated until the context is released, also where a later call needs
 * a larger one (mlip_learn_memory_bytes counts both).  Replay it in order with
 * the context's calls, and not after the context, or a plan whose step it has,
 * is released.  All results are the same from run to run: nothing is summed in
 * an order that depends on the scheduling of work-groups.
 */
typedef struct mlip_learn mlip_learn;
typedef enum { MLIP_F32 = 0, MLIP_BF16 = 1 } mlip_dtype;

/* Create a context on the current HIP device.  Errors: MLIP_E_ARG,
   MLIP_E_OOM, MLIP_E_HIP; mlip_learn_last_error(NULL) then says why. */
mlip_status mlip_learn_create(void* hip_stream, mlip_learn** out);
const char* mlip_learn_last_error(const mlip_learn* ctx);
mlip_status mlip_learn_memory_bytes(const mlip_learn* ctx, size_t* bytes);
/* Release the context after its stream's work (NULL is ignored). */
void mlip_learn_destroy(mlip_learn* ctx);

/*
 * Route n rows (atoms) to top_k of n_experts experts (energy heads).
 *   logits_dev  f32 or bf16 [n][n_experts], rows row_stride values apart
 *   kinds_dev   int32 [n] and allowed_dev uint8 [n_kinds][n_experts], or both
 *               NULL: row i may use expert e only where
 *               allowed[kinds[i]][e] != 0; a row whose kind is outside
 *               [0, n_kinds) uses none.  A logit of -infinity takes its expert
 *               out too.  What stands at places that are out is not looked at
 *               (it may be NaN)
 *   experts_dev int32 [n][top_k], the experts of the largest logits in falling
 *               order (equal logits: the lower index first), -1 where fewer
 *               are left
 *   gates_dev   f32 [n][top_k], 0 at -1: with MLIP_GATES_CHOSEN the softmax
 *               over the chosen experts' logits, with MLIP_GATES_ALL their
 *               probabilities p_ie, the softmax over all that the row may use
 *               (float32; one below 2^-126 of the row's largest is 0)
 *   counts_dev  int32 [n_experts + 1], entries per expert, then the number of
 *               rows that have any expert
 *   loss_dev    f32 [1], the balance loss n_experts sum_e f_e P_e with f_e =
 *               counts_e / sum counts and P_e the mean of p_ie over the rows
 *               that have any expert: 1 where all experts are used alike, up to
 *               n_experts where one is; 0 without such rows
 * A NaN (or +infinity) among the logits a row may use makes all its gates NaN,
 * those at -1 too (a NaN is never chosen).
 * mlip_route_backward writes the logits' gradient (their type, [n][n_experts]
 * contiguous) of sum(dgates gates) + dloss loss: the choice of experts and the
 * shares f_e are constants of it.  experts_dev and counts_dev are what
 * mlip_route wrote for the same logits; dgates_dev [n][top_k] (not looked at
 * where experts is -1) or NULL, dloss_dev [1] or NULL: none.
 * n in [0, 2^31 / top_k), n_experts 1..256, top_k 1..16 and <= n_experts.
 * Errors: MLIP_E_ARG, MLIP_E_STATE, MLIP_E_OOM, MLIP_E_HIP.
 */
typedef enum { MLIP_GATES_CHOSEN = 0, MLIP_GATES_ALL = 1 } mlip_gates;
typedef struct {
  int32_t n_experts;
  int32_t top_k;
  int32_t n_kinds;     /* rows of allowed_dev; 0 without it */
  int32_t gates;       /* mlip_gates */
  int32_t dtype;       /* mlip_dtype of the logits and their gradient */
  int64_t row_stride;  /* values between rows of the logits, >= n_experts */
} mlip_route_params;

mlip_status mlip_route(mlip_learn* ctx, const mlip_route_params* p, int64_t n, const void* logits_dev,
                       const int32_t* kinds_dev, const uint8_t* allowed_dev, int32_t* experts_dev, float* gates_dev,
                       int32_t* counts_dev, float* loss_dev);
mlip_status mlip_route_backward(mlip_learn* ctx, const mlip_route_params* p, int64_t n, const void* logits_dev,
                                const int32_t* kinds_dev, const uint8_t* allowed_dev, const int32_t* experts_dev,
                                const int32_t* counts_dev, const float* dgates_dev, const float* dloss_dev,
                                void* dlogits_dev);

/*
 * Group n_entries routed entries (experts_dev, [n][top_k] flat, or one species
 * per atom) by expert: order_dev int32 [n_entries] receives the entries'
 * indices, those of expert e at offsets_dev[e] .. offsets_dev[e + 1] - 1 in
 * rising order, and after offsets_dev[n_experts] those whose id is outside
 * [0, n_experts).  offsets_dev int32 [n_experts + 1].
 * n_entries in [0, 2^31), n_experts 1..256.  Errors: MLIP_E_ARG, MLIP_E_STATE,
 * MLIP_E_OOM, MLIP_E_HIP.
 */
mlip_status mlip_group(mlip_learn* ctx, int64_t n_entries, int32_t n_experts, const int32_t* experts_dev,
                       int32_t* offsets_dev, int32_t* order_dev);

/*
 * The energy heads (Eq. 6; layout and formula of a head table at
 * mlip_weight_count, hidden width 64) of n rows, each through the top_k heads it
 * is routed to: energy_i = sum_s gate_is v_is with v_is the value of head
 * experts_is at row i, and gradients of sum_i denergy_i energy_i.
 *   x_dev       f32 or bf16 [n][width], rows row_stride values apart
 *   weights_dev f32 [n_experts][values of a head]
 *   offsets_dev, order_dev  the entries [n][top_k] grouped by head, as
 *               mlip_group writes them (for species as experts: top_k 1)
 *   gates_dev   f32 [n][top_k], or NULL: 1.  denergy_dev f32 [n], or NULL: 1
 * Outputs, each NULL where it is not wanted:
 *   energy_dev  f32 [n]; entries without a head (-1) add nothing, and a row
 *               without any has energy and gradients of 0
 *   dx_dev      x's type, [n][width] contiguous
 *   dweights_dev f32 [n_experts][values of a head], 0 for heads without rows
 *   dgates_dev  f32 [n][top_k], denergy_i v_is, 0 at entries without a head
 * Products, activations and sums are float32 whatever x's type; values of bf16
 * are rounded to nearest once, at the end.  An infinity, or a value of 2^128 (1 -
 * 2^-9) or more in size, makes what depends on it NaN.
 * n in [0, 2^31 / top_k), n_experts 1..256, width 1..1024, hidden 1..8, top_k
 * 1..16.  Errors: MLIP_E_ARG, MLIP_E_STATE, MLIP_E_OOM, MLIP_E_HIP.
 */
typedef struct {
  int32_t n_experts;
  int32_t width;       /* inputs of a head, (lmax + 1) k for descriptors */
  int32_t hidden;      /* hidden layers */
  int32_t top_k;
  int32_t dtype;       /* mlip_dtype of x and dx */
  int64_t row_stride;  /* values between rows of x, >= width */
} mlip_heads_params;

/* Values of weights_dev; 0 if the parameters are invalid. */
size_t mlip_heads_weight_count(const mlip_heads_params* p);
mlip_status mlip_heads(mlip_learn* ctx, const mlip_heads_params* p, int64_t n, const void* x_dev,
                       const float* weights_dev, const int32_t* offsets_dev, const int32_t* order_dev,
                       const float* gates_dev, const float* denergy_dev, float* energy_dev, void* dx_dev,
                       float* dweights_dev, float* dgates_dev);

/*
 * Layers of experts wider than the energy heads (hidden width 64): rows are
 * brought into the experts' order, go through matrix products and activations,
 * and come back with weights.  Between the products rows are held in 8 bits, so a
 * result is a step function of its inputs, and the gradients are those of the layers
 * without that rounding: they serve training, and values that are not differentiated
 * again, not an energy whose derivative is to be the force on an atom.
 *
 * mlip_sort: entry i top_k + s (row i, its s-th expert) stands at place p with
 * order[p] = i top_k + s (offsets_dev, order_dev as mlip_group writes them):
 *   sorted_dev  [n top_k][width] contiguous: sorted[p] = x[order[p] / top_k] for
 *               p < offsets[n_experts]; rows from there on (entries without an
 *               expert) are left as they are.  NULL: places alone, x is not read
 *   places_dev  int32 [n][top_k]: p, or -1 for an entry without an expert
 * mlip_combine: out_i = sum_s gates_is y[places_is] in float32, in the order of s,
 * out_dev [n][width] contiguous; entries without an expert add nothing and their
 * gates are not looked at.  gates_dev f32 [n][top_k] or NULL: 1.  Without gates,
 * and given the gradient in sorted_dev, it is mlip_sort's gradient in x.
 * mlip_combine_backward: of sum dout . out, dy_dev [n top_k][width] contiguous,
 * dy[places_is] = gates_is dout_i (other rows are left as they are), and, unless
 * NULL, dgates_dev f32 [n][top_k], dout_i . y[places_is], 0 for an entry without
 * an expert (y_dev is needed for it alone).
 * x, y and dout are f32 or bf16 (dtype), rows *_stride values apart; their
 * results have their type.  No output may overlap an input.
 * n in [0, 2^31 / top_k), n_experts 1..256, top_k 1..16, width 1..65536.
 * Errors: MLIP_E_ARG, MLIP_E_HIP.
 */
typedef struct {
  int32_t n_experts;   /* of offsets_dev, where there is one */
  int32_t top_k;
  int32_t width;
  int32_t dtype;       /* mlip_dtype of the rows */
} mlip_rows_params;

mlip_status mlip_sort(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const void* x_dev, int64_t x_stride,
                      const int32_t* offsets_dev, const int32_t* order_dev, void* sorted_dev, int32_t* places_dev);
mlip_status mlip_combine(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const void* y_dev, int64_t y_stride,
                         const int32_t* places_dev, const float* gates_dev, void* out_dev);
mlip_status mlip_combine_backward(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const void* dout_dev,
                                  int64_t dout_stride, const void* y_dev, int64_t y_stride, const int32_t* places_dev,
                                  const float* gates_dev, void* dy_dev, float* dgates_dev);

/*
 * Rows in 8 bits: for every 128 values of a row (the last block of a row may be
 * shorter) a power of two 2^e and a code each of 4 exponent and 3 mantissa bits
 * beside the sign, s (1 + f/8) 2^(E - 7) 2^e, for E = 0 s f/8 2^-6 2^e; 0x7f and
 * 0xff are NaN.  With a the largest finite size of the block, a = f 2^q, 1 <= f < 2:
 * e = q - 8 if f <= 1.75, else q - 7, kept within -100..120; codes are the values
 * times 2^-e rounded to nearest, ties to even, and to 15/16 2^128 instead of 2^128,
 * which float32 has not.  An infinity or a NaN is held as NaN and leaves its
 * block's others alone.
 *   codes uint8 [rows][mlip_row8_codes(width)], width rounded up to a multiple of
 *         128, zeros behind the row's end; aligned to 16 bytes
 *   exps  uint8 [rows][mlip_row8_exps(width)], e + 127 of each block, rounded up
 *         to a multiple of four, zeros behind the last; aligned to 4 bytes
 * (whole blocks: 64 and 129 values take 132 and 260 bytes, more than in bf16)
 * mlip_pack8 packs n rows, or, with offsets_dev and order_dev (both or neither),
 * their entries in the experts' order as mlip_sort would write them: n top_k rows,
 * those from offsets[n_experts] on left as they are.  mlip_unpack8 writes the
 * values of n packed rows, x_dev [n][width] contiguous in dtype; both types hold
 * them without rounding.
 * mlip_pack8_weights packs matrices w_dev f32 or bf16 [n_experts][outputs][inputs]
 * with one power of two for 128 x 128 values (the same rule):
 *   codes  [n_experts][outputs][mlip_row8_codes(inputs)]
 *   exps   [n_experts][ceil(outputs / 128)][mlip_row8_exps(inputs)]
 * and their transposes, with the same values:
 *   t_codes [n_experts][inputs][mlip_row8_codes(outputs)]
 *   t_exps  [n_experts][ceil(inputs / 128)][mlip_row8_exps(outputs)]
 * either pair may be NULL.
 * Errors: MLIP_E_ARG, MLIP_E_HIP.
 */
int64_t mlip_row8_codes(int32_t width);
int64_t mlip_row8_exps(int32_t width);
mlip_status mlip_pack8(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const void* x_dev, int64_t x_stride,
                       const int32_t* offsets_dev, const int32_t* order_dev, uint8_t* codes_dev, uint8_t* exps_dev);
mlip_status mlip_unpack8(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const uint8_t* codes_dev,
                         const uint8_t* exps_dev, void* x_dev);

/*
 * Products of packed rows and matrices.  m rows stand in the experts' order:
 * expert e has rows offsets[e] .. offsets[e + 1] - 1 (offsets_dev int32
 * [n_experts + 1], rising; NULL with n_experts 1: all rows), and rows from
 * offsets[n_experts] on are neither read nor written.
 * mlip_product8: y_p = W_e x_p + c_e, y_dev [m][outputs] contiguous in dtype,
 * bias_dev f32 [n_experts][outputs] or NULL.  With the transposes and dy for x
 * (inputs and outputs exchanged) it is the gradient in x.
 * Sums from block to block are float32.  In float32 y has the accuracy of float32
 * products of the packed values; for bf16, whose results are rounded to 8
 * bits, the matrix instruction adds eight neighbouring products at a time with
 * their bits below 2^-13 of the largest one cut off (rms 1.5e-5 of a sum of normally
 * distributed values, at most 7 x 2^-13 of the largest product of each eight).
 * mlip_product8_weights: dweights_dev f32 [n_experts][outputs][inputs],
 * sum_p dy_p x_p^T over the expert's rows, and, unless NULL, dbias_dev f32
 * [n_experts][outputs], sum_p dy_p; 0 for experts without rows.  Float32 sums of
 * the packed values' products, in dbias of the packed values (a caller who has dy
 * in more bits may sum that instead); dtype is not looked at beyond its range.  A NaN in
 * a row gives NaN wherever it is a factor.  No output may overlap an input.
 * m in [0, 2^31), n_experts 1..256, inputs and outputs 1..65536, and (m / 128 +
 * n_experts) outputs / 128, and n_experts inputs outputs / 2^14, below 2^22.
 * Errors: MLIP_E_ARG, and of mlip_product8_weights MLIP_E_STATE, MLIP_E_OOM; MLIP_E_HIP.
 */
typedef struct {
  int32_t n_experts;
  int32_t inputs;
  int32_t outputs;
  int32_t dtype;       /* mlip_dtype of w and of y */
} mlip_product8_params;

mlip_status mlip_pack8_weights(mlip_learn* ctx, const mlip_product8_params* p, const void* w_dev, uint8_t* codes_dev,
                               uint8_t* exps_dev, uint8_t* t_codes_dev, uint8_t* t_exps_dev);
mlip_status mlip_product8(mlip_learn* ctx, const mlip_product8_params* p, int64_t m, const uint8_t* x_codes_dev,
                          const uint8_t* x_exps_dev, const uint8_t* w_codes_dev, const uint8_t* w_exps_dev,
                          const int32_t* offsets_dev, const float* bias_dev, void* y_dev);
mlip_status mlip_product8_weights(mlip_learn* ctx, const mlip_product8_params* p, int64_t m, const uint8_t* dy_codes_dev,
                                  const uint8_t* dy_exps_dev, const uint8_t* x_codes_dev, const uint8_t* x_exps_dev,
                                  const int32_t* offsets_dev, float* dweights_dev, float* dbias_dev);

/*
 * An activation that keeps its argument in 8 bits for the backward pass:
 *   h = r + silu(z), silu(z) = z / (1 + exp(-z));  r = residual_dev or NULL: 0
 *   dz = dh silu'(z^), silu'(z) = s (1 + z (1 - s)), s = 1 / (1 + exp(-z)), with z^
 *   the kept z's values (the residual's gradient is dh)
 * in float32.  z, r, dh: n rows of `width` values in dtype, *_stride values apart;
 * h_dev, dz_dev [n][width] contiguous in dtype.  h_codes_dev, h_exps_dev and
 * dz_codes_dev, dz_exps_dev are what mlip_pack8 gives for h and dz as they are
 * written, for the next product; kept_codes_dev, kept_exps_dev what it gives for z.
 * Outputs that are not wanted are NULL (kept: nothing will be differentiated).
 * h may be z or r, and dz dh, where their rows are contiguous; apart from that no
 * output may overlap an input.  silu(-infinity) is NaN.  p->n_experts and top_k are not used beyond their range.
 * Errors: MLIP_E_ARG, MLIP_E_HIP.
 */
mlip_status mlip_activate8(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const void* z_dev, int64_t z_stride,
                           const void* residual_dev, int64_t residual_stride, void* h_dev, uint8_t* h_codes_dev,
                           uint8_t* h_exps_dev, uint8_t* kept_codes_dev, uint8_t* kept_exps_dev);
mlip_status mlip_activate8_backward(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const uint8_t* kept_codes_dev,
                                    const uint8_t* kept_exps_dev, const void* dh_dev, int64_t dh_stride, void* dz_dev,
                                    uint8_t* dz_codes_dev, uint8_t* dz_exps_dev);

/*
 * AdamW over many tensors at once (the tables of a potential are hundreds to
 * thousands: eight tensors for every pair of species and ten for every
 * species), in one launch:
 *   m' = beta1 m + (1 - beta1) g,  v' = beta2 v + (1 - beta2) g^2,  g the gradient
 *   times grad_scale,
 *   p' = p (1 - lr weight_decay [tensors with decay])
 *        - lr / (1 - beta1^step) m' / (sqrt(v') / sqrt(1 - beta2^step) + eps)
 * in float32; bf16 parameters are rounded to nearest at the end.
 *
 * A plan holds the tensors' places and the stream, and is made once.  The
 * moments are the caller's: the tensors' elements back to back in the order of
 * the plan, float32, or with state_bits 8 one code each and one exponent for
 * every 256 elements of a tensor (the last block of a tensor is shorter):
 *   exponent byte e + 127, the block's |values| < 2^e
 *   m  sign, 4 exponent bits E, 3 mantissa bits: (1 + f/8) 2^(E - 15) 2^e, for
 *      E = 0 f/8 2^-14 2^e; 0x7f is NaN
 *   v  4 exponent and 4 mantissa bits: (1 + f/16) 2^(E - 15) 2^e, for E = 0 f/16
 *      2^-14 2^e; 0xff is NaN
 * All zero bytes are zero moments.  The update uses m' and v' before they are
 * rounded.  Rounding is up or down at random, up with the probability of the
 * part that is cut off (to nearest, v would never change: a step moves it by
 * less than half of what its codes are apart); the random bits are mixed from
 * `seed` (another one each step) and the element's place, so a step can be
 * repeated bit for bit.  An element whose moment is not finite keeps NaN and
 * leaves its block's others alone; a size of 2^127 and more is held as the
 * largest code.
 * A v that is not 0 is not rounded to 0: less than 2^-18 2^e is held as that.
 * So where an element's gradients stay below 1/512 to 1/362 of the largest of
 * its block (the root of v's share of 2^e), its v is too large and its steps are
 * shorter than with 32 bits, by the root of v / (2^-18 2^e).  Tensors whose
 * gradients spread wider than that within 256 neighbours want 32 bits.
 *
 * mlip_adamw_create  tensors: host array, copied; into_dev, for all tensors or
 *                    for none: where new parameters go (NULL: param_dev), equal
 *                    to param_dev or apart from it.  Errors:
 *                    MLIP_E_ARG, MLIP_E_OOM, MLIP_E_HIP, text from
 *                    mlip_adamw_last_error(NULL).  Synchronises
 * mlip_adamw_state_count  elements of each moment, and exponents of each (0
 *                    with 32 bits)
 * mlip_adamw_step    reads the state `from` and writes `into` (NULL: `from`
 *                    again); with into_dev and a second state a step can be
 *                    dropped by not using what it wrote.  reverse != 0 reads
 *                    the parameters at into_dev and writes param_dev
 * mlip_adamw_moments the values 8-bit moments stand for, float32 [elements]
 */
typedef struct mlip_adamw mlip_adamw;
typedef struct {
  void* param_dev;
  void* into_dev;
  const void* grad_dev;
  int64_t n;
  int32_t param_dtype;  /* mlip_dtype */
  int32_t grad_dtype;   /* mlip_dtype */
  int32_t decay;        /* whether weight_decay applies */
} mlip_adamw_tensor;
typedef struct {
  int64_t step;         /* this step's number, from 1 */
  double lr, beta1, beta2, eps, weight_decay;
  double grad_scale;    /* factor on the gradients: 1, a clipping factor, or 1 / loss scale */
  uint32_t seed;        /* of the rounding of 8-bit moments */
} mlip_adamw_params;
typedef struct {
  void* m_dev;
  void* v_dev;
  uint8_t* m_exp_dev;   /* 8 bits only */
  uint8_t* v_exp_dev;
} mlip_adamw_state;

mlip_status mlip_adamw_create(const mlip_adamw_tensor* tensors, int64_t n_tensors, int32_t state_bits,
                              void* hip_stream, mlip_adamw** out);
const char* mlip_adamw_last_error(const mlip_adamw* plan);
mlip_status mlip_adamw_state_count(const mlip_adamw* plan, int64_t* elements, int64_t* blocks);
void mlip_adamw_destroy(mlip_adamw* plan);
mlip_status mlip_adamw_step(mlip_adamw* plan, const mlip_adamw_params* p, const mlip_adamw_state* from,
                            const mlip_adamw_state* into, int32_t reverse);
mlip_status mlip_adamw_moments(mlip_adamw* plan, const mlip_adamw_state* state, float* m_out_dev, float* v_out_dev);

#ifdef __cplusplus
}
#endif

#endif /* MLIP_H */
