/*
 * pdn.h -- C ABI of the chunkwise preconditioned delta rule on MI355X (gfx950).
 *
 * Computes, for every batch b and head h independently, the recurrence of
 * "Preconditioned DeltaNet" (arXiv 2604.21100), Sec. 3.5, Eq. precond_end2end,
 * in its three instantiations (PDN: no decay; PGDN: scalar decay; PKDA:
 * per-key-channel decay -- the decayed forms of Sec. 3.5 and App. D):
 *
 *   A_t  = exp(gP_t) A_{t-1} + betaP_t (k_t * k_t)            diagonal key Gram
 *   r_t  = log(A_t) - exp(logAScale_h)
 *   B_t  = exp(-log(x) * r_t / (1 + |r_t|))                    in [1/x, x]
 *   kt_t = B_t * k_t                                           write key
 *   S_t  = alpha_t S_{t-1} + beta_t (v_t - alpha_t S_{t-1} k_t) kt_t^T
 *   o_t  = scale * S_t q_t
 *
 * with S_t in R^{dv x dk} (the paper's orientation), alpha_t = exp(g_t) a
 * scalar (PGDN) or a dk-vector acting as S Diag(alpha_t) (PKDA).  The library
 * evaluates it with the chunkwise-parallel form of Eq. chunkwise_atk_form /
 * App. D (UT transform T = (I + tril(Diag(beta) K Kt^T, -1))^{-1} Diag(beta),
 * W = T K, U = T V, inter-chunk state scan, chunk output).
 *
 * Conventions
 *   - Every tensor argument is a DEVICE pointer to dense row-major memory owned
 *     by the caller.  The library never allocates or frees device memory; all
 *     scratch lives in a caller-provided workspace (pdn_workspace_size), except
 *     for pdn_chunk_fwd_noalloc's fixed per-device array (see there).
 *   - Layouts: q, k, ktilde, dq, dk: [B, T, H, dk];  v, o, dO, dv: [B, T, H, dv];
 *     beta, betaP, gP and a scalar gate g: [B, T, H];  a per-channel gate g:
 *     [B, T, H, dk];  logAScale: [H];  A0, A_T: [B, H, dk];
 *     S0, S_T, dS_T, dS0: [B, H, dk, dv] holding S^T (the transpose of the
 *     paper's S), i.e. element (b, h, i, j) is S[j][i].
 *   - q, k, v, o, ktilde and their gradients use the problem's io dtype
 *     (IEEE fp32 or bfloat16); every other tensor is fp32.
 *   - Byte offsets inside a chunk of q, k, v, o and their gradients are 32-bit:
 *     (min(T, chunk) - 1) * H * max(dk, dv) * element size must stay below
 *     2^32 - 1024 (in bf16 at d = 128 and T >= chunk = 64: H up to 266304).
 *     Nothing checks it.
 *   - Calls are asynchronous on the given HIP stream (a hipStream_t passed as
 *     void*; NULL = the null stream).  Inputs, outputs and workspace must stay
 *     valid until the stream work completes.
 *   - Errors: every argument is validated on the host BEFORE any HIP call;
 *     on a validation failure the function returns the first failing code
 *     and writes nothing.  A failed kernel launch returns PDN_ERR_HIP and
 *     leaves the outputs undefined.  Values are not inspected: NaN / Inf in
 *     the inputs propagate.  No exception, abort or printf crosses the ABI.
 *   - Apart from pdn_chunk_fwd_noalloc (which shares one fixed scratch array
 *     per device), the library keeps no mutable global state: calls are
 *     re-entrant and may run concurrently on different streams with
 *     distinct workspaces.
 */
#ifndef PDN_H
#define PDN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PDN_ABI_VERSION 7

typedef enum {
  PDN_OK = 0,
  PDN_ERR_NULL = 1,        /* a required pointer is NULL                       */
  PDN_ERR_SHAPE = 2,       /* B, T, H negative or sizes overflow               */
  PDN_ERR_DTYPE = 3,       /* unknown io dtype                                 */
  PDN_ERR_UNSUPPORTED = 4, /* dk, dv or chunk outside the built kernels (dk, dv
                              in {64, 128}, chunk in {32, 64}), or a mode
                              the entry point does not cover                 */
  PDN_ERR_ALIGN = 5,       /* a tensor is not 16-byte aligned                  */
  PDN_ERR_ALIAS = 6,       /* an output overlaps an input or another output    */
  PDN_ERR_WORKSPACE = 7,   /* workspace NULL, too small or misaligned          */
  PDN_ERR_VALUE = 8,       /* bad scalar (x < 1, non-finite x/scale, ridge <= 0
                              for DIAG_SM / ATQ) or enum (knorm other than
                              NONE without SQUASH), or a gate pointer
                              inconsistent with the gate kind               */
  PDN_ERR_HIP = 9,         /* a HIP launch failed                              */
  PDN_ERR_SCRATCH = 10     /* pdn_chunk_fwd_noalloc: the problem's workspace
                              exceeds PDN_NOALLOC_SCRATCH_BYTES              */
} pdn_status;

typedef enum { PDN_F32 = 0, PDN_BF16 = 1 } pdn_dtype;

typedef enum {
  PDN_GATE_NONE = 0,    /* PDN:  alpha_t = 1                        */
  PDN_GATE_SCALAR = 1,  /* PGDN: alpha_t = exp(g_t), g [B,T,H]      */
  PDN_GATE_CHANNEL = 2  /* PKDA: alpha_t = exp(g_t), g [B,T,H,dk]   */
} pdn_gate;

/* Admissible per-channel decay (PDN_GATE_CHANNEL).  Inside a chunk the
 * decay between tokens t <= r of one channel, exp(G_r - G_t) with G the
 * in-chunk prefix sum of that channel's g, is applied as the product of two
 * fp32 factors split at a reference row of each 16-token block (forward
 * interaction matrices and the backward's intra-chunk products).  One of
 * the two is the exponential of up to 15 consecutive log-decays with the
 * sign flipped, so every run of 15 consecutive g of a channel must sum to
 * more than -87 (a mean log-decay above -5.8 per token, alpha above 0.003);
 * below that the factor overflows and outputs and gradients hold Inf / NaN.
 * Nothing checks the range.  The scalar gate has no such limit.           */

typedef enum {
  PDN_PRECOND_SQUASH = 0,   /* write key of Eq. precond_end2end (the method) */
  PDN_PRECOND_IDENTITY = 1, /* kt = k: plain DeltaNet / GDN / KDA            */
  PDN_PRECOND_EXTERNAL = 2, /* kt supplied by the caller in `ktilde`         */
  /* Unstable ATK (App. D, "ATK (unstable) preconditioner recurrence"; the
   * Sherman-Morrison form of Sec. 3.4): with the same A recurrence and
   * P_t = Diag(A_{t-1} + ridge)^{-1} (the state BEFORE token t),
   *   kt_t = P_t k_t / (1 + k_t^T P_t k_t)
   * and the delta rule above.  Forward only.                               */
  PDN_PRECOND_DIAG_SM = 3,
  /* Preconditioned linear attention, apply-to-query (Sec. 3.3 chunkwise PLA
   * form; App. D, "ATQ preconditioner recurrence"; P-Mamba-2 with a scalar
   * gate, PGLA with a per-channel gate): no delta rule,
   *   S_t = alpha_t S_{t-1} + beta_t v_t k_t^T
   *   o_t = scale * S_t (q_t / (A_t + ridge))          (A_t: current state)
   * ktilde is unused (write key = read key).  Forward only.                */
  PDN_PRECOND_ATQ = 4
} pdn_precond;

/* Normalisation factor on the SQUASH write key (the ablation of App. E,
 * "Stable parameterization", table of normalisation factors): with
 * m_t = k_t^T B_t k_t,
 *   kt_t = B_t k_t * { 1 | 1 / m_t | 1 / (1 + m_t) | beta_t / (alpha_t + beta_t m_t) }
 * alpha_t = exp(g_t) for a scalar gate, 1 without a gate.  NONE is the
 * method; the others are forward only, SQUASH only, and BETA is not
 * defined for a per-channel gate (PDN_ERR_UNSUPPORTED).                    */
typedef enum {
  PDN_KNORM_NONE = 0,
  PDN_KNORM_M = 1,      /* 1 / m_t                                          */
  PDN_KNORM_1PM = 2,    /* 1 / (1 + m_t)                                    */
  PDN_KNORM_BETA = 3    /* beta_t / (alpha_t + beta_t m_t)                  */
} pdn_knorm;

typedef struct {
  int64_t B, T, H;     /* batch, sequence length, heads; 0 is allowed      */
  int32_t dk, dv;      /* head dims: each 64 or 128                         */
  int32_t chunk;       /* chunk length C: 32 or 64 (the paper's form for
                          any C; results differ only by rounding)        */
  pdn_dtype io;        /* dtype of q, k, v, o, ktilde and their gradients   */
  pdn_gate gate;
  pdn_precond precond;
  float x;             /* squash range [1/x, x]; x >= 1 (paper: 1.5)        */
  float scale;         /* output scale (paper: 1.0)                         */
  float ridge;         /* DIAG_SM and ATQ: the ridge lambda > 0 added to A
                          before the elementwise inverse; ignored otherwise */
  pdn_knorm knorm;     /* SQUASH write-key normalisation; NONE otherwise    */
} pdn_problem;

typedef struct {
  const void* q;             /* [B,T,H,dk] io                                */
  const void* k;             /* [B,T,H,dk] io  (read key)                    */
  const void* v;             /* [B,T,H,dv] io                                */
  const float* beta;         /* [B,T,H]                                      */
  const float* g;            /* NULL for GATE_NONE, else [B,T,H] / [B,T,H,dk] */
  const float* beta_p;       /* [B,T,H]; SQUASH, DIAG_SM, ATQ               */
  const float* g_p;          /* [B,T,H] or NULL (alpha^P = 1); as beta_p     */
  const float* log_a_scale;  /* [H]; mu_h = exp(.); SQUASH only              */
  const float* A0;           /* [B,H,dk] or NULL (= 0); as beta_p            */
  const float* S0;           /* [B,H,dk,dv] (S^T) or NULL (= 0)              */
  const void* ktilde;        /* [B,T,H,dk] io; EXTERNAL only                 */
} pdn_inputs;

typedef struct {
  void* o;      /* [B,T,H,dv] io                                             */
  float* S_T;   /* [B,H,dk,dv] final state S_T^T, or NULL                    */
  float* A_T;   /* [B,H,dk] final preconditioner state, or NULL (SQUASH,
                   DIAG_SM, ATQ)                                             */
} pdn_fwd_out;

typedef struct {
  void* dq;              /* [B,T,H,dk] io                                    */
  void* dk;              /* [B,T,H,dk] io                                    */
  void* dv;              /* [B,T,H,dv] io                                    */
  float* dbeta;          /* [B,T,H]                                          */
  float* dg;             /* [B,T,H] / [B,T,H,dk]; NULL iff GATE_NONE         */
  float* dS0;            /* [B,H,dk,dv] or NULL                              */
  float* dbeta_p;        /* [B,T,H] or NULL (SQUASH)                         */
  float* dg_p;           /* [B,T,H] or NULL (SQUASH)                         */
  float* dlog_a_scale;   /* [H] or NULL (SQUASH)                             */
  float* dA0;            /* [B,H,dk] or NULL (SQUASH)                        */
  void* dktilde;         /* [B,T,H,dk] io, EXTERNAL only, or NULL            */
} pdn_bwd_out;

/* Bytes of workspace pdn_chunk_fwd (with_bwd = 0) or pdn_chunk_bwd
 * (with_bwd = 1) needs for this problem.  Host-only, no HIP call.  (A forward
 * of up to eight tokens may run as the token recurrence, which uses none of
 * it; the size is the same, and so is every check of it.)
 * Returns PDN_ERR_NULL / SHAPE / DTYPE / UNSUPPORTED / VALUE for a bad
 * problem; *bytes is written only on PDN_OK. */
pdn_status pdn_workspace_size(const pdn_problem* problem, int with_bwd,
                              size_t* bytes);

/* Number of sequence segments the forward state scan of this problem runs
 * in (1: one pass over the chunks).  A scan workgroup holds one head's
 * 32-column state slab on one compute unit, so with few heads (B * H *
 * dv / 32 far below the 256 compute units of MI355X) most of the chip
 * would idle.  The chunks are then cut into S >= 3 segments: segment 0
 * runs from S0 while every middle segment runs from zero and, with its
 * values zeroed, from the identity (giving its d_k x d_k transition Phi,
 * S_end^T = Phi S_start^T + local end, the chunkwise recurrence being
 * affine in the state); the exact start of each segment is composed from
 * those, and segments 1 .. S - 1 run again from it.  The result is the same
 * recurrence up to fp32 rounding.  S depends only on the problem's sizes,
 * as does the workspace (which holds the segment states).  Host-only, no
 * HIP call; errors as pdn_workspace_size. */
pdn_status pdn_scan_segments(const pdn_problem* problem, int* segments);

/* Forward pass (Eq. chunkwise_atk_form with the preconditioner of Eq.
 * precond_end2end; decayed forms of App. D).  Writes o and, when non-NULL,
 * S_T and A_T.  `ws` must be 256-byte aligned and at least
 * pdn_workspace_size(problem, 0) bytes.  Asynchronous on `hip_stream`. */
pdn_status pdn_chunk_fwd(const pdn_problem* problem, const pdn_inputs* in,
                         pdn_fwd_out* out, void* ws, size_t ws_bytes,
                         void* hip_stream);

/* pdn_chunk_fwd without a workspace argument, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  It computes exactly what pdn_chunk_fwd
 * computes, with the same kernels, using as its workspace a fixed scratch
 * array of PDN_NOALLOC_SCRATCH_BYTES (64 MiB) that the library holds in
 * every device it runs on, from the library's loading on that device until
 * the process ends.  It calls no hipMalloc / hipFree or other allocating
 * routine; its first call on a device looks up that device's array once.
 *
 * Limit: pdn_workspace_size(problem, 0, &n) must give n <=
 * PDN_NOALLOC_SCRATCH_BYTES, else PDN_ERR_SCRATCH (returned, like every
 * other validation failure, before any HIP call).  For example, bf16 with
 * d_k = d_v = 128 and a scalar gate needs about 0.53 KB per token-head:
 * B*T*H up to about 120k (B=1, T=8192, H=14).
 *
 * Sharing: every call on one device uses that device's single array, which
 * keeps the last call's contents (the forward overwrites every byte it reads
 * before reading it, so nothing needs clearing).  Calls that overlap in time
 * on one device -- on different streams, or from different host threads
 * without ordering -- race on the array and give undefined results; order
 * them on one stream.  Arguments, outputs and errors otherwise as
 * pdn_chunk_fwd. */
#define PDN_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)
pdn_status pdn_chunk_fwd_noalloc(const pdn_problem* problem, const pdn_inputs* in,
                                 pdn_fwd_out* out, void* hip_stream);

/* PDN_NOALLOC_SCRATCH_BYTES of the built library. */
size_t pdn_noalloc_scratch_bytes(void);

/* pdn_chunk_fwd that also records caller-created HIP events (hipEvent_t
 * handles passed as void*) on `hip_stream` at the stage boundaries, for
 * timing individual kernels:
 *   stage_events[0]  before the preconditioner scan (k1_*; empty unless
 *                    SQUASH, DIAG_SM or ATQ)
 *   stage_events[1]  after it / before the per-chunk prep kernel (k2)
 *   stage_events[2]  after k2 / before the inter-chunk scan + output (k3)
 *   stage_events[3]  after k3
 * (k3: the state scan of either io type.)  A forward of up to eight tokens may
 * run as the token recurrence, one launch between [2] and [3]: the stages
 * before it are then empty, or in pdn_chunk_fwd_train as above with the
 * recurrence in k3's place.
 * n_events must be 4 (else PDN_ERR_VALUE); a NULL entry is not recorded
 * (each record costs a few microseconds of GPU time between kernels, so a
 * caller timing one stage passes only its two boundaries).  The events stay
 * owned by the caller; results are identical to pdn_chunk_fwd. */
#define PDN_FWD_STAGE_EVENTS 4
pdn_status pdn_chunk_fwd_events(const pdn_problem* problem, const pdn_inputs* in,
                                pdn_fwd_out* out, void* ws, size_t ws_bytes,
                                void* hip_stream, void* const* stage_events,
                                int n_events);

/* Backward pass: gradients of <dO, o> + <dS_T, S_T> with respect to every
 * input of pdn_chunk_fwd (App. C, backward pseudocode).  dO is [B,T,H,dv]
 * io; dS_T is [B,H,dk,dv] fp32 or NULL (= 0).  The forward intermediates are
 * recomputed; `ws` must hold pdn_workspace_size(problem, 1) bytes.  The
 * output pointers dbeta_p, dg_p, dlog_a_scale, dA0 and dS0 may be NULL to
 * skip them.  SQUASH, IDENTITY and EXTERNAL only (DIAG_SM, ATQ:
 * PDN_ERR_UNSUPPORTED), and knorm NONE only. */
pdn_status pdn_chunk_bwd(const pdn_problem* problem, const pdn_inputs* in,
                         const void* dO, const float* dS_T, pdn_bwd_out* out,
                         void* ws, size_t ws_bytes, void* hip_stream);

/* pdn_chunk_bwd that also records caller-created HIP events on `hip_stream`
 * at its stage boundaries (n_events must be PDN_BWD_STAGE_EVENTS):
 *   [0] start  [1] after the preconditioner recompute (k1_*)
 *   [2] after the per-chunk prep recompute (k2, backward mode)
 *   [3] after the state-saving forward scan (k3, or the token recurrence)
 *   [4] after the reverse state-adjoint scan (r1)
 *   [5] after the per-chunk adjoints and gradients (p12)
 *   [6] after the preconditioner's reverse scan (pc_*) or the key combine
 * NULL entries are not recorded.  Results are identical to pdn_chunk_bwd. */
#define PDN_BWD_STAGE_EVENTS 7
pdn_status pdn_chunk_bwd_events(const pdn_problem* problem, const pdn_inputs* in,
                                const void* dO, const float* dS_T, pdn_bwd_out* out,
                                void* ws, size_t ws_bytes, void* hip_stream,
                                void* const* stage_events, int n_events);

/* Training pair.  pdn_chunk_fwd_train computes exactly what pdn_chunk_fwd
 * computes and also leaves in `ws` the forward intermediates the backward
 * reads (per-chunk solve factors, chunk-start states, the X and E rows, the
 * write-key rows, ...), so that pdn_chunk_bwd_train can skip the
 * recompute of the forward that pdn_chunk_bwd performs.  This trades memory
 * for time: `ws` must hold at least pdn_workspace_size(problem, 1, &bytes) bytes
 * (the backward's workspace) for both calls.
 *
 * Contract: pdn_chunk_bwd_train must receive the same problem, the same
 * input pointers with unchanged contents and the same `ws` as the preceding
 * pdn_chunk_fwd_train, with no other call writing `ws` in between (the
 * library cannot detect a violation; results are then undefined, but every
 * access stays inside the declared buffers).  pdn_chunk_bwd_train leaves the
 * saved intermediates intact, so it may be called again for another dO.
 * The backward's restrictions apply to both calls (fp32 io only with
 * d_k = d_v = 64; no DIAG_SM or ATQ; knorm NONE: PDN_ERR_UNSUPPORTED).
 *
 * stage_events: NULL with n_events = 0, or PDN_FWD_STAGE_EVENTS /
 * PDN_BWD_STAGE_EVENTS caller-created events recorded as in the _events
 * variants (the backward's recompute stages are then empty). */
pdn_status pdn_chunk_fwd_train(const pdn_problem* problem, const pdn_inputs* in,
                               pdn_fwd_out* out, void* ws, size_t ws_bytes,
                               void* hip_stream, void* const* stage_events,
                               int n_events);
pdn_status pdn_chunk_bwd_train(const pdn_problem* problem, const pdn_inputs* in,
                               const void* dO, const float* dS_T, pdn_bwd_out* out,
                               void* ws, size_t ws_bytes, void* hip_stream,
                               void* const* stage_events, int n_events);

/* ---------------------------------------------------------------- serving
 * A server keeps the states of its sequences in a pool and runs ragged batches
 * of them.  pdn_slot_fwd advances states over one or many tokens (decoding,
 * prompts); pdn_slot_draft scores drafted tokens without moving the state and
 * applies the ones a verification accepted in the next call's pass over the
 * state; pdn_draft_verify is that verification.  All of it stays on the
 * device: `accepted` of one is `accepted` of the other.
 *
 * Tokens of a batch are packed: q, k [tokens, Hk, dk], v, o [tokens, H, dv],
 * beta, beta_p, g_p and a scalar g [tokens, H], a per-channel g
 * [tokens, H, dk], ktilde [tokens, Hk, dk].  Value head h reads the query and
 * key of head h / (H / Hk).  pdn_problem's B is the number of sequences, T the
 * most tokens one of them has (a longer one is cut there), chunk is unused.
 * The recurrence, its modes and the meaning of the other members are those of
 * pdn_chunk_fwd; states and products are fp32 for both io types.
 * Log-decays, a channel's too, and g_p may be as low as the type goes, and -inf
 * (the state, or a channel of it, is forgotten: e.g. a document's first token).
 * A NaN or Inf in a token shows in that sequence and slot only, from that token
 * on (one of a query in that token's o, one of a value in its column; a NaN of
 * beta_p or g_p with SQUASH in A only, which then gives the write keys' gain x).
 * B H must be below 2^22.
 *
 * `starts`, `slot`, `slot_out`, `fresh`, `accepted` are device arrays, read by
 * the kernels and not checked on the host; whatever they hold, accesses stay
 * inside the declared tensors: row numbers are clamped to [0, tokens], and a
 * sequence whose slot is outside [0, slots) is left out (its rows of o, and
 * every slot, stay as they were: padding of a batch).  Rows of o that belong
 * to no sequence stay as they were.
 * A slot written by one sequence of a call must not be read or written by
 * another of the same call; several may read one slot (forks of a state).
 * Nothing checks it; the states concerned, and outputs of the readers, are
 * then undefined. */
typedef struct {
  int64_t tokens;           /* rows of the packed token tensors                */
  int64_t slots;            /* states in the pool                              */
  int64_t Hk;               /* query / key heads, a divisor of H; 0: H         */
  int64_t q_stride, k_stride, v_stride; /* elements from a token's row to the
                               next (q, k, v may be slices of one projection's
                               rows; whole multiples of 16 bytes, at most 2^25);
                               0: dense                                        */
  const int32_t* starts;    /* [B + 1] first row of each sequence, and the end of
                               the last; NULL: B sequences of T rows           */
  const int32_t* slot;      /* [B] slot a sequence's state is read from; NULL: its
                               own number                                      */
  const int32_t* slot_out;  /* [B] slot it is written to; NULL: slot           */
  const int32_t* fresh;     /* [B] non-zero: start from a zero state (nothing is
                               read from the slot); NULL: none does            */
  float* S;                 /* [slots, H, dk, dv] S^T                          */
  float* A;                 /* [slots, H, dk]; SQUASH, DIAG_SM, ATQ, else NULL */
  /* pdn_slot_draft only (NULL and 0 in pdn_slot_fwd): */
  float* tape;              /* [slots, tape_tokens, H, R] records of pending tokens,
                               R = dk + dv + (per-channel gate: dk, else 4) + (A: dk):
                               write key, correction e_t, log-decay summed from the first
                               pending token (without the per-channel gate four
                               times the same; the decay between two records
                               is as exact as fp32 has their sums), A_t        */
  int64_t tape_tokens;      /* >= T                                            */
  int32_t* pending;         /* [slots, H] records a slot has (of every head the
                               same); zero at first                            */
  const int32_t* accepted;  /* [B] pending tokens of the sequence that hold, first
                               ones first; NULL: none                          */
} pdn_slots;

/* Advances each sequence's state over its tokens: reads it from `slot`, writes
 * the state after the last token (S, A) to `slot_out`, and o.  in->S0 and in->A0
 * must be NULL (PDN_ERR_VALUE).  One launch, no workspace.  Tokens pending
 * on a tape are not looked at: apply or drop them first (pdn_slot_draft).
 * A head's tokens run on one compute unit, one chunk after the other: one long
 * prompt of few heads is faster through pdn_chunk_fwd (16 heads x 2048 tokens in
 * bf16: 71 us against 319), whose bf16 states are less exact. */
pdn_status pdn_slot_fwd(const pdn_problem* problem, const pdn_inputs* in,
                        const pdn_slots* slots, void* o, void* hip_stream);

/* Scores drafted tokens.  Of the tokens pending in `slot` the first
 * min(accepted, pending) are applied to the state, the others dropped; the
 * state then goes to `slot_out` (S, A), the new tokens' outputs to o, and the new
 * tokens are left pending in slot_out's tape.  A sequence without rows only
 * has its accepted tokens applied.  fresh: nothing is applied, the state is zero. */
pdn_status pdn_slot_draft(const pdn_problem* problem, const pdn_inputs* in,
                          const pdn_slots* slots, void* o, void* hip_stream);

/* Verifies drafted tokens by the target's probabilities.  A sequence's rows are
 * the tokens it was fed (ids): one that is certain, then the drafts.  p[row] is the
 * target's distribution after that token, q[row] the distribution that token was
 * drafted from (unused for a sequence's first; q NULL: each draft had
 * probability one), both [rows, V] in `dtype`.  Draft t + 1 holds iff those before
 * it do and u[t] q[t+1][x] < p[t][x], x its id (an id outside [0, V) does not
 * hold).  accepted[n]: the tokens that hold, the first and the drafts.
 * token[n]: drawn with r[n] by inversion (the first j whose running sum is
 * over r times the whole) from max(p - q, 0) of the first refused draft (from p
 * where that is zero everywhere), or from p after the last draft; -1 where no
 * token has a positive weight.  A sequence without rows: 0 and -1.
 * u: [rows] (a sequence's last is unused), r: [N], in [0, 1).  p and q need
 * not be normalised; NaN counts as zero weight (an infinite sum: the last token
 * with a weight is taken).  `starts` as in pdn_slots
 * (NULL: rows / N rows each).  Sums are taken in 64 bits.
 * `ws` must be 256-byte aligned, of pdn_draft_verify_workspace_size bytes. */
pdn_status pdn_draft_verify_workspace_size(int64_t N, int64_t V, size_t* bytes);
pdn_status pdn_draft_verify(int64_t N, int64_t rows, int64_t V, pdn_dtype dtype,
                            const void* p, const void* q, const int32_t* ids,
                            const float* u, const float* r, const int32_t* starts,
                            int32_t* accepted, int32_t* token, void* ws,
                            size_t ws_bytes, void* hip_stream);

/* ------------------------------------------------- around the rule in a block
 * What a block does between its matrix products and the rule: the residual sum
 * with the norms on both sides of it, and the norms over each head's channels.
 * Forward and backward, for training batches and for a server's few rows alike.
 *
 * Weights, the scale and their gradients are fp32, sums and factors too; the
 * tensors of rows are fp32 or bf16, rounded once when they are written.  They
 * need to be aligned to an element only (16 bytes are faster).  Rows do not
 * depend on each other: a NaN or Inf shows in its own row, and in the gradients of
 * the vectors.  A row's squares are summed in fp32: one whose sum passes 3.4e38 is out
 * of range (its norm is zeros; the gradients through that norm, and of the vectors on
 * it, are NaN).  Gradients of vectors are summed in one order, so a call's results are
 * the same each time.  No call allocates. */

typedef struct {
  int64_t rows, D;      /* rows of D channels; D from 1 to 16384               */
  pdn_dtype io;         /* y, u, du, dy                                        */
  pdn_dtype stream;     /* residual, h, dh, dresidual                          */
  int32_t post_norm;    /* non-zero: y is normed itself                        */
  float alpha;          /* the branch's factor; finite                         */
  float eps;            /* > 0, finite                                         */
} pdn_rnorm;

/* A block's output joins the residual stream; the next block's input is its norm:
 *   a = y, or with post_norm  y / sqrt(mean(y^2) + eps) * post_weight
 *   h = residual + alpha * scale * a
 *   u = h / sqrt(mean(h^2) + eps) * weight
 * (u of h before its rounding.)  residual [rows, D] or NULL (= 0); weight,
 * post_weight, scale [D] or NULL (= 1; post_weight without post_norm is
 * PDN_ERR_VALUE); h NULL: not written.  h may be residual itself (updated in
 * place, stream dtype); nothing else may overlap. */
pdn_status pdn_residual_norm(const pdn_rnorm* problem, const void* y, const void* residual,
                             const float* weight, const float* post_weight, const float* scale,
                             void* u, void* h, void* hip_stream);

/* Gradients of <du, u> + <dh, h>, from the h that the forward wrote (or, where
 * none was, its like).  dh: NULL (= 0).  y is needed with post_norm and for dscale.
 * dresidual and the vectors' gradients may be NULL to skip them; a vector that is
 * not given has none (PDN_ERR_VALUE).  dresidual may be dh itself.  `ws`: 256-byte
 * aligned, of at least pdn_residual_norm_bwd_workspace_size bytes; none without a
 * vector's gradient. */
pdn_status pdn_residual_norm_bwd_workspace_size(const pdn_rnorm* problem, size_t* bytes);
pdn_status pdn_residual_norm_bwd(const pdn_rnorm* problem, const void* du, const void* dh,
                                 const void* h, const void* y, const float* weight,
                                 const float* post_weight, const float* scale, void* dy,
                                 void* dresidual, float* dweight, float* dpost_weight,
                                 float* dscale, void* ws, size_t ws_bytes, void* hip_stream);

typedef enum {
  PDN_NORM_RMS = 0,     /* x / sqrt(mean(x^2) + eps): a recurrence's output    */
  PDN_NORM_L2 = 1       /* x / sqrt(sum(x^2) + eps): queries and keys          */
} pdn_norm;
typedef enum {
  PDN_ACT_NONE = 0,     /* no gate                                             */
  PDN_ACT_SILU = 1,     /* z / (1 + exp(-z))                                   */
  PDN_ACT_SIGMOID = 2   /* 1 / (1 + exp(-z))                                   */
} pdn_act;

typedef struct {
  int64_t tokens, H;    /* tensors [tokens, H, d], a token's row dense; H below
                           2^24, H d up to 2^26                                */
  int32_t d;            /* channels of a head; from 1 to 512                   */
  pdn_dtype io;         /* every tensor of rows                                */
  pdn_norm norm;
  pdn_act act;
  int32_t head_weight;  /* weight and dweight are 0: [d], else: [H, d]         */
  float eps;            /* > 0, finite                                         */
  int64_t x_stride, z_stride, y_stride, dy_stride, dx_stride, dz_stride;
                        /* elements from a token's row to the next, at least
                           H d (rows may be slices of wider ones); 0: dense    */
} pdn_hnorm;

/* y = norm(x) * weight * act(z), over each head's channels.  weight: NULL (= 1); z:
 * NULL iff PDN_ACT_NONE.  y may be x itself (same stride); nothing else may
 * overlap, but rows of one stride may interleave. */
pdn_status pdn_head_norm(const pdn_hnorm* problem, const void* x, const void* z,
                         const float* weight, void* y, void* hip_stream);

/* Gradients of <dy, y>.  dz: NULL iff PDN_ACT_NONE; dweight: NULL to skip it, or
 * without a weight.  dx may be dy itself (same stride).  `ws` as above. */
pdn_status pdn_head_norm_bwd_workspace_size(const pdn_hnorm* problem, size_t* bytes);
pdn_status pdn_head_norm_bwd(const pdn_hnorm* problem, const void* dy, const void* x,
                             const void* z, const float* weight, void* dx, void* dz,
                             float* dweight, void* ws, size_t ws_bytes, void* hip_stream);

/* ------------------------------------------------------ from logits to tokens
 * pdn_logits makes of logits the probabilities that pdn_draft_verify reads;
 * pdn_token_counts keeps the table of tokens that a sequence has had, in the same
 * slots as its state.  A round: pdn_slot_draft .. logits -> pdn_logits ->
 * pdn_draft_verify -> pdn_token_counts with its `accepted`, and pdn_slot_draft again.
 *
 * A count is 32 bits: the lower 31 how often the sequence generated the token, the
 * sign bit set if the prompt has it.
 *
 * Rows are packed as in pdn_draft_verify: `starts` [N + 1], NULL for rows / N rows
 * each.  Lists on the device are not checked: row numbers are clamped to [0, rows],
 * a sequence whose slot is outside [0, slots) is left out (its rows of `out`, and
 * the table, stay as they were), tokens outside [0, V) count for nothing.  Rows that
 * belong to no sequence stay as they were.  rows (for the counts N) times V / 2048, rounded
 * up, must be below 2^24. */

typedef struct {
  int64_t rows, V, N;        /* N sequences                                     */
  pdn_dtype dtype;           /* logits                                          */
  pdn_dtype out_dtype;
  int32_t probs;             /* 0: the changed logits, else probabilities       */
  int64_t stride;            /* elements from a row of logits to the next, at
                                least V; 0: V.  Rows of out are dense           */
  const void* logits;        /* [rows, V]                                       */
  const int32_t* starts;
  const float* temperature;  /* [N], or NULL (= 1)                              */
  const float* repetition;   /* [N] or NULL (= 1)                               */
  const float* presence;     /* [N] or NULL (= 0)                               */
  const float* frequency;    /* [N] or NULL (= 0)                               */
  const int32_t* counts;     /* [slots, V] or NULL (= 0)                        */
  int64_t slots;             /* rows of counts                                  */
  const int32_t* slot;       /* [N] or NULL (the sequence's own number); with
                                counts only                                     */
  const int32_t* ids;        /* [rows] tokens fed (as for pdn_draft_verify), not
                                in the table yet: row t of a sequence counts
                                those of its rows up to t.  NULL: none          */
  const int32_t* bias_starts;/* [N + 1] a sequence's entries of the next two, or
                                NULL                                            */
  const int32_t* bias_ids;   /* [biases]; of a token listed twice in a sequence
                                the last entry holds                            */
  const float* bias_values;  /* [biases]                                        */
  int64_t biases;
  const int32_t* mask;       /* [masks, (V + 31) / 32]: token j is allowed where
                                bit j % 32 of word j / 32 is set; or NULL       */
  int64_t masks;
  const int32_t* mask_rows;  /* [rows] a row's mask, outside [0, masks): none.
                                NULL: its own number (masks >= rows)            */
} pdn_logits_args;

/* Token j of a row, c its count (table and ids), l its logit:
 *   l = l > 0 ? l / repetition : l * repetition    if c > 0 or the prompt has it
 *   l = (l - frequency * c) - presence             if c > 0
 *   l = l + bias
 *   l = -inf                                       if the mask does not allow it
 * each step rounded to fp32.  out: l, or p = softmax(l / temperature); with a
 * temperature that is not above 0 (or NaN) one at the largest l (the lowest token of
 * several), else zero.  A row in which nothing is left (every l -inf) is zeros:
 * pdn_draft_verify then gives token -1.  Tokens at +inf share the probability.
 * A NaN in a place that the mask forbids is not seen; any other makes its row NaN.
 * out [rows, V] may be the logits themselves (same dtype, dense); nothing else may
 * overlap.  All row tensors need to be aligned to an element only.  `ws`: 256-byte
 * aligned, of pdn_logits_workspace_size bytes (none without probs). */
pdn_status pdn_logits_workspace_size(int64_t rows, int64_t V, size_t* bytes);
pdn_status pdn_logits(const pdn_logits_args* args, void* out, void* ws, size_t ws_bytes,
                      void* hip_stream);

/* Adds tokens to the table: of each sequence's ids the first accepted[n] (NULL: all),
 * as generated ones, or with `prompt` as the prompt's.  The counts are read from
 * slot[n] (NULL: n; `fresh` non-zero: zero, nothing is read) and written to slot_out[n]
 * (NULL: slot; another one: a fork).  Without slot_out and fresh only the tokens'
 * own entries are touched.  A slot written by one sequence must not be read or written
 * by another of the same call, but sequences may add to one slot without slot_out and
 * fresh.  accepted is pdn_draft_verify's: the tokens fed that hold. */
pdn_status pdn_token_counts(int64_t N, int64_t rows, int64_t V, int64_t slots, int32_t prompt,
                            const int32_t* ids, const int32_t* starts, const int32_t* slot,
                            const int32_t* slot_out, const int32_t* fresh,
                            const int32_t* accepted, int32_t* counts, void* hip_stream);

/* Static, NUL-terminated description of a status code. */
const char* pdn_status_string(pdn_status status);

/* PDN_ABI_VERSION of the built library. */
int pdn_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* PDN_H */
