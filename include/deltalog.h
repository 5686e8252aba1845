/*
 * deltalog.h -- C ABI of libdeltalog.so: DeltaLog one-token decode state update for
 * linear-attention recurrences (the Table 1 operators: GDN, KDA, RWKV6, linear
 * attention, RetNet, GLA) on AMD Instinct MI355X (gfx950).
 *
 * The method (deferred materialisation of recurrent states, Sec. 3): the dense
 * recurrent state of each (slot, head) is kept as a dense base S plus a bounded log of
 * compact update factors.  Most decode steps read S once, replay the live log, emit
 * the output and append one entry (Eq. 5); every M-th step folds the log and the
 * current token back into S with a single dense write (Eq. 6).  The represented
 * state is always Eq. 7:
 *
 *     S_logical = D(ell) S + sum_{i<L} D(ell - Lam_i) K_i U_i^T,   D(l) = diag(exp l)
 *
 * and equals the eager recurrence of Eq. 3 (Table 1 instantiations) in exact
 * arithmetic.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Every data pointer is a DEVICE pointer (hipMalloc'd or a torch CUDA tensor),
 *    owned by the caller.  The library never allocates, frees or synchronises; all
 *    work is enqueued on the caller's `stream`, and buffers must stay alive until the
 *    stream has executed it.  Calls on distinct buffers are re-entrant and thread-safe.
 *  - Arrays are dense, row-major, with the shapes given below.  B = desc->num_slots,
 *    H = desc->heads, C = desc->merge_interval - 1 (live-log capacity),
 *    dl = 1 for GDN and RetNet (one log-decay per head), dl = dk for KDA, RWKV6 and
 *    GLA (per key); linear attention has no decay (no lam_log or lam).
 *  - The state matrix of a head is dk x dv, rows indexed by the key dimension; the
 *    decay D(.) scales rows (Eq. 2); outputs are o = x^T S (length dv).
 *  - `slots` is a device int32 array of n distinct slot ids in [0, B): token row i
 *    drives slot slots[i].  slots == NULL means the identity and requires n == B,
 *    except that n == 0 is always a no-op: once the descriptor is valid and 0 <= n <= B
 *    it returns DL_OK without looking at any pointer.
 *    Duplicate ids in one call race (undefined).
 *  - Token arrays are packed by token row: [n, H, ...].  Outputs are written by token
 *    row, fp32, [n, H, dv].  `o` must not alias any input or state buffer.
 *  - Every argument check happens on the host BEFORE any HIP call; a failing check
 *    returns a negative dl_status and enqueues nothing (so the checks can be exercised
 *    without a GPU).  A failed launch returns DL_E_HIP.  Corruption that only the
 *    device can see (a slot id outside [0, B), a live length outside [0, C]) makes the
 *    affected (slot, head) skip its work and ORs a code into *state->err (if non-NULL):
 *    1 = bad slot id, 2 = live length out of range.
 *  - Alignment: S, k_log, u_log, q, k, v and o must be 16-byte aligned, and so must
 *    lam_log when dl == dk (KDA, RWKV6, GLA: its rows are read 16 bytes at a time);
 *    the other float/int32 arrays 4-byte aligned.
 *  - Supported shapes: dk, dv in {64, 128}; 1 <= M <= 64.
 */
#ifndef DELTALOG_H
#define DELTALOG_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DL_ABI_VERSION 4
#define DL_MAX_MERGE_INTERVAL 64

typedef enum {
  DL_OK = 0,
  DL_E_NULL = -1,        /* a required pointer is NULL                                  */
  DL_E_SHAPE = -2,       /* B, H, n or slot-list shape inconsistent                     */
  DL_E_DTYPE = -3,       /* dtype combination not allowed                               */
  DL_E_ALIGN = -4,       /* pointer not aligned as required                             */
  DL_E_UNSUPPORTED = -5, /* dk/dv/M/op outside the supported set                        */
  DL_E_HIP = -6,         /* the kernel launch failed                                    */
  DL_E_VERSION = -7,     /* desc->abi_version != DL_ABI_VERSION                         */
  DL_E_SCRATCH = -8      /* needs more than DL_NOALLOC_SCRATCH_BYTES of scratch          */
} dl_status;

typedef enum {
  DL_OP_GDN = 0,
  DL_OP_KDA = 1,
  DL_OP_RWKV6 = 2,
  DL_OP_LINATTN = 3,
  DL_OP_RETNET = 4,
  DL_OP_GLA = 5
} dl_op;
typedef enum { DL_F32 = 0, DL_BF16 = 1 } dl_dtype;

/* Problem description (host memory, read during the call only).
 * Operators (Table 1, Eq. 3):
 *   GDN     head-wise scalar decay, delta-rule pair (k, beta (v - k^T D(lambda) S)),
 *           post-update readout o = q^T S_t;
 *   KDA     per-key decay, the same pair and readout;
 *   RWKV6   per-key decay, pair (k, v), bonus readout o = r^T (S_{t-1} + diag(u) k v^T);
 *   LINATTN no decay, pair (phi(k), v) with phi applied by the caller, o = q^T S_t
 *           (Eq. 1);
 *   RETNET  head-wise scalar decay gamma_t = exp(lambda_t), pair (k, v), o = q^T S_t;
 *   GLA     per-key decay, pair (k, v), o = q^T S_t.
 * dl (the log-decay width) is dk for KDA, RWKV6 and GLA and 1 for GDN and RetNet;
 * linear attention has no log-decay and touches neither lam_log nor lam.
 * The cumulative log-decay ell of Sec. 3.1 is not a buffer here: Eq. 5 writes ell and
 * the new snapshot Lam_log[L] with the same value and Eq. 6 resets ell together with L,
 * so ell is always the newest snapshot Lam_log[L-1], or 0 when L = 0, and the library
 * reads it from there. */
typedef struct {
  int32_t abi_version;    /* must be DL_ABI_VERSION                                      */
  int32_t op;             /* dl_op                                                       */
  int32_t num_slots;      /* B >= 1: slots in the state buffers                          */
  int32_t heads;          /* H >= 1                                                      */
  int32_t dk, dv;         /* key / value head dims, each 64 or 128                       */
  int32_t merge_interval; /* M in [1, 64]: one merge every M steps (Sec. 3.1); C = M-1   */
  int32_t in_dtype;       /* dl_dtype of q/r, k, v; K_log stores exact copies of k       */
  int32_t u_log_dtype;    /* dl_dtype of U_log: DL_F32 for GDN/KDA (corrected values),   */
                          /* == in_dtype for the others (exact copies of v)              */
  int32_t state_dtype;    /* dl_dtype of the dense state S: DL_F32, or DL_BF16 (all       */
                          /* arithmetic in fp32, S rounded to bf16 -- nearest even -- on  */
                          /* every store; every other buffer keeps its dtype)            */
} dl_desc;

/* DeltaLog physical state (Sec. 3.1 list of buffers, less ell: see dl_desc), one entry
 * per (slot, head). */
typedef struct {
  void*    S;        /* [B,H,dk,dv] state_dtype dense base                               */
  void*    k_log;    /* [B,H,C,dk]  in_dtype   key-side factors   (may be NULL if C == 0) */
  void*    u_log;    /* [B,H,C,dv]  u_log_dtype value-side factors (may be NULL if C == 0)*/
  float*   lam_log;  /* [B,H,C,dl]  fp32 snapshot of ell per entry (may be NULL if C == 0)*/
                     /*             16-byte aligned when dl == dk, else 4-byte            */
                     /*             for dl == 1 stored entry-major, [B,C,H]               */
                     /*             (ignored, may be NULL, for LINATTN)                  */
  int32_t* len;      /* [B,H]       live-log length L in [0, C]                          */
  int32_t* err;      /* [1]         sticky device error word (see above); may be NULL    */
} dl_state;

/* Current-token inputs: the per-token interface of Eq. 3, one row per listed slot. */
typedef struct {
  const void*  q;    /* [n,H,dk] in_dtype: query (the receptance r for RWKV6)            */
  const void*  k;    /* [n,H,dk] in_dtype: key, the key-side factor a_t                  */
  const void*  v;    /* [n,H,dv] in_dtype: value                                         */
  const float* beta; /* [n,H]    fp32 delta-rule write strength (GDN/KDA); else ignored  */
  const float* lam;  /* [n,H,dl] fp32 per-step log-decay lambda_t = log(alpha_t) <= 0     */
                     /*          (ignored, may be NULL, for LINATTN)                     */
  const float* u;    /* [H,dk]   fp32 RWKV6 bonus (per-head parameter); NULL otherwise   */
} dl_token;

/* Eager dense step (Eq. 3): S <- D(lambda) S + a b^T with the readout of Table 1, for
 * the listed slots of a dense state S [B,H,dk,dv] of state_dtype (no log).  Writes
 * o [n,H,dv].
 * This is the baseline that reads and writes the whole state every token (Sec. 2.3).
 * desc->merge_interval is validated but otherwise ignored. */
int dl_eager_step(const dl_desc* desc, void* S, const dl_token* tok, float* o,
                  const int32_t* slots, int32_t n, hipStream_t stream);

/* One DeltaLog decode step (Alg. 1) for the listed slots: per (slot, head) read the
 * base once, replay the live log, write the output, then append the factors
 * (Eq. 5) if L < C, else merge log and token into the base (Eq. 6) and reset L (the
 * cumulative log-decay restarts at 0).  With M == 1 every step merges and the result
 * equals dl_eager_step. */
int dl_append_step(const dl_desc* desc, const dl_state* state, const dl_token* tok,
                   float* o, const int32_t* slots, int32_t n, hipStream_t stream);

/* Merge now, at any live length L in [0, C] (Eq. 6 is defined for general L).
 * tok != NULL: consume the token exactly like the merge branch of dl_append_step and
 *              write o (required).
 * tok == NULL: flush -- materialise Eq. 7 into the base and reset (slot reuse,
 *              eviction, checkpoint; Sec. 4 slot lifecycle); o is ignored. */
int dl_merge(const dl_desc* desc, const dl_state* state, const dl_token* tok, float* o,
             const int32_t* slots, int32_t n, hipStream_t stream);

/* Read-only readout of the represented state (Eq. 7): o = x^T S_logical for a query
 * x [n,H,dk] in in_dtype.  Mutates nothing.  (No RWKV6 bonus: there is no token.) */
int dl_readout(const dl_desc* desc, const dl_state* state, const void* q, float* o,
               const int32_t* slots, int32_t n, hipStream_t stream);

/* Value-tiled DeltaLog step (Sec. 3.3, the kernel ownership path): the same operation
 * as dl_append_step (results equal up to floating-point reassociation), with each
 * (slot, head) state split along the value dimension into value_tiles tiles of
 * dk x dv/value_tiles, one workgroup each.  Two launches on the stream (one if C == 0):
 *   [ReplayPrep]  split_replay != 0 and C > 0 only: the key-side replay coefficients
 *                 q^T D(ell - Lam_i) K_i and k^T D(ell - Lam_i) K_i of every live entry,
 *                 once per (row, head), into the caller's workspace (fp32), and the
 *                 commit of L (from which the tiles tell the L they act on);
 *   AppendDecode  per value tile: stream the tile, replay the log on its columns (with
 *                 the prepared coefficients, or recomputing them per tile when
 *                 split_replay == 0), write the output slice, append the tile's U_log
 *                 shard (tile 0 also writes K_log[L] and Lam_log[L]) or merge the tile;
 *   [Finalize]    split_replay == 0 and C > 0 only: commit L exactly once per (row, head).
 * value_tiles: 2 or 4.  Only state_dtype == DL_F32 (else DL_E_DTYPE).
 * workspace: device memory of at least dl_tiled_workspace_bytes(desc, n) bytes, 16-byte
 * aligned, owned by the caller; required when split_replay != 0 and C > 0, ignored
 * otherwise.  Its contents are scratch: overwritten, never read across calls.  Calls
 * that share a workspace must not overlap.  If a later launch fails, DL_E_HIP is
 * returned and the earlier launch of the call may already be enqueued.  With split replay
 * one more launch then takes the committed lengths back, and the state is as before the
 * call (if that launch fails too, the state must be taken as partly stepped); with fused
 * replay the tiles have run and their lengths are not committed, and the state must be
 * taken as partly stepped. */
int dl_append_step_tiled(const dl_desc* desc, const dl_state* state, const dl_token* tok,
                         float* o, const int32_t* slots, int32_t n, int32_t value_tiles,
                         int32_t split_replay, void* workspace, size_t workspace_bytes,
                         hipStream_t stream);

/* Bytes of workspace dl_append_step_tiled needs for n rows with split replay:
 * n * H * 2 * (M - 1) * sizeof(float) (0 when M == 1).  Writes *bytes. */
int dl_tiled_workspace_bytes(const dl_desc* desc, int32_t n, size_t* bytes);

/* Size of the fixed scratch of dl_append_step_tiled_noalloc, per GPU. */
#define DL_NOALLOC_SCRATCH_BYTES (4u << 20)

/* For callers that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): dl_append_step_tiled with split
 * replay, its workspace taken from a scratch array of DL_NOALLOC_SCRATCH_BYTES that the
 * library holds in device memory, one per GPU, for the life of the process.  The caller
 * still passes the state, token and output buffers; the call allocates and frees
 * nothing and enqueues exactly the launches of dl_append_step_tiled(..., split_replay=1,
 * ...), with the same state after a launch that fails.
 * The scratch needed is dl_tiled_workspace_bytes(desc, n); a call that needs more than
 * DL_NOALLOC_SCRATCH_BYTES returns DL_E_SCRATCH (after the argument checks, before any
 * HIP call) and enqueues nothing.
 * Every call on a GPU shares that GPU's scratch: calls that may overlap on one GPU (on
 * different streams, or from different threads without ordering) race and must not be
 * issued; calls ordered on one stream are safe.  The scratch keeps the last call's
 * contents; a call reads only what it wrote itself.  On its first call on a device the
 * entry point looks up that device's scratch address (a HIP runtime query, no
 * allocation) and keeps it; a failed lookup returns DL_E_HIP. */
int dl_append_step_tiled_noalloc(const dl_desc* desc, const dl_state* state,
                                 const dl_token* tok, float* o, const int32_t* slots,
                                 int32_t n, int32_t value_tiles, hipStream_t stream);

/* ---------------------------------------------------------------- whole sequences
 * The recurrence over ragged batches of sequences (prompts, training documents): token
 * rows of all sequences packed one after the other, [N, H, ...], sequence i with its own
 * initial and final state (a slot of a [B,H,dk,dv] buffer).  Lengths live in device memory;
 * the host knows n (sequences) and N (token rows the buffers hold) only.  Sequences may be
 * empty: their state passes through.  Rows behind the last sequence belong to nobody: they
 * are never used, and output rows there stay as they were. */
#define DL_CHUNK 32   /* tokens of a chunk of the tables below */

#define DL_MAX_HEADS 65536   /* of whole-sequence calls */

/* Chunk rows the tables of n sequences with up to `tokens` token rows have. */
#define DL_MAX_CHUNKS(n, tokens) ((tokens) / DL_CHUNK + (n))

/* Chunk tables and slot maps of a ragged batch (device memory, owned by the caller). */
typedef struct {
  int32_t* cu_tokens; /* [n+1] first token row of each sequence; [n] = rows in use         */
  int32_t* cu_chunks; /* [n+1] first chunk of each sequence; [n] = chunks in use           */
  int32_t* chunks;    /* [DL_MAX_CHUNKS(n,N), 4], 16-byte aligned: (sequence, first token  */
                      /*       row, tokens, slot); (-1, 0, 0, -1) past the chunks in use   */
  int32_t* row_slot;  /* [N]   slot of every token row; -1 past the rows in use            */
  int32_t* seq_slot;  /* [n]   slot of every sequence                                      */
  int32_t* order;     /* [n]   the sequences, longest first up to 1024 of them (dl_prefill */
                      /*       starts them in this order), as they come with more          */
} dl_tables;

/* Build the tables from lens [n] (device) and slots (device int32 [n], or NULL: sequence i
 * has slot i, which requires n <= num_slots; ids of sequences that run are distinct, two on
 * one slot race on its final state).  What only the device can see is ORed into
 * *err (device, may be NULL): 1 = a slot id outside [0, num_slots) (the sequence's slot
 * becomes -1, and dl_prefill and dl_prefill_backward skip it), 4 = a length below 0 (taken
 * as 0) or past the N token rows (cut there).  n == 0 is a no-op. */
int dl_chunk_tables(const int32_t* lens, const int32_t* slots, int32_t n, int32_t tokens,
                    int32_t num_slots, const dl_tables* tables, int32_t* err,
                    hipStream_t stream);

/* Bytes of workspace dl_prefill (backward == 0) or dl_prefill and dl_prefill_backward
 * (backward != 0) need for n sequences and N token rows.  Writes *bytes. */
int dl_prefill_workspace_bytes(const dl_desc* desc, int32_t n, int32_t tokens,
                               int32_t backward, size_t* bytes);

/* The recurrence over whole sequences (Eq. 3, token by token in exact arithmetic): for
 * every sequence of the tables, from S_in[slot] (S_in == NULL: zero) to S_out[slot] (both
 * [B,H,dk,dv] of state_dtype; S_out may be S_in), with o [N,H,dv] in in_dtype -- a prompt's
 * outputs go on to products in that type, and a state read back in it would not gain from
 * wider ones.  tok holds N rows.  Products, sums, decays and states are fp32 (fp32 results are
 * within some 4e-7 of the exact ones, relative to their norm), and o and S_out are rounded once;
 * only factors that go into a bf16 o alone are good to 2^-17.  Log-decays are summed in fp32 from a
 * chunk's start, so the decay between two tokens behind a gate of 0 (which counts as -104) in the
 * same chunk is good to some 1e-5.  Outputs must not overlap inputs, S_out = S_in apart.
 * The log of a DeltaLog state is not looked at: flush it first (dl_merge without a token)
 * where S_in is the base of a state with a log, and reset len where S_out is.
 * tables: as dl_chunk_tables left them for the same n and N (row_slot is not read).
 * workspace: at least dl_prefill_workspace_bytes(desc, n, N, 0, ..) bytes, 256-byte
 * aligned; scratch, never read across calls; calls that share one must not overlap.
 * With no token rows (N == 0) the pointers to rows may be NULL.
 * desc->merge_interval is validated but otherwise ignored.  At most DL_MAX_HEADS heads
 * (else DL_E_SHAPE).  n == 0 is a no-op.
 * A value that is infinite or NaN (a log-decay too) stays within its sequence and head, but may
 * reach outputs of up to 31 tokens before its own (its chunk's), and an infinite one may come out
 * as NaN.  Log-decays above 0 are taken at their value, as by the decode calls. */
int dl_prefill(const dl_desc* desc, const void* S_in, void* S_out, const dl_token* tok, void* o,
               const dl_tables* tables, int32_t n, int32_t tokens, void* workspace,
               size_t workspace_bytes, hipStream_t stream);

/* Gradients, shaped as what they belong to; dq, dk, dv in in_dtype, dS in state_dtype. */
typedef struct {
  void*  dq;    /* [N,H,dk]                                                              */
  void*  dk;    /* [N,H,dk]                                                              */
  void*  dv;    /* [N,H,dv]                                                              */
  float* dbeta; /* [N,H] (GDN/KDA; else ignored)                                         */
  float* dlam;  /* [N,H,dl] (ignored for LINATTN)                                        */
  float* du;    /* [H,dk] (RWKV6; else ignored)                                          */
  void*  dS;    /* [B,H,dk,dv] of the initial states; may be NULL.  Slots that no        */
                /* sequence has stay as they were.                                       */
} dl_grads;

/* Backward pass of dl_prefill: from d_o [N,H,dv] (in_dtype) and dS_out [B,H,dk,dv] (of the
 * final states, state_dtype; NULL: zero) to every gradient, for the same S_in, tok and
 * tables as the forward call.  Nothing is kept from the forward call: the states are
 * computed again.  S_in is read, so a forward call that wrote its states in place has
 * destroyed what this call needs.  dS may be dS_out; no other gradient may overlap an input or
 * another gradient (dv is written while v is still read).
 * workspace: dl_prefill_workspace_bytes(desc, n, N, 1, ..) bytes, 256-byte aligned. */
int dl_prefill_backward(const dl_desc* desc, const void* S_in, const dl_token* tok,
                        const void* d_o, const void* dS_out, const dl_grads* grads,
                        const dl_tables* tables, int32_t n, int32_t tokens, void* workspace,
                        size_t workspace_bytes, hipStream_t stream);

/* ---------------------------------------------------------------- around a recurrence
 * What a layer puts in front of the recurrences above -- a short causal convolution of every
 * channel, norms and rotations of queries and keys -- and the recurrence whose decay differs by
 * channel and state.  Whole sequences are packed as above and use the same dl_tables (of which
 * these calls read cu_tokens and seq_slot only); single tokens take a slot list as the decode
 * calls do.  n == 0 is a no-op; rows behind the last sequence are never used, and output rows
 * there stay as they were.
 *  - Token rows that are inputs may be columns of a wider array: *_stride counts the elements
 *    from one row to the next, at least a row's width, a multiple of 8 and up to
 *    DL_MAX_STRIDE.  Arrays of in_dtype and states are 16-byte aligned, fp32 parameters and int32 arrays 4-byte aligned.  Outputs
 *    and gradients are dense.
 *  - Products, sums, states' arithmetic and statistics are fp32; every output is rounded once.
 *  - Outputs must not overlap inputs or each other, s_out = s_in apart.  Calls on distinct
 *    buffers are re-entrant; calls that share a workspace must not overlap.
 *  - Sums over tokens, rows or channels (gradients of parameters, of B and C) are taken in an
 *    order that depends on sizes alone: the same call gives the same bits.
 *  - Slots that are listed twice in one call race (undefined). */

#define DL_MAX_STRIDE (1 << 24)

typedef enum { DL_ACT_NONE = 0, DL_ACT_SILU = 1 } dl_activation;

/* Short causal convolution of every channel c of D, W taps:
 *   a_t = bias + sum_j w[c,j] x_{t-W+1+j},   y_t = a_t or silu(a_t) = a_t / (1 + e^-a_t),
 * x_t with t < 0 being the state: the W - 1 inputs before the first token, oldest first. */
typedef struct {
  int32_t abi_version;  /* must be DL_ABI_VERSION                                       */
  int32_t num_slots;    /* B >= 1                                                       */
  int32_t channels;     /* D >= 8, a multiple of 8                                      */
  int32_t width;        /* W: 2, 3 or 4                                                 */
  int32_t activation;   /* dl_activation                                                */
  int32_t in_dtype;     /* dl_dtype of x, y, the states and their gradients             */
} dl_conv_desc;

typedef struct {
  const void*  x;       /* [N,D] in_dtype                                               */
  int64_t      x_stride;
  const float* w;       /* [D,W] fp32, the newest input's tap last                      */
  const float* bias;    /* [D] fp32, or NULL: none                                      */
} dl_conv_rows;

typedef struct {
  void*  dx;            /* [N,D] in_dtype                                               */
  float* dw;            /* [D,W] fp32                                                   */
  float* dbias;         /* [D] fp32 (ignored without a bias)                            */
  void*  ds;            /* [B,W-1,D] of the states before, or NULL.  Slots that no      */
                        /* sequence has stay as they were.                              */
} dl_conv_grads;

/* One token per listed slot: y [n,D] from s_in [B,W-1,D] and x [n,D]; s_out (may be s_in) gets
 * the listed slots' new states. */
int dl_conv_step(const dl_conv_desc* desc, const void* s_in, void* s_out,
                 const dl_conv_rows* rows, void* y, const int32_t* slots, int32_t n,
                 hipStream_t stream);

/* Whole sequences, each from s_in[slot] (s_in == NULL: zeros) to s_out[slot] (may be s_in). */
int dl_conv_prefill(const dl_conv_desc* desc, const void* s_in, void* s_out,
                    const dl_conv_rows* rows, void* y, const dl_tables* tables, int32_t n,
                    int32_t tokens, hipStream_t stream);

/* Bytes of workspace dl_conv_backward needs.  Writes *bytes. */
int dl_conv_workspace_bytes(const dl_conv_desc* desc, int32_t n, int32_t tokens, size_t* bytes);

/* Gradients of dl_conv_prefill from dy [N,D] and ds_out [B,W-1,D] (of the final states; NULL:
 * zero), for the same s_in, rows and tables.  Nothing is kept from the forward call.  The
 * gradients of s_in must not overlap ds_out.  workspace: 256-byte aligned. */
int dl_conv_backward(const dl_conv_desc* desc, const void* s_in, const dl_conv_rows* rows,
                     const void* dy, const void* ds_out, const dl_conv_grads* grads,
                     const dl_tables* tables, int32_t n, int32_t tokens, void* workspace,
                     size_t workspace_bytes, hipStream_t stream);

/* Norms of queries and keys, head by head, with the rotation by position in the same pass.  For
 * a head x of d places: n = scale w . x / sqrt(c sum x^2 + eps), c = 1 (L2) or 1 / d (root mean
 * square); no norm: n = scale w . x; scale is q_scale for queries, 1 for keys.  Then pair i of
 * the first rot places -- (i, rot/2 + i) for halves, (2i, 2i + 1) for pairs -- turns by the angle
 * pos freq[i] (the product in 64 bits): (a cos - b sin, a sin + b cos).  Every head is written rep
 * times, output heads h rep .. h rep + rep - 1, for recurrences whose heads share keys.  Any rows:
 * prompts, training, one token a slot.  What is infinite or NaN stays in its head; a head whose sum of
 * squares is beyond fp32 has the norm infinity, and comes out 0. */
typedef enum { DL_NORM_NONE = 0, DL_NORM_L2 = 1, DL_NORM_RMS = 2 } dl_norm;
typedef enum { DL_TURN_NONE = 0, DL_TURN_HALVES = 1, DL_TURN_PAIRS = 2 } dl_turn;

typedef struct {
  int32_t abi_version;  /* must be DL_ABI_VERSION                                       */
  int32_t heads;        /* H >= 1 of the inputs; H rep <= DL_MAX_HEADS                  */
  int32_t head_dim;     /* d: 64 or 128                                                 */
  int32_t rep;          /* >= 1                                                         */
  int32_t norm;         /* dl_norm                                                      */
  int32_t turn;         /* dl_turn                                                      */
  int32_t rot;          /* places that turn: a multiple of 16 up to d; 0 without turn   */
  int32_t in_dtype;     /* dl_dtype of q, k, outputs and their gradients                */
  float eps;            /* 2^-126 (the smallest normal fp32 number) or above with a norm */
  float q_scale;
} dl_qk_desc;

typedef struct {
  const void*    q;     /* [n,H,d] in_dtype                                             */
  const void*    k;     /* [n,H,d] in_dtype                                             */
  int64_t        q_stride, k_stride;
  const int32_t* pos;   /* [n] positions (may be NULL without turn)                     */
  const float*   freq;  /* [rot/2] fp32, radians a position (may be NULL without turn)  */
  const float*   wq;    /* [d] fp32 weights, both or (NULL) neither                     */
  const float*   wk;
  const int32_t* used;  /* [1] rows in use, as dl_tables' cu_tokens + n (device); rows  */
                        /* behind them stay untouched.  NULL: all n                     */
} dl_qk_rows;

typedef struct {
  void*  dq;            /* [n,H,d] in_dtype                                             */
  void*  dk;
  float* dwq;           /* [d] fp32 (ignored without weights)                           */
  float* dwk;
} dl_qk_grads;

/* q_out, k_out [n,H rep,d]. */
int dl_qk_norm(const dl_qk_desc* desc, const dl_qk_rows* rows, void* q_out, void* k_out,
               int32_t n, hipStream_t stream);

/* Bytes of workspace dl_qk_norm_backward needs (with weights; without them it may be NULL).
 * Writes *bytes. */
int dl_qk_workspace_bytes(const dl_qk_desc* desc, int32_t n, size_t* bytes);

/* Gradients of dl_qk_norm from dq_out, dk_out [n,H rep,d], for the same rows. */
int dl_qk_norm_backward(const dl_qk_desc* desc, const dl_qk_rows* rows, const void* dq_out,
                        const void* dk_out, const dl_qk_grads* grads, int32_t n, void* workspace,
                        size_t workspace_bytes, hipStream_t stream);

/* Selective state space scan: channel c of D has S states, with its own decays.  With
 * d_t = softplus(dt_t + dt_bias), softplus(r) = log(1 + e^r):
 *   h_t = exp(d_t A) . h_{t-1} + d_t x_t B_t,   y_t = (<C_t, h_t> + skip x_t) silu(z_t),
 * A and h_t [S] per channel (A <= 0 forgets; taken at its value), B_t and C_t [S] the same for
 * all channels, skip and z left out where NULL.  Whole sequences are cut into stretches that run
 * side by side, of a length that goes by the call's tokens: what a sequence's results round to
 * depends on how many rows the call has.
 * A value that is infinite or NaN stays in its sequence, and in its channel unless it is one of
 * B or C; an infinite one may come out as NaN, and so may what follows decays above 1 whose product
 * over a sequence's tokens is beyond fp32.  Steps are at most as large as fp32 holds; the
 * hardware's exponential takes decays below 2^-126 for 0. */
typedef struct {
  int32_t abi_version;  /* must be DL_ABI_VERSION                                       */
  int32_t num_slots;    /* >= 1                                                         */
  int32_t channels;     /* D >= 8, a multiple of 8                                      */
  int32_t states;       /* S: 16, 32 or 64                                              */
  int32_t in_dtype;     /* dl_dtype of x, dt, z, B, C, y and their gradients            */
} dl_ssm_desc;          /* states are fp32, [num_slots,D,S]                             */

typedef struct {
  const void*  x;       /* [N,D] in_dtype                                               */
  const void*  dt;      /* [N,D] in_dtype                                               */
  const void*  z;       /* [N,D] in_dtype, or NULL: no gate                             */
  const void*  B;       /* [N,S] in_dtype                                               */
  const void*  C;       /* [N,S] in_dtype                                               */
  int64_t      x_stride, dt_stride, z_stride, b_stride, c_stride;
  const float* A;       /* [D,S] fp32                                                   */
  const float* skip;    /* [D] fp32, or NULL                                            */
  const float* dt_bias; /* [D] fp32, or NULL                                            */
} dl_ssm_rows;

typedef struct {
  void*  dx;            /* [N,D] in_dtype, and so on                                    */
  void*  ddt;
  void*  dz;            /* ignored without z                                            */
  void*  dB;            /* [N,S]                                                        */
  void*  dC;
  float* dA;            /* [D,S]                                                        */
  float* dskip;         /* [D]; ignored without skip                                    */
  float* dbias;         /* [D]; ignored without dt_bias                                 */
  float* ds;            /* [num_slots,D,S] of the states before, or NULL.  Slots that   */
                        /* no sequence has stay as they were.                           */
} dl_ssm_grads;

/* One token per listed slot: y [n,D] from h_in and one row each; h_out (may be h_in) gets the
 * listed slots' new states. */
int dl_ssm_step(const dl_ssm_desc* desc, const float* h_in, float* h_out, const dl_ssm_rows* rows,
                void* y, const int32_t* slots, int32_t n, hipStream_t stream);

/* Bytes of workspace dl_ssm_prefill (backward == 0) or dl_ssm_prefill and dl_ssm_backward
 * (backward != 0) need for this n and these tokens (other ones can need more); may be 0, and the
 * workspace NULL then.  Large calls: forward some 17 MiB, backward about 0.75 tokens x channels x
 * states bytes with 16 states and 1.3 with 32 or 64 (4096 tokens of 4096 x 16: 195 MiB; 16384 of
 * 1024 x 64: 1268 MiB), most of it the states before every tile of 8 (4) tokens.  Writes *bytes. */
int dl_ssm_workspace_bytes(const dl_ssm_desc* desc, int32_t n, int32_t tokens, int32_t backward,
                           size_t* bytes);

/* Whole sequences, each from h_in[slot] (h_in == NULL: zeros) to h_out[slot] (may be h_in).
 * workspace: 256-byte aligned. */
int dl_ssm_prefill(const dl_ssm_desc* desc, const float* h_in, float* h_out,
                   const dl_ssm_rows* rows, void* y, const dl_tables* tables, int32_t n,
                   int32_t tokens, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Gradients of dl_ssm_prefill from dy [N,D] and dh_out (of the final states; NULL: zero), for the
 * same h_in, rows and tables.  Nothing is kept from the forward call.  The gradients of h_in must
 * not overlap dh_out. */
int dl_ssm_backward(const dl_ssm_desc* desc, const float* h_in, const dl_ssm_rows* rows,
                    const void* dy, const float* dh_out, const dl_ssm_grads* grads,
                    const dl_tables* tables, int32_t n, int32_t tokens, void* workspace,
                    size_t workspace_bytes, hipStream_t stream);

/* Human-readable name of a dl_status value (static storage). */
const char* dl_status_str(int status);

/* DL_ABI_VERSION of the loaded library. */
int dl_abi_version(void);

/* The compiler flags the library's kernels were built with beyond the optimisation
 * level and target (static storage), so that measurements can be matched to the exact
 * build that produced them. */
const char* dl_build_flags(void);

#ifdef __cplusplus
}
#endif

#endif /* DELTALOG_H */
