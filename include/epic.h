/* epic.h - C ABI of the MI355X (gfx950) validity-check hot path of EPIC
 * (Efficient and Parallel Inference under CFG constraints, arxiv 2606.00722).
 *
 * Per denoising step a diffusion LM proposes (position, token) commits for a
 * batch of partially masked token sequences.  This library decides, for every
 * proposal, whether the sequence stays completable under a context-free
 * grammar (Sec. 3: Valid_G(x, D) = 1[L(G) cap C_{x+D} != empty], masked runs
 * read as Sigma*), and then chooses the relaxed compatible subset of the
 * valid proposals to commit together (Sec. 4.3, Alg. 4).
 *
 * Conventions for every call:
 *  - Pointers named d_* are device pointers (HIP device memory, e.g. PyTorch
 *    tensors); all other pointers are host pointers.  Host data is copied
 *    before the call returns; the caller keeps ownership of everything it
 *    passes in.
 *  - Device work is enqueued on `stream` and the call returns without
 *    waiting; outputs are valid after the stream is synchronised.
 *  - A context is used by one host thread at a time; distinct contexts are
 *    independent.  Calls on one context that overlap on different streams
 *    must not share a workspace.
 *  - Errors detectable on the host are returned immediately as a negative
 *    epic_status and nothing is enqueued.  Errors that only the device can
 *    see mark the affected candidate (verdict 2) and set a sticky device flag
 *    that epic_ctx_device_error() reads after synchronising.
 */
#ifndef EPIC_H
#define EPIC_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  EPIC_OK = 0,
  EPIC_ERR_NULL = -1,        /* a required pointer is NULL */
  EPIC_ERR_ARG = -2,         /* a size or index argument is out of range */
  EPIC_ERR_CAPACITY = -3,    /* larger than the context or workspace was sized for */
  EPIC_ERR_LEXER = -4,       /* lexer DFA malformed (start accepts, not trim, bad label) */
  EPIC_ERR_GRAMMAR = -5,     /* undefined symbol, start not a nonterminal, too large */
  EPIC_ERR_VOCAB = -6,       /* token empty or longer than 8 bytes */
  EPIC_ERR_HIP = -7,         /* a HIP runtime call failed */
  EPIC_ERR_STATE = -8,       /* memo not built yet */
  EPIC_ERR_UNSUPPORTED = -9  /* outside the sizes the library supports (see below) */
} epic_status;

/* Device-side sticky error bits, read by epic_ctx_device_error(). */
#define EPIC_DEV_BAD_CANDIDATE 1u  /* position not masked, token/sequence/position out of range */
#define EPIC_DEV_CAPACITY 2u       /* a chart or graph buffer overflowed: verdict 2 written */
#define EPIC_DEV_BAD_SELECT 4u     /* duplicate positions or NaN confidence among valid candidates */
/* With EPIC_DEV_CAPACITY, bit 8+i names the buffer that overflowed: i = 1 chart
 * slots of one row, 2 slot hash, 3 row tasks, 4 chart entries, 5 graph nodes,
 * 6 in-edges of a node, 7 frontier, 8 emission events. */

typedef struct epic_ctx epic_ctx;

/* Lexer DFA: the compiled lexical map (Alg. 1 "compile the lexical map").
 * States 0..num_states-1, state 0 is the start state and must not accept;
 * every state must reach an accepting state (trim).  trans[q*256 + byte] is
 * the successor or -1.  accept[q] is -1 (not accepting), -2 (a skip lexeme
 * such as whitespace) or a grammar terminal id.  Lexing is greedy with one
 * byte of lookahead and no backtracking: a lexeme ends when the next byte has
 * no transition; the earlier-listed rule already decided the label.
 * Supported: num_states <= 256. */
typedef struct {
  int32_t num_states;
  const int16_t* trans;
  const int16_t* accept;
} epic_lexer_desc;

/* Grammar G = (V, Sigma_lex, P, S) (Sec. 3).  Terminals are 0..T-1,
 * nonterminals T..T+N-1; production p is lhs[p] -> rhs[rhs_offsets[p] ..
 * rhs_offsets[p+1]).  Empty right-hand sides are allowed.
 * Supported: T <= 63, N <= 64, at most 512 dotted items (sum of |rhs|+1,
 * plus two for the augmented start production). */
typedef struct {
  int32_t num_terminals, num_nonterminals, start, num_productions;
  const int32_t* lhs;
  const int32_t* rhs_offsets;
  const int32_t* rhs;
} epic_grammar_desc;

/* Tokenizer vocabulary Gamma: token t has bytes[offsets[t] .. offsets[t+1]),
 * 1 to 8 bytes. */
typedef struct {
  int32_t vocab_size;
  const uint8_t* bytes;
  const int32_t* offsets;
} epic_vocab_desc;

/* Create a context: validates the descriptors, builds the constant tables
 * (dotted items, prediction closure, the lexer's gap automaton reduced to its
 * left-language classes, the regular cover of App. A.2), uploads them and
 * allocates the memo table (vocab_size * num_states * 16 bytes).  max_batch,
 * max_seq_len and max_cands bound later calls (max_seq_len <= 1024).
 * *out receives the context. */
epic_status epic_ctx_create(const epic_lexer_desc* lexer, const epic_grammar_desc* grammar,
                            const epic_vocab_desc* vocab, int32_t max_batch, int32_t max_seq_len,
                            int32_t max_cands, epic_ctx** out);

void epic_ctx_destroy(epic_ctx* ctx);

/* Bytes of device workspace that epic_validate_batch,
 * epic_select_compatible and epic_commit_fallback need (the caller allocates
 * it, 256-byte aligned, and zeroes it once after allocating it).
 * Besides per-call scratch the workspace keeps, between calls, the recorded
 * walks of each sequence (its chart state at every masked run, tagged with the
 * context and the sequence walked).  A later call on the same context and
 * workspace resumes a sequence's walk at the last recorded masked run that
 * starts at or before the first token that changed.  Records of another
 * context (other tables, another process, or a context since destroyed) fail
 * the tag check and the sequence is walked from the start, as in a zeroed
 * workspace.  The tag covers the record headers, not the chart storage they
 * point into, so the caller must zero a newly allocated workspace (memory
 * that held this context's earlier workspace could otherwise carry valid
 * headers over overwritten charts) and must not modify it between calls;
 * under these two rules results do not depend on its contents, only the time
 * taken does. */
size_t epic_workspace_bytes(const epic_ctx* ctx);

/* Number of graph nodes one masked run contributes: the left-language
 * classes of the lexer's gap automaton (diagnostics; 2 for lexers whose
 * whitespace can separate any two lexemes: inside whitespace, and after
 * anything else). */
int32_t epic_gap_classes(const epic_ctx* ctx);

/* Number of 32-bit words of an item bitset (diagnostics; the productions'
 * dotted items packed so that none straddles a word, rounded up to a power
 * of two; each chart entry stores this many words). */
int32_t epic_item_words(const epic_ctx* ctx);

/* Alg. 2, lexing memoization: for every token t and lexer state q the greedy
 * lexing of t's bytes from q, without a final flush, into the context's memo
 * table.  Entry (t, q) sits at byte offset (t*num_states + q)*16:
 *   [0..1] state after the token (little-endian u16, 0xFFFF = the lexer dies)
 *   [2]    number of emissions (skip lexemes included)
 *   [3]    emission mask: bit j set when reading byte j ended a lexeme
 *   [4..11] emitted labels in order (terminal id, 0xFF = skip), unused = 0
 *   [12..15] zero.  A dead entry is all zero except bytes 0..1.
 * Enqueued on `stream`; must complete before validation reads the memo. */
epic_status epic_lexmemo_build(epic_ctx* ctx, hipStream_t stream);

/* Copy the memo table to host memory (bytes >= vocab_size*num_states*16).
 * Synchronous. */
epic_status epic_memo_export(const epic_ctx* ctx, void* host_dst, size_t bytes);

/* Validity of each proposal (Sec. 3 Valid; Alg. 3 is the recogniser):
 * verdict[c] = Valid_G(x_b, {(pos[c], tok[c])}) for b = cand_seq[c], i.e. 1
 * if x_b with token tok[c] at position pos[c] can still be completed into a
 * sentence of L(G), else 0; 2 if the candidate is malformed (sequence or
 * position out of range, position not masked in x_b, token out of range).
 * d_seqs: int32 [B*n] row-major, -1 = MASK.  d_cand_*: int32 [C].
 * d_verdict: uint8 [C].  Every candidate is judged against the same x_b.
 * d_workspace: at least epic_workspace_bytes(ctx) bytes.
 * A launch that shares prefixes carries the number of the call, by which its
 * walks wait for records of this very call: a HIP graph that captured the call
 * repeats the number, so it must not be replayed on other sequences
 * (epic_validate_batch_noalloc can be). */
epic_status epic_validate_batch(epic_ctx* ctx, const int32_t* d_seqs, int32_t B, int32_t n,
                                const int32_t* d_cand_seq, const int32_t* d_cand_pos,
                                const int32_t* d_cand_tok, int32_t C, uint8_t* d_verdict,
                                void* d_workspace, size_t workspace_bytes, hipStream_t stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, serving loops that must not allocate, harnesses that forbid
 * hipMalloc): epic_validate_batch without a workspace.  The verdicts are
 * epic_validate_batch's.  The walks keep their charts in a scratch array of
 * 256 MiB that the library holds in device memory, one per GPU, from the
 * first context created on that GPU until the process ends; the call itself
 * calls no hipMalloc, hipFree or other allocating routine.  Every call on a
 * GPU shares that GPU's array, so calls that overlap on one GPU (other
 * streams, contexts or host threads) race: the caller serialises them.
 * Nothing in the array must start at zero (a walk writes every chart row
 * before reading it, and nothing is kept between calls: no prefix sharing,
 * no walk records).  As many walks run at once as chart slots of the
 * context fit in the array (at most 1024); EPIC_ERR_CAPACITY when not even
 * one fits (the slot size grows with the context's max_seq_len and item
 * words: about 11 MB for 16-word items at 256 or more tokens). */
epic_status epic_validate_batch_noalloc(epic_ctx* ctx, const int32_t* d_seqs, int32_t B, int32_t n,
                                        const int32_t* d_cand_seq, const int32_t* d_cand_pos,
                                        const int32_t* d_cand_tok, int32_t C, uint8_t* d_verdict,
                                        hipStream_t stream);

/* Relaxed compatible-subset selection (Alg. 4): per sequence, the candidates
 * with verdict 1 are sorted by descending confidence (float32, ties to the
 * lower candidate index) and passed to RelaxedSelect followed by
 * ExactShrink; halves put the first ceil(|C|/2) candidates on the
 * high-confidence side.  The relaxed check is the emptiness test of the
 * regular cover intersected with the completion automaton (App. A.2);
 * the exact check is Valid.  d_selected: uint8 [C], 1 = in the returned
 * subset B (empty, or at least two candidates whose joint application is
 * exactly valid).  A sequence whose verdict-1 candidates repeat a position or
 * carry a NaN confidence selects nothing and sets EPIC_DEV_BAD_SELECT; one
 * with more than 64 verdict-1 candidates selects nothing and sets
 * EPIC_DEV_CAPACITY; a verdict-1 candidate that is not a legal update sets
 * EPIC_DEV_BAD_CANDIDATE.
 * d_counts (optional, device int64 [2]) accumulates the number of cover and
 * exact checks Alg. 4 calls.  Some calls are answered without a walk: a
 * repeated check, or one an answered check decides (a pass carries to
 * subsets, a failure to supersets, an exact pass to the cover check, a cover
 * failure to the exact check); the answer is the one the walk would give. */
epic_status epic_select_compatible(epic_ctx* ctx, const int32_t* d_seqs, int32_t B, int32_t n,
                                   const int32_t* d_cand_seq, const int32_t* d_cand_pos,
                                   const int32_t* d_cand_tok, const float* d_conf,
                                   const uint8_t* d_verdict, int32_t C, uint8_t* d_selected,
                                   int64_t* d_counts, void* d_workspace, size_t workspace_bytes,
                                   hipStream_t stream);

/* The sequential fallback that follows the relaxed batch in EPIC decoding
 * (App. C.1: Alg. 1 and the paragraph after it): per sequence b,
 * with the selected set B (d_selected, as written by epic_select_compatible)
 * committed to x_b, the other candidates of b are taken by descending
 * confidence (float32, ties to the lower candidate index); each is committed
 * when x_b + (everything committed so far) + c is valid (Sec. 3 Valid), until
 * d_num_commit[b] - |B| more are committed (n_t of the step) or the
 * candidates run out.  Candidates with verdict != 1 are never committed: a
 * candidate invalid on x_b stays invalid once more masked positions are
 * filled.  d_num_commit: device int32 [B].  d_accepted: uint8 [C], 1 = the
 * fallback committed the candidate (B's candidates and the others 0); the
 * caller applies B and the accepted candidates to x.  Inputs are not
 * modified.  The same input rules as epic_select_compatible apply: a sequence
 * whose verdict-1 candidates repeat a position or carry a NaN confidence, or
 * number more than 64, commits nothing and sets the corresponding flag. */
epic_status epic_commit_fallback(epic_ctx* ctx, const int32_t* d_seqs, int32_t B, int32_t n,
                                 const int32_t* d_cand_seq, const int32_t* d_cand_pos, const int32_t* d_cand_tok,
                                 const float* d_conf, const uint8_t* d_verdict, const uint8_t* d_selected,
                                 const int32_t* d_num_commit, int32_t C, uint8_t* d_accepted, void* d_workspace,
                                 size_t workspace_bytes, hipStream_t stream);

/* Synchronise `stream`, then read and clear the sticky device error bits
 * (EPIC_DEV_*) into *flags. */
epic_status epic_ctx_device_error(epic_ctx* ctx, hipStream_t stream, uint32_t* flags);

/* Diagnostics: synchronise `stream`, then read and clear the work counters
 * accumulated by all walks since the last call: out[0] graph walks (one per
 * validity or cover check), out[1] chart entries written (origin slots of
 * Earley rows: 4*W bytes of items for W item words and a 4-byte origin),
 * out[2] memo entries read (16 bytes each), out[3] graph nodes built, out[4]
 * chart entries pulled by completion and scan steps (items and origin read),
 * out[5] of those, entries with an item that advanced. */
epic_status epic_ctx_work_counters(epic_ctx* ctx, hipStream_t stream, int64_t* out);

/* Diagnostics: per-kernel timing.  With enable != 0, every kernel the
 * context launches from then on is bracketed by two HIP events recorded on the
 * stream it is launched on (the events cost a few microseconds per launch).
 * Off by default. */
epic_status epic_ctx_set_timing(epic_ctx* ctx, int32_t enable);

/* Witness extraction (failure recovery, Sec. 4): how much of the search
 * state lives in LDS rather than in the witness workspace.  The back-trace
 * indexes up to max_proofs proofs in LDS, then moves its proof index to the
 * workspace for the rest of that sequence's search (0: the workspace's index
 * from the start); the byte search keeps a masked run's visited set in LDS
 * when it fits in max_vis_words 32-bit words, else in the workspace.  Where
 * they live changes only the speed, not which completions can be found.
 * 0 <= max_proofs <= 8192 and 0 <= max_vis_words <= 4096 (the defaults are
 * the maxima), else EPIC_ERR_ARG and the settings are unchanged.  Applies to
 * later epic_witness calls on the context. */
epic_status epic_ctx_set_witness_lds(epic_ctx* ctx, int32_t max_proofs, int32_t max_vis_words);

/* Diagnostics: synchronise `stream`, then read and clear, per kernel kind k
 * (0 lexing memo, 1 base walks of prefix sharing, 2 candidate walks of
 * validation, 3 selection (the walks it used: its own, and the helpers'
 * speculated walks whose results it took or drew an answer from),
 * 4 sequential fallback, 5 speculation bookkeeping (state clear, work
 * accounting), 6 speculated checks whose results the selection did not take
 * (no launches of their own, their time is the selection's)): ms[k]
 * the summed event durations of its timed launches, launches[k] their
 * number, work[k*6 .. k*6+5] the work counters of its walks (as
 * epic_ctx_work_counters).  Host arrays of 7, 7 and 42 elements. */
epic_status epic_ctx_kernel_stats(epic_ctx* ctx, hipStream_t stream, double* ms, int64_t* launches, int64_t* work);

/* Witness extraction for failure recovery (Sec. 4): when decoding stops
 * early, the output is completed from a witness of the current partial
 * sequence, which is completable because every committed update was checked.
 * For each sequence b of d_seqs (int32 [B*n], -1 = MASK), d_status[b]
 * (int32) is 1 when x_b is valid and a completion was found, 0 when x_b is
 * not valid, -1 when a token is out of range (EPIC_DEV_BAD_CANDIDATE), -2
 * when a buffer is too small (the witness workspace, bytes_per_seq or
 * max_gaps; EPIC_DEV_CAPACITY), -3 when no completion was found (not expected
 * for a valid x_b).  With status 1, d_gap_len[b*max_gaps + j] (int32) is the
 * number of bytes that fill the j-th maximal masked run of x_b, and
 * d_bytes[b*bytes_per_seq ..] holds the bytes of the runs in order: x_b with
 * every run replaced by its bytes lexes into a sentence of L(G).  A masked
 * run reads any byte string (the paper's over-approximation of masked
 * regions), so a filling is a byte string, not a number of tokens.
 * d_witness_ws: device memory of epic_witness_workspace_bytes(ctx, B) bytes,
 * 256-byte aligned, owned by the caller; d_workspace is the context's
 * workspace (its chart slots hold the walks).  B may not exceed the walk
 * slots of the context (min(max(max_cands, max_batch), 1024)):
 * EPIC_ERR_CAPACITY.  Asynchronous on stream. */
size_t epic_witness_workspace_bytes(const epic_ctx* ctx, int32_t B);
epic_status epic_witness(epic_ctx* ctx, const int32_t* d_seqs, int32_t B, int32_t n, uint8_t* d_bytes,
                         int32_t bytes_per_seq, int32_t* d_gap_len, int32_t max_gaps, int32_t* d_status,
                         void* d_witness_ws, size_t witness_ws_bytes, void* d_workspace, size_t workspace_bytes,
                         hipStream_t stream);

/* Diagnostics: LDS streaming microbenchmark, the measurement behind the LDS
 * peak that walk kernels are compared with.  Launches `blocks` workgroups of
 * `threads` threads (a multiple of 64, at most 1024) on `stream`; each
 * workgroup fills 64 KiB of LDS, then every thread reads `iters` 16-byte
 * vectors from it at consecutive addresses (no bank conflicts), so the
 * launch reads blocks * threads * iters * 16 bytes of LDS.  d_sink: device
 * uint32 [8]; workgroup 0's thread 0 writes the shader-clock ticks (sink[2],
 * sink[3]: low, high word) and the constant-rate wall-clock ticks (sink[4],
 * sink[5]) it measured around its read loop; the caller times the launch
 * with events on the same stream.  Returns EPIC_ERR_ARG for sizes out of
 * range. */
epic_status epic_diag_lds_stream(int32_t blocks, int32_t threads, int32_t iters, uint32_t* d_sink,
                                 hipStream_t stream);

/* Shader-clock and wall-clock rates of the current device in kHz (as the
 * runtime reports them), for epic_diag_lds_stream's tick counts. */
epic_status epic_diag_clock_rates(int32_t* shader_khz, int32_t* wall_khz);

/* ---- What comes before and around the check: logits rows ----------------
 *
 * A denoiser answers with logits.  The three operators below make proposals of
 * them (epic_sample, epic_propose) and train the denoiser on a teacher's
 * (epic_distill_*).  They need no context: they know nothing of the grammar.
 *
 * Rows.  Row (b, i), 0 <= b < batch and 0 <= i < rows, holds the `vocab` logits
 * of sequence b at position start[b] + i of its n tokens, elements
 * data[b*seq_stride + i*row_stride + 0 .. vocab): a window of `rows` positions
 * per sequence (the active block in block decoding).  d_start (int32 [batch])
 * NULL: every window starts at position 0.  A row counts when its position is
 * inside the sequence and masked there (d_seqs int32 [batch*n], -1 = MASK);
 * with d_seqs NULL (then n and d_start are not read) every row counts.  Rows
 * that do not count are not read: they may hold anything.
 *
 * data is a device pointer aligned to its element; rows need no more alignment
 * and no particular stride (a stride of 0 repeats a row; the rows of a gradient
 * must not overlap).  1 <= vocab <= 262144, else EPIC_ERR_UNSUPPORTED; batch *
 * rows < 2^30, else EPIC_ERR_ARG (of epic_propose batch * per_seq too); offsets
 * are 64-bit.  batch * rows = 0 is no error.  The calls allocate nothing, keep
 * nothing and may be captured in a HIP graph; the same inputs give the same
 * bits, whatever else is in the batch. */
typedef enum { EPIC_F32 = 0, EPIC_F16 = 1, EPIC_BF16 = 2 } epic_dtype;

typedef struct {
  void* data;        /* device */
  int32_t dtype;     /* epic_dtype */
  int32_t batch;     /* sequences */
  int32_t rows;      /* rows per sequence */
  int32_t vocab;     /* logits per row */
  int64_t seq_stride; /* elements from a sequence's first row to the next's */
  int64_t row_stride; /* elements from a row to the next of its sequence */
} epic_rows_desc;

/* Sampling with temperature, top-k, top-p and min-p from given uniform
 * numbers: one token and its confidence for every row that counts.
 *
 * With M the row's largest logit and T its temperature, token t has
 *   x_t = (l_t - M) * c,  c = log2(e) / T rounded to float32, at most 1e30,
 *   e_t = 2^x_t,  w_t = floor(2^31 * e_t + 1/2),  a whole number; W = sum of all
 *   w_t
 * (x, e and the sum with 1/2 in float32).  Sums of whole numbers depend on no
 * order, so neither does the token drawn.  A weight is off by up to half a unit:
 * tokens below 2^-32 of the likeliest one's probability are never drawn.
 * NaN and -inf logits have w = 0 and are never drawn.
 * Tokens are ordered by descending logit, ties to the lower id.  Kept are the
 * tokens that pass all of
 *   top-k (k > 0):   the first k; S their mass (else S = W);
 *   top-p (p < 1):   the shortest prefix whose mass is at least
 *                    max(1, floor(S * floor(2^24 p) / 2^24)), p <= 0: the first;
 *   min-p (q > 0):   w_t >= floor(2^31 q + 1/2), q capped at 1.
 * With D the mass kept and U = floor(2^24 u), u the row's uniform number
 * (capped to [0, 1 - 2^-24], NaN: 0), the token is the lowest id at which the
 * kept mass up to it exceeds floor(D * U / 2^24).  Its confidence is
 * 2^31 e_t / W: its probability at that temperature before the filters.
 * T <= 0 is greedy: the first of the order, with its probability at T = 1.
 *
 * d_uniform: float32 [batch*rows].  Settings per sequence, NULL for the default:
 * d_temperature float32 [batch] (1), d_top_k int32 (off), d_top_p float32
 * (off), d_min_p float32 (off); NaN in top-p or min-p means off.
 * d_tok int32 [batch*rows], d_conf float32 [batch*rows]: -1 and 0 for a row
 * that does not count, has no finite logit, has a logit of +inf or a NaN
 * temperature.  A mask of the type's lowest finite value is a finite logit:
 * beside an ordinary one its weight is 0, a row of nothing else is uniform. */
epic_status epic_sample(const epic_rows_desc* logits, const int32_t* d_seqs, int32_t n, const int32_t* d_start,
                        const float* d_uniform, const float* d_temperature, const int32_t* d_top_k,
                        const float* d_top_p, const float* d_min_p, int32_t* d_tok, float* d_conf,
                        hipStream_t stream);

/* Proposals of a step from sampled tokens: of each sequence the per_seq most
 * confident rows (float32, descending, ties to the lower row) that have a
 * token, as the candidate arrays that epic_validate_batch,
 * epic_select_compatible and epic_commit_fallback read.
 * d_tok int32 and d_conf float32 [batch*rows] as epic_sample writes them; a
 * row with a token below 0 or a NaN confidence is no proposal.  d_start as
 * above, or NULL.  1 <= per_seq <= 64 (what selection takes of a sequence).
 * Sequence b's candidates are d_cand_*[d_offsets[b] .. d_offsets[b+1]), most
 * confident first, position = d_start[b] + row; d_offsets int32 [batch+1]
 * starts at 0, and d_offsets[batch] is the C of the calls that follow.  The
 * arrays hold batch*per_seq entries; those past the last candidate are set to
 * -1 (confidence 0). */
epic_status epic_propose(const int32_t* d_tok, const float* d_conf, int32_t batch, int32_t rows,
                         const int32_t* d_start, int32_t per_seq, int32_t* d_cand_seq, int32_t* d_cand_pos,
                         int32_t* d_cand_tok, float* d_cand_conf, int32_t* d_offsets, hipStream_t stream);

/* Distillation from a teacher's top logits: the divergence of the student's
 * rows from the teacher, which is known by K entries (id, logit) per row.
 * With z = l / tau the student's scaled logits, S the set of the row's listed
 * ids and t_k the teacher's logits:
 *   with d_teacher_lse (float32 [batch*rows], the teacher's logsumexp of t /
 *   tau over its whole vocabulary): q_k = exp(t_k/tau - lse_T), and
 *   q_rest = max(0, 1 - sum q_k) is what the teacher leaves to the rest;
 *   without (NULL): q = softmax of t / tau over the entries, q_rest = 0.
 *   lse_rest = log sum_{j not in S} exp(z_j), lse = log sum_j exp(z_j),
 *   p = exp(z - lse), p_rest = exp(lse_rest - lse),
 *   loss = tau^2 (sum_k q_k (log q_k - log p_k) + q_rest (log q_rest - log p_rest)),
 *   d loss / d l_j = tau (p_j - q_j) for j in S (q_j: the sum of j's entries),
 *                    tau exp(z_j - lse_rest) (p_rest - q_rest) for the others.
 * An entry with a negative id is absent; an entry of logit -inf is listed with
 * q = 0.  When every finite logit of the row is listed, q_rest counts as 0.  A
 * row that does not count, whose student logits are all -inf, or that has no
 * entry (without d_teacher_lse: none but -inf) has loss 0 and gradient 0; an id
 * >= vocab gives loss NaN and gradient 0.  NaN and +inf elsewhere among the
 * student's logits, the entries' and d_teacher_lse give NaN.  z and t / tau are
 * float32: a logit whose quotient is not finite there counts as that infinity.
 * Exponentials below 2^-126 may count as 0.
 *
 * d_top_idx int32 and d_top_logit float32 [batch*rows*K], 1 <= K <= 1024, ids
 * in any order; 0 < tau < inf with log2(e) / tau finite in float32 (tau > 4.24e-39),
 * else EPIC_ERR_ARG.  d_loss float32 [batch*rows].  d_stats float32
 * [batch*rows*2] receives lse and lse_rest of each row for the backward pass.
 * Gradients: grad (its data, of the logits' type and shape, strides of its
 * own, rounded to nearest even from float32) receives weight[row] times the
 * derivative above for every row (0 in rows that do not count); it may be the
 * logits themselves (the same data and strides), but not otherwise overlap
 * them.  d_weight float32 [batch*rows]: the upstream gradient of each row's
 * loss (NULL: 1).
 * epic_distill_forward writes losses and stats and, when grad is not NULL, the
 * gradient with one reading of the logits.  epic_distill_backward writes the
 * gradient from the stats of an earlier forward pass over the same inputs. */
epic_status epic_distill_forward(const epic_rows_desc* logits, const int32_t* d_seqs, int32_t n,
                                 const int32_t* d_start, const int32_t* d_top_idx, const float* d_top_logit, int32_t K,
                                 const float* d_teacher_lse, float tau, float* d_loss, float* d_stats,
                                 const float* d_weight, const epic_rows_desc* grad, hipStream_t stream);
epic_status epic_distill_backward(const epic_rows_desc* logits, const int32_t* d_seqs, int32_t n,
                                  const int32_t* d_start, const int32_t* d_top_idx, const float* d_top_logit,
                                  int32_t K, const float* d_teacher_lse, float tau, const float* d_stats,
                                  const float* d_weight, const epic_rows_desc* grad, hipStream_t stream);

const char* epic_status_string(epic_status s);

#ifdef __cplusplus
}
#endif

#endif /* EPIC_H */
