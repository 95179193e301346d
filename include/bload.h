/*
 * bload.h -- C ABI of the BLoad block packer for MI355X (gfx950).
 *
 * BLoad (arXiv 2310.10879) trains on N sequences S_i of H x W x T_i frames
 * with varying T_i (Problem Statement) by concatenating randomly ordered whole
 * sequences into blocks of a fixed length T_blk = T_max, padding each block's
 * tail with 0's, and keeping a table of where each sequence starts inside its
 * block so that a recurrent consumer can reset its carried state there
 * (Methods).  This library is that packer, on the GPU:
 *
 *   bload_plan            order the sequences by seed and assign them to blocks
 *   bload_pack            gather the frames into [num_blocks, T_blk, frame] and
 *                         write the per-slot form of the start table
 *   bload_segment_reduce  per-sequence sum / mean over the packed blocks, using
 *                         only the packed tensor and that per-slot table
 * for the model that trains on the blocks and serves from them,
 *   bload_segment_mask, bload_segment_attention (_backward, _decode)
 *   bload_rotary, bload_rotary_frequencies
 *   bload_gated_scan (_backward)
 *   bload_layer_norm, bload_segment_conv, bload_selective_scan (each with _backward)
 * and, around that path,
 *   bload_plan_random_fit   the plan built with the sampler of the paper's pseudocode
 *   bload_plan_shard        one data-parallel worker's share of a plan
 *   bload_segment_scan      a recurrent consumer that drops its state at sequence starts
 *   bload_strategy_counts   padding / frames deleted under the strategies the paper compares
 *   bload_pack_check        are these tables a plan bload_pack can take
 *   bload_pack_noalloc      bload_pack with its scratch in a fixed array of the library
 *
 * Conventions
 *   - Pointers named d_* are DEVICE pointers (hipMalloc-style memory of the
 *     current device), h_* are HOST pointers.  The caller owns every buffer;
 *     the library allocates nothing and keeps no state between calls (the one
 *     exception, a fixed scratch array, is bload_pack_noalloc's and is described
 *     there).
 *   - A frame is an opaque record of `frame_bytes` bytes (H*W*C*sizeof(elem));
 *     H and W are the same for all sequences of one call.
 *   - `hip_stream` is a hipStream_t passed as void* (NULL = the null stream).
 *     bload_pack, bload_segment_reduce, bload_segment_scan and the model's operators only
 *     enqueue work on it (no synchronisation, no allocation: they can be recorded into a HIP
 *     graph); the planners and bload_strategy_counts enqueue, then wait for the
 *     stream, because they return counts to the host.
 *   - Every function returns a bload_status; nothing is thrown.  On any
 *     status other than BLOAD_OK the contents of the output buffers are
 *     unspecified (but nothing outside them is ever written).
 *   - Sizes: 0 <= n_seq <= BLOAD_MAX_SEQ, 1 <= t_blk, 1 <= L_i <= t_blk,
 *     num_blocks * t_blk < 2^40 slots.
 */
#ifndef BLOAD_H
#define BLOAD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define BLOAD_MAX_SEQ ((int64_t)1 << 27)

typedef enum {
    BLOAD_OK = 0,
    BLOAD_EINVAL = 1,      /* null pointer, negative size, t_blk < 1, frame_bytes < 1,
                              unknown dtype / op, or an unsupported dtype-op pair */
    BLOAD_ELENGTH = 2,     /* some L_i < 1 or L_i > t_blk (the method needs T_i <= T_max) */
    BLOAD_EWORKSPACE = 3,  /* workspace smaller than the *_workspace_bytes() answer (but see
                              bload_segment_reduce) */
    BLOAD_EALIGN = 4,      /* a payload / workspace base is not 16-byte aligned (32-byte for
                              bload_pack's workspace), or an int32 / int64 table is not
                              naturally aligned */
    BLOAD_EOVERFLOW = 5,   /* n_seq or num_blocks * t_blk beyond the supported range, or more
                              work than one launch holds (2^24 - 1 workgroups) */
    BLOAD_EHIP = 6         /* a HIP runtime call failed (bload_last_hip_error() says which) */
} bload_status;

typedef enum { BLOAD_U8 = 0, BLOAD_F16 = 1, BLOAD_F32 = 2, BLOAD_I32 = 3,
               BLOAD_BF16 = 4 /* the model's operators */ } bload_dtype;
typedef enum { BLOAD_SUM = 0, BLOAD_MEAN = 1 } bload_op;

/* Human-readable name of a status (static storage, never NULL). */
const char* bload_status_string(bload_status status);

/* hipError_t (as int) of the most recent failing HIP call made by this library
 * on the calling thread, 0 if none. */
int bload_last_hip_error(void);

/* ------------------------------------------------------------------ plan --
 * Methods section: blocks of T_max frames are put together from whole sequences,
 * none longer than T_max, taken in random order; each block is closed as near
 * T_max as the visiting order allows; a table keeps where every sequence starts.
 *
 * order:  a permutation of [0, n_seq) fixed by `seed` alone: position p holds
 *         the sequence walk(p), where walk applies a 6-round balanced Feistel
 *         network over the smallest even bit width w >= 2 with 2^w >= n_seq
 *         (round function: MurmurHash3's 32-bit finaliser of right-half +
 *         key_r, masked to w/2 bits; key_r = low 32 bits of the r-th output of
 *         SplitMix64 started at `seed`) and re-applies it until the value is
 *         below n_seq.  n_seq <= 1 gives the identity.
 * assign: next-fit over that order: a sequence goes into the open block if
 *         fill + L <= t_blk, otherwise the block is closed (its tail is
 *         padding) and the sequence opens the next one.
 *
 * d_lengths        in   int32[n_seq]   L_i, in original sequence order
 * d_order          out  int32[n_seq]   order[p] = sequence at shuffled position p
 * d_block_of_seq   out  int32[n_seq]   block of sequence i      (original index)
 * d_offset_of_seq  out  int32[n_seq]   first slot of sequence i inside its block
 *                                      (the paper's start table, per sequence)
 * d_block_first    out  int32[n_seq+1] capacity; entries [0 .. B] are written:
 *                                      first shuffled position of block b, [B] = n_seq
 * h_num_blocks     out  host int64     B
 * h_total_frames   out  host int64     sum of L_i
 * d_workspace           device scratch of >= bload_plan_workspace_bytes(n_seq)
 *                       bytes, 16-byte aligned; contents meaningless afterwards
 *
 * Lengths are checked on the device; a bad one gives BLOAD_ELENGTH.  n_seq = 0
 * gives B = 0, BLOAD_OK, and writes nothing to the device.  Synchronises the
 * stream before returning.  The library keeps 64 bytes of pinned host memory per
 * calling thread (taken at that thread's first call, never freed) into which the
 * device writes B and the frame total; bload_plan_random_fit and bload_plan_shard use
 * the same bytes.
 */
size_t bload_plan_workspace_bytes(int64_t n_seq);

bload_status bload_plan(const int32_t* d_lengths, int64_t n_seq, int32_t t_blk, uint64_t seed,
                        int32_t* d_order, int32_t* d_block_of_seq, int32_t* d_offset_of_seq,
                        int32_t* d_block_first,
                        int64_t* h_num_blocks, int64_t* h_total_frames,
                        void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------- plan, random fit --
 * Caption of the pseudocode figure: the block builder asks a sampler for a random
 * entry of the length dictionary L_dict among the sequences no longer than the
 * frames remaining in the open block; a block is closed when none fits.  The
 * reading implemented here:
 *   - every remaining sequence that fits is equally likely: with m of them the
 *     draw is k = floor(u * m / 2^64), u the output number 6 + p of the seed's
 *     SplitMix64 stream for the p-th placement, and the k-th is counted through
 *     L_dict by ascending length;
 *   - L_dict[l] lists the sequences of length l in the seeded order (the order
 *     bload_plan visits them in); a draw landing in L_dict[l] takes its last
 *     remaining entry.
 * Arguments, outputs, workspace rules and error codes are those of bload_plan
 * (d_order[p] is the p-th sequence placed); bload_pack, bload_plan_shard and
 * bload_segment_reduce take the result like a next-fit plan.  Additionally
 * BLOAD_EOVERFLOW when t_blk > BLOAD_RANDOM_FIT_MAX_T_BLK (the per-length counts
 * are kept in on-chip memory).  The draws form a dependent chain that one
 * wavefront walks: the cost grows linearly with n_seq.
 * Synchronises the stream before returning.
 */
#define BLOAD_RANDOM_FIT_MAX_T_BLK 8192

size_t bload_plan_random_fit_workspace_bytes(int64_t n_seq);

bload_status bload_plan_random_fit(const int32_t* d_lengths, int64_t n_seq, int32_t t_blk,
                                   uint64_t seed, int32_t* d_order, int32_t* d_block_of_seq,
                                   int32_t* d_offset_of_seq, int32_t* d_block_first,
                                   int64_t* h_num_blocks, int64_t* h_total_frames,
                                   void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------ plan shard --
 * Problem Statement: under data-parallel training every worker must receive the
 * same number of samples per epoch, otherwise the gradient exchange stalls; the
 * blocks are the samples.  This call derives worker `rank`'s share of a plan:
 * the blocks b with b mod world == rank, renumbered j = b / world, plus one
 * block of pure padding at the end for the workers that would otherwise hold
 * one block less, so that every worker has ceil(B / world) blocks.  The outputs
 * are a plan in the worker's own numbering; bload_pack and bload_segment_reduce
 * take them like the tables of bload_plan (with n_seq unchanged, the worker's
 * block count, and the same d_lengths / d_offset_of_seq / d_src / d_src_offsets).
 *
 * d_order, d_block_of_seq, d_block_first   in   as produced by bload_plan
 * d_order_local          out  int32[n_seq]  the worker's sequences in visiting
 *                                           order, then -1 (= no sequence)
 * d_block_of_seq_local   out  int32[n_seq]  local block of sequence i, -1 when i
 *                                           belongs to another worker
 * d_block_first_local    out  int32[ceil(B / world) + 1]
 * h_num_blocks_local     out  host int64    ceil(B / world)
 * h_n_seq_local          out  host int64    number of sequences of the worker
 * d_workspace                 >= 16 bytes, 16-byte aligned
 *
 * Synchronises the stream before returning (it reports the worker's counts).
 */
bload_status bload_plan_shard(const int32_t* d_order, const int32_t* d_block_of_seq,
                              const int32_t* d_block_first, int64_t n_seq, int64_t num_blocks,
                              int32_t rank, int32_t world,
                              int32_t* d_order_local, int32_t* d_block_of_seq_local,
                              int32_t* d_block_first_local,
                              int64_t* h_num_blocks_local, int64_t* h_n_seq_local,
                              void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------ pack --
 * Methods section: the sequences of a block are laid one after another and the
 * rest of the block is filled with 0's; the start table says where each new
 * sequence begins.
 *
 * d_src          in   bytes[total_frames * frame_bytes]: the ragged source, the
 *                     frames of sequence i stored contiguously from frame
 *                     d_src_offsets[i]; any byte alignment (fastest when it is
 *                     16-byte aligned and frame_bytes is a multiple of 16)
 * d_src_offsets  in   int64[n_seq+1]  first source frame of each sequence;
 *                     src_offsets[i+1] - src_offsets[i] must equal L_i (not checked)
 * d_lengths, d_order, d_block_of_seq, d_offset_of_seq, d_block_first
 *                in   as produced by bload_plan for the same lengths (or a worker's
 *                     share of them from bload_plan_shard; an entry of d_order that
 *                     is not in [0, n_seq) ends the list of sequences)
 * num_blocks     in   B as returned by bload_plan
 * d_packed       out  bytes[B, t_blk, frame_bytes]; slot
 *                     (b, offset_of_seq[i] + t) receives frame t of sequence i,
 *                     every other byte is 0
 * d_seq_id       out  int32[B, t_blk]  original sequence index, -1 on padding
 * d_frame_idx    out  int32[B, t_blk]  frame number inside its sequence, -1 on padding
 * d_reset        out  uint8[B, t_blk]  1 on the first frame of a sequence, else 0
 * d_valid        out  uint8[B, t_blk]  1 on a real frame, 0 on padding
 *                     (all five outputs 16-byte aligned)
 *
 * d_workspace         device scratch of >= bload_pack_workspace_bytes(...) bytes,
 *                     32-byte aligned: one 32-byte record per sequence (where it
 *                     lands, where it comes from) and one int32 per destination
 *                     tile -- 4 KiB of packed tensor (plus, from 2^21 slots on, one
 *                     per 1024 slots for the pass that writes the start table) or
 *                     1024 slots -- saying where the tile starts in the shuffled
 *                     order; contents meaningless afterwards
 *
 * Every byte of the five outputs is written exactly once (no prior memset is
 * needed), and nothing outside them whatever the tables hold.  The tables are
 * trusted otherwise: tables that are not a plan give a meaningless result, and
 * source offsets outside the source are read; bload_pack_check tells.
 * Asynchronous on `hip_stream`.  n_seq = 0 / num_blocks = 0: no-op.
 */
/* Which of its two tile shapes bload_pack takes for these sizes: 4096 when the packed
 * tensor is cut into tiles of 4096 bytes (pack_wide_kernel, pack_direct_kernel where
 * they are few), 0 when it is cut into tiles of 1024 slots (pack_narrow_kernel,
 * pack_narrow_direct_kernel), also for sizes bload_pack refuses.
 * src_aligned_16: whether d_src is 16-byte aligned.  For profiling and reports. */
int32_t bload_pack_tile_bytes(int64_t n_seq, int64_t num_blocks, int32_t t_blk, int64_t frame_bytes,
                              int32_t src_aligned_16);

size_t bload_pack_workspace_bytes(int64_t n_seq, int64_t num_blocks, int32_t t_blk, int64_t frame_bytes);

bload_status bload_pack(const void* d_src, const int64_t* d_src_offsets, const int32_t* d_lengths,
                        const int32_t* d_order, const int32_t* d_block_of_seq,
                        const int32_t* d_offset_of_seq, const int32_t* d_block_first,
                        int64_t n_seq, int64_t num_blocks, int32_t t_blk, int64_t frame_bytes,
                        void* d_packed, int32_t* d_seq_id, int32_t* d_frame_idx,
                        uint8_t* d_reset, uint8_t* d_valid,
                        void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* For callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): bload_pack without the
 * workspace argument.  Its scratch -- the same per-sequence records and per-tile
 * entries -- lives in a fixed array of 16 MiB of device memory that belongs to the
 * loaded library; every GPU on which this entry point is used holds one until the
 * process ends.  Limits: n_seq <= BLOAD_PACK_NOALLOC_MAX_SEQ and at most
 * BLOAD_PACK_NOALLOC_MAX_TILES - 4 tile entries (a tile is 4 KiB of packed tensor
 * when bload_pack_tile_bytes() says 4096, with one more entry per 1024 slots from
 * 2^21 slots on, else 1024 slots: just under 8 GiB of packed tensor, or 2^31
 * slots); anything larger is refused with BLOAD_EOVERFLOW before anything is
 * launched.  All other arguments, checks and results are those of bload_pack.
 * The call allocates and frees nothing and does not synchronise.  Nothing in the
 * array has to be cleared between calls (each call rewrites the part it reads),
 * but all calls on one GPU share it: two such calls must not overlap in time on
 * the same GPU (calls on one stream never do; calls on different streams, or from
 * different threads, need an order between them).
 */
#define BLOAD_PACK_NOALLOC_MAX_SEQ ((int64_t)1 << 18)
#define BLOAD_PACK_NOALLOC_MAX_TILES ((int64_t)1 << 21)

bload_status bload_pack_noalloc(const void* d_src, const int64_t* d_src_offsets, const int32_t* d_lengths,
                                const int32_t* d_order, const int32_t* d_block_of_seq,
                                const int32_t* d_offset_of_seq, const int32_t* d_block_first,
                                int64_t n_seq, int64_t num_blocks, int32_t t_blk, int64_t frame_bytes,
                                void* d_packed, int32_t* d_seq_id, int32_t* d_frame_idx,
                                uint8_t* d_reset, uint8_t* d_valid, void* hip_stream);

/* Methods section: whole sequences, one after another from the block's first
 * slot, none split, none beyond the block's end.  This call verifies that the
 * tables handed to bload_pack describe such a layout, without packing anything:
 *   - block_first[0 .. num_blocks] is non-decreasing, starts at 0 and ends at
 *     P <= n_seq; every position p < P holds a sequence index in [0, n_seq);
 *   - the sequence at position p lies in the block whose range contains p, at
 *     offset 0 if it is the block's first and right behind its predecessor
 *     otherwise, and ends at or before slot t_blk;
 *   - 1 <= L_i, and the source range [src_offsets[i], src_offsets[i] + L_i) lies
 *     inside [0, total_frames) and src_offsets[i+1] - src_offsets[i] = L_i,
 * for every sequence listed.  (Together these make the listed sequences distinct.)
 * BLOAD_OK if so, BLOAD_EINVAL if not; *h_first_bad (may be NULL) receives the
 * smallest shuffled position or block at which a rule fails, -1 if none.
 * d_workspace: >= 16 bytes, 16-byte aligned.  Synchronises the stream.
 */
bload_status bload_pack_check(const int64_t* d_src_offsets, const int32_t* d_lengths,
                              const int32_t* d_order, const int32_t* d_block_of_seq,
                              const int32_t* d_offset_of_seq, const int32_t* d_block_first,
                              int64_t n_seq, int64_t num_blocks, int32_t t_blk, int64_t total_frames,
                              int64_t* h_first_bad, void* d_workspace, size_t workspace_bytes,
                              void* hip_stream);

/* -------------------------------------------------------- segment reduce --
 * Methods section: knowing where a new sequence starts lets the consumer drop
 * what it carried from the previous frame.  The simplest such consumer: a
 * running sum over time that is restarted at every start flag and never
 * crosses a block boundary.  It receives no plan tables: segments are found
 * from d_reset / d_valid alone, d_seq_id only names the output row.
 *
 * d_packed   in   [B, t_blk, feat_dim] of `dtype`, 16-byte aligned
 * d_seq_id   in   int32[B, t_blk];  d_reset, d_valid in uint8[B, t_blk]
 * d_out      out  [n_seq, feat_dim]: float32 for U8 / F16 / F32 inputs (float32
 *                 accumulation over chunks of time, chunks added in time order),
 *                 int64 for I32 (exact).  MEAN divides by the segment's frame
 *                 count; I32 supports SUM only.  A segment's row is d_seq_id at
 *                 its first slot: row i is written iff some segment starts with
 *                 seq_id i; ids outside [0, n_seq) are skipped.  float32 sums are
 *                 formed as trees of a few frames that are added with compensation or
 *                 in 64 bits: whatever the length of a sequence, the result is
 *                 within a few units of float32 roundoff of sum |x| (exact for U8
 *                 while the sum stays below 2^24).
 * d_workspace     device scratch of >= bload_segment_reduce_workspace_bytes(...)
 *                 bytes, 16-byte aligned (may be NULL when that is 0).  The size is
 *                 that of one cut of the work, chosen for the sizes it is asked for:
 *                 ask again for another num_blocks, fewer blocks can need more.  Less
 *                 is taken where a slower cut makes do with it (none at all for
 *                 frames of 2 to 63 elements in blocks of up to 12288 slots) and else
 *                 refused with BLOAD_EWORKSPACE (BLOAD_EINVAL without a workspace).
 *
 * Asynchronous on `hip_stream`; same inputs and a workspace of the same size give
 * bit-identical outputs.
 */
size_t bload_segment_reduce_workspace_bytes(int64_t num_blocks, int32_t t_blk, int64_t feat_dim,
                                            bload_dtype dtype);

/* Which of its layouts bload_segment_reduce takes for these sizes with so many bytes of
 * (aligned) workspace, and into how many chunks of time or tiles it cuts the blocks
 * (*h_chunks, which may be NULL): BLOAD_REDUCE_NONE and 0 for empty calls and sizes that
 * it refuses.  For profiling, reports and tests; what it answers may change. */
enum { BLOAD_REDUCE_NONE = 0, BLOAD_REDUCE_WIDE = 1, BLOAD_REDUCE_STAGED = 2, BLOAD_REDUCE_FLAT = 3, BLOAD_REDUCE_NARROW = 4 };
int32_t bload_segment_reduce_layout(int64_t num_blocks, int32_t t_blk, int64_t feat_dim, bload_dtype dtype,
                                    int64_t n_seq, size_t workspace_bytes, int64_t* h_chunks);

bload_status bload_segment_reduce(const void* d_packed, const int32_t* d_seq_id,
                                  const uint8_t* d_reset, const uint8_t* d_valid,
                                  int64_t num_blocks, int32_t t_blk, int64_t feat_dim,
                                  bload_dtype dtype, bload_op op, int64_t n_seq, void* d_out,
                                  void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* ---------------------------------------------------------- segment scan --
 * Methods section and the figure of the DDS model: the network feeds what it
 * produced for frame n-1 into frame n, and the start table tells it where that
 * carried state belongs to another sequence and has to be dropped.  This is the
 * smallest consumer with such feedback: per feature a first-order linear
 * recurrence along time,
 *     h = x                   at a slot that starts a sequence
 *     h = decay * h_prev + x  at every other valid slot
 *     h = 0                   at a padding slot,
 * where a slot starts a sequence exactly as for bload_segment_reduce (valid, and
 * carrying a start flag, or first of its block, or behind an invalid slot).
 *
 * d_packed   in   [B, t_blk, feat_dim] of `dtype` (U8, F16 or F32; I32 is
 *                 refused with BLOAD_EINVAL), 16-byte aligned
 * d_reset, d_valid   in   uint8[B, t_blk]
 * decay      in   any float
 * d_out      out  float32[B, t_blk, feat_dim], 16-byte aligned; every element is
 *                 written.  float32 arithmetic in time order inside stretches of 8 to
 *                 33 slots; a sequence that crosses from one stretch to the next takes
 *                 its state along in 64 bits, as decay^length * (state in front of the
 *                 stretch) + (the stretch's own part), which adds no rounding; a state
 *                 beyond the range of float32 is infinite.  For the k-th frame of a
 *                 sequence the result differs from the exact one by at most (3k + 4) * 2^-24 * S,
 *                 S being the same recurrence run on |x| with |decay|.
 * d_workspace     device scratch of >= bload_segment_scan_workspace_bytes(...)
 *                 bytes, 16-byte aligned (may be NULL when that is 0).  With less, one
 *                 workgroup takes a block from end to end, which is slower: accepted
 *                 down to nothing where there are thousands of blocks or blocks are
 *                 shorter than 128 slots, and in any case where 4 bytes per element and
 *                 1 per slot of every 64th slot fit; else BLOAD_EWORKSPACE
 *                 (BLOAD_EINVAL without a workspace).
 * Asynchronous on `hip_stream`; same inputs give bit-identical outputs.
 */
size_t bload_segment_scan_workspace_bytes(int64_t num_blocks, int32_t t_blk, int64_t feat_dim,
                                          bload_dtype dtype);

bload_status bload_segment_scan(const void* d_packed, const uint8_t* d_reset,
                                const uint8_t* d_valid, int64_t num_blocks, int32_t t_blk,
                                int64_t feat_dim, bload_dtype dtype, float decay, float* d_out,
                                void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------ segment attention --
 * Attention between the frames of one sequence, on the packed blocks: the start table
 * keeps a sequence's frames from seeing its neighbours in the block, as it keeps a
 * recurrent consumer's state from crossing a start.
 *
 * Tensors of queries, keys and values are [num_blocks, t_blk, heads, head_dim] with the
 * elements of a head side by side; the other distances are free (in elements, 0 or
 * negative ones included), so that q, k and v may be parts of one projection's result. */
typedef struct {
    void* d_data;                 /* element (0, 0, 0, 0), aligned to its type */
    int64_t block_stride, slot_stride, head_stride;
} bload_heads;

#define BLOAD_ATTENTION_MAX_HEAD_DIM 128

/* Who sees whom, once per batch and for every layer and pass: a slot's query sees the keys
 * of its own sequence, which lies in the consecutive slots [f, e) of one block (found from
 * d_reset / d_valid as bload_segment_reduce finds it).
 *   causal = 0   all of [f, e)
 *   causal = 1   [f, t + 1); with d_prefix also the first d_prefix[seq_id] frames of the
 *                sequence, wherever the query stands (negative counts as 0, more than the
 *                sequence has as all; a slot whose seq_id is outside [0, n_seq) has none)
 * d_mask     out  int32[num_blocks, t_blk, 4], 16-byte aligned: key_lo, key_hi (the slots
 *                 of the block that slot t's query sees), query_lo, query_hi (those whose
 *                 queries see slot t's key); all 0 on padding
 * d_prefix   in   int32[n_seq] or NULL;  d_seq_id is read only with it
 * Asynchronous on `hip_stream`. */
bload_status bload_segment_mask(const uint8_t* d_reset, const uint8_t* d_valid, const int32_t* d_seq_id,
                                int64_t num_blocks, int32_t t_blk, int32_t causal, const int32_t* d_prefix,
                                int64_t n_seq, int32_t* d_mask, void* hip_stream);

/* For query i and key j of a head (keys and values are shared by heads_q / heads_kv
 * consecutive heads of queries):
 *     s = scale q_i.k_j;   with cap > 0: s = cap tanh(s / cap);   s = s - slope |i - j|
 *     out_i = sum_j softmax_j(s) v_j over the keys that the mask lets i see
 * A row that sees nothing (padding) is 0 and its lse -infinity.  What is not seen has no
 * part in a result, infinite or NaN as it may be.  (That takes time: rows whose neighbours in
 * the block, up to 127 slots from what they see, are not finite are computed again one by one;
 * 127 of them that see 2048 slots each take some 60 ms.)  A value that is seen and infinite makes
 * its element of the result infinite, or NaN where its probability is 0 in the type.
 *
 * dtype      F16, BF16 or F32 (of q, k, v and out); head_dim 1 .. BLOAD_ATTENTION_MAX_HEAD_DIM
 * scale      > 0;  cap >= 0 (0: none; from 2^100 on all alike);  d_slopes  in  float32[heads_q] or NULL
 * d_mask     from bload_segment_mask.  Any other intervals do as well; they are cut to
 *            [0, t_blk), and the backward pass needs the two of each slot to agree.
 * d_lse      out  float32[num_blocks, heads_q, t_blk] or NULL: ln sum e^s, for the
 *                 backward pass
 * out_rest   out  like out, or NULL: what rounding to the type took from out (16-bit types;
 *                 0 for F32), from which the backward pass forms do.out more exactly
 * Products are those of the type with sums in 32 bits; probabilities are rounded to the
 * type before they meet v.  Asynchronous on `hip_stream`, no workspace; same inputs give
 * bit-identical outputs. */
bload_status bload_segment_attention(const bload_heads* q, const bload_heads* k, const bload_heads* v, const int32_t* d_mask,
                                     int64_t num_blocks, int32_t t_blk, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                                     bload_dtype dtype, float scale, float cap, const float* d_slopes, const bload_heads* out,
                                     float* d_lse, const bload_heads* out_rest, void* hip_stream);

/* Gradients of sum(out * dout) by q, k and v (dk and dv summed over the heads that share
 * them; no gradient of scale, cap and slopes).  out, d_lse and, where it was written,
 * out_rest are those of the forward call with the same arguments; the outputs must not
 * overlap any input.  For 16-bit types probabilities and the gradients of scores are rounded to
 * the type's precision before they meet dout, q and k; for F16 scaled by powers of two, so that
 * they keep it however small or large dout is.
 * d_workspace: >= bload_segment_attention_backward_workspace_bytes() bytes, 16-byte aligned.
 * Asynchronous on `hip_stream`; bit-identical like the forward pass. */
size_t bload_segment_attention_backward_workspace_bytes(int64_t num_blocks, int32_t t_blk, int32_t heads_q);

bload_status bload_segment_attention_backward(const bload_heads* dout, const bload_heads* q, const bload_heads* k,
                                              const bload_heads* v, const bload_heads* out, const float* d_lse,
                                              const bload_heads* out_rest, const int32_t* d_mask, int64_t num_blocks,
                                              int32_t t_blk, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                                              bload_dtype dtype, float scale, float cap, const float* d_slopes,
                                              const bload_heads* dq, const bload_heads* dk, const bload_heads* dv,
                                              void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* The form for single tokens: one query for every sequence, which sees all of the sequence's
 * frames; the packed blocks are the cache of keys and values.  The query stands at the
 * sequence's last frame (for slopes).
 * q, out          [n_seq, heads_q, head_dim]: block_stride is the distance of two sequences,
 *                 slot_stride is not used
 * k, v            [num_blocks, t_blk, heads_kv, head_dim]
 * d_block_of_seq, d_offset_of_seq, d_lengths  in  int32[n_seq]: sequence i lies in the slots
 *                 [offset, offset + length) of its block.  A sequence without frames, or one
 *                 that does not lie inside the blocks (block -1 of another worker's share), gives 0.
 * d_workspace     >= bload_segment_attention_decode_workspace_bytes(...) bytes, 16-byte aligned
 *                 (may be NULL when that is 0)
 * The rest is bload_segment_attention's.  Asynchronous on `hip_stream`. */
size_t bload_segment_attention_decode_workspace_bytes(int64_t n_seq, int32_t t_blk, int32_t heads_q, int32_t heads_kv,
                                                      int32_t head_dim);

bload_status bload_segment_attention_decode(const bload_heads* q, const bload_heads* k, const bload_heads* v,
                                            const int32_t* d_block_of_seq, const int32_t* d_offset_of_seq, const int32_t* d_lengths,
                                            int64_t n_seq, int64_t num_blocks, int32_t t_blk, int32_t heads_q, int32_t heads_kv,
                                            int32_t head_dim, bload_dtype dtype, float scale, float cap, const float* d_slopes,
                                            const bload_heads* out, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* ----------------------------------------------------------- gated scan --
 * bload_segment_scan with a gate for every element in place of one decay, a state that may be
 * handed in and out, and a backward pass.  Per feature, along the slots of a block:
 *     h = gate * h_prev + x   where the slot goes on: it is valid, carries no start flag and the
 *                             slot in front of it is valid; the first slot of a block goes on
 *                             from d_state_in, where that is given and the slot carries no flag
 *     h = x                   where it starts a sequence
 *     h = 0                   on padding
 * Blocks of one slot (t_blk = 1) with a state in and out are the form for single tokens.
 *
 * d_gate, d_x  in   [B, t_blk, feat_dim] of `dtype` (F16, BF16 or F32), aligned to an element
 * d_reset, d_valid  in  uint8[B, t_blk]
 * d_state_in   in   float32[B, feat_dim] or NULL (no state: the first slot starts a sequence)
 * d_out        out  [B, t_blk, feat_dim] of `dtype`: h; every element is written; overlaps no input
 * d_state_out  out  float32[B, feat_dim] or NULL: h of the last slot, unrounded; may be
 *                   d_state_in where t_blk <= 8, and is refused (BLOAD_EINVAL) where it meets
 *                   d_state_in in any other way
 * d_workspace       device scratch of >= bload_gated_scan_workspace_bytes(...) bytes, 16-byte
 *                   aligned (may be NULL when that is 0); one answer for both passes
 * States are held in 32 bits.  What is cut off by a start or by padding has no part in a
 * result, infinite or NaN as it may be.  The product of the gates of consecutive slots has
 * to stay inside float32 (it does where no |gate| is above 1).
 * Asynchronous on `hip_stream`; same inputs give bit-identical outputs. */
size_t bload_gated_scan_workspace_bytes(int64_t num_blocks, int32_t t_blk, int64_t feat_dim, bload_dtype dtype);

bload_status bload_gated_scan(const void* d_gate, const void* d_x, const uint8_t* d_reset, const uint8_t* d_valid,
                              int64_t num_blocks, int32_t t_blk, int64_t feat_dim, bload_dtype dtype, const float* d_state_in,
                              void* d_out, float* d_state_out, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Gradients of sum(out * dout) + sum(state_out * dstate_out) by gate, x and state_in.
 * d_out, d_state_in  in   of the forward pass; dgate is formed with the rounded states of d_out
 * d_dstate_out       in   float32[B, feat_dim] or NULL
 * d_dgate, d_dx      out  [B, t_blk, feat_dim] of `dtype`, every element written, overlapping no input
 * d_dstate_in        out  float32[B, feat_dim] or NULL (0 where the first slot does not go on); may be
 *                         d_dstate_out or d_state_in where t_blk <= 8, else refused where it meets one */
bload_status bload_gated_scan_backward(const void* d_dout, const void* d_gate, const void* d_out, const uint8_t* d_reset,
                                       const uint8_t* d_valid, int64_t num_blocks, int32_t t_blk, int64_t feat_dim,
                                       bload_dtype dtype, const float* d_state_in, const float* d_dstate_out, void* d_dgate,
                                       void* d_dx, float* d_dstate_in, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* --------------------------------------------------------------- rotary --
 * Rotary positions: the pairs of the first rot_dim elements of every head (elements i and
 * i + rot_dim / 2, or 2 i and 2 i + 1) are turned by position * d_freq[i] radians and multiplied
 * by `scale`; the elements behind are handed through.  inverse = 1 turns back: the gradient.
 *
 * x, out       [num_blocks, t_blk, heads, head_dim] of F16, BF16 or F32; out may be x;
 *              rot_dim even, 2 .. BLOAD_ROTARY_MAX_DIM, head_dim up to 65536
 * d_positions  in   int32[num_blocks, t_blk]: frame_idx of bload_pack, or any others; negative
 *                   ones are padding, whose elements become 0
 * d_freq       in   float32[rot_dim / 2], radians per frame
 * Angles are formed in 64 bits.  Asynchronous on `hip_stream`, no workspace. */
#define BLOAD_ROTARY_MAX_DIM 4096
typedef enum { BLOAD_ROTARY_HALF = 0, BLOAD_ROTARY_INTERLEAVED = 1 } bload_rotary_layout;

bload_status bload_rotary(const bload_heads* x, const int32_t* d_positions, int64_t num_blocks, int32_t t_blk, int32_t heads,
                          int32_t head_dim, bload_dtype dtype, const float* d_freq, int32_t rot_dim, bload_rotary_layout layout,
                          float scale, int32_t inverse, const bload_heads* out, void* hip_stream);

/* base^(-2 i / rot_dim) for the pairs i, stretched for contexts `factor` times as long as the
 * model was trained on: with trained = 0 all are divided by factor; with trained > 0 (in frames)
 * those of fewer than `slow` turns over that length are divided, those of more than `fast` kept,
 * and the ones between mixed in proportion (slow < fast).  Host only. */
bload_status bload_rotary_frequencies(int32_t rot_dim, double base, double factor, int64_t trained, double slow, double fast,
                                      float* h_freq);

/* ------------------------------------------------------------ layer norm --
 * Rows of features brought to one size: with s = x, or x + residual rounded to the type,
 *     m = mean(s) (center = 1) or 0 (center = 0: root mean square norm)
 *     out = (s - m) / sqrt(mean((s - m)^2) + eps) * weight + bias
 * over the `dim` elements of each head of each slot: heads = 1 for a slot's features as a whole, the heads of queries and keys
 * for a norm of each.
 *
 * x, residual, out, sum   [num_blocks, t_blk, heads, dim] of F16, BF16 or F32; residual may be NULL.  out may be x, and sum
 *                 residual, with the same strides; else outputs overlap no input
 * d_valid         in   uint8[num_blocks, t_blk] or NULL (all valid): rows of padding are not read, and become 0
 * eps             >= 0
 * d_weight, d_bias in  float32[dim], or NULL for ones and zeros
 * sum             out  s, or NULL
 * d_stats         out  float32[num_blocks, t_blk, heads, 2], 8-byte aligned, or NULL: mean and 1 / deviation, for the backward pass
 * The mean, the mean square and everything per element are in 32 bits.  num_blocks * t_blk * heads < 2^31, dim up to
 * BLOAD_LAYER_NORM_MAX_DIM.  Asynchronous on `hip_stream`, no workspace; same inputs give bit-identical outputs. */
#define BLOAD_LAYER_NORM_MAX_DIM (1 << 21)

bload_status bload_layer_norm(const bload_heads* x, const bload_heads* residual, const uint8_t* d_valid, int64_t num_blocks,
                              int32_t t_blk, int32_t heads, int32_t dim, bload_dtype dtype, int32_t center, float eps,
                              const float* d_weight, const float* d_bias, const bload_heads* out, const bload_heads* sum,
                              float* d_stats, void* hip_stream);

/* Gradients of sum(out * dout) + sum(sum * dsum) by s (which is that by x and by residual), weight and bias.
 * x               in   what was normalised: the forward call's x, or its sum where it had a residual
 * d_stats         in   of the forward call;  dsum  in  like x, or NULL
 * dx              out  like x, 0 on padding; may be dout or dsum with the same strides
 * d_dweight, d_dbias out float32[dim], or NULL; written also where there are no rows
 * d_workspace     >= bload_layer_norm_backward_workspace_bytes() bytes, 16-byte aligned (may be NULL without d_dweight and d_dbias)
 * Asynchronous on `hip_stream`; bit-identical like the forward pass. */
size_t bload_layer_norm_backward_workspace_bytes(int64_t num_blocks, int32_t t_blk, int32_t heads, int32_t dim, bload_dtype dtype);

bload_status bload_layer_norm_backward(const bload_heads* dout, const bload_heads* x, const float* d_stats, const uint8_t* d_valid,
                                       int64_t num_blocks, int32_t t_blk, int32_t heads, int32_t dim, bload_dtype dtype, int32_t center,
                                       const float* d_weight, const bload_heads* dsum, const bload_heads* dx, float* d_dweight,
                                       float* d_dbias, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* -------------------------------------------------------- segment conv --
 * A short causal convolution of every feature by itself inside the sequences: per slot t of a block
 *     p = bias + sum_j weight[d][taps - 1 - j] x[t - j]
 * over the taps j that reach no further back than t's sequence, and out = p, or with silu = 1 p / (1 + e^-p); 0 on padding.  A
 * slot goes on from the one in front of it as in bload_gated_scan, and the first slot of a block from the state, where that is
 * given and the slot carries no start flag.  Blocks of one slot with a state in and out are the form for single tokens.
 *
 * x, out       [num_blocks, t_blk, feat_dim] of F16, BF16 or F32 (bload_heads whose head_stride is not used); out overlaps no input
 * d_weight     in   float32[feat_dim, taps], taps 1 .. BLOAD_CONV_MAX_TAPS;  d_bias  in  float32[feat_dim] or NULL
 * d_reset, d_valid  in  uint8[num_blocks, t_blk]
 * d_state_in   in   [num_blocks, taps - 1, feat_dim] of `dtype` or NULL: the inputs in front of the first slot, the oldest first
 * d_state_out  out  the same behind the last slot, 0 where its sequence (or padding) does not reach, or NULL; may be d_state_in
 *                   where t_blk <= 8, and is refused (BLOAD_EINVAL) where it meets d_state_in in any other way
 * Sums are in 32 bits.  What lies in another sequence has no part in a result, infinite or NaN as it may be.
 * Asynchronous on `hip_stream`, no workspace; same inputs give bit-identical outputs. */
#define BLOAD_CONV_MAX_TAPS 8

bload_status bload_segment_conv(const bload_heads* x, const float* d_weight, const float* d_bias, const uint8_t* d_reset,
                                const uint8_t* d_valid, int64_t num_blocks, int32_t t_blk, int32_t feat_dim, int32_t taps,
                                bload_dtype dtype, int32_t silu, const void* d_state_in, const bload_heads* out, void* d_state_out,
                                void* hip_stream);

/* Gradients of sum(out * dout) + sum(state_out * dstate_out) by x, weight, bias and state_in.
 * d_dstate_out  in   like the state, or NULL
 * dx            out  like x, every element written (0 on padding), overlapping no input
 * d_dweight, d_dbias  out  float32[feat_dim, taps] and [feat_dim], or NULL; written also where there are no blocks
 * d_dstate_in   out  like the state, or NULL; overlaps neither state nor d_dstate_out (BLOAD_EINVAL)
 * d_workspace   >= bload_segment_conv_backward_workspace_bytes() bytes, 16-byte aligned (may be NULL without d_dweight and d_dbias) */
size_t bload_segment_conv_backward_workspace_bytes(int64_t num_blocks, int32_t t_blk, int32_t feat_dim, int32_t taps, bload_dtype dtype);

bload_status bload_segment_conv_backward(const bload_heads* dout, const bload_heads* x, const float* d_weight, const float* d_bias,
                                         const uint8_t* d_reset, const uint8_t* d_valid, int64_t num_blocks, int32_t t_blk,
                                         int32_t feat_dim, int32_t taps, bload_dtype dtype, int32_t silu, const void* d_state_in,
                                         const void* d_dstate_out, const bload_heads* dx, float* d_dweight, float* d_dbias,
                                         void* d_dstate_in, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------ selective scan --
 * A state space whose steps, inputs and outputs go by the frame: every channel d keeps `states` states h_n, and per slot
 *     step = dt + dt_bias[d], or with softplus = 1 ln(1 + e^(dt + dt_bias[d]))
 *     h_n = e^(step rate[d][n]) h_n + step b_n x   where the slot goes on (as in bload_gated_scan),
 *     h_n = step b_n x                             where it starts a sequence, and 0 on padding
 *     y = sum_n c_n h_n + skip[d] x;   out = y z / (1 + e^-z), or y without z; 0 on padding
 * b and c are shared by the feat_dim / groups consecutive channels of a group.  Blocks of one slot with a state in and out are
 * the form for single tokens. */
#define BLOAD_SELECTIVE_MAX_STATES 64

typedef struct {
    bload_heads x, dt, z;            /* [num_blocks, t_blk, feat_dim] of `dtype` (head_stride is not used); z.d_data may be NULL */
    bload_heads b, c;                /* [num_blocks, t_blk, groups, states] of `dtype` */
    const float* d_rate;             /* float32[feat_dim, states]: negative where states fade */
    const float* d_skip;             /* float32[feat_dim] or NULL */
    const float* d_dt_bias;          /* float32[feat_dim] or NULL */
    const uint8_t *d_reset, *d_valid;        /* uint8[num_blocks, t_blk] */
    const float* d_state_in;         /* float32[num_blocks, feat_dim, states] or NULL (no state: the first slot starts a sequence) */
    int64_t num_blocks;
    int32_t t_blk, feat_dim, states, groups; /* states 1 .. BLOAD_SELECTIVE_MAX_STATES; groups divides feat_dim */
    bload_dtype dtype;               /* F16, BF16 or F32 */
    int32_t softplus;
} bload_selective;

/* out          out  like x, every element written; overlaps no input
 * d_state_out  out  like the state, or NULL: the state of the last slot; may be d_state_in where t_blk <= 8, and is refused
 *                   (BLOAD_EINVAL) where it meets d_state_in in any other way
 * d_saved      out  bload_selective_scan_saved_bytes() bytes, for the backward pass, or NULL: the state in front of every 16th slot
 * d_workspace  >= bload_selective_scan_workspace_bytes() bytes, 16-byte aligned (may be NULL when that is 0)
 * States, steps and sums are in 32 bits.  What lies in another sequence or in padding has no part in a result, infinite or NaN as
 * it may be.  Asynchronous on `hip_stream`; same inputs give bit-identical outputs. */
size_t bload_selective_scan_workspace_bytes(int64_t num_blocks, int32_t t_blk, int32_t feat_dim, int32_t states, int32_t groups);
size_t bload_selective_scan_saved_bytes(int64_t num_blocks, int32_t t_blk, int32_t feat_dim, int32_t states, int32_t groups);

bload_status bload_selective_scan(const bload_selective* s, const bload_heads* out, float* d_state_out, float* d_saved,
                                  void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Gradients of sum(out * dout) + sum(state_out * dstate_out) by x, dt, rate, b, c, skip, z, dt_bias and state_in.
 * s, d_saved     in   the forward call's
 * d_dstate_out   in   float32[num_blocks, feat_dim, states] or NULL
 * dx, ddt, db, dc, dz  out  like their inputs, every element written (0 on padding), overlapping no input; dz is not used without z
 * d_drate, d_dskip, d_ddt_bias  out  float32 like their inputs, or NULL; written also where there are no blocks
 * d_dstate_in    out  like the state, or NULL (0 where the first slot does not go on); meets neither state nor d_dstate_out (BLOAD_EINVAL)
 * d_workspace    >= bload_selective_scan_backward_workspace_bytes() bytes, 16-byte aligned */
size_t bload_selective_scan_backward_workspace_bytes(int64_t num_blocks, int32_t t_blk, int32_t feat_dim, int32_t states, int32_t groups);

bload_status bload_selective_scan_backward(const bload_selective* s, const bload_heads* dout, const float* d_saved,
                                           const float* d_dstate_out, const bload_heads* dx, const bload_heads* ddt, float* d_drate,
                                           const bload_heads* db, const bload_heads* dc, float* d_dskip, const bload_heads* dz,
                                           float* d_ddt_bias, float* d_dstate_in, void* d_workspace, size_t workspace_bytes,
                                           void* hip_stream);

/* -------------------------------------------------------- strategy counts --
 * Problem Statement and Table 1 (rows "padding amount" and "# frames deleted"):
 * what the strategies compared there cost on a given set of lengths, counted in
 * frames, without materialising anything.
 *   pad to the longest  every sequence padded to t_max:  n_seq * t_max - sum(L)
 *   chunk sampling      every sequence cut into pieces of t_chunk frames, each a
 *                       sample of its own, nothing padded: sum(floor(L / t_chunk))
 *                       samples, sum(L mod t_chunk) frames deleted
 *   block packing       num_blocks * t_blk - sum(L), for the plan's num_blocks
 * ("mix pad" of Table 1 is not defined in the paper and is not counted.)
 *
 * d_lengths   in   int32[n_seq], every L >= 0
 * t_max       in   pad-to-longest target; <= 0 means "the longest sequence found"
 * t_chunk     in   >= 1
 * num_blocks, t_blk   in   as returned by / given to a planner (0, 0 to skip)
 * h_counts    out  host struct, see below
 * d_workspace      >= 64 bytes, 16-byte aligned
 *
 * Synchronises the stream before returning.
 */
typedef struct bload_strategy_counts_t {
    int64_t total_frames;       /* sum(L) */
    int64_t longest;            /* max(L), 0 when n_seq == 0 */
    int64_t pad_to_longest;     /* frames of padding when every sequence is padded */
    int64_t pad_blocks;         /* frames of padding in the packed blocks */
    int64_t chunk_samples;      /* pieces of t_chunk frames */
    int64_t chunk_deleted;      /* frames that fill no piece */
} bload_strategy_counts_t;

bload_status bload_strategy_counts(const int32_t* d_lengths, int64_t n_seq, int32_t t_max,
                                   int32_t t_chunk, int64_t num_blocks, int32_t t_blk,
                                   bload_strategy_counts_t* h_counts, void* d_workspace,
                                   size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* BLOAD_H */
