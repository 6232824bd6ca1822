/*
 * libmala -- C ABI of the B200 (sm_100a) MassAlloc Attention (MALA) hot path.
 *
 * The operator is the one the paper's Methodology section states for a query head and its
 * key/value head: QK^T scores are formed for every legal causal tile; a forward tile is skipped
 * when, for every relevant row, rowmax(S) - m - log(l) < log(tau / L_q) (Eq. 3, Algorithm 1);
 * a backward tile is skipped when S - lse < log(tau / L_q) on all its valid entries (Eq. 4,
 * Algorithm 2); split-KV decode applies the forward rule per split against the split's partial
 * normalizer with L = N_k and merges the partials ("Fused decoding execution").  tau = 0 selects
 * the dense FullAttn kernels (Section 2.3: tau -> 0 recovers FullAttn).
 *
 * Conventions common to all calls
 *   - Every pointer is a DEVICE pointer owned by the caller unless stated otherwise; the library
 *     never frees or retains one.  Tensors are bf16 views [B, N, H, d] given as a base pointer and
 *     element strides (sb, sn, sh); the last dimension is contiguous.  Base pointers must be
 *     16-byte aligned and all strides multiples of 8 elements (16 bytes).
 *   - d is a multiple of 8 between 8 and 256 for the forward calls (mala_fwd*) and the decode calls on a bf16 cache
 *     (mala_decode, _multi, _paged, _static), between 8 and 128 for the backward calls and a multiple of 16 up to
 *     128 for the calls on an e4m3 cache (the paper's symbols put no limit on d_h, Section 2.1; its models use 128).
 *     The kernels exist for 64, 128 and 256 columns; another head size runs on the next of them at that size's cost
 *     (the missing columns are read as zeros and never stored).
 *     Hq must be a multiple of Hkv; query head h uses key/value head h / (Hq / Hkv).  N may be any positive length (the last tile may be ragged).
 *   - scale (> 0, finite) multiplies the fp32 scores; lse is in nats, of the scaled scores, over
 *     the retained set.  tau >= 0, finite.
 *   - Tile partition: mala_tile_shape() reports it; forward and backward use the same partition.
 *   - Two environment variables, read once per process, change what a call does around its launches (both off by
 *     default): MALA_NVTX=1 makes every launching call an NVTX range of its own name; MALA_DEBUG=1 makes error
 *     reporting synchronous -- the call waits for its stream and returns MALA_ERR_CUDA or MALA_ERR_DEVICE_TIMEOUT
 *     itself (with a line on stderr) instead of leaving the error to a later call.  A debug call therefore
 *     synchronises, which a call otherwise never does.
 *   - Calls are asynchronous on `cuda_stream` (a cudaStream_t, may be NULL for the default
 *     stream), allocate nothing and never synchronise.  `ws` is caller-provided scratch of at
 *     least mala_workspace_bytes() bytes, 256-byte aligned; its contents are undefined afterwards.
 *   - Return value: MALA_OK or a negative MALA_ERR_* code; nothing is launched on error.
 *     A bounded device-side wait that expires does not hang: the kernels finish, later launches
 *     become no-ops, and mala_device_status() reports MALA_ERR_DEVICE_TIMEOUT until cleared.
 */
#ifndef MALA_H_
#define MALA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MALA_OK 0
#define MALA_ERR_INVALID_ARG (-1)        /* NULL pointer, non-positive size, bad tau / scale */
#define MALA_ERR_UNSUPPORTED (-2)        /* d not a multiple of 8 in the call's range, Hq % Hkv != 0, too many splits ... */
#define MALA_ERR_MISALIGNED (-3)         /* pointer / stride alignment rules above violated */
#define MALA_ERR_WORKSPACE_TOO_SMALL (-4)
#define MALA_ERR_WRONG_ARCH (-5)         /* current device is not compute capability 10.x */
#define MALA_ERR_CUDA (-6)               /* a CUDA runtime call or launch failed */
#define MALA_ERR_TENSOR_MAP (-7)         /* the driver rejected a TMA tensor map */
#define MALA_ERR_DEVICE_TIMEOUT (-8)     /* a bounded device-side wait expired (status word) */
#define MALA_ERR_STATIC_SCRATCH_EXCEEDED (-9) /* mala_decode_static: problem exceeds the built-in scratch */

/* Size of the scratch array compiled into the library for mala_decode_static (24 MiB per device). */
#define MALA_STATIC_SCRATCH_BYTES (24u << 20)

#define MALA_OP_FWD 0
#define MALA_OP_BWD 1
#define MALA_OP_DECODE 2

typedef struct { const void* p; int64_t sb, sn, sh; } mala_tin;   /* read-only bf16 [B,N,H,d] view */
typedef struct { void* p; int64_t sb, sn, sh; } mala_tout;        /* written bf16 [B,N,H,d] view */

/* Optional telemetry (any member may be NULL; the struct pointer itself may be NULL).
 *   retained_per_block : u32, overwritten.  fwd [B,Hq,Tr] (per query block), bwd [B,Hq,Tc] (per key
 *                        block and query head), decode [B,Hkv,num_splits].
 *   tile_bitmask       : u32 words, overwritten.  fwd [B,Hq,Tr,ceil(Tc/32)], bit j of row i set iff
 *                        tile (i,j) was retained; bwd [B,Hq,Tc,ceil(Tr/32)], bit i of row j;
 *                        decode [B,Hkv,num_splits,ceil(tiles_per_split/32)].  Meant for parity checks.
 *   totals             : u64[2], ACCUMULATED: += retained tiles, += legal (visited) tiles. */
typedef struct {
  uint32_t* retained_per_block;
  uint32_t* tile_bitmask;
  uint64_t* totals;
} mala_stats;

/* Algorithm 1 (forward / prefill).  q [B,N,Hq,d]; k, v [B,N,Hkv,d]; o [B,N,Hq,d]; lse fp32 [B,Hq,N].
 * causal != 0: equal-length causal attention, L_q = q + 1, tiles visited from the diagonal toward
 * earlier keys.  causal == 0: every key legal, L_q = N, tiles visited from the last to the first. */
int mala_fwd(mala_tin q, mala_tin k, mala_tin v, mala_tout o, float* lse, const mala_stats* st, int B, int Hq,
             int Hkv, int N, int d, int causal, float scale, float tau, void* ws, size_t ws_bytes,
             void* cuda_stream);

/* Algorithm 2 (backward).  o, dout [B,N,Hq,d]; lse as written by mala_fwd; dq [B,N,Hq,d];
 * dk, dv [B,N,Hkv,d] (summed over the query heads of the group).  D = rowsum(O o dO) is computed
 * from the given o.  dQ is accumulated in fp32 in the workspace and converted at the end. */
int mala_bwd(mala_tin q, mala_tin k, mala_tin v, mala_tin o, mala_tin dout, const float* lse, mala_tout dq,
             mala_tout dk, mala_tout dv, const mala_stats* st, int B, int Hq, int Hkv, int N, int d, int causal,
             float scale, float tau, void* ws, size_t ws_bytes, void* cuda_stream);

/* Algorithms 1 and 2 with fewer queries than keys (chunked prefill; cross attention when causal == 0).
 * q, o, dout, dq [B,Nq,Hq,d]; k, v, dk, dv [B,Nk,Hkv,d]; lse fp32 [B,Hq,Nq].
 * causal != 0: the queries are the LAST Nq of the Nk positions (Nk >= Nq): query row q attends to the keys
 * 0 .. q + Nk - Nq and L_q = q + 1 + Nk - Nq, the number of keys it sees (Section 2.1); a query block visits its
 * tiles from its diagonal toward earlier keys.  The query blocks follow the key positions -- block i holds the rows q
 * with 128 i <= q + (Nk - Nq) % 128 < 128 (i + 1), so the first block of a chunk that starts inside a tile is a short
 * one -- and the result therefore equals rows Nk - Nq .. Nk - 1 of the equal-length call on the whole sequence wherever
 * the chunk holds a whole block of that call (for the backward: with dout zero on the earlier rows).
 * Both calls take any Nk >= Nq.
 * causal == 0: every key legal for every query, L_q = Nk, any Nq and Nk.
 * Telemetry: fwd retained_per_block [B,Hq,Tq], tile_bitmask [B,Hq,Tq,ceil(ceil(Nk/128)/32)] with
 * Tq = ceil((Nq + (Nk - Nq) % 128) / 128) (causal) or ceil(Nq/128);
 * bwd retained_per_block [B,Hq,ceil(Nk/128)], tile_bitmask [B,Hq,ceil(Nk/128),ceil(Tq/32)].
 * Workspace of the backward: mala_workspace_bytes(MALA_OP_BWD, B, Hq, Hkv, Nq + (Nk - Nq) % 128, d, 0) when causal
 * (the accumulator holds whole query blocks), mala_workspace_bytes(MALA_OP_BWD, B, Hq, Hkv, Nq, d, 0) otherwise.  Everything else as
 * mala_fwd / mala_bwd, which are these calls with Nq = Nk = N. */
int mala_fwd_chunk(mala_tin q, mala_tin k, mala_tin v, mala_tout o, float* lse, const mala_stats* st, int B, int Hq,
                   int Hkv, int Nq, int Nk, int d, int causal, float scale, float tau, void* ws, size_t ws_bytes,
                   void* cuda_stream);
int mala_bwd_chunk(mala_tin q, mala_tin k, mala_tin v, mala_tin o, mala_tin dout, const float* lse, mala_tout dq,
                   mala_tout dk, mala_tout dv, const mala_stats* st, int B, int Hq, int Hkv, int Nq, int Nk, int d,
                   int causal, float scale, float tau, void* ws, size_t ws_bytes, void* cuda_stream);

/* mala_fwd_chunk with the keys cut into num_splits ranges that run on different SMs: for a short chunk of queries
 * against a long context (where mala_fwd_chunk has fewer query blocks than the GPU has SMs).  The key blocks
 * 0 .. ceil(Nk/128)-1 are cut into num_splits contiguous ranges of ceil(ceil(Nk/128)/num_splits) blocks; every range
 * runs Algorithm 1 on its blocks with its own running state, i.e. its skip test sees the range's PARTIAL normalizer
 * (the split-local rule of "Fused decoding execution"; more conservative than the unsplit test), and the ranges are
 * merged by lse = log sum_s exp(lse_s), o = sum_s exp(lse_s - lse) o_s.  num_splits = 1 is mala_fwd_chunk; tau = 0
 * gives FullAttn for any num_splits.  Telemetry as for mala_fwd_chunk.  ws: device scratch of
 * mala_workspace_bytes(MALA_OP_FWD, B, Hq, Hkv, Nq, d, num_splits) bytes, 256-byte aligned.  B * num_splits <= 65535. */
int mala_fwd_chunk_split(mala_tin q, mala_tin k, mala_tin v, mala_tout o, float* lse, const mala_stats* st, int B,
                         int Hq, int Hkv, int Nq, int Nk, int d, int causal, float scale, float tau, int num_splits,
                         void* ws, size_t ws_bytes, void* cuda_stream);

/* Algorithms 1 and 2 on B packed sequences of different lengths (self attention, equal query and key lengths per
 * sequence).  q, o, dout, dq are [1,total,Hq,d] tensors, k, v, dk, dv [1,total,Hkv,d] (sb is ignored); sequence b
 * holds the rows cu_seqlens[b] .. cu_seqlens[b+1]-1; cu_seqlens: device int32 [B+1], non-decreasing, cu_seqlens[0] = 0,
 * cu_seqlens[B] = total; max_seqlen >= every length (it sizes the grid and the telemetry).  Every sequence is treated
 * exactly as a mala_fwd / mala_bwd call on its own rows (its own tile partition, starting at its first row; its own
 * L_q).  lse: fp32 [Hq,total].  Telemetry as for mala_fwd / mala_bwd with N = max_seqlen (rows of blocks a sequence
 * does not have stay zero).  Workspace of the backward:
 * mala_workspace_bytes(MALA_OP_BWD, 1, Hq, Hkv, total + 128 * B, d, 0).  The tile that holds a sequence's last rows
 * also covers the first rows of the next one: those never reach a result, but they must be finite numbers. */
int mala_fwd_varlen(mala_tin q, mala_tin k, mala_tin v, const int32_t* cu_seqlens, mala_tout o, float* lse,
                    const mala_stats* st, int B, int Hq, int Hkv, int total, int max_seqlen, int d, int causal,
                    float scale, float tau, void* ws, size_t ws_bytes, void* cuda_stream);
int mala_bwd_varlen(mala_tin q, mala_tin k, mala_tin v, mala_tin o, mala_tin dout, const float* lse,
                    const int32_t* cu_seqlens, mala_tout dq, mala_tout dk, mala_tout dv, const mala_stats* st, int B,
                    int Hq, int Hkv, int total, int max_seqlen, int d, int causal, float scale, float tau, void* ws,
                    size_t ws_bytes, void* cuda_stream);

/* Algorithm 1 on B packed sequences each of which has more keys than queries -- a batch of prefill chunks behind
 * cached prefixes.  q, o [1,total_q,Hq,d] with sequence b in rows cu_seqlens_q[b] .. cu_seqlens_q[b+1]-1; k, v
 * [1,total_k,Hkv,d] with its keys in rows cu_seqlens_k[b] .. cu_seqlens_k[b+1]-1 (both device int32 [B+1]).  Every
 * sequence is treated exactly as a mala_fwd_chunk call on its own rows: causal != 0 puts its queries at its last
 * positions (it must not have more queries than keys: such a sequence is left untouched), its query blocks follow its
 * key positions, L_q is the number of keys the row sees; causal == 0: every key of the sequence legal, L = its number
 * of keys.  max_seqlen_q / max_seqlen_k >= every length.  lse fp32 [Hq,total_q].  Telemetry as for mala_fwd_chunk
 * with Tq = ceil((max_seqlen_q + 127) / 128) and ceil(max_seqlen_k / 128) key blocks. */
int mala_fwd_varlen_prefix(mala_tin q, mala_tin k, mala_tin v, const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k,
                           mala_tout o, float* lse, const mala_stats* st, int B, int Hq, int Hkv, int total_q,
                           int total_k, int max_seqlen_q, int max_seqlen_k, int d, int causal, float scale, float tau,
                           void* ws, size_t ws_bytes, void* cuda_stream);

/* Algorithm 2 for mala_fwd_varlen_prefix: every sequence is treated exactly as a mala_bwd_chunk call on its own
 * rows, with the query blocks following its key positions as in the forward call.  o, dout, dq like q; dk, dv like k;
 * lse fp32 [Hq,total_q] as the forward call wrote it.  A sequence without queries (or, causal != 0, with more queries
 * than keys) gets zero dk / dv rows (and zero dq rows).  Telemetry as for mala_bwd_chunk with ceil(max_seqlen_k / 128)
 * key blocks and Tq = ceil((max_seqlen_q + 127) / 128).  Workspace:
 * mala_workspace_bytes(MALA_OP_BWD, 1, Hq, Hkv, total_q + 384 * B, d, 0).  As for the other packed calls, the tiles at
 * a sequence's ends also cover rows of its neighbours, which must be finite numbers. */
int mala_bwd_varlen_prefix(mala_tin q, mala_tin k, mala_tin v, mala_tin o, mala_tin dout, const float* lse,
                           const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, mala_tout dq, mala_tout dk,
                           mala_tout dv, const mala_stats* st, int B, int Hq, int Hkv, int total_q, int total_k,
                           int max_seqlen_q, int max_seqlen_k, int d, int causal, float scale, float tau, void* ws,
                           size_t ws_bytes, void* cuda_stream);

/* mala_fwd_varlen_prefix with the keys and values held in pages: a batch of prefill chunks behind prefixes that
 * live in a paged cache (the chunks' own keys and values already written to their pages).  q, o [1,total_q,Hq,d]
 * packed by cu_seqlens_q (device int32 [B+1]); kpages, vpages [num_pages, page_size, Hkv, d] with page_size a multiple
 * of 128, or 8, 16, 32 or 64 (a tile is then put together from 128 / page_size pages, each with its own table
 * lookup, at reduced throughput); block_table device int32 [B, max_pages_per_seq] (keys page_size*x .. of sequence b in page
 * block_table[b][x]); seqlens_k device int32 [B], the keys sequence b holds, clamped to
 * max_pages_per_seq * page_size (what its block-table row can map), its queries being its last positions
 * (a sequence with no keys, or with fewer keys than queries when causal != 0, is left untouched).  Slots of a mapped
 * page beyond the sequence's length must hold finite numbers.  Everything else as mala_fwd_varlen_prefix with
 * max_seqlen_k = max_pages_per_seq * page_size. */
int mala_fwd_paged(mala_tin q, mala_tin kpages, mala_tin vpages, const int32_t* cu_seqlens_q, const int32_t* block_table,
                   const int32_t* seqlens_k, mala_tout o, float* lse, const mala_stats* st, int B, int Hq, int Hkv,
                   int total_q, int max_seqlen_q, int num_pages, int page_size, int max_pages_per_seq, int d, int causal,
                   float scale, float tau, void* ws, size_t ws_bytes, void* cuda_stream);

/* Split-KV decode of one new token per sequence ("Fused decoding execution").  q [B,1,Hq,d] (sn is
 * ignored); kcache, vcache [B,Nk,Hkv,d], the newest token's key/value included; o [B,1,Hq,d];
 * lse_opt fp32 [B,Hq] or NULL.  The Hq/Hkv query heads of one KV head are the rows of one tile; the
 * key range is cut into num_splits contiguous chunks of ceil(ceil(Nk/num_splits)/128)*128 keys,
 * each visited newest tile first with its own running state, L = Nk; partials are merged by the
 * normalizer-aware reduction.  Requires Hq/Hkv <= 16. */
int mala_decode(mala_tin q, mala_tin kcache, mala_tin vcache, mala_tout o, float* lse_opt, const mala_stats* st,
                int B, int Hq, int Hkv, int Nk, int d, float scale, float tau, int num_splits, void* ws,
                size_t ws_bytes, void* cuda_stream);

/* mala_decode over an 8-bit KV cache: the same operator ("Fused decoding execution"; the paper keeps the cache intact,
 * and so does this call -- only the storage type differs) on keys and values stored as e4m3 with one fp32 scale per
 * (sequence, KV head, 128-key tile):
 *     k[b, n, h, :] = kscale[b, h, n / 128] * e4m3(kcache8[b, n, h, :]),   v likewise with vscale.
 * The result is that of mala_decode on those dequantised values (the step streams half the bytes).
 * kcache8, vcache8: 8-bit [B,Nk,Hkv,d] views, strides in ELEMENTS (= bytes), multiples of 16; kscale, vscale: device
 * fp32 [B,Hkv,ceil(Nk/128)].  d a multiple of 16, at most 128; Hq/Hkv <= 8 (MALA_ERR_UNSUPPORTED otherwise).  q, o,
 * lse_opt, telemetry, splits and merge as in mala_decode.
 * Workspace: mala_workspace_bytes(MALA_OP_DECODE, B, Hq, Hkv, Nk, 128, num_splits). */
int mala_decode_fp8(mala_tin q, mala_tin kcache8, mala_tin vcache8, const float* kscale, const float* vscale,
                    mala_tout o, float* lse_opt, const mala_stats* st, int B, int Hq, int Hkv, int Nk, int d, float scale,
                    float tau, int num_splits, void* ws, size_t ws_bytes, void* cuda_stream);

/* mala_decode_fp8 with Sq new tokens per sequence: the rule and the layout of mala_decode_multi (q, o [B,Sq,Hq,d],
 * lse_opt [B,Sq,Hq], the new tokens' keys and values in the last Sq positions of the caches, token s at position
 * Nk - Sq + s with L = Nk - Sq + s + 1) on the storage of mala_decode_fp8.  Requires Sq * Hq/Hkv <= 8 and Sq <= Nk
 * (MALA_ERR_UNSUPPORTED otherwise); Sq = 1 is mala_decode_fp8.
 * Workspace: mala_workspace_bytes(MALA_OP_DECODE, B * Sq, Hq, Hkv, Nk, 128, num_splits). */
int mala_decode_fp8_multi(mala_tin q, mala_tin kcache8, mala_tin vcache8, const float* kscale, const float* vscale,
                          mala_tout o, float* lse_opt, const mala_stats* st, int B, int Hq, int Hkv, int Nk, int Sq, int d,
                          float scale, float tau, int num_splits, void* ws, size_t ws_bytes, void* cuda_stream);

/* mala_decode_fp8 over a paged 8-bit cache with one length per sequence: the layout of mala_decode_paged (one new token
 * per sequence) with the storage of mala_decode_fp8.  kpages8, vpages8: 8-bit [num_pages, page_size, Hkv, d] views
 * (strides in elements = bytes, multiples of 16), page_size a multiple of 128, or 16, 32 or 64 (MALA_ERR_UNSUPPORTED
 * otherwise); kscale, vscale: device fp32 [num_pages, Hkv, max(1, page_size/128)], the scale of tile y of page x at
 * [x][h][y] -- one scale per 128-key tile of a page, or one per page where a page is smaller than a tile (a tile is then
 * put together from 128 / page_size pages, each key scaled by its own page's scale; the skip rule's tile stays 128
 * keys).  block_table, seqlens, the split layout (Nk = max_pages_per_seq*page_size), the
 * clamping of seqlens, entries outside the pool (read as zeros) and telemetry as in mala_decode_paged; slots of a
 * mapped page beyond the sequence's length must hold codes other than e4m3's two NaN codes, 0x7f and 0xff (a
 * zero-initialised or recycled page does): their keys are masked out of the scores, but their values are multiplied by
 * zero probabilities.  (Where such slots share a scale with real keys -- the rest of the sequence's last page -- a
 * scale orders of magnitude above the real values' costs those values, and the step's 8-bit probabilities, precision:
 * quantise a page from the slots in use.)  d, Hq/Hkv and the workspace as in mala_decode_fp8. */
int mala_decode_fp8_paged(mala_tin q, mala_tin kpages8, mala_tin vpages8, const float* kscale, const float* vscale,
                          const int32_t* block_table, const int32_t* seqlens, mala_tout o, float* lse_opt,
                          const mala_stats* st, int B, int Hq, int Hkv, int num_pages, int page_size,
                          int max_pages_per_seq, int d, float scale, float tau, int num_splits, void* ws, size_t ws_bytes,
                          void* cuda_stream);

/* Split-KV decode of Sq new tokens per sequence at once (a verification step of speculative decoding, or a short
 * chunk).  q, o [B,Sq,Hq,d]; lse_opt fp32 [B,Sq,Hq] or NULL; kcache, vcache [B,Nk,Hkv,d] with the keys and values of
 * the Sq new tokens already in the last Sq positions.  Token s (0 = oldest) sits at position Nk - Sq + s, attends to
 * the keys before and at its own position and has L = Nk - Sq + s + 1, the number of keys it sees (Section 2.1).
 * The Sq * Hq/Hkv rows that share a KV head form one tile (one row that needs a key block retains it for all; a
 * row that sees no key of a block does not constrain it); requires Sq * Hq/Hkv <= 16 and Sq <= Nk.  Splits,
 * telemetry and merge as in mala_decode; Sq = 1 is mala_decode.
 * Workspace: mala_workspace_bytes(MALA_OP_DECODE, B * Sq, Hq, Hkv, Nk, d, num_splits). */
int mala_decode_multi(mala_tin q, mala_tin kcache, mala_tin vcache, mala_tout o, float* lse_opt, const mala_stats* st,
                      int B, int Hq, int Hkv, int Nk, int Sq, int d, float scale, float tau, int num_splits, void* ws,
                      size_t ws_bytes, void* cuda_stream);

/* Split-KV decode over a paged cache with one length per sequence (the serving-side layout of "Fused decoding
 * execution"; the rule itself is the one of mala_decode / mala_decode_multi with seqlens[b] in the place of Nk).
 * q, o [B,Sq,Hq,d], Sq >= 1 new tokens per sequence whose keys are the last Sq of the sequence's seqlens[b] keys
 * (Sq * Hq/Hkv <= 16; Sq = 1: sn of q and o is ignored); lse_opt fp32 [B,Sq,Hq] or NULL.
 * kpages, vpages [num_pages, page_size, Hkv, d] (sb = page stride, sn = key stride, sh = head stride);
 * page_size is a multiple of 128, or 8, 16, 32 or 64 (a 128-key tile is then fetched as several copies, which costs
 * throughput; MALA_ERR_UNSUPPORTED for any other size).  block_table: device int32
 * [B, max_pages_per_seq]; keys page_size*x .. page_size*(x+1)-1 of sequence b live in page block_table[b][x]
 * (entries beyond the sequence's length are never read; an entry outside [0, num_pages) reads zeros).
 * seqlens: device int32 [B], keys held by each sequence, clamped to [0, max_pages_per_seq*page_size], or NULL
 * if every sequence holds max_pages_per_seq*page_size keys; a token that sees no key (a sequence without keys, or
 * with fewer keys than new tokens) gets o = 0, lse = -inf.
 * The key positions 0 .. max_pages_per_seq*page_size-1 are cut into num_splits chunks as in mala_decode with
 * Nk = max_pages_per_seq*page_size; splits beyond a sequence's length are empty.  Telemetry shapes as for
 * mala_decode with that Nk.  The values stored in a mapped page beyond the sequence's length must be finite
 * bf16 numbers (a zero-initialised or recycled page is): they never reach the result, but the tile that holds
 * the newest key is multiplied as a whole.  Workspace: mala_workspace_bytes(MALA_OP_DECODE, B * Sq, Hq, Hkv,
 * max_pages_per_seq*page_size, d, num_splits).  The library reads block_table and seqlens on the device, on
 * cuda_stream, and keeps neither. */
int mala_decode_paged(mala_tin q, mala_tin kpages, mala_tin vpages, const int32_t* block_table,
                      const int32_t* seqlens, mala_tout o, float* lse_opt, const mala_stats* st, int B, int Hq,
                      int Hkv, int num_pages, int page_size, int max_pages_per_seq, int Sq, int d, float scale,
                      float tau, int num_splits, void* ws, size_t ws_bytes, void* cuda_stream);

/* ---- Attention with a learned relative position bias ------------------------------------------------------------
 * The calls above with one more term in the scores: x = scale * q.k + table[bucket(delta)][h] for query head h and
 * delta = key position - query position, where the queries are the last Nq of the Nk positions (query row q sits at
 * q + Nk - Nq, also when not causal).  Everything that the calls above say of scores holds for x: the skip test, lse
 * (in nats), the retained sets.
 *   Buckets.  bidirectional != 0: half of the buckets, h = num_buckets / 2 (num_buckets even), belong to each side; the
 *   keys after the query take the upper half, and n = |delta|.  bidirectional == 0: all h = num_buckets are for the keys
 *   before the query, n = max(-delta, 0).  With e = h / 2 (rounded down): n < e lies in bucket n of its side, n >= e in
 *   bucket e + floor((h - e) ln(n / e) / ln(max_distance / e)), at most h - 1; a distance that lies exactly on a border
 *   belongs to the bucket that begins there.  2 <= num_buckets <= 128 (4 <= when bidirectional), e < max_distance <= 65536.
 *   table: bf16, entry of bucket b and query head h at [b * sb + h].  Finite values, or -inf: keys of such a bucket are
 *   masked, and a row that sees no other key gets o = 0, lse = -inf and no gradient.
 *   Scores are in fp32: a row whose keys all have biases of magnitude M has scores to M 2^-24, and one of nothing
 *   but a type's lowest values weighs its keys alike (its lse is about -1.4e38).
 *   The backward calls have P from lse: to |lse| 2^-23 of it, and rows with |lse| >= 2^20, where every visible key or the heaviest
 *   ones have a bias as large as that, get no gradient.
 * Head sizes: multiples of 8 up to 128 in all of these calls.  Not causal: any Nq and Nk.
 * ws: mala_bias_workspace_bytes() bytes, 256-byte aligned (the forward calls need it too: the table laid out by distance). */
typedef struct {
  const void* table;                 /* bf16 [num_buckets, Hq] */
  int64_t sb;                        /* elements from one bucket to the next */
  int num_buckets, max_distance, bidirectional;
} mala_rel_bias;

/* mala_fwd_chunk / mala_bwd_chunk with a bias (HOST pointer, read during the call; its table is a device pointer).
 * dtable: bf16, overwritten, entry of bucket b and head h at [b * dtable_sb + h] (dtable_sb >= Hq): the sum of
 * dS = P o (dP - D) over batch entries and all retained query-key pairs with that bucket, kept in fp32 and added up in a
 * fixed order.  With tau > 0 the backward tests and works tile by tile in one pass. */
int mala_fwd_bias(mala_tin q, mala_tin k, mala_tin v, const mala_rel_bias* bias, mala_tout o, float* lse,
                  const mala_stats* st, int B, int Hq, int Hkv, int Nq, int Nk, int d, int causal, float scale, float tau,
                  void* ws, size_t ws_bytes, void* cuda_stream);
int mala_bwd_bias(mala_tin q, mala_tin k, mala_tin v, mala_tin o, mala_tin dout, const float* lse,
                  const mala_rel_bias* bias, mala_tout dq, mala_tout dk, mala_tout dv, void* dtable, int64_t dtable_sb,
                  const mala_stats* st, int B, int Hq, int Hkv, int Nq, int Nk, int d, int causal, float scale, float tau,
                  void* ws, size_t ws_bytes, void* cuda_stream);

/* mala_fwd_varlen_prefix / mala_bwd_varlen_prefix with a bias (pass the same offsets twice for self attention).  A sequence
 * without keys (or, causal != 0, with more queries than keys) gets o = 0, lse = -inf and zero gradients. */
int mala_fwd_varlen_bias(mala_tin q, mala_tin k, mala_tin v, const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k,
                         const mala_rel_bias* bias, mala_tout o, float* lse, const mala_stats* st, int B, int Hq, int Hkv,
                         int total_q, int total_k, int max_seqlen_q, int max_seqlen_k, int d, int causal, float scale,
                         float tau, void* ws, size_t ws_bytes, void* cuda_stream);
int mala_bwd_varlen_bias(mala_tin q, mala_tin k, mala_tin v, mala_tin o, mala_tin dout, const float* lse,
                         const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, const mala_rel_bias* bias, mala_tout dq,
                         mala_tout dk, mala_tout dv, void* dtable, int64_t dtable_sb, const mala_stats* st, int B, int Hq,
                         int Hkv, int total_q, int total_k, int max_seqlen_q, int max_seqlen_k, int d, int causal,
                         float scale, float tau, void* ws, size_t ws_bytes, void* cuda_stream);

/* mala_decode_paged with a bias; a new token's position is that of its own key. */
int mala_decode_paged_bias(mala_tin q, mala_tin kpages, mala_tin vpages, const int32_t* block_table,
                           const int32_t* seqlens, const mala_rel_bias* bias, mala_tout o, float* lse_opt,
                           const mala_stats* st, int B, int Hq, int Hkv, int num_pages, int page_size,
                           int max_pages_per_seq, int Sq, int d, float scale, float tau, int num_splits, void* ws,
                           size_t ws_bytes, void* cuda_stream);

/* Scratch of the calls with a bias: op MALA_OP_FWD, MALA_OP_BWD or MALA_OP_DECODE; B sequences of up to Nq queries (decode: Sq)
 * and Nk keys; total_q: all query rows of packed sequences, 0 for the calls that are not packed; num_splits for
 * decode only.  Returns 0 for unsupported arguments. */
size_t mala_bias_workspace_bytes(int op, int B, int Hq, int Hkv, int Nq, int Nk, int total_q, int d, int num_splits,
                                 int num_buckets, int max_distance);

/* ---- Filling a paged cache ----------------------------------------------------------------------------------------
 * What the paged calls read, made on the GPU: a serving step of B requests releases the pages of finished requests, gives
 * the others pages for their new tokens, and writes the tokens' keys and values into them.  All pointers are device
 * pointers; nothing is read back to the host, so the calls can be captured in a CUDA graph.
 *
 * Pages are those of the paged calls (8, 16, 32, 64 or a multiple of 128 keys).  free_pages [num_pages] lists the free pages in its
 * first free_count[0] entries; pages are taken off its end and given back behind it.  No output may be an input's buffer
 * (block_table and free_pages apart): the next step reads what this one wrote.  B <= 16384, B * max_pages_per_seq
 * below 2^31, at most 2^30 rows in a call.
 *
 * mala_page_tables: request b holds seqlens[b] tokens, whose pages stand in the first ceil(seqlens[b] / page_size) entries of its
 * row of block_table [B, max_pages_per_seq], and gets new_tokens[b] more (below 0: none).
 *   block_table     the new pages are entered behind the old ones; page number x that the step hands out, in the order of the
 *                   requests, is free_pages[free_count[0] - 1 - x]
 *   cu_seqlens      [B + 1] first row of each request among the step's new tokens (the sum of new_tokens below 2^31: with more,
 *                   what the call gives has no meaning, but stays within its buffers)
 *   seqlens_out     [B] tokens that it holds afterwards
 *   slots           int64 [rows] for each new token page * page_size + place in the page; -1 in rows behind the last request
 *                   and for tokens without a place.  rows may be smaller or larger than the number of new tokens.
 *   free_count_out  [1] free pages that are left
 * A request that does not fit its row of the table, or that needs pages after the free ones have run out, gets none: its
 * seqlens_out is its seqlens and its slots are -1 (requests that need no page are served all the same). */
int mala_page_tables(const int32_t* seqlens, const int32_t* new_tokens, int32_t* block_table, const int32_t* free_pages,
                     const int32_t* free_count, int32_t* cu_seqlens, int32_t* seqlens_out, int64_t* slots,
                     int32_t* free_count_out, int B, int max_pages_per_seq, int page_size, int num_pages, int rows,
                     void* cuda_stream);

/* The pages of the requests with done[b] != 0 (bytes) go behind the free ones, request by request in the order of their
 * tables; their seqlens_out is 0, the others' their seqlens.  block_table is left as it is. */
int mala_release_pages(const uint8_t* done, const int32_t* seqlens, const int32_t* block_table, int32_t* free_pages,
                       const int32_t* free_count, int32_t* seqlens_out, int32_t* free_count_out, int B, int max_pages_per_seq,
                       int page_size, int num_pages, void* cuda_stream);

/* k, v: bf16 [rows, Hkv, d] views (sn = row stride, sh = head stride, sb ignored); row t goes to slot slots[t] of kpages, vpages
 * [num_pages, page_size, Hkv, d], rows whose slot is negative or beyond the pool nowhere.  d a multiple of 8 up to 256.
 * A slot stands for one row at most: one that is given twice holds, 8 columns by 8 columns, either row's. */
int mala_cache_write(mala_tin k, mala_tin v, const int64_t* slots, mala_tout kpages, mala_tout vpages, int rows, int Hkv,
                     int num_pages, int page_size, int d, void* cuda_stream);

/* The same into e4m3 pages with the scales of mala_decode_fp8_paged (kscale, vscale [num_pages, Hkv, max(1, page_size/128)]):
 * d a multiple of 16 up to 128, page_size not 8.  The keys that share a scale are a unit (a tile of 128, or a smaller page).
 * With m the largest magnitude among the unit's new rows of a head: a unit whose first key is among them gets the scale
 * m / 448 (1 where m is 0); in another one, which holds keys already, the scale s becomes max(s, m / 448), and where that is
 * larger the codes of the keys before the new ones are rounded again, e4m3(code * s_old / s_new).  New codes are
 * e4m3(x / s), rounded to nearest even.  Values must be finite.  The rows of a unit must be neighbours with consecutive
 * slots, as mala_page_tables gives them, and no other call may write to these units at the same time. */
int mala_cache_write_fp8(mala_tin k, mala_tin v, const int64_t* slots, mala_tout kpages8, mala_tout vpages8, float* kscale,
                         float* vscale, int rows, int Hkv, int num_pages, int page_size, int d, void* cuda_stream);

/* mala_page_tables that also gives the positions of the new tokens in their sequences: int32 [rows], 0 in rows without a slot. */
int mala_page_tables_positions(const int32_t* seqlens, const int32_t* new_tokens, int32_t* block_table, const int32_t* free_pages,
                               const int32_t* free_count, int32_t* cu_seqlens, int32_t* seqlens_out, int64_t* slots,
                               int32_t* positions, int32_t* free_count_out, int B, int max_pages_per_seq, int page_size,
                               int num_pages, int rows, void* cuda_stream);

/* ---- Reading a paged cache back -----------------------------------------------------------------------------------
 * Keys and values of B sequences out of their pages, packed one sequence behind the other: k_out, v_out bf16
 * [rows, Hkv, d] views (sn = row stride, sh = head stride, sb ignored), cu_seqlens [B + 1] (written) the first row of each.
 * kpages, vpages, block_table [B, max_pages_per_seq] and seqlens [B] as for mala_decode_paged / mala_fwd_paged; a length counts as
 * what its row of the table can map.  rows: room in the outputs, at least the sum of the lengths; of a sequence that reaches
 * beyond it only what fits is there, in cu_seqlens too.  A key whose page is not one of the pool's is 0.  The first 128 rows behind the last
 * sequence (as far as there are) are set to 0, so that the tiles of the packed calls may cover them; the others stay as they were.
 * d a multiple of 8 up to 256; B <= 16384 and at most 2^30 rows. */
int mala_cache_read(mala_tin kpages, mala_tin vpages, const int32_t* block_table, const int32_t* seqlens, mala_tout k_out,
                    mala_tout v_out, int32_t* cu_seqlens, int B, int Hkv, int num_pages, int page_size,
                    int max_pages_per_seq, int rows, int d, void* cuda_stream);

/* The same out of e4m3 pages with the scales of mala_decode_fp8_paged: bf16(scale * code), rounded once.  d a multiple of 16 up to 128,
 * page_size not 8. */
int mala_cache_read_fp8(mala_tin kpages8, mala_tin vpages8, const float* kscale, const float* vscale,
                        const int32_t* block_table, const int32_t* seqlens, mala_tout k_out, mala_tout v_out,
                        int32_t* cu_seqlens, int B, int Hkv, int num_pages, int page_size, int max_pages_per_seq, int rows,
                        int d, void* cuda_stream);

/* mala_fwd_paged over an e4m3 cache: keys and values are scale * code, not rounded on their way (the codes are multiplied, the scales come in
 * at the softmax; beyond 2^-60 .. 2^60, or not positive, bf16(scale * code)).  total_k: room for keys in the workspace, at least the sum of
 * seqlens_k (see mala_cache_read_fp8 for what lies beyond it: the sequences that reach beyond have no meaningful result).
 * A sequence's result is the same whatever the other sequences' keys and values are, infinities and NaNs among them.
 * Workspace: mala_paged_fp8_workspace_bytes.  d a multiple of 16 up to 128, page_size not 8, B <= 16384, total_k <= 2^30; everything else as
 * mala_fwd_paged; telemetry laid out for max_seqlen_k = min(max_pages_per_seq * page_size, total_k). */
int mala_fwd_paged_fp8(mala_tin q, mala_tin kpages8, mala_tin vpages8, const float* kscale, const float* vscale,
                       const int32_t* cu_seqlens_q, const int32_t* block_table, const int32_t* seqlens_k, mala_tout o,
                       float* lse, const mala_stats* st, int B, int Hq, int Hkv, int total_q, int max_seqlen_q, int total_k,
                       int num_pages, int page_size, int max_pages_per_seq, int d, int causal, float scale, float tau,
                       void* ws, size_t ws_bytes, void* cuda_stream);
/* 0 for unsupported arguments */
size_t mala_paged_fp8_workspace_bytes(int B, int Hkv, int total_k, int d);

/* mala_fwd_paged_fp8 with the keys of every sequence cut into num_splits ranges of ceil(ceil(seqlen_k/128)/num_splits) blocks that run on
 * different SMs, for few and short prompts behind long prefixes; test, merge and telemetry as in mala_fwd_chunk_split.
 * Workspace: mala_paged_fp8_split_workspace_bytes.  B * num_splits <= 65535.  num_splits = 1 is mala_fwd_paged_fp8; the suggested count
 * takes the lengths that the host knows, max_seqlen_k = min(max_pages_per_seq * page_size, total_k) (sm_count 0: the current device's). */
int mala_fwd_paged_fp8_split(mala_tin q, mala_tin kpages8, mala_tin vpages8, const float* kscale, const float* vscale,
                             const int32_t* cu_seqlens_q, const int32_t* block_table, const int32_t* seqlens_k, mala_tout o,
                             float* lse, const mala_stats* st, int B, int Hq, int Hkv, int total_q, int max_seqlen_q, int total_k,
                             int num_pages, int page_size, int max_pages_per_seq, int d, int causal, float scale, float tau,
                             int num_splits, void* ws, size_t ws_bytes, void* cuda_stream);
size_t mala_paged_fp8_split_workspace_bytes(int B, int Hq, int Hkv, int max_seqlen_q, int total_k, int d, int num_splits);
int mala_paged_fp8_suggest_splits(int B, int Hq, int max_seqlen_q, int max_seqlen_k, int total_k, int sm_count);

/* ---- Rotary positions ---------------------------------------------------------------------------------------------
 * The first `rotary` columns of a head's row (even, 2 .. d) are rotated in pairs by the angle position * inv_freq[i]: pair i is
 * the columns i and i + rotary / 2, or, interleaved != 0, 2 i and 2 i + 1:
 *     (y1, y2) -> magnitude * (y1 cos - y2 sin, y2 cos + y1 sin);   columns from rotary on stay as they are.
 * inv_freq: DEVICE pointer, doubles [rotary / 2], radians per position (scaled for long contexts or not); the struct itself is read during the
 * call.  Angles are exact to 2^-31 of a turn wherever the position lies, their cosines and sines to 2^-23.
 * norm (may be NULL): before its rotation each head's row is normed, y = x / sqrt(mean(x^2) + eps) * weight, over all d columns;
 * weights [d] on the device, bf16 or (weights_fp32 != 0) fp32, NULL: 1.  All arithmetic is fp32, rounded once to bf16.
 * d a multiple of 8 up to 256; at most 2^30 rows per tensor. */
typedef struct { const double* inv_freq; int rotary; int interleaved; float magnitude; } mala_rotary;
typedef struct { const void* q_weight; const void* k_weight; int weights_fp32; float eps; } mala_head_norm;

/* q, q_out [B,Nq,Hq,d]; k, k_out [B,Nk,Hkv,d] (k.p and k_out.p NULL: no keys).  The queries are the last Nq of the Nk positions, as in
 * mala_fwd_chunk.  positions: int32 [B,Nk], or NULL for 0 .. Nk - 1 (query row n of entry b has positions[b][n + Nk - Nq]); any
 * int32 value.  An output may be its own input (same view); otherwise they must not overlap. */
int mala_rotary_fwd(mala_tin q, mala_tin k, const int32_t* positions, const mala_rotary* rotary, const mala_head_norm* norm,
                    mala_tout q_out, mala_tout k_out, int B, int Nq, int Nk, int Hq, int Hkv, int d, void* cuda_stream);

/* Its gradients: dq, dk those of the outputs, dq_out, dk_out those of q and k (an output may be its own incoming gradient, not q or k).
 * With a norm: q, k as they went into mala_rotary_fwd, and dq_weight, dk_weight fp32 [d] (either may be NULL), overwritten with the weights'
 * gradients, summed over rows and heads in fp32 in a fixed order; ws of mala_rotary_workspace_bytes(d), 256-byte aligned (not needed where both
 * are NULL).  Without one q, k and ws are ignored and dq_weight, dk_weight must be NULL. */
int mala_rotary_bwd(mala_tin dq, mala_tin dk, mala_tin q, mala_tin k, const int32_t* positions, const mala_rotary* rotary,
                    const mala_head_norm* norm, mala_tout dq_out, mala_tout dk_out, float* dq_weight, float* dk_weight, int B,
                    int Nq, int Nk, int Hq, int Hkv, int d, void* ws, size_t ws_bytes, void* cuda_stream);

/* Packed sequences: q [1,total_q,Hq,d], k [1,total_k,Hkv,d], offsets as in mala_fwd_varlen_prefix (pass the same twice for self attention):
 * the key in row t of sequence b has position t - cu_seqlens_k[b], and its queries are the last positions.  Rows that no sequence has are copied
 * as they are (their gradients too) and have no part in the weights' gradients. */
int mala_rotary_fwd_varlen(mala_tin q, mala_tin k, const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k,
                           const mala_rotary* rotary, const mala_head_norm* norm, mala_tout q_out, mala_tout k_out, int B,
                           int Hq, int Hkv, int total_q, int total_k, int d, void* cuda_stream);
int mala_rotary_bwd_varlen(mala_tin dq, mala_tin dk, mala_tin q, mala_tin k, const int32_t* cu_seqlens_q,
                           const int32_t* cu_seqlens_k, const mala_rotary* rotary, const mala_head_norm* norm,
                           mala_tout dq_out, mala_tout dk_out, float* dq_weight, float* dk_weight, int B, int Hq, int Hkv,
                           int total_q, int total_k, int d, void* ws, size_t ws_bytes, void* cuda_stream);
size_t mala_rotary_workspace_bytes(int d);

/* A serving step in one call: q [rows,Hq,d] is rotated into q_out (which may be q itself), k [rows,Hkv,d] into its slots of kpages, v goes to its
 * slots of vpages (views, slots and pages as for mala_cache_write; rows without a slot: q_out only).  positions int32 [rows], as
 * mala_page_tables_positions gives them. */
int mala_rotary_write(mala_tin q, mala_tin k, mala_tin v, const int32_t* positions, const int64_t* slots,
                      const mala_rotary* rotary, const mala_head_norm* norm, mala_tout q_out, mala_tout kpages,
                      mala_tout vpages, int rows, int Hq, int Hkv, int num_pages, int page_size, int d, void* cuda_stream);

/* The same into e4m3 pages, by the rules of mala_cache_write_fp8 (on the rotated keys in fp32: codes and scales are rounded once, not
 * behind a rounding to bf16). */
int mala_rotary_write_fp8(mala_tin q, mala_tin k, mala_tin v, const int32_t* positions, const int64_t* slots,
                          const mala_rotary* rotary, const mala_head_norm* norm, mala_tout q_out, mala_tout kpages8,
                          mala_tout vpages8, float* kscale, float* vscale, int rows, int Hq, int Hkv, int num_pages,
                          int page_size, int d, void* cuda_stream);

/* Decode for callers that cannot allocate device memory.  (The paper has no counterpart: this entry point
 * exists for integration reasons only and computes exactly what mala_decode computes.)
 *
 * Some callers of this library have no way to obtain scratch memory at the point of the call: code
 * that runs inside a serving engine's pre-sized memory plan where every byte of the device pool is
 * already assigned, a plug-in that receives only its input and output buffers from the host framework,
 * or a latency-critical path that must not touch an allocator (cudaMalloc synchronises the device and
 * may fail under fragmentation).  For them this variant keeps the split partials -- the only scratch
 * the decode path needs -- in an array that is part of the library image: MALA_STATIC_SCRATCH_BYTES of
 * global memory on every GPU that loads the library, held until the process exits.  The caller still
 * passes all inputs and outputs; the call itself allocates nothing and frees nothing.
 *
 * Limits and rules
 *   - mala_workspace_bytes(MALA_OP_DECODE, ...) for the same arguments must not exceed
 *     MALA_STATIC_SCRATCH_BYTES; otherwise nothing is launched and
 *     MALA_ERR_STATIC_SCRATCH_EXCEEDED is returned (use fewer splits, or mala_decode with your own ws).
 *   - All calls on one device share the one array.  Two calls whose kernels can overlap on the GPU
 *     (different streams, or different host threads on different streams) race on it and give wrong
 *     results: keep calls on a device in one stream, or order them with events.  The array keeps the
 *     previous call's contents between calls; the kernels overwrite every entry they later read, so no
 *     clearing is needed.
 *   - The first call on each device looks up the array's device address (a one-time
 *     cudaGetSymbolAddress with that device current).  Make that first call outside any stream capture.
 *   - No telemetry (mala_stats) is available through this entry point.
 * Arguments, layouts, result and error codes otherwise as mala_decode. */
int mala_decode_static(mala_tin q, mala_tin kcache, mala_tin vcache, mala_tout o, float* lse_opt, int B, int Hq,
                       int Hkv, int Nk, int d, float scale, float tau, int num_splits, void* cuda_stream);

/* A split count for mala_decode and its variants (host only; nothing is launched).  The skip test of a split sees
 * only that split's partial normalizer ("Fused decoding execution"), so it passes more often the longer the split:
 * the best count is the SMALLEST one that still spreads the B * Hkv * num_splits work items evenly over the SMs.
 * Items differ in how many tiles they retain, so an SM needs several of them to even that out.
 * Returned: the smallest S with at least six items per SM and at least two tiles per split (without the first
 * condition where the two cannot both hold) whose longest per-SM queue, ceil(B*Hkv*S / sm_count) items of
 * ceil(ceil(Nk/128) / S) tiles each, is within 4 % of the shortest such queue any admissible S gives.
 * Nk: the (longest) cache length; sm_count <= 0: the current device's SM count is used.
 * Returns the count (>= 1) or a negative MALA_ERR_* code. */
int mala_decode_suggest_splits(int B, int Hkv, int Nk, int sm_count);

/* Scratch bytes needed by one call of `op` (MALA_OP_*); N is Nk for decode; num_splits is ignored
 * for fwd / bwd.  Returns 0 for unsupported arguments. */
size_t mala_workspace_bytes(int op, int B, int Hq, int Hkv, int N, int d, int num_splits);

/* Tile partition of `op` for head size d: Bq query rows x Bk keys.  For decode Bq is reported as 0
 * (the rows are the Hq/Hkv packed query heads).  Returns MALA_OK or MALA_ERR_UNSUPPORTED. */
int mala_tile_shape(int op, int d, int* Bq, int* Bk);

/* Reads the current device's status word into *code_out (MALA_OK or MALA_ERR_DEVICE_TIMEOUT) and, if
 * clear != 0, resets it.  Synchronises the device.  HOST pointer. */
int mala_device_status(int* code_out, int clear);

/* ---- Test support (not part of the operator) ------------------------------------------------------------------
 * Every wait inside the kernels is bounded (Conventions, last item).  This call makes one such wait run out on
 * purpose, in the only way that harms nothing: it launches a single small thread block whose one waiting thread
 * polls, with the kernels' own wait routine, a barrier that nobody ever arrives on, gives up after limit_cycles
 * clock cycles (1 .. 1e8; the kernels themselves use about 2 s), records MALA_ERR_DEVICE_TIMEOUT in the device's
 * status word and returns through the normal exit.  Nothing faults, traps or waits without a limit.  Afterwards
 * mala_device_status reports the code, and every later launch of this library on the device returns at once
 * without touching its outputs until the word is cleared (mala_device_status with clear != 0).
 * Asynchronous on cuda_stream; MALA_OK or a negative MALA_ERR_* code (MALA_ERR_INVALID_ARG for a limit out of range). */
int mala_test_expire_wait(long long limit_cycles, void* cuda_stream);

const char* mala_strerror(int code);
int mala_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MALA_H_ */
