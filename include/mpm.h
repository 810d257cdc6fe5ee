/*
 * mpm.h -- C ABI of the Mutual Pair Merging (MPM) token-reduction path,
 * implemented with hand-written HIP kernels for MI355X (gfx950, CDNA4).
 *
 * MPM (arXiv 2604.05718, Sec. 3.2, Alg. 1) reduces the N x D image tokens of a
 * ViT block input:
 *   1. normalise each token to unit L2 norm and form the cosine affinity
 *      S = Xn Xn^T with the diagonal excluded (Eq. 1);
 *   2. b(i) = argmax_{j != i} S_ij;
 *   3. keep the mutual pairs (b(b(i)) = i), lower index as representative;
 *   4. give clusters (pairs and singletons) compact ids r(i) by a
 *      left-to-right scan (Alg. 1), partners inherit the representative's id;
 *   5. replace each cluster by the mean of its members (Eq. 2).
 * Merge maps of successive insertions compose as r*(i) = r2(r1(i)) (Eq. 3),
 * and the full grid is rebuilt by a gather Z_up[i] = Z[r*(i)] (Eq. 4).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - All array pointers are DEVICE pointers owned by the caller. The library
 *   allocates and frees nothing.
 * - Every call is asynchronous on `stream` (a hipStream_t; NULL = the null
 *   stream) and never synchronises the host. Counts and offsets stay on the
 *   device; the caller reads them when it needs them.
 * - Token rows are D contiguous elements; rows are 16-byte aligned
 *   (D % 8 == 0 for bfloat16, D % 4 == 0 for float32) and base pointers are
 *   16-byte aligned.
 * - A batch holds B images of at most N tokens each. Token rows are either
 *   DENSE (offsets pointer NULL: image b owns rows [b*N, b*N + N)) or PACKED
 *   (offsets pointer = device int32[B+1], image b owns rows
 *   [off[b], off[b+1]), n_b = off[b+1] - off[b] with 0 <= n_b <= N, offsets
 *   non-decreasing). An empty image (n_b = 0) gets no merged rows and a map of
 *   -1. Packed offsets are data on the device; violating these rules is
 *   undefined behaviour, not a reported error.
 * - Per-token integer arrays (nb, map) use a [B][N] slot layout: entry
 *   b*N + i belongs to token i of image b, for i < n_b. Ids are 0-based and
 *   image-local.
 * - Ties: the argmax keeps the lowest index j among equal scores.
 * - `schedule` (an mpm_schedule value) picks the affinity kernel's work
 *   decomposition for that call only; results never depend on it.
 * - Argument errors are reported synchronously, before anything is launched:
 *     MPM_ERR_INVALID_ARG  null or misaligned pointer, B < 1, N < 1, D < 1,
 *                          D not a multiple of 8 (bf16) / 4 (f32), bad dtype,
 *                          unknown schedule;
 *     MPM_ERR_UNSUPPORTED  N above MPM_MAX_N, B above MPM_MAX_B, D above MPM_MAX_D;
 *     MPM_ERR_WORKSPACE    workspace smaller than mpm_workspace_bytes;
 *     MPM_ERR_HIP          a launch failed; mpm_last_hip_error() holds the
 *                          hipError_t (per host thread).
 *   Device-side faults surface at the caller's next synchronisation.
 * - Results are deterministic: the same inputs give bitwise-identical outputs.
 * - Reentrant: no mutable global state besides the per-thread last HIP error
 *   and, for mpm_merge_noalloc and the checked mode below, the device address of
 *   a library array per GPU (set once). Calls that share a workspace must be
 *   ordered (one stream, or events).
 * - Fault injection: with MPM_FAULT_INJECT=launch in the environment (read once,
 *   at the first call), every entry point that would launch a kernel returns
 *   MPM_ERR_HIP with hipErrorLaunchFailure recorded, after its argument checks and
 *   before any HIP call, so that callers' error paths can be tested without a GPU.
 * - Checked mode (debugging): with MPM_CHECKED=1 in the environment (read once, at
 *   the first call), every entry point also validates on the device the data
 *   preconditions that are otherwise undefined behaviour, before launching its
 *   operation: packed offsets (0 <= n_b <= N; merged-row offsets also at most the
 *   tokens they come from, within B*N rows; the padded layout's any n_b >= 0), token
 *   values and given inverse norms (finite; norms positive), grid positions (in
 *   range, rows non-decreasing), neighbours (in [0, n_b), not the token itself, -1
 *   for a one-token image), merged-row sources (in [0, n_b)) and maps (in [-1, N),
 *   or [-1, n_z) where they index merged rows). Offsets are validated first; the
 *   rows they address must exist. On a violation the call returns
 *   MPM_ERR_INVALID_ARG and launches nothing of its operation (mpm_run_schedule
 *   checks each insertion's input so, and may have run those before it). A checked call
 *   synchronises its stream (it reads the verdict back; so not under graph
 *   capture), and checked calls are serialised by a lock. Without the variable
 *   nothing of this runs.
 */
#ifndef MPM_H
#define MPM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MPM_OK = 0,
    MPM_ERR_INVALID_ARG = 1,
    MPM_ERR_UNSUPPORTED = 2,
    MPM_ERR_WORKSPACE = 3,
    MPM_ERR_HIP = 4
} mpm_status;

typedef enum {
    MPM_F32 = 0,   /* float32 storage, float32 arithmetic */
    MPM_BF16 = 1   /* bfloat16 storage, float32 accumulation */
} mpm_dtype;

/*
 * Work schedule of the affinity kernel. The affinity of an image is symmetric
 * (Eq. 1), so MPM_SCHEDULE_SYMMETRIC computes only the 256 x 256 blocks on and
 * above the block diagonal and takes each off-diagonal block's argmax in both
 * directions (about half the matrix-core work for large images, for a
 * cross-lane reduction per block); when an XCD group's blocks would leave a
 * last round on at most half of its workgroups (rows a whole number of
 * 128-byte chunks), that many diagonal blocks run in a second launch as two
 * halves of their queries each. MPM_SCHEDULE_FULL_64 computes every pair of
 * 64 x 64 blocks, so that a small batch (a single image of 1024 tokens has 16
 * blocks of 256 x 256 but 256 of 64 x 64) still occupies every compute unit.
 * MPM_SCHEDULE_AUTO takes the 64 x 64 blocks for small batches (at most 32
 * blocks of 256 x 256 among them), else whichever of the symmetric schedule (on
 * 256 x 256 or, where those would leave compute units idle, 128 x 128 blocks)
 * and the full one an estimate of the launch finds faster. The choice applies
 * to rows whose byte length is a multiple of 64; for other rows the library
 * always picks. The partials (and everything reduced from them) are
 * bit-identical under every schedule.
 */
typedef enum {
    MPM_SCHEDULE_AUTO = 0,
    MPM_SCHEDULE_FULL = 1,      /* every (query block, candidate tile) pair of 256 x 256 */
    MPM_SCHEDULE_SYMMETRIC = 2, /* pairs on and above the block diagonal only */
    MPM_SCHEDULE_FULL_64 = 3    /* every pair of 64 x 64 blocks (small batches) */
} mpm_schedule;

#define MPM_MAX_N 16384   /* tokens per image */
#define MPM_MAX_B 65535   /* images per call */
#define MPM_MAX_D 16384   /* channels per token */

/* Library version string, e.g. "mpm 0.3.0 gfx950". Never NULL. (0.3.0: mpm_attention_call and mpm_norm_call have
 * fields at their end that say what becomes of rows of no image; zeros there are the calls as they were.) */
const char* mpm_version(void);

/* Human-readable name of a status code. Never NULL. */
const char* mpm_status_string(int status);

/* hipError_t of the last MPM_ERR_HIP returned on this host thread (0 if none). */
int mpm_last_hip_error(void);

/*
 * Device workspace of mpm_affinity, mpm_affinity_compact, mpm_argmax and
 * mpm_merge: bytes needed for a batch of B images of at most N tokens. The
 * caller allocates it (256-byte aligned) and owns it; calls ordered on one
 * stream may reuse it, for any B and N it is large enough for. Layout, as byte
 * offsets returned by mpm_workspace_offsets (each 256-byte aligned):
 *   sync  int32[MPM_MAX_B + 1]  arrival counters of the fused compaction
 *                               (always at offset 0, the same for every shape);
 *   nb    int32[B*N]            nearest neighbour per token (slot layout);
 *   src   int32[2*B*N]          (representative, partner) of cluster k of image
 *                               b at 2*(b*N + k) (partner == representative for
 *                               a singleton);
 *   pv    float[B*T*N], pi int32[B*T*N]  per-candidate-tile argmax partials,
 *                               T = ceil(N / 64) slots per token: tile t of image b
 *                               for token i at (b*T + t)*N + i; a launch fills the
 *                               first ceil(n_b / w) slots, w = the block width it
 *                               runs (mpm_affinity_block_rows).
 * A workspace needs no preparation: each call sets what it counts in to zero
 * first, and leaves the words of the sync region that it used zero (an
 * interrupted call may not). Returns 0 for B < 1 or N < 1.
 */
size_t mpm_workspace_bytes(int32_t B, int32_t N);

/* Byte offsets of the workspace regions listed above; any pointer may be NULL.
 * Returns MPM_OK, or MPM_ERR_INVALID_ARG for B < 1 or N < 1. */
int mpm_workspace_offsets(int32_t B, int32_t N, size_t* sync, size_t* nb, size_t* src, size_t* pv, size_t* pi);

/*
 * Zeroes the sync region of a workspace of ws_bytes bytes (at least the
 * region's 256 KB) with a fill kernel on `stream` (no memset node, so it may
 * be captured in a HIP graph). Not needed: calls clear the words they use.
 */
int mpm_workspace_init(void* ws, size_t ws_bytes, void* stream);

/*
 * Cosine affinity and its self-masked row argmax, per candidate tile (Eq. 1
 * and the argmax of Sec. 3.2), into the workspace partials: for every query i
 * and candidate tile t, the best score (x_i . x_j) / max(||x_j||, 1e-12) over
 * the tile's candidates j != i, j < n_b, and that j (lowest j among equal
 * scores). The dot products are accumulated in float32 on MFMA from the
 * stored values (bfloat16 products are exact in float32); the N x N affinity
 * is never written to memory. Dividing by ||x_i|| too would not move the
 * argmax of row i, so it is not applied.
 *   x, x_off: rows of dtype `dt`, dense or packed;
 *   x_inv (may be NULL): the inverse row norms 1 / max(||x_r||, 1e-12), one
 *     float per row of x (packed like x; rows past an image's end are not
 *     read), given instead of summed in the kernel's K loop (about a tenth of
 *     its time), as mpm_pair_average writes them for the next insertion's
 *     input (Sec. 3.3). Bfloat16 rows whose byte length is a multiple of 64
 *     only: other rows return MPM_ERR_UNSUPPORTED with a non-NULL x_inv;
 *   start_event / stop_event (may be NULL): hipEvent_t the caller created
 *     (timing enabled) and owns, bound to the kernels' own dispatches
 *     (hipExtLaunchKernel): start to the first launch, stop to the last, so
 *     hipEventElapsedTime(start, stop) is the step's duration on the device
 *     without extra stream commands. The step is one launch, or two when the
 *     symmetric schedule runs deferred diagonal blocks in a second launch.
 */
int mpm_affinity(const void* x, const int32_t* x_off, const float* x_inv, int32_t B, int32_t N, int32_t D,
                 int32_t dt, int32_t schedule, void* ws, size_t ws_bytes, void* start_event, void* stop_event,
                 void* stream);

/*
 * One insertion's affinity step and compaction step (Sec. 3.2, Alg. 1 steps 2-6)
 * in one call: mpm_affinity, then the compaction kernel, which reduces each
 * image's partials to nb (larger score, then smaller index; images with more
 * than a few candidate tiles are reduced by a separate parallel launch first),
 * tests the pairs for mutuality, marks representatives and assigns compact ids
 * by a left-to-right scan, one workgroup per image. Each image's workgroup adds
 * its cluster count to the offsets of the images after it (y_off is cleared by
 * the affinity launch, so it must not alias x_off); beyond 256 images the one
 * that finishes the last image (found with the arrival counter in the
 * workspace's sync region, no waiting) turns the counts into offsets. Writes
 *   map[b*N + i] = r(i) for i < n_b, -1 for n_b <= i < N;
 *   y_off[0] = 0, y_off[b+1] = y_off[b] + n'_b (int32[B+1]);
 *   the workspace's nb and src regions (src read by mpm_pair_average).
 * The timing events are bound to the affinity kernel's dispatches only.
 * Arguments as mpm_affinity otherwise.
 */
int mpm_affinity_compact(const void* x, const int32_t* x_off, const float* x_inv, int32_t B, int32_t N, int32_t D,
                         int32_t dt, int32_t schedule, int32_t* map, int32_t* y_off, void* ws, size_t ws_bytes,
                         void* start_event, void* stop_event, void* stream);

/*
 * The schedule (MPM_SCHEDULE_FULL, MPM_SCHEDULE_SYMMETRIC or
 * MPM_SCHEDULE_FULL_64, never AUTO) that mpm_affinity runs for B images of at
 * most N tokens of D channels of dtype dt under `schedule` on the current
 * device, written to *used (a host pointer). For reporting the matrix-core
 * work a call issues: about 2 * w^2 * D flops per w x w block, nb^2 blocks per
 * image of nb = ceil(n_b / w) blocks under the full schedules and nb (nb + 1) / 2
 * under the symmetric one, w = mpm_affinity_block_rows. This is the schedule of a call
 * without offsets, and MPM_SCHEDULE_FULL for rows whose byte length is not a multiple of
 * 64, which do not take the argument; mpm_affinity_plan reports what any call runs.
 * Returns MPM_OK, MPM_ERR_INVALID_ARG for bad sizes, an unknown schedule or a NULL
 * pointer, or MPM_ERR_HIP when the device cannot be queried.
 */
int mpm_affinity_schedule_used(int32_t B, int32_t N, int32_t D, int32_t dt, int32_t schedule, int32_t* used);

/*
 * The rows of the square blocks mpm_affinity runs for B images of at most N tokens of D
 * channels of dtype dt under `schedule` on the current device, without offsets
 * (packed = 0) or with them, written to *rows (a host pointer): 64, 128 or 256. This is
 * the token width w of one partial in the workspace. For reporting. Returns MPM_OK,
 * MPM_ERR_INVALID_ARG for bad sizes, an unknown schedule or a NULL pointer, or
 * MPM_ERR_HIP when the device cannot be queried.
 */
int mpm_affinity_block_rows(int32_t B, int32_t N, int32_t D, int32_t dt, int32_t schedule, int32_t packed,
                            int32_t* rows);

/*
 * What mpm_affinity runs for such a call, rows of any width, without offsets (packed = 0)
 * or with them: the schedule to *used (MPM_SCHEDULE_FULL, MPM_SCHEDULE_SYMMETRIC or
 * MPM_SCHEDULE_FULL_64) and the rows of its square blocks to *rows, as
 * mpm_affinity_block_rows. Returns as mpm_affinity_block_rows.
 */
int mpm_affinity_plan(int32_t B, int32_t N, int32_t D, int32_t dt, int32_t schedule, int32_t packed, int32_t* used,
                      int32_t* rows);

/*
 * The block size mpm_merge_local's affinity runs for this shape, window and requested
 * block_rows on the current device, written to *rows (a host pointer): 256 or 128
 * (square blocks on the symmetric schedule; with block_rows 0, whichever an estimate of
 * the launch on a full raster grid of grid_w columns, at this window, finds faster), or
 * N for rows whose byte length is not a multiple of 64, which do not take the argument
 * (mpm_local_tile_rows reports their blocks too). For reporting. Returns MPM_OK,
 * MPM_ERR_INVALID_ARG for bad sizes, grid_w, window or block_rows (as mpm_merge_local) or
 * a NULL pointer, or MPM_ERR_HIP when the device cannot be queried.
 */
int mpm_local_block_rows(int32_t B, int32_t N, int32_t D, int32_t dt, int32_t grid_w, int32_t window,
                         int32_t block_rows, int32_t* rows);

/*
 * The rows of the square blocks mpm_merge_local's affinity runs, and the token width of one
 * partial in its workspace, for rows of any width: 128 or 256. Otherwise as
 * mpm_local_block_rows.
 */
int mpm_local_tile_rows(int32_t B, int32_t N, int32_t D, int32_t dt, int32_t grid_w, int32_t window,
                        int32_t block_rows, int32_t* rows);

/*
 * Nearest neighbours: mpm_affinity (norms summed in the kernel), then the
 * reduction of the partials.
 *   nb[b*N + i] = argmax_{j != i, j < n_b} cos(x_i, x_j), lowest j on equal
 *                 scores; -1 when n_b == 1. Entries i >= n_b are not written.
 *   best[b*N + i] (optional, may be NULL) = the float32 cosine of that pair.
 * nb and best are caller arrays (not the workspace).
 */
int mpm_argmax(const void* x, const int32_t* x_off, int32_t B, int32_t N, int32_t D, int32_t dt, int32_t schedule,
               int32_t* nb, float* best, void* ws, size_t ws_bytes, void* stream);

/*
 * Mutual pairs and compact ids (Sec. 3.2, Alg. 1) from given neighbours nb
 * (slot layout, values in [0, n_b) or -1 for n_b == 1).
 *   map[b*N + i] = r(i) for i < n_b, -1 for n_b <= i < N;
 *   src[2*(b*N + k)], src[2*(b*N + k) + 1] = (representative, partner) of
 *     cluster k < n'_b (partner == representative for a singleton);
 *   y_off[0] = 0, y_off[b+1] = y_off[b] + n'_b.
 * x_off: the offsets of the tokens nb was computed on (NULL = dense, n_b = N).
 * Two launches (one workgroup per image, then the offsets).
 */
int mpm_pair_compact(const int32_t* nb, const int32_t* x_off, int32_t B, int32_t N, int32_t* map, int32_t* src,
                     int32_t* y_off, void* stream);

/*
 * Cluster means (Eq. 2), packed by the offsets the compaction wrote:
 *   y[y_off[b] + k] = mean of the rows src names for cluster k of image b,
 *     computed in float32 and rounded once (nearest even) to `dt`; a
 *     singleton is copied bit for bit;
 *   y_inv (optional, may be NULL): y_inv[y_off[b] + k] = 1 / max(||y_k||, 1e-12)
 *     from the stored values of y in float32, summed in a fixed order (the same
 *     on every run): the x_inv of y for the next insertion's affinity.
 * src in the slot layout above (the workspace's src region after
 * mpm_affinity_compact, or mpm_pair_compact's output); y has room for
 * y_off[B] rows (at most B*N). x as in mpm_affinity.
 */
int mpm_pair_average(const void* x, const int32_t* x_off, const int32_t* src, const int32_t* y_off, int32_t B,
                     int32_t N, int32_t D, int32_t dt, void* y, float* y_inv, void* stream);

/*
 * One MPM insertion (Alg. 1) = mpm_affinity_compact, then mpm_pair_average
 * (src from the workspace), in order on `stream`.
 *   x, x_off, x_inv: input tokens (dense or packed) and optional given inverse
 *       norms, as in mpm_affinity;
 *   y, y_off: merged tokens, packed (capacity B*N rows), offsets int32[B+1];
 *   y_inv (may be NULL): inverse norms of the merged rows, as in mpm_pair_average;
 *   map: int32[B*N] merge map in slot layout (-1 beyond n_b);
 *   ws: workspace of at least mpm_workspace_bytes(B, N) bytes; nb and src are
 *       readable there after the call.
 * Feed (y, y_off, y_inv) as (x, x_off, x_inv) of the next insertion.
 */
int mpm_merge(const void* x, const int32_t* x_off, const float* x_inv, int32_t B, int32_t N, int32_t D, int32_t dt,
              int32_t schedule, void* y, int32_t* y_off, float* y_inv, int32_t* map, void* ws, size_t ws_bytes,
              void* stream);

/*
 * One locality-constrained insertion: mpm_merge with the candidates of each token
 * restricted to a window around it on the token grid, the mitigation of the
 * quadratic affinity that the paper proposes (Sec. 5, also Sec. 4.3). A token's
 * position is its raster index on a grid of grid_w columns (row = pos / grid_w,
 * column = pos % grid_w):
 *   x_inv (may be NULL): given inverse norms of the rows of x, as in mpm_affinity;
 *   y_inv (may be NULL): inverse norms of the merged rows, as in mpm_pair_average;
 *   pos (may be NULL): int32 per row of x, packed like x; NULL means each token's
 *       index in its image (the raster order of a full grid, as for a first
 *       insertion); positions must be non-decreasing in row along each image;
 *   window >= 0: j is a candidate of i when |row_i - row_j| <= window and
 *       |col_i - col_j| <= window;
 *   block_rows: 0, 128 or 256: the rows of the square blocks the affinity runs in
 *       (0: the library's pick, as mpm_local_block_rows reports); results never
 *       depend on it;
 *   nb[i] = argmax over the candidates of the cosine (lowest j on equal scores), or
 *       -1 when the window holds no other token (i is then a singleton);
 *   y_pos[y_off[b] + k] = the position of cluster k's representative (int32, packed
 *       like y): the pos of the merged rows for the next insertion, which keeps the
 *       raster order since ids follow the left-to-right scan.
 * Feed (y, y_off, y_inv, y_pos) as (x, x_off, x_inv, pos) of the next insertion.
 * Only the candidate tiles a query block's window reaches are computed. The
 * workspace as in mpm_merge (nb and src readable after the call). start_event /
 * stop_event (may be NULL) are bound to the affinity kernel's dispatch, as in
 * mpm_affinity. Errors as mpm_merge, plus MPM_ERR_INVALID_ARG for grid_w < 1,
 * grid_w > MPM_MAX_N, window < 0 or another block_rows. Positions outside
 * [0, grid_w * MPM_MAX_N) are undefined behaviour.
 */
int mpm_merge_local(const void* x, const int32_t* x_off, const float* x_inv, const int32_t* pos, int32_t B,
                    int32_t N, int32_t D, int32_t dt, int32_t grid_w, int32_t window, int32_t block_rows, void* y,
                    int32_t* y_off, float* y_inv, int32_t* y_pos, int32_t* map, void* ws, size_t ws_bytes,
                    void* start_event, void* stop_event, void* stream);

/* The buffers of one insertion of mpm_run_schedule, as mpm_merge's arguments of the same
 * names: y_inv may be NULL (the last insertion's is not written); y_pos is used (and needed)
 * under the locality constraint only; nb and src are readable in ws after the call. */
typedef struct mpm_insertion {
    void* y;
    int32_t* y_off;
    float* y_inv;
    int32_t* y_pos;
    int32_t* map;
    void* ws;
} mpm_insertion;

/*
 * A whole schedule in one call: `insertions` (1 to 3) insertions with identity blocks in
 * between (Sec. 3.3), the first on the dense tokens x, each next one on the packed rows,
 * norms and positions of the one before; the composed map (Eq. 3) and the gather back to the
 * grid (Eq. 4):
 *   window < 0: each insertion as mpm_merge(..., schedule, ...) (grid_w, block_rows not used);
 *   window >= 0: each as mpm_merge_local(..., grid_w, window, block_rows, ...);
 *   ins[s]: insertion s's buffers, whose workspaces (ws_bytes bytes each) must not overlap;
 *   rstar: the composed map, int32[B*N] in slot layout (not used, may be NULL, with one
 *       insertion, whose map is the composed one);
 *   out: [B][N][D], out[b][i] = the last insertion's merged row of token i.
 * Results are those of the separate calls, bit for bit. The last pair average writes the
 * merged rows and the grid in one pass. Errors as mpm_merge and mpm_merge_local, plus
 * MPM_ERR_INVALID_ARG for insertions < 1 or overlapping workspaces and MPM_ERR_UNSUPPORTED
 * for more than 3 insertions. In checked mode each insertion's input is validated before that
 * insertion, as the separate calls do: x before anything is launched; where finite tokens
 * overflow in a merged row or its norm, the next insertion is refused, with the buffers of the
 * insertions before it written and the others, rstar and out, not.
 */
int mpm_run_schedule(const void* x, int32_t B, int32_t N, int32_t D, int32_t dt, int32_t schedule, int32_t grid_w,
                     int32_t window, int32_t block_rows, const mpm_insertion* ins, int32_t insertions,
                     size_t ws_bytes, int32_t* rstar, void* out, void* stream);

/*
 * Padded batch layout (the paper pads each batch to its longest image, Sec. 4.2): the
 * packed rows of B images (offsets z_off, int32[B+1], as the merges write them) to a
 * dense [B][P][row_bytes] array, image b's rows first and zero rows after them:
 *   out[b][k] = z[z_off[b] + k] for k < min(n_b, P), zeros for n_b <= k < P.
 * For the parts of a model that need equal-length images (batched attention with a
 * key mask), while the per-token parts keep the packed rows. Rows are copied as
 * bytes: row_bytes a positive multiple of 16 (any dtype, several heads' features in
 * one row, ...). P is the caller's choice, usually the batch's largest n_b (read from
 * z_off) or N. Errors: MPM_ERR_INVALID_ARG for B < 1, P < 1, a row size that is not a
 * positive multiple of 16 or bad pointers; MPM_ERR_UNSUPPORTED for B, P or rows above
 * the maxima (MPM_MAX_B, MPM_MAX_N, 4 * MPM_MAX_D bytes).
 */
int mpm_pad(const void* z, const int32_t* z_off, int32_t B, int32_t P, int32_t row_bytes, void* out, void* stream);

/* The inverse of mpm_pad: z[z_off[b] + k] = padded[b][k] for k < min(n_b, P); padded
 * rows k >= n_b are not read. Arguments and errors as mpm_pad. */
int mpm_unpad(const void* padded, const int32_t* z_off, int32_t B, int32_t P, int32_t row_bytes, void* z,
              void* stream);

/*
 * mpm_merge for callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation): the workspace
 * is a file-scope device array of MPM_NOALLOC_SCRATCH_BYTES that each GPU the
 * library runs on holds until the process ends; its address is looked up on the
 * first call on a GPU, whose stream also gets one small fill kernel that clears
 * its arrival counters. No call allocates or frees anything (no hipMalloc,
 * hipFree or allocating library routine). Shapes whose mpm_workspace_bytes(B, N)
 * exceed the array return MPM_ERR_WORKSPACE (B = 64 at N = 1024, B = 16 at
 * N = 4096 and B = 32 at N = 2304 fit). Every call on a GPU shares that GPU's
 * array and leaves its arrival counters zero, but its other contents are the last
 * call's: calls that overlap on one GPU (several streams or threads) race and give
 * wrong results, so order them. Arguments, results and other errors as mpm_merge
 * (without the workspace, so nb and src are not readable).
 */
#define MPM_NOALLOC_SCRATCH_BYTES (48u << 20)
int mpm_merge_noalloc(const void* x, const int32_t* x_off, const float* x_inv, int32_t B, int32_t N, int32_t D,
                      int32_t dt, int32_t schedule, void* y, int32_t* y_off, float* y_inv, int32_t* map, void* stream);

/*
 * Composition of merge maps (Eq. 3): map_ab[b*N + i] = map_b[b*N + map_a[b*N + i]],
 * or -1 where map_a[b*N + i] < 0. Both maps in slot layout; map_a's values
 * index image b's entries of map_b. map_ab may alias map_a.
 */
int mpm_compose(const int32_t* map_a, const int32_t* map_b, int32_t B, int32_t N,
                int32_t* map_ab, void* stream);

/*
 * Gather reconstruction (Eq. 4) with E special rows in front.
 *   out is dense [B][E + N][D];
 *   out[b][e]     = z_spec[b][e]                   for e < E (z_spec [B][E][D]; may be NULL iff E == 0);
 *   out[b][E + i] = z[z_off[b] + map[b*N + i]]     for map >= 0 (bit copy),
 *                   zeros                          where map < 0.
 * z, z_off: merged rows, packed (z_off NULL = dense [B][N][D] rows).
 */
int mpm_unmerge(const void* z, const int32_t* z_off, const int32_t* map, const void* z_spec, int32_t E,
                int32_t B, int32_t N, int32_t D, int32_t dt, void* out, void* stream);

/*
 * Composition folded into the gather (Eq. 3 and Eq. 4 in one pass over the grid):
 *   r*(i) = map_b[b*N + map_a[b*N + i]], or -1 where map_a[b*N + i] < 0;
 *   out as mpm_unmerge with map = r*;
 *   map_ab (optional, may be NULL) receives r* in slot layout.
 * map_ab must not alias map_a or map_b (MPM_ERR_INVALID_ARG if it does). Other
 * arguments and errors as mpm_unmerge and mpm_compose.
 */
int mpm_compose_unmerge(const void* z, const int32_t* z_off, const int32_t* map_a, const int32_t* map_b,
                        int32_t* map_ab, const void* z_spec, int32_t E, int32_t B, int32_t N, int32_t D, int32_t dt,
                        void* out, void* stream);

/* ---- The blocks between the merges: attention over packed images with a learned relative
 * position bias, and the norms around a block. Conventions as above; NaN and infinities in the
 * inputs flow through as in the formulas (checked mode validates the offsets only). ---- */

#define MPM_MAX_HEADS 1024   /* query heads of an attention call */
#define MPM_MAX_HEAD_DIM 128 /* channels of a head */
#define MPM_MAX_SPAN 63      /* largest axis offset with a bias of its own */

/* Rows of several heads: head j of row r is dh contiguous elements at p + r * row + j * head
 * (strides in elements, each a whole number of 16 bytes, >= 0; p 16-byte aligned). Views into the
 * rows of one fused projection are taken as they are. */
typedef struct mpm_heads {
    void* p;
    int64_t row;
    int64_t head;
} mpm_heads;

/*
 * The shape and the optional inputs of an attention call.
 *   B images; queries dense (q_off NULL: Nq rows an image) or packed (q_off int32[B+1], at most Nq
 *   rows an image), keys and values likewise by k_off and Nk. Nq, Nk <= MPM_MAX_N.
 *   H query heads share Hk key heads (H a multiple of Hk): query head h reads key head h / (H / Hk).
 *   dh channels a head, a multiple of 8 (bf16) or 4 (f32), at most MPM_MAX_HEAD_DIM.
 *   scale: the factor of q . k (finite).
 *   bias (may be NULL): float[H][W][W], W = 2 span + 1, 0 <= span <= MPM_MAX_SPAN, as
 *     mpm_bias_expand writes it: bias[h][span + r][span + c] is added to the score of a query and a
 *     key whose grid positions differ by r rows and c columns (query minus key), each offset held
 *     to [-span, span]. Positions are raster indices on a grid of grid_h x grid_w cells
 *     (1 <= grid_h, grid_w <= MPM_MAX_N): q_pos, k_pos int32 per row, packed like q and k, or
 *     NULL for each row's index in its image (the raster order of a full grid). Any order of
 *     positions is taken; one outside the grid counts as the nearest cell index.
 *     An entry, or a key's bias below, beyond 2.35e38 in magnitude counts as that (infinities stay infinite).
 *   k_bias (may be NULL): float per key row, added to its scores for every query and head (for
 *     merged rows the log of the tokens they stand for). A key with -inf is dropped: its rows of
 *     k and v take no part, whatever they hold, and their gradients are zero. A constant: no
 *     gradient is computed for it.
 *   q_rows, k_rows: with q_off (k_off), how many rows out and dq (dk and dv) have if those of no image, before off[0]
 *     and from off[B] on, are to get zeros; 0: they are not written.
 */
typedef struct mpm_attention_call {
    int32_t B, Nq, Nk, H, Hk, dh, dt;
    float scale;
    const int32_t* q_off;
    const int32_t* k_off;
    const float* bias;
    int32_t span, grid_h, grid_w;
    const int32_t* q_pos;
    const int32_t* k_pos;
    const float* k_bias;
    int32_t q_rows, k_rows;
} mpm_attention_call;

/*
 * Attention of each image's queries over its keys:
 *   s = scale q . k + bias + k_bias,  out = softmax(s) v,
 * scores, softmax statistics and sums in float32, out rounded once to dt. A query without a key
 * (an image with none, or all dropped or at -inf) gets zeros. Bfloat16 rounds the
 * probabilities, before their division, to bfloat16 for their product with v, and divides by the sum of
 * the rounded ones. Sums are kept before the division: values of v of 2^96 and more in magnitude may
 * overflow them, and those below 2^-86 lose precision.
 *   lse (may be NULL): float [query row][H][2], contiguous, 8-byte aligned, needed for the gradients: the
 *     maximum m that was taken from the scores and l = log2 sum 2^(s log2(e) - m), both in base 2: the
 *     log-sum-exp is (m + l) ln 2 (a query without a key: -inf, 0). Two numbers, since under a mask
 *     value such as -1e9 on every key one float32 would not hold both;
 *   ws: device workspace of mpm_attention_workspace_bytes(call) bytes (0 for many shapes: may be
 *     NULL then), 256-byte aligned, used where few queries have their keys split over workgroups.
 * Errors: MPM_ERR_INVALID_ARG for NULL or misaligned pointers, sizes below 1, dh, H or strides as
 * above, bad dt, a span, grid or scale outside its range, q_rows or k_rows below 0; MPM_ERR_UNSUPPORTED for B, Nq, Nk,
 * H or dh above their maxima; MPM_ERR_WORKSPACE; MPM_ERR_HIP.
 */
size_t mpm_attention_workspace_bytes(const mpm_attention_call* call);
int mpm_attention(const mpm_attention_call* call, const mpm_heads* q, const mpm_heads* k, const mpm_heads* v,
                  const mpm_heads* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * The gradients of mpm_attention from its inputs, its out and lse, and dout (dtype dt):
 *   dq, dk, dv (dtype dt; rows and strides of their own), dk and dv summed over the query heads
 *     that share a key head;
 *   dbias (may be NULL; only with bias): float[H][W][W], the sum of the score gradients of every
 *     pair at each offset, over all images (mpm_bias_gradient takes it to the table's).
 * Rows of dq, dk and dv that belong to an image are all written. Results do not depend on the order workgroups run in.
 * dbias is summed in 64-bit integers of a unit found for every image and head: score gradients below 2^-40
 * of the largest there are lost. One that is not finite makes all of its head's dbias NaN.
 * ws: mpm_attention_backward_workspace_bytes(call) bytes. With a bias most of them are dbias's partial
 * sums, W * W floats for every image, head and 64 to 256 queries; a call whose dbias is NULL needs only
 * what the size of the same call without its bias is (bias NULL). Errors as mpm_attention, plus
 * MPM_ERR_INVALID_ARG for dbias without bias.
 */
size_t mpm_attention_backward_workspace_bytes(const mpm_attention_call* call);
int mpm_attention_backward(const mpm_attention_call* call, const mpm_heads* dout, const mpm_heads* q,
                           const mpm_heads* k, const mpm_heads* v, const mpm_heads* out, const float* lse,
                           const mpm_heads* dq, const mpm_heads* dk, const mpm_heads* dv, float* dbias, void* ws,
                           size_t ws_bytes, void* stream);

/*
 * The learned relative position bias by buckets. lut int32[2 span + 1] gives the bucket, in
 * [0, nb), of an axis offset -span ... span; a pair's bucket is lut[row offset] * nb + lut[column
 * offset]; table [nb * nb][H] of dtype dt holds the learned values.
 *   mpm_bias_expand: bias[h][r][c] = table[lut[r] * nb + lut[c]][h], float [H][W][W];
 *   mpm_bias_gradient: dtable[bucket][h] = the sum of dbias[h] over the bucket's offsets in a fixed
 *     order, rounded once to dt; buckets without an offset get zeros.
 * A lut value outside [0, nb) counts as the nearest bucket in mpm_bias_expand and as none in
 * mpm_bias_gradient. Errors: MPM_ERR_INVALID_ARG for bad pointers, nb < 1, H < 1, span < 0 or dt;
 * MPM_ERR_UNSUPPORTED for span > MPM_MAX_SPAN, H > MPM_MAX_HEADS or nb > 2 * MPM_MAX_SPAN + 1.
 */
int mpm_bias_expand(const void* table, const int32_t* lut, int32_t nb, int32_t span, int32_t H, int32_t dt,
                    float* bias, void* stream);
int mpm_bias_gradient(const float* dbias, const int32_t* lut, int32_t nb, int32_t span, int32_t H, int32_t dt,
                      void* dtable, void* stream);

typedef enum {
    MPM_NORM_LAYER = 0, /* (t - mean) / sqrt(variance + eps) * w + b */
    MPM_NORM_RMS = 1    /* t / sqrt(mean square + eps) * w (+ b where given) */
} mpm_norm_kind;

/*
 * The parameters of the norms around a block, each of D values of dtype dt unless said otherwise:
 *   R rows of D values (16-byte rows, as tokens), contiguous;
 *   w, b: the norm before the next block (w NULL: none; b NULL: no shift);
 *   post_w, post_b: the norm after this block (post_w NULL: none);
 *   scale (may be NULL): the residual scale;
 *   gate (may be NULL): gate_per_row 0: one row an image, [B][D], the rows of image b given by
 *     off (int32[B+1]; NULL: R / B rows each); gate_per_row 1: [R][D] (B and off are not used);
 *   clear: what becomes of the rows outside every image (with a gate by image and off): 0: they are not written;
 *     MPM_CLEAR_ROWS: zeros in h, dx and df, and with MPM_CLEAR_SUM in y as well (which must not be x then).
 */
#define MPM_CLEAR_ROWS 1
#define MPM_CLEAR_SUM 2
typedef struct mpm_norm_call {
    int32_t R, D, dt, kind;
    float eps;
    int32_t B, gate_per_row;
    const int32_t* off;
    const void* w;
    const void* b;
    const void* post_w;
    const void* post_b;
    const void* scale;
    const void* gate;
    int32_t clear;
} mpm_norm_call;

/*
 * A block's output f into the residual stream x, and the next block's input:
 *   u = post_norm(f) or f,  y = x + scale * gate * u,  h = norm(y),
 * in float32 with y and h rounded once to dt (h is of the sum before y's rounding).
 *   h: NULL if and only if w is; y may alias x;
 *   stats (may be NULL): float[R][4], (mean, 1 / deviation) of f and of y, for the gradients.
 * Rows outside every image (with a gate by image and off) are written only as `clear` says.
 * Errors: MPM_ERR_INVALID_ARG for NULL or misaligned (16-byte) pointers, sizes below 1, D as for tokens,
 * eps < 0 or not finite, a shift without its weight, B that does not divide R (gate by image, off NULL),
 * bad dt, kind or clear, MPM_CLEAR_SUM with y at x; MPM_ERR_UNSUPPORTED for D > MPM_MAX_D or B >
 * MPM_MAX_B; MPM_ERR_HIP.
 */
int mpm_residual_norm(const mpm_norm_call* call, const void* x, const void* f, void* y, void* h, float* stats,
                      void* stream);

/*
 * Its gradients, from dy (into y from past this block; NULL: zero) and dh (into h; NULL if and only if
 * w is), the stored y, f and stats:
 *   dx, df [R][D]; dw, db, dpost_w, dpost_b, dscale [D]; dgate shaped as gate: each needed if and
 *   only if its parameter is given. All of dtype dt; sums over rows are kept in float32, in a fixed order.
 * The rows of y are normed as they are stored, rounded to dt, with the statistics of the unrounded sum.
 * ws: mpm_residual_norm_backward_workspace_bytes(call) bytes. Errors as mpm_residual_norm,
 * plus MPM_ERR_WORKSPACE.
 */
typedef struct mpm_norm_grads {
    void* dx;
    void* df;
    void* dw;
    void* db;
    void* dpost_w;
    void* dpost_b;
    void* dscale;
    void* dgate;
} mpm_norm_grads;

size_t mpm_residual_norm_backward_workspace_bytes(const mpm_norm_call* call);
int mpm_residual_norm_backward(const mpm_norm_call* call, const void* dy, const void* dh, const void* y,
                               const void* f, const float* stats, const mpm_norm_grads* grads, void* ws,
                               size_t ws_bytes, void* stream);

/* ---- Rotary positions, products in 8-bit integers and group norm: an encoder whose positions are
 * rotations, its serving form, and the norm of the decoder on the rebuilt grid. Conventions as above; NaN
 * and infinities flow through as in the formulas (checked mode validates the offsets only). ---- */

typedef enum {
    MPM_ROTARY_HALVES = 0, /* pair p of a head: channels p and p + pairs */
    MPM_ROTARY_PAIRS = 1   /* pair p of a head: channels 2 p and 2 p + 1 */
} mpm_rotary_layout;

#define MPM_MAX_AXES 3

/*
 * Rows of heads and the angles they are turned by.
 *   R rows of H heads of dh channels (a multiple of 8 (bf16) or 4 (f32), at most MPM_MAX_HEAD_DIM), of
 *   which the first 2 * pairs are turned, pair by pair, and the others pass.
 *   axes (1 ... MPM_MAX_AXES) axes of a grid of grid[0] x ... x grid[axes - 1] cells (at most 2^31 - 1),
 *   the last one running fastest: (row, column) of an image, (time, row, column) of a clip.
 *   pos: int32[R], each row's raster index on that grid (any order; one outside the grid counts as the
 *     nearest cell index); NULL: its index in its image.
 *   freq: float [axes][pairs], or [H][axes][pairs] with freq_per_head: a row at cell (c_0, ...) turns
 *     pair p by sum_a c_a freq[a][p] radians. Angles are formed in 64 bits.
 *   off (may be NULL): int32[B+1], the packed images. Rows before off[0] and from off[B] on belong to no
 *     image and are not turned. NULL: every row is turned, in images of R / B rows each.
 */
typedef struct mpm_rotary_call {
    int32_t R, H, dh, dt;
    int32_t pairs, layout;
    int32_t axes, grid[MPM_MAX_AXES];
    int32_t freq_per_head;
    const float* freq;
    const int32_t* pos;
    int32_t B;
    const int32_t* off;
} mpm_rotary_call;

/*
 * out = x with every pair (a, b) turned to (a cos - b sin, a sin + b cos), in float32 and rounded once to
 * dt; by the negative angle with inverse != 0. out may be x; otherwise the two must not overlap.
 * Rows of no image are not written. Bfloat16 takes the processor's sine and cosine (absolute error
 * below 2^-19), float32 the library's (a few 2^-24).
 * Errors: MPM_ERR_INVALID_ARG for NULL or misaligned pointers, sizes below 1, dh or strides as for
 * mpm_attention, pairs above dh / 2, a grid of more than 2^31 - 1 cells, bad dt, layout or axes, B that does
 * not divide R (off NULL); MPM_ERR_UNSUPPORTED for H > MPM_MAX_HEADS, dh > MPM_MAX_HEAD_DIM or
 * B > MPM_MAX_B; MPM_ERR_HIP.
 */
int mpm_rotary(const mpm_rotary_call* call, const mpm_heads* x, const mpm_heads* out, int32_t inverse, void* stream);

/*
 * The gradients of mpm_rotary from dout:
 *   dx: dout turned by the negative angles (zeros in rows of no image); may be dout itself;
 *   dfreq (may be NULL): float, shaped as freq: the sum over rows (and over heads, where they share
 *     frequencies) of c_a (x_1 dx_2 - x_2 dx_1), dx before its rounding; x (only with dfreq; else NULL) is the
 *     forward call's x, and dx must not overlap it. Sums in float32 in a workgroup, in 64 bits over them, in
 *     a fixed order; with bfloat16 rows, of terms formed with the processor's sine and cosine.
 * ws: mpm_rotary_backward_workspace_bytes(call) bytes with dfreq; none without. Errors as mpm_rotary,
 * MPM_ERR_INVALID_ARG for dfreq without x or x without dfreq, and MPM_ERR_WORKSPACE.
 */
size_t mpm_rotary_backward_workspace_bytes(const mpm_rotary_call* call);
int mpm_rotary_backward(const mpm_rotary_call* call, const mpm_heads* dout, const mpm_heads* x, const mpm_heads* dx,
                        float* dfreq, void* ws, size_t ws_bytes, void* stream);

typedef enum {
    MPM_ACT_NONE = 0,
    MPM_ACT_RELU = 1, /* max(z, 0); slope 0 at 0 */
    MPM_ACT_SILU = 2, /* z / (1 + e^-z), the exponential within (1 + |z|) 2^-23 of itself */
    /* z (1 + erf(z / sqrt 2)) / 2. For results (or gradients) of dtype bfloat16 the factor of z is a fit, within
     * 2^-17 + z^2 2^-22 of itself down to z = -11 and 2^-100 of the result below; its slope uses the same factor. */
    MPM_ACT_GELU = 3
} mpm_activation;

#define MPM_I8 2           /* signed 8-bit steps, as mpm_quantize_rows writes them (an mpm_dtype of x only) */
#define MPM_MAX_K8 65536   /* widest row of 8-bit steps: sums of products stay below 2^30 */
#define MPM_MAX_N8 1048576 /* most output channels of mpm_linear_int8 */

/*
 * Rows of K values (dtype dt, a multiple of 8 (bf16) or 4 (f32); row r at x + r * x_row elements, x_row a whole
 * number of 16 bytes) as signed 8-bit steps with a scale each:
 *   scale[r] = max(max_k |x| / 127, 2^-126), rounded to float32;
 *   q[r][k] = x / scale[r] rounded to the nearest integer, ties to even, held to [-127, 127]: the rounding of
 *     the real quotient, not of its float32 value.
 * A row with a NaN or an infinity gets the scale NaN and steps 0. q rows are K bytes and zeros up to the next
 * multiple of 16. Errors: MPM_ERR_INVALID_ARG for NULL or misaligned (q, x: 16, scale: 4) pointers, sizes
 * below 1, K or x_row as above, bad dt; MPM_ERR_UNSUPPORTED for K > MPM_MAX_K8; MPM_ERR_HIP.
 */
int mpm_quantize_rows(const void* x, int32_t R, int32_t K, int64_t x_row, int32_t dt, int8_t* q, float* scale,
                      void* stream);

/*
 * A product in 8-bit integers, with a scale for each token and each output channel:
 *   out[m][n] = act(x_scale[m] w_scale[n] (sum_k q[m][k] w[n][k]) + bias[n]),
 * the sum exact in 32-bit integers, the rest in float32, rounded once to dt (the scales are multiplied into
 * the sum one after the other, x_scale 2^-24 first and then w_scale 2^24: x_scale below 2^-102 loses
 * precision, w_scale has to be below 2^104).
 *   M tokens of K values; x_dt MPM_I8: x holds the steps, rows of K bytes rounded up to a multiple of 16, and
 *     x_scale their scales; MPM_F32 / MPM_BF16: x holds values, rows at x_row elements as in mpm_quantize_rows,
 *     which are turned into steps on the way (x_scale NULL);
 *   w: int8 [N] rows of K bytes rounded up to a multiple of 16 (mpm_quantize_rows of the weights [N][K]). The
 *     bytes from K on are multiplied too: x's or w's have to be zero, as mpm_quantize_rows leaves them;
 *   w_scale: float[N]; bias (may be NULL): N values of dtype dt;
 *   out: row m at out + m * out_row elements, out_row >= N (any alignment of whole elements; rows of whole
 *     16 bytes are written fastest). out must not overlap the inputs.
 *   ws: mpm_linear_int8_workspace_bytes(call) bytes (0 for steps, and for few results), 256-byte aligned.
 * Errors: MPM_ERR_INVALID_ARG for NULL or misaligned pointers (x, w: 16 bytes; w_scale, x_scale: 4; bias,
 * out: an element), sizes below 1, K or strides as above, bad dt, x_dt or act, x_scale that does not go with
 * x_dt; MPM_ERR_UNSUPPORTED for K > MPM_MAX_K8 or N > MPM_MAX_N8; MPM_ERR_WORKSPACE; MPM_ERR_HIP.
 */
typedef struct mpm_linear8_call {
    int32_t M, N, K, x_dt, dt, act;
    int64_t x_row, out_row;
    const float* x_scale;
    const int8_t* w;
    const float* w_scale;
    const void* bias;
} mpm_linear8_call;

size_t mpm_linear_int8_workspace_bytes(const mpm_linear8_call* call);
int mpm_linear_int8(const mpm_linear8_call* call, const void* x, void* out, void* ws, size_t ws_bytes, void* stream);

/*
 * Group norm with an activation, channels last. B images of rows of C channels (16-byte rows, as tokens;
 * contiguous, R in all): dense (off NULL: R / B rows each) or packed (off int32[B+1]); groups divides C. Per
 * image and group of C / groups channels, over all its rows:
 *   t = (x - mean) / sqrt(variance + eps),  y = act(t w + b)
 * (w, b: C values of dtype dt each, may be NULL: ones, zeros; b only with w).
 */
typedef struct mpm_group_norm_call {
    int32_t R, C, groups, dt, act;
    float eps;
    int32_t B;
    const int32_t* off;
    const void* w;
    const void* b;
} mpm_group_norm_call;

/*
 * Forward: statistics and the rest in float32, y rounded once to dt; y may be x itself. A NaN or an infinity among a
 * group's values leaves NaN in all of them; so may finite values 2^60 and more away from its mean. Rows of no image are
 * not written. stats (may be NULL): float[B][groups][2], mean and 1 / deviation (zeros for an empty image).
 * Backward, from dy, x and stats: dx (zeros in rows of no image; may be dy or x itself), and dw, db (C values of
 * dtype dt, each asked for if and only if w, b is given), summed over the images in a fixed order.
 * ws: the given number of bytes (may be 0), 256-byte aligned.
 * Errors: MPM_ERR_INVALID_ARG for NULL or misaligned (16-byte; stats: 8) pointers, sizes below 1, C as for
 * tokens, groups that do not divide C, eps < 0 or not finite, b without w, bad dt or act, B that does not divide R
 * (off NULL); MPM_ERR_UNSUPPORTED for C > MPM_MAX_D or B > MPM_MAX_B; MPM_ERR_WORKSPACE; MPM_ERR_HIP.
 */
size_t mpm_group_norm_workspace_bytes(const mpm_group_norm_call* call);
int mpm_group_norm(const mpm_group_norm_call* call, const void* x, void* y, float* stats, void* ws, size_t ws_bytes,
                   void* stream);
size_t mpm_group_norm_backward_workspace_bytes(const mpm_group_norm_call* call);
int mpm_group_norm_backward(const mpm_group_norm_call* call, const void* dy, const void* x, const float* stats, void* dx,
                            void* dw, void* db, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MPM_H */
