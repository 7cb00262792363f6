/*
 * adatopk_measure.h -- measurement hooks of libadatopk (benchmarks, profiling and tests only).
 *
 * Not part of the compressor's contract: these calls exist so that a benchmark can
 * time the individual kernels of a compress / decompress call with HIP events on the
 * caller's stream, and can measure plain streaming kernels (the ceilings that the
 * HBM roofline fractions are compared with, and the known-size copy that hardware
 * counter readings are scaled by).  They keep process-global state, create HIP events
 * and synchronise; none of them may be used concurrently with another call.
 */
#ifndef ADATOPK_MEASURE_H
#define ADATOPK_MEASURE_H

#include <stddef.h>
#include <stdint.h>

#include "adatopk.h"

#ifdef __cplusplus
extern "C" {
#endif

/* on != 0: from now on every kernel of a compress / decompress call is launched with a
 * start and a stop HIP event that carry the timestamps of the dispatch itself (events are
 * created as they are needed).  on == 0: plain launches.  Returns ADATOPK_OK or
 * ADATOPK_ERUNTIME. */
adatopk_status adatopk_measure_enable(int32_t on);

/* Number of kernel stages a timed call can report, and their names (static strings):
 * the kernels of compress in launch order, then those of the two decompress calls. */
int32_t adatopk_measure_stage_count(void);
const char *adatopk_measure_stage_name(int32_t stage);

/* Waits for the stop events of the kernels launched since the last read and stores the
 * summed duration of the launches of every stage (a batch is launched in groups; the first 64 of
 * a stage count) in milliseconds into
 * ms_out[adatopk_measure_stage_count()] (host memory); stages that did not run since
 * the last read are reported as -1.  Returns ADATOPK_OK or ADATOPK_ERUNTIME. */
adatopk_status adatopk_measure_read(float *ms_out);

/* For tests of the compress of a single tensor whose sample misled it: from now on the kernel that then makes
 * the exact passes is launched without its last `missing_workgroups` workgroups, as if they started too late;
 * those that are there do their chunks for them.  Wrong results for a tensor whose sample did not mislead.
 * 0: all workgroups.  wait_rounds: how often a workgroup looks for the others before it gives up (the call then
 * ends with a NaN error norm); negative: as in the product library. */
void adatopk_measure_judge(int32_t missing_workgroups, int32_t wait_rounds);

/* Byte offset in the workspace of a call over `n_total` elements of
 *   ADATOPK_MEASURE_CLAIMS        (a single tensor whose sample misled it) who worked: per chunk 1 + the number of the
 *                                 workgroup that took it, 0 if none had to (uint32)
 *   ADATOPK_MEASURE_CHUNK_COUNTS  per chunk its candidates, more than a quarter of the chunk's length: the chunk
 *                                 has no list (uint32)
 *   ADATOPK_MEASURE_PART_COUNTS   (fp32) per part of a chunk's candidates how many lie above the k-th key's window bin; not
 *                                 written for empty parts (uint32) */
#define ADATOPK_MEASURE_CLAIMS 0
#define ADATOPK_MEASURE_CHUNK_COUNTS 1
#define ADATOPK_MEASURE_PART_COUNTS 2
size_t adatopk_measure_workspace_offset(int32_t what, int64_t n_total, int32_t num_segments, adatopk_dtype dtype);

/* For tests of every form of a kernel: how a call of these sizes is cut up.  Host only, EINVAL for sizes that the call refuses or has nothing to
 * do for.
 *   weight_grad  out[0], out[1]  sides of a tile of results     out[2]  1: each load is bounded for itself (small matrices, rows far apart)
 *                out[3]          shares of the tokens; more than one are joined by a second kernel
 *   layernorm    out[0]          lanes to a row                 out[1]  octets of a row to a lane
 *                out[2]          rows under way at a time
 *                out[3]          backward pass with the weight's gradient: 0 if that is added up along with the rows, otherwise the number of
 *                                shares of the rows in which it is, apart from them
 *   fp8_product  out[0]          side of a tile, 0: a few tokens     out[1]  1: the tile's wavefronts take turns along the sum
 *                out[2]          shares of the sum; more than one are joined by a second kernel
 *                out[3]          1: the tiles behind the last full round are done in quarters
 *   muon_update  eight products, three numbers each (sides of a tile, and what out[2] is above, + 64 where its wavefronts take turns along the sum): X X^T, A A,
 *                B X and the last step's B X, which writes w, from pairs, then from their h alone
 *   muon_update_next   B X of a step that others follow, four numbers each (sides of a tile, 1: its wavefronts take turns along the sum, 1: its operands change
 *                places): from pairs, from their h alone with another such step behind it, and with one from pairs behind it */
adatopk_status adatopk_measure_weight_grad_cut(int64_t rows, int64_t n_out, int64_t n_in, adatopk_dtype dt, int64_t dy_stride, int32_t *out);
adatopk_status adatopk_measure_layernorm_cut(int64_t rows, int64_t cols, int32_t backward, int32_t *out);
adatopk_status adatopk_measure_fp8_product_cut(int64_t rows, int64_t n_out, int64_t n_in, adatopk_dtype dt, int32_t *out);
adatopk_status adatopk_measure_muon_update_cut(int64_t rows, int64_t cols, int32_t *out);
adatopk_status adatopk_measure_muon_update_next_cut(int64_t rows, int64_t cols, int32_t *out);

/* Plain streaming kernels on `hip_stream`; all pointers are device memory, 16-byte
 * aligned; bytes must be a multiple of 16.
 *   copy:      dst[i] = src[i]                        (reads bytes, writes bytes)
 *   read_only: folds src into one word at sink[0]     (reads bytes)
 *   fill:      dst[i] = 0, the kernel decompress uses (writes bytes) */
adatopk_status adatopk_measure_copy(void *dst, const void *src, size_t bytes, void *hip_stream);
adatopk_status adatopk_measure_read_only(const void *src, size_t bytes, uint32_t *sink, void *hip_stream);
adatopk_status adatopk_measure_fill(void *dst, size_t bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ADATOPK_MEASURE_H */
