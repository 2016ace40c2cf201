// The contraction behind the linear cross entropy: one tcgen05 kernel over CTA pairs whose operands may be K-major or
// MN-major (a matrix used as it lies in memory or transposed) and whose epilogue is the loss's.
#pragma once
#include <cstdint>

#include "common.cuh"
#include "xent_plan.cuh"

namespace cert {

struct XentMap { alignas(64) unsigned char bytes[128]; };   // a CUtensorMap

enum { XENT_EPI_LSE = 0, XENT_EPI_PROB = 1, XENT_EPI_STORE = 2, XENT_EPI_ROW = 3 };

// D[m][n] = sum over k of A[m][k] * B[n][k] with 16-bit operands and fp32 accumulators.
// A float32 operand is held as three bfloat16 parts side by side, x = x0 + x1 + x2 (8 bits of mantissa each); `segs`
// products of parts (a_part[i], b_part[i]) then make up one product of matrices.
struct XentGemmArgs {
    // sizes; a count on the device, where given, replaces the host's upper bound
    int M, N, K;
    const int *m_count, *k_count;
    int bn;                          // columns of a tile: a multiple of 32 (LSE), of 64 (PROB, ROW) or of 128 (STORE), up to 256
    int a_mn;                        // STORE: A is MN-major (its rows are read as columns), else K-major; B is MN-major
    int most_splits, split_kb, pairs;   // K in up to this many ranges, each with a slab of its own (see xent_splits)
    int raster;                      // row panels that are walked together (see the tile order in the kernel)
    int segs;
    signed char a_part[8], b_part[8];
    int a_pitch, b_pitch;            // elements between two parts, along the operand's contiguous axis
    int a_mn0, a_k0, b_mn0, b_k0;    // where the operand's rows / K range start in its tensor map
    int bf16;                        // operand type: bfloat16, else float16
    int *status;
    // LSE and PROB: the logits are acc + bias[n]; column n of this launch is class class0 + n
    const float *bias;               // fp32, readable up to N rounded up to 32 (ROW: to the tile's end); or null
    int class0;
    const int *target;               // [rows] class of each row
    // LSE: per row and slot (two slots per column tile) the running maximum (log2 units) and sum; target's logit
    float2 *partial;                 // [slots][rows_pad]
    int rows_pad, slot0;
    float *target_logit;             // [rows]
    // PROB: p * prob_scale as 16-bit numbers, prob_parts parts; column sums of p over groups of 32 rows
    const float2 *stat;              // [rows] maximum m of z log2 e, and log2 of the sum of 2^(z log2 e - m)
    void *prob;
    long long prob_ld;
    int prob_parts, prob_pitch;
    float prob_log2_scale;           // p is stored times 2^this
    float *colsum;                   // [groups of 32 rows][colsum_ld] or null
    int colsum_ld;
    // (written through shared memory by TMA, 32 rows x 32 columns at a time, see out_map in launch_xent_*)
    // ROW (all classes in one column tile): the statistics are the tile's own, then as PROB; the rows' losses and their sums
    // over groups of 32 rows
    float *row_losses;               // [rows of the call] or null
    const int *row_of;               // [rows] row of the call
    double *loss_sum;                // [groups of 32 rows]
    // STORE: out = acc * scale in `out_type`, or accumulated in fp32
    void *out;
    int out_type;
    long long out_ld, out_split_stride;
    int add;                         // add to what is there (fp32 only)
    int tma_out;                     // the launch's output map covers out: whole groups of 32 rows go there by TMA
    int rows_16;                     // rows start on 16-byte boundaries (where the lanes store them)
    int split_rows;                  // rows of the map from one K range's slab to the next
    float out_scale;
    const int *count;                // non-null: out_scale is divided by max(1, *count) (mean reduction)
    const int *row_map;              // non-null: row m goes to row row_map[m]
};

bool xent_gemm_prepare();
bool xent_make_map(XentMap *m, const void *base, bool bf16, long long inner, long long outer, long long pitch_elems,
                   int box_inner, int box_outer);
// Map of an output in blocks of 32 x 32 (needs a 16-byte aligned base and pitch); false where TMA cannot write it.
bool xent_make_out_map(XentMap *m, const void *base, int type, long long inner, long long outer, long long pitch_elems);
// LSE, PROB and ROW take K-major operands; `out` is the map of the probabilities (PROB, ROW).
void launch_xent_gemm(int epi, int pairs, const XentMap &a, const XentMap &b, const XentMap &out, const XentGemmArgs &args, cudaStream_t st);
// One or two STORE products (the second with N = 0: one) in one launch, the first's tiles before the second's.
struct XentProduct { XentMap a, b, out; XentGemmArgs args; };
void launch_xent_store(int pairs, const XentProduct &first, const XentProduct &second, cudaStream_t st);

}  // namespace cert
