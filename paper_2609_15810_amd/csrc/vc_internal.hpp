// Internal launch arguments and launchers (not part of the public ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vc_attn.h"

namespace vc {

struct PrepArgs {
  const uint16_t *Q, *K, *V;
  const int32_t *perm, *q_perm;
  const float *rope_cos, *rope_sin;
  int8_t* q;
  float* q_scale;
  int8_t* k;
  float* k_scale;
  float* k_mean;
  uint8_t* v;
  float* v_scale;
  uint16_t* v_mean;
  uint8_t *q_mxs, *k_mxs;  // E8M0 scale bytes (MXFP4 only)
  float* ws_ksum;   // [B*H][T][128] per-block key channel sums
  float* ws_vamax;  // [B*H][T][128] per-block residual maxima
  float* ws_vinv;   // [B*H][128]    448 / amax (0 for an all-zero channel)
  int N, T, F, Ht, Wd;
  float inv_w, inv_hw;  // 1/Wd and 1/(Ht*Wd) in fp32: estimates for the token-position divisions
  int rope, hadamard, smooth_k, smooth_v;
  int qk_fmt;
};

struct FwdArgs {
  const int8_t* q;
  const float* q_scale;
  const int8_t* k;
  const float* k_scale;
  const uint8_t* v;
  const float* v_scale;
  const uint16_t* v_mean;
  const uint8_t *q_mxs, *k_mxs;  // E8M0 scale bytes (MXFP4 only)
  const int32_t* q_perm;
  uint16_t* O;
  uint8_t* p_codes;  // debugging: the probability codes of every tile [B*H][N][128 T], or null
  int N, T;
  float kappa;      // sm_scale * log2(e) (/ 128 with the Hadamard rotation), rounded once to fp32
  float cbias;      // fl(120 + beta)
  int p_mode, smooth_v;
  int qk_fmt;
  int first;        // a launch's first workgroup (in order of head and query)
};

// How a call's rows are dealt to the attention kernels: n8 workgroups of 256 queries, n4 of 128 and n1 of
// 32, each counted in order of head and query (a head's last workgroup may be ragged); first4 and first1 are
// the positions of the first ones behind those before them.
struct ForwardPlan {
  int n8, first4, n4, first1, n1;
};

struct GroupArgs {
  const uint16_t* V;
  float* centroids;
  int32_t *labels, *perm, *inv_perm;
  // workspace (k-means)
  int8_t* codes;      // [B*H][N][128] INT8 codes of V
  float* scale;       // [B*H] max |V|
  float* amax_part;   // [B*H][nblk] its partial maxima
  int8_t* cent8;      // [2][B*H][k][128] the centroids of a round and the one before
  int32_t* sums;      // [3][B*H][sums_head] member sums [k][128] and counts [k] of three rounds in turn
  int32_t* hist;      // [B*H][nsort][k] final label counts per 1024 tokens
  int BH, N, F, Ht, Wd, k, iters, warm_start, mode, cube_t, cube_h, cube_w;
  int nblk;           // 256-token blocks per head
  int sums_head;      // k * 129 rounded up to 16 bytes
  int nsort;          // 1024-token blocks per head
  int atok;           // tokens per assignment workgroup (a multiple of 256)
};

// One of the tensors (queries, keys) of the norm and rotation: rows [b, h, n] of d channels at element
// strides, and for the backward pass the gradient of its output (grad) with out the gradient of its input
struct NormRopeTensor {
  const uint16_t *in, *grad;
  uint16_t* out;
  int64_t in_sb, in_sh, in_sn, grad_sb, grad_sh, grad_sn, out_sb, out_sh, out_sn;
  const float* weight;   // of the norm, or null (ones)
  float* dw;
  float* dw_part;        // [workgroups][weights] partial sums, or null (no weight gradient)
  float inv_span;        // 1 / channels under one norm
  int H, weights;
  int W, P;              // waves that share a token; slots of theirs that work on its heads
  uint32_t groups;       // of tokens
};

struct NormRopeArgs {
  NormRopeTensor t[2];
  int ntensors;
  int64_t tokens;        // B * N
  int N, d, dtype, norm, layout, rot;
  float eps, sign;       // sign of the sines
  const float *cos_t, *sin_t;
  const int32_t* pos;    // [B][N] table rows, or null
  int rows;              // of the tables on a line
  int past;              // store results past the caches
  int grid, F, Ht, Wd;   // grid: positions on the latent grid, tables of frames, rows and columns
};

// A strided tensor of 16-bit rows
struct Strided {
  uint16_t* p;
  int64_t sb, sh, sn;
};

// Attention of Hq query heads of M queries to Hk = Hq / G key heads of N keys. The query rows of a key head are
// counted through its G query heads: R = G M rows.
struct CrossArgs {
  Strided Q, K, V, O, dO, dQ, dK, dV;
  int B, Hq, Hk, G, M, N, R, d, dtype;
  float c;               // score scale times log2(e)
  float scale;           // score scale
  const int32_t* k_len;  // [B], or null
  const int32_t* idx;    // [B][N] the keys that count, in order, then the others; or null
  const int32_t* count;  // [B] how many count (with idx)
  float* lse;            // [B][Hq][M] natural logarithm of the softmax's sum
  // keys split over workgroups: `splits` parts of `chunk` keys, joined from
  int splits, chunk;
  float* part_o;         // [splits][B Hk][R][d] unnormalised outputs (backward: parts of dQ)
  float* part_ml;        // [splits][B Hk][R][2] running maximum (log2 units) and sum (backward: sums of P dP and of P)
  // backward
  float* stats;          // [B][Hq][cross_stat_rows(M)][2] lse in log2 units and delta
  int row_splits, row_chunk;   // row tiles split over workgroups that form dK and dV
  float* part_kv;        // [row_splits][2][B Hk][N][d] parts of dK and dV
};

hipError_t launch_prep(const PrepArgs& a, int BH, hipStream_t s);
ForwardPlan forward_plan(int N, int BH, int qk_fmt, int p_mode);
hipError_t launch_forward(FwdArgs a, int BH, hipStream_t s);
hipError_t launch_group(const GroupArgs& a, int BH, hipStream_t s);
hipError_t launch_fp8_score_product(const uint8_t* a, const uint8_t* b, const float* c_in, float* out, int n,
                                    hipStream_t s);

hipError_t launch_norm_rope(NormRopeArgs a, hipStream_t s);
hipError_t launch_norm_rope_backward(NormRopeArgs a, hipStream_t s);
int norm_rope_parts(int64_t tokens, int ntensors);   // workgroups of the backward kernel for each tensor

// Which keys count, as a list: idx [B][N], count [B]
hipError_t launch_cross_keys(const uint8_t* k_mask, int64_t stride, const int32_t* k_len, int B, int N, int32_t* idx,
                             int32_t* count, hipStream_t s);
// How a call's keys are split (a.splits, a.chunk), and for the backward pass its rows (a.row_splits, a.row_chunk)
void cross_plan(CrossArgs& a);
void cross_plan_backward(CrossArgs& a);
int cross_stat_rows(int M);   // rows of a query head's statistics
hipError_t launch_cross_forward(const CrossArgs& a, hipStream_t s);
hipError_t launch_cross_backward(const CrossArgs& a, hipStream_t s);

// VC_OK, or VC_ERR_HIP with the error kept for vc_last_hip_error
vc_status hip_status(hipError_t e);

}  // namespace vc

// The plan of a call, for tests on the host (not part of the public ABI): n8, first4, n4, first1, n1.
extern "C" void vc_internal_forward_plan(int32_t N, int32_t BH, int32_t qk_fmt, int32_t p_mode, int32_t plan[5]);
