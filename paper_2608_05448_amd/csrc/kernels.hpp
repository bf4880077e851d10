// Launch interfaces between the C ABI (abi.hip) and the kernels. Internal to the library.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dbl {

constexpr int kTile = 128;            // vocabulary tile of the two-level log-prob form
constexpr int kTilesPerChunk = 32;    // vocabulary tiles per workgroup in the V-streaming kernels
constexpr int kMaxR = 64;             // categories handled by one wavefront

struct HeadArgs {
  int64_t M, V;
  int d;
  bool dtype_bf16;
  const void* h;
  const void* w;
  float* tls;
  float* lmass;
  float* lse;
  int32_t* argmax;      // [M] or null: lowest-index argmax of each row's logits
  uint64_t* amax_keys;  // workspace [M] when argmax is requested
};

// The branch log-probabilities and block description shared by the sampler and verifier.
struct BlockArgs {
  int64_t B, K, R, V;
  int nT;
  const float* tls;
  const float* lmass;
  const float* lse;
  const float* prior;  // [B, R]
  float z_temp;
  uint64_t seed, step;
  int64_t seq_offset;
};

struct SampleArgs {
  BlockArgs blk;
  int32_t* z_out;
  int32_t* x_out;
};

struct VerifyArgs {
  BlockArgs blk;
  const int32_t* x;     // [B, K]
  const float* logp;    // [B, Kp, V]
  int64_t Kp;
  bool trajectory;      // expected-length mode: no accept test, no residual
  int32_t* n_accept;    // [B] (verify only)
  int32_t* next_token;  // [B] (verify only)
  float* beta;          // [B, K] or null
  float* al;            // [B] or null
  float* exp_len;       // [B] or null
  double* wpost;        // workspace [B, K, R]: posterior weights
  float* beta_part;     // workspace [B*K, nchunk]
  uint64_t* res_tiles;  // workspace [B, nT]
  uint64_t* p_tiles;    // workspace [B, nT]
};

// Greedy-branch mode: the branch tokens replace the branch log-probabilities (blk.tls, lmass and
// lse are unused).
struct GreedyArgs {
  BlockArgs blk;
  const int32_t* xhat;  // [B, K, R] branch tokens argmax_v q_k(v | z)
  int32_t* z_out;       // sample: [B]
  int32_t* x_out;       // sample: [B, K]
  const int32_t* x;     // verify: [B, K] draft or trajectory
  const float* logp;    // verify: [B, Kp, V]
  int64_t Kp;
  bool trajectory;
  int32_t* n_accept;
  int32_t* next_token;
  float* beta;
  float* al;
  float* exp_len;
  double* wpost;        // workspace [B, K, R]
  uint64_t* res_tiles;  // workspace [B, nT]
  uint64_t* p_tiles;    // workspace [B, nT]
};

// Training-objective forward along target trajectories.
struct ObjectiveArgs {
  BlockArgs blk;
  const int32_t* x;     // [B, K] target trajectory
  const float* logp;    // [B, K, V]
  float tau;
  float* log_r;         // [B, K] or null
  float* S;             // [B, K] or null
  int32_t* ell_tau;     // [B]
  float* J;             // [B]
  float* nll;           // [B]
};

// Category hidden expander (bf16): out[m, z*d + j] = h[m, j] + (W h[m])[z*d + j] + c[z*d + j].
struct ExpandArgs {
  int64_t M, R;
  int d;
  const void* h;   // [M, d]
  const void* W;   // [R*d, d]
  const void* c;   // [R*d]
  void* out;       // [M, R*d]
};

// Category-prior head (bf16 inputs, fp32 logits): ell[b, z] = U[z] . h_anchor[b] + e[z].
struct PriorHeadArgs {
  int64_t B;
  int R, d;
  const void* h_anchor;  // [B, d]
  const void* U;         // [R, d]
  const void* e;         // [R]
  float* ell;            // [B, R]
};

// Target sampling transform: rows of logits -> filtered log-probabilities. Per row the optional
// workspace holds kFilterRowBytes (segment results, candidate lists or mass bins, by the filters
// asked for) and 16 bytes for the row's cut.
constexpr int kFilterRowBytes = 32768;
struct FilterCut {
  uint32_t key_above, key_at;  // logit keys at or above key_above are kept, and those at or above
  uint32_t last_id;            // key_at whose id is at most last_id
  uint32_t done;               // the row is already written
};

struct FilterArgs {
  int64_t N, V;
  const float* logits;  // [N, V]
  float temperature;
  int64_t top_k;        // 0: off
  float top_p;          // 1: off
  float* logp;          // [N, V]
  char* row_ws = nullptr;         // workspace [N, kFilterRowBytes] or null
  FilterCut* cuts = nullptr;      // workspace [N]
};

// Early-determinism estimate from sampled target blocks.
struct DeterminismArgs {
  int64_t M, b, V;
  const int32_t* x;     // [M, b]
  const float* logp;    // [M, b, V]
  float* terms;         // [M]
  float* mean;          // scalar or null
};

// One row that is trained on, as the head's training kernels see it. The gradient of its negative
// log-likelihood with respect to the logits, g (p_v - [v = token]), is handled as scale * u_v with
// u_v = exp(logit_v - shift') (shift' = lse + ln q) and u = at_token at the token.
// bf16: q = 1 - p_token = -expm1(-nll), scale = g q, so that u is -1 at the token (exact in bf16) and p_v / q
// elsewhere: the rounding of u to bf16 then touches the other ids only, whose errors average out, and never
// the one entry that most of the gradient rests on. q is kept from below by 2^-24, the rounding of a binary32
// probability near 1 (at_token = -(1 - p) / q there, in [-1, 0]). nll = lse - logit is off by lse's rounding
// (about 2e-6 at 20), and q with it: in a row that is as sure of its token as that, the other ids' u may be
// above 1 and do not add up to the token's, which leaves the gradient off by about g times nll's error, as it
// is in binary32 throughout. fp32: q = 1.
struct alignas(16) TrainRow {
  float shift;     // bf16: (lse + ln q) log2(e); fp32: lse
  float at_token;
  float scale;
  int32_t token;
};

// The training head's GEMM over the rows that count (bf16): tile log-masses and token logits, or the
// scaled logits' gradient u over a piece of the vocabulary.
struct HeadTrainArgs {
  int64_t M;             // rows there can be
  int64_t V;             // ids of w (of the piece)
  int d;
  const void* h;         // [M, d] rows that count first
  const void* w;         // [V, d]
  const int32_t* count;  // rows that count
  const TrainRow* rows;  // [M]
  float* lmass;          // nll: [M, nT]
  float* tgt;            // nll: [M]
  void* grad;            // gradient: [M, ldg]
  int64_t ldg, vbase;
};

// dbl_head_nll and its gradient; workspace pointers are carved out by the ABI.
struct NllArgs {
  int64_t P, R, V;       // positions, categories
  int d;
  bool bf16;
  const void* h;         // [P, R, d]
  const void* w;         // [V, d]
  const int32_t* x;      // [P]
  float* nll;            // [P, R] out (backward: in)
  float* lse;            // [P, R] out (backward: in)
  const float* g;        // backward: [P, R]
  void* dh;              // backward: [P, R, d]
  void* dw;              // backward: [V, d] or null
  void* hc;              // workspace [M, d]: rows that count
  void* hs;              // workspace [M, d]: the same times their scale (dw)
  TrainRow* rows;        // workspace [M]
  int32_t* inv;          // workspace [P]: place of a position among those that count, or -1
  int32_t* count;        // workspace
  float* lmass;          // workspace [M, nT]
  float* tgt;            // workspace [M]
  void* grad;            // workspace [M, piece]
  float* part;           // workspace [splits, M, d]
  float* dw_part;        // workspace [dw_splits, ids of a piece, d]
  int64_t piece;         // ids per piece, a multiple of 256
  int splits, dw_splits;
};

struct ExpandBackwardArgs {
  int64_t P, R;
  int d;
  const void* h;         // [P, d]
  const void* W;         // [R*d, d]
  const void* dout;      // [P, R*d]
  void* dh;              // [P, d] or null
  void* dW;              // [R*d, d] or null
  void* dc;              // [R*d] or null
  float* part;           // workspace [splits, P, d]
  float* dW_part;        // workspace [dW_splits, R*d, d]
  int splits, dW_splits;
};

// One tensor of a set of gradients.
struct GradTensor {
  const void* g;
  void* out;             // clipping only
  int64_t n;
  int32_t bf16;
};

// Ids of the vocabulary that the head's backward pass takes at a time: as many as give a gradient of
// about 1 GiB, at least 8192, in equal pieces of a multiple of 4096 (a single piece: of 256).
constexpr int64_t kPieceBytes = int64_t(1) << 30;
inline int64_t nll_piece(int64_t M, int64_t V, int elem) {
  const int64_t most = kPieceBytes / (elem * (M > 0 ? M : 1));
  const int64_t cap = most < 8192 ? 8192 : most / 4096 * 4096;
  const int64_t pieces = (V + cap - 1) / cap;
  const int64_t each = (V + pieces - 1) / pieces;
  const int64_t unit = pieces > 1 ? 4096 : 256;
  return (each + unit - 1) / unit * unit;
}

// The kernel of a bf16 product [nb, na] over K terms (both: both operands lie across the sum): 256 x 256
// tiles, one workgroup to a CU; 256-column tiles of up to 128 rows, one to a CU; smaller tiles; for short
// sums with both operands across them, a stream over the output. The last against the smaller tiles, us
// (terms x output columns x rows): 200 x 4096 x 151936 317 and 477, 128 x 4096 x 151936 213 and 246, 256 x
// 4096 x 32768 72 and 96, 100 x 2048 x 50000 38 and 50; but 168 x 1000 x 50257 34 and 31, 250 x 1024 x
// 20000 25 and 20, 60 x 2560 x 151936 125 and 128, 30 x 2048 x 151936 118 and 107. The smaller tiles against
// the 256 x 256 ones below 512 terms: 300 x 4096 x 151936 548 and 609, 400 x 2048 x 50000 118 and 127, 480 x
// 2560 x 151936 453 and 460.
enum ProdKind : int { kProdPp = 0, kProdFew = 1, kProdSmall = 2, kProdStream = 3 };
inline ProdKind prod_kind(bool both, int64_t na, int64_t nb, int64_t K) {
  if (na > 128 && nb > 128 && K >= 512) return kProdPp;
  if (!both) return na > 128 && nb <= 128 ? kProdFew : kProdSmall;
  return K > 64 && K <= 256 && na > 256 && na * nb >= (int64_t(1) << 26) ? kProdStream : kProdSmall;
}

// How many parts the sum over K of an [nb, na] product is split into (one operand across the sum).
// 256 x 256 tiles: the split with the least time for whole rounds of 256 workgroups, at 1.7 us a 64-deep
// stage and 20 us a tile for its stores and their sum. Others: as many as one round of workgroups holds,
// of 256 terms at least.
inline int grad_splits(int64_t na, int64_t nb, int64_t K) {
  if (na <= 0 || nb <= 0 || K <= 0) return 1;
  const ProdKind kind = prod_kind(false, na, nb, K);
  if (kind == kProdPp) {
    const int64_t tiles = ((na + 255) / 256) * ((nb + 255) / 256), stages = (K + 63) / 64;
    int best = 1;
    int64_t least = 0;
    for (int s = 1; s <= 64 && stages / s >= 4; ++s) {
      const int64_t t = (tiles * s + 255) / 256 * ((stages + s - 1) / s * 17 + 200);
      if (s == 1 || t < least) {
        least = t;
        best = s;
      }
    }
    return best;
  }
  const int64_t s = kind == kProdFew ? 256 / ((na + 255) / 256)
                                     : 512 / (((na + 127) / 128) * ((nb + 127) / 128));
  const int64_t most = (K + 255) / 256;
  return static_cast<int>(s < 1 ? 1 : s < most ? s : most);
}

// Rows up to which the fp32 kernel takes tiles of 32 rows.
constexpr int64_t kF32FewRows = 32;
// Tile log-masses of a row: of 128 ids, in fp32 of 32.
inline int64_t nll_tiles(bool bf16, int64_t V) { return bf16 ? (V + kTile - 1) / kTile : (V + 31) / 32; }

// The splits for fp32, whose kernel has 128 x 64 tiles and 32-deep stages: small problems are bound by the
// walk over K (a stage takes about 2 us to load), so parts have 32 terms at least.
inline int grad_splits_f32(int64_t na, int64_t nb, int64_t K) {
  if (na <= 0 || nb <= 0 || K <= 0) return 1;
  const int64_t s = 768 / (((na + 127) / 128) * ((nb + 63) / 64)), most = (K + 31) / 32;
  return static_cast<int>(s < 1 ? 1 : s < most ? s : most);
}

// The same for a product with both operands across the sum (the weight gradients): small outputs of many
// rows would leave most CUs idle. The split with the least time, in ns: whole rounds of 256 workgroups, a
// stage's time in each and 5 us for its ends; parts written and read at 5 TB/s, and one more launch. One part,
// and that split with the launch that adds the parts, us: 1000 x 512 outputs of 8192 rows 145 and 30 (24 + 6);
// 2048 x 512 of 4096 rows 75 and 29 (22 + 7); fp32 2000 x 256 of 8192 rows 380 and 114 (109 + 5), 256 x 64 of
// 2048 rows 97 and 14 (11 + 3).
inline int weight_splits(bool bf16, int64_t na, int64_t nb, int64_t K) {
  if (na <= 0 || nb <= 0 || K <= 0) return 1;
  const ProdKind kind = bf16 ? prod_kind(true, na, nb, K) : kProdSmall;
  if (kind == kProdStream) return 1;
  const bool pp = kind == kProdPp;
  const int64_t ta = pp ? 256 : 128, tb = pp ? 256 : bf16 ? 128 : 64, deep = pp ? 64 : 32;
  const int64_t stage = pp ? 1150 : bf16 ? 470 : 1500;
  const int64_t tiles = ((na + ta - 1) / ta) * ((nb + tb - 1) / tb), stages = (K + deep - 1) / deep;
  int best = 1;
  int64_t least = 0;
  for (int s = 1; s <= 64 && tiles * s <= 512 && (s == 1 || stages / s >= 4); ++s) {
    const int64_t t = (tiles * s + 255) / 256 * ((stages + s - 1) / s * stage + 5000) +
                      (s > 1 ? 4000 + s * na * nb / 625 : 0);
    if (s == 1 || t < least) {
      least = t;
      best = s;
    }
  }
  return best;
}

// Microscaled rows: blocks of 32 values that share a power of two (one byte b for 2^(b - 127)), in 4 bits
// (e2m1, two to a byte, the even value low) or 8 (e4m3); a row of d values is padded with zeros to mx_row(d).
constexpr int kMxBlock = 32, kMxPad = 128;
inline int64_t mx_row(int64_t d) { return (d + kMxPad - 1) / kMxPad * kMxPad; }

struct MxQuantArgs {
  int64_t M;
  int d, bits;
  bool bf16;
  const void* x;        // [M, d]; dequantisation: out
  void* codes;          // [M, mx_row(d) * bits / 8]
  uint8_t* scales;      // [M, mx_row(d) / 32]
};

// Norm: h = x + residual (rounded to the type), y = h / sqrt(mean(h^2) + eps) * weight.
struct MxNormArgs {
  MxQuantArgs q;
  const void* residual; // [M, d] or null
  const void* weight;   // [d]
  float eps;
  void* sum;            // [M, d] or null
  void* y;              // [M, d] or null
};

// Product of microscaled rows h [M, d] (4 or 8 bits) and w [V, d] (4 bits): logits, or the head's
// two-level form.
struct MxProductArgs {
  int64_t M, V;
  int dp;               // mx_row(d)
  int bits;             // of h
  const void* h;
  const uint8_t* hs;
  const void* w;
  const uint8_t* ws;
  void* logits;         // [M, V], or null: the two-level form
  bool bf16;            // type of the logits
  float* tls;           // [M, V]
  float* lmass;         // [M, nT]
  float* lse;           // [M]
  int32_t* argmax;      // [M] or null
  uint64_t* amax_keys;  // workspace [M]
};

// One token per row of logits.
struct DrawArgs {
  int64_t N, V;
  bool bf16;
  const void* logits;   // [N, V]
  const uint32_t* words;
  float temperature, top_p, min_p;
  int64_t top_k;
  const float *temperatures, *top_ps, *min_ps;  // [N] or null: the number beside each
  const int32_t* top_ks;
  int32_t* token;       // [N]
  float* logprob;       // [N]
  char* ws;
};
// The draw's rows are split into segments of this many ids, and the segments of a row among its workgroups (parts).
constexpr int kDrawSeg = 4096;
// Segments of a row: up to 7 ids more than V, where a row starts inside a 16-byte word.
inline int64_t draw_segments(int64_t V) { return (V + 7 + kDrawSeg - 1) / kDrawSeg; }
constexpr int kDrawBins = 4096, kDrawList = 4096;
struct DrawState {       // of a row
  uint32_t count;        // entries of the list
  uint32_t mode;         // what the launches that follow do (see draw.hip)
  uint32_t cut_bin, by;  // where the cut falls, and what makes it
  uint64_t need;
  float low;             // logits below it are not kept
  uint32_t unused[9];
};
static_assert(sizeof(DrawState) == 64, "the row's arrays follow it");
// A row's workspace, for G segments: the state; by part (G at most) the maximum; by segment the sum and the maxima
// of 128 ids each; the list; the bins' masses and counts.
struct DrawLayout {
  size_t top, sum, maxima, list, mass, count, total;
  __host__ __device__ explicit DrawLayout(int64_t G) {
    top = sizeof(DrawState);
    sum = top + 8 * G;
    maxima = sum + 8 * G;
    list = (maxima + kDrawSeg / 128 * 4 * G + 255) / 256 * 256;
    mass = list + 8 * kDrawList;
    count = mass + 8 * kDrawBins;
    total = count + 4 * kDrawBins;
  }
};
inline size_t draw_row_bytes(int64_t V) { return DrawLayout(draw_segments(V)).total; }

constexpr int64_t kMaxThreads = 0xffffffffll;     // of a launch; what is more is dropped without an error
inline bool fits_launch(int64_t blocks, int threads) { return blocks <= kMaxThreads / threads; }
constexpr int64_t kMaxTrainRows = (1 << 24) - 1;  // a workgroup of 256 each

constexpr int64_t kMaxTensors = int64_t(1) << 20;  // of a norm or clipping call
constexpr int kNormSet = 180;      // tensors of one launch of the gradient norm
constexpr int kNormBlocks = 1024;  // its workgroups, and partial sums, at most
inline int64_t norm_parts(int64_t n) { return (n + kNormSet - 1) / kNormSet * kNormBlocks; }
constexpr int64_t kMaxGradElements = int64_t(1) << 40;  // of all tensors (chunks are numbered in 31 bits)

inline int n_chunks(int nT) { return (nT + kTilesPerChunk - 1) / kTilesPerChunk; }

hipError_t launch_head(const HeadArgs& a, hipStream_t stream);
hipError_t launch_sample(const SampleArgs& a, hipStream_t stream);
hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream);
hipError_t launch_sample_greedy(const GreedyArgs& a, hipStream_t stream);
hipError_t launch_verify_greedy(const GreedyArgs& a, hipStream_t stream);
hipError_t launch_objective(const ObjectiveArgs& a, hipStream_t stream);
hipError_t launch_expand(const ExpandArgs& a, hipStream_t stream);
hipError_t launch_prior_head(const PriorHeadArgs& a, hipStream_t stream);
hipError_t launch_head_train(const HeadTrainArgs& a, bool grad, hipStream_t stream);
hipError_t launch_nll(const NllArgs& a, hipStream_t stream);
hipError_t launch_nll_backward(const NllArgs& a, hipStream_t stream);
hipError_t launch_expand_backward(const ExpandBackwardArgs& a, hipStream_t stream);
hipError_t launch_grad_norm(const GradTensor* t, int64_t n, double* part, float* norm,
                            hipStream_t stream);
hipError_t launch_clip_grads(const GradTensor* t, int64_t n, const float* norm, float max_norm,
                             hipStream_t stream);
hipError_t launch_filter(const FilterArgs& a, hipStream_t stream);
hipError_t launch_determinism(const DeterminismArgs& a, hipStream_t stream);
hipError_t launch_argmax_clear(uint64_t* amax, int64_t M, hipStream_t stream);
hipError_t launch_lse(const float* lmass, float* lse, const uint64_t* amax, int32_t* argmax, int64_t M,
                      int nT, hipStream_t stream);
hipError_t launch_mx_quantize(const MxQuantArgs& a, hipStream_t stream);
hipError_t launch_mx_dequantize(const MxQuantArgs& a, hipStream_t stream);
hipError_t launch_mx_norm(const MxNormArgs& a, hipStream_t stream);
hipError_t launch_mx_product(const MxProductArgs& a, hipStream_t stream);
hipError_t launch_draw(const DrawArgs& a, hipStream_t stream);
hipError_t launch_read_probe(const void* buf, int64_t bytes, float* partials, int64_t n_partials,
                             hipStream_t stream);

}  // namespace dbl
