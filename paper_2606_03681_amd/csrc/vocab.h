// Kernels of the operators over discrete values (include/tfm_vocab.h): embedding rows and their
// gradient, distillation from a teacher's top logits, adjusted logits, sampling.
#pragma once

#include "common.h"

namespace tfm {

constexpr int VOCAB_VMAX = 1 << 18;  // most classes of a row of logits
constexpr int DISTILL_KMAX = 256;    // most teacher entries of a row

// Where row (i, j, k) of ids [n0][n1][n2] lies among the activations, in elements.
struct EmbedGeo {
  int64_t N;            // n0 n1 n2
  int64_t stride[3];
  uint64_t m1, m2;      // floor(2^64 / n1) + 1 and of n2, 0 for 1
  int32_t n1, n2;
  int32_t E, V;
  float scale;
};

template <class TT, class TO>
hipError_t launch_embed_fwd(const EmbedGeo& g, const int32_t* ids, const TT* table, TO* out,
                            int accumulate, hipStream_t s);
size_t embed_bwd_bytes(const EmbedGeo& g);
template <class TO>
hipError_t launch_embed_bwd(const EmbedGeo& g, const int32_t* ids, const TO* dout, float* dtable,
                            int accumulate, void* ws, hipStream_t s);

struct DistillGeo {
  int64_t N, ld;
  int32_t V, k, tail;
  float tau, alpha;
  const int32_t* idx;
  const float* top;
  const float* lse;      // null unless tail
  const int32_t* labels; // nullable
  const float* weights;  // nullable
  const int32_t* ncls;   // nullable
  float* row_loss;       // caller's or scratch
  double* wsum;          // scratch: partial sums of the weights
  int32_t nwsum;         // their number
  double* lsum;          // scratch: partial sums of the weighted losses (as many at most)
  void* split;           // scratch of split rows
};
// Bytes of that scratch: few long rows are split over workgroups.
size_t distill_split_bytes(int64_t N, int32_t V, int32_t k);

constexpr int DISTILL_WPARTS = 256;  // most partial sums of the weights
hipError_t launch_distill_weights(DistillGeo& g, hipStream_t s);
template <class T>
hipError_t launch_distill_rows(const DistillGeo& g, const T* logits, T* dlogits, hipStream_t s);
hipError_t launch_distill_total(const DistillGeo& g, float* loss, hipStream_t s);

struct AdjustGeo {
  int64_t N, ld, ld_out, ld_history, ld_bias, ld_allowed;
  int32_t V, n_hist, n_bias;
  const int32_t* ncls;      // nullable, as are all but bias_idx and bias where n_bias > 0
  const int32_t* history;
  const int32_t* n_history;
  const float* repetition;
  const float* presence;
  const float* frequency;
  const int32_t* bias_idx;
  const float* bias;
  const uint32_t* allowed;
};
template <class T>
hipError_t launch_adjust(const AdjustGeo& g, const T* logits, T* out, hipStream_t s);

struct SampleGeo {
  int64_t N, ld;
  int32_t V;
  const int32_t* ncls;   // the settings are nullable
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int32_t* token;
  float* logprob;        // nullable
};
template <class T>
hipError_t launch_sample(const SampleGeo& g, const T* logits, hipStream_t s);

}  // namespace tfm
