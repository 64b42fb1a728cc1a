// Arguments of the sampling kernel (sample_kernels.hip).
#pragma once
#include <hip/hip_runtime.h>

namespace cfpp {

enum { kLogitsF16 = 1, kLogitsF32 = 2 };
constexpr int kSampleMaxVocab = 1 << 18;   // (weights of up to 2^45 each: their sum fits 63 bits)

struct SampleParams {
    const void *logits;
    long long stride;                // values from row to row
    int vocab;
    // of each row; null: 1, all, 1, 0
    const float *temperature;
    const int *top_k;
    const float *top_p, *min_p;
    const float *uniform;
    int *tokens;
    float *probs;                    // or null
    int *kept;                       // or null
    // a generation loop's row, or null: uniform is that of the position, the token goes to tokens[position + 1] (0 where there is none) and the position advances
    int *pos;
    int max_seq;
};

hipError_t launch_sample(const SampleParams &P, int type, int n_rows, hipStream_t s);

}  // namespace cfpp
