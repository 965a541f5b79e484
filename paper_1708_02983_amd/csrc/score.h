// What the other parts of the library need of the kernels that score tokens.
#pragma once
#include "logits.h"

namespace easgd {

// What a program gives to learn from tokens that it has (see easgd_token_loss in include/easgd.h).
struct TokensGiven {
    const int *tokens;
    const float *weight;
    float bonus, temperature;
    float *logprob, *entropy;
};

// The checks of these arguments that every call shares; EASGD_OK, or the error with its message set.
int check_tokens(const char *name, const TokensGiven &t, bool rows);

// Losses and gradients of rows of at most SCORE_SHORT_V fp32 logits that come as the sum of `parts` matrices, added in
// ascending order: the last layer of a network whose logits product was split over its sum.
static constexpr int SCORE_SHORT_V = 1024;
void score_logits(const float *logits, int parts, size_t part_stride, size_t rows, int classes, const TokensGiven &t, float scale,
                  float *row_loss, float *dlogits, void *stream);

}  // namespace easgd
