// What the other parts of the library need of the distillation kernels.
#pragma once
#include "logits.h"

namespace easgd {

// What a teacher gives for rows of logits (see include/easgd.h).
struct TeacherGiven {
    const int *indices;
    const float *values, *lse;
    int k;
    const int *labels;
    float temperature, hard;
};

// The checks of a teacher's arguments that every call shares; EASGD_OK, or the error with its message set.
int check_teacher(const char *name, const TeacherGiven &t, bool rows);

// Losses and gradients of rows of at most DISTILL_SHORT_V fp32 logits that come as the sum of `parts` matrices, added in
// ascending order: the last layer of a network whose logits product was split over its sum.
static constexpr int DISTILL_SHORT_V = 1024;
void distill_logits(const float *logits, int parts, size_t part_stride, size_t rows, int classes, const TeacherGiven &t, float scale,
                    float *row_loss, float *dlogits, void *stream);

}  // namespace easgd
