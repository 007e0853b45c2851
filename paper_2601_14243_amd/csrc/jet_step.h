// Arguments of the operators of a training step around the blocks: embedding, layer norm, gradient norm and clipping.
#pragma once
#include <stdint.h>

#include "jet_step_plan.h"

namespace jet {

struct EmbedArgs {
    const void* ids;              // int64 or int32 [T]
    bool wide;                    // int64
    long T, rows, first;          // tokens; rows of the table, which are those of ids first ..
    int H;
    float scale;
    bool f32;                     // the table's (gradient's) type, else bf16
    const void* w;                // forward
    uint16_t* y;
    const uint16_t* dy;           // gradient
    void* dw;
    bool add;                     // to what dw holds
};

struct NormArgs {
    const uint16_t *x, *res, *gamma, *beta;   // res, beta may be null; in the backward pass res is the gradient beside the norm
    float eps;
    long M;
    int K;
    uint16_t *y, *sum;            // forward: y or the E4M3 pair; sum with res
    uint8_t* q;
    float* s;
    const uint16_t* dy;           // backward
    bool layer;                   // with the mean, else RMS
    uint16_t* dx;
    float *dgamma, *dbeta;
    float* partial;
};

}  // namespace jet
