// Launcher of beams.hip.  Its arguments have been checked.
#pragma once
#include "../../include/llmint8.h"
#include "common.h"

namespace llmint8 {

struct BeamArgs {  // llmint8_beam_select's arguments
    const void* logits;
    long long ld;
    int items, beams, vocab;
    const float* scores;
    const int* ended;
    int eos, n_out;
    float* scores_out;
    int *parent, *token, *ended_out, *status;
};
int beam_parts(long long rows, int vocab);  // pieces that a row is cut into
size_t beam_ws(long long rows, int vocab, int n_out);
hipError_t launch_beam_select(const BeamArgs& a, bool f32, void* ws, hipStream_t st);

}  // namespace llmint8
