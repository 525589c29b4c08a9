// Choice of the next beams: the launch interface between the C ABI (lessdec_beams_api.hip) and the kernel file.
#pragma once

#include "lessdec_common.h"
#include "lessdec.h"

namespace lessdec {

constexpr int kBeamTile = 512;                       // logits that a wave takes at a time
constexpr int kBeamParts = 64;                       // of a row, at most: a lane each when they are joined

struct BeamArgs {
  int groups, beams, vocab, picks, end_token;
  int parts, per;                                    // of a row; logits in one
  const void *logits;
  long stride;
  const float *score;
  const unsigned char *ended;
  int *parent, *token;
  float *next_score;
  unsigned char *next_ended;
  int *counters;                                     // [rows + groups], 0 before and after a call
  unsigned long long *sums, *lists, *scores;         // [rows][parts][2], [rows][parts][picks], [rows][picks]
  int *tokens;                                       // [rows][picks]
};
hipError_t launch_beam_select(const BeamArgs &a, int dtype, hipStream_t st);

}  // namespace lessdec
