// C ABI of the choice of beams: argument checks and the launch.  Nothing here allocates, synchronises or keeps state between calls.
#include "lessdec_beams.h"

namespace {

using namespace lessdec;

inline bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

bool shape_ok(const lessdec_beam_desc *d)
{
  if (!d) return false;
  if (d->groups < 1 || d->beams < 1 || d->beams > LESSDEC_MAX_BEAMS || (long)d->groups * d->beams > 1L << 20) return false;
  if (d->vocab < 1 || d->vocab > 1 << 28 || d->picks < 1 || d->picks > LESSDEC_MAX_PICKS) return false;
  if (d->dtype != LESSDEC_DTYPE_F32 && d->dtype != LESSDEC_DTYPE_F16 && d->dtype != LESSDEC_DTYPE_BF16) return false;
  return d->end_token >= -1 && d->end_token < d->vocab;
}

// Parts of a row: as many as make kEnough workgroups of all rows (five to a compute unit, which the registers hold), a tile for each wave at least.
constexpr int kEnough = 1280;
void split(const lessdec_beam_desc *d, int *parts, int *per)
{
  const long rows = (long)d->groups * d->beams, unit = 4 * kBeamTile, units = (d->vocab + unit - 1) / unit;
  long n = (kEnough + rows - 1) / rows;
  n = n < units ? n : units;
  n = n < kBeamParts ? n : kBeamParts;
  const long each = (units + n - 1) / n;
  *parts = (int)((units + each - 1) / each);
  *per = (int)(each * unit);
}

struct Layout {
  size_t sums, lists, scores, tokens, total;
};
Layout layout(const lessdec_beam_desc *d, int parts)
{
  const size_t rows = (size_t)d->groups * d->beams, picks = (size_t)d->picks;
  Layout l;
  l.sums = align_up((rows + d->groups) * sizeof(int));
  l.lists = l.sums + align_up(rows * parts * 16);
  l.scores = l.lists + align_up(rows * parts * picks * 8);
  l.tokens = l.scores + align_up(rows * picks * 8);
  l.total = l.tokens + align_up(rows * picks * 4);
  return l;
}

}  // namespace

extern "C" {

size_t lessdec_beam_workspace_bytes(const lessdec_beam_desc *desc)
{
  if (!shape_ok(desc)) return 0;
  int parts, per;
  split(desc, &parts, &per);
  return layout(desc, parts).total;
}

int lessdec_beam_select(const lessdec_beam_desc *desc, const void *logits, int64_t row_stride, const float *score, const uint8_t *ended,
                        int32_t *parent, int32_t *token, float *next_score, uint8_t *next_ended, void *hip_stream)
{
  if (!shape_ok(desc)) return LESSDEC_EINVAL;
  const size_t size = desc->dtype == LESSDEC_DTYPE_F32 ? 4 : 2;
  const long stride = row_stride == 0 ? desc->vocab : (long)row_stride;
  if (stride < desc->vocab || stride > 1L << 40) return LESSDEC_EINVAL;
  if (!logits || !score || !parent || !token || !next_score || !aligned(logits, size) || !aligned(score, 4) || !aligned(parent, 4) ||
      !aligned(token, 4) || !aligned(next_score, 4))
    return LESSDEC_EINVAL;
  if (ended && desc->end_token < 0) return LESSDEC_EINVAL;
  if (parent == token) return LESSDEC_EINVAL;
  // in place only where a prompt's picks take the place of its beams
  if (desc->picks != desc->beams && (next_score == score || (ended && next_ended == ended))) return LESSDEC_EINVAL;
  BeamArgs a;
  split(desc, &a.parts, &a.per);
  const Layout l = layout(desc, a.parts);
  if (!desc->workspace || !aligned(desc->workspace, 256) || desc->workspace_bytes < l.total) return LESSDEC_EWORKSPACE;
  a.groups = desc->groups; a.beams = desc->beams; a.vocab = desc->vocab; a.picks = desc->picks; a.end_token = desc->end_token;
  a.logits = logits; a.stride = stride; a.score = score; a.ended = ended;
  a.parent = parent; a.token = token; a.next_score = next_score; a.next_ended = next_ended;
  char *w = static_cast<char *>(desc->workspace);
  a.counters = reinterpret_cast<int *>(w);
  a.sums = reinterpret_cast<unsigned long long *>(w + l.sums);
  a.lists = reinterpret_cast<unsigned long long *>(w + l.lists);
  a.scores = reinterpret_cast<unsigned long long *>(w + l.scores);
  a.tokens = reinterpret_cast<int *>(w + l.tokens);
  return launch_beam_select(a, desc->dtype, (hipStream_t)hip_stream) == hipSuccess ? LESSDEC_OK : LESSDEC_EHIP;
}

}  // extern "C"
