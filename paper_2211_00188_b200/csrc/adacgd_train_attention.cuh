// Declarations shared by the units of attention (adacgd_train.h): adacgd_train_attention.cu has the kernels that take any type,
// alignment and head length; adacgd_train_attention_mma.cu those for the 16-bit types on the tensor cores.
#pragma once

#include "adacgd_train.cuh"

namespace adacgd {

// Each returns the number of kernels launched, -1 after a failed launch, or 0 where it does not take the call.
int launch_attention_mma(const adacgd_attention_args& a, const Where& at);
int launch_attention_backward_mma(const adacgd_attention_backward_args& a, const Where& at);

// Sequences are cut into tiles of B rows.  With seq_start the host does not know their lengths: sequence q gets the tile numbers
// from floor(start / B) + q on, which leaves room for ceil(length / B) of them, and the numbers behind a sequence's last tile do nothing.
inline long long tile_slots(const adacgd_attention_inputs& a, int B) {
  if (a.seq_start) return a.tokens / B + a.sequences;
  const long long each = a.tokens / a.sequences;
  return a.sequences * ((each + B - 1) / B);
}

struct Tile {
  long long row;   // the sequence's first row
  int length;      // and its rows
  int first;       // the tile's first row within it
};
// A tile by its number.  False: there is none.  Called by whole warps with the same arguments: a warp looks at 32 sequences a round.
__device__ __forceinline__ bool tile_of(const adacgd_attention_inputs& a, long long slot, int B, Tile* t) {
  long long q = 0, tile, lo, hi;
  if (a.seq_start) {
    // a lane holds the start of sequence l + lane * step; in the last round the steps are one and the next lane's is the end
    long long l = 0, h = a.sequences, start;
    int m;
    for (;;) {
      const long long step = (h - l + 30) / 31, at = l + (threadIdx.x & 31) * step;
      start = a.seq_start[at < a.sequences ? at : a.sequences];
      start = start < 0 ? 0 : (start > a.tokens ? a.tokens : start);
      m = __popc(__ballot_sync(0xffffffffu, at < h && (threadIdx.x & 31) < 31 && start / B + at <= slot));   // the last that begins at or before the slot
      if (m > 0) --m;
      if (step == 1) break;
      l += m * step;
      h = l + step < h ? l + step : h;
    }
    q = l + m;
    lo = __shfl_sync(0xffffffffu, start, m);
    hi = __shfl_sync(0xffffffffu, start, m + 1);
    if (hi < lo) hi = lo;
    tile = slot - (lo / B + q);
  } else {
    const long long each = a.tokens / a.sequences, per = (each + B - 1) / B;
    q = slot / per;
    tile = slot - q * per;
    lo = q * each;
    hi = lo + each;
  }
  if (tile < 0 || tile * B >= hi - lo) return false;
  t->row = lo;
  t->length = (int)(hi - lo);
  t->first = (int)(tile * B);
  return true;
}

}  // namespace adacgd
