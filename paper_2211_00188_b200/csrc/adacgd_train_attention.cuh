// Declarations shared by the units of attention (adacgd_train.h): adacgd_train_attention.cu has the kernels that take any type,
// alignment and head length; adacgd_train_attention_mma.cu those for the 16-bit types on the tensor cores.
#pragma once

#include "adacgd_train.cuh"

namespace adacgd {

// Each returns the number of kernels launched, -1 after a failed launch, or 0 where it does not take the call.
int launch_attention_mma(const adacgd_attention_args& a, const Where& at);
int launch_attention_backward_mma(const TrainScratch& ws, const adacgd_attention_backward_args& a, const Where& at);

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
// A tile by its number.  False: there is none.  All threads of a CTA may call it with the same arguments.
__device__ __forceinline__ bool tile_of(const adacgd_attention_inputs& a, long long slot, int B, Tile* t) {
  long long q = 0, tile, lo, hi;
  if (a.seq_start) {
    long long l = 0, h = a.sequences;                // the last q whose numbers begin at or before the slot
    while (h - l > 1) {
      const long long mid = (l + h) >> 1;
      long long s = a.seq_start[mid];
      s = s < 0 ? 0 : (s > a.tokens ? a.tokens : s);
      if (s / B + mid <= slot) l = mid; else h = mid;
    }
    q = l;
    seq_bounds(a.seq_start, q, a.tokens, 0, &lo, &hi);
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
