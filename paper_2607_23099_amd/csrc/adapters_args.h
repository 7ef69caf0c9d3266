// Arguments of the adapters' kernels, and the launches that other files have.
#pragma once

#include <cstdint>

#include <hip/hip_runtime.h>

namespace damoe {

struct DownArgs {
  const void* x;   // rows that are contracted (x, dy)
  int64_t ldx;
  const void* w;   // A [L][r][C], or B [L][C][r]
  const int32_t* perm;
  const int32_t* off;
  const float* scale;  // of a segment's sums, or NULL
  float* part;     // [parts][T][rp], or NULL: with one part, what `up` takes and u are written
  void* ready;     // Ready, groups of places from each segment's first on
  float* u;        // [T][r] or NULL
  int32_t L, T, C, r, rp;
  int32_t places;  // of a block
  int32_t units;   // of columns that a block takes
};

struct UpArgs {
  const float* part;  // [parts][T][rp], joined here (UpJoin)
  void* ready;        // else: Ready
  int32_t parts;
  float* u;           // UpJoin: NULL, or the joined sums [T][r]
  const void* w;      // B [L][C][r], or A [L][r][C]
  const float* scale;
  const int32_t* perm;
  const int32_t* off;
  const void* add;
  int64_t lda;
  void* y;
  int64_t ldy;
  char* spare;        // not UpJoin: kSpare bytes that nothing reads
  int32_t L, T, C, r, rp, places;
};

struct OuterArgs {
  const void* x;       // rows (x, dy)
  int64_t ldx;
  const void* by_rank; // the other factor, of `sums`, or (of few places) as it is:
  const float* part;   // [parts][T][ld]
  int32_t parts, ld;
  const float* scale;  // of a segment's sums, or NULL
  const int32_t* perm;
  const int32_t* off;
  float* out;          // dA [L][r][C], or dB [L][C][r]
  float* slots;        // parts of segments of several chunks, laid out as the output
  int32_t n_slots;     // no more are there, whatever the offsets are
  int32_t L, T, C, r, rp, chunk, accumulate;
};

// y in one launch, where the work that blocks then share costs less than a second one.
bool adapters_few(int32_t T, int32_t L, int32_t rp, int32_t K, int32_t N, int32_t ydtype, int32_t wdtype);
hipError_t adapters_in_one(DownArgs a, const UpArgs& b, int32_t xdtype, int32_t wdtype, int32_t ydtype, hipStream_t stream);

// dx, dA and dB in one launch.  Few rows: behind `down`, which has left g's parts, a segment is one chunk and empty ones are
// cleared; joined: behind `sums`.
bool adapters_grad_few(int32_t T, int32_t L, int32_t r, int32_t K, int32_t N, int32_t xdtype, int32_t ydtype);
bool adapters_grad_joined(int32_t T, int32_t L, int32_t r, int32_t K, int32_t N, int32_t xdtype, int32_t ydtype);
hipError_t adapters_grad_in_one(const OuterArgs& b, const OuterArgs& a, UpArgs x, bool few, int32_t dtype, int32_t wdtype,
                                hipStream_t stream);

}  // namespace damoe
