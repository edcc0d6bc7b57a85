// Device code shared by the cached-history kernels: sequence lookup, page lookup and the
// rotation's angles.
#pragma once

#include "cast_common.h"

namespace cast {

// Division of 0 <= x by a fixed d >= 1 through one 64-bit product: exact for x * d < 2^40
// and x < 2^24 d (the entry points refuse sizes past that).
struct FastDiv {
  unsigned long long magic;
  int d;
};
inline FastDiv fast_div(int d) {
  return FastDiv{((1ull << 40) + (unsigned long long)d - 1) / (unsigned long long)d, d};
}
__device__ __forceinline__ int div_by(int x, FastDiv f) {
  return (int)(((unsigned long long)(unsigned)x * f.magic) >> 40);
}

// The sequences of a call as the kernels read them.  Garbage in the device arrays gives
// garbage results, never an access outside the tensors.
struct KvSeqs {
  const int32_t* cu;
  const int32_t* len;
  const int32_t* table;
  int n_seq, n_tok, max_pages;
  int max_tokens;                // max_pages * page
  FastDiv page;
};

__device__ __forceinline__ int seq_row(const KvSeqs& s, int b) { return min(max(s.cu[b], 0), s.n_tok); }
__device__ __forceinline__ int seq_len(const KvSeqs& s, int b) { return min(max(s.len[b], 0), s.max_tokens); }

// The last b in [0, n_seq) with start(b) <= x, for a start() that does not decrease and
// start(0) <= x: 64 probes per step, one per lane (one step up to 64 sequences).  Every
// lane of the wave calls it with the same x.
template <class F>
__device__ __forceinline__ int find_seq(int n_seq, int x, F&& start) {
  const int lane = threadIdx.x & 63;
  int lo = 0, cnt = n_seq;
  while (cnt > 1) {
    const int step = (cnt + 63) >> 6;
    const int b = lo + lane * step;
    const unsigned long long hit = __ballot(b < lo + cnt && start(b) <= x);
    const int c = max(__popcll(hit), 1);
    const int at = (c - 1) * step;
    lo += at;
    cnt = min(step, cnt - at);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Two e4m3 codes, the lower or upper ones of a word, under the scale of an exponent byte, as bf16:
// code * 2^(byte - 127), exactly where bf16 has that (always from byte 3 to 246), infinite past its
// range; all NaN for byte 255.
__device__ __forceinline__ float byte_scale(int e) { return __uint_as_float((uint32_t)e << 23); }
template <bool HI>
__device__ __forceinline__ uint32_t widen2(uint32_t codes, float sc) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, sc, HI));
}

// The rotation as the kernels read it.
struct Rope {
  const double* turns;
  const uint8_t* axis;
  const int32_t* pos;            // [n, n_axes], or NULL: the token's index in its sequence
  int rot, inter, n_axes;
  float amp;
  float sign;                    // -1: transposed
};

__device__ __forceinline__ int rope_axis(const Rope& r, int j) {
  return r.axis == nullptr ? 0 : min((int)r.axis[j], r.n_axes - 1);
}

// The angle of a pair at position p: k quarter turns and the rest r of one, r in [-0.5, 0.5].
// Whole turns of `turns` go first, so p times the rest stays below 2^33 quarters, whose
// integer part the addition of 1.5 * 2^52 leaves in the sum's low bits; r is rounded once.
// (In fp32 p = 10^6 and turns ~ 0.16 would leave no angle at all: 2^-24 * 1.6e5 = 0.01 turns.)
struct Angle {
  int k;
  float r;
};
__device__ __forceinline__ double quarter_turns(double turns) { return 4.0 * (turns - rint(turns)); }
__device__ __forceinline__ Angle rope_angle(double quarters, int p) {
  constexpr double kInt = 6755399441055744.0;    // 1.5 * 2^52
  const double t = fma((double)p, quarters, kInt);
  return Angle{(int)__double_as_longlong(t), (float)fma((double)p, quarters, kInt - t)};
}

}  // namespace cast
