// Rotary positions, appending to a paged cache with the rotation on the way, and reading
// pages back as bf16 blocks.  All three are bound by HBM (or, for a few tokens, by the
// latency of one launch): every value is read once, converted in registers, written once.
// 28160 tokens of 24 heads of 128 channels rotated: 66 us, 5.2 TB/s; 24960 tokens of 12 heads
// appended in bf16: 62 us, 4.9 TB/s; 15000 tokens of 8 heads in e4m3, half of the channels
// rotated: 28 us, 3.3 TB/s (the angles and the two passes over a page take as long as the
// memory), read back as bf16 29 us; a frame of 1560 tokens of 12 heads as one e4m3 page 17 us
// (three launches of 7.8, 3.8 and 6.7), sixteen of them 84; 16 e4m3 pages of 3520 tokens of 24
// heads read: 171 us, 6.1 TB/s.
#include <algorithm>

#include "kv_device.h"

namespace cast {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kTok = 4;          // tokens per block of the rotating kernels: 4 x 64 pairs = one angle a thread
constexpr int kMaxPairs = 64;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ float to_f32(uint16_t w) { return __uint_as_float((uint32_t)w << 16); }
__device__ __forceinline__ float to_f32(float w) { return w; }
__device__ __forceinline__ void from_f32(uint16_t* p, float v) { *p = (uint16_t)pack_bf16(v, 0.0f); }
__device__ __forceinline__ void from_f32(float* p, float v) { *p = v; }

// eight consecutive channels
__device__ __forceinline__ void load8(const uint16_t* p, float* f) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16lo(w[i]);
    f[2 * i + 1] = bf16hi(w[i]);
  }
}
__device__ __forceinline__ void load8(const float* p, float* f) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[i] = a[i];
    f[4 + i] = b[i];
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const float* f) {
  *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
}
__device__ __forceinline__ void store8(float* p, const float* f) {
  *reinterpret_cast<f32x4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
}

// How the channels of a head are shared out over threads ("items"), each with both
// channels of its pairs, so that out may be x itself:
//   2  half layout, rot a multiple of 16: item i < rot/16 takes chunks i and i + rot/16 of
//      eight channels, the others a chunk of the channels that pass through
//   1  interleaved layout, rot a multiple of 8: item i takes chunk i
//   0  any rot, any alignment: item j < rot/2 takes pair j, the others one channel
struct Items {
  int mode, per_head;
  FastDiv div;                   // by per_head
};
Items plan_items(int rot, int inter, int dh, bool wide) {
  Items t;
  t.mode = wide && !inter && rot % 16 == 0 ? 2 : wide && (inter || rot == 0) && rot % 8 == 0 ? 1 : 0;
  t.per_head = t.mode == 2 ? rot / 16 + (dh - rot) / 8 : t.mode == 1 ? dh / 8 : rot / 2 + (dh - rot);
  t.div = fast_div(t.per_head);
  return t;
}

// cs[j] = (cos, sin) of pair j, x and y the same head's row in and out
template <class T>
__device__ __forceinline__ void rotate_item(const T* x, T* y, int i, int mode, int rot, int inter,
                                            const f32x2* cs) {
  if (mode == 2) {
    const int half = rot >> 1;
    if (i < (rot >> 4)) {
      float a[8], b[8], p[8], q[8];
      load8(x + 8 * i, a);
      load8(x + 8 * i + half, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const f32x2 c = cs[8 * i + e];
        p[e] = fmaf(a[e], c.x, -(b[e] * c.y));
        q[e] = fmaf(a[e], c.y, b[e] * c.x);
      }
      store8(y + 8 * i, p);
      store8(y + 8 * i + half, q);
      return;
    }
    const int c = rot + 8 * (i - (rot >> 4));
    float a[8];
    load8(x + c, a);
    store8(y + c, a);
  } else if (mode == 1) {
    float a[8];
    load8(x + 8 * i, a);
    if (8 * i < rot) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x2 c = cs[4 * i + e];
        const float u = a[2 * e], w = a[2 * e + 1];
        a[2 * e] = fmaf(u, c.x, -(w * c.y));
        a[2 * e + 1] = fmaf(u, c.y, w * c.x);
      }
    }
    store8(y + 8 * i, a);
  } else if (i < (rot >> 1)) {
    const int c0 = inter ? 2 * i : i, c1 = inter ? 2 * i + 1 : i + (rot >> 1);
    const f32x2 c = cs[i];
    const float u = to_f32(x[c0]), w = to_f32(x[c1]);
    from_f32(y + c0, fmaf(u, c.x, -(w * c.y)));
    from_f32(y + c1, fmaf(u, c.y, w * c.x));
  } else {
    const int c = rot + (i - (rot >> 1));
    y[c] = x[c];
  }
}

// a (cos, sin) of an angle.  Of the rest of a quarter turn, r of [-1/8, 1/8] in turns,
//   sin(2 pi r) = r (2 pi + P(r^2)),  cos(2 pi r) = 1 + r^2 Q(r^2)
// with P and Q fitted over that range to less than 1e-8 (2 pi in two parts): least squares on
// Chebyshev points, the weights multiplied by the errors until these level out (Lawson's
// algorithm), the coefficients then rounded to fp32.  Off by at most
// 7.5e-8, about one fp32 step of 1.  v_cos and v_sin of an fp32 angle are off by up to 2.2e-7:
// they put 18 of the 15 million codes of 15000 tokens of 8 heads on the other side of a
// rounding, this 9 (means of six caches), and saved 4 of the append's 32 us.
__device__ __forceinline__ f32x2 cos_sin(Angle t, float amp) {
  const float r = 0.25f * t.r, s = r * r;
  const float p = fmaf(fmaf(fmaf(-75.7257843f, s, 81.5995178f), s, -41.3416977f), s, -1.74845553e-7f);
  const float q = fmaf(fmaf(fmaf(59.4235306f, s, -85.4488068f), s, 64.9393692f), s, -19.7392082f);
  const float sn = fmaf(r, 6.28318548f, r * p), cn = fmaf(s, q, 1.0f);
  const unsigned k = (unsigned)t.k;
  const float c = (k & 1) ? sn : cn, d = (k & 1) ? cn : sn;
  return f32x2{__uint_as_float(__float_as_uint(c) ^ (((k + 1) & 2) << 30)) * amp,
               __uint_as_float(__float_as_uint(d) ^ ((k & 2) << 30)) * amp};
}

// (cos, sin) of the block's tokens' pairs into LDS: token of the block tt, position of axis
// a given by pos_of(tt, a).
template <class F>
__device__ __forceinline__ void fill_angles(f32x2 (*cs)[kMaxPairs], const Rope& r, F&& pos_of) {
  const int pairs = r.rot >> 1;
  for (int t = threadIdx.x; t < kTok * kMaxPairs; t += kThreads) {
    const int tt = t / kMaxPairs, j = t % kMaxPairs;
    if (j < pairs) {
      const f32x2 c = cos_sin(rope_angle(quarter_turns(r.turns[j]), pos_of(tt, rope_axis(r, j))), r.amp);
      cs[tt][j] = f32x2{c.x, c.y * r.sign};
    }
  }
}

// ---------------------------------------------------------------------------
// cast_rope
// ---------------------------------------------------------------------------
// One block takes kTok tokens and one of gridDim.y shares of the heads; the angles of a
// token are formed once per block and shared by its heads.  Few tokens: the heads are
// shared out over more blocks (latency); many: one block takes them all.
template <class T>
__global__ __launch_bounds__(kThreads) void rope_kernel(const T* x, long long xt, long long xh, T* y,
                                                        long long yt, long long yh, int n, int H,
                                                        int heads, Rope r, Items it) {
  __shared__ f32x2 cs[kTok][kMaxPairs];
  const int t0 = blockIdx.x * kTok, nt = min(kTok, n - t0);
  fill_angles(cs, r, [&](int tt, int a) { return r.pos[(long long)min(t0 + tt, n - 1) * r.n_axes + a]; });
  __syncthreads();
  const int h0 = blockIdx.y * heads, nh = min(heads, H - h0);
  const int per_tok = nh * it.per_head;
#pragma unroll 2
  for (int i = threadIdx.x; i < nt * per_tok; i += kThreads) {
    const int tt = i / per_tok, rem = i - tt * per_tok;
    const int h = div_by(rem, it.div), item = rem - h * it.per_head;
    const long long t = t0 + tt;
    rotate_item(x + t * xt + (h0 + h) * xh, y + t * yt + (h0 + h) * yh, item, it.mode, r.rot, r.inter, cs[tt]);
  }
}

// ---------------------------------------------------------------------------
// cast_kv_append, bf16 cache (and the queries of both)
// ---------------------------------------------------------------------------
struct AppendArgs {
  KvSeqs s;
  Rope r;
  Items it;                      // rotation of one head
  const uint16_t* k;
  const uint16_t* v;
  const uint16_t* q;
  uint16_t* q_out;
  void* kc;
  void* vc;
  uint8_t* ke;
  uint8_t* ve;
  long long ks, vs, qs;          // token strides
  int H, Hq, dh, pages, page;
  int heads;                     // heads of K, V and Q together per block
  int q_blocks_x, q_shares;      // 8-bit: blocks of the queries in front of the pages'
  int part_log2;                 // 8-bit, long pages: tokens of a part
  FastDiv page_parts;            // by the parts of a page
};

// Sequence, index in it and row of the cache (-1: none) of a call's row: one wave per row.
__device__ __forceinline__ void locate(const AppendArgs& a, int row, int* index, int* slot, int* mine) {
  const int b = find_seq(a.s.n_seq, row, [&](int i) { return seq_row(a.s, i); });
  const int beg = seq_row(a.s, b), end = seq_row(a.s, b + 1);
  const int t = seq_len(a.s, b) - (end - row);
  const bool in = row >= beg && row < end;
  int at = -1;
  if (in && t >= 0) {
    const int p = div_by(t, a.s.page);
    const int id = a.s.table[(long long)b * a.s.max_pages + p];
    if (id >= 0 && id < a.pages) at = id * a.page + (t - p * a.page);
  }
  *index = t;
  *slot = at;
  *mine = in;
}

// Heads are counted K 0 .. H, V .. 2 H, Q .. 2 H + Hq; block (x, y) takes kTok tokens and
// the heads [y heads, (y + 1) heads) of that count, from `first` on.
__device__ __forceinline__ void append_rows(const AppendArgs& a, int bx, int by, int first,
                                            f32x2 (*cs)[kMaxPairs], int* index, int* slot, int* mine) {
  const int t0 = bx * kTok, n = a.s.n_tok, nt = min(kTok, n - t0);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave < nt) locate(a, t0 + wave, index + wave, slot + wave, mine + wave);
  __syncthreads();
  if (a.r.rot > 0) {
    fill_angles(cs, a.r, [&](int tt, int ax) {
      const int t = min(tt, nt - 1);
      return a.r.pos != nullptr ? a.r.pos[(long long)(t0 + t) * a.r.n_axes + ax] : index[t];
    });
    __syncthreads();
  }
  const int h0 = first + by * a.heads, nh = min(a.heads, 2 * a.H + a.Hq - h0);
  const int per_tok = nh * a.it.per_head;
  const long long row = (long long)a.H * a.dh;
  for (int i = threadIdx.x; i < nt * per_tok; i += kThreads) {
    const int tt = i / per_tok, rem = i - tt * per_tok;
    int h = div_by(rem, a.it.div);
    const int item = rem - h * a.it.per_head;
    h += h0;
    const long long t = t0 + tt;
    if (h < 2 * a.H) {
      if (slot[tt] < 0) continue;
      const bool is_v = h >= a.H;
      if (is_v) h -= a.H;
      const uint16_t* x = is_v ? a.v + t * a.vs + h * a.dh : a.k + t * a.ks + h * a.dh;
      uint16_t* y = static_cast<uint16_t*>(is_v ? a.vc : a.kc) + (long long)slot[tt] * row + h * a.dh;
      if (is_v) {
        // the items of a head cover its channels in some order: copy the same ones
        if (a.it.mode == 2) {
          const bool two = item < (a.r.rot >> 4);
          const int c = two ? 8 * item : a.r.rot + 8 * (item - (a.r.rot >> 4));
          const u32x4 w = *reinterpret_cast<const u32x4*>(x + c);
          if (two) {
            const u32x4 w2 = *reinterpret_cast<const u32x4*>(x + c + (a.r.rot >> 1));
            *reinterpret_cast<u32x4*>(y + c + (a.r.rot >> 1)) = w2;
          }
          *reinterpret_cast<u32x4*>(y + c) = w;
        } else if (a.it.mode == 1) {
          *reinterpret_cast<u32x4*>(y + 8 * item) = *reinterpret_cast<const u32x4*>(x + 8 * item);
        } else if (item < a.dh / 8) {
          *reinterpret_cast<u32x4*>(y + 8 * item) = *reinterpret_cast<const u32x4*>(x + 8 * item);
        }
      } else {
        rotate_item(x, y, item, a.it.mode, a.r.rot, a.r.inter, cs[tt]);
      }
    } else if (mine[tt]) {
      h -= 2 * a.H;
      rotate_item(a.q + t * a.qs + h * a.dh, a.q_out + (t * a.Hq + h) * a.dh, item, a.it.mode, a.r.rot, a.r.inter, cs[tt]);
    }
  }
}

__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  __shared__ f32x2 cs[kTok][kMaxPairs];
  __shared__ int index[kTok], slot[kTok], mine[kTok];
  append_rows(a, blockIdx.x, blockIdx.y, 0, cs, index, slot, mine);
}

// ---------------------------------------------------------------------------
// cast_kv_append, e4m3 cache
// ---------------------------------------------------------------------------
// Four values as e4m3 codes (nearest even) under 1/scale `inv`: |v * inv| <= 448 for finite
// v, infinities and NaN become NaN.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
}
// 2^-e for -127 < e <= 128 (below 2^-126 a subnormal)
__device__ __forceinline__ float inverse_scale(int e) { return __uint_as_float(e < 127 ? (uint32_t)(127 - e) << 23 : 0x00400000u >> (e - 127)); }

// the least e >= -117 with top <= 448 * 2^e (448 = 0.875 * 2^9)
__device__ __forceinline__ int need_exp(float top) {
  if (!(top > 0.0f)) return -117;
  int e;
  const float m = frexpf(top, &e);
  return max(e - 9 + (m > 0.875f ? 1 : 0), -117);
}

__device__ __forceinline__ void unpack8(u32x4 w, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16lo(w[i]);
    f[2 * i + 1] = bf16hi(w[i]);
  }
}

// The new rows of one (page, head, K or V): the largest magnitude gives the exponent, then
// the codes are written.  An item is two chunks of eight channels; a thread keeps one item
// of every `step`-th token, so the frequencies of its pairs are read once and an angle
// serves both channels of its pair.
//   MODE 0  no rotation: chunks 2 i and 2 i + 1
//        1  half layout, rot a multiple of 16: items < rot/16 take chunks i and i + rot/16
//        2  interleaved
//        3  half layout, any rot: partners are read one by one
// kKeep items are loaded together and stay in registers between the two passes; longer
// pages are read again (from the L2).
struct PageRows {
  const uint16_t* src;           // the call's first row of the page, this head
  long long ss;                  // its token stride
  uint8_t* page;                 // row 0 of the page, this head
  long long cs;                  // its row stride
  uint8_t* exponent;
  int had, n, row0, index0;      // earlier tokens, new ones; first call row and index in the sequence
};
constexpr int kKeep = 2;

// The first `rows` tokens of a page, at channel `at` from its head on, rounded to an exponent
// that has grown by `up`.
__device__ __forceinline__ void round_again(const PageRows& g, int at, int rows, int up, int dh) {
  if (rows == 0 || up <= 0) return;
  const int ipr = dh >> 4, shift = 31 - __clz(ipr), item = threadIdx.x & (ipr - 1), step = kThreads >> shift;
  const float down = up < 127 ? inverse_scale(up) : 0.0f;
  for (int t = threadIdx.x >> shift; t < rows; t += step) {
    u32x4* p = reinterpret_cast<u32x4*>(g.page + t * g.cs + at + 16 * item);
    const u32x4 w = *p;
    u32x4 o;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
      o[k] = codes4(lo.x, lo.y, hi.x, hi.y, down);
    }
    *p = o;
  }
}

// PHASE kFind and kStore are the two passes alone, over rows that stay in registers: kFind
// leaves the exponent that the rows need as the first byte of their first row, where kStore's
// codes come to lie.
enum Phase { kBoth, kFind, kStore };
template <int MODE, int NH, int PHASE>
__device__ __forceinline__ void store_page(const Rope& r, const PageRows& g, int dh, float (*tops)[kThreads / 64]) {
  const int ipr = dh >> 4, shift = 31 - __clz(ipr);            // items per row
  const int item = threadIdx.x & (ipr - 1), t0 = threadIdx.x >> shift, step = kThreads >> shift;
  const int half = r.rot >> 1;
  int c0 = 16 * item, c1 = c0 + 8;               // first channels of the item's chunks
  bool turns = MODE != 0 && c0 < r.rot;
  if (MODE == 1) {
    turns = item < (r.rot >> 4);
    if (turns) {
      c0 = 8 * item;
      c1 = c0 + half;
    }
  }
  constexpr int NF = MODE == 0 ? 1 : MODE == 3 ? 16 : 8;       // angles of an item
  double freq[NF];
  uint32_t axes = 0;                             // two bits each
  if (MODE != 0 && turns) {
#pragma unroll
    for (int e = 0; e < NF; ++e) {
      const int ch = c0 + e;
      const int j = MODE == 1 ? ch : MODE == 2 ? (c0 >> 1) + e : ch >= half ? ch - half : ch;
      const int jj = min(j, half - 1);
      freq[e] = quarter_turns(r.turns[jj]);
      axes |= (uint32_t)rope_axis(r, jj) << (2 * e);
    }
  }
  auto fetch = [&](int base, float (&y)[NH][kKeep][16]) __attribute__((always_inline)) {
    u32x4 w[NH][kKeep][2];
#pragma unroll
    for (int j = 0; j < kKeep; ++j) {
      const uint16_t* row = g.src + min(base + t0 + j * step, g.n - 1) * g.ss;
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        w[h][j][0] = *reinterpret_cast<const u32x4*>(row + h * dh + c0);
        w[h][j][1] = *reinterpret_cast<const u32x4*>(row + h * dh + c1);
      }
    }
#pragma unroll
    for (int j = 0; j < kKeep; ++j) {
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        unpack8(w[h][j][0], y[h][j]);
        unpack8(w[h][j][1], y[h][j] + 8);
      }
      if (MODE == 0 || !turns) continue;
      const int t = min(base + t0 + j * step, g.n - 1);
      const int32_t* pos = r.pos != nullptr ? r.pos + (long long)(g.row0 + t) * r.n_axes : nullptr;
      const int p0 = pos != nullptr ? pos[0] : g.index0 + t;
      auto angle = [&](int e) {
        return cos_sin(rope_angle(freq[e], r.n_axes > 1 && pos != nullptr ? pos[(axes >> (2 * e)) & 3] : p0), r.amp);
      };
      const uint16_t* row = g.src + t * g.ss;
#pragma unroll
      for (int e = 0; e < NF; ++e) {
        if (MODE == 3) {
          const int ch = c0 + e;
          if (ch < r.rot) {
            const f32x2 a = angle(e);
#pragma unroll
            for (int h = 0; h < NH; ++h) {
              const float o = to_f32(row[h * dh + (ch < half ? ch + half : ch - half)]);
              y[h][j][e] = fmaf(y[h][j][e], a.x, ch < half ? -(o * a.y) : o * a.y);
            }
          }
        } else {
          const int u = MODE == 1 ? e : 2 * e, z = MODE == 1 ? 8 + e : 2 * e + 1;
          if (MODE == 1 || c0 + 2 * e < r.rot) {
            const f32x2 a = angle(e);
#pragma unroll
            for (int h = 0; h < NH; ++h) {
              const float yu = y[h][j][u], yz = y[h][j][z];
              y[h][j][u] = fmaf(yu, a.x, -(yz * a.y));
              y[h][j][z] = fmaf(yu, a.y, yz * a.x);
            }
          }
        }
      }
    }
  };
  float top[NH];
#pragma unroll
  for (int h = 0; h < NH; ++h) top[h] = 0.0f;
  auto look = [&](const float (&y)[NH][kKeep][16]) __attribute__((always_inline)) {   // (repeated last rows do no harm)
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int j = 0; j < kKeep; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float m = fabsf(y[h][j][e]);
          top[h] = m < INFINITY ? fmaxf(top[h], m) : top[h];   // false for NaN, too
        }
  };
  int old[NH];
#pragma unroll
  for (int h = 0; h < NH; ++h) old[h] = (int)g.exponent[h] - 127;
  const int batch = kKeep * step;
  float keep[NH][kKeep][16];
#pragma unroll 1
  for (int base = 0; base < g.n; base += batch) {
    fetch(base, keep);
    if (PHASE != kStore) look(keep);
  }
  int ex[NH];
  if constexpr (PHASE == kStore) {
#pragma unroll
    for (int h = 0; h < NH; ++h) ex[h] = old[h];
  } else {
#pragma unroll
    for (int h = 0; h < NH; ++h) {
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) top[h] = fmaxf(top[h], __shfl_xor(top[h], d));
      if ((threadIdx.x & 63) == 0) tops[h][threadIdx.x >> 6] = top[h];
    }
    __syncthreads();                             // (also: every thread has read the old exponents)
#pragma unroll
    for (int h = 0; h < NH; ++h) {
#pragma unroll
      for (int w = 0; w < kThreads / 64; ++w) top[h] = fmaxf(top[h], tops[h][w]);
      const int need = need_exp(top[h]);
      ex[h] = PHASE == kBoth && g.had > 0 ? max(old[h], need) : need;
      if (threadIdx.x == 0) *(PHASE == kBoth ? g.exponent + h : g.page + g.had * g.cs + h * dh) = (uint8_t)(ex[h] + 127);
    }
    if (PHASE == kFind) return;
  }
#pragma unroll 1
  for (int base = 0; base < g.n; base += batch) {
    if (g.n > batch) fetch(base, keep);
#pragma unroll
    for (int j = 0; j < kKeep; ++j) {
      const int t = base + t0 + j * step;
      if (t < g.n) {
        uint8_t* at = g.page + (g.had + t) * g.cs;
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          const float inv = inverse_scale(ex[h]);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float* y = &keep[h][j][8 * k];
            *reinterpret_cast<u32x2*>(at + h * dh + (k == 0 ? c0 : c1)) =
                u32x2{codes4(y[0], y[1], y[2], y[3], inv), codes4(y[4], y[5], y[6], y[7], inv)};
          }
        }
      }
    }
  }
  if constexpr (PHASE == kBoth) {
#pragma unroll
    for (int h = 0; h < NH; ++h) round_again(g, h * dh, g.had, ex[h] - old[h], dh);
  }
}

// Rows lo .. hi of sequence b (end: its last call row + 1, len: its length), which lie in its page p.
__device__ __forceinline__ bool rows_of(const AppendArgs& a, int b, int end, int len, int p, int lo, int hi, int h, bool is_v,
                                        PageRows& g) {
  const int id = a.s.table[(long long)b * a.s.max_pages + p];
  if (id < 0 || id >= a.pages) return false;
  g.had = lo - p * a.page;
  g.n = hi - lo;
  g.row0 = end - (len - lo);
  g.index0 = lo;
  g.ss = is_v ? a.vs : a.ks;
  g.src = (is_v ? a.v : a.k) + h * a.dh + (long long)g.row0 * g.ss;
  g.cs = (long long)a.H * a.dh;
  g.page = static_cast<uint8_t*>(is_v ? a.vc : a.kc) + ((long long)id * a.page * a.H + h) * a.dh;
  g.exponent = (is_v ? a.ve : a.ke) + (long long)id * a.H + h;
  return true;
}
// The units of a launch: a number x for the rows, times V's heads and groups of nh of K's.
__device__ __forceinline__ int unit_rows(const AppendArgs& a, int unit, int nh, int& h, bool& is_v) {
  const int groups = a.H / nh, x = unit / (groups + a.H), rem = unit - x * (groups + a.H);
  is_v = rem >= groups;
  h = is_v ? rem - groups : rem * nh;
  return x;
}

// One block per (page of a sequence that the call writes, head of V or NH heads of K, which
// share their angles).  The call's pages
// of sequence b are numbered from cu[b] / page + 2 b (a sequence of n tokens meets at most
// ceil(n / page) + 1 pages, so the ranges do not meet).  KM: how keys are rotated.
__device__ __forceinline__ bool page_rows(const AppendArgs& a, int unit, int nh, PageRows& g, bool& is_v) {
  int h;
  const int x = unit_rows(a, unit, nh, h, is_v);
  const int b = find_seq(a.s.n_seq, x, [&](int i) { return div_by(seq_row(a.s, i), a.s.page) + 2 * i; });
  const int beg = seq_row(a.s, b), end = seq_row(a.s, b + 1), len = seq_len(a.s, b);
  const int first = max(len - (end - beg), 0);   // rows before token 0 are dropped
  const int p = div_by(first, a.s.page) + (x - (div_by(beg, a.s.page) + 2 * b));
  const int lo = max(first, p * a.page), hi = min(len, (p + 1) * a.page);
  if (x < div_by(beg, a.s.page) + 2 * b || end <= beg || lo >= hi) return false;
  return rows_of(a, b, end, len, p, lo, hi, h, is_v, g);
}

// Long pages: parts of 2^part_log2 rows, from a page's first row on.  n tokens meet at most
// n / part + n / page + 4 of them (n - 1 steps from token to token cross one border in a part's
// rows but for the short last part of each page they pass, and the two at their ends), so those
// of sequence b are numbered from cu[b] / part + cu[b] / page + 4 b: the grid goes by the tokens
// of the call, not by what its pages could hold.
__device__ __forceinline__ int parts_of(const AppendArgs& a, int n) { return (n >> a.part_log2) + div_by(n, a.s.page); }
__device__ __forceinline__ bool part_rows(const AppendArgs& a, int unit, int nh, PageRows& g, bool& is_v) {
  int h;
  const int x = unit_rows(a, unit, nh, h, is_v);
  const int b = find_seq(a.s.n_seq, x, [&](int i) { return parts_of(a, seq_row(a.s, i)) + 4 * i; });
  const int beg = seq_row(a.s, b), end = seq_row(a.s, b + 1), len = seq_len(a.s, b);
  const int j = x - (parts_of(a, beg) + 4 * b);
  if (end <= beg || j < 0 || j >= parts_of(a, end - beg) + 4) return false;
  const int first = max(len - (end - beg), 0), p0 = div_by(first, a.s.page);
  const int at = p0 * a.page_parts.d + ((first - p0 * a.page) >> a.part_log2) + j;
  const int p = div_by(at, a.page_parts), r0 = (at - p * a.page_parts.d) << a.part_log2;
  const int lo = max(first, p * a.page + r0), hi = min(len, p * a.page + min(r0 + (1 << a.part_log2), a.page));
  if (lo >= hi) return false;
  return rows_of(a, b, end, len, p, lo, hi, h, is_v, g);
}

template <int KM, int NH>
__global__ __launch_bounds__(kThreads) void append8_kernel(AppendArgs a) {
  __shared__ f32x2 cs[kTok][kMaxPairs];
  __shared__ int index[kTok], slot[kTok], mine[kTok];
  __shared__ float tops[NH][kThreads / 64];
  const int nq = a.q_blocks_x * a.q_shares;
  if ((int)blockIdx.x < nq) {
    append_rows(a, blockIdx.x % a.q_blocks_x, blockIdx.x / a.q_blocks_x, 2 * a.H, cs, index, slot, mine);
    return;
  }
  PageRows g;
  bool is_v;
  if (!page_rows(a, blockIdx.x - nq, NH, g, is_v)) return;
  if (is_v) store_page<0, 1, kBoth>(a.r, g, a.dh, tops);
  else store_page<KM, NH, kBoth>(a.r, g, a.dh, tops);
}

// Long pages, in three launches: the exponents that a block per part and head finds its rows to
// need (and the queries), the page's exponent from them, the codes.
template <int KM, int NH, int PHASE>
__global__ __launch_bounds__(kThreads) void append8_part_kernel(AppendArgs a) {
  __shared__ f32x2 cs[kTok][kMaxPairs];
  __shared__ int index[kTok], slot[kTok], mine[kTok];
  __shared__ float tops[NH][kThreads / 64];
  const int nq = PHASE == kFind ? a.q_blocks_x * a.q_shares : 0;
  if (PHASE == kFind && (int)blockIdx.x < nq) {
    append_rows(a, blockIdx.x % a.q_blocks_x, blockIdx.x / a.q_blocks_x, 2 * a.H, cs, index, slot, mine);
    return;
  }
  PageRows g;
  bool is_v;
  if (!part_rows(a, blockIdx.x - nq, NH, g, is_v)) return;
  if (is_v) store_page<0, 1, PHASE>(a.r, g, a.dh, tops);
  else store_page<KM, NH, PHASE>(a.r, g, a.dh, tops);
}
__global__ __launch_bounds__(kThreads) void append8_exponent_kernel(AppendArgs a) {
  PageRows g;
  bool is_v;
  if (!page_rows(a, blockIdx.x, 1, g, is_v)) return;
  const int old = (int)*g.exponent - 127;
  __syncthreads();                               // (every thread has read it)
  int need = g.page[g.had * g.cs];               // at the parts' first rows
#pragma unroll 8
  for (int row = ((g.had >> a.part_log2) + 1) << a.part_log2; row < g.had + g.n; row += 1 << a.part_log2)
    need = max(need, (int)g.page[row * g.cs]);
  const int e = g.had > 0 ? max(old, need - 127) : need - 127;
  if (threadIdx.x == 0) *g.exponent = (uint8_t)(e + 127);
  round_again(g, 0, g.had, e - old, a.dh);
}

// ---------------------------------------------------------------------------
// cast_kv_read
// ---------------------------------------------------------------------------
// A thread writes 16-byte chunks (eight channels), a block's width apart, so a wave writes
// 1 KB in a row; grid (parts of a page, page, K or V).
struct ReadArgs {
  const void* k;
  const void* v;
  const uint8_t* ke;
  const uint8_t* ve;
  const int32_t* idx;
  uint16_t* ko;
  uint16_t* vo;
  int pages, H;
  long long chunks;              // 16-byte chunks of bf16 in a page
  int cph_log2;                  // chunks per head
  FastDiv heads;                 // by H
};

template <bool F8>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a) {
  const bool is_v = a.ko == nullptr || blockIdx.z == 1;
  const int i = blockIdx.y;
  const int id = a.idx[i];
  uint16_t* out = (is_v ? a.vo : a.ko) + (long long)i * a.chunks * 8;
  const long long step = (long long)gridDim.x * kThreads;
  if (id < 0 || id >= a.pages) {
    for (long long c = (long long)blockIdx.x * kThreads + threadIdx.x; c < a.chunks; c += step)
      *reinterpret_cast<u32x4*>(out + 8 * c) = u32x4{0u, 0u, 0u, 0u};
    return;
  }
  const uint8_t* src = static_cast<const uint8_t*>(is_v ? a.v : a.k) + (long long)id * a.chunks * (F8 ? 8 : 16);
  const uint8_t* ex = F8 ? (is_v ? a.ve : a.ke) + (long long)id * a.H : nullptr;
#pragma unroll 4
  for (long long c = (long long)blockIdx.x * kThreads + threadIdx.x; c < a.chunks; c += step) {
    if constexpr (F8) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(src + 8 * c);
      const int at = (int)(c >> a.cph_log2), head = at - div_by(at, a.heads) * a.H;   // at: token and head
      const float sc = byte_scale(ex[head]);
      *reinterpret_cast<u32x4*>(out + 8 * c) = u32x4{widen2<false>(w.x, sc), widen2<true>(w.x, sc), widen2<false>(w.y, sc), widen2<true>(w.y, sc)};
    } else {
      *reinterpret_cast<u32x4*>(out + 8 * c) = *reinterpret_cast<const u32x4*>(src + 16 * c);
    }
  }
}

Rope make_rope(const cast_rope_params_t* p, const int32_t* pos, int transpose) {
  Rope r{};
  if (p == nullptr) return r;
  r.turns = p->turns;
  r.axis = p->n_axes > 1 ? p->axis : nullptr;
  r.pos = pos;
  r.rot = p->rot_dim;
  r.inter = p->interleaved;
  r.n_axes = p->n_axes;
  r.amp = p->amplitude;
  r.sign = transpose ? -1.0f : 1.0f;
  return r;
}

// `pages`, `parts`: how many of them the call can meet
template <int KM, int NH>
void launch_append8_parts(const AppendArgs& a, long long pages, long long parts, hipStream_t stream) {
  const unsigned nq = a.q_blocks_x * a.q_shares, units = (unsigned)(parts * (a.H + a.H / NH));
  hipLaunchKernelGGL((append8_part_kernel<KM, NH, kFind>), dim3(nq + units), dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL(append8_exponent_kernel, dim3((unsigned)pages * 2 * a.H), dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL((append8_part_kernel<KM, NH, kStore>), dim3(units), dim3(kThreads), 0, stream, a);
}

// heads per block: all of them once there are blocks for every compute unit several
// times over, else shared out down to about two items a thread
int heads_per_block(int tok_blocks, int heads, int per_head) {
  const int least = std::max(1, 2 * kThreads / (kTok * per_head));
  int shares = std::max(1, 1024 / std::max(tok_blocks, 1));
  int hpb = (heads + shares - 1) / shares;
  return std::min(std::max(hpb, least), heads);
}

}  // namespace

KvSeqs make_seqs(const cast_kv_seqs_t& s, int page) {
  return KvSeqs{s.cu, s.len, s.table, s.n_seq, s.n_tok, s.max_pages, s.max_pages * page, fast_div(page)};
}

cast_status_t launch_rope(const void* x, int dtype, int n, int H, int dh, long long xt, long long xh,
                          const int32_t* pos, const cast_rope_params_t& p, int transpose, void* out,
                          long long yt, long long yh, bool wide, hipStream_t stream) {
  Rope r = make_rope(&p, pos, transpose);
  const Items it = plan_items(r.rot, r.inter, dh, wide);
  const int heads = heads_per_block((n + kTok - 1) / kTok, H, it.per_head);
  constexpr int kMost = 1 << 25;                 // tokens of a launch, whose threads must stay below 2^32
  for (long long at = 0; at < n; at += kMost) {
    const int m = (int)std::min<long long>(n - at, kMost);
    const dim3 grid((m + kTok - 1) / kTok, (H + heads - 1) / heads);
    r.pos = pos + at * r.n_axes;
    if (dtype == 0)
      hipLaunchKernelGGL((rope_kernel<float>), grid, dim3(kThreads), 0, stream, static_cast<const float*>(x) + at * xt,
                         xt, xh, static_cast<float*>(out) + at * yt, yt, yh, m, H, heads, r, it);
    else
      hipLaunchKernelGGL((rope_kernel<uint16_t>), grid, dim3(kThreads), 0, stream,
                         static_cast<const uint16_t*>(x) + at * xt, xt, xh, static_cast<uint16_t*>(out) + at * yt, yt,
                         yh, m, H, heads, r, it);
  }
  return check_launch("rope");
}

cast_status_t launch_kv_append(const cast_kv_cache_t& c, const cast_kv_seqs_t& s, const void* k, long long ks,
                               const void* v, long long vs, const cast_rope_params_t* rope, const int32_t* pos,
                               const void* q, long long qs, int Hq, void* q_out, hipStream_t stream) {
  AppendArgs a{};
  a.s = make_seqs(s, c.page);
  a.r = make_rope(rope, pos, 0);
  a.it = plan_items(a.r.rot, a.r.inter, c.dh, true);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.q = static_cast<const uint16_t*>(q);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.kc = c.k;
  a.vc = c.v;
  a.ke = c.k_exp;
  a.ve = c.v_exp;
  a.ks = ks;
  a.vs = vs;
  a.qs = qs;
  a.H = c.H;
  a.Hq = q != nullptr ? Hq : 0;
  a.dh = c.dh;
  a.pages = c.pages;
  a.page = c.page;
  const int bx = (s.n_tok + kTok - 1) / kTok;
  if (c.dtype == 1) {
    const int all = 2 * c.H + a.Hq;
    a.heads = heads_per_block(bx, all, a.it.per_head);
    hipLaunchKernelGGL(append_kernel, dim3(bx, (all + a.heads - 1) / a.heads), dim3(kThreads), 0, stream, a);
  } else {
    if (a.Hq > 0) {
      a.heads = heads_per_block(bx, a.Hq, a.it.per_head);
      a.q_blocks_x = bx;
      a.q_shares = (a.Hq + a.heads - 1) / a.heads;
    }
    // every page counted holds a token, or is a sequence's first or last (see page_rows, part_rows)
    const long long pages = (long long)s.n_tok / c.page + 2ll * s.n_seq;
    // The rows of a part stay in a block's registers.  Where sequences bring many more
    // to longer pages, several blocks share a page and head, at the price of two more launches:
    // a frame of 1560 tokens and 12 heads that is a page 17 us, 98 with one block each; 4 x
    // 6240 tokens in such pages 89 and 133, in pages of 12480 94 and 412; 2 x 300 of 8 heads in
    // pages of 300 13.6 and 22; 64 x 200 in pages of 4096 48 and 45, where the two sides meet;
    // but 2 x 300 in pages of 100 13.5 and 11.
    // Two heads of K to a block where that leaves a thousand: 15000 tokens of 8 heads in
    // pages of 64 29 us and 25.5; but 8 x 512 tokens 10.8 and 11.4, 2 x 300 in pages of 100 11
    // and 13.
    const int part = kKeep * kThreads * 16 / c.dh;
    a.part_log2 = c.dh == 32 ? 8 : c.dh == 64 ? 7 : 6;
    a.page_parts = fast_div((c.page + part - 1) / part);
    const long long parts = (long long)s.n_tok / part + s.n_tok / c.page + 4ll * s.n_seq;
    const int mode = a.r.rot == 0 ? 0 : a.r.inter ? 2 : a.r.rot % 16 == 0 ? 1 : 3;
    const long long nq = (long long)a.q_blocks_x * a.q_shares, most = 1ll << 24;
    auto heads_of = [&](long long n) { return (mode == 1 || mode == 2) && c.H % 2 == 0 && n * c.H >= 1024 ? 2 : 1; };
    int nh = heads_of(parts);
    if (c.page > 4 * part && s.n_tok / s.n_seq > 2 * part && nq + parts * (c.H + c.H / nh) < most) {
      if (mode == 0) launch_append8_parts<0, 1>(a, pages, parts, stream);
      else if (mode == 1 && nh == 2) launch_append8_parts<1, 2>(a, pages, parts, stream);
      else if (mode == 1) launch_append8_parts<1, 1>(a, pages, parts, stream);
      else if (mode == 2 && nh == 2) launch_append8_parts<2, 2>(a, pages, parts, stream);
      else if (mode == 2) launch_append8_parts<2, 1>(a, pages, parts, stream);
      else launch_append8_parts<3, 1>(a, pages, parts, stream);
      return check_launch("kv_append");
    }
    nh = heads_of(pages);
    const long long blocks = nq + pages * (c.H + c.H / nh);
    if (blocks >= most) return fail(CAST_ERR_UNSUPPORTED, "kv_append: %lld workgroups are too many", blocks);
    const dim3 grid((unsigned)blocks);
    if (mode == 0) hipLaunchKernelGGL((append8_kernel<0, 1>), grid, dim3(kThreads), 0, stream, a);
    else if (mode == 1 && nh == 2) hipLaunchKernelGGL((append8_kernel<1, 2>), grid, dim3(kThreads), 0, stream, a);
    else if (mode == 1) hipLaunchKernelGGL((append8_kernel<1, 1>), grid, dim3(kThreads), 0, stream, a);
    else if (mode == 2 && nh == 2) hipLaunchKernelGGL((append8_kernel<2, 2>), grid, dim3(kThreads), 0, stream, a);
    else if (mode == 2) hipLaunchKernelGGL((append8_kernel<2, 1>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((append8_kernel<3, 1>), grid, dim3(kThreads), 0, stream, a);
  }
  return check_launch("kv_append");
}

cast_status_t launch_kv_read(const cast_kv_cache_t& c, const int32_t* idx, int m, void* ko, void* vo,
                             hipStream_t stream) {
  ReadArgs a{};
  a.k = c.k;
  a.v = c.v;
  a.ke = c.k_exp;
  a.ve = c.v_exp;
  a.idx = idx;
  a.ko = static_cast<uint16_t*>(ko);
  a.vo = static_cast<uint16_t*>(vo);
  a.pages = c.pages;
  a.H = c.H;
  a.cph_log2 = c.dh == 32 ? 2 : c.dh == 64 ? 3 : 4;
  a.heads = fast_div(c.H);
  a.chunks = (long long)c.page * c.H << a.cph_log2;
  const unsigned parts = (unsigned)std::min<long long>((a.chunks + 4 * kThreads - 1) / (4 * kThreads), 65535);
  const unsigned z = ko != nullptr && vo != nullptr ? 2 : 1;
  // pages beyond the grid's limit of rows go in further launches
  for (long long at = 0; at < m; at += 65535) {
    ReadArgs b = a;
    b.idx = idx + at;
    if (ko != nullptr) b.ko = a.ko + at * a.chunks * 8;
    if (vo != nullptr) b.vo = a.vo + at * a.chunks * 8;
    const dim3 grid(parts, (unsigned)std::min(m - at, 65535ll), z);
    if (c.dtype == 2) hipLaunchKernelGGL((read_kernel<true>), grid, dim3(kThreads), 0, stream, b);
    else hipLaunchKernelGGL((read_kernel<false>), grid, dim3(kThreads), 0, stream, b);
  }
  return check_launch("kv_read");
}

}  // namespace cast
