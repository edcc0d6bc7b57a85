// Attention over a paged cache, bf16 or e4m3: ragged sequences, grouped heads, causal or
// not, a window of the past with the first tokens kept visible.
//
// One pass over the keys with the running maximum and sum of the softmax.  The rows of a
// KV head are its query heads' rows of consecutive tokens (row = token * g + head in the
// group), so grouped heads fill the matrix tiles and read each key once.  Per wave: 32
// rows, and of a key tile
//   S^T = K Q^T       A = 32 keys, B = Q^T held in registers; one row per lane column, so
//                     maximum and sum need the lane's own values and one half-wave swap
//   O^T += V^T P^T    B = P^T straight from the S^T accumulators as bf16, A = V^T from a
//                     row-major LDS tile through the transposing read
// e4m3 codes become bf16 on the way (exactly: their scales are powers of two), so both
// cache types share everything after the load.
//
// Three kernels, chosen by the rows of a sequence (kv_attn_plan):
//   rows   16 rows per workgroup (decoding; of bf16 up to 8 where keys are cut).  Its waves
//          take neighbouring heads and walk key tiles by themselves, keys straight from
//          memory into MFMA operands, values through a private LDS tile; no barrier until the
//          results are joined.  Bound by HBM: 16 streams of up to 8192 bf16 keys (288 MB) 54
//          us, 4 of up to 131072 e4m3 keys (819 MB) 154 us, 5.3 TB/s; their joins 7 and 10 us.
//   tiles  128 rows per workgroup; its four waves share 64-key tiles in LDS, copied one tile
//          ahead.  Bound by the softmax's VALU work: chunks of 64-wide heads 144 us, 700
//          TFLOP/s (VALU 57% of the cycles, matrix cores 30%).
//   pairs  256 rows of 128 channels per workgroup, its waves in two groups that take turns on
//          the matrix cores and the VALU.  28160 keys by 4 x 3520 rows of 24 heads 1090
//          TFLOP/s; 13000 causal rows of prompts up to 4096 long, 28 key tiles a workgroup,
//          361 to 379 us, 790 to 830 TFLOP/s (matrix cores 38%: start and end of a workgroup
//          lie bare).
// Long key ranges with few row tiles are cut into pieces by the lengths the device sees (16
// streams of 400 to 8192 keys, 64 rows of each: 116 us cut by the bound on the lengths, 94
// so); a further kernel joins them.
#include <algorithm>
#include <utility>

#include "kv_device.h"

namespace cast {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void glb_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kThreads = 256;
constexpr int kTileRows = 128;   // rows per workgroup of the tiles kernel
constexpr int kTileKeys = 64;
constexpr int kMinWaveKeys = 128;    // keys that a wave of the rows kernel walks at least, before a range is cut
constexpr int kFewRows = 16;     // rows per workgroup of the rows kernel
// keys per tile and wave of the rows kernel: 16 KB of K and V at 128 channels, as much in
// flight for codes, and 16 KB of both for 64 channels of bf16
constexpr int row_keys(int dh, bool f8) { return dh == 128 && !f8 ? 32 : 64; }
// its workgroups per compute unit (waves per SIMD)
constexpr int row_groups(int dh) { return dh < 128 ? 3 : 2; }
constexpr int kMaxPieces = 128;
constexpr int kJoinWays = 8;   // threads that share the pieces of a row, from as many pieces on (at like lengths)
// s_waitcnt vmcnt(0) that leaves expcnt and lgkmcnt free
constexpr int kVmcnt0 = 0x0F70;
// The running maximum moves only when a tile exceeds it by more than this, in log2 units
// (see softmax).  With 2^8, keys whose logits spread by 6 moved some wave's maximum in nearly
// every tile (chunks of 64-wide heads 177 us, so 144; the frame over an 8-bit window 167 and 145).
constexpr float kMaxSlack = 16.0f;
constexpr float kJoinScale = 0x1p-14f;  // of a piece in a sum of up to 2^14 of them
// "no key seen yet": below every finite scaled score, so the first visible key moves it
constexpr float kNoMax = -3.0e38f;
constexpr float kLn2 = 0.69314718055994531f;

struct KvAttnArgs {
  const uint16_t* q;
  long long qs;
  const uint8_t* k;
  const uint8_t* v;
  const uint8_t* ke;
  const uint8_t* ve;
  KvSeqs s;
  uint16_t* out;
  float* lse;
  float* part_o;                 // normalised: [slabs][n_tok * Hq][dh], or [items][wh][rows][dh]
  float* part_lse;               // log2 domain: [slabs][n_tok * Hq], or [items][wh][rows]
  int Hq, H, g, pages, page;
  int causal, window, sinks;     // window 0: none
  int slabs, least;              // tiles kernels: pieces of a row tile at most, key tiles of a piece at least
  int target, max_items;         // pieces wanted (0: none is cut); rows kernel: work items at most
  int wh, hgroups;               // rows kernel: heads of a workgroup (1, 2 or 4), H / wh
  int2* meta;                    // rows kernel: first item and pieces of [row tile][head group]
  int* cuts;                     // tiles kernels: pieces of [n_tok * Hq]
  float sl2;                     // scale * log2(e)
};

template <int V>
struct IC {
  static constexpr int value = V;
};
template <int B, int E, class F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (B < E) {
    f(IC<B>{});
    static_for<B + 1, E>(f);
  }
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// LDS images: chunk c (16 bytes) of tile row r is stored at chunk c ^ swz(r), CPR chunks
// per row.  K: ds_read_b128 of one chunk by 32 consecutive rows; V: the transposing read's
// 4 rows x 32 bytes per 16 lanes; both conflict-free.
__device__ __forceinline__ constexpr int kswz(int r, int cpr) { return (r / (16 / cpr)) & (cpr - 1); }
__device__ __forceinline__ constexpr int vswz(int r, int cpr) { return ((2 * (r & 3)) ^ (8 * (r & 1))) & (cpr - 1); }

__device__ __forceinline__ u32x4 widen8(uint32_t a, uint32_t b, float sc) {
  return u32x4{widen2<false>(a, sc), widen2<true>(a, sc), widen2<false>(b, sc), widen2<true>(b, sc)};
}

// ---- the row tile of a workgroup and the key tiles it meets ----------------------------
struct RowTile {
  int b, beg, n_rows, row0;      // sequence, its first call row, its rows (tokens * g), first row here
  int len, off;                  // its length; position of its first token of the call
  int ts, tw, dir, nt;           // logical key tile u: u < ts ? u : tw + dir (u - ts); nt in all
};
// the key tiles that rows at positions p_lo .. p_hi of a sequence of `len` meet
template <int TK>
__device__ __forceinline__ void key_tiles(const KvAttnArgs& a, RowTile& t, int p_lo, int p_hi, int len) {
  const int hi = max(a.causal ? min(p_hi + 1, len) : len, 0);
  const int lo = a.window > 0 ? min(max(p_lo - a.window + 1, 0), hi) : 0;
  const int sk = a.window > 0 ? min(a.sinks, hi) : 0;
  const int te = (hi + TK - 1) / TK;
  t.ts = (sk + TK - 1) / TK;
  const int first = max(lo / TK, t.ts);
  t.nt = t.ts + max(te - first, 0);
  // Row tiles that run at the same time should be at the same keys.  Windows of rows that are
  // not causal differ in where they begin and end together, so they are walked from the end
  // (a 30x52 frame, window 7800, 12 heads of 128: 110 us; 153 from the beginning, where the
  // row tiles read up to 24 key tiles apart, past the L2).
  const bool back = a.window > 0 && !a.causal;
  t.tw = back ? te - 1 : first;
  t.dir = back ? -1 : 1;
}
// Row tiles of the call: those of sequence b are numbered from floor(cu[b] g / TM) + b,
// which leaves room for its partial tile.
template <int TM>
__device__ __forceinline__ int first_tile(const KvAttnArgs& a, int b) {
  return (int)((unsigned)(seq_row(a.s, b) * a.g) / (unsigned)TM) + b;
}
// row tile k of sequence b, which has call rows beg .. beg + n and is len long
template <int TM, int TK>
__device__ __forceinline__ bool place(const KvAttnArgs& a, int b, int beg, int n, int len, int k, RowTile& t) {
  t.b = b;
  t.beg = beg;
  t.n_rows = n * a.g;
  if (k < 0 || (long long)k * TM >= t.n_rows) return false;
  t.row0 = k * TM;
  t.len = len;
  t.off = t.len - n;
  key_tiles<TK>(a, t, t.off + t.row0 / a.g, t.off + (min(t.row0 + TM, t.n_rows) - 1) / a.g, t.len);
  return true;
}
template <int TM, int TK>
__device__ __forceinline__ bool place(const KvAttnArgs& a, int b, int k, RowTile& t) {
  const int beg = seq_row(a.s, b);
  return place<TM, TK>(a, b, beg, max(seq_row(a.s, b + 1) - beg, 0), seq_len(a.s, b), k, t);
}
// x-th row tile of the call
template <int TM, int TK>
__device__ __forceinline__ bool row_tile(const KvAttnArgs& a, int x, RowTile& t) {
  const int b = find_seq(a.s.n_seq, x, [&](int i) { return first_tile<TM>(a, i); });
  return place<TM, TK>(a, b, x - first_tile<TM>(a, b), t);
}
// Sums over a wave by row shifts and broadcasts in the registers (shuffles go through the LDS
// and take ten times as long): inclusive prefix sums of the lanes.
template <int CTRL, int ROWS, class T>
__device__ __forceinline__ T dpp_add(T v) {
  return v + __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
template <class T>
__device__ __forceinline__ T prefix_sum(T v) {
  v = dpp_add<0x111, 0xf>(v);                  // row_shr 1, 2, 4, 8: rows of 16 lanes
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  v = dpp_add<0x142, 0xa>(v);                  // lane 15 of rows 0 and 2 into rows 1 and 3
  return dpp_add<0x143, 0xc>(v);               // lane 31 into rows 2 and 3
}
__device__ __forceinline__ int lane_value(int v, int l) { return __builtin_amdgcn_readlane(v, l); }

// A sequence of the call: its rows and length, its row tiles and the key tiles they meet.
struct SeqWork {
  int beg, n, len, rt, nt;
};
template <int TM, int TK>
__device__ __forceinline__ SeqWork seq_work(const KvAttnArgs& a, int b) {
  SeqWork w{0, 0, 0, 0, 0};
  if (b >= a.s.n_seq) return w;
  w.beg = seq_row(a.s, b);
  w.n = max(seq_row(a.s, b + 1) - w.beg, 0);
  w.len = seq_len(a.s, b);
  if (w.n == 0) return w;
  w.rt = (w.n * a.g + TM - 1) / TM;
  if (a.target == 0) return w;                       // (nt is for those who cut)
  RowTile t;
  key_tiles<TK>(a, t, w.len - w.n, w.len - 1, w.len);
  w.nt = t.nt;
  return w;
}
// The key tiles of a piece with which the call, `groups` times over, makes about a.target of
// them, at most target + groups row tiles.  FIT (the tiles kernels, where a piece more than the
// card holds costs a whole round): the first of this mean and three larger sizes that makes at
// most a.target, else the largest.  `w` is the lane's first sequence.
template <int TM, int TK, bool FIT>
__device__ __forceinline__ int piece_tiles(const KvAttnArgs& a, const SeqWork& w, int groups, int least) {
  const int lane = threadIdx.x & 63;
  float sum = 0.0f;
  for (int c = 0; c < a.s.n_seq; c += 64) {
    const SeqWork v = c == 0 ? w : seq_work<TM, TK>(a, c + lane);
    sum += (float)v.rt * (float)v.nt;
  }
  sum = __int_as_float(lane_value(__float_as_int(prefix_sum(sum)), 63));
  const int mean = max(least, (int)fminf(ceilf(sum * (float)groups * (FIT ? 0.9999f : 1.0001f) / (float)a.target), 1.0e7f));
  if constexpr (!FIT) return mean;
  int per[4], n[4];
  float inv[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    per[i] = mean + ((mean * i * (i + 3) + 31) >> 5);   // 1, 1.125, 1.31, 1.56 times
    inv[i] = __builtin_amdgcn_rcpf((float)per[i]);
    n[i] = 0;
  }
  for (int c = 0; c < a.s.n_seq; c += 64) {
    const SeqWork v = c == 0 ? w : seq_work<TM, TK>(a, c + lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) n[i] += v.rt * max(1, (int)ceilf((float)v.nt * inv[i] - 1e-3f));   // (near enough to choose by)
  }
  int best = per[3];
#pragma unroll
  for (int i = 2; i >= 0; --i) best = (long long)lane_value(prefix_sum(n[i]), 63) * groups <= a.target ? per[i] : best;
  return best;
}

// The work of a workgroup of the tiles kernels: row tile, head, and the logical key tiles
// [u0, u1), which are piece z of `pieces`.  The grid has room for every way to share the rows
// out among the sequences; what is there is counted, so that the workgroups with nothing to
// do are the last ones of the grid.  (With a spare row tile numbered after each sequence's,
// 512 rows over 16384 keys of 8 heads took 81 us and 511 rows, which need no spare one, 58:
// while the idle ones start and leave, others pile up on the compute units that are free.)
// Workgroup b runs on XCD b mod 8.  Each XCD takes a run of the (head, sequence, piece, row
// tile) list, so the row tiles that read the same keys share its L2, and walks it from the
// end: of causal rows the last tiles are the longest, and the shortest should finish the call.
// (With heads over all XCDs and short tiles first: prompts 463 us for 425, chunks of 64-wide
// heads 232 for 195.)
struct Unit {
  RowTile t;
  int h, z, pieces, u0, u1;
};
template <int TM, int TK>
__device__ __forceinline__ bool my_unit(const KvAttnArgs& a, Unit& un) {
  const int lane = threadIdx.x & 63;
  SeqWork w = seq_work<TM, TK>(a, lane);
  int per = 0x3fffffff;
  if (a.target > 0) per = piece_tiles<TM, TK, true>(a, w, a.H, a.least);
  // (slabs: a sequence much longer than the others is cut no finer than they allow)
  auto pieces_of = [&](const SeqWork& v) __attribute__((always_inline)) -> int {
    return a.target > 0 ? min(max(1, (v.nt + per - 1) / per), a.slabs) : 1;
  };
  int total = 0;
  for (int c = 0; c < a.s.n_seq; c += 64) {
    const SeqWork v = c == 0 ? w : seq_work<TM, TK>(a, c + lane);
    total += lane_value(prefix_sum(v.rt * pieces_of(v)), 63);
  }
  const int grid = gridDim.x;
  total = min(max(total, 0), grid / a.H);            // (the bound, whatever the offsets hold)
  const int n = total * a.H, b = blockIdx.x, x = b & 7, j = b >> 3, share = n >> 3, rest = n & 7;
  const int mine = share + (x < rest ? 1 : 0);
  if (j >= mine) return false;
  const int unit = x * share + min(x, rest) + mine - 1 - j;
  un.h = unit / total;
  const int at = unit - un.h * total;
  int base = 0;
  for (int c = 0; c < a.s.n_seq; c += 64) {
    if (c > 0) w = seq_work<TM, TK>(a, c + lane);
    const int pieces = pieces_of(w), there = w.rt * pieces, incl = prefix_sum(there);
    const unsigned long long hit = __ballot(at - base < incl);
    if (hit != 0) {
      const int l = __ffsll((long long)hit) - 1;
      const int rt = lane_value(w.rt, l), local = at - base - lane_value(incl - there, l);
      un.pieces = lane_value(pieces, l);
      un.z = local / max(rt, 1);
      if (local < 0 || un.z >= un.pieces) return false;   // (sums that wrapped: offsets that hold garbage)
      if (!place<TM, TK>(a, c + l, lane_value(w.beg, l), lane_value(w.n, l), lane_value(w.len, l), local - un.z * rt, un.t))
        return false;
      const int size = a.target > 0 ? (lane_value(w.nt, l) + un.pieces - 1) / un.pieces : un.t.nt;
      un.u0 = (int)min((long long)un.z * size, (long long)un.t.nt);
      un.u1 = min(un.u0 + min(size, un.t.nt), un.t.nt);
      return true;
    }
    base += lane_value(incl, 63);
  }
  return false;
}

// A lane's row, and which keys it sees: j < hi, and j >= lo or j < sinks.
struct RowLimits {
  int hi, lo;
};
__device__ __forceinline__ RowLimits row_limits(const KvAttnArgs& a, const RowTile& t, int p) {
  return RowLimits{a.causal ? min(p + 1, t.len) : t.len, a.window > 0 ? p - a.window + 1 : 0};
}

// Whether a key tile [j0, j0 + TK) is seen by none (0), some (1) or all (2) of the rows at
// positions p0 .. p1; `there`: BITS bits, set where the keys exist.  Sign bits instead of
// comparisons: branches would cut up the products beside which this is worked out.
struct KindBounds {
  int c0, c1;                    // the last key that row p0, row p1 sees
  int w0, w1;                    // the last key before their windows
  int sinks;
};
__device__ __forceinline__ KindBounds kind_bounds(const KvAttnArgs& a, int len, int p0, int p1) {
  const int far = 1 << 30;       // (positions, lengths and windows are at most that)
  return KindBounds{a.causal ? min(p0, len - 1) : len - 1, a.causal ? min(p1, len - 1) : len - 1, a.window > 0 ? max(p0 - a.window, -1) : -1,
                    a.window > 0 ? max(p1 - a.window, -1) : -1, min(a.sinks, far)};
}
__device__ __forceinline__ int less(int x, int y) { return (int)((unsigned)(x - y) >> 31); }   // 1 where x < y
template <int TK, int BITS = TK>
__device__ __forceinline__ int tile_kind(const KindBounds& k, int j0, unsigned long long there) {
  const int last = j0 + TK - 1, n = (int)__popcll(there);
  const int none = less(n, 1) | less(k.c1, j0) | (less(last, k.w0 + 1) & less(k.sinks, j0 + 1));
  const int full = less(BITS - 1, n) & less(last, k.c0 + 1) & (less(k.w1, j0) | less(last, k.sinks));
  return (1 + full) & (none - 1);
}

// a byte of ones for each of eight bits
__device__ __forceinline__ unsigned long long bytes_of(unsigned long long bits) {
  const unsigned long long x = (bits * 0x0101010101010101ull) & 0x8040201008040201ull;
  return (((x + 0x7f7f7f7f7f7f7f7full) >> 7) & 0x0101010101010101ull) * 0xff;
}

// The lane's visible keys among j0 .. j0 + 31 as bits (of those in `there`).
__device__ __forceinline__ uint32_t below(int n) {   // bits 0 .. n - 1
  return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u;
}
__device__ __forceinline__ uint32_t visible_bits(RowLimits r, int sinks, int j0, uint32_t there) {
  return there & below(r.hi - j0) & (~below(r.lo - j0) | below(sinks - j0));
}
// S^T accumulator element e of block kb belongs to key kb * 32 + 8 (e / 4) + 4 hf + e % 4.
template <int NB>
__device__ __forceinline__ void mask_scores(f32x16 (&sn)[NB], int j0, int hf, RowLimits r, int sinks,
                                            unsigned long long there) {
#pragma unroll
  for (int kb = 0; kb < NB; ++kb) {
    const uint32_t bits = visible_bits(r, sinks, j0 + 32 * kb, (uint32_t)(there >> (32 * kb))) >> (4 * hf);
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (((bits >> (8 * (e / 4) + e % 4)) & 1) == 0) sn[kb][e] = -INFINITY;
  }
}

// The running maximum is kept `lead` above the scores', in log2 units, so exponentials start at
// 2^-lead and reach 2^(kMaxSlack - lead), which is 2^-bits for a sequence of less than 2^bits keys:
// those of a row sum to less than one, and their products with the values to less than the largest
// value, which may be the type's.  (With the maximum at the scores' own, finite values above 2^111
// could give infinite rows.)  What falls below 2^-126 is lost, as ever: 2^-80 of the largest
// exponential at most, and products below 2^-80 in size (of 2^30 keys; 2^-98 of 4096).  The
// exponent's argument is off by 2^-20 for up to 2^15 keys, by 2^-19 for more.
struct Lead {
  float lead, bound, scale;      // bound 2^(kMaxSlack - lead), scale 2^lead
};
__device__ __forceinline__ Lead lead_of(int len) {
  const int bits = 32 - __clz(len);
  return Lead{kMaxSlack + (float)bits, __uint_as_float((uint32_t)(127 - bits) << 23),
              __uint_as_float((uint32_t)(127 + (int)kMaxSlack + bits) << 23)};
}

// Exponentials of a tile against the running maximum, in place of the scores (a second set
// would cost the registers of two waves per SIMD at 64-wide heads), packed as P^T operands,
// and their sum.  A lane's sum of at most the bound shows that no score is far above the maximum,
// which then may stay; else the scores are formed again, the maximum is taken over the tile, moved, and the sums
// so far scaled down.
template <int NB, int ND, class S>
__device__ __forceinline__ void softmax(f32x16 (&sn)[NB], S&& scores, bf16x8 (&pp)[NB][2], float& m_run, float& l_run,
                                        f32x16 (&acc)[ND], float sl2, const Lead& ld) {
  auto exps = [&]() __attribute__((always_inline)) -> float {
    float rs[4];
#pragma unroll
    for (int e = 0; e < NB * 16; ++e) {
      const float p = __builtin_amdgcn_exp2f(fmaf(sn[e / 16][e % 16], sl2, -m_run));
      sn[e / 16][e % 16] = p;
      rs[e % 4] = e < 4 ? p : rs[e % 4] + p;
    }
    return (rs[0] + rs[1]) + (rs[2] + rs[3]);
  };
  float sum = exps();
  if (__ballot(!(sum <= ld.bound)) != 0ull) {
    scores();
    float pm = sn[0][0];
#pragma unroll
    for (int e = 1; e < NB * 16; ++e) pm = fmaxf(pm, sn[e / 16][e % 16]);
    const float cand = fmaxf(m_run, fmaf(half_swap_max(pm), sl2, ld.lead));
    const bool up = cand > m_run + kMaxSlack;
    const float m_new = up ? cand : m_run;
    const float corr = __builtin_amdgcn_exp2f(m_run - m_new);
    l_run *= corr;
    m_run = m_new;
    if (__ballot(up) != 0ull) {
#pragma unroll
      for (int db = 0; db < ND; ++db) acc[db] *= corr;
    }
    sum = exps();
  }
#pragma unroll
  for (int g = 0; g < 2 * NB; ++g) {
    const f32x16& p = sn[g / 2];
    const int b = 8 * (g % 2);
    pp[g / 2][g % 2] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(p[b], p[b + 1]), pack_bf16x2(p[b + 2], p[b + 3]),
                                                        pack_bf16x2(p[b + 4], p[b + 5]), pack_bf16x2(p[b + 6], p[b + 7])});
  }
  l_run += sum;
}

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// O^T += V^T P^T of a tile that every row sees.  read(db, kb, s2): the A operand of channels
// 32 db .. and keys 32 kb + 16 s2 ..
template <int NB, int ND, class R>
__device__ __forceinline__ void values(R&& read, const bf16x8 (&pp)[NB][2], f32x16 (&acc)[ND]) {
  constexpr int N = 2 * NB * ND, AHEAD = N < 3 ? N : 3;
  bf16x8 op[N];
  auto rd = [&](auto uu) __attribute__((always_inline)) {
    constexpr int u = decltype(uu)::value;
    op[u] = read(u % ND, u / (2 * ND), (u / ND) % 2);
  };
  static_for<0, AHEAD>([&](auto u) { rd(u); });
  static_for<0, N>([&](auto uu) {
    constexpr int u = decltype(uu)::value;
    if constexpr (u + AHEAD < N) rd(IC<u + AHEAD>{});
    acc[u % ND] = mfma(op[u], pp[u / (2 * ND)][(u / ND) % 2], acc[u % ND]);
    __builtin_amdgcn_sched_barrier(0);
  });
}

// Infinities and NaN at places that a row does not see must add nothing to it, but there
// P = 0 and 0 * inf is NaN.  So a tile that some row sees only in part is looked through for
// them (exponent bits all set), and if it holds any its product is formed in three: the
// finite values, and 0/1 images of where +inf (or NaN) and -inf (or NaN) lie under 0/1
// weights; a row that meets only +inf gets that, only -inf that, both or a NaN a NaN.
__device__ __forceinline__ uint32_t special_bits(uint32_t w) { return (w & 0x7f807f80u) + 0x00800080u; }   // bits 15, 31
__device__ __forceinline__ uint32_t special_bits(bf16x8 op) {
  const u32x4 w = __builtin_bit_cast(u32x4, op);
  return (special_bits(w.x) | special_bits(w.y)) | (special_bits(w.z) | special_bits(w.w));
}
enum Part { kFinite, kPlus, kMinus };
template <Part P>
__device__ __forceinline__ bf16x8 part_of(bf16x8 op) {
  u32x4 w = __builtin_bit_cast(u32x4, op);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = special_bits(w[i]) & 0x80008000u;
    const uint32_t nan = m & (((w[i] & 0x007f007fu) + 0x007f007fu) << 8), sign = w[i] & 0x80008000u;
    if (P == kFinite) w[i] &= ~((m >> 15) * 0xffffu);
    else w[i] = ((m & ((P == kPlus ? ~sign : sign) | nan)) >> 15) * 0x3f80u;
  }
  return __builtin_bit_cast(bf16x8, w);
}
// 1 where a weight is not zero
__device__ __forceinline__ bf16x8 seen_weights(bf16x8 p8) {
  u32x4 p = __builtin_bit_cast(u32x4, p8);
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = ((((p[i] & 0x7fff7fffu) + 0x7fff7fffu) & 0x80008000u) >> 15) * 0x3f80u;
  return __builtin_bit_cast(bf16x8, p);
}
// Adds infinity times the sign where the count is above 0: the count times 3e38 twice (not
// fused with the sum, which would take the product without its overflow).
template <int N, class V>
__device__ __forceinline__ void add_infinity(V& acc, V count, float sign) {
#pragma clang fp contract(off)
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float c = count[e] * 3.0e38f;
    acc[e] += c * (3.0e38f * sign);
  }
}
// A step of the special products is done before the next begins: they are rare and should
// not cost the loop around them registers.
#define PIN(x) asm volatile("" : "+v"(x))
template <int NB, int ND, class R>
__device__ __forceinline__ bool has_special(R&& read) {
  uint32_t m = 0;
#pragma unroll
  for (int g = 0; g < 2 * NB; ++g)
#pragma unroll
    for (int db = 0; db < ND; ++db) {
      m |= special_bits(read(db, g / 2, g % 2));
      PIN(m);
    }
  return __ballot((m & 0x80008000u) != 0) != 0ull;
}
template <int NB, int ND, class R>
__device__ __forceinline__ void values_special(R&& read, const bf16x8 (&pp)[NB][2], f32x16 (&acc)[ND]) {
#pragma unroll
  for (int db = 0; db < ND; ++db) {
#pragma unroll
    for (int g = 0; g < 2 * NB; ++g) {
      acc[db] = mfma(part_of<kFinite>(read(db, g / 2, g % 2)), pp[g / 2][g % 2], acc[db]);
      PIN(acc[db]);
    }
    f32x16 count{};
#pragma unroll
    for (int g = 0; g < 2 * NB; ++g) {
      count = mfma(part_of<kPlus>(read(db, g / 2, g % 2)), seen_weights(pp[g / 2][g % 2]), count);
      PIN(count);
    }
    add_infinity<16>(acc[db], count, 1.0f);
    PIN(acc[db]);
    count = f32x16{};
#pragma unroll
    for (int g = 0; g < 2 * NB; ++g) {
      count = mfma(part_of<kMinus>(read(db, g / 2, g % 2)), seen_weights(pp[g / 2][g % 2]), count);
      PIN(count);
    }
    add_infinity<16>(acc[db], count, -1.0f);
    PIN(acc[db]);
  }
}

// A row's place in the call and its result: 16-byte-aligned groups of four channels.
__device__ __forceinline__ void put4(const KvAttnArgs& a, long long row, int dh, int d, f32x4 o) {
  *reinterpret_cast<u32x2*>(a.out + row * dh + d) = u32x2{pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w)};
}

// A lane's row of a tiles kernel: normalised into the output, or as piece z of it.
template <int DH, int ND>
__device__ __forceinline__ void finish(const KvAttnArgs& a, const Unit& un, long long row, int hf, bool any, float m_run,
                                       float l_run, const f32x16 (&acc)[ND]) {
  const float l = l_run + __shfl_xor(l_run, 32);
  const bool some = l != 0.0f;               // true for NaN, too
  const float inv = some ? 1.0f / l : 0.0f;
  const Lead ld = lead_of(un.t.len);
  const float l2 = some ? (m_run - ld.lead) + __log2f(l * ld.scale) : -INFINITY;
  const long long at = (long long)un.z * a.s.n_tok * a.Hq + row;
  if (a.target > 0 && un.z == 0 && hf == 0) a.cuts[row] = un.pieces;
  if (un.pieces > 1) {
    if (hf == 0) a.part_lse[at] = l2;
    if (!any) return;
  } else if (a.lse != nullptr && hf == 0) {
    a.lse[row] = l2 * kLn2;
  }
#pragma unroll
  for (int db = 0; db < ND; ++db)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) {
      const f32x4 o{acc[db][4 * g4] * inv, acc[db][4 * g4 + 1] * inv, acc[db][4 * g4 + 2] * inv, acc[db][4 * g4 + 3] * inv};
      const int d = db * 32 + 8 * g4 + 4 * hf;
      if (un.pieces > 1) *reinterpret_cast<f32x4*>(a.part_o + at * DH + d) = o;
      else put4(a, row, DH, d, o);
    }
}

// ---------------------------------------------------------------------------
// tiles
// ---------------------------------------------------------------------------
// RUNS (both tiles kernels): pages of a multiple of copy_rows(DH) tokens.  Then the rows of
// one copy instruction of a wave, which start at a multiple of it, lie side by side in one
// page, and their place is one number for the wave; else every lane fetches its row's place
// from the lane that looked it up.  (The LDS, which that goes through, is as busy as the matrix cores.)
constexpr int copy_rows(int dh) { return 1024 / dh; }
// Codes of a tile come in 16-byte loads, dh / 16 to a row: load i of a wave covers copy_rows(dh)
// rows from this one on.  A tile of 32-wide heads has a load for two of the four waves; the
// others have none (-1): their rows would lie behind the tile's, which nothing looked up.
constexpr int code_loads(int dh) { return (kTileKeys * dh / 16 + kThreads - 1) / kThreads; }
constexpr int code_rows(int dh, int wave, int i) {
  const int first = (wave + i * (kThreads / 64)) * copy_rows(dh);
  return code_loads(dh) * kThreads * 16 / dh > kTileKeys && first >= kTileKeys ? -1 : first;
}

template <int DH, bool F8, bool RUNS>
__global__ __launch_bounds__(kThreads, DH == 128 ? 2 : DH == 64 ? 3 : 4) void kv_tiles_kernel(KvAttnArgs a) {
  constexpr int CPR = DH / 8, ROWB = DH * 2, ND = DH / 32, TK = kTileKeys;
  constexpr int NSLOT = DH / 32;             // 1-KB copies of a bf16 tile per wave
  constexpr int RSTEP = 2048 / DH;           // tile rows between them
  constexpr int C8 = DH / 16;                // 16-byte chunks of a row of codes
  constexpr int N8 = code_loads(DH);
  // separate objects: the compiler sees that copies do not touch the buffer being read
  __shared__ __attribute__((aligned(1024))) uint16_t lds_k0[TK * DH];
  __shared__ __attribute__((aligned(1024))) uint16_t lds_k1[TK * DH];
  __shared__ __attribute__((aligned(1024))) uint16_t lds_v0[TK * DH];
  __shared__ __attribute__((aligned(1024))) uint16_t lds_v1[TK * DH];

  Unit un;
  if (!my_unit<kTileRows, TK>(a, un)) return;
  const RowTile& t = un.t;
  const int h = un.h, u0 = un.u0, u1 = un.u1;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hf = lane >> 5;

  // the lane's row; rows past the end repeat the last one and are not stored
  const int w0 = t.row0 + wave * 32;
  const bool live = w0 < t.n_rows;
  const int r = min(w0 + l32, t.n_rows - 1);
  const int tok = r / a.g, hq = h * a.g + (r - tok * a.g);
  const int p0 = t.off + min(w0, t.n_rows - 1) / a.g, p1 = t.off + min(w0 + 31, t.n_rows - 1) / a.g;
  const RowLimits lim = row_limits(a, t, t.off + tok);
  const KindBounds kb = kind_bounds(a, t.len, p0, p1);
  const Lead ld = lead_of(t.len);
  bf16x8 qreg[DH / 16];
  {
    const uint16_t* qp = a.q + (long long)(t.beg + tok) * a.qs + hq * DH + 8 * hf;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) qreg[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qp + 16 * i));
  }

  // ---- key lookup: lane l of every wave looks up key l of a tile
  const int32_t* table = a.s.table + (long long)t.b * a.s.max_pages;
  auto tile_of = [&](int u) { return u < t.ts ? u : t.tw + t.dir * (u - t.ts); };
  struct Look { int key, id, rem; };
  auto look = [&](int u) __attribute__((always_inline)) -> Look {
    Look k;
    k.key = tile_of(min(u, t.nt - 1)) * TK + lane;
    // (RUNS: a run past the end stands in for itself from the last key's run)
    const int kk = RUNS ? (k.key < t.len ? k.key : ((t.len - 1) & -copy_rows(DH)) + (k.key & (copy_rows(DH) - 1)))
                        : min(k.key, t.len - 1);
    const int pg = div_by(kk, a.s.page);
    k.id = table[pg];
    k.rem = kk - pg * a.page;
    return k;
  };
  // row of the cache of the lane's key (row 0 of page 0 where there is none), and which exist
  auto resolve = [&](const Look& k, unsigned long long& there) __attribute__((always_inline)) -> int {
    const bool in = k.id >= 0 && k.id < a.pages;
    there = __ballot(in && k.key < t.len);
    return in ? k.id * a.page + k.rem : 0;
  };
  const long long row_bytes = (long long)a.H * DH * (F8 ? 1 : 2), head_bytes = (long long)h * DH * (F8 ? 1 : 2);

  // ---- copies
  const int brow = wave * (512 / DH) + lane / CPR;
  const int kofs = ((lane % CPR) ^ kswz(brow, CPR)) * 16, vofs = ((lane % CPR) ^ vswz(brow, CPR)) * 16;
  auto copy_bf16 = [&](int slot, uint16_t* kd, uint16_t* vd) __attribute__((always_inline)) {
    static_for<0, NSLOT>([&](auto rr) {
      constexpr int i = decltype(rr)::value;
      const int lb = (wave + 4 * i) * 1024;
      const uint8_t *kp, *vp;
      if constexpr (RUNS) {
        const long long at = (long long)__builtin_amdgcn_readlane(slot, wave * (512 / DH) + i * RSTEP) * row_bytes + head_bytes;
        kp = a.k + at + (unsigned)(lane / CPR * (int)row_bytes + kofs);
        vp = a.v + at + (unsigned)(lane / CPR * (int)row_bytes + vofs);
      } else {
        const long long at = (long long)__shfl(slot, brow + i * RSTEP) * row_bytes + head_bytes;
        kp = a.k + at + kofs;
        vp = a.v + at + vofs;
      }
      __builtin_amdgcn_global_load_lds((glb_void*)kp, (lds_void*)(reinterpret_cast<char*>(kd) + lb), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((glb_void*)vp, (lds_void*)(reinterpret_cast<char*>(vd) + lb), 16, 0, 0);
    });
  };
  u32x4 ck[N8], cv[N8];
  int ex = 0;                                // exponent bytes of the lane's key: K | V << 8
  auto load8 = [&](int slot, int id) __attribute__((always_inline)) {
    const long long pe = (long long)(id >= 0 && id < a.pages ? id : 0) * a.H + h;
    ex = (int)a.ke[pe] | (int)a.ve[pe] << 8;
#pragma unroll
    for (int i = 0; i < N8; ++i) {
      const int c = tid + i * kThreads, first = code_rows(DH, wave, i);
      if (first < 0) continue;
      long long at = head_bytes;
      if constexpr (RUNS) {
        at += (long long)__builtin_amdgcn_readlane(slot, first) * row_bytes + (unsigned)(lane / C8 * (int)row_bytes + (lane % C8) * 16);
      } else {
        at += (long long)__shfl(slot, c / C8) * row_bytes + (c % C8) * 16;
      }
      ck[i] = *reinterpret_cast<const u32x4*>(a.k + at);
      cv[i] = *reinterpret_cast<const u32x4*>(a.v + at);
    }
  };
  auto store8 = [&](uint16_t* kd, uint16_t* vd) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N8; ++i) {
      const int c = tid + i * kThreads, row = c / C8, ch = 2 * (c % C8), first = code_rows(DH, wave, i);
      if (first < 0) continue;
      int e;
      if constexpr (RUNS) e = __builtin_amdgcn_readlane(ex, first);
      else e = __shfl(ex, row);
      const float sk = byte_scale(e & 255), sv = byte_scale(e >> 8);
      char* kr = reinterpret_cast<char*>(kd) + row * ROWB;
      char* vr = reinterpret_cast<char*>(vd) + row * ROWB;
      *reinterpret_cast<u32x4*>(kr + ((ch ^ kswz(row, CPR)) * 16)) = widen8(ck[i].x, ck[i].y, sk);
      *reinterpret_cast<u32x4*>(kr + (((ch + 1) ^ kswz(row, CPR)) * 16)) = widen8(ck[i].z, ck[i].w, sk);
      *reinterpret_cast<u32x4*>(vr + ((ch ^ vswz(row, CPR)) * 16)) = widen8(cv[i].x, cv[i].y, sv);
      *reinterpret_cast<u32x4*>(vr + (((ch + 1) ^ vswz(row, CPR)) * 16)) = widen8(cv[i].z, cv[i].w, sv);
    }
  };

  // ---- LDS reads (bytes within a tile); see kswz, vswz
  const unsigned kbase = (unsigned)(l32 * ROWB + ((hf ^ kswz(l32, CPR)) * 16));
  unsigned vbase;
  {
    const int gq = lane >> 4, la = lane & 15;
    const int vr = 4 * (gq >> 1) + (la >> 2);
    const int c = 2 * (gq & 1) + ((la & 3) >> 1);
    vbase = (unsigned)(vr * ROWB + ((c ^ vswz(vr, CPR)) * 16) + 8 * (la & 1));
  }
  // (the XORs are formed again at each use: opaque() keeps them out of registers across the loop)
  auto opaque = [](unsigned x) { asm volatile("" : "+v"(x)); return x; };
  auto read_k = [&](const uint16_t* kt, unsigned kb0, int i, int kb) __attribute__((always_inline)) -> bf16x8 {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(
        reinterpret_cast<const char*>(kt) + (kb0 ^ (32u * i)) + kb * 32 * ROWB));
  };
  auto read_v = [&](const uint16_t* vt, unsigned vb0, int db, int kb, int s2) __attribute__((always_inline)) -> bf16x8 {
    const lds_char* p = (const lds_char*)(vt) + (vb0 ^ (64u * db)) + (32 * kb + 16 * s2) * ROWB;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * ROWB)));
    return __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
  };

  f32x16 acc[ND];
#pragma unroll
  for (int db = 0; db < ND; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[db][e] = 0.0f;
  float m_run = kNoMax, l_run = 0.0f;

  unsigned long long there = 0, there_next = 0;
  Look nxt{};
  if (u0 < u1) {
    const Look first = look(u0);
    const int slot = resolve(first, there);
    if constexpr (F8) {
      load8(slot, first.id);
      store8(lds_k0, lds_v0);
    } else {
      copy_bf16(slot, lds_k0, lds_v0);
    }
    nxt = look(u0 + 1);
    __builtin_amdgcn_s_waitcnt(kVmcnt0);
  }
  __syncthreads();
  // one tile; buffers of parity P are read, the others filled with the next tile
  auto tile = [&](auto par, int u) __attribute__((always_inline)) {
    constexpr int P = decltype(par)::value;
    const uint16_t* kt = P == 0 ? lds_k0 : lds_k1;
    const uint16_t* vt = P == 0 ? lds_v0 : lds_v1;
    uint16_t* kn = P == 0 ? lds_k1 : lds_k0;
    uint16_t* vn = P == 0 ? lds_v1 : lds_v0;
    const bool more = u + 1 < u1;
    if (more) {
      const int slot = resolve(nxt, there_next);
      if constexpr (F8) load8(slot, nxt.id);
      else copy_bf16(slot, kn, vn);
      nxt = look(u + 2);
    }
    const int j0 = tile_of(u) * TK;
    const int kind = live ? tile_kind<TK>(kb, j0, there) : 0;
    if (kind != 0) {
      f32x16 sn[2];
      const unsigned vb0 = opaque(vbase);
      auto scores = [&]() __attribute__((always_inline)) {
        constexpr int N = 2 * (DH / 16), AHEAD = 3;
        const unsigned kb0 = opaque(kbase);
        bf16x8 op[N];
        static_for<0, AHEAD>([&](auto uu) { constexpr int i = decltype(uu)::value; op[i] = read_k(kt, kb0, i / 2, i % 2); });
        static_for<0, N>([&](auto uu) {
          constexpr int i = decltype(uu)::value, n = i + AHEAD;
          if constexpr (n < N) op[n] = read_k(kt, kb0, n / 2, n % 2);
          sn[i % 2] = mfma(op[i], qreg[i / 2], i < 2 ? f32x16{} : sn[i % 2]);
          __builtin_amdgcn_sched_barrier(0);
        });
        if (kind == 1) mask_scores<2>(sn, j0, hf, lim, a.sinks, there);
      };
      scores();
      bf16x8 pp[2][2];
      softmax<2, ND>(sn, scores, pp, m_run, l_run, acc, a.sl2, ld);
      auto rd = [&](int db, int kb, int s2) __attribute__((always_inline)) { return read_v(vt, vb0, db, kb, s2); };
      if (kind == 1 && has_special<2, ND>(rd)) values_special<2, ND>(rd, pp, acc);
      else values<2, ND>(rd, pp, acc);
    }
    if constexpr (F8) {
      if (more) store8(kn, vn);
    }
    there = there_next;
    __builtin_amdgcn_s_waitcnt(kVmcnt0);
    __syncthreads();
  };
#pragma unroll 1
  for (int u = u0; u < u1; u += 2) {
    tile(IC<0>{}, u);
    if (u + 1 >= u1) break;
    tile(IC<1>{}, u + 1);
  }

  if (w0 + l32 < t.n_rows)
    finish<DH>(a, un, (long long)(t.beg + tok) * a.Hq + hq, hf, u0 < u1, m_run, l_run, acc);
}

// ---------------------------------------------------------------------------
// pairs
// ---------------------------------------------------------------------------
// 128-wide heads, many rows: 256 rows and eight waves per workgroup, one per compute unit.
// Wave w runs on SIMD w mod 4, so every SIMD holds a wave of group A (0-3) and one of group
// B (4-7).  The groups take turns, a barrier between: while one forms S of tile j and O of
// tile j - 1 on the matrix core, the other does its softmax on the VALU.  B runs one
// interval behind: in interval 2 j A multiplies for tile j and B takes the softmax of
// j - 1, in 2 j + 1 A the softmax of j and B the products of j.  A fetches K[j + 1] at the
// start of interval 2 j + 1, B V[j + 1] at the start of 2 j + 2, each into the buffer that
// held tile j - 1, which no product of that interval reads.  (The tiles kernel leaves the
// overlap of two workgroups to chance: matrix cores 30% busy, VALU 39%.)
constexpr int kPairRows = 256, kPairThreads = 512;

template <bool F8, bool RUNS>
__global__ __launch_bounds__(kPairThreads, 2) void kv_pairs_kernel(KvAttnArgs a) {
  constexpr int DH = 128, CPR = DH / 8, ROWB = DH * 2, ND = DH / 32, TK = kTileKeys;
  constexpr int C8 = DH / 16;                // 16-byte chunks of a row of codes
  __shared__ __attribute__((aligned(1024))) uint16_t lds_k0[TK * DH];
  __shared__ __attribute__((aligned(1024))) uint16_t lds_k1[TK * DH];
  __shared__ __attribute__((aligned(1024))) uint16_t lds_v0[TK * DH];
  __shared__ __attribute__((aligned(1024))) uint16_t lds_v1[TK * DH];
  __shared__ __attribute__((aligned(1024))) uint16_t lds_zero[TK * DH];   // values of a tile that was not seen

  Unit un;
  if (!my_unit<kPairRows, TK>(a, un)) return;
  const RowTile& t = un.t;
  const int h = un.h, u0 = un.u0, u1 = un.u1;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave >> 2, l32 = lane & 31, hf = lane >> 5;

  const int w0 = t.row0 + wave * 32;
  const bool live = w0 < t.n_rows;
  const int r = min(w0 + l32, t.n_rows - 1);
  const int tok = r / a.g, hq = h * a.g + (r - tok * a.g);
  const int p0 = t.off + min(w0, t.n_rows - 1) / a.g, p1 = t.off + min(w0 + 31, t.n_rows - 1) / a.g;
  const RowLimits lim = row_limits(a, t, t.off + tok);
  const KindBounds kb = kind_bounds(a, t.len, p0, p1);
  const Lead ld = lead_of(t.len);
  bf16x8 qreg[DH / 16];
  {
    const uint16_t* qp = a.q + (long long)(t.beg + tok) * a.qs + hq * DH + 8 * hf;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) qreg[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qp + 16 * i));
  }

  // ---- key lookup, as in the tiles kernel
  const int32_t* table = a.s.table + (long long)t.b * a.s.max_pages;
  auto tile_of = [&](int u) { return u < t.ts ? u : t.tw + t.dir * (u - t.ts); };
  struct Look { int key, id, rem; };
  auto look = [&](int u) __attribute__((always_inline)) -> Look {
    Look k;
    k.key = tile_of(min(u, t.nt - 1)) * TK + lane;
    // (RUNS: a run past the end stands in for itself from the last key's run)
    const int kk = RUNS ? (k.key < t.len ? k.key : ((t.len - 1) & -copy_rows(DH)) + (k.key & (copy_rows(DH) - 1)))
                        : min(k.key, t.len - 1);
    const int pg = div_by(kk, a.s.page);
    k.id = table[pg];
    k.rem = kk - pg * a.page;
    return k;
  };
  const long long row_bytes = (long long)a.H * DH * (F8 ? 1 : 2), head_bytes = (long long)h * DH * (F8 ? 1 : 2);
  int slot = 0, exp_at = 0;                  // of the lane's key: row of the cache; of codes page * H + h
  auto resolve = [&](const Look& k, unsigned long long& there) __attribute__((always_inline)) {
    const bool in = k.id >= 0 && k.id < a.pages;
    there = __ballot(in && k.key < t.len);
    slot = in ? k.id * a.page + k.rem : 0;
    if (F8) exp_at = (in ? k.id : 0) * a.H + h;
  };

  // With RUNS one lookup serves eight tiles: lane l looks up the run of eight keys
  // l mod 8 of tile l / 8 of a window of them, and keeps its address.  (Looked up tile by
  // tile, a tile cost 55 more vector and 55 more scalar instructions than the products and
  // the softmax take, 4 x 3520 rows of 24 heads on
  // 28160 keys 4856 us, so and with the reads' offsets kept in registers 4468.)
  constexpr int GR = copy_rows(DH), GPT = TK / GR, TPW = 64 / GPT;
  static_assert(GPT == 8, "eight runs per tile: a byte of the window's mask");
  int win_id = 0, win_rem = 0;               // the next window's lookup
  unsigned run_lo = 0, run_hi = 0;           // this window's addresses
  unsigned long long runs = 0;               // which of its runs exist
  auto open_window = [&](int u) __attribute__((always_inline)) {
    const int key = tile_of(min(u + lane / GPT, t.nt - 1)) * TK + lane % GPT * GR;
    const int kk = key < t.len ? key : (t.len - 1) & -GR;
    const int pg = div_by(kk, a.s.page);
    win_id = table[pg];
    win_rem = kk - pg * a.page;
  };

  // ---- a group's four waves copy a tile: bf16 straight into LDS, codes through registers
  const int cw = wave & 3;
  const int brow = cw * 4 + lane / CPR;
  const int cofs = ((lane % CPR) ^ (grp == 0 ? kswz(brow, CPR) : vswz(brow, CPR))) * 16;
  const uint8_t* src = (grp == 0 ? a.k : a.v) + head_bytes;
  const uint8_t* exps = grp == 0 ? a.ke : a.ve;
  const int tg = tid & 255;
  int ex = 0;                                // codes: exponent byte of the lane's key or run
  auto enter_window = [&]() __attribute__((always_inline)) {
    const bool in = win_id >= 0 && win_id < a.pages;
    runs = __ballot(in);
    const uint8_t* at = src + (long long)(in ? win_id * a.page + win_rem : 0) * row_bytes;
    run_lo = (unsigned)(unsigned long long)at;
    run_hi = (unsigned)((unsigned long long)at >> 32);
    if (F8) ex = exps[(in ? win_id : 0) * a.H + h];
  };
  // run (in its tile) of a wave's copy i, and the lane's place from there
  auto run_of = [&](int i) { return F8 ? cw + 4 * i : 2 * i + (cw >> 1); };
  const unsigned lane_at = F8 ? (unsigned)(lane / C8 * (int)row_bytes + lane % C8 * 16)
                              : (unsigned)(((cw & 1) * 4 + lane / CPR) * (int)row_bytes + cofs);
  auto opaque = [](unsigned x) { asm volatile("" : "+v"(x)); return x; };
  auto place = [&](int i, int wt) __attribute__((always_inline)) -> const uint8_t* {   // wt: tile of the window
    if constexpr (RUNS) {
      const int l = wt * GPT + run_of(i);
      const unsigned long long at = (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)run_hi, l) << 32 |
                                    (unsigned)__builtin_amdgcn_readlane((int)run_lo, l);
      return reinterpret_cast<const uint8_t*>(at) + opaque(lane_at);   // (opaque: scalar base + lane offset)
    } else {
      const int c = tg + 256 * i;
      return src + (long long)__shfl(slot, F8 ? c / C8 : brow + 16 * i) * row_bytes + (F8 ? c % C8 * 16 : cofs);
    }
  };
  auto copy_bf16 = [&](uint16_t* dst, int wt) __attribute__((always_inline)) {
    static_for<0, 4>([&](auto rr) {
      constexpr int i = decltype(rr)::value;
      __builtin_amdgcn_global_load_lds((glb_void*)place(i, wt), (lds_void*)(reinterpret_cast<char*>(dst) + (cw + 4 * i) * 1024), 16, 0, 0);
    });
  };
  u32x4 code[2];
  auto load8 = [&](int wt) __attribute__((always_inline)) {
    if (!RUNS) ex = exps[exp_at];
#pragma unroll
    for (int i = 0; i < 2; ++i) code[i] = *reinterpret_cast<const u32x4*>(place(i, wt));
  };
  auto store8 = [&](uint16_t* dst, int wt) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = tg + 256 * i, row = c / C8, ch = 2 * (c % C8);
      int e;
      if constexpr (RUNS) e = __builtin_amdgcn_readlane(ex, wt * GPT + run_of(i));
      else e = __shfl(ex, row);
      const float sc = byte_scale(e);
      const int sw = grp == 0 ? kswz(row, CPR) : vswz(row, CPR);
      char* at = reinterpret_cast<char*>(dst) + row * ROWB;
      *reinterpret_cast<u32x4*>(at + ((ch ^ sw) * 16)) = widen8(code[i].x, code[i].y, sc);
      *reinterpret_cast<u32x4*>(at + (((ch + 1) ^ sw) * 16)) = widen8(code[i].z, code[i].w, sc);
    }
  };

  // ---- LDS reads (bytes within a tile); see kswz, vswz
  const unsigned kbase = (unsigned)(l32 * ROWB + ((hf ^ kswz(l32, CPR)) * 16));
  unsigned vbase;
  {
    const int gq = lane >> 4, la = lane & 15;
    const int vr = 4 * (gq >> 1) + (la >> 2);
    const int c = 2 * (gq & 1) + ((la & 3) >> 1);
    vbase = (unsigned)(vr * ROWB + ((c ^ vswz(vr, CPR)) * 16) + 8 * (la & 1));
  }
  auto read_k = [&](const uint16_t* kt, unsigned kb0, int i, int kb) __attribute__((always_inline)) -> bf16x8 {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(
        reinterpret_cast<const char*>(kt) + (kb0 ^ (32u * i)) + kb * 32 * ROWB));
  };
  auto read_v = [&](const uint16_t* vt, unsigned vb0, int db, int kb, int s2) __attribute__((always_inline)) -> bf16x8 {
    const lds_char* p = (const lds_char*)(vt) + (vb0 ^ (64u * db)) + (32 * kb + 16 * s2) * ROWB;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * ROWB)));
    return __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
  };

  f32x16 acc[ND];
#pragma unroll
  for (int db = 0; db < ND; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[db][e] = 0.0f;
  f32x16 sn[2];
  bf16x8 pp[2][2];
#pragma unroll
  for (int g = 0; g < 4; ++g) pp[g / 2][g % 2] = bf16x8{};
  float m_run = kNoMax, l_run = 0.0f;
  bool has_p = false;                        // pp holds a tile whose products are to come

  // ---- S of tile j and O of tile j - 1, one MFMA of each per step, operands read three
  //      steps ahead; step i: S chain i % 2, channels 16 (i / 2); O block i % 4, keys
  //      (kb, s2) = (i / 8, (i / 4) % 2).  also(i) is issued beside step i.
  auto products = [&](const uint16_t* kt, const uint16_t* vt, auto with_o, auto&& also) __attribute__((always_inline)) {
    constexpr bool O = decltype(with_o)::value != 0;
    constexpr int N = 16, AHEAD = 3;
    const unsigned kb0 = kbase, vb0 = vbase;
    bf16x8 opk[N], opv[N];
    auto rd = [&](auto uu) __attribute__((always_inline)) {
      constexpr int i = decltype(uu)::value;
      opk[i] = read_k(kt, kb0, i / 2, i % 2);
      if constexpr (O) opv[i] = read_v(vt, vb0, i % ND, i / (2 * ND), (i / ND) % 2);
    };
    static_for<0, AHEAD>([&](auto i) { rd(i); });
    static_for<0, N>([&](auto uu) {
      constexpr int i = decltype(uu)::value;
      if constexpr (i + AHEAD < N) rd(IC<i + AHEAD>{});
      sn[i % 2] = mfma(opk[i], qreg[i / 2], i < 2 ? f32x16{} : sn[i % 2]);
      if constexpr (O) acc[i % ND] = mfma(opv[i], pp[i / (2 * ND)][(i / ND) % 2], acc[i % ND]);
      also(uu);
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  const int n = u1 - u0;
  // keys of tile j that exist, and of the next ones: bits per key, with RUNS per run
  unsigned long long there = 0, there_next = 0, there_far = 0;
  Look nxt{};
  constexpr int D = F8 ? 2 : 1;              // tiles from the products' to the one being fetched
  // Codes go through registers, and are fetched a tile earlier than they are stored: the
  // fetch of tile j + 2 follows the store of j + 1 at the start of an interval and has until
  // the next such start.
  auto runs_of = [&](int wt) { return (runs >> (wt * GPT)) & 0xff; };
  if (n > 0) {
    for (int x = tid; x < TK * DH / 8; x += kPairThreads) reinterpret_cast<u32x4*>(lds_zero)[x] = u32x4{0u, 0u, 0u, 0u};
    if constexpr (RUNS) {
      open_window(u0);
      enter_window();
      open_window(u0 + TPW);
      there = runs_of(0);
    } else {
      resolve(look(u0), there);
    }
    if constexpr (F8) {
      load8(0);
      store8(grp == 0 ? lds_k0 : lds_v0, 0);
      if constexpr (RUNS) there_next = runs_of(1);
      else resolve(look(u0 + 1), there_next);
      load8(1);
    } else {
      copy_bf16(grp == 0 ? lds_k0 : lds_v0, 0);
    }
    if constexpr (!RUNS) nxt = look(u0 + D);
    if constexpr (!F8) __builtin_amdgcn_s_waitcnt(kVmcnt0);
    __syncthreads();
    if (grp == 1) __syncthreads();
    auto kind_of = [&](int j, unsigned long long th) __attribute__((always_inline)) {
      return -((int)live & less(j, n)) & tile_kind<TK, RUNS ? GPT : TK>(kb, tile_of(u0 + j) * TK, th);
    };
    int kind = kind_of(0, there), kind_next = 0;
    auto step = [&](auto par, int j) __attribute__((always_inline)) {
      constexpr int P = decltype(par)::value;
      const uint16_t* kc = P == 0 ? lds_k0 : lds_k1;     // K[j]
      const uint16_t* vc = P == 0 ? lds_v0 : lds_v1;     // V[j]
      uint16_t* kn = P == 0 ? lds_k1 : lds_k0;           // K[j - 1], then K[j + 1]
      uint16_t* vn = P == 0 ? lds_v1 : lds_v0;           // V[j - 1], then V[j + 1]
      const int j0 = tile_of(u0 + j) * TK;
      const int wt = (j + 1) % TPW, wd = (j + D) % TPW;  // tiles j + 1 and j + D in their windows
      // What tile j + 1 needs to know is worked out beside the products, where the wave waits
      // for the matrix core anyway.
      auto prepare = [&](auto uu) __attribute__((always_inline)) {
        constexpr int i = decltype(uu)::value;
        if constexpr (!RUNS && i == 1) resolve(nxt, F8 ? there_far : there_next);
        if constexpr (!RUNS && i == 5) nxt = look(u0 + j + D + 1);
        if constexpr (RUNS && !F8 && i == 5) there_next = runs_of(wt);
        if constexpr (i == 9) kind_next = kind_of(j + 1, there_next);
      };
      auto next_window = [&]() __attribute__((always_inline)) {
        if (RUNS && wd == 0) {                           // (no copy from the last one is to come)
          enter_window();
          open_window(u0 + j + D + TPW);
        }
      };
      if constexpr (!F8) next_window();
      // (one path for both products: with a path for each case the accumulators moved between
      // registers; a product that is not wanted meets zeros or is not looked at)
      if (kind != 0 || has_p) products(kc, has_p ? vn : lds_zero, IC<1>{}, prepare);
      else static_for<0, 16>(prepare);
      has_p = kind != 0;
      __syncthreads();
      if constexpr (F8) {
        if (j + 1 < n) store8(grp == 0 ? kn : vn, wt);
        if (j + 2 < n) {
          next_window();
          load8(wd);
        }
        if constexpr (RUNS) there_far = runs_of(wd);
      } else if (j + 1 < n) {
        copy_bf16(grp == 0 ? kn : vn, wt);
      }
      if (kind != 0) {
        auto mask = [&]() __attribute__((always_inline)) {
          if (kind == 1) mask_scores<2>(sn, j0, hf, lim, a.sinks, RUNS ? bytes_of(there) : there);
        };
        mask();
        PIN(sn[0]);
        PIN(sn[1]);
        softmax<2, ND>(sn, [&]() __attribute__((always_inline)) {
          products(kc, vc, IC<0>{}, [](auto) {});        // K[j] is still there
          mask();
        }, pp, m_run, l_run, acc, a.sl2, ld);
        if (kind == 1) {
          const unsigned vb0 = opaque(vbase);
          auto rd = [&](int db, int kb, int s2) __attribute__((always_inline)) { return read_v(vc, vb0, db, kb, s2); };
          if (has_special<2, ND>(rd)) {
            values_special<2, ND>(rd, pp, acc);
            has_p = false;
          }
        }
      }
      there = there_next;
      if constexpr (F8) there_next = there_far;
      kind = kind_next;
      // (the barrier's fence does not wait for copies into LDS; codes may still be on their way)
      if constexpr (!F8) __builtin_amdgcn_s_waitcnt(kVmcnt0);
      __syncthreads();
    };
#pragma unroll 1
    for (int j = 0; j <= n; j += 2) {
      step(IC<0>{}, j);
      if (j + 1 > n) break;
      step(IC<1>{}, j + 1);
    }
    if (grp == 0) __syncthreads();           // B's extra interval at the start
  }
  if (w0 + l32 < t.n_rows)
    finish<DH>(a, un, (long long)(t.beg + tok) * a.Hq + hq, hf, n > 0, m_run, l_run, acc);
}

// ---------------------------------------------------------------------------
// rows
// ---------------------------------------------------------------------------
// v_mfma_f32_16x16x32_bf16: of 16 rows an accumulator takes a quarter of the registers that
// 32x32 tiles need, which leaves room for two workgroups per compute unit (three of narrow
// heads), each wave with a whole key tile on its way.
//
// The four waves take wh = 4, 2 or 1 neighbouring heads (whatever divides H) and share each
// head's key tiles 4 / wh ways.  Waves that walk the same tokens in step read them whole
// lines side by side: with the waves on one head, each 128-byte line of codes was a DRAM
// access of its own, and 4 contexts of up to 131072 tokens stood at 4.4 TB/s with 33 MB in
// flight.
//
// Work list.  The call's work is shared out by the lengths the device sees, not by their
// bound: with T the key tiles of all row tiles, a piece is P = T (H / wh) / target key tiles
// (128 keys a wave at least), so there are about `target` pieces of like size however ragged
// the batch.  (Cut by the bound on the lengths, 16 streams of 300 to 8100 tokens ran as 2048
// workgroups of at most 4 key tiles a wave, half of them empty: 154 us.)  Item x of the
// list: sequence by sequence, row tile, piece, head group (fastest).
struct Item {
  RowTile t;
  int hg, z, pieces, item0;      // head group, piece of `pieces`, item of piece 0 (the next: + hgroups)
  int tile_id, per;              // number of the row tile in the call, key tiles of a piece
};
template <int TM, int TK>
__device__ __forceinline__ bool find_item(const KvAttnArgs& a, int x, Item& it) {
  const int lane = threadIdx.x & 63, n_seq = a.s.n_seq;
  SeqWork w = seq_work<TM, TK>(a, lane);
  int per = 0x3fffffff;
  if (a.target > 0) per = piece_tiles<TM, TK, false>(a, w, a.hgroups, kMinWaveKeys / TK * (kThreads / 64 / a.wh));
  int base = 0;
  for (int c = 0; c < n_seq; c += 64) {
    if (c > 0) w = seq_work<TM, TK>(a, c + lane);
    const int pieces = max(1, (w.nt + per - 1) / per);
    const int mine = w.rt * pieces * a.hgroups, incl = prefix_sum(mine);
    const unsigned long long hit = __ballot(x - base < incl);
    if (hit != 0) {
      const int l = __ffsll((long long)hit) - 1;
      const int first = base + lane_value(incl - mine, l);
      it.pieces = lane_value(pieces, l);
      it.per = a.target > 0 ? (lane_value(w.nt, l) + it.pieces - 1) / it.pieces : per;   // (even pieces)
      const int local = x - first, rest = local / a.hgroups;
      if (local < 0) return false;                   // (sums that wrapped: offsets that hold garbage)
      it.hg = local - rest * a.hgroups;
      const int k = rest / it.pieces;
      it.z = rest - k * it.pieces;
      it.item0 = first + k * it.pieces * a.hgroups + it.hg;
      it.tile_id = first_tile<TM>(a, c + l) + k;
      return place<TM, TK>(a, c + l, lane_value(w.beg, l), lane_value(w.n, l), lane_value(w.len, l), k, it.t);
    }
    base += lane_value(incl, 63);
  }
  return false;
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// max over the four quarters of a wave
__device__ __forceinline__ float quarter_max(float x) {
  const u32x2 s = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return half_swap_max(fmaxf(__uint_as_float(s.x), __uint_as_float(s.y)));
}

template <int DH, bool F8>
__global__ __launch_bounds__(kThreads, row_groups(DH)) void kv_rows_kernel(KvAttnArgs a) {
  constexpr int CPR = DH / 8, ROWB = DH * 2, TK = row_keys(DH, F8), W = kThreads / 64, TM = kFewRows;
  constexpr int SUB = TK / 32, R = 2 * SUB;          // 32-key halves; a lane's rows: l16 + 16 r
  constexpr int NT = DH / 32;                        // contraction steps of S, 32 channels each
  constexpr int ND = DH / 16;                        // 16-channel blocks of O^T
  // Loads of a lane: rows l16 and l16 + 16 of the tile; bf16 16 bytes (channels 32 i + 8
  // quarter ..) for each step; codes 16 bytes (channels 64 i + 16 quarter ..) for two steps,
  // or, of 32-wide heads, 8 bytes for the one step
  constexpr int NL = F8 ? (DH == 32 ? 1 : DH / 64) : NT;
  constexpr bool HALF = F8 && DH == 32;
  __shared__ __attribute__((aligned(1024))) char smem[W * (TM * DH * 4 > 32 * ROWB ? TM * DH * 4 : 32 * ROWB)];
  __shared__ float sm[W][TM], sl[W][TM];

  Item it;
  if (!find_item<TM, TK>(a, blockIdx.x, it)) return;
  const RowTile& t = it.t;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ways = W / a.wh;                         // waves that share a head's key tiles
  const int h = it.hg * a.wh + wave % a.wh;
  const int l16 = lane & 15, qd = lane >> 4;
  const int u0 = min(it.z * it.per, t.nt), u1 = min(u0 + min(it.per, t.nt), t.nt);
  const int nrows = min(TM, t.n_rows - t.row0);
  const int p0 = t.off + t.row0 / a.g, p1 = t.off + (t.row0 + nrows - 1) / a.g;
  const KindBounds kb = kind_bounds(a, t.len, p0, p1);
  const Lead ld = lead_of(t.len);
  RowLimits lim;
  bf16x8 qreg[NT];
  const int r = t.row0 + min(l16, nrows - 1);
  const int tok = r / a.g, hq = h * a.g + (r - tok * a.g);
  lim = row_limits(a, t, t.off + tok);
  const uint16_t* qp = a.q + (long long)(t.beg + tok) * a.qs + hq * DH;
#pragma unroll
  for (int i = 0; i < NT; ++i)
    qreg[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(
        qp + (F8 && !HALF ? 64 * (i / 2) + 16 * qd + 8 * (i % 2) : 32 * i + 8 * qd)));
  const int32_t* table = a.s.table + (long long)t.b * a.s.max_pages;
  auto tile_of = [&](int u) { return u < t.ts ? u : t.tw + t.dir * (u - t.ts); };
  // lane l looks up key l (mod TK) of a tile
  struct Look { int key, id, rem; };
  auto look = [&](int u) __attribute__((always_inline)) -> Look {
    Look k;
    k.key = tile_of(min(u, t.nt - 1)) * TK + (lane & (TK - 1));
    const int kk = min(k.key, t.len - 1);
    const int pg = div_by(kk, a.s.page);
    k.id = table[pg];
    k.rem = kk - pg * a.page;
    return k;
  };
  const long long row_bytes = (long long)a.H * DH * (F8 ? 1 : 2);
  const int lane_bytes = h * DH * (F8 ? 1 : 2) + qd * (HALF ? 8 : 16);
  u32x4 kr[R][NL], vr[R][NL];
  int ke[R], ve[R], ve_cur[R];
  auto load_rows = [&](const uint8_t* base, const long long (&at)[R], u32x4 (&to)[R][NL], int r0, int r1) __attribute__((always_inline)) {
#pragma unroll
    for (int r = r0; r < r1; ++r)
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        if constexpr (HALF) {
          const u32x2 w = *reinterpret_cast<const u32x2*>(base + at[r]);
          to[r][i] = u32x4{w.x, w.y, 0u, 0u};
        } else {
          to[r][i] = *reinterpret_cast<const u32x4*>(base + at[r] + 64 * i);
        }
      }
  };
  char* vt = smem + wave * (32 * ROWB);
  auto vsw = [](int row) { return 2 * ((row / (16 / CPR)) & (CPR / 2 - 1)); };
  // byte offsets in the value tile from which a lane writes and reads; their XORs with a
  // chunk are formed again at each use (opaque() keeps them out of registers across the loop)
  auto opaque = [](unsigned x) { asm volatile("" : "+v"(x)); return x; };
  const unsigned vwr = (unsigned)(l16 * ROWB);
  auto store_v = [&](unsigned wr, int sub) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 2 * sub; r < 2 * sub + 2; ++r) {
      char* at = vt + wr + 16 * (r & 1) * ROWB;      // rows l16 and l16 + 16 have the same swizzle
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const u32x4 w = vr[r][i];
        if constexpr (HALF) {
          *reinterpret_cast<u32x4*>(at + ((qd ^ vsw(l16)) * 16)) = widen8(w.x, w.y, byte_scale(ve_cur[r]));
        } else if constexpr (F8) {
          const float sc = byte_scale(ve_cur[r]);
          const int ch = 8 * i + 2 * qd;
          *reinterpret_cast<u32x4*>(at + ((ch ^ vsw(l16)) * 16)) = widen8(w.x, w.y, sc);
          *reinterpret_cast<u32x4*>(at + (((ch + 1) ^ vsw(l16)) * 16)) = widen8(w.z, w.w, sc);
        } else {
          *reinterpret_cast<u32x4*>(at + (((4 * i + qd) ^ vsw(l16)) * 16)) = w;
        }
      }
    }
  };
  // V^T operand of channels 16 db + l16, keys 16 (i / 4) + 4 qd + i % 4: the order in which
  // S^T leaves them.  Of 16 lanes lane x reads row x / 4 and 4 channels from 4 (x % 4) on.
  const int tr = 4 * qd + (l16 >> 2), trc = (l16 & 3) >> 1;
  const unsigned vrd0 = (unsigned)(tr * ROWB + (trc ^ vsw(tr)) * 16 + 8 * (l16 & 1));
  auto read_v = [&](unsigned rd, int db) __attribute__((always_inline)) -> bf16x8 {
    const lds_char* p = (const lds_char*)(vt) + (rd ^ (32u * db));
    // rows tr and tr + 16 have the same swizzle
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * ROWB)));
    return __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
  };

  f32x4 acc[ND];
  float m_run, l_run;
  m_run = kNoMax;
  l_run = 0.0f;
#pragma unroll
  for (int db = 0; db < ND; ++db) acc[db] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  unsigned long long there = 0, there_next = 0;
  long long at[R];
  // places of the lane's rows (row 0 of page 0 for keys that do not exist)
  auto resolve = [&](const Look& k, unsigned long long& th) __attribute__((always_inline)) {
    const bool in = k.id >= 0 && k.id < a.pages;
    th = __ballot(in && k.key < t.len) & (TK == 64 ? ~0ull : 0xffffffffull);
    const int id = in ? k.id : 0, slot = in ? k.id * a.page + k.rem : 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      at[r] = (long long)__shfl(slot, l16 + 16 * r) * row_bytes + lane_bytes;
      if constexpr (F8) {
        const long long pe = (long long)__shfl(id, l16 + 16 * r) * a.H + h;
        ke[r] = a.ke[pe];
        ve[r] = a.ve[pe];
      }
    }
  };
  Look nxt{};
  int u = u0 + wave / a.wh;
  if (u < u1) {
    const Look first = look(u);
    resolve(first, there);
    load_rows(a.k, at, kr, 0, R);
    load_rows(a.v, at, vr, 0, R);
    nxt = look(u + ways);
  }
#pragma unroll 1
  for (; u < u1; u += ways) {
    const bool more = u + ways < u1;
    const int j0 = tile_of(u) * TK;
    f32x4 sn[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float sc = 0.0f;
      if constexpr (F8) sc = byte_scale(ke[r]);
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        bf16x8 op;
        if constexpr (F8) {
          const u32x4 w = kr[r][i / 2];
          op = __builtin_bit_cast(bf16x8, i % 2 == 0 ? widen8(w.x, w.y, sc) : widen8(w.z, w.w, sc));
        } else {
          op = __builtin_bit_cast(bf16x8, kr[r][i]);
        }
        sn[r] = mfma16(op, qreg[i], i == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : sn[r]);
      }
    }
    if constexpr (F8) {
#pragma unroll
      for (int r = 0; r < R; ++r) ve_cur[r] = ve[r];
    }
    const int kind = tile_kind<TK>(kb, j0, there);
    if (more) {
      resolve(nxt, there_next);
      load_rows(a.k, at, kr, 0, R);
      nxt = look(u + 2 * ways);
    }
    bf16x8 pp[SUB];
    if (kind != 0) {
      if (kind == 1) {
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) {
          const uint32_t bits = visible_bits(lim, a.sinks, j0 + 32 * sub, (uint32_t)(there >> (32 * sub))) >> (4 * qd);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (((bits >> (16 * (e / 4) + e % 4)) & 1) == 0) sn[2 * sub + e / 4][e % 4] = -INFINITY;
        }
      }
      // (see softmax)
      float pe[8 * SUB];
      auto exps = [&]() __attribute__((always_inline)) -> float {
        float rs[4];
#pragma unroll
        for (int e = 0; e < 8 * SUB; ++e) {
          pe[e] = __builtin_amdgcn_exp2f(fmaf(sn[e / 4][e % 4], a.sl2, -m_run));
          rs[e % 4] = e < 4 ? pe[e] : rs[e % 4] + pe[e];
        }
        return (rs[0] + rs[1]) + (rs[2] + rs[3]);
      };
      float sum = exps();
      if (__ballot(!(sum <= ld.bound)) != 0ull) {
        float pm = sn[0][0];
#pragma unroll
        for (int e = 1; e < 8 * SUB; ++e) pm = fmaxf(pm, sn[e / 4][e % 4]);
        const float cand = fmaxf(m_run, fmaf(quarter_max(pm), a.sl2, ld.lead));
        const bool up = cand > m_run + kMaxSlack;
        const float m_new = up ? cand : m_run;
        const float corr = __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= corr;
        m_run = m_new;
#pragma unroll
        for (int db = 0; db < ND; ++db) acc[db] *= corr;
        sum = exps();
      }
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub) {
        const float* p = &pe[8 * sub];
        pp[sub] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]),
                                                   pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])});
      }
      l_run += sum;
    }
    // values, 32 keys at a time through the wave's LDS tile
#pragma unroll
    for (int sub = 0; sub < SUB; ++sub) {
      store_v(opaque(vwr), sub);
      const unsigned vrd = opaque(vrd0);
      bool special = false;
      if (kind == 1) {
        uint32_t m = 0;
#pragma unroll
        for (int db = 0; db < ND; ++db) {
          m |= special_bits(read_v(vrd, db));
          PIN(m);
        }
        special = __ballot((m & 0x80008000u) != 0) != 0ull;
      }
      // (special tiles fetch the next values later: together with them they need more registers)
      if (more && !special) load_rows(a.v, at, vr, 2 * sub, 2 * sub + 2);
      if (kind == 0) continue;
      if (!special) {
#pragma unroll
        for (int db = 0; db < ND; ++db) {
          const bf16x8 op = read_v(vrd, db);
          acc[db] = mfma16(op, pp[sub], acc[db]);
        }
      } else {
#pragma unroll
        for (int db = 0; db < ND; ++db) {
          const bf16x8 op = read_v(vrd, db);
          const f32x4 zero{0.0f, 0.0f, 0.0f, 0.0f};
          const bf16x8 w = seen_weights(pp[sub]);
          acc[db] = mfma16(part_of<kFinite>(op), pp[sub], acc[db]);
          add_infinity<4>(acc[db], mfma16(part_of<kPlus>(op), w, zero), 1.0f);
          add_infinity<4>(acc[db], mfma16(part_of<kMinus>(op), w, zero), -1.0f);
          PIN(acc[db]);
        }
        if (more) load_rows(a.v, at, vr, 2 * sub, 2 * sub + 2);
      }
    }
    there = there_next;
  }

  // ---- join the waves of a head: weights 2^(m_w - max m)
  float l = l_run + __shfl_xor(l_run, 16);
  l += __shfl_xor(l, 32);
  if (qd == 0) {
    sm[wave][l16] = m_run;
    sl[wave][l16] = l;
  }
  __syncthreads();                                   // (the value tiles are read no more)
  float* part = reinterpret_cast<float*>(smem);
  if (l16 < nrows) {
#pragma unroll
    for (int db = 0; db < ND; ++db)
      *reinterpret_cast<f32x4*>(part + (wave * TM + l16) * DH + 16 * db + 4 * qd) = acc[db];
  }
  __syncthreads();
  if (a.target > 0 && it.z == 0 && tid == 0) a.meta[(long long)it.tile_id * a.hgroups + it.hg] = make_int2(it.item0, it.pieces);
  const int per_head = nrows * (DH / 4);
  for (int i = tid; i < a.wh * per_head; i += kThreads) {
    const int hw = i / per_head, j = i - hw * per_head;
    const int ql = j / (DH / 4), d = 4 * (j % (DH / 4));
    float m = kNoMax;
    for (int w = hw; w < W; w += a.wh) m = fmaxf(m, sm[w][ql]);
    float lt = 0.0f;
    f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
    for (int w = hw; w < W; w += a.wh) {
      if (sl[w][ql] == 0.0f) continue;               // saw no key
      const float c = __builtin_amdgcn_exp2f(sm[w][ql] - m);
      lt += c * sl[w][ql];
      o += c * *reinterpret_cast<const f32x4*>(part + (w * TM + ql) * DH + d);
    }
    const bool some = lt != 0.0f;                    // true for NaN, too
    o *= some ? 1.0f / lt : 0.0f;
    const float l2 = some ? (m - ld.lead) + __log2f(lt * ld.scale) : -INFINITY;
    if (it.pieces > 1) {
      const long long at = ((long long)blockIdx.x * a.wh + hw) * TM + ql;
      *reinterpret_cast<f32x4*>(a.part_o + at * DH + d) = o;
      if (d == 0) a.part_lse[at] = l2;
    } else {
      const int rr = t.row0 + ql, tk = rr / a.g;
      const long long row = (long long)(t.beg + tk) * a.Hq + (it.hg * a.wh + hw) * a.g + (rr - tk * a.g);
      put4(a, row, DH, d, o);
      if (a.lse != nullptr && d == 0) a.lse[row] = l2 * kLn2;
    }
  }
}

// Join of the pieces of a row that the rows kernel cut: with l_z the log2 log-sum-exp and
// O_z the normalised output of piece z, O = sum 2^(l_z - max) O_z / sum 2^(l_z - max).
// Pieces without a visible key (-inf) add nothing.  One workgroup per row, its threads
// shared out over four channels each and, in step, the pieces; grid (row tile, head, row).
template <int DH>
__global__ __launch_bounds__(kThreads) void kv_rows_join_kernel(KvAttnArgs a) {
  constexpr int TM = kFewRows, PER = DH / 4, WAYS = kThreads / PER;
  __shared__ float red[kThreads / 64];
  __shared__ f32x4 part[kThreads];
  __shared__ float sums[WAYS];
  const int ql = blockIdx.z, tid = threadIdx.x;
  const int hg = blockIdx.y / a.wh, hw = blockIdx.y - hg * a.wh;
  const int2 meta = a.meta[(long long)blockIdx.x * a.hgroups + hg];
  // (the bounds hold for whatever lies in the workspace: a row tile that does not exist has no
  // entry of this call, which is found out below, after the first loads are on their way)
  if (meta.y < 2 || meta.x < 0 || meta.x >= a.max_items || meta.y > (a.max_items - 1 - meta.x) / a.hgroups + 1) return;
  auto slot = [&](int z) { return ((long long)(meta.x + z * a.hgroups) * a.wh + hw) * TM + ql; };
  const float first = tid < meta.y ? a.part_lse[slot(tid)] : -INFINITY;
  RowTile t;
  if (!row_tile<TM, 32>(a, blockIdx.x, t) || ql >= t.n_rows - t.row0) return;
  float m = first;
  for (int z = tid + kThreads; z < meta.y; z += kThreads) {
    const float l = a.part_lse[slot(z)];
    m = l > m || l != l ? l : m;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const float o = __shfl_xor(m, d);
    m = o > m || o != o ? o : m;
  }
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) m = red[w] > m || red[w] != red[w] ? red[w] : m;
  const int way = tid / PER, d = 4 * (tid % PER);
  float w = 0.0f;
  f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int z = way; z < meta.y; z += WAYS) {
    const float l = a.part_lse[slot(z)];
    const f32x4 p = *reinterpret_cast<const f32x4*>(a.part_o + slot(z) * DH + d);
    const float c = l == m ? 1.0f : __builtin_amdgcn_exp2f(l - m);
    if (l != -INFINITY) {
      w += c;
      o += (c * kJoinScale) * p;
    }
  }
  part[tid] = o;
  if (d == 0) sums[way] = w;
  __syncthreads();
  if (way != 0) return;
#pragma unroll 1
  for (int k = 1; k < WAYS; ++k) {
    w += sums[k];
    o += part[k * PER + tid];
  }
  const bool some = w != 0.0f;
  o *= some ? (1.0f / kJoinScale) / w : 0.0f;
  const int rr = t.row0 + ql, tk = rr / a.g;
  const long long row = (long long)(t.beg + tk) * a.Hq + blockIdx.y * a.g + (rr - tk * a.g);
  put4(a, row, DH, d, o);
  if (a.lse != nullptr && d == 0) a.lse[row] = some ? (m + __log2f(w)) * kLn2 : -INFINITY;
}

// Join of the pieces of every row that the tiles kernels cut, as above.  WAYS threads share
// the pieces of four channels of a row.
template <int DH, int WAYS>
__global__ __launch_bounds__(kThreads) void kv_join_kernel(KvAttnArgs a) {
  constexpr int PER = DH / 4, ROWS = kThreads / (PER * WAYS);
  __shared__ f32x4 part[kThreads];
  __shared__ float tops[kThreads / PER], sums[kThreads / PER];
  const long long rows = (long long)a.s.n_tok * a.Hq;
  const int tid = threadIdx.x, slot = tid / PER, way = slot % WAYS, first = slot - way, d = 4 * (tid % PER);
  const long long row = (long long)blockIdx.x * ROWS + slot / WAYS;
  const bool there = row < rows;
  const float* lse = a.part_lse + (there ? row : 0);
  const float* o_z = a.part_o + (there ? row : 0) * DH + d;
  // (rows of no sequence hold whatever lies in the workspace; they are left alone below)
  const float early = there && way < a.slabs ? lse[way * rows] : -INFINITY;
  const int pieces = there ? min(a.cuts[row], a.slabs) : 0;
  float m = way < pieces ? early : -INFINITY;
#pragma unroll 4
  for (int z = way + WAYS; z < pieces; z += WAYS) {
    const float l = lse[z * rows];
    m = l > m || l != l ? l : m;
  }
  if constexpr (WAYS > 1) {
    if (d == 0) tops[slot] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < WAYS; ++k) {
      const float l = tops[first + k];
      m = l > m || l != l ? l : m;
    }
  }
  float w = 0.0f;
  f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int z = way; z < pieces; z += WAYS) {
    const float l = lse[z * rows];
    const f32x4 p = *reinterpret_cast<const f32x4*>(o_z + z * rows * DH);
    const float c = l == m ? 1.0f : __builtin_amdgcn_exp2f(l - m);
    if (l != -INFINITY) {   // else nothing was written
      w += c;
      o += (c * kJoinScale) * p;
    }
  }
  if constexpr (WAYS > 1) {
    part[tid] = o;
    if (d == 0) sums[slot] = w;
    __syncthreads();
    if (way != 0) return;
#pragma unroll
    for (int k = 1; k < WAYS; ++k) {
      w += sums[first + k];
      o += part[tid + k * PER];
    }
  }
  if (pieces < 2) return;                          // whole, and written
  const int tok = (int)(row / a.Hq);
  if (tok < seq_row(a.s, 0) || tok >= seq_row(a.s, a.s.n_seq)) return;   // of no sequence: left alone
  const bool some = w != 0.0f;
  o *= some ? (1.0f / kJoinScale) / w : 0.0f;
  put4(a, row, DH, d, o);
  if (a.lse != nullptr && d == 0) a.lse[row] = some ? (m + __log2f(w)) * kLn2 : -INFINITY;
}

template <int DH, int WAYS>
void launch_join(const KvAttnArgs& a, hipStream_t stream) {
  const long long threads = (long long)a.s.n_tok * a.Hq * (DH / 4) * WAYS;
  hipLaunchKernelGGL((kv_join_kernel<DH, WAYS>), dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads),
                     0, stream, a);
}

template <int DH, bool F8>
void launch_rows(const KvAttnArgs& a, const KvAttnPlan& p, hipStream_t stream) {
  const int items = p.target > 0 ? p.max_items : p.row_tiles * a.hgroups;
  hipLaunchKernelGGL((kv_rows_kernel<DH, F8>), dim3(items), dim3(kThreads), 0, stream, a);
  if (p.target > 0)
    hipLaunchKernelGGL((kv_rows_join_kernel<DH>), dim3(p.row_tiles, a.H, kFewRows), dim3(kThreads), 0, stream, a);
}

template <int DH, bool F8, bool RUNS>
void launch_tiles(const KvAttnArgs& a, const KvAttnPlan& p, hipStream_t stream) {
  const dim3 grid((p.row_tiles * a.H) + p.target);
  if constexpr (DH == 128) {
    if (p.rows == kPairRows) {
      hipLaunchKernelGGL((kv_pairs_kernel<F8, RUNS>), grid, dim3(kPairThreads), 0, stream, a);
      return;
    }
  }
  hipLaunchKernelGGL((kv_tiles_kernel<DH, F8, RUNS>), grid, dim3(kThreads), 0, stream, a);
}

template <int DH, bool F8>
void launch_as(const KvAttnArgs& a, const KvAttnPlan& p, hipStream_t stream) {
  if (p.rows == kFewRows) return launch_rows<DH, F8>(a, p, stream);
  if (a.page % copy_rows(DH) == 0) launch_tiles<DH, F8, true>(a, p, stream);
  else launch_tiles<DH, F8, false>(a, p, stream);
  if (p.target > 0 && p.pieces >= kJoinWays) launch_join<DH, kJoinWays>(a, stream);
  else if (p.target > 0) launch_join<DH, 1>(a, stream);
}

}  // namespace

// (host code's view of code_rows, for tests)
int kv_attn_code_rows(int dh, int wave, int i) { return i < code_loads(dh) ? code_rows(dh, wave, i) : -1; }

KvAttnPlan kv_attn_plan(long long n_tok, int n_seq, int g, int H, int dh, bool f8, long long max_len, int window, int sinks,
                        int cus) {
  KvAttnPlan p{};
  const long long rows = n_tok * g, mean = (rows + n_seq - 1) / n_seq;
  long long keys = max_len;
  if (window > 0) keys = std::min(keys, (long long)window + (mean + g - 1) / g + sinks + 2 * kTileKeys);
  const long long nt = (keys + kTileKeys - 1) / kTileKeys;
  auto units = [&](long long tile_rows) { return n_seq * ((mean + tile_rows - 1) / tile_rows) * H; };
  // Rows per workgroup, by their mean over the sequences (8 heads of 128 in bf16 unless said).
  // The rows kernel up to 16 of codes, which the tiles kernel widens once for 128 rows, for
  // few as for many (one sequence of 131072: 64 us, as 128-row tiles 86), and of bf16 where
  // nothing is cut (256 of 512 tokens 94 and 117); else up to 8 (16 streams of 300 to 8100
  // tokens, 4 rows 63 and 69; 16 rows 64 and 50; 8 of 4096, 16 rows 40 and 32).
  // From 17 on the half-filled tiles win: 8 of 4096, 17 rows 46 us and 30, 32 rows 58 and 32.
  // Pairs beyond 128 rows of 128 channels, if they can be cut into enough pieces to fill the
  // card: 8 of 4096 with 192 rows 51 us, 57 in tiles; 768 rows 107 and 140; but 4 of 1024
  // with 192 rows, 64 pieces, 30 and 25.  (Tiles below that switch have no more pieces, and so
  // no more workspace, than pairs above it: 3/4 cus / units at most.)
  const bool pairs = dh == 128 && mean > kTileRows && units(kPairRows) * ((nt + 7) / 8) >= cus * 3 / 4;
  const int few = f8 || units(kTileRows) > cus ? kFewRows : kFewRows / 2;
  p.rows = mean <= few ? kFewRows : pairs ? kPairRows : kTileRows;
  p.wh = H % 4 == 0 ? 4 : H % 2 == 0 ? 2 : 1;
  // at most, over all ways to share the rows out
  p.row_tiles = (int)(p.rows == kFewRows ? rows / p.rows + n_seq : (rows + (long long)n_seq * (p.rows - 1)) / p.rows);
  if (cus <= 0 || n_tok < 1) return p;
  if (p.rows < kTileRows) {
    // workgroups resident at once, less the partial pieces that the row tiles end with
    const long long resident = (long long)cus * row_groups(dh), items = units(kFewRows) / p.wh;
    if (keys <= kMinWaveKeys * (kThreads / 64 / p.wh) || items >= resident) return p;
    p.target = (int)std::max(resident - items / 2, resident / 2);
    p.max_items = p.target + p.row_tiles * (H / p.wh) + 1;
    p.part_bytes = align_up((size_t)p.max_items * p.wh * p.rows * dh * 4);
    p.lse_bytes = align_up((size_t)p.max_items * p.wh * p.rows * 4);
    p.bytes = p.part_bytes + p.lse_bytes + align_up((size_t)p.row_tiles * (H / p.wh) * sizeof(int2));
    return p;
  }
  const long long resident = (long long)cus * (p.rows == kPairRows ? 1 : 2), items = units(p.rows);
  // Key tiles of a piece: a piece of few rows leaves little to join (48 rows over 4 x 1024
  // keys: 17 us with 4 tiles at least, 22 with 8; 128 rows over 16384: 48 and 36).
  p.least = (int)std::clamp(mean / 16, 4ll, 8ll);
  // A sequence is cut into at most four times as many pieces as all would be at one length.
  const long long want = resident / std::max(items, 1ll);
  const long long most = std::min<long long>(kMaxPieces, (nt + p.least - 1) / p.least);
  p.pieces = (int)std::min(want, most);
  if (p.pieces < 2) return p;
  p.slabs = (int)std::min(4 * want, most);
  p.target = (int)resident;
  p.part_bytes = align_up((size_t)p.slabs * n_tok * H * g * dh * 4);
  p.lse_bytes = align_up((size_t)p.slabs * n_tok * H * g * 4);
  p.bytes = p.part_bytes + p.lse_bytes + align_up((size_t)n_tok * H * g * 4);
  return p;
}

cast_status_t launch_kv_attn(const void* q, long long q_stride, int Hq, const cast_kv_cache_t& c,
                             const cast_kv_seqs_t& s, int causal, int window, int sinks, float scale, void* out,
                             float* lse, const KvAttnPlan& plan, void* workspace, hipStream_t stream) {
  KvAttnArgs a{};
  a.q = static_cast<const uint16_t*>(q);
  a.qs = q_stride;
  a.k = static_cast<const uint8_t*>(c.k);
  a.v = static_cast<const uint8_t*>(c.v);
  a.ke = c.k_exp;
  a.ve = c.v_exp;
  a.s = make_seqs(s, c.page);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.part_o = static_cast<float*>(workspace);
  a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.part_bytes);
  a.meta = reinterpret_cast<int2*>(static_cast<char*>(workspace) + plan.part_bytes + plan.lse_bytes);
  a.cuts = reinterpret_cast<int*>(a.meta);
  a.wh = plan.wh;
  a.hgroups = c.H / plan.wh;
  a.target = plan.target;
  a.max_items = plan.max_items;
  a.Hq = Hq;
  a.H = c.H;
  a.g = Hq / c.H;
  a.pages = c.pages;
  a.page = c.page;
  a.causal = causal;
  a.window = window;
  a.sinks = window > 0 ? sinks : 0;
  a.slabs = plan.slabs;
  a.least = plan.least;
  a.sl2 = scale * 1.4426950408889634f;
  const bool f8 = c.dtype == 2;
  switch (c.dh) {
    case 32: f8 ? launch_as<32, true>(a, plan, stream) : launch_as<32, false>(a, plan, stream); break;
    case 64: f8 ? launch_as<64, true>(a, plan, stream) : launch_as<64, false>(a, plan, stream); break;
    default: f8 ? launch_as<128, true>(a, plan, stream) : launch_as<128, false>(a, plan, stream); break;
  }
  return check_launch("kv_attn");
}

}  // namespace cast
