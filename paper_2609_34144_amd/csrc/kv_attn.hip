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
// Two kernels:
//   tiles  128 rows per workgroup; its four waves share 64-key tiles in LDS, copied one
//          tile ahead.  Bound by the matrix cores and the softmax's VALU work.
//   rows   32 rows per workgroup (few rows: decoding); each wave takes every fourth 32-key
//          tile by itself, keys straight from memory into MFMA operands, values through a
//          private LDS tile; no barrier until the four results are joined.  Bound by HBM.
// Long key ranges with few row tiles are cut into pieces, joined by a second kernel.
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
constexpr int kRows = 32;        // of the rows kernel
constexpr int kRowKeys = 32;     // keys per tile and wave there
constexpr int kMaxPieces = 128;
// s_waitcnt vmcnt(0) that leaves expcnt and lgkmcnt free
constexpr int kVmcnt0 = 0x0F70;
// The running maximum moves only when a tile exceeds it by more than 2^8 (see softmax).
constexpr float kMaxSlack = 8.0f;
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
  float* part_o;                 // [pieces][n_tok * Hq][dh], normalised
  float* part_lse;               // [pieces][n_tok * Hq], log2 domain
  int Hq, H, g, pages, page;
  int causal, window, sinks;     // window 0: none
  int npieces, piece_tiles;
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
// max over lanes l and l ^ 32 (not __builtin_bit_cast(float, s.y): on an element of a vector
// it reads the vector's first)
__device__ __forceinline__ float half_swap_max(float x) {
  const u32x2 s = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return fmaxf(__uint_as_float(s.x), __uint_as_float(s.y));
}

// LDS images: chunk c (16 bytes) of tile row r is stored at chunk c ^ swz(r), CPR chunks
// per row.  K: ds_read_b128 of one chunk by 32 consecutive rows; V: the transposing read's
// 4 rows x 32 bytes per 16 lanes; both conflict-free.
__device__ __forceinline__ constexpr int kswz(int r, int cpr) { return (r / (16 / cpr)) & (cpr - 1); }
__device__ __forceinline__ constexpr int vswz(int r, int cpr) { return ((2 * (r & 3)) ^ (8 * (r & 1))) & (cpr - 1); }

// eight e4m3 codes (two dwords) times 2^(exponent of sc), exact in bf16
__device__ __forceinline__ u32x4 widen8(uint32_t a, uint32_t b, float sc) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, sc, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, sc, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, sc, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, sc, true))};
}
__device__ __forceinline__ float byte_scale(int e) { return __uint_as_float((uint32_t)e << 23); }

// ---- the row tile of a workgroup and the key tiles it meets ----------------------------
struct RowTile {
  int b, beg, n_rows, row0;      // sequence, its first call row, its rows (tokens * g), first row here
  int len, off;                  // its length; position of its first token of the call
  int ts, tw, nt;                // logical key tile u: u < ts ? u : tw + u - ts; nt in all
};
// x-th row tile of the call (tiles of TM rows; sequence b's are numbered from
// floor(cu[b] g / TM) + b, which leaves room for its partial tile)
template <int TM, int TK>
__device__ __forceinline__ bool row_tile(const KvAttnArgs& a, int x, RowTile& t) {
  auto start = [&](int i) { return (int)((unsigned)(seq_row(a.s, i) * a.g) / (unsigned)TM) + i; };
  t.b = find_seq(a.s.n_seq, x, start);
  t.beg = seq_row(a.s, t.b);
  const int n = max(seq_row(a.s, t.b + 1) - t.beg, 0), k = x - start(t.b);
  t.n_rows = n * a.g;
  if (k < 0 || (long long)k * TM >= t.n_rows) return false;
  t.row0 = k * TM;
  t.len = seq_len(a.s, t.b);
  t.off = t.len - n;
  const int p_lo = t.off + t.row0 / a.g, p_hi = t.off + (min(t.row0 + TM, t.n_rows) - 1) / a.g;
  const int hi = max(a.causal ? min(p_hi + 1, t.len) : t.len, 0);
  const int lo = a.window > 0 ? min(max(p_lo - a.window + 1, 0), hi) : 0;
  const int sk = a.window > 0 ? min(a.sinks, hi) : 0;
  const int te = (hi + TK - 1) / TK;
  t.ts = (sk + TK - 1) / TK;
  t.tw = max(lo / TK, t.ts);
  t.nt = t.ts + max(te - t.tw, 0);
  return true;
}
// logical key tiles [u0, u1) of piece z
__device__ __forceinline__ void piece_range(const KvAttnArgs& a, int nt, int z, int& u0, int& u1) {
  const int per = max(a.piece_tiles, (nt + a.npieces - 1) / a.npieces);
  u0 = min(z * per, nt);
  u1 = min(u0 + per, nt);
}

// A lane's row, and which keys it sees: j < hi, and j >= lo or j < sinks.
struct RowLimits {
  int hi, lo;
};
__device__ __forceinline__ RowLimits row_limits(const KvAttnArgs& a, const RowTile& t, int p) {
  return RowLimits{a.causal ? min(p + 1, t.len) : t.len, a.window > 0 ? p - a.window + 1 : 0};
}

// Whether a key tile [j0, j0 + TK) is seen by none (0), some (1) or all (2) of the rows at
// positions p0 .. p1; `there`: bit per key, set where the key exists.
template <int TK>
__device__ __forceinline__ int tile_kind(const KvAttnArgs& a, int j0, int p0, int p1, unsigned long long there) {
  const unsigned long long all = TK == 64 ? ~0ull : (1ull << TK) - 1;
  if (there == 0) return 0;
  if (a.causal && j0 > p1) return 0;
  const bool win = a.window > 0;
  if (win && j0 + TK - 1 <= p0 - a.window && j0 >= a.sinks) return 0;
  const bool full = there == all && (!a.causal || j0 + TK - 1 <= p0) &&
                    (!win || j0 > p1 - a.window || j0 + TK - 1 < a.sinks);
  return full ? 2 : 1;
}

// S^T accumulator element e of block kb belongs to key kb * 32 + 8 (e / 4) + 4 hf + e % 4.
template <int NB>
__device__ __forceinline__ void mask_scores(f32x16 (&sn)[NB], int j0, int hf, RowLimits r, int sinks,
                                            unsigned long long there) {
  const unsigned long long bits = there >> (4 * hf);
#pragma unroll
  for (int kb = 0; kb < NB; ++kb)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int c = kb * 32 + 8 * (e / 4) + e % 4;
      const int key = j0 + c + 4 * hf;
      const bool seen = key < r.hi && (key >= r.lo || key < sinks) && ((bits >> c) & 1) != 0;
      if (!seen) sn[kb][e] = -INFINITY;
    }
}

// Exponentials of a tile against the running maximum, packed as P^T operands, and their
// sum.  A lane's sum of at most 2^8 shows that no score is far above the maximum, which
// then may stay (probabilities up to 2^8 do no harm in fp32 sums and bf16 operands); else
// the maximum is taken over the tile, moved, and the sums so far scaled down.
template <int NB, int ND>
__device__ __forceinline__ void softmax(const f32x16 (&sn)[NB], bf16x8 (&pp)[NB][2], float& m_run, float& l_run,
                                        f32x16 (&acc)[ND], float sl2) {
  float pe[NB * 16], rs[4];
  auto exps = [&]() __attribute__((always_inline)) -> float {
#pragma unroll
    for (int e = 0; e < NB * 16; ++e) {
      pe[e] = __builtin_amdgcn_exp2f(fmaf(sn[e / 16][e % 16], sl2, -m_run));
      rs[e % 4] = e < 4 ? pe[e] : rs[e % 4] + pe[e];
    }
    return (rs[0] + rs[1]) + (rs[2] + rs[3]);
  };
  float sum = exps();
  if (__ballot(!(sum <= 256.0f)) != 0ull) {
    float pm = sn[0][0];
#pragma unroll
    for (int e = 1; e < NB * 16; ++e) pm = fmaxf(pm, sn[e / 16][e % 16]);
    const float cand = fmaxf(m_run, half_swap_max(pm) * sl2);
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
    const float* p = &pe[8 * g];
    pp[g / 2][g % 2] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]),
                                                        pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])});
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
  });
}

// The same where some row does not see some key.  There P = 0, and 0 times an infinity or
// NaN that lies at the invisible place must add nothing: the tile's product is formed
// apart, and if it is not finite, from the finite values plus the signs of the others at
// the keys whose weight is not zero (both signs, or a NaN, give NaN).
template <int NB, int ND, class R>
__device__ __forceinline__ void values_masked(R&& read, const bf16x8 (&pp)[NB][2], f32x16 (&acc)[ND]) {
#pragma unroll
  for (int db = 0; db < ND; ++db) {
    f32x16 t{};
#pragma unroll
    for (int g = 0; g < 2 * NB; ++g) t = mfma(read(db, g / 2, g % 2), pp[g / 2][g % 2], t);
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 16; ++e) bad |= !(fabsf(t[e]) < INFINITY);
    if (__ballot(bad) != 0ull) {
      f32x16 fin{}, pos{}, neg{};
#pragma unroll 1
      for (int g = 0; g < 2 * NB; ++g) {
        u32x4 v = __builtin_bit_cast(u32x4, read(db, g / 2, g % 2)), vp, vn, w;
        bf16x8 p8 = pp[0][0];
#pragma unroll
        for (int x = 1; x < 2 * NB; ++x)
          if (g == x) p8 = pp[x / 2][x % 2];
        const u32x4 p = __builtin_bit_cast(u32x4, p8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          vp[i] = vn[i] = w[i] = 0;
#pragma unroll
          for (int s = 0; s < 32; s += 16) {
            const uint32_t one = 0x3f80u << s, x = (v[i] >> s) & 0xffffu;
            if ((x & 0x7f80u) == 0x7f80u) {
              if (x != 0xff80u) vp[i] |= one;
              if (x != 0x7f80u) vn[i] |= one;
              v[i] &= ~(0xffffu << s);
            }
            if (((p[i] >> s) & 0x7fffu) != 0) w[i] |= one;
          }
        }
        const bf16x8 seen = __builtin_bit_cast(bf16x8, w);
        fin = mfma(__builtin_bit_cast(bf16x8, v), p8, fin);
        pos = mfma(__builtin_bit_cast(bf16x8, vp), seen, pos);
        neg = mfma(__builtin_bit_cast(bf16x8, vn), seen, neg);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e)
        t[e] = (fin[e] + (pos[e] > 0.0f ? INFINITY : 0.0f)) + (neg[e] > 0.0f ? -INFINITY : 0.0f);
    }
    acc[db] += t;
  }
}

// A row's place in the call and its result: 16-byte-aligned groups of four channels.
__device__ __forceinline__ void put4(const KvAttnArgs& a, long long row, int dh, int d, f32x4 o) {
  *reinterpret_cast<u32x2*>(a.out + row * dh + d) = u32x2{pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w)};
}

// ---------------------------------------------------------------------------
// tiles
// ---------------------------------------------------------------------------
template <int DH, bool F8>
__global__ __launch_bounds__(kThreads, 2) void kv_tiles_kernel(KvAttnArgs a) {
  constexpr int CPR = DH / 8, ROWB = DH * 2, ND = DH / 32, TK = kTileKeys;
  constexpr int NSLOT = DH / 32;             // 1-KB copies of a bf16 tile per wave
  constexpr int RSTEP = 2048 / DH;           // tile rows between them
  constexpr int C8 = DH / 16;                // 16-byte chunks of a row of codes
  constexpr int N8 = (TK * C8 + kThreads - 1) / kThreads;
  // separate objects: the compiler sees that copies do not touch the buffer being read
  __shared__ __attribute__((aligned(1024))) uint16_t lds_k0[TK * DH];
  __shared__ __attribute__((aligned(1024))) uint16_t lds_k1[TK * DH];
  __shared__ __attribute__((aligned(1024))) uint16_t lds_v0[TK * DH];
  __shared__ __attribute__((aligned(1024))) uint16_t lds_v1[TK * DH];

  RowTile t;
  if (!row_tile<kTileRows, TK>(a, blockIdx.x, t)) return;
  const int h = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hf = lane >> 5;
  int u0, u1;
  piece_range(a, t.nt, blockIdx.z, u0, u1);

  // the lane's row; rows past the end repeat the last one and are not stored
  const int w0 = t.row0 + wave * 32;
  const bool live = w0 < t.n_rows;
  const int r = min(w0 + l32, t.n_rows - 1);
  const int tok = r / a.g, hq = h * a.g + (r - tok * a.g);
  const int p0 = t.off + min(w0, t.n_rows - 1) / a.g, p1 = t.off + min(w0 + 31, t.n_rows - 1) / a.g;
  const RowLimits lim = row_limits(a, t, t.off + tok);
  bf16x8 qreg[DH / 16];
  {
    const uint16_t* qp = a.q + (long long)(t.beg + tok) * a.qs + hq * DH + 8 * hf;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) qreg[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qp + 16 * i));
  }

  // ---- key lookup: lane l of every wave looks up key l of a tile
  const int32_t* table = a.s.table + (long long)t.b * a.s.max_pages;
  auto tile_of = [&](int u) { return u < t.ts ? u : t.tw + (u - t.ts); };
  struct Look { int key, id, rem; };
  auto look = [&](int u) __attribute__((always_inline)) -> Look {
    Look k;
    k.key = tile_of(min(u, t.nt - 1)) * TK + lane;
    const int kk = min(k.key, t.len - 1);
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
      const long long at = (long long)__shfl(slot, brow + i * RSTEP) * row_bytes + head_bytes;
      const int lb = (wave + 4 * i) * 1024;
      __builtin_amdgcn_global_load_lds((glb_void*)(a.k + at + kofs), (lds_void*)(reinterpret_cast<char*>(kd) + lb), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((glb_void*)(a.v + at + vofs), (lds_void*)(reinterpret_cast<char*>(vd) + lb), 16, 0, 0);
    });
  };
  u32x4 ck[N8], cv[N8];
  int ex = 0;                                // exponent bytes of the lane's key: K | V << 8
  auto load8 = [&](int slot, int id) __attribute__((always_inline)) {
    const long long pe = (long long)(id >= 0 && id < a.pages ? id : 0) * a.H + h;
    ex = (int)a.ke[pe] | (int)a.ve[pe] << 8;
#pragma unroll
    for (int i = 0; i < N8; ++i) {
      const int c = tid + i * kThreads, row = min(c / C8, TK - 1);
      const long long at = (long long)__shfl(slot, row) * row_bytes + head_bytes + (c % C8) * 16;
      ck[i] = *reinterpret_cast<const u32x4*>(a.k + at);
      cv[i] = *reinterpret_cast<const u32x4*>(a.v + at);
    }
  };
  auto store8 = [&](uint16_t* kd, uint16_t* vd) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N8; ++i) {
      const int c = tid + i * kThreads, row = c / C8, ch = 2 * (c % C8);
      const int e = __shfl(ex, min(row, TK - 1));
      if (row < TK) {
        const float sk = byte_scale(e & 255), sv = byte_scale(e >> 8);
        char* kr = reinterpret_cast<char*>(kd) + row * ROWB;
        char* vr = reinterpret_cast<char*>(vd) + row * ROWB;
        *reinterpret_cast<u32x4*>(kr + ((ch ^ kswz(row, CPR)) * 16)) = widen8(ck[i].x, ck[i].y, sk);
        *reinterpret_cast<u32x4*>(kr + (((ch + 1) ^ kswz(row, CPR)) * 16)) = widen8(ck[i].z, ck[i].w, sk);
        *reinterpret_cast<u32x4*>(vr + ((ch ^ vswz(row, CPR)) * 16)) = widen8(cv[i].x, cv[i].y, sv);
        *reinterpret_cast<u32x4*>(vr + (((ch + 1) ^ vswz(row, CPR)) * 16)) = widen8(cv[i].z, cv[i].w, sv);
      }
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
  auto read_k = [&](const uint16_t* kt, int i, int kb) __attribute__((always_inline)) -> bf16x8 {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(
        reinterpret_cast<const char*>(kt) + (kbase ^ (32u * i)) + kb * 32 * ROWB));
  };
  auto read_v = [&](const uint16_t* vt, int db, int kb, int s2) __attribute__((always_inline)) -> bf16x8 {
    const lds_char* p = (const lds_char*)(vt) + (vbase ^ (64u * db)) + (32 * kb + 16 * s2) * ROWB;
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
    const int kind = live ? tile_kind<TK>(a, j0, p0, p1, there) : 0;
    if (kind != 0) {
      f32x16 sn[2];
      constexpr int N = 2 * (DH / 16), AHEAD = 3;
      bf16x8 op[N];
      static_for<0, AHEAD>([&](auto uu) { constexpr int i = decltype(uu)::value; op[i] = read_k(kt, i / 2, i % 2); });
      static_for<0, N>([&](auto uu) {
        constexpr int i = decltype(uu)::value, n = i + AHEAD;
        if constexpr (n < N) op[n] = read_k(kt, n / 2, n % 2);
        sn[i % 2] = mfma(op[i], qreg[i / 2], i < 2 ? f32x16{} : sn[i % 2]);
      });
      if (kind == 1) mask_scores<2>(sn, j0, hf, lim, a.sinks, there);
      bf16x8 pp[2][2];
      softmax<2, ND>(sn, pp, m_run, l_run, acc, a.sl2);
      auto rd = [&](int db, int kb, int s2) __attribute__((always_inline)) { return read_v(vt, db, kb, s2); };
      if (kind == 2) values<2, ND>(rd, pp, acc);
      else values_masked<2, ND>(rd, pp, acc);
    }
    if constexpr (F8) {
      if (more) store8(kn, vn);
    }
    there = there_next;
    __builtin_amdgcn_s_waitcnt(kVmcnt0);
    __syncthreads();
  };
  int u = u0;
  for (; u + 1 < u1; u += 2) {
    tile(IC<0>{}, u);
    tile(IC<1>{}, u + 1);
  }
  if (u < u1) tile(IC<0>{}, u);

  if (w0 + l32 >= t.n_rows) return;
  const float l = l_run + __shfl_xor(l_run, 32);
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  const float l2 = l > 0.0f || l != l ? m_run + __log2f(l) : -INFINITY;
  const long long row = (long long)(t.beg + tok) * a.Hq + hq;
  if (a.npieces > 1) {
    const long long at = (long long)blockIdx.z * a.s.n_tok * a.Hq + row;
    if (hf == 0) a.part_lse[at] = l2;
    if (u0 < u1) {
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4)
          *reinterpret_cast<f32x4*>(a.part_o + at * DH + db * 32 + 8 * g4 + 4 * hf) =
              f32x4{acc[db][4 * g4] * inv, acc[db][4 * g4 + 1] * inv, acc[db][4 * g4 + 2] * inv, acc[db][4 * g4 + 3] * inv};
    }
    return;
  }
#pragma unroll
  for (int db = 0; db < ND; ++db)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4)
      put4(a, row, DH, db * 32 + 8 * g4 + 4 * hf,
           f32x4{acc[db][4 * g4] * inv, acc[db][4 * g4 + 1] * inv, acc[db][4 * g4 + 2] * inv, acc[db][4 * g4 + 3] * inv});
  if (a.lse != nullptr && hf == 0) a.lse[row] = l2 * kLn2;
}

// ---------------------------------------------------------------------------
// rows
// ---------------------------------------------------------------------------
template <int DH, bool F8>
__global__ __launch_bounds__(kThreads, 2) void kv_rows_kernel(KvAttnArgs a) {
  constexpr int CPR = DH / 8, ROWB = DH * 2, ND = DH / 32, TK = kRowKeys, W = kThreads / 64;
  constexpr int NK = F8 ? DH / 32 : DH / 16;         // 16-byte loads of a lane's key half
  constexpr int CV = F8 ? DH / 16 : DH / 8;          // 16-byte chunks of a value row in memory
  constexpr int NV = TK * CV / 64;                   // loads of a value tile per lane
  constexpr int VSTEP = 64 / CV;                     // rows between them
  // value tiles, one per wave; afterwards the waves' results
  __shared__ __attribute__((aligned(1024))) char smem[W * kRows * DH * 4];
  __shared__ float sm[W][kRows], sl[W][kRows];

  RowTile t;
  if (!row_tile<kRows, TK>(a, blockIdx.x, t)) return;
  const int h = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hf = lane >> 5;
  int u0, u1;
  piece_range(a, t.nt, blockIdx.z, u0, u1);
  const int nrows = min(kRows, t.n_rows - t.row0);
  const int r = t.row0 + min(l32, nrows - 1);
  const int tok = r / a.g, hq = h * a.g + (r - tok * a.g);
  const int p0 = t.off + t.row0 / a.g, p1 = t.off + (t.row0 + nrows - 1) / a.g;
  const RowLimits lim = row_limits(a, t, t.off + tok);
  // Q^T in the order in which the lane gets its key's channels: bf16 16 i + 8 hf ..; codes
  // come 16 to a load, so 32 (i / 2) + 16 hf + 8 (i % 2) ..
  bf16x8 qreg[DH / 16];
  {
    const uint16_t* qp = a.q + (long long)(t.beg + tok) * a.qs + hq * DH;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i)
      qreg[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(
          qp + (F8 ? 32 * (i / 2) + 16 * hf + 8 * (i % 2) : 16 * i + 8 * hf)));
  }
  const int32_t* table = a.s.table + (long long)t.b * a.s.max_pages;
  auto tile_of = [&](int u) { return u < t.ts ? u : t.tw + (u - t.ts); };
  struct Look { int key, id, rem; };
  auto look = [&](int u) __attribute__((always_inline)) -> Look {
    Look k;
    k.key = tile_of(min(u, t.nt - 1)) * TK + l32;
    const int kk = min(k.key, t.len - 1);
    const int pg = div_by(kk, a.s.page);
    k.id = table[pg];
    k.rem = kk - pg * a.page;
    return k;
  };
  const long long row_bytes = (long long)a.H * DH * (F8 ? 1 : 2), head_bytes = (long long)h * DH * (F8 ? 1 : 2);
  u32x4 kr[NK], vr[NV];
  int ex = 0;
  auto load_k = [&](int slot) __attribute__((always_inline)) {
    const uint8_t* p = a.k + (long long)slot * row_bytes + head_bytes + 16 * hf;
#pragma unroll
    for (int i = 0; i < NK; ++i) kr[i] = *reinterpret_cast<const u32x4*>(p + 32 * i);
  };
  auto load_v = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int row = lane / CV + i * VSTEP;
      vr[i] = *reinterpret_cast<const u32x4*>(a.v + (long long)__shfl(slot, row) * row_bytes + head_bytes + (lane % CV) * 16);
    }
  };
  auto load_e = [&](int id) __attribute__((always_inline)) {
    if constexpr (F8) {
      const long long pe = (long long)(id >= 0 && id < a.pages ? id : 0) * a.H + h;
      ex = (int)a.ke[pe] | (int)a.ve[pe] << 8;
    }
  };
  char* vt = smem + wave * (TK * ROWB);
  auto store_v = [&](int e) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int row = lane / CV + i * VSTEP;
      char* at = vt + row * ROWB;
      if constexpr (F8) {
        const float sc = byte_scale(__shfl(e, row) >> 8);
        const int ch = 2 * (lane % CV);
        *reinterpret_cast<u32x4*>(at + ((ch ^ vswz(row, CPR)) * 16)) = widen8(vr[i].x, vr[i].y, sc);
        *reinterpret_cast<u32x4*>(at + (((ch + 1) ^ vswz(row, CPR)) * 16)) = widen8(vr[i].z, vr[i].w, sc);
      } else {
        *reinterpret_cast<u32x4*>(at + (((lane % CV) ^ vswz(row, CPR)) * 16)) = vr[i];
      }
    }
  };
  unsigned vbase;
  {
    const int gq = lane >> 4, la = lane & 15;
    const int row = 4 * (gq >> 1) + (la >> 2);
    const int c = 2 * (gq & 1) + ((la & 3) >> 1);
    vbase = (unsigned)(row * ROWB + ((c ^ vswz(row, CPR)) * 16) + 8 * (la & 1));
  }
  auto read_v = [&](int db, int, int s2) __attribute__((always_inline)) -> bf16x8 {
    const lds_char* p = (const lds_char*)(vt) + (vbase ^ (64u * db)) + 16 * s2 * ROWB;
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

  auto resolve = [&](const Look& k, unsigned long long& there) __attribute__((always_inline)) -> int {
    const bool in = k.id >= 0 && k.id < a.pages;
    there = __ballot(in && k.key < t.len) & 0xffffffffull;
    return in ? k.id * a.page + k.rem : 0;
  };
  unsigned long long there = 0, there_next = 0;
  Look nxt{};
  int u = u0 + wave;
  if (u < u1) {
    const Look first = look(u);
    const int slot = resolve(first, there);
    load_e(first.id);
    load_k(slot);
    load_v(slot);
    nxt = look(u + W);
  }
#pragma unroll 1
  for (; u < u1; u += W) {
    const bool more = u + W < u1;
    const int j0 = tile_of(u) * TK;
    const int e_cur = ex;
    f32x16 sn[1];
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) {
      bf16x8 op;
      if constexpr (F8) {
        const u32x4 w = kr[i / 2];
        const float sc = byte_scale(e_cur & 255);
        op = __builtin_bit_cast(bf16x8, i % 2 == 0 ? widen8(w.x, w.y, sc) : widen8(w.z, w.w, sc));
      } else {
        op = __builtin_bit_cast(bf16x8, kr[i]);
      }
      sn[0] = mfma(op, qreg[i], i == 0 ? f32x16{} : sn[0]);
    }
    int slot = 0;
    if (more) {
      slot = resolve(nxt, there_next);
      load_e(nxt.id);
      load_k(slot);
      nxt = look(u + 2 * W);
    }
    store_v(e_cur);
    if (more) load_v(slot);
    const int kind = tile_kind<TK>(a, j0, p0, p1, there);
    if (kind != 0) {
      if (kind == 1) mask_scores<1>(sn, j0, hf, lim, a.sinks, there);
      bf16x8 pp[1][2];
      softmax<1, ND>(sn, pp, m_run, l_run, acc, a.sl2);
      if (kind == 2) values<1, ND>(read_v, pp, acc);
      else values_masked<1, ND>(read_v, pp, acc);
    }
    there = there_next;
  }

  // ---- join the four waves: weights 2^(m_w - max m)
  const float l = l_run + __shfl_xor(l_run, 32);
  if (hf == 0) {
    sm[wave][l32] = m_run;
    sl[wave][l32] = l;
  }
  __syncthreads();
  float* part = reinterpret_cast<float*>(smem) + wave * kRows * DH;
  if (l32 < nrows) {
#pragma unroll
    for (int db = 0; db < ND; ++db)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        *reinterpret_cast<f32x4*>(part + l32 * DH + db * 32 + 8 * g4 + 4 * hf) =
            f32x4{acc[db][4 * g4], acc[db][4 * g4 + 1], acc[db][4 * g4 + 2], acc[db][4 * g4 + 3]};
  }
  __syncthreads();
  for (int i = tid; i < nrows * (DH / 4); i += kThreads) {
    const int ql = i / (DH / 4), d = 4 * (i % (DH / 4));
    float m = sm[0][ql];
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, sm[w][ql]);
    float lt = 0.0f;
    f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (sl[w][ql] == 0.0f) continue;         // saw no key
      const float c = __builtin_amdgcn_exp2f(sm[w][ql] - m);
      lt += c * sl[w][ql];
      o += c * *reinterpret_cast<const f32x4*>(reinterpret_cast<float*>(smem) + (w * kRows + ql) * DH + d);
    }
    const bool some = lt != 0.0f;              // true for NaN, too
    o *= some ? 1.0f / lt : 0.0f;
    const float l2 = some ? m + __log2f(lt) : -INFINITY;
    const int rr = t.row0 + ql, tk = rr / a.g;
    const long long row = (long long)(t.beg + tk) * a.Hq + h * a.g + (rr - tk * a.g);
    if (a.npieces > 1) {
      const long long at = (long long)blockIdx.z * a.s.n_tok * a.Hq + row;
      *reinterpret_cast<f32x4*>(a.part_o + at * DH + d) = o;
      if (d == 0) a.part_lse[at] = l2;
    } else {
      put4(a, row, DH, d, o);
      if (a.lse != nullptr && d == 0) a.lse[row] = l2 * kLn2;
    }
  }
}

// Join of the pieces of every row: with l_z the log2 log-sum-exp and O_z the normalised
// output of piece z, O = sum 2^(l_z - max) O_z / sum 2^(l_z - max).  One thread per four
// channels of a row; pieces without a visible key (-inf) are not read.
template <int DH>
__global__ __launch_bounds__(kThreads) void kv_join_kernel(KvAttnArgs a) {
  const long long rows = (long long)a.s.n_tok * a.Hq;
  const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
  const long long row = i / (DH / 4);
  const int d = 4 * (int)(i % (DH / 4));
  if (row >= rows) return;
  const int tok = (int)(row / a.Hq);
  if (tok < seq_row(a.s, 0) || tok >= seq_row(a.s, a.s.n_seq)) return;   // of no sequence: left alone
  float m = -INFINITY;
  for (int z = 0; z < a.npieces; ++z) {
    const float l = a.part_lse[z * rows + row];
    m = l > m || l != l ? l : m;
  }
  float w = 0.0f;
  f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
  for (int z = 0; z < a.npieces; ++z) {
    const float l = a.part_lse[z * rows + row];
    if (l == -INFINITY) continue;
    const float c = l == m ? 1.0f : __builtin_amdgcn_exp2f(l - m);
    w += c;
    o += c * *reinterpret_cast<const f32x4*>(a.part_o + (z * rows + row) * DH + d);
  }
  const bool some = w != 0.0f;
  o *= some ? 1.0f / w : 0.0f;
  put4(a, row, DH, d, o);
  if (a.lse != nullptr && d == 0) a.lse[row] = some ? (m + __log2f(w)) * kLn2 : -INFINITY;
}

template <int DH, bool F8>
void launch_as(const KvAttnArgs& a, const KvAttnPlan& p, hipStream_t stream) {
  const dim3 grid(p.row_tiles, a.H, p.pieces);
  if (p.few_rows) hipLaunchKernelGGL((kv_rows_kernel<DH, F8>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((kv_tiles_kernel<DH, F8>), grid, dim3(kThreads), 0, stream, a);
  if (p.pieces > 1) {
    const long long threads = (long long)a.s.n_tok * a.Hq * (DH / 4);
    hipLaunchKernelGGL((kv_join_kernel<DH>), dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                       stream, a);
  }
}

}  // namespace

KvAttnPlan kv_attn_plan(long long n_tok, int n_seq, int g, int H, int dh, long long max_len, int window, int sinks,
                        int cus) {
  KvAttnPlan p{};
  const long long rows = n_tok * g, mean = (rows + n_seq - 1) / n_seq;
  p.few_rows = mean <= 2 * kRows;
  const int tm = p.few_rows ? kRows : kTileRows, tk = p.few_rows ? kRowKeys : kTileKeys;
  p.row_tiles = (int)(rows / tm + n_seq);
  p.pieces = 1;
  p.piece_tiles = 1;
  if (cus <= 0 || n_tok < 1) return p;
  const long long units = (long long)n_seq * ((mean + tm - 1) / tm) * H;
  long long keys = max_len;
  if (window > 0) keys = std::min(keys, (long long)window + (mean + g - 1) / g + sinks + 2 * tk);
  const long long nt = (keys + tk - 1) / tk;
  const long long least = p.few_rows ? 16 : 8;       // key tiles of a piece
  const long long want = (long long)cus * (p.few_rows ? 8 : 2) / std::max(units, 1ll);
  const long long most = std::min<long long>(std::min<long long>(want, kMaxPieces), (nt + least - 1) / least);
  if (most < 2) return p;
  p.piece_tiles = (int)((nt + most - 1) / most);
  p.pieces = (int)((nt + p.piece_tiles - 1) / p.piece_tiles);
  p.part_bytes = align_up((size_t)most * n_tok * H * g * dh * 4);
  p.bytes = p.part_bytes + align_up((size_t)most * n_tok * H * g * 4);
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
  a.part_lse = plan.pieces > 1 ? reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.part_bytes) : nullptr;
  a.Hq = Hq;
  a.H = c.H;
  a.g = Hq / c.H;
  a.pages = c.pages;
  a.page = c.page;
  a.causal = causal;
  a.window = window;
  a.sinks = window > 0 ? sinks : 0;
  a.npieces = plan.pieces;
  a.piece_tiles = plan.piece_tiles;
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
