// Attention of several query rows per sequence over the paged int4/int2 cache,
// with the exponential itself: the drafted nodes of a tree (turbo_attn_tree), or
// one row per query head over a choice of groups (turbo_attn_selected).
//
// For a row with query q and a visible token t,
//   x_t = sm_scale * q . K_t,   o = sum_t e^(x_t) V_t / sum_t e^(x_t),
// K_t, V_t the values the cache stands for: (code * s^int + z^int) * s for a
// cached group, code * s for the buffer, fp16 for a drafted node.  One pass over
// the tokens in tiles of 64 with the running maximum m and sum l of each row,
// everything in binary32 but the operands of the matrix instructions:
//  * K and V as fp16 integers code * s^int + z^int times a power of two (exact), q
//    as given: the products of Q K^T are exact, their sums binary32;
//  * the weights P, rounded to fp16 (relative 2^-11, as the output's own rounding).
// The scale of a tile's V goes into its weights, so that the products of all tiles
// add up in the accumulators with no pass over them in between: with e = log2 of the
// tile's scale (x in units of log2 from here on)
//   P_t = 2^(x_t + e - m + 7),  O += P V,  l += 2^-e sum_t P_t,  m ~ max (x_t + e),
// o = O / l.  m follows the maximum only when it is more than 8 behind (the row's
// sums are then rescaled), so 2^7 leaves P below 2^15 and terms down to 2^-21 of the
// row's largest in fp16's normal range.  l sums P before it is rounded.
//
// The tokens of the G query heads of a KV head are one matrix of G * T rows.  A
// wave takes 16 of them and a tile:
//   S^T = K q^T   (16x16x32 fp16 MFMA; A row m of block mb: token
//                  16 (m >> 2) + 4 mb + (m & 3) of the tile)
//   O^T += V^T P^T (A row m of block cb: channel 32 (cb >> 1) + 2 m + (cb & 1))
// With this order of tokens lane (n, g4) -- n = lane & 15 the query row, g4 =
// lane >> 4 -- holds the scores of the 16 tokens of page g4, which are the ones
// its operand of the second product needs: P never leaves the registers, and the
// row's m and l are the lane's own.  With this order of channels the lanes' codes of V
// are contiguous in every load, and a lane's outputs runs of 8 channels.
#include "turbo_common.h"
#include "stream_loads.h"
#include <algorithm>

namespace turbo {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
// q, the nodes' keys and values and o may lie at any fp16 boundary
typedef unsigned u4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u1_any __attribute__((aligned(2)));

struct RowsArgs {
  const unsigned short* q;   // fp16 [B][Hq][T][128]
  const unsigned short* kt;  // fp16 [B][Hkv][T][128] (null: no nodes)
  const unsigned short* vt;
  const unsigned long long* mask;  // [B][T][mwords]; null: node i sees 0 .. i
  int mwords;
  const int* tree_lens;      // [B]; null: T
  const int* sel;            // [B][Hkv][nsel] groups to attend; null: all
  int nsel;
  const uint8_t* pages;
  const int8_t* gmeta;       // [slots][Hkv][4][128]
  const float* gscale;       // [slots][Hkv][2]
  int npages, nslots;        // min(num_pages, INT_MAX), min(num_slots, INT_MAX)
  int page_bytes;
  unsigned long long int2_mask;
  const int* seq_lens;       // [B]
  const int* block_table;    // [B][4*max_groups]
  const int* group_table;    // [B][max_groups]
  int max_groups;
  int B, Hq, Hkv, G, T;
  float sm_log2e;            // sm_scale * log2(e)
  const int8_t* tk;          // Sec. 3.3 buffer (null: none)
  const int8_t* tv;
  const float* tscale;
  int ntiles_row;            // row tiles in the grid
  int nchunk;                // chunks in the grid
  int min_len;               // tiles of a chunk, at least
  float* ws;                 // [B][Hq][T][nchunk][132]: m, l, -, -, O[128]
  unsigned short* o;         // fp16 [B][Hq][T][128]
  float* lse;                // [B][Hq][T] or null
};

constexpr int kRowsWaves = 4;   // waves of a work-group, a tile each in turn
constexpr float kPShift = 7.0f;

// The tiles of sequence b: cached groups (or choices), the buffer, the nodes.
struct RowsSeq {
  int ng;      // cached groups
  int nt;      // buffered tokens
  int tl;      // nodes
  int nlist;   // tiles of cached groups
  int ntile;   // all tiles
  int len;     // tiles of a chunk
  int nparts;  // chunks
};

__device__ __forceinline__ RowsSeq rows_seq(const RowsArgs& a, int b) {
  RowsSeq s;
  const int len = a.seq_lens[b];
  s.ng = min(max(len / 64, 0), a.max_groups);
  s.nt = a.tk ? min(max(len - 64 * s.ng, 0), 63) : 0;
  s.tl = a.tree_lens ? min(max(a.tree_lens[b], 0), a.T) : a.T;
  s.nlist = a.sel ? a.nsel : s.ng;
  s.ntile = s.nlist + (s.nt > 0) + (a.kt ? (s.tl + 63) / 64 : 0);
  s.len = max(a.min_len, ceil_div(s.ntile, a.nchunk));
  s.nparts = ceil_div(s.ntile, s.len);
  return s;
}

// The work of a work-group; false past the last.  They go to the eight XCDs in turn:
// the row tiles of a chunk, which read the same codes, to one of them.  The first
// chunks of all heads come first, the second ones after them, so that the chunks that
// short sequences do not have lie together, not on some of the XCDs; the heads, whose
// bits and so whose work may differ, are rotated by the sequence.
__device__ __forceinline__ bool rows_place(const RowsArgs& a, int& b, int& kh, int& s, int& rt) {
  const unsigned span = 8u * a.ntiles_row;
  rt = (int)(blockIdx.x % span >> 3);
  const int u = (int)(blockIdx.x / span * 8 + (blockIdx.x & 7));
  s = u / (a.B * a.Hkv);
  const int bh = u - s * (a.B * a.Hkv);
  b = bh / a.Hkv;
  kh = (bh - b * a.Hkv + b) % a.Hkv;
  return s < a.nchunk;
}

__device__ __forceinline__ f4 mfma_h(u32x4_t a, u32x4_t b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a),
                                                __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

__device__ __forceinline__ unsigned h2_fma(unsigned a, unsigned b, unsigned c) {
  return __builtin_bit_cast(
      unsigned, __builtin_elementwise_fma(__builtin_bit_cast(h2, a), __builtin_bit_cast(h2, b),
                                          __builtin_bit_cast(h2, c)));
}
__device__ __forceinline__ unsigned h2_add(unsigned a, unsigned b) {
  return __builtin_bit_cast(unsigned, __builtin_bit_cast(h2, a) + __builtin_bit_cast(h2, b));
}
__device__ __forceinline__ unsigned h2_mul(unsigned a, unsigned b) {
  return __builtin_bit_cast(unsigned, __builtin_bit_cast(h2, a) * __builtin_bit_cast(h2, b));
}
__device__ __forceinline__ unsigned h2_of(float lo, float hi) {
  const h2 x = {(_Float16)lo, (_Float16)hi};
  return __builtin_bit_cast(unsigned, x);
}

// Codes to fp16.  A field of a half's low bits, masked, is the subnormal number
// field * 2^-24, and one fused multiply-add by a power of two times s^int and to
// z^int makes of it (code s + z) 2^-kDown, exactly: no conversion.  Pair i of a word
// (int4: nibbles i and i + 4; int2: fields i and i + 8) is brought to the lowest or
// second lowest field of its half, whose factors differ by 2^bits: a shift for every
// two pairs.  Exact, and s' finite, for the s^int this library writes (at most 16
// with 4 bits, 80 with 2).  9 instructions for 8 codes of 4 bits; by way of
// 1 + code / 16 it takes 12.
template <int BITS>
constexpr int kDown = BITS == 4 ? 13 : 15;

template <int BITS>
__device__ __forceinline__ unsigned code_pair(unsigned w, int i) {
  constexpr unsigned m = BITS == 4 ? 0x000f000fu : 0x00030003u;
  return (w >> (2 * BITS * (i >> 1))) & (i & 1 ? m << BITS : m);
}

// 2^e as fp16 in both halves.
constexpr unsigned h2_exp2(int e) {  // (subnormal below 2^-14)
  const unsigned h = e >= -14 ? (unsigned)(15 + e) << 10 : 1u << (24 + e);
  return h | h << 16;
}

// s^int and z^int of two channels (bytes at bits 0-7 and 16-23) as fp16 integers.
// (0x6400 | x is 1024 + x.)
__device__ __forceinline__ unsigned scale_h2(unsigned s) {
  return h2_add(s | 0x64006400u, 0xe400e400u);
}
__device__ __forceinline__ unsigned zero_h2(unsigned z) {
  return h2_add((z ^ 0x00800080u) | 0x64006400u, 0xe480e480u);
}
// Factors of pairs in the lowest (odd = 0) and second lowest field, and z 2^-kDown.
template <int BITS>
__device__ __forceinline__ unsigned scale_at(unsigned s, int odd) {
  return h2_mul(s, odd ? h2_exp2(24 - kDown<BITS> - BITS) : h2_exp2(24 - kDown<BITS>));
}
template <int BITS>
__device__ __forceinline__ unsigned zero_at(unsigned z) {
  return h2_mul(z, h2_exp2(-kDown<BITS>));
}
__device__ __forceinline__ unsigned h2_splat(unsigned x, int hi) {
  const h2 v = __builtin_bit_cast(h2, x);
  const h2 y = hi ? h2{v[1], v[1]} : h2{v[0], v[0]};
  return __builtin_bit_cast(unsigned, y);
}

// int8 pair (bytes at bits 0-7 and 16-23, high bits flipped) to fp16.
__device__ __forceinline__ unsigned int8_pair(unsigned x) {
  return h2_add(x | 0x64006400u, h2_of(-1152.0f, -1152.0f));
}

// Order of a tile's 32 channels of lane group g4 over the four k-steps: register jj
// of step ks holds channels 32 g4 + first(ks, jj) and that + dist.
enum { kOrd4 = 0, kOrd2 = 1, kOrdNat = 2 };
template <int ORD>
__device__ __forceinline__ int chan_lo(int ks, int jj) {
  return ORD == kOrd4 ? 8 * ks + jj : ORD == kOrd2 ? 16 * (ks >> 1) + 4 * (ks & 1) + jj : 8 * ks + 2 * jj;
}
template <int ORD>
constexpr int kChanDist = ORD == kOrd4 ? 4 : (ORD == kOrd2 ? 8 : 1);

// The wave's query rows as the B operand of S^T, in one of these orders.
template <int NT>
struct RowsQ {
  u32x4_t x[NT][4];
  long at[NT];  // row of q, o and lse; -1 past the last
  int node[NT];
};

template <int NT, int ORD>
__device__ __forceinline__ void load_q(const RowsArgs& a, RowsQ<NT>& Q) {
  const int g4 = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    unsigned raw[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u4_any x = {0, 0, 0, 0};
      if (Q.at[t] >= 0) x = reinterpret_cast<const u4_any*>(a.q + Q.at[t] * 128 + 32 * g4)[i];
      raw[4 * i] = x.x; raw[4 * i + 1] = x.y; raw[4 * i + 2] = x.z; raw[4 * i + 3] = x.w;
    }
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const int c = chan_lo<ORD>(ks, jj);
        if (ORD == kOrdNat) {
          Q.x[t][ks][jj] = raw[c >> 1];
        } else {
          const unsigned lo = raw[c >> 1], hi = raw[(c + kChanDist<ORD>) >> 1];
          Q.x[t][ks][jj] = __builtin_amdgcn_perm(hi, lo, c & 1 ? 0x07060302u : 0x05040100u);
        }
      }
  }
}

// Running state of the wave's rows: O^T (channel 32 e + 8 g4 + 2 r + hi in
// o[t][2 e + hi][r]), maximum (in units of log2) and this lane's part of the sum.
template <int NT>
struct RowsState {
  f4 o[NT][8];
  float m[NT], l[NT];
};

// Scores of a tile to weights.  S holds the products of row tile t, x = S * c2; ex
// and inv are log2 of the scale of the tile's V and its inverse; where MASKED, bit
// 4 mb + r of vis says whether token (mb, r) of the lane's page is visible.  Brings
// the state to the tile's maximum and returns P as the B operand of O^T: PAIR4 pairs
// tokens (8 ks + jj, + 4) of the page, else (4 ks + jj, + 8).
template <int NT, bool PAIR4, bool MASKED>
__device__ __forceinline__ void rows_softmax(RowsState<NT>& st, int t, f4 (&S)[4], float c2, float ex,
                                             float inv, unsigned vis, u32x4_t (&P)[2]) {
  if (MASKED) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = S[i >> 2][i & 3] * c2;
      S[i >> 2][i & 3] = (vis >> i) & 1u ? x : -INFINITY;
    }
    c2 = 1.0f;
  }
  // (plain maxima: a matrix result must not be read by inline asm, before which the
  // compiler inserts no wait states)
  float mx = S[0][0];
#pragma unroll
  for (int i = 1; i < 16; ++i) mx = fmaxf(mx, S[i >> 2][i & 3]);
  mx = __builtin_fmaf(max_xor32_nn(max_xor16_nn(mx)), c2, ex);  // (c2 >= 0)
  const float mo = st.m[t];
  const bool up = mx > mo + 8.0f;
  if (__any(up)) {
    const float mn = up ? mx : mo;
    // (a row that has seen nothing yet: its sums are zero)
    const float al = mo == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mo - mn);
    st.m[t] = mn;
    st.l[t] *= al;
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) st.o[t][cb] *= al;
  }
  const float off = st.m[t] == -INFINITY ? 0.0f : (kPShift + ex) - st.m[t];  // (all -inf: P = 0)
  float l[4] = {};
#pragma unroll
  for (int mb = 0; mb < 4; ++mb)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      S[mb][r] = __builtin_amdgcn_exp2f(MASKED ? S[mb][r] + off : __builtin_fmaf(S[mb][r], c2, off));
      l[r] += S[mb][r];
    }
  st.l[t] = __builtin_fmaf((l[0] + l[1]) + (l[2] + l[3]), inv, st.l[t]);
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int jj = 0; jj < 4; ++jj)
      P[ks][jj] = PAIR4 ? h2_of(S[2 * ks][jj], S[2 * ks + 1][jj]) : h2_of(S[ks][jj], S[ks + 2][jj]);
}

// log2 and inverse of the scale of a tile's V, brought to its operands.  Below 2^-60
// (zero, or a scale whose values all round to zero in fp16) it counts as 2^-60, which
// both functions and the sums stand.
__device__ __forceinline__ void value_scale(float sv, float up, float& ex, float& inv) {
  float s = sv * up;
  s = s < 0x1p-60f ? 0x1p-60f : s;  // (NaN stays)
  ex = __builtin_amdgcn_logf(s);
  inv = __builtin_amdgcn_rcpf(s);
}

// ---- a cached group ------------------------------------------------------------
// Table entries and scales of 64 tiles, lane i holding the i-th: one round of loads for
// 64 steps, and no step waits for a table entry before its codes can leave.
struct RowsTab {
  int pg[4];     // pages, 0 where there is nothing to attend
  int slot;      // -1 where there is nothing to attend
  float sk, sv;
};

// Lane i: the tile j + i * STEP of the list, attended below j1.
template <int STEP>
__device__ __forceinline__ void load_tab(const RowsArgs& a, int b, int kh, const RowsSeq& sq, int j,
                                         int j1, RowsTab& T) {
  j += (int)(threadIdx.x & 63) * STEP;
  bool ok = j < j1;
  int g = ok ? j : 0;
  if (a.sel) g = ok ? a.sel[((long)b * a.Hkv + kh) * a.nsel + j] : 0;
  ok = ok && g >= 0 && g < sq.ng;
  T.slot = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i) T.pg[i] = 0;
  T.sk = T.sv = 0.0f;
  if (ok) {
    const int* bt = a.block_table + ((long)b * a.max_groups + g) * 4;
    const int slot = a.group_table[(long)b * a.max_groups + g];
    int pg[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      pg[i] = bt[i];
      ok = ok && pg[i] >= 0 && pg[i] < a.npages;
    }
    if (ok && slot >= 0 && slot < a.nslots) {
      T.slot = slot;
#pragma unroll
      for (int i = 0; i < 4; ++i) T.pg[i] = pg[i];
      const float* gs = a.gscale + ((long)slot * a.Hkv + kh) * 2;
      T.sk = gs[0];
      T.sv = gs[1];
    }
  }
}

// Codes and metadata of a group.
template <int BITS>
struct RowsGroup {
  unsigned k[4][BITS];     // codes of token (m, mb), the lane's 32 channels
  unsigned v[8 * BITS / 2];  // codes of channels 32 e + 2 n and + 1, the lane's page
  uint2 ks, kz;            // s^int, z^int of the 8 channels that hold the lane's pair
  unsigned vs, vz;         // of channels 2 lane and + 1
};

// K and V of the i-th tile of T.  One with nothing to attend loads page 0 and slot 0,
// so that as many loads are in flight on every path.
__device__ __forceinline__ long tab_page(const RowsArgs& a, const RowsTab& T, int i, int p) {
  int pg[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) pg[k] = __builtin_amdgcn_readlane(T.pg[k], i);
  const int lo = p & 1 ? pg[1] : pg[0], hi = p & 1 ? pg[3] : pg[2];
  return (long)(p & 2 ? hi : lo) * a.page_bytes;
}
__device__ __forceinline__ const int8_t* tab_meta(const RowsArgs& a, const RowsTab& T, int i, int kh) {
  const int slot = max(__builtin_amdgcn_readlane(T.slot, i), 0);
  return a.gmeta + ((long)slot * a.Hkv + kh) * 512;
}

template <int BITS>
__device__ __forceinline__ void load_group_k(const RowsArgs& a, int kh, int head_off, const RowsTab& T,
                                             int i, RowsGroup<BITS>& x) {
  const int lane = threadIdx.x & 63, n = lane & 15, g4 = lane >> 4;
  const uint8_t* kp =
      a.pages + tab_page(a, T, i, n >> 2) + head_off + (n & 3) * 16 * BITS + 4 * BITS * g4;
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) {
    if constexpr (BITS == 4) {
      const u32x4_t w = load_nt4(kp + 4 * mb * 16 * BITS);
      x.k[mb][0] = w.x; x.k[mb][1] = w.y; x.k[mb][2] = w.z; x.k[mb][3] = w.w;
    } else {
      const u32x2_t w = load_nt2(kp + 4 * mb * 16 * BITS);
      x.k[mb][0] = w.x; x.k[mb][1] = w.y;
    }
  }
  // the lane converts pair (ks, jj) = (n >> 2, n & 3) of its channels
  constexpr int ORD = BITS == 4 ? kOrd4 : kOrd2;
  const int8_t* meta = tab_meta(a, T, i, kh) + 32 * g4 + (chan_lo<ORD>(n >> 2, n & 3) & ~3);
  x.ks = make_uint2(*reinterpret_cast<const unsigned*>(meta),
                    *reinterpret_cast<const unsigned*>(meta + kChanDist<ORD>));
  x.kz = make_uint2(*reinterpret_cast<const unsigned*>(meta + 128),
                    *reinterpret_cast<const unsigned*>(meta + 128 + kChanDist<ORD>));
}

template <int BITS>
__device__ __forceinline__ void load_group_v(const RowsArgs& a, int kh, int head_off, const RowsTab& T,
                                             int i, RowsGroup<BITS>& x) {
  const int lane = threadIdx.x & 63, n = lane & 15, g4 = lane >> 4;
  const uint8_t* vp = a.pages + tab_page(a, T, i, g4) + head_off + 256 * BITS + n * 4 * BITS;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (BITS == 4) {
      const u32x4_t w = load_nt4(vp + 256 * e);
      x.v[4 * e] = w.x; x.v[4 * e + 1] = w.y; x.v[4 * e + 2] = w.z; x.v[4 * e + 3] = w.w;
    } else {
      const u32x2_t w = load_nt2(vp + 128 * e);
      x.v[2 * e] = w.x; x.v[2 * e + 1] = w.y;
    }
  }
  const int8_t* meta = tab_meta(a, T, i, kh);
  x.vs = *reinterpret_cast<const unsigned short*>(meta + 256 + 2 * lane);
  x.vz = *reinterpret_cast<const unsigned short*>(meta + 384 + 2 * lane);
}

// S^T = K q^T of a group.
template <int BITS, int NT>
__device__ __forceinline__ void group_scores(const RowsGroup<BITS>& x, const RowsQ<NT>& Q,
                                             f4 (&S)[NT][4], uint2* szk) {
  const int lane = threadIdx.x & 63, n = lane & 15, g4 = lane >> 4;
  // factors and zero points of the lane group's channel pairs, exchanged through LDS
  {
    const int sh = 8 * (n & 3);
    const unsigned s = scale_h2(((x.ks.x >> sh) & 0xffu) | (((x.ks.y >> sh) & 0xffu) << 16));
    const unsigned z = zero_h2(((x.kz.x >> sh) & 0xffu) | (((x.kz.y >> sh) & 0xffu) << 16));
    wave_sync();
    szk[lane] = make_uint2(n & 1 ? scale_at<BITS>(s, 1) : scale_at<BITS>(s, 0), zero_at<BITS>(z));
    wave_sync();
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int mb = 0; mb < 4; ++mb) S[t][mb] = f4{0, 0, 0, 0};
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    uint2 sz[4];
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) sz[jj] = szk[16 * g4 + 4 * ks + jj];
#pragma unroll
    for (int mb = 0; mb < 4; ++mb) {
      u32x4_t A;
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const unsigned c = BITS == 4 ? code_pair<BITS>(x.k[mb][ks], jj)
                                     : code_pair<BITS>(x.k[mb][ks >> 1], 4 * (ks & 1) + jj);
        A[jj] = h2_fma(c, sz[jj].x, sz[jj].y);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) S[t][mb] = mfma_h(A, Q.x[t][ks], S[t][mb]);
    }
  }
}

// O^T += V^T P^T of a group.
template <int BITS, int NT>
__device__ __forceinline__ void group_values(const RowsGroup<BITS>& x, const u32x4_t (&P)[NT][2],
                                             RowsState<NT>& st, uint4* szv) {
  const int lane = threadIdx.x & 63, n = lane & 15;
  {  // factors and zero points of channel pairs, one a lane, exchanged through LDS
    const unsigned s = scale_h2(__builtin_amdgcn_perm(0u, x.vs, 0x0c010c00u));
    const unsigned z = zero_h2(__builtin_amdgcn_perm(0u, x.vz, 0x0c010c00u));
    wave_sync();
    szv[lane] = make_uint4(scale_at<BITS>(s, 0), scale_at<BITS>(s, 1), zero_at<BITS>(z), 0u);
    wave_sync();
  }
#pragma unroll
  for (int c2 = 0; c2 < 4; ++c2) {  // channels 32 c2 + 2 n and + 1
    const uint4 sz = szv[16 * c2 + n];
    const unsigned s0 = sz.x, s1 = sz.y, zd = sz.z;
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
      const int cb = 2 * c2 + hi;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        u32x4_t A;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          const unsigned c = BITS == 4 ? code_pair<BITS>(x.v[2 * cb + ks], jj)
                                       : code_pair<BITS>(x.v[cb], 4 * ks + jj);
          A[jj] = h2_fma(c, h2_splat(jj & 1 ? s1 : s0, hi), h2_splat(zd, hi));
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) st.o[t][cb] = mfma_h(A, P[t][ks], st.o[t][cb]);
      }
    }
  }
}

// ---- the int8 buffer ---------------------------------------------------------------
// Q in order kOrd4.
template <int NT>
__device__ __forceinline__ void step_buffer(const RowsArgs& a, long u, int nt, const RowsQ<NT>& Q,
                                            RowsState<NT>& st) {
  const int lane = threadIdx.x & 63, n = lane & 15, g4 = lane >> 4;
  f4 S[NT][4];
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) {
    const int8_t* kr = a.tk + (u * 64 + 16 * (n >> 2) + 4 * mb + (n & 3)) * 128 + 32 * g4;
    unsigned w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = reinterpret_cast<const unsigned*>(kr)[i] ^ 0x80808080u;
#pragma unroll
    for (int t = 0; t < NT; ++t) S[t][mb] = f4{0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      u32x4_t A;
#pragma unroll
      for (int jj = 0; jj < 4; ++jj)
        A[jj] = int8_pair(__builtin_amdgcn_perm(w[2 * ks + 1], w[2 * ks], 0x0c040c00u + 0x00010001u * jj));
#pragma unroll
      for (int t = 0; t < NT; ++t) S[t][mb] = mfma_h(A, Q.x[t][ks], S[t][mb]);
    }
  }
  const float sk = a.tscale[2 * u];
  float ex, inv;
  value_scale(a.tscale[2 * u + 1], 1.0f, ex, inv);
  const int live = min(max(nt - 16 * g4, 0), 16);
  u32x4_t P[NT][2];
#pragma unroll
  for (int t = 0; t < NT; ++t)
    rows_softmax<NT, true, true>(st, t, S[t], sk * a.sm_log2e, ex, inv, (1u << live) - 1u, P[t]);
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) {
    const int8_t* vr = a.tv + (u * 128 + 32 * (cb >> 1) + 2 * n + (cb & 1)) * 64 + 16 * g4;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const unsigned w0 = reinterpret_cast<const unsigned*>(vr)[2 * ks] ^ 0x80808080u;
      const unsigned w1 = reinterpret_cast<const unsigned*>(vr)[2 * ks + 1] ^ 0x80808080u;
      u32x4_t A;
#pragma unroll
      for (int jj = 0; jj < 4; ++jj)
        A[jj] = int8_pair(__builtin_amdgcn_perm(w1, w0, 0x0c040c00u + 0x00010001u * jj));
#pragma unroll
      for (int t = 0; t < NT; ++t) st.o[t][cb] = mfma_h(A, P[t][ks], st.o[t][cb]);
    }
  }
}

// ---- 64 drafted nodes ------------------------------------------------------------
__device__ __forceinline__ bool nonfinite_h2(unsigned x) {
  return (x & 0x7c00u) == 0x7c00u || (x & 0x7c000000u) == 0x7c000000u;
}

// Which of the lane's 16 nodes of tile j a row (node `node` of the tree) sees.
__device__ __forceinline__ unsigned nodes_visible(const RowsArgs& a, int b, int j, int tl, long at,
                                                  int node) {
  const int g4 = (threadIdx.x & 63) >> 4;
  const int live = min(max(tl - 64 * j - 16 * g4, 0), 16);
  unsigned long long w = 0;
  if (at >= 0) {
    if (a.mask) {
      w = a.mask[((long)b * a.T + node) * a.mwords + j];
    } else {
      const int c = node + 1 - 64 * j;  // nodes of this tile up to the row's own
      w = c >= 64 ? ~0ull : (c > 0 ? (1ull << c) - 1ull : 0ull);
    }
  }
  return (unsigned)(w >> (16 * g4)) & ((1u << live) - 1u);
}

// Adds the values of tile j (rows of vb) that are not finite to the rows that see
// their node.
template <int NT, bool PAIR4>
__device__ void nodes_nonfinite(const RowsArgs& a, const unsigned short* vb, int j, int tl,
                                const u32x4_t (&P)[NT][2], const unsigned (&vis)[NT],
                                RowsState<NT>& st) {
  const int lane = threadIdx.x & 63, n = lane & 15, g4 = lane >> 4;
  const int cnt = min(tl - 64 * j, 64);
  for (int i = 0; i < cnt; ++i) {
    const unsigned short* vr = vb + (64L * j + i) * 128 + 8 * g4;
    const int from = 16 * (i >> 4) + n;  // lane that holds the row's p of token i
    // register (ks, jj) and half of token i & 15 of the page
    const int tok = i & 15;
    const int reg = PAIR4 ? (tok >> 3) * 4 + (tok & 3) : tok & 7;
    const bool high = PAIR4 ? tok & 4 : tok & 8;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      unsigned w = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) w = reg == k ? P[t][k >> 2][k & 3] : w;
      if (high) w >>= 16;
      const unsigned pw = __shfl((int)(w & 0xffffu), from);
      const unsigned seen = __shfl((int)vis[t], from) >> tok;
      const float p = (float)__builtin_bit_cast(_Float16, (unsigned short)pw);
      if (!(seen & 1u)) continue;
#pragma unroll
      for (int cb = 0; cb < 8; ++cb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const unsigned short x = vr[32 * (cb >> 1) + 2 * r + (cb & 1)];
          if ((x & 0x7c00u) == 0x7c00u) st.o[t][cb][r] += p * (float)__builtin_bit_cast(_Float16, x);
        }
    }
  }
}

// Nodes 64 j .. of the sequence's tl; Q in order kOrdNat.  A value that is not
// finite must not reach the rows that do not see its node (0 * NaN): it takes no
// part in the products and is added to the rows that do afterwards.
template <int NT>
__device__ __forceinline__ void step_nodes(const RowsArgs& a, int b, long u, int j, int tl,
                                           const RowsQ<NT>& Q, RowsState<NT>& st) {
  const int lane = threadIdx.x & 63, n = lane & 15, g4 = lane >> 4;
  const unsigned short* kb = a.kt + u * a.T * 128;
  const unsigned short* vb = a.vt + u * a.T * 128;
  f4 S[NT][4];
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) {
    const int tok = 64 * j + 16 * (n >> 2) + 4 * mb + (n & 3);
#pragma unroll
    for (int t = 0; t < NT; ++t) S[t][mb] = f4{0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      u4_any A = {0, 0, 0, 0};
      if (tok < tl) A = reinterpret_cast<const u4_any*>(kb + (long)tok * 128 + 32 * g4)[ks];
#pragma unroll
      for (int t = 0; t < NT; ++t)
        S[t][mb] = mfma_h(u32x4_t{A.x, A.y, A.z, A.w}, Q.x[t][ks], S[t][mb]);
    }
  }
  u32x4_t P[NT][2];
  unsigned vis[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    vis[t] = nodes_visible(a, b, j, tl, Q.at[t], Q.node[t]);
    rows_softmax<NT, true, true>(st, t, S[t], a.sm_log2e, 0.0f, 1.0f, vis[t], P[t]);
  }
  bool bad = false;
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    unsigned v[8][4];  // token 8 ks + i of the page, channels 32 e + 2 n and + 1
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int tok = 64 * j + 16 * g4 + 8 * ks + i;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[i][e] = 0u;
        if (tok < tl) v[i][e] = *reinterpret_cast<const u1_any*>(vb + (long)tok * 128 + 32 * e + 2 * n);
        bad = bad || nonfinite_h2(v[i][e]);
      }
    }
    if (__any(bad)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if ((v[i][e] & 0x7c00u) == 0x7c00u) v[i][e] &= 0xffff0000u;
          if ((v[i][e] & 0x7c000000u) == 0x7c000000u) v[i][e] &= 0xffffu;
        }
    }
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) {
      u32x4_t A;
#pragma unroll
      for (int jj = 0; jj < 4; ++jj)
        A[jj] = __builtin_amdgcn_perm(v[jj + 4][cb >> 1], v[jj][cb >> 1],
                                      cb & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int t = 0; t < NT; ++t) st.o[t][cb] = mfma_h(A, P[t][ks], st.o[t][cb]);
    }
  }
  if (__any(bad)) nodes_nonfinite<NT, true>(a, vb, j, tl, P, vis, st);
}

// Row `at` of o and lse from its merged state (8 channels from c0).
__device__ __forceinline__ void rows_store(const RowsArgs& a, long at, int c0, float m, float l,
                                           const float (&o)[8]) {
  const bool none = l == 0.0f;  // no visible token
  const float inv = none ? 0.0f : 1.0f / l;
  u4_any y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = h2_of(o[2 * e] * inv, o[2 * e + 1] * inv);
  *reinterpret_cast<u4_any*>(a.o + at * 128 + c0) = y;
  constexpr float kLn2 = 0x1.62e430p-1f;
  if (a.lse && c0 == 0) a.lse[at] = none ? -INFINITY : (m + (__builtin_log2f(l) - kPShift)) * kLn2;
}

// (m, l, o) and another state of the same row.
__device__ __forceinline__ void rows_join(float& m, float& l, float (&o)[8], float pm, float pl,
                                          const float (&v)[8]) {
  const float mn = fmaxf(m, pm);
  const float f = m == mn ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
  const float g = pm == mn ? 1.0f : __builtin_amdgcn_exp2f(pm - mn);
  m = mn;
  l = __builtin_fmaf(g, pl, f * l);
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = __builtin_fmaf(g, v[e], f * o[e]);
}

// ---- few rows ----------------------------------------------------------------------
// A wave takes a tile with all its work-group's rows, the four waves the tiles of a chunk
// in turn.  64 x 8190 tokens, 40/10 heads, int4 and int2: 32 groups, 4 rows, 36 us, 4.0
// TB/s; all groups, 20 rows, 156 us, 3.6 TB/s, bound by vector issue (590 instructions a
// tile) and, at three and two waves per SIMD, by the wait for the codes.
constexpr int kRowsLds = 132;  // floats of a row's state in LDS

template <int BITS, int NT>
__device__ __forceinline__ void rows_tiles(const RowsArgs& a, int b, int kh, int head_off,
                                           const RowsSeq& sq, int j0, int j1, RowsQ<NT>& Q,
                                           RowsState<NT>& st, uint2* szk, uint4* szv) {
  const int w = threadIdx.x >> 6;
  const long u = (long)b * a.Hkv + kh;
  int j = j0 + w;
  const int je = min(j1, sq.nlist);
  if (j < je) {
    load_q<NT, BITS == 4 ? kOrd4 : kOrd2>(a, Q);
    const int cnt = ceil_div(je - j, kRowsWaves);
    RowsTab T;
    load_tab<kRowsWaves>(a, b, kh, sq, j, je, T);
    RowsGroup<BITS> x;
    load_group_k<BITS>(a, kh, head_off, T, 0, x);
    load_group_v<BITS>(a, kh, head_off, T, 0, x);
    // each half's next codes are requested as soon as its registers are free
    for (int i = 0; i < cnt; ++i) {
      const int at = i & 63, next = (i + 1) & 63;
      const bool live = __builtin_amdgcn_readlane(T.slot, at) >= 0;
      const float sk = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(T.sk), at));
      const float sv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(T.sv), at));
      if (next == 0) load_tab<kRowsWaves>(a, b, kh, sq, j + kRowsWaves * (i + 1), je, T);
      f4 S[NT][4];
      group_scores<BITS, NT>(x, Q, S, szk);
      load_group_k<BITS>(a, kh, head_off, T, next, x);
      if (live) {
        constexpr float up = 1 << kDown<BITS>;
        float ex, inv;
        value_scale(sv, up, ex, inv);
        u32x4_t P[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
          rows_softmax<NT, BITS == 4, false>(st, t, S[t], sk * (a.sm_log2e * up), ex, inv, 0, P[t]);
        group_values<BITS, NT>(x, P, st, szv);
      }
      load_group_v<BITS>(a, kh, head_off, T, next, x);
    }
    j += kRowsWaves * cnt;
  }
  if (j < j1 && j == sq.nlist && sq.nt > 0) {
    load_q<NT, kOrd4>(a, Q);
    step_buffer<NT>(a, u, sq.nt, Q, st);
    j += kRowsWaves;
  }
  if (j < j1) {
    load_q<NT, kOrdNat>(a, Q);
    for (; j < j1; j += kRowsWaves)
      step_nodes<NT>(a, b, u, j - sq.nlist - (sq.nt > 0), sq.tl, Q, st);
  }
}

template <int NT>
__global__ __launch_bounds__(64 * kRowsWaves) void k_attn_rows(RowsArgs a) {
  __shared__ __attribute__((aligned(16))) float part[kRowsWaves][16][kRowsLds];
  __shared__ uint2 szk[kRowsWaves][64];
  __shared__ uint4 szv[kRowsWaves][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, g4 = lane >> 4;
  int b, kh, s, rt;
  if (!rows_place(a, b, kh, s, rt)) return;
  const RowsSeq sq = rows_seq(a, b);
  const int base = 16 * NT * rt, rows = a.G * sq.tl;
  if (base >= rows || s >= max(sq.nparts, 1)) return;
  RowsQ<NT> Q;
  RowsState<NT> st;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = base + 16 * t + n;
    const int h = row / sq.tl;
    Q.node[t] = row - h * sq.tl;
    Q.at[t] = row < rows ? ((long)b * a.Hq + kh * a.G + h) * a.T + Q.node[t] : -1;
    st.m[t] = -INFINITY;
    st.l[t] = 0.0f;
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) st.o[t][cb] = f4{0, 0, 0, 0};
  }
  const int head_off = 512 * (4 * kh - 2 * __popcll(a.int2_mask & ((1ull << kh) - 1ull)));
  const int j0 = s * sq.len, j1 = min(j0 + sq.len, sq.ntile);
  if ((a.int2_mask >> kh) & 1ull)
    rows_tiles<2, NT>(a, b, kh, head_off, sq, j0, j1, Q, st, szk[w], szv[w]);
  else
    rows_tiles<4, NT>(a, b, kh, head_off, sq, j0, j1, Q, st, szk[w], szv[w]);
  // the waves' states to LDS, and their merge: 16 lanes a row
  const int row = threadIdx.x >> 4, c0 = 8 * (threadIdx.x & 15);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float l = add_xor32(st.l[t] + __shfl_xor(st.l[t], 16));
    float* p = part[w][n];
    if (t > 0) __syncthreads();
    if (g4 == 0) *reinterpret_cast<float2*>(p) = make_float2(st.m[t], l);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f4 x = st.o[t][2 * e], y = st.o[t][2 * e + 1];
      float* d = p + 4 + 32 * e + 8 * g4;
      *reinterpret_cast<f4*>(d) = f4{x[0], y[0], x[1], y[1]};
      *reinterpret_cast<f4*>(d + 4) = f4{x[2], y[2], x[3], y[3]};
    }
    __syncthreads();
    const int at_row = base + 16 * t + row;
    if (at_row >= rows) continue;
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kRowsWaves; ++i) m = fmaxf(m, part[i][row][0]);
    float ls = 0.0f, o[8] = {};
#pragma unroll
    for (int i = 0; i < kRowsWaves; ++i) {
      const float* q = part[i][row];
      const float f = q[0] == m ? 1.0f : __builtin_amdgcn_exp2f(q[0] - m);
      ls = __builtin_fmaf(f, q[1], ls);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = __builtin_fmaf(f, q[4 + c0 + e], o[e]);
    }
    const int h = at_row / sq.tl;
    const long at = ((long)b * a.Hq + kh * a.G + h) * a.T + (at_row - h * sq.tl);
    if (sq.nparts <= 1) {
      rows_store(a, at, c0, m, ls, o);
    } else {
      float* q = a.ws + (at * a.nchunk + s) * kWsStride;
      *reinterpret_cast<float4*>(q + kWsO + c0) = make_float4(o[0], o[1], o[2], o[3]);
      *reinterpret_cast<float4*>(q + kWsO + c0 + 4) = make_float4(o[4], o[5], o[6], o[7]);
      if (c0 == 0) *reinterpret_cast<float2*>(q) = make_float2(m, ls);
    }
  }
}

// ---- many rows: tiles expanded once per work-group -------------------------------
// With T * G rows per KV head the expansion of the codes, two thirds of a tile's vector
// instructions for 16 rows, is shared: the NW waves of a work-group take 32 rows each,
// expand their part of the next tile into LDS, in the order in which its lanes hold the
// operands, and read all of this one.  Two buffers, one barrier a tile.  2 x 32/8 heads,
// 16384 tokens, 256 nodes: 158 us, 884 TFLOP/s, with eight waves (four: 5 % more, but
// less of a ragged batch's last tile is empty); each wave by itself, 216.  The vector
// units are busy 55 % of the time and the matrix cores 36 %.
template <int NW>
constexpr int kWideRows = 32 * NW;

struct WideTile {
  u32x4_t k[4][4][64];  // [ks][mb][lane]
  u32x4_t v[8][2][64];  // [cb][ks][lane]
};

// What a wave expands of a tile: of K, m-block w & 3, all four k-steps (NW = 4) or two
// of them; of V, channels 32 w + 2 n and + 1, or one of those of w >> 1.
template <int BITS, int NW>
struct WideRaw {
  static constexpr int kWords = BITS * 4 / NW;
  unsigned k[kWords], v[kWords];
  uint2 ks, kz;
  unsigned vs, vz;  // s^int, z^int of the channels in bits 0-7 (and 8-15)
};

template <int WORDS>
__device__ __forceinline__ void load_words(const uint8_t* p, unsigned (&x)[WORDS]) {
  if constexpr (WORDS == 4) {
    const uint4 c = *reinterpret_cast<const uint4*>(p);
    x[0] = c.x; x[1] = c.y; x[2] = c.z; x[3] = c.w;
  } else if constexpr (WORDS == 2) {
    const uint2 c = *reinterpret_cast<const uint2*>(p);
    x[0] = c.x; x[1] = c.y;
  } else {
    x[0] = *reinterpret_cast<const unsigned*>(p);
  }
}

template <int BITS, int NW>
__device__ __forceinline__ void wide_load(const RowsArgs& a, int kh, int head_off, const RowsTab& T,
                                          int i, WideRaw<BITS, NW>& x) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, g4 = lane >> 4;
  load_words(a.pages + tab_page(a, T, i, n >> 2) + head_off + (4 * (w & 3) + (n & 3)) * 16 * BITS +
                 4 * BITS * g4 + 2 * BITS * (w >> 2),
             x.k);
  load_words(a.pages + tab_page(a, T, i, g4) + head_off + 256 * BITS +
                 (NW == 4 ? (32 * w + 2 * n) : (32 * (w >> 1) + 2 * n + (w & 1))) * 2 * BITS,
             x.v);
  constexpr int ORD = BITS == 4 ? kOrd4 : kOrd2;
  const int8_t* meta = tab_meta(a, T, i, kh);
  const int8_t* mk = meta + 32 * g4 + (chan_lo<ORD>(n >> 2, n & 3) & ~3);
  x.ks = make_uint2(*reinterpret_cast<const unsigned*>(mk),
                    *reinterpret_cast<const unsigned*>(mk + kChanDist<ORD>));
  x.kz = make_uint2(*reinterpret_cast<const unsigned*>(mk + 128),
                    *reinterpret_cast<const unsigned*>(mk + 128 + kChanDist<ORD>));
  if constexpr (NW == 4) {
    x.vs = *reinterpret_cast<const unsigned short*>(meta + 256 + 32 * w + 2 * n);
    x.vz = *reinterpret_cast<const unsigned short*>(meta + 384 + 32 * w + 2 * n);
  } else {
    x.vs = *reinterpret_cast<const unsigned char*>(meta + 256 + 32 * (w >> 1) + 2 * n + (w & 1));
    x.vz = *reinterpret_cast<const unsigned char*>(meta + 384 + 32 * (w >> 1) + 2 * n + (w & 1));
  }
}

template <int BITS, int NW>
__device__ __forceinline__ void wide_expand(const WideRaw<BITS, NW>& x, WideTile& d, uint2* szk) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, g4 = lane >> 4;
  {
    const int sh = 8 * (n & 3);
    const unsigned s = scale_h2(((x.ks.x >> sh) & 0xffu) | (((x.ks.y >> sh) & 0xffu) << 16));
    const unsigned z = zero_h2(((x.kz.x >> sh) & 0xffu) | (((x.kz.y >> sh) & 0xffu) << 16));
    wave_sync();
    szk[lane] = make_uint2(n & 1 ? scale_at<BITS>(s, 1) : scale_at<BITS>(s, 0), zero_at<BITS>(z));
    wave_sync();
  }
  const int k0 = NW == 4 ? 0 : 2 * (w >> 2);
#pragma unroll
  for (int kk = 0; kk < 16 / NW; ++kk) {
    u32x4_t A;
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      const uint2 sz = szk[16 * g4 + 4 * (k0 + kk) + jj];
      const unsigned c = BITS == 4 ? code_pair<BITS>(x.k[kk], jj)
                                   : code_pair<BITS>(x.k[kk >> 1], 4 * (kk & 1) + jj);
      A[jj] = h2_fma(c, sz.x, sz.y);
    }
    d.k[k0 + kk][w & 3][lane] = A;
  }
  const unsigned pick = NW == 4 ? 0x0c010c00u : 0x0c000c00u;
  const unsigned s = scale_h2(__builtin_amdgcn_perm(0u, x.vs, pick));
  const unsigned z = zero_h2(__builtin_amdgcn_perm(0u, x.vz, pick));
  const unsigned s0 = scale_at<BITS>(s, 0), s1 = scale_at<BITS>(s, 1), zd = zero_at<BITS>(z);
#pragma unroll
  for (int hi = 0; hi < 8 / NW; ++hi)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      u32x4_t A;
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const unsigned c = BITS == 4 ? code_pair<BITS>(x.v[2 * hi + ks], jj)
                                     : code_pair<BITS>(x.v[hi], 4 * ks + jj);
        A[jj] = h2_fma(c, h2_splat(jj & 1 ? s1 : s0, hi), h2_splat(zd, hi));
      }
      d.v[8 / NW * w + hi][ks][lane] = A;
    }
}

// The buffer's 64 rows (those past the last are masked), as the codes of the head's
// groups are ordered.
template <int BITS>
__device__ __forceinline__ void wide_buffer(const RowsArgs& a, long u, WideTile& d) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, g4 = lane >> 4;
  constexpr int ORD = BITS == 4 ? kOrd4 : kOrd2;
  const int8_t* kr = a.tk + (u * 64 + 16 * (n >> 2) + 4 * w + (n & 3)) * 128 + 32 * g4;
  unsigned kw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) kw[i] = reinterpret_cast<const unsigned*>(kr)[i] ^ 0x80808080u;
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    u32x4_t A;
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      const int c = chan_lo<ORD>(ks, jj), e = c + kChanDist<ORD>;
      A[jj] = int8_pair(__builtin_amdgcn_perm(kw[e >> 2], kw[c >> 2], 0x0c040c00u + 0x00010001u * (c & 3)));
    }
    d.k[ks][w][lane] = A;
  }
#pragma unroll
  for (int hi = 0; hi < 2; ++hi) {
    const int8_t* vr = a.tv + (u * 128 + 32 * w + 2 * n + hi) * 64 + 16 * g4;
    unsigned vw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) vw[i] = reinterpret_cast<const unsigned*>(vr)[i] ^ 0x80808080u;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      u32x4_t A;
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const int lo = BITS == 4 ? 2 * ks : ks, up = BITS == 4 ? 2 * ks + 1 : ks + 2;
        A[jj] = int8_pair(__builtin_amdgcn_perm(vw[up], vw[lo], 0x0c040c00u + 0x00010001u * jj));
      }
      d.v[2 * w + hi][ks][lane] = A;
    }
  }
}

// Nodes 64 j ..; returns whether a value was not finite (it is zero in the tile).
template <int BITS>
__device__ __forceinline__ bool wide_nodes(const RowsArgs& a, long u, int j, int tl, WideTile& d) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, g4 = lane >> 4;
  constexpr int ORD = BITS == 4 ? kOrd4 : kOrd2;
  const int tok = 64 * j + 16 * (n >> 2) + 4 * w + (n & 3);
  unsigned raw[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u4_any x = {0, 0, 0, 0};
    if (tok < tl) x = reinterpret_cast<const u4_any*>(a.kt + (u * a.T + tok) * 128 + 32 * g4)[i];
    raw[4 * i] = x.x; raw[4 * i + 1] = x.y; raw[4 * i + 2] = x.z; raw[4 * i + 3] = x.w;
  }
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    u32x4_t A;
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      const int c = chan_lo<ORD>(ks, jj);
      A[jj] = __builtin_amdgcn_perm(raw[(c + kChanDist<ORD>) >> 1], raw[c >> 1],
                                    c & 1 ? 0x07060302u : 0x05040100u);
    }
    d.k[ks][w][lane] = A;
  }
  unsigned v[16];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int t = 64 * j + 16 * g4 + i;
    v[i] = t < tl ? *reinterpret_cast<const u1_any*>(a.vt + (u * a.T + t) * 128 + 32 * w + 2 * n) : 0u;
    bad = bad || nonfinite_h2(v[i]);
    if ((v[i] & 0x7c00u) == 0x7c00u) v[i] &= 0xffff0000u;
    if ((v[i] & 0x7c000000u) == 0x7c000000u) v[i] &= 0xffffu;
  }
#pragma unroll
  for (int hi = 0; hi < 2; ++hi)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      u32x4_t A;
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const int lo = BITS == 4 ? 8 * ks + jj : 4 * ks + jj, up = lo + (BITS == 4 ? 4 : 8);
        A[jj] = __builtin_amdgcn_perm(v[up], v[lo], hi ? 0x07060302u : 0x05040100u);
      }
      d.v[2 * w + hi][ks][lane] = A;
    }
  return __any(bad);
}

template <int NW>
struct WideLds {
  WideTile tile[2];
  uint2 szk[NW][64];
  int bad[4];  // a wave met a node's value that is not finite
};

// Order of a block of 16 fragment reads from LDS and the 32 matrix instructions they
// feed: four reads ahead of every eight instructions (128 cycles, about a read's
// latency).  Left alone, the compiler reads each fragment right before its use.
__device__ __forceinline__ void wide_order() {
  __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, 8, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, 8, 0);
}

// S^T = K q^T and O^T += V^T P^T of the tile in LDS.
__device__ __forceinline__ void wide_scores(const WideTile& d, const RowsQ<2>& Q, f4 (&S)[2][4]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int mb = 0; mb < 4; ++mb) S[t][mb] = f4{0, 0, 0, 0};
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int mb = 0; mb < 4; ++mb) {
      const u32x4_t A = d.k[ks][mb][lane];
#pragma unroll
      for (int t = 0; t < 2; ++t) S[t][mb] = mfma_h(A, Q.x[t][ks], S[t][mb]);
    }
  wide_order();
}
__device__ __forceinline__ void wide_values(const WideTile& d, const u32x4_t (&P)[2][2],
                                            RowsState<2>& st) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int cb = 0; cb < 8; ++cb)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const u32x4_t A = d.v[cb][ks][lane];
#pragma unroll
      for (int t = 0; t < 2; ++t) st.o[t][cb] = mfma_h(A, P[t][ks], st.o[t][cb]);
    }
  wide_order();
}

template <int BITS, int NW>
__device__ __forceinline__ void wide_tiles(const RowsArgs& a, int b, int kh, int head_off,
                                           const RowsSeq& sq, int j0, int j1, bool work, RowsQ<2>& Q,
                                           RowsState<2>& st, WideLds<NW>& L) {
  const int w = threadIdx.x >> 6;
  const long u = (long)b * a.Hkv + kh;
  const int je = min(j1, sq.nlist);
  load_q<2, BITS == 4 ? kOrd4 : kOrd2>(a, Q);
  if (j0 < je) {  // cached groups
    const int cnt = je - j0;
    RowsTab T;
    load_tab<1>(a, b, kh, sq, j0, je, T);
    WideRaw<BITS, NW> raw;
    wide_load<BITS, NW>(a, kh, head_off, T, 0, raw);
    float sk = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(T.sk), 0));
    float sv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(T.sv), 0));
    bool live = __builtin_amdgcn_readlane(T.slot, 0) >= 0;
    wide_expand<BITS, NW>(raw, L.tile[0], L.szk[w]);
    wide_load<BITS, NW>(a, kh, head_off, T, 1, raw);
    for (int i = 0; i < cnt; ++i) {
      __syncthreads();
      const float ski = sk, svi = sv;
      const bool livei = live;
      // the next tile to the other buffer, and its successor's codes requested (past
      // the end: page 0 and slot 0, expanded to no use)
      const int at = (i + 1) & 63;
      sk = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(T.sk), at));
      sv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(T.sv), at));
      live = __builtin_amdgcn_readlane(T.slot, at) >= 0;
      if (at == 63) load_tab<1>(a, b, kh, sq, j0 + i + 2, je, T);
      wide_expand<BITS, NW>(raw, L.tile[(i + 1) & 1], L.szk[w]);
      wide_load<BITS, NW>(a, kh, head_off, T, (i + 2) & 63, raw);
      if (!work || !livei) continue;
      f4 S[2][4];
      wide_scores(L.tile[i & 1], Q, S);
      constexpr float up = 1 << kDown<BITS>;
      float ex, inv;
      value_scale(svi, up, ex, inv);
      u32x4_t P[2][2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
        rows_softmax<2, BITS == 4, false>(st, t, S[t], ski * (a.sm_log2e * up), ex, inv, 0, P[t]);
      wide_values(L.tile[i & 1], P, st);
    }
  }
  // the buffer and the nodes
  for (int j = max(je, j0); j < j1; ++j) {
    const bool buffer = j == sq.nlist && sq.nt > 0;
    const int node = j - sq.nlist - (sq.nt > 0);
    __syncthreads();
    if (w < 4) {
      if (buffer) {
        wide_buffer<BITS>(a, u, L.tile[0]);
      } else {
        const bool bad = wide_nodes<BITS>(a, u, node, sq.tl, L.tile[0]);
        if ((threadIdx.x & 63) == 0) L.bad[w] = bad;
      }
    }
    __syncthreads();
    if (!work) continue;
    f4 S[2][4];
    wide_scores(L.tile[0], Q, S);
    float c2 = a.sm_log2e, ex = 0.0f, inv = 1.0f;
    if (buffer) {
      c2 *= a.tscale[2 * u];
      value_scale(a.tscale[2 * u + 1], 1.0f, ex, inv);
    }
    u32x4_t P[2][2];
    unsigned vis[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int g4 = (threadIdx.x & 63) >> 4;
      vis[t] = buffer ? (1u << min(max(sq.nt - 16 * g4, 0), 16)) - 1u
                      : nodes_visible(a, b, node, sq.tl, Q.at[t], Q.node[t]);
      rows_softmax<2, BITS == 4, true>(st, t, S[t], c2, ex, inv, vis[t], P[t]);
    }
    wide_values(L.tile[0], P, st);
    if (!buffer && (L.bad[0] | L.bad[1] | L.bad[2] | L.bad[3]))
      nodes_nonfinite<2, BITS == 4>(a, a.vt + u * a.T * 128, node, sq.tl, P, vis, st);
  }
}

template <int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_attn_wide(RowsArgs a) {
  __shared__ __attribute__((aligned(16))) WideLds<NW> L;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, g4 = lane >> 4;
  int b, kh, s, rt;
  if (!rows_place(a, b, kh, s, rt)) return;
  const RowsSeq sq = rows_seq(a, b);
  const int rows = a.G * sq.tl;
  if (kWideRows<NW> * rt >= rows || s >= max(sq.nparts, 1)) return;
  const int base = kWideRows<NW> * rt + 32 * w;
  RowsQ<2> Q;
  RowsState<2> st;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int row = base + 16 * t + n;
    const int h = row / sq.tl;
    Q.node[t] = row - h * sq.tl;
    Q.at[t] = row < rows ? ((long)b * a.Hq + kh * a.G + h) * a.T + Q.node[t] : -1;
    st.m[t] = -INFINITY;
    st.l[t] = 0.0f;
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) st.o[t][cb] = f4{0, 0, 0, 0};
  }
  const int head_off = 512 * (4 * kh - 2 * __popcll(a.int2_mask & ((1ull << kh) - 1ull)));
  const int j0 = s * sq.len, j1 = min(j0 + sq.len, sq.ntile);
  const bool work = base < rows;
  if (j0 < j1) {
    if ((a.int2_mask >> kh) & 1ull)
      wide_tiles<2, NW>(a, b, kh, head_off, sq, j0, j1, work, Q, st, L);
    else
      wide_tiles<4, NW>(a, b, kh, head_off, sq, j0, j1, work, Q, st, L);
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const float l = add_xor32(st.l[t] + __shfl_xor(st.l[t], 16));
    if (Q.at[t] < 0) continue;
    float* ws = a.ws + (Q.at[t] * a.nchunk + s) * kWsStride;
    if (sq.nparts > 1 && g4 == 0) *reinterpret_cast<float2*>(ws) = make_float2(st.m[t], l);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c0 = 32 * e + 8 * g4;
      const f4 x = st.o[t][2 * e], y = st.o[t][2 * e + 1];
      const float o[8] = {x[0], y[0], x[1], y[1], x[2], y[2], x[3], y[3]};
      if (sq.nparts <= 1) {
        rows_store(a, Q.at[t], c0, st.m[t], l, o);
      } else {
        *reinterpret_cast<float4*>(ws + kWsO + c0) = make_float4(o[0], o[1], o[2], o[3]);
        *reinterpret_cast<float4*>(ws + kWsO + c0 + 4) = make_float4(o[4], o[5], o[6], o[7]);
      }
    }
  }
}

// Rows of several chunks.  Q groups of 16 lanes merge a row's states, each every Q-th
// (four at a time, their loads together), then the groups: a wave a row where few rows
// have many states, four rows a wave otherwise.
template <int Q>
__global__ __launch_bounds__(256) void k_rows_merge(RowsArgs a) {
  const int lane = threadIdx.x & 63, c0 = 8 * (lane & 15);
  const long at = ((long)blockIdx.x * 16 + (threadIdx.x >> 4)) / Q;
  if (at >= (long)a.B * a.Hq * a.T) return;
  const long bh = at / a.T;
  const int b = (int)(bh / a.Hq);
  const RowsSeq sq = rows_seq(a, b);
  if (at - bh * a.T >= sq.tl || sq.nparts <= 1) return;
  const float* ws = a.ws + at * a.nchunk * kWsStride;
  float m = -INFINITY, l = 0.0f, o[8] = {};
  for (int i0 = (lane >> 4) % Q; i0 < sq.nparts; i0 += 4 * Q) {
    float pm[4], pl[4];
    float4 x[4], y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = i0 + Q * k;
      pm[k] = -INFINITY;
      pl[k] = 0.0f;
      x[k] = y[k] = make_float4(0, 0, 0, 0);
      if (i < sq.nparts) {
        const float* p = ws + (long)i * kWsStride;
        pm[k] = p[0];
        pl[k] = p[1];
        x[k] = *reinterpret_cast<const float4*>(p + kWsO + c0);
        y[k] = *reinterpret_cast<const float4*>(p + kWsO + c0 + 4);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float v[8] = {x[k].x, x[k].y, x[k].z, x[k].w, y[k].x, y[k].y, y[k].z, y[k].w};
      rows_join(m, l, o, pm[k], pl[k], v);
    }
  }
#pragma unroll
  for (int d = 16; d < 16 * Q; d += d) {
    float v[8];
    const float pm = __shfl_xor(m, d), pl = __shfl_xor(l, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __shfl_xor(o[e], d);
    rows_join(m, l, o, pm, pl, v);
  }
  if (Q == 1 || lane < 16) rows_store(a, at, c0, m, l, o);
}

// Query rows of a work-group: one or two tiles of 16 for every wave (the second shares
// the codes' expansion), or 32 a wave of four or eight.  One tile where that many
// work-groups leave the GPU half empty: 1 x 32/8 heads, 4000 tokens, 64 rows a KV head,
// 13.9 us with 16-row tiles and 16.1 with 32-row ones.
inline int rows_tile(int B, int Hkv, int G, int T) {
  const int rows = G * T;
  if (rows > 64) return rows <= 512 ? kWideRows<4> : kWideRows<8>;
  return rows <= 16 || (long)B * Hkv * ceil_div(rows, 16) <= 64 ? 16 : 32;
}
inline int rows_tiles_per_head(int B, int Hkv, int G, int T) {
  return ceil_div(G * T, rows_tile(B, Hkv, G, T));
}

// Chunks of a sequence, at most, and their tiles, at least.  As many as give the GPU two
// work-groups of four waves per CU (one where few heads have to fill it, so that fewer
// states are merged: 13.9 us against 16.0 in the case above), with a tile for every
// wave (eight where the waves share them).  Where the heads fill the GPU by themselves,
// up to 16 chunks of 32 tiles or more, so that a long sequence does not outlast the rest
// of a ragged batch; a chunk's state costs as much as about 8 tiles of 128 rows.  16 x
// 64/8 heads, ragged <= 257 tiles, 120 .. 504 rows: 1 chunk 555 us, 4 307, 8 (33 tiles)
// 289; 64 x 10 heads, 130 tiles of 20 rows: 1 chunk 193 us, 2 180, 3 189.  The tables'
// width bounds the chunks, the sequence's own length divides them.
struct RowsSplit {
  int chunks, min_len;
};
inline RowsSplit rows_split(int B, int Hkv, int G, int T, int max_tiles) {
  const int tile = rows_tile(B, Hkv, G, T);
  const bool wide = tile > 32;
  const int units = (int)std::min<long>((long)B * Hkv * rows_tiles_per_head(B, Hkv, G, T) * (tile > 128 ? 2 : 1), 512);
  RowsSplit r = {ceil_div(!wide && units <= 32 ? 256 : 512, units), wide ? 8 : kRowsWaves};
  if (units >= 256) {
    r.chunks = std::max(r.chunks, std::min(16, ceil_div(max_tiles, wide ? 36 : 72)));
    r.min_len = 32;
  }
  r.chunks = std::max(1, std::min(r.chunks, ceil_div(max_tiles, r.min_len)));
  return r;
}

inline long rows_groups(const RowsArgs& a) {
  return ((long)a.B * a.Hkv * a.nchunk + 7) / 8 * 8 * a.ntiles_row;
}

inline hipError_t launch_attn_rows(const RowsArgs& a, hipStream_t stream) {
  const dim3 groups((unsigned)rows_groups(a));
  switch (rows_tile(a.B, a.Hkv, a.G, a.T)) {
    case 16: hipLaunchKernelGGL((k_attn_rows<1>), groups, dim3(64 * kRowsWaves), 0, stream, a); break;
    case 32: hipLaunchKernelGGL((k_attn_rows<2>), groups, dim3(64 * kRowsWaves), 0, stream, a); break;
    case kWideRows<4>: hipLaunchKernelGGL((k_attn_wide<4>), groups, dim3(256), 0, stream, a); break;
    default: hipLaunchKernelGGL((k_attn_wide<8>), groups, dim3(512), 0, stream, a); break;
  }
  if (a.nchunk > 1) {
    const long rows = (long)a.B * a.Hq * a.T;
    if (rows <= 4096)
      hipLaunchKernelGGL((k_rows_merge<4>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, a);
    else
      hipLaunchKernelGGL((k_rows_merge<1>), dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace turbo
