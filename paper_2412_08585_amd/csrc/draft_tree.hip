// Drafted trees around the attention that checks them: the ancestor bits of their
// nodes (turbo_tree_mask) and the append of an accepted path to the int8 buffer and
// the cache (turbo_append_path).
#include "turbo_common.h"

namespace turbo {

// ---- ancestors -------------------------------------------------------------------
struct TreeMaskArgs {
  const int* parents;        // [B][T]
  const int* tree_lens;      // [B]
  int T, words;
  unsigned long long* mask;  // [B][T][words]
  int* depth;                // [B][T] or null
};

// One work-group per tree, one thread per node.  Round k gives every node the
// ancestors within 2^k steps and the node 2^k steps up: log2(T) rounds in LDS, with
// no chain of dependent reads as long as the tree is deep.  1.8 us (16 nodes: a launch) to
// 4.2 us (256 trees of 200 nodes, 2 MB).
__global__ __launch_bounds__(TURBO_MAX_TREE) void k_tree_mask(TreeMaskArgs a) {
  constexpr int W = TURBO_MAX_TREE / 64;
  __shared__ unsigned long long bits[TURBO_MAX_TREE][W];
  __shared__ int up[TURBO_MAX_TREE];
  const int b = blockIdx.x, i = threadIdx.x;
  const int tl = min(max(a.tree_lens[b], 0), a.T);
  unsigned long long m[W] = {};
  int p = -1;
  if (i < tl) {
    m[i >> 6] = 1ull << (i & 63);
    p = a.parents[(long)b * a.T + i];
    p = p >= 0 && p < i ? p : -1;
  }
  for (int span = 1; span < tl; span *= 2) {
#pragma unroll
    for (int k = 0; k < W; ++k) bits[i][k] = m[k];
    up[i] = p;
    __syncthreads();
    if (p >= 0) {
#pragma unroll
      for (int k = 0; k < W; ++k) m[k] |= bits[p][k];
      p = up[p];
    }
    __syncthreads();
  }
  if (i >= a.T) return;
  int n = 0;
  unsigned long long* dst = a.mask + ((long)b * a.T + i) * a.words;
#pragma unroll
  for (int k = 0; k < W; ++k) {
    n += __popcll(m[k]);
    if (k < a.words) dst[k] = m[k];
  }
  if (a.depth) a.depth[(long)b * a.T + i] = n - 1;
}

inline hipError_t launch_tree_mask(const TreeMaskArgs& a, int B, hipStream_t stream) {
  hipLaunchKernelGGL(k_tree_mask, dim3((unsigned)B), dim3(TURBO_MAX_TREE), 0, stream, a);
  return hipGetLastError();
}

// ---- append of an accepted path -----------------------------------------------------
struct AppendPathArgs {
  const unsigned short* kt;  // fp16 [B][Hkv][T][128]
  const unsigned short* vt;
  const int* path;           // [B][max_path] nodes
  const int* path_lens;      // [B]
  int T, max_path;
  AppendArgs c;              // buffer, cache, tables, lengths before (knew, vnew unused)
};

// Filling up is the rare part of the append, and the slowest of its work-groups: its
// code runs once in each, straight from memory, so that fetching it is most of its
// time.  It is kept short (loops that stay loops): 256 sequences of which a tenth
// fills a buffer, 11.9 us without this part, 19.1 with it, 30 with its loops unrolled.

// The rows that the buffer held before the call, into the tiles.
__device__ __forceinline__ void path_held(const AppendArgs& c, long u, int held, int8_t* ktile,
                                          int8_t* vtile) {
  const int tid = threadIdx.x;
  const int t = tid >> 2, c0 = 32 * (tid & 3);
  const unsigned* s = reinterpret_cast<const unsigned*>(c.tk + (u * 64 + t) * 128 + c0);
  unsigned* d = reinterpret_cast<unsigned*>(ktile + t * kTileStride + c0);
  if (t < held) {
#pragma unroll 4
    for (int k = 0; k < 8; ++k) d[k] = s[k];
  }
  const int cc = tid >> 1, t0 = 32 * (tid & 1);
  const unsigned* v = reinterpret_cast<const unsigned*>(c.tv + (u * 128 + cc) * 64 + t0);
#pragma unroll 2
  for (int k = 0; k < 8; ++k) {
    const unsigned w = v[k];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (t0 + 4 * k + e < held) vtile[(t0 + 4 * k + e) * kTileStride + cc] = (int8_t)(w >> (8 * e));
  }
}

struct PathMeta {
  int s[2][128], z[2][128], inv[2][128];  // of K and V: s^int, z^int, 2^20 / (2 s) + 1
};

__device__ __forceinline__ unsigned path_code(const PathMeta& m, int v, int c, int q) {
  return (unsigned)((2 * (q - m.z[v][c]) + m.s[v][c]) * m.inv[v][c]) >> 20;
}

// The full buffer in the tiles to group g of sequence b: step 2 (the integers of
// step2_channel).
__device__ __forceinline__ void path_flush(const AppendArgs& a, int b, int h, long g, float sK, float sV,
                                           const int8_t* ktile, const int8_t* vtile, PathMeta& m) {
  const int tid = threadIdx.x, c = tid & 127, v = tid >> 7;
  const int bits = ((a.int2_mask >> h) & 1ull) ? 2 : 4;
  bool ok = g < a.max_groups;
  int slot = 0;
  const int* bt = a.block_table + ((long)b * a.max_groups + g) * 4;
  if (ok) {
    int bad = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) bad |= bt[k] < 0 || bt[k] >= a.num_pages;
    slot = a.group_table[(long)b * a.max_groups + g];
    ok = !bad && slot >= 0 && slot < a.num_slots;
  }
  __syncthreads();
  if (ok) {
    const long at = (long)slot * a.Hkv + h;
    {
      const int8_t* tile = v ? vtile : ktile;
      int mn = 127, mx = -128;
#pragma unroll 8
      for (int t = 0; t < 64; ++t) {
        const int q = tile[t * kTileStride + c];
        mn = min(mn, q);
        mx = max(mx, q);
      }
      const int levels = (1 << bits) - 1;
      const int s = max(1, (mx - mn + levels - 1) / levels);
      m.s[v][c] = s;
      m.z[v][c] = mn;
      m.inv[v][c] = (1 << 20) / (2 * s) + 1;
      int8_t* meta = a.gmeta + at * 512 + 256 * v + c;
      meta[0] = (int8_t)s;
      meta[128] = (int8_t)mn;
      if (c == 0) a.gscale[at * 2 + v] = v ? sV : sK;
    }
    __syncthreads();
    const int head_off = 512 * (4 * h - 2 * __popcll(a.int2_mask & ((1ull << h) - 1ull)));
    // K, token-major: token tid / 4, 32 channels; V, channel-major: channel tid / 2, two
    // pages of 16 tokens: 32 codes each, word by word
    const int t = tid >> 2, c0 = 32 * (tid & 3), cv = tid >> 1, t0 = 32 * (tid & 1);
    unsigned* kd = reinterpret_cast<unsigned*>(a.pages + (long)bt[t >> 4] * a.page_bytes + head_off +
                                               (t & 15) * 16 * bits + (tid & 3) * 4 * bits);
    for (int i = 0; i < bits; ++i) {
      unsigned wk = 0, wv = 0;
#pragma unroll 2
      for (int e = 0; e < 32 / bits; ++e) {
        const int x = 32 / bits * i + e;
        wk |= path_code(m, 0, c0 + x, ktile[t * kTileStride + c0 + x]) << (bits * e);
        wv |= path_code(m, 1, cv, vtile[(t0 + x) * kTileStride + cv]) << (bits * e);
      }
      kd[i] = wk;
      const int page = bt[(t0 >> 4) + (2 * i >= bits)];
      reinterpret_cast<unsigned*>(a.pages + (long)page * a.page_bytes + head_off + 256 * bits +
                                  cv * 2 * bits)[i & (bits / 2 - 1)] = wv;
    }
  }
  __syncthreads();
}

// The m low bytes of word to dst (at r in its aligned run of 64), in as few stores as
// its alignment allows: every channel's run is a line of its own.
__device__ __forceinline__ void path_bytes(int8_t* dst, int r, int m, unsigned long long word) {
  while (m > 0) {
    const int n = (r & 1) || m < 2 ? 1 : ((r & 2) || m < 4 ? 2 : 4);
    if (n == 4)
      *reinterpret_cast<unsigned*>(dst) = (unsigned)word;
    else if (n == 2)
      *reinterpret_cast<unsigned short*>(dst) = (unsigned short)word;
    else
      *dst = (int8_t)word;
    dst += n;
    r += n;
    m -= n;
    word >>= 8 * n;
  }
}

// One work-group per (sequence, KV head), one thread per channel of K (0 .. 127) and
// of V.  The nodes' codes go to the buffer rows seq_len mod 64 onwards, eight nodes'
// loads at a time, and, if a buffer fills up, to the tiles in LDS that it is
// compressed from; the rows it held before are read only then.  A few KB per
// work-group: bound by the latency of lengths, path, keys and stores (3.8 us for one
// sequence, 19 for 256 of 10 heads).
__global__ __launch_bounds__(256, 6) void k_append_path(AppendPathArgs a) {
  __shared__ int8_t ktile[64 * kTileStride];
  __shared__ int8_t vtile[64 * kTileStride];
  __shared__ PathMeta meta;
  const long u = blockIdx.x;
  const int b = (int)(u / a.c.Hkv), h = (int)(u % a.c.Hkv);
  const int tid = threadIdx.x, c = tid & 127, lane = tid & 63;
  const bool isv = tid >= 128;
  const int len = a.c.seq_lens[b];
  if (len < 0) return;
  const int n = min(max(a.path_lens[b], 0), a.max_path);
  const float sK = a.c.tscale[2 * u], sV = a.c.tscale[2 * u + 1];
  const float inv = univ_inv(isv ? sV : sK);
  const unsigned short* src = (isv ? a.vt : a.kt) + u * a.T * 128 + c;
  int8_t* tile = isv ? vtile : ktile;
  const bool fills = (long)(len & 63) + n >= 64;
  int held = len & 63;  // rows of the buffer that LDS does not have
  long p = len;
  for (int i0 = 0; i0 < n; i0 += 64) {
    // the next 64 nodes, a lane each, up to the first that is none
    int node = -1;  // (read before n is known)
    if (i0 + lane < a.max_path) node = a.path[(long)b * a.max_path + i0 + lane];
    const unsigned long long ends = ~__ballot(i0 + lane < n && node >= 0 && node < a.T);
    const int cnt = ends ? __builtin_ctzll(ends) : 64;
    for (int i = 0; i < cnt;) {  // up to eight, and no further than the buffer's end
      const int r = (int)(p & 63), m = min(min(8, cnt - i), 64 - r);
      _Float16 x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] = (_Float16)0.0f;
        if (k < m)
          x[k] = __builtin_bit_cast(
              _Float16, src[(long)__builtin_amdgcn_readlane(node, i + k) * 128]);
      }
      unsigned long long word = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (k >= m) break;
        const int code = quant_univ((float)x[k], inv);
        if (fills) tile[(r + k) * kTileStride + c] = (int8_t)code;
        if (!isv) a.c.tk[(u * 64 + r + k) * 128 + c] = (int8_t)code;
        word |= (unsigned long long)(code & 0xff) << (8 * k);
      }
      if (isv) path_bytes(a.c.tv + (u * 128 + c) * 64 + r, r, m, word);
      i += m;
      p += m;
      if (r + m == 64) {
        if (held > 0) path_held(a.c, u, held, ktile, vtile);
        held = 0;
        path_flush(a.c, b, h, (p >> 6) - 1, sK, sV, ktile, vtile, meta);
      }
    }
    if (cnt < 64) break;
  }
}

inline hipError_t launch_append_path(const AppendPathArgs& a, int B, hipStream_t stream) {
  hipLaunchKernelGGL(k_append_path, dim3((unsigned)(B * a.c.Hkv)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace turbo
