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
// no chain of dependent reads as long as the tree is deep.
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

// One work-group per (sequence, KV head).  The nodes' codes go to the buffer rows
// seq_len mod 64 onwards and, in LDS, to the tiles a full buffer is compressed from;
// the rows it held before are read only then.
__global__ __launch_bounds__(256) void k_append_path(AppendPathArgs a) {
  __shared__ int8_t ktile[64 * kTileStride];
  __shared__ int8_t vtile[64 * kTileStride];
  __shared__ uint8_t ctile[64 * kTileStride];
  const long u = blockIdx.x;
  const int b = (int)(u / a.c.Hkv), h = (int)(u % a.c.Hkv);
  const int tid = threadIdx.x, c = tid & 127;
  const bool isv = tid >= 128;
  const int len = a.c.seq_lens[b];
  if (len < 0) return;
  const int n = min(max(a.path_lens[b], 0), a.max_path);
  const int* path = a.path + (long)b * a.max_path;
  const float sK = a.c.tscale[2 * u], sV = a.c.tscale[2 * u + 1];
  const float inv = univ_inv(isv ? sV : sK);
  const unsigned short* src = (isv ? a.vt : a.kt) + u * a.T * 128 + c;
  int8_t* tile = isv ? vtile : ktile;
  int held = len & 63;  // rows of the buffer that LDS does not have
  long p = len;
  for (int i = 0; i < n; ++i, ++p) {
    const int node = path[i];
    if (node < 0 || node >= a.T) return;  // ends the path
    const int r = (int)(p & 63);
    const int code = quant_univ((float)__builtin_bit_cast(_Float16, src[(long)node * 128]), inv);
    tile[r * kTileStride + c] = (int8_t)code;
    if (isv)
      a.c.tv[(u * 128 + c) * 64 + r] = (int8_t)code;
    else
      a.c.tk[(u * 64 + r) * 128 + c] = (int8_t)code;
    if (r != 63) continue;
    const long g = p >> 6;
    if (held > 0) {
      {
        const int t = tid >> 2, c0 = 32 * (tid & 3);
        if (t < held) {
          const uint4* s = reinterpret_cast<const uint4*>(a.c.tk + (u * 64 + t) * 128 + c0);
          uint4* d = reinterpret_cast<uint4*>(ktile + t * kTileStride + c0);
          d[0] = s[0];
          d[1] = s[1];
        }
      }
      const int cc = tid >> 1, t0 = 32 * (tid & 1);
      const uint4* s = reinterpret_cast<const uint4*>(a.c.tv + (u * 128 + cc) * 64 + t0);
      const uint4 x0 = s[0], x1 = s[1];
      const unsigned w[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
      for (int k = 0; k < 32; ++k)
        if (t0 + k < held) vtile[(t0 + k) * kTileStride + cc] = (int8_t)(w[k >> 2] >> (8 * (k & 3)));
      held = 0;
    }
    bool ok = g < a.c.max_groups;
    long page[4] = {};
    long slot = 0;
    if (ok) {
      const int* bt = a.c.block_table + ((long)b * a.c.max_groups + g) * 4;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        page[k] = bt[k];
        ok = ok && page[k] >= 0 && page[k] < a.c.num_pages;
      }
      slot = a.c.group_table[(long)b * a.c.max_groups + g];
      ok = ok && slot >= 0 && slot < a.c.num_slots;
    }
    __syncthreads();
    if (ok) {
      const int bits = ((a.c.int2_mask >> h) & 1ull) ? 2 : 4;
      const int head_off = 512 * (4 * h - 2 * __popcll(a.c.int2_mask & ((1ull << h) - 1ull)));
      int8_t* meta = a.c.gmeta + (slot * a.c.Hkv + h) * 512;
      float* gs = a.c.gscale + (slot * a.c.Hkv + h) * 2;
      compress_k(ktile, ctile, bits, meta, gs, sK, page, a.c.pages, a.c.page_bytes, head_off, tid);
      compress_v(vtile, bits, meta, gs + 1, sV, page, a.c.pages, a.c.page_bytes, head_off, tid);
    }
    __syncthreads();
  }
}

inline hipError_t launch_append_path(const AppendPathArgs& a, int B, hipStream_t stream) {
  hipLaunchKernelGGL(k_append_path, dim3((unsigned)(B * a.c.Hkv)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace turbo
