// Choice of the cached groups that a decoding step attends (turbo_select_groups).
//
// The step-2 metadata of a group bounds its keys: channel c of K^{q1} lies between
// z_c and z_c + L s_c, L = 2^bits - 1.  So for the int8 codes q of a query row,
//   I = sum_c max(q_c z_c, q_c (z_c + L s_c))
//     = sum_c q_c z_c + L sum_c max(q_c, 0) s_c
// is the largest sum any key of the group could reach: an integer, two dot products
// over the 256 metadata bytes of the group's K, 3 % (4 bits) of what attending the
// group reads.  fl(fl(I * s_Q) * s_K) bounds the score up to the common factor.
//
// A few hundred bytes to a megabyte in all: bound by a chain of latencies, not by bytes
// or sums.  511 groups of 8 heads, 64 chosen, 9.7 us; 32 x 8 heads of up to 255 groups,
// eight rows, 11.5 us; with bounds and choice in two launches 14.4 and 16.5.
#include "turbo_common.h"

namespace turbo {

struct SelectArgs {
  const unsigned short* q;   // fp16 [B][Hq][128]
  const int8_t* gmeta;       // [slots][Hkv][4][128]
  const float* gscale;       // [slots][Hkv][2]
  int npages, nslots;        // min(num_pages, INT_MAX), min(num_slots, INT_MAX)
  unsigned long long int2_mask;
  const int* seq_lens;       // [B]
  const int* block_table;    // [B][4*max_groups]
  const int* group_table;    // [B][max_groups]
  int max_groups;
  int B, Hq, Hkv, G;
  int nsel, first, last;
  float* ws;                 // [B][Hq][max_groups] bounds
  int* sel;                  // [B][Hkv][nsel]
};

constexpr int kSelThreads = 512;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kBoundGroups = kSelThreads / 4;  // four lanes a group
constexpr int kBoundRound = 4;                 // groups of a lane in flight
constexpr int kSelLdsFloats = 12288;           // bounds kept in LDS, at most

// Query rows of (b, kh) as int8 codes and scales, the way the decode quantizes them.
__device__ __forceinline__ void select_quantize(const SelectArgs& a, int b, int kh, int (*q8)[32],
                                                float* sq) {
  const int lane = threadIdx.x & 63;
  for (int r = threadIdx.x >> 6; r < a.G; r += kSelWaves) {
    const unsigned short* src = a.q + ((long)b * a.Hq + kh * a.G + r) * 128 + 2 * lane;
    const float x0 = (float)__builtin_bit_cast(_Float16, src[0]);
    const float x1 = (float)__builtin_bit_cast(_Float16, src[1]);
    const float amax = wave_max_fast(fmaxf(fabsf(x0), fabsf(x1)));
    const float inv = amax > 0.0f ? kQmax / amax : 0.0f;
    const int c0 = min(119, max(-119, rne_mul(x0, inv)));
    const int c1 = min(119, max(-119, rne_mul(x1, inv)));
    reinterpret_cast<unsigned short*>(q8[r])[lane] = (unsigned short)((c0 & 0xff) | ((c1 & 0xff) << 8));
    if (lane == 0) sq[r] = amax / kQmax;
  }
}

// Table entries of the thread's groups g0 + 128 i (four lanes a group), read before
// the sequence's length is known: slot and the lane's page, -1 past the table.
struct SelectTab {
  int slot[kBoundRound], pg[kBoundRound];
};

__device__ __forceinline__ void select_tab(const SelectArgs& a, int b, int g0, SelectTab& t) {
#pragma unroll
  for (int i = 0; i < kBoundRound; ++i) {
    const int g = g0 + (threadIdx.x >> 2) + i * kBoundGroups;
    t.slot[i] = t.pg[i] = -1;
    if (g < a.max_groups) {
      t.slot[i] = a.group_table[(long)b * a.max_groups + g];
      t.pg[i] = a.block_table[((long)b * a.max_groups + g) * 4 + (threadIdx.x & 3)];
    }
  }
}

// Bounds of the groups of t below ng to bounds[r][g] (rows `stride` apart): 32
// channels a lane, the loads of all its groups before the first sum.  NaN marks a
// group whose table entries are out of range; a bound that is not a number is stored
// as -inf.
__device__ __forceinline__ void select_bounds(const SelectArgs& a, int kh, int g0, int ng,
                                              const SelectTab& t, const int (*q8)[32], const float* sq,
                                              float* bounds, int stride) {
  const int part = threadIdx.x & 3;
  g0 += threadIdx.x >> 2;
  int s[kBoundRound][8], z[kBoundRound][8];
  float sk[kBoundRound];
  bool bad[kBoundRound];
#pragma unroll
  for (int i = 0; i < kBoundRound; ++i) {
    int x = g0 + i * kBoundGroups >= ng || t.slot[i] < 0 || t.slot[i] >= a.nslots || t.pg[i] < 0 ||
            t.pg[i] >= a.npages;
    x |= __builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true);  // the quad's four pages
    x |= __builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true);
    bad[i] = x;
    sk[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s[i][k] = z[i][k] = 0;
    if (!bad[i]) {
      const int8_t* meta = a.gmeta + ((long)t.slot[i] * a.Hkv + kh) * 512 + 32 * part;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int4 x4 = reinterpret_cast<const int4*>(meta)[k];
        const int4 y4 = reinterpret_cast<const int4*>(meta + 128)[k];
        s[i][4 * k] = x4.x; s[i][4 * k + 1] = x4.y; s[i][4 * k + 2] = x4.z; s[i][4 * k + 3] = x4.w;
        z[i][4 * k] = y4.x; z[i][4 * k + 1] = y4.y; z[i][4 * k + 2] = y4.z; z[i][4 * k + 3] = y4.w;
      }
      sk[i] = a.gscale[((long)t.slot[i] * a.Hkv + kh) * 2];
    }
  }
  const int L = (a.int2_mask >> kh) & 1ull ? 3 : 15;
  for (int r = 0; r < a.G; ++r) {
    int qw[8];
    unsigned pos[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      qw[k] = q8[r][8 * part + k];
      // bytes below zero to 0: their sign bits spread over the byte
      const unsigned neg = ((unsigned)qw[k] >> 7) & 0x01010101u;
      pos[k] = (unsigned)qw[k] & ~(neg * 0xffu);
    }
    const float sr = sq[r];
#pragma unroll
    for (int i = 0; i < kBoundRound; ++i) {
      const int g = g0 + i * kBoundGroups;
      int sum = 0;
      unsigned up = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        sum = __builtin_amdgcn_sdot4(qw[k], z[i][k], sum, false);
        up = __builtin_amdgcn_udot4(pos[k], (unsigned)s[i][k], up, false);
      }
      sum += L * (int)up;
      sum += __builtin_amdgcn_mov_dpp(sum, 0xB1, 0xf, 0xf, true);
      sum += __builtin_amdgcn_mov_dpp(sum, 0x4E, 0xf, 0xf, true);
      if (part == 0 && g < ng) {
        float v = ((float)sum * sr) * sk[i];
        v = v == v ? v : -INFINITY;
        bounds[(long)r * stride + g] = bad[i] ? __builtin_nanf("") : v;
      }
    }
  }
}

// Bounds of 512 groups of a (sequence, KV head) to the workspace.
__global__ __launch_bounds__(kSelThreads) void k_group_bounds(SelectArgs a, int nblk) {
  __shared__ __attribute__((aligned(16))) int q8[16][32];  // codes, 4 per word
  __shared__ float sq[16];
  int u = blockIdx.x;
  const int blk = u % nblk;
  u /= nblk;
  const int b = u / a.Hkv, kh = u - b * a.Hkv;
  const int ng = min(max(a.seq_lens[b] / 64, 0), a.max_groups);
  const int g0 = blk * kBoundGroups * kBoundRound;
  if (g0 >= ng) return;
  SelectTab t;
  select_tab(a, b, g0, t);
  select_quantize(a, b, kh, q8, sq);
  __syncthreads();
  select_bounds(a, kh, g0, ng, t, q8, sq,
                a.ws + ((long)b * a.Hq + kh * a.G) * a.max_groups, a.max_groups);
}

// Unsigned key in the order of the floats (not NaN); 0 and ~0 are below and above all.
__device__ __forceinline__ unsigned order_key(float x) {
  const unsigned u = __float_as_uint(x + 0.0f);  // (-0 is +0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Inclusive sums over the lanes of a wave: within rows of 16 by DPP shifts, then the
// last lanes of the rows before.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row 0 to 1, 2 to 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2, 3
  return v;
}

// The choice of one (sequence, KV head) from its bounds (rows `stride` apart), by a
// work-group.  Score of a group: the largest over the G rows of fl(bound - the row's
// largest bound), so that every row's best group scores 0 whatever the size of its
// scores.  The num_select-th largest key is found digit by digit (four of 8 bits,
// counted in LDS; every wave reads the counts for itself); the groups above it and
// the first ones equal to it are written in ascending order.
__device__ __forceinline__ void select_pick(const SelectArgs& a, int ng, float* bounds, int stride,
                                            int* sel) {
  __shared__ float rowmax[16];
  __shared__ int hist[4][256];
  __shared__ int wsum[2][kSelWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  hist[tid >> 8][tid & 255] = hist[2 + (tid >> 8)][tid & 255] = 0;
  for (int r = w; r < a.G; r += kSelWaves) {
    float m = -INFINITY;
#pragma unroll 8
    for (int g = lane; g < ng; g += 64) m = fmaxf(m, bounds[(long)r * stride + g]);
    m = wave_max_fast(m);
    if (lane == 0) rowmax[r] = m;
  }
  __syncthreads();
  // keys in place of the first row's bounds, read back by the thread that wrote them
  unsigned* keys = reinterpret_cast<unsigned*>(bounds);
  for (int g = tid; g < ng; g += kSelThreads) {
    unsigned key = 0;
    const float b0 = bounds[g];
    if (b0 == b0) {  // (NaN: out of range in every row)
      float v = fmaxf(-INFINITY, b0 - rowmax[0]);
#pragma unroll 4
      for (int r = 1; r < a.G; ++r) v = fmaxf(v, bounds[(long)r * stride + g] - rowmax[r]);
      key = g < a.first || g >= ng - a.last ? ~0u : order_key(v);
    }
    keys[g] = key;
  }
  // the digits of the smallest chosen key
  unsigned prefix = 0;
  int want = a.nsel;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int shift = 24 - 8 * d;
    for (int g = tid; g < ng; g += kSelThreads) {
      const unsigned k = keys[g];
      if (k != 0 && (d == 0 || (k >> (shift + 8)) == (prefix >> (shift + 8))))
        atomicAdd(&hist[d][(k >> shift) & 255u], 1);
    }
    __syncthreads();
    // lane i: digits 255 - 4 i downwards
    int c[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += c[i] = hist[d][255 - 4 * lane - i];
    int before = wave_scan(sum);
    const int all = __builtin_amdgcn_readlane(before, 63);
    before -= sum;
    // the digit at which the count reaches `want`; digit 0, and all of them, where
    // there are fewer
    int digit = -1, rest = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (before < want && before + c[i] >= want) {
        digit = 255 - 4 * lane - i;
        rest = want - before;
      }
      before += c[i];
    }
    const unsigned long long hit = __ballot(digit >= 0);
    const int from = hit ? __builtin_ctzll(hit) : 0;
    digit = __builtin_amdgcn_readlane(digit, from);
    rest = __builtin_amdgcn_readlane(rest, from);
    prefix |= (unsigned)(hit ? digit : 0) << shift;
    want = hit ? rest : all;
  }
  // above the threshold, and the first `want` equal to it
  int above = 0, equal = 0;
  for (int g0 = 0; g0 < ng; g0 += kSelThreads) {
    const int g = g0 + tid;
    const unsigned k = g < ng ? keys[g] : 0u;
    const unsigned long long gt = __ballot(k > prefix), eq = __ballot(k != 0 && k == prefix);
    const unsigned long long lower = (1ull << lane) - 1ull;
    if (g0 > 0) __syncthreads();
    if (lane == 0) {
      wsum[0][w] = __popcll(gt);
      wsum[1][w] = __popcll(eq);
    }
    __syncthreads();
    int na = above + __popcll(gt & lower), ne = equal + __popcll(eq & lower);
#pragma unroll
    for (int i = 0; i < kSelWaves; ++i) {
      const int x = wsum[0][i], y = wsum[1][i];
      if (i < w) {
        na += x;
        ne += y;
      }
      above += x;
      equal += y;
    }
    const bool is_eq = (eq >> lane) & 1ull;
    if (((gt >> lane) & 1ull) || (is_eq && ne < want)) sel[na + min(ne, want)] = g;
  }
  for (int i = above + min(equal, want) + tid; i < a.nsel; i += kSelThreads) sel[i] = -1;
}

// One work-group per (sequence, KV head): the choice from the workspace's bounds, or
// (FUSED) from bounds it computes into LDS.
template <bool FUSED>
__global__ __launch_bounds__(kSelThreads) void k_group_pick(SelectArgs a) {
  __shared__ __attribute__((aligned(16))) int q8[FUSED ? 16 : 1][32];
  __shared__ float sq[16];
  __shared__ float lds[FUSED ? kSelLdsFloats : 1];
  const int u = blockIdx.x;
  const int b = u / a.Hkv, kh = u - b * a.Hkv;
  const int ng = min(max(a.seq_lens[b] / 64, 0), a.max_groups);
  int* sel = a.sel + (long)u * a.nsel;
  if constexpr (FUSED) {
    SelectTab t;
    select_tab(a, b, 0, t);
    select_quantize(a, b, kh, q8, sq);
    __syncthreads();
    for (int g0 = 0; g0 < ng; g0 += kBoundGroups * kBoundRound) {
      if (g0 > 0) select_tab(a, b, g0, t);
      select_bounds(a, kh, g0, ng, t, q8, sq, lds, a.max_groups);
    }
    __syncthreads();
    select_pick(a, ng, lds, a.max_groups, sel);
  } else {
    select_pick(a, ng, a.ws + ((long)b * a.Hq + kh * a.G) * a.max_groups, a.max_groups, sel);
  }
}

// One launch where the bounds fit LDS and one work-group reads its groups' metadata
// soon enough, by itself (1024 groups: 256 KB) or as one of as many as there are CUs.
inline bool select_fused(int B, int Hkv, int G, int max_groups) {
  return (long)G * max_groups <= kSelLdsFloats && (max_groups <= 1024 || (long)B * Hkv >= 256);
}

inline hipError_t launch_select_groups(const SelectArgs& a, hipStream_t stream) {
  const dim3 units((unsigned)(a.B * a.Hkv)), threads(kSelThreads);
  if (select_fused(a.B, a.Hkv, a.G, a.max_groups)) {
    hipLaunchKernelGGL((k_group_pick<true>), units, threads, 0, stream, a);
    return hipGetLastError();
  }
  const int nblk = ceil_div(a.max_groups, kBoundGroups * kBoundRound);
  hipLaunchKernelGGL(k_group_bounds, dim3((unsigned)((long)a.B * a.Hkv * nblk)), threads, 0, stream, a,
                     nblk);
  hipLaunchKernelGGL((k_group_pick<false>), units, threads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace turbo
