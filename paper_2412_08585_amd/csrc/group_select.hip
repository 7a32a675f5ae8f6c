// Choice of the cached groups that a decoding step attends (turbo_select_groups).
//
// The step-2 metadata of a group bounds its keys: channel c of K^{q1} lies between
// z_c and z_c + L s_c, L = 2^bits - 1.  So for the int8 codes q of a query row,
//   I = sum_c max(q_c z_c, q_c (z_c + L s_c))
//     = sum_c q_c z_c + L sum_c max(q_c, 0) s_c
// is the largest sum any key of the group could reach: an integer, two dot products
// over the 256 metadata bytes of the group's K, 3 % (4 bits) of what attending the
// group reads.  fl(fl(I * s_Q) * s_K) bounds the score up to the common factor.
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

constexpr int kBoundGroups = 64;  // groups of a work-group of k_group_bounds

// One work-group per 64 groups of a (sequence, KV head): four lanes per group, 32
// channels each, for all G rows.  NaN marks a group whose table entries are out of
// range (a bound that is not a number is stored as -inf).
__global__ __launch_bounds__(256) void k_group_bounds(SelectArgs a, int nblk) {
  __shared__ __attribute__((aligned(16))) int q8[16][32];  // codes, 4 per word
  __shared__ float sq[16];
  int u = blockIdx.x;
  const int blk = u % nblk;
  u /= nblk;
  const int b = u / a.Hkv, kh = u - b * a.Hkv;
  const int ng = min(max(a.seq_lens[b] / 64, 0), a.max_groups);
  if (blk * kBoundGroups >= ng) return;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  for (int r = w; r < a.G; r += 4) {  // Q to int8, as the decode quantizes it
    const unsigned short* src = a.q + ((long)b * a.Hq + kh * a.G + r) * 128 + 2 * lane;
    const float x0 = (float)__builtin_bit_cast(_Float16, src[0]);
    const float x1 = (float)__builtin_bit_cast(_Float16, src[1]);
    const float amax = wave_max(fmaxf(fabsf(x0), fabsf(x1)));
    const float inv = amax > 0.0f ? kQmax / amax : 0.0f;
    const int c0 = min(119, max(-119, rne_mul(x0, inv)));
    const int c1 = min(119, max(-119, rne_mul(x1, inv)));
    reinterpret_cast<unsigned short*>(q8[r])[lane] = (unsigned short)((c0 & 0xff) | ((c1 & 0xff) << 8));
    if (lane == 0) sq[r] = amax / kQmax;
  }
  __syncthreads();
  const int g = blk * kBoundGroups + (threadIdx.x >> 2), part = threadIdx.x & 3;
  if (g >= ng) return;
  const int slot = a.group_table[(long)b * a.max_groups + g];
  const int pg = a.block_table[((long)b * a.max_groups + g) * 4 + part];
  int bad = slot < 0 || slot >= a.nslots || pg < 0 || pg >= a.npages;
  bad |= __shfl_xor(bad, 1);
  bad |= __shfl_xor(bad, 2);
  int s[8] = {}, z[8] = {};
  float sk = 0.0f;
  if (!bad) {
    const int8_t* meta = a.gmeta + ((long)slot * a.Hkv + kh) * 512 + 32 * part;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int4 x = reinterpret_cast<const int4*>(meta)[i];
      const int4 y = reinterpret_cast<const int4*>(meta + 128)[i];
      s[4 * i] = x.x; s[4 * i + 1] = x.y; s[4 * i + 2] = x.z; s[4 * i + 3] = x.w;
      z[4 * i] = y.x; z[4 * i + 1] = y.y; z[4 * i + 2] = y.z; z[4 * i + 3] = y.w;
    }
    sk = a.gscale[((long)slot * a.Hkv + kh) * 2];
  }
  const int L = (a.int2_mask >> kh) & 1ull ? 3 : 15;
  for (int r = 0; r < a.G; ++r) {
    int sum = 0;
    unsigned up = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int qw = q8[r][8 * part + i];
      // bytes below zero to 0: their sign bits spread over the byte
      const unsigned neg = ((unsigned)qw >> 7) & 0x01010101u;
      const unsigned pos = (unsigned)qw & ~(neg * 0xffu);
      sum = __builtin_amdgcn_sdot4(qw, z[i], sum, false);
      up = __builtin_amdgcn_udot4(pos, (unsigned)s[i], up, false);
    }
    sum += L * (int)up;
    sum += __shfl_xor(sum, 1);
    sum += __shfl_xor(sum, 2);
    if (part == 0) {
      float v = ((float)sum * sq[r]) * sk;
      v = v == v ? v : -INFINITY;
      a.ws[((long)b * a.Hq + kh * a.G + r) * a.max_groups + g] = bad ? __builtin_nanf("") : v;
    }
  }
}

// Unsigned key in the order of the floats (not NaN); 0 and ~0 are below and above all.
__device__ __forceinline__ unsigned order_key(float x) {
  const unsigned u = __float_as_uint(x + 0.0f);  // (-0 is +0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kPickThreads = 256;

// Sum over the work-group of flags, and the number of them before this thread.
__device__ __forceinline__ int block_rank(bool f, int* wsum, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const unsigned long long m = __ballot(f);
  __syncthreads();
  if (lane == 0) wsum[w] = __popcll(m);
  __syncthreads();
  int before = __popcll(m & ((1ull << lane) - 1ull));
  total = 0;
#pragma unroll
  for (int i = 0; i < kPickThreads / 64; ++i) {
    if (i < w) before += wsum[i];
    total += wsum[i];
  }
  return before;
}

// One work-group per (sequence, KV head).  Score of a group: the largest over the G
// rows of fl(bound - the row's largest bound), so that every row's best group scores
// 0 whatever the size of its scores.  The num_select-th largest key is found digit by
// digit (four of 8 bits, counted in LDS); the groups above it and the first ones
// equal to it are written in ascending order.
__global__ __launch_bounds__(kPickThreads) void k_group_pick(SelectArgs a) {
  __shared__ float rowmax[16];
  __shared__ int hist[256];
  __shared__ int wsum[kPickThreads / 64];
  __shared__ int found[2];
  const int u = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int b = u / a.Hkv, kh = u - b * a.Hkv;
  const int ng = min(max(a.seq_lens[b] / 64, 0), a.max_groups);
  int* sel = a.sel + (long)u * a.nsel;
  float* bounds = a.ws + ((long)b * a.Hq + kh * a.G) * a.max_groups;
  for (int r = w; r < a.G; r += kPickThreads / 64) {
    float m = -INFINITY;
    for (int g = lane; g < ng; g += 64) m = fmaxf(m, bounds[(long)r * a.max_groups + g]);
    m = wave_max(m);
    if (lane == 0) rowmax[r] = m;
  }
  __syncthreads();
  // keys in place of the first row's bounds, read back by the thread that wrote them
  unsigned* keys = reinterpret_cast<unsigned*>(bounds);
  for (int g = tid; g < ng; g += kPickThreads) {
    unsigned key = 0;
    const float b0 = bounds[g];
    if (b0 == b0) {  // (NaN: out of range in every row)
      float v = -INFINITY;
      for (int r = 0; r < a.G; ++r)
        v = fmaxf(v, bounds[(long)r * a.max_groups + g] - rowmax[r]);
      key = g < a.first || g >= ng - a.last ? ~0u : order_key(v);
    }
    keys[g] = key;
  }
  // the digits of the smallest chosen key
  unsigned prefix = 0;
  int want = a.nsel;
  for (int shift = 24; shift >= 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    for (int g = tid; g < ng; g += kPickThreads) {
      const unsigned k = keys[g];
      if (k != 0 && (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))))
        atomicAdd(&hist[(k >> shift) & 255u], 1);
    }
    __syncthreads();
    if (w == 0) {  // lane i: digits 255 - 4 i downwards
      int c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += c[i] = hist[255 - 4 * lane - i];
      int before = sum;
      for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(before, o);
        if (lane >= o) before += x;
      }
      const int all = __shfl(before, 63);
      before -= sum;
      if (lane == 0 && all < want) {  // fewer groups than wanted: every one is chosen
        found[0] = 0;
        found[1] = all;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (before < want && before + c[i] >= want && all >= want) {
          found[0] = 255 - 4 * lane - i;
          found[1] = want - before;
        }
        before += c[i];
      }
    }
    __syncthreads();
    prefix |= (unsigned)found[0] << shift;
    want = found[1];
    __syncthreads();
  }
  // above the threshold, and the first `want` equal to it
  int out = 0, equal = 0;
  for (int g0 = 0; g0 < ng; g0 += kPickThreads) {
    const int g = g0 + tid;
    const unsigned k = g < ng ? keys[g] : 0u;
    int n;
    const bool eq = k != 0 && k == prefix;
    const int re = equal + block_rank(eq, wsum, n);
    equal += n;
    const bool take = k > prefix || (eq && re < want);
    const int at = out + block_rank(take, wsum, n);
    if (take) sel[at] = g;
    out += n;
  }
  for (int i = out + tid; i < a.nsel; i += kPickThreads) sel[i] = -1;
}

inline hipError_t launch_select_groups(const SelectArgs& a, hipStream_t stream) {
  const int nblk = ceil_div(a.max_groups, kBoundGroups);
  hipLaunchKernelGGL(k_group_bounds, dim3((unsigned)((long)a.B * a.Hkv * nblk)), dim3(256), 0, stream,
                     a, nblk);
  hipLaunchKernelGGL(k_group_pick, dim3((unsigned)(a.B * a.Hkv)), dim3(kPickThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace turbo
