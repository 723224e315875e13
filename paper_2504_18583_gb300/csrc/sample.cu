// One token a row from temperature, top-k, top-p and min-p, drawn with a given
// uniform number.
//
//   x_i = (z_i - max z) / T,  w_i = e^x_i                   order: z descending, then i ascending
//   top-k: the first k;  top-p: those whose mass before them, of the top-k's, is below p times it;
//   min-p: w_i >= m (the largest has w = 1);  the first is always kept
//   token = the lowest i with  sum_{kept j <= i} w_j > u * sum_{kept} w_j
//
// Weights are summed as whole multiples of 2^-40 in 64 bits: integer sums have
// no order, so neither the threads' atomics nor the split over CTAs changes a
// result, and a cut or a draw is exact for those weights (32-bit floating sums
// over 1e5 entries move a draw's boundaries by 1e-7 each).
//
// What bounds it: HBM for many rows (each logit is read once and stays in
// shared memory), dependent steps for few.  A cluster of up to eight CTAs holds
// a row, an index range each.  Sorting is avoided: one histogram over
// max z - z (1024 bins, counts and the sums of the places within a bin, which
// give a bin's mass to 1e-5) finds the bins that the cuts fall into, and only
// entries that can matter are sorted:
//   A  top-k set:   the bins up to the k-th entry hold at most 2048 entries: one
//                   CTA sorts them and does all the rest;
//   B  top-p only:  the same with the bins up to the nucleus' end, and the
//                   exact sum of all weights;
//   C  otherwise:   exact sums around the cut's bin, whose entries alone are
//                   sorted (a bin of more than 2048 entries, ties as a rule: by
//                   bisection over (z, i)); then one pass draws in index order.
#include <cuda_fp16.h>

#include "common.cuh"
#include "tree.h"

namespace pard {

namespace {

constexpr int kSmpThreads = 512;
constexpr int kSmpWarps = kSmpThreads / 32;
constexpr int kBins = 1024;
constexpr int kList = 2048;            // entries one CTA sorts
constexpr int kSmpMaxCluster = 8;
constexpr int kSliceBytes = 64 * 1024; // a CTA's share of a row: two CTAs an SM
constexpr float kRange = 28.5f;        // e^-28.5 * 2^40 rounds to 0
constexpr float kWeightOne = 1099511627776.0f;  // 2^40
static_assert(kBins == 2 * kSmpThreads && kList == 4 * kSmpThreads, "bins and entries a thread");

struct Exchange {  // what a CTA tells its cluster; two, used in turn
  float top, low;
  int top_at;
  unsigned long long a, b, c;
};

struct SmpShared {
  uint64_t list[kList];
  uint32_t count[kBins], place[kBins];
  Exchange ex[2];
  unsigned long long warp64[kSmpWarps];
  float warp_top[kSmpWarps], warp_low[kSmpWarps];
  int warp_at[kSmpWarps];
  uint32_t warp_cnt[kSmpWarps];
  float warp_mass[kSmpWarps];
  int n_list, found;
  int bin_k, bin_p;
  uint32_t before_k;
  float mass_k;
  unsigned long long reply;  // the leader's answer to its cluster
  int again;
};

__device__ __forceinline__ uint32_t ld_cluster32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 ld_cluster32x2(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ unsigned long long ld_cluster64(uint32_t a) {
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
  return v;
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
// a NaN is never drawn
__device__ __forceinline__ float clean(float z) { return z == z ? z : -INFINITY; }

// ascending keys: z descending, then index ascending
__device__ __forceinline__ uint64_t entry_key(float z, int i) {
  const uint32_t u = __float_as_uint(z == 0.f ? 0.f : z);  // both zeros are equal
  const uint32_t up = u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
  return (uint64_t)(~up) << 32 | (uint32_t)i;
}
__device__ __forceinline__ float key_z(uint64_t key) {
  const uint32_t up = ~(uint32_t)(key >> 32);
  return __uint_as_float(up ^ ((up >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}

__device__ __forceinline__ unsigned long long warp_sum64(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ unsigned long long warp_scan64(unsigned long long v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += t;
  }
  return v;
}

// A row's shared state and the passes over one CTA's slice of it.
template <typename T>
struct Row {
  SmpShared& sh;
  const T* buf;    // this CTA's entries
  int lo, n;       // their first index, and how many
  int rank, size;  // place in the cluster
  int tid, lane, warp;
  int turn;        // which exchange is next
  float top, temp, scale, range, log_min_p;

  __device__ float z(int i) const { return clean(to_f32(buf[i])); }
  __device__ float dist(float v) const { return v == top ? 0.f : top - v; }
  __device__ int bin(float d) const { return min(kBins - 1, (int)(d * scale)); }
  __device__ float expo(float v) const { return v == top ? 0.f : __fdiv_rn(v - top, temp); }
  __device__ float weight(float v) const { return v == -INFINITY ? 0.f : expf(expo(v)); }
  // w >= min_p, told by the exponents: next to 1 the weights have no bits left
  __device__ bool likely(float v) const { return expo(v) >= log_min_p; }
  __device__ unsigned long long whole(float w) const { return (unsigned long long)__float2ll_rn(w * kWeightOne); }
  __device__ unsigned long long mass(float v) const { return dist(v) > range ? 0ull : whole(weight(v)); }

  // sums of three 64-bit values over the CTA
  __device__ void block_sum(unsigned long long (&v)[3]) {
#pragma unroll
    for (int e = 0; e < 3; ++e) {
      const unsigned long long w = warp_sum64(v[e]);
      __syncthreads();
      if (lane == 0) sh.warp64[warp] = w;
      __syncthreads();
      unsigned long long t = 0;
      for (int i = 0; i < kSmpWarps; ++i) t += sh.warp64[i];
      v[e] = t;
    }
  }
  // and over the cluster
  __device__ void cluster_total(unsigned long long (&v)[3]) {
    block_sum(v);
    Exchange* mine = &sh.ex[turn];
    if (tid == 0) { mine->a = v[0]; mine->b = v[1]; mine->c = v[2]; }
    cluster_sync();
    v[0] = v[1] = v[2] = 0;
    for (int r = 0; r < size; ++r) {
      v[0] += ld_cluster64(mapa_shared(&mine->a, r));
      v[1] += ld_cluster64(mapa_shared(&mine->b, r));
      v[2] += ld_cluster64(mapa_shared(&mine->c, r));
    }
    turn ^= 1;
  }

  // Entries of bins [b0, b1] at or before `most` into this CTA's list (the
  // caller knows that they fit).
  __device__ void collect(int b0, int b1, uint64_t most) {
    __syncthreads();
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kSmpThreads) {
      const float v = z(i), d = dist(v);
      if (d > range) continue;
      const int b = bin(d);
      if (b < b0 || b > b1) continue;
      const uint64_t key = entry_key(v, lo + i);
      if (key <= most) {
        const int at = atomicAdd(&sh.n_list, 1);
        if (at < kList) sh.list[at] = key;
      }
    }
    __syncthreads();
  }
  // The leader's list takes the other CTAs' entries; returns the total.  A
  // cluster_sync lies between collect() and this.
  __device__ int pull() {
    int total = min(sh.n_list, kList);
    for (int r = 1; r < size; ++r) {
      const int c = min((int)ld_cluster32(mapa_shared(&sh.n_list, r)), kList - total);
      const uint32_t from = mapa_shared(sh.list, r);
      for (int i = tid; i < c; i += kSmpThreads) sh.list[total + i] = ld_cluster64(from + 8 * i);
      total += c;
    }
    __syncthreads();
    return total;
  }
  // Sorts the list's first m entries, ascending; returns the padded length.
  __device__ int sort(int m) {
    int len = 2;
    while (len < m) len <<= 1;
    for (int i = m + tid; i < len; i += kSmpThreads) sh.list[i] = ~0ull;
    __syncthreads();
    for (int k = 2; k <= len; k <<= 1)
      for (int j = k >> 1; j > 0; j >>= 1) {
        for (int t = tid; t < len / 2; t += kSmpThreads) {
          const int i = 2 * t - (t & (j - 1)), p = i + j;
          const uint64_t x = sh.list[i], y = sh.list[p];
          if ((x > y) == ((i & k) == 0)) { sh.list[i] = y; sh.list[p] = x; }
        }
        __syncthreads();
      }
    return len;
  }
  // Of four consecutive weights a thread: what lies before the thread's first.
  __device__ unsigned long long scan_before(const unsigned long long (&v)[4]) {
    const unsigned long long own = v[0] + v[1] + v[2] + v[3];
    const unsigned long long inc = warp_scan64(own, lane);
    __syncthreads();
    if (lane == 31) sh.warp64[warp] = inc;
    __syncthreads();
    unsigned long long before = inc - own;
    for (int i = 0; i < warp; ++i) before += sh.warp64[i];
    return before;
  }

  // Smallest key whose entries up to it (at or before `most`) reach `bar`:
  // their count, or their mass.  The answer lies in bin b.
  __device__ uint64_t bisect(int b, bool by_mass, double bar, uint64_t most) {
    uint32_t zl = 0xFFFFFFFFu, zh = 0;
    for (int i = tid; i < n; i += kSmpThreads) {
      const float v = z(i), d = dist(v);
      if (d > range || bin(d) != b) continue;
      const uint32_t k = (uint32_t)(entry_key(v, 0) >> 32);
      zl = min(zl, k);
      zh = max(zh, k);
    }
    zl = __reduce_min_sync(0xffffffffu, zl);
    zh = __reduce_max_sync(0xffffffffu, zh);
    __syncthreads();
    if (lane == 0) sh.warp64[warp] = (unsigned long long)zl << 32 | zh;
    __syncthreads();
    for (int i = 0; i < kSmpWarps; ++i) {
      zl = min(zl, (uint32_t)(sh.warp64[i] >> 32));
      zh = max(zh, (uint32_t)sh.warp64[i]);
    }
    Exchange* mine = &sh.ex[turn];
    if (tid == 0) mine->a = (unsigned long long)zl << 32 | zh;
    cluster_sync();
    for (int r = 0; r < size; ++r) {
      const unsigned long long v = ld_cluster64(mapa_shared(&mine->a, r));
      zl = min(zl, (uint32_t)(v >> 32));
      zh = max(zh, (uint32_t)v);
    }
    turn ^= 1;
    // over z, then over the index among the entries of that z
    while (zl < zh) {
      const uint32_t mid = zl + (zh - zl) / 2;
      if (reaches((uint64_t)mid << 32 | 0xFFFFFFFFu, by_mass, bar, most)) zh = mid; else zl = mid + 1;
    }
    uint32_t il = 0, ih = (uint32_t)kSampleMaxVocab;
    while (il < ih) {
      const uint32_t mid = il + (ih - il) / 2;
      if (reaches((uint64_t)zl << 32 | mid, by_mass, bar, most)) ih = mid; else il = mid + 1;
    }
    return (uint64_t)zl << 32 | il;
  }
  __device__ bool reaches(uint64_t key, bool by_mass, double bar, uint64_t most) {
    key = key < most ? key : most;
    unsigned long long v[3] = {0, 0, 0};
    for (int i = tid; i < n; i += kSmpThreads) {
      const float f = z(i);
      if (entry_key(f, lo + i) <= key) v[0] += by_mass ? mass(f) : 1ull;
    }
    cluster_total(v);
    return (double)v[0] >= bar;
  }
};

}  // namespace

template <typename T>
__global__ void __launch_bounds__(kSmpThreads, 2) sample_kernel(const SampleArgs a, int per_cta) {
  extern __shared__ __align__(16) uint8_t smem[];
  SmpShared& sh = *reinterpret_cast<SmpShared*>(smem);
  uint8_t* raw = smem + (sizeof(SmpShared) + 15) / 16 * 16;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster_rank(), size = (int)cluster_size();
  const int row = blockIdx.x / size;
  const int lo = min(rank * per_cta, a.vocab), n = min(per_cta, a.vocab - lo);
  const T* src = reinterpret_cast<const T*>(a.logits) + (int64_t)row * a.stride + lo;
  // the slice lies in shared memory at its global address modulo 16, so that
  // its middle moves in 16-byte pieces whatever the row's alignment
  const int shift = (int)(reinterpret_cast<uintptr_t>(src) & 15);
  T* buf = reinterpret_cast<T*>(raw + shift);
  const int head = min(n, shift ? (16 - shift) / (int)sizeof(T) : 0);
  constexpr int kPer = 16 / (int)sizeof(T);
  const int pieces = (n - head) / kPer;

  float top = -INFINITY, low = INFINITY;
  int top_at = 0x7FFFFFFF;
  auto see = [&](float v, int i) {
    v = clean(v);
    if (v > top || (v == top && i < top_at)) { top = v; top_at = i; }
    if (v > -INFINITY) low = fminf(low, v);
  };
  {
    const uint4* s4 = reinterpret_cast<const uint4*>(src + head);
    uint4* d4 = reinterpret_cast<uint4*>(buf + head);
    for (int p0 = 0; p0 < pieces; p0 += 8 * kSmpThreads) {
      uint4 v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int p = p0 + e * kSmpThreads + tid;
        if (p < pieces) v[e] = __ldcs(s4 + p);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int p = p0 + e * kSmpThreads + tid;
        if (p >= pieces) continue;
        d4[p] = v[e];
        const T* q = reinterpret_cast<const T*>(&v[e]);
#pragma unroll
        for (int j = 0; j < kPer; ++j) see(to_f32(q[j]), lo + head + p * kPer + j);
      }
    }
    const int tail = n - head - pieces * kPer;
    if (tid < head + tail) {
      const int i = tid < head ? tid : n - tail + (tid - head);
      const T v = src[i];
      buf[i] = v;
      see(to_f32(v), lo + i);
    }
  }
  for (int i = tid; i < kBins; i += kSmpThreads) sh.count[i] = sh.place[i] = 0;
  // the row's largest entry (its lowest index) and smallest finite one
  warp_argmax(top, top_at);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
  if (lane == 0) { sh.warp_top[warp] = top; sh.warp_at[warp] = top_at; sh.warp_low[warp] = low; }
  __syncthreads();
  for (int i = 0; i < kSmpWarps; ++i) {
    argmax_merge(top, top_at, sh.warp_top[i], sh.warp_at[i]);
    low = fminf(low, sh.warp_low[i]);
  }
  if (tid == 0) { sh.ex[0].top = top; sh.ex[0].top_at = top_at; sh.ex[0].low = low; }
  cluster_sync();
#pragma unroll 1
  for (int r = 0; r < size; ++r) {
    const float t = __uint_as_float(ld_cluster32(mapa_shared(&sh.ex[0].top, r)));
    argmax_merge(top, top_at, t, (int)ld_cluster32(mapa_shared(&sh.ex[0].top_at, r)));
    low = fminf(low, __uint_as_float(ld_cluster32(mapa_shared(&sh.ex[0].low, r))));
  }
  const float temp = a.temperature ? a.temperature[row] : 1.0f;
  if (top == -INFINITY || !(temp > 0.f)) {  // nothing to draw from, or the largest entry
    if (rank == 0 && tid == 0) {
      a.token[row] = top == -INFINITY ? -1 : top_at;
      a.logprob[row] = top == -INFINITY ? -INFINITY : 0.f;
    }
    cluster_sync();  // no CTA leaves while another reads its shared memory
    return;
  }
  const float p = a.top_p ? a.top_p[row] : 1.0f;
  const float min_p = a.min_p ? fminf(a.min_p[row], 1.0f) : 0.f;
  const float log_min_p = min_p > 0.f ? logf(min_p) : -INFINITY;
  const double u = (double)fminf(fmaxf(a.u[row], 0.f), 0.99999994f);
  const int k = a.top_k ? a.top_k[row] : 0;
  bool need_k = k > 0 && k < a.vocab, need_p = p < 1.0f;
  const float range = fminf(kRange * temp, top - low);
  Row<T> R{sh, buf, lo, n, rank, size, tid, lane, warp, 1, top, temp, range > 1e-30f ? kBins / range : 0.f, range, log_min_p};

  uint64_t last = ~0ull;  // the last entry that top-k and top-p keep
  if (need_k || need_p) {
    // ---- histogram over the distance from the largest entry ------------------
    for (int i = tid; i < n; i += kSmpThreads) {
      const float d = R.dist(R.z(i));
      if (d > range) continue;
      const int b = R.bin(d);
      atomicAdd(&sh.count[b], 1u);
      if (need_p) atomicAdd(&sh.place[b], (uint32_t)(fminf(fmaxf(d * R.scale - b, 0.f), 1.f) * 65535.f));
    }
    cluster_sync();
    uint32_t cnt[2] = {0, 0};
    float plc[2] = {0.f, 0.f};
    for (int r = 0; r < size; ++r) {
      const uint2 c = ld_cluster32x2(mapa_shared(&sh.count[2 * tid], r));
      cnt[0] += c.x;
      cnt[1] += c.y;
      if (need_p) {
        const uint2 q = ld_cluster32x2(mapa_shared(&sh.place[2 * tid], r));
        plc[0] += q.x * (1.f / 65535.f);
        plc[1] += q.y * (1.f / 65535.f);
      }
    }
    // a bin's mass from its count and its entries' mean place within it
    const float step = R.scale > 0.f ? 1.f / (R.scale * temp) : 0.f;
    float ms[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (need_p && cnt[e]) ms[e] = cnt[e] * __expf(-(2 * tid + e + plc[e] / cnt[e]) * step);
    uint32_t ci = cnt[0] + cnt[1];
    float mi = ms[0] + ms[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t tc = __shfl_up_sync(0xffffffffu, ci, o);
      const float tm = __shfl_up_sync(0xffffffffu, mi, o);
      if (lane >= o) { ci += tc; mi += tm; }
    }
    if (lane == 31) { sh.warp_cnt[warp] = ci; sh.warp_mass[warp] = mi; }
    if (tid == 0) { sh.bin_k = -1; sh.bin_p = kBins - 1; }
    __syncthreads();
    uint32_t n_all = 0;
    float m_all = 0.f, m_mine = 0.f;
    for (int i = 0; i < kSmpWarps; ++i) {
      if (i == warp) { ci += n_all; m_mine = m_all; }
      n_all += sh.warp_cnt[i];
      m_all += sh.warp_mass[i];
    }
    mi += m_mine;
    // cumulative up to and including each of this thread's two bins
    const uint32_t cc[2] = {ci - cnt[1], ci};
    const float mm[2] = {mi - ms[1], mi};
    need_k = need_k && n_all >= (uint32_t)k;  // else all that can be drawn is kept
    if (need_k) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (cc[e] >= (uint32_t)k && cc[e] - cnt[e] < (uint32_t)k) {
          sh.bin_k = 2 * tid + e;
          sh.before_k = cc[e] - cnt[e];
          // the top-k's mass, its last bin's taken in proportion
          sh.mass_k = mm[e] - ms[e] + ms[e] * ((float)(k - (int)(cc[e] - cnt[e])) / cnt[e]);
        }
    }
    __syncthreads();
    if (need_p) {
      const float m_bar = p * (need_k ? sh.mass_k : m_all);
      const int at = p <= 0.f ? 0 : mm[0] >= m_bar ? 2 * tid : mm[1] >= m_bar ? 2 * tid + 1 : kBins - 1;
      const int first = __reduce_min_sync(0xffffffffu, at);
      if (lane == 0) atomicMin(&sh.bin_p, first);
    }
    __syncthreads();
    const int bin_k = sh.bin_k;
    int bin_p = sh.bin_p;
    if (need_k && bin_p > bin_k) bin_p = bin_k;
    // entries up to a bin, from the thread that holds it
    const int few_bin = need_k ? bin_k : min(bin_p + 2, kBins - 1);
    if (tid == 0) sh.found = 0;
    __syncthreads();
    if ((few_bin >> 1) == tid) sh.found = (int)cc[few_bin & 1];
    __syncthreads();
    const int few = sh.found;
    if ((need_k || need_p) && few <= kList) {
      // ---- A, B: one CTA sorts all that can be kept ----------------------------
      unsigned long long sums[3] = {0, 0, 0};
      R.collect(0, few_bin, ~0ull);
      if (!need_k) {
        for (int i = tid; i < n; i += kSmpThreads) sums[0] += R.mass(R.z(i));
        R.cluster_total(sums);
      } else {
        cluster_sync();
      }
      if (rank == 0) {
        const int m = R.pull();
        R.sort(m);
        unsigned long long W[4];
        bool fits[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * tid + e;
          const bool in = i < m && (!need_k || i < k);
          const float v = in ? key_z(sh.list[i]) : -INFINITY;
          W[e] = R.whole(R.weight(v));
          fits[e] = in && R.likely(v);
        }
        unsigned long long before = R.scan_before(W);
        unsigned long long all = 0;  // the list's mass: the top-k's
        for (int i = 0; i < kSmpWarps; ++i) all += sh.warp64[i];
        const double bar = (double)p * (double)(need_k ? all : sums[0]);
        const int limit = need_k ? min(m, k) : m;
        const bool short_list = need_p && !need_k && (double)all < bar;
        // kept entries are a prefix: the weights fall along the list
        int kept = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * tid + e;
          if (i < limit && (i == 0 || ((!need_p || (double)before < bar) && fits[e]))) kept = i + 1;
          before += W[e];
        }
        if (tid == 0) { sh.found = 1; sh.again = short_list; }
        __syncthreads();
        atomicMax(&sh.found, kept);
        __syncthreads();
        const int m2 = sh.found;
        if (!short_list) {
          // the kept entries in index order: (index, z's key)
          __syncthreads();
          for (int i = tid; i < m2; i += kSmpThreads) {
            const uint64_t key = sh.list[i];
            sh.list[i] = key << 32 | key >> 32;
          }
          R.sort(m2);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * tid + e;
            W[e] = i < m2 ? R.whole(R.weight(key_z(sh.list[i] << 32))) : 0ull;
          }
          unsigned long long upto = R.scan_before(W);
          unsigned long long S = 0;
          for (int i = 0; i < kSmpWarps; ++i) S += sh.warp64[i];
          const double t = u * (double)S;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * tid + e;
            const double was = (double)upto;
            upto += W[e];
            if (i < m2 && (double)upto > t && (i == 0 || was <= t)) {
              a.token[row] = (int)(sh.list[i] >> 32);
              a.logprob[row] = -log1pf((float)(S - W[e]) / (float)W[e]);
            }
          }
        }
      }
      cluster_sync();
      if (need_k || !ld_cluster32(mapa_shared(&sh.again, 0))) {
        cluster_sync();
        return;
      }
      cluster_sync();
    }
    // ---- C: the last entry of the top-k, then that of the nucleus --------------
    // answers: the leader sorts a bin's entries and replies with a key
    if (need_k) {
      __syncthreads();
      if ((bin_k >> 1) == tid) sh.found = (int)cnt[bin_k & 1];
      __syncthreads();
      if (sh.found <= kList) {
        const uint32_t before_k = sh.before_k;
        R.collect(bin_k, bin_k, ~0ull);
        cluster_sync();
        if (rank == 0) {
          R.sort(R.pull());
          if (tid == 0) sh.reply = sh.list[k - 1 - before_k];
        }
        cluster_sync();
        last = ld_cluster64(mapa_shared(&sh.reply, 0));
        cluster_sync();
      } else {
        last = R.bisect(bin_k, false, (double)k, ~0ull);
      }
    }
    if (need_p) {
      const uint64_t most = last;
      unsigned long long v[3];
      double bar;
      // exact masses before and in the bin; the estimate is rarely a bin off
      while (true) {
        v[0] = v[1] = v[2] = 0;
        for (int i = tid; i < n; i += kSmpThreads) {
          const float f = R.z(i), d = R.dist(f);
          if (d > range || entry_key(f, lo + i) > most) continue;
          const unsigned long long W = R.whole(R.weight(f));
          const int b = R.bin(d);
          v[0] += W;
          if (b < bin_p) v[1] += W;
          if (b == bin_p) v[2] += W;
        }
        R.cluster_total(v);
        bar = (double)p * (double)v[0];
        if (bin_p > 0 && (double)v[1] >= bar) --bin_p;
        else if (bin_p < kBins - 1 && (double)(v[1] + v[2]) < bar) ++bin_p;
        else break;
      }
      __syncthreads();
      if ((bin_p >> 1) == tid) sh.found = (int)cnt[bin_p & 1];
      __syncthreads();
      if (sh.found <= kList) {
        R.collect(bin_p, bin_p, most);
        cluster_sync();
        if (rank == 0) {
          const int m = R.pull();
          R.sort(m);
          unsigned long long W[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * tid + e;
            W[e] = i < m ? R.whole(R.weight(key_z(sh.list[i]))) : 0ull;
          }
          unsigned long long before = v[1] + R.scan_before(W);
          if (tid == 0) sh.found = 1;
          __syncthreads();
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * tid + e;
            if (i < m && (double)before < bar) atomicMax(&sh.found, i + 1);
            before += W[e];
          }
          __syncthreads();
          if (tid == 0) sh.reply = sh.list[sh.found - 1];
        }
        cluster_sync();
        last = ld_cluster64(mapa_shared(&sh.reply, 0));
      } else {
        last = R.bisect(bin_p, true, bar, most);
      }
    }
  }
  // ---- the draw, in index order: warps own consecutive ranges ------------------
  const int per_warp = (n + 32 * kSmpWarps - 1) / (32 * kSmpWarps) * 32;
  const int w0 = min(n, warp * per_warp), w1 = min(n, w0 + per_warp);
  auto kept_mass = [&](int i) -> unsigned long long {
    const float v = R.z(i);
    if (R.dist(v) > range || entry_key(v, lo + i) > last) return 0ull;
    return R.likely(v) ? R.whole(R.weight(v)) : 0ull;
  };
  unsigned long long own = 0;
  for (int i = w0 + lane; i < w1; i += 32) own += kept_mass(i);
  own = warp_sum64(own);
  __syncthreads();
  if (lane == 0) sh.warp64[warp] = own;
  __syncthreads();
  unsigned long long mine = 0, before_warp = 0;
  for (int i = 0; i < kSmpWarps; ++i) {
    if (i == warp) before_warp = mine;
    mine += sh.warp64[i];
  }
  Exchange* e = &sh.ex[R.turn];
  if (tid == 0) e->a = mine;
  cluster_sync();
  unsigned long long S = 0, before = 0;
  for (int r = 0; r < size; ++r) {
    const unsigned long long v = ld_cluster64(mapa_shared(&e->a, r));
    if (r < rank) before += v;
    S += v;
  }
  const double t = u * (double)S;
  before += before_warp;
  // the first warp whose range passes the target; u < 1 keeps the target below S
  if (own && (double)before <= t && (double)(before + own) > t) {
    for (int i0 = w0; i0 < w1; i0 += 32) {
      const int i = i0 + lane;
      const unsigned long long W = i < w1 ? kept_mass(i) : 0ull;
      const unsigned long long inc = before + warp_scan64(W, lane);
      const uint32_t past = __ballot_sync(0xffffffffu, (double)inc > t);
      if (past) {
        if (lane == __ffs(past) - 1) {
          a.token[row] = lo + i;
          a.logprob[row] = -log1pf((float)(S - W) / (float)W);
        }
        break;
      }
      before = __shfl_sync(0xffffffffu, inc, 31);
    }
  }
  cluster_sync();
}

template <typename T>
static void run_sample(const SampleArgs& a, cudaStream_t s) {
  // as many CTAs a row as keep a slice within 64 KB; more where rows are few
  const int64_t bytes = (int64_t)a.vocab * sizeof(T);
  int size = (int)((bytes + kSliceBytes - 1) / kSliceBytes);
  while (size < kSmpMaxCluster && a.rows * size < 152 && a.vocab / (size + 1) >= 2048) ++size;
  if (size > kSmpMaxCluster) size = kSmpMaxCluster;
  const int per_cta = (a.vocab + 8 * size - 1) / (8 * size) * 8;
  const int smem = (int)((sizeof(SmpShared) + 15) / 16 * 16 + 16 + ((size_t)per_cta * sizeof(T) + 15) / 16 * 16);
  static int configured = 0;
  if (smem > configured) {
    const cudaError_t e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) throw e;
    configured = smem;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.rows * size);
  cfg.blockDim = dim3(kSmpThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, sample_kernel<T>, a, per_cta);
  if (e != cudaSuccess) throw e;
}

void launch_sample(const SampleArgs& a, cudaStream_t s) {
  if (a.dtype == DT_BF16) run_sample<__nv_bfloat16>(a, s);
  else if (a.dtype == DT_F16) run_sample<__half>(a, s);
  else run_sample<float>(a, s);
}

}  // namespace pard
