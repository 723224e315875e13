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
// A cluster of up to eight CTAs holds a row, an index range each, in shared
// memory, so each logit is read once.  Nothing is sorted or compared but the
// entries that a cut can depend on:
//   A  top-k: any k entries bound the k-th from below; the threads' largest
//      entries (4096 a row) are counted into 1024 bins over max z - z, and the
//      entries up to the k-th one's bin, a few more than k, go to one CTA, which
//      does the rest: up to 256 are compared each with all others, which gives
//      every one its place and the mass before it in one step where a sort is a
//      chain of them; more are sorted;
//   B  top-p alone: counts of the largest entries, and of one in eight of the
//      others, give each bin's mass and its error; between the bins where the cut
//      may lie by five of these errors, one pass has all entries by finer bins, and
//      the exact masses of what is kept for sure and of all; every CTA compares the
//      entries of the fine bin that the cut falls into;
//   C  whatever these do not cover (ties by the thousand, extreme temperatures, a
//      guess that failed): a histogram of all entries, exact masses around the
//      cut's bin, and, in a bin of more than 2048 entries, bisection over (z, i).
// The draw is a scan in index order: masses of CTAs, then of warps' ranges, then
// of the entries of the one range that the target falls into.
//
// What bounds it.  Many rows: the latency of the steps.  464 rows of 128256
// floats take 201 to 210 us, a sixth of HBM's rate (35 us): a top-p row 55000 clocks,
// of which the exact pass is 10000 (40 instructions an entry), reading 6000,
// and the rest some fifteen meetings of a CTA or the cluster; a top-k row 20000
// and its leader 10000 more.  Two CTAs an SM overlap (issue slots 41% busy); 16
// warps each, two slices, are what shared memory holds, and reading the row from
// L2 in every pass instead, with four CTAs an SM, took 1081 us.  One row: 10 us.
#include <cuda_fp16.h>

#include "common.cuh"
#include "per_device.h"
#include "tree.h"

namespace pard {

namespace {

constexpr int kSmpThreads = 512;
constexpr int kSmpWarps = kSmpThreads / 32;
constexpr int kBins = 1024;
constexpr int kFine = 256;             // bins of the entries that a cut may fall among
constexpr int kList = 2048;            // entries one CTA sorts
constexpr int kFew = 256;              // up to here, each is compared with all others instead
constexpr int kSmpMaxCluster = 8;
constexpr float kRange = 28.5f;        // e^-28.5 * 2^40 rounds to 0
constexpr float kWeightOne = 1099511627776.0f;  // 2^40
static_assert(kBins == 2 * kSmpThreads && kList == 4 * kSmpThreads && 2 * kFine == kSmpThreads && 2 * kFew == kSmpThreads,
              "bins and entries a thread");

struct Exchange {  // what a CTA tells its cluster; two, used in turn
  float top, low;
  int n;
  unsigned long long a, b, c;
};

// Whole weights rint(w 2^40) summed in 32-bit halves at full rate: a sum with
// 1.5 * 2^23 leaves a whole number in the low bits, which add as integers (a
// lane has at most 256 weights of a row: the halves stay within 32 bits).
struct Halves {
  int hi = 0, lo = 0;
  static constexpr float kMagic = 12582912.0f;  // 1.5 * 2^23
  static __device__ __forceinline__ Halves of(float w) {
    const float a = fmaf(w, 1048576.0f, kMagic), h = a - kMagic;          // rint(w 2^20)
    const float b = fmaf(fmaf(w, 1048576.0f, -h), 1048576.0f, kMagic);    // the rest, in 2^-40
    return {__float_as_int(a) - 0x4B400000, __float_as_int(b) - 0x4B400000};
  }
  __device__ __forceinline__ void add(Halves w, bool in = true) {
    hi += in ? w.hi : 0;
    lo += in ? w.lo : 0;
  }
  __device__ __forceinline__ unsigned long long total() const { return (unsigned long long)((long long)hi * 1048576 + lo); }
};

struct SmpShared {
  uint64_t list[kList];
  struct alignas(16) Pair { unsigned long long key, mass; };
  // `few` follows after the counts' last use by any CTA
  union {
    struct { uint32_t count[kBins], place[kBins]; };
    Pair few[kFew];
  };
  unsigned long long mass[kFine];
  uint64_t cut[kFew];
  Exchange ex[2];
  unsigned long long warp64[kSmpWarps], above[kSmpWarps], part[3][kSmpWarps];
  int first[kSmpMaxCluster + 1];
  float warp_top[kSmpWarps], warp_low[kSmpWarps];
  uint32_t warp_cnt[kSmpWarps];
  float warp_mass[kSmpWarps];
  int n_list, found;
  int bin_k, bin_p;
  uint32_t before_k;
  float mass_k, warp_var[kSmpWarps];
  unsigned long long reply;  // the leader's answer to its cluster
  unsigned long long cut_key;
  int n_cut;
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
  float top, temp, inv_temp, scale, range, log_min_p;
  bool tame;       // finite, and far from the ends of the exponents' range

  __device__ float z(int i) const { return clean(to_f32(buf[i])); }
  __device__ float dist(float v) const { return v == top ? 0.f : top - v; }
  __device__ int bin(float d) const { return min(kBins - 1, (int)(d * scale)); }
  // (v - top) / temp, correctly rounded: the reciprocal's product and one
  // correction by its exact remainder (Markstein, IBM J. Res. Dev. 34, 1990),
  // where nothing over- or underflows on the way, else the division
  __device__ float expo(float v) const {
    const float d = v - top;
    if (!tame) return v == top ? 0.f : __fdiv_rn(d, temp);
    const float q = d * inv_temp;
    return fmaf(fmaf(-q, temp, d), inv_temp, q);
  }
  __device__ float weight(float v) const { return v == -INFINITY ? 0.f : expf(expo(v)); }
  // w >= min_p, told by the exponents: next to 1 the weights have no bits left
  __device__ bool likely(float v) const { return expo(v) >= log_min_p; }
  __device__ unsigned long long whole(float w) const { return (unsigned long long)__float2ll_rn(w * kWeightOne); }
  __device__ unsigned long long mass(float v) const { return dist(v) > range ? 0ull : whole(weight(v)); }
  // place among the bins, as a real number; more than kBins: no weight
  __device__ float place(float v) const { return (top - v) * scale; }

  // what an entry of a place before p has at least, and some others have too
  __device__ float at_least(float p) const { return __fsub_rd(top, (p + 1.f) / scale); }

  // a word of every CTA of the cluster, summed: a lane reads one
  __device__ int cluster_int(const int* mine) {
    return (int)__reduce_add_sync(0xffffffffu, lane < size ? ld_cluster32(mapa_shared(mine, lane)) : 0u);
  }
  __device__ unsigned long long cluster_sum64(const unsigned long long* mine) {
    return warp_sum64(lane < size ? ld_cluster64(mapa_shared(mine, lane)) : 0ull);
  }
  // the warps' values that lie in shared memory: all of them, and those before this one
  __device__ unsigned long long warps_total(const unsigned long long* of, unsigned long long* before) {
    const unsigned long long x = lane < kSmpWarps ? of[lane] : 0ull;
    *before = warp_sum64(lane < warp ? x : 0ull);
    return warp_sum64(x);
  }
  // sums of three 64-bit values over the cluster
  __device__ void cluster_total(unsigned long long (&v)[3]) {
#pragma unroll
    for (int e = 0; e < 3; ++e) {
      v[e] = warp_sum64(v[e]);
      if (lane == 0) sh.part[e][warp] = v[e];
    }
    __syncthreads();
    Exchange* mine = &sh.ex[turn];
    if (warp == 0) {
      unsigned long long b, t[3];
#pragma unroll
      for (int e = 0; e < 3; ++e) t[e] = warps_total(sh.part[e], &b);
      if (lane == 0) { mine->a = t[0]; mine->b = t[1]; mine->c = t[2]; }
    }
    cluster_sync();
    v[0] = cluster_sum64(&mine->a);
    v[1] = cluster_sum64(&mine->b);
    v[2] = cluster_sum64(&mine->c);
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
    const int c = lane < size ? min((int)ld_cluster32(mapa_shared(&sh.n_list, lane)), kList) : 0;
    int inc = c;
#pragma unroll
    for (int o = 1; o < kSmpMaxCluster; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += t;
    }
    if (warp == 0 && lane <= kSmpMaxCluster) sh.first[lane] = lane < kSmpMaxCluster ? inc - c : inc;
    const int total = min(__shfl_sync(0xffffffffu, inc, kSmpMaxCluster - 1), kList);
    __syncthreads();
    const int own = sh.first[1];
    for (int i = own + tid; i < total; i += kSmpThreads) {
      int r = 1;
#pragma unroll
      for (int e = 2; e < kSmpMaxCluster; ++e) r += i >= sh.first[e];
      sh.list[i] = ld_cluster64(mapa_shared(sh.list, r) + 8 * (i - sh.first[r]));
    }
    __syncthreads();
    return total;
  }
  // Sorts the list's first m entries, ascending: bitonic, an entry a thread in
  // registers (steps within a warp are shuffles) for up to 512, else in place.
  __device__ void sort(int m) {
    int len = 32;
    while (len < m) len <<= 1;
    if (len <= kSmpThreads) {
      uint64_t x = tid < m ? sh.list[tid] : ~0ull;
#pragma unroll 1
      for (int k = 2; k <= len; k <<= 1)
#pragma unroll 1
        for (int j = k >> 1; j > 0; j >>= 1) {
          uint64_t y;
          if (j >= 32) {
            __syncthreads();
            sh.list[tid] = x;
            __syncthreads();
            y = sh.list[tid ^ j];
          } else {
            y = __shfl_xor_sync(0xffffffffu, x, j);
          }
          const bool low = ((tid & j) == 0) == ((tid & k) == 0);  // this thread keeps the smaller
          x = low ? (x < y ? x : y) : (x < y ? y : x);
        }
      __syncthreads();
      sh.list[tid] = x;
      __syncthreads();
      return;
    }
    for (int i = m + tid; i < len; i += kSmpThreads) sh.list[i] = ~0ull;
    __syncthreads();
#pragma unroll 1
    for (int k = 2; k <= len; k <<= 1)
#pragma unroll 1
      for (int j = k >> 1; j > 0; j >>= 1) {
        for (int t = tid; t < len / 2; t += kSmpThreads) {
          const int i = 2 * t - (t & (j - 1)), p = i + j;
          const uint64_t x = sh.list[i], y = sh.list[p];
          if ((x > y) == ((i & k) == 0)) { sh.list[i] = y; sh.list[p] = x; }
        }
        __syncthreads();
      }
  }
  // Of four consecutive weights a thread: what lies before the thread's first,
  // and the total.
  __device__ unsigned long long scan_before(const unsigned long long (&v)[4], unsigned long long* total) {
    const unsigned long long own = v[0] + v[1] + v[2] + v[3];
    const unsigned long long inc = warp_scan64(own, lane);
    __syncthreads();
    if (lane == 31) sh.warp64[warp] = inc;
    __syncthreads();
    unsigned long long before;
    *total = warps_total(sh.warp64, &before);
    return before + inc - own;
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
    {
      const unsigned long long v = ld_cluster64(mapa_shared(&mine->a, lane < size ? lane : 0));
      zl = __reduce_min_sync(0xffffffffu, min(zl, (uint32_t)(v >> 32)));
      zh = __reduce_max_sync(0xffffffffu, max(zh, (uint32_t)v));
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
  // Of the up to kFew entries in sh.few and this thread's, entry `e`: how many
  // come before it, and their mass.  Threads of one entry are neighbours, `parts`
  // of them, and each looks at every parts-th.
  template <typename Before>
  __device__ void few_before(int m, int e, int parts, Before&& is_before, int* rank_of, unsigned long long* mass_of) {
    int r = 0;
    unsigned long long b = 0;
    if (e - (lane / parts) < m) {
#pragma unroll 4
      for (int j = tid % parts; j < m; j += parts) {
        const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(&sh.few[j]);
        if (is_before(o.x)) { ++r; b += o.y; }
      }
      for (int o = parts / 2; o > 0; o >>= 1) {
        r += __shfl_xor_sync(0xffffffffu, r, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
      }
    }
    *rank_of = r;
    *mass_of = b;
  }
  // sum of one value a thread over the CTA
  __device__ unsigned long long block_sum64(unsigned long long v) {
    v = warp_sum64(v);
    if (lane == 0) sh.warp64[warp] = v;
    __syncthreads();
    return warp_sum64(lane < kSmpWarps ? sh.warp64[lane] : 0ull);
  }
  // finish_list for up to kFew entries: each thread (or two, or four) compares its
  // entry with all others, which takes fewer dependent steps than sorting.
  __device__ void finish_few(int m, int k, bool need_p, float p, double u, int32_t* token, float* logprob) {
    const int parts = m <= kFew / 2 ? 4 : 2, e = tid / parts;
    const bool own = e < m && tid % parts == 0;
    const uint64_t key = e < m ? sh.list[e] : ~0ull;
    const float v = key_z(key);
    const unsigned long long W = e < m ? whole(weight(v)) : 0ull;
    if (own) sh.few[e] = {key, W};
    __syncthreads();
    int r;
    unsigned long long before;
    few_before(m, e, parts, [&](unsigned long long o) { return o < key; }, &r, &before);
    const unsigned long long all = block_sum64(own && r < k ? W : 0ull);  // the top-k's mass
    const double bar = (double)p * (double)all;
    const bool kept = own && r < k && (r == 0 || (likely(v) && (!need_p || (double)before < bar)));
    // then in index order
    if (own) sh.few[e] = {key << 32 | key >> 32, kept ? W : 0ull};
    __syncthreads();
    const uint32_t index = (uint32_t)key;
    unsigned long long upto;
    few_before(m, e, parts, [&](unsigned long long o) { return (uint32_t)(o >> 32) < index; }, &r, &upto);
    const unsigned long long S = block_sum64(kept ? W : 0ull);
    const double t = u * (double)S;
    if (kept && (double)upto <= t && (double)(upto + W) > t) {
      *token = (int)index;
      *logprob = -log1pf((float)(S - W) / (float)W);
    }
  }
  // The cut among up to kFew entries of all CTAs (their n_cut and cut; a
  // cluster_sync lies before this): the last whose mass before it is below the
  // bar.  Every CTA finds it for itself.
  __device__ uint64_t cut_few(int m, unsigned long long from, double bar) {
    const int c = lane < size ? (int)ld_cluster32(mapa_shared(&sh.n_cut, lane)) : 0;
    int inc = c;
#pragma unroll
    for (int o = 1; o < kSmpMaxCluster; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += t;
    }
    const int exc = inc - c;
    const int e = tid / 2;
    int r = 0;
#pragma unroll
    for (int o = 0; o < kSmpMaxCluster - 1; ++o) r += e >= __shfl_sync(0xffffffffu, inc, o);
    const int at = e - __shfl_sync(0xffffffffu, exc, r);
    const uint64_t key = e < m ? ld_cluster64(mapa_shared(&sh.cut[at], r)) : ~0ull;
    if (e < m && (tid & 1) == 0) sh.few[e] = {key, mass(key_z(key))};
    __syncthreads();
    unsigned long long before;
    few_before(m, e, 2, [&](unsigned long long o) { return o < key; }, &r, &before);
    if (e < m && (tid & 1) == 0 && (double)(from + before) < bar) atomicMax(&sh.cut_key, (unsigned long long)key);
    __syncthreads();
    return sh.cut_key;
  }
  // Sorts the list's m entries and returns the last that a nucleus keeps, of
  // which `before` lies before the list: the last whose mass before it is below
  // the bar, or the first.
  __device__ uint64_t cut_list(int m, unsigned long long before, double bar) {
    sort(m);
    unsigned long long W[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 4 * tid + e;
      W[e] = i < m ? whole(weight(key_z(sh.list[i]))) : 0ull;
    }
    unsigned long long all;
    before += scan_before(W, &all);
    if (tid == 0) sh.found = 1;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 4 * tid + e;
      if (i < m && (double)before < bar) atomicMax(&sh.found, i + 1);
      before += W[e];
    }
    __syncthreads();
    return sh.list[sh.found - 1];
  }
  // The whole rest of a row whose first k entries are among the list's m: the
  // leader sorts them, cuts and draws.
  __device__ void finish_list(int m, int k, bool need_p, float p, double u, int32_t* token, float* logprob) {
    sort(m);
    unsigned long long W[4];
    bool fits[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 4 * tid + e;
      const bool in = i < m && i < k;
      const float v = in ? key_z(sh.list[i]) : -INFINITY;
      W[e] = whole(weight(v));
      fits[e] = in && likely(v);
    }
    unsigned long long all;  // the top-k's mass
    unsigned long long before = scan_before(W, &all);
    const double bar = (double)p * (double)all;
    // kept entries are a prefix: the weights fall along the list
    int kept = 1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 4 * tid + e;
      if (fits[e] && (!need_p || (double)before < bar)) kept = max(kept, i + 1);
      before += W[e];
    }
    if (tid == 0) sh.found = 1;
    __syncthreads();
    kept = __reduce_max_sync(0xffffffffu, kept);
    if (lane == 0) atomicMax(&sh.found, kept);
    __syncthreads();
    const int m2 = sh.found;
    __syncthreads();
    // the kept entries in index order: (index, z's key)
    for (int i = tid; i < m2; i += kSmpThreads) {
      const uint64_t key = sh.list[i];
      sh.list[i] = key << 32 | key >> 32;
    }
    sort(m2);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 4 * tid + e;
      W[e] = i < m2 ? whole(weight(key_z(sh.list[i] << 32))) : 0ull;
    }
    unsigned long long S, upto = scan_before(W, &S);
    const double t = u * (double)S;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 4 * tid + e;
      const double was = (double)upto;
      upto += W[e];
      if (i < m2 && (double)upto > t && (i == 0 || was <= t)) {
        *token = (int)(sh.list[i] >> 32);
        *logprob = -log1pf((float)(S - W[e]) / (float)W[e]);
      }
    }
  }
  __device__ unsigned long long kept_mass(int i, uint64_t last) const {
    const float v = z(i);
    if (dist(v) > range || entry_key(v, lo + i) > last) return 0ull;
    return likely(v) ? whole(weight(v)) : 0ull;
  }
  // The draw in index order, of kept entries (key up to `last`, likely enough);
  // `own`: the mass of this warp's range [w0, w1), the same in all its lanes.
  __device__ void draw(int w0, int w1, unsigned long long own, uint64_t last, double u, int32_t* token, float* logprob) {
    __syncthreads();
    if (lane == 0) sh.warp64[warp] = own;
    __syncthreads();
    unsigned long long own_before;
    const unsigned long long mine = warps_total(sh.warp64, &own_before);
    Exchange* e = &sh.ex[turn];
    if (tid == 0) e->a = mine;
    cluster_sync();
    const unsigned long long of = lane < size ? ld_cluster64(mapa_shared(&e->a, lane)) : 0ull;
    const unsigned long long S = warp_sum64(of);
    unsigned long long before = own_before + warp_sum64(lane < rank ? of : 0ull);
    const double t = u * (double)S;
    // this CTA reads no other's shared memory from here on
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    // the CTA, and in it the warp, whose range passes the target (u < 1 keeps it below S)
    if (mine && (double)(before - own_before) <= t && (double)(before - own_before + mine) > t) {
      if (lane == 0 && own && (double)before <= t && (double)(before + own) > t) {
        sh.first[0] = w0;
        sh.first[1] = w1;
        sh.reply = before;
      }
      __syncthreads();
      const int r0 = sh.first[0], r1 = sh.first[1];
      before = sh.reply;
      for (int i0 = r0; i0 < r1; i0 += 4 * kSmpThreads) {
        unsigned long long W[4], all;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int i = i0 + 4 * tid + q;
          W[q] = i < r1 ? kept_mass(i, last) : 0ull;
        }
        unsigned long long upto = before + scan_before(W, &all);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const double was = (double)upto;
          upto += W[q];
          if (W[q] && was <= t && (double)upto > t) {
            *token = lo + i0 + 4 * tid + q;
            *logprob = -log1pf((float)(S - W[q]) / (float)W[q]);
          }
        }
        before += all;
      }
    }
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
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
  const int pieces = (n - head) / kPer, tail = n - head - pieces * kPer;
  auto largest = [](const T* x) {
    float m = to_f32(x[0]);
#pragma unroll
    for (int e = 1; e < kPer; ++e) m = fmaxf(m, to_f32(x[e]));
    return m;
  };

  pdl_trigger();
  pdl_wait();
  const float temp = a.temperature ? a.temperature[row] : 1.0f;
  const float p = a.top_p ? a.top_p[row] : 1.0f;
  const float min_p = a.min_p ? fminf(a.min_p[row], 1.0f) : 0.f;
  const float log_min_p = min_p > 0.f ? logf(min_p) : -INFINITY;
  const double u = (double)fminf(fmaxf(a.u[row], 0.f), 0.99999994f);
  const int k = a.top_k ? a.top_k[row] : 0;
  float top = -INFINITY;  // a NaN is no maximum
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
        for (int j = 0; j < kPer; ++j) top = fmaxf(top, to_f32(q[j]));
      }
    }
    if (tid < head + tail) {
      const int i = tid < head ? tid : n - tail + (tid - head);
      const T v = src[i];
      buf[i] = v;
      top = fmaxf(top, to_f32(v));
    }
  }
  for (int i = tid; i < kBins; i += kSmpThreads) sh.count[i] = sh.place[i] = 0;
  // the row's largest entry
  const float thread_top = top;
  top = warp_max(top);
  if (lane == 0) sh.warp_top[warp] = top;
  __syncthreads();
  top = warp_max(sh.warp_top[lane % kSmpWarps]);
  if (tid == 0) sh.ex[0].top = top;
  cluster_sync();
  {
    const float t = lane < size ? __uint_as_float(ld_cluster32(mapa_shared(&sh.ex[0].top, lane))) : -INFINITY;
    top = warp_max(t);
  }
  // whatever follows, the row gets an answer
  if (rank == 0 && tid == 0) {
    a.token[row] = -1;
    a.logprob[row] = -INFINITY;
  }
  if (top == -INFINITY) {  // nothing to draw from
    cluster_sync();        // no CTA leaves while another reads its shared memory
    return;
  }
  if (!(temp > 0.f)) {  // the largest entry's lowest index
    int at = 0x7FFFFFFF;
    for (int i = n - 1 - tid; i >= 0; i -= kSmpThreads)
      if (to_f32(buf[i]) == top) at = lo + i;
    at = __reduce_min_sync(0xffffffffu, at);
    if (tid == 0) sh.found = 0x7FFFFFFF;
    __syncthreads();
    if (lane == 0) atomicMin(&sh.found, at);
    __syncthreads();
    if (tid == 0) sh.ex[1].n = sh.found;
    cluster_sync();
    if (rank == 0 && tid == 0) {
      for (int r = 0; r < size; ++r) at = min(at, (int)ld_cluster32(mapa_shared(&sh.ex[1].n, r)));
      a.token[row] = at;
      a.logprob[row] = 0.f;
    }
    cluster_sync();
    return;
  }
  bool need_k = k > 0 && k < a.vocab, need_p = p < 1.0f;
  const float inv_temp = 1.0f / temp;
  const bool tame = top < INFINITY && temp > 1e-12f && temp < 1e12f;
  float range = kRange * temp;
  Row<T> R{sh, buf, lo, n, rank, size, tid, lane, warp, 1, top, temp, inv_temp, kBins / range, range, log_min_p, tame};

  uint64_t last = ~0ull;  // the last entry that top-k and top-p keep
  unsigned long long own = 0;  // the kept mass of this warp's range
  bool summed = false;
  const int per_warp = (n + 32 * kSmpWarps - 1) / (32 * kSmpWarps) * 32;
  const int w0 = min(n, warp * per_warp), w1 = min(n, w0 + per_warp);
  bool general = need_k || need_p;
  if (general && tame) {
    // ---- A, B: few entries can matter; a guess finds them ------------------------
    // Counted: each thread's largest entry.  Any k of them bound the k-th entry
    // of the row from below.  Where top-p asks for masses, each CTA also counts
    // all its entries as large as the 128th of its threads' (one in a hundred or so), and
    // one in eight of the others.
    const float own_place = R.place(thread_top);
    if (own_place < (float)kBins) atomicAdd(&sh.count[(int)own_place], 1u);
    if (tid == 0) {
      sh.bin_k = sh.bin_p = kBins;
      sh.n_list = sh.n_cut = 0;
      sh.cut_key = 0;
    }
    if (tid < kFine) sh.mass[tid] = 0;
    if (need_k) cluster_sync(); else __syncthreads();
    // this thread's two bins of all CTAs, their loads together
    uint2 bins[kSmpMaxCluster];
    auto gather = [&]() {
#pragma unroll
      for (int r = 0; r < kSmpMaxCluster; ++r)
        bins[r] = r < size ? ld_cluster32x2(mapa_shared(sh.count + 2 * tid, r)) : make_uint2(0, 0);
    };
    uint32_t cnt[2] = {0, 0};
    if (need_k) {
      gather();
#pragma unroll
      for (int r = 0; r < kSmpMaxCluster; ++r) { cnt[0] += bins[r].x; cnt[1] += bins[r].y; }
    } else {
      cnt[0] = sh.count[2 * tid];
      cnt[1] = sh.count[2 * tid + 1];
    }
    // first bins up to which the counts, or the masses, reach a bar
    auto first_bin = [&](bool lo_reaches, bool hi_reaches, int* where) {
      const int at = lo_reaches ? 2 * tid : hi_reaches ? 2 * tid + 1 : kBins;
      const int first = __reduce_min_sync(0xffffffffu, at);
      if (lane == 0 && first < kBins) atomicMin(where, first);
    };
    {
      uint32_t ci = cnt[0] + cnt[1];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xffffffffu, ci, o);
        if (lane >= o) ci += t;
      }
      if (lane == 31) sh.warp_cnt[warp] = ci;
      __syncthreads();
      ci += __reduce_add_sync(0xffffffffu, lane < warp ? sh.warp_cnt[lane] : 0);
      const uint32_t want = need_k ? (uint32_t)k : (uint32_t)kSmpThreads / 4;
      first_bin(ci - cnt[1] >= want, ci >= want, &sh.bin_k);
      __syncthreads();
    }
    if (!need_k) {
      const float heavy = (float)min(sh.bin_k + 1, kBins);
      // (16 bytes of 512 threads a turn; a warp looks closely at every eighth of its
      // pieces, so that what is looked at is spread over the slice, and else only at
      // those that hold a heavy entry)
      const int spread = pieces > 4 * kSmpThreads ? 7 : 0;
      const float maybe = R.at_least(heavy);
      auto counted = [&](T x, bool look) {
        const float t = R.place(to_f32(x));
        if (t < heavy) atomicAdd(&sh.place[(int)t], 1u);
        else if (look && t < (float)kBins) atomicAdd(&sh.place[(int)t], 0x10000u);
      };
#pragma unroll 2
      for (int at = tid, turn = warp; at < pieces; at += kSmpThreads, ++turn) {
        const uint4 raw = reinterpret_cast<const uint4*>(buf + head)[at];
        const T* x = reinterpret_cast<const T*>(&raw);
        const bool look = (turn & spread) == 0;
        if (!look && !(largest(x) >= maybe)) continue;
#pragma unroll
        for (int e = 0; e < kPer; ++e) counted(x[e], look);
      }
      if (tid < head + tail) counted(buf[tid < head ? tid : n - tail + (tid - head)], true);
      __syncthreads();
      // (how many pieces were looked at closely, of all)
      const int turns = pieces / kSmpThreads, rest = pieces - turns * kSmpThreads, first = 32 * (-turns & 7);
      auto of_warp = [](int k) { return min(32, max(0, k)); };
      const int seen = spread ? 64 * turns + of_warp(rest - first) + of_warp(rest - first - 256) : pieces;
      const float step = range / (kBins * temp), each = seen > 0 ? (float)pieces / (float)seen : 1.f;
      // a bin's entries as they are reckoned, and the variance of that number in
      // units of the bin's weight (of an entry that is counted, only its place in
      // the bin is unknown: a uniform one's variance is 1/12): 16 bits each
      float w[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int b = 2 * tid + e;
        const uint32_t both = sh.place[b];  // all counted, and one in eight: 16 bits each (a wrap spoils a guess only)
        const float seldom = each * (both >> 16), every = both & 0xFFFF;
        w[e] = __expf(-(b + 0.5f) * step);
        sh.count[b] = __half_as_ushort(__float2half_rn(fminf(every + seldom, 65000.f))) |
                      (__float_as_uint(each * seldom + every * (step * step / 12.f)) & 0xFFFF0000u);
      }
      if (tid == 0) sh.bin_k = kBins;
      cluster_sync();
      gather();
      float ms[2] = {0.f, 0.f}, vs[2] = {0.f, 0.f};
#pragma unroll
      for (int r = 0; r < kSmpMaxCluster; ++r) {
        const uint32_t c[2] = {bins[r].x, bins[r].y};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          ms[e] += __half2float(__ushort_as_half((unsigned short)(c[e] & 0xFFFF))) * w[e];
          vs[e] += __uint_as_float(c[e] & 0xFFFF0000u) * w[e] * w[e];
        }
      }
      float mi = ms[0] + ms[1], vi = vs[0] + vs[1];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const float tm = __shfl_up_sync(0xffffffffu, mi, o), tv = __shfl_up_sync(0xffffffffu, vi, o);
        if (lane >= o) { mi += tm; vi += tv; }
      }
      if (lane == 31) { sh.warp_mass[warp] = mi; sh.warp_var[warp] = vi; }
      __syncthreads();
      const float m = lane < kSmpWarps ? sh.warp_mass[lane] : 0.f, v = lane < kSmpWarps ? sh.warp_var[lane] : 0.f;
      mi += warp_sum(lane < warp ? m : 0.f);
      vi += warp_sum(lane < warp ? v : 0.f);
      const float m_all = warp_sum(m), v_all = warp_sum(v);
      // The cut lies where what is before, less p of all, turns positive: that is
      // (1 - p) of what is before less p of what is after, and its error is small
      // where p is near 1, as what is after is.
      auto past = [&](float before, float var, float sign) {
        const float after = fmaxf(m_all - before, 0.f);
        const float err = sqrtf((1.f - p) * (1.f - p) * var + p * p * fmaxf(v_all - var, 0.f));
        return (1.f - p) * before - p * after >= sign * (5.f * err + 0.001f * fminf(before, after));
      };
      first_bin(past(mi - ms[1], vi - vs[1], -1.f), past(mi, vi, -1.f), &sh.bin_k);
      first_bin(past(mi - ms[1], vi - vs[1], 1.f), past(mi, vi, 1.f), &sh.bin_p);
      __syncthreads();
    }
    // Top-k: places before `inner` are the candidates.  Top-p: places before
    // `inner` are kept for sure, those from `outer` on are not.
    const float inner = need_k ? (float)min(sh.bin_k + 1, kBins) : (float)min(sh.bin_k, kBins - 1);
    const float outer = (float)min(sh.bin_p + 1, kBins);
    const bool guess = !need_k || sh.bin_k < kBins;
    const float finer = kFine / (outer - inner);
    auto fine_bin = [&](float t) { return min(kFine - 1, (int)((t - inner) * finer)); };
    if (guess && need_k) {
      const float maybe = R.at_least(inner);
      auto listed = [&](T x, int i) {
        const float v = to_f32(x);
        if (R.place(v) < inner) {
          const int at = atomicAdd(&sh.n_list, 1);
          if (at < kList) sh.list[at] = entry_key(v, lo + i);
        }
      };
#pragma unroll 4
      for (int at = tid; at < pieces; at += kSmpThreads) {
        const uint4 raw = reinterpret_cast<const uint4*>(buf + head)[at];
        const T* x = reinterpret_cast<const T*>(&raw);
        if (!(largest(x) >= maybe)) continue;
#pragma unroll
        for (int e = 0; e < kPer; ++e) listed(x[e], head + at * kPer + e);
      }
      if (tid < head + tail) {
        const int i = tid < head ? tid : n - tail + (tid - head);
        listed(buf[i], i);
      }
      __syncthreads();
      cluster_sync();
      if (R.cluster_int(&sh.n_list) <= kList) {
        const int m = rank == 0 ? R.pull() : 0;
        cluster_sync();  // the others leave: only the leader goes on
        if (rank == 0) {
          if (m <= kFew) R.finish_few(m, k, need_p, p, u, a.token + row, a.logprob + row);
          else R.finish_list(m, k, need_p, p, u, a.token + row, a.logprob + row);
        }
        return;
      }
      cluster_sync();
    } else if (guess) {
      // the exact masses before `inner` and of all, and the entries between
      Halves all, sure;
      unsigned long long between = 0;
#pragma unroll 4
      for (int i = w0 + lane; i < w1; i += 32) {
        const float v = to_f32(buf[i]), t = R.place(v);
        const Halves w = Halves::of(t <= (float)kBins ? expf(R.expo(v)) : 0.f);
        all.add(w);
        sure.add(w, t < inner);
        if (t >= inner && t < outer) {
          const int at = atomicAdd(&sh.n_list, 1);
          if (at < kList) sh.list[at] = entry_key(v, lo + i);
          const unsigned long long W = w.total();
          between += W;
          atomicAdd(&sh.mass[fine_bin(t)], W);
        }
      }
      const unsigned long long mine = warp_sum64(sure.total());
      if (lane == 0) sh.above[warp] = mine;
      unsigned long long v[3] = {all.total(), sure.total(), between};
      R.cluster_total(v);
      const double bar = (double)p * (double)v[0];
      bool fits = (double)v[1] < bar && (double)(v[1] + v[2]) >= bar;
      if (fits) {
        // the fine bin that the cut falls into, exactly: two threads a bin, each for
        // every other CTA
        unsigned long long f = 0;
#pragma unroll
        for (int r = 0; r < kSmpMaxCluster; r += 2)
          if (r + (tid & 1) < size) f += ld_cluster64(mapa_shared(&sh.mass[tid / 2], r + (tid & 1)));
        f += __shfl_xor_sync(0xffffffffu, f, 1);
        const unsigned long long inc = warp_scan64((tid & 1) ? f : 0ull, lane);
        if (lane == 31) sh.warp64[warp] = inc;
        __syncthreads();
        unsigned long long before;
        R.warps_total(sh.warp64, &before);
        before += v[1] + inc - f;
        if ((tid & 1) && (double)before < bar && (double)(before + f) >= bar) { sh.found = tid / 2; sh.reply = before; }
        __syncthreads();
        const int fine = sh.found, n_mine = sh.n_list;
        const unsigned long long m_before = sh.reply;
        // its entries: from the list, or, where that was too short, from all
        const bool listed = n_mine <= kList;
        uint64_t keep[kList / kSmpThreads];
        auto in_fine = [&](float t) { return t >= inner && t < outer && fine_bin(t) == fine; };
        auto cut_add = [&](uint64_t key) {
          const int at = atomicAdd(&sh.n_cut, 1);
          if (at < kFew) sh.cut[at] = key;
        };
        if (listed) {
#pragma unroll
          for (int e = 0; e < kList / kSmpThreads; ++e) {
            const int i = e * kSmpThreads + tid;
            keep[e] = i < n_mine ? sh.list[i] : ~0ull;  // (no entry's key: its z is a NaN)
            if (in_fine(R.place(key_z(keep[e])))) cut_add(keep[e]);
          }
        } else {
#pragma unroll 4
          for (int i = tid; i < n; i += kSmpThreads) {
            const float v = to_f32(buf[i]);
            if (in_fine(R.place(v))) cut_add(entry_key(v, lo + i));
          }
        }
        cluster_sync();
        const int n_cut = R.cluster_int(&sh.n_cut);
        if (n_cut <= kFew) {
          last = R.cut_few(n_cut, m_before, bar);
        } else {
          // many: in front of the list, for the leader to sort
          fits = n_cut <= kList;
          if (fits) {
            if (tid == 0) sh.n_list = 0;
            __syncthreads();
            if (listed) {
#pragma unroll
              for (int e = 0; e < kList / kSmpThreads; ++e)
                if (in_fine(R.place(key_z(keep[e])))) sh.list[atomicAdd(&sh.n_list, 1)] = keep[e];
            } else {
              for (int i = tid; i < n; i += kSmpThreads) {
                const float v = to_f32(buf[i]);
                if (in_fine(R.place(v))) sh.list[atomicAdd(&sh.n_list, 1)] = entry_key(v, lo + i);
              }
            }
            cluster_sync();
            if (rank == 0) {
              const uint64_t key = R.cut_list(R.pull(), m_before, bar);
              if (tid == 0) sh.reply = key;
            }
            cluster_sync();
            last = ld_cluster64(mapa_shared(&sh.reply, 0));
          }
        }
        if (fits) {
          general = false;
          if (listed && log_min_p == -INFINITY) {
            // kept: what was sure, and the entries between up to the cut
#pragma unroll
            for (int e = 0; e < kList / kSmpThreads; ++e)
              if (e * kSmpThreads + tid < n_mine && keep[e] <= last)
                atomicAdd(&sh.above[((int)(uint32_t)keep[e] - lo) / per_warp], R.mass(key_z(keep[e])));
            __syncthreads();
            own = sh.above[warp];
            summed = true;
          }
        }
      }
      if (general) cluster_sync();  // masses and counts are taken again below
    } else {
      cluster_sync();  // the counts have been read: they are taken again below
    }
  }
  if (general) {
    // ---- C: any k, any ties, any range -------------------------------------------
    if (tid == 0) sh.found = 0;
    for (int i = tid; i < kBins; i += kSmpThreads) sh.count[i] = sh.place[i] = 0;
    float low = INFINITY;
    for (int i = tid; i < n; i += kSmpThreads) {
      const float v = R.z(i);
      if (v > -INFINITY) low = fminf(low, v);
    }
    low = -warp_max(-low);
    if (lane == 0) sh.warp_top[warp] = low;
    __syncthreads();
    low = -warp_max(-sh.warp_top[lane % kSmpWarps]);
    Exchange* mine = &sh.ex[R.turn];
    if (tid == 0) mine->low = low;
    cluster_sync();
    for (int r = 0; r < size; ++r) low = fminf(low, __uint_as_float(ld_cluster32(mapa_shared(&mine->low, r))));
    R.turn ^= 1;
    range = R.range = fminf(kRange * temp, top - low);
    R.scale = range > 1e-30f ? kBins / range : 0.f;
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
    // the last entry of the top-k, then that of the nucleus;
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
        // (a bar of 0 is reached before any entry; the largest is kept all the same)
        bar = fmax((double)p * (double)v[0], 1.0);
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
          const uint64_t key = R.cut_list(R.pull(), v[1], bar);
          if (tid == 0) sh.reply = key;
        }
        cluster_sync();
        last = ld_cluster64(mapa_shared(&sh.reply, 0));
      } else {
        last = R.bisect(bin_p, true, bar, most);
      }
    }
  }
  // ---- the draw, in index order: warps own consecutive ranges ------------------
  if (!summed) {
    if (tame) {
      const float z_last = last == ~0ull ? -INFINITY : key_z(last);
      const int i_last = (int)(uint32_t)last - lo;
      Halves sum;
#pragma unroll 4
      for (int i = w0 + lane; i < w1; i += 32) {
        const float v = to_f32(buf[i]), x = R.expo(v);
        const bool in = top - v <= R.range && x >= log_min_p && (v > z_last || (v == z_last && i <= i_last));
        sum.add(Halves::of(in ? expf(x) : 0.f));
      }
      own = sum.total();
    } else {
      for (int i = w0 + lane; i < w1; i += 32) own += R.kept_mass(i, last);
    }
    own = warp_sum64(own);
  }
  R.draw(w0, w1, own, last, u, a.token + row, a.logprob + row);
}

// How many CTAs share a row.  Rows run in rounds of as many clusters as the GPU
// holds (a cluster stays within one group of SMs, so sizes differ in what they
// leave idle: of 128256 floats a row 36 clusters of 8 run at once, or 46 of 6), and
// a round takes the time of a CTA's entries and of its dependent steps, which
// cost as much as some 18000 entries.  464 such rows took 244 us with 6,
// 272 with 7, 270 with 8; one row is fastest with 8.
struct Shape {
  int size, per_cta, smem;
};
template <typename T>
static Shape shape_of(int rows, int vocab) {
  constexpr int kMaxShared = 227 * 1024;
  static OncePerDevice allowed;
  const int dev = current_device();
  allowed.get(dev, [] { return allow_shared(sample_kernel<T>, kMaxShared); });
  // clusters at once, of the last device and vocabulary
  thread_local int of_dev = -1, of_vocab = 0, active[kSmpMaxCluster + 1];
  const bool known = of_dev == dev && of_vocab == vocab;
  if (!known) of_vocab = 0;  // until all of them are
  Shape best{};
  int64_t best_cost = INT64_MAX;
  for (int size = 1; size <= kSmpMaxCluster; ++size) {
    if (size > 1 && vocab / size < 2048) break;  // (best holds a size: one CTA has room for 4096 entries)
    const int per_cta = (vocab + 8 * size - 1) / (8 * size) * 8;
    const int smem = (int)((sizeof(SmpShared) + 15) / 16 * 16 + 16 + ((size_t)per_cta * sizeof(T) + 15) / 16 * 16);
    if (smem > kMaxShared) continue;
    if (!known) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3((unsigned)size);
      cfg.blockDim = dim3(kSmpThreads);
      cfg.dynamicSmemBytes = smem;
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = size;
      attr[0].val.clusterDim.y = 1;
      attr[0].val.clusterDim.z = 1;
      cfg.attrs = attr;
      cfg.numAttrs = 1;
      const cudaError_t e = cudaOccupancyMaxActiveClusters(&active[size], sample_kernel<T>, &cfg);
      if (e != cudaSuccess) throw e;
    }
    if (active[size] < 1) continue;
    const int64_t cost = (int64_t)((rows + active[size] - 1) / active[size]) * (per_cta + 18000);
    if (cost < best_cost) {
      best_cost = cost;
      best = {size, per_cta, smem};
    }
  }
  of_dev = dev;
  of_vocab = vocab;
  if (best.size == 0) throw cudaErrorInvalidConfiguration;
  return best;
}

template <typename T>
static void run_sample(const SampleArgs& a, cudaStream_t s) {
  const Shape shape = shape_of<T>(a.rows, a.vocab);
  launch_in_turn(sample_kernel<T>, dim3((unsigned)a.rows * shape.size), kSmpThreads, shape.smem, shape.size, s, a, shape.per_cta);
}

void launch_sample(const SampleArgs& a, cudaStream_t s) {
  if (a.dtype == DT_BF16) run_sample<__nv_bfloat16>(a, s);
  else if (a.dtype == DT_F16) run_sample<__half>(a, s);
  else run_sample<float>(a, s);
}

}  // namespace pard
