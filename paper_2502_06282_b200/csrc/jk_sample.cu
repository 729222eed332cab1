// jk_sample: temperature, top-k, top-p and min-p over rows of logits, the draw of a token and the filtered
// rows (the sampled form of arXiv 2502.06282, Sec. 2.1 steps 2-3, draws with a temperature only).
//
// Logits are compared through their ordered 32-bit image (larger logit = larger unsigned integer).  Every filter
// is a prefix of (logit descending, index ascending), so the kept set is a threshold on the image plus a number of
// tokens equal to the threshold, lowest index first.  Both thresholds (by count for top-k, by weight for top-p) are
// found in a histogram of the row:
//   - a bin is the upper half of the image (sign, exponent, 7 bits), over the 18 octaves that hold the largest
//     magnitude with a weight; what is nearer to zero falls into two bins of its own, zero into one, what weighs
//     nothing into a last one;
//   - the bin that holds the threshold is resolved exactly: if it has one value (every bf16 bin) there is nothing
//     left to do, else its members (a few tens of 1e5, as a rule) are gathered and compared with one another,
//     and if they are more than SMP_LIST, a histogram of the bin's images follows, at most three of them;
//   - when all tokens down to that bin fit the list, filters and draw are carried out on the list.
// Weights are fixed-point numbers of 64 bits, unit 2^-SH (SH = 45 up to 2^17 tokens, less beyond, so that a row's
// sum stays below 2^62): sums do not depend on an order and are the same on every run, and a histogram can hold them in
// two 32-bit counters.  A bin of one value needs its count alone: bf16 rows take one atomic per element and one
// exponential per bin.
//
// A row belongs to a cluster of 1 to 8 blocks; histograms are added up in its first block's shared memory.
//
// Measured (B200, graph replay on the same inputs; in brackets calls one after the other on inputs that leave L2 in
// between): one row of 32000 in fp32 with top-k 50 and top-p 12.4 us (12.9), of which a pass over the row takes 1 us and
// each of the cluster's barriers 0.7; 240 rows of 128256 in bf16 (62 MB in, 123 MB out: 29 us of HBM time) with top-p,
// min-p, draw and filtered rows 108 us (115): largest logit 10, histogram 33 (the latency of its
// shared-memory atomics, 2.4 cycles of bank conflicts each, and instruction fetch), scan of the bins 8, output and weights 32, search for the token
// 7; some SMs hold two rows, others one.
#include <math.h>

#include "jk_common.cuh"

#define SMP_THREADS 512
#define SMP_WARPS (SMP_THREADS / 32)
#define SMP_CLUSTER 8
#define SMP_LIST 256                  // candidates that are compared with one another
#define SMP_OCTAVES 18
#define SMP_BINS 5120                 // >= 2 * 128 * SMP_OCTAVES + 4, a multiple of SMP_THREADS
#define SMP_LEVEL 4096                // bins of a histogram of images
#define SMP_NOTHING 0x007fffffu       // the image of -inf
#define SMP_BIG 3.402823466e38f

typedef unsigned long long u64;

// Larger value, larger image; NaN like -inf, +inf like the largest float.
__device__ __forceinline__ uint32_t smp_key(float z) {
  if (z != z) z = -INFINITY;
  z = fminf(z, SMP_BIG) + 0.f;                           // (-0 and +0 are one value)
  const uint32_t b = __float_as_uint(z);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float smp_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

struct smp_state {                    // of the row: decided by the cluster's first block, copied to the others
  int stage;                          // what comes next: one of SMP_*
  uint32_t klo, khi;                  // images of the bin that holds the threshold
  int n, before;                      // tokens in it and above it
  u64 before_m, total, target;        // weight above it, of all tokens of the filter, and to be reached
  uint32_t thr;                       // result: threshold, tokens equal to it that stay, and that there are
  int ties, eq;
  int n_list, first, done_tok;
  int win;                            // run of the row that holds the draw
  u64 win_before;                     // weight in front of it
  long long goal;
};
enum { SMP_GATHER_ALL, SMP_GATHER_BIN, SMP_REFINE, SMP_FOUND };

struct smp_shared {
  alignas(16) uint32_t cnt[SMP_BINS], lo[SMP_BINS], hi[SMP_BINS];  // (lo and hi hold a table of weights for the draw)
  double table[16];                   // 2^(j / 16): one entry per pair of banks, so that no two lanes collide
  smp_state st;
  // candidates: image and complement of the index in one word, so that a larger word comes first in the order; weight
  alignas(16) u64 lc[SMP_LIST], lw[SMP_LIST];
  u64 wsum[SMP_CLUSTER * SMP_WARPS];  // per warp of the cluster (first block's copy)
  int weq[SMP_CLUSTER * SMP_WARPS];
  u64 red[SMP_WARPS];
  int redi[SMP_WARPS];
  uint32_t kmax;                      // of this block's part
  int rest;
};

__device__ __forceinline__ uint32_t smp_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

// Weights: exp((z - zmax) / T) in units of 2^-sh.  2^(n / 16) from a table, the rest (at most ln2 / 32) by the power
// series to the sixth term: 5e-16 off, next to the 4e-15 of the reduced argument.
struct smp_weight {
  double zmax, inv_t, magic;
  float cut;                          // below: less than half a unit
  const double* table;
  __device__ __forceinline__ u64 operator()(float z) const {
    const double x = ((double)z - zmax) * inv_t;         // (without branches, so that several can be under way)
    const double big = 6755399441055744.0;               // 1.5 * 2^52: the integer part stands in the low bits
    const double nb = fma(x, 23.083120654223414219, big);  // 16 / ln 2
    const int n = __double2loint(nb);
    const double r = fma(nb - big, -0.043321698784996581, x);  // ln 2 / 16
    double p = fma(r, 1.0 / 720.0, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    const double t = table[n & 15];
    const double w = __hiloint2double(__double2hiint(t) + ((n >> 4) << 20), __double2loint(t)) * p;
    const u64 units = (u64)__double_as_longlong(w + magic) - (u64)__double_as_longlong(magic);
    return z >= cut ? units : 0ull;
  }
};

// Bins of the first histogram.
struct smp_map1 {
  uint32_t mz, mb, mn;                // upper half of the largest |z| of positive tokens, of the smallest, of negative ones
  int np, nn;                         // bins of positive and of negative values
  float cut;                          // below: no weight
  uint32_t kcut, kfloor;
  bool bf16;
  __device__ void set(uint32_t kmax, uint32_t floor_key, float lowest, bool is_bf16) {
    const float zmax = smp_value(kmax);
    cut = lowest;
    kcut = smp_key(cut);
    kfloor = floor_key;
    bf16 = is_bf16;
    const uint32_t mzm = (__float_as_uint(zmax) >> 16) & 0x7fffu, mcut = (__float_as_uint(cut) >> 16) & 0x7fffu;
    const uint32_t mt = max(mzm, mcut), oct = mt >> 7;
    mb = oct >= SMP_OCTAVES ? (oct - (SMP_OCTAVES - 1)) << 7 : 1u;
    mz = mzm;
    mn = zmax < 0.f ? max(mb, mzm) : mb;
    np = zmax > 0.f && mzm >= mb ? (int)(mzm - mb) + 1 : 0;
    nn = cut < 0.f && mcut >= mn ? (int)(mcut - mn) + 1 : 0;
  }
  __device__ __forceinline__ int bins() const { return np + nn + 4; }
  __device__ __forceinline__ int bin(float z) const {    // z >= cut, not above the largest float
    const int b = (int)__float_as_uint(z), m = (b >> 16) & 0x7fff;
    if (m < (int)mb) return z == 0.f ? np + 1 : z > 0.f ? np : np + 2;
    return b < 0 ? m + (np + 3 - (int)mn) : (int)mz - m;
  }
  __device__ void range(int b, uint32_t& klo, uint32_t& khi) const {
    if (b < np) {
      klo = (0x8000u | (mz - b)) << 16;
      khi = klo | 0xffffu;
      if (bf16 && mz - b != 0x7f7fu) khi = klo;
    } else if (b == np) {
      klo = 0x80000001u;
      khi = ((0x8000u | mb) << 16) - 1u;
    } else if (b == np + 1) {
      klo = khi = 0x80000000u;
    } else if (b == np + 2) {
      klo = ~((0x8000u | mb) << 16) + 1u;
      khi = 0x7ffffffeu;
    } else if (b < np + 3 + nn) {
      const uint32_t m = mn + (b - np - 3);
      khi = ~((0x8000u | m) << 16);
      klo = khi - 0xffffu;
      if (bf16 && m != 0x7f7fu) klo = khi;
    } else {
      klo = SMP_NOTHING + 1u;
      khi = kcut - 1u;
      klo = max(klo, kfloor + 1u);
      return;
    }
    if (klo != khi) klo = max(klo, kcut);
    klo = max(klo, kfloor + 1u);
  }
  // one value: its weight follows from the count
  __device__ __forceinline__ bool single(int b) const {
    if (b == np + 1) return true;
    return bf16 && ((b < np && mz - b != 0x7f7fu) || (b >= np + 3 && b < np + 3 + nn && mn + (b - np - 3) != 0x7f7fu));
  }
};

template <typename T, int VEC> __device__ __forceinline__ void smp_unpack(const uint32_t (&raw)[VEC * sizeof(T) / 4 ? VEC * sizeof(T) / 4 : 1], float (&z)[VEC]) {
  if constexpr (VEC == 1) {
    z[0] = __uint_as_float(raw[0]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) z[i] = __uint_as_float(raw[i]);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i += 2) {
      z[i] = __uint_as_float(raw[i / 2] << 16);
      z[i + 1] = __uint_as_float(raw[i / 2] & 0xffff0000u);
    }
  }
}

template <typename T, int VEC>
__global__ void __launch_bounds__(SMP_THREADS, 2) k_sample(
    const T* __restrict__ logits, long long stride, int V, int C, int sh, const float* __restrict__ temperature,
    const int32_t* __restrict__ top_k, const float* __restrict__ top_p, const float* __restrict__ min_p,
    const float* __restrict__ u, int32_t* __restrict__ out_tok, float* __restrict__ out_logits) {
  constexpr int RAW = VEC * sizeof(T) / 4 ? VEC * sizeof(T) / 4 : 1;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  smp_shared& S = *reinterpret_cast<smp_shared*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x / C, rank = C > 1 ? (int)smp_rank() : 0;
  smp_shared* S0 = C > 1 ? jk_cluster_map(&S, 0) : &S;          // the first block's
  auto sync = [&]() {
    if (C > 1) {
      asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
      __syncthreads();
    }
  };
  // the first block's state to the others, before a barrier of the cluster
  auto publish = [&]() {
    __syncthreads();
    if (C > 1) {
      constexpr int WORDS = sizeof(smp_state) / 4;
      for (int i = tid; i < (C - 1) * WORDS; i += SMP_THREADS)
        reinterpret_cast<uint32_t*>(&jk_cluster_map(&S, 1 + i / WORDS)->st)[i % WORDS] = reinterpret_cast<const uint32_t*>(&S.st)[i % WORDS];
    }
  };
  for (int i = tid; i < SMP_BINS / 4; i += SMP_THREADS) {
    reinterpret_cast<uint4*>(S.cnt)[i] = make_uint4(0u, 0u, 0u, 0u);
    reinterpret_cast<uint4*>(S.lo)[i] = make_uint4(0u, 0u, 0u, 0u);
    reinterpret_cast<uint4*>(S.hi)[i] = make_uint4(0u, 0u, 0u, 0u);
  }
  bool clean = true;                                     // the bins are empty
  if (tid < 16) S.table[tid] = exp2(tid / 16.0);
  jk_pdl_wait();
  jk_pdl_trigger();
  const T* z0 = logits + (size_t)r * stride;
  float* out = out_logits ? out_logits + (size_t)r * V : nullptr;
  // every warp of the cluster owns a run of the row, in index order
  const int nv = V / VEC;
  const int W = C * SMP_WARPS, chunk = ((nv + W - 1) / W + 31) / 32 * 32, gw = rank * SMP_WARPS + warp;
  const int v_begin = (int)min((long long)nv, (long long)gw * chunk), v_end = (int)min((long long)nv, (long long)v_begin + chunk);
  auto load = [&](int v, uint32_t (&raw)[RAW]) {
    if constexpr (VEC == 1) {
      raw[0] = __float_as_uint(jk_to_float(z0[v]));
    } else if constexpr (RAW == 4) {
      const uint4 x = __ldg(reinterpret_cast<const uint4*>(z0) + v);
      raw[0] = x.x; raw[1] = x.y; raw[2] = x.z; raw[3] = x.w;
    } else {
      const uint2 x = __ldg(reinterpret_cast<const uint2*>(z0) + v);
      raw[0] = x.x; raw[1] = x.y;
    }
  };
  // f(index of the lane's vector, its VEC values) for the vectors of the warp's run
  auto each = [&](auto f) {
    int v = v_begin + lane;
    for (; v + 96 < v_end; v += 128) {                   // four loads on their way at a time
      uint32_t raw[4][RAW];
#pragma unroll
      for (int i = 0; i < 4; ++i) load(v + 32 * i, raw[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float z[VEC];
        smp_unpack<T, VEC>(raw[i], z);
        f(v + 32 * i, z);
      }
    }
    for (; v < v_end; v += 32) {
      uint32_t raw[RAW];
      load(v, raw);
      float z[VEC];
      smp_unpack<T, VEC>(raw, z);
      f(v, z);
    }
  };

  // ---------------------------------------------------------------- largest logit
  {
    float mx = -INFINITY;
    each([&](int, const float (&z)[VEC]) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) mx = fmaxf(mx, z[i]);  // (a NaN is passed over)
    });
    mx = jk_warp_max(mx);
    if (lane == 0) S.redi[warp] = (int)smp_key(mx);
    __syncthreads();
    if (tid == 0) {
      uint32_t k = 0u;
      for (int i = 0; i < SMP_WARPS; ++i) k = max(k, (uint32_t)S.redi[i]);
      S.kmax = k;
      S.st.first = 0x7fffffff;
      S.st.n_list = 0;
      S.st.done_tok = 0;
    }
  }
  sync();
  uint32_t kmax = 0u;
  for (int i = 0; i < C; ++i) kmax = max(kmax, C > 1 ? jk_cluster_map(&S.kmax, i)[0] : S.kmax);
  auto fill = [&](int keep_index, float value) {         // one token, or none
    if (!out) return;
    each([&](int v, const float (&)[VEC]) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) out[(size_t)v * VEC + i] = v * VEC + i == keep_index ? value : -INFINITY;
    });
  };
  const float temp = temperature ? temperature[r] : 1.f;
  if (kmax <= SMP_NOTHING) {                             // nothing but -inf
    fill(-1, 0.f);
    if (out_tok && rank == 0 && tid == 0) out_tok[r] = -1;
    sync();                                              // (shared memory of a block that has left is not read)
    return;
  }
  if (!(temp > 0.f)) {                                   // greedy
    int first = 0x7fffffff;
    each([&](int v, const float (&z)[VEC]) {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (smp_key(z[i]) == kmax) first = min(first, v * VEC + i);
    });
    first = __reduce_min_sync(0xffffffffu, first);
    if (lane == 0 && first != 0x7fffffff) atomicMin(&S0->st.first, first);
    sync();
    first = S0->st.first;
    fill(first, 0.f);
    if (out_tok && rank == 0 && tid == 0) out_tok[r] = first;
    sync();
    return;
  }
  const float zmax = smp_value(kmax);
  smp_weight weight;
  weight.zmax = (double)zmax;
  weight.inv_t = 1.0 / (double)temp;
  // exp(-x) < 2^-(sh + 1), half a unit, and some more: those weigh nothing, and the reduced argument stays in range
  weight.cut = fmaxf((float)((double)zmax - (0.6931471805599454 * (sh + 1) + 1.0) * (double)temp), -SMP_BIG);
  weight.magic = __hiloint2double((1023 + 52 - sh) << 20, 0);
  weight.table = S.table;

  // ---------------------------------------------------------------- thresholds
  const int k = top_k ? top_k[r] : 0;
  const float p = top_p ? top_p[r] : 1.f, mp = min_p ? min_p[r] : 0.f;
  const float uu = out_tok ? u[r] : 0.f;
  // image of the lowest logit that min_p leaves
  uint32_t kb = SMP_NOTHING + 1u;
  if (mp > 0.f) {
    const double bound = fmin(0.0, (double)temp * log((double)mp));
    auto ok = [&](uint32_t key) { return (double)smp_value(key) - (double)zmax >= bound; };
    // The sum's image or, where the sum was rounded down, the next one.  Not where zmax + bound is next to zero: the
    // difference to zmax is then the same for every float around zero, 2^29 of them and more, and all of them pass.
    const uint32_t low = kb;
    kb = smp_key(fmaxf((float)((double)zmax + bound), -SMP_BIG));
    if (!ok(kb)) ++kb;                                   // (zmax passes: kb is not above it)
    if (!ok(kb) || (kb > low && ok(kb - 1u))) {
      uint32_t fails = low, passes = kmax;               // (larger images pass if smaller ones do)
      while (fails < passes) {
        const uint32_t mid = fails + (passes - fails) / 2u;
        if (ok(mid)) passes = mid;
        else fails = mid + 1u;
      }
      kb = passes;
    }
  }
  auto block_sum = [&](u64 v) {                          // of one block, every thread
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if (lane == 0) S.red[warp] = v;
    __syncthreads();
    u64 t = 0ull;
#pragma unroll
    for (int i = 0; i < SMP_WARPS; ++i) t += S.red[i];
    return t;
  };
  auto reach = [&](u64 total) {                          // weight to be reached, at least one unit
    const double x = (double)p * (double)total;
    u64 t = x > 0.0 ? (u64)x : 0ull;
    if ((double)t < x) ++t;
    return min(max(t, 1ull), total);
  };
  // the draw is the first kept token whose cumulative weight exceeds this: u of the sum, never all of it
  auto draw_goal = [&](u64 all) {
    const long long most = (long long)all - 1;
    return uu >= 0.f && uu < 1.f ? min((long long)((double)uu * (double)all), most) : uu < 0.f ? 0ll : most;
  };
  auto ties_by_weight = [&](u64 missing, u64 w, int most) {  // tokens of weight w until `missing` is reached
    const u64 n = (missing + w - 1ull) / max(w, 1ull);
    return (int)min(n, (u64)most);
  };

  // Finds the threshold among the tokens above floor_key; ties_f of the eq_f tokens equal to it take part in the
  // total and come last.  Everything that is decided is decided by the first block.
  auto select = [&](bool by_weight, uint32_t floor_key, int ties_f, int eq_f) {
    smp_map1 map;
    map.set(kmax, floor_key, weight.cut, sizeof(T) == 2);
    const float z_floor = smp_value(floor_key);
    uint32_t klo = 0u, khi = 0xffffffffu;
    int shift = 0;
    for (int level = 0;; ++level) {
      // ------------------------------------------------ histogram
      const int nb = level == 0 ? map.bins() : (int)((khi - klo) >> shift) + 1;
      if (!clean) {
        for (int i = tid; i < SMP_BINS / 4; i += SMP_THREADS) {
          reinterpret_cast<uint4*>(S.cnt)[i] = make_uint4(0u, 0u, 0u, 0u);
          reinterpret_cast<uint4*>(S.lo)[i] = make_uint4(0u, 0u, 0u, 0u);
          reinterpret_cast<uint4*>(S.hi)[i] = make_uint4(0u, 0u, 0u, 0u);
        }
        __syncthreads();
      }
      clean = false;
      auto add_weight = [&](int b, u64 w) {
        const uint32_t l = (uint32_t)w, old = atomicAdd(&S.lo[b], l);
        const uint32_t h = (uint32_t)(w >> 32) + (old + l < old ? 1u : 0u);
        if (h) atomicAdd(&S.hi[b], h);
      };
      auto add = [&](int b, bool weigh, float z) {
        atomicAdd(&S.cnt[b], 1u);
        if (weigh) add_weight(b, weight(z));
      };
      if (level == 0) {
        // (one comparison, false for a NaN; no float is above the largest)
        float lowest = smp_value(max(map.kcut, floor_key + 1u));
        if (lowest == INFINITY) lowest = __int_as_float(0x7fffffff);
        int rest = 0;
        const int np3 = map.np + 3 - (int)map.mn, mb = (int)map.mb, mz = (int)map.mz;
        each([&](int, const float (&zz)[VEC]) {
          if constexpr (sizeof(T) == 2) {
            // bins of one value are counted; the few other tokens come after the vector
            uint32_t odd = 0u;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              const int b = (int)__float_as_uint(zz[i]), m = (b >> 16) & 0x7fff;
              const bool in = zz[i] >= lowest, usual = m >= mb && m < 0x7f7f;
              if (in && usual) atomicAdd(&S.cnt[b < 0 ? m + np3 : mz - m], 1u);
              odd |= in && !usual ? 1u << i : 0u;
              if (!by_weight) rest += !in && zz[i] > -INFINITY;
            }
            if (odd) {
#pragma unroll
              for (int i = 0; i < VEC; ++i) {
                if (!((odd >> i) & 1u)) continue;
                const float z = fminf(zz[i], SMP_BIG);
                const int b = map.bin(z);
                add(b, by_weight && !map.single(b), z);
              }
            }
          } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              if (zz[i] >= lowest) atomicAdd(&S.cnt[map.bin(fminf(zz[i], SMP_BIG))], 1u);
              else if (!by_weight) rest += zz[i] > -INFINITY;
            }
            if (by_weight) {
              u64 w[VEC];
#pragma unroll
              for (int i = 0; i < VEC; ++i) w[i] = weight(fminf(zz[i], SMP_BIG));
#pragma unroll
              for (int i = 0; i < VEC; ++i)
                if (zz[i] >= lowest && zz[i] != 0.f) add_weight(map.bin(fminf(zz[i], SMP_BIG)), w[i]);
            }
          }
        });
        rest = __reduce_add_sync(0xffffffffu, rest);
        if (lane == 0 && rest) atomicAdd(&S.cnt[nb - 1], (uint32_t)rest);
      } else {
        const float z_lo = smp_value(klo);
        each([&](int, const float (&zz)[VEC]) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            if (!(zz[i] >= z_lo)) continue;
            const uint32_t key = smp_key(zz[i]);
            if (key >= klo && key <= khi) add((int)((khi - key) >> shift), by_weight && shift > 0, smp_value(key));
          }
        });
      }
      sync();
      if (C > 1) {
        // block `rank` adds up its part of the bins in the first block's memory
        const int quads = (nb + 3) / 4, per = (quads + C - 1) / C, q1 = min(quads, (rank + 1) * per);
        for (int q = rank * per + tid; q < q1; q += SMP_THREADS) {
          uint32_t n[4] = {0u, 0u, 0u, 0u};
#pragma unroll
          for (int i = 0; i < SMP_CLUSTER; ++i) {
            const uint4 c = reinterpret_cast<const uint4*>(jk_cluster_map(&S, i < C ? i : 0)->cnt)[q];
            if (i < C) { n[0] += c.x; n[1] += c.y; n[2] += c.z; n[3] += c.w; }
          }
          reinterpret_cast<uint4*>(S0->cnt)[q] = make_uint4(n[0], n[1], n[2], n[3]);
        }
        if (by_weight) {
          for (int q = rank * per + tid; q < q1; q += SMP_THREADS) {
            u64 m[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
            for (int i = 0; i < SMP_CLUSTER; ++i) {
              const smp_shared* o = jk_cluster_map(&S, i < C ? i : 0);
              const uint4 l = reinterpret_cast<const uint4*>(o->lo)[q], h = reinterpret_cast<const uint4*>(o->hi)[q];
              if (i < C) {
                m[0] += (u64)h.x << 32 | l.x; m[1] += (u64)h.y << 32 | l.y;
                m[2] += (u64)h.z << 32 | l.z; m[3] += (u64)h.w << 32 | l.w;
              }
            }
            reinterpret_cast<uint4*>(S0->lo)[q] = make_uint4((uint32_t)m[0], (uint32_t)m[1], (uint32_t)m[2], (uint32_t)m[3]);
            reinterpret_cast<uint4*>(S0->hi)[q] =
                make_uint4((uint32_t)(m[0] >> 32), (uint32_t)(m[1] >> 32), (uint32_t)(m[2] >> 32), (uint32_t)(m[3] >> 32));
          }
        }
        sync();
      }
      // ------------------------------------------------ the bin that holds the threshold (first block)
      if (rank == 0) {
        const int per = (nb + SMP_THREADS - 1) / SMP_THREADS, b0 = min(nb, tid * per), b1 = min(nb, b0 + per);
        auto range = [&](int b, uint32_t& lo, uint32_t& hi) {
          if (level == 0) {
            map.range(b, lo, hi);
          } else {
            hi = khi - ((uint32_t)b << shift);
            lo = max(klo, hi - ((1u << shift) - 1u));
          }
        };
        if (by_weight) {
          // (bins by turns: the ones that hold anything stand together)
          // (fp32 has one such bin there, that of zero)
          const bool one = sizeof(T) == 4 && level == 0;
#pragma unroll 2
          for (int b = one ? map.np + 1 + (tid ? nb : 0) : tid; b < nb; b += SMP_THREADS) {
            uint32_t lo, hi;
            range(b, lo, hi);
            const u64 w = (u64)S.cnt[b] * weight(smp_value(lo));
            if (level == 0 ? map.single(b) : shift == 0) {
              S.lo[b] = (uint32_t)w;
              S.hi[b] = (uint32_t)(w >> 32);
            }
          }
          __syncthreads();
        }
        int n = 0;
        u64 m = 0ull;
        for (int b = b0; b < b1; ++b) {
          n += S.cnt[b];
          if (by_weight) m += (u64)S.hi[b] << 32 | S.lo[b];
        }
        // prefix sums over the threads
        int n_in = n;
        u64 m_in = m;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int a = __shfl_up_sync(0xffffffffu, n_in, o);
          const u64 c = __shfl_up_sync(0xffffffffu, m_in, o);
          if (lane >= o) { n_in += a; m_in += c; }
        }
        if (lane == 31) { S.redi[warp] = n_in; S.red[warp] = m_in; }
        __syncthreads();
        u64 total = 0ull;
        int n_all = 0;
        for (int i = 0; i < SMP_WARPS; ++i) {
          if (i < warp) { n_in += S.redi[i]; m_in += S.red[i]; }
          total += S.red[i];
          n_all += S.redi[i];
        }
        const int base_n = level == 0 ? 0 : S.st.before;
        const u64 base_m = level == 0 ? 0ull : S.st.before_m;
        u64 target = 0ull;
        if (by_weight) {
          const u64 wf = ties_f > 0 ? weight(z_floor) : 0ull;
          const u64 all = total + (u64)ties_f * wf;
          target = level == 0 ? reach(all) : S.st.target;
          if (level == 0 && tid == 0) { S.st.total = all; }
          if (level == 0 && target > total) {            // the tokens at the floor take part
            if (tid == 0) {
              S.st.thr = floor_key;
              S.st.ties = ties_by_weight(target - total, wf, ties_f);
              S.st.eq = eq_f;
              S.st.stage = SMP_FOUND;
            }
          }
        } else if (level == 0 && n_all <= k) {           // no more tokens than top_k
          if (tid == 0) {
            S.st.thr = SMP_NOTHING + 1u;
            S.st.ties = S.st.eq = V;
            S.st.stage = SMP_FOUND;
          }
        }
        __syncthreads();                                 // (base_n and base_m have been read)
        n_in += base_n;
        m_in += base_m;
        int n_before = n_in - n;
        u64 m_before = m_in - m;
        const bool mine = by_weight ? m_before < target && target <= m_in : n_before < k && k <= n_in;
        if (mine && !(by_weight && level == 0 && target > total) && !(!by_weight && level == 0 && n_all <= k)) {
          for (int b = b0; b < b1; ++b) {
            const int c = (int)S.cnt[b];
            const u64 w = by_weight ? (u64)S.hi[b] << 32 | S.lo[b] : 0ull;
            if (by_weight ? target > m_before + w : k > n_before + c) {
              n_before += c;
              m_before += w;
              continue;
            }
            uint32_t lo, hi;
            range(b, lo, hi);
            S.st.klo = lo;
            S.st.khi = hi;
            S.st.n = c;
            S.st.before = n_before;
            S.st.before_m = m_before;
            S.st.target = target;
            // (the list may hold all tokens only where nothing below the floor is left out)
            if (n_before + c <= SMP_LIST) {
              S.st.stage = SMP_GATHER_ALL;
            } else if (lo == hi) {
              S.st.stage = SMP_FOUND;
              S.st.thr = lo;
              S.st.eq = c;
              S.st.ties = by_weight ? ties_by_weight(target - m_before, weight(smp_value(lo)), c) : k - n_before;
            } else {
              S.st.stage = c <= SMP_LIST ? SMP_GATHER_BIN : SMP_REFINE;
            }
            break;
          }
        }
      }
      if (rank == 0) publish();
      sync();
      const int stage = S.st.stage;
      klo = S.st.klo;
      khi = S.st.khi;
      if (stage == SMP_FOUND) break;
      if (stage == SMP_REFINE) {
        shift = 0;
        while (((khi - klo) >> shift) >= SMP_LEVEL) ++shift;
        __syncthreads();
        continue;
      }
      // ------------------------------------------------ candidates
      const uint32_t top = stage == SMP_GATHER_ALL ? 0xffffffffu : khi;
      const float z_lo = smp_value(klo);
      each([&](int v, const float (&zz)[VEC]) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          if (!(zz[i] >= z_lo)) continue;
          const uint32_t key = smp_key(zz[i]);
          if (key >= klo && key <= top) {
            const int at = atomicAdd(&S0->st.n_list, 1);
            if (at < SMP_LIST) S0->lc[at] = (u64)key << 32 | (uint32_t)~(v * VEC + i);
          }
        }
      });
      sync();
      if (rank == 0) {
        const int n = min(S.st.n_list, SMP_LIST);
        const u64 me = tid < n ? S.lc[tid] : 0ull;
        const uint32_t key = (uint32_t)(me >> 32);
        const int idx = (int)~(uint32_t)me;
        const u64 w = tid < n ? weight(smp_value(key)) : 0ull;
        if (tid >= n && tid < SMP_LIST) S.lc[tid] = 0ull;  // (behind every candidate, without weight)
        if (tid < SMP_LIST) S.lw[tid] = w;
        if (tid == 0) S.st.thr = 0xffffffffu;
        __syncthreads();
        // Tokens, and their weight, in front of candidate tid (mod SMP_LIST): half of the list per half of the block.
        // On the whole list that is the order's rank, for a bin's the tokens of larger value.
        int front = 0;
        u64 front_m = 0ull;
        {
          const int c = tid & (SMP_LIST - 1), half = ((n + 7) >> 3) * 4, j0 = tid < SMP_LIST ? 0 : half;
          const u64 than = stage == SMP_GATHER_ALL ? S.lc[c] : S.lc[c] | 0xffffffffull;
          if ((c & ~31) < n) {
#pragma unroll 4
            for (int j = j0; j < min(j0 + half, SMP_LIST); j += 2) {
              const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(&S.lc[j]), ow = *reinterpret_cast<const ulonglong2*>(&S.lw[j]);
              if (o.x > than) { ++front; front_m += ow.x; }
              if (o.y > than) { ++front; front_m += ow.y; }
            }
          }
          if (tid >= SMP_LIST) {
            S.cnt[c] = (uint32_t)front;
            S.lo[c] = (uint32_t)front_m;
            S.hi[c] = (uint32_t)(front_m >> 32);
          }
          __syncthreads();
          if (tid < SMP_LIST) {
            front += (int)S.cnt[c];
            front_m += (u64)S.hi[c] << 32 | S.lo[c];
          }
        }
        if (stage == SMP_GATHER_BIN) {
          front += S.st.before;
          front_m += S.st.before_m;
          if (tid < n && (by_weight ? front_m < S.st.target : front < k)) atomicMin(&S.st.thr, key);
          if (tid == 0) S.st.eq = 0;
          __syncthreads();
          if (tid < n && key == S.st.thr) atomicAdd(&S.st.eq, 1);
          __syncthreads();
          if (tid < n && key == S.st.thr)                // (equal values written by each of them)
            S.st.ties = by_weight ? ties_by_weight(S.st.target - front_m, w, S.st.eq) : min(S.st.eq, k - front);
        } else {
          // everything is on the list: the filters, then the draw
          bool keep = tid < n && (by_weight || front < k);
          u64 target = S.st.target;
          if (!by_weight) target = reach(block_sum(keep ? w : 0ull));
          if (p < 1.f) keep = keep && front_m < target;
          keep = keep && key >= kb;
          const u64 kept = block_sum(keep ? w : 0ull);
          if (keep) atomicMin(&S.st.thr, key);
          if (tid < SMP_LIST) S.lw[tid] = keep ? w : 0ull;
          if (tid == 0) { S.st.first = 0x7fffffff; S.st.ties = 0; S.st.eq = 0; S.st.done_tok = 1; }
          __syncthreads();
          if (tid < n && key == S.st.thr) {
            atomicAdd(&S.st.eq, 1);
            if (keep) atomicAdd(&S.st.ties, 1);
          }
          if (out_tok) {
            const long long goal = draw_goal(kept);
            if (keep) {
              u64 run = 0ull;
#pragma unroll 4
              for (int j = 0; j < n; j += 2) {
                const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(&S.lc[j]), ow = *reinterpret_cast<const ulonglong2*>(&S.lw[j]);
                if ((uint32_t)o.x >= (uint32_t)me) run += ow.x;
                if ((uint32_t)o.y >= (uint32_t)me) run += ow.y;
              }
              if ((long long)run > goal) atomicMin(&S.st.first, idx);
            }
            __syncthreads();
            if (tid == 0) out_tok[r] = S.st.first;
          }
        }
        __syncthreads();
        if (tid == 0) S.st.n_list = 0;
        publish();
      }
      sync();
      break;
    }
  };
  uint32_t thr = SMP_NOTHING + 1u;
  int ties = V, eq = V;
  bool done = false;
  if (k > 0 && k < V) {
    select(false, SMP_NOTHING, 0, 0);
    thr = S.st.thr;
    ties = S.st.ties;
    eq = S.st.eq;
    done = S.st.done_tok != 0;
  }
  if (p < 1.f && !done) {
    const bool cuts = ties < V;                          // (tokens at top_k's threshold are counted apart)
    select(true, cuts ? thr : SMP_NOTHING, cuts ? ties : 0, cuts ? eq : 0);
    thr = S.st.thr;
    ties = S.st.ties;
    eq = S.st.eq;
    done = S.st.done_tok != 0;
  }
  if (kb > thr) { thr = kb; ties = eq = V; }

  // ---------------------------------------------------------------- the row and the draw
  const bool draw = out_tok && !done;
  if (out || draw) {
    // tokens equal to the threshold in front of this warp's run, where only some of them stay
    const bool some = ties < eq;
    const float zt = smp_value(thr);                     // z >= zt: at or above the threshold (+inf too, no NaN)
    int tie = 0;
    if (some) {
      int n = 0;
      each([&](int, const float (&zz)[VEC]) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) n += zz[i] >= zt && fminf(zz[i], SMP_BIG) == zt;
      });
      n = __reduce_add_sync(0xffffffffu, n);
      if (lane == 0) S0->weq[gw] = n;
      sync();
      if (rank == 0 && warp == 0) {                      // (lane l: W / 32 runs)
        constexpr int PER = SMP_CLUSTER * SMP_WARPS / 32;
        const int per = (W + 31) / 32, i0 = lane * per;
        int c[PER], mine = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          c[i] = i < per && i0 + i < W ? S.weq[i0 + i] : 0;
          mine += c[i];
        }
        int run = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, run, o);
          if (lane >= o) run += y;
        }
        run -= mine;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          if (i < per && i0 + i < W) S.weq[i0 + i] = run;
          run += c[i];
        }
      }
      sync();
      tie = S0->weq[gw];
    }
    // The kept tokens of vector v (none where !in), t: tokens equal to the threshold in front of the warp's vectors
    auto kept_of = [&](bool in, const float (&z)[VEC], int& t) {
      uint32_t keep = 0u;
#pragma unroll
      for (int i = 0; i < VEC; ++i) keep |= z[i] >= zt ? 1u << i : 0u;
      if (!in) keep = 0u;
      if (some) {
        uint32_t same = 0u;
#pragma unroll
        for (int i = 0; i < VEC; ++i) same |= fminf(z[i], SMP_BIG) == zt ? 1u << i : 0u;
        same &= keep;
        if (__any_sync(0xffffffffu, same != 0u)) {
          int x = __popc(same);
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
          }
          int at = t + x - __popc(same);
#pragma unroll
          for (int i = 0; i < VEC; ++i)
            if ((same >> i) & 1u) { if (at >= ties) keep &= ~(1u << i); ++at; }
          t += __shfl_sync(0xffffffffu, x, 31);
        }
      }
      return keep;
    };
    // f(vector, values, kept) for vectors [va, vb), in index order; the whole warp takes part
    auto kept_each = [&](int va, int vb, int t, auto f) {
      int v = va + lane;
      for (; v - lane + 128 <= vb; v += 128) {
        uint32_t raw[4][RAW];
#pragma unroll
        for (int q = 0; q < 4; ++q) load(v + 32 * q, raw[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float z[VEC];
          smp_unpack<T, VEC>(raw[q], z);
          const uint32_t keep = kept_of(true, z, t);
          f(v + 32 * q, z, keep);
        }
      }
      for (; v - lane < vb; v += 32) {
        uint32_t raw[RAW] = {};
        if (v < vb) load(v, raw);
        float z[VEC];
        smp_unpack<T, VEC>(raw, z);
        const uint32_t keep = kept_of(v < vb, z, t);
        if (v < vb) f(v, z, keep);
      }
    };
    auto write = [&](int v, const float (&z)[VEC], uint32_t keep) {
      float o[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        o[i] = (keep >> i) & 1u ? fmaxf(-SMP_BIG, fminf(SMP_BIG, fminf(z[i], SMP_BIG) / temp)) : -INFINITY;
      if constexpr (VEC == 4) __stcs(reinterpret_cast<float4*>(out) + v, make_float4(o[0], o[1], o[2], o[3]));
      else __stcs(out + v, o[0]);
    };
    auto write_nothing = [&](int v) {
      if constexpr (VEC == 4) __stcs(reinterpret_cast<float4*>(out) + v, make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY));
      else __stcs(out + v, -INFINITY);
    };
    if (!draw && !some) {
      each([&](int v, const float (&z)[VEC]) {
        uint32_t keep = 0u;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (z[i] >= zt) keep |= 1u << i;
        if (keep) write(v, z, keep);
        else write_nothing(v);
      });
    } else {
      // Weights of kept tokens.  bf16 takes them from a table by bin; fp32 forms those of a vector together, whether or
      // not all of its tokens stay: one at a time, each behind a branch, took twice as long.
      smp_map1 map;
      u64* wt = reinterpret_cast<u64*>(S.lo);
      const bool by_bin = sizeof(T) == 2 && draw;
      if (by_bin) {
        map.set(kmax, SMP_NOTHING, weight.cut, true);
        const int nb = map.np + 3 + map.nn;
        for (int b = tid; b < nb; b += SMP_THREADS) {
          uint32_t lo, hi;
          map.range(b, lo, hi);
          if (hi >= thr && map.single(b)) wt[b] = weight(smp_value(lo));
        }
        __syncthreads();
      }
      const float z_low = fmaxf(zt, weight.cut);
      // Twice: over all runs, then the block of the run that holds the draw over that run's parts, of which the warp
      // that holds it goes through its own token by token.
      int v0 = v_begin, v1 = v_end;
      long long goal = 0;
      for (int round = 0; round < 2; ++round) {
        u64 sum = 0ull;
        kept_each(v0, v1, tie, [&](int v, const float (&z)[VEC], uint32_t keep) {
          if (out && round == 0) {
            if (keep) write(v, z, keep);
            else write_nothing(v);
          }
          if (!keep) return;
          if (by_bin) {
            const int np3 = map.np + 3 - (int)map.mn, mb = (int)map.mb, mz = (int)map.mz;
            uint32_t odd = 0u;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              const int b = (int)__float_as_uint(z[i]), m = (b >> 16) & 0x7fff;
              const bool in = ((keep >> i) & 1u) && z[i] >= z_low, usual = m >= mb && m < 0x7f7f;
              if (in && usual) sum += wt[b < 0 ? m + np3 : mz - m];
              odd |= in && !usual ? 1u << i : 0u;
            }
            if (odd) {
#pragma unroll
              for (int i = 0; i < VEC; ++i)
                if ((odd >> i) & 1u) sum += weight(fminf(z[i], SMP_BIG));
            }
          } else if (draw) {
            u64 w[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[i] = weight(fminf(z[i], SMP_BIG));
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum += (keep >> i) & 1u ? w[i] : 0ull;
          }
        });
        if (!draw) break;
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (round == 0) {
          if (lane == 0) S0->wsum[gw] = sum;
          sync();
          // the first run whose end passes the goal
          if (rank == 0) {
            if (warp == 0) {                               // (lane l: W / 32 runs)
              constexpr int PER = SMP_CLUSTER * SMP_WARPS / 32;
              const int per = (W + 31) / 32, i0 = lane * per;
              u64 ws[PER], mine = 0ull;
#pragma unroll
              for (int i = 0; i < PER; ++i) {
                ws[i] = i < per && i0 + i < W ? S.wsum[i0 + i] : 0ull;
                mine += ws[i];
              }
              u64 incl = mine;
#pragma unroll
              for (int o = 1; o < 32; o <<= 1) {
                const u64 y = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += y;
              }
              const long long goal = draw_goal(__shfl_sync(0xffffffffu, incl, 31));
              u64 run = incl - mine;
#pragma unroll
              for (int i = 0; i < PER; ++i) {
                if ((long long)run <= goal && (long long)(run + ws[i]) > goal) {
                  S.st.win = i0 + i;
                  S.st.win_before = run;
                  S.st.goal = goal;
                }
                run += ws[i];
              }
            }
            publish();
          }
          sync();
          const int win = S.st.win;
          if (win / SMP_WARPS != rank) break;
          goal = S.st.goal;
          const int w0 = (int)min((long long)nv, (long long)win * chunk), w1 = (int)min((long long)nv, (long long)w0 + chunk);
          const int part = ((w1 - w0 + SMP_WARPS - 1) / SMP_WARPS + 31) / 32 * 32;
          v0 = min(w1, w0 + warp * part);
          v1 = min(w1, v0 + part);
          if (some) {
            int n = 0;
            for (int v = v0 + lane; v < v1; v += 32) {
              uint32_t raw[RAW];
              load(v, raw);
              float z[VEC];
              smp_unpack<T, VEC>(raw, z);
#pragma unroll
              for (int i = 0; i < VEC; ++i) n += z[i] >= zt && fminf(z[i], SMP_BIG) == zt;
            }
            n = __reduce_add_sync(0xffffffffu, n);
            if (lane == 0) S.redi[warp] = n;
            __syncthreads();
            tie = S0->weq[win];
            for (int i = 0; i < warp; ++i) tie += S.redi[i];
          }
        } else {
          if (lane == 0) S.red[warp] = sum;
          __syncthreads();
          u64 run = S.st.win_before;
          for (int i = 0; i < warp; ++i) run += S.red[i];
          if ((long long)run <= goal && (long long)(run + sum) > goal) {
            int t = tie;
            for (int v = v0 + lane; v - lane < v1; v += 32) {
              uint32_t raw[RAW] = {};
              if (v < v1) load(v, raw);
              float z[VEC];
              smp_unpack<T, VEC>(raw, z);
              const uint32_t keep = kept_of(v < v1, z, t);
              u64 w[VEC], x = 0ull;
#pragma unroll
              for (int i = 0; i < VEC; ++i) {
                w[i] = (keep >> i) & 1u ? weight(fminf(z[i], SMP_BIG)) : 0ull;
                x += w[i];
              }
              const u64 own = x;
#pragma unroll
              for (int o = 1; o < 32; o <<= 1) {
                const u64 y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
              }
              const uint32_t hit = __ballot_sync(0xffffffffu, keep && (long long)(run + x) > goal);
              if (hit) {
                if (lane == __ffs(hit) - 1) {
                  u64 c = run + x - own;
                  int tok = -1;
#pragma unroll
                  for (int i = 0; i < VEC; ++i) {
                    c += w[i];
                    if (tok < 0 && ((keep >> i) & 1u) && (long long)c > goal) tok = v * VEC + i;
                  }
                  out_tok[r] = tok;
                }
                break;
              }
              run += __shfl_sync(0xffffffffu, x, 31);
            }
          }
        }
      }
    }
  }
  sync();                                                // (the first block's memory is read until here)
}

template <typename T, int VEC>
static int smp_launch(jk_ctx* ctx, cudaStream_t st, int rows, const void* logits, int64_t stride, const float* temperature,
                      const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* out_tok,
                      float* out_logits) {
  const int V = ctx->cfg.vocab;
  const size_t smem = sizeof(smp_shared);
  JK_CUDA_CHECK(ctx, cudaFuncSetAttribute(k_sample<T, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  // Blocks per row: at least 2048 tokens each, and no more blocks than three per SM (two at a time run there).  One row of
  // 128256 in fp32 with top-p: 8 blocks 33 us, 4 46, 2 73, 1 116; 32 rows: 52, 56, 87, 148; 240 rows: 1 block 233, 2 236,
  // 4 255; in bf16 129, 147, 180.
  int C = SMP_CLUSTER;
  while (C > 1 && ((long long)rows * C > 3ll * ctx->sm_count || V / C < 2048)) C >>= 1;
  int bits = 0;
  while (bits < 31 && (1ll << bits) < V) ++bits;
  const int sh = bits <= 17 ? 45 : 62 - bits;
  jk_launch_pdl_cluster(k_sample<T, VEC>, dim3((unsigned)rows * C), dim3(SMP_THREADS), (unsigned)C, smem, st,
                        (const T*)logits, (long long)stride, V, C, sh, temperature, top_k, top_p, min_p, u, out_tok,
                        out_logits);
  JK_LAUNCH_CHECK(ctx);
  return JK_OK;
}

extern "C" int jk_sample(jk_ctx* ctx, void* stream, int32_t rows, const void* logits, int32_t logits_dtype,
                         int64_t row_stride, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, const float* u, int32_t* out_tok,
                         float* out_logits) {
  if (!ctx || !logits || (!out_tok && !out_logits) || (out_tok && !u)) return JK_ERR_NULL;
  if (logits_dtype != JK_F32 && logits_dtype != JK_BF16) return JK_ERR_DTYPE;
  const int V = ctx->cfg.vocab;
  if (rows < 1 || row_stride < V) return JK_ERR_SHAPE;
  if ((uintptr_t)logits % jk_elem_size(logits_dtype)) return JK_ERR_ALIGN;
  const void* words[] = {temperature, top_k, top_p, min_p, u, out_tok, out_logits};
  for (const void* p : words)
    if ((uintptr_t)p & 3) return JK_ERR_ALIGN;
  if (out_logits) {
    // the filtered rows are written while the logits are still read
    const uintptr_t z0 = (uintptr_t)logits, z1 = z0 + ((size_t)(rows - 1) * row_stride + V) * jk_elem_size(logits_dtype);
    const uintptr_t o0 = (uintptr_t)out_logits, o1 = o0 + (size_t)rows * V * 4;
    if (z0 < o1 && o0 < z1) return JK_ERR_SHAPE;
  }
  const int rc = jk_ensure_device_info(ctx);
  if (rc != JK_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  JK_PROF(ctx, st, JK_ST_SAMPLE);
  // four tokens per access where every row of the input and of the output starts on four tokens' boundary
  const int es = jk_elem_size(logits_dtype);
  const bool wide = V % 4 == 0 && row_stride % 4 == 0 && (uintptr_t)logits % (4 * es) == 0 && (uintptr_t)out_logits % 16 == 0;
  auto go = logits_dtype == JK_BF16 ? (wide ? smp_launch<__nv_bfloat16, 4> : smp_launch<__nv_bfloat16, 1>)
                                    : (wide ? smp_launch<float, 4> : smp_launch<float, 1>);
  return go(ctx, st, rows, logits, row_stride, temperature, top_k, top_p, min_p, u, out_tok, out_logits);
}
