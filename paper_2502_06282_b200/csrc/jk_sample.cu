// jk_sample: temperature, top-k, top-p and min-p over rows of logits, the draw of a token and the filtered
// rows (the sampled form of arXiv 2502.06282, Sec. 2.1 steps 2-3, draws with a temperature only).
//
// Logits are compared through their ordered 32-bit image (larger logit = larger unsigned integer).  Every filter
// is a prefix of (logit descending, index ascending), so the kept set is a threshold on the image plus a number of
// tokens equal to the threshold, lowest index first.  Both thresholds (by count for top-k, by weight for top-p) are
// found in a histogram of the row:
//   - a bin is the upper half of the image (sign, exponent, 7 bits), over the 20 octaves that hold the largest
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
#include <math.h>

#include "jk_common.cuh"

#define SMP_THREADS 512
#define SMP_WARPS (SMP_THREADS / 32)
#define SMP_CLUSTER 8
#define SMP_LIST 256                  // candidates that are compared with one another
#define SMP_OCTAVES 20
#define SMP_BINS 5632                 // >= 2 * 128 * SMP_OCTAVES + 4, a multiple of SMP_THREADS
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

struct smp_state {                    // of the row, in the cluster's first block
  int stage;                          // what comes next: one of SMP_*
  uint32_t klo, khi;                  // images of the bin that holds the threshold
  int n, before;                      // tokens in it and above it
  u64 before_m, total, target;        // weight above it, of all tokens of the filter, and to be reached
  uint32_t thr;                       // result: threshold, tokens equal to it that stay, and that there are
  int ties, eq;
  int n_list, first, done_tok;
};
enum { SMP_GATHER_ALL, SMP_GATHER_BIN, SMP_REFINE, SMP_FOUND };

struct smp_shared {
  uint32_t cnt[SMP_BINS], lo[SMP_BINS], hi[SMP_BINS];
  double table[64];                   // 2^(j / 64)
  smp_state st;
  uint32_t lkey[SMP_LIST];
  int lidx[SMP_LIST];
  u64 lw[SMP_LIST];
  u64 wsum[SMP_CLUSTER * SMP_WARPS];  // per warp of the cluster (first block's copy)
  int wlast[SMP_CLUSTER * SMP_WARPS], weq[SMP_CLUSTER * SMP_WARPS];
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
// a generic address of the same variable in block `rank` of the cluster
template <typename P> __device__ __forceinline__ P* smp_map(P* p, uint32_t rank) {
  u64 a;
  asm("mapa.u64 %0, %1, %2;" : "=l"(a) : "l"((u64)p), "r"(rank));
  return reinterpret_cast<P*>(a);
}

// Weights: exp((z - zmax) / T) in units of 2^-sh.  2^(n / 64) from a table, the rest (at most ln2 / 128) by the power
// series to the fifth term: 4e-17 off, next to the 4e-15 of the reduced argument.
struct smp_weight {
  double zmax, inv_t, limit, magic;
  const double* table;
  __device__ __forceinline__ u64 operator()(float z) const {
    const double x = ((double)z - zmax) * inv_t;
    if (!(x >= limit)) return 0ull;
    const double big = 6755399441055744.0;               // 1.5 * 2^52: the integer part stands in the low bits
    const double nb = fma(x, 92.332482616893656877, big);  // 64 / ln 2
    const int n = __double2loint(nb);
    const double r = fma(nb - big, -0.010830424696249145248, x);
    double p = fma(r, 1.0 / 120.0, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    const double t = table[n & 63];
    const double w = __hiloint2double(__double2hiint(t) + ((n >> 6) << 20), __double2loint(t)) * p;
    return (u64)__double_as_longlong(w + magic) - (u64)__double_as_longlong(magic);
  }
};

// Bins of the first histogram.
struct smp_map1 {
  uint32_t mz, mb, mn;                // upper half of the largest |z| of positive tokens, of the smallest, of negative ones
  int np, nn;                         // bins of positive and of negative values
  float cut;                          // below: no weight
  uint32_t kcut, kfloor;
  bool bf16;
  __device__ void set(uint32_t kmax, uint32_t floor_key, float T, double limit, bool is_bf16) {
    const float zmax = smp_value(kmax);
    const double c = (double)zmax + (limit - 1.0) * (double)T;
    cut = fmaxf((float)c, -SMP_BIG);
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
    const uint32_t b = __float_as_uint(z), m = (b >> 16) & 0x7fffu;
    if (z == 0.f) return np + 1;
    if (m < mb) return z > 0.f ? np : np + 2;
    return z > 0.f ? (int)(mz - m) : np + 3 + (int)(m - mn);
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
  smp_shared* S0 = C > 1 ? smp_map(&S, 0) : &S;          // the first block's
  auto sync = [&]() {
    if (C > 1) {
      asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
      __syncthreads();
    }
  };
  jk_pdl_wait();
  jk_pdl_trigger();
  const T* z0 = logits + (size_t)r * stride;
  float* out = out_logits ? out_logits + (size_t)r * V : nullptr;
  // every warp of the cluster owns a run of the row, in index order
  const int nv = V / VEC;
  const int W = C * SMP_WARPS, chunk = ((nv + W - 1) / W + 31) / 32 * 32, gw = rank * SMP_WARPS + warp;
  const int v_begin = (int)min((long long)nv, (long long)gw * chunk), v_end = (int)min((long long)nv, (long long)v_begin + chunk);
  // f(index of the lane's vector, its VEC values); lanes behind the run's end get NaN and index -1 where `all`
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
    if (tid < 64) S.table[tid] = exp2(tid / 64.0);
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
  for (int i = 0; i < C; ++i) kmax = max(kmax, C > 1 ? smp_map(&S.kmax, i)[0] : S.kmax);
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
  weight.limit = -0.6931471805599454 * (sh + 1);         // half a unit and below: nothing
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
    kb = smp_key(fmaxf((float)((double)zmax + bound), -SMP_BIG));
    while (kb > SMP_NOTHING + 1u && ok(kb - 1u)) --kb;
    while (!ok(kb)) ++kb;
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
  auto ties_by_weight = [&](u64 missing, u64 w, int most) {  // tokens of weight w until `missing` is reached
    const u64 n = (missing + w - 1ull) / max(w, 1ull);
    return (int)min(n, (u64)most);
  };

  // Finds the threshold among the tokens above floor_key (tokens that are equal to it add `extra` of weight, and
  // ties_f of eq_f of them count).  Everything that is decided is decided by the first block.
  auto select = [&](bool by_weight, uint32_t floor_key, int ties_f, int eq_f) {
    smp_map1 map;
    map.set(kmax, floor_key, temp, weight.limit, sizeof(T) == 2);
    const float z_floor = smp_value(floor_key);
    uint32_t klo = 0u, khi = 0xffffffffu;
    int shift = 0;
    for (int level = 0;; ++level) {
      // ------------------------------------------------ histogram
      const int nb = level == 0 ? map.bins() : (int)((khi - klo) >> shift) + 1;
      for (int i = tid; i < nb; i += SMP_THREADS) {
        S.cnt[i] = 0u;
        if (by_weight) { S.lo[i] = 0u; S.hi[i] = 0u; }
      }
      __syncthreads();
      auto add = [&](int b, bool weigh, float z) {
        atomicAdd(&S.cnt[b], 1u);
        if (weigh) {
          const u64 w = weight(z);
          const uint32_t l = (uint32_t)w, old = atomicAdd(&S.lo[b], l);
          const uint32_t h = (uint32_t)(w >> 32) + (old + l < old ? 1u : 0u);
          if (h) atomicAdd(&S.hi[b], h);
        }
      };
      if (level == 0) {
        int rest = 0;
        each([&](int, const float (&zz)[VEC]) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const float z = fminf(zz[i], SMP_BIG);       // (a NaN becomes the largest float)
            if (z > z_floor && zz[i] == zz[i]) {
              if (z >= map.cut) {
                const int b = map.bin(z);
                add(b, by_weight && !map.single(b), z);
              } else {
                ++rest;
              }
            }
          }
        });
        rest = __reduce_add_sync(0xffffffffu, rest);
        if (lane == 0 && rest) atomicAdd(&S.cnt[nb - 1], (uint32_t)rest);
      } else {
        each([&](int, const float (&zz)[VEC]) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const uint32_t key = smp_key(zz[i]);
            if (key >= klo && key <= khi) add((int)((khi - key) >> shift), by_weight && shift > 0, smp_value(key));
          }
        });
      }
      sync();
      if (C > 1) {
        // block `rank` adds up its part of the bins in the first block's memory
        const int per = (nb + C - 1) / C, b1 = min(nb, (rank + 1) * per);
        for (int b = rank * per + tid; b < b1; b += SMP_THREADS) {
          uint32_t n = 0u;
          u64 m = 0ull;
          for (int i = 0; i < C; ++i) {
            smp_shared* o = smp_map(&S, i);
            n += o->cnt[b];
            if (by_weight) m += (u64)o->hi[b] << 32 | o->lo[b];
          }
          S0->cnt[b] = n;
          if (by_weight) { S0->lo[b] = (uint32_t)m; S0->hi[b] = (uint32_t)(m >> 32); }
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
        int n = 0;
        u64 m = 0ull;
        for (int b = b0; b < b1; ++b) {
          const uint32_t c = S.cnt[b];
          n += c;
          if (by_weight) {
            if (c && (level == 0 ? map.single(b) : shift == 0)) {
              uint32_t lo, hi;
              range(b, lo, hi);
              const u64 w = (u64)c * weight(smp_value(lo));
              S.lo[b] = (uint32_t)w;
              S.hi[b] = (uint32_t)(w >> 32);
            }
            m += (u64)S.hi[b] << 32 | S.lo[b];
          }
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
      sync();
      const int stage = S0->st.stage;
      klo = S0->st.klo;
      khi = S0->st.khi;
      if (stage == SMP_FOUND) break;
      if (stage == SMP_REFINE) {
        shift = 0;
        while (((khi - klo) >> shift) >= SMP_LEVEL) ++shift;
        __syncthreads();
        continue;
      }
      // ------------------------------------------------ candidates
      const uint32_t top = stage == SMP_GATHER_ALL ? 0xffffffffu : khi;
      each([&](int v, const float (&zz)[VEC]) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const uint32_t key = smp_key(zz[i]);
          if (key >= klo && key <= top) {
            const int at = atomicAdd(&S0->st.n_list, 1);
            if (at < SMP_LIST) { S0->lkey[at] = key; S0->lidx[at] = v * VEC + i; }
          }
        }
      });
      sync();
      if (rank == 0) {
        const int n = min(S.st.n_list, SMP_LIST);
        const uint32_t key = tid < n ? S.lkey[tid] : 0u;
        const int idx = tid < n ? S.lidx[tid] : 0;
        const u64 w = tid < n ? weight(smp_value(key)) : 0ull;
        if (tid < n) S.lw[tid] = w;
        if (tid == 0) S.st.thr = 0xffffffffu;
        __syncthreads();
        if (stage == SMP_GATHER_BIN) {
          int above = S.st.before, same = 0;
          u64 above_m = S.st.before_m;
          if (tid < n) {
            for (int j = 0; j < n; ++j) {
              const uint32_t kj = S.lkey[j];
              same += kj == key;
              if (kj > key) { ++above; above_m += S.lw[j]; }
            }
            if (by_weight ? above_m < S.st.target : above < k) atomicMin(&S.st.thr, key);
          }
          __syncthreads();
          if (tid < n && key == S.st.thr) {              // (equal values written by each of them)
            S.st.eq = same;
            S.st.ties = by_weight ? ties_by_weight(S.st.target - above_m, w, same) : min(same, k - above);
          }
        } else {
          // everything on the list: rank and weight before each token, then the filters, then the draw
          int better = 0;
          u64 before = 0ull;
          if (tid < n) {
            for (int j = 0; j < n; ++j) {
              const uint32_t kj = S.lkey[j];
              if (kj > key || (kj == key && S.lidx[j] < idx)) { ++better; before += S.lw[j]; }
            }
          }
          bool keep = tid < n && (by_weight || better < k);
          u64 target = S.st.target;
          if (!by_weight) target = reach(block_sum(keep ? w : 0ull));
          if (p < 1.f) keep = keep && before < target;
          keep = keep && key >= kb;
          const u64 kept = block_sum(keep ? w : 0ull);
          if (keep) atomicMin(&S.st.thr, key);
          if (tid < n) S.lw[tid] = keep ? w : 0ull;
          if (tid == 0) { S.st.first = 0x7fffffff; S.st.ties = 0; S.st.eq = 0; S.st.done_tok = 1; }
          __syncthreads();
          if (tid < n && key == S.st.thr) {
            atomicAdd(&S.st.eq, 1);
            if (keep) atomicAdd(&S.st.ties, 1);
          }
          if (out_tok) {
            const long long goal = uu >= 0.f ? (long long)((double)uu * (double)kept) : uu < 0.f ? -1ll : 0x7fffffffffffffffll;
            u64 run = 0ull;
            int last = -1;
            if (keep) {
              for (int j = 0; j < n; ++j)
                if (S.lidx[j] <= idx) run += S.lw[j];
              if ((long long)run > goal) atomicMin(&S.st.first, idx);
              last = idx;
            }
            last = __reduce_max_sync(0xffffffffu, last);
            if (lane == 0) S.redi[warp] = last;
            __syncthreads();
            if (tid == 0) {
              int t = S.st.first;
              if (t == 0x7fffffff)
                for (int i = 0; i < SMP_WARPS; ++i) t = i == 0 ? S.redi[0] : max(t, S.redi[i]);
              out_tok[r] = t;
            }
          }
        }
        __syncthreads();
        if (tid == 0) S.st.n_list = 0;
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
    thr = S0->st.thr;
    ties = S0->st.ties;
    eq = S0->st.eq;
    done = S0->st.done_tok != 0;
    sync();
  }
  if (p < 1.f && !done) {
    const bool cuts = ties < V;                          // (tokens at top_k's threshold are counted apart)
    select(true, cuts ? thr : SMP_NOTHING, cuts ? ties : 0, cuts ? eq : 0);
    thr = S0->st.thr;
    ties = S0->st.ties;
    eq = S0->st.eq;
    done = S0->st.done_tok != 0;
    sync();
  }
  if (kb > thr) { thr = kb; ties = eq = V; }

  // ---------------------------------------------------------------- the row and the draw
  const bool draw = out_tok && !done;
  if (out || draw) {
    // tokens equal to the threshold in front of this warp's run, where only some of them stay
    const bool some = ties < eq;
    int tie = 0;
    if (some) {
      int n = 0;
      each([&](int, const float (&zz)[VEC]) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) n += smp_key(zz[i]) == thr;
      });
      n = __reduce_add_sync(0xffffffffu, n);
      if (lane == 0) S0->weq[gw] = n;
      sync();
      for (int i = lane; i < gw; i += 32) tie += S0->weq[i];
      tie = __reduce_add_sync(0xffffffffu, tie);
    }
    // f(vector or -1, values, kept): the whole warp, in index order
    auto kept_each = [&](auto f) {
      const int t0 = tie;
      int t = t0;
      for (int v = v_begin + lane; v - lane < v_end; v += 32) {
        uint32_t raw[RAW] = {};
        const bool in = v < v_end;
        if (in) load(v, raw);
        float z[VEC];
        smp_unpack<T, VEC>(raw, z);
        uint32_t keep = 0u, same = 0u;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const uint32_t key = in ? smp_key(z[i]) : 0u;
          if (key >= thr) keep |= 1u << i;
          if (key == thr) same |= 1u << i;
        }
        if (some) {
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
        if (!f(in ? v : -1, z, keep)) break;
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
    if (!draw && !some) {
      each([&](int v, const float (&z)[VEC]) {
        uint32_t keep = 0u;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (smp_key(z[i]) >= thr) keep |= 1u << i;
        write(v, z, keep);
      });
    } else {
      u64 sum = 0ull;
      int last = -1;
      kept_each([&](int v, const float (&z)[VEC], uint32_t keep) {
        if (v >= 0 && out) write(v, z, keep);
        if (draw && keep) {
#pragma unroll
          for (int i = 0; i < VEC; ++i)
            if ((keep >> i) & 1u) { sum += weight(fminf(z[i], SMP_BIG)); last = v * VEC + i; }
        }
        return true;
      });
      if (draw) {
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        last = __reduce_max_sync(0xffffffffu, last);
        if (lane == 0) { S0->wsum[gw] = sum; S0->wlast[gw] = last; }
        sync();
        // the first run whose end passes the goal; the last kept token if none does
        u64 all = 0ull, before = 0ull;
        int end = -1;
        for (int i = lane; i < W; i += 32) {
          const u64 s = S0->wsum[i];
          all += s;
          if (i < gw) before += s;
          end = max(end, S0->wlast[i]);
        }
        for (int o = 16; o > 0; o >>= 1) {
          all += __shfl_xor_sync(0xffffffffu, all, o);
          before += __shfl_xor_sync(0xffffffffu, before, o);
        }
        end = __reduce_max_sync(0xffffffffu, end);
        const long long goal = uu >= 0.f ? (long long)((double)uu * (double)all) : uu < 0.f ? -1ll : 0x7fffffffffffffffll;
        if (goal >= (long long)all) {
          if (gw == 0 && lane == 0) out_tok[r] = end;
        } else if (last >= 0 && (long long)(before + sum) > goal) {
          // is an earlier run with a kept token past it too?
          bool earlier = false;
          u64 run = 0ull;
          for (int i = 0; i < gw; ++i) {
            run += S0->wsum[i];
            earlier |= S0->wlast[i] >= 0 && (long long)run > goal;
          }
          if (!earlier) {
            run = before;
            kept_each([&](int v, const float (&z)[VEC], uint32_t keep) {
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
                return false;
              }
              run += __shfl_sync(0xffffffffu, x, 31);
              return true;
            });
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
  // Blocks per row: as many as the machine takes at once (three blocks fit an SM), and at least 2048 tokens each.
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
