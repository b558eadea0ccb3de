// Log-probabilities of given tokens under softmax(z / T), with entropy and the most likely
// alternatives, and their gradient in the logits.
//
//   y_x = (z_x - max) / T,  S = sum exp(y),  W = sum exp(y) y  (both W <= 0 and log S >= 0)
//   log p_x = y_x - log S,  H = log S - W / S      (a difference of terms of opposite sign: no cancellation)
//   d/dz_x = ([x = id] g - p_x (g + gH (log p_x + H))) / T
//
// Forward: one pass over the logits.  A wave takes a stretch of one row (4096 ids; a quarter
// of that in float32 and half in bf16 where there are few rows), all its loads in flight before the first exponential,
// and leaves the stretch's (max, S, W) and, where alternatives are asked for, the maxima of groups of its
// lanes' ids, which cost nothing beside the stretch's own: no barrier, nothing shared between waves.  Then one
// wave (or, with alternatives, one workgroup) per row joins the stretches; the alternatives come from the few
// groups whose maxima reach a bound, which are read again.
// Backward: one elementwise pass.  Both are bound by HBM: 4096 x 151936 float32 forward 378 us (6.6 TB/s), bf16 backward
// 486 us (5.1 TB/s; a copy of 2 GiB reaches 4.9); the bf16 forward (238 us, 5.2 TB/s) by its exponentials too.
// 64 x 151936 float32 with 8 alternatives: 15.4 us, of which each of the two launches takes about half.
#include "common.h"
#include "forward.h"

namespace gm {

namespace {
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;
constexpr float kLowest = -16384.f;    // exponents (of 2) below this are 0 already; finite, so that 0 * y is 0

typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned int u32x4h_t __attribute__((ext_vector_type(4), aligned(2)));
typedef __bf16 bfx2_t __attribute__((ext_vector_type(2)));
typedef float fx2_t __attribute__((ext_vector_type(2)));

// kPer consecutive logits in 16 bytes, at any element (global loads of 16 bytes take any alignment);
// bf16 stays packed and is widened where it is used
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int kPer = 4;
  f32x4u_t r;
  __device__ __forceinline__ void load(const float *p) { r = *reinterpret_cast<const f32x4u_t *>(p); }
  __device__ __forceinline__ void load_once(const float *p) {   // read once per launch
    r = __builtin_nontemporal_load(reinterpret_cast<const f32x4u_t *>(p));
  }
  __device__ __forceinline__ float get(int i) const { return r[i]; }
  __device__ __forceinline__ void set(int i, float v) { r[i] = v; }
  __device__ __forceinline__ void set2(int i, float a, float b) {
    r[i] = a;
    r[i + 1] = b;
  }
  // keeps what was computed from the values from being held for their next use
  __device__ __forceinline__ void opaque() {}
  template <bool NT> __device__ __forceinline__ void store(float *p) const {
    if (NT) __builtin_nontemporal_store(r, reinterpret_cast<f32x4u_t *>(p));
    else *reinterpret_cast<f32x4u_t *>(p) = r;
  }
  static __device__ __forceinline__ float one(const float *p) { return *p; }
  static __device__ __forceinline__ void put(float *p, float v) { *p = v; }
};
template <> struct Vec<bf16> {
  static constexpr int kPer = 8;
  u32x4h_t r;
  __device__ __forceinline__ void load(const bf16 *p) { r = *reinterpret_cast<const u32x4h_t *>(p); }
  __device__ __forceinline__ void load_once(const bf16 *p) {
    r = __builtin_nontemporal_load(reinterpret_cast<const u32x4h_t *>(p));
  }
  __device__ __forceinline__ float get(int i) const {
    return __uint_as_float(i & 1 ? r[i >> 1] & 0xffff0000u : r[i >> 1] << 16);
  }
  __device__ __forceinline__ void set(int i, float v) {     // (a bf16 value: from `one`, or an infinity)
    const uint32_t h = __float_as_uint(v) >> 16;
    r[i >> 1] = i & 1 ? (r[i >> 1] & 0x0000ffffu) | h << 16 : (r[i >> 1] & 0xffff0000u) | h;
  }
  __device__ __forceinline__ void set2(int i, float a, float b) {   // values i, i + 1 (i even), round to nearest even
    r[i >> 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(fx2_t{a, b}, bfx2_t));
  }
  __device__ __forceinline__ void opaque() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w = r[i];
      asm volatile("" : "+v"(w));
      r[i] = w;
    }
  }
  template <bool NT> __device__ __forceinline__ void store(bf16 *p) const {
    if (NT) __builtin_nontemporal_store(r, reinterpret_cast<u32x4h_t *>(p));
    else *reinterpret_cast<u32x4h_t *>(p) = r;
  }
  static __device__ __forceinline__ float one(const bf16 *p) { return bf16_to_f32(p->bits); }
  static __device__ __forceinline__ void put(bf16 *p, float v) { p->bits = f32_to_bf16(v); }
};

// Reductions over groups of lanes in the vector ALU (DPP): pairs, quads, 8, 16; the four rows of 16 by shuffles.
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int LANES> __device__ __forceinline__ float group_max(float v) {   // over LANES neighbours: 1, 4, 16 or 64
  if (LANES >= 4) {
    v = fmaxf(v, dpp<0xB1>(v));      // quad_perm 1, 0, 3, 2
    v = fmaxf(v, dpp<0x4E>(v));      // quad_perm 2, 3, 0, 1
  }
  if (LANES >= 16) {
    v = fmaxf(v, dpp<0x141>(v));     // row_half_mirror
    v = fmaxf(v, dpp<0x140>(v));     // row_mirror
  }
  if (LANES >= 64) {
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    v = fmaxf(v, __shfl_xor(v, 32, kWave));
  }
  return v;
}
__device__ __forceinline__ float lanes_sum(float v) {
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  v += dpp<0x141>(v);
  v += dpp<0x140>(v);
  v += __shfl_xor(v, 16, kWave);
  return v + __shfl_xor(v, 32, kWave);
}

__device__ __forceinline__ uint32_t order_key(float x) {   // larger float, larger key (-0 as +0)
  uint32_t u = __float_as_uint(x);
  if (u == 0x80000000u) u = 0u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Over one stretch of one row, with exponents of 2: S = sum 2^(z L - ref), W = sum 2^(z L - ref) (z L - ref), where
// L is log2 e / T in float32 and ref is max L rounded to float32: whatever its rounding, it is the same one
// for every term and for the join.
struct LpPart {
  float max, s, w, ref;
};

// ---------------------------------------------------------------- forward
// LG: lanes per group of the alternatives' selection (a group is LG neighbouring lanes' ids of all loads of a
// stretch, lp_group_id), 0: no group maxima are wanted
template <typename T, int kVecs, int LG>
__global__ __launch_bounds__(256) void lp_part_kernel(int M, int V, int parts, const T *__restrict__ logits, long ld,
                                                      float scale, LpPart *__restrict__ out,
                                                      float *__restrict__ groups) {
  constexpr int kPer = Vec<T>::kPer, kIds = 64 * kPer * kVecs;
  const int lane = threadIdx.x & 63, part = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (part >= parts) return;
  const int lo = part * kIds;
  for (long r = blockIdx.x; r < M; r += gridDim.x) {
    const T *row = logits + r * ld;
    Vec<T> v[kVecs];
    if (lo + kIds <= V) {
#pragma unroll
      for (int u = 0; u < kVecs; ++u) v[u].load_once(row + lo + (u * 64 + lane) * kPer);
    } else {
#pragma unroll
      for (int u = 0; u < kVecs; ++u) {
        const int x = lo + (u * 64 + lane) * kPer;
        if (x + kPer <= V) {
          v[u].load(row + x);
        } else {
#pragma unroll
          for (int i = 0; i < kPer; ++i) v[u].set(i, x + i < V ? Vec<T>::one(row + x + i) : -INFINITY);
        }
      }
    }
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < kVecs; ++u)
#pragma unroll
      for (int i = 0; i < kPer; i += 2) m = fmaxf(m, fmaxf(v[u].get(i), v[u].get(i + 1)));
    if constexpr (LG > 0) {
      const float g = group_max<LG>(m);
      if (lane % LG == 0) groups[(r * parts + part) * (64 / LG) + lane / LG] = g;
    }
    m = group_max<64>(m);
    // a stretch of -inf only: S and W are 0 (a NaN, which the maximum passes over, still reaches S)
    float ref = m == -INFINITY ? 0.f : m * scale;
    float s[2] = {0.f, 0.f}, w[2] = {0.f, 0.f};
    auto sums = [&](auto exponent) {
#pragma unroll
      for (int u = 0; u < kVecs; ++u) {
        v[u].opaque();
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const float y = exponent(v[u].get(i)), e = __builtin_amdgcn_exp2f(y);
          s[i & 1] += e;
          w[i & 1] += e * fmaxf(y, kLowest);
        }
      }
    };
    if (fabsf(ref) < INFINITY) {
      sums([&](float z) { return __builtin_fmaf(z, scale, -ref); });
    } else {       // max / T is past float32's range (or the row holds +inf): from the difference, which is not
      sums([&](float z) { return (z - m) * scale; });
    }
    const float S = lanes_sum(s[0] + s[1]), W = lanes_sum(w[0] + w[1]);
    if (lane == 0) out[r * parts + part] = LpPart{m, S, W, ref};
  }
}

struct LpRow {
  float max;        // largest logit
  double s, log_s, ent;      // s = sum exp((z - max) / T)
};
// The row's statistics from its stretches, in every lane of the wave that asks (a fixed order).  A stretch's
// terms are 2^(z L - ref); relative to the row's maximum they are 2^(ref - max L) of that, in float64.
__device__ __forceinline__ LpRow lp_join(const LpPart *__restrict__ p, int parts, float scale) {
  const int lane = threadIdx.x & 63;
  LpPart c[kLpMaxParts / 64];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kLpMaxParts / 64; ++i) {
    if (64 * i >= parts) break;
    c[i] = 64 * i + lane < parts ? p[64 * i + lane] : LpPart{-INFINITY, 0.f, 0.f, 0.f};
    m = fmaxf(m, c[i].max);
  }
  LpRow r;
  r.max = wave_max(m);
  const double top = (double)r.max * (double)scale;
  double s = 0.0, w = 0.0;
#pragma unroll
  for (int i = 0; i < kLpMaxParts / 64; ++i) {
    if (64 * i >= parts) break;
    if (c[i].s != 0.f) {                 // (also a NaN)
      const double ref = fabsf(c[i].ref) < INFINITY ? (double)c[i].ref : (double)c[i].max * (double)scale;
      const double y = c[i].max == -INFINITY ? 0.0 : ref - top;
      const double f = exp2(y);
      s += c[i].s * f;
      if (f != 0.0) w += (c[i].w + c[i].s * y) * f;
    }
  }
  r.s = wave_sum(s);
  w = wave_sum(w);
  r.log_s = r.s == 0.0 ? -INFINITY : log(r.s);
  r.ent = r.s == 0.0 ? 0.0 : r.log_s - w / r.s * kLn2;
  return r;
}
template <typename T>
__device__ __forceinline__ void lp_write(const LpRow &st, long r, int V, const T *__restrict__ row, double inv_t,
                                         const LpOut &o) {
  if (o.logp) {
    const int id = o.ids[r];
    if (id >= V) raise_dev_err(o.dev_err, GM_DEVERR_TOKEN);
    float lp = 0.f;
    if (id >= 0 && id < V) {
      const double z = Vec<T>::one(row + id);
      lp = st.s == 0.0 ? -INFINITY : (float)((z - (double)st.max) * inv_t - st.log_s);
    }
    o.logp[r] = lp;
  }
  if (o.entropy) o.entropy[r] = (float)st.ent;
  if (o.stats) o.stats[r] = gm_token_stats{st.max, (float)st.s};
}

template <typename T>
__global__ __launch_bounds__(256) void lp_row_kernel(int M, int V, int parts, const T *__restrict__ logits, long ld,
                                                     float scale, double inv_t, const LpPart *__restrict__ part,
                                                     LpOut o) {
  const long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= M) return;
  const LpRow st = lp_join(part + r * parts, parts, scale);
  if ((threadIdx.x & 63) == 0) lp_write(st, r, V, logits + r * ld, inv_t, o);
}

// Lane l of the wave holds the keys of groups 64 i + l; keys of groups past n are 0 and not counted.
constexpr int kKeys = kLpMaxGroups / 64;
// groups whose key is at least c
__device__ __forceinline__ int groups_from(const uint32_t (&key)[kKeys], int n, uint32_t c) {
  const int lane = threadIdx.x & 63;
  int cnt = 0;
#pragma unroll
  for (int i = 0; i < kKeys; ++i) {
    if (64 * i >= n) break;
    cnt += __popcll(__ballot(64 * i + lane < n && key[i] >= c));
  }
  return cnt;
}
__device__ __forceinline__ float key_value(uint32_t k) {   // the float of an order key
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
// Logits by rank: larger first, the lower id first among equals.
__device__ __forceinline__ unsigned long long rank_key(int id, uint32_t key) {
  return (unsigned long long)key << 32 | (uint32_t)(0x7fffffff - id);
}

// One workgroup per row: statistics (wave 1), then the alternatives.
// Wave 0 bounds them from the group maxima: the topk-th largest of its 64 lanes' own maxima is reached by topk
// groups at least, so nothing below that bound t is among the best, and the groups that reach it hold all that
// is.  Where more than kLpWins do (many alternatives), t becomes the topk-th largest group maximum.  Where that many
// still do (long ties), only the groups above t are read, fewer than topk; what is missing then are the lowest
// ids whose logit is t itself, which one ordered pass over the row finds.
constexpr int kLpWins = 128;
template <typename T>
__global__ __launch_bounds__(256) void lp_top_kernel(int M, int V, int parts, int vecs, int lg, int topk,
                                                     const T *__restrict__ logits, long ld, float scale, double inv_t,
                                                     const LpPart *__restrict__ part,
                                                     const float *__restrict__ groups, LpOut o) {
  constexpr int kPer = Vec<T>::kPer, kCap = 1024;
  __shared__ int win[kLpWins];             // the groups that are read
  __shared__ uint32_t thr_sh;
  __shared__ int n_sh, wins_sh, ties_sh, cnt_sh[4];
  __shared__ unsigned long long cand[kCap];
  __shared__ LpRow st_sh;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const long r = blockIdx.x;
  const T *row = logits + r * ld;
  const int per_part = 64 / lg, n_groups = parts * per_part;
  if (w == 1) {
    const LpRow st = lp_join(part + r * parts, parts, scale);
    if (lane == 0) {
      st_sh = st;
      lp_write(st, r, V, row, inv_t, o);
    }
  }
  if (w == 0) {
    uint32_t key[kKeys], best = 0;
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      if (64 * i >= n_groups) break;
      key[i] = 64 * i + lane < n_groups ? order_key(groups[r * n_groups + 64 * i + lane]) : 0u;
      best = max(best, key[i]);
    }
    uint32_t t = 0;
    for (int bit = 31; bit >= 0; --bit)
      if (__popcll(__ballot(best >= (t | 1u << bit))) >= topk) t |= 1u << bit;
    if (groups_from(key, n_groups, t) > kLpWins) {
      t = 0;                 // the largest t that at least topk groups reach (or one that topk reach exactly)
      for (int bit = 31; bit >= 0; --bit) {
        const int cnt = groups_from(key, n_groups, t | 1u << bit);
        if (cnt >= topk) t |= 1u << bit;
        if (cnt == topk) break;
      }
    }
    const bool ties = groups_from(key, n_groups, t) > kLpWins;
    int at = 0;
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      if (64 * i >= n_groups) break;
      const bool take = 64 * i + lane < n_groups && (ties ? key[i] > t : key[i] >= t);
      const unsigned long long mt = __ballot(take);
      if (take) win[at + __popcll(mt & ((1ull << lane) - 1))] = 64 * i + lane;
      at += __popcll(mt);
    }
    if (lane == 0) {
      thr_sh = t;
      wins_sh = at;
      ties_sh = ties;
      n_sh = 0;
    }
  }
  __syncthreads();
  const LpRow st = st_sh;
  if (st.s != st.s) {       // NaN or +inf in the row: no order that means anything
    if (tid < topk) {
      o.top_ids[r * topk + tid] = -1;
      o.top_logp[r * topk + tid] = (float)st.s;
    }
    return;
  }
  const int wins = wins_sh;
  const bool ties = ties_sh;
  const uint32_t t = thr_sh;
  const unsigned long long from = (unsigned long long)t << 32 | (ties ? 0xffffffffull : 0ull);   // ranks above it count
  // calls f(rank key) for the ids of those groups, four loads of a thread in flight
  auto scan = [&](auto f) {
    const int log_lg = 31 - __clz(lg), log_vecs = 31 - __clz(vecs), log_pieces = log_lg + log_vecs;
    const int pieces = wins << log_pieces;
    for (int i0 = tid; i0 < pieces; i0 += 4 * 256) {
      Vec<T> v[4];
      int x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = i0 + 256 * e;
        x[e] = V;
        if (i >= pieces) continue;
        const int g = win[i >> log_pieces], j = i & ((1 << log_pieces) - 1), u = j >> log_lg;
        x[e] = ((((g / per_part) << log_vecs) + u) * 64 + (g % per_part << log_lg) + (j & (lg - 1))) * kPer;
        if (x[e] + kPer <= V) v[e].load(row + x[e]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (x[e] + kPer <= V) {
#pragma unroll
          for (int q = 0; q < kPer; ++q) f(rank_key(x[e] + q, order_key(v[e].get(q))));
        } else {
#pragma unroll
          for (int q = 0; q < kPer; ++q)
            if (x[e] + q < V) f(rank_key(x[e] + q, order_key(Vec<T>::one(row + x[e] + q))));
        }
      }
    }
  };
  auto push = [&](unsigned long long c) {           // (the list's order does not matter: it is ranked below)
    const int at = atomicAdd(&n_sh, 1);
    if (at < kCap) cand[at] = c;
  };
  scan([&](unsigned long long c) {
    if (c > from) push(c);
  });
  __syncthreads();
  if (n_sh > kCap) {
    // More candidates than the list holds (long runs of the largest logits): the topk-th best by bisection,
    // 64 counts over the groups, which the caches hold by now.
    unsigned long long c0 = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long c = c0 | 1ull << bit;
      int cnt = 0;
      scan([&](unsigned long long x) { cnt += x >= c; });
#pragma unroll
      for (int s = 32; s > 0; s >>= 1) cnt += __shfl_xor(cnt, s, kWave);
      __syncthreads();
      if (lane == 0) cnt_sh[w] = cnt;
      __syncthreads();
      if (cnt_sh[0] + cnt_sh[1] + cnt_sh[2] + cnt_sh[3] >= topk) c0 = c;
    }
    __syncthreads();
    if (tid == 0) n_sh = 0;
    __syncthreads();
    scan([&](unsigned long long c) {
      if (c >= c0) push(c);
    });
    __syncthreads();
  }
  int n = n_sh;
  if (ties && n < topk) {
    // the lowest ids with logit t, in order: kPer neighbours a thread, its places behind those of the threads before it
    for (int x0 = 0; x0 < V && n < topk; x0 += 256 * kPer) {
      const int x = x0 + tid * kPer;
      int hits = 0;                        // bit q: id x + q
      if (x + kPer <= V) {
        Vec<T> v;
        v.load(row + x);
#pragma unroll
        for (int q = 0; q < kPer; ++q) hits |= int(order_key(v.get(q)) == t) << q;
      } else {
        for (int q = 0; q < kPer && x + q < V; ++q) hits |= int(order_key(Vec<T>::one(row + x + q)) == t) << q;
      }
      int before = __popc(hits);           // inclusive sum over the wave
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) {
        const int y = __shfl_up(before, s, kWave);
        if (lane >= s) before += y;
      }
      __syncthreads();
      if (lane == 63) cnt_sh[w] = before;
      __syncthreads();
      int at = n + before - __popc(hits);
      for (int i = 0; i < w; ++i) at += cnt_sh[i];
      for (; hits && at < topk; hits &= hits - 1) cand[at++] = rank_key(x + __ffs(hits) - 1, t);
      n = min(topk, n + cnt_sh[0] + cnt_sh[1] + cnt_sh[2] + cnt_sh[3]);
    }
    __syncthreads();
  }
  for (int i = tid; i < n; i += 256) {
    const unsigned long long me = cand[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += cand[j] > me;
    if (rank >= topk) continue;
    o.top_ids[r * topk + rank] = 0x7fffffff - (int)(uint32_t)me;
    o.top_logp[r * topk + rank] =
        st.s == 0.0 ? -INFINITY
                    : (float)(((double)key_value(uint32_t(me >> 32)) - (double)st.max) * inv_t - st.log_s);
  }
}

// ---------------------------------------------------------------- gradient
constexpr int kGradThreads = 256;
// Gradients of this size and more pass the caches by.  Measured with streaming / ordinary stores: 311 MB 120.5 / 126.2 us,
// 156 MB 60.5 / 64.4, 52 MB 21.5 / 17.0, 39 MB 15.3 / 12.9.
constexpr size_t kGradStreamBytes = size_t(128) << 20;
template <typename T> constexpr int kGradIds = 4 * kGradThreads * Vec<T>::kPer;    // four loads in flight per thread

template <typename T, bool NT>
__global__ __launch_bounds__(kGradThreads) void lp_grad_kernel(int M, int V, const T *logits, long ld, float scale,
                                                               float inv_t, const int32_t *__restrict__ ids,
                                                               const gm_token_stats *__restrict__ stats,
                                                               const float *__restrict__ ent,
                                                               const float *__restrict__ g_logp,
                                                               const float *__restrict__ g_ent, T *grad, long ldg) {
  constexpr int kPer = Vec<T>::kPer;
  const int lo = blockIdx.y * kGradIds<T> + threadIdx.x * kPer;
  for (long r = blockIdx.x; r < M; r += gridDim.x) {
    const T *row = logits + r * ld;
    T *out = grad + r * ldg;
    Vec<T> v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int x = lo + u * kGradThreads * kPer;
      if (x + kPer <= V) {
        if (NT) v[u].load_once(row + x);
        else v[u].load(row + x);
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[u].set(i, x + i < V ? Vec<T>::one(row + x + i) : 0.f);
      }
    }
    const gm_token_stats st = stats[r];
    int id = ids ? ids[r] : -1;
    if (id >= V) id = -1;
    const float g = id >= 0 ? g_logp[r] : 0.f, gh = g_ent ? g_ent[r] : 0.f;
    // grad = e (a + b y) with e = exp2(y), y = (z - max) / T log2 e
    float a = 0.f, b = 0.f;
    if (st.sum != 0.f) {
      const float k = -inv_t / st.sum;
      a = gh != 0.f ? k * (g + gh * (ent[r] - logf(st.sum))) : k * g;
      b = k * gh * (float)kLn2;
    }
    const float hot = st.sum != 0.f ? g * inv_t : 0.f;
    const float ref = st.max == -INFINITY ? 0.f : st.max;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int x = lo + u * kGradThreads * kPer;
      if (x >= V) break;
      Vec<T> o;
      float d[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const float y = (v[u].get(i) - ref) * scale;
        d[i] = __builtin_amdgcn_exp2f(y) * (a + b * fmaxf(y, kLowest));
        if (x + i == id) d[i] += hot;
      }
#pragma unroll
      for (int i = 0; i < kPer; i += 2) o.set2(i, d[i], d[i + 1]);
      if (x + kPer <= V) {
        o.template store<NT>(out + x);
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (x + i < V) Vec<T>::put(out + x + i, d[i]);
      }
    }
  }
}

// rows per launch dimension: a grid's dimension holds less than 2^32 threads
unsigned grid_rows(int M) { return (unsigned)(M < (1 << 20) ? M : (1 << 20)); }

// 16-byte loads per lane and stretch: as many as make 4096 ids (16 in float32, 8 in bf16) where there are 16384 such
// stretches (64 Mi logits) and more, else 4.  Measured with many / 4: 4096 x 151936 float32 378 / 404 us, bf16 238 / 243,
// 8192 x 32000 float32 206 / 217 (with four alternatives), 4096 x 32000 bf16 51 / 54, 1024 x 151936 float32 101 / 101;
// 1024 x 50257 40 / 36, 256 x 151936 32 / 29, 64 x 151936 17.9 / 15.4 (with eight).
constexpr int kLpWaves = 16384;
int lp_vecs(int M, int V, int per) {
  const int most = 64 / per;
  return (long)M * V / (64 * per * most) >= kLpWaves ? most : 4;
}
int lp_parts(int M, int V, int per) {
  const int ids = 64 * per * lp_vecs(M, V, per);
  return (V + ids - 1) / ids;
}
static_assert(kMaxVocab / (64 * 4 * 4) <= kLpMaxParts, "a wave joins a row's stretches");
// Lanes per group: as few as leave at most 1024 groups a row (a wave holds 2048): at least 64 groups, of at most
// 512 ids, so that the group maxima bound the 64th best logit.  Against 16 lanes throughout, 64 rows of 151936 bf16
// take 14.0 us (15.1), 16 float32 rows with 64 alternatives 25.8 (26.7); with at most 2048 groups a row 17.3 (bf16).
int lp_group_lanes(int parts) { return parts <= 16 ? 1 : parts <= 64 ? 4 : 16; }
static_assert(kLpMaxParts * 64 / 16 <= kLpMaxGroups && 128 * 64 / 16 <= kLpMaxGroups, "a wave holds a row's groups");

template <typename T>
void run_logprobs(int M, int V, const T *logits, long ld, double inv_t, int topk, const LpOut &o, char *ws,
                  hipStream_t s) {
  constexpr int kPer = Vec<T>::kPer;
  const int vecs = lp_vecs(M, V, kPer), parts = lp_parts(M, V, kPer), lg = lp_group_lanes(parts);
  Carve c;
  LpPart *part = (LpPart *)(ws + c.take(sizeof(LpPart) * (size_t)M * parts));
  float *groups = topk > 0 ? (float *)(ws + c.take(sizeof(float) * (size_t)M * parts * (64 / lg))) : nullptr;
  const float scale = (float)(inv_t / kLn2);
  {
    TraceScope ts("logprob_parts", s);
    const dim3 grid(grid_rows(M), (parts + 3) / 4);
    auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, M, V, parts, logits, ld, scale, part, groups);
    };
    constexpr int kMost = 64 / kPer;
    if (topk == 0) launch(vecs == kMost ? lp_part_kernel<T, kMost, 0> : lp_part_kernel<T, 4, 0>);
    else if (lg == 1) launch(vecs == kMost ? lp_part_kernel<T, kMost, 1> : lp_part_kernel<T, 4, 1>);
    else if (lg == 4) launch(vecs == kMost ? lp_part_kernel<T, kMost, 4> : lp_part_kernel<T, 4, 4>);
    else launch(vecs == kMost ? lp_part_kernel<T, kMost, 16> : lp_part_kernel<T, 4, 16>);
  }
  TraceScope ts(topk > 0 ? "logprob_top" : "logprob_rows", s);
  if (topk > 0)
    hipLaunchKernelGGL(lp_top_kernel<T>, dim3(M), dim3(256), 0, s, M, V, parts, vecs, lg, topk, logits, ld, scale,
                       inv_t, part, groups, o);
  else
    hipLaunchKernelGGL(lp_row_kernel<T>, dim3((unsigned)(((long)M + 3) / 4)), dim3(256), 0, s, M, V, parts, logits, ld,
                       scale, inv_t, part, o);
}
}  // namespace

size_t logprobs_workspace(int M, int V, int topk) {
  size_t most = 0;
  for (int per = 4; per <= 8; per *= 2) {      // float32 and bf16
    const size_t parts = (size_t)M * lp_parts(M, V, per);
    Carve c;
    c.take(sizeof(LpPart) * parts);
    if (topk > 0) c.take(sizeof(float) * parts * (64 / lp_group_lanes(lp_parts(M, V, per))));
    if (c.off > most) most = c.off;
  }
  return most;
}

void launch_token_logprobs(int M, int V, int dtype, const void *logits, long ld, float temperature, int topk,
                           const LpOut &o, char *ws, hipStream_t s) {
  const double inv_t = 1.0 / (double)temperature;
  if (dtype == GM_BF16) run_logprobs(M, V, (const bf16 *)logits, ld, inv_t, topk, o, ws, s);
  else run_logprobs(M, V, (const float *)logits, ld, inv_t, topk, o, ws, s);
}

void launch_token_logprobs_grad(int M, int V, int dtype, const void *logits, long ld, float temperature,
                                const int32_t *ids, const gm_token_stats *stats, const float *entropy,
                                const float *g_logp, const float *g_entropy, void *grad, long ld_grad, hipStream_t s) {
  TraceScope ts("logprob_grad", s);
  const double inv_t = 1.0 / (double)temperature;
  const float scale = (float)(inv_t / kLn2);
  auto launch = [&](auto kernel, auto *z, auto *g, int per_block) {
    hipLaunchKernelGGL(kernel, dim3(grid_rows(M), (V + per_block - 1) / per_block), dim3(kGradThreads), 0, s, M, V, z,
                       ld, scale, (float)inv_t, ids, stats, entropy, g_logp, g_entropy, g, ld_grad);
  };
  const bool nt = (size_t)M * V * (dtype == GM_BF16 ? 2 : 4) >= kGradStreamBytes;
  if (dtype == GM_BF16) launch(nt ? lp_grad_kernel<bf16, true> : lp_grad_kernel<bf16, false>, (const bf16 *)logits, (bf16 *)grad, kGradIds<bf16>);
  else launch(nt ? lp_grad_kernel<float, true> : lp_grad_kernel<float, false>, (const float *)logits, (float *)grad, kGradIds<float>);
}

}  // namespace gm
