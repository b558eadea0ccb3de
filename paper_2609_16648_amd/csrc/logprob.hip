// Log-probabilities of given tokens under softmax(z / T), with entropy and the most likely
// alternatives, and their gradient in the logits.
//
//   y_x = (z_x - max) / T,  S = sum exp(y),  W = sum exp(y) y  (both W <= 0 and log S >= 0)
//   log p_x = y_x - log S,  H = log S - W / S      (a difference of terms of opposite sign: no cancellation)
//   d/dz_x = ([x = id] g - p_x (g + gH (log p_x + H))) / T
// y is taken from the difference of the logits, not from z / T: it is exact near the maximum, and a
// mask of the type's lowest value stays finite.
//
// Forward: one pass over the logits.  A workgroup takes a chunk of 16384 ids of one row, all its
// loads in flight before the first exponential, and leaves (max, S, W) of the chunk, and, where
// alternatives are asked for, the maximum of every run of ids (lp_run); then one wave (or, with
// alternatives, one workgroup) per row joins the chunks.  The topk best ids, ordered by (logit
// descending, id ascending), lie in the topk best runs, ordered by (maximum descending, run
// ascending): the row's second kernel finds those among the run maxima and reads them again.
// Backward: one elementwise pass.  Both are bound by HBM.
#include "common.h"
#include "forward.h"

namespace gm {

namespace {
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;
constexpr float kLowest = -16384.f;    // exponents (of 2) below this are 0 already; finite, so that 0 * y is 0

typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short u16x8u_t __attribute__((ext_vector_type(8), aligned(2)));

// kPer consecutive logits in 16 bytes, at any element (global loads of 16 bytes take any alignment)
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int kPer = 4;
  f32x4u_t r;
  __device__ __forceinline__ void load(const float *p) { r = *reinterpret_cast<const f32x4u_t *>(p); }
  __device__ __forceinline__ float get(int i) const { return r[i]; }
  __device__ __forceinline__ void set(int i, float v) { r[i] = v; }
  template <bool NT> __device__ __forceinline__ void store(float *p) const {
    if (NT) __builtin_nontemporal_store(r, reinterpret_cast<f32x4u_t *>(p));
    else *reinterpret_cast<f32x4u_t *>(p) = r;
  }
  static __device__ __forceinline__ float one(const float *p) { return *p; }
  static __device__ __forceinline__ void put(float *p, float v) { *p = v; }
};
template <> struct Vec<bf16> {
  static constexpr int kPer = 8;
  u16x8u_t r;
  __device__ __forceinline__ void load(const bf16 *p) { r = *reinterpret_cast<const u16x8u_t *>(p); }
  __device__ __forceinline__ float get(int i) const { return bf16_to_f32(r[i]); }
  __device__ __forceinline__ void set(int i, float v) { r[i] = f32_to_bf16(v); }
  template <bool NT> __device__ __forceinline__ void store(bf16 *p) const {
    if (NT) __builtin_nontemporal_store(r, reinterpret_cast<u16x8u_t *>(p));
    else *reinterpret_cast<u16x8u_t *>(p) = r;
  }
  static __device__ __forceinline__ float one(const bf16 *p) { return bf16_to_f32(p->bits); }
  static __device__ __forceinline__ void put(bf16 *p, float v) { p->bits = f32_to_bf16(v); }
};

__device__ __forceinline__ uint32_t order_key(float x) {   // larger float, larger key (-0 as +0)
  uint32_t u = __float_as_uint(x);
  if (u == 0x80000000u) u = 0u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float block_max4(float v, float *sh) {   // 256 threads
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3]));
}

struct LpChunk {       // over one chunk of one row; S and W with exponents of 2
  float max, pad;
  double s, w;
};

// ---------------------------------------------------------------- forward
template <typename T, bool RUNS>
__global__ __launch_bounds__(256) void lp_chunk_kernel(int M, int V, int nch, int nruns, int run_len, const T *__restrict__ logits,
                                                       long ld, float scale, LpChunk *__restrict__ out,
                                                       float *__restrict__ runs) {
  constexpr int kPer = Vec<T>::kPer, kVecs = kLpChunk / (256 * kPer);
  __shared__ float sh_max[4];
  __shared__ double sh_s[16], sh_w[16];
  const int tid = threadIdx.x, lo = blockIdx.y * kLpChunk;
  for (long r = blockIdx.x; r < M; r += gridDim.x) {
    const T *row = logits + r * ld;
    Vec<T> v[kVecs];
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      const int x = lo + (u * 256 + tid) * kPer;
      if (x + kPer <= V) {
        v[u].load(row + x);
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[u].set(i, x + i < V ? Vec<T>::one(row + x + i) : -INFINITY);
      }
    }
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      float mv = v[u].get(0);
#pragma unroll
      for (int i = 1; i < kPer; ++i) mv = fmaxf(mv, v[u].get(i));
      m = fmaxf(m, mv);
      if (RUNS) {
        // run_len consecutive ids lie in run_len / kPer neighbouring lanes of one load
        float rm = mv;
        for (int o = 1; o < run_len / kPer; o <<= 1) rm = fmaxf(rm, __shfl_xor(rm, o, kWave));
        const int x = lo + (u * 256 + tid) * kPer;
        if (x % run_len == 0 && x < V) runs[r * nruns + x / run_len] = rm;
      }
    }
    m = block_max4(m, sh_max);
    // a chunk of -inf only: S and W are 0 (a NaN, which the maximum passes over, still reaches S)
    const float ref = m == -INFINITY ? 0.f : m;
    float s[2] = {0.f, 0.f}, w[2] = {0.f, 0.f};
#pragma unroll
    for (int u = 0; u < kVecs; ++u)
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const float y = (v[u].get(i) - ref) * scale;
        const float e = __builtin_amdgcn_exp2f(y);
        s[i & 1] += e;
        w[i & 1] += e * fmaxf(y, kLowest);
      }
    const double S = block_sum((double)s[0] + (double)s[1], sh_s), W = block_sum((double)w[0] + (double)w[1], sh_w);
    if (tid == 0) out[r * nch + blockIdx.y] = LpChunk{m, 0.f, S, W};
    __syncthreads();
  }
}

struct LpRow {
  float max;        // largest logit
  double s, log_s, ent;
};
// The row's statistics from its chunks, in every lane of the wave that asks (chunk order is fixed).
__device__ __forceinline__ LpRow lp_join(const LpChunk *__restrict__ ch, int nch, float scale) {
  const int lane = threadIdx.x & 63;
  const LpChunk c = lane < nch ? ch[lane] : LpChunk{-INFINITY, 0.f, 0.0, 0.0};
  LpRow r;
  r.max = wave_max(c.max);
  double s = 0.0, w = 0.0;
  if (c.s != 0.0) {                      // (also a NaN)
    const double y = c.max == -INFINITY ? 0.0 : ((double)c.max - (double)r.max) * (double)scale;
    const double f = exp2(y);
    s = c.s * f;
    w = f == 0.0 ? 0.0 : (c.w + c.s * y) * f;
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
__global__ __launch_bounds__(256) void lp_row_kernel(int M, int V, int nch, const T *__restrict__ logits, long ld,
                                                     float scale, double inv_t, const LpChunk *__restrict__ chunks,
                                                     LpOut o) {
  const long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= M) return;
  const LpRow st = lp_join(chunks + r * nch, nch, scale);
  if ((threadIdx.x & 63) == 0) lp_write(st, r, V, logits + r * ld, inv_t, o);
}

// Lane l of the wave holds keys of runs 64 i + l; keys of runs past nruns are 0 and not counted.
constexpr int kRunsPerLane = 32;
static_assert(kMaxVocab / 256 <= 64 * kRunsPerLane && 16384 / 32 <= 64 * kRunsPerLane, "a wave holds a row's runs");
// runs whose key is at least c
__device__ __forceinline__ int runs_from(const uint32_t (&key)[kRunsPerLane], int nruns, uint32_t c) {
  const int lane = threadIdx.x & 63;
  int cnt = 0;
#pragma unroll
  for (int i = 0; i < kRunsPerLane; ++i)
    if (64 * i < nruns) cnt += __popcll(__ballot(64 * i + lane < nruns && key[i] >= c));
  return cnt;
}

// One workgroup per row: statistics, then the alternatives.
template <typename T>
__global__ __launch_bounds__(256) void lp_top_kernel(int M, int V, int nch, int nruns, int run_len, int topk,
                                                     const T *__restrict__ logits, long ld, float scale, double inv_t,
                                                     const LpChunk *__restrict__ chunks,
                                                     const float *__restrict__ runs, LpOut o) {
  constexpr int kPer = Vec<T>::kPer, kCap = 1024;
  __shared__ int win[64];                  // the best runs, ascending in id
  __shared__ uint32_t thr_sh;
  __shared__ int n_sh, wins_sh, cnt_sh[4];
  __shared__ unsigned long long cand[kCap];
  __shared__ LpRow st_sh;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const long r = blockIdx.x;
  const T *row = logits + r * ld;
  if (w == 1) {
    const LpRow st = lp_join(chunks + r * nch, nch, scale);
    if (lane == 0) {
      st_sh = st;
      lp_write(st, r, V, row, inv_t, o);
    }
  }
  if (w == 0) {
    // the topk best runs: a lane holds runs 64 i + lane
    uint32_t key[kRunsPerLane];
#pragma unroll
    for (int i = 0; i < kRunsPerLane; ++i)
      key[i] = 64 * i + lane < nruns ? order_key(runs[r * nruns + 64 * i + lane]) : 0u;
    const int want = topk < nruns ? topk : nruns;
    uint32_t t = 0;                      // the largest t that at least `want` runs reach
    for (int bit = 31; bit >= 0; --bit)
      if (runs_from(key, nruns, t | 1u << bit) >= want) t |= 1u << bit;
    int eq_left = want - (t == 0xffffffffu ? 0 : runs_from(key, nruns, t + 1)), at = 0;
#pragma unroll
    for (int i = 0; i < kRunsPerLane; ++i) {        // runs in ascending order
      if (64 * i >= nruns) break;
      const bool in = 64 * i + lane < nruns, eq = in && key[i] == t;
      const unsigned long long me = __ballot(eq), below = (1ull << lane) - 1;
      const bool take = (in && key[i] > t) || (eq && __popcll(me & below) < eq_left);
      const unsigned long long mt = __ballot(take);
      if (take) win[at + __popcll(mt & below)] = 64 * i + lane;
      at += __popcll(mt);
      eq_left -= min(eq_left, __popcll(me));
    }
    if (lane == 0) {
      thr_sh = t;
      wins_sh = at;
      n_sh = 0;
    }
  }
  __syncthreads();
  if (st_sh.s != st_sh.s) {       // NaN or +inf in the row: no order that means anything
    if (tid < topk) {
      o.top_ids[r * topk + tid] = -1;
      o.top_logp[r * topk + tid] = (float)st_sh.s;
    }
    return;
  }
  // Ids of those runs whose logit reaches the last run's maximum: with topk runs there are at least topk of
  // them, and no other id is among the best (fewer runs than topk: every id counts).
  const int wins = wins_sh;
  const uint32_t t = wins < topk ? 0u : thr_sh;
  // calls f(id, key) for the ids of the best runs
  auto scan = [&](auto f) {
    const int vecs = run_len / kPer;
    for (int i = tid; i < wins * vecs; i += 256) {
      const int x = win[i / vecs] * run_len + i % vecs * kPer;
      if (x + kPer <= V) {
        Vec<T> v;
        v.load(row + x);
#pragma unroll
        for (int q = 0; q < kPer; ++q) f(x + q, order_key(v.get(q)));
      } else {
#pragma unroll
        for (int q = 0; q < kPer; ++q)
          if (x + q < V) f(x + q, order_key(Vec<T>::one(row + x + q)));
      }
    }
  };
  auto composite = [](int id, uint32_t key) { return (unsigned long long)key << 32 | (uint32_t)(0x7fffffff - id); };
  auto push = [&](int id, uint32_t key) {           // (the list's order does not matter: it is ranked below)
    const int at = atomicAdd(&n_sh, 1);
    if (at < kCap) cand[at] = composite(id, key);
  };
  scan([&](int id, uint32_t key) {
    if (key >= t) push(id, key);
  });
  __syncthreads();
  if (n_sh > kCap) {
    // More candidates than the list holds (long runs of equal or of the largest logits): the topk-th
    // best composite key by bisection, 64 counts over the runs, which the caches hold by now.
    unsigned long long c0 = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long c = c0 | 1ull << bit;
      int cnt = 0;
      scan([&](int id, uint32_t key) { cnt += composite(id, key) >= c; });
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
    scan([&](int id, uint32_t key) {
      if (composite(id, key) >= c0) push(id, key);
    });
    __syncthreads();
  }
  const int n = n_sh;
  const LpRow st = st_sh;
  for (int i = tid; i < n; i += 256) {
    const unsigned long long me = cand[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += cand[j] > me;
    if (rank >= topk) continue;
    const int id = 0x7fffffff - (int)(uint32_t)me;
    const double z = Vec<T>::one(row + id);
    o.top_ids[r * topk + rank] = id;
    o.top_logp[r * topk + rank] = st.s == 0.0 ? -INFINITY : (float)((z - (double)st.max) * inv_t - st.log_s);
  }
}

// ---------------------------------------------------------------- gradient
constexpr int kGradThreads = 256;
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
        v[u].load(row + x);
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
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const float y = (v[u].get(i) - ref) * scale;
        float d = __builtin_amdgcn_exp2f(y) * (a + b * fmaxf(y, kLowest));
        if (x + i == id) d += hot;
        o.set(i, d);
      }
      if (x + kPer <= V) {
        o.template store<NT>(out + x);
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (x + i < V) Vec<T>::put(out + x + i, o.get(i));
      }
    }
  }
}

// rows per launch dimension: a grid's dimension holds less than 2^32 threads
unsigned grid_rows(int M) { return (unsigned)(M < (1 << 20) ? M : (1 << 20)); }
}  // namespace

static_assert(kMaxVocab / kLpChunk <= 64, "a wave joins a row's chunks");

size_t logprobs_workspace(int M, int V, int topk) {
  Carve c;
  c.take(sizeof(LpChunk) * (size_t)M * lp_chunks(V));
  if (topk > 0) c.take(sizeof(float) * (size_t)M * lp_runs(V));
  return c.off;
}

template <typename T>
static void run_logprobs(int M, int V, const T *logits, long ld, double inv_t, int topk, const LpOut &o, char *ws,
                         hipStream_t s) {
  const int nch = lp_chunks(V), nruns = lp_runs(V);
  Carve c;
  LpChunk *chunks = (LpChunk *)(ws + c.take(sizeof(LpChunk) * (size_t)M * nch));
  float *runs = topk > 0 ? (float *)(ws + c.take(sizeof(float) * (size_t)M * nruns)) : nullptr;
  const float scale = (float)(inv_t / kLn2);
  {
    TraceScope ts("logprob_chunks", s);
    const dim3 grid(grid_rows(M), nch);
    if (topk > 0)
      hipLaunchKernelGGL((lp_chunk_kernel<T, true>), grid, dim3(256), 0, s, M, V, nch, nruns, lp_run(V), logits, ld, scale, chunks,
                         runs);
    else
      hipLaunchKernelGGL((lp_chunk_kernel<T, false>), grid, dim3(256), 0, s, M, V, nch, nruns, lp_run(V), logits, ld, scale,
                         chunks, runs);
  }
  TraceScope ts(topk > 0 ? "logprob_top" : "logprob_rows", s);
  if (topk > 0)
    hipLaunchKernelGGL(lp_top_kernel<T>, dim3(M), dim3(256), 0, s, M, V, nch, nruns, lp_run(V), topk, logits, ld, scale, inv_t,
                       chunks, runs, o);
  else
    hipLaunchKernelGGL(lp_row_kernel<T>, dim3((unsigned)(((long)M + 3) / 4)), dim3(256), 0, s, M, V, nch, logits, ld,
                       scale, inv_t, chunks, o);
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
  if (dtype == GM_BF16) launch(lp_grad_kernel<bf16, false>, (const bf16 *)logits, (bf16 *)grad, kGradIds<bf16>);
  else launch(lp_grad_kernel<float, false>, (const float *)logits, (float *)grad, kGradIds<float>);
}

}  // namespace gm
