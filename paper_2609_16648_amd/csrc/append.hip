// Append of new positions to the paged cache: per-head RMSNorm of q and k, the rotation, and
// the scatter of K and V into the pre-swizzled 16-token tiles (gm.h).
//
//   y = x / sqrt(mean(x^2) + eps) * w          (qk_norm)
//   (y_c, y_{c+d/2}) -> (y_c cos t - y_{c+d/2} sin t, y_{c+d/2} cos t + y_c sin t),
//   t = position * base^(-2c/d)
//
// Work: a unit is one 16-token tile of the cache that a sequence's new slots touch, so every
// K and V tile is written by one workgroup in whole 16-byte pieces: in V's layout four tokens of
// a channel are neighbours, and a lane that holds a quad of tokens and sixteen channels
// transposes them in registers.  (Sequences begin at any slot: units cut in slot space keep the
// quads whole where units of 16 rows would not.)  A workgroup takes the rotations of its 16
// tokens once, into LDS, for all heads; its four waves take the heads in turn, a wave 16 tokens
// of one q or k head, or of the 2 (head_dim 128) or 4 (64) v heads that fill its lanes.
// Bound by HBM: every row is read once and written once.  32.6K rows of 32 + 8 + 8 bf16 heads of 128 (802 MB) take
// 189 us, 4.2 TB/s, where a copy of 2 GiB reaches 4.9; V through LDS instead of the register transpose took 204.
//
// Precision: the angle in float64 as a fraction of a turn (positions reach 32K and beyond, where a
// float32 angle is off by 1e-3), its sine and cosine in float32; norm and rotation in float32,
// outputs rounded once to the model dtype.
#include "common.h"
#include "tree.h"

namespace gm {

namespace {
typedef unsigned short u16x8_t __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bfx2_t __attribute__((ext_vector_type(2)));
typedef float fx2_t __attribute__((ext_vector_type(2)));

// Eight consecutive elements (rows may start at any element: global loads of 16 bytes take any alignment)
template <typename T> struct Eight;
template <> struct Eight<bf16> {
  u16x8_t r;
  __device__ __forceinline__ void load(const bf16 *p) { r = *reinterpret_cast<const u16x8_t *>(p); }
  __device__ __forceinline__ void zero() { r = u16x8_t{0, 0, 0, 0, 0, 0, 0, 0}; }
  __device__ __forceinline__ float get(int i) const { return bf16_to_f32(r[i]); }
  static __device__ __forceinline__ void store(bf16 *p, const float (&f)[8]) {   // round to nearest even
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(fx2_t{f[2 * i], f[2 * i + 1]}, bfx2_t));
    *reinterpret_cast<u16x8_t *>(p) = __builtin_bit_cast(u16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
  }
};
template <> struct Eight<float> {
  f32x4u_t a, b;
  __device__ __forceinline__ void load(const float *p) {
    a = *reinterpret_cast<const f32x4u_t *>(p);
    b = *reinterpret_cast<const f32x4u_t *>(p + 4);
  }
  __device__ __forceinline__ void zero() { a = b = f32x4u_t{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ float get(int i) const { return i < 4 ? a[i] : b[i - 4]; }
  static __device__ __forceinline__ void store(float *p, const float (&f)[8]) {
    *reinterpret_cast<f32x4u_t *>(p) = f32x4u_t{f[0], f[1], f[2], f[3]};
    *reinterpret_cast<f32x4u_t *>(p + 4) = f32x4u_t{f[4], f[5], f[6], f[7]};
  }
};

// one V piece: channel x of the low eight and of the high eight, tokens 0..3 of each
__device__ __forceinline__ void store_quad(bf16 *p, const Eight<bf16> (&lo)[4], const Eight<bf16> (&hi)[4], int x) {
  *reinterpret_cast<uint4 *>(p) =
      make_uint4(lo[0].r[x] | (uint32_t(lo[1].r[x]) << 16), lo[2].r[x] | (uint32_t(lo[3].r[x]) << 16),
                 hi[0].r[x] | (uint32_t(hi[1].r[x]) << 16), hi[2].r[x] | (uint32_t(hi[3].r[x]) << 16));
}
__device__ __forceinline__ void store_quad(float *p, const Eight<float> (&lo)[4], const Eight<float> (&hi)[4], int x) {
  *reinterpret_cast<float4 *>(p) = make_float4(lo[0].get(x), lo[1].get(x), lo[2].get(x), lo[3].get(x));
  *reinterpret_cast<float4 *>(p + 4) = make_float4(hi[0].get(x), hi[1].get(x), hi[2].get(x), hi[3].get(x));
}
__device__ __forceinline__ void put(bf16 *p, const Eight<bf16> &e, int x) { p->bits = e.r[x]; }
__device__ __forceinline__ void put(float *p, const Eight<float> &e, int x) { *p = e.get(x); }

// Units of the sequences before b: floor(row_start[b] / 16) + 2 b.  n rows span at most
// floor((n + 14) / 16) + 1 <= floor(n / 16) + 2 tiles, and floor(x + n) - floor(x) >= floor(n):
// every sequence has the units it needs, with no sum over the batch; units past its tiles end at once.
__device__ __forceinline__ long units_before(long row, int b) { return (row >> 4) + 2L * b; }

template <typename T, int D>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  // q and k: kRowLanes lanes hold a row's low half and its high half, eight channels each: whole 128-byte lines per
  // load and store; kIters passes over the 16 tokens
  constexpr int kHalf = D / 2, kRowLanes = kHalf / 8, kIters = 16 * kRowLanes / 64;
  __shared__ __attribute__((aligned(16))) float2 rot[16][kHalf + 2];   // (cos, sin) of token s and pair c; rows four banks apart
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const long u = blockIdx.x;
  // the sequence of this unit: the last one with at most u units before it
  int b;
  if (a.row_start) {
    // 256 places at a time, each round within one step of the round before
    int lo = 0;
    for (int len = a.B, step = 0; step != 1; len = min(step, a.B - lo)) {
      step = (len + 255) / 256;
      const int i = tid * step;
      const int n = __syncthreads_count(i < len && units_before(a.row_start[lo + min(i, len - 1)], lo + i) <= u);
      if (n > 1) lo += (n - 1) * step;
    }
    b = lo;
  } else {
    const int R = a.T / a.B;
    b = (int)(16 * u / (R + 32));       // units_before is between b (R + 32) / 16 - 1 and b (R + 32) / 16
    if (b >= a.B) b = a.B - 1;
    if (b + 1 < a.B && units_before((long)(b + 1) * R, b + 1) <= u) ++b;
  }
  long r0, n;
  if (a.row_start) {
    r0 = a.row_start[b];
    n = a.row_start[b + 1] - r0;
  } else {
    n = a.T / a.B;
    r0 = b * n;
  }
  const int m = a.seq_lens[b];
  const long first = u - units_before(r0, b);           // this unit's tile among the sequence's new ones
  if (first < 0 || n <= 0) return;
  const long slot0 = (((long)m >> 4) + first) << 4;     // the tile's first slot
  if (slot0 >= m + n) return;
  auto row_of = [&](int s) -> long {                    // the row that goes to token s, or -1
    const long i = slot0 + s - m, r = r0 + i;
    return i >= 0 && i < n && r >= 0 && r < a.T ? r : -1;
  };
  // the tile's place
  long kv_base = -1;
  {
    const long pi = slot0 / a.page_size;
    const int page = slot0 >= 0 && pi < a.max_pages ? a.block_table[(long)b * a.max_pages + pi] : -1;
    if (page >= 0 && page < a.num_pages) kv_base = (long)page * a.n_kv * a.page_size * D + (slot0 % a.page_size) * D;
    else if (tid == 0 && blockIdx.y == 0) raise_dev_err(a.dev_err, GM_DEVERR_PAGE);
  }
  {
    // thread t holds pair t % kHalf throughout
    const int c = tid % kHalf;
    const double turns = exp2(-2.0 * c / D * a.log2_base) * 0.15915494309189535;   // per position, / 2 pi
    for (int s = tid / kHalf; s < 16; s += 256 / kHalf) {
      const long r = row_of(s);
      const long pos = r < 0 ? 0 : (a.offsets ? (long)m + a.offsets[r] : slot0 + s);
      const double x = (double)pos * turns;
      float sn, cs;
      sincospif(2.f * (float)(x - rint(x)), &sn, &cs);
      rot[s][c] = make_float2(cs, sn);
    }
  }
  __syncthreads();
  constexpr int kVLanes = D / 4, kVHeads = 64 / kVLanes;    // lanes of one v head, v heads per wave
  const int n_rot = a.n_heads + a.n_kv;
  const int tasks = n_rot + (a.n_kv + kVHeads - 1) / kVHeads;
  for (int task = blockIdx.y * 4 + w; task < tasks; task += gridDim.y * 4) {
    if (task < n_rot) {
      const bool is_q = task < a.n_heads;
      const int h = is_q ? task : task - a.n_heads;
      const T *const src = (const T *)(is_q ? a.q : a.k);
      const T *const nw = (const T *)(is_q ? a.q_norm : a.k_norm);
      const int j = lane % kRowLanes, c = 8 * j;
      Eight<T> lo[kIters], hi[kIters], wl, wh;
      long r[kIters];
#pragma unroll
      for (int i = 0; i < kIters; ++i) {
        r[i] = row_of(lane / kRowLanes + i * (64 / kRowLanes));
        lo[i].zero();
        hi[i].zero();
        if (r[i] >= 0) {
          const T *p = src + r[i] * (is_q ? a.q_stride : a.k_stride) + (long)h * D + c;
          lo[i].load(p);
          hi[i].load(p + kHalf);
        }
      }
      if (nw) {
        wl.load(nw + c);
        wh.load(nw + c + kHalf);
      }
#pragma unroll
      for (int i = 0; i < kIters; ++i) {
        const int s = lane / kRowLanes + i * (64 / kRowLanes);
        float inv = 1.f;
        if (nw) {
          float ss = 0.f;
#pragma unroll
          for (int x = 0; x < 8; ++x) ss += lo[i].get(x) * lo[i].get(x) + hi[i].get(x) * hi[i].get(x);
#pragma unroll
          for (int o = 1; o < kRowLanes; o <<= 1) ss += __shfl_xor(ss, o, kWave);
          inv = 1.0f / sqrtf(ss / (float)D + a.eps);
        }
        if (r[i] < 0 || (!is_q && kv_base < 0)) continue;
        float y1[8], y2[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          float p = lo[i].get(x), q = hi[i].get(x);
          if (nw) {
            p = p * inv * wl.get(x);
            q = q * inv * wh.get(x);
          }
          const float2 t = rot[s][c + x];
          y1[x] = p * t.x - q * t.y;
          y2[x] = q * t.x + p * t.y;
        }
        if (is_q) {
          T *o = (T *)a.q_out + (r[i] * a.n_heads + h) * D + c;
          Eight<T>::store(o, y1);
          Eight<T>::store(o + kHalf, y2);
        } else {
          T *o = (T *)a.k_pages + kv_base + (long)h * a.page_size * D;
          Eight<T>::store(o + k_tile_off(s, c), y1);
          Eight<T>::store(o + k_tile_off(s, c + kHalf), y2);
        }
      }
    } else {
      const int h = (task - n_rot) * kVHeads + lane / kVLanes, l = lane % kVLanes;
      const int quad = l / (D / 16), g = l % (D / 16);   // four tokens; eight channels and the eight 16 on
      const int c = (g >> 1) * 32 + (g & 1) * 8;
      if (h >= a.n_kv || kv_base < 0) continue;
      Eight<T> lo[4], hi[4];
      int live = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const long r = row_of(4 * quad + e);
        lo[e].zero();
        hi[e].zero();
        if (r >= 0) {
          const T *p = (const T *)a.v + r * a.v_stride + (long)h * D + c;
          lo[e].load(p);
          hi[e].load(p + 16);
          live |= 1 << e;
        }
      }
      T *const o = (T *)a.v_pages + kv_base + (long)h * a.page_size * D + v_tile_off(4 * quad, c);
      if (live == 15) {
#pragma unroll
        for (int x = 0; x < 8; ++x) store_quad(o + 8 * x, lo, hi, x);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (!(live >> e & 1)) continue;
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            put(o + 8 * x + e, lo[e], x);
            put(o + 8 * x + 4 + e, hi[e], x);
          }
        }
      }
    }
  }
}
}  // namespace

void launch_kv_append(const AppendArgs &a, hipStream_t s) {
  const long units = (a.T >> 4) + 2L * a.B;
  if (a.T <= 0 || a.B <= 0) return;
  TraceScope ts("kv_append", s);
  const int tasks = a.n_heads + a.n_kv + (a.n_kv * a.head_dim / 4 + 63) / 64;
  // Few units: their heads are dealt to more workgroups, until about 2048 of them (eight per CU).  Measured with 2048 /
  // 8192 / 16384, bf16, 32 q and 8 KV heads of 128: 32 prompts of 37 to 2001 rows 189 / 207 / 200 us, 256 trees of 4 nodes
  // 22 / 30 / 30, 64 trees of 16 nodes 14.6 / 14.8 / 14.3: more workgroups repeat the rotations and the table reads.
  int y = (int)((2048 + units - 1) / units);
  const int most = (tasks + 3) / 4;
  if (y > most) y = most;
  const dim3 grid((unsigned)units, y);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a); };
  if (a.dtype == GM_BF16) launch(kv_append_kernel<bf16, 128>);
  else if (a.head_dim == 64) launch(kv_append_kernel<float, 64>);
  else launch(kv_append_kernel<float, 128>);
}

}  // namespace gm
