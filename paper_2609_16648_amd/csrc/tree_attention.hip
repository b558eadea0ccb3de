// Attention of a draft tree's nodes over the cache: node i of sequence b attends to the committed positions and
// to the nodes of its mask (its ancestors and itself).  The rows of a KV head are its query heads times the
// nodes, (n_heads / n_kv_heads) * N, up to 4096.
//
// Up to 32 rows: the kernel of the verify attention (attention.h), whose waves stream K and V straight into
// operand registers, one wave per KV head; bound by HBM: 32 sequences of 16K to 32K tokens, 8 KV heads, 4 query heads
// each and 8 nodes take 512 us, 6.3 TB/s.  (The kernel below takes 517 there; 138 / 141 us at 64 sequences of 1K to 4K,
// 129 / 135 with 5 nodes.)
// More rows (tree_attn_kernel): the workgroup brings each KV tile into LDS once for all of its rows.
//    Up to 64 rows: four heads, a wave of 64 rows each.  Up to 128: two heads, and more: one, with eight waves of 32
//    rows, two per SIMD (further rows: further workgroups).
//  * S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16: a lane holds half of the tokens of one query,
//    so a row's maximum takes one exchange between lanes and P goes into the second product without one.
//  * K and V go from memory into LDS without passing registers, in stages of 32 tokens (a pair of tiles) of the
//    workgroup's heads, 128 KiB of them: 2, 4 or 8 stages.  A window of a range's tiles is listed once: a stage's places
//    in the pool, and whether it ends its sequence.
//    Four heads: each wave brings its own head's tiles, reads a stage's operands into registers at once
//    and gives its place to the stage after next; no wave waits for another.  Fewer heads: a barrier per two stages
//    says that they have arrived for all waves and that the two before have been read (a barrier for each: 306 us
//    where this takes 294).
//  * P is split into bf16 hi + lo parts, two products per V operand: the weights keep 16 bits.
//  * Work partition, partials and their combination are the verify attention's.
// 64 sequences of 1K to 4K tokens with 16 nodes (64 rows a head, 675 MB): 157 us with the combination, bound by HBM (4.3
// TB/s) and the 2 x 32 MB of partials.  32 sequences of 0.5K to 8.7K tokens with 64 nodes (256 rows a head): 294 us, 231
// GFLOP with the second part of P at 0.87 PFLOP/s, where a product of 8192^3 reaches 1.18 on this card.  Neither fewer
// vector instructions, nor whole-rate V reads, nor two groups of waves that take turns at the matrix unit and the weights
// changed that by more than 3%.
#include "attention.h"

namespace gm {

namespace {
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kTreeLds = 128 * 1024;      // bytes of the stages

// n KiB (4 or 2) from memory (uniform) into LDS (uniform), n x 16 bytes per lane, counted in vmcnt; off = 16 * lane.  In
// asm, so that the compiler does not put a wait for it before every LDS read (it cannot tell the stages apart): the
// kernel waits itself (wait_vm).  No register is written.  The instructions' offsets count on both sides.
template <int n> __device__ __forceinline__ void load_to_lds(uint32_t lds, const uint16_t *src, uint32_t off) {
  if (n == 4)
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %2, %1 nt\n\t"
        "global_load_lds_dwordx4 %2, %1 offset:1024 nt\n\t"
        "global_load_lds_dwordx4 %2, %1 offset:2048 nt\n\t"
        "global_load_lds_dwordx4 %2, %1 offset:%3 nt" ::"s"(lds), "s"(src), "v"(off), "n"(3 * 1024)
        : "memory", "m0");
  else
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %2, %1 nt\n\t"
        "global_load_lds_dwordx4 %2, %1 offset:1024 nt" ::"s"(lds), "s"(src), "v"(off)
        : "memory", "m0");
}
// until at most n vector memory operations of this wave are under way (older ones complete first)
template <int n> __device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory");
}

constexpr int tree_block(int HG) { return HG == 4 ? 256 : 512; }

// HG: heads per workgroup
template <int HG>
__global__ __launch_bounds__(tree_block(HG)) void tree_attn_kernel(AttnK a) {
  constexpr int kBlock = tree_block(HG), kWaves = kBlock / 64;
  constexpr int NT = HG == 4 ? 2 : 1;            // 32-row query tiles per wave
  constexpr int WPH = kWaves / HG;               // waves per head
  constexpr int kStage = HG * 16384, kRing = kTreeLds / kStage;
  constexpr int kLoads = kStage / 1024 / kWaves;   // loads per wave and stage
  constexpr bool kShared = HG < 4;               // the waves read each other's loads
  constexpr int kTurn = kShared ? 2 : 1;         // stages per barrier
  constexpr int kLater = kShared ? kRing - 2 * kTurn : 1;   // stages behind the awaited one that may be under way
  __shared__ int scan_sh[16];
  __shared__ int cum_sh[kBlock + 1], m0_sh[kBlock], bl_sh[kBlock];
  constexpr int kWin = kBlock;                   // tiles per window
  __shared__ int slot_sh[kWin];
  __shared__ int4 list_sh[kWin];                 // the window's stages (struct Stage)
  // per stage K tiles [HG][2], then V tiles [HG][2], as they lie in the pool
  extern __shared__ __attribute__((aligned(16))) uint8_t stage_sh[];

  const int tid = threadIdx.x, lane = tid & 63, j = lane & 31, g = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = blockIdx.x, kvh0 = blockIdx.y * HG, hw = w / WPH, kvh = kvh0 + hw;
  const int rows = a.G * a.R, row0 = ((int)blockIdx.z * WPH + w % WPH) * 32 * NT;
  const bool wave_ok = kvh < a.n_kv && row0 < rows;    // other waves only bring tiles
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)stage_sh;

  const bool one_chunk = a.B <= kBlock, writer = part == 0 && blockIdx.y == 0 && blockIdx.z == 0;
  int TT = 0, T1 = 0, cb1 = 0, m1 = 0, r1 = 0;
  if (one_chunk) {
    T1 = tid < a.B ? seq_tiles(a, tid, m1, r1) : 0;
    cb1 = block_excl_scan(T1, scan_sh, &TT);
    if (writer && tid < a.B) a.cum[tid] = cb1;
  } else {
    for (int c = 0; c < a.B; c += kBlock) {
      const int T = c + tid < a.B ? seq_tiles(a, c + tid, m1, r1) : 0;
      int tot;
      const int cb = TT + block_excl_scan(T, scan_sh, &tot);
      if (writer && c + tid < a.B) a.cum[c + tid] = cb;
      TT += tot;
    }
  }
  if (writer && tid == 0) a.cum[a.B] = TT;
  const int s = part_begin(part, TT, a.parts), e = part_begin(part + 1, TT, a.parts);
  if (s >= e) return;
  const int tpp = a.page_size >> 4;

  // this lane's queries: rows row0 + 32 t + j
  int qi[NT], qoff[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = row0 + 32 * t + j;
    qi[t] = r < rows && wave_ok ? r % a.R : -1;
    qoff[t] = qi[t] >= 0 ? (qi[t] * a.n_heads + kvh * a.G + r / a.R) * 128 : 0;
  }
  // the segment being computed (see attn_mfma_kernel)
  int b = -1, m0 = 0, L = 0, cb = 0, seq_end = 0;
  bool dead = false;
  uint32_t wild = 0;
  bf16x8_t qf[NT][8];
  unsigned long long anc[NT];
  bool node[NT];
  float m[NT], l[NT];
  f32x16_t O[NT][4];

  auto begin = [&](int c, int q) {
    b = c + q;
    m0 = __builtin_amdgcn_readfirstlane(m0_sh[q]);
    const int blen = __builtin_amdgcn_readfirstlane(bl_sh[q]);
    L = m0 + blen;
    cb = __builtin_amdgcn_readfirstlane(cum_sh[q]);
    seq_end = __builtin_amdgcn_readfirstlane(cum_sh[q + 1]);
    dead = false;
    wild = 0;
    const uint16_t *qb = a.q + (long)b * a.R * a.n_heads * 128;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      node[t] = qi[t] >= 0 && qi[t] < blen;
      anc[t] = node[t] ? a.masks[(long)b * a.R + qi[t]] : 0ull;
      if (blen < kMaxNodes) anc[t] &= (1ull << blen) - 1;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        qf[t][k] = as_bf16x8(qi[t] >= 0 ? *reinterpret_cast<const uint4 *>(qb + qoff[t] + 16 * k + 8 * g)
                                        : make_uint4(0, 0, 0, 0));
      m[t] = -INFINITY;
      l[t] = 0.f;
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[t][q4][i] = 0.f;
    }
  };
  auto finish = [&]() {
    const bool whole = cb >= s && seq_end <= e;
    if (wild) {
      // V that is inf or NaN stayed out of the products (0 * inf is NaN): added here, weight aside, for the rows
      // that see its token
#pragma unroll 1
      for (int tok = m0 & ~15; tok < L; ++tok) {
        const int tile = tok >> 4, d = tok - m0;
        if (!(wild >> (tile - m0 / 16) & 1)) continue;
        const int page = a.bt[(long)b * a.max_pages + tile / tpp];
        const uint16_t *v = a.vp + ((long)page * a.n_kv + kvh) * a.page_size * 128 + (long)(tile % tpp) * 2048;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float f = bf16_to_f32(v[v_tile_off(tok & 15, 32 * c + 8 * (i >> 2) + 4 * g + (i & 3))]);
            if (!(fabsf(f) < INFINITY)) {
#pragma unroll
              for (int t = 0; t < NT; ++t)
                if ((d < 0) | bool(anc[t] >> (d & 63) & 1)) O[t][c][i] += f;
            }
          }
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float lu = l[t] + __shfl_xor(l[t], 32, kWave);
      const int r = row0 + 32 * t + j;
      if (qi[t] < 0) continue;
      if (!whole) {
        const long prow = ((long)(part + b) * a.n_kv + kvh) * a.rows_pad + r;
        if (g == 0) a.part_ml[prow] = make_float2(m[t], lu);
        float *dst = a.part_o + prow * 128 + 4 * g;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<floatx4_t *>(dst + 32 * c + 8 * i) =
                floatx4_t{O[t][c][4 * i], O[t][c][4 * i + 1], O[t][c][4 * i + 2], O[t][c][4 * i + 3]};
      } else {
        const bool live = node[t] && m[t] != -INFINITY;
        const float inv = 1.f / lu;
        uint16_t *dst = a.out + (long)b * a.R * a.n_heads * 128 + qoff[t] + 4 * g;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float f[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) f[x] = live ? O[t][c][4 * i + x] * inv : 0.f;
            *reinterpret_cast<uint2 *>(dst + 32 * c + 8 * i) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
          }
      }
    }
  };

  bf16x8_t kf[8];         // K's operands of a stage
  auto read_k = [&](const uint8_t *st) {
    const uint8_t *kt = st + hw * 8192 + (j >> 4) * 4096 + g * 256 + (j & 15) * 16;
#pragma unroll
    for (int k = 0; k < 8; ++k) kf[k] = as_bf16x8(*reinterpret_cast<const uint4 *>(kt + k * 512));
  };
  // S[t][4 i + r]: the score of token 8 i + 4 g + r of the stage and query 32 t + j, unscaled
  auto scores = [&](f32x16_t (&S)[NT]) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) S[t][i] = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int t = 0; t < NT; ++t) S[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], qf[t][k], S[t], 0, 0, 0);
  };
  uint4 vf[2][4];         // V's: tokens 4 g .. + 3 and 8 + 4 g .. + 3 of tile k, channel 32 c + j
  auto read_v = [&](const uint8_t *st) {
    const uint8_t *vt = st + (HG + hw) * 8192 + g * 256 + (j & 15) * 16 + (j >> 4) * 8;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint8_t *p = vt + k * 4096 + c * 1024;
        const uint2 x = *reinterpret_cast<const uint2 *>(p), y = *reinterpret_cast<const uint2 *>(p + 512);
        vf[k][c] = make_uint4(x.x, x.y, y.x, y.y);
      }
  };
  // The masks of the tokens tb .. tb + 31, of which those below lim are there, and the rows' maxima brought up to date.
  auto settle = [&](f32x16_t (&S)[NT], int tb, int lim, bool mask) {
    if (mask) {
      // entries past the last node are nothing; nodes' values that are inf or NaN are kept for the end (finish)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bool nodes = tb + 16 * k + 16 > m0;
        bool mine = false;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t v[4] = {vf[k][c].x, vf[k][c].y, vf[k][c].z, vf[k][c].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int left = lim - (tb + 16 * k + 8 * (i >> 1) + 4 * g + 2 * (i & 1));
            v[i] = left <= 0 ? 0u : left == 1 ? v[i] & 0x0000ffffu : v[i];
            const uint32_t f = finite_or_0(v[i]);
            mine = mine | (f != v[i]);
            v[i] = nodes ? f : v[i];
          }
          vf[k][c] = make_uint4(v[0], v[1], v[2], v[3]);
        }
        if (nodes && __any(mine)) wild |= 1u << (tb / 16 + k - m0 / 16);
      }
    }
    float tmax[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (mask) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          // without branches: the tile's 32 tests are a few instructions each
          const int tok = tb + 8 * (i >> 2) + 4 * g + (i & 3), d = tok - m0;
          const bool seen = (tok < lim) & ((d < 0) | ((d < kMaxNodes) & bool(anc[t] >> (d & 63) & 1)));
          S[t][i] = seen ? S[t][i] : -INFINITY;
        }
      }
      // the larger of a pair as the median with infinity: fmaxf would first canonicalise every product's result
      float x0 = __builtin_amdgcn_fmed3f(S[t][0], S[t][1], INFINITY);
#pragma unroll
      for (int i = 2; i < 16; i += 2) x0 = fmaxf(x0, __builtin_amdgcn_fmed3f(S[t][i], S[t][i + 1], INFINITY));
      // (the other half of the wave holds the row's other tokens)
      const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x0), __float_as_uint(x0), false, false);
      tmax[t] = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * a.scale_log2;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const bool up = tmax[t] > m[t] + kLazyLog2;
      if (__any(up)) {
        const float mn = up ? fmaxf(m[t], tmax[t]) : m[t];
        const float alpha = (!up || mn == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f(m[t] - mn);
        l[t] *= alpha;
#pragma unroll
        for (int c = 0; c < 4; ++c) O[t][c] *= alpha;
        m[t] = mn;
      }
    }
  };
  // O += P V; the weights of query tile 1 are computed while the products of tile 0 run, six vector instructions
  // behind each
  auto weigh = [&](f32x16_t (&S)[NT]) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float ref = m[t] == -INFINITY ? 0.f : m[t];     // (a row that has seen nothing: every score is -inf)
      bf16x8_t hi[2], lo[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t h[4], q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(S[t][8 * k + 2 * i], a.scale_log2, -ref));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(S[t][8 * k + 2 * i + 1], a.scale_log2, -ref));
          l[t] += p0;
          l[t] += p1;
          h[i] = pack_bf16(p0, p1);
          q[i] = pack_bf16(p0 - __uint_as_float(h[i] << 16), p1 - __uint_as_float(h[i] & 0xffff0000u));
        }
        hi[k] = as_bf16x8(make_uint4(h[0], h[1], h[2], h[3]));
        lo[k] = as_bf16x8(make_uint4(q[0], q[1], q[2], q[3]));
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int c = 0; c < 4; ++c) O[t][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vf[k][c]), hi[k], O[t][c], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < 4; ++c) O[t][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vf[k][c]), lo[k], O[t][c], 0, 0, 0);
      }
    }
    if (NT > 1) __builtin_amdgcn_sched_group_barrier(0x402, 100, 0);
#pragma unroll
    for (int i = 0; i < 16 * (NT - 1); ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x402, 6, 0);
    }
  };

  // A stage: up to two neighbouring tiles of a sequence, in scalar registers.
  struct Stage {
    int slot0, slot1;       // places in the pool (a tile that is absent, or on a bad page: some other one's)
    int x;                  // first tile
    int seq, there;         // sequence in the chunk; tiles that are there, up to a bad page
    bool bad, last;         // a bad page; the segment's last stage
  };
  auto stage = [&](const int4 &v) {
    const int meta = __builtin_amdgcn_readfirstlane(v.z);
    return Stage{__builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y),
                 __builtin_amdgcn_readfirstlane(v.w), meta & 0xffff, meta >> 16 & 3, (meta >> 18 & 1) != 0,
                 (meta >> 19 & 1) != 0};
  };
  const uint32_t off = lane * 16;
  auto fetch = [&](const Stage &f, int p) {
    // this wave's units of 4 KiB: K and V, both tiles, of its own head (HG = 4); one unit (2); half a unit (1)
#pragma unroll
    for (int q = 0; q < (HG == 4 ? 4 : 1); ++q) {
      const int u = HG == 4 ? (q >> 1) * 8 + hw * 2 + (q & 1) : HG == 2 ? w : w >> 1;
      const int h = (u >> 1) % HG, kv = u / (2 * HG), head = min(kvh0 + h, a.n_kv - 1);
      const uint16_t *src = (kv ? a.vp : a.kp) + (long)head * a.page_size * 128 + (long)(f.slot0 + (u & 1) * (f.slot1 - f.slot0)) * 2048;
      const uint32_t dst = lds0 + p * kStage + u * 4096;
      if (HG > 1) load_to_lds<4>(dst, src, off);
      else load_to_lds<2>(dst + (w & 1) * 2048, src + (w & 1) * 1024, off);
    }
  };
  // until a stage has arrived, with `later` stages fetched behind it (the window's last ones arrive together)
  auto arrived = [&](int later) {
    if (later >= kLater) wait_vm<kLater * kLoads>();
    else wait_vm<0>();
  };

  int run = 0;
  for (int c = 0; c < a.B; c += kBlock) {
    int T, cbt, tot;
    if (one_chunk) {
      T = T1;
      cbt = cb1;
      tot = TT;
    } else {
      T = c + tid < a.B ? seq_tiles(a, c + tid, m1, r1) : 0;
      cbt = run + block_excl_scan(T, scan_sh, &tot);
    }
    const int cbeg = run, cend = run + tot;
    run = cend;
    if (cend <= s) continue;
    if (cbeg >= e) break;
    __syncthreads();
    cum_sh[tid] = cbt;
    if (tid == 0) cum_sh[kBlock] = cend;
    m0_sh[tid] = m1;
    bl_sh[tid] = r1;
    const int xe = min(e, cend);
    for (int x0 = max(s, cbeg); x0 < xe; x0 += kWin) {
      const int nt = min(kWin, xe - x0);
      __syncthreads();
      int seq = 0;
      if (const int i = tid; i < nt) {              // a thread per tile
        int lo = 0, hi = min(kBlock, a.B - c);
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (cum_sh[mid] <= x0 + i) lo = mid;
          else hi = mid;
        }
        const int t = x0 + i - cum_sh[lo], pi = t / tpp;
        const int page = pi < a.max_pages ? a.bt[(long)(c + lo) * a.max_pages + pi] : -1;
        const bool ok = page >= 0 && page < a.num_pages;
        if (!ok) raise_dev_err(a.dev_err, GM_DEVERR_PAGE);
        seq = lo;
        slot_sh[i] = ok ? page * a.n_kv * tpp + t % tpp : -1;
      }
      // the stages: pairs of tiles counted from where the sequence begins in this window
      const int x = x0 + tid;
      const bool first = tid < nt && ((x - max(cum_sh[seq], x0)) & 1) == 0;
      int stages;
      const int at = block_excl_scan(first, scan_sh, &stages);      // (its barriers also order slot_sh)
      if (first) {
        const int end = min(cum_sh[seq + 1], x0 + nt), n = min(2, end - x);
        const int s0 = slot_sh[tid], s1 = n > 1 ? slot_sh[tid + 1] : s0;
        const int there = s0 < 0 ? 0 : s1 < 0 ? 1 : n;
        const bool last = x + n == min(e, cum_sh[seq + 1]);
        list_sh[at] = make_int4(max(s0, 0), max(s1, 0), seq | there << 16 | (there < n) << 18 | last << 19, x);
      }
      __syncthreads();
      // Stage f lies in place f % kRing.  `next` is the next one to fetch: kFetch of them before the first is computed,
      // then one per stage.
      constexpr int kFetch = kShared ? kRing - kTurn : 2;
      int next = min(kFetch, stages);
      for (int f = 0; f < next; ++f) fetch(stage(list_sh[f]), f);
      Stage cur = stage(list_sh[0]), ahead = stage(list_sh[min(next, stages - 1)]);
      auto fetch_next = [&]() {
        if (next < stages) fetch(ahead, next++ % kRing);
      };
      // (waves without rows compute along: what they hold is written nowhere)
      for (int k = 0; k < stages; ++k) {
        const int4 cur_v = list_sh[min(k + 1, stages - 1)];
        int4 ahead_v;
        const uint8_t *const st = stage_sh + k % kRing * kStage;
        if (kShared) {
          if (k % kTurn == 0) {
            arrived(next - 1 - min(k + kTurn - 1, stages - 1));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int f = 0; f < kTurn; ++f)
              if (next < stages) {
                fetch(stage(list_sh[next]), next % kRing);
                ++next;
              }
          }
        } else {
          arrived(next - 1 - k);
          ahead_v = list_sh[min(k + kFetch + 1, stages - 1)];
        }
        if (b != c + cur.seq) begin(c, cur.seq);
        read_k(st);
        __builtin_amdgcn_sched_barrier(0);
        f32x16_t S[NT];
        scores(S);
        read_v(st);
        __builtin_amdgcn_sched_barrier(0);
        if (!kShared) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          fetch_next();
        }
        const int there = dead ? 0 : cur.there;
        dead = dead || cur.bad;
        const int tb = 16 * (cur.x - cb);
        const bool last = cur.last;
        settle(S, tb, min(L, tb + 16 * there), there < 2 || tb + 32 > m0);
        cur = stage(cur_v);
        if (!kShared) ahead = stage(ahead_v);
        weigh(S);
        if (last && wave_ok) finish();
      }
      wait_vm<0>();
    }
  }
}

// Up to 32 rows of a KV head go to attn_mfma_kernel, more to tree_attn_kernel with as many heads per workgroup as give a
// head's rows waves of their own.  Measured (us, combination included; 64 sequences of 1K to 4K tokens with 8 KV heads):
// 48 and 64 rows with four heads 157 and 162, two 198 and 199; 96 and 128 rows with two 203 and 215, one 286 and 303,
// four and a workgroup per 64 rows 237 and 237; 256 rows (32 sequences of 0.5K to 8.7K) with one 304, four 350.  One
// sequence of 4001 tokens and 64 rows alone is faster with two heads (24 against 30).
struct TreeGeom {
  bool wide;
  int heads_per_group, groups, row_groups, rows_pad, block, rt;
};
TreeGeom tree_geom(int rows, int n_kv) {
  TreeGeom g;
  g.wide = rows > 32;
  g.rt = rows <= 16 ? 1 : 2;
  g.heads_per_group = !g.wide || rows <= 64 ? 4 : rows <= 128 ? 2 : 1;
  g.row_groups = g.wide ? (rows + 255) / 256 : 1;
  g.rows_pad = g.wide ? (rows + 63) / 64 * 64 : g.rt * 16;
  if (!g.wide && g.heads_per_group > n_kv) g.heads_per_group = n_kv;
  g.groups = (n_kv + g.heads_per_group - 1) / g.heads_per_group;
  g.block = g.wide ? 256 : 64 * g.heads_per_group;
  return g;
}

// kernels that reserve more LDS than a launch may by itself say so once per device
template <typename F>
void reserve(F *kernel, int bytes, std::atomic<uint32_t> &ready) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) dev = 31;
  if (dev < 31 && (ready.load() >> dev & 1)) return;
  (void)hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (dev < 31) ready.fetch_or(1u << dev);
}
template <int RT>
void launch_narrow(const AttnK &k, const TreeGeom &g, hipStream_t s) {
  static std::atomic<uint32_t> ready{0};
  reserve(attn_mfma_kernel<true, RT, true>, kAttnLdsReserve, ready);
  hipLaunchKernelGGL((attn_mfma_kernel<true, RT, true>), dim3(k.parts, g.groups), dim3(g.block), kAttnLdsReserve, s, k);
}
template <int HG>
void launch_wide(const AttnK &k, const TreeGeom &g, hipStream_t s) {
  static std::atomic<uint32_t> ready{0};
  reserve(tree_attn_kernel<HG>, kTreeLds, ready);
  hipLaunchKernelGGL(tree_attn_kernel<HG>, dim3(k.parts, g.groups, g.row_groups), dim3(tree_block(HG)), kTreeLds, s,
                     k);
}
}  // namespace

AttnPlan plan_tree_attention(const gm_model_config &cfg, int B, int N) {
  AttnPlan p{};
  if (cfg.dtype != GM_BF16) return p;
  const TreeGeom g = tree_geom(cfg.n_heads / cfg.n_kv_heads * N, cfg.n_kv_heads);
  p.rows_pad = g.rows_pad;
  const int parts = attn_resident_groups(g.block) / (g.groups * g.row_groups);
  p.parts = parts < 1 ? 1 : parts;
  Carve c;     // the partial of (range p, sequence b) is in slot p + b
  const size_t n = (size_t)(p.parts + B) * cfg.n_kv_heads * p.rows_pad;
  p.part_o = c.take(n * 128 * sizeof(float));
  p.part_ml = c.take(n * sizeof(float2));
  p.cum = c.take((size_t)(B + 1) * sizeof(int32_t));
  p.total = c.off;
  return p;
}

void run_tree_attention(const AttnArgs &a, const uint64_t *masks, const AttnPlan &p, char *ws, hipStream_t s) {
  if (a.B == 0) return;
  if (a.dtype != GM_BF16) {
    launch_attn_f32<true>(a, masks, s);
    return;
  }
  const TreeGeom g = tree_geom(a.n_heads / a.n_kv * a.R, a.n_kv);
  AttnGeom geo{};
  geo.heads_per_group = g.heads_per_group;
  geo.waves_per_head = 1;
  AttnK k = attn_k(a, p, geo, ws);
  k.masks = (const unsigned long long *)masks;
  {
    TraceScope ts(a.trace, s);
    if (g.wide && g.heads_per_group == 4) launch_wide<4>(k, g, s);
    else if (g.wide && g.heads_per_group == 2) launch_wide<2>(k, g, s);
    else if (g.wide) launch_wide<1>(k, g, s);
    else if (g.rt == 1) launch_narrow<1>(k, g, s);
    else launch_narrow<2>(k, g, s);
  }
  launch_attn_combine(k, a.trace_combine, s);
}

}  // namespace gm
