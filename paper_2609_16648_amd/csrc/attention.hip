// Verify attention (Sec. 3.1, Eq. verification-context): the query at block
// position i of sequence b attends causally to cache positions 0 .. m_b + i.
// The kernels are in attention.h.
#include "attention.h"

namespace gm {

// Workgroups of `block` threads that one device holds at once (queried once per
// block size and device; a fixed guess when no device answers).  The LDS
// reservation makes this one per CU.
int attn_resident_groups(int block) {
  static std::atomic<int> cache[16][kAttnWavesPerGroup + 1];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 16) return 256;
  const int wv = block / 64;
  int v = cache[dev][wv].load();
  if (v > 0) return v;
  int per_cu = 0, cus = 0;
  const void *kernels[] = {(const void *)attn_mfma_kernel<true, 1, false>, (const void *)attn_mfma_kernel<true, 2, false>,
                           (const void *)attn_mfma_kernel<false, 2, false>};
  bool ok = true;
  for (const void *f : kernels)
    ok = ok && hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, kAttnLdsReserve) == hipSuccess;
  if (!ok || hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, attn_mfma_kernel<true, 2, false>, block, kAttnLdsReserve) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || per_cu < 1 || cus < 1) {
    (void)hipGetLastError();
    return 256;
  }
  v = per_cu * cus;
  cache[dev][wv].store(v);
  return v;
}

AttnPlan plan_attention(const gm_model_config &cfg, int B, int R) {
  AttnPlan p{};
  const int G = cfg.n_heads / cfg.n_kv_heads;
  const int rows = G * R;
  const int nt = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
  p.rows_pad = nt * 16;
  if (cfg.dtype != GM_BF16) return p;
  const AttnGeom g = attn_geom(cfg, p.rows_pad);
  long parts = attn_resident_groups(g.block) / g.groups;
  // One range per workgroup that the chip holds, however long: every further round of workgroups
  // fills its rings again, writes more partials, and the last one leaves CUs idle (256 sequences
  // of 512-8704 tokens: 840 us with one round, 898 us in 4.25 rounds of at most 4096 tokens;
  // 32 sequences of 16-32K tokens: 500 us with one round, 530 with two, 577 with four).
  if (parts < 1) parts = 1;
  p.parts = (int)parts;
  // the partial of (range p, sequence b) is in slot p + b
  Carve c;
  const size_t n = (size_t)(parts + B) * cfg.n_kv_heads * p.rows_pad;
  p.part_o = c.take(n * 128 * sizeof(float));
  p.part_ml = c.take(n * sizeof(float2));
  p.cum = c.take((size_t)(B + 1) * sizeof(int32_t));
  p.total = c.off;
  return p;
}

AttnArgs attn_args(const gm_model_config &cfg, const gm_kv_cache &c, int layer, int B, int R,
                   const int32_t *base_lens, int base_off, const int32_t *blk_len) {
  AttnArgs a{};
  a.dtype = cfg.dtype;
  a.B = B;
  a.R = R;
  a.n_heads = cfg.n_heads;
  a.n_kv = cfg.n_kv_heads;
  a.head_dim = cfg.head_dim;
  a.page_size = c.page_size;
  a.max_pages = c.max_pages_per_seq;
  a.num_pages = c.num_pages;
  a.k_pages = c.k_pages[layer];
  a.v_pages = c.v_pages[layer];
  a.block_table = c.block_table;
  a.base_lens = base_lens;
  a.base_off = base_off;
  a.blk_len = blk_len;
  a.blk_len_add = 0;
  a.scale = 1.0f / sqrtf((float)cfg.head_dim);
  a.trace = "attn";
  a.trace_combine = "attn_combine";
  return a;
}

void run_attention(const AttnArgs &a, const AttnPlan &p, char *ws, hipStream_t s) {
  if (a.B == 0) return;
  if (a.dtype != GM_BF16) {
    launch_attn_f32<false>(a, nullptr, s);
    return;
  }
  gm_model_config cfg{};
  cfg.n_kv_heads = a.n_kv;
  const AttnGeom geo = attn_geom(cfg, p.rows_pad);
  const AttnK k = attn_k(a, p, geo, ws);
  {
    TraceScope ts(a.trace, s);
    const dim3 grid(k.parts, geo.groups), block(geo.block);
    if (geo.rt_per_wave == 1)
      hipLaunchKernelGGL((attn_mfma_kernel<true, 1, false>), grid, block, kAttnLdsReserve, s, k);
    else if (geo.waves_per_head == 1)
      hipLaunchKernelGGL((attn_mfma_kernel<true, 2, false>), grid, block, kAttnLdsReserve, s, k);
    else
      hipLaunchKernelGGL((attn_mfma_kernel<false, 2, false>), grid, block, kAttnLdsReserve, s, k);
  }
  launch_attn_combine(k, a.trace_combine, s);
}

}  // namespace gm
