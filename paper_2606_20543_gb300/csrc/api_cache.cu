// api_cache.cu — the extern "C" entry points of the paged 8-bit cache and the
// sampler (include/ssd.h): host-side argument checks and launches on the
// caller's stream.  No allocation, no synchronisation.
#include <math.h>

#include "kernels.cuh"

using namespace ssd;

namespace {

ssd_status from_cuda(cudaError_t e) { return e == cudaSuccess ? SSD_OK : SSD_ERR_CUDA; }

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

ssd_status check_grid(const ssd_grid* g) {
  if (g == nullptr) return SSD_ERR_INVALID_ARG;
  if (g->grid_h <= 0 || g->grid_w <= 0 || g->prefix_len < 0) return SSD_ERR_SHAPE;
  if (g->row_stride != g->grid_w && g->row_stride != g->grid_w + 1) return SSD_ERR_SHAPE;
  if ((int64_t)g->grid_h * g->row_stride + g->prefix_len > INT32_MAX / 2) return SSD_ERR_SHAPE;
  return SSD_OK;
}

bool block_ok(int32_t block) { return block == 16 || block == 32 || block == 64 || block == 128; }

int32_t log2_of(int32_t x) {
  int32_t n = 0;
  while ((1 << n) < x) ++n;
  return n;
}

ssd_status check_cache(const ssd_block_cache* c) {
  if (c == nullptr) return SSD_ERR_INVALID_ARG;
  if (c->num_blocks <= 0 || c->block <= 0 || c->Hkv <= 0 || c->d <= 0) return SSD_ERR_SHAPE;
  if (!block_ok(c->block) || (c->d != 64 && c->d != 128)) return SSD_ERR_UNSUPPORTED;
  if ((int64_t)c->num_blocks * c->Hkv > INT32_MAX / c->block) return SSD_ERR_UNSUPPORTED;
  if (c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr)
    return SSD_ERR_INVALID_ARG;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))
    return SSD_ERR_INVALID_ARG;
  return SSD_OK;
}

}  // namespace

extern "C" {

ssd_status ssd_cache_plan(const ssd_grid* grid, int32_t B, int32_t block, int32_t max_blocks,
                          int32_t N_max, const int32_t* cache_len, const int32_t* n_new,
                          const int32_t* held, const int32_t* ring, int32_t ring_size,
                          const int64_t* head, const int64_t* tail, int64_t* next_head,
                          int32_t* block_table, int32_t* n_blocks, int64_t* slots, int32_t* pos,
                          int32_t* status, ssd_stream_t stream) {
  if (pos != nullptr) {
    const ssd_status s = check_grid(grid);
    if (s != SSD_OK) return s;
  }
  if (B < 0 || max_blocks <= 0 || N_max <= 0 || ring_size <= 0 || block <= 0) return SSD_ERR_SHAPE;
  if (!block_ok(block) || max_blocks > INT32_MAX / 2 / block || N_max > INT32_MAX / 4)
    return SSD_ERR_UNSUPPORTED;
  if (B == 0) return SSD_OK;
  for (const void* p : {(const void*)cache_len, (const void*)n_new, (const void*)held,
                        (const void*)ring, (const void*)head, (const void*)tail,
                        (const void*)next_head, (const void*)block_table, (const void*)n_blocks,
                        (const void*)slots, (const void*)status})
    if (p == nullptr) return SSD_ERR_INVALID_ARG;
  if (!aligned(head, 8) || !aligned(tail, 8) || !aligned(next_head, 8) || !aligned(slots, 8))
    return SSD_ERR_INVALID_ARG;
  // every block reads head, and held while another writes n_blocks
  if (next_head == head || next_head == tail || n_blocks == held) return SSD_ERR_INVALID_ARG;
  CachePlanArgs a{};
  if (pos != nullptr) a.grid = *grid;
  a.B = B;
  a.block_log = log2_of(block);
  a.max_blocks = max_blocks;
  a.N_max = N_max;
  a.cache_len = cache_len;
  a.n_new = n_new;
  a.held = held;
  a.ring = ring;
  a.ring_size = ring_size;
  a.head = head;
  a.tail = tail;
  a.next_head = next_head;
  a.block_table = block_table;
  a.n_blocks = n_blocks;
  a.slots = slots;
  a.pos = pos;
  a.status = status;
  return from_cuda(launch_cache_plan(a, (cudaStream_t)stream));
}

ssd_status ssd_rotary_table(int32_t n_pos, int32_t pairs, const float* freq, float* table,
                            ssd_stream_t stream) {
  if (n_pos <= 0 || pairs <= 0) return SSD_ERR_SHAPE;
  if ((int64_t)n_pos * pairs > INT32_MAX) return SSD_ERR_UNSUPPORTED;
  if (freq == nullptr || table == nullptr || !aligned(table, 8)) return SSD_ERR_INVALID_ARG;
  return from_cuda(launch_rotary_table(n_pos, pairs, freq, table, (cudaStream_t)stream));
}

ssd_status ssd_cache_append(const ssd_block_cache* cache, const ssd_rotary* rotary, int32_t B,
                            int32_t N_max, int32_t Hq, const int32_t* n_new, const int64_t* slots,
                            const int32_t* pos, const void* q, int64_t ldq, const void* k,
                            int64_t ldk, const void* v, int64_t ldv, void* q_out, int32_t* status,
                            ssd_stream_t stream) {
  ssd_status s = check_cache(cache);
  if (s != SSD_OK) return s;
  if (rotary == nullptr) return SSD_ERR_INVALID_ARG;
  if (B < 0 || N_max <= 0 || Hq <= 0) return SSD_ERR_SHAPE;
  const int32_t d = cache->d, Hkv = cache->Hkv;
  if (Hq % Hkv != 0 || rotary->n_pos <= 0) return SSD_ERR_SHAPE;
  int64_t pairs = 0;
  for (int i = 0; i < 3; ++i) {
    if (rotary->sec[i] < 0) return SSD_ERR_SHAPE;
    pairs += rotary->sec[i];
  }
  if (pairs != d / 2) return SSD_ERR_SHAPE;
  if (ldq < (int64_t)Hq * d || ldk < (int64_t)Hkv * d || ldv < (int64_t)Hkv * d) return SSD_ERR_SHAPE;
  if (ldq % 8 != 0 || ldk % 8 != 0 || ldv % 8 != 0) return SSD_ERR_SHAPE;
  if ((int64_t)Hq * d > INT32_MAX / 2 || (int64_t)B * N_max > INT32_MAX / Hq)
    return SSD_ERR_UNSUPPORTED;
  if (B == 0) return SSD_OK;
  for (const void* p : {(const void*)n_new, (const void*)slots, (const void*)pos, q, k, v,
                        (const void*)q_out, (const void*)rotary->table, (const void*)status})
    if (p == nullptr) return SSD_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, (const void*)q_out})
    if (!aligned(p, 16)) return SSD_ERR_INVALID_ARG;
  if (!aligned(slots, 8) || !aligned(rotary->table, 8)) return SSD_ERR_INVALID_ARG;
  if (q_out == q && ldq != (int64_t)Hq * d) return SSD_ERR_INVALID_ARG;
  CacheAppendArgs a{};
  a.cache = *cache;
  a.rot = *rotary;
  a.B = B;
  a.N_max = N_max;
  a.Hq = Hq;
  a.n_new = n_new;
  a.slots = slots;
  a.pos = pos;
  a.q = q;
  a.k = k;
  a.v = v;
  a.ldq = ldq;
  a.ldk = ldk;
  a.ldv = ldv;
  a.q_out = q_out;
  a.status = status;
  return from_cuda(launch_cache_append(a, (cudaStream_t)stream));
}

size_t ssd_cache_attention_workspace(int32_t B, int32_t Hq, int32_t Hkv, int32_t d, int32_t D_max,
                                     int32_t L_max) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || d <= 0 || D_max <= 0 || L_max <= 0) return 0;
  return cache_attention_workspace(B, Hq, Hkv, d, D_max, L_max);
}

ssd_status ssd_cache_attention(const ssd_grid* grid, const ssd_block_cache* cache, int32_t B,
                               int32_t Hq, const int32_t* cache_len, const int32_t* n_drafts,
                               const int32_t* draft_pos, const int32_t* key_start, int32_t D_max,
                               const int32_t* block_table, int32_t max_blocks, const void* q,
                               float scale, void* o, float* lse, void* workspace,
                               size_t workspace_bytes, int32_t* status, ssd_stream_t stream) {
  ssd_status s = check_grid(grid);
  if (s != SSD_OK) return s;
  s = check_cache(cache);
  if (s != SSD_OK) return s;
  if (B < 0 || Hq <= 0 || D_max <= 0 || max_blocks <= 0) return SSD_ERR_SHAPE;
  if (Hq % cache->Hkv != 0) return SSD_ERR_SHAPE;
  if (max_blocks > INT32_MAX / 2 / cache->block) return SSD_ERR_UNSUPPORTED;
  if ((int64_t)B * cache->Hkv > 65535) return SSD_ERR_UNSUPPORTED;
  if ((int64_t)D_max * (Hq / cache->Hkv) > 65535 * 16) return SSD_ERR_UNSUPPORTED;
  if ((int64_t)B * D_max * Hq > INT32_MAX / 2) return SSD_ERR_UNSUPPORTED;
  if (B == 0) return SSD_OK;
  for (const void* p : {(const void*)cache_len, (const void*)n_drafts, (const void*)block_table, q,
                        (const void*)o, (const void*)status})
    if (p == nullptr) return SSD_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(o, 16)) return SSD_ERR_INVALID_ARG;
  if (!(scale >= 0.f) || !isfinite(scale)) return SSD_ERR_INVALID_ARG;
  const size_t need = cache_attention_workspace(B, Hq, cache->Hkv, cache->d, D_max,
                                                max_blocks * cache->block);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return SSD_ERR_WORKSPACE;
  if (need > 0 && !aligned(workspace, 16)) return SSD_ERR_INVALID_ARG;
  CacheAttnArgs a{};
  a.grid = *grid;
  a.cache = *cache;
  a.B = B;
  a.Hq = Hq;
  a.D_max = D_max;
  a.max_blocks = max_blocks;
  a.cache_len = cache_len;
  a.n_drafts = n_drafts;
  a.draft_pos = draft_pos;
  a.key_start = key_start;
  a.block_table = block_table;
  a.q = q;
  a.scale = scale;
  a.o = o;
  a.lse = lse;
  a.status = status;
  return from_cuda(launch_cache_attention(a, workspace, (cudaStream_t)stream));
}

ssd_status ssd_sample(int32_t rows, int32_t V, const void* logits, int32_t logits_bf16, int64_t ld,
                      const ssd_sampling* sampling, const ssd_rng* rng, int32_t* out_tok,
                      float* prob, int32_t* kept, int32_t* status, ssd_stream_t stream) {
  if (rows < 0 || V <= 0 || ld < V) return SSD_ERR_SHAPE;
  if (sampling == nullptr || rng == nullptr) return SSD_ERR_INVALID_ARG;
  if (logits_bf16 != 0 && logits_bf16 != 1) return SSD_ERR_INVALID_ARG;
  if (V > kSampleMaxV) return SSD_ERR_UNSUPPORTED;
  if (sampling->temperatures == nullptr &&
      (!(sampling->temperature >= 0.f) || !isfinite(sampling->temperature)))
    return SSD_ERR_INVALID_ARG;
  if (sampling->top_ps == nullptr && !(sampling->top_p > 0.f && sampling->top_p <= 1.f))
    return SSD_ERR_INVALID_ARG;
  if (sampling->min_ps == nullptr && !(sampling->min_p >= 0.f && sampling->min_p <= 1.f))
    return SSD_ERR_INVALID_ARG;
  if (sampling->top_ks == nullptr && sampling->top_k < 0) return SSD_ERR_INVALID_ARG;
  if (sampling->n_drafts != nullptr && sampling->D_max <= 0) return SSD_ERR_SHAPE;
  if (rows == 0) return SSD_OK;
  if (logits == nullptr || out_tok == nullptr || status == nullptr) return SSD_ERR_INVALID_ARG;
  if (!aligned(logits, logits_bf16 ? 2 : 4)) return SSD_ERR_INVALID_ARG;
  if (rng->uniforms != nullptr && !aligned(rng->uniforms, 8)) return SSD_ERR_INVALID_ARG;
  SampleArgs a{};
  a.rows = rows;
  a.V = V;
  a.logits = logits;
  a.bf16 = logits_bf16;
  a.ld = ld;
  a.s = *sampling;
  a.rng = *rng;
  a.out_tok = out_tok;
  a.prob = prob;
  a.kept = kept;
  a.status = status;
  return from_cuda(launch_sample(a, (cudaStream_t)stream));
}

}  // extern "C"
