// Attention of draft trees over a paged cache: entry points.
#include "../../include/stand.h"

#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "attention.cuh"
#include "attention_plain.cuh"
#include "attention_tensor.cuh"
#include "launch.cuh"

using namespace stand;

namespace {

constexpr int64_t MOST_CHAIN = 65536;  // query rows per sequence without a mask

bool attention_valid(const stand_attention* c) {
  if (!c || c->B < 1 || c->N < 1 || c->N > MOST_CHAIN || c->heads_kv < 1 || c->heads_q < 1 || c->heads_q % c->heads_kv != 0) return false;
  if (c->dim < 1 || c->dim > ATTN_DIM_MAX || c->dtype < STAND_DTYPE_F32 || c->dtype > STAND_DTYPE_F16) return false;
  if (c->page_size < 16 || c->page_size > 4096 || c->page_size % 16 != 0 || c->pages < 0 || c->max_pages < 0) return false;
  if (!(c->scale > 0.0f && c->scale < INFINITY) || c->heads_q > 65535 || (long long)c->max_pages * c->page_size > (1ll << 30)) return false;
  if ((long long)c->N * (c->heads_q / c->heads_kv) >= (1ll << 20) || (long long)c->B * c->heads_kv > (1ll << 24)) return false;
  if ((c->own_v_stride != 0 && c->own_v_stride != 1) || c->reserved != 0) return false;
  for (int i = 0; i < 3; ++i)
    if (c->q_stride[i] < 0 || c->kv_stride[i] < 0 || c->cache_stride[i] < 0 || (c->own_v_stride && c->v_stride[i] < 0)) return false;
  return true;
}

}  // namespace

extern "C" {

size_t stand_tree_attention_scratch_bytes(const stand_attention* c) {
  if (!attention_valid(c)) return 0;
  const int group = c->heads_q / c->heads_kv;
  const size_t plain = ta_scratch_bytes(PA_ROWS, c->dim, plain_ctas(c->dim));
  if (c->dtype == STAND_DTYPE_F32 || group > TA_ROWS) return plain;
  const size_t tensor = ta_scratch_bytes(tensor_tile_rows(c->N, group), c->dim, tensor_ctas(c->dim));
  return tensor > plain ? tensor : plain;  // alignment decides, and that is not known here
}

int stand_tree_attention(const stand_attention* c, const void* dev_q, const void* dev_k, const void* dev_v, const void* dev_cache_k,
                         const void* dev_cache_v, const int32_t* dev_table, const int64_t* dev_len, const uint32_t* dev_mask,
                         int64_t mask_stride, const int32_t* dev_tree_tokens, void* dev_scratch, size_t scratch_bytes, void* dev_out,
                         float* dev_lse, void* cu_stream) {
  if (!attention_valid(c) || !dev_q || !dev_k || !dev_v || !dev_len || !dev_out) return STAND_E_ARG;
  if (c->max_pages > 0 && (!dev_table || !dev_cache_k || !dev_cache_v)) return STAND_E_ARG;
  if (!aligned(c->dtype == STAND_DTYPE_F32 ? 4 : 2, dev_q, dev_k, dev_v, dev_cache_k, dev_cache_v, dev_out) || !aligned(8, dev_len) ||
      !aligned(4, dev_table, dev_mask, dev_tree_tokens, dev_lse))
    return STAND_E_ARG;
  if (dev_mask && (c->N > STAND_MAX_NODES || mask_stride < 0)) return STAND_E_ARG;
  if (!dev_scratch || ((uintptr_t)dev_scratch & 255) != 0 || scratch_bytes < stand_tree_attention_scratch_bytes(c)) return STAND_E_WORKSPACE;
  AttnParams p;
  p.q = (const char*)dev_q; p.k = (const char*)dev_k; p.v = (const char*)dev_v;
  p.cache_k = (const char*)dev_cache_k; p.cache_v = (const char*)dev_cache_v; p.table = dev_table; p.len = (const long long*)dev_len;
  p.mask = dev_mask; p.mask_stride = mask_stride; p.tree = dev_tree_tokens; p.out = (char*)dev_out; p.lse = dev_lse;
  p.B = c->B; p.N = c->N; p.heads_q = c->heads_q; p.heads_kv = c->heads_kv; p.group = c->heads_q / c->heads_kv; p.dim = c->dim;
  p.page = c->page_size; p.pages = c->pages; p.cols = c->max_pages; p.mask_words = (c->N + 31) / 32;
  p.scale2 = (float)((double)c->scale * 1.4426950408889634);
  for (int i = 0; i < 3; ++i) {
    p.q_stride[i] = c->q_stride[i];
    p.k_stride[i] = c->kv_stride[i];
    p.v_stride[i] = c->own_v_stride ? c->v_stride[i] : c->kv_stride[i];
    p.cache_stride[i] = c->cache_stride[i];
  }
  cudaStream_t st = (cudaStream_t)cu_stream;
  int dev = -1, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return STAND_E_CUDA;
  if (tensor_takes(p, c->dtype)) {
    const int dp = tensor_dim(p.dim);
    const bool bf = c->dtype == STAND_DTYPE_BF16;
    const unsigned limit = wait_limit();
    int rc;
    if (dp == 64) rc = bf ? launch_tensor_parts<64, true>(p, dev_scratch, sms, limit, st) : launch_tensor_parts<64, false>(p, dev_scratch, sms, limit, st);
    else if (dp == 128) rc = bf ? launch_tensor_parts<128, true>(p, dev_scratch, sms, limit, st) : launch_tensor_parts<128, false>(p, dev_scratch, sms, limit, st);
    else rc = bf ? launch_tensor_parts<256, true>(p, dev_scratch, sms, limit, st) : launch_tensor_parts<256, false>(p, dev_scratch, sms, limit, st);
    if (rc != STAND_E_ARG) return rc;  // strides that the copy unit cannot take: the other kernel
  }
  if (c->dtype == STAND_DTYPE_F32) return launch_plain_attention<float>(p, dev_scratch, sms, st);
  if (c->dtype == STAND_DTYPE_BF16) return launch_plain_attention<__nv_bfloat16>(p, dev_scratch, sms, st);
  return launch_plain_attention<__half>(p, dev_scratch, sms, st);
}

int stand_tree_mask(const int32_t* host_parent, int32_t n, uint32_t* host_mask) {
  if (!host_parent || !host_mask || n < 1 || n > STAND_MAX_NODES || host_parent[0] != -1) return STAND_E_ARG;
  for (int u = 1; u < n; ++u)
    if (host_parent[u] < 0 || host_parent[u] >= u) return STAND_E_ARG;
  const int words = (n + 31) / 32;
  memset(host_mask, 0, (size_t)n * words * sizeof(uint32_t));
  for (int u = 0; u < n; ++u) {
    uint32_t* row = host_mask + (size_t)u * words;
    if (u > 0) memcpy(row, host_mask + (size_t)host_parent[u] * words, words * sizeof(uint32_t));
    row[u >> 5] |= 1u << (u & 31);
  }
  return STAND_OK;
}

}  // extern "C"
