// What the calls around a decode step share: rows, rotary positions, the 8-bit cache and their checks.
#pragma once
#include <algorithm>
#include <cmath>

#include "locks_internal.cuh"

#define KVQ_SLOT_BOUND 592       // upper bound on the CTAs of the token attention kernel (148 SMs x 4)
#define KVQ_ROWS 16              // query rows of a problem at most
#define KVQ_CHUNK_SLOTS 148      // CTAs of the chunk attention kernel at most where it splits the tokens
#define KVQ_CHUNK_ROWS 256       // query rows of one of them
#define KVQ_TINY_BITS 0x0D800000u   // 2^-100: a page whose largest magnitude is below it is stored as zeros

struct KvqCache {   // the 8-bit cache as the kernels take it
  char *k, *v;
  int64_t sb, sh, st;
  float *ks, *vs, *kt, *vt;
  const int32_t *block_table, *seq_lens;
  int num_blocks, Hkv, Pmax, B, tail_pages;
#ifdef __CUDACC__
  // first element of the tail's page that `page` of request b has, of KV head h
  __device__ __forceinline__ int64_t tail_at(int b, int h, int page) const {
    return ((((int64_t)b * Hkv + h) * tail_pages + (page & (tail_pages - 1))) * B) * LOCKS_D;
  }
#endif
};

static inline KvqCache kvq_cache(const locks_ctx *c, const locks_kvq *kv) {
  return KvqCache{reinterpret_cast<char *>(kv->k), reinterpret_cast<char *>(kv->v), kv->stride_block, kv->stride_head, kv->stride_token,
                  kv->k_scale, kv->v_scale, kv->k_tail, kv->v_tail, kv->block_table, kv->seq_lens, kv->num_blocks,
                  c->cfg.num_kv_heads, c->Pmax, c->B, kv->tail_pages == 2 ? 2 : 1};
}

static inline int kvq_check(const locks_ctx *c, const locks_kvq *kv, int batch) {
  if (!c || !kv || !kv->k || !kv->v || !kv->k_scale || !kv->v_scale || !kv->k_tail || !kv->v_tail || !kv->block_table || !kv->seq_lens)
    return LOCKS_ERR_INVALID_ARG;
  if (c->cfg.kv_dtype != LOCKS_BF16) return LOCKS_ERR_UNSUPPORTED;
  if (batch <= 0 || batch > c->cfg.max_batch || kv->num_blocks <= 0) return LOCKS_ERR_INVALID_ARG;
  if (kv->fmt != LOCKS_KVQ_INT && kv->fmt != LOCKS_KVQ_FLOAT) return LOCKS_ERR_INVALID_ARG;
  if (kv->tail_pages < 0 || kv->tail_pages > 2) return LOCKS_ERR_INVALID_ARG;
  if (kv->stride_block <= 0 || kv->stride_head <= 0 || kv->stride_token < LOCKS_D) return LOCKS_ERR_INVALID_ARG;
  if ((kv->stride_block | kv->stride_head | kv->stride_token) % 16) return LOCKS_ERR_INVALID_ARG;
  if (((uintptr_t)kv->k | (uintptr_t)kv->v | (uintptr_t)kv->k_tail | (uintptr_t)kv->v_tail) % 16) return LOCKS_ERR_INVALID_ARG;
  if (((uintptr_t)kv->k_scale | (uintptr_t)kv->v_scale) % 4) return LOCKS_ERR_INVALID_ARG;
  return LOCKS_OK;
}

// attention of many rows per KV head (kvq_chunk.cu); cu is not null
int locks_launch_kvq_chunk(locks_ctx *c, const void *q, const int32_t *cu, int n, const locks_kvq *kv, int batch, void *out, float *lse, cudaStream_t st);

// token attention: partials of the problems that several CTAs share, of whom each leaves at most two
// chunk attention: of 256 rows in each CTA of its splits, with one number a row
static_assert(KVQ_CHUNK_SLOTS * KVQ_CHUNK_ROWS <= 4 * KVQ_SLOT_BOUND * KVQ_ROWS, "");
static inline size_t kvq_part_floats() { return (size_t)std::max(2 * KVQ_SLOT_BOUND * KVQ_ROWS, KVQ_CHUNK_SLOTS * KVQ_CHUNK_ROWS) * LOCKS_D; }
static inline size_t kvq_ml_floats() { return (size_t)2 * KVQ_SLOT_BOUND * KVQ_ROWS * 2; }

#ifdef __CUDACC__
// Value of a code, exactly, in fp16.  Signed bytes: with the sign bit flipped, byte u = code + 128; 0x6400 | u is 1024 + u, and
// 1152 off it is the code.
__device__ __forceinline__ uint32_t half2_sub(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
template <int FMT> __device__ __forceinline__ uint32_t kvq_flip(uint32_t w) { return FMT == LOCKS_KVQ_INT ? w ^ 0x80808080u : w; }
// bytes 0, 1 (lo) and 2, 3 (hi) of a flipped word
template <int FMT> __device__ __forceinline__ void kvq_halves(uint32_t w, uint32_t &lo, uint32_t &hi) {
  if (FMT == LOCKS_KVQ_INT) {
    lo = half2_sub(__byte_perm(w, 0x64646464u, 0x4140), 0x64806480u);
    hi = half2_sub(__byte_perm(w, 0x64646464u, 0x4342), 0x64806480u);
  } else {
    asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
  }
}
#endif
