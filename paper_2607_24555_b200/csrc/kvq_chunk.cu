// Attention over the 8-bit paged cache for chunks of prompts: many query rows per KV head (kvq_attend.cu has the formula, and the form
// for few rows).
//
// A CTA takes 128 rows, the G heads of 128 / G consecutive tokens of one request, and walks the tokens that they see in tiles of 64.
// Both products run on the fifth-generation tensor cores, accumulators in tensor memory: S [128 x 64] = Q K^T (two buffers), O [128 x
// 128] += P V.  Four warps convert: codes to fp16 (exactly: numbers up to 127, or e4m3 numbers) in shared memory, tile j + 1 while tile
// j is multiplied; K [token][dim] is the K-major operand of the first product, V in the same layout the MN-major one of the
// second.  Four warps do the softmax, a thread per row, which needs no exchange between lanes; weights go to shared memory in fp16.
// One thread issues S of tile j + 1 before it waits for the weights of tile j, so that the tensor cores work through a softmax.
// Two CTAs share an SM.
//
// Key scales are factors of the scores.  A page's value scale goes into its weights, relative to a power of two that is at least twice
// the largest value scale so far.  A row's weights are 2^7 p relative to a maximum that is let grow by 2^8 before the output is
// rescaled (in tensor memory: rarely more than once or twice a row), so they stay below 2^15, and normal in fp16 down to 2^-21 of the
// largest.  Bound by the softmax threads and the conversion, which share the issue slots (about 450 and 270 cycles of a tile, whose
// products take 524).
#include "kvq.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kRows = 128, kTok = 64, kThreads = 288;   // warps 0 .. 3 softmax, 4 .. 7 conversion, 8 issues
// shared memory, all tiles in rows of 128 bytes with their 16-byte pieces exchanged by row (piece ^ row % 8):
// queries [2 x 64 dims][128 rows]; two stages of K and V [2 x 64 dims][64 tokens]; weights [128 rows]
constexpr int kQBytes = 2 * kRows * 128, kKvTile = 2 * kTok * 128;
constexpr int kOffKv = kQBytes, kOffP = kOffKv + 4 * kKvTile, kOffMisc = kOffP + kRows * 128;
struct Misc {
  uint64_t kv_full[2], kv_empty[2], s_full[2], p_full, pv_done, q_full, drained;
  float scale[2][2][4];   // [stage][K, V][16-token part]
  int there[2][4];        // [stage][part]
  float red[8];
  int found[4];
  uint32_t tmem;
  int slow;               // the unfinished page has values that are not finite
};
constexpr int kSmem = kOffMisc + (int)sizeof(Misc);
static_assert(kSmem <= 115712, "two CTAs an SM");
constexpr int kTmemCols = 256, kColO = 128;   // S at columns 0 and 64

// weights are 2^kTop p relative to a maximum that may be exceeded by 2^8, times at most 1/2
constexpr float kTop = 8.f;

struct ChunkParams {
  const __nv_bfloat16 *q;
  const int32_t *cu;
  KvqCache c;
  __nv_bfloat16 *out;
  float *lse;
  int32_t *status;
  int n, batch, Hq, G, tile_tokens, log_b;
  float c2;
};

__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}
// the power of two that brings a magnitude to 2^top .. 2^(top + 1)
__device__ __forceinline__ float power_to(float amax, int top) {
  const int e = (int)(__float_as_uint(amax) >> 23) - 127;
  return amax < 1e-30f ? 1.f : __uint_as_float((uint32_t)(min(max(top - e, -126), 127) + 127) << 23);
}
// piece `piece` (eight fp16) of row `row` of a tile with rows of 128 bytes
__device__ __forceinline__ uint32_t at128(int row, int piece) { return row * 128 + ((piece ^ (row & 7)) << 4); }

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(*reinterpret_cast<unsigned long long *>(&d))
      : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)),
        "l"(*reinterpret_cast<unsigned long long *>(&c)));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(*reinterpret_cast<unsigned long long *>(&d))
      : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(*reinterpret_cast<unsigned long long *>(&d))
      : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)));
  return d;
}
__device__ __forceinline__ uint4 load_if(const void *src, bool there) {   // 16 bytes, or zeros
  uint4 y;
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %5, 0;\n mov.b32 %0, 0;\n mov.b32 %1, 0;\n mov.b32 %2, 0;\n mov.b32 %3, 0;\n"
               " @p ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n}\n"
               : "=&r"(y.x), "=&r"(y.y), "=&r"(y.z), "=&r"(y.w)
               : "l"(src), "r"((int)there));
  return y;
}
// ---- tensor memory and the instructions that work on it
__device__ __forceinline__ void tmem_ld32(uint32_t (&r)[32], uint32_t at) {   // 32 columns of this thread's lane
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]) : "r"(at));
}
__device__ __forceinline__ void tmem_ld8(uint32_t (&r)[8], uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(at));
}
__device__ __forceinline__ void tmem_st32(const uint32_t (&r)[32], uint32_t at) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};\n" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(at));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint64_t *bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t *bar) {   // arrives when this thread's products so far are done
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Operand descriptor: rows of 128 bytes, swizzled, eight rows (1024 bytes) to the next eight; lbo: bytes from 64 elements of the major
// dimension to the next 64 (MN-major operands).  Version 1, layout type 2 (128-byte swizzle).
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t lbo) {
  return (uint64_t)((at >> 4) & 0x3fff) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// fp16 by fp16 to fp32, 128 rows, n columns; b_mn: the second operand is MN-major
template <int n, int b_mn>
__device__ __forceinline__ constexpr uint32_t instruction() { return 1u << 4 | (uint32_t)b_mn << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(kRows >> 4) << 24; }

__device__ __forceinline__ uint32_t f32_bits(float x) { return __float_as_uint(x); }

template <int FMT>
__global__ void __launch_bounds__(kThreads, 2) kvq_chunk_kernel(const __grid_constant__ ChunkParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  Misc &ms = *reinterpret_cast<Misc *>(smem + kOffMisc);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int Hkv = p.c.Hkv, h = blockIdx.x % Hkv, B = p.c.B;
  pdl_trigger();
  pdl_wait();
  // ---- the row tile of this CTA: a request's tiles from the last one on, so that the ones that see most start first
  if (tid == 0) {
    ms.found[0] = -1;
    ms.slow = 0;
  }
  __syncthreads();
  if (warp == 0) {
    int before = 0;
    const int want = blockIdx.x / Hkv;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
      int n = 0, row0 = 0;
      if (b0 + lane < p.batch) {
        row0 = p.cu[b0 + lane];
        n = p.cu[b0 + lane + 1] - row0;
        if (n < 0 || row0 < 0 || row0 > p.n - n) {
          set_status(p.status, LOCKS_ERR_BAD_BLOCK);
          n = 0;
        }
      }
      const int tiles = (n + p.tile_tokens - 1) / p.tile_tokens;
      int end = tiles;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, end, o);
        if (lane >= o) end += y;
      }
      const int at = want - before - (end - tiles);
      if (at >= 0 && at < tiles) { ms.found[0] = b0 + lane; ms.found[1] = tiles - 1 - at; ms.found[2] = row0; ms.found[3] = n; }
      before += __shfl_sync(0xffffffffu, end, 31);
    }
  }
  __syncthreads();
  const int b = ms.found[0];
  if (b < 0) return;
  const int j0 = ms.found[1] * p.tile_tokens, row0 = ms.found[2] + j0, n = ms.found[3];
  const int toks = min(p.tile_tokens, n - j0), rows = toks * p.G;
  const int T = max(p.c.seq_lens[b], 0);
  const int seen0 = T - n + j0 + 1;      // tokens that the tile's first token sees
  const int full_pages = T / B;
  if (T > 0 && (T - 1) / B >= p.c.Pmax && tid == 0) set_status(p.status, LOCKS_ERR_BAD_BLOCK);
  const int last = min(min(seen0 + toks - 1, T), p.c.Pmax * B);   // tokens that the tile's last token sees
  const int codes_end = min(last, full_pages * B);                // of them, those in codes
  const int tiles = last > 0 ? (codes_end + kTok - 1) / kTok : 0;
  const int tail_tiles = full_pages < p.c.Pmax && last > full_pages * B ? (last - full_pages * B + 31) / 32 : 0;
  const int nt = tiles + tail_tiles;     // then the unfinished page, 32 tokens at a time
  if (tid == 0) {
    mbar_init(&ms.kv_full[0], 128); mbar_init(&ms.kv_full[1], 128);
    mbar_init(&ms.kv_empty[0], 1); mbar_init(&ms.kv_empty[1], 1);
    mbar_init(&ms.s_full[0], 1); mbar_init(&ms.s_full[1], 1);
    mbar_init(&ms.p_full, 128); mbar_init(&ms.pv_done, 1); mbar_init(&ms.q_full, 128); mbar_init(&ms.drained, 1);
    fence_barrier_init();
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&ms.tmem)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = ms.tmem;
  const uint32_t base = smem_u32(smem);
  bool ok = true;   // no wait of this thread has run out

  if (warp == 8) {
    // ------------------------------------------------------------------------------------------ issue
    if (lane == 0 && nt > 0) {
      auto issue_s = [&](int j) {
        if (!(ok = ok && mbar_wait(&ms.kv_full[j & 1], (j >> 1) & 1))) return;
        fence_after();
        const uint32_t k = base + kOffKv + (j & 1) * 2 * kKvTile;
#pragma unroll
        for (int s = 0; s < 8; ++s)   // 16 dims a step: 32 bytes on in a row of 64 dims, then the other 64
          mma_f16_ss(tmem + 64 * (j & 1), operand(base + (s >> 2) * kRows * 128 + (s & 3) * 32, 16), operand(k + (s >> 2) * kTok * 128 + (s & 3) * 32, 16), instruction<kTok, 0>(), s > 0);
        mma_commit(&ms.s_full[j & 1]);
      };
      ok = mbar_wait(&ms.q_full, 0);
      if (ok) issue_s(0);
      for (int j = 0; j < nt && ok; ++j) {
        if (j + 1 < nt) issue_s(j + 1);
        if (!(ok = ok && mbar_wait(&ms.p_full, j & 1))) break;
        fence_after();
        const uint32_t v = base + kOffKv + (j & 1) * 2 * kKvTile + kKvTile;
#pragma unroll
        for (int s = 0; s < 4; ++s)   // 16 tokens a step
          mma_f16_ss(tmem + kColO, operand(base + kOffP + s * 32, 16), operand(v + s * 16 * 128, kTok * 128), instruction<LOCKS_D, 1>(), j > 0 || s > 0);
        mma_commit(&ms.kv_empty[j & 1]);
        mma_commit(&ms.pv_done);
      }
      mma_commit(&ms.drained);
      ok = mbar_wait(&ms.drained, 0) && ok;   // nothing is under way when the tensor memory is given back
    }
    __syncwarp();
  } else if (warp >= 4) {
    // ------------------------------------------------------------------------------------------ conversion
    const int ct = tid - 128, piece = ct & 7, tok = ct >> 3;   // 16 dims of tokens tok + 16 i, i.e. of part i
    int blk[4], my_blk = 0;   // (my_blk: of part ct % 4, whose scale of K, V threads 0 .. 3, 4 .. 7 fetch)
    uint4 k[4], v[4];
    float my_scale = 0.f;
    int my_there = 0;
    const int32_t *row = p.c.block_table + (int64_t)b * p.c.Pmax;
    const char *kp = p.c.k + (int64_t)h * p.c.sh + piece * 16, *vp = p.c.v + (int64_t)h * p.c.sh + piece * 16;
    auto blocks = [&](int tile) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int pos = tile * kTok + 16 * i;
        blk[i] = pos < codes_end ? row[pos >> p.log_b] : -1;
      }
      const int pos = tile * kTok + 16 * (ct & 3);
      my_blk = pos < codes_end ? row[pos >> p.log_b] : -1;
    };
    auto is_there = [&](int block) { return (uint32_t)block < (uint32_t)p.c.num_blocks; };
    auto fetch = [&](int tile) {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int pos = tile * kTok + 16 * i;
        const bool good = is_there(blk[i]);
        bad |= !good && pos < codes_end;
        const int64_t off = good ? (int64_t)blk[i] * p.c.sb + (int64_t)((pos & (B - 1)) + tok) * p.c.st : 0;
        k[i] = load_if(kp + off, good);
        v[i] = load_if(vp + off, good);
      }
      if (bad && ct == 0) set_status(p.status, LOCKS_ERR_BAD_BLOCK);
      const bool good = is_there(my_blk);
      my_scale = ct < 8 && good ? (ct < 4 ? p.c.ks : p.c.vs)[(int64_t)my_blk * Hkv + h] : 0.f;
      my_there = good;
      blocks(tile + 1);
    };
    auto put = [&](uint8_t *tile, int row, int dim_piece, const uint32_t (&f)[4]) {   // eight dims from 8 dim_piece on
      *reinterpret_cast<uint4 *>(tile + (dim_piece >> 3) * kTok * 128 + at128(row, dim_piece & 7)) = make_uint4(f[0], f[1], f[2], f[3]);
    };
    if (tiles > 0) {
      blocks(0);
      fetch(0);
    }
    for (int j = 0; j < nt; ++j) {
      const int stage = j & 1;
      uint8_t *kt = smem + kOffKv + stage * 2 * kKvTile, *vt = kt + kKvTile;
      if (j >= 2 && ok) ok = mbar_wait(&ms.kv_empty[stage], ((j >> 1) - 1) & 1);   // (run out: on, so that no barrier waits for this thread)
      if (j < tiles) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = tok + 16 * i;
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const uint4 y = kv ? v[i] : k[i];
            const uint32_t word[4] = {y.x, y.y, y.z, y.w};
            uint32_t f[2][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) kvq_halves<FMT>(kvq_flip<FMT>(word[e]), f[e >> 1][2 * (e & 1)], f[e >> 1][2 * (e & 1) + 1]);
            // (of a row's eight threads, four write the second half first: their pieces lie in eight different banks' groups)
            const bool turn = piece & 4;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t w[4] = {turn ? f[1 - e][0] : f[e][0], turn ? f[1 - e][1] : f[e][1], turn ? f[1 - e][2] : f[e][2], turn ? f[1 - e][3] : f[e][3]};
              put(kv ? vt : kt, row, 2 * piece + (turn ? 1 - e : e), w);
            }
          }
        }
        if (ct < 8) ms.scale[stage][ct >> 2][ct & 3] = my_scale;
        if (ct < 4) ms.there[stage][ct] = my_there;
        if (j + 1 < tiles) fetch(j + 1);
      } else {
        // a thread: 32 dims of one token of 32, as fp16 times a power of two of the 32 tokens' largest; keys in two parts (22 bits), the
        // second in rows 32 on; values' rows 32 on are zero
        const int pos = full_pages * B + 32 * (j - tiles), tt = ct >> 2, d0 = 32 * (ct & 3);
        const int64_t at = (((int64_t)b * Hkv + h) * B + pos - full_pages * B + tt) * LOCKS_D + d0;
        const float *src[2] = {p.c.kt + at, p.c.vt + at};
        const bool in = pos + tt < T;
        float amax[2] = {0.f, 0.f}, up[2];
        bool odd = false;
        if (in) {
#pragma unroll
          for (int kv = 0; kv < 2; ++kv)
#pragma unroll 2
            for (int i = 0; i < 8; ++i) {
              const float4 y = reinterpret_cast<const float4 *>(src[kv])[i];
              amax[kv] = fmaxf(amax[kv], fmaxf(fmaxf(finite_abs(y.x), finite_abs(y.y)), fmaxf(finite_abs(y.z), finite_abs(y.w))));
              if (kv) odd |= !(fabsf(y.x) < INFINITY && fabsf(y.y) < INFINITY && fabsf(y.z) < INFINITY && fabsf(y.w) < INFINITY);
            }
        }
        if (odd) ms.slow = 1;
        asm volatile("bar.sync 1, 128;\n" ::: "memory");   // the reductions before are used
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const float y = warp_max(amax[kv]);
          if (lane == 0) ms.red[4 * kv + warp - 4] = y;
        }
        asm volatile("bar.sync 1, 128;\n" ::: "memory");
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) up[kv] = power_to(fmaxf(fmaxf(ms.red[4 * kv], ms.red[4 * kv + 1]), fmaxf(ms.red[4 * kv + 2], ms.red[4 * kv + 3])), 14);
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
          uint32_t hi[4], lo[4], val[4], zero[4] = {0, 0, 0, 0};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float2 y = make_float2(0.f, 0.f), z = y;
            if (in) { y = *reinterpret_cast<const float2 *>(src[0] + 8 * i + 2 * e); z = *reinterpret_cast<const float2 *>(src[1] + 8 * i + 2 * e); }
            y.x *= up[0]; y.y *= up[0];
            hi[e] = pack_f16(y.x, y.y);
            const float2 r = __half22float2(*reinterpret_cast<__half2 *>(&hi[e]));
            lo[e] = pack_f16(fabsf(y.x) < INFINITY ? y.x - r.x : 0.f, fabsf(y.y) < INFINITY ? y.y - r.y : 0.f);
            // (values that are not finite are added at the end, to the rows that see them)
            val[e] = pack_f16(fabsf(z.x) < INFINITY ? z.x * up[1] : 0.f, fabsf(z.y) < INFINITY ? z.y * up[1] : 0.f);
          }
          const int dim_piece = d0 / 8 + i;
          put(kt, tt, dim_piece, hi);
          put(kt, tt + 32, dim_piece, lo);
          put(vt, tt, dim_piece, val);
          put(vt, tt + 32, dim_piece, zero);
        }
        if (ct < 4) {
          ms.scale[stage][0][ct] = 1.f / up[0];
          ms.scale[stage][1][ct] = ct < 2 ? 1.f / up[1] : 0.f;
          ms.there[stage][ct] = ct < 2;
        }
      }
      fence_async_proxy();
      mbar_arrive(&ms.kv_full[stage]);
    }
  } else {
    // ------------------------------------------------------------------------------------------ softmax: thread = row
    const int r = tid, jr = r / p.G, g = r - jr * p.G;
    const bool real = r < rows;
    float cr;
    {
      const uint4 *src = reinterpret_cast<const uint4 *>(p.q + ((int64_t)(row0 + jr) * p.Hq + h * p.G + g) * LOCKS_D);
      float amax = 0.f;
      if (real) {
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
          const uint4 w = src[i];
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) amax = fmaxf(amax, fmaxf(finite_abs(__uint_as_float(u[e] << 16)), finite_abs(__uint_as_float(u[e] & 0xFFFF0000u))));
        }
      }
      const float up = power_to(amax, 0);
      cr = p.c2 / up;
#pragma unroll 4
      for (int i = 0; i < 16; ++i) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (real) w = src[i];
        uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = pack_f16(__uint_as_float(u[e] << 16) * up, __uint_as_float(u[e] & 0xFFFF0000u) * up);
        *reinterpret_cast<uint4 *>(smem + (i >> 3) * kRows * 128 + at128(r, i & 7)) = make_uint4(u[0], u[1], u[2], u[3]);
      }
    }
    fence_async_proxy();
    mbar_arrive(&ms.q_full);
    const int lim = real ? seen0 + jr : last;   // this row sees the first lim tokens
    const uint32_t lane_at = tmem + ((uint32_t)(32 * warp) << 16);
    float m = -INFINITY, l = 0.f, vref = 0.f;
    for (int j = 0; j < nt && ok; ++j) {
      const int stage = j & 1;
      const bool tail = j >= tiles;
      const int pos = tail ? full_pages * B + 32 * (j - tiles) : j * kTok;
      ok = mbar_wait(&ms.s_full[stage], (j >> 1) & 1) && mbar_wait(&ms.kv_full[stage], (j >> 1) & 1);   // (the second: the scales)
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      fence_after();
      float f[4], vs[4];
      bool all_there = true;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[i] = cr * ms.scale[stage][0][i];
        vs[i] = ms.scale[stage][1][i];
        all_there = all_there && ms.there[stage][i];
      }
      // who sees what: 64 bits of the tile's tokens (parts that are not there are seen by nobody)
      uint64_t sees = ~0ull;
      const bool mask = pos + (tail ? 32 : kTok) > seen0 || !all_there || tail;
      if (mask) {
        const int left = lim - pos;
        sees = left <= 0 ? 0ull : (left >= 64 ? ~0ull : (1ull << left) - 1);
        if (tail) sees &= 0xffffffffull;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!ms.there[stage][i]) sees &= ~(0xffffull << (16 * i));
      }
      // the scores of half a tile; of the unfinished page, with what fp16 left of the keys
      uint32_t s[32];
      auto scores = [&](int half) {
        tmem_ld32(s, lane_at + 64 * stage + 32 * half);
        tmem_wait_ld();
        if (tail && half == 0) {
#pragma unroll
          for (int c = 0; c < 32; c += 8) {
            uint32_t rest[8];
            tmem_ld8(rest, lane_at + 64 * stage + 32 + c);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i) s[c + i] = f32_bits(__uint_as_float(s[c + i]) + __uint_as_float(rest[i]));
          }
        }
      };
      // the tile's maximum
      float mx = -INFINITY;
      if (mask) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          scores(half);
          const uint32_t bits = (uint32_t)(sees >> (32 * half));
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if ((bits >> i) & 1) mx = fmaxf(mx, __uint_as_float(s[i]) * f[2 * half + (i >> 4)]);
        }
      } else {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          tmem_ld32(s, lane_at + 64 * stage + 32 * half);
          tmem_wait_ld();
          float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            m0 = fmaxf(m0, __uint_as_float(s[i]));
            m1 = fmaxf(m1, __uint_as_float(s[16 + i]));
          }
          mx = fmaxf(mx, fmaxf(m0 * f[2 * half], m1 * f[2 * half + 1]));
        }
      }
      // the row's maximum, and the values' reference
      float fix = 1.f;
      if (mx > m + 8.f) {   // (also the first that is seen: the row's output and sum are zero then)
        fix = m == -INFINITY ? 1.f : ex2f(m - mx);
        l *= fix;
        m = mx;
      }
      const float vmax = fmaxf(fmaxf(vs[0], vs[1]), fmaxf(vs[2], vs[3]));   // (a NaN is not a larger one)
      if (2.f * vmax > vref) {
        const float to = __uint_as_float(min((f32_bits(vmax) >> 23) + 2u, 254u) << 23);
        fix *= vref / to;
        vref = to;
      }
      const float inv = vref > 0.f ? 1.f / vref : 0.f, off = kTop - (m == -INFINITY ? 0.f : m);
      // the product before has read the weights' memory, and its output is there to be rescaled
      if (j > 0) {
        ok = mbar_wait(&ms.pv_done, (j - 1) & 1);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        fence_after();
        if (__any_sync(0xffffffffu, fix != 1.f)) {
#pragma unroll 1
          for (int c = 0; c < LOCKS_D; c += 32) {
            tmem_ld32(s, lane_at + kColO + c);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) s[i] = f32_bits(__uint_as_float(s[i]) * fix);
            tmem_st32(s, lane_at + kColO + c);
          }
          tmem_wait_st();
        }
      }
      // weights, eight in a 16-byte piece
      auto weights = [&](int half, bool masked) {
        const uint32_t bits = (uint32_t)(sees >> (32 * half));
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int piece = 0; piece < 4; ++piece) {
          const float ff = f[2 * half + (piece >> 1)], vv = vs[2 * half + (piece >> 1)] * inv;
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int e = 8 * piece + 2 * i;
            const float2 y = fma2(make_float2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), make_float2(ff, ff), make_float2(off, off));
            float2 q = make_float2(ex2f(y.x), ex2f(y.y)), z = mul2(q, make_float2(vv, vv));
            if (masked) {   // (nothing of a scale of NaN, nor of a score)
              if (!((bits >> e) & 1)) q.x = z.x = 0.f;
              if (!((bits >> (e + 1)) & 1)) q.y = z.y = 0.f;
            }
            sum = add2(sum, q);
            w[i] = pack_f16(z.x, z.y);
          }
          *reinterpret_cast<uint4 *>(smem + kOffP + at128(r, 4 * half + piece)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        l += sum.x + sum.y;
      };
      if (mask) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          scores(half);
          weights(half, true);
        }
      } else {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          tmem_ld32(s, lane_at + 64 * stage + 32 * half);
          tmem_wait_ld();
          weights(half, false);
        }
      }
      fence_async_proxy();
      fence_before();
      mbar_arrive(&ms.p_full);
    }
    // ---- results
    if (nt > 0 && ok) ok = mbar_wait(&ms.pv_done, (nt - 1) & 1);
    const bool good = __all_sync(0xffffffffu, ok);
    fence_after();
    const int64_t row = (int64_t)(row0 + jr) * p.Hq + h * p.G + g;
    const float scale = l == 0.f ? 0.f : vref / l;   // (0: nothing seen)
    const bool slow = tail_tiles > 0 && ms.slow;     // (written before the last tiles' barriers)
#pragma unroll 1
    for (int c = 0; c < LOCKS_D; c += 32) {
      uint32_t s[32];
      if (nt > 0 && good) {
        tmem_ld32(s, lane_at + kColO + c);
        tmem_wait_ld();
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i] = 0;
      }
      if (slow) {
        const float *vt = p.c.vt + (((int64_t)b * Hkv + h) * B) * LOCKS_D + c;
#pragma unroll 1
        for (int k = 0; full_pages * B + k < min(lim, last); ++k)
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float y = vt[k * LOCKS_D + i];
            if (!(fabsf(y) < INFINITY)) s[i] = f32_bits(__uint_as_float(s[i]) + y);
          }
      }
      if (real && ok) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // (a row that has seen nothing is zero whatever lies in its output)
            const float a = __uint_as_float(s[8 * i + 2 * e]), z = __uint_as_float(s[8 * i + 2 * e + 1]);
            y[e] = l == 0.f ? 0u : pack_bf16(a * scale, z * scale);
          }
          *reinterpret_cast<uint4 *>(p.out + row * LOCKS_D + c + 8 * i) = make_uint4(y[0], y[1], y[2], y[3]);
        }
      }
    }
    if (real && ok && p.lse) p.lse[row] = l == 0.f ? -INFINITY : ((m == -INFINITY ? 0.f : m) - kTop + log2f(l)) * kLn2;
    fence_before();
  }
  if (!ok) set_status(p.status, LOCKS_ERR_TIMEOUT);
  __syncthreads();
  if (warp == 8) {
    __syncwarp();
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kTmemCols));
  }
}

}  // namespace

int locks_launch_kvq_chunk(locks_ctx *c, const void *q, const int32_t *cu, int n, const locks_kvq *kv, int batch, void *out, float *lse, cudaStream_t st) {
  ChunkParams p = {};
  p.q = reinterpret_cast<const __nv_bfloat16 *>(q); p.cu = cu; p.c = kvq_cache(c, kv);
  p.out = reinterpret_cast<__nv_bfloat16 *>(out); p.lse = lse; p.status = c->status;
  p.n = n; p.batch = batch; p.Hq = c->cfg.num_q_heads; p.G = c->G;
  p.tile_tokens = kRows / c->G;
  p.log_b = c->B == 64 ? 6 : (c->B == 32 ? 5 : 4);
  p.c2 = c->cfg.sm_scale * kLog2e;
  const int64_t grid = ((int64_t)n / p.tile_tokens + batch) * c->cfg.num_kv_heads;   // a request's last tile may be short
  if (grid > INT32_MAX) return LOCKS_ERR_TOO_LARGE;
#define KVQ_CHUNK(F_)                                                                                                         \
  do {                                                                                                                        \
    if (locks_attrs_needed(LOCKS_ATTR_KVQ_CHUNK + F_))                                                                        \
      cudaFuncSetAttribute(kvq_chunk_kernel<F_>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);                         \
    locks_launch_pdl(kvq_chunk_kernel<F_>, dim3((unsigned)grid), dim3(kThreads), kSmem, st, p);                               \
  } while (0)
  if (kv->fmt == LOCKS_KVQ_INT) KVQ_CHUNK(LOCKS_KVQ_INT);
  else KVQ_CHUNK(LOCKS_KVQ_FLOAT);
#undef KVQ_CHUNK
  return locks_check_launch(c);
}
