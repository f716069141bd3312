// Attention over the 8-bit paged cache for chunks of prompts: many query rows per KV head (kvq_attend.cu has the formula, and the form
// for few rows).
//
// A CTA takes two times 128 rows, the G heads of 2 (128 / G) consecutive tokens of one request, and walks the tokens that they see in
// tiles of 128.  Both products run on the fifth-generation tensor cores, accumulators in tensor memory: for each 128 rows S [128 x 128]
// = Q K^T and O [128 x 128] += P V, all 512 columns.  Eight warps convert codes to fp16 (exactly: numbers up to 127, or e4m3 numbers)
// in shared memory, tile j + 1 while tile j is multiplied; K [token][dim] is the K-major operand of the first product, V in the same
// layout the MN-major one of the second.  Eight warps do the softmax, a thread per row, which needs no exchange between lanes; a row's
// weights go, in fp16, where its scores were, and are the second product's first operand from there.  One thread issues: while one 128
// rows' softmax is under way the tensor cores work for the other 128.
//
// Key scales are factors of the scores.  A page's value scale goes into its weights, relative to a power of two that is at least twice
// the largest value scale that the row has seen.  A row's weights are 2^8 p relative to a maximum that may be exceeded by 2^8 before the output is
// rescaled (in tensor memory: rarely more than once or twice a row), so they stay below 2^15, and normal in fp16 down to 2^-20 of the
// largest.
//
// Why 2 x 128 rows: a tile's conversion and its way through shared memory serve twice as many rows, and the two take turns on the tensor
// cores.  Why the scores are read once: a maximum that may be exceeded needs no second pass, and the next 32 columns' maximum hides
// between these 32's exponentials.  Registers are split by warps' kind (setmaxnreg).  Where blocks of 256 rows are fewer than SMs, the
// tokens that each sees are shared by several CTAs, and a second kernel joins them.
// Measured, 1024 tokens of 32 heads over 8 KV heads after 15277: 374 us, 708 TFLOP/s, 0.42 of a library matrix product's rate (with 128 of 148
// SMs at work: a CTA for each block); without the softmax 252, without products and conversion 276 (of 369 then).  Pipes are about half busy
// (exponentials 50 %, tensor cores 40 %, issue 43 %): bound by the latencies of a chain of softmax and products with two softmax warps a
// scheduler.  One request's tokens after 16K: 46 us (32 tokens), 74 (128), 210 (512).  Accumulators add up in the tensor cores' fp32.
#include <algorithm>
#include <type_traits>

#include "kvq.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kRows = 128, kTok = 128, kParts = kTok / 16;
constexpr int kSoft = 256, kConv = 256, kThreads = kSoft + kConv + 128;   // warps 0 .. 7 softmax, 8 .. 15 conversion, 16 issues, three idle
// registers a thread: of the launch, then of the three kinds; their sum is the launch's
constexpr int kRegs = 96, kSoftRegs = 136, kConvRegs = 80, kIssueRegs = 48;
static_assert(kRegs * kThreads == kSoftRegs * kSoft + kConvRegs * kConv + kIssueRegs * 128, "");
// shared memory, all tiles in rows of 128 bytes with their 16-byte pieces exchanged by row (piece ^ row % 8):
// queries [2][2 x 64 dims][128 rows]; two stages of K and V [2 x 64 dims][128 tokens]
constexpr int kQTile = 2 * kRows * 128, kKvTile = 2 * kTok * 128;
constexpr int kOffKv = 2 * kQTile, kOffMisc = kOffKv + 4 * kKvTile;
struct Misc {
  uint64_t kv_full[2], kv_empty[2], s_full[2], p_full[2], q_full, o_full;
  float scale[2][2][kParts];   // [stage][K, V][16-token part]
  uint32_t there[2];           // [stage]: a bit per part
  float red[16];
  int found[6];
  uint32_t tmem;
  int slow;                    // the unfinished page has values that are not finite
};
constexpr int kSmem = kOffMisc + (int)sizeof(Misc);
static_assert(kSmem <= 227 * 1024, "one CTA an SM");
constexpr int kTmemCols = 512, kColO = 256;   // S (and weights) of the two 128 rows at columns 0 and 128, O at 256 and 384
// weights are 2^kTop p relative to a maximum that may be exceeded by 2^8, times at most 1/2
constexpr float kTop = 8.f;

struct ChunkParams {
  const __nv_bfloat16 *q;
  const int32_t *cu;
  KvqCache c;
  __nv_bfloat16 *out;
  float *lse, *part, *part_lse;   // (partials of the splits: [block, head][split][2 x 128 rows], normalised, and log2 of their sums)
  int32_t *status;
  int n, batch, Hq, G, tile_tokens, log_b, slots;   // tile_tokens: of 128 rows; slots: CTAs that may leave partials
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
// ---- tensor memory and the instructions that work on it.  Loads, stores and their waits are a whole warp's: behind code that branches by
// lane (rows differ in what they see) the kernel brings the lanes together before the next of them: a chunk of 1024 tokens 369.6 -> 373.7 us.
// (In each of these functions: 381.)
template <int N> __device__ __forceinline__ void tmem_ld(uint32_t *r, uint32_t at) {   // N columns of this thread's lane
  if constexpr (N == 32)
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]) : "r"(at));
  else
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(at));
}
template <int N> __device__ __forceinline__ void tmem_st(const uint32_t *r, uint32_t at) {
  static_assert(N == 16, "");
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};\n" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(at));
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
// first operand in tensor memory: two fp16 a column
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
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

// A unit of work: a block of 2 tile_tokens tokens of a request, and which share of the tokens that it sees.  Blocks are numbered request
// by request, a request's from the last one on, so that the ones that see most start first; where there are few, each is split so that
// the slots are all used.
struct Block {
  int b, j0, row0, n;   // request (< 0: none), its token and row at which the block starts, tokens of the request
  int index, splits;
};
// unit: index * per_index * splits + something smaller, or the index itself (per_index 0)
__device__ __forceinline__ Block find_block(const ChunkParams &p, int unit, int per_index, int (&found)[6]) {
  const int tokens = 2 * p.tile_tokens;
  if (threadIdx.x == 0) found[0] = -1;
  __syncthreads();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    auto blocks_of = [&](int b, int &row0, int &n) -> int {
      n = row0 = 0;
      if (b < p.batch) {
        row0 = p.cu[b];
        n = p.cu[b + 1] - row0;
        if (n < 0 || row0 < 0 || row0 > p.n - n) {
          set_status(p.status, LOCKS_ERR_BAD_BLOCK);
          n = 0;
        }
      }
      return (n + tokens - 1) / tokens;
    };
    int total = 0, row0, n;
    for (int b0 = 0; b0 < p.batch; b0 += 32) total += blocks_of(b0 + lane, row0, n);
    total = __reduce_add_sync(0xffffffffu, total);
    const int splits = max(1, p.slots / max(1, min(total, p.slots) * p.c.Hkv)), want = per_index ? unit / (per_index * splits) : unit;
    int before = 0;
    for (int b0 = 0; b0 < p.batch && before <= want; b0 += 32) {
      const int blocks = blocks_of(b0 + lane, row0, n);
      int end = blocks;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, end, o);
        if (lane >= o) end += y;
      }
      const int at = want - before - (end - blocks);
      if (at >= 0 && at < blocks) { found[0] = b0 + lane; found[1] = blocks - 1 - at; found[2] = row0; found[3] = n; }
      before += __shfl_sync(0xffffffffu, end, 31);
    }
    if (lane == 0) { found[4] = want; found[5] = splits; }
  }
  __syncthreads();
  const int j0 = found[1] * tokens;
  return Block{found[0], j0, found[2] + j0, found[3], found[4], found[5]};
}

template <int FMT>
__global__ void __launch_bounds__(kThreads, 1) kvq_chunk_kernel(const __grid_constant__ ChunkParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  Misc &ms = *reinterpret_cast<Misc *>(smem + kOffMisc);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int Hkv = p.c.Hkv, B = p.c.B, cta_tokens = 2 * p.tile_tokens;
  pdl_trigger();
  pdl_wait();
  if (tid == 0) ms.slow = 0;
  const Block at = find_block(p, blockIdx.x, Hkv, ms.found);
  const int b = at.b, j0 = at.j0, row0 = at.row0, n = at.n;
  if (b < 0) return;
  const int splits = at.splits, split = blockIdx.x % splits, h = blockIdx.x / splits % Hkv;
  const int toks = min(cta_tokens, n - j0), halves = toks > p.tile_tokens ? 2 : 1;   // of 128 rows
  const int T = max(p.c.seq_lens[b], 0);
  const int seen0 = T - n + j0 + 1;      // tokens that the CTA's first token sees
  const int full_pages = T >> p.log_b;
  if (T > 0 && (T - 1) >> p.log_b >= p.c.Pmax && tid == 0) set_status(p.status, LOCKS_ERR_BAD_BLOCK);
  const int last = min(min(seen0 + toks - 1, T), p.c.Pmax * B);   // tokens that the CTA's last token sees
  const int codes_end = min(last, full_pages * B);                // of them, those in codes
  // ---- tiles of 128 tokens, then the unfinished page (fewer than 64); of them this CTA's share: nt from tile0 on, `tiles` of them codes
  const int all_codes = last > 0 ? (codes_end + kTok - 1) / kTok : 0;
  const int64_t all = all_codes + (full_pages < p.c.Pmax && last > full_pages * B);
  const int tile0 = (int)(all * split / splits), nt = (int)(all * (split + 1) / splits) - tile0;
  const int tiles = min(max(all_codes - tile0, 0), nt), tail_tiles = nt - tiles;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ms.kv_full[i], kConv); mbar_init(&ms.kv_empty[i], 1);
      mbar_init(&ms.s_full[i], 1); mbar_init(&ms.p_full[i], kRows);
    }
    mbar_init(&ms.q_full, kSoft); mbar_init(&ms.o_full, 1);
    fence_barrier_init();
  }
  if (warp == 16) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&ms.tmem)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = ms.tmem;
  const uint32_t base = smem_u32(smem);
  bool ok = true;   // no wait of this thread has run out

  if (warp >= 16) {
    // ------------------------------------------------------------------------------------------ issue
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kIssueRegs));
    if (tid == kSoft + kConv && nt > 0) {
      auto issue_s = [&](int j, int t) {
        const uint32_t q = base + t * kQTile, k = base + kOffKv + (j & 1) * 2 * kKvTile;
#pragma unroll
        for (int s = 0; s < 8; ++s)   // 16 dims a step: 32 bytes on in a row of 64 dims, then the other 64
          mma_f16_ss(tmem + 128 * t, operand(q + (s >> 2) * kRows * 128 + (s & 3) * 32, 16), operand(k + (s >> 2) * kTok * 128 + (s & 3) * 32, 16), instruction<kTok, 0>(), s > 0);
        mma_commit(&ms.s_full[t]);
      };
      auto tile_there = [&](int j) {
        if (ok) ok = mbar_wait(&ms.kv_full[j & 1], (j >> 1) & 1);
        fence_after();
      };
      ok = mbar_wait(&ms.q_full, 0);
      tile_there(0);
      if (ok)
        for (int t = 0; t < halves; ++t) issue_s(0, t);
      // a half's scores of tile j + 1 take the place of its weights of tile j, which the product before them has read: products are
      // done in the order in which they are issued
      for (int j = 0; j < nt && ok; ++j) {
        const uint32_t v = base + kOffKv + (j & 1) * 2 * kKvTile + kKvTile;
        for (int t = 0; t < halves && ok; ++t) {
          if (!(ok = mbar_wait(&ms.p_full[t], j & 1))) break;
          fence_after();
#pragma unroll
          for (int s = 0; s < 8; ++s)   // 16 tokens a step
            mma_f16_ts(tmem + kColO + 128 * t, tmem + 128 * t + 8 * s, operand(v + s * 16 * 128, kTok * 128), instruction<LOCKS_D, 1>(), j > 0 || s > 0);
          if (t == halves - 1) mma_commit(&ms.kv_empty[j & 1]);
          if (j + 1 < nt) {
            if (t == 0) tile_there(j + 1);
            if (ok) issue_s(j + 1, t);
          }
        }
      }
      mma_commit(&ms.o_full);
      ok = mbar_wait(&ms.o_full, 0) && ok;   // nothing is under way when the tensor memory is given back
    }
    __syncwarp();
  } else if (warp >= 8) {
    // ------------------------------------------------------------------------------------------ conversion
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kConvRegs));
    const int ct = tid - kSoft, piece = ct & 7, tok = ct >> 3;   // 16 dims of tokens tok + 32 i
    int blk[4], my_blk = 0, my_there = 0;   // (my_blk: of part ct % 8, whose scale of K, V threads 0 .. 7, 8 .. 15 fetch)
    uint4 k[4], v[4];
    float my_scale = 0.f;
    const int left = codes_end - tile0 * kTok;   // tokens in codes from tile0 on, and their pages
    const int32_t *row = p.c.block_table + (int64_t)b * p.c.Pmax + ((tile0 * kTok) >> p.log_b);
    const char *kp = p.c.k + (int64_t)h * p.c.sh + piece * 16, *vp = p.c.v + (int64_t)h * p.c.sh + piece * 16;
    auto blocks = [&](int tile) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int pos = tile * kTok + 32 * i + (tok & 16);
        blk[i] = pos < left ? row[pos >> p.log_b] : -1;
      }
      const int pos = tile * kTok + 16 * (ct & 7);
      my_blk = pos < left ? row[pos >> p.log_b] : -1;
    };
    auto is_there = [&](int block) { return (uint32_t)block < (uint32_t)p.c.num_blocks; };
    auto fetch = [&](int tile) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int pos = tile * kTok + 32 * i + tok;
        const bool good = is_there(blk[i]);
        const int64_t off = good ? (int64_t)blk[i] * p.c.sb + (int64_t)(pos & (B - 1)) * p.c.st : 0;
        k[i] = load_if(kp + off, good);
        v[i] = load_if(vp + off, good);
      }
      my_there = is_there(my_blk);
      if (!my_there && tile * kTok + 16 * (ct & 7) < left) set_status(p.status, LOCKS_ERR_BAD_BLOCK);
      my_scale = ct < 16 && my_there ? (ct < 8 ? p.c.ks : p.c.vs)[(int64_t)my_blk * Hkv + h] : 0.f;
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
        const int turn = piece >> 2;   // of a row's eight threads, four write the second eight first: all write to different banks
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const uint4 y = kv ? v[i] : k[i];
            const uint32_t word[4] = {turn ? y.z : y.x, turn ? y.w : y.y, turn ? y.x : y.z, turn ? y.y : y.w};
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              uint32_t f[4];
              kvq_halves<FMT>(kvq_flip<FMT>(word[2 * e]), f[0], f[1]);
              kvq_halves<FMT>(kvq_flip<FMT>(word[2 * e + 1]), f[2], f[3]);
              put(kv ? vt : kt, tok + 32 * i, 2 * piece + (e ^ turn), f);
            }
          }
        if (ct < 16) ms.scale[stage][ct >> 3][ct & 7] = my_scale;
        if (warp == 8) {
          const uint32_t there = __ballot_sync(0xffffffffu, my_there) & 0xff;
          if (lane == 0) ms.there[stage] = there;
        }
        if (j + 1 < tiles) fetch(j + 1);
      } else {
        // a thread: 32 dims of one token of 64, as fp16 times a power of two of the 64 tokens' largest; keys in two parts (22 bits), the
        // second in rows 64 on; values' rows 64 on are zero
        const int tt = ct >> 2, d0 = 32 * (ct & 3);
        const int64_t at = p.c.tail_at(b, h, full_pages) + tt * LOCKS_D + d0;
        const float *src[2] = {p.c.kt + at, p.c.vt + at};
        const bool in = full_pages * B + tt < T;
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
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const float y = warp_max(amax[kv]);
          if (lane == 0) ms.red[8 * kv + warp - 8] = y;
        }
        __syncwarp();
        asm volatile("bar.sync 1, %0;\n" ::"n"(kConv) : "memory");
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          float y = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) y = fmaxf(y, ms.red[8 * kv + i]);
          up[kv] = power_to(y, 14);
        }
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
          put(kt, tt + 64, dim_piece, lo);
          put(vt, tt, dim_piece, val);
          put(vt, tt + 64, dim_piece, zero);
        }
        if (ct < 8) {
          ms.scale[stage][0][ct] = 1.f / up[0];
          ms.scale[stage][1][ct] = ct < 4 ? 1.f / up[1] : 0.f;
        }
        if (ct == 0) ms.there[stage] = 0xf;
      }
      fence_async_proxy();
      mbar_arrive(&ms.kv_full[stage]);
    }
  } else {
    // ------------------------------------------------------------------------------------------ softmax: thread = row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kSoftRegs));
    const int t = warp >> 2, r = tid & 127;
    const int first = seen0 + t * p.tile_tokens - tile0 * kTok;   // tokens from tile0 on that the first of these 128 rows sees
    // this thread's token within the CTA, and its row of q and out (asked for again after the loop, so that the loop need not keep them)
    auto place = [&](int r, int &jr, int64_t &row) -> bool {
      jr = t * p.tile_tokens + r / p.G;
      row = (int64_t)(row0 + jr) * p.Hq + h * p.G + r % p.G;
      return r < p.tile_tokens * p.G && jr < toks;
    };
    float cr;
    int lim;   // this row sees the first lim tokens from tile0 on
    {
      int jr;
      int64_t row;
      const bool real = place(r, jr, row);
      lim = (real ? seen0 + jr : last) - tile0 * kTok;
      const uint4 *src = reinterpret_cast<const uint4 *>(p.q + row * LOCKS_D);
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
        *reinterpret_cast<uint4 *>(smem + t * kQTile + (i >> 3) * kRows * 128 + at128(r, i & 7)) = make_uint4(u[0], u[1], u[2], u[3]);
      }
    }
    fence_async_proxy();
    mbar_arrive(&ms.q_full);
    const int tail_pos = full_pages * B - tile0 * kTok;
    const uint32_t s_at = tmem + 128 * t + ((uint32_t)(32 * (warp & 3)) << 16), o_at = s_at + kColO;
    float m = -INFINITY, l = 0.f;                  // m: a whole number
    float vref = 0x1p-126f, inv = 0x1p126f;   // values' reference, 1 / vref
    const int mine = t < halves ? nt : 0;
    for (int j = 0; j < mine && ok; ++j) {
      const int stage = j & 1;
      const bool tail = j >= tiles;
      const int pos = tail ? tail_pos : j * kTok;
      ok = mbar_wait(&ms.s_full[t], j & 1) && mbar_wait(&ms.kv_full[stage], (j >> 1) & 1);   // (the second: the scales)
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      fence_after();
      const uint32_t there = ms.there[stage];
      const bool mask = pos + (tail ? 64 : kTok) > first || there != 0xff;
      // which of columns 32 i .. are seen (of parts that are not there, none)
      auto seen = [&](int i) -> uint32_t {
        const int left = lim - pos - 32 * i;
        uint32_t y = left <= 0 ? 0u : (left >= 32 ? ~0u : (1u << left) - 1);
        if (!((there >> (2 * i)) & 1)) y &= 0xffff0000u;
        if (!((there >> (2 * i + 1)) & 1)) y &= 0x0000ffffu;
        return y;
      };
      // ---- output and the tile's weights so far (their first `columns` columns) times fix, a power of two
      auto rescale = [&](float fix, int columns) {
        __syncwarp();
        if (j > 0) {   // (the scores are there: the product before them is done)
#pragma unroll 1
          for (int c = 0; c < LOCKS_D; c += 16) {
            uint32_t y[16];
            tmem_ld<16>(y, o_at + c);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = f32_bits(__uint_as_float(y[i]) * fix);
            tmem_st<16>(y, o_at + c);
          }
        }
        const __half2 by = __float2half2_rn(fix);
#pragma unroll 1
        for (int c = 0; c < columns; c += 16) {
          tmem_wait_st();
          uint32_t y[16];
          tmem_ld<16>(y, s_at + c);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const __half2 z = __hmul2(*reinterpret_cast<__half2 *>(&y[i]), by);
            y[i] = *reinterpret_cast<const uint32_t *>(&z);
          }
          tmem_st<16>(y, s_at + c);
        }
        tmem_wait_st();
      };
      // the largest value scale of the pages that this row sees
      const float *ks = ms.scale[stage][0], *vs = ms.scale[stage][1];
      float vmax = 0.f;
      if (mask) {
#pragma unroll
        for (int i = 0; i < kParts; ++i)
          if (pos + 16 * i < lim && ((there >> i) & 1)) vmax = fmaxf(vmax, vs[i]);   // (a NaN is not a larger one)
      } else {
#pragma unroll
        for (int i = 0; i < kParts; ++i) vmax = fmaxf(vmax, vs[i]);
      }
      // ---- 32 tokens at a time: weights, and between them the maximum of the next 32
      uint32_t buf[2][32];
      float2 sum = make_float2(0.f, 0.f);
      auto walk = [&](auto masked_) {
        constexpr bool kMasked = decltype(masked_)::value;
        if (kMasked) __syncwarp();
        uint32_t bits[2] = {~0u, ~0u};
        auto maximum = [&](int i) -> float {   // of columns 32 i .., which are loaded
          uint32_t *s = buf[i & 1];
          if (kMasked) {
            if (tail && i < 2) {   // what fp16 left of the keys
#pragma unroll
              for (int c = 0; c < 32; c += 16) {
                uint32_t rest[16];
                tmem_ld<16>(rest, s_at + 64 + 32 * i + c);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) s[c + e] = f32_bits(__uint_as_float(s[c + e]) + __uint_as_float(rest[e]));
              }
            }
            bits[i & 1] = seen(i);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!((bits[i & 1] >> e) & 1)) s[e] = 0xff800000u;   // -inf
          }
          float mx = -INFINITY;
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            float y = __uint_as_float(s[16 * part]), z = __uint_as_float(s[16 * part + 1]);
#pragma unroll
            for (int e = 2; e < 16; e += 4) {
              y = fmaxf(y, fmaxf(__uint_as_float(s[16 * part + e]), __uint_as_float(s[16 * part + e + 1])));
              if (e + 2 < 16) z = fmaxf(z, fmaxf(__uint_as_float(s[16 * part + e + 2]), __uint_as_float(s[16 * part + e + 3])));
            }
            mx = fmaxf(mx, fmaxf(y, z) * (cr * ks[2 * i + part]));
          }
          return mx;
        };
        tmem_ld<32>(buf[0], s_at);
        tmem_wait_ld();
        tmem_ld<32>(buf[1], s_at + 32);
        float mx = maximum(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t *s = buf[i & 1];
          const bool up = mx > m + 8.f;   // (also the first that is seen: the row's output and sum are zero then)
          const bool up_v = i == 0 && 2.f * vmax > vref;
          if (__any_sync(0xffffffffu, up || up_v)) {
            const float to = up ? ceilf(mx) : m, fix = up && m != -INFINITY ? ex2f(m - to) : 1.f;
            sum.x *= fix; sum.y *= fix; l *= fix;
            m = to;
            float fix_v = 1.f;
            if (up_v) {
              const uint32_t e = min((f32_bits(vmax) >> 23) + 2u, 252u);
              inv = __uint_as_float((254u - e) << 23);
              fix_v = vref * inv;
              vref = __uint_as_float(e << 23);
            }
            rescale(fix * fix_v, 16 * i);
          }
          const float off = kTop - (m == -INFINITY ? 0.f : m);
          uint32_t w[16];
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            const float f = cr * ks[2 * i + part], vv = vs[2 * i + part] * inv;
            if (part == 1 && i < 3) {
              if (kMasked) __syncwarp();
              tmem_wait_ld();
              mx = maximum(i + 1);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const int e = 16 * part + 2 * k;
              const float2 y = fma2(make_float2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), make_float2(f, f), make_float2(off, off));
              float2 q = make_float2(ex2f(y.x), ex2f(y.y)), z = mul2(q, make_float2(vv, vv));
              if (kMasked) {   // (nothing of a scale of NaN, nor of a score)
                if (!((bits[i & 1] >> e) & 1)) q.x = z.x = 0.f;
                if (!((bits[i & 1] >> (e + 1)) & 1)) q.y = z.y = 0.f;
              }
              sum = add2(sum, q);
              w[8 * part + k] = pack_f16(z.x, z.y);
            }
          }
          if (kMasked) __syncwarp();
          tmem_st<16>(w, s_at + 16 * i);
          if (i < 2) tmem_ld<32>(buf[i & 1], s_at + 32 * (i + 2));
        }
      };
      if (mask) walk(std::true_type());
      else walk(std::false_type());
      l += sum.x + sum.y;
      tmem_wait_st();
      fence_before();
      mbar_arrive(&ms.p_full[t]);
    }
    // ---- results
    if (mine > 0 && ok) ok = mbar_wait(&ms.o_full, 0);
    const bool good = __all_sync(0xffffffffu, ok);
    fence_after();
    int jr, again = r;
    int64_t row;
    asm volatile("" : "+r"(again));
    const bool real = place(again, jr, row);
    const float scale = l == 0.f ? 0.f : vref / l;   // (0: nothing seen)
    const bool slow = tail_tiles > 0 && ms.slow;     // (written before the last tile's barrier)
#pragma unroll 1
    for (int c = 0; c < LOCKS_D; c += 32) {
      uint32_t s[32];
      __syncwarp();   // (behind the stores, and the loop over what is not finite, of the columns before)
      if (mine > 0 && good) {
        tmem_ld<32>(s, o_at + c);
        tmem_wait_ld();
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i] = 0;
      }
      if (slow) {
        const float *vt = p.c.vt + p.c.tail_at(b, h, full_pages) + c;
#pragma unroll 1
        for (int k = 0; tail_pos + k < min(lim, last - tile0 * kTok); ++k)
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float y = vt[k * LOCKS_D + i];
            if (!(fabsf(y) < INFINITY)) s[i] = f32_bits(__uint_as_float(s[i]) + y);
          }
      }
      if (real && good && splits > 1) {
        float4 *part = reinterpret_cast<float4 *>(p.part + ((int64_t)blockIdx.x * kSoft + tid) * LOCKS_D + c);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          part[i] = make_float4(__uint_as_float(s[4 * i]) * scale, __uint_as_float(s[4 * i + 1]) * scale, __uint_as_float(s[4 * i + 2]) * scale, __uint_as_float(s[4 * i + 3]) * scale);
      } else if (real && good) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)   // (a row that has seen nothing is zero whatever lies in its output)
            y[e] = l == 0.f ? 0u : pack_bf16(__uint_as_float(s[8 * i + 2 * e]) * scale, __uint_as_float(s[8 * i + 2 * e + 1]) * scale);
          *reinterpret_cast<uint4 *>(p.out + row * LOCKS_D + c + 8 * i) = make_uint4(y[0], y[1], y[2], y[3]);
        }
      }
    }
    if (real && good) {
      const float lse2 = l == 0.f ? -INFINITY : (m == -INFINITY ? 0.f : m) - kTop + log2f(l);
      if (splits > 1) p.part_lse[blockIdx.x * kSoft + tid] = lse2;
      else if (p.lse) p.lse[row] = lse2 * kLn2;
    }
    fence_before();
  }
  if (!ok) set_status(p.status, LOCKS_ERR_TIMEOUT);
  __syncthreads();
  if (warp == 16) {
    __syncwarp();
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kTmemCols));
  }
}

// Joins the splits of 16 of a block's 256 rows, a warp a row, a lane four dims.
constexpr int kJoinRows = 16;
__global__ void __launch_bounds__(32 * kJoinRows) kvq_chunk_join_kernel(const __grid_constant__ ChunkParams p) {
  __shared__ int found[6];
  const int lane = threadIdx.x & 31, h = blockIdx.y, G = p.G, cta_tokens = 2 * p.tile_tokens;
  pdl_trigger();
  pdl_wait();
  const int block = blockIdx.x / (kSoft / kJoinRows), r = blockIdx.x % (kSoft / kJoinRows) * kJoinRows + (threadIdx.x >> 5);
  const Block at = find_block(p, block, 0, found);
  const int of_half = r % kRows, jr = r / kRows * p.tile_tokens + of_half / G, splits = at.splits;
  if (at.b < 0 || splits == 1 || of_half >= p.tile_tokens * G || jr >= min(cta_tokens, at.n - at.j0)) return;
  const int64_t first = ((int64_t)block * p.c.Hkv + h) * splits, row = (int64_t)(at.row0 + jr) * p.Hq + h * G + of_half % G;
  float m = -INFINITY;
  for (int s = lane; s < splits; s += 32) m = fmaxf(m, p.part_lse[(first + s) * kSoft + r]);
  m = warp_max(m);
  const float ms = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    const float w = ex2f(p.part_lse[(first + s) * kSoft + r] - ms);
    if (w == 0.f) continue;   // (nothing seen)
    const float4 y = *reinterpret_cast<const float4 *>(p.part + ((first + s) * kSoft + r) * LOCKS_D + 4 * lane);
    sum += w;
    o.x = fmaf(w, y.x, o.x); o.y = fmaf(w, y.y, o.y); o.z = fmaf(w, y.z, o.z); o.w = fmaf(w, y.w, o.w);
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  *reinterpret_cast<uint2 *>(p.out + row * LOCKS_D + 4 * lane) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
  if (lane == 0 && p.lse) p.lse[row] = sum == 0.f ? -INFINITY : (ms + log2f(sum)) * kLn2;
}

}  // namespace

// Blocks of 256 rows that `n` tokens of `batch` requests may make, per KV head: most when all requests but one have a single token
static int64_t chunk_blocks(const locks_ctx *c, int n, int batch) {
  const int tokens = 2 * (kRows / c->G);
  return n <= batch ? n : (n - batch) / tokens + batch;
}

int locks_launch_kvq_chunk(locks_ctx *c, const void *q, const int32_t *cu, int n, const locks_kvq *kv, int batch, void *out, float *lse, cudaStream_t st) {
  ChunkParams p = {};
  p.q = reinterpret_cast<const __nv_bfloat16 *>(q); p.cu = cu; p.c = kvq_cache(c, kv);
  p.out = reinterpret_cast<__nv_bfloat16 *>(out); p.lse = lse; p.status = c->status;
  p.n = n; p.batch = batch; p.Hq = c->cfg.num_q_heads; p.G = c->G;
  p.tile_tokens = kRows / c->G;
  p.log_b = c->B == 64 ? 6 : (c->B == 32 ? 5 : 4);
  p.c2 = c->cfg.sm_scale * kLog2e;
  // Few blocks: the tokens that each sees are split, so that every SM has a share (not where rows, unless they are padding, leave no two
  // slots for each block)
  const int64_t blocks = chunk_blocks(c, n, batch), ctas = blocks * c->cfg.num_kv_heads;
  const int slots = std::min(c->num_sms, KVQ_CHUNK_SLOTS), joined = slots / (2 * c->cfg.num_kv_heads);   // at most so many blocks are split
  p.slots = ((int64_t)n + 2 * p.tile_tokens - 1) / (2 * p.tile_tokens) <= joined ? slots : 0;
  p.part = c->kvq_part; p.part_lse = reinterpret_cast<float *>(c->kvq_ml);
  const int64_t grid = std::max<int64_t>(ctas, p.slots);   // (no slot without a CTA)
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
  const int rc = locks_check_launch(c);
  if (rc != LOCKS_OK || !p.slots) return rc;
  const dim3 rows((unsigned)std::min<int64_t>(blocks, joined) * (kSoft / kJoinRows), c->cfg.num_kv_heads);
  locks_launch_pdl(kvq_chunk_join_kernel, rows, dim3(32 * kJoinRows), 0, st, p);
  return locks_check_launch(c);
}
