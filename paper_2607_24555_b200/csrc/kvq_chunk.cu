// Attention over the 8-bit paged cache for chunks of prompts: many query rows per KV head (kvq_attend.cu has the formula, and the form
// for few rows).
//
// A CTA takes 128 rows, the G heads of 128 / G consecutive tokens of one request, and walks the tokens that they see in tiles of 64:
// codes come by 16-byte asynchronous copies two tiles ahead, all threads turn a tile into fp16 in shared memory (exactly: numbers up
// to 127 or e4m3 numbers; once for 128 rows), and each warp multiplies its 32 rows by 32 tokens at a time, keeping scores and outputs in
// registers; weights pass from the first product to the second in registers.  Two CTAs share an SM, so that one converts while the
// other multiplies.  Key scales are factors of the scores; a page's value scale goes into its weights, relative to a running power
// of two that is at least the largest value scale so far (weights are 2^15 p times at most 1: normal in fp16 down to 2^-29).
// Bound by the m16n8k16 instruction, of which an SM retires one in two cycles (580 TFLOP/s), and by the shared-memory reads that
// feed it, 97 bytes a cycle of 128.
#include "kvq.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMt = 1, kWarps = 8, kThreads = 32 * kWarps, kRows = 16 * kMt * kWarps, kTok = 64;   // kMt: 16-row tiles of a warp
// shared memory: queries [128][256 bytes]; K and V tiles in fp16 [64][256 bytes] each; two raw tiles (K, V: [64][128 bytes] each)
constexpr int kQBytes = kRows * 256, kHalfTile = kTok * 256, kRawTile = 2 * kTok * 128;
constexpr int kOffK = kQBytes, kOffV = kOffK + kHalfTile, kOffRaw = kOffV + kHalfTile, kOffMisc = kOffRaw + 2 * kRawTile;
constexpr int kSmem = kOffMisc + 256;   // scales of two raw tiles' four 16-token parts (K, V), reductions

struct ChunkParams {
  const __nv_bfloat16 *q;
  const int32_t *cu;
  KvqCache c;
  __nv_bfloat16 *out;
  float *lse;
  int32_t *status;
  int n, batch, Hq, G, tile_tokens;
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
__device__ __forceinline__ void copy16(void *dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
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
// 16-byte piece `piece` of row `row` of an fp16 tile (rows of 256 bytes): pieces change places with the row, so that eight rows' pieces
// of one ldmatrix lie in different banks
__device__ __forceinline__ uint32_t at256(int row, int piece) { return row * 256 + ((piece ^ (row & 7)) << 4); }

template <int FMT>
__global__ void __launch_bounds__(kThreads, 2) kvq_chunk_kernel(const __grid_constant__ ChunkParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];   // (rows of 256 bytes begin at multiples of 256: pieces change by exclusive or)
  float *scale_s = reinterpret_cast<float *>(smem + kOffMisc);       // [2 raw tiles][K, V][4 parts] and what is there: [2][4] ints behind
  int *kind_s = reinterpret_cast<int *>(smem + kOffMisc + 64);       // [2][4]: 0 nothing, 1 codes
  float *red_s = reinterpret_cast<float *>(smem + kOffMisc + 128);   // [2][kWarps]
  int *found_s = reinterpret_cast<int *>(smem + kOffMisc + 192);     // [4]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, x = lane >> 2, t = lane & 3;
  const int Hkv = p.c.Hkv, h = blockIdx.x % Hkv, B = p.c.B;
  pdl_trigger();
  pdl_wait();
  // ---- the row tile of this CTA: requests' tiles counted from the last one on, so that the ones that see most start first
  if (tid == 0) found_s[0] = -1;
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
      if (at >= 0 && at < tiles) { found_s[0] = b0 + lane; found_s[1] = tiles - 1 - at; found_s[2] = row0; found_s[3] = n; }
      before += __shfl_sync(0xffffffffu, end, 31);
    }
  }
  __syncthreads();
  const int b = found_s[0];
  if (b < 0) return;
  const int j0 = found_s[1] * p.tile_tokens, row0 = found_s[2] + j0, n = found_s[3];
  const int toks = min(p.tile_tokens, n - j0), rows = toks * p.G;
  int T = max(p.c.seq_lens[b], 0);
  const int seen0 = T - n + j0 + 1;      // tokens that the tile's first token sees
  const int full_pages = T / B;
  if ((T - 1) / B >= p.c.Pmax && T > 0 && tid == 0) set_status(p.status, LOCKS_ERR_BAD_BLOCK);
  const int last = min(min(seen0 + toks - 1, T), p.c.Pmax * B);   // tokens that the tile's last token sees
  const int codes_end = min(min(last, full_pages * B), p.c.Pmax * B);   // of them, those in codes
  const int tiles = last > 0 ? (codes_end + kTok - 1) / kTok : 0;

  // ---- queries: fp16 times a power of two, two threads a row (64 dims each)
  float c_row;   // what undoes it, times sm_scale log2 e
  {
    const int qr = tid >> 1, i0 = 8 * (tid & 1), j = qr / p.G, g = qr - j * p.G;
    const uint4 *src = reinterpret_cast<const uint4 *>(p.q + ((int64_t)(row0 + j) * p.Hq + h * p.G + g) * LOCKS_D);
    float amax = 0.f;
    if (qr < rows) {
#pragma unroll
      for (int i = i0; i < i0 + 8; ++i) {
        const uint4 w = src[i];
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) amax = fmaxf(amax, fmaxf(finite_abs(__uint_as_float(u[e] << 16)), finite_abs(__uint_as_float(u[e] & 0xFFFF0000u))));
      }
    }
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    const float up = power_to(amax, 0);
    c_row = p.c2 / up;
#pragma unroll
    for (int i = i0; i < i0 + 8; ++i) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (qr < rows) w = src[i];
      uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] = pack_f16(__uint_as_float(u[e] << 16) * up, __uint_as_float(u[e] & 0xFFFF0000u) * up);
      *reinterpret_cast<uint4 *>(smem + at256(qr, i)) = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
  // rows of this lane: 16 kMt warp + 16 mt + x + 8 c; lane 2 r of a warp has row r's factor
  float cr[kMt][2];
  int lim[kMt][2];
#pragma unroll
  for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = 16 * mt + x + 8 * c;
      cr[mt][c] = __shfl_sync(0xffffffffu, c_row, 2 * r);
      lim[mt][c] = 16 * kMt * warp + r < rows ? seen0 + (16 * kMt * warp + r) / p.G : last;
    }

  // ---- raw tiles: 16-byte copies, and the scales of the four 16-token parts; block ids are fetched a tile ahead of them
  int blk[2];
  auto blocks = [&](int tile) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int pos = tile * kTok + 16 * ((tid >> 7) + 2 * i);
      blk[i] = pos < codes_end ? p.c.block_table[(int64_t)b * p.c.Pmax + pos / B] : -1;
    }
  };
  auto issue = [&](int tile, int stage) {
    uint8_t *raw = smem + kOffRaw + stage * kRawTile;
    if (tile < tiles) {
      // a thread's copies: piece tid & 7 of token (tid >> 3) % 16 of parts (tid >> 7) + 2 i
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int i = (tid >> 7) + 2 * k, pos = tile * kTok + 16 * i, block = blk[k];
        const bool good = block >= 0 && block < p.c.num_blocks;
        const int tok = (tid >> 3) & 15;
        if (!good && pos < codes_end && (tid & 127) == 0) set_status(p.status, LOCKS_ERR_BAD_BLOCK);
        uint8_t *dk = raw + (16 * i + tok) * 128 + (tid & 7) * 16;
        if (good) {
          const int64_t off = (int64_t)block * p.c.sb + (int64_t)h * p.c.sh + (int64_t)(pos % B + tok) * p.c.st + (tid & 7) * 16;
          copy16(dk, p.c.k + off);
          copy16(dk + kRawTile / 2, p.c.v + off);
        }
        if ((tid & 127) == 0) {
          kind_s[4 * stage + i] = good;
          scale_s[8 * stage + i] = good ? p.c.ks[(int64_t)block * Hkv + h] : 0.f;
          scale_s[8 * stage + 4 + i] = good ? p.c.vs[(int64_t)block * Hkv + h] : 0.f;
        }
      }
      blocks(tile + 1);
    }
    cp_async_commit();
  };

  float o[kMt][16][4];   // rows as above (c0 c1: row x, c2 c3: row x + 8), dims 8 nt + 2 t, + 1
  float m[kMt][2], l[kMt][2];
  float vref = 0x1p-126f;   // a power of two, at least the largest value scale so far
#pragma unroll
  for (int mt = 0; mt < kMt; ++mt) {
#pragma unroll
    for (int nt = 0; nt < 16; ++nt) o[mt][nt][0] = o[mt][nt][1] = o[mt][nt][2] = o[mt][nt][3] = 0.f;
    m[mt][0] = m[mt][1] = -INFINITY;
    l[mt][0] = l[mt][1] = 0.f;
  }
  auto raise_vref = [&](float vs) {   // (no part has a larger scale; a NaN is not a larger one)
    if (vs > vref) {
      const float to = __uint_as_float(min(((__float_as_uint(vs) >> 23) & 255u) + 1u, 254u) << 23), f = vref / to;
      vref = to;
#pragma unroll
      for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
        for (int nt = 0; nt < 16; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[mt][nt][e] *= f;
    }
  };
  // Scores (times f0, f1 for the two 16-token parts, in place) -> weights times the parts' value scales; a masked score is -inf already
  auto weigh = [&](float (&s)[kMt][4][4], float ks0, float ks1, float vs0, float vs1, bool masked) {
#pragma unroll
    for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float f0 = cr[mt][c] * ks0, f1 = cr[mt][c] * ks1;
        float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          m0 = fmaxf(m0, fmaxf(s[mt][nt][2 * c], s[mt][nt][2 * c + 1]));
          m1 = fmaxf(m1, fmaxf(s[mt][nt + 2][2 * c], s[mt][nt + 2][2 * c + 1]));
        }
        float mx = fmaxf(m0 * f0, m1 * f1);
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        const float mn = fmaxf(m[mt][c], mx), ms = mn == -INFINITY ? 0.f : mn;
        if (__any_sync(0xffffffffu, mn != m[mt][c])) {
          const float a = ex2f(m[mt][c] - ms);
          l[mt][c] *= a;
#pragma unroll
          for (int nt = 0; nt < 16; ++nt) { o[mt][nt][2 * c] *= a; o[mt][nt][2 * c + 1] *= a; }
        }
        m[mt][c] = mn;
        const float2 off = make_float2(15.f - ms, 15.f - ms);
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int nt = 0; nt < 4; ++nt) {
          const float f = nt < 2 ? f0 : f1, v = nt < 2 ? vs0 : vs1;
          const float2 y = fma2(make_float2(s[mt][nt][2 * c], s[mt][nt][2 * c + 1]), make_float2(f, f), off);
          const float2 q = make_float2(ex2f(y.x), ex2f(y.y));
          sum = add2(sum, q);
          float2 w = mul2(q, make_float2(v, v));
          if (masked) {   // (nothing of a scale of NaN)
            if (s[mt][nt][2 * c] == -INFINITY) w.x = 0.f;
            if (s[mt][nt][2 * c + 1] == -INFINITY) w.y = 0.f;
          }
          s[mt][nt][2 * c] = w.x;
          s[mt][nt][2 * c + 1] = w.y;
        }
        l[mt][c] += sum.x + sum.y;
      }
  };
  // ldmatrix addresses of this lane for piece 0 of the first row: rows are 256 bytes apart, pieces change by exclusive or
  const uint32_t q_addr = smem_u32(smem) + at256(16 * kMt * warp + (lane & 15), lane >> 4);
  // K rows are the columns of the second operand: matrices (tokens 0 .. 7, dims 0 .. 7), (0 .. 7, 8 .. 15), (8 .. 15, 0 .. 7), (8 .. 15, 8 .. 15)
  const uint32_t k_addr = smem_u32(smem) + kOffK + at256((lane & 7) + 8 * (lane >> 4), (lane >> 3) & 1);
  // 16 tokens by 16 dims of V, transposed: matrices (tokens 0 .. 7, dims 0 .. 7), (8 .. 15, 0 .. 7), (0 .. 7, 8 .. 15), (8 .. 15, 8 .. 15)
  const uint32_t v_addr = smem_u32(smem) + kOffV + at256(lane & 15, lane >> 4);
  // 32 tokens from row k0 of the K and V tiles on; their places start at pos.  ks, vs: of their two 16-token parts (vs relative to
  // vref), ok0, ok1: whether they are there.  tail: the K tile's rows k0 + 32 .. hold what fp16 left of the keys in rows k0 ..; slow:
  // values are taken from vt (fp32)
  auto step = [&](int k0, int pos, float ks0, float ks1, float vs0, float vs1, bool ok0, bool ok1, bool tail, bool slow, const float *vt) {
    float s[kMt][4][4];
#pragma unroll
    for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) s[mt][nt][0] = s[mt][nt][1] = s[mt][nt][2] = s[mt][nt][3] = 0.f;
    uint32_t k_row = k_addr + k0 * 256;
#pragma unroll 1
    for (int part = 0; part < (tail ? 2 : 1); ++part, k_row += 32 * 256) {
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        uint32_t a[kMt][4], kf[2][4];
#pragma unroll
        for (int mt = 0; mt < kMt; ++mt) ldsm4(a[mt], (q_addr ^ (32 * ks)) + 4096 * mt);
#pragma unroll
        for (int g = 0; g < 2; ++g) ldsm4(kf[g], (k_row ^ (32 * ks)) + 4096 * g);
#pragma unroll
        for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
          for (int nt = 0; nt < 4; ++nt) mma_f16(s[mt][nt], a[mt][0], a[mt][1], a[mt][2], a[mt][3], kf[nt >> 1][2 * (nt & 1)], kf[nt >> 1][2 * (nt & 1) + 1]);
      }
    }
    if (pos + 32 > seen0 || !(ok0 && ok1)) {   // some row does not see all of them
#pragma unroll
      for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
        for (int nt = 0; nt < 4; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool sees = pos + 8 * nt + 2 * t + (e & 1) < lim[mt][e >> 1] && (nt < 2 ? ok0 : ok1);
            s[mt][nt][e] = sees ? s[mt][nt][e] * (nt < 2 ? ks0 : ks1) : -INFINITY;
          }
      weigh(s, 1.f, 1.f, vs0, vs1, true);
    } else {
      weigh(s, ks0, ks1, vs0, vs1, false);
    }
    uint32_t pf[kMt][4][2];   // weights as A fragments: [rows][8 tokens][row x, x + 8]
#pragma unroll
    for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) { pf[mt][nt][0] = pack_f16(s[mt][nt][0], s[mt][nt][1]); pf[mt][nt][1] = pack_f16(s[mt][nt][2], s[mt][nt][3]); }
    if (!slow) {
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          uint32_t vf[4];
          ldsm4_trans(vf, ((v_addr + k0 * 256) ^ (32 * d)) + 4096 * g);
#pragma unroll
          for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              mma_f16(o[mt][2 * d + e], pf[mt][2 * g][0], pf[mt][2 * g][1], pf[mt][2 * g + 1][0], pf[mt][2 * g + 1][1], vf[2 * e], vf[2 * e + 1]);
        }
    } else {   // values that are not finite: token by token in fp32, so that a row takes nothing of a token that it does not see
#pragma unroll 1
      for (int k = 0; k < 32 && pos + k < T; ++k) {
#pragma unroll
        for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float mine = 0.f;
#pragma unroll
            for (int nt = 0; nt < 4; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if ((k >> 3) == nt && (k & 1) == e) mine = s[mt][nt][2 * c + e];
            const float y = __shfl_sync(0xffffffffu, mine, (lane & ~3) + ((k & 7) >> 1));
            if (pos + k < lim[mt][c]) {
#pragma unroll
              for (int nt = 0; nt < 16; ++nt) {
                const float2 v = *reinterpret_cast<const float2 *>(vt + (int64_t)k * LOCKS_D + 8 * nt + 2 * t);
                o[mt][nt][2 * c] = fmaf(y, v.x, o[mt][nt][2 * c]);
                o[mt][nt][2 * c + 1] = fmaf(y, v.y, o[mt][nt][2 * c + 1]);
              }
            }
          }
      }
    }
  };

  // ---- tiles of codes, then the unfinished page, 32 tokens at a time
  const int tail_end = min(last, T), tail_tiles = full_pages < p.c.Pmax && tail_end > full_pages * B ? (tail_end - full_pages * B + 31) / 32 : 0;
  blocks(0);
  issue(0, 0);
#pragma unroll 1
  for (int tile = 0; tile < tiles + tail_tiles; ++tile) {
    const int stage = tile & 1;
    const bool tail = tile >= tiles;
    float4 ks, vs;
    int4 kind;
    int pos = tile * kTok;
    bool slow = false;
    const float *vt = nullptr;
    if (!tail) {
      issue(tile + 1, stage ^ 1);
      cp_async_wait<1>();
      __syncthreads();   // the tile's bytes and scales are there; the last tile's fp16 form is used
      const uint8_t *raw = smem + kOffRaw + stage * kRawTile;
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // 16 codes: piece tid & 7 of row (tid >> 3) + 32 (i % 2), of K for i < 2, then of V
        const int row = (tid >> 3) + 32 * (i & 1), piece = tid & 7;
        const bool key = i < 2;
        uint4 y = *reinterpret_cast<const uint4 *>(raw + (key ? 0 : kRawTile / 2) + row * 128 + piece * 16);
        if (!kind_s[4 * stage + (row >> 4)]) y = make_uint4(0, 0, 0, 0);
        const uint32_t word[4] = {y.x, y.y, y.z, y.w};
        uint32_t f[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) kvq_halves<FMT>(kvq_flip<FMT>(word[e]), f[2 * e], f[2 * e + 1]);
        uint8_t *dst = smem + (key ? kOffK : kOffV);
        *reinterpret_cast<uint4 *>(dst + at256(row, 2 * piece)) = make_uint4(f[0], f[1], f[2], f[3]);
        *reinterpret_cast<uint4 *>(dst + at256(row, 2 * piece + 1)) = make_uint4(f[4], f[5], f[6], f[7]);
      }
      ks = *reinterpret_cast<const float4 *>(scale_s + 8 * stage);
      vs = *reinterpret_cast<const float4 *>(scale_s + 8 * stage + 4);
      kind = *reinterpret_cast<const int4 *>(kind_s + 4 * stage);
      __syncthreads();
    } else {
      // a thread: 16 dims of one token, as fp16 times a power of two of the 32 tokens' largest; keys in two parts (22 bits)
      pos = full_pages * B + 32 * (tile - tiles);
      const int tok = tid >> 3, d0 = 16 * (tid & 7);
      const int64_t at = (((int64_t)b * Hkv + h) * B + pos - full_pages * B) * LOCKS_D;
      vt = p.c.vt + at;
      const float *src[2] = {p.c.kt + at + tok * LOCKS_D + d0, vt + tok * LOCKS_D + d0};
      float amax[2] = {0.f, 0.f}, up[2];
      bool odd = false;
      if (pos + tok < T) {
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll 4
          for (int i = 0; i < 16; ++i) {
            const float y = src[kv][i];
            amax[kv] = fmaxf(amax[kv], finite_abs(y));
            if (kv == 1) odd |= !(fabsf(y) < INFINITY);
          }
      }
      __syncthreads();   // the last tile's fp16 form and the last reductions are used
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const float y = warp_max(amax[kv]);
        if (lane == 0) red_s[kWarps * kv + warp] = y;
      }
      slow = __syncthreads_or(odd);
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        float y = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) y = fmaxf(y, red_s[kWarps * kv + w]);
        up[kv] = power_to(y, 14);
      }
#pragma unroll 1
      for (int i = 0; i < 2; ++i) {
        uint32_t k_hi[4], k_lo[4], v_hi[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float2 y = make_float2(0.f, 0.f), z = y;
          if (pos + tok < T) { y = *reinterpret_cast<const float2 *>(src[0] + 8 * i + 2 * e); z = *reinterpret_cast<const float2 *>(src[1] + 8 * i + 2 * e); }
          y.x *= up[0]; y.y *= up[0];
          k_hi[e] = pack_f16(y.x, y.y);
          const float2 r = __half22float2(*reinterpret_cast<__half2 *>(&k_hi[e]));
          k_lo[e] = pack_f16(fabsf(y.x) < INFINITY ? y.x - r.x : 0.f, fabsf(y.y) < INFINITY ? y.y - r.y : 0.f);
          v_hi[e] = pack_f16(z.x * up[1], z.y * up[1]);
        }
        const int piece = d0 / 8 + i;
        *reinterpret_cast<uint4 *>(smem + kOffK + at256(tok, piece)) = make_uint4(k_hi[0], k_hi[1], k_hi[2], k_hi[3]);
        *reinterpret_cast<uint4 *>(smem + kOffK + at256(tok + 32, piece)) = make_uint4(k_lo[0], k_lo[1], k_lo[2], k_lo[3]);
        *reinterpret_cast<uint4 *>(smem + kOffV + at256(tok, piece)) = make_uint4(v_hi[0], v_hi[1], v_hi[2], v_hi[3]);
      }
      ks = make_float4(1.f / up[0], 1.f / up[0], 0.f, 0.f);
      const float v1 = slow ? 1.f : 1.f / up[1];
      vs = make_float4(v1, v1, 0.f, 0.f);
      kind = make_int4(1, 1, 0, 0);
      __syncthreads();
    }
    raise_vref(fmaxf(fmaxf(vs.x, vs.y), fmaxf(vs.z, vs.w)));
    const float inv = 1.f / vref;
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
      const bool ok0 = half ? kind.z : kind.x, ok1 = half ? kind.w : kind.y;
      if (!(ok0 || ok1) || pos + 32 * half >= last) continue;
      step(32 * half, pos + 32 * half, half ? ks.z : ks.x, half ? ks.w : ks.y, (half ? vs.z : vs.x) * inv, (half ? vs.w : vs.y) * inv, ok0, ok1, tail, slow, vt);
    }
  }
  cp_async_wait<0>();
  // ---- results
#pragma unroll
  for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float sum = l[mt][c];
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      const int r = 16 * kMt * warp + 16 * mt + x + 8 * c;
      if (r >= rows) continue;
      const int j = r / p.G, g = r - j * p.G;
      const int64_t row = (int64_t)(row0 + j) * p.Hq + h * p.G + g;
      const float f = sum == 0.f ? 0.f : vref / sum;   // (0: nothing seen)
      uint32_t *dst = reinterpret_cast<uint32_t *>(p.out + row * LOCKS_D + 2 * t);
#pragma unroll
      for (int nt = 0; nt < 16; ++nt) dst[4 * nt] = pack_bf16(o[mt][nt][2 * c] * f, o[mt][nt][2 * c + 1] * f);
      if (p.lse && t == 0) p.lse[row] = sum == 0.f ? -INFINITY : ((m[mt][c] == -INFINITY ? 0.f : m[mt][c]) - 15.f + log2f(sum)) * kLn2;
    }
}

}  // namespace

int locks_launch_kvq_chunk(locks_ctx *c, const void *q, const int32_t *cu, int n, const locks_kvq *kv, int batch, void *out, float *lse, cudaStream_t st) {
  ChunkParams p = {};
  p.q = reinterpret_cast<const __nv_bfloat16 *>(q); p.cu = cu; p.c = kvq_cache(c, kv);
  p.out = reinterpret_cast<__nv_bfloat16 *>(out); p.lse = lse; p.status = c->status;
  p.n = n; p.batch = batch; p.Hq = c->cfg.num_q_heads; p.G = c->G;
  p.tile_tokens = kRows / c->G;
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
