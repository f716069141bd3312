// Attention over the 8-bit paged cache, for single tokens and a few tokens per request:
//   o_r = sum_i softmax_i(q_r . k_i s_k(i) sm_scale) v_i s_v(i)   over the tokens i that row r sees.
//
// Codes are numbers that fp16 holds exactly, so both products run on the tensor cores in fp16.  A query row goes in times a power of
// two that brings its largest element to 1 .. 2 (undone on the scores in fp32; elements down to 2^-17 of the largest go in exactly, smaller
// ones within 2^-25 of it, which is where fp16 ends), a page's key scale is a factor of its
// scores, and P V of 16 tokens joins the fp32 output by one rounding multiply-add with the page's value scale, so that no scale meets
// fp16's range.  Weights go in as 2^15 p in fp16 (within 2^-11 of each, and normal down to p = 2^-29); the sum that divides is that of
// the unrounded ones.  Scores, maxima, sums and outputs are fp32.
//
// Signed codes: byte u = code + 128 (its sign bit flipped) with a zero byte above it is the fp16 number 2^-24 u, without any
// arithmetic.  So the products are those of u, and what 128 adds to them, 128 sum_d q_d and 128 sum_i p_i, is taken off by the
// accumulators' start: the first is known once per row, the second is one more MMA, with ones for values.  (As differences of
// numbers 1024 + u and 1152 the conversions were 176 of a tile's 500 instructions; 8 x 32K tokens took 116 us.)
//
// A problem is a (request, KV head, row tile): up to 8 or 16 query rows, the G heads of one or several tokens.  The pairs of 16-token tiles
// of all problems form one line that is cut into equal shares, one per CTA, whatever the lengths: a CTA's share is a few segments of
// problems, and a problem that several CTAs share is put together by the last of them, or by a second kernel where they are many.
// A warp streams every fourth pair of a segment through a ring in shared memory and reads it as MMA fragments: the order of
// dimensions in q k and of tokens and dimensions in p v is free, and is chosen such that a lane's bytes are 16-byte pieces of rows.
// Measured, 32 query heads: 8 x 32K tokens over 8 KV heads 94 to 98 us (5.5 TB/s, 0.84 of a copy's bandwidth, which bounds it); one
// request of 1M tokens over 2 KV heads 114 when the chip is busy all the time (0.72; 101 in short runs; signed codes 119: the issue of
// conversions and products for 16 rows); 2048 listed tokens of 8 requests 21, of which 5 are bytes: the chain page id, block, scale,
// codes, and the join (attention over the same pages of a 16-bit cache: 15 to 19 in one graph, so 8 bits save memory there, not time).
#include <algorithm>

#include "kvq.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kRowPad = LOCKS_D + 4;   // floats of a row of a warp's partial
constexpr int kUnfinished = -2;        // in a block's place: the unfinished page
constexpr int kMostLead = 24;          // pairs that a problem's start costs a CTA that has another one's end before it
constexpr int kTailPairs = 5;           // pairs that a warp reads while another works on an unfinished page (2 to 5 alike; chat traffic 59.5 to 56.6 us)
constexpr int kMinShare = kWarps;      // places of a share at least: a pair per warp
constexpr int kJoinWarps = 8;
constexpr int kManyShares = 16;        // CTAs per problem from which on the partials are put together by a second kernel

struct QAttParams {
  const __nv_bfloat16 *q;
  const int32_t *cu;
  KvqCache c;
  const int32_t *ids, *cnt;
  __nv_bfloat16 *out;
  float *lse;
  float *part;       // [2 CTAs][KVQ_ROWS][128]: CTA c leaves the problem that it goes on with in 2 c, the one that it begins in 2 c + 1
  float2 *part_ml;   // [2 CTAs][KVQ_ROWS] running max, sum
  int32_t *done;     // [CTAs] partials of the problem that CTA c begins (zero between launches)
  int32_t *status;
  int n, batch, Hq, Hkv, G, kvdiv, kbud, sub_shift;   // sub_shift: a page is 2^sub_shift tiles of 16 tokens
  int tile_tokens;   // tokens of a row tile
  float c2;          // sm_scale log2 e
};

__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(*reinterpret_cast<unsigned long long *>(&d))
      : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)),
        "l"(*reinterpret_cast<unsigned long long *>(&c)));
  return d;
}
// (No cache hint: an instance of the hinted form in this file's tile loop raised "illegal instruction" on sm_100a.)
__device__ __forceinline__ void copy16(void *dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

// One request's part of the line: its length, tokens, first row, pairs of tiles of a problem, row tiles (problems: times KV heads)
struct Request { int T, n, row0, pairs, row_tiles; };

__device__ __forceinline__ Request request_at(const QAttParams &p, int b) {
  Request r;
  r.row0 = b;
  r.n = 1;
  r.T = max(p.c.seq_lens[b], 0);   // (a length below zero: an empty sequence)
  if (p.cu) {
    r.row0 = p.cu[b];
    r.n = p.cu[b + 1] - r.row0;
    if (r.n < 0 || r.row0 < 0 || r.row0 > p.n - r.n) {   // rows that are not there
      set_status(p.status, LOCKS_ERR_BAD_BLOCK);
      r.n = 0;
    }
  }
  if (p.ids) {
    r.pairs = ((p.kbud << p.sub_shift) + 1) >> 1;
  } else {
    int pages = r.T > 0 ? (r.T - 1) / p.c.B + 1 : 0;
    if (pages > p.c.Pmax) { set_status(p.status, LOCKS_ERR_BAD_BLOCK); pages = p.c.Pmax; }
    r.pairs = max(((pages << p.sub_shift) + 1) >> 1, 1);   // (an empty sequence's problem writes its zeros all the same)
  }
  r.row_tiles = (r.n + p.tile_tokens - 1) / p.tile_tokens;
  return r;
}

// 32 requests, a lane each: where their places end within the 32; the warp's total in lane 31
__device__ __forceinline__ int scan_places(int mine, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, mine, o);
    if (lane >= o) mine += x;
  }
  return mine;
}

// The line as a warp knows it: the first 32 requests (most batches: all), its length and the CTAs' share of it.  (The host sees to it
// that the length fits 32 bits; all: 0 where the offsets are such that it does not.)  A problem's pairs come after `lead` places that stand for what its start costs: its queries, first
// blocks and tiles, and joining its warps' partials take a CTA some 10 us, as long as 24 pairs do.  Without them a CTA with two
// problems in its share ends that much later (24 requests of 211 .. 9001 tokens, 8 heads: 76 us; 6 places 66, 24 places 51).  A quarter of
// the share at most: where shares are short every CTA has a start of its own, and places without work would leave CTAs idle.
struct Line {
  Request r;                   // lane: request
  int end, all, lead, share;   // end: of the lane's request's places
  __device__ __forceinline__ int places(const QAttParams &p, const Request &x) const { return (lead + x.pairs) * x.row_tiles * p.Hkv; }
  __device__ __forceinline__ void read(const QAttParams &p, int lane, int ctas) {
    r = Request{0, 0, 0, 0, 0};
    if (lane < p.batch) r = request_at(p, lane);
    int pairs = __reduce_add_sync(0xffffffffu, r.pairs * r.row_tiles);
    const uint32_t most = (uint32_t)p.batch + (uint32_t)p.n;   // row tiles at most, which the host has counted with
    uint32_t problems = __reduce_add_sync(0xffffffffu, (uint32_t)r.row_tiles);
    for (int b0 = 32; b0 < p.batch && problems <= most; b0 += 32) {
      Request x = {0, 0, 0, 0, 0};
      if (b0 + lane < p.batch) x = request_at(p, b0 + lane);
      pairs += __reduce_add_sync(0xffffffffu, x.pairs * x.row_tiles);
      problems += __reduce_add_sync(0xffffffffu, (uint32_t)x.row_tiles);
    }
    if (problems > most) {   // offsets that do not ascend give rows to several requests: a longer line than 32 bits may hold
      set_status(p.status, LOCKS_ERR_BAD_BLOCK);
      pairs = problems = 0;
    }
    lead = min(pairs * p.Hkv / (4 * ctas), kMostLead);
    all = (pairs + lead * (int)problems) * p.Hkv;
    share = max((all - 1) / ctas + 1, kMinShare);
    end = scan_places(places(p, r), lane);
  }
  // The request that holds place u (below `all`), and where its places begin
  __device__ __forceinline__ void find(const QAttParams &p, int u, int lane, int &b, int &begin, Request &req) const {
    Request x = r;
    int to = end, at = to - places(p, x);
    uint32_t has = __ballot_sync(0xffffffffu, u >= at && u < to);
    b = 0;
    while (!has && b + 32 < p.batch) {
      const int before = __shfl_sync(0xffffffffu, to, 31);
      b += 32;
      x = Request{0, 0, 0, 0, 0};
      if (b + lane < p.batch) x = request_at(p, b + lane);
      to = before + scan_places(places(p, x), lane);
      at = to - places(p, x);
      has = __ballot_sync(0xffffffffu, u >= at && u < to);
    }
    const int l = has ? __ffs(has) - 1 : 0;
    b += l;
    begin = __shfl_sync(0xffffffffu, at, l);
    req.T = __shfl_sync(0xffffffffu, x.T, l); req.n = __shfl_sync(0xffffffffu, x.n, l); req.row0 = __shfl_sync(0xffffffffu, x.row0, l);
    req.pairs = __shfl_sync(0xffffffffu, x.pairs, l); req.row_tiles = __shfl_sync(0xffffffffu, x.row_tiles, l);
  }
};
// Outputs are kept times 2^15 (of the weights) and this: the unit of signed codes' fp16 form; for e4m3, so that large scales stay in range
template <int FMT> constexpr float kUnit = FMT == LOCKS_KVQ_INT ? 0x1p-24f : 0x1p-15f;

// largest finite magnitude over a warp -> the power of two that brings it to 2^top .. 2^(top + 1)
__device__ __forceinline__ float power_to(float amax, int top) {
  const int e = (int)(__float_as_uint(amax) >> 23) - 127;
  return amax < 1e-30f ? 1.f : __uint_as_float((uint32_t)(min(max(top - e, -126), 127) + 127) << 23);
}
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}

// The row tile's queries as B fragments: lane (x, t) holds four dims of row x (+ 8) per step, 64 (s / 4) + 16 t + 4 (s % 4) ..
// Of rows 2 t, 2 t + 1 (+ 8), rs: what undoes their power of two, times c2; start: what signed codes' 128 adds to the sum of products,
// taken off.
template <int NH>
__device__ __forceinline__ void fetch_queries(const QAttParams &p, int64_t row0, int h, int rows, int x, int t, uint4 (&w)[NH][4]) {
#pragma unroll
  for (int hh = 0; hh < NH; ++hh) {
    const int r = x + 8 * hh, j = r / p.G, g = r - j * p.G;
    const __nv_bfloat16 *qr = p.q + ((row0 + j) * p.Hq + h * p.G + g) * LOCKS_D + 16 * t;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[hh][i] = r < rows ? *reinterpret_cast<const uint4 *>(qr + (i >> 1) * 64 + 8 * (i & 1)) : make_uint4(0, 0, 0, 0);
  }
}
template <int NH>
__device__ __forceinline__ void take_queries(const QAttParams &p, const uint4 (&raw)[NH][4], int t, uint32_t (&qf)[NH][8][2], float2 (&rs)[NH], float2 (&start)[NH]) {
#pragma unroll
  for (int hh = 0; hh < NH; ++hh) {
    const uint4 (&w)[4] = raw[hh];
    float amax = 0.f;
    float v[8][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * i + (e >> 1)][2 * (e & 1)] = __uint_as_float(u[e] << 16);
        v[2 * i + (e >> 1)][2 * (e & 1) + 1] = __uint_as_float(u[e] & 0xFFFF0000u);
      }
    }
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) amax = fmaxf(amax, finite_abs(v[s][e]));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    const float up = power_to(amax, 0);
    const float back = p.c2 / up;
    rs[hh] = make_float2(__shfl_sync(0xffffffffu, back, 8 * t), __shfl_sync(0xffffffffu, back, 8 * t + 4));
    float sum = 0.f;   // of the elements as the products take them
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        qf[hh][s][e] = pack_f16(v[s][2 * e] * up, v[s][2 * e + 1] * up);
        const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&qf[hh][s][e]));
        sum += y.x;
        sum += y.y;
      }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    sum *= -0x1p-17f;
    start[hh] = make_float2(__shfl_sync(0xffffffffu, sum, 8 * t), __shfl_sync(0xffffffffu, sum, 8 * t + 4));
  }
}

// D = A B + C, with registers of its own for C (a start that several products share is not copied)
__device__ __forceinline__ void mma_f16_from(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, float c0, float c1, float c2, float c3) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};\n"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}

// transpose of an 8 x 8 matrix of 16-bit elements, lane (x, t) holding elements 2 t, 2 t + 1 of row x
__device__ __forceinline__ uint32_t movm_trans(uint32_t v) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
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
__device__ __forceinline__ float2 max2(float2 a, float2 b) { return make_float2(fmaxf(a.x, b.x), fmaxf(a.y, b.y)); }

// Running softmax of the row tile in a warp's registers, of rows 2 t, 2 t + 1 (+ 8) in every lane
template <int NH>
struct Running {
  float2 m[NH], l[NH];   // maximum (log2 units); the share of the sum of this lane's tokens
  float4 o[8][NH];       // dims 16 x + 2 i (.x, .y) and 16 x + 2 i + 1 (.z, .w)
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) {
      m[hh] = make_float2(-INFINITY, -INFINITY);
      l[hh] = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i][hh] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  // Scores of H tiles (tokens x and x + 8 of each, by the two rows) -> weights times 2^15 (pw; as B fragments pb).  f: what the sums of
  // products stand for, in log2 units.  MASK: some row does not see all of the tile, whose first token's place is pos
  template <int H, bool MASK>
  __device__ __forceinline__ void weights(const float (&s)[H][NH][4], const float2 (&f)[H][NH], const int2 (&lim)[NH], int pos, int x, uint32_t (&pb)[H][NH][2], float (&pw)[H][NH][4]) {
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) {
      float2 v[H][2], mx = make_float2(-INFINITY, -INFINITY);
#pragma unroll
      for (int w = 0; w < H; ++w) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          v[w][e] = make_float2(s[w][hh][2 * e], s[w][hh][2 * e + 1]);
          if (MASK) {
            v[w][e] = mul2(v[w][e], f[w][hh]);
            if (pos + x + 8 * e >= lim[hh].x) v[w][e].x = -INFINITY;
            if (pos + x + 8 * e >= lim[hh].y) v[w][e].y = -INFINITY;
          }
        }
        const float2 m2 = max2(v[w][0], v[w][1]);
        mx = max2(mx, MASK ? m2 : mul2(m2, f[w][hh]));
      }
#pragma unroll
      for (int k = 4; k < 32; k <<= 1) mx = max2(mx, make_float2(__shfl_xor_sync(0xffffffffu, mx.x, k), __shfl_xor_sync(0xffffffffu, mx.y, k)));
      const float2 mn = max2(m[hh], mx), ms = make_float2(mn.x == -INFINITY ? 0.f : mn.x, mn.y == -INFINITY ? 0.f : mn.y);
      if (__any_sync(0xffffffffu, mn.x != m[hh].x || mn.y != m[hh].y)) {   // some row's maximum rose
        const float2 a = make_float2(ex2f(m[hh].x - ms.x), ex2f(m[hh].y - ms.y));
        l[hh] = mul2(l[hh], a);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 lo = mul2(make_float2(o[i][hh].x, o[i][hh].y), a), hi = mul2(make_float2(o[i][hh].z, o[i][hh].w), a);
          o[i][hh] = make_float4(lo.x, lo.y, hi.x, hi.y);
        }
      }
      m[hh] = mn;
      const float2 off = make_float2(15.f - ms.x, 15.f - ms.y);
#pragma unroll
      for (int w = 0; w < H; ++w) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float2 y = MASK ? add2(v[w][e], off) : fma2(v[w][e], f[w][hh], off);
          const float2 q = make_float2(ex2f(y.x), ex2f(y.y));
          l[hh] = add2(l[hh], q);
          pw[w][hh][2 * e] = q.x;
          pw[w][hh][2 * e + 1] = q.y;
          pb[w][hh][e] = movm_trans(pack_f16(q.x, q.y));
        }
      }
    }
  }
  // Two dims' values of a tile's tokens join the outputs, times f; start: the accumulators' (both of rows 2 t, 2 t + 1)
  __device__ __forceinline__ void outputs(int i, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&pb)[NH][2], const float2 (&start)[NH], const float2 (&f)[NH]) {
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) {
      float c[4];
      mma_f16_from(c, a0, a1, a2, a3, pb[hh][0], pb[hh][1], start[hh].x, start[hh].y, start[hh].x, start[hh].y);
      const float2 lo = fma2(make_float2(c[0], c[1]), f[hh], make_float2(o[i][hh].x, o[i][hh].y));
      const float2 hi = fma2(make_float2(c[2], c[3]), f[hh], make_float2(o[i][hh].z, o[i][hh].w));
      o[i][hh] = make_float4(lo.x, lo.y, hi.x, hi.y);
    }
  }
  // into the warp's partial: [rows][kRowPad] outputs, [rows] (max, sum).  JOIN: `times` over, to what is there
  template <bool JOIN>
  __device__ __forceinline__ void leave(float *wo, float2 *wml, int x, int t, float times) {
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) {
      float2 sum = l[hh];
#pragma unroll
      for (int k = 4; k < 32; k <<= 1) sum = add2(sum, make_float2(__shfl_xor_sync(0xffffffffu, sum.x, k), __shfl_xor_sync(0xffffffffu, sum.y, k)));
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int r = 2 * t + c + 8 * hh;
        float mn = c ? m[hh].y : m[hh].x, total = c ? sum.y : sum.x, fo = 0.f, fn = 1.f;
        if (JOIN) {
          const float2 old = wml[r];
          const float mine = mn;
          mn = fmaxf(old.x, mine);
          fo = mn == -INFINITY ? 1.f : ex2f(old.x - mn);
          fn = times * (mn == -INFINITY ? 1.f : ex2f(mine - mn));
          total = old.y * fo + total * fn;
          __syncwarp();
        }
        if (x == 0) wml[r] = make_float2(mn, total);
        float *w = wo + r * kRowPad + 16 * x;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          float4 y = c ? make_float4(o[i][hh].y, o[i][hh].w, o[i + 1][hh].y, o[i + 1][hh].w) : make_float4(o[i][hh].x, o[i][hh].z, o[i + 1][hh].x, o[i + 1][hh].z);
          if (JOIN) {
            const float4 z = *reinterpret_cast<const float4 *>(w + 2 * i);
            y = make_float4(fmaf(y.x, fn, z.x * fo), fmaf(y.y, fn, z.y * fo), fmaf(y.z, fn, z.z * fo), fmaf(y.w, fn, z.w * fo));
          }
          *reinterpret_cast<float4 *>(w + 2 * i) = y;
        }
      }
    }
  }
};

template <int NH> struct Queries {   // as fragments, and what undoes their power of two, times sm_scale log2 e
  uint32_t f[NH][8][2];
  float2 rs[NH];
};
// 16 places of the unfinished page (fp32), from pos on, joined to the warp's partial `times` over.  Elements go to fp16 times a power
// of two of the tile's largest, values rounded (2^-11 of each), keys in two parts.  Out of line: its registers would be the tile loop's.
template <int NH, int FMT>
__device__ __noinline__ void tail_tile(const Queries<NH> &q, int T, int2 lim0, int2 lim1, const float *kt, const float *vt, int pos, float times, float *wo, float2 *wml) {
  const int lane = threadIdx.x & 31, x = lane >> 2, t = lane & 3;
  uint32_t pb[1][NH][2];
  float2 f[1][NH];
  float pw[1][NH][4], s[1][NH][4];
  int2 lim[NH];
  lim[0] = lim0;
  lim[NH - 1] = NH == 1 ? lim0 : lim1;
  Running<NH> run;
  run.clear();
  float4 k[2][8];
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      k[w][i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (pos + x + 8 * w < T) k[w][i] = *reinterpret_cast<const float4 *>(kt + (x + 8 * w) * LOCKS_D + (i >> 2) * 64 + 16 * t + 4 * (i & 3));
    }
  float4 v[4][4];   // 16 dims of tokens 2 t, 2 t + 1, 8 + 2 t, 9 + 2 t
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int tok = 2 * t + (e & 1) + 4 * (e & 2);
      v[e][i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (pos + tok < T) v[e][i] = *reinterpret_cast<const float4 *>(vt + tok * LOCKS_D + 16 * x + 4 * i);
    }
  float amax = 0.f;
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      amax = fmaxf(amax, fmaxf(fmaxf(finite_abs(k[w][i].x), finite_abs(k[w][i].y)), fmaxf(finite_abs(k[w][i].z), finite_abs(k[w][i].w))));
  float up = power_to(warp_max(amax), 14);
  bool odd = false;   // an infinity or a NaN
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      odd |= !(fabsf(k[w][i].x) < INFINITY && fabsf(k[w][i].y) < INFINITY && fabsf(k[w][i].z) < INFINITY && fabsf(k[w][i].w) < INFINITY);
  const bool finite_tile = !__any_sync(0xffffffffu, odd);
#pragma unroll
  for (int hh = 0; hh < NH; ++hh) s[0][hh][0] = s[0][hh][1] = s[0][hh][2] = s[0][hh][3] = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {   // in two parts: 22 bits of each
    uint32_t a[4], rest[4];       // token x, x + 8; dims 0 1, 2 3 of the four
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float2 y = e ? make_float2(k[w][i].z * up, k[w][i].w * up) : make_float2(k[w][i].x * up, k[w][i].y * up);
        a[w + 2 * e] = pack_f16(y.x, y.y);
        const float2 z = __half22float2(*reinterpret_cast<__half2 *>(&a[w + 2 * e]));
        rest[w + 2 * e] = pack_f16(y.x - z.x, y.y - z.y);
      }
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) {
      mma_f16(s[0][hh], a[0], a[1], a[2], a[3], q.f[hh][i][0], q.f[hh][i][1]);
      if (finite_tile) mma_f16(s[0][hh], rest[0], rest[1], rest[2], rest[3], q.f[hh][i][0], q.f[hh][i][1]);
    }
  }
#pragma unroll
  for (int hh = 0; hh < NH; ++hh) f[0][hh] = make_float2(q.rs[hh].x / up, q.rs[hh].y / up);
  run.template weights<1, true>(s, f, lim, pos, x, pb, pw);
  amax = 0.f;
  odd = false;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      amax = fmaxf(amax, fmaxf(fmaxf(finite_abs(v[e][i].x), finite_abs(v[e][i].y)), fmaxf(finite_abs(v[e][i].z), finite_abs(v[e][i].w))));
      odd |= !(fabsf(v[e][i].x) < INFINITY && fabsf(v[e][i].y) < INFINITY && fabsf(v[e][i].z) < INFINITY && fabsf(v[e][i].w) < INFINITY);
    }
  up = power_to(warp_max(amax), 14);
  if (!__any_sync(0xffffffffu, odd)) {
    float2 back[NH], zero[NH];
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) { back[hh] = make_float2(kUnit<FMT> / up, kUnit<FMT> / up); zero[hh] = make_float2(0.f, 0.f); }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      run.outputs(2 * i, pack_f16(v[0][i].x * up, v[1][i].x * up), pack_f16(v[0][i].y * up, v[1][i].y * up), pack_f16(v[2][i].x * up, v[3][i].x * up), pack_f16(v[2][i].y * up, v[3][i].y * up), pb[0], zero, back);
      run.outputs(2 * i + 1, pack_f16(v[0][i].z * up, v[1][i].z * up), pack_f16(v[0][i].w * up, v[1][i].w * up), pack_f16(v[2][i].z * up, v[3][i].z * up), pack_f16(v[2][i].w * up, v[3][i].w * up), pb[0], zero, back);
    }
  } else {   // token by token in fp32, so that a row takes nothing of a token that it does not see
#pragma unroll 1
    for (int k2 = 0; k2 < 16 && pos + k2 < T; ++k2) {
      const int from = 4 * (k2 & 7) + t;   // who has the token's weights of rows 2 t, 2 t + 1
#pragma unroll
      for (int hh = 0; hh < NH; ++hh) {
        const float w0 = kUnit<FMT> * __shfl_sync(0xffffffffu, k2 < 8 ? pw[0][hh][0] : pw[0][hh][2], from);
        const float w1 = kUnit<FMT> * __shfl_sync(0xffffffffu, k2 < 8 ? pw[0][hh][1] : pw[0][hh][3], from);
        const bool s0 = pos + k2 < lim[hh].x, s1 = pos + k2 < lim[hh].y;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 y = *reinterpret_cast<const float2 *>(vt + k2 * LOCKS_D + 16 * x + 2 * i);
          if (s0) { run.o[i][hh].x = fmaf(w0, y.x, run.o[i][hh].x); run.o[i][hh].z = fmaf(w0, y.y, run.o[i][hh].z); }
          if (s1) { run.o[i][hh].y = fmaf(w1, y.x, run.o[i][hh].y); run.o[i][hh].w = fmaf(w1, y.y, run.o[i][hh].w); }
        }
      }
    }
  }
  run.template leave<true>(wo, wml, x, t, times);
}

// Partials of CTAs c, c + step, .. c1 of the problem that begins in CTA c0: row r, four dims; N loads at a time
template <int N>
__device__ __forceinline__ float4 join_partials(const QAttParams &p, int c0, int c, int c1, int step, int r, int d4, float &M, float &L) {
  M = -INFINITY;
  L = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  for (; c <= c1; c += N * step) {
    float2 ml[N];
    float4 y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int ci = c + i * step, s = 2 * ci + (ci == c0 ? 1 : 0);
      ml[i] = make_float2(-INFINITY, 0.f);
      y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (ci <= c1) {
        ml[i] = __ldcg(p.part_ml + s * KVQ_ROWS + r);
        y[i] = __ldcg(reinterpret_cast<const float4 *>(p.part + ((int64_t)s * KVQ_ROWS + r) * LOCKS_D + d4));
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float mn = fmaxf(M, ml[i].x), fo = mn == -INFINITY ? 1.f : ex2f(M - mn), fn = mn == -INFINITY ? 1.f : ex2f(ml[i].x - mn);
      L = L * fo + ml[i].y * fn;
      a.x = a.x * fo + y[i].x * fn; a.y = a.y * fo + y[i].y * fn; a.z = a.z * fo + y[i].z * fn; a.w = a.w * fo + y[i].w * fn;
      M = mn;
    }
  }
  return a;
}

// Output rows: one row's four dims from its maximum, sum and unnormalised mean
template <int FMT>
__device__ __forceinline__ void finish_dims(const QAttParams &p, int64_t row, int d4, float4 a, float M, float L) {
  const float inv = L == 0.f ? 0.f : 1.f / kUnit<FMT> / L;   // (0: nothing seen)
  *reinterpret_cast<uint2 *>(p.out + row * LOCKS_D + d4) = make_uint2(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv));
  if (p.lse && d4 == 0) p.lse[row] = L == 0.f ? -INFINITY : ((M == -INFINITY ? 0.f : M) - 15.f + log2f(L)) * kLn2;
}

// A warp's ring: pairs of tiles; a tile is 4 KB (keys, then values; 16 rows of 128 bytes).  16-byte pieces of a row are stored at piece
// ^ 4 (row % 2) (keys) and piece ^ 2 (row / 2 % 4) (values): then the eight lanes that read together, two rows' pieces 4 c .. 4 c + 3
// (keys) or four rows' pieces 2 c, 2 c + 1 (values), touch every bank once.
constexpr int kTile = 2 * 16 * LOCKS_D, kPair = 2 * kTile;
template <int NH> constexpr int kStages = NH == 1 ? 2 : 3;
template <int NH> constexpr int kCtasPerSm = NH == 1 ? 3 : 2;
template <int NH> constexpr int kRing = kStages<NH> * kPair;
template <int NH> constexpr int token_smem() { return kWarps * kRing<NH> + 16; }
static_assert(kRing<1> >= 8 * (kRowPad * 4 + 8) && kRing<2> >= 16 * (kRowPad * 4 + 8), "a warp's partial takes its ring's place");

template <int FMT> constexpr float kScaleUnit = FMT == LOCKS_KVQ_INT ? 1.f : kUnit<FMT>;   // (signed codes come in their unit)

// codes of a word (flipped, if signed) as fp16 in units of kUnit (signed) or 1
template <int FMT> __device__ __forceinline__ void halves(uint32_t w, uint32_t &lo, uint32_t &hi) {
  if (FMT == LOCKS_KVQ_INT) { lo = __byte_perm(w, 0, 0x4140); hi = __byte_perm(w, 0, 0x4342); }
  else kvq_halves<LOCKS_KVQ_FLOAT>(w, lo, hi);
}

template <int NH, int FMT, bool CONTIG>
__global__ void __launch_bounds__(kThreads, kCtasPerSm<NH>) kvq_token_kernel(const __grid_constant__ QAttParams p) {
  extern __shared__ __align__(128) uint8_t ring_s[];
  constexpr int R = 8 * NH, S = kStages<NH>;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, x = lane >> 2, t = lane & 3;
  uint8_t *ring = ring_s + warp * kRing<NH>;
  auto part_of = [&](int w) { return reinterpret_cast<float *>(ring_s + w * kRing<NH>); };   // [R][kRowPad], then [R] (max, sum)
  auto ml_of = [&](int w) { return reinterpret_cast<float2 *>(part_of(w) + R * kRowPad); };
  int &last_s = *reinterpret_cast<int *>(ring_s + kWarps * kRing<NH>);
  pdl_trigger();
  pdl_wait();
  Line line;
  line.read(p, lane, gridDim.x);
  const int share = line.share, lead = line.lead;
  if ((int64_t)share * blockIdx.x >= line.all) return;
  int u = share * blockIdx.x, b = -1, begin = 0;
  const int u_end = min((int64_t)u + share, (int64_t)line.all);
  Request req = {0, 0, 0, 0, 0};
  // 16-byte copies: copy i of a tile moves piece lane & 7 of row (lane >> 3) + 4 i
  const int cr = lane >> 3, cc = lane & 7;
  const uint32_t k_dst = cr * 128 + ((cc ^ (4 * (cr & 1))) << 4), v_dst = 2048 + cr * 128 + ((cc ^ (2 * (cr >> 1))) << 4);
  const int64_t st = CONTIG ? LOCKS_D : p.c.st, c_off = (int64_t)cr * st + cc * 16;
  while (u < u_end) {
    if (b < 0 || u >= begin + line.places(p, req)) line.find(p, u, lane, b, begin, req);
    const int span = lead + req.pairs, prob = (u - begin) / span, prob_begin = begin + prob * span;   // problem of the request
    const int seg0 = max(u - prob_begin - lead, 0), seg1 = min(req.pairs, u_end - prob_begin - lead);
    u = prob_begin + lead + max(seg1, 0);
    if (seg1 <= seg0) continue;   // (nothing but some of the problem's lead)
    const int h = prob % p.Hkv, rt = prob / p.Hkv, hkv = h / p.kvdiv, kv_heads = p.Hkv / p.kvdiv;
    const int j0 = rt * p.tile_tokens, toks = min(p.tile_tokens, req.n - j0), rows = toks * p.G;
    const int T = req.T, B = p.c.B, full_pages = T > 0 ? T / B : 0;
    int tiles = p.c.Pmax << p.sub_shift;   // (a dense problem's further tiles lie behind its tokens)
    if (p.ids) {
      int npages = p.cnt[(int64_t)b * p.Hkv + h];
      if (npages < 0 || npages > p.kbud) {
        if (tid == 0) set_status(p.status, LOCKS_ERR_BAD_BLOCK);
        npages = npages < 0 ? 0 : p.kbud;
      }
      tiles = npages << p.sub_shift;
    }
    const int lim_min = T - req.n + j0 + 1;   // what the row tile's first token sees
    // ---- the segment's pairs: this warp's are pair_at(j).  Blocks and scales of 16 pairs at a time, a lane per tile.  Where the problem's last
    // pair, with its unfinished page, is among them, the warp that has it gets kTailPairs fewer than the others.
    const int sub_mask = (1 << p.sub_shift) - 1, end = min(seg1, (tiles + 1) >> 1), count = max(end - seg0, 0);
    const int fewer = end == min(req.pairs, (tiles + 1) >> 1) && T & (B - 1) && count ? min(kTailPairs, (count - 1) / (kWarps - 1)) : 0;
    const int owner = (count - 1 - (kWarps - 1) * fewer) & (kWarps - 1), more = warp == owner ? 0 : fewer;
    const int first = seg0 + warp - (warp > owner), rest = seg0 + (kWarps - 1) * fewer + warp - kWarps * more;   // (pairs of the first `more` rounds, of the others)
    auto pair_at = [&](int j) { return j < more ? first + (kWarps - 1) * j : rest + kWarps * j; };
    const int mine = max((count - (kWarps - 1) * fewer - warp + kWarps - 1) / kWarps, 0) + more;
    struct Batch {
      int blk, page;         // block, page of this lane's tile
      float ks, vs;
      uint32_t have, easy;   // tiles of codes; those among them that every row sees whole.  Not uniform bits of the others: 0
    };
    auto tile_at = [&](int jb) { return 2 * pair_at(jb + (lane >> 1)) + (lane & 1); };
    auto page_at = [&](int tile) { return p.ids ? p.ids[((int64_t)b * p.Hkv + h) * p.kbud + (tile >> p.sub_shift)] : tile >> p.sub_shift; };
    auto resolve = [&](int jb) {
      const int tile = tile_at(jb);
      Batch r = {-1, 0, 0.f, 0.f, 0, 0};
      if (tile < min(tiles, 2 * end)) {
        r.page = page_at(tile);
        if (r.page < 0 || r.page >= p.c.Pmax) {
          set_status(p.status, LOCKS_ERR_BAD_BLOCK);
        } else if (r.page < full_pages) {
          r.blk = p.c.block_table[(int64_t)b * p.c.Pmax + r.page];
          if (r.blk < 0 || r.blk >= p.c.num_blocks) {
            r.blk = -1;
            set_status(p.status, LOCKS_ERR_BAD_BLOCK);
          } else {
            const int64_t at = (int64_t)r.blk * kv_heads + hkv;
            r.ks = p.c.ks[at];
            r.vs = p.c.vs[at];
          }
        } else if (r.page == full_pages && r.page * B + (tile & sub_mask) * 16 < T) {
          r.blk = kUnfinished;
        }
      }
      __syncwarp();
      r.have = __ballot_sync(0xffffffffu, r.blk >= 0);
      r.easy = __ballot_sync(0xffffffffu, r.blk >= 0 && r.page * B + (tile & sub_mask) * 16 + 16 <= lim_min);
      return r;
    };
    uint4 raw[NH][4];
    fetch_queries<NH>(p, req.row0 + j0, h, rows, x, t, raw);
    Batch cur = resolve(0), next = cur;
    auto issue = [&](int j, const Batch &r) {   // a pair's copies
      uint8_t *dst = ring + (j % S) * kPair;
      const int l = 2 * (j & 15);
      if (j < mine) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const int bk = __shfl_sync(0xffffffffu, r.blk, l + w);
          if ((r.have >> (l + w)) & 1) {
            const int sub = (2 * pair_at(j) + w) & sub_mask;
            const int64_t off = (int64_t)bk * p.c.sb + (int64_t)hkv * p.c.sh + (int64_t)(sub * 16) * st + c_off;
            const char *kp = p.c.k + off, *vp = p.c.v + off;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              copy16(dst + w * kTile + k_dst + 512 * i, kp + 4 * i * st);
              copy16(dst + w * kTile + (v_dst ^ (64 * (i & 1))) + 512 * i, vp + 4 * i * st);
            }
          }
        }
      }
      cp_async_commit();
    };
#pragma unroll
    for (int j = 0; j < S - 1; ++j) issue(j, cur);
    uint32_t qf[NH][8][2];
    float2 rs[NH], start[NH];
    take_queries<NH>(p, raw, t, qf, rs, start);
    int2 lim[NH];    // rows 2 t, 2 t + 1 (+ 8) see the first lim tokens
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) {
      const int r = 2 * t + 8 * hh;
      lim[hh] = make_int2(r < rows ? lim_min + r / p.G : T, r + 1 < rows ? lim_min + (r + 1) / p.G : T);
    }
    Running<NH> run;
    run.clear();
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) {
      if (FMT == LOCKS_KVQ_INT) rs[hh] = make_float2(rs[hh].x * 0x1p24f, rs[hh].y * 0x1p24f);
      else start[hh] = make_float2(0.f, 0.f);
    }
    // scores of a tile: two chains of four steps
    auto scores = [&](const uint8_t *kt, float (&s)[NH][4]) {
      float c[2][NH][4];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t at = x * 128 + (((4 * half + t) ^ (4 * (x & 1))) << 4);
        const uint4 y0 = *reinterpret_cast<const uint4 *>(kt + at), y1 = *reinterpret_cast<const uint4 *>(kt + at + 1024);
        const uint32_t w0[4] = {y0.x, y0.y, y0.z, y0.w}, w1[4] = {y1.x, y1.y, y1.z, y1.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = 4 * half + i;
          uint32_t a[4];   // token x, x + 8; dims 0 1, 2 3 of the four
          halves<FMT>(kvq_flip<FMT>(w0[i]), a[0], a[2]);
          halves<FMT>(kvq_flip<FMT>(w1[i]), a[1], a[3]);
#pragma unroll
          for (int hh = 0; hh < NH; ++hh) {
            if (k == 0) mma_f16_from(c[0][hh], a[0], a[1], a[2], a[3], qf[hh][k][0], qf[hh][k][1], start[hh].x, start[hh].y, start[hh].x, start[hh].y);
            else if (k == 4) mma_f16_from(c[1][hh], a[0], a[1], a[2], a[3], qf[hh][k][0], qf[hh][k][1], 0.f, 0.f, 0.f, 0.f);
            else mma_f16(c[half][hh], a[0], a[1], a[2], a[3], qf[hh][k][0], qf[hh][k][1]);
          }
        }
      }
#pragma unroll
      for (int hh = 0; hh < NH; ++hh)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[hh][e] = c[0][hh][e] + c[1][hh][e];
    };
    auto values = [&](const uint8_t *vt, const uint32_t (&pb)[NH][2], const float2 (&fv)[NH]) {
      float2 from[NH];
#pragma unroll
      for (int hh = 0; hh < NH; ++hh) {
        from[hh] = make_float2(0.f, 0.f);
        if (FMT == LOCKS_KVQ_INT) {   // 128 sum of weights
          float c[4];
          mma_f16_from(c, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u, pb[hh][0], pb[hh][1], 0.f, 0.f, 0.f, 0.f);
          from[hh] = make_float2(-0x1p-17f * c[0], -0x1p-17f * c[1]);
        }
      }
      uint4 v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const uint4 *>(vt + (2 * t + (e & 1) + 4 * (e & 2)) * 128 + ((x ^ (2 * t)) << 4));
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        auto word = [&](int e) { return kvq_flip<FMT>(w == 0 ? v[e].x : (w == 1 ? v[e].y : (w == 2 ? v[e].z : v[e].w))); };
        const uint32_t a0 = word(0), a1 = word(1), a2 = word(2), a3 = word(3);
        uint32_t ha[4][2];   // [dim][token pair]
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint32_t lo = c ? a2 : a0, hi = c ? a3 : a1;
          halves<FMT>(__byte_perm(lo, hi, 0x5140), ha[0][c], ha[1][c]);
          halves<FMT>(__byte_perm(lo, hi, 0x7362), ha[2][c], ha[3][c]);
        }
        run.outputs(2 * w, ha[0][0], ha[1][0], ha[0][1], ha[1][1], pb, from, fv);
        run.outputs(2 * w + 1, ha[2][0], ha[3][0], ha[2][1], ha[3][1], pb, from, fv);
      }
    };
    // times that this warp takes each 16-token part of the unfinished page, 16 bits a part: where all pages are read, the parts that lie
    // in the segment go to different warps, the owner's first; of a page table, the parts that the warp meets
    uint64_t tails = 0;
    if (!p.ids && T & (B - 1) && full_pages < p.c.Pmax)
      for (int sub = 0; sub * 16 < (T & (B - 1)); ++sub) {
        const int pair = ((full_pages << p.sub_shift) + sub) >> 1;
        if (pair >= seg0 && pair < end && ((owner + sub) & (kWarps - 1)) == warp) tails += 1ull << (16 * sub);
      }
#pragma unroll 1
    for (int j = 0; j < mine; ++j) {
      const int jn = j + S - 1, l = 2 * (j & 15);
      if ((jn & 15) == 8) next = resolve((jn & ~15) + 16);   // half a batch early
      if ((jn & 15) < S - 1 && jn >= 16) issue(jn, next);    // (pair j + S - 1 is of the next batch, pair j of this one)
      else issue(jn, cur);
      cp_async_wait<S - 1>();
      __syncwarp();
      const uint8_t *pair = ring + (j % S) * kPair;
      const float ks[2] = {__shfl_sync(0xffffffffu, cur.ks, l), __shfl_sync(0xffffffffu, cur.ks, l + 1)};
      const float vs[2] = {__shfl_sync(0xffffffffu, cur.vs, l) * kScaleUnit<FMT>, __shfl_sync(0xffffffffu, cur.vs, l + 1) * kScaleUnit<FMT>};
      if (((cur.easy >> l) & 3) == 3) {
        float s[2][NH][4], pw[2][NH][4];
        float2 f[2][NH];
        uint32_t pb[2][NH][2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          scores(pair + w * kTile, s[w]);
#pragma unroll
          for (int hh = 0; hh < NH; ++hh) f[w][hh] = make_float2(rs[hh].x * ks[w], rs[hh].y * ks[w]);
        }
        run.template weights<2, false>(s, f, lim, 0, x, pb, pw);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          float2 fv[NH];
#pragma unroll
          for (int hh = 0; hh < NH; ++hh) fv[hh] = make_float2(vs[w], vs[w]);
          values(pair + w * kTile + 2048, pb[w], fv);
        }
      } else {
#pragma unroll 1
        for (int w = 0; w < 2; ++w) {
          const int sub = (2 * pair_at(j) + w) & sub_mask;
          const int pos = __shfl_sync(0xffffffffu, cur.page, l + w) * B + sub * 16;
          if (!((cur.have >> (l + w)) & 1)) {
            if (p.ids && __shfl_sync(0xffffffffu, cur.blk, l + w) == kUnfinished) tails += 1ull << (16 * sub);
            continue;
          }
          float s[1][NH][4], pw[1][NH][4];
          float2 f[1][NH], fv[NH];
          uint32_t pb[1][NH][2];
          scores(pair + w * kTile, s[0]);
#pragma unroll
          for (int hh = 0; hh < NH; ++hh) {   // rows that see nothing of the tile take nothing of it, not even a NaN that its scale may be
            f[0][hh] = make_float2(rs[hh].x * (w ? ks[1] : ks[0]), rs[hh].y * (w ? ks[1] : ks[0]));
            fv[hh] = make_float2(pos < lim[hh].x ? (w ? vs[1] : vs[0]) : 0.f, pos < lim[hh].y ? (w ? vs[1] : vs[0]) : 0.f);
          }
          run.template weights<1, true>(s, f, lim, pos, x, pb, pw);
          values(pair + w * kTile + 2048, pb[0], fv);
        }
      }
      if ((j & 15) == 15) cur = next;
      __syncwarp();
    }
    // ---- the warps' partials
    cp_async_wait<0>();
    __syncwarp();
    run.template leave<false>(part_of(warp), ml_of(warp), x, t, 1.f);
    __syncwarp();
#pragma unroll 1
    for (int sub = 0; tails; ++sub, tails >>= 16) {
      if (!(tails & 0xffff)) continue;
      const int64_t at = p.c.tail_at(b, hkv, full_pages) + 16 * sub * LOCKS_D;
      Queries<NH> q;   // (a copy: what a call takes by address lies in memory)
#pragma unroll
      for (int hh = 0; hh < NH; ++hh) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { q.f[hh][i][0] = qf[hh][i][0]; q.f[hh][i][1] = qf[hh][i][1]; }
        q.rs[hh] = FMT == LOCKS_KVQ_INT ? make_float2(rs[hh].x * 0x1p-24f, rs[hh].y * 0x1p-24f) : rs[hh];
      }
      tail_tile<NH, FMT>(q, T, lim[0], lim[NH - 1], p.c.kt + at, p.c.vt + at, full_pages * B + 16 * sub, (float)(tails & 0xffff), part_of(warp), ml_of(warp));
      __syncwarp();
    }
    __syncthreads();
    const bool whole = seg0 == 0 && seg1 == req.pairs;
    const int slot = 2 * blockIdx.x + (seg0 == 0 ? 1 : 0);
    auto row_of = [&](int r) { const int j = r / p.G; return (int64_t)(req.row0 + j0 + j) * p.Hq + h * p.G + (r - j * p.G); };
    for (int i = tid; i < rows * (LOCKS_D / 4); i += kThreads) {
      const int r = i >> 5, d4 = 4 * (i & 31);
      float M = -INFINITY, L = 0.f;
      float2 ml[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) { ml[w] = ml_of(w)[r]; M = fmaxf(M, ml[w].x); }
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = M == -INFINITY ? 1.f : ex2f(ml[w].x - M);   // (a sum of NaN stays)
        const float4 y = *reinterpret_cast<const float4 *>(part_of(w) + r * kRowPad + d4);
        L += ml[w].y * f;
        a.x = fmaf(y.x, f, a.x); a.y = fmaf(y.y, f, a.y); a.z = fmaf(y.z, f, a.z); a.w = fmaf(y.w, f, a.w);
      }
      if (whole) {
        finish_dims<FMT>(p, row_of(r), d4, a, M, L);
      } else {
        __stcg(reinterpret_cast<float4 *>(p.part + ((int64_t)slot * KVQ_ROWS + r) * LOCKS_D + d4), a);
        if (d4 == 0) __stcg(p.part_ml + slot * KVQ_ROWS + r, make_float2(M, L));
      }
    }
    if (!whole && p.done) {   // the last of the problem's CTAs puts its partials together, in their order
      const int c0 = (prob_begin + lead) / share, c1 = (prob_begin + lead + req.pairs - 1) / share;
      __syncthreads();
      if (tid == 0) {
        __threadfence();   // what the CTA has written, which the barrier orders before
        last_s = atomicAdd(p.done + c0, 1) == c1 - c0;
        __threadfence();
      }
      __syncthreads();
      if (last_s) {
        for (int i = tid; i < rows * (LOCKS_D / 4); i += kThreads) {
          const int r = i >> 5, d4 = 4 * (i & 31);
          float M, L;
          const float4 a = join_partials<8>(p, c0, c0, c1, 1, r, d4, M, L);
          finish_dims<FMT>(p, row_of(r), d4, a, M, L);
        }
        if (tid == 0) p.done[c0] = 0;   // ready for the next launch
      }
    }
    __syncthreads();   // the partials' memory is the rings'
  }
}

// Problems that many CTAs share: a CTA per output row puts their partials together, a warp every eighth of them.
template <int FMT>
__global__ void __launch_bounds__(32 * kJoinWarps) kvq_join_kernel(const __grid_constant__ QAttParams p, int ctas) {
  __shared__ float4 a_s[kJoinWarps][32];
  __shared__ float2 ml_s[kJoinWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int hq = blockIdx.x, row = blockIdx.y, h = hq / p.G;
  pdl_trigger();
  pdl_wait();
  // the row's request (all warps alike), and where its part of the line begins
  int b = p.cu ? -1 : row;
  for (int b0 = 0; p.cu && b0 < p.batch; b0 += 32) {
    const uint32_t has = __ballot_sync(0xffffffffu, b0 + lane < p.batch && p.cu[b0 + lane] <= row && row < p.cu[b0 + lane + 1]);
    if (has) { b = b0 + __ffs(has) - 1; break; }
  }
  if (b < 0) return;
  const Request req = request_at(p, b);
  const int j = row - req.row0;
  if (j >= req.n) return;   // (offsets out of range)
  Line line;
  line.read(p, lane, ctas);
  if (line.all == 0) return;
  const int share = line.share;
  int before = 0;   // places of the requests before
  if (b < 32) {
    before = __shfl_sync(0xffffffffu, line.end - line.places(p, line.r), b);
  } else {
    before = __shfl_sync(0xffffffffu, line.end, 31);
    for (int b0 = 32; b0 < b; b0 += 32) before += __reduce_add_sync(0xffffffffu, b0 + lane < b ? line.places(p, request_at(p, b0 + lane)) : 0);
  }
  const int rt = j / p.tile_tokens, r = (j - rt * p.tile_tokens) * p.G + hq - h * p.G;
  const int at = before + (rt * p.Hkv + h) * (line.lead + req.pairs) + line.lead;   // its first pair
  const int c0 = at / share, c1 = (at + req.pairs - 1) / share;
  if (c0 == c1) return;     // finished by its CTA
  float M, L;
  const float4 a = join_partials<8>(p, c0, c0 + warp, c1, kJoinWarps, r, 4 * lane, M, L);
  a_s[warp][lane] = a;
  if (lane == 0) ml_s[warp] = make_float2(M, L);
  __syncthreads();
  if (warp) return;
  M = -INFINITY; L = 0.f;
  for (int w = 0; w < kJoinWarps; ++w) M = fmaxf(M, ml_s[w].x);
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int w = 0; w < kJoinWarps; ++w) {
    const float f = M == -INFINITY ? 1.f : ex2f(ml_s[w].x - M);
    const float4 y = a_s[w][lane];
    L += ml_s[w].y * f;
    o.x = fmaf(y.x, f, o.x); o.y = fmaf(y.y, f, o.y); o.z = fmaf(y.z, f, o.z); o.w = fmaf(y.w, f, o.w);
  }
  finish_dims<FMT>(p, (int64_t)row * p.Hq + hq, 4 * lane, o, M, L);
}

}  // namespace

extern "C" int locks_kvq_attend(locks_ctx *ctx, const void *q, const int32_t *cu_tokens, int num_tokens, const locks_kvq *kv, int batch,
                                const int32_t *page_ids, const int32_t *page_count, void *out, float *lse, locks_stream stream) {
  int rc = kvq_check(ctx, kv, batch);
  if (rc != LOCKS_OK) return rc;
  if (!q || !out || ((uintptr_t)q | (uintptr_t)out) % 16 || (uintptr_t)lse % 4 || num_tokens < 1) return LOCKS_ERR_INVALID_ARG;
  if ((page_ids == nullptr) != (page_count == nullptr) || (page_ids && cu_tokens) || (!cu_tokens && num_tokens != batch)) return LOCKS_ERR_INVALID_ARG;
  QAttParams p = {};
  p.q = reinterpret_cast<const __nv_bfloat16 *>(q); p.cu = cu_tokens; p.c = kvq_cache(ctx, kv); p.ids = page_ids; p.cnt = page_count;
  p.out = reinterpret_cast<__nv_bfloat16 *>(out); p.lse = lse;
  p.part = ctx->kvq_part; p.part_ml = ctx->kvq_ml; p.done = ctx->kvq_done; p.status = ctx->status;
  p.n = num_tokens; p.batch = batch; p.Hq = ctx->cfg.num_q_heads; p.Hkv = ctx->cfg.num_kv_heads; p.G = ctx->G; p.kvdiv = 1; p.kbud = ctx->k;
  if (ctx->cfg.combine == LOCKS_COMBINE_PER_HEAD && page_ids) { p.kvdiv = p.G; p.Hkv = p.Hq; p.G = 1; }   // a page table per query head
  p.sub_shift = ctx->B == 64 ? 2 : (ctx->B == 32 ? 1 : 0);
  p.c2 = ctx->cfg.sm_scale * kLog2e;
  // Chunks of prompts, from 96 query rows a KV head and request on average, and 768 in all (20 to 24 tokens of 32 heads): the form with 256
  // rows a CTA.  Measured either side, us, this form and that, 32 query heads: one request at 16301 with 8 KV heads 41 / 43 (16 tokens),
  // 58 / 46 (32), 183 / 74 (128), 1361 / 374 (1024); six at 6000 113 / 60 (32 each); with 2 KV heads 38 / 32 (8 each); 24 at 3000 with 8 KV
  // heads 132 / 138 (16 each), 246 / 139 (32).  Also where the line of this form may not fit 32 bits.  (The host knows the average alone: a
  // batch of a chunk and single tokens takes one form for both, which costs up to 2.4 times what two calls do: 512 tokens beside 31 single ones at
  // 8000 533 us, as two calls 221; 1024 beside 15 337 and 257; 2048 beside 24 at 16000 1205 and 823.)
  const int64_t problem = (((int64_t)(page_ids ? p.kbud : p.c.Pmax) << p.sub_shift) + 1) / 2 + kMostLead;   // places at most
  const bool fits = (batch + (cu_tokens ? (int64_t)num_tokens : 0)) * p.Hkv * problem <= INT32_MAX;
  if (cu_tokens && (!fits || ((int64_t)num_tokens * p.G >= (int64_t)96 * batch && (int64_t)num_tokens * p.Hq >= 768))) {
    ctx->last_launches = 0;
    return locks_launch_kvq_chunk(ctx, q, cu_tokens, num_tokens, kv, batch, out, lse, (cudaStream_t)stream);
  }
  if (!fits) return LOCKS_ERR_TOO_LARGE;
  // 8 rows a tile where a request's rows fit on average, else 16
  const bool wide = p.G > 8 || (int64_t)num_tokens * p.G > (int64_t)8 * batch;
  p.tile_tokens = (wide ? 16 : 8) / p.G;
  int ctas = ctx->num_sms * (wide ? kCtasPerSm<2> : kCtasPerSm<1>);
  if (ctas > KVQ_SLOT_BOUND) ctas = KVQ_SLOT_BOUND;
  // Few problems, each shared by many CTAs: a kernel of its own puts the partials together, row by row, side by side
  const int64_t problems = (cu_tokens ? std::max<int64_t>(batch, num_tokens / p.tile_tokens) : batch) * p.Hkv;
  const bool join = ctas >= kManyShares * problems;
  if (join) p.done = nullptr;
  const bool contig = kv->stride_token == LOCKS_D;
  ctx->last_launches = 0;
#define KVQ_TOKEN(NH_, F_, C_)                                                                                                        \
  do {                                                                                                                                \
    if (wide != (NH_ == 2) || kv->fmt != F_ || contig != C_) break;                                                                   \
    if (locks_attrs_needed(LOCKS_ATTR_KVQ + 4 * (NH_ - 1) + 2 * F_ + C_))                                                             \
      cudaFuncSetAttribute(kvq_token_kernel<NH_, F_, C_>, cudaFuncAttributeMaxDynamicSharedMemorySize, token_smem<NH_>());            \
    locks_launch_pdl(kvq_token_kernel<NH_, F_, C_>, dim3(ctas), dim3(kThreads), token_smem<NH_>(), (cudaStream_t)stream, p);          \
  } while (0)
  KVQ_TOKEN(1, LOCKS_KVQ_INT, true);
  KVQ_TOKEN(1, LOCKS_KVQ_INT, false);
  KVQ_TOKEN(1, LOCKS_KVQ_FLOAT, true);
  KVQ_TOKEN(1, LOCKS_KVQ_FLOAT, false);
  KVQ_TOKEN(2, LOCKS_KVQ_INT, true);
  KVQ_TOKEN(2, LOCKS_KVQ_INT, false);
  KVQ_TOKEN(2, LOCKS_KVQ_FLOAT, true);
  KVQ_TOKEN(2, LOCKS_KVQ_FLOAT, false);
#undef KVQ_TOKEN
  if ((rc = locks_check_launch(ctx)) != LOCKS_OK || !join) return rc;
  const dim3 rows(p.Hq, num_tokens);
  if (kv->fmt == LOCKS_KVQ_INT) locks_launch_pdl(kvq_join_kernel<LOCKS_KVQ_INT>, rows, dim3(32 * kJoinWarps), 0, (cudaStream_t)stream, p, ctas);
  else locks_launch_pdl(kvq_join_kernel<LOCKS_KVQ_FLOAT>, rows, dim3(32 * kJoinWarps), 0, (cudaStream_t)stream, p, ctas);
  return locks_check_launch(ctx);
}
