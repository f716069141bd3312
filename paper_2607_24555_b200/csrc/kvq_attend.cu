// Attention over the 8-bit paged cache, for single tokens and a few tokens per request:
//   o_r = sum_i softmax_i(q_r . k_i s_k(i) sm_scale) v_i s_v(i)   over the tokens i that row r sees.
//
// Codes are whole numbers (or e4m3 numbers) that fp16 holds exactly, so both products run on the tensor cores in fp16: a query row goes
// in times a power of two that brings its largest element to 1 .. 2 (exact, and undone on the scores in fp32), a page's key scale
// is a factor of its 16 scores, and P V of a tile starts from zero and joins the fp32 output by one rounding multiply-add with the
// page's value scale, so that no scale meets fp16's range.  P is rounded to fp16 (2^-12 of each weight; the sum of the weights
// is that of the unrounded ones).  Scores, maxima, sums and outputs are fp32.
//
// A problem is a (request, KV head, row tile): up to 8 or 16 query rows, the G heads of one or several tokens.  The 16-token tiles of all problems
// form one line that is cut into equal shares, one per CTA, whatever the lengths: a CTA's share is a few segments of problems, and
// a problem that several CTAs share is put together by the last of them.  A warp streams every fourth tile of a segment from global
// memory straight into MMA fragments, a tile ahead: the order of dimensions in q k and of tokens and dimensions in p v is free, and is
// chosen such that a lane's bytes are 16-byte pieces of rows.
#include "kvq.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kRowPad = LOCKS_D + 4;   // floats of a row of a warp's partial
constexpr int kMinShare = 2 * kWarps;  // tiles of a share at least: two per warp

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

// One request's share of the line: its tokens, its length, tiles of a problem, problems (row tiles x KV heads)
struct Request { int T, n, row0, tiles, row_tiles; };

__device__ __forceinline__ Request request_at(const QAttParams &p, int b) {
  Request r;
  r.row0 = b;
  r.n = 1;
  r.T = p.c.seq_lens[b];
  if (p.cu) {
    r.row0 = p.cu[b];
    r.n = p.cu[b + 1] - r.row0;
    if (r.n < 0 || r.row0 < 0 || r.row0 > p.n - r.n) {   // rows that are not there
      set_status(p.status, LOCKS_ERR_BAD_BLOCK);
      r.n = 0;
    }
  }
  if (p.ids) {
    r.tiles = p.kbud << p.sub_shift;
  } else {
    int pages = r.T > 0 ? (r.T - 1) / p.c.B + 1 : 0;
    if (pages > p.c.Pmax) { set_status(p.status, LOCKS_ERR_BAD_BLOCK); pages = p.c.Pmax; }
    r.tiles = max(pages << p.sub_shift, 1);   // (an empty sequence's problem writes its zeros all the same)
  }
  r.row_tiles = (r.n + p.tile_tokens - 1) / p.tile_tokens;
  return r;
}

// The request that holds place u of the line: where its places begin.  All lanes of a warp take part.
__device__ __forceinline__ bool find_request(const QAttParams &p, int64_t u, int lane, int &b, int64_t &begin, Request &req) {
  int64_t before = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 32) {
    const int i = b0 + lane;
    Request r = {0, 0, 0, 0, 0};
    if (i < p.batch) r = request_at(p, i);
    const int64_t mine = (int64_t)r.tiles * r.row_tiles * p.Hkv;
    int64_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += x;
    }
    const int64_t at = before + sum - mine;
    const uint32_t has = __ballot_sync(0xffffffffu, u >= at && u < at + mine);
    if (has) {
      const int l = __ffs(has) - 1;
      b = b0 + l;
      begin = __shfl_sync(0xffffffffu, at, l);
      req.T = __shfl_sync(0xffffffffu, r.T, l); req.n = __shfl_sync(0xffffffffu, r.n, l); req.row0 = __shfl_sync(0xffffffffu, r.row0, l);
      req.tiles = __shfl_sync(0xffffffffu, r.tiles, l); req.row_tiles = __shfl_sync(0xffffffffu, r.row_tiles, l);
      return true;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  return false;
}
__device__ __forceinline__ int64_t line_length(const QAttParams &p, int lane) {
  int64_t all = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 32)
    if (b0 + lane < p.batch) {
      const Request r = request_at(p, b0 + lane);
      all += (int64_t)r.tiles * r.row_tiles * p.Hkv;
    }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
  return all;
}

__device__ __forceinline__ int64_t share_of(int64_t all) { return max((all + gridDim.x - 1) / (int64_t)gridDim.x, (int64_t)kMinShare); }

// largest finite magnitude over a warp -> the power of two that brings it to 2^top .. 2^(top + 1)
__device__ __forceinline__ float power_to(float amax, int top) {
  const int e = (int)(__float_as_uint(amax) >> 23) - 127;
  return amax < 1e-30f ? 1.f : __uint_as_float((uint32_t)(min(max(top - e, -126), 127) + 127) << 23);
}
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}

// The row tile's queries as A fragments: lane (x, t) holds four dims of row x (+ 8) per step, 64 (s / 4) + 16 t + 4 (s % 4) ..
// Returns 2^-e c2, which undoes the power of two.
template <int NH>
__device__ __forceinline__ void load_queries(const QAttParams &p, int64_t row0, int h, int rows, int x, int t, uint32_t (&qf)[NH][8][2], float (&rs)[NH]) {
#pragma unroll
  for (int hh = 0; hh < NH; ++hh) {
    const int r = x + 8 * hh, j = r / p.G, g = r - j * p.G;
    const __nv_bfloat16 *qr = p.q + ((row0 + j) * p.Hq + h * p.G + g) * LOCKS_D + 16 * t;
    uint4 w[4] = {};
    if (r < rows) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const uint4 *>(qr + (i >> 1) * 64 + 8 * (i & 1));
    }
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
    rs[hh] = p.c2 / up;
#pragma unroll
    for (int s = 0; s < 8; ++s) { qf[hh][s][0] = pack_f16(v[s][0] * up, v[s][1] * up); qf[hh][s][1] = pack_f16(v[s][2] * up, v[s][3] * up); }
  }
}

__device__ __forceinline__ void mma_f16_z(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// Running softmax of the row tile in a warp's registers
template <int NH>
struct Running {
  float m[NH], l[NH];   // row x (+ 8): maximum (log2 units), this lane's share of the sum
  float4 o[8][NH];      // dims 16 x + 2 i (.x, .y) and 16 x + 2 i + 1 (.z, .w) of rows 2 t, 2 t + 1 (+ 8)
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) {
      m[hh] = -INFINITY;
      l[hh] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i][hh] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  // Scores of tokens x, x + 8 of a tile -> weights of tokens 2 t, 2 t + 1, 8 + 2 t, 9 + 2 t (pw; as B fragments pb).  f[hh]: what
  // the sums of products stand for, in log2 units; pos: place of the tile's first token; mask: some row does not see all of it
  __device__ __forceinline__ void weights(const float (&s)[2][4], const float (&f)[NH], const int (&lim)[NH], int pos, bool mask, int t, uint32_t (&pb)[NH][2], float (&pw)[NH][4]) {
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) {
      float sv[4] = {s[0][2 * hh] * f[hh], s[0][2 * hh + 1] * f[hh], s[1][2 * hh] * f[hh], s[1][2 * hh + 1] * f[hh]};
      if (mask) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (pos + 2 * t + (e & 1) + 4 * (e & 2) >= lim[hh]) sv[e] = -INFINITY;
      }
      float mx = fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      const float mn = fmaxf(m[hh], mx), ms = mn == -INFINITY ? 0.f : mn;
      if (__any_sync(0xffffffffu, mn != m[hh])) {   // some row's maximum rose
        const float a = ex2f(m[hh] - ms);
        l[hh] *= a;
        const float a0 = __shfl_sync(0xffffffffu, a, 8 * t), a1 = __shfl_sync(0xffffffffu, a, 8 * t + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) { o[i][hh].x *= a0; o[i][hh].y *= a1; o[i][hh].z *= a0; o[i][hh].w *= a1; }
      }
      m[hh] = mn;
#pragma unroll
      for (int e = 0; e < 4; ++e) { pw[hh][e] = ex2f(sv[e] - ms); l[hh] += pw[hh][e]; }
      pb[hh][0] = pack_f16(pw[hh][0], pw[hh][1]);
      pb[hh][1] = pack_f16(pw[hh][2], pw[hh][3]);
    }
  }
  // Two dims' values of the tile's tokens join the outputs, times f (of rows 2 t, 2 t + 1)
  __device__ __forceinline__ void outputs(int i, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&pb)[NH][2], const float2 (&f)[NH]) {
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) {
      float c[4];
      mma_f16_z(c, a0, a1, a2, a3, pb[hh][0], pb[hh][1]);
      const float2 lo = fma2(make_float2(c[0], c[1]), f[hh], make_float2(o[i][hh].x, o[i][hh].y));
      const float2 hi = fma2(make_float2(c[2], c[3]), f[hh], make_float2(o[i][hh].z, o[i][hh].w));
      o[i][hh] = make_float4(lo.x, lo.y, hi.x, hi.y);
    }
  }
  // into the warp's partial: [rows][kRowPad] outputs, [rows] (max, sum); `times` over, joined to what is there
  __device__ __forceinline__ void leave(float *wo, float2 *wml, int x, int t, bool join, float times) {
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) {
      float sum = l[hh];
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      float f_old = 0.f, f_new = 1.f, mn = m[hh];
      sum *= times;
      if (join) {
        const float2 old = wml[x + 8 * hh];
        mn = fmaxf(old.x, m[hh]);
        f_old = mn == -INFINITY ? 1.f : ex2f(old.x - mn);
        f_new = mn == -INFINITY ? 1.f : ex2f(m[hh] - mn);
        sum = old.y * f_old + sum * f_new;
      }
      f_new *= times;
      __syncwarp();
      if (t == 0) wml[x + 8 * hh] = make_float2(mn, sum);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float fo = __shfl_sync(0xffffffffu, f_old, 8 * t + 4 * c), fn = __shfl_sync(0xffffffffu, f_new, 8 * t + 4 * c);
        float *w = wo + (2 * t + c + 8 * hh) * kRowPad + 16 * x;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          float4 y = c ? make_float4(o[i][hh].y, o[i][hh].w, o[i + 1][hh].y, o[i + 1][hh].w) : make_float4(o[i][hh].x, o[i][hh].z, o[i + 1][hh].x, o[i + 1][hh].z);
          if (join) {
            const float4 z = *reinterpret_cast<const float4 *>(w + 2 * i);
            y = make_float4(fmaf(y.x, fn, z.x * fo), fmaf(y.y, fn, z.y * fo), fmaf(y.z, fn, z.z * fo), fmaf(y.w, fn, z.w * fo));
          }
          *reinterpret_cast<float4 *>(w + 2 * i) = y;
        }
      }
    }
  }
};

// 16 places of the unfinished page (fp32), from pos on, joined to the warp's partial `times` over.  Elements go to fp16 by a power of
// two of the tile's largest (2^-11 of each).  Not part of the tile loop: its registers would be the loop's.
template <int NH>
__device__ __forceinline__ void tail_tile(const QAttParams &p, int64_t row0, int h, int rows, int T, const int (&lim)[NH], const float *kt, const float *vt, int pos, float times, float *wo, float2 *wml) {
  const int lane = threadIdx.x & 31, x = lane >> 2, t = lane & 3;
  uint32_t qf[NH][8][2], pb[NH][2];
  float rs[NH], pw[NH][4], s[2][4], f[NH];
  load_queries<NH>(p, row0, h, rows, x, t, qf, rs);
  Running<NH> run;
  run.clear();
  float4 k[2][8];
  float amax = 0.f;
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      k[w][i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (pos + x + 8 * w < T) k[w][i] = *reinterpret_cast<const float4 *>(kt + (x + 8 * w) * LOCKS_D + (i >> 2) * 64 + 16 * t + 4 * (i & 3));
      amax = fmaxf(amax, fmaxf(fmaxf(finite_abs(k[w][i].x), finite_abs(k[w][i].y)), fmaxf(finite_abs(k[w][i].z), finite_abs(k[w][i].w))));
    }
  float up = power_to(warp_max(amax), 14);
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    s[w][0] = s[w][1] = s[w][2] = s[w][3] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      mma_f16(s[w], qf[0][i][0], NH == 2 ? qf[NH - 1][i][0] : 0u, qf[0][i][1], NH == 2 ? qf[NH - 1][i][1] : 0u, pack_f16(k[w][i].x * up, k[w][i].y * up), pack_f16(k[w][i].z * up, k[w][i].w * up));
  }
#pragma unroll
  for (int hh = 0; hh < NH; ++hh) f[hh] = rs[hh] / up;
  run.weights(s, f, lim, pos, true, t, pb, pw);
  // values: 16 dims of tokens 2 t, 2 t + 1, 8 + 2 t, 9 + 2 t
  float4 v[4][4];
  amax = 0.f;
  bool odd = false;   // an infinity or a NaN
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int tok = 2 * t + (e & 1) + 4 * (e & 2);
      v[e][i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (pos + tok < T) v[e][i] = *reinterpret_cast<const float4 *>(vt + tok * LOCKS_D + 16 * x + 4 * i);
      const float a = fmaxf(fmaxf(finite_abs(v[e][i].x), finite_abs(v[e][i].y)), fmaxf(finite_abs(v[e][i].z), finite_abs(v[e][i].w)));
      amax = fmaxf(amax, a);
      odd |= !(fabsf(v[e][i].x) < INFINITY && fabsf(v[e][i].y) < INFINITY && fabsf(v[e][i].z) < INFINITY && fabsf(v[e][i].w) < INFINITY);
    }
  up = power_to(warp_max(amax), 14);
  if (!__any_sync(0xffffffffu, odd)) {
    float2 back[NH];
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) back[hh] = make_float2(1.f / up, 1.f / up);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      run.outputs(2 * i, pack_f16(v[0][i].x * up, v[1][i].x * up), pack_f16(v[0][i].y * up, v[1][i].y * up), pack_f16(v[2][i].x * up, v[3][i].x * up), pack_f16(v[2][i].y * up, v[3][i].y * up), pb, back);
      run.outputs(2 * i + 1, pack_f16(v[0][i].z * up, v[1][i].z * up), pack_f16(v[0][i].w * up, v[1][i].w * up), pack_f16(v[2][i].z * up, v[3][i].z * up), pack_f16(v[2][i].w * up, v[3][i].w * up), pb, back);
    }
  } else {   // token by token in fp32, so that a row takes nothing of a token that it does not see
#pragma unroll 1
    for (int k2 = 0; k2 < 16 && pos + k2 < T; ++k2) {
      const int e = (k2 & 1) + (k2 >> 3) * 2, from = (k2 & 7) >> 1;   // the weight's place: element e of the lanes with t = from
#pragma unroll
      for (int hh = 0; hh < NH; ++hh) {
        const float w = e == 0 ? pw[hh][0] : (e == 1 ? pw[hh][1] : (e == 2 ? pw[hh][2] : pw[hh][3]));
        const float w0 = __shfl_sync(0xffffffffu, w, 8 * t + from), w1 = __shfl_sync(0xffffffffu, w, 8 * t + 4 + from);
        const bool s0 = pos + k2 < __shfl_sync(0xffffffffu, lim[hh], 8 * t), s1 = pos + k2 < __shfl_sync(0xffffffffu, lim[hh], 8 * t + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 y = *reinterpret_cast<const float2 *>(vt + k2 * LOCKS_D + 16 * x + 2 * i);
          if (s0) { run.o[i][hh].x = fmaf(w0, y.x, run.o[i][hh].x); run.o[i][hh].z = fmaf(w0, y.y, run.o[i][hh].z); }
          if (s1) { run.o[i][hh].y = fmaf(w1, y.x, run.o[i][hh].y); run.o[i][hh].w = fmaf(w1, y.y, run.o[i][hh].w); }
        }
      }
    }
  }
  run.leave(wo, wml, x, t, true, times);
}

// Output rows: one row's four dims from its maximum, sum and unnormalised mean
__device__ __forceinline__ void finish_dims(const QAttParams &p, int64_t row, int d4, float4 a, float M, float L) {
  const float inv = L == 0.f ? 0.f : 1.f / L;   // (0: nothing seen)
  *reinterpret_cast<uint2 *>(p.out + row * LOCKS_D + d4) = make_uint2(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv));
  if (p.lse && d4 == 0) p.lse[row] = L == 0.f ? -INFINITY : ((M == -INFINITY ? 0.f : M) + log2f(L)) * kLn2;
}

// A warp's ring: tiles of 4 KB (keys, then values; 16 rows of 128 bytes).  16-byte pieces of a row are stored at piece ^ 4 (row % 2)
// (keys) and piece ^ 2 (row / 2 % 4) (values): then the eight lanes that read together, two rows' pieces 4 c .. 4 c + 3 (keys) or four
// rows' pieces 2 c, 2 c + 1 (values), touch every bank once.
constexpr int kTile = 2 * 16 * LOCKS_D;
template <int NH> constexpr int kStages = NH == 1 ? 3 : 6;
template <int NH> constexpr int kRing = kStages<NH> * kTile;
template <int NH> constexpr int token_smem() { return kWarps * kRing<NH> + 16; }
static_assert(kRing<1> >= 8 * (kRowPad * 4 + 8) && kRing<2> >= 16 * (kRowPad * 4 + 8), "a warp's partial takes its ring's place");
template <int NH> constexpr int kCtasPerSm = NH == 1 ? 4 : 2;

template <int NH, int FMT>
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
  const int64_t all = line_length(p, lane);
  const int64_t share = share_of(all);
  int64_t u = share * blockIdx.x;
  const int64_t u_end = min(u + share, all);
  int b = -1;
  int64_t begin = 0;
  Request req = {0, 0, 0, 0, 0};
  // 16-byte copies: copy i moves piece lane & 7 of row (lane >> 3) + 4 i
  const int cr = lane >> 3, cc = lane & 7;
  const uint32_t k_dst = cr * 128 + ((cc ^ (4 * (cr & 1))) << 4), v_dst = 2048 + cr * 128 + ((cc ^ (2 * (cr >> 1))) << 4);
  const int64_t c_off = (int64_t)cr * p.c.st + cc * 16;
  while (u < u_end) {
    if (b < 0 || u >= begin + (int64_t)req.tiles * req.row_tiles * p.Hkv)
      if (!find_request(p, u, lane, b, begin, req)) return;   // (not reached: u lies on the line)
    const int prob = (int)((u - begin) / req.tiles);            // problem of the request
    const int64_t prob_begin = begin + (int64_t)prob * req.tiles;
    const int seg0 = (int)(u - prob_begin), seg1 = (int)min((int64_t)req.tiles, u_end - prob_begin);
    const int h = prob % p.Hkv, rt = prob / p.Hkv, hkv = h / p.kvdiv, kv_heads = p.Hkv / p.kvdiv;
    const int j0 = rt * p.tile_tokens, toks = min(p.tile_tokens, req.n - j0), rows = toks * p.G;
    const int T = req.T, B = p.c.B, full_pages = T > 0 ? T / B : 0;
    int npages = 0;
    if (p.ids) {
      npages = p.cnt[(int64_t)b * p.Hkv + h];
      if (npages < 0 || npages > p.kbud) {
        if (tid == 0) set_status(p.status, LOCKS_ERR_BAD_BLOCK);
        npages = npages < 0 ? 0 : p.kbud;
      }
    }
    const int tiles_here = p.ids ? min(seg1, npages << p.sub_shift) : (T > 0 ? seg1 : 0);
    // ---- the segment's tiles: this warp's are seg0 + warp + 4 j
    const int first = seg0 + warp, sub_mask = (1 << p.sub_shift) - 1;
    const int mine = tiles_here > first ? (tiles_here - first + kWarps - 1) / kWarps : 0;
    // blocks and scales of 32 tiles at a time, a lane each.  block -1: nothing to read here (out of range, past the end); -2: the unfinished page
    int blk = -1, blk_next = -1, page_l = 0, page_next = 0;
    float ks_l = 0.f, vs_l = 0.f, ks_next = 0.f, vs_next = 0.f;
    uint64_t tails = 0;   // times that each 16-token part of the unfinished page is listed, 16 bits a part
    auto resolve = [&](int jb, int &bk, int &pg, float &ks, float &vs) {
      const int idx = first + (jb + lane) * kWarps;
      bk = -1; pg = 0; ks = vs = 0.f;
      if (idx < tiles_here) {
        pg = idx >> p.sub_shift;
        if (p.ids) pg = p.ids[((int64_t)b * p.Hkv + h) * p.kbud + pg];
        if (pg < 0 || pg >= p.c.Pmax) {
          set_status(p.status, LOCKS_ERR_BAD_BLOCK);
        } else if (pg < full_pages) {
          bk = p.c.block_table[(int64_t)b * p.c.Pmax + pg];
          if (bk < 0 || bk >= p.c.num_blocks) {
            bk = -1;
            set_status(p.status, LOCKS_ERR_BAD_BLOCK);
          } else {
            const int64_t at = (int64_t)bk * kv_heads + hkv;
            ks = p.c.ks[at];
            vs = p.c.vs[at];
          }
        } else if (pg == full_pages && pg * B + (idx & sub_mask) * 16 < T) {
          bk = -2;
        }
      }
    };
    resolve(0, blk, page_l, ks_l, vs_l);
    auto sub_of = [&](int j) { return (first + j * kWarps) & sub_mask; };
    auto issue = [&](int j, int bk) {
      if (j < mine && bk >= 0) {
        uint8_t *dst = ring + (j % S) * kTile;
        const int64_t off = (int64_t)bk * p.c.sb + (int64_t)hkv * p.c.sh + (int64_t)(sub_of(j) * 16) * p.c.st + c_off;
        const char *kp = p.c.k + off, *vp = p.c.v + off;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          copy16(dst + k_dst + 512 * i, kp + 4 * i * p.c.st);
          copy16(dst + (v_dst ^ (64 * (i & 1))) + 512 * i, vp + 4 * i * p.c.st);
        }
      }
      cp_async_commit();
    };
#pragma unroll
    for (int j = 0; j < S - 1; ++j) issue(j, __shfl_sync(0xffffffffu, blk, j));
    uint32_t qf[NH][8][2];
    float rs[NH];   // 2^e of the row, times sm_scale log2 e
    load_queries<NH>(p, req.row0 + j0, h, rows, x, t, qf, rs);
    int lim[NH];    // row x (+ 8) sees the first lim tokens
#pragma unroll
    for (int hh = 0; hh < NH; ++hh) lim[hh] = x + 8 * hh < rows ? T - req.n + j0 + (x + 8 * hh) / p.G + 1 : T;
    const int lim_min = T - req.n + j0 + 1;   // what the tile's first token sees
    Running<NH> run;
    run.clear();
#pragma unroll 1
    for (int j = 0; j < mine; ++j) {
      const int jn = j + S - 1;
      if ((jn & 31) == 16) resolve(jn + 16, blk_next, page_next, ks_next, vs_next);   // half a batch early
      const bool over = (jn & 31) < S - 1 && jn >= 32;   // tile j + S - 1 is of the next batch, tile j of this one
      issue(jn, __shfl_sync(0xffffffffu, over ? blk_next : blk, jn & 31));
      cp_async_wait<S - 1>();
      __syncwarp();
      const int bk = __shfl_sync(0xffffffffu, blk, j & 31), pos = __shfl_sync(0xffffffffu, page_l, j & 31) * B + sub_of(j) * 16;
      const float ks = __shfl_sync(0xffffffffu, ks_l, j & 31), vs = __shfl_sync(0xffffffffu, vs_l, j & 31);
      if (bk == -2) tails += 1ull << (16 * sub_of(j));
      if (bk >= 0) {
        const uint8_t *kt = ring + (j % S) * kTile, *vt = kt + 2048;
        float s[2][4];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const uint4 y = *reinterpret_cast<const uint4 *>(kt + (x + 8 * w) * 128 + (((4 * c + t) ^ (4 * (x & 1))) << 4));
            const uint32_t word[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int st = 4 * c + i;
              uint32_t lo, hi;
              kvq_halves<FMT>(kvq_flip<FMT>(word[i]), lo, hi);
              if (st == 0) mma_f16_z(s[w], qf[0][st][0], NH == 2 ? qf[NH - 1][st][0] : 0u, qf[0][st][1], NH == 2 ? qf[NH - 1][st][1] : 0u, lo, hi);
              else mma_f16(s[w], qf[0][st][0], NH == 2 ? qf[NH - 1][st][0] : 0u, qf[0][st][1], NH == 2 ? qf[NH - 1][st][1] : 0u, lo, hi);
            }
          }
        }
        uint32_t pb[NH][2];
        float pw[NH][4], f[NH];
        float2 fv[NH];
#pragma unroll
        for (int hh = 0; hh < NH; ++hh) { f[hh] = rs[hh] * ks; fv[hh] = make_float2(vs, vs); }
        const bool mask = pos + 16 > lim_min;
        run.weights(s, f, lim, pos, mask, t, pb, pw);
        if (mask) {   // rows that see nothing of the tile take nothing of it, not even a NaN that its scale may be
#pragma unroll
          for (int hh = 0; hh < NH; ++hh) {
            if (pos >= __shfl_sync(0xffffffffu, lim[hh], 8 * t)) fv[hh].x = 0.f;
            if (pos >= __shfl_sync(0xffffffffu, lim[hh], 8 * t + 4)) fv[hh].y = 0.f;
          }
        }
        uint4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tok = 2 * t + (e & 1) + 4 * (e & 2);
          v[e] = *reinterpret_cast<const uint4 *>(vt + tok * 128 + ((x ^ (2 * t)) << 4));
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          auto word = [&](int e) { return kvq_flip<FMT>(w == 0 ? v[e].x : (w == 1 ? v[e].y : (w == 2 ? v[e].z : v[e].w))); };
          const uint32_t a0 = word(0), a1 = word(1), a2 = word(2), a3 = word(3);
          uint32_t ha[4][2];   // [dim][token pair]
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const uint32_t lo = c ? a2 : a0, hi = c ? a3 : a1;
            kvq_halves<FMT>(__byte_perm(lo, hi, 0x5140), ha[0][c], ha[1][c]);
            kvq_halves<FMT>(__byte_perm(lo, hi, 0x7362), ha[2][c], ha[3][c]);
          }
          run.outputs(2 * w, ha[0][0], ha[1][0], ha[0][1], ha[1][1], pb, fv);
          run.outputs(2 * w + 1, ha[2][0], ha[3][0], ha[2][1], ha[3][1], pb, fv);
        }
      }
      if ((j & 31) == 31) { blk = blk_next; page_l = page_next; ks_l = ks_next; vs_l = vs_next; }
      __syncwarp();
    }
    // ---- the warps' partials
    cp_async_wait<0>();
    __syncwarp();
    run.leave(part_of(warp), ml_of(warp), x, t, false, 1.f);
    __syncwarp();
    for (int sub = 0; tails; ++sub, tails >>= 16) {
      if (!(tails & 0xffff)) continue;
      const int64_t at = (((int64_t)b * kv_heads + hkv) * B + 16 * sub) * LOCKS_D;
      tail_tile<NH>(p, req.row0 + j0, h, rows, T, lim, p.c.kt + at, p.c.vt + at, full_pages * B + 16 * sub, (float)(tails & 0xffff), part_of(warp), ml_of(warp));
      __syncwarp();
    }
    __syncthreads();
    const bool whole = seg0 == 0 && seg1 == req.tiles;
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
        finish_dims(p, row_of(r), d4, a, M, L);
      } else {
        __stcg(reinterpret_cast<float4 *>(p.part + ((int64_t)slot * KVQ_ROWS + r) * LOCKS_D + d4), a);
        if (d4 == 0) __stcg(p.part_ml + slot * KVQ_ROWS + r, make_float2(M, L));
      }
    }
    if (!whole) {   // the last of the problem's CTAs puts its partials together, in their order
      const int c0 = (int)(prob_begin / share), c1 = (int)((prob_begin + req.tiles - 1) / share);
      __threadfence();
      __syncthreads();
      if (tid == 0) last_s = atomicAdd(p.done + c0, 1) == c1 - c0;
      __syncthreads();
      if (last_s) {
        __threadfence();
        for (int i = tid; i < rows * (LOCKS_D / 4); i += kThreads) {
          const int r = i >> 5, d4 = 4 * (i & 31);
          float M = -INFINITY, L = 0.f;
          float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int c = c0; c <= c1; ++c) {
            const int s = 2 * c + (c == c0 ? 1 : 0);
            const float2 ml = __ldcg(p.part_ml + s * KVQ_ROWS + r);
            const float4 y = __ldcg(reinterpret_cast<const float4 *>(p.part + ((int64_t)s * KVQ_ROWS + r) * LOCKS_D + d4));
            const float mn = fmaxf(M, ml.x), fo = mn == -INFINITY ? 1.f : ex2f(M - mn), fn = mn == -INFINITY ? 1.f : ex2f(ml.x - mn);
            L = L * fo + ml.y * fn;
            a.x = a.x * fo + y.x * fn; a.y = a.y * fo + y.y * fn; a.z = a.z * fo + y.z * fn; a.w = a.w * fo + y.w * fn;
            M = mn;
          }
          finish_dims(p, row_of(r), d4, a, M, L);
        }
        if (tid == 0) p.done[c0] = 0;   // ready for the next launch
      }
    }
    __syncthreads();   // the partials' memory is the rings'
    u = prob_begin + seg1;
  }
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
  // 8 rows a tile where a request's rows fit on average, else 16
  const bool wide = p.G > 8 || (int64_t)num_tokens * p.G > (int64_t)8 * batch;
  p.tile_tokens = (wide ? 16 : 8) / p.G;
  int ctas = ctx->num_sms * (wide ? kCtasPerSm<2> : kCtasPerSm<1>);
  if (ctas > KVQ_SLOT_BOUND) ctas = KVQ_SLOT_BOUND;
  ctx->last_launches = 0;
#define KVQ_TOKEN(NH_, F_)                                                                                                            \
  do {                                                                                                                                \
    if (locks_attrs_needed(LOCKS_ATTR_KVQ + 2 * (NH_ - 1) + F_))                                                                      \
      cudaFuncSetAttribute(kvq_token_kernel<NH_, F_>, cudaFuncAttributeMaxDynamicSharedMemorySize, token_smem<NH_>());                \
    locks_launch_pdl(kvq_token_kernel<NH_, F_>, dim3(ctas), dim3(kThreads), token_smem<NH_>(), (cudaStream_t)stream, p);              \
  } while (0)
  if (!wide && kv->fmt == LOCKS_KVQ_INT) KVQ_TOKEN(1, LOCKS_KVQ_INT);
  else if (!wide) KVQ_TOKEN(1, LOCKS_KVQ_FLOAT);
  else if (kv->fmt == LOCKS_KVQ_INT) KVQ_TOKEN(2, LOCKS_KVQ_INT);
  else KVQ_TOKEN(2, LOCKS_KVQ_FLOAT);
#undef KVQ_TOKEN
  return locks_check_launch(ctx);
}
