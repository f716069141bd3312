// Rotary positions (one axis or several), and appends of new tokens to the paged caches with the rotation on the way.
//
// A pair (a, b) of a head's dimensions turns by the angle position x frequency: (a cos - b sin, a sin + b cos).  Angles are formed in
// fp64 turns (at position 10^6 the product's rounding to fp32 would be 0.03 rad), reduced to a fraction of a turn, and only then
// go to fp32; rows are turned in fp32 and rounded once.  (An fp32 row is within 5.6e-8 of the exact one, relative, where sines and cosines in
// fp64 would leave 4.2e-8; a bf16 row's rounding is 1.7e-3.)  A token's cosines and sines are worked out once, in shared memory, for
// all of its heads.
#include <algorithm>

#include "kvq.cuh"

namespace {

struct Rows {   // strides in elements
  const char *p;
  int64_t st, sh;
};

__device__ __forceinline__ float2 turn(int pos, float inv_freq) {
  double t = (double)pos * (double)inv_freq * 0.15915494309189533576888;   // turns: over 2 pi
  t -= rint(t);
  float s, c;
  sincospif((float)(t + t), &s, &c);
  return make_float2(c, s);
}

// eight consecutive dimensions
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float *v) {
  const uint4 w = *reinterpret_cast<const uint4 *>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const float *p, float *v) {
  const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float *v) {
  *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ void store8(float *p, const float *v) {
  reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// A head's 128 dimensions are eight units of 16: unit u < rot / 16 holds pairs 8 u .. 8 u + 7, the others what is not rotated.  A unit
// is two runs of eight dimensions; where they begin:
__device__ __forceinline__ void unit_runs(int u, int rot, int inter, int &lo, int &hi) {
  if (inter || u >= rot / 16) { lo = 16 * u; hi = lo + 8; }
  else { lo = 8 * u; hi = rot / 2 + lo; }
}
// A token's cosines and sines lie such that the eight units of a head read 16 bytes each side by side: pair f = 8 u + 2 e + c of the
// token at 16 e + 2 u + c.
__device__ __forceinline__ int turn_at(int f) { return 16 * ((f >> 1) & 3) + 2 * (f >> 3) + (f & 1); }
__device__ __forceinline__ void unit_turns(const float2 *token, int u, float2 (&cs)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float4 c = reinterpret_cast<const float4 *>(token)[8 * e + u];
    cs[2 * e] = make_float2(c.x, c.y);
    cs[2 * e + 1] = make_float2(c.z, c.w);
  }
}
// v: the runs' values, cs: cosines and sines of the unit's pairs
__device__ __forceinline__ void unit_turn(float (&v)[16], const float2 (&cs)[8], int inter) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = inter ? v[2 * i] : v[i], b = inter ? v[2 * i + 1] : v[8 + i];
    const float x = fmaf(a, cs[i].x, -b * cs[i].y), y = fmaf(a, cs[i].y, b * cs[i].x);
    if (inter) { v[2 * i] = x; v[2 * i + 1] = y; }
    else { v[i] = x; v[8 + i] = y; }
  }
}

// A unit's two runs as they lie in memory
template <typename T> struct Raw {
  static constexpr int N = sizeof(T) == 2 ? 1 : 2;   // 16-byte pieces of a run
  uint4 w[2 * N];
  __device__ __forceinline__ void load(const T *p, int lo, int hi) {
#pragma unroll
    for (int i = 0; i < N; ++i) { w[i] = reinterpret_cast<const uint4 *>(p + lo)[i]; w[N + i] = reinterpret_cast<const uint4 *>(p + hi)[i]; }
  }
  __device__ __forceinline__ void store(T *p, int lo, int hi) const {
#pragma unroll
    for (int i = 0; i < N; ++i) { reinterpret_cast<uint4 *>(p + lo)[i] = w[i]; reinterpret_cast<uint4 *>(p + hi)[i] = w[N + i]; }
  }
  __device__ __forceinline__ void get(float (&v)[16]) const {
    load8(reinterpret_cast<const T *>(&w[0]), v);
    load8(reinterpret_cast<const T *>(&w[N]), v + 8);
  }
  __device__ __forceinline__ void set(const float (&v)[16]) {
    store8(reinterpret_cast<T *>(&w[0]), v);
    store8(reinterpret_cast<T *>(&w[N]), v + 8);
  }
};

struct RopeParams {
  locks_rotary rot;
  const int32_t *positions, *cu;
  Rows q, qo, k, ko, v;      // ko: locks_rope only
  int n, Hq, Hk, Hv, batch;  // Hq, Hk, Hv: heads of each that this call takes (0: none)
  int tokens;                // of a CTA
  // the cache of locks_append_rows
  char *kc, *vc;
  int64_t sb, sh, st;
  const int32_t *block_table, *seq_lens;
  int num_blocks, Pmax, B;
  int32_t *status;
};

// A CTA of NT threads takes one token row (ONE), or up to kRopeTokens: NT / 8 heads at a time, each by eight threads of which one has a
// unit.  A thread fetches four units at a time, of four tokens (ONE: of four of its heads), while it turns the four before.  Bound by
// the chain of a few round trips when there are few tokens (lengths and offsets; block; and rows, which are fetched meanwhile), by
// memory when there are many.  8191 tokens of 32 + 8 heads are turned in 33 us (5.1 TB/s, 0.77 of a copy's bandwidth; 26 at all of it; fp32 72,
// 51 at all of it), 24 in 3 to 4; 4K tokens appended in 24.8 (4.8 TB/s; fp32 55 of 37), 32 in 3.5 to 4.4.
constexpr int kRopeThreads = 128, kRopeTokens = 16, kAhead = 4;

struct RowsShared {
  float2 cs[kRopeTokens][64];
  int64_t at[kRopeTokens];   // the token's row in the cache (elements), or -1
  int owner[kRopeTokens], pos[kRopeTokens];
};

template <typename T, bool APPEND, bool ONE, int NT>
__device__ __forceinline__ void rope_rows(const RopeParams &p, int cta, RowsShared &sm) {
  auto &cs_s = sm.cs;
  auto &at_s = sm.at;
  auto &owner_s = sm.owner;
  auto &pos_s = sm.pos;
  const int tid = threadIdx.x, row0 = cta * p.tokens, toks = ONE ? 1 : min(p.tokens, p.n - row0), half = p.rot.rot_dim / 2, u = tid & 7, inter = p.rot.interleaved;
  constexpr int kEach = NT / 64, kTurns = ONE ? 1 : (kRopeTokens + kEach - 1) / kEach;
  const int f = tid & 63, t0 = tid >> 6;   // this thread's frequency, for tokens t0, t0 + kEach, ..
  float inv = 0.f;
  int axis = 0;
  if (f < half) { inv = p.rot.inv_freq[f]; axis = p.rot.axis[f]; }
  int lo, hi;
  unit_runs(u, p.rot.rot_dim, inter, lo, hi);
  const int heads = p.Hq + p.Hk + p.Hv, hi_off = hi - lo;
  const bool mine = u < p.rot.rot_dim / 16;
  // Units in batches of kAhead: of head (tid >> 3) + NT / 8 pass, tokens t .. t + kAhead - 1; ONE: of the token's heads of kAhead passes
  const int passes = (heads + NT / 8 - 1) / (NT / 8), slots = ONE ? kAhead : (toks + kAhead - 1) / kAhead * kAhead;
  struct Batch {
    int pass, t;
    __device__ __forceinline__ void on(int slots) {
      if (ONE || (t += kAhead) == slots) { t = 0; pass += ONE ? kAhead : 1; }
    }
  };
  auto head_of = [&](const Batch &k, int i) { return (tid >> 3) + NT / 8 * (ONE ? k.pass + i : k.pass); };
  auto token_of = [&](const Batch &k, int i) { return ONE ? 0 : k.t + i; };
  struct Line { const char *p; int64_t st; };   // a head's row of the CTA's first token (values are chosen: a reference chosen would be fetched lane by lane)
  auto source = [&](int h) {
    const bool q = h < p.Hq, k = !q && h < p.Hq + p.Hk;
    const int64_t st = q ? p.q.st : (k ? p.k.st : p.v.st), sh = q ? p.q.sh : (k ? p.k.sh : p.v.sh);
    return Line{(q ? p.q.p : (k ? p.k.p : p.v.p)) + (row0 * st + (h - (q ? 0 : (k ? p.Hq : p.Hq + p.Hk))) * sh + lo) * (int64_t)sizeof(T), st * (int64_t)sizeof(T)};
  };
  Raw<T> x[2][kAhead];
  Batch from = {0, 0}, to = {0, 0};
  auto fetch = [&](Raw<T> (&y)[kAhead]) {
    const Batch k = from;
    from.on(slots);
    Line l = source(head_of(k, 0));
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (ONE && i) l = source(head_of(k, i));
      if (head_of(k, i) < heads && token_of(k, i) < toks) y[i].load(reinterpret_cast<const T *>(l.p + token_of(k, i) * l.st), 0, hi_off);
    }
  };
  int pos[kTurns];
  if (p.positions && f < half) {
#pragma unroll
    for (int i = 0; i < kTurns; ++i) pos[i] = t0 + kEach * i < toks ? p.positions[(int64_t)axis * p.n + row0 + t0 + kEach * i] : 0;
  }
  if (APPEND) {
    // whose rows these are: the request with cu[b] <= row < cu[b + 1]
    if (tid < kRopeTokens) owner_s[tid] = -1;
    __syncthreads();
    if (!p.cu) {
      if (tid < toks) {
        const int len = p.seq_lens[row0 + tid];
        pos_s[tid] = len - 1;
        if (len != 0) owner_s[tid] = row0 + tid;   // (a length of zero: no token)
      }
    } else {
      for (int b = tid; b < p.batch; b += NT) {
        const int c0 = p.cu[b], c1 = p.cu[b + 1], len = p.seq_lens[b];
        for (int t = max(c0 - row0, 0); t < min(c1 - row0, toks); ++t) {
          owner_s[t] = b;
          pos_s[t] = c1 - c0 > len ? -1 : (int)max((int64_t)len - c1 + row0 + t, (int64_t)-1);
        }
      }
    }
  }
  fetch(x[0]);
  if (APPEND) {
    __syncthreads();
    if (tid < toks) {
      int64_t at = -1;
      if (owner_s[tid] >= 0 && p.Hk) {   // (else a row behind the last request's)
        const int place = pos_s[tid], page = place < 0 ? -1 : place / p.B;
        int block = -1;
        if (page >= 0 && page < p.Pmax) block = p.block_table[(int64_t)owner_s[tid] * p.Pmax + page];
        if (block >= 0 && block < p.num_blocks) at = (int64_t)block * p.sb + (int64_t)(place - page * p.B) * p.st;
        else set_status(p.status, LOCKS_ERR_BAD_BLOCK);
      }
      at_s[tid] = at;
    }
    if (!p.positions && f < half) {
#pragma unroll
      for (int i = 0; i < kTurns; ++i) pos[i] = t0 + kEach * i < toks ? pos_s[t0 + kEach * i] : 0;
    }
  }
  if (f < half) {
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
      if (t0 + kEach * i < toks) cs_s[t0 + kEach * i][turn_at(f)] = turn(pos[i], inv);
  }
  __syncthreads();
  auto give = [&](Raw<T> (&y)[kAhead]) {
    const Batch k = to;
    to.on(slots);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = head_of(k, i), t = token_of(k, i);
      if (h >= heads || t >= toks || (APPEND && owner_s[t] < 0)) continue;
      const bool q = h < p.Hq, key = h < p.Hq + p.Hk;
      if (mine && key) {
        float v[16];
        float2 cs[8];
        y[i].get(v);
        unit_turns(cs_s[t], u, cs);
        unit_turn(v, cs, inter);
        y[i].set(v);
      }
      T *d;
      if (q || !APPEND) {
        d = reinterpret_cast<T *>(const_cast<char *>(q ? p.qo.p : p.ko.p)) + (int64_t)(row0 + t) * (q ? p.qo.st : p.ko.st) + (h - (q ? 0 : p.Hq)) * (q ? p.qo.sh : p.ko.sh);
      } else {
        if (at_s[t] < 0) continue;
        d = reinterpret_cast<T *>(key ? p.kc : p.vc) + at_s[t] + (h - p.Hq - (key ? 0 : p.Hk)) * p.sh;
      }
      y[i].store(d + lo, 0, hi_off);
    }
  };
#pragma unroll 1
  while (true) {
    if (from.pass < passes) fetch(x[1]);
    give(x[0]);
    if (to.pass >= passes) break;
    if (from.pass < passes) fetch(x[0]);
    give(x[1]);
    if (to.pass >= passes) break;
  }
}

template <typename T, bool APPEND, bool ONE>
__global__ void __launch_bounds__(kRopeThreads) rope_rows_kernel(const __grid_constant__ RopeParams p) {
  __shared__ __align__(16) RowsShared sm;
  pdl_trigger();
  pdl_wait();
  rope_rows<T, APPEND, ONE, kRopeThreads>(p, blockIdx.x, sm);
}

// ------------------------------------------------------------------------------------------------ the 8-bit cache
struct QAppendParams {
  RopeParams r;    // rotation, positions, offsets, rows; its Hq heads of queries alone
  int q_ctas;      // the first CTAs take the query rows
  KvqCache c;
  int32_t *status;
};

constexpr int kMostTokens = 1 << 30;   // places stay far from 32 bits' end
constexpr int kQWarps = 8, kQThreads = kQWarps * 32;

__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
// x / scale, rounded to nearest: the product with the rounded reciprocal, and one correction by the remainder (Markstein 1990), which
// a multiply-add gives exactly
__device__ __forceinline__ float quotient(float x, float scale, float inv) {
  const float q = x * inv;
  return fmaf(fmaf(-q, scale, x), inv, q);
}
template <int FMT> __device__ __forceinline__ uint32_t code4(const float *v, float scale, float inv) {   // rounded to even
  float q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = quotient(v[i], scale, inv);
  if (FMT == LOCKS_KVQ_INT) {   // (at most 127 and a rounding)
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = (uint32_t)__float2int_rn(q[i]);
    return __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
  }
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(q[1]), "f"(q[0]));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(q[3]), "f"(q[2]));
  return (uint32_t)lo | (uint32_t)hi << 16;
}

// Query rows, and a CTA per (request, page that gets tokens and is complete afterwards), all KV heads; the first of a request's also takes
// its unfinished last page, whose tokens replace the tail that the first page has been put together from.  A warp has 16 tokens of a
// head's keys or values in registers (a lane: a unit of four tokens), so that the largest magnitude is known before a code is
// written and everything is read once; pages of 32 and 64 tokens are two and four warps'
// work.  The CTA's cosines and sines serve all heads.  Twelve prompts of 1.1K tokens on average with 32 heads of queries: 73 us (4.3 TB/s; 48 at a
// copy's bandwidth), signed codes 75, in pages of 32 and 64 tokens 82 and 99 (fewer CTAs, and a head's turn after the other); 8 single tokens 6.3 to 6.9.
// EARLY (where offsets are given, so that pages get many tokens): the first round's rows are fetched before the cosines are worked out (12
// prompts together: 82 to 73 us; one token per request, where it would wait for nothing, 6.3 to 6.9 from the registers that it costs).
template <int FMT, bool EARLY>
__global__ void __launch_bounds__(kQThreads, 2) kvq_append_kernel(const __grid_constant__ QAppendParams a) {
  extern __shared__ __align__(16) float2 cs_s[];   // [B][64]
  __shared__ int found_s[5];         // request, item of it, first row, new tokens, length
  __shared__ int warp_s[kQWarps];
  __shared__ uint32_t amax_s[kQWarps];
  pdl_trigger();
  pdl_wait();
  const RopeParams &p = a.r;
  if ((int)blockIdx.x < a.q_ctas) {
    if (p.tokens == 1) rope_rows<__nv_bfloat16, true, true, kQThreads>(p, blockIdx.x, *reinterpret_cast<RowsShared *>(cs_s));
    else rope_rows<__nv_bfloat16, true, false, kQThreads>(p, blockIdx.x, *reinterpret_cast<RowsShared *>(cs_s));
    return;
  }
  const KvqCache &c = a.c;
  // this thread's frequency (fetched lane by lane, so once)
  const int f = threadIdx.x & 63;
  float inv_freq = 0.f;
  int axis = 0;
  if (f < p.rot.rot_dim / 2) { inv_freq = p.rot.inv_freq[f]; axis = p.rot.axis[f]; }
  const int cta = blockIdx.x - a.q_ctas, ctas = gridDim.x - a.q_ctas;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = c.B;
  const int half = p.rot.rot_dim / 2, u = lane & 7, inter = p.rot.interleaved;
  int lo, hi;
  unit_runs(u, p.rot.rot_dim, inter, lo, hi);
  const bool mine = u < p.rot.rot_dim / 16;
  int b = cta, item = 0, row0 = b, n = 1;
  if (p.cu) {
    // the request that this CTA's item belongs to: a running sum of the requests' items
    if (tid == 0) found_s[0] = -1;
    int before = 0;
    for (int b0 = 0; b0 < p.batch; b0 += kQThreads) {
      const int i = b0 + tid;
      int items = 0, c0 = 0, m = 0, T = 0;
      if (i < p.batch) {
        c0 = p.cu[i];
        m = p.cu[i + 1] - c0;
        T = c.seq_lens[i];
        if (m != 0 && (m < 0 || m > T || T > kMostTokens || c0 < 0 || c0 > p.n - m)) {
          set_status(a.status, LOCKS_ERR_BAD_BLOCK);
          m = 0;
        }
        if (m > 0) items = max(1, T / B - (T - m) / B);   // (at most one more than p.n / B)
      }
      int sum = items;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += x;
      }
      if (lane == 31) warp_s[warp] = sum;
      __syncthreads();
      int all = 0;
#pragma unroll
      for (int w = 0; w < kQWarps; ++w) {
        if (w < warp) sum += warp_s[w];
        all += warp_s[w];
      }
      const int at = cta - before - (sum - items);
      if (at >= 0 && at < items) { found_s[0] = i; found_s[1] = at; found_s[2] = c0; found_s[3] = m; found_s[4] = T; }
      before += all;
      __syncthreads();
      if (before > cta && cta + 1 < ctas) break;   // (the last CTA looks at every request)
    }
    if (cta + 1 == ctas && before > ctas && tid == 0) set_status(a.status, LOCKS_ERR_BAD_BLOCK);   // offsets that go back: some items have no CTA
    if (found_s[0] < 0) return;
    b = found_s[0]; item = found_s[1]; row0 = found_s[2]; n = found_s[3];
  }
  const int T = p.cu ? found_s[4] : c.seq_lens[b];
  if (T < n || T > kMostTokens) {   // (one token per request: none at a length of zero)
    if (tid == 0 && T != 0) set_status(a.status, LOCKS_ERR_BAD_BLOCK);
    return;
  }
  const int start = T - n;
  const int sub_shift = B == 64 ? 2 : (B == 32 ? 1 : 0);   // a page is 2^sub_shift warps' work
  const int p0 = start / B, last = T / B;
  // keep: a page's rows into the tail, and nothing else
  auto do_page = [&](int page, bool keep) {
    const int first = page * B, t0 = max(first, start), t1 = min(first + B, T);
    const bool complete = !keep && first + B <= T;
    const int tasks = 2 * c.Hkv, per_round = kQWarps >> sub_shift, sub = warp & ((1 << sub_shift) - 1), at0 = first + 16 * sub + (lane >> 3);
    auto row_at = [&](int task, int pos) {
      const bool key = !(task & 1);
      return reinterpret_cast<const __nv_bfloat16 *>(key ? p.k.p : p.v.p) + (int64_t)(row0 + pos - start) * (key ? p.k.st : p.v.st) + (int64_t)(task >> 1) * (key ? p.k.sh : p.v.sh);
    };
    Raw<__nv_bfloat16> raw[4];
    auto fetch = [&](int task) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int pos = at0 + 4 * i;
        if (task < tasks && pos >= t0 && pos < t1) raw[i].load(row_at(task, pos), lo, hi);
      }
    };
    if (EARLY) fetch(warp >> sub_shift);
    if (f < half)
      for (int t = t0 + (tid >> 6); t < t1; t += kQThreads / 64) {
        const int row = row0 + t - start;
        cs_s[(t - t0) * 64 + turn_at(f)] = turn(p.positions ? p.positions[(int64_t)axis * p.n + row] : t, inv_freq);
      }
    int block = -1;
    if (complete) {
      if (page < c.Pmax) block = c.block_table[(int64_t)b * c.Pmax + page];
      if (block < 0 || block >= c.num_blocks) {
        block = -1;
        if (tid == 0) set_status(a.status, LOCKS_ERR_BAD_BLOCK);
      }
    }
    const bool fits = page < c.Pmax;
    if (!fits && !complete && tid == 0) set_status(a.status, LOCKS_ERR_BAD_BLOCK);
    auto turned = [&](float (&x)[16], int t) {   // t: token of this page's new ones
      float2 cs[8];
      unit_turns(cs_s + t * 64, u, cs);
      unit_turn(x, cs, inter);
    };
    // ---- keys and values
    __syncthreads();   // the cosines are there
    for (int r = 0; r < tasks; r += per_round) {
      if (EARLY && r) fetch(r + (warp >> sub_shift));
      const int task = r + (warp >> sub_shift), h = task >> 1;
      const bool live = task < tasks, key = !(task & 1);
      float *tail = (key ? c.kt : c.vt) + c.tail_at(b, h, page);
      float x[4][16];
      float top = 0.f;
      if (live) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int pos = at0 + 4 * i;
          if (pos < t0) {
            if (complete) { load8(tail + (pos - first) * LOCKS_D + lo, x[i]); load8(tail + (pos - first) * LOCKS_D + hi, x[i] + 8); }
          } else if (pos < t1) {
            if (EARLY) {
              raw[i].get(x[i]);
            } else {
              const __nv_bfloat16 *s = row_at(task, pos);
              load8(s + lo, x[i]);
              load8(s + hi, x[i] + 8);
            }
          }
        }
      }
      if (live && key && mine) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int pos = at0 + 4 * i;
          if (pos >= t0 && pos < t1) turned(x[i], pos - t0);
        }
      }
      if (complete) {
        if (live) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = max_nan(top, fabsf(x[i][e]));
        }
        uint32_t amax = __reduce_max_sync(0xffffffffu, __float_as_uint(top));   // (as whole numbers in the order of magnitudes, NaN last)
        if (sub_shift) {
          if (lane == 0) amax_s[warp] = amax;
          __syncthreads();
          const int w0 = warp & ~((1 << sub_shift) - 1);
          for (int w = 0; w < 1 << sub_shift; ++w) amax = max(amax, amax_s[w0 + w]);
          __syncthreads();
        }
        if (live && block >= 0) {
          float scale = __fdiv_rn(__uint_as_float(amax), FMT == LOCKS_KVQ_INT ? 127.f : 448.f);
          const bool codes = amax >= KVQ_TINY_BITS && amax < 0x7f800000u;
          if (!codes) scale = amax < KVQ_TINY_BITS ? 0.f : __uint_as_float(0x7fffffffu);
          const float inv = 1.f / scale;
          char *dst = (key ? c.k : c.v) + (int64_t)block * c.sb + (int64_t)h * c.sh;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            char *d = dst + (int64_t)(16 * sub + 4 * i + (lane >> 3)) * c.st;
            const uint2 a = codes ? make_uint2(code4<FMT>(x[i], scale, inv), code4<FMT>(x[i] + 4, scale, inv)) : make_uint2(0, 0);
            const uint2 c = codes ? make_uint2(code4<FMT>(x[i] + 8, scale, inv), code4<FMT>(x[i] + 12, scale, inv)) : make_uint2(0, 0);
            *reinterpret_cast<uint2 *>(d + lo) = a;
            *reinterpret_cast<uint2 *>(d + hi) = c;
          }
          if (lane == 0 && sub == 0) (key ? c.ks : c.vs)[(int64_t)block * c.Hkv + h] = scale;
        }
      }
      // (a page that is complete keeps its rows where the tail has two pages, so that the sequence may be shortened into it: 12 prompts
      // 72.7 us with one page, 78.4 with two, single tokens 6.4 and 6.6)
      if (live && fits && (!complete || (c.tail_pages == 2 && page == p0 && page == last - 1))) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int pos = at0 + 4 * i;
          if (pos >= t0 && pos < t1) { store8(tail + (pos - first) * LOCKS_D + lo, x[i]); store8(tail + (pos - first) * LOCKS_D + hi, x[i] + 8); }
        }
      }
    }
  };
  if (!EARLY) {   // a single token: its page, and none behind it that has tokens
    do_page(p0, false);
    return;
  }
  bool keep = false;
#pragma unroll 1
  for (int page = p0 + item;;) {
    do_page(page, keep);
    if (item || last == p0) break;
    if (c.tail_pages == 2 && page == p0 && last - 1 != p0) { page = last - 1; keep = true; }
    else if (page != last && T % B) { page = last; keep = false; }
    else break;
    __syncthreads();   // the tail's old tokens have been read, the cosines used
  }
}

// ------------------------------------------------------------------------------------------------ host
int rows_ok(const locks_ctx *c, const locks_rows *r) {
  if (!r->p || (uintptr_t)r->p % 16) return 0;
  const int64_t m = c->cfg.kv_dtype == LOCKS_BF16 ? 8 : 4;
  return r->stride_token % m == 0 && r->stride_head % m == 0;
}
Rows rows(const locks_rows *r) {
  return r ? Rows{reinterpret_cast<const char *>(r->p), r->stride_token, r->stride_head} : Rows{nullptr, 0, 0};
}

int rotary_ok(const locks_rotary *r) {
  if (r->rot_dim < 16 || r->rot_dim > LOCKS_D || r->rot_dim % 16 || r->num_axes < 1 || r->num_axes > LOCKS_MAX_AXES) return LOCKS_ERR_INVALID_ARG;
  if (r->interleaved != 0 && r->interleaved != 1) return LOCKS_ERR_INVALID_ARG;
  for (int i = 0; i < r->rot_dim / 2; ++i)
    if (r->axis[i] >= r->num_axes || !std::isfinite(r->inv_freq[i])) return LOCKS_ERR_INVALID_ARG;
  return LOCKS_OK;
}

// what the two appends check alike
int append_ok(const locks_ctx *c, const locks_rotary *rot, const int32_t *cu, int n, const locks_rows *q, const locks_rows *qo,
              const locks_rows *k, const locks_rows *v, int batch) {
  if (!c || !k || !v || !rows_ok(c, k) || !rows_ok(c, v) || n < 1 || (!cu && n != batch)) return LOCKS_ERR_INVALID_ARG;
  if ((q == nullptr) != (qo == nullptr) || (q && (!rot || !rows_ok(c, q) || !rows_ok(c, qo)))) return LOCKS_ERR_INVALID_ARG;
  return rot ? rotary_ok(rot) : LOCKS_OK;
}

// Token rows a CTA: one while there are CTAs to spare, then so many that all CTAs are there at once (a chain of lengths, blocks and
// angles is paid once for all of a CTA's), up to sixteen
int rows_per_cta(const locks_ctx *c, int n) { return std::min((n - 1) / (4 * c->num_sms) + 1, kRopeTokens); }
template <bool APPEND> void launch_rows(locks_ctx *c, RopeParams &p, cudaStream_t st) {
  p.tokens = rows_per_cta(c, p.n);
  const dim3 grid((p.n - 1) / p.tokens + 1), block(kRopeThreads);
  const bool bf = c->cfg.kv_dtype == LOCKS_BF16;
  if (p.tokens == 1 && bf) locks_launch_pdl(rope_rows_kernel<__nv_bfloat16, APPEND, true>, grid, block, 0, st, p);
  else if (p.tokens == 1) locks_launch_pdl(rope_rows_kernel<float, APPEND, true>, grid, block, 0, st, p);
  else if (bf) locks_launch_pdl(rope_rows_kernel<__nv_bfloat16, APPEND, false>, grid, block, 0, st, p);
  else locks_launch_pdl(rope_rows_kernel<float, APPEND, false>, grid, block, 0, st, p);
}

}  // namespace

extern "C" int locks_rope(locks_ctx *ctx, const locks_rotary *rot, const int32_t *positions, int num_tokens, const locks_rows *q,
                          const locks_rows *q_out, const locks_rows *k, const locks_rows *k_out, locks_stream stream) {
  if (!ctx || !rot || !positions || num_tokens < 1) return LOCKS_ERR_INVALID_ARG;
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr) || (!q && !k)) return LOCKS_ERR_INVALID_ARG;
  for (const locks_rows *r : {q, q_out, k, k_out})
    if (r && !rows_ok(ctx, r)) return LOCKS_ERR_INVALID_ARG;
  int rc = rotary_ok(rot);
  if (rc != LOCKS_OK) return rc;
  RopeParams p = {};
  p.rot = *rot; p.positions = positions; p.n = num_tokens;
  p.q = rows(q); p.qo = rows(q_out); p.k = rows(k); p.ko = rows(k_out);
  p.Hq = q ? ctx->cfg.num_q_heads : 0; p.Hk = k ? ctx->cfg.num_kv_heads : 0;
  ctx->last_launches = 0;
  launch_rows<false>(ctx, p, (cudaStream_t)stream);
  return locks_check_launch(ctx);
}

extern "C" int locks_append_rows(locks_ctx *ctx, const locks_rotary *rot, const int32_t *positions, const int32_t *cu_tokens, int num_tokens,
                            const locks_rows *q, const locks_rows *q_out, const locks_rows *k_new, const locks_rows *v_new,
                            const locks_kv *kv, int batch, locks_stream stream) {
  if (!ctx || !kv || !kv->k || !kv->v || !kv->block_table || !kv->seq_lens) return LOCKS_ERR_INVALID_ARG;
  if (batch <= 0 || batch > ctx->cfg.max_batch || kv->num_blocks <= 0) return LOCKS_ERR_INVALID_ARG;
  if (kv->stride_block <= 0 || kv->stride_head <= 0 || kv->stride_token < LOCKS_D) return LOCKS_ERR_INVALID_ARG;
  if ((kv->stride_block | kv->stride_head | kv->stride_token) % (ctx->cfg.kv_dtype == LOCKS_BF16 ? 8 : 4)) return LOCKS_ERR_INVALID_ARG;
  if (((uintptr_t)kv->k | (uintptr_t)kv->v) % 16) return LOCKS_ERR_INVALID_ARG;
  int rc = append_ok(ctx, rot, cu_tokens, num_tokens, q, q_out, k_new, v_new, batch);
  if (rc != LOCKS_OK) return rc;
  RopeParams p = {};
  if (rot) p.rot = *rot;
  p.positions = positions; p.cu = cu_tokens; p.n = num_tokens; p.batch = batch;
  p.q = rows(q); p.qo = rows(q_out); p.k = rows(k_new); p.v = rows(v_new);
  p.Hq = q ? ctx->cfg.num_q_heads : 0; p.Hk = p.Hv = ctx->cfg.num_kv_heads;
  p.kc = reinterpret_cast<char *>(kv->k); p.vc = reinterpret_cast<char *>(kv->v);
  p.sb = kv->stride_block; p.sh = kv->stride_head; p.st = kv->stride_token;
  p.block_table = kv->block_table; p.seq_lens = kv->seq_lens; p.num_blocks = kv->num_blocks; p.Pmax = ctx->Pmax; p.B = ctx->B;
  p.status = ctx->status;
  ctx->last_launches = 0;
  launch_rows<true>(ctx, p, (cudaStream_t)stream);
  return locks_check_launch(ctx);
}

extern "C" int locks_kvq_append(locks_ctx *ctx, const locks_rotary *rot, const int32_t *positions, const int32_t *cu_tokens, int num_tokens,
                                const locks_rows *q, const locks_rows *q_out, const locks_rows *k_new, const locks_rows *v_new,
                                const locks_kvq *kv, int batch, locks_stream stream) {
  int rc = kvq_check(ctx, kv, batch);
  if (rc != LOCKS_OK) return rc;
  if ((rc = append_ok(ctx, rot, cu_tokens, num_tokens, q, q_out, k_new, v_new, batch)) != LOCKS_OK) return rc;
  QAppendParams a = {};
  RopeParams &p = a.r;
  if (rot) p.rot = *rot;
  p.positions = positions; p.cu = cu_tokens; p.n = num_tokens; p.batch = batch;
  p.q = rows(q); p.qo = rows(q_out); p.k = rows(k_new); p.v = rows(v_new);
  p.Hq = q ? ctx->cfg.num_q_heads : 0;
  p.seq_lens = kv->seq_lens; p.B = ctx->B; p.Pmax = ctx->Pmax; p.status = ctx->status;
  p.tokens = rows_per_cta(ctx, num_tokens);
  a.q_ctas = q ? (num_tokens - 1) / p.tokens + 1 : 0;
  a.c = kvq_cache(ctx, kv); a.status = ctx->status;
  // a request with m new tokens completes at most (m + B - 1) / B pages, and has an item at least
  const int64_t grid = (cu_tokens ? (int64_t)num_tokens / ctx->B + batch : batch) + a.q_ctas;
  if (grid > INT32_MAX) return LOCKS_ERR_TOO_LARGE;
  const size_t smem = std::max((size_t)ctx->B * 64 * sizeof(float2), sizeof(RowsShared));
  ctx->last_launches = 0;
#define KVQ_APPEND(F_, E_) \
  if (kv->fmt == F_ && (cu_tokens != nullptr) == E_) locks_launch_pdl(kvq_append_kernel<F_, E_>, dim3((unsigned)grid), dim3(kQThreads), smem, (cudaStream_t)stream, a)
  KVQ_APPEND(LOCKS_KVQ_INT, false);
  KVQ_APPEND(LOCKS_KVQ_INT, true);
  KVQ_APPEND(LOCKS_KVQ_FLOAT, false);
  KVQ_APPEND(LOCKS_KVQ_FLOAT, true);
#undef KVQ_APPEND
  return locks_check_launch(ctx);
}
