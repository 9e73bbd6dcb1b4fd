// Log-probabilities of given tokens, the entropy and the most likely alternatives of rows of logits, and the gradient of
// the first two into the logits.
//
//   z_i = x_i / T,  m = max_i x_i,  r = sum over i, without one occurrence of the maximum, of exp((x_i - m) / T)
//   L = log(1 + r),  log p_i = (x_i - m) / T - L
//   H = -sum_i p_i log p_i = L - sum_i exp((x_i - m) / T) (x_i - m) / T / (1 + r)
//   d x_i = (1 / T) ( g (delta_it - p_i) - h p_i (log p_i + H) )          g = d log p_t, h = d H
// The maximum's own 1 is kept out of r, so that log1p(r) is exact to fp32 for a row that is nearly sure of one token.
//
// Forward: one pass over the row, 16 bytes a load, four loads (a batch) in flight per thread.  A thread keeps a running maximum,
// moved once per batch, and its sums of e and e (x - m) relative to it; the block (and, for few rows, the up to eight
// blocks of a cluster that share a row) joins them at the end.  The alternatives cost no second pass: the k-th largest of
// the threads' own maxima is a lower bound of the k-th largest logit, so only the few threads whose maximum reaches it can
// hold one, and their warps read again out of L2 the batch of four vectors that held such a thread's maximum, or all its elements
// if another batch reaches the bound too.  The same re-reading makes r exact when it is
// small: only the thread that holds the maximum added it to anything.
#pragma once
#include "common.cuh"

namespace hift {

constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2E = 1.4426950408889634f, kLogLn2 = 0.6931471805599453f;
constexpr int kLpMaxTop = 32;
constexpr int kLpCand = 512;              // alternatives a block can collect before it falls back to whole passes
constexpr int kLpBatch = 4;
constexpr int kLpThreads = 256;           // at most, of a block

__device__ __forceinline__ float lp_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 16 bytes of logits: V elements as V / 2 pairs
template <typename T> struct LpVec;
template <> struct LpVec<float> {
  static constexpr int V = 4;
  __device__ static uint4 missing() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
  __device__ static float max(const uint4& v) { return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w))); }
  __device__ static void pairs(const uint4& v, float (&a)[2], float (&b)[2]) {
    a[0] = __uint_as_float(v.x); b[0] = __uint_as_float(v.y); a[1] = __uint_as_float(v.z); b[1] = __uint_as_float(v.w);
  }
  __device__ static uint4 join(const float (&a)[2], const float (&b)[2]) {
    return make_uint4(__float_as_uint(a[0]), __float_as_uint(b[0]), __float_as_uint(a[1]), __float_as_uint(b[1]));
  }
};
template <> struct LpVec<bf16> {
  static constexpr int V = 8;
  __device__ static uint4 missing() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
  __device__ static float max(const uint4& v) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
  }
  __device__ static void pairs(const uint4& v, float (&a)[4], float (&b)[4]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { a[i] = __uint_as_float(w[i] << 16); b[i] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  __device__ static uint4 join(const float (&a)[4], const float (&b)[4]) {
    uint4 v;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(a[i], b[i]);
    return v;
  }
};

// A row as 16-byte vectors: `head` elements before the first aligned address, nv vectors, the rest.  The up to 2 (V - 1)
// single elements outside the vectors are numbered 0 .. ns - 1.
struct LpRow { int head, nv, ns; };
template <typename T>
__device__ __forceinline__ LpRow lp_row(const T* x, int n) {
  constexpr int V = LpVec<T>::V;
  LpRow r;
  const int off = (int)(((uintptr_t)x & 15) / sizeof(T));
  r.head = min(n, (V - off) % V);
  r.nv = (n - r.head) / V;
  r.ns = n - r.nv * V;
  return r;
}
template <typename T>
__device__ __forceinline__ int lp_single(const LpRow& r, int s) { return s < r.head ? s : r.nv * LpVec<T>::V + s; }

// orders like the value (-0 = +0), -inf lowest; for values that are not NaN
__device__ __forceinline__ uint32_t lp_order(float v) {
  const uint32_t o = __float_as_uint(v + 0.0f);
  return (o & 0x80000000u) ? ~o : (o | 0x80000000u);
}
__device__ __forceinline__ float lp_value(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o); }
constexpr uint32_t kLpNone = 0x007fffffu;         // lp_order(-inf)

// largest key of the warp: the values first, then the indexes among the lanes that hold the largest value
__device__ __forceinline__ unsigned long long lp_warp_max(unsigned long long key) {
  const uint32_t hi = (uint32_t)(key >> 32);
  const uint32_t mh = __reduce_max_sync(0xffffffffu, hi);
  const uint32_t ml = __reduce_max_sync(0xffffffffu, hi == mh ? (uint32_t)key : 0u);
  return ((unsigned long long)mh << 32) | ml;
}
// one warp: the n largest of the `have` keys (distinct, or 0 for none) in falling order into out (0: no more).  Few keys: a key's
// place is the number of larger ones, counted by every lane for its own; many: n rounds of the largest that is left.
__device__ __forceinline__ void lp_select(const unsigned long long* keys, int have, int n, unsigned long long* out, int lane) {
  if (have <= 96) {
    if (lane < kLpMaxTop) out[lane] = 0ull;
    unsigned long long q[3];
    int above[3] = {0, 0, 0};
#pragma unroll
    for (int j = 0; j < 3; ++j) q[j] = lane + 32 * j < have ? keys[lane + 32 * j] : 0ull;
    __syncwarp();
#pragma unroll 4
    for (int i = 0; i < have; ++i) {
      const unsigned long long k = keys[i];
#pragma unroll
      for (int j = 0; j < 3; ++j) above[j] += k > q[j];
    }
#pragma unroll
    for (int j = 0; j < 3; ++j) if (q[j] != 0ull && above[j] < n) out[above[j]] = q[j];
    __syncwarp();
    return;
  }
  unsigned long long last = ~0ull;
  for (int k = 0; k < n; ++k) {
    unsigned long long mine = 0ull;
    for (int i = lane; i < have; i += 32) { const unsigned long long q = keys[i]; if (q < last && q > mine) mine = q; }
    mine = lp_warp_max(mine);
    if (lane == 0) out[k] = mine;
    last = mine ? mine : 1ull;
  }
  __syncwarp();
}

struct LpShared {
  float red[4][kLpThreads / 32];                       // per warp: maximum, sum, weighted sum
  uint32_t tmax[kLpThreads];
  uint8_t few[kLpThreads];                // per warp: its lanes that can hold an alternative
  unsigned long long cand[kLpCand];
  unsigned long long top[kLpMaxTop];
  unsigned long long best;
  float m, rest, u, own_rest;             // of this block: maximum, r, sum of e log2 e; the owner's part of r
  int has, owner, count;
  uint32_t bound;
};

struct LpArgs {
  const int32_t* tokens;
  int vocab, n_top;
  int64_t ld, rows;
  float scale, scale2;                    // 1 / T and log2(e) / T, each rounded once
  float *logp, *entropy, *stats, *top_logp;
  int32_t *top_ids, *bad;
};

template <typename T>
__global__ void __launch_bounds__(kLpThreads) token_logprobs_kernel(const T* logits, LpArgs a) {
  constexpr int V = LpVec<T>::V;
  __shared__ LpShared sh;
  uint32_t parts, part;                   // blocks of the cluster that share the row
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(part));
  const int64_t row = blockIdx.x / parts;
  pdl_launch_next();
  pdl_wait_prior();                       // loads below are plain ones: the read-only path (2 us less at 4096 x 50257) promises that nothing
                                          // writes the logits while this kernel runs, and a producer in front of it may still be doing so
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nt = blockDim.x, nw = nt >> 5;
  const T* x = logits + row * a.ld;
  const int tok = a.tokens[row];
  if (tok < 0 || tok >= a.vocab) {        // uniform over the cluster
    if (part == 0) {
      if (tid == 0) {
        if (tok >= 0 && a.bad) *a.bad = 1;
        a.logp[row] = 0.f;
        if (a.entropy) a.entropy[row] = 0.f;
        if (a.stats) { a.stats[row] = 0.f; a.stats[a.rows + row] = 0.f; }
      }
      if (tid < a.n_top) { a.top_ids[row * a.n_top + tid] = -1; a.top_logp[row * a.n_top + tid] = -INFINITY; }
    }
    return;
  }
  const float xt = to_f(x[tok]);
  const LpRow rw = lp_row(x, a.vocab);
  const uint4* xv = reinterpret_cast<const uint4*>(x + rw.head);
  const int per = (rw.nv + (int)parts - 1) / (int)parts;
  const int v0 = min(rw.nv, per * (int)part), v1 = min(rw.nv, v0 + per);
  const int ns = part == 0 ? rw.ns : 0;   // the single elements go to the first block's first threads
  const float s2 = a.scale2;

  // ---- one pass: maximum, sum of e, sum of e log2 e (bounded, unlike e (x - m)), all relative to the thread's running maximum
  float tmax = -INFINITY, m = kLowest;
  float tmax2 = -INFINITY;                // largest logit outside the batch that holds the thread's maximum (the first such batch)
  int at_max = -1;                        // that batch's first vector; -1: the single element
  uint64_t s = 0ull, u = 0ull;            // pairs of partial sums
  auto move_max = [&](float top, int batch) {
    tmax2 = fmaxf(tmax2, fminf(tmax, top));
    if (top > tmax) at_max = batch;
    tmax = fmaxf(tmax, top);
    const float mn = fmaxf(m, top), d = (m - mn) * s2, f = lp_ex2(d), dc = f > 0.f ? d : 0.f;     // d is 0 where the maximum stays
    const uint64_t ff = f2_pack(f, f);
    u = f2_mul(f2_fma(s, f2_pack(dc, dc), u), ff);
    s = f2_mul(s, ff);
    m = mn;
  };
  auto add_pair = [&](float p, float q, uint64_t nm, uint64_t sc) {
    const uint64_t d = f2_add(f2_pack(p, q), nm), t = f2_mul(d, sc);
    float t0, t1;
    f2_unpack(t, t0, t1);
    const uint64_t e = f2_pack(lp_ex2(t0), lp_ex2(t1));
    s = f2_add(s, e);
    u = f2_fma(e, f2_pack(fmaxf(t0, kLowest), fmaxf(t1, kLowest)), u);     // 0 x -inf would be NaN
  };
  const uint64_t sc = f2_pack(s2, s2);
  if (tid < ns) {
    const float v = to_f(x[lp_single<T>(rw, tid)]);
    move_max(v, -1);
    add_pair(v, -INFINITY, f2_pack(-m, -m), sc);
  }
  for (int c = v0 + tid; c < v1; c += kLpBatch * nt) {
    uint4 w[kLpBatch];
#pragma unroll
    for (int k = 0; k < kLpBatch; ++k) w[k] = c + k * nt < v1 ? xv[c + k * nt] : LpVec<T>::missing();
    float top = LpVec<T>::max(w[0]);
#pragma unroll
    for (int k = 1; k < kLpBatch; ++k) top = fmaxf(top, LpVec<T>::max(w[k]));
    move_max(top, c);
    const uint64_t nm = f2_pack(-m, -m);
#pragma unroll
    for (int k = 0; k < kLpBatch; ++k) {
      float p[V / 2], q[V / 2];
      LpVec<T>::pairs(w[k], p, q);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) add_pair(p[i], q[i], nm, sc);
    }
  }
  // ---- the block's maximum, its owner, and the sums relative to it
  sh.tmax[tid] = lp_order(tmax);
  const float wm = warp_max(m);
  if (lane == 0) sh.red[0][warp] = wm;
  if (tid == 0) { sh.owner = 1 << 30; sh.count = 0; sh.best = 0ull; }
  __syncthreads();
  float M = kLowest;
  for (int i = 0; i < nw; ++i) M = fmaxf(M, sh.red[0][i]);
  float s0, s1, u0, u1;
  f2_unpack(s, s0, s1);
  f2_unpack(u, u0, u1);
  {
    const float d = (m - M) * s2, f = lp_ex2(d);
    float st = s0 + s1, ut = u0 + u1;
    ut = f > 0.f ? (ut + st * d) * f : 0.f;                            // (a NaN shows in the sum below)
    st *= f;
    const bool own = tmax == M;
    const unsigned who = __ballot_sync(0xffffffffu, own);
    if (who != 0u && lane == 0) atomicMin(&sh.owner, warp * 32 + __ffs(who) - 1);
    st = warp_sum(st);
    ut = warp_sum(ut);
    if (lane == 0) { sh.red[1][warp] = st; sh.red[2][warp] = ut; }
  }
  // ---- a lower bound of the k-th largest: of the threads' maxima the k-th
  const bool want_top = a.n_top > 0;
  if (want_top && warp == 0) {
    uint32_t key[kLpThreads / 32], bound = kLpNone;
#pragma unroll
    for (int i = 0; i < kLpThreads / 32; ++i) key[i] = i < nw ? sh.tmax[lane + 32 * i] : 0u;
    for (int k = 0; k < a.n_top; ++k) {
      uint32_t best = key[0];
#pragma unroll
      for (int i = 1; i < kLpThreads / 32; ++i) best = max(best, key[i]);
      const uint32_t top = __reduce_max_sync(0xffffffffu, best);
      if (top <= kLpNone) { bound = kLpNone; break; }
      bound = top;
      const unsigned who = __ballot_sync(0xffffffffu, best == top);
      if (lane == __ffs(who) - 1) {
        bool gone = false;
#pragma unroll
        for (int i = 0; i < kLpThreads / 32; ++i) if (!gone && key[i] == top) { key[i] = 0u; gone = true; }
      }
    }
    if (lane == 0) sh.bound = bound;
  }
  __syncthreads();
  float S = 0.f, U = 0.f;
  for (int i = 0; i < nw; ++i) { S += sh.red[1][i]; U += sh.red[2][i]; }
  const int owner = sh.owner;
  const bool has = owner < (1 << 30);                                   // something above -inf
  float R = has ? S - 1.0f : S;
  // every element of thread i, read again by its warp: lane j takes the thread's j-th vector, lane 31 a single element
  auto reread = [&](int i, auto&& see) {
    for (int c = v0 + i + lane * nt; c < v1; c += 32 * nt) {
      const uint4 w = xv[c];
      float p[V / 2], q[V / 2];
      LpVec<T>::pairs(w, p, q);
#pragma unroll
      for (int k = 0; k < V / 2; ++k) { see(p[k], rw.head + c * V + 2 * k); see(q[k], rw.head + c * V + 2 * k + 1); }
    }
    if (lane == 31 && i < ns) { const int at = lp_single<T>(rw, i); see(to_f(x[at]), at); }
  };
  if (has && R < 1.0f) {                                                // r is small: 1 + r has lost bits of it
    if (warp == owner >> 5) {
      float mine = 0.f, ties = 0.f;                                     // the owner's elements without one maximum
      reread(owner, [&](float v, int) { if (v == M) ties += 1.0f; else mine += lp_ex2((v - M) * s2); });
      mine = warp_sum(mine) + (warp_sum(ties) - 1.0f);
      if (lane == 0) sh.own_rest = mine;
    }
    // the other threads' sums, joined again without the owner's
    const float d = m - M;
    float st = tid == owner ? 0.f : (s0 + s1) * lp_ex2(d * s2);
    st = warp_sum(st);
    if (lane == 0) sh.red[3][warp] = st;
    __syncthreads();
    R = sh.own_rest;
    for (int i = 0; i < nw; ++i) R += sh.red[3][i];
  }
  // ---- alternatives: the threads whose maximum reaches the bound
  const bool poison = !(S < INFINITY);                                  // a NaN or +inf among the logits
  if (want_top && !poison && has) {
    const uint32_t least = max(sh.bound, kLpNone + 1u);
    const bool can = sh.tmax[tid] >= least, wide = can && lp_order(tmax2) >= least;
    uint8_t* few = sh.few + warp * 32;
    auto list = [&](bool in) {                                          // the warp's lanes that answer yes, and how many
      const unsigned who = __ballot_sync(0xffffffffu, in);
      __syncwarp();
      if (in) few[__popc(who & ((1u << lane) - 1u))] = (uint8_t)lane;
      __syncwarp();
      return __popc(who);
    };
    auto see = [&](float v, int at) {
      const uint32_t o = lp_order(v);
      if (o >= least) {
        const int slot = atomicAdd(&sh.count, 1);
        if (slot < kLpCand) sh.cand[slot] = ((unsigned long long)o << 32) | (uint32_t)~at;
      }
    };
    auto see_vector = [&](int c) {
      float p[V / 2], q[V / 2];
      LpVec<T>::pairs(xv[c], p, q);
#pragma unroll
      for (int e = 0; e < V / 2; ++e) { see(p[e], rw.head + c * V + 2 * e); see(q[e], rw.head + c * V + 2 * e + 1); }
    };
    auto see_single = [&](int i) {
      if (i < ns) { const int at = lp_single<T>(rw, i); see(to_f(x[at]), at); }
    };
    // most of them reach it in one batch only: a lane takes one vector of a thread's batch
    const int one = list(can && !wide) * kLpBatch;
    for (int k0 = 0; k0 < one; k0 += 32) {
      const int k = min(k0 + lane, one - 1), i = few[k / kLpBatch], b = __shfl_sync(0xffffffffu, at_max, i), c = b + (k % kLpBatch) * nt;
      if (k0 + lane >= one) continue;
      if (b < 0) { if (k % kLpBatch == 0) see_single(warp * 32 + i); }
      else if (c < v1) see_vector(c);
    }
    // of the others all elements: a lane takes one vector of one of them at a time
    const int each = (v1 - v0 + nt - 1) / nt + (ns > 0 ? 1 : 0), items = list(wide) * each;
    for (int k = lane; k < items && *(volatile int*)&sh.count <= kLpCand; k += 32) {
      const int i = warp * 32 + few[k / each], j = k % each, c = v0 + i + j * nt;
      if (ns > 0 && j == each - 1) see_single(i);                       // the thread's single element
      else if (c < v1) see_vector(c);
    }
    __syncthreads();
    if (sh.count <= kLpCand) {
      if (warp == 0) lp_select(sh.cand, sh.count, a.n_top, sh.top, lane);
    } else {                                                            // a great many equal logits: one pass per alternative
      unsigned long long last = ~0ull;
      for (int k = 0; k < a.n_top; ++k) {
        unsigned long long mine = 0ull;
        auto see = [&](float v, int at) {
          const unsigned long long q = ((unsigned long long)lp_order(v) << 32) | (uint32_t)~at;
          if (v > -INFINITY && q < last && q > mine) mine = q;
        };
        for (int c = v0 + tid; c < v1; c += nt) {
          float p[V / 2], q[V / 2];
          LpVec<T>::pairs(xv[c], p, q);
#pragma unroll
          for (int i = 0; i < V / 2; ++i) { see(p[i], rw.head + c * V + 2 * i); see(q[i], rw.head + c * V + 2 * i + 1); }
        }
        if (tid < ns) { const int at = lp_single<T>(rw, tid); see(to_f(x[at]), at); }
        mine = lp_warp_max(mine);
        if (lane == 0 && mine) atomicMax(&sh.best, mine);
        __syncthreads();
        last = sh.best;
        __syncthreads();
        if (tid == 0) { sh.top[k] = last; sh.best = 0ull; }
        if (last == 0ull) last = 1ull;
        __syncthreads();
      }
    }
  } else if (want_top && tid < kLpMaxTop) {
    sh.top[tid] = 0ull;
  }
  // ---- join the blocks of a cluster in the first one
  if (tid == 0) { sh.m = M; sh.rest = poison ? S : R; sh.u = U; sh.has = has; }
  if (parts > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  } else {
    __syncthreads();
  }
  if (part == 0 && warp == 0) {
    float m_all = sh.m, r_all = sh.rest, u_all = sh.u;
    int has_all = sh.has;
    bool bad = poison;
    unsigned long long* list = sh.top;
    if (parts > 1) {
      auto remote = [&](const void* p, uint32_t rank) {
        uint32_t r;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
        return r;
      };
      auto ldf = [&](const void* p, uint32_t rank) { float v; asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote(p, rank))); return v; };
      float pm = 0.f, pr = 0.f, pu = 0.f, ph = 0.f;                     // lane k: what block k found
      if (lane < (int)parts) { pm = ldf(&sh.m, lane); pr = ldf(&sh.rest, lane); pu = ldf(&sh.u, lane); ph = ldf(&sh.has, lane); }
      for (uint32_t k = 1; k < parts; ++k) {
        const float mk = __shfl_sync(0xffffffffu, pm, k), rk = __shfl_sync(0xffffffffu, pr, k), uk = __shfl_sync(0xffffffffu, pu, k);
        const int hk = __float_as_int(__shfl_sync(0xffffffffu, ph, k));
        bad = bad || !(rk < INFINITY);
        if (mk > m_all || (!has_all && hk)) {                          // the other one's maximum leads
          const float d = (m_all - mk) * s2, f = lp_ex2(d), w = r_all + (has_all ? 1.f : 0.f);
          u_all = uk + (f > 0.f ? (u_all + w * d) * f : 0.f);
          r_all = rk + w * f;
          m_all = mk;
        } else {
          const float d = (mk - m_all) * s2, f = lp_ex2(d), w = rk + (hk ? 1.f : 0.f);
          u_all += f > 0.f ? (uk + w * d) * f : 0.f;
          r_all += w * f;
        }
        has_all |= hk;
      }
      if (want_top) {
        for (int i = lane; i < (int)parts * a.n_top; i += 32) {
          unsigned long long q;
          asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(q) : "r"(remote(&sh.top[i % a.n_top], (uint32_t)(i / a.n_top))));
          sh.cand[i] = q;
        }
        __syncwarp();
        lp_select(sh.cand, (int)parts * a.n_top, a.n_top, sh.top, lane);
      }
    }
    const float nanv = __int_as_float(0x7fc00000);
    const bool empty = !has_all && !bad;
    const float L = log1pf(r_all);
    if (lane == 0) {
      a.logp[row] = empty ? -INFINITY : bad ? nanv : (xt - m_all) * a.scale - L;
      if (a.entropy) a.entropy[row] = empty ? 0.f : bad ? nanv : L - u_all * kLogLn2 / (1.0f + r_all);
      if (a.stats) { a.stats[row] = bad ? nanv : empty ? -INFINITY : m_all; a.stats[a.rows + row] = empty ? 0.f : bad ? nanv : L; }
    }
    for (int k = lane; k < a.n_top; k += 32) {
      const unsigned long long q = bad ? 0ull : list[k];
      a.top_ids[row * a.n_top + k] = q ? (int32_t)~(uint32_t)q : -1;
      a.top_logp[row * a.n_top + k] = bad ? nanv : q ? (lp_value((uint32_t)(q >> 32)) - m_all) * a.scale - L : -INFINITY;
    }
  }
  if (parts > 1)                                                        // the peers' shared memory stays until it has been read
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Threads of a block and blocks per row.  Small blocks: the end of a row (sums, alternatives) is a chain of short steps that other
// rows' blocks on the same SM hide (4096 x 50257 bf16: 86 us with 256 threads, 78 with 128 on one card, 83 on others), down to 64 or 32 threads for short
// rows, where that end is most of the work, as long as the SMs stay full (16384 x 4000: 74 us with 128, 58 with 64, 48 with 32; 16384 x
// 16000: 125, 111, 120; but 4096 x 50257 with 64: 85); but enough threads in all, or loads in flight run short (512 x 128000:
// 75 us with 128, 51 with 256; 2048 x 4000: 11 us with 128, 26 with 64).  While the rows alone still leave
// SMs idle, up to eight blocks (a cluster) share a row, as long as each has two vectors a thread.  148 SMs are assumed; on a device with another
// number only the speed would change.
inline void lp_shape(int64_t rows, int64_t vocab, int vec, int* threads, int* parts) {
  const int64_t nv = vocab / vec, fill = 148 * 1024;
  int th = 32;
  while (th < 128 && nv > 4 * th) th *= 2;
  for (int few = 32; few < th; few *= 2)
    if (rows * few >= 148 * 1536 && nv <= 32 * few) th = few;             // (ends the loop)
  if (th == 128 && rows * th < fill && nv > 8 * th) th = kLpThreads;
  int p = 1;
  while (p < 8 && rows * th * p < fill && nv >= 2 * p * th) p *= 2;
  *threads = th;
  *parts = p;
}
template <typename T>
inline cudaError_t launch_token_logprobs(cudaStream_t st, const T* logits, const LpArgs& a) {
  int th, parts;
  lp_shape(a.rows, a.vocab, LpVec<T>::V, &th, &parts);
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3((unsigned)(a.rows * parts));
  cfg.blockDim = dim3(th);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled();
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = parts; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = parts > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T>, logits, a);
}

// ------------------------------------------------------------------ gradient
// From the saved maximum, L and H; one pass, each element read and written once.  A task is up to 4 vectors per thread of a row;
// blocks walk the tasks.  VEC: logits and gradient rows share their alignment, so both move 16 bytes at a time.
struct LpBwdArgs {
  const int32_t* tokens;
  int vocab, chunks;
  int64_t ld, rows;
  float scale;
  const float *stats, *entropy, *dlogp, *dentropy;
};
template <typename T, bool VEC>
__global__ void __launch_bounds__(128) token_logprobs_bwd_kernel(const T* logits, T* dlogits, LpBwdArgs a) {
  constexpr int V = LpVec<T>::V;
  const int tid = threadIdx.x, nt = blockDim.x;
  pdl_launch_next();
  pdl_wait_prior();
  for (int64_t task = blockIdx.x; task < a.rows * a.chunks; task += gridDim.x) {
    const int64_t row = task / a.chunks;
    const int part = (int)(task % a.chunks);
    const T* x = logits + row * a.ld;
    T* d = dlogits + row * a.ld;
    LpRow rw;
    uint4 w[4];
    const int first = part * 4 * nt + tid;
    if (VEC) {                                               // under way before the row's scalars are known
      rw = lp_row(x, (int)a.ld);
      const uint4* xv = reinterpret_cast<const uint4*>(x + rw.head);
#pragma unroll
      for (int k = 0; k < 4; ++k) if (first + k * nt < rw.nv) w[k] = xv[first + k * nt];
    }
    const int tok = a.tokens[row];
    const float m = a.stats[row], L = a.stats[a.rows + row];
    const bool zero = tok < 0 || tok >= a.vocab || m == -INFINITY;
    const float g = a.dlogp ? a.dlogp[row] * a.scale : 0.f, h = a.dentropy ? a.dentropy[row] * a.scale : 0.f;
    const float hH = a.dentropy ? h * a.entropy[row] : 0.f, c0 = g + hH, s = a.scale;
    auto plain = [&](float v) {                              // any column but the token's
      const float lp = fmaf(v - m, s, -L);
      return -lp_ex2(lp * kLog2E) * fmaf(h, fmaxf(lp, -200.f), c0);        // p is 0 below -200; p x -inf would be NaN
    };
    auto grad = [&](float v, int64_t at) {
      if (zero || at >= a.vocab) return 0.f;
      if (at != tok) return plain(v);
      const float lp = fmaf(v - m, s, -L);
      return -expm1f(lp) * g - lp_ex2(lp * kLog2E) * fmaf(h, fmaxf(lp, -200.f), hH);     // 1 - p of a token that is nearly sure
    };
    if (VEC) {
      uint4* dv = reinterpret_cast<uint4*>(d + rw.head);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = first + k * nt;
        if (c >= rw.nv) break;
        const int64_t at = rw.head + (int64_t)c * V;
        float p[V / 2], q[V / 2];
        LpVec<T>::pairs(w[k], p, q);
        if (!zero && at + V <= a.vocab && (unsigned)(tok - at) >= (unsigned)V) {
#pragma unroll
          for (int i = 0; i < V / 2; ++i) { p[i] = plain(p[i]); q[i] = plain(q[i]); }
        } else {
#pragma unroll
          for (int i = 0; i < V / 2; ++i) { p[i] = grad(p[i], at + 2 * i); q[i] = grad(q[i], at + 2 * i + 1); }
        }
        dv[c] = LpVec<T>::join(p, q);
      }
      if (part == 0 && tid < rw.ns) { const int at = lp_single<T>(rw, tid); d[at] = from_f<T>(grad(zero ? 0.f : to_f(x[at]), at)); }
    } else {
      for (int64_t c = (int64_t)part * 4 * nt * V + tid; c < min(a.ld, ((int64_t)part + 1) * 4 * nt * V); c += nt) d[c] = from_f<T>(grad(zero ? 0.f : to_f(x[c]), c));
    }
  }
}
template <typename T>
inline cudaError_t launch_token_logprobs_bwd(cudaStream_t st, const T* logits, T* dlogits, LpBwdArgs a) {
  constexpr int V = LpVec<T>::V;
  const int64_t nv = (a.ld + V - 1) / V;
  int th = 32;
  while (th < 128 && nv > 4 * th) th *= 2;
  a.chunks = (int)((nv + 4 * th - 1) / (4 * th));
  const int64_t tasks = a.rows * a.chunks;
  const unsigned grid = (unsigned)(tasks < (1 << 30) ? tasks : (1 << 30));
  const bool vec = (((uintptr_t)logits ^ (uintptr_t)dlogits) & 15) == 0;
  return launch_pdl(vec ? token_logprobs_bwd_kernel<T, true> : token_logprobs_bwd_kernel<T, false>, dim3(grid), dim3(th), 0, st, logits, dlogits, a);
}

}  // namespace hift
