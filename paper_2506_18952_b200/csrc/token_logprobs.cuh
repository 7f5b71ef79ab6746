// token_logprobs.cuh - log probabilities of given tokens, their ranks, the entropy of a row and its top alternatives, from
// logits in memory.  Part of hola_verify.cu (inside its anonymous namespace).
//
// One pass over a row of V logits:  m = max l,  s = sum e^(l-m),  t = sum e^(l-m)(l-m),  logZ = m + ln s,  H = ln s - t/s,
// logprob(x) = (l[x] - m) - ln s,  rank(x) = #{v : l[v] > l[x], or l[v] = l[x] and v < x},  and the n entries that come first in the
// order (logit descending, id ascending).  A row is one CTA's or is cut into parts for the CTAs of a cluster, which merge over
// distributed shared memory; thread i of a part takes groups of eight neighbouring entries i, i + 256, ...
//
// The alternatives cost the pass next to nothing: every thread keeps the maximum of what it has seen (which the running sums
// need anyway) and the group that it first met it in.  Let the n-th best of the threads' (maximum, group) pairs in the order
// (value descending, group ascending) be (w, g): at least n entries lie at or before it (those maxima), so every one of the
// part's n best has a value above w, or w itself in a group up to g.  Only threads whose own pair is at or before (w, g) can hold
// such entries; a warp reads those threads' groups again, out of the L2, and keeps the best 32 it meets.

constexpr int kLpThreads = 256;
constexpr int kLpWarps = kLpThreads / 32;
constexpr int kLpGroup = 8;            // neighbouring entries that a thread takes at once
constexpr int kLpMaxTop = 32;          // alternatives: a sorted list lies across a warp, one entry per lane
constexpr int kLpTok = 4;              // tokens ranked in one pass (counters in registers)
constexpr int kLpMaxCluster = 8;

struct LpParams {
  const void* logits;
  long long row_stride;        // entries from one row to the next
  int rows, V;
  int T, t0, tn;               // tokens per row; the part of them that this launch ranks and scores
  int n_top;
  const int* tokens;           // [rows][T], or null
  const int* draft_tok;        // emitted form (accept_len not null): [B][k], rows = B (k + 1), T = 1
  const int* accept_len;
  const int* next_tok;
  int k;
  const float* logZ_in;        // [rows], or null: the sums are made
  float* logprob;              // [rows][T]
  int* rank;                   // [rows][T], or null
  float* entropy;              // [rows], or null
  float* logZ;                 // [rows], or null
  int* top_ids;                // [rows][n_top]
  float* top_logprobs;
  unsigned* status;            // or null
};

// What a CTA knows of its part of a row when it has seen it.
struct LpPart {
  float m, s, t;
  unsigned bad;
  int count[kLpTok];
};

// Floats in the order of their values as unsigned whole numbers (one zero; NaN does not occur).
__device__ __forceinline__ uint32_t lp_order(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float lp_value(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ uint64_t lp_key(float x, int at) {
  return static_cast<uint64_t>(lp_order(x)) << 32 | static_cast<uint32_t>(~at);
}
// ln p = (l - m) - ln s from a row's own sums (the rounding of m + ln s, relative to m, stays out of it), l - logZ under a given
// logZ (m = 0, ln s = logZ).  Where nothing is left of a row every entry has probability 0.
__device__ __forceinline__ float lp_logprob(float l, float m, float ls) {
  return m == -CUDART_INF_F || ls == -CUDART_INF_F ? -CUDART_INF_F : (l - m) - ls;
}
// A difference of maxima that is kept finite when multiplied by a sum of 2^31 terms: masks may be as low as the type goes.
__device__ __forceinline__ float lp_below(float a, float b) { return fmaxf(a - b, -1e28f); }

// Sorted lists across a warp: lane i holds the i-th largest key (0: none).
__device__ __forceinline__ uint64_t lp_exchange(uint64_t a, int stride, bool larger) {
  const uint64_t b = __shfl_xor_sync(0xffffffffu, a, stride);
  return (a > b) == larger ? a : b;
}
__device__ __forceinline__ uint64_t lp_sort(uint64_t a, int lane) {                 // bitonic sort (Batcher)
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int stride = size >> 1; stride > 0; stride >>= 1)
      a = lp_exchange(a, stride, ((lane & size) == 0) == ((lane & stride) == 0));
  return a;
}
// The 32 largest of two sorted lists, sorted; `reversed`: the second one from its end.
__device__ __forceinline__ uint64_t lp_merge(uint64_t a, uint64_t reversed, int lane) {
  if (reversed > a) a = reversed;
#pragma unroll
  for (int stride = 16; stride > 0; stride >>= 1) a = lp_exchange(a, stride, (lane & stride) == 0);
  return a;
}
// The lists of all warps of the CTA into warp 0's.  `lists`: [kLpWarps][32] in shared memory.
__device__ __forceinline__ uint64_t lp_merge_warps(uint64_t a, uint64_t* lists, int warp, int lane) {
  lists[warp * 32 + lane] = a;
#pragma unroll
  for (int step = 1; step < kLpWarps; step <<= 1) {
    __syncthreads();
    if ((warp & (2 * step - 1)) == 0) {
      a = lp_merge(a, lists[(warp + step) * 32 + 31 - lane], lane);
      lists[warp * 32 + lane] = a;
    }
  }
  return a;
}

__device__ __forceinline__ float min3(float a, float b, float c) {
  float d;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {     // NaN where one of them is
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// 16 bytes that this kernel never sees change, past the L1.
__device__ __forceinline__ uint4 load_once(const void* p) {
  uint4 x;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p));
  return x;
}

// Eight neighbouring logits as loaded and as fp32.
template <typename T>
struct LpRaw {
  static constexpr int kPieces = kLpGroup * sizeof(T) / 16;
  uint4 x[kPieces];
};
__device__ __forceinline__ float lp_float(float x) { return x; }
__device__ __forceinline__ float lp_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float lp_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void lp_expand(const LpRaw<float>& r, float* f) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    f[4 * i] = __uint_as_float(r.x[i].x); f[4 * i + 1] = __uint_as_float(r.x[i].y);
    f[4 * i + 2] = __uint_as_float(r.x[i].z); f[4 * i + 3] = __uint_as_float(r.x[i].w);
  }
}
__device__ __forceinline__ void lp_expand(const LpRaw<__nv_bfloat16>& r, float* f) {
  const uint32_t w[4] = {r.x[0].x, r.x[0].y, r.x[0].z, r.x[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void lp_expand(const LpRaw<__half>& r, float* f) {
  const uint32_t w[4] = {r.x[0].x, r.x[0].y, r.x[0].z, r.x[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    f[2 * i] = y.x;
    f[2 * i + 1] = y.y;
  }
}

// A row as groups that start on 16-byte boundaries: group j holds entries 8 j - off ... 8 j - off + 7, the first and the last
// one perhaps fewer (what they lack reads as -inf).
template <typename T>
struct LpRow {
  const T* base;               // entry -off, on a 16-byte boundary (not read before entry 0)
  int off, V, groups;          // groups whole_begin .. whole_end - 1 are whole
  int whole_begin, whole_end;
  __device__ __forceinline__ LpRow(const T* row, int V_) : V(V_) {
    off = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
    base = row - off;
    groups = static_cast<int>((static_cast<long long>(V_) + off + kLpGroup - 1) / kLpGroup);
    whole_begin = off ? 1 : 0;
    whole_end = static_cast<int>((static_cast<long long>(V_) + off) / kLpGroup);
  }
  __device__ __forceinline__ bool whole(int j) const { return j >= whole_begin && j < whole_end; }
  __device__ __forceinline__ LpRaw<T> fetch(int j) const {        // (whole groups)
    LpRaw<T> r;
    const char* p = reinterpret_cast<const char*>(base + static_cast<size_t>(j) * kLpGroup);
#pragma unroll
    for (int i = 0; i < LpRaw<T>::kPieces; ++i) r.x[i] = load_once(p + 16 * i);
    return r;
  }
  __device__ __forceinline__ void get(int j, float* f) const {
    if (whole(j)) {
      lp_expand(fetch(j), f);
    } else {
#pragma unroll
      for (int i = 0; i < kLpGroup; ++i) {
        const long long v = static_cast<long long>(j) * kLpGroup - off + i;
        f[i] = v >= 0 && v < V ? lp_float(base[v + off]) : -CUDART_INF_F;
      }
    }
  }
  __device__ __forceinline__ int first(int j) const { return j * kLpGroup - off; }
};

// One thread's view of its part of the row.
template <bool kSums, bool kTop, bool kRank>
struct LpThread {
  float m, s, t;
  int at;                      // group that the maximum was first met in
  bool bad;
  int count[kLpTok];

  __device__ __forceinline__ explicit LpThread(int first) : s(0.f), t(0.f), at(first), bad(false), count{0, 0, 0, 0} {
    m = -CUDART_INF_F;
  }

  __device__ __forceinline__ void take(const float* f, int j, int v0, const float* lx, const int* x, float lx_min, int n) {
    const float hi = max3_nan(max3_nan(f[0], f[1], f[2]), max3_nan(f[3], f[4], f[5]), max3_nan(f[6], f[7], f[7]));
    if (!(hi < CUDART_INF_F)) { bad = true; return; }
    if (kRank && hi >= lx_min) {
#pragma unroll
      for (int q = 0; q < kLpTok; ++q) {
        if (q < n && hi >= lx[q]) {
#pragma unroll
          for (int i = 0; i < kLpGroup; ++i)
            count[q] += f[i] > lx[q] || (f[i] == lx[q] && v0 + i < x[q] && v0 + i >= 0) ? 1 : 0;
        }
      }
    }
    if (hi > m) {
      if (kSums && m != -CUDART_INF_F) {
        const float d = lp_below(m, hi), e = ex2_approx(d * kLog2e);
        t = e * (t + d * s);
        s *= e;
      }
      m = hi;
      at = j;
    }
    if (!kSums || hi == -CUDART_INF_F) return;
    const float lo = min3(min3(f[0], f[1], f[2]), min3(f[3], f[4], f[5]), fminf(f[6], f[7]));
    if (lo > -1e37f) {
      const uint64_t mm = pack2(-m, -m), l2e = pack2(kLog2e, kLog2e);
      uint64_t s2 = pack2(0.f, 0.f), a2 = pack2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kLpGroup / 2; ++i) {
        const uint64_t d2 = add2(pack2(f[2 * i], f[2 * i + 1]), mm);
        float x0, x1;
        unpack2(mul2(d2, l2e), x0, x1);
        const uint64_t e2 = pack2(ex2_approx(x0), ex2_approx(x1));
        s2 = add2(s2, e2);
        a2 = fma2(e2, d2, a2);
      }
      float a, b, c, d;
      unpack2(s2, a, b);
      unpack2(a2, c, d);
      s += a + b;
      t += c + d;
    } else {
      // masked entries (-inf, or as low as the type goes): differences are kept finite, their exponentials are zeros
#pragma unroll
      for (int i = 0; i < kLpGroup; ++i) {
        const float d = lp_below(f[i], m), e = ex2_approx(d * kLog2e);
        s += e;
        t = fmaf(e, d, t);
      }
    }
  }
};

// What bounds it: HBM for large batches; for a few rows the chain token -> its logit -> pass -> merges.
template <typename T, bool kSums, bool kTop, bool kRank>
__global__ void __launch_bounds__(kLpThreads, 4) token_logprobs_kernel(const LpParams p, int C) {
  __shared__ uint64_t lists[kLpWarps * 32];
  __shared__ uint64_t fresh[kLpWarps][32];               // candidates a warp has met and not sorted in yet
  __shared__ uint64_t cluster_lists[kLpMaxCluster][kTop ? 32 : 1];
  __shared__ uint8_t looked_at[kLpWarps][32];
  __shared__ LpPart warp_parts[kLpWarps];
  __shared__ LpPart cluster_parts[kLpMaxCluster];
  __shared__ uint64_t limit;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = blockIdx.x / C, part = blockIdx.x - row * C;
  // the other CTAs of the cluster have started (looked at before anything is sent to them)
  if (C > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
  grid_dependency_wait();
  grid_dependency_release();

  // The part's groups.
  const LpRow<T> r(static_cast<const T*>(p.logits) + static_cast<size_t>(row) * p.row_stride, p.V);
  const int per = (r.groups + C - 1) / C;
  const int j_end = min(r.groups, (part + 1) * per), j_begin = min(part * per, j_end);

  // What the row is asked for.  (Emitted form: row j of a sequence holds a token up to its accept length.)
  int j_seq = 0, len = 0;
  unsigned flags = 0;
  if (p.accept_len) {
    const int b = row / (p.k + 1);
    j_seq = row - b * (p.k + 1);
    len = p.accept_len[b];
    const bool valid = len >= 0 && len <= p.k;
    if (!valid || j_seq > len) {                         // (the same in every CTA of the cluster)
      if (C > 1) asm volatile("barrier.cluster.wait;" ::: "memory");
      if (part != 0) return;
      // no token: nothing is read; an accept length that cannot be: NaN
      const float none = valid ? 0.f : CUDART_NAN_F;
      if (tid == 0) {
        p.logprob[row] = none;
        if (kRank) p.rank[row] = -1;
        if (!valid && p.status) atomicOr(p.status, HOLA_FLAG_BAD_TOKEN);
      }
      if (kTop && tid < p.n_top) {
        p.top_ids[static_cast<size_t>(row) * p.n_top + tid] = -1;
        p.top_logprobs[static_cast<size_t>(row) * p.n_top + tid] = none;
      }
      return;
    }
  }

  // The first groups are on their way while the tokens and their logits are looked up.
  constexpr int kUnroll = 4 / LpRaw<T>::kPieces;
  constexpr int kAhead = (kUnroll - 1) * kLpThreads;
  LpRaw<T> raw[kUnroll];
  const int whole_end = min(j_end, r.whole_end);
  int j = j_begin + tid;
  const bool ragged_first = j < j_end && j < r.whole_begin;
  if (ragged_first) j += kLpThreads;
  bool more = j + kAhead < whole_end;
  if (more) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) raw[u] = r.fetch(j + u * kLpThreads);
  }

  int x[kLpTok];
  float lx[kLpTok], lx_min = CUDART_INF_F;
  const int n = p.tn;
#pragma unroll
  for (int q = 0; q < kLpTok; ++q) {
    x[q] = -1;
    if (kRank && q < n) {
      x[q] = p.accept_len ? (j_seq < len ? p.draft_tok[static_cast<size_t>(row / (p.k + 1)) * p.k + j_seq] : p.next_tok[row / (p.k + 1)])
                          : p.tokens[static_cast<size_t>(row) * p.T + p.t0 + q];
    }
    const bool have = x[q] >= 0 && x[q] < p.V;
    lx[q] = have ? lp_float(r.base[static_cast<size_t>(x[q]) + r.off]) : CUDART_NAN_F;
    if (have) lx_min = fminf(lx_min, lx[q]);
  }

  LpThread<kSums, kTop, kRank> th(j_begin + tid);
  if (ragged_first) {
    float f[kLpGroup];
    r.get(0, f);
    th.take(f, 0, r.first(0), lx, x, lx_min, n);
  }
  while (more) {
    LpRaw<T> now[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) now[u] = raw[u];
    const int next = j + kUnroll * kLpThreads;
    more = next + kAhead < whole_end;
    if (more) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) raw[u] = r.fetch(next + u * kLpThreads);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float f[kLpGroup];
      lp_expand(now[u], f);
      th.take(f, j + u * kLpThreads, r.first(j + u * kLpThreads), lx, x, lx_min, n);
    }
    j = next;
  }
  for (; j < j_end; j += kLpThreads) {
    float f[kLpGroup];
    r.get(j, f);
    th.take(f, j, r.first(j), lx, x, lx_min, n);
  }

  // The threads' sums and counts, over the warp and the CTA.
  const float wm = warp_max_f32(th.m);
  LpPart mine;
  mine.m = wm;
  mine.s = mine.t = 0.f;
  if (kSums) {
    const float d = th.m == -CUDART_INF_F ? 0.f : lp_below(th.m, wm), e = ex2_approx(d * kLog2e);
    mine.s = e * th.s;
    mine.t = e * fmaf(d, th.s, th.t);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      mine.s += __shfl_xor_sync(0xffffffffu, mine.s, o);
      mine.t += __shfl_xor_sync(0xffffffffu, mine.t, o);
    }
  }
  mine.bad = __any_sync(0xffffffffu, th.bad) ? 1u : 0u;
#pragma unroll
  for (int q = 0; q < kLpTok; ++q) mine.count[q] = kRank ? __reduce_add_sync(0xffffffffu, th.count[q]) : 0;
  if (lane == 0) warp_parts[warp] = mine;

  uint64_t best = 0;                                     // kTop: warp 0's sorted list of the part's best entries
  if (kTop) {
    const uint64_t own = th.at < j_end ? lp_key(th.m, th.at) : 0;
    const uint64_t all = lp_merge_warps(lp_sort(own, lane), lists, warp, lane);
    if (warp == 0 && lane == p.n_top - 1) limit = all;
    __syncthreads();
    const uint64_t lim = limit;                          // (0: fewer threads than that hold anything)
    const float w = lp_value(static_cast<uint32_t>(lim >> 32));
    const int g = static_cast<int>(~static_cast<uint32_t>(lim));
    const unsigned look = __ballot_sync(0xffffffffu, own != 0 && own >= lim);
    int waiting = 0;
    // The groups of those threads, dealt out to the lanes.
    if (look >> lane & 1u) looked_at[warp][__popc(look & ((1u << lane) - 1u))] = static_cast<uint8_t>(lane);
    __syncwarp();
    const int steps = (j_end - j_begin + kLpThreads - 1) / kLpThreads;         // groups per thread at most
    const int total = __popc(look) * steps;
    for (int i0 = 0; i0 < total; i0 += 32) {
      const int i = i0 + lane;
      float f[kLpGroup];
      int jj = -1;
      if (i < total) {
        const int who = i / steps;
        jj = j_begin + warp * 32 + looked_at[warp][who] + (i - who * steps) * kLpThreads;
        if (jj >= j_end) jj = -1;
      }
      if (jj >= 0) r.get(jj, f);
      const int v0 = r.first(jj);
#pragma unroll
      for (int e = 0; e < kLpGroup; ++e) {
        const bool in = jj >= 0 && v0 + e >= 0 && v0 + e < p.V && (lim == 0 || f[e] > w || (f[e] == w && jj <= g));
        const unsigned mask = __ballot_sync(0xffffffffu, in);
        if (!mask) continue;
        const int fit = __popc(mask);
        if (waiting + fit > 32) {                        // full: sort what waits into the list
          __syncwarp();
          const uint64_t a = lp_sort(lane < waiting ? fresh[warp][lane] : 0, lane);
          best = lp_merge(best, __shfl_sync(0xffffffffu, a, 31 - lane), lane);
          waiting = 0;
          __syncwarp();
        }
        if (in) fresh[warp][waiting + __popc(mask & ((1u << lane) - 1u))] = lp_key(f[e], v0 + e);
        waiting += fit;
      }
    }
    __syncwarp();
    if (waiting > 0) {
      const uint64_t a = lp_sort(lane < waiting ? fresh[warp][lane] : 0, lane);
      best = lp_merge(best, __shfl_sync(0xffffffffu, a, 31 - lane), lane);
    }
    best = lp_merge_warps(best, lists, warp, lane);      // (the lists of before are read no more)
  } else {
    __syncthreads();
  }

  // Warp 0: the CTA's part, to the first CTA of the cluster.
  if (warp == 0) {
    LpPart w8 = {-CUDART_INF_F, 0.f, 0.f, 0u, {0, 0, 0, 0}};
    if (lane < kLpWarps) w8 = warp_parts[lane];
    const float m = warp_max_f32(w8.m);
    if (kSums) {
      const float d = w8.m == -CUDART_INF_F ? 0.f : lp_below(w8.m, m), e = ex2_approx(d * kLog2e);
      w8.t = e * fmaf(d, w8.s, w8.t);
      w8.s *= e;
    }
    w8.m = m;
#pragma unroll
    for (int o = kLpWarps / 2; o > 0; o >>= 1) {
      w8.s += __shfl_xor_sync(0xffffffffu, w8.s, o);
      w8.t += __shfl_xor_sync(0xffffffffu, w8.t, o);
      w8.bad |= __shfl_xor_sync(0xffffffffu, w8.bad, o);
#pragma unroll
      for (int q = 0; q < kLpTok; ++q) w8.count[q] += __shfl_xor_sync(0xffffffffu, w8.count[q], o);
    }
    if (C > 1) asm volatile("barrier.cluster.wait;" ::: "memory");
    LpPart* to = C > 1 ? cg::this_cluster().map_shared_rank(&cluster_parts[part], 0) : &cluster_parts[part];
    if (lane == 0) *to = w8;
    if (kTop) {
      uint64_t* to_list = C > 1 ? cg::this_cluster().map_shared_rank(&cluster_lists[part][0], 0) : &cluster_lists[part][0];
      to_list[lane] = best;
    }
    __syncwarp();
  } else if (C > 1) {
    asm volatile("barrier.cluster.wait;" ::: "memory");
  }
  if (C > 1) cluster_sync_all();
  if (part != 0 || warp != 0) return;

  // The row.
  LpPart all = cluster_parts[0];
  if (kTop) best = cluster_lists[0][lane];
  for (int c = 1; c < C; ++c) {
    const LpPart o = cluster_parts[c];
    if (kSums && o.m != -CUDART_INF_F) {
      const float m = fmaxf(all.m, o.m);
      const float da = all.m == -CUDART_INF_F ? 0.f : lp_below(all.m, m), db = lp_below(o.m, m);
      const float ea = ex2_approx(da * kLog2e), eb = ex2_approx(db * kLog2e);
      all.t = ea * fmaf(da, all.s, all.t) + eb * fmaf(db, o.s, o.t);
      all.s = ea * all.s + eb * o.s;
      all.m = m;
    }
    all.bad |= o.bad;
#pragma unroll
    for (int q = 0; q < kLpTok; ++q) all.count[q] += o.count[q];
    if (kTop) best = lp_merge(best, cluster_lists[c][31 - lane], lane);
  }
  float m = 0.f, ls, logZ, H = 0.f;
  if (!kSums) {
    ls = logZ = p.logZ_in[row];
  } else if (all.bad) {
    m = ls = logZ = H = CUDART_NAN_F;
  } else if (all.m == -CUDART_INF_F) {
    m = ls = logZ = -CUDART_INF_F;                       // nothing is left of the row
  } else {
    m = all.m;
    ls = logf(all.s);
    logZ = m + ls;
    H = fmaxf(0.f, ls - quotient(all.t, all.s));
  }
  if (all.bad) flags |= HOLA_FLAG_BAD_LOGIT;
  if (lane == 0) {
    if (kSums && p.entropy) p.entropy[row] = H;
    if (kSums && p.logZ) p.logZ[row] = logZ;
  }
  // (no token: 0; one that the vocabulary does not have: NaN)
  if (kRank) {
    if (lane < n) {
      int tok = x[0], before = all.count[0];
      float l = lx[0];
#pragma unroll
      for (int q = 1; q < kLpTok; ++q)
        if (lane == q) { tok = x[q]; before = all.count[q]; l = lx[q]; }
      const size_t at = static_cast<size_t>(row) * p.T + p.t0 + lane;
      const bool have = tok >= 0 && tok < p.V, none = !p.accept_len && tok == -1;
      if (!have && !none) flags |= HOLA_FLAG_BAD_TOKEN;
      p.logprob[at] = have ? lp_logprob(l, m, ls) : none ? 0.f : CUDART_NAN_F;
      p.rank[at] = have && !all.bad ? before : -1;
    }
  } else {
    for (int q = lane; q < p.T; q += 32) {
      const int tok = !p.accept_len ? p.tokens[static_cast<size_t>(row) * p.T + q]
                      : j_seq < len ? p.draft_tok[static_cast<size_t>(row / (p.k + 1)) * p.k + j_seq] : p.next_tok[row / (p.k + 1)];
      const bool have = tok >= 0 && tok < p.V, none = !p.accept_len && tok == -1;
      if (!have && !none) flags |= HOLA_FLAG_BAD_TOKEN;
      p.logprob[static_cast<size_t>(row) * p.T + q] =
          have ? lp_logprob(lp_float(r.base[static_cast<size_t>(tok) + r.off]), m, ls) : none ? 0.f : CUDART_NAN_F;
    }
  }
  if (kTop && lane < p.n_top) {
    const size_t at = static_cast<size_t>(row) * p.n_top + lane;
    p.top_ids[at] = all.bad ? -1 : static_cast<int>(~static_cast<uint32_t>(best));
    p.top_logprobs[at] = all.bad ? CUDART_NAN_F : lp_logprob(lp_value(static_cast<uint32_t>(best >> 32)), m, ls);
  }
  if (p.status) {
    __syncwarp();
    flags = __reduce_or_sync(0xffffffffu, flags);
    if (lane == 0 && flags) atomicOr(p.status, flags);
  }
}

// The tokens' own entries alone: log probabilities where logZ is known and neither ranks nor alternatives are asked for.
template <typename T>
__global__ void __launch_bounds__(128) gather_logprobs_kernel(const LpParams p) {
  grid_dependency_wait();
  grid_dependency_release();
  const long long i = static_cast<long long>(blockIdx.x) * 128 + threadIdx.x;
  if (i >= static_cast<long long>(p.rows) * p.T) return;
  const int row = static_cast<int>(i / p.T);
  int tok = -1;
  bool none = false;
  if (p.accept_len) {
    const int b = row / (p.k + 1), j = row - b * (p.k + 1), len = p.accept_len[b];
    const bool valid = len >= 0 && len <= p.k;
    none = valid && j > len;
    if (valid && !none) tok = j < len ? p.draft_tok[static_cast<size_t>(b) * p.k + j] : p.next_tok[b];
  } else {
    tok = p.tokens[i];
    none = tok == -1;
  }
  const bool have = tok >= 0 && tok < p.V;
  const T* row_at = static_cast<const T*>(p.logits) + static_cast<size_t>(row) * p.row_stride;
  p.logprob[i] = have ? lp_logprob(lp_float(row_at[tok]), 0.f, p.logZ_in[row]) : none ? 0.f : CUDART_NAN_F;
  if (!have && !none && p.status) atomicOr(p.status, HOLA_FLAG_BAD_TOKEN);
}

// CTAs per row: enough for four on every SM, as long as a thread keeps a group or two of its own.
int lp_cluster(int num_sms, int rows, int V) {
  int C = 1;
  while (C < kLpMaxCluster && static_cast<long long>(rows) * C < 4ll * num_sms && V / (2 * C) >= kLpThreads * kLpGroup) C <<= 1;
  return C;
}

template <typename T, bool kSums, bool kTop, bool kRank>
cudaError_t launch_logprobs(const LpParams& p, int C, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.rows) * C); cfg.blockDim = dim3(kLpThreads); cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(C); attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = C > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, kSums, kTop, kRank>, p, C);
}

template <typename T>
cudaError_t run_logprobs(LpParams p, int num_sms, cudaStream_t stream) {
  const bool sums = !p.logZ_in, top = p.n_top > 0, rank = p.rank != nullptr;
  if (!sums && !top && !rank) {
    if (p.T == 0) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((static_cast<long long>(p.rows) * p.T + 127) / 128)); cfg.blockDim = dim3(128);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, gather_logprobs_kernel<T>, p);
  }
  const int C = lp_cluster(num_sms, p.rows, p.V);
  // More tokens than a pass has counters for: their ranks take a pass each four.
  cudaError_t e = cudaSuccess;
  for (p.t0 = 0; e == cudaSuccess && (p.t0 == 0 || (rank && p.t0 < p.T)); p.t0 += kLpTok) {
    p.tn = p.T - p.t0 < kLpTok ? p.T - p.t0 : kLpTok;
    const bool first = p.t0 == 0;
    if (!first) { p.entropy = nullptr; p.logZ = nullptr; }
    e = top && first ? (sums ? (rank ? launch_logprobs<T, true, true, true>(p, C, stream) : launch_logprobs<T, true, true, false>(p, C, stream))
                             : (rank ? launch_logprobs<T, false, true, true>(p, C, stream) : launch_logprobs<T, false, true, false>(p, C, stream)))
        : sums ? (rank ? launch_logprobs<T, true, false, true>(p, C, stream) : launch_logprobs<T, true, false, false>(p, C, stream))
               : launch_logprobs<T, false, false, true>(p, C, stream);
  }
  return e;
}
