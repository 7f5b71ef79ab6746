// token_logprobs.cuh - log probabilities of given tokens, their ranks, the entropy of a row and its top alternatives, from
// logits in memory.  Part of hola_verify.cu (inside its anonymous namespace).
//
// One pass over a row of V logits:  m = max l,  s = sum e^(l-m),  t = sum e^(l-m)(l-m),  logZ = m + ln s,  H = ln s - t/s,
// logprob(x) = (l[x] - m) - ln s,  rank(x) = #{v : l[v] > l[x], or l[v] = l[x] and v < x},  and the n entries that come first in the
// order (logit descending, id ascending).  A row is one CTA's or is cut into parts for the CTAs of a cluster, which merge over
// distributed shared memory; thread i of a part takes groups i, i + 256, ... of 32 bytes (one load each).
//
// The alternatives cost the pass next to nothing: every thread keeps the maximum of what it has seen and the group that it first
// met it in.  Every eight threads put the best of their (maximum, group) pairs, in the order (value descending, group ascending),
// on a board of 32 (every four on one of 64, for more than twenty alternatives); let the n-th best there be (w, g).  At least n entries lie at or before it (those maxima), so every one of the
// part's n best has a value above w, or w itself in a group up to g.  Only threads whose own pair is at or before (w, g) can hold
// such entries.  The group of their maximum is read again, out of the L2, and their other groups where the second-best may qualify
// too.  What qualifies (n entries and some more) goes to the row's first CTA, which places each entry by counting those before it.

constexpr int kLpThreads = 256;
constexpr int kLpWarps = kLpThreads / 32;
constexpr int kLpSpots = 128;          // entries that a part may send unsorted; beyond that it sends its 32 best
constexpr float kLpSlack = 4.f;        // how far a maximum may rise above the point that the sums are taken about
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
  int spots;                   // entries it sends
};

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
// The first `n` of 32 waiting keys into a sorted list.  (Out of line: rarely called, and code that is not fetched costs nothing.)
__device__ __noinline__ uint64_t lp_take_in(uint64_t best, const uint64_t* waiting, int n) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  const uint64_t a = lp_sort(lane < n ? waiting[lane] : 0, lane);
  best = lp_merge(best, __shfl_sync(0xffffffffu, a, 31 - lane), lane);
  __syncwarp();
  return best;
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

__device__ __forceinline__ float lp_float(float x) { return x; }
__device__ __forceinline__ float lp_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float lp_float(__half x) { return __half2float(x); }

// A token that is ranked.  An entry comes before it where its logit is larger, or as large and its id smaller: in groups before the
// token's own where !(l <= below), `below` the type's next number under its logit (for -inf a NaN, and every entry counts), in groups
// behind it where !(l <= l[x]).
template <typename T>
struct LpToken {
  int x;
  float l;
  uint32_t limit[2];           // 0: behind it, 1: before it; the number's bits, 16-bit ones twice
  __device__ __forceinline__ void set(int x_, bool have, const T* at) {
    x = x_;
    uint32_t b;
    if (sizeof(T) == 4) {
      b = have ? *reinterpret_cast<const uint32_t*>(at) : 0x7fffffffu;
      l = __uint_as_float(b);
      if (b == 0x80000000u) b = 0u;
      limit[0] = b;
      limit[1] = b == 0u ? 0x80000001u : b & 0x80000000u ? b + 1u : b - 1u;
    } else {
      b = have ? *reinterpret_cast<const uint16_t*>(at) : 0x7fffu;
      LpGroup<T> g;
      g.w[0] = b;
      l = g.entry(0);
      if (b == 0x8000u) b = 0u;
      limit[0] = b * 0x10001u;
      limit[1] = (b == 0u ? 0x8001u : b & 0x8000u ? b + 1u : b - 1u) * 0x10001u;
    }
  }
};

// Entries of the group above a limit (or not comparable with it): 1.0 for each, added up two at a time.
template <typename T>
__device__ __forceinline__ int lp_count(const LpGroup<T>& g, uint32_t limit) {
  if (sizeof(T) == 4) {
    uint64_t n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      g.pair(i, a, b);
      asm("set.gtu.f32.f32 %0, %0, %1;" : "+f"(a) : "f"(__uint_as_float(limit)));
      asm("set.gtu.f32.f32 %0, %0, %1;" : "+f"(b) : "f"(__uint_as_float(limit)));
      n = add2(n, pack2(a, b));
    }
    float a, b;
    unpack2(n, a, b);
    return static_cast<int>(a + b);
  }
  LpGroup<T> n;
  n.w[0] = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (std::is_same<T, __nv_bfloat16>::value) {
      const __nv_bfloat162 one = __hgtu2(*reinterpret_cast<const __nv_bfloat162*>(&g.w[i]), *reinterpret_cast<const __nv_bfloat162*>(&limit));
      const __nv_bfloat162 sum = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&n.w[0]), one);
      n.w[0] = *reinterpret_cast<const uint32_t*>(&sum);
    } else {
      const __half2 one = __hgtu2(*reinterpret_cast<const __half2*>(&g.w[i]), *reinterpret_cast<const __half2*>(&limit));
      const __half2 sum = __hadd2(*reinterpret_cast<const __half2*>(&n.w[0]), one);
      n.w[0] = *reinterpret_cast<const uint32_t*>(&sum);
    }
  }
  float a, b;
  n.pair(0, a, b);
  return static_cast<int>(a + b);
}

// One thread's view of its part of the row.  Its sums are taken about `ref`, which trails the maximum by kLpSlack at most: a rise of
// the maximum then rarely makes a warp rescale.  In units of ln 2: x = l log2 e - ref log2 e, s = sum 2^x, t = sum 2^x x.
template <typename T, bool kSums, bool kTop, int kRank>
struct LpThread {
  static constexpr int E = LpGroup<T>::kEntries;
  float m, second;             // maximum, and that of the other groups
  float ref, rise, shift;      // rise: where the next rescaling is due; shift = -ref log2 e
  uint64_t s2, t2;             // two halves of either sum
  int at;                      // group that holds the maximum, the first one that does
  bool bad;
  int count[kRank ? kRank : 1];

  __device__ __forceinline__ explicit LpThread(int first) : shift(0.f), s2(0), t2(0), at(first), bad(false) {
    m = second = ref = rise = -CUDART_INF_F;
#pragma unroll
    for (int q = 0; q < (kRank ? kRank : 1); ++q) count[q] = 0;
  }

  // Groups j, j + kLpThreads ... (N of them), by all lanes of a warp together (a lane without one brings a group of -inf); v0: the first
  // one's first entry.  kPlain: they are whole and come behind those before them.
  template <bool kPlain, int N>
  __device__ __forceinline__ void take(const LpGroup<T>* g, int j, int v0, const LpToken<T>* tok, float l_min, bool ragged) {
    float top[N], most;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      top[u] = g[u].largest();
      if (!kSums) bad = bad || !(top[u] < CUDART_INF_F);
      if (kTop) {
        second = fmaxf(second, fminf(top[u], m));
        if (top[u] > m || (!kPlain && top[u] == m && j < at)) at = j + u * kLpThreads;
      }
      m = fmaxf(m, top[u]);
      most = u ? fmaxf(most, top[u]) : top[u];
    }
    // seldom: the maximum rises, or there are entries before a token
    if (__any_sync(0xffffffffu, (kSums && most > rise) || (kRank && most >= l_min))) {
      if (kRank && most >= l_min) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
          const int v = v0 + u * kLpThreads * E;
#pragma unroll
          for (int q = 0; q < kRank; ++q) {
            if (!(top[u] >= tok[q].l)) continue;
            if (ragged || (v <= tok[q].x && v + E > tok[q].x)) {
#pragma unroll
              for (int i = 0; i < E; ++i) {
                const float l = g[u].entry(i);
                count[q] += v + i >= 0 && (l > tok[q].l || (l == tok[q].l && v + i < tok[q].x)) ? 1 : 0;
              }
            } else {
              count[q] += lp_count(g[u], v < tok[q].x ? tok[q].limit[1] : tok[q].limit[0]);
            }
          }
        }
      }
      if (kSums && most > rise) {
        const float old = shift;
        // (Rounded, the shift is off by up to 2^-24 of itself, in every exponent alike: 0.05 at most here.  Beyond, where it would be
        // the exponents that count, NaN: every group goes the long way below, from differences.)
        shift = fabsf(most) < 5e5f ? -most * kLog2e : CUDART_NAN_F;
        if (ref != -CUDART_INF_F) {
          float dx = shift - old;
          if (!(dx == dx)) {                             // one of them from differences: x of the same logit, now less then
            const float now = shift == shift ? fmaf(ref, kLog2e, shift) : (ref - most) * kLog2e;
            dx = now - (old == old ? fmaf(ref, kLog2e, old) : 0.f);
          }
          dx = fmaxf(dx, -1e28f);
          const float e = ex2_approx(dx);
          const uint64_t e2 = pack2(e, e);
          t2 = mul2(fma2(pack2(dx, dx), s2, t2), e2);
          s2 = mul2(s2, e2);
        }
        ref = most;
        rise = most + kLpSlack;
      }
    }
    if (!kSums) return;
    const uint64_t l2e = pack2(kLog2e, kLog2e), sh = pack2(shift, shift);
    uint64_t ps[2] = {0, 0}, pt[2] = {0, 0};
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int i = 0; i < E / 2; ++i) {
        float a, b;
        g[u].pair(i, a, b);
        const uint64_t x = fma2(pack2(a, b), l2e, sh);
        unpack2(x, a, b);
        const uint64_t e = pack2(ex2_approx(a), ex2_approx(b));
        ps[i & 1] = u == 0 && i < 2 ? e : add2(ps[i & 1], e);
        pt[i & 1] = u == 0 && i < 2 ? mul2(e, x) : fma2(e, x, pt[i & 1]);
      }
    const uint64_t both = add2(pt[0], pt[1]);
    float a, b;
    unpack2(both, a, b);
    if (a + b == a + b) {
      s2 = add2(s2, add2(ps[0], ps[1]));
      t2 = add2(t2, both);
      return;
    }
    // 0 * -inf: entries that are masked (-inf, or as low as the type goes), or too large for x; or there is no distribution
    const float from = shift == shift ? fmaf(ref, kLog2e, shift) : 0.f;       // (about the same point as everything else)
#pragma unroll
    for (int u = 0; u < N; ++u) {
      if (!(top[u] < CUDART_INF_F)) {
        bad = true;
      } else if (top[u] != -CUDART_INF_F) {
        float s = 0.f, t = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float x = fmaf(lp_below(g[u].entry(i), ref), kLog2e, from), e = ex2_approx(x);
          s += e;
          t = fmaf(e, x, t);
        }
        s2 = add2(s2, pack2(s, 0.f));
        t2 = add2(t2, pack2(t, 0.f));
      }
    }
  }

  // The sums about the thread's own maximum: m, sum e^(l-m), sum e^(l-m)(l-m).
  __device__ __forceinline__ void sums(float& s, float& t) const {
    float a, b, c, d;
    unpack2(s2, a, b);
    unpack2(t2, c, d);
    s = a + b;
    t = c + d;
    if (m == -CUDART_INF_F) return;
    const float x = shift == shift ? fmaf(m, kLog2e, shift) : (m - ref) * kLog2e;     // (of the maximum, as it was summed)
    const float e = ex2_approx(-x);
    t = kLn2 * (e * fmaf(-x, s, t));
    s *= e;
  }
};

// Entries of group j at or before (w, g_last) to the part's spots, as far as there is room.
template <typename T>
__device__ __forceinline__ void lp_send(const LpGroup<T>& g, const LpRow<T>& r, int j, uint64_t lim, float w, int g_last, uint64_t* spots,
                                        int* n_spots) {
  if (lim != 0) {
    const float top = g.largest();
    if (!(top > w || (top == w && j <= g_last))) return;
  }
  const int v0 = r.first(j);
  unsigned which = 0;
#pragma unroll
  for (int e = 0; e < LpGroup<T>::kEntries; ++e) {
    const float l = g.entry(e);
    which |= (lim == 0 || l > w || (l == w && j <= g_last)) && v0 + e >= 0 && v0 + e < r.V ? 1u << e : 0u;
  }
  if (!which) return;
  int spot = atomicAdd(n_spots, __popc(which));
#pragma unroll
  for (int e = 0; e < LpGroup<T>::kEntries; ++e)
    if (which >> e & 1u) {
      if (spot < kLpSpots) spots[spot] = lp_key(g.entry(e), v0 + e);
      ++spot;
    }
}

// Writes what a row without a token gets (see the header), or one whose accept length cannot be.
__device__ __forceinline__ void lp_no_token(const LpParams& p, int row, bool valid, bool rank) {
  const float none = valid ? 0.f : CUDART_NAN_F;
  if (threadIdx.x == 0) {
    p.logprob[row] = none;
    if (rank) p.rank[row] = -1;
    if (!valid && p.status) atomicOr(p.status, HOLA_FLAG_BAD_TOKEN);
  }
  if (threadIdx.x < p.n_top) {
    p.top_ids[static_cast<size_t>(row) * p.n_top + threadIdx.x] = -1;
    p.top_logprobs[static_cast<size_t>(row) * p.n_top + threadIdx.x] = none;
  }
}

// CTAs per SM, by registers: what 16-bit logits are expanded to and the alternatives' bookkeeping do not fit 64 together, nor do two
// groups of fp32 on the way (us at 80 / at 64 registers: 192 x 32000 bf16, 8 alternatives 12.7 / 15.0; 384 x 128256 fp32, 20
// alternatives 42.5 / 46.5; but 2304 x 128256 bf16, none 134.3 / 116.2).
template <typename T>
constexpr int lp_per_sm(bool sums, bool top) { return (sums && top && sizeof(T) == 2) || sizeof(T) == 4 ? 3 : 4; }

// What bounds it: HBM for large batches; for a few rows the chain token -> its logit -> pass -> board -> second look -> counting.
// N: groups that a thread takes together.
template <typename T, bool kSums, bool kTop, int kRank, int N>
__global__ void __launch_bounds__(kLpThreads, lp_per_sm<T>(kSums, kTop)) token_logprobs_kernel(const LpParams p, int C) {
  constexpr int E = LpGroup<T>::kEntries;
  __shared__ uint64_t spots[kTop ? kLpMaxCluster : 1][kLpSpots];       // first CTA: what every part sends
  __shared__ LpPart parts[kLpMaxCluster];
  __shared__ uint64_t own_spots[kTop ? kLpSpots : 1];
  __shared__ uint64_t side[kTop ? kLpMaxCluster * kLpSpots : 1];       // first CTA: all of it, and each entry's place
  __shared__ int before_it[kTop ? kLpMaxCluster * kLpSpots : 1];
  __shared__ float row_m, row_ls;
  __shared__ uint64_t lists[kTop ? kLpWarps * 32 : 1];   // board, or the warps' sorted lists
  __shared__ uint64_t fresh[kTop ? kLpWarps : 1][32];
  __shared__ uint8_t looked_at[kLpWarps][32];
  __shared__ LpPart warp_parts[kLpWarps];
  __shared__ int n_spots;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = blockIdx.x / C, part = blockIdx.x - row * C;
  // the other CTAs of the cluster have started (looked at before anything is sent to them)
  if (C > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
  if (tid == 0) n_spots = 0;
  grid_dependency_wait();
  grid_dependency_release();

  // The part's groups.
  const LpRow<T> r(static_cast<const T*>(p.logits) + static_cast<size_t>(row) * p.row_stride, p.V);
  const int per = (r.groups + C - 1) / C;
  const int j_end = min(r.groups, (part + 1) * per), j_begin = min(part * per, j_end);

  // What the row is asked for.  (Emitted form: row j of a sequence holds a token up to its accept length.)
  int j_seq = 0, len = 0;
  if (p.accept_len) {
    const int b = row / (p.k + 1);
    j_seq = row - b * (p.k + 1);
    len = p.accept_len[b];
    const bool valid = len >= 0 && len <= p.k;
    if (!valid || j_seq > len) {                         // (the same in every CTA of the cluster)
      if (C > 1) asm volatile("barrier.cluster.wait;" ::: "memory");
      if (part == 0) lp_no_token(p, row, valid, kRank > 0);
      return;
    }
  }

  // Rounds in which every thread has N whole groups, and some for what is left; the row's first group, where it lacks entries, has one
  // of its own.  The first groups are on their way while the tokens and their logits are looked up.
  const int j_first = max(j_begin, min(r.whole_begin, j_end)), rounds = max(0, min(j_end, r.whole_end) - j_first) / (N * kLpThreads);
  // What is on the way stays in its registers until it is used (a copy waits for it): rounds by turns.  384 x 32000 fp32, one / two on
  // the way: 15.1 / 13.3 us out of HBM, 10.3 / 10.6 out of the L2; two of two groups each, 384 x 128256: 42.5 / 48.6, no registers left
  // for it; 16-bit logits, 192 x 32000: 12.7 / 13.1.  Bulk prefetches into the L2 instead: 13.4 and 11.4 us, 42.5 -> 48.1.
  constexpr int D = sizeof(T) == 4 && N == 1 ? 2 : 1;
  LpGroup<T> next[D][N];
  const T* ptr = r.base + static_cast<size_t>(j_first + tid) * E;
#pragma unroll
  for (int d = 0; d < D; ++d)
    if (d < rounds) {
#pragma unroll
      for (int u = 0; u < N; ++u) next[d][u].load(ptr + (d * N + u) * kLpThreads * E);
    }

  LpToken<T> tok[kRank ? kRank : 1];
  float l_min = CUDART_INF_F;
  const int n = p.tn;
#pragma unroll
  for (int q = 0; q < kRank; ++q) {
    int x = -1;
    if (q < n)
      x = p.accept_len ? (j_seq < len ? p.draft_tok[static_cast<size_t>(row / (p.k + 1)) * p.k + j_seq] : p.next_tok[row / (p.k + 1)])
                       : p.tokens[static_cast<size_t>(row) * p.T + p.t0 + q];
    const bool have = x >= 0 && x < p.V;
    tok[q].set(x, have, r.base + (have ? static_cast<size_t>(x) + r.off : 0));
    if (have) l_min = fminf(l_min, tok[q].l);
  }

  int j = j_first + tid;
  LpThread<T, kSums, kTop, kRank> th(j);
#pragma unroll 1
  for (int i = 0; i < rounds; i += D) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      if (d > 0 && i + d >= rounds) break;
      LpGroup<T> g[N];
#pragma unroll
      for (int u = 0; u < N; ++u) g[u] = next[d][u];
      if (i + d + D < rounds) {
#pragma unroll
        for (int u = 0; u < N; ++u) next[d][u].load(ptr + (D * N + u) * kLpThreads * E);
      }
      ptr += N * kLpThreads * E;
      th.template take<true, N>(g, j, r.first(j), tok, l_min, false);
      j += N * kLpThreads;
    }
  }
#pragma unroll 1
  for (int i = 0; i <= N; ++i, j += kLpThreads) {        // (less than N groups a thread and a ragged one; the first)
    if (i == N) {
      if (j_begin == j_first || warp != 0) break;
      j = lane == 0 ? 0 : j_end;
    } else if (j - tid >= j_end) {
      continue;
    }
    const bool some = j < j_end, ragged = !some || !r.whole(j);
    LpGroup<T> g = r.none();
    if (some) g = r.get(j);
    th.template take<false, 1>(&g, j, some ? r.first(j) : INT32_MAX - E, tok, l_min, ragged);
  }

  // The threads' sums and counts, over the warp.
  LpPart mine;
  mine.m = warp_max_f32(th.m);
  mine.s = mine.t = 0.f;
  mine.spots = 0;
  if (kSums) {
    th.sums(mine.s, mine.t);
    const float d = th.m == -CUDART_INF_F ? 0.f : lp_below(th.m, mine.m), e = ex2_approx(d * kLog2e);
    mine.t = e * fmaf(d, mine.s, mine.t);
    mine.s *= e;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      mine.s += __shfl_xor_sync(0xffffffffu, mine.s, o);
      mine.t += __shfl_xor_sync(0xffffffffu, mine.t, o);
    }
  }
  mine.bad = __any_sync(0xffffffffu, th.bad) ? 1u : 0u;
#pragma unroll
  for (int q = 0; q < kLpTok; ++q) mine.count[q] = q < kRank ? __reduce_add_sync(0xffffffffu, th.count[q < kRank ? q : 0]) : 0;
  if (lane == 0) warp_parts[warp] = mine;

  if (kTop) {
    const uint64_t own = th.at < j_end ? lp_key(th.m, th.at) : 0;       // (a thread without a group: nothing)
    // (fewer threads to a place of the board where not all of them have groups)
    const int held = j_end - j_begin, board = p.n_top > 20 ? 64 : 32;
    int share = kLpThreads / board;
    while (share > 1 && held <= share / 2 * board) share >>= 1;
    uint64_t a = own;
    for (int o = 1; o < share; o <<= 1) {
      const uint64_t b = __shfl_xor_sync(0xffffffffu, a, o);
      if (b > a) a = b;
    }
    if ((lane & (share - 1)) == 0 && tid < board * share) lists[tid / share] = a;
    __syncthreads();
    // every warp for itself: the n-th best on the board (its keys differ, but for empty ones)
    uint64_t lim = 0;                                    // (0: fewer hold anything)
    for (int at = 0; at < board; at += 32) {
      const uint64_t key = lists[at + lane];
      int before = 0;
#pragma unroll 8
      for (int i = 0; i < board; ++i) before += lists[i] > key ? 1 : 0;
      const unsigned nth = __ballot_sync(0xffffffffu, key != 0 && before == p.n_top - 1);
      if (nth) lim = __shfl_sync(0xffffffffu, key, __ffs(nth) - 1);
    }
    float w = lp_value(static_cast<uint32_t>(lim >> 32));
    int g_last = static_cast<int>(~static_cast<uint32_t>(lim));
    // Masked rows: fewer entries than alternatives are left, the others are -inf by rising id.  The part's first ones serve, where 64
    // entries hold enough of them (otherwise: as where there is no room).
    const bool masked = lim != 0 && w == -CUDART_INF_F;
    if (masked) {
      g_last = -1;                                       // (entries above w only)
      if (warp == 0) {
        const int v_begin = max(0, r.first(j_begin)), v_end = min(p.V, r.first(j_end));
        const int v = v_begin + 2 * lane;
        const bool a = v < v_end && lp_float(r.base[static_cast<size_t>(v) + r.off]) == w,
                   b = v + 1 < v_end && lp_float(r.base[static_cast<size_t>(v) + 1 + r.off]) == w;
        const unsigned as = __ballot_sync(0xffffffffu, a), bs = __ballot_sync(0xffffffffu, b), below = (1u << lane) - 1u;
        const int found = __popc(as) + __popc(bs), place = __popc(as & below) + __popc(bs & below);
        const bool enough = found >= p.n_top || v_end - v_begin <= 64;
        int first = 0;
        if (lane == 0) first = atomicAdd(&n_spots, enough ? min(found, p.n_top) : kLpSpots + 1);
        first = __shfl_sync(0xffffffffu, first, 0);
        if (enough && a && place < p.n_top && first + place < kLpSpots) own_spots[first + place] = lp_key(w, v);
        if (enough && b && place + (a ? 1 : 0) < p.n_top && first + place + (a ? 1 : 0) < kLpSpots)
          own_spots[first + place + (a ? 1 : 0)] = lp_key(w, v + 1);
      }
    }
    const bool mine_too = masked ? th.m > w : own != 0 && own >= lim;
    const bool again = mine_too && (lim == 0 || (masked ? th.second > w : th.second >= w));
    if (mine_too && !again) lp_send(r.get(th.at), r, th.at, lim, w, g_last, own_spots, &n_spots);
    // The groups of a thread, the row's first one last; dealt out to the lanes.
    const int steps = (j_end - j_first + kLpThreads - 1) / kLpThreads + (j_begin < j_first ? 1 : 0);
    auto group_of = [&](int i) {
      const int who = i / steps, k = i - who * steps, t = warp * 32 + looked_at[warp][who];
      const int jj = j_first + t + k * kLpThreads;
      return k == steps - 1 && j_begin < j_first ? (t == 0 ? 0 : j_end) : jj;
    };
    const unsigned look = __ballot_sync(0xffffffffu, again);
    if (look) {
      if (again) looked_at[warp][__popc(look & ((1u << lane) - 1u))] = static_cast<uint8_t>(lane);
      __syncwarp();
      const int total = __popc(look) * steps;
      for (int i = lane; i < total; i += 32) {
        const int jj = group_of(i);
        if (jj < j_end) lp_send(r.get(jj), r, jj, lim, w, g_last, own_spots, &n_spots);
      }
    }
    __syncthreads();
    if (n_spots > kLpSpots) {
      // More than there is room for (the best entries crowd together, or many are equal): with the n-th best of ALL threads' pairs for
      // a limit, the part's 32 best by sorted lists, from all groups of the threads that may hold some.
      __syncthreads();                                   // (everyone has seen n_spots, and the board)
      const uint64_t firsts = lp_merge_warps(lp_sort(own, lane), lists, warp, lane);
      if (warp == 0 && lane == p.n_top - 1) own_spots[0] = firsts;
      __syncthreads();
      lim = own_spots[0];
      w = lp_value(static_cast<uint32_t>(lim >> 32));
      g_last = static_cast<int>(~static_cast<uint32_t>(lim));
      const bool holds = own != 0 && own >= lim;
      const unsigned all = __ballot_sync(0xffffffffu, holds);
      if (holds) looked_at[warp][__popc(all & ((1u << lane) - 1u))] = static_cast<uint8_t>(lane);
      __syncwarp();
      const int total = __popc(all) * steps;
      uint64_t best = 0;
      int waiting = 0;
#pragma unroll 1
      for (int i0 = 0; i0 < total; i0 += 32) {
        const int i = i0 + lane;
        int jj = -1;
        if (i < total) {
          jj = group_of(i);
          if (jj >= j_end) jj = -1;
        }
        LpGroup<T> g = {};
        if (jj >= 0) g = r.get(jj);
        const int v0 = r.first(jj);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float l = g.entry(e);
          const bool in = jj >= 0 && v0 + e >= 0 && v0 + e < p.V && (lim == 0 || l > w || (l == w && jj <= g_last));
          const unsigned mask = __ballot_sync(0xffffffffu, in);
          if (!mask) continue;
          const int fit = __popc(mask);
          if (waiting + fit > 32) {                      // full: what waits goes into the list
            best = lp_take_in(best, fresh[warp], waiting);
            waiting = 0;
          }
          if (in) fresh[warp][waiting + __popc(mask & ((1u << lane) - 1u))] = lp_key(l, v0 + e);
          waiting += fit;
        }
      }
      best = lp_take_in(best, fresh[warp], waiting);
      __syncthreads();
      best = lp_merge_warps(best, lists, warp, lane);
      if (warp == 0) own_spots[lane] = best;
      if (tid == 0) n_spots = 32;
      __syncthreads();
    }
  } else {
    __syncthreads();
  }

  // The part, to the first CTA of the cluster.
  if (C > 1) asm volatile("barrier.cluster.wait;" ::: "memory");
  if (warp == 0) {
    LpPart all = {-CUDART_INF_F, 0.f, 0.f, 0u, {0, 0, 0, 0}, 0};
    if (lane < kLpWarps) all = warp_parts[lane];
    const float m = warp_max_f32(all.m);
    if (kSums) {
      const float d = all.m == -CUDART_INF_F ? 0.f : lp_below(all.m, m), e = ex2_approx(d * kLog2e);
      all.t = e * fmaf(d, all.s, all.t);
      all.s *= e;
    }
    all.m = m;
#pragma unroll
    for (int o = kLpWarps / 2; o > 0; o >>= 1) {
      all.s += __shfl_xor_sync(0xffffffffu, all.s, o);
      all.t += __shfl_xor_sync(0xffffffffu, all.t, o);
      all.bad |= __shfl_xor_sync(0xffffffffu, all.bad, o);
#pragma unroll
      for (int q = 0; q < kRank; ++q) all.count[q] += __shfl_xor_sync(0xffffffffu, all.count[q], o);
    }
    all.spots = kTop ? n_spots : 0;
    LpPart* to = C > 1 ? cg::this_cluster().map_shared_rank(&parts[part], 0) : &parts[part];
    if (lane == 0) *to = all;
  } else if (kTop && warp <= kLpSpots / 32) {
    uint64_t* to = C > 1 ? cg::this_cluster().map_shared_rank(&spots[part][0], 0) : &spots[part][0];
    const int i = (warp - 1) * 32 + lane;
    if (i < n_spots) to[i] = own_spots[i];
  }
  if (C > 1) cluster_sync_all();
  else __syncthreads();
  if (part != 0 || (!kTop && warp != 0)) return;

  // What the parts sent, side by side: warp c copies part c's.
  int total = 0;
  if (kTop) {
    const int sent = lane < C ? parts[lane].spots : 0;
    int upto = sent;
#pragma unroll
    for (int o = 1; o < kLpMaxCluster; o <<= 1) {
      const int below = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += below;
    }
    total = __shfl_sync(0xffffffffu, upto, kLpMaxCluster - 1);
    const int mine = __shfl_sync(0xffffffffu, sent, warp), first = __shfl_sync(0xffffffffu, upto, warp) - mine;
#pragma unroll 1
    for (int i = lane; i < mine; i += 32) {
      side[first + i] = spots[warp][i];
      before_it[first + i] = 0;
    }
    __syncthreads();
    // Every entry's place is the number of those before it: a warp compares all of them with an eighth of them.
    const int slice = (total + kLpWarps - 1) / kLpWarps, from = warp * slice, to = min(total, from + slice);
    if (from < to) {
#pragma unroll 1
      for (int i = lane; i < total; i += 32) {
        const uint64_t key = side[i];
        int n_before = 0;
#pragma unroll 4
        for (int k = from; k < to; ++k) n_before += side[k] > key ? 1 : 0;
        atomicAdd(&before_it[i], n_before);
      }
    }
  }

  // The row, by warp 0.
  if (warp == 0) {
    LpPart all = {-CUDART_INF_F, 0.f, 0.f, 0u, {0, 0, 0, 0}, 0};
    if (lane < C) all = parts[lane];
    const bool bad = __any_sync(0xffffffffu, all.bad != 0);
    float m = 0.f, ls, logZ, H = 0.f;
    if (kSums) {
      m = warp_max_f32(all.m);
      const float d = all.m == -CUDART_INF_F ? 0.f : lp_below(all.m, m), e = ex2_approx(d * kLog2e);
      float s = e * all.s, t = e * fmaf(d, all.s, all.t);
#pragma unroll
      for (int o = kLpMaxCluster / 2; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        t += __shfl_xor_sync(0xffffffffu, t, o);
      }
      if (bad) {
        m = ls = logZ = H = CUDART_NAN_F;
      } else if (m == -CUDART_INF_F) {
        ls = logZ = m;                                   // nothing is left of the row
      } else {
        ls = logf(s);
        logZ = m + ls;
        H = fmaxf(0.f, ls - quotient(t, s));
      }
      ls = __shfl_sync(0xffffffffu, ls, 0);              // (lanes beyond the parts hold other sums)
    } else {
      ls = logZ = p.logZ_in[row];
    }
    if (lane == 0) {
      if (kSums && p.entropy) p.entropy[row] = H;
      if (kSums && p.logZ) p.logZ[row] = logZ;
      row_m = bad ? CUDART_NAN_F : m;
      row_ls = ls;
    }
    unsigned flags = bad ? HOLA_FLAG_BAD_LOGIT : 0u;
    // (no token: 0; one that the vocabulary does not have: NaN)
    if (kRank) {
#pragma unroll
      for (int q = 0; q < kRank; ++q) all.count[q] = __reduce_add_sync(0xffffffffu, all.count[q]);
      if (lane < n) {
        int x = tok[0].x, before = all.count[0];
        float l = tok[0].l;
#pragma unroll
        for (int q = 1; q < kRank; ++q)
          if (lane == q) { x = tok[q].x; before = all.count[q]; l = tok[q].l; }
        const size_t at = static_cast<size_t>(row) * p.T + p.t0 + lane;
        const bool have = x >= 0 && x < p.V, none = !p.accept_len && x == -1;
        if (!have && !none) flags |= HOLA_FLAG_BAD_TOKEN;
        p.logprob[at] = have ? lp_logprob(l, m, ls) : none ? 0.f : CUDART_NAN_F;
        p.rank[at] = have && !bad ? before : -1;
      }
    } else {
      for (int q = lane; q < p.T; q += 32) {
        const int x = !p.accept_len ? p.tokens[static_cast<size_t>(row) * p.T + q]
                      : j_seq < len ? p.draft_tok[static_cast<size_t>(row / (p.k + 1)) * p.k + j_seq] : p.next_tok[row / (p.k + 1)];
        const bool have = x >= 0 && x < p.V, none = !p.accept_len && x == -1;
        if (!have && !none) flags |= HOLA_FLAG_BAD_TOKEN;
        p.logprob[static_cast<size_t>(row) * p.T + q] =
            have ? lp_logprob(lp_float(r.base[static_cast<size_t>(x) + r.off]), m, ls) : none ? 0.f : CUDART_NAN_F;
      }
    }
    if (p.status) {
      __syncwarp();
      flags = __reduce_or_sync(0xffffffffu, flags);
      if (lane == 0 && flags) atomicOr(p.status, flags);
    }
  }
  if (kTop) {
    __syncthreads();
    const size_t at = static_cast<size_t>(row) * p.n_top;
    const float m = row_m, ls = row_ls;
    if (m != m) {
      if (tid < p.n_top) { p.top_ids[at + tid] = -1; p.top_logprobs[at + tid] = CUDART_NAN_F; }
      return;
    }
#pragma unroll 1
    for (int i = tid; i < total; i += kLpThreads) {
      const int place = before_it[i];
      const uint64_t key = side[i];
      if (place < p.n_top) {
        p.top_ids[at + place] = static_cast<int>(~static_cast<uint32_t>(key));
        p.top_logprobs[at + place] = lp_logprob(lp_value(static_cast<uint32_t>(key >> 32)), m, ls);
      }
    }
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

// CTAs per row: up to three on an SM, as long as a thread keeps a group or two of its own.  Start, merges and the second look are
// latency, some 4 us a CTA, which more CTAs only add to, and a second wave for a few of them costs as much as the first.  us with 1 /
// 2 / 4 / 8: 69 x 50003 fp16 18.3 / 14.8 / 15.4 / 23.0; 192 x 32000 bf16 13.7 / 12.7 / 18.4 / 30.3; 384 x 128256 fp32 42.5 / 49.5 /
// 63.2 / 99.9; 5 x 32000 fp32 9.5 / 7.8 / 6.7 / 7.0.  The rule takes the best of them for the second and third, one doubling too many
// for the first and the last (four and eight: 4 % above the best).  Rows of the emitted form that return at once count like the others.
int lp_cluster(int num_sms, int rows, int V) {
  int C = 1;
  while (C < kLpMaxCluster && 2ll * rows * C <= 3ll * num_sms && V / (2 * C) >= 8 * kLpThreads) C <<= 1;
  return C;
}

template <typename T, bool kSums, bool kTop, int kRank, int N>
cudaError_t launch_logprobs(const LpParams& p, int C, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.rows) * C); cfg.blockDim = dim3(kLpThreads); cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(C); attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = C > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, kSums, kTop, kRank, N>, p, C);
}

// One token per row is the rule: the pass then carries one comparison instead of kLpTok.  Long rows of fp32 are taken two groups at a
// time, which halves what each costs beside its sums and doubles what is on the way (us, one / two: 384 x 128256, one CTA a row,
// 63 groups a thread 46.2 / 42.5; 32000 entries, 16 groups a thread 10.6 / 11.3 out of the L2, 13.3 / 13.1 out of HBM; 16-bit logits
// 116 / 142).
template <typename T, bool kSums, bool kTop, int N>
cudaError_t launch_logprobs_of(const LpParams& p, bool rank, int C, cudaStream_t stream) {
  return !rank ? launch_logprobs<T, kSums, kTop, 0, N>(p, C, stream)
         : p.tn == 1 ? launch_logprobs<T, kSums, kTop, 1, N>(p, C, stream) : launch_logprobs<T, kSums, kTop, kLpTok, N>(p, C, stream);
}
template <typename T, bool kSums, bool kTop>
cudaError_t launch_logprobs_of(const LpParams& p, bool rank, int C, cudaStream_t stream) {
  const bool two = sizeof(T) == 4 && p.V / C >= 32 * kLpThreads * (kLpGroupBytes / 4);
  return two ? launch_logprobs_of<T, kSums, kTop, sizeof(T) == 4 ? 2 : 1>(p, rank, C, stream)
             : launch_logprobs_of<T, kSums, kTop, 1>(p, rank, C, stream);
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
    e = top && first ? (sums ? launch_logprobs_of<T, true, true>(p, rank, C, stream) : launch_logprobs_of<T, false, true>(p, rank, C, stream))
                     : (sums ? launch_logprobs_of<T, true, false>(p, rank, C, stream) : launch_logprobs_of<T, false, false>(p, rank, C, stream));
  }
  return e;
}
