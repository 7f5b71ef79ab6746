// beams.cuh - one step of a beam search around the LM head: the best continuations over all beams and the vocabulary, and the beams'
// states put in the order of their parents.  Part of decode_ops.cu (inside its anonymous namespace).
//
// Selection.  Candidate (w, v) of a sequence has c = (score[w] - logZ[w]) + l[w][v] and the key c * weight[w], both in 64 bits; the n
// first in the order (key descending, beam ascending, logit descending, id ascending) are kept.  One pass over the logits in 32 bits:
// a = fma(l, weight, b), b = (score - logZ) weight rounded, is within 2^-24 (|a| + |b|) of the key.  A cluster of CTAs takes a sequence,
// every CTA a part of each row; a thread keeps the two largest a of its groups, those groups, and the largest of its other groups.
// Eight threads each put the best of theirs on a place of a board of 32 (four each on one of 64, for more than twenty candidates); let
// the n-th best there be w.  At least n candidates have a >= w, so each of the part's n best has a >= w - 2^-22 (|w| + max |b|): twice
// the bound above for either side, and the roundings of this line.  Only threads whose own largest is that large hold such entries;
// their two groups (all of theirs, where a third is as large) are read again, out of the L2, and what qualifies is placed, by keys in
// 64 bits, by counting those before it.  The n best go to the sequence's first CTA in their order, which merges the parts' lists.

constexpr int kBsThreads = 256;
constexpr int kBsWarps = kBsThreads / 32;
constexpr int kBsMaxBeams = 32, kBsMaxKept = 32;
constexpr int kBsMaxCluster = 16;
constexpr int kBsSpots = 64;           // candidates that a part may send unsorted; beyond that it sends its 32 best
constexpr int kBsAhead = 6;            // groups of a thread that are on the way
constexpr int kBsMaxV = 1 << 27;       // ids share a word with a beam and a logit

struct BsParams {
  const void* logits;
  long long seq_stride, beam_stride;   // entries
  int B, W, V, n;
  const float* logZ;                   // [B][W]
  const float* score;                  // [B][W]
  const uint8_t* finished;             // [B][W], or null
  const float* weight;                 // [B][W], or null: 1
  int end_token, keep_slots;
  float* score_out;                    // [B][n]
  int* parent;
  int* token;
  uint8_t* finished_out;               // or null
  unsigned* status;                    // or null
};

// A candidate in its order: the larger (hi, lo) comes first.  hi: the key; lo: beam (5 bits, reversed), logit (32), id (27, reversed).
struct BsCand {
  uint64_t hi, lo;
};
// (without branches: 103 candidates against one another 4.1 us with them)
__device__ __forceinline__ bool bs_before(const BsCand& a, const BsCand& b) {
  return static_cast<bool>(static_cast<int>(a.hi > b.hi) | (static_cast<int>(a.hi == b.hi) & static_cast<int>(a.lo > b.lo)));
}
__device__ __forceinline__ uint64_t bs_order(double x) {
  const uint64_t b = static_cast<uint64_t>(__double_as_longlong(x + 0.0));
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ uint64_t bs_low(int beam, float l, int id) {
  return static_cast<uint64_t>(31 - beam) << 59 | static_cast<uint64_t>(lp_order(l)) << 27 | static_cast<uint32_t>(kBsMaxV - 1 - id);
}
__device__ __forceinline__ int bs_beam(uint64_t lo) { return 31 - static_cast<int>(lo >> 59); }
__device__ __forceinline__ float bs_logit(uint64_t lo) { return lp_value(static_cast<uint32_t>(lo >> 27)); }
__device__ __forceinline__ int bs_id(uint64_t lo) { return kBsMaxV - 1 - static_cast<int>(lo & (kBsMaxV - 1)); }

// Sorted lists across a warp, as in token_logprobs.cuh, of candidates; {0, 0}: none.
__device__ __forceinline__ BsCand bs_exchange(const BsCand& a, int stride, bool first) {
  const BsCand b = {__shfl_xor_sync(0xffffffffu, a.hi, stride), __shfl_xor_sync(0xffffffffu, a.lo, stride)};
  return bs_before(a, b) == first ? a : b;
}
// The 32 first of two sorted lists, sorted; `reversed`: the second one from its end.
__device__ __forceinline__ BsCand bs_merge(BsCand a, const BsCand& reversed, int lane) {
  if (bs_before(reversed, a)) a = reversed;
#pragma unroll
  for (int stride = 16; stride > 0; stride >>= 1) a = bs_exchange(a, stride, (lane & stride) == 0);
  return a;
}
__device__ __noinline__ BsCand bs_take_in(BsCand best, const BsCand* waiting, int n) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  BsCand a = {0, 0};
  if (lane < n) a = waiting[lane];
#pragma unroll 1
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll 1
    for (int stride = size >> 1; stride > 0; stride >>= 1) a = bs_exchange(a, stride, ((lane & size) == 0) == ((lane & stride) == 0));
  const BsCand r = {__shfl_sync(0xffffffffu, a.hi, 31 - lane), __shfl_sync(0xffffffffu, a.lo, 31 - lane)};
  best = bs_merge(best, r, lane);
  __syncwarp();
  return best;
}

// A live beam's row, and this CTA's part of its whole groups of 32 bytes.  The first and the last group, where they lack entries, are the
// first CTA's (`edge`, or -1).
struct BsRow {
  double off, weight;
  const void* row;
  const unsigned char* at;             // group `begin`
  float b, w32;
  int beam, begin, count;
  int edge[2];
};

struct BsShared {
  BsRow rows[kBsMaxBeams];
  uint2 spots[kBsSpots];               // entries of this part: logit; row (5 bits) and id (27)
  BsCand own[kBsWarps * 32];           // this part's candidates (the ended beams among the first part's), or the warps' sorted lists
  int before_it[kBsSpots + kBsMaxBeams];
  BsCand sent[kBsMaxCluster][32];      // first CTA: every part's best, sorted
  int sent_by[kBsMaxCluster];          // their number
  BsCand waiting[kBsWarps][32];        // also: lists on their way through the merge
  uint64_t keys[kBsThreads];           // the threads' largest
  uint64_t board[kBsWarps][64];
  uint8_t looked_at[kBsWarps][32];
  unsigned bad_from[kBsMaxCluster];    // rows that hold NaN or +inf, as every CTA of the cluster has found them
  unsigned bad_here;
  int width, n_own;                    // width: groups of the row that has most of them in this part
  float b_max;
};

// a: the key in 32 bits.  (Kept finite: a mask may be as low as the type goes.  -inf is no candidate; NaN stays.)
__device__ __forceinline__ float bs_approx(float l, float w32, float b) {
  const float a = fmaf(l, w32, b);
  return fabsf(a) == CUDART_INF_F && fabsf(l) != CUDART_INF_F ? copysignf(3.402823466e38f, a) : a;
}

// Entries of group j of a row whose a is at least thr, to the part's spots.
template <typename T>
__device__ __forceinline__ void bs_note(BsShared& s, int li, int V, int j, float thr) {
  const BsRow& row = s.rows[li];
  const LpRow<T> r(static_cast<const T*>(row.row), V);
  const LpGroup<T> g = r.get(j);
  unsigned which = 0;
#pragma unroll
  for (int e = 0; e < LpGroup<T>::kEntries; ++e) {
    const float l = g.entry(e);
    which |= l > -CUDART_INF_F && bs_approx(l, row.w32, row.b) >= thr ? 1u << e : 0u;
  }
  if (!which) return;
  int spot = atomicAdd(&s.n_own, __popc(which));
  const uint32_t at = static_cast<uint32_t>(li) << 27 | static_cast<uint32_t>(r.first(j) & (kBsMaxV - 1));
#pragma unroll
  for (int e = 0; e < LpGroup<T>::kEntries; ++e)
    if (which >> e & 1u) {
      // (a row's first group may begin before entry 0: added up within 27 bits)
      if (spot < kBsSpots)
        s.spots[spot] = make_uint2(__float_as_uint(g.entry(e)), static_cast<uint32_t>(li) << 27 | ((at + static_cast<uint32_t>(e)) & (kBsMaxV - 1)));
      ++spot;
    }
}

// What bounds it: HBM for large batches; for a few rows the chain beams -> pass -> board -> second look -> cluster -> counting.
template <typename T>
__global__ void __launch_bounds__(kBsThreads, 2) beam_select_kernel(const BsParams p, int C) {
  extern __shared__ __align__(16) unsigned char bs_smem[];
  BsShared& s = *reinterpret_cast<BsShared*>(bs_smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int seq = blockIdx.x / C, part = blockIdx.x - seq * C;
  if (tid == 0) { s.n_own = 0; s.bad_here = 0; }
  if (tid < kBsMaxCluster) s.bad_from[tid] = 0;
  // (the other CTAs of the cluster have started, and their words stand at zero: looked at before anything is sent)
  if (C > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  grid_dependency_wait();
  grid_dependency_release();

  // The beams, by every warp for itself; warp 0 writes them down.
  unsigned flags = 0;
  float score = -CUDART_INF_F, logZ = 0.f, weight = 1.f;
  bool ended = false;
  if (lane < p.W) {
    const size_t at = static_cast<size_t>(seq) * p.W + lane;
    score = p.score[at];
    ended = p.finished && p.finished[at];
    if (p.weight) weight = p.weight[at];
    if (!ended) logZ = p.logZ[at];
  }
  // (of what is no beam nothing but the score counts)
  const bool bad_beam = score != -CUDART_INF_F && (!(score < CUDART_INF_F) || !(logZ < CUDART_INF_F) || !(weight > 0.f && weight < CUDART_INF_F));
  const bool there = !bad_beam && score != -CUDART_INF_F, reads = there && !ended && logZ != -CUDART_INF_F;
  if (__any_sync(0xffffffffu, bad_beam)) flags |= HOLA_FLAG_BAD_LOGIT;
  const unsigned ended_mask = __ballot_sync(0xffffffffu, there && ended);
  unsigned excluded = 0;                                 // rows that have turned out to hold NaN or +inf

  for (;;) {
    const unsigned live_mask = __ballot_sync(0xffffffffu, reads && !(excluded >> lane & 1u));
    const int live = __popc(live_mask);
    if (warp == 0) {
      const double off = static_cast<double>(score) - static_cast<double>(logZ);
      // (kept finite: an entry of -inf stays -inf beside it)
      const float b = fminf(fmaxf(static_cast<float>(off * static_cast<double>(weight)), -3.402823466e38f), 3.402823466e38f);
      if (live_mask >> lane & 1u) {
        BsRow& row = s.rows[__popc(live_mask & ((1u << lane) - 1u))];
        const T* at = static_cast<const T*>(p.logits) + static_cast<size_t>(seq) * p.seq_stride + static_cast<size_t>(lane) * p.beam_stride;
        const LpRow<T> r(at, p.V);
        const int whole = max(r.whole_end - r.whole_begin, 0), per = (whole + C - 1) / C, first = min(part * per, whole);
        row.off = off; row.weight = weight; row.row = at; row.b = b; row.w32 = weight; row.beam = lane;
        row.begin = r.whole_begin + first;
        row.count = min(per, whole - first);
        row.at = reinterpret_cast<const unsigned char*>(r.base) + static_cast<size_t>(row.begin) * kLpGroupBytes;
        row.edge[0] = part == 0 && r.whole_begin == 1 ? 0 : -1;
        row.edge[1] = part == 0 && r.whole_end < r.groups && r.whole_end >= r.whole_begin ? r.whole_end : -1;
      }
      const float most = warp_max_f32(live_mask >> lane & 1u ? fabsf(b) : 0.f);
      if (lane == 0) s.b_max = most;
      __syncwarp();
      const int width = __reduce_max_sync(0xffffffffu, lane < live ? s.rows[lane].count : 0);
      if (lane == 0) s.width = width;
    }
    __syncthreads();

    // The pass: the part's groups, `width` places for those of every row, dealt out to the threads in rounds, kBsAhead of them on the
    // way.  (So short rows, or many CTAs to a sequence, leave no thread idle: 2 x 16 x 10864 fp16 95.8 us with rounds of one row each,
    // and too few on the board for a limit.)
    float m = -CUDART_INF_F, second = -CUDART_INF_F, third = -CUDART_INF_F;
    int at = 0, at_second = 0;                           // rounds of the two largest; `rounds`: an edge
    const int width = s.width, rounds = static_cast<int>((static_cast<long long>(live) * width + kBsThreads - 1) / kBsThreads);
    auto take = [&](float top, float w32, float b, bool have, int beam, int where) {
      if (have && !(top < CUDART_INF_F)) atomicOr(&s.bad_here, 1u << beam);
      const float a = have ? bs_approx(top, w32, b) : -CUDART_INF_F;
      third = fmaxf(third, fminf(a, second));
      if (a > second) at_second = a > m ? at : where;
      second = fmaxf(second, fminf(a, m));
      if (a > m) at = where;
      m = fmaxf(m, a);
    };
    // Group of this thread in a round: row and place in it (row `live` or a place that the row lacks: none).
    auto group_of = [&](int round, int thread, int* j) {
      const int f = round * kBsThreads + thread, li = f / width;
      *j = f - li * width;
      return li;
    };
    if (rounds > 0) {
      const int q = kBsThreads / width, r = kBsThreads - q * width;
      int j_a = 0, li_a = group_of(0, tid, &j_a), j = j_a, li = li_a;        // of the round that is loaded next, and of the one that is looked at
      int count_a = 0, count = 0, beam = 0;
      float w32 = 1.f, b = 0.f;
      const unsigned char* row_at = nullptr;
      auto reload_a = [&]() {
        count_a = 0;
        if (li_a < live) { row_at = s.rows[li_a].at; count_a = s.rows[li_a].count; }
      };
      auto reload = [&]() {
        count = 0;
        if (li < live) { count = s.rows[li].count; w32 = s.rows[li].w32; b = s.rows[li].b; beam = s.rows[li].beam; }
      };
      reload_a();
      reload();
      LpGroup<T> next[kBsAhead];
      auto load = [&](LpGroup<T>& g) {
        if (j_a < count_a) g.load(reinterpret_cast<const T*>(row_at + static_cast<size_t>(j_a) * kLpGroupBytes));
        j_a += r;
        const bool over = j_a >= width;
        if (over) j_a -= width;
        if (over || q > 0) {
          li_a += q + (over ? 1 : 0);
          reload_a();
        }
      };
#pragma unroll
      for (int d = 0; d < kBsAhead; ++d)
        if (d < rounds) load(next[d]);
#pragma unroll 1
      for (int i = 0; i < rounds; i += kBsAhead) {
#pragma unroll
        for (int d = 0; d < kBsAhead; ++d) {
          if (i + d >= rounds) break;
          const float top = next[d].largest();
          if (i + d + kBsAhead < rounds) load(next[d]);
          take(top, w32, b, j < count, beam, i + d);
          j += r;
          const bool over = j >= width;
          if (over) j -= width;
          if (over || q > 0) {
            li += q + (over ? 1 : 0);
            reload();
          }
        }
      }
    }
    // (a thread of the first CTA for each edge)
    const int my_edge = tid < 2 * live ? s.rows[tid >> 1].edge[tid & 1] : -1;
    if (my_edge >= 0) {
      const BsRow& row = s.rows[tid >> 1];
      take(LpRow<T>(static_cast<const T*>(row.row), p.V).get_ragged(my_edge).largest(), row.w32, row.b, true, row.beam, rounds);
    }

    // The board: the n-th best of the threads' largest, taken together by eight or four that lie apart.  (Neighbouring threads have
    // neighbouring groups, and one beam's groups may hold all that is good: with neighbours on one place the limit would be another
    // beam's, and far too low.)
    {
      const int board = p.n > 20 ? 64 : 32;
      s.keys[tid] = m > -CUDART_INF_F ? lp_key(m, tid) : 0;
      __syncthreads();
      // (by every warp for itself)
      uint64_t place[2] = {0, 0};
#pragma unroll
      for (int w = 0; w < kBsWarps; ++w) {
        const uint64_t a = s.keys[w * 32 + lane];
        if (board == 64 && (w & 1)) place[1] = a > place[1] ? a : place[1];
        else place[0] = a > place[0] ? a : place[0];
      }
      s.board[warp][lane] = place[0];
      s.board[warp][32 + lane] = place[1];
      __syncwarp();
      uint64_t lim = 0;
      for (int at = 0; at < board; at += 32) {
        const uint64_t key = at ? place[1] : place[0];
        int before = 0;
#pragma unroll 8
        for (int i = 0; i < board; ++i) before += s.board[warp][i] > key ? 1 : 0;
        const unsigned nth = __ballot_sync(0xffffffffu, key != 0 && before == p.n - 1);
        if (nth) lim = __shfl_sync(0xffffffffu, key, __ffs(nth) - 1);
      }
      // (offsets beyond 1e30, where the bound on a would run over: everything qualifies)
      float thr = -CUDART_INF_F;
      if (lim != 0 && s.b_max < 1e30f) {
        const float w = lp_value(static_cast<uint32_t>(lim >> 32));
        thr = w - (2.384185791015625e-7f * (fabsf(w) + s.b_max) + 1e-37f);
      }
      const bool mine = m > -CUDART_INF_F && m >= thr, again = mine && third >= thr && third > -CUDART_INF_F;
      if (mine && !again) {
        const int groups = second > -CUDART_INF_F && second >= thr ? 2 : 1;
#pragma unroll 1
        for (int q = 0; q < groups; ++q) {
          const int t = q ? at_second : at;
          int li = tid >> 1, j = my_edge;
          if (t < rounds) {
            li = group_of(t, tid, &j);
            j += s.rows[li].begin;
          }
          bs_note<T>(s, li, p.V, j, thr);
        }
      }
      if (again && my_edge >= 0) bs_note<T>(s, tid >> 1, p.V, my_edge, thr);
      // (seldom) threads with more than two such groups: all of theirs, dealt out to the warp's lanes
      const unsigned look = __ballot_sync(0xffffffffu, again);
      if (look) {
        if (again) s.looked_at[warp][__popc(look & ((1u << lane) - 1u))] = static_cast<uint8_t>(lane);
        __syncwarp();
        const int who = __popc(look), total = rounds * who;
        for (int i = lane; i < total; i += 32) {
          int j;
          const int li = group_of(i / who, warp * 32 + s.looked_at[warp][i % who], &j);
          if (li < live && j < s.rows[li].count) bs_note<T>(s, li, p.V, s.rows[li].begin + j, thr);
        }
      }
    }
    __syncthreads();
    int mine = s.n_own;
    if (mine <= kBsSpots) {
      if (tid < mine) {
        const uint2 e = s.spots[tid];
        const BsRow& row = s.rows[e.y >> 27];
        const float l = __uint_as_float(e.x);
        s.own[tid] = {bs_order((row.off + static_cast<double>(l)) * row.weight), bs_low(row.beam, l, static_cast<int>(e.y & (kBsMaxV - 1)))};
      }
    } else {
      // More than there is room for (equal or masked entries, or the best crowd together): the part's 32 best by sorted lists, from
      // every entry's key in 64 bits.
      __syncthreads();                                   // (everyone has seen n_own)
      BsCand best = {0, 0};
      int waiting = 0;
      // (a warp's lanes bring a group each, of one row or, edges, of several)
      auto look = [&](const BsRow& row, int j) {
        LpGroup<T> g = LpRow<T>::none();
        const LpRow<T> r(static_cast<const T*>(row.row), p.V);
        if (j >= 0) g = r.get(j);
        const int v0 = r.first(j);
        BsCand worst = {__shfl_sync(0xffffffffu, best.hi, p.n - 1), __shfl_sync(0xffffffffu, best.lo, p.n - 1)};
        const float top = g.largest();
        const bool any = j >= 0 && top > -CUDART_INF_F && bs_order((row.off + static_cast<double>(top)) * row.weight) >= worst.hi;
        if (!__any_sync(0xffffffffu, any)) return;
#pragma unroll 1
        for (int e = 0; e < LpGroup<T>::kEntries; ++e) {
          float l = -CUDART_INF_F;
#pragma unroll
          for (int i = 0; i < LpGroup<T>::kEntries; ++i) l = i == e ? g.entry(i) : l;
          const BsCand c = {bs_order((row.off + static_cast<double>(l)) * row.weight), bs_low(row.beam, l, v0 + e)};
          const bool in = any && l > -CUDART_INF_F && bs_before(c, worst);
          const unsigned mask = __ballot_sync(0xffffffffu, in);
          if (!mask) continue;
          const int fit = __popc(mask);
          if (waiting + fit > 32) {
            best = bs_take_in(best, s.waiting[warp], waiting);
            waiting = 0;
            worst = {__shfl_sync(0xffffffffu, best.hi, p.n - 1), __shfl_sync(0xffffffffu, best.lo, p.n - 1)};
          }
          if (in) s.waiting[warp][waiting + __popc(mask & ((1u << lane) - 1u))] = c;
          waiting += fit;
        }
      };
#pragma unroll 1
      for (int li = 0; li < live; ++li) {
#pragma unroll 1
        for (int j0 = warp * 32; j0 < s.rows[li].count; j0 += kBsThreads)
          look(s.rows[li], j0 + lane < s.rows[li].count ? s.rows[li].begin + j0 + lane : -1);
      }
      if (warp * 32 < 2 * live) look(s.rows[min(tid >> 1, live - 1)], my_edge);
      best = bs_take_in(best, s.waiting[warp], waiting);
      s.own[tid] = best;
      __syncthreads();
      int before = 0;
      for (int i = 0; i < kBsWarps * 32; ++i) before += bs_before(s.own[i], best) ? 1 : 0;
      __syncthreads();
      if (best.hi != 0 && before < 32) s.own[before] = best;       // (candidates differ, so their places do)
      mine = __syncthreads_count(best.hi != 0 && before < 32);
    }

    // Ended beams have one candidate each: the first part's.
    if (part == 0) {
      if (warp == kBsWarps - 1 && (ended_mask >> lane & 1u))
        s.own[mine + __popc(ended_mask & ((1u << lane) - 1u))] = {bs_order(static_cast<double>(score) * weight), bs_low(lane, 0.f, p.end_token)};
      mine += __popc(ended_mask);
    }
    if (tid < mine) s.before_it[tid] = 0;
    __syncthreads();
    // Every candidate's place is the number of those before it: half of the threads look at half of them each.
    constexpr int kHalf = kBsThreads / 2;
    static_assert(kBsSpots + kBsMaxBeams <= kHalf, "a thread for each candidate");
    BsCand c = {0, 0};
    if ((tid & (kHalf - 1)) < mine) {
      c = s.own[tid & (kHalf - 1)];
      const int half = (mine + 1) / 2, from = tid < kHalf ? 0 : half, to = tid < kHalf ? half : mine;
      int before = 0;
#pragma unroll 8
      for (int k = from; k < to; ++k) before += bs_before(s.own[k], c) ? 1 : 0;
      atomicAdd(&s.before_it[tid & (kHalf - 1)], before);
    }
    __syncthreads();
    // To the sequence's first CTA: the best; to every CTA: the rows found bad.
    if (C > 1) asm volatile("barrier.cluster.wait;" ::: "memory");
    if (tid < mine) {
      const int place = s.before_it[tid];
      if (place < p.n) (C > 1 ? cg::this_cluster().map_shared_rank(&s.sent[part][0], 0) : &s.sent[part][0])[place] = c;
    }
    if (tid == kBsThreads - 1) *(C > 1 ? cg::this_cluster().map_shared_rank(&s.sent_by[part], 0) : &s.sent_by[part]) = min(mine, p.n);
    if (warp == 3 && lane < C) *(C > 1 ? cg::this_cluster().map_shared_rank(&s.bad_from[part], lane) : &s.bad_from[part]) = s.bad_here;
    if (C > 1) cluster_sync_all();
    else __syncthreads();
    const unsigned found = __reduce_or_sync(0xffffffffu, lane < C ? s.bad_from[lane] : 0u) & ~excluded;
    if (!found) break;
    // Seldom: the limits may stem from rows that have no distribution.  Once more without them.
    excluded |= found;
    flags |= HOLA_FLAG_BAD_LOGIT;
    __syncthreads();
    if (tid == 0) s.n_own = 0;
    if (C > 1) {
      cluster_sync_all();
      asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    } else {
      __syncthreads();
    }
  }
  if (part != 0) return;

  // The parts' lists, merged: warp w takes those of parts w and w + 8, then the other warps'.  Lane i: the i-th kept.
  BsCand c = {0, 0};
  if (warp < C && lane < s.sent_by[warp]) c = s.sent[warp][lane];
  if (warp + kBsWarps < C) {
    BsCand r = {0, 0};
    if (31 - lane < s.sent_by[warp + kBsWarps]) r = s.sent[warp + kBsWarps][31 - lane];
    c = bs_merge(c, r, lane);
  }
#pragma unroll 1
  for (int step = 1; step < min(C, kBsWarps); step <<= 1) {
    if ((warp & (2 * step - 1)) == step) s.waiting[warp][lane] = c;
    __syncthreads();
    if ((warp & (2 * step - 1)) == 0 && warp + step < C) c = bs_merge(c, s.waiting[warp + step][31 - lane], lane);
  }
  if (warp != 0) return;

  const bool have = lane < p.n && c.hi != 0;
  const int beam = have ? bs_beam(c.lo) : 0;
  const float from_score = __shfl_sync(0xffffffffu, score, beam), from_logZ = __shfl_sync(0xffffffffu, logZ, beam);
  const bool was_ended = have && (ended_mask >> beam & 1u);
  const float out_score = !have ? -CUDART_INF_F
                          : was_ended ? from_score
                          : static_cast<float>((static_cast<double>(from_score) - static_cast<double>(from_logZ)) + static_cast<double>(bs_logit(c.lo)));
  const int token = have ? bs_id(c.lo) : -1;
  int slot = lane;
  if (p.keep_slots) {
    // the first child of a beam goes to its slot, the others take the free ones in order
    const unsigned same = __match_any_sync(0xffffffffu, have ? beam : -1 - lane);
    const bool stays = have && __ffs(same) - 1 == lane;
    unsigned free = ~__reduce_or_sync(0xffffffffu, stays ? 1u << beam : 0u);
    const unsigned waits = __ballot_sync(0xffffffffu, lane < p.n && !stays);
    if (stays) {
      slot = beam;
    } else {
      for (int i = __popc(waits & ((1u << lane) - 1u)); i > 0; --i) free &= free - 1u;
      slot = __ffs(free) - 1;
    }
  }
  if (lane < p.n) {
    const size_t at = static_cast<size_t>(seq) * p.n + slot;
    p.score_out[at] = out_score;
    p.parent[at] = have ? beam : -1;
    p.token[at] = token;
    if (p.finished_out) p.finished_out[at] = have && (was_ended || (p.end_token >= 0 && token == p.end_token)) ? 1 : 0;
  }
  if (p.status && lane == 0 && flags) atomicOr(p.status, flags);
}

// CTAs per sequence: as many as leave all clusters of the call room on the chip at once (`fit`: clusters of so many CTAs that it holds; up to
// fifteen sixteenths of them, for the last ones share SMs), and a thread three groups or more.  us with 1 / 2 / 4 / 8 / 16: 1 x 4 x 32000
// fp32 12.5 / 9.4 / 7.8 / 7.1 / 6.8; 23 x 3 x 50003 fp16 14.0 / 10.9 / 10.4 / 10.2 / 16.8 (two waves); 64 x 6 x 32000 fp32 27.7 / 19.1 /
// 15.7 / 26.3 / 41.2; 32 x 5 x 128256 bf16 41.3 / 25.3 / 18.4 / 18.1 (with 7: 16.1); 4 x 2 x 5000 fp32 5.0 / 5.3 / 5.4 / 6.1 / 11.2.
int bs_cluster(int B, int W, int V, int elem, const int* fit) {
  const long long groups = static_cast<long long>(W) * V / (kLpGroupBytes / elem);
  for (int C = kBsMaxCluster; C > 1; C = C > 8 ? 8 : C - 1)
    if (16ll * B <= 15ll * fit[C] && groups / C >= 3 * kBsThreads) return C;
  return 1;
}

template <typename T>
cudaError_t launch_beam_select(const BsParams& p, const int* fit, cudaStream_t stream) {
  const int C = bs_cluster(p.B, p.W, p.V, static_cast<int>(sizeof(T)), fit);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.B) * C); cfg.blockDim = dim3(kBsThreads); cfg.stream = stream;
  cfg.dynamicSmemBytes = sizeof(BsShared);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(C); attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = C > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, beam_select_kernel<T>, p, C);
}

template <typename T>
cudaError_t configure_select() {
  const cudaError_t e = cudaFuncSetAttribute(beam_select_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(sizeof(BsShared)));
  return e != cudaSuccess ? e : cudaFuncSetAttribute(beam_select_kernel<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
}
// Also: how many clusters of 1 .. kBsMaxCluster CTAs the device holds at once (the types' kernels are alike in what they need).
cudaError_t configure_beams(int* fit) {
  cudaError_t e = configure_select<float>();
  if (e == cudaSuccess) e = configure_select<__nv_bfloat16>();
  if (e == cudaSuccess) e = configure_select<__half>();
  for (int C = 1; e == cudaSuccess && C <= kBsMaxCluster; ++C) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(C)); cfg.blockDim = dim3(kBsThreads); cfg.dynamicSmemBytes = sizeof(BsShared);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(C); attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    fit[C] = 0;
    // (a size that the device does not hold at all is none that is taken)
    if (cudaOccupancyMaxActiveClusters(&fit[C], beam_select_kernel<float>, &cfg) != cudaSuccess) { fit[C] = 0; cudaGetLastError(); }
  }
  return e;
}

// ------------------------------------------------------------------------------------------------ reordering
// new[b][i] = old[b][parent[b][i]], any number of states.  A CTA takes a piece of the bytes of all beams of one sequence (of one layer,
// one head).  Where no place that changes has children of its own (copies into another buffer; a selection that keeps slots), every
// parent's words are read once and written to all of its children.  Else, in place, a thread takes its words of every beam that changes
// into registers and then writes them, so that any order of the parents will do: no other thread touches these bytes.  In place, beams
// that stay (parent[i] = i) are neither read, but for their children, nor written.  Bound by HBM, whose latency eight words of 16 bytes a
// thread on the way hide.
constexpr int kBrThreads = 128;
constexpr int kBrStates = 24;          // states of one launch (launch parameters)

struct BrState {
  const unsigned char* src;
  unsigned char* dst;
  long long seq, beam, outer0, outer1; // strides in bytes
  long long to_seq, to_beam, to_outer0, to_outer1;
  long long run, position;             // bytes that lie side by side; bytes of a position (0: all of the run is moved)
  unsigned n0, n1;                     // outer axes
  unsigned pieces;                     // of a run
  unsigned piece;                      // bytes of one: 8 words a thread, of 16 bytes, 4, 2 or 1, as the state's addresses allow
  unsigned first_cta;
};
struct BrParams {
  BrState s[kBrStates];
  int count, B, W, n, in_place;
  int split;                           // CTAs that share the parents of a piece
  long long parent_stride;
  const int* parent;
  const int* used;
  unsigned* status;
};
constexpr int kBrWords = 8;            // words of a piece that a thread takes

// Every parent's words to its children: `sources` parents, children[k] as bits.
template <typename V>
__device__ __forceinline__ void br_spread(const BrState& st, const unsigned char* src, unsigned char* dst, long long begin, long long end,
                                          const int* from, const unsigned* children, int first, int sources, int split) {
  constexpr int U = kBrWords;
  constexpr int kStep = kBrThreads * sizeof(V);
#pragma unroll 1
  for (long long at = begin + static_cast<long long>(threadIdx.x) * sizeof(V); at < end; at += U * kStep) {
    const int left = static_cast<int>(end - at);
#pragma unroll 1
    for (int k = first; k < sources; k += split) {
      V v[U];
      const unsigned char* x = src + from[k] * st.beam + at;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u * kStep < left) v[u] = *reinterpret_cast<const V*>(x + u * kStep);
#pragma unroll 1
      for (unsigned c = children[k]; c; c &= c - 1u) {
        unsigned char* y = dst + (__ffs(c) - 1) * st.to_beam + at;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u * kStep < left) *reinterpret_cast<V*>(y + u * kStep) = v[u];
      }
    }
  }
}

// In any order: M beams that change at most; U words of each that a thread has on the way.
template <typename V, int M, int U>
__device__ __forceinline__ void br_move(const BrState& st, const unsigned char* src, unsigned char* dst, long long begin, long long end,
                                        const int* to, const int* from, int moves) {
  constexpr int kStep = kBrThreads * sizeof(V);
#pragma unroll 1
  for (long long at = begin + static_cast<long long>(threadIdx.x) * sizeof(V); at < end; at += U * kStep) {
    const int left = static_cast<int>(end - at);
    V v[U][M];
#pragma unroll
    for (int i = 0; i < M; ++i)
      if (i < moves) {
        const unsigned char* x = src + from[i] * st.beam + at;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u * kStep < left) v[u][i] = *reinterpret_cast<const V*>(x + u * kStep);
      }
#pragma unroll
    for (int i = 0; i < M; ++i)
      if (i < moves) {
        unsigned char* x = dst + to[i] * st.to_beam + at;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u * kStep < left) *reinterpret_cast<V*>(x + u * kStep) = v[u][i];
      }
  }
}
template <typename V>
__device__ __forceinline__ void br_move_any(const BrState& st, const unsigned char* src, unsigned char* dst, long long begin, long long end,
                                            const int* to, const int* from, int moves) {
  if (moves <= 4) br_move<V, 4, 4>(st, src, dst, begin, end, to, from, moves);
  else if (moves <= 8) br_move<V, 8, 2>(st, src, dst, begin, end, to, from, moves);
  else if (moves <= 16) br_move<V, 16, 1>(st, src, dst, begin, end, to, from, moves);
  else br_move<std::conditional_t<sizeof(V) == 16, uint2, V>, 32, 1>(st, src, dst, begin, end, to, from, moves);       // (64 registers)
}

__global__ void __launch_bounds__(kBrThreads, 5) beam_reorder_kernel(const __grid_constant__ BrParams p) {
  __shared__ int to[32], from[32];
  __shared__ unsigned children[32];
  __shared__ int n_moves, n_sources;                     // n_sources 0: in any order
  grid_dependency_wait();
  grid_dependency_release();
  int k = 0;
  const unsigned cta = blockIdx.x / static_cast<unsigned>(p.split);
  const int share = static_cast<int>(blockIdx.x - cta * static_cast<unsigned>(p.split));
  while (k + 1 < p.count && cta >= p.s[k + 1].first_cta) ++k;
  const BrState& st = p.s[k];
  unsigned x = cta - st.first_cta;
  const unsigned piece = x % st.pieces; x /= st.pieces;
  const unsigned b = x % static_cast<unsigned>(p.B); x /= static_cast<unsigned>(p.B);
  const unsigned i1 = x % st.n1, i0 = x / st.n1;
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    int from_beam = -1;
    bool bad = false;
    if (lane < p.n) {
      from_beam = p.parent[static_cast<long long>(b) * p.parent_stride + lane];
      bad = from_beam < -1 || from_beam >= p.W;
    }
    const bool moves = !bad && from_beam >= 0 && !(p.in_place && from_beam == lane);
    const unsigned mask = __ballot_sync(0xffffffffu, moves), below = (1u << lane) - 1u;
    const unsigned parents = __reduce_or_sync(0xffffffffu, moves ? 1u << from_beam : 0u);
    const unsigned same = __match_any_sync(0xffffffffu, moves ? from_beam : -1);
    const bool any_order = p.in_place && (mask & parents) != 0;
    if (any_order) {
      if (moves) {
        to[__popc(mask & below)] = lane;
        from[__popc(mask & below)] = from_beam;
      }
    } else if (moves && __ffs(same) - 1 == lane) {
      const int at = __popc(parents & ((1u << from_beam) - 1u));
      from[at] = from_beam;
      children[at] = same;
    }
    if (lane == 0) { n_moves = __popc(mask); n_sources = any_order ? 0 : __popc(parents); }
    if (__any_sync(0xffffffffu, bad) && lane == 0 && p.status) atomicOr(p.status, HOLA_FLAG_BAD_BEAM);
  }
  __syncthreads();
  const int moves = n_moves;
  long long run = st.run;
  if (p.used && st.position > 0) {
    const long long filled = static_cast<long long>(max(p.used[b], 0)) * st.position;
    run = filled < run ? filled : run;
  }
  const long long begin = static_cast<long long>(piece) * st.piece, end = begin + st.piece < run ? begin + st.piece : run;
  if (moves == 0 || begin >= end) return;
  const unsigned char* src = st.src + (b * st.seq + i0 * st.outer0 + i1 * st.outer1);
  unsigned char* dst = st.dst + (b * st.to_seq + i0 * st.to_outer0 + i1 * st.to_outer1);
  // whole words, and what is left of the last one byte by byte (a last position may end anywhere)
  const int word = static_cast<int>(st.piece / (kBrWords * kBrThreads));
  const long long words_end = end - (end - begin) % word;
  const int sources = n_sources;
  if (sources) {
    if (word == 16) br_spread<uint4>(st, src, dst, begin, words_end, from, children, share, sources, p.split);
    else if (word == 4) br_spread<uint32_t>(st, src, dst, begin, words_end, from, children, share, sources, p.split);
    else if (word == 2) br_spread<uint16_t>(st, src, dst, begin, words_end, from, children, share, sources, p.split);
    else br_spread<unsigned char>(st, src, dst, begin, words_end, from, children, share, sources, p.split);
    br_spread<unsigned char>(st, src, dst, words_end, end, from, children, share, sources, p.split);
  } else if (share == 0) {
    if (word == 16) br_move_any<uint4>(st, src, dst, begin, words_end, to, from, moves);
    else if (word == 4) br_move_any<uint32_t>(st, src, dst, begin, words_end, to, from, moves);
    else if (word == 2) br_move_any<uint16_t>(st, src, dst, begin, words_end, to, from, moves);
    else br_move_any<unsigned char>(st, src, dst, begin, words_end, to, from, moves);
    br_move_any<unsigned char>(st, src, dst, words_end, end, to, from, moves);
  }
}

// Bytes of a piece of a state: by the widest word that all its addresses are multiples of.
unsigned br_piece(const hola_beam_state& s) {
  uintptr_t all = reinterpret_cast<uintptr_t>(s.src) | reinterpret_cast<uintptr_t>(s.dst) | static_cast<uintptr_t>(s.seq_stride | s.beam_stride | s.dst_seq_stride |
                                                                                                                 s.dst_beam_stride);
  for (int i = 0; i < 2; ++i)
    if (s.outer[i] > 1) all |= static_cast<uintptr_t>(s.outer_stride[i] | s.dst_outer_stride[i]);
  return kBrWords * kBrThreads * (all % 16 == 0 ? 16u : all % 4 == 0 ? 4u : all % 2 == 0 ? 2u : 1u);
}

cudaError_t launch_beam_reorder(const BrParams& p, unsigned ctas, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas); cfg.blockDim = dim3(kBrThreads); cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, beam_reorder_kernel, p);
}
