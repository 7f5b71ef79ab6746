// adapters.cuh - low-rank adapters of many requests beside the LM head.  Part of hola_verify.cu (inside its anonymous namespace).
//
// Sequence b uses adapter a = ids[b] (or none): its k + 1 verify rows x[r] get the logits of the head W + s_a B_a A_a,
//   l[r,v] = sum_h W[v,h] x[r,h] + sum_i B_a[v,i] u[r,i],   u[r,i] = s_a sum_h A_a[i,h] x[r,h],   i < rank.
//
//   adapter_down_kernel  u, ahead of the GEMM: one CTA per sequence, 16 ranks and 16 rows, whose warps share the hidden channels; and
//       one CTA that sorts the batch's rows by adapter into tiles of eight.
//   adapter_up_kernel    behind the GEMM, whatever its weight mode: adds the second product to the stored logits and makes the
//       rows' softmax statistics anew, in the form in which the GEMM's epilogue leaves them (partials of each row), so that
//       everything behind reads them as before.  Rows without an adapter are left alone.
// Both products run on bf16 operands with fp32 accumulation; u, which is fp32, enters the second one as three bf16 planes that
// add up to it exactly (8 significant bits each), so that no rounding is added to what an fp32 product would have.  That holds for
// finite factors; where one is not (an entry of B masks with -inf, say), a zero in one plane or planes of opposite signs make NaN of a
// product that is infinite: entries that come out as NaN are taken again as fp32 products.
//
// (Why not inside the GEMM, as further K blocks [B_0 B_1 ...] against rows that are zero but for their own slot's columns: a number
// that is not finite in one slot would reach the rows of every other request as 0 * inf, and each block costs all rows' MMAs.)

constexpr int kAdMaxRank = 128;
constexpr int kAdDownWarps = 16;
constexpr int kAdUpWarps = 4;
constexpr int kAdRows = 8;             // verify rows of a tile: the N of the MMA
constexpr int kAdChunk = 64;           // vocabulary entries per warp step
constexpr int kAdMaxSorted = 2048;     // sequences up to which rows of different sequences share tiles

// Up to eight verify rows that use one adapter.
struct AdapterTile {
  int adapter, n, row[kAdRows];
};

struct AdapterParams {
  const uint16_t* A;           // bf16 [slots][rank][H]
  const uint16_t* Bm;          // bf16 [slots][V][rank]
  const float* scale;          // [slots], or null: 1
  const int* ids;              // [B]
  int slots, rank;
  int B, rows_per_seq, H, V;
  const uint16_t* hidden;      // [B][rows_per_seq][H]
  float* u;                    // [rows][kAdMaxRank]
  AdapterTile* tiles;          // [max_tiles]
  int* n_tiles;                // how many the batch needs
  int max_tiles;
  float* logits;
  int ldl;
  float4* partials;
  int part_stride, nparts;
  int want_arg;
  unsigned* status;
  int clear_status;
};

__device__ __forceinline__ void mma_bf16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Which adapter a sequence uses; -1: none (also where the index is out of range, which the first CTA reports).
__device__ __forceinline__ int adapter_of(const AdapterParams& p, int b) {
  const int a = p.ids[b];
  return a >= 0 && a < p.slots ? a : -1;
}

// The batch's rows by adapter, in tiles of eight, by one CTA.  Sequences with the same adapter keep their order; a sequence finds its
// place by looking at all others: B^2 comparisons, which up to some 100 sequences are hidden behind the loads of the other CTAs and
// beyond are what the kernel takes (us, H = 1024, two rows each: 64 sequences 5.3, 256 16, 512 42, 1024 140, 2048 516).  Beyond
// kAdMaxSorted sequences every one has tiles of its own (2049: 48).
__device__ __forceinline__ void adapter_tiles(const AdapterParams& p) {
  __shared__ int ids[kAdMaxSorted], users[kAdMaxSorted];
  const int tid = threadIdx.x, nthr = blockDim.x, k1 = p.rows_per_seq, B = p.B;
  const int per_seq = (k1 + kAdRows - 1) / kAdRows;
  if (B > kAdMaxSorted) {
    for (int i = tid; i < B * per_seq; i += nthr) {
      const int b = i / per_seq, j0 = (i - b * per_seq) * kAdRows, a = adapter_of(p, b);
      AdapterTile& t = p.tiles[i];
      t.adapter = a;
      t.n = a < 0 ? 0 : min(kAdRows, k1 - j0);
      for (int j = 0; j < kAdRows; ++j) t.row[j] = b * k1 + j0 + j;
    }
    if (tid == 0) *p.n_tiles = B * per_seq;
    return;
  }
  if (tid == 0) *p.n_tiles = 0;
  for (int b = tid; b < B; b += nthr) ids[b] = adapter_of(p, b);
  __syncthreads();
  for (int b = tid; b < B; b += nthr) {                  // how many use the adapter, at its first user; 0 at the others
    int n = 0, before = 0;
    for (int c = 0; c < B; ++c) {
      const bool same = ids[c] == ids[b];
      n += same ? 1 : 0;
      before += same && c < b ? 1 : 0;
    }
    users[b] = ids[b] < 0 || before > 0 ? 0 : n;
  }
  __syncthreads();
  for (int b = tid; b < B; b += nthr) {
    if (ids[b] < 0) continue;
    int first = 0, before = 0, all = 0;
    for (int c = 0; c < B; ++c) {
      if (ids[c] < ids[b]) first += (users[c] * k1 + kAdRows - 1) / kAdRows;
      if (ids[c] == ids[b]) {
        all += users[c];
        before += c < b ? 1 : 0;
      }
    }
    for (int j = 0; j < k1; ++j) {
      const int i = before * k1 + j;
      AdapterTile& t = p.tiles[first + i / kAdRows];
      t.row[i % kAdRows] = b * k1 + j;
      if (i % kAdRows == 0) {
        t.adapter = ids[b];
        t.n = min(kAdRows, all * k1 - i);
        if (t.n == all * k1 - i) atomicMax(p.n_tiles, first + i / kAdRows + 1);        // (the adapter's last one)
      }
    }
  }
}

// The order of the channels inside a sum is free, so lane (g, q) of a warp loads 16 bytes = 8 neighbouring channels of its row and
// hands them to two MMAs: channels 8q .. 8q+3 in the places the first one gives lane q, 8q+4 .. 8q+7 in those of the second.
__global__ void __launch_bounds__(kAdDownWarps * 32, 1) adapter_down_kernel(const AdapterParams p) {
  __shared__ float sums[kAdDownWarps][16][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int b = blockIdx.x, i0 = blockIdx.y * 16, j0 = blockIdx.z * 16;
  grid_dependency_wait();
  grid_dependency_release();
  if (b == p.B) {
    if (blockIdx.y != 0 || blockIdx.z != 0) return;
    if (warp == 0 && p.status) {
      bool bad = false;
      for (int i = lane; i < p.B; i += 32) bad = bad || p.ids[i] < -1 || p.ids[i] >= p.slots;
      const unsigned flags = __any_sync(0xffffffffu, bad) ? HOLA_FLAG_BAD_ADAPTER : 0u;
      if (lane == 0) {
        if (p.clear_status) *p.status = flags;
        else if (flags) atomicOr(p.status, flags);
      }
    }
    adapter_tiles(p);
    return;
  }
  const int a = adapter_of(p, b);
  if (a < 0) return;
  const int rows = min(16, p.rows_per_seq - j0), ranks = min(16, p.rank - i0);
  const float scale = p.scale ? p.scale[a] : 1.f;
  const uint16_t* x = p.hidden + (static_cast<size_t>(b) * p.rows_per_seq + j0) * p.H;
  const uint16_t* A = p.A + (static_cast<size_t>(a) * p.rank + i0) * p.H;
  float d[2][4] = {};
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 4
  for (int h0 = warp * 32; h0 < p.H; h0 += kAdDownWarps * 32) {
    const int h = h0 + 8 * q;                            // (H is a multiple of 8)
    const bool in = h < p.H;
    const uint4 x0 = in && g < rows ? *reinterpret_cast<const uint4*>(x + static_cast<size_t>(g) * p.H + h) : zero;
    const uint4 x1 = in && g + 8 < rows ? *reinterpret_cast<const uint4*>(x + static_cast<size_t>(g + 8) * p.H + h) : zero;
    const uint4 a0 = in && g < ranks ? *reinterpret_cast<const uint4*>(A + static_cast<size_t>(g) * p.H + h) : zero;
    const uint4 a1 = in && g + 8 < ranks ? *reinterpret_cast<const uint4*>(A + static_cast<size_t>(g + 8) * p.H + h) : zero;
    const uint32_t f0[4] = {x0.x, x1.x, x0.y, x1.y}, f1[4] = {x0.z, x1.z, x0.w, x1.w};
    mma_bf16(d[0], f0, a0.x, a0.y);
    mma_bf16(d[1], f0, a1.x, a1.y);
    mma_bf16(d[0], f1, a0.z, a0.w);
    mma_bf16(d[1], f1, a1.z, a1.w);
  }
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[warp][g + 8 * (e >> 1)][8 * n + 2 * q + (e & 1)] = d[n][e];
  __syncthreads();
  const int j = threadIdx.x >> 4, i = threadIdx.x & 15;
  if (threadIdx.x < 256 && j < rows) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kAdDownWarps; ++w) s += sums[w][j][i];
    p.u[(static_cast<size_t>(b) * p.rows_per_seq + j0 + j) * kAdMaxRank + i0 + i] = s * scale;
  }
}

// Running statistics of a row about a point that trails the maximum by 4 at most, so that a rise of the maximum rarely makes a
// warp rescale.  In units of ln 2: x = (l - ref) log2 e, s = sum 2^x, t = sum 2^x x.  (Differences first: one addition more a pair
// than l log2 e + shift, whose shift would be off by 2^-24 of itself, which large logits turn into sums of zero or infinity.)
struct RowStats {
  float m, ref;                // (a row's first step: -inf and 0)
  uint64_t s2, t2;             // two halves of either sum
  int arg;
  __device__ __forceinline__ void clear() {
    m = -CUDART_INF_F;
    ref = 0.f;
    s2 = t2 = 0;
    arg = 0x7fffffff;
  }
  __device__ __forceinline__ float rise() const { return m == -CUDART_INF_F ? m : ref + 4.f; }
  // Eight logits and their largest; entry i is vocabulary entry v(i), rising with i.  First what is seldom (the maximum rises by
  // more than 4, the arg-max is wanted), then the sums.  kSome: logits that are -inf are none.
  template <typename Entry>
  __device__ __forceinline__ void rises(const float* l, float top, int want_arg, Entry v) {
    if (want_arg && top > m) {
      int first = 0;
#pragma unroll
      for (int i = 7; i > 0; --i)
        if (l[i] == top) first = v(i);
      arg = l[0] == top ? v(0) : first;
    }
    if (top > rise()) {
      if (m != -CUDART_INF_F) {
        const float dx = fmaxf((ref - top) * kLog2e, -1e30f), e = ex2_approx(dx);            // (finite: e is 0 there)
        const uint64_t e2 = pack2(e, e);
        t2 = mul2(fma2(pack2(dx, dx), s2, t2), e2);
        s2 = mul2(s2, e2);
      }
      ref = top;
    }
  }
  template <bool kSome>
  __device__ __forceinline__ void add(const float* l, float top) {
    m = fmaxf(m, top);
    const uint64_t l2e = pack2(kLog2e, kLog2e), from = pack2(-ref, -ref);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint64_t x = mul2(add2(pack2(l[2 * i], l[2 * i + 1]), from), l2e);
      float a, b;
      unpack2(x, a, b);
      const uint64_t e = pack2(ex2_approx(a), ex2_approx(b));
      if (kSome) x = pack2(fmaxf(a, -1e30f), fmaxf(b, -1e30f));       // (0 * -inf)
      s2 = add2(s2, e);
      t2 = fma2(e, x, t2);
    }
  }
  // Entries of -inf, which the sums are not kept clear of in whole steps, have made NaN (0 * -inf) of t.
  __device__ __forceinline__ bool lost() const {
    float a, b, c, d;
    unpack2(s2, a, b);
    unpack2(t2, c, d);
    return a + b > 0.f && a + b < CUDART_INF_F && c + d != c + d;
  }
  __device__ __forceinline__ Stats stats() const {
    float a, b, c, d;
    unpack2(s2, a, b);
    unpack2(t2, c, d);
    const float s = a + b;
    if (s == 0.f) return stats_empty();
    if (!(s < CUDART_INF_F)) return Stats{CUDART_NAN_F, CUDART_NAN_F, CUDART_NAN_F, arg};       // (no distribution)
    const float x = (m - ref) * kLog2e, e = ex2_approx(-x);                   // (x of the maximum, as it was summed)
    return Stats{m, s * e, kLn2 * (e * fmaf(-x, s, c + d)), arg};
  }
};

// One entry of the second product, rank by rank; b: the entry's row of B.
__device__ __noinline__ float adapter_product(const uint16_t* b, const float* u, int rank) {
  float s = 0.f;
#pragma unroll 1
  for (int i = 0; i < rank && s == s; ++i) s = fmaf(__uint_as_float(static_cast<uint32_t>(b[i]) << 16), u[i], s);
  return s;
}

// A warp step covers 64 vocabulary entries, the M of four MMAs, and the tile's eight rows, their N.  Lane (g, q) holds entries g, 8 + g,
// 16 + g ... of rows 2 q and 2 q + 1.  Rows of the logits that start on 16-byte boundaries (kVec) are loaded and stored 16 bytes a lane,
// a step ahead, and change hands in shared memory; others lane by lane, eight of which share a sector.  Every lane sums the same
// entries in the same order either way.  (Bulk copies in place of the loads and stores, three buffers of 256-byte rows a warp, took
// as long: a copy keeps its lane some 100 cycles, and memory bounds both.)
//
// As in the first product, the order of the ranks is free.  Sixteen at a time, lane q loads four (8 bytes) of a row of B; where whole
// blocks of 32 ranks are known beforehand (kR: the rank, or 0), eight (16 bytes) for two MMA steps.
template <int kR>
__device__ __forceinline__ int adapter_rank(int k, int q) {      // first of the four ranks that lane q holds in step k
  return kR % 32 == 0 && kR > 0 ? 32 * (k >> 1) + 8 * q + 4 * (k & 1) : 16 * k + 4 * q;
}
constexpr int kAdPitch = kAdChunk + 4;                           // (floats from row to row: no two rows of a step on the same banks)

// What bounds it: at V = 128256 memory, short of its limit.  64 adapters of rank 16, 384 rows: 262 MB of B and the logits in and out,
// 197 MB each, 132 us from the first CTA's start to the last one's end, 5.0 TB/s; 16 adapters of rank 32 for 28 rows 35 us, 4.6 TB/s.
// At V = 32000 the latency of a warp's step, load -> shared memory -> MMA -> sums -> shared memory -> store with one step asked for ahead:
// 48 tiles of 16 adapters 26 us, 18 of them the steps (87 MB at 4.9 TB/s out of the L2, with 24 % of the warps, 34 % of the issue slots
// and 21 % of DRAM's rate in use under a profiler), the rest start and end.  Without the stores 5 us less of 26, without the sums 1,
// without two of the three planes 1.
constexpr int kAdUpCtas = 4;                                     // per SM, by registers
template <bool kVec, int kR>
__global__ void __launch_bounds__(kAdUpWarps * 32, kAdUpCtas) adapter_up_kernel(const AdapterParams p) {
  constexpr int kSteps = (kR + 15) / 16;                 // 0: not known beforehand
  constexpr bool kAhead = kR == 8 || kR == 16;           // a step's ranks are asked for while the step before is worked on
  __shared__ uint2 planes[3][kR ? kSteps : kAdMaxRank / 16][kAdRows][4];         // [plane][16 ranks][row][q]
  __shared__ float4 warp_stats[kAdUpWarps][kAdRows];
  __shared__ __align__(16) float buffer[kVec ? kAdUpWarps : 1][kVec ? kAdRows : 1][kAdPitch];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int rank = kR ? kR : p.rank, steps = kR ? kSteps : (rank + 15) >> 4;
  grid_dependency_wait();
  // The CTAs are dealt out to the tiles that there are: P parts of the vocabulary each, in one go as far as there are enough CTAs.
  const int n_tiles = *p.n_tiles, chunks = (p.V + kAdChunk - 1) / kAdChunk;
  if (n_tiles == 0) return;
  const int P = max(1, min(min(static_cast<int>(gridDim.x) / n_tiles, p.nparts), (chunks + kAdUpWarps - 1) / kAdUpWarps));
  const int per = (chunks + P - 1) / P;
  for (int item = blockIdx.x; item < n_tiles * P; item += gridDim.x) {
    const int part = item / n_tiles;
    const AdapterTile& tile = p.tiles[item - part * n_tiles];
    const int n = tile.n;
    if (n == 0) continue;
    const int c_begin = part * per + warp, c_end = min(chunks, (part + 1) * per);

    // This lane's two rows of the logits (one that the tile lacks: its first one, read and not written), from entry 4 g or g on, and B from
    // entry g and its first rank on.
    const bool have[2] = {2 * q < n, 2 * q + 1 < n};
    float* at[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) at[h] = p.logits + static_cast<size_t>(tile.row[have[h] ? 2 * q + h : 0]) * p.ldl + (kVec ? 4 * g : g);
    const uint16_t* Bm = p.Bm + static_cast<size_t>(tile.adapter) * p.V * rank;
    float4 near[2][2];                                   // (kVec) logits of the next step
    auto fetch = [&](int c) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        near[h][0] = *reinterpret_cast<const float4*>(at[h] + c * kAdChunk);
        near[h][1] = *reinterpret_cast<const float4*>(at[h] + c * kAdChunk + 32);
      }
    };
    const int c_whole = min(c_end, p.V / kAdChunk);      // steps before it are whole
    if (kVec && c_begin < c_whole) fetch(c_begin);
    auto row = [&](int c, int e) {                       // (a ragged step: entries past the vocabulary read its last row)
      const int v = c * kAdChunk + 8 * e + g;
      return Bm + static_cast<size_t>(c < c_whole ? v : min(v, p.V - 1)) * rank;
    };
    uint2 ahead[8];
    auto ask = [&](int c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ahead[e] = make_uint2(0u, 0u);
        if (kR == 16 || 4 * q < kR) ahead[e] = *reinterpret_cast<const uint2*>(row(c, e) + 4 * q);
      }
    };
    if (kAhead && c_begin < c_end) ask(c_begin);

    for (int i = threadIdx.x; i < steps * kAdRows * 4; i += kAdUpWarps * 32) {
      const int k = i >> 5, r = (i >> 2) & 7, qq = i & 3;
      uint32_t w[3][2] = {};
      if (r < n) {
        const float4 u4 = *reinterpret_cast<const float4*>(p.u + static_cast<size_t>(tile.row[r]) * kAdMaxRank + adapter_rank<kR>(k, qq));
        float u[4] = {u4.x, u4.y, u4.z, u4.w};
#pragma unroll
        for (int pl = 0; pl < 3; ++pl)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const __nv_bfloat16 h = __float2bfloat16_rn(u[e]);
            u[e] -= __bfloat162float(h);                 // (exact)
            w[pl][e >> 1] |= static_cast<uint32_t>(__bfloat16_as_ushort(h)) << (16 * (e & 1));
          }
      }
#pragma unroll
      for (int pl = 0; pl < 3; ++pl) planes[pl][k][r][qq] = make_uint2(w[pl][0], w[pl][1]);
    }
    __syncthreads();
    RowStats st[2];
    st[0].clear(); st[1].clear();
    for (int c = c_begin; c < c_end; c += kAdUpWarps) {
      const int v0 = c * kAdChunk, vg = v0 + g;
      const bool whole = c < c_whole;
      float l[2][8];
      if (kVec && whole) {
        __syncwarp();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          *reinterpret_cast<float4*>(&buffer[warp][2 * q + h][4 * g]) = near[h][0];
          *reinterpret_cast<float4*>(&buffer[warp][2 * q + h][32 + 4 * g]) = near[h][1];
        }
        __syncwarp();
        if (c + kAdUpWarps < c_whole) fetch(c + kAdUpWarps);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 8; ++e) l[h][e] = buffer[warp][2 * q + h][8 * e + g];
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 8; ++e) l[h][e] = whole || vg + 8 * e < p.V ? at[h][v0 + 8 * e - (kVec ? 3 * g : 0)] : -CUDART_INF_F;
      }
      float d[4][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) d[t][0] = d[t][1] = d[t][2] = d[t][3] = 0.f;
      if (kAhead) {
        uint2 w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = ahead[e];
        if (c + kAdUpWarps < c_end) ask(c + kAdUpWarps);
#pragma unroll
        for (int pl = 2; pl >= 0; --pl) {
          const uint2 u = planes[pl][0][g][q];
#pragma unroll
          for (int t = 0; t < 4; ++t) {                  // entries 16 t + g at m = g, 16 t + 8 + g at m = g + 8
            const uint32_t f[4] = {w[2 * t].x, w[2 * t + 1].x, w[2 * t].y, w[2 * t + 1].y};
            mma_bf16(d[t], f, u.x, u.y);
          }
        }
      } else if (kR % 32 == 0 && kR > 0) {
#pragma unroll 1
        for (int k = 0; k < kSteps; k += 2) {
          uint4 w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = *reinterpret_cast<const uint4*>(row(c, e) + 16 * k + 8 * q);
#pragma unroll
          for (int pl = 2; pl >= 0; --pl) {
            const uint2 u0 = planes[pl][k][g][q], u1 = planes[pl][k + 1][g][q];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const uint32_t f0[4] = {w[2 * t].x, w[2 * t + 1].x, w[2 * t].y, w[2 * t + 1].y},
                             f1[4] = {w[2 * t].z, w[2 * t + 1].z, w[2 * t].w, w[2 * t + 1].w};
              mma_bf16(d[t], f0, u0.x, u0.y);
              mma_bf16(d[t], f1, u1.x, u1.y);
            }
          }
        }
      } else {
#pragma unroll 1
        for (int k = 0; k < steps; ++k) {
          const bool in = 16 * k + 4 * q < rank;
          uint2 w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            w[e] = make_uint2(0u, 0u);
            if (in) w[e] = *reinterpret_cast<const uint2*>(row(c, e) + 16 * k + 4 * q);
          }
#pragma unroll
          for (int pl = 2; pl >= 0; --pl) {
            const uint2 u = planes[pl][k][g][q];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const uint32_t f[4] = {w[2 * t].x, w[2 * t + 1].x, w[2 * t].y, w[2 * t + 1].y};
              mma_bf16(d[t], f, u.x, u.y);
            }
          }
        }
      }
      // (Both rows in one stretch of code: a lane without them carries numbers that nobody reads.)
      float top[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int e = 0; e < 8; ++e) l[h][e] += d[e >> 1][2 * (e & 1) + h];         // (past the vocabulary: -inf + something)
        if (!whole) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (vg + 8 * e >= p.V) l[h][e] = -CUDART_INF_F;
        }
        top[h] = max3_nan(max3_nan(max3_nan(l[h][0], l[h][1], l[h][2]), max3_nan(l[h][3], l[h][4], l[h][5]), l[h][6]), l[h][7], l[h][7]);
      }
      if (__any_sync(0xffffffffu, p.want_arg || !(top[0] <= st[0].rise()) || !(top[1] <= st[1].rise()))) {
        if (top[0] != top[0] || top[1] != top[1]) {
          unsigned which = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) which |= l[i >> 3][i & 7] != l[i >> 3][i & 7] && have[i >> 3] ? 1u << i : 0u;
#pragma unroll 1
          for (; which; which &= which - 1u) {
            const int at_i = __ffs(which) - 1, h = at_i >> 3, e = at_i & 7;
            float x = (h ? at[1] : at[0])[v0 + 8 * e - (kVec ? 3 * g : 0)];
            if (x == x) x += adapter_product(row(c, e), p.u + static_cast<size_t>(tile.row[2 * q + h]) * kAdMaxRank, rank);
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (i == at_i) l[i >> 3][i & 7] = x;
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)                    // (the largest of those that are numbers)
            top[h] = fmaxf(max3(max3(l[h][0], l[h][1], l[h][2]), max3(l[h][3], l[h][4], l[h][5]), l[h][6]), l[h][7]);
        }
        st[0].rises(l[0], top[0], p.want_arg, [&](int e) { return vg + 8 * e; });
        st[1].rises(l[1], top[1], p.want_arg, [&](int e) { return vg + 8 * e; });
      }
      if (whole) {
        st[0].template add<false>(l[0], top[0]);
        st[1].template add<false>(l[1], top[1]);
      } else if (vg < p.V) {
        st[0].template add<true>(l[0], top[0]);
        st[1].template add<true>(l[1], top[1]);
      }
      if (kVec && whole) {
        __syncwarp();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 8; ++e) buffer[warp][2 * q + h][8 * e + g] = l[h][e];
        __syncwarp();
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (have[h]) {
            *reinterpret_cast<float4*>(at[h] + v0) = *reinterpret_cast<const float4*>(&buffer[warp][2 * q + h][4 * g]);
            *reinterpret_cast<float4*>(at[h] + v0 + 32) = *reinterpret_cast<const float4*>(&buffer[warp][2 * q + h][32 + 4 * g]);
          }
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (have[h] && (whole || vg + 8 * e < p.V)) at[h][v0 + 8 * e - (kVec ? 3 * g : 0)] = l[h][e];
      }
    }
    // (rows with entries of -inf: the sums once more, clear of them, from what has been stored)
    if (__any_sync(0xffffffffu, st[0].lost() || st[1].lost())) {
      __syncwarp();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (!st[h].lost() || !have[h]) continue;
        st[h].clear();
#pragma unroll 1
        for (int c = c_begin; c < c_end; c += kAdUpWarps) {
          const int vg = c * kAdChunk + g;
          float l[8], top = -CUDART_INF_F;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            l[e] = vg + 8 * e < p.V ? at[h][vg + 8 * e - (kVec ? 4 * g : g)] : -CUDART_INF_F;
            top = fmaxf(top, l[e]);
          }
          st[h].rises(l, top, p.want_arg, [&](int e) { return vg + 8 * e; });
          st[h].template add<true>(l, top);
        }
      }
      __syncwarp();
    }
    // a row's statistics over the eight lanes that hold it, then over the warps
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      Stats s = st[h].stats();
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        Stats x;
        x.m = __shfl_xor_sync(0xffffffffu, s.m, o); x.s = __shfl_xor_sync(0xffffffffu, s.s, o);
        x.t = __shfl_xor_sync(0xffffffffu, s.t, o); x.arg = __shfl_xor_sync(0xffffffffu, s.arg, o);
        s = stats_merge(s, x);
      }
      if (g == 0) warp_stats[warp][2 * q + h] = make_float4(s.m, s.s, s.t, __int_as_float(s.arg));
    }
    __syncthreads();
    if (threadIdx.x < n) {
      Stats all = stats_empty();
#pragma unroll
      for (int w = 0; w < kAdUpWarps; ++w) {
        const float4 x = warp_stats[w][threadIdx.x];
        all = stats_merge(all, Stats{x.x, x.y, x.z, __float_as_int(x.w)});
      }
      p.partials[static_cast<size_t>(tile.row[threadIdx.x]) * p.part_stride + part] = make_float4(all.m, all.s, all.t, __int_as_float(all.arg));
    }
    if (part == 0) {                                       // what the GEMM left beyond this kernel's parts counts no more
      const int stale = p.nparts - P;
      for (int i = threadIdx.x; i < n * stale; i += kAdUpWarps * 32)
        p.partials[static_cast<size_t>(tile.row[i / stale]) * p.part_stride + P + i % stale] =
            make_float4(-CUDART_INF_F, 0.f, 0.f, __int_as_float(0x7fffffff));
    }
    __syncthreads();                                     // (the planes and the warps' statistics have been read)
  }
}

// Tiles that a batch may need: whole ones, and one more for each adapter; or those of every sequence by itself.
int adapter_max_tiles(int B, int k1, int slots) {
  const long long own = static_cast<long long>(B) * ((k1 + kAdRows - 1) / kAdRows);
  const long long shared = static_cast<long long>(B) * k1 / kAdRows + (B < slots ? B : slots);
  return static_cast<int>(B <= kAdMaxSorted && shared < own ? shared : own);
}

cudaError_t launch_adapter_down(const AdapterParams& p, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.B + 1), static_cast<unsigned>((p.rank + 15) / 16), static_cast<unsigned>((p.rows_per_seq + 15) / 16));
  cfg.blockDim = dim3(kAdDownWarps * 32); cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, adapter_down_kernel, p);
}

cudaError_t launch_adapter_up(const AdapterParams& p, int num_sms, cudaStream_t stream) {
  // As many CTAs as fit (by registers), a chunk per warp at least.
  const int chunks = (p.V + kAdChunk - 1) / kAdChunk, resident = kAdUpCtas;
  const long long most = static_cast<long long>(p.max_tiles) * ((chunks + kAdUpWarps - 1) / kAdUpWarps);
  const unsigned grid = static_cast<unsigned>(most < resident * num_sms ? most : resident * num_sms);
  const bool vec = p.ldl % 4 == 0 && (reinterpret_cast<uintptr_t>(p.logits) & 15u) == 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kAdUpWarps * 32); cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  auto* kernel = adapter_up_kernel<true, 0>;
  switch (p.rank) {
    case 8: kernel = vec ? adapter_up_kernel<true, 8> : adapter_up_kernel<false, 8>; break;
    case 16: kernel = vec ? adapter_up_kernel<true, 16> : adapter_up_kernel<false, 16>; break;
    case 32: kernel = vec ? adapter_up_kernel<true, 32> : adapter_up_kernel<false, 32>; break;
    case 64: kernel = vec ? adapter_up_kernel<true, 64> : adapter_up_kernel<false, 64>; break;
    default: kernel = vec ? adapter_up_kernel<true, 0> : adapter_up_kernel<false, 0>;
  }
  return cudaLaunchKernelEx(&cfg, kernel, p);
}
