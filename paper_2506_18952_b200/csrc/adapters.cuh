// adapters.cuh - low-rank adapters of many requests beside the LM head.  Part of hola_verify.cu (inside its anonymous namespace).
//
// Sequence b uses adapter a = ids[b] (or none): its k + 1 verify rows x[r] get the logits of the head W + s_a B_a A_a,
//   l[r,v] = sum_h W[v,h] x[r,h] + sum_i B_a[v,i] u[r,i],   u[r,i] = s_a sum_h A_a[i,h] x[r,h],   i < rank.
//
//   adapter_down_kernel  u, ahead of the GEMM: one CTA per sequence, 16 ranks and 16 rows, whose warps share the hidden channels.
//   adapter_up_kernel    behind the GEMM, whatever its weight mode: adds the second product to the stored logits and makes the
//       rows' softmax statistics anew, in the form in which the GEMM's epilogue leaves them (partials of each row), so that
//       everything behind reads them as before.  Rows without an adapter are left alone.
// Both products run on bf16 operands with fp32 accumulation; u, which is fp32, enters the second one as three bf16 planes that
// add up to it exactly (8 significant bits each), so that no rounding is added to what an fp32 product would have.

constexpr int kAdMaxRank = 128;
constexpr int kAdDownWarps = 16;
constexpr int kAdUpWarps = 4;
constexpr int kAdChunk = 32;           // vocabulary entries per warp step

struct AdapterParams {
  const uint16_t* A;           // bf16 [slots][rank][H]
  const uint16_t* Bm;          // bf16 [V][pitch]: slot s at columns s * rank
  const float* scale;          // [slots], or null: 1
  const int* ids;              // [B]
  int slots, rank, pitch;
  int B, rows_per_seq, H, V;
  const uint16_t* hidden;      // [B][rows_per_seq][H]
  float* u;                    // [rows][kAdMaxRank]
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

// The order of the channels inside a sum is free, so lane (g, q) of a warp loads 16 bytes = 8 neighbouring channels of its row and
// hands them to two MMAs: channels 8q .. 8q+3 in the places the first one gives lane q, 8q+4 .. 8q+7 in those of the second.
__global__ void __launch_bounds__(kAdDownWarps * 32) adapter_down_kernel(const AdapterParams p) {
  __shared__ float sums[kAdDownWarps][16][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int b = blockIdx.x, i0 = blockIdx.y * 16, j0 = blockIdx.z * 16;
  grid_dependency_wait();
  grid_dependency_release();
  if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && warp == 0 && p.status) {
    bool bad = false;
    for (int i = lane; i < p.B; i += 32) bad = bad || p.ids[i] < -1 || p.ids[i] >= p.slots;
    const unsigned flags = __any_sync(0xffffffffu, bad) ? HOLA_FLAG_BAD_ADAPTER : 0u;
    if (lane == 0) {
      if (p.clear_status) *p.status = flags;
      else if (flags) atomicOr(p.status, flags);
    }
  }
  const int a = adapter_of(p, b);
  if (a < 0) return;
  const int rows = min(16, p.rows_per_seq - j0), ranks = min(16, p.rank - i0);
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
    p.u[(static_cast<size_t>(b) * p.rows_per_seq + j0 + j) * kAdMaxRank + i0 + i] = p.scale ? s * p.scale[a] : s;
  }
}

__device__ __forceinline__ void stats_fold8(const float* v, int vocab0, int want_arg, Stats& st) {
  const float cmax = fmaxf(max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), v[6]), v[7]);
  if (cmax > st.m) {
    if (st.m != -CUDART_INF_F) {
      const float d = st.m - cmax, sc = ex2_approx(d * kLog2e);
      st.t = sc * (st.t + d * st.s);
      st.s *= sc;
    }
    st.m = cmax;
    if (want_arg) {
      int first = 0;
#pragma unroll
      for (int i = 7; i > 0; --i)
        if (v[i] == cmax) first = i;
      st.arg = vocab0 + (v[0] == cmax ? 0 : first);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (v[i] == -CUDART_INF_F) continue;                 // (entries past the vocabulary)
    const float d = v[i] - st.m, e = ex2_approx(d * kLog2e);
    st.s += e;
    st.t = fmaf(e, d, st.t);
  }
}

// A warp step covers 32 vocabulary entries and 16 rows: column n of tile j of the four MMAs stands for entry 8 (n / 2) + 2 j + n % 2,
// so that a lane ends up with eight neighbouring entries of rows g and g + 8.
template <bool kVec>
__global__ void __launch_bounds__(kAdUpWarps * 32) adapter_up_kernel(const AdapterParams p, int P) {
  __shared__ uint2 planes[3][kAdMaxRank / 16][16][4];    // [plane][16 ranks][row][q]: ranks 4q .. 4q+3 of the sixteen
  __shared__ float4 warp_stats[kAdUpWarps][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int b = blockIdx.x, part = blockIdx.y;
  grid_dependency_wait();
  const int a = adapter_of(p, b);
  if (a < 0) return;
  const int chunks = (p.V + kAdChunk - 1) / kAdChunk, per = (chunks + P - 1) / P;
  const int c_end = min(chunks, (part + 1) * per);
  const int steps = (p.rank + 15) >> 4;
  const uint16_t* Bm = p.Bm + static_cast<size_t>(a) * p.rank;
  for (int j0 = 0; j0 < p.rows_per_seq; j0 += 16) {
    const int rows = min(16, p.rows_per_seq - j0);
    const size_t row0 = static_cast<size_t>(b) * p.rows_per_seq + j0;
    __syncthreads();
    for (int i = threadIdx.x; i < steps * 64; i += kAdUpWarps * 32) {
      const int k = i >> 6, r = (i >> 2) & 15, qq = i & 3;
      uint32_t w[3][2] = {};
      if (r < rows) {
        const float4 u4 = *reinterpret_cast<const float4*>(p.u + (row0 + r) * kAdMaxRank + 16 * k + 4 * qq);
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
    Stats st[2] = {stats_empty(), stats_empty()};
    for (int c = part * per + warp; c < c_end; c += kAdUpWarps) {
      const int v0 = c * kAdChunk + 8 * q;               // this lane's entries
      float l[2][8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = g + 8 * h;
        const float* at = p.logits + (row0 + r) * p.ldl + v0;
#pragma unroll
        for (int e = 0; e < 8; ++e) l[h][e] = -CUDART_INF_F;
        if (r < rows) {
          if (kVec && v0 + 8 <= p.V) {
            const float4 x = *reinterpret_cast<const float4*>(at), y = *reinterpret_cast<const float4*>(at + 4);
            l[h][0] = x.x; l[h][1] = x.y; l[h][2] = x.z; l[h][3] = x.w;
            l[h][4] = y.x; l[h][5] = y.y; l[h][6] = y.z; l[h][7] = y.w;
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (v0 + e < p.V) l[h][e] = at[e];
          }
        }
      }
      float d[4][4] = {};
      for (int k = 0; k < steps; ++k) {
        uint32_t f[3][4];
#pragma unroll
        for (int pl = 0; pl < 3; ++pl) {
          const uint2 x = planes[pl][k][g][q], y = planes[pl][k][g + 8][q];
          f[pl][0] = x.x; f[pl][1] = y.x; f[pl][2] = x.y; f[pl][3] = y.y;
        }
        const bool in = 16 * k + 4 * q < p.rank;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int v = c * kAdChunk + 8 * (g >> 1) + 2 * j + (g & 1);
          uint2 w = make_uint2(0u, 0u);
          if (in && v < p.V) w = *reinterpret_cast<const uint2*>(Bm + static_cast<size_t>(v) * p.pitch + 16 * k + 4 * q);
#pragma unroll
          for (int pl = 2; pl >= 0; --pl) mma_bf16(d[j], f[pl], w.x, w.y);
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = g + 8 * h;
        if (r >= rows) continue;
        float* at = p.logits + (row0 + r) * p.ldl + v0;
#pragma unroll
        for (int e = 0; e < 8; ++e) l[h][e] += d[e >> 1][2 * h + (e & 1)];       // (past the vocabulary: -inf + 0)
        if (kVec && v0 + 8 <= p.V) {
          *reinterpret_cast<float4*>(at) = make_float4(l[h][0], l[h][1], l[h][2], l[h][3]);
          *reinterpret_cast<float4*>(at + 4) = make_float4(l[h][4], l[h][5], l[h][6], l[h][7]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (v0 + e < p.V) at[e] = l[h][e];
        }
        if (v0 < p.V) stats_fold8(l[h], v0, p.want_arg, st[h]);
      }
    }
    // a row's statistics over the four lanes that hold it, then over the warps
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        Stats x;
        x.m = __shfl_xor_sync(0xffffffffu, st[h].m, o); x.s = __shfl_xor_sync(0xffffffffu, st[h].s, o);
        x.t = __shfl_xor_sync(0xffffffffu, st[h].t, o); x.arg = __shfl_xor_sync(0xffffffffu, st[h].arg, o);
        st[h] = stats_merge(st[h], x);
      }
      if (q == 0) warp_stats[warp][g + 8 * h] = make_float4(st[h].m, st[h].s, st[h].t, __int_as_float(st[h].arg));
    }
    __syncthreads();
    if (threadIdx.x < rows) {
      Stats all = stats_empty();
#pragma unroll
      for (int w = 0; w < kAdUpWarps; ++w) {
        const float4 x = warp_stats[w][threadIdx.x];
        all = stats_merge(all, Stats{x.x, x.y, x.z, __float_as_int(x.w)});
      }
      p.partials[(row0 + threadIdx.x) * p.part_stride + part] = make_float4(all.m, all.s, all.t, __int_as_float(all.arg));
    }
    if (part == 0) {                                     // what the GEMM left beyond this kernel's parts counts no more
      const int stale = p.nparts - P;
      for (int i = threadIdx.x; i < rows * stale; i += kAdUpWarps * 32)
        p.partials[(row0 + i / stale) * p.part_stride + P + i % stale] =
            make_float4(-CUDART_INF_F, 0.f, 0.f, __int_as_float(0x7fffffff));
    }
  }
}

cudaError_t launch_adapter_down(const AdapterParams& p, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.B), static_cast<unsigned>((p.rank + 15) / 16), static_cast<unsigned>((p.rows_per_seq + 15) / 16));
  cfg.blockDim = dim3(kAdDownWarps * 32); cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, adapter_down_kernel, p);
}

cudaError_t launch_adapter_up(const AdapterParams& p, int num_sms, cudaStream_t stream) {
  // Parts of the vocabulary: eight CTAs per SM, a chunk per warp at least, and no more partials than a row has room for.
  const int chunks = (p.V + kAdChunk - 1) / kAdChunk;
  int P = (8 * num_sms + p.B - 1) / p.B;
  if (P > (chunks + kAdUpWarps - 1) / kAdUpWarps) P = (chunks + kAdUpWarps - 1) / kAdUpWarps;
  if (P > p.nparts) P = p.nparts;
  if (P < 1) P = 1;
  const bool vec = p.ldl % 4 == 0 && (reinterpret_cast<uintptr_t>(p.logits) & 15u) == 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.B), static_cast<unsigned>(P));
  cfg.blockDim = dim3(kAdUpWarps * 32); cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return vec ? cudaLaunchKernelEx(&cfg, adapter_up_kernel<true>, p, P) : cudaLaunchKernelEx(&cfg, adapter_up_kernel<false>, p, P);
}
