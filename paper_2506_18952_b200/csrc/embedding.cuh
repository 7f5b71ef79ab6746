// embedding.cuh - rows of a table by token, and the gradient of the table.  Part of decode_ops.cu (inside its anonymous namespace).

// ------------------------------------------------------------------------------------------------ lookup
// out[r] = add[r] + scale * W[tok[r]], every operation one rounding in fp32 (the scale of a quantised row first), the result rounded
// once more where it is stored in 16 bits.
constexpr int kEmThreads = 128;
constexpr int kEmMaxH = 1 << 30;       // channels: 32 bits count them, and a step of 65535 slices (at most 2^27 channels) beyond the last one

// Types of rows in memory (hola_t_dtype).
enum { kTabF32 = HOLA_T_F32, kTabBf16 = HOLA_T_BF16, kTabF16 = HOLA_T_F16, kTabInt8 = HOLA_T_INT8, kTabMixed = HOLA_T_MIXED };
__host__ __device__ constexpr int tab_bytes(int t) { return t == kTabF32 ? 4 : t == kTabInt8 ? 1 : 2; }

struct EmParams {
  const void* tokens;
  int wide;                            // 64-bit ids
  long long N;
  int V, H;
  long long v_offset, V_global;
  const void *table, *table_end, *add_end;      // (ends of what may be read)
  long long row_stride;                // channels
  const float* w_scale;
  hola_wmix mix;
  float scale;
  const void* add;
  long long add_stride;
  void* out;
  long long out_stride;
  unsigned* status;
};

// Row of the table that a token names; -1: none.  `bad`: no token at all.
__device__ __forceinline__ int em_row(const void* tokens, int wide, long long r, int V, long long v_offset, long long V_global, bool* bad) {
  const long long t = wide ? static_cast<const long long*>(tokens)[r] : static_cast<const int*>(tokens)[r];
  *bad = t < -1 || t >= V_global;
  const long long v = t - v_offset;
  return t >= 0 && v >= 0 && v < V ? static_cast<int>(v) : -1;
}

// n (8 or 1) channels as loaded, and as fp32.
template <int kType, int n>
struct EmWord {
  static constexpr int kBytes = tab_bytes(kType) * n;
  uint32_t w[kBytes < 4 ? 1 : kBytes / 4];
  __device__ __forceinline__ void load(const void* p) {
    if (kBytes == 32) {
      constexpr int k = kBytes < 4 ? 1 : kBytes / 4;
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1 % k]), "=r"(w[2 % k]), "=r"(w[3 % k]), "=r"(w[4 % k]), "=r"(w[5 % k]), "=r"(w[6 % k]), "=r"(w[7 % k])
                   : "l"(p) : "memory");
    } else if (kBytes == 16) {
      const uint4 a = *static_cast<const uint4*>(p);
      w[0] = a.x; w[1 % (kBytes < 4 ? 1 : kBytes / 4)] = a.y; w[2 % (kBytes < 4 ? 1 : kBytes / 4)] = a.z;
      w[3 % (kBytes < 4 ? 1 : kBytes / 4)] = a.w;
    } else if (kBytes == 8) {
      const uint2 a = *static_cast<const uint2*>(p);
      w[0] = a.x; w[1 % (kBytes < 4 ? 1 : kBytes / 4)] = a.y;
    } else if (kBytes == 4) {
      w[0] = *static_cast<const uint32_t*>(p);
    } else if (kBytes == 2) {
      w[0] = *static_cast<const uint16_t*>(p);
    } else {
      w[0] = *static_cast<const uint8_t*>(p);
    }
  }
  __device__ __forceinline__ void store(void* p) const {
    constexpr int k = kBytes < 4 ? 1 : kBytes / 4;
    if (kBytes == 32)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                   ::"l"(p), "r"(w[0]), "r"(w[1 % k]), "r"(w[2 % k]), "r"(w[3 % k]), "r"(w[4 % k]), "r"(w[5 % k]), "r"(w[6 % k]), "r"(w[7 % k])
                   : "memory");
    else if (kBytes == 16) *static_cast<uint4*>(p) = make_uint4(w[0], w[1 % k], w[2 % k], w[3 % k]);
    else if (kBytes == 4) *static_cast<uint32_t*>(p) = w[0];
    else if (kBytes == 2) *static_cast<uint16_t*>(p) = static_cast<uint16_t>(w[0]);
  }
  __device__ __forceinline__ float get(int i) const {
    if (kType == kTabF32) return __uint_as_float(w[i]);
    if (kType == kTabBf16) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    if (kType == kTabF16) return __half2float(__ushort_as_half(static_cast<unsigned short>(w[i / 2] >> (16 * (i & 1)))));
    return static_cast<float>(static_cast<int>(w[i / 4] << (24 - 8 * (i & 3))) >> 24);
  }
};

// n channels to memory, rounded to nearest even.
template <int kType, int n>
__device__ __forceinline__ void em_store(void* p, const float* x) {
  if (kType == kTabF32) {
    if (n == 8) {
      asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                   ::"l"(p), "f"(x[0]), "f"(x[1 % n]), "f"(x[2 % n]), "f"(x[3 % n]), "f"(x[4 % n]), "f"(x[5 % n]), "f"(x[6 % n]), "f"(x[7 % n])
                   : "memory");
    } else if (n == 4) {
      *static_cast<float4*>(p) = make_float4(x[0], x[1 % n], x[2 % n], x[3 % n]);
    } else {
      *static_cast<float*>(p) = x[0];
    }
    return;
  }
  if (n >= 4) {
    constexpr int kPairs = n / 2 < 4 ? 4 : n / 2;
    uint32_t h[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float a = x[(2 * i) % n], b = x[(2 * i + 1) % n];
      if (kType == kTabBf16) {
        const __nv_bfloat162 y = __floats2bfloat162_rn(a, b);
        h[i] = *reinterpret_cast<const uint32_t*>(&y);
      } else {
        const __half2 y = __floats2half2_rn(a, b);
        h[i] = *reinterpret_cast<const uint32_t*>(&y);
      }
    }
    if (n == 16)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                   ::"l"(p), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]), "r"(h[4 % kPairs]), "r"(h[5 % kPairs]), "r"(h[6 % kPairs]), "r"(h[7 % kPairs])
                   : "memory");
    else if (n == 8) *static_cast<uint4*>(p) = make_uint4(h[0], h[1], h[2], h[3]);
    else *static_cast<uint2*>(p) = make_uint2(h[0], h[1]);
  } else {
    *static_cast<uint16_t*>(p) = kType == kTabBf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(x[0])) : __half_as_ushort(__float2half_rn(x[0]));
  }
}
template <int n>
__device__ __forceinline__ void em_store_as(int type, void* base, long long at, const float* x) {
  if (type == kTabF32) em_store<kTabF32, n>(static_cast<float*>(base) + at, x);
  else if (type == kTabBf16) em_store<kTabBf16, n>(static_cast<uint16_t*>(base) + at, x);
  else em_store<kTabF16, n>(static_cast<uint16_t*>(base) + at, x);
}
template <int n>
__device__ __forceinline__ void em_load_as(int type, const void* base, long long at, float* x) {
  if (type == kTabF32) {
    EmWord<kTabF32, n> w;
    w.load(static_cast<const float*>(base) + at);
#pragma unroll
    for (int i = 0; i < n; ++i) x[i] = w.get(i);
  } else {
    EmWord<kTabBf16, n> w;
    w.load(static_cast<const uint16_t*>(base) + at);
    EmWord<kTabF16, n> f;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof w.w / 4); ++i) f.w[i] = w.w[i];
#pragma unroll
    for (int i = 0; i < n; ++i) x[i] = type == kTabBf16 ? w.get(i) : f.get(i);
  }
}

// Eight channels from any address: the aligned 16 bytes that hold them, on their way, and shifted into place later.  What else these hold is of
// the same tensor; at its ends, where it would not be, channel by channel.
template <int kType>
struct EmRaw {
  static constexpr int kSize = tab_bytes(kType), kNeed = 8 * kSize, kGranules = (kNeed + 15) / 16 + 1;
  uint32_t w[4 * kGranules];
  unsigned shift;
  // Channels h .. h + 7 of a row of H (those outside it are not used) of a tensor from begin to end.
  __device__ __forceinline__ void load(const void* begin, const void* end, long long row, int h, int H) {
    const unsigned char* at = static_cast<const unsigned char*>(begin) + (row + h) * kSize;
    shift = static_cast<unsigned>(reinterpret_cast<uintptr_t>(at) & 15u);
    const unsigned char* first = at - shift;
    const int granules = static_cast<int>(shift + kNeed + 15) / 16;
    if (first >= static_cast<const unsigned char*>(begin) && first + 16 * granules <= static_cast<const unsigned char*>(end)) {
#pragma unroll
      for (int i = 0; i < kGranules; ++i)
        if (i < granules) {
          const uint4 y = *reinterpret_cast<const uint4*>(first + 16 * i);
          w[4 * i] = y.x; w[4 * i + 1] = y.y; w[4 * i + 2] = y.z; w[4 * i + 3] = y.w;
        }
    } else {
      ragged(at, h, H);
    }
  }
  __device__ __forceinline__ void ragged(const unsigned char* at, int h, int H) {
    uint32_t y[kNeed / 4];
#pragma unroll
    for (int i = 0; i < kNeed / 4; ++i) y[i] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (h + e >= 0 && h + e < H) {
        if (kSize == 4) y[e * kSize / 4] = *reinterpret_cast<const uint32_t*>(at + e * kSize);
        else if (kSize == 2) y[e * kSize / 4] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(at + e * kSize)) << (16 * (e & 1));
        else y[e * kSize / 4] |= static_cast<uint32_t>(at[e]) << (8 * (e & 3));
      }
#pragma unroll
    for (int i = 0; i < kNeed / 4; ++i) w[i] = y[i];
    shift = 0;
  }
  __device__ __forceinline__ EmWord<kType, 8> get() {
#pragma unroll
    for (int i = 0; i + 1 < 4 * kGranules; ++i) w[i] = shift & 4u ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i + 2 < 4 * kGranules; ++i) w[i] = shift & 8u ? w[i + 2] : w[i];
    EmWord<kType, 8> x;
#pragma unroll
    for (int i = 0; i < kNeed / 4; ++i) x.w[i] = __funnelshift_r(w[i], w[i + 1], 8 * (shift & 3u));
    return x;
  }
};

// n channels of a row of a mixed-width head: group of 256 rows -> its width and its place among the rows of that width.
template <int n>
__device__ __forceinline__ void em_mixed(const hola_wmix& mix, int H, int v, int h, float* x) {
  const int width = mix.group_width[v >> 8];
  const size_t row = static_cast<size_t>(mix.group_row[v >> 8]) + (v & 255);
  if (width == 16) {
    EmWord<kTabBf16, n> w;
    w.load(static_cast<const uint16_t*>(mix.W16) + row * H + h);
#pragma unroll
    for (int i = 0; i < n; ++i) x[i] = w.get(i);
  } else if (width == 8) {
    EmWord<kTabInt8, n> w;
    w.load(static_cast<const uint8_t*>(mix.W8) + row * H + h);
#pragma unroll
    for (int i = 0; i < n; ++i) x[i] = w.get(i);
  } else {
    // two codes a byte, the even channel in the low nibble; a power of two for every 128 channels
    const uint8_t* at = static_cast<const uint8_t*>(mix.W4) + (row * H + h) / 2;
    const uint32_t codes = n == 8 ? *reinterpret_cast<const uint32_t*>(at) : static_cast<uint32_t>(*at) >> (4 * (h & 1));
    const int e = mix.shift4[static_cast<size_t>(h / 128) * mix.rows4 + row];
#pragma unroll
    for (int i = 0; i < n; ++i) x[i] = static_cast<float>((static_cast<int>(codes << (28 - 4 * i)) >> 28) << e);
  }
}

// n: channels that a thread takes at once, 8 where everything is aligned, 16 where rows of 8 or 16 bits become results of 16; kWide: results
// of 32 bits, else of 16 (`f16`: which).  A CTA takes kRows rows at a time, or as many times that as leave no thread idle where rows are
// short (`lanes`: threads of a row, a power of two).  Bound by HBM: rows in, rows out.  us: 128 / 256 threads 16384 x 4096 bf16 33.2 /
// 35.6; 8 / 16 channels 33.1 / 31.8, 20000 x 4096 int8 41 / 34; rows one by one instead of four at a time 2304 x 4096 int8 18.3 -> 13.1.
template <int kType, int n>                            // rows on the way together
__host__ __device__ constexpr int em_rows() { return kType == kTabF32 || kType == kTabMixed || (n == 16 && kType != kTabInt8) ? 2 : 4; }

// kShort: several rows side by side in a CTA (addresses that all threads share are cheaper: 16384 x 4096 bf16 36.2 -> 33.2 us).
template <int kType, bool kWide, bool kAdd, bool kShort, int n>
__global__ void __launch_bounds__(kEmThreads, 8) embed_kernel(const __grid_constant__ EmParams p, int f16, int some_rows, int lanes_log2) {
  constexpr bool kCodes = kType == kTabInt8 || kType == kTabMixed, kMixed = kType == kTabMixed;
  constexpr int kWord = kMixed ? kTabBf16 : kType, kRows = em_rows<kType, n>(), kOut = kWide ? kTabF32 : kTabBf16;
  constexpr int kWords = n == 1 ? 4 : 1;                 // words of a row that a thread has on the way
  grid_dependency_wait();
  grid_dependency_release();
  const int lanes = kShort ? 1 << lanes_log2 : kEmThreads, lane = static_cast<int>(threadIdx.x) & (lanes - 1);
  const long long r0 = kShort ? (static_cast<long long>(blockIdx.x) * (kEmThreads >> lanes_log2) + (threadIdx.x >> lanes_log2)) * some_rows
                              : static_cast<long long>(blockIdx.x) * some_rows;
  const int rows = static_cast<int>(p.N - r0 < some_rows ? p.N - r0 : some_rows);          // (less than one: none)
  int v[kRows];
  float ws[kRows];
  bool any_bad = false;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    v[i] = -1;
    ws[i] = 1.f;
    if (i < rows) {
      bool bad;
      v[i] = em_row(p.tokens, p.wide, r0 + i, p.V, p.v_offset, p.V_global, &bad);
      any_bad = any_bad || bad;
      if (kCodes && v[i] >= 0) ws[i] = p.w_scale[v[i]];
    }
  }
  if (any_bad && p.status && lane == 0 && blockIdx.y == 0) atomicOr(p.status, HOLA_FLAG_BAD_TOKEN);
  // (what is neither scaled nor added to nor converted is passed on as it is)
  const bool as_is = !kAdd && p.scale == 1.f && (kWide ? kType == kTabF32 : kType == (f16 ? kTabF16 : kTabBf16));
  const int apart = lanes * n;                           // a thread's words
#pragma unroll 1
  for (int h0 = static_cast<int>(blockIdx.y) * apart * kWords + lane * n; h0 < p.H; h0 += static_cast<int>(gridDim.y) * apart * kWords) {
    EmWord<kWord, n> w[kRows][kWords];
    float x[kMixed ? kRows : 1][kMixed ? kWords : 1][n];
    EmWord<kOut, n> add[kAdd ? kRows : 1][kWords];
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
      for (int u = 0; u < kWords; ++u) {
        const int h = h0 + u * apart;
        if (kWords > 1 && h >= p.H) continue;
        if (v[i] >= 0) {
          if (kMixed) em_mixed<n>(p.mix, p.H, v[i], h, x[kMixed ? i : 0][kMixed ? u : 0]);
          else w[i][u].load(static_cast<const unsigned char*>(p.table) + (v[i] * p.row_stride + h) * tab_bytes(kWord));
        }
        if (kAdd && i < rows) add[kAdd ? i : 0][u].load(static_cast<const unsigned char*>(p.add) + ((r0 + i) * p.add_stride + h) * tab_bytes(kOut));
      }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (i >= rows) break;
#pragma unroll
      for (int u = 0; u < kWords; ++u) {
        const int h = h0 + u * apart;
        if (kWords > 1 && h >= p.H) continue;
        unsigned char* to = static_cast<unsigned char*>(p.out) + ((r0 + i) * p.out_stride + h) * tab_bytes(kOut);
        float y[n];
        if (v[i] >= 0) {
          if (as_is) {
            w[i][u].store(to);
            continue;
          }
#pragma unroll
          for (int c = 0; c < n; ++c) {
            y[c] = kMixed ? x[kMixed ? i : 0][kMixed ? u : 0][c] : w[i][u].get(c);
            if (kCodes) y[c] = __fmul_rn(y[c], ws[i]);
            y[c] = __fmul_rn(y[c], p.scale);
          }
        } else {
#pragma unroll
          for (int c = 0; c < n; ++c) y[c] = 0.f;
        }
        if (kAdd) {
          const EmWord<kOut, n>& a = add[kAdd ? i : 0][u];
          if (!kWide && f16) {
            EmWord<kTabF16, n> b;
#pragma unroll
            for (int c = 0; c < static_cast<int>(sizeof a.w / 4); ++c) b.w[c] = a.w[c];
#pragma unroll
            for (int c = 0; c < n; ++c) y[c] = __fadd_rn(b.get(c), y[c]);
          } else {
#pragma unroll
            for (int c = 0; c < n; ++c) y[c] = __fadd_rn(a.get(c), y[c]);
          }
        }
        if (!kWide && f16) em_store<kTabF16, n>(to, y);
        else em_store<kOut, n>(to, y);
      }
    }
  }
}

template <int kType, bool kWide, bool kAdd, int n>
cudaError_t launch_embed(const EmParams& p, int out_type, int num_sms, cudaStream_t stream) {
  constexpr int kAtOnce = n == 1 ? 4 : n;
  static_assert(65535ll * kEmThreads * kAtOnce <= INT32_MAX - kEmMaxH, "a channel behind the row still fits 32 bits");
  // (fewer threads to a row where the last of several slices would leave more than an eighth of them idle)
  int log2 = 0;
  while ((1 << log2) < kEmThreads && (1 << log2) * kAtOnce < p.H) ++log2;
  const long long chunks = (static_cast<long long>(p.H) + kAtOnce - 1) / kAtOnce;
  auto idle = [&](int log) { return ((chunks + (1 << log) - 1) >> log << log) - chunks; };
  while (log2 > 5 && 8 * idle(log2) > chunks && idle(log2 - 1) < idle(log2)) --log2;
  const int lanes = 1 << log2;
  const long long slices = (p.H + lanes * kAtOnce - 1) / (lanes * kAtOnce);
  const int slots = kEmThreads / lanes;
  // several rows at a time where there are CTAs enough all the same
  const int rows = p.N * slices >= 2ll * em_rows<kType, n>() * slots * num_sms ? em_rows<kType, n>() : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((p.N + rows * slots - 1) / (rows * slots)), static_cast<unsigned>(slices > 65535 ? 65535 : slices));
  cfg.blockDim = dim3(kEmThreads); cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  const int f16 = out_type == kTabF16 ? 1 : 0;
  if (n == 1 || lanes < kEmThreads) return cudaLaunchKernelEx(&cfg, embed_kernel<kType, kWide, kAdd, true, n>, p, f16, rows, log2);
  return cudaLaunchKernelEx(&cfg, embed_kernel<kType, kWide, kAdd, n == 1, n>, p, f16, rows, log2);
}
// The same where rows start anywhere: a thread takes 8 channels that lie side by side on an aligned address of the result (or, at a row's ends,
// what there is of them), out of the aligned words that hold them in the table.  us, channel by channel / so: 3000 x 4097 bf16 18.7 / 12.7,
// 5000 x 1001 8.6 / 6.0.
template <int kType, bool kWide, bool kAdd>
__global__ void __launch_bounds__(kEmThreads, 8) embed_any_kernel(const __grid_constant__ EmParams p, int f16, int lanes_log2) {
  constexpr int kRows = kType == kTabF32 || kAdd ? 1 : 2, kOut = kWide ? kTabF32 : kTabBf16, kOutSize = tab_bytes(kOut);
  grid_dependency_wait();
  grid_dependency_release();
  const int lanes = 1 << lanes_log2, lane = static_cast<int>(threadIdx.x) & (lanes - 1);
  const long long r0 = (static_cast<long long>(blockIdx.x) * (kEmThreads >> lanes_log2) + (threadIdx.x >> lanes_log2)) * kRows;
  const int rows = static_cast<int>(p.N - r0 < kRows ? p.N - r0 : kRows);
  int v[kRows], lead[kRows];                             // lead: channels ahead of the first aligned address of the result
  float ws[kRows];
  bool any_bad = false;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    v[i] = -1;
    ws[i] = 1.f;
    lead[i] = 0;
    if (i < rows) {
      bool bad;
      v[i] = em_row(p.tokens, p.wide, r0 + i, p.V, p.v_offset, p.V_global, &bad);
      any_bad = any_bad || bad;
      if (kType == kTabInt8 && v[i] >= 0) ws[i] = p.w_scale[v[i]];
      const uintptr_t to = reinterpret_cast<uintptr_t>(p.out) + static_cast<uintptr_t>((r0 + i) * p.out_stride) * kOutSize;
      lead[i] = static_cast<int>((0 - to) & (8 * kOutSize - 1)) / kOutSize;
    }
  }
  if (any_bad && p.status && lane == 0 && blockIdx.y == 0) atomicOr(p.status, HOLA_FLAG_BAD_TOKEN);
#pragma unroll 1
  for (int c = static_cast<int>(blockIdx.y) * lanes + lane; 8 * (c - 1) < p.H; c += static_cast<int>(gridDim.y) * lanes) {
    EmRaw<kType> w[kRows];
    EmRaw<kOut> add[kAdd ? kRows : 1];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int h = lead[i] + 8 * (c - 1);
      if (h <= -8 || h >= p.H) continue;
      if (v[i] >= 0) w[i].load(p.table, p.table_end, v[i] * p.row_stride, h, p.H);
      if (kAdd && i < rows) add[kAdd ? i : 0].load(p.add, p.add_end, (r0 + i) * p.add_stride, h, p.H);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int h = lead[i] + 8 * (c - 1);
      if (i >= rows || h <= -8 || h >= p.H) continue;
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = 0.f;
      if (v[i] >= 0) {
        const EmWord<kType, 8> x = w[i].get();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y[e] = x.get(e);
          if (kType == kTabInt8) y[e] = __fmul_rn(y[e], ws[i]);
          y[e] = __fmul_rn(y[e], p.scale);
        }
      }
      if (kAdd) {
        const EmWord<kOut, 8> a = add[kAdd ? i : 0].get();
        EmWord<kTabF16, 8> b;
#pragma unroll
        for (int k = 0; k < 4; ++k) b.w[k] = a.w[k];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = __fadd_rn(!kWide && f16 ? b.get(e) : a.get(e), y[e]);
      }
      unsigned char* to = static_cast<unsigned char*>(p.out) + ((r0 + i) * p.out_stride + h) * kOutSize;
      if (h >= 0 && h + 8 <= p.H) {
        if (!kWide && f16) em_store<kTabF16, 8>(to, y);
        else em_store<kOut, 8>(to, y);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (h + e >= 0 && h + e < p.H) {
            if (!kWide && f16) em_store<kTabF16, 1>(to + e * kOutSize, y + e);
            else em_store<kOut, 1>(to + e * kOutSize, y + e);
          }
      }
    }
  }
}

template <int kType, bool kWide, bool kAdd>
cudaError_t launch_embed_any(const EmParams& p, int out_type, cudaStream_t stream) {
  constexpr int kRows = kType == kTabF32 || kAdd ? 1 : 2;
  const int chunks = static_cast<int>((static_cast<long long>(p.H) + 15) / 8);
  int log2 = 0;
  while ((1 << log2) < kEmThreads && 1 << log2 < chunks) ++log2;
  const int lanes = 1 << log2, slots = kEmThreads / lanes * kRows, slices = (chunks + lanes - 1) / lanes;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((p.N + slots - 1) / slots), static_cast<unsigned>(slices > 65535 ? 65535 : slices));
  cfg.blockDim = dim3(kEmThreads); cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, embed_any_kernel<kType, kWide, kAdd>, p, out_type == kTabF16 ? 1 : 0, log2);
}
template <int kType>
cudaError_t launch_embed_any_of(const EmParams& p, int out_type, cudaStream_t stream) {
  if (out_type == kTabF32)
    return p.add ? launch_embed_any<kType, true, true>(p, out_type, stream) : launch_embed_any<kType, true, false>(p, out_type, stream);
  return p.add ? launch_embed_any<kType, false, true>(p, out_type, stream) : launch_embed_any<kType, false, false>(p, out_type, stream);
}

template <int kType, int n>
cudaError_t launch_embed_as(const EmParams& p, int out_type, int num_sms, cudaStream_t stream) {
  if (out_type == kTabF32)
    return p.add ? launch_embed<kType, true, true, n>(p, out_type, num_sms, stream) : launch_embed<kType, true, false, n>(p, out_type, num_sms, stream);
  return p.add ? launch_embed<kType, false, true, n>(p, out_type, num_sms, stream) : launch_embed<kType, false, false, n>(p, out_type, num_sms, stream);
}
// Sixteen channels at once: results of 16 bits from rows of 8 or 16.
template <int kType>
cudaError_t launch_embed_16_of(const EmParams& p, int out_type, int num_sms, cudaStream_t stream) {
  return p.add ? launch_embed<kType, false, true, 16>(p, out_type, num_sms, stream) : launch_embed<kType, false, false, 16>(p, out_type, num_sms, stream);
}
cudaError_t launch_embed_16(const EmParams& p, int type, int out_type, int num_sms, cudaStream_t stream) {
  return type == kTabInt8 ? launch_embed_16_of<kTabInt8>(p, out_type, num_sms, stream)
         : type == kTabBf16 ? launch_embed_16_of<kTabBf16>(p, out_type, num_sms, stream) : launch_embed_16_of<kTabF16>(p, out_type, num_sms, stream);
}
// words: eight channels of every row start on an aligned address.
cudaError_t launch_embed_of(const EmParams& p, int type, int out_type, bool words, int num_sms, cudaStream_t stream) {
  switch (type) {
    case kTabF32: return words ? launch_embed_as<kTabF32, 8>(p, out_type, num_sms, stream) : launch_embed_any_of<kTabF32>(p, out_type, stream);
    case kTabBf16: return words ? launch_embed_as<kTabBf16, 8>(p, out_type, num_sms, stream) : launch_embed_any_of<kTabBf16>(p, out_type, stream);
    case kTabF16: return words ? launch_embed_as<kTabF16, 8>(p, out_type, num_sms, stream) : launch_embed_any_of<kTabF16>(p, out_type, stream);
    case kTabInt8: return words ? launch_embed_as<kTabInt8, 8>(p, out_type, num_sms, stream) : launch_embed_any_of<kTabInt8>(p, out_type, stream);
    default: return words ? launch_embed_as<kTabMixed, 8>(p, out_type, num_sms, stream) : launch_embed_as<kTabMixed, 1>(p, out_type, num_sms, stream);
  }
}

// ------------------------------------------------------------------------------------------------ gradient
// dW[v] = scale * sum of g[r] over the rows r with tok[r] = v, in rising r, in fp32.  Two launches (few tokens: embed_grad_few_kernel).
//
// 1. Tokens sorted (stable), with nothing exchanged between the CTAs: each takes a range of ids and reads all tokens, every warp a
//    stretch of them, lists those inside its range, and counts those below it (where its part of the sorted order begins).  Counts per
//    (id, warp), and a scan over them, give every warp the place of its first occurrence of every id.  Ranges are cut at the even marks
//    V j / U and at the marks (V + 1)^(i / Z) together, for vocabularies are numbered by falling frequency: no range holds more than 1 / U
//    of the ids nor, where p(id) is about 1 / (id + 1), much more than 1 / Z of the tokens (or one id).  Where the frequent ids lie side
//    by side further up, a CTA or two list most of the tokens (32768 x 4096, 512 ids from 100000 on: 166 us, from 0 on 88).  Bound by
//    latency; N x 4 or 8 bytes per CTA out of the L2.
// 2. Sums.  The sorted order is cut into windows; the rows of a token lie side by side there, in pieces of at most `S`.  A CTA adds up
//    the pieces that begin in its window, for a slice of 1024 channels (256 where there are no more).  A token with one piece is finished
//    by it; the pieces of the others go to the workspace, and the CTA that comes last adds them up in their order.  So the result does
//    not depend on the schedule. The whole table's gradient: further CTAs write zeros to the rows that no token names.  Bound by HBM.
constexpr int kEsThreads = 1024, kEsWarps = 32;
constexpr int kEsZipf = 74;            // Z
constexpr int kEsList = 512, kEsMaxList = 1024;       // tokens that a warp lists before it counts them: as many as there is room for
constexpr int kEsLoads = 8;            // 32 tokens each that a warp has on the way
constexpr int kEsMaxShared = 216 * 1024;       // shared memory of a CTA
constexpr int kEsIdBits = 11;          // ids of a range (with what is left of 32 bits for places in a warp's stretch)
constexpr int kEgThreads = 128, kEgFewThreads = 32, kEgEach = 8;       // threads of a CTA of the sums; where a row has at most 256 channels
constexpr int kEgMaxWindow = 64, kEgMaxPiece = 1024;
constexpr int kEgRanges = 256;         // ranges of ids whose distinct ones are added up beforehand
constexpr int kEgAhead = 8;            // rows of a thread on the way (those that start anywhere)
constexpr long long kEgMaxTokens = 1 << 25;      // what is left of a list's words for places in the stretch of one of 16 warps
constexpr int kEgPlanSms = 148;        // what the work is cut for (the workspace has to be known without a device)

struct EgParams {
  const void* tokens;
  int wide;
  int N, V, H;
  long long v_offset, V_global;
  int even, buckets, R, warps, chunk, list;      // sort: U, ranges of ids and how many a range holds at most, warps that count, tokens of a warp
                                       // and how many of them it lists
  int few;                             // one launch does it, see embed_grad_few_kernel
  int S, S_log2, window, slices, blank;      // sums: piece, window, slices of the channels; rows of a CTA that writes zeros
  const void* grad;
  long long g_stride;
  float scale;
  void* out;
  long long out_stride;
  int accumulate, by_rows;
  int* ids_out;                        // by_rows: the distinct tokens, rising
  int* count_out;
  // workspace
  int4* places;                        // [N] in sorted order: row, id, where the id's rows begin and end
  int2* numbers;                       // [N] by_rows: the id's range, its number among the distinct ones there
  int* first;                          // [V + 1] the whole table: where an id's rows begin
  int* distinct;                       // [buckets]
  int* valid;                          // tokens that have a row
  unsigned* done;                      // [ceil(N / S)][slices] pieces of a token that have arrived
  float* partial;                      // [2 ceil(N / S)][slices x channels of a slice]
  unsigned* status;
};

// Number of even marks V j / U (1 <= j < U) that are at most x.
__device__ __forceinline__ int es_even_upto(int x, int V, int U) {
  const long long j = ((static_cast<long long>(x) + 1) * U - 1) / V;
  return static_cast<int>(j < U - 1 ? j : U - 1);
}

// Shared memory of the sort, of `ids` ids at most in a range: [warp][id] counters (`pitch` of them a warp), per id where its rows begin and
// how many distinct ids lie before it, the warps' lists.
struct EsLayout {
  int pitch, heads, lists, total;
  __host__ __device__ EsLayout(int ids, int warps, int list, int cell) {
    pitch = (ids + 1) & ~1;
    heads = (pitch * warps * cell + 15) & ~15;
    lists = heads + (ids + 1) * 8;
    total = lists + warps * list * 4;
  }
};

// Cell: counters of a warp's tokens per id, 16 bits where there are few enough tokens; Token: as they lie in memory.
template <typename Cell, typename Token>
__global__ void __launch_bounds__(kEsThreads, 1) embed_sort_kernel(const __grid_constant__ EgParams p) {
  extern __shared__ __align__(16) unsigned char es_smem[];
  __shared__ int warp_below[kEsWarps];
  __shared__ uint64_t warp_sum[kEsWarps];
  __shared__ int mark[kEsZipf], range[2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = blockIdx.x;
  // The range: marks g and g + 1 of both kinds together (even ones before equal others).
  int place = 0;
  if (tid < kEsZipf - 1) {
    const float x = exp2f(log2f(static_cast<float>(p.V) + 1.f) * (static_cast<float>(tid + 1) / kEsZipf));
    mark[tid] = min(static_cast<int>(fminf(x, static_cast<float>(p.V))), p.V);
    place = tid + 1 + es_even_upto(mark[tid], p.V, p.even);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int r = g + e;
    const int before = __syncthreads_count(tid < kEsZipf - 1 && place < r);
    if (tid == 0) range[e] = r == 0 ? 0 : r == p.buckets ? p.V : static_cast<int>(static_cast<long long>(p.V) * (r - before) / p.even);
    __syncthreads();
    if (tid < kEsZipf - 1 && place == r && r < p.buckets) range[e] = mark[tid];
  }
  __syncthreads();
  const int lo = range[0], R = range[1] - lo;
  const EsLayout lay(p.R, p.warps, p.list, static_cast<int>(sizeof(Cell)));
  Cell* cells = reinterpret_cast<Cell*>(es_smem) + warp * lay.pitch;
  int2* heads = reinterpret_cast<int2*>(es_smem + lay.heads);
  uint32_t* list = reinterpret_cast<uint32_t*>(es_smem + lay.lists) + warp * p.list;
  for (int i = tid; i < lay.heads / 16; i += kEsThreads) reinterpret_cast<uint4*>(es_smem)[i] = make_uint4(0, 0, 0, 0);
  grid_dependency_wait();
  grid_dependency_release();
  // (counters of the second launch)
  const long long pieces = static_cast<long long>((p.N + p.S - 1) / p.S) * p.slices;
  for (long long i = static_cast<long long>(g) * kEsThreads + tid; i < pieces; i += static_cast<long long>(p.buckets) * kEsThreads) p.done[i] = 0;
  __syncthreads();

  const long long begin = static_cast<long long>(warp) * p.chunk;
  const int len = warp < p.warps ? static_cast<int>(min(static_cast<long long>(p.chunk), max(p.N - begin, 0ll))) : 0;
  int below = 0, n = 0;
  bool any_bad = false;
  const bool looks = g + 1 == p.buckets;                 // for what is no token at all (the last range's ids are rare ones)
  // Row of the table; none: above every row (as differences that wrap are).
  const unsigned V_global = static_cast<unsigned>(p.V_global), v_offset = static_cast<unsigned>(p.v_offset);
  auto row_of = [&](Token x, bool* inside) {
    unsigned t = static_cast<unsigned>(x);
    if (sizeof(Token) == 8 && static_cast<uint64_t>(x) >> 32 != 0) t = 0xffffffffu;
    *inside = t < V_global;
    return *inside ? t - v_offset : 0xffffffffu;
  };
  // One pass over the warp's stretch, one batch ahead; full(): the list may not hold the next tokens.
  auto stream = [&](bool count, auto&& full) {
    const Token* at = static_cast<const Token*>(p.tokens) + begin + lane;
    Token next[kEsLoads];
#pragma unroll
    for (int u = 0; u < kEsLoads; ++u) {
      next[u] = -1;
      if (32 * u + lane < len) next[u] = at[32 * u];
    }
#pragma unroll 1
    for (int r0 = 0; r0 < len; r0 += 32 * kEsLoads) {
      at += 32 * kEsLoads;
      const int left = len - r0 - 32 * kEsLoads - lane;
#pragma unroll
      for (int u = 0; u < kEsLoads; ++u) {
        bool inside;
        const unsigned v = row_of(next[u], &inside);
        if (count) {
          if (looks) any_bad = any_bad || (!inside && next[u] != -1);
          below += v < static_cast<unsigned>(lo) ? 1 : 0;
        }
        next[u] = -1;
        if (32 * u < left) next[u] = at[32 * u];
        const unsigned id = v - static_cast<unsigned>(lo);
        const bool mine = id < static_cast<unsigned>(R);
        const unsigned in = __ballot_sync(0xffffffffu, mine);
        if (in) {
          if (mine) list[n + __popc(in & ((1u << lane) - 1u))] = static_cast<uint32_t>(r0 + 32 * u + lane) << kEsIdBits | id;
          n += __popc(in);
        }
      }
      if (n > p.list - 32 * kEsLoads) full();
    }
  };
  auto count_list = [&]() {
    __syncwarp();
    for (int i = 0; i < n; i += 32) {
      // (lanes without a token: an id that there is not)
      const unsigned id = i + lane < n ? list[i + lane] & ((1u << kEsIdBits) - 1u) : 0xffffffffu;
      const unsigned same = __match_any_sync(0xffffffffu, id);
      if (i + lane < n && __ffs(same) - 1 == lane) cells[id] += static_cast<Cell>(__popc(same));
      __syncwarp();
    }
  };
  bool again = false;                                    // the list did not hold all
  stream(true, [&]() { count_list(); n = 0; again = true; });
  count_list();
  below = __reduce_add_sync(0xffffffffu, below);
  if (lane == 0) warp_below[warp] = below;
  if (__any_sync(0xffffffffu, any_bad) && lane == 0 && p.status) atomicOr(p.status, HOLA_FLAG_BAD_TOKEN);
  __syncthreads();

  // Per id: exclusive sums over the warps (two ids of 16 bits in one word; neither half runs over).  Over the ids: tokens in the upper half,
  // distinct ids in the lower.
  const int i0 = 2 * tid;
  unsigned all[2] = {0, 0};
  if (i0 < R) {
    using Pair = std::conditional_t<sizeof(Cell) == 2, uint32_t, uint2>;
    Pair* word = reinterpret_cast<Pair*>(reinterpret_cast<Cell*>(es_smem) + i0);
    const int step = lay.pitch / 2;
    Pair run = {};
#pragma unroll 8
    for (int w = 0; w < p.warps; ++w) {
      const Pair c = word[w * step];
      word[w * step] = run;
      if constexpr (sizeof(Cell) == 2) run += c;
      else run = make_uint2(run.x + c.x, run.y + c.y);
    }
    if constexpr (sizeof(Cell) == 2) { all[0] = run & 0xffffu; all[1] = run >> 16; }
    else { all[0] = run.x; all[1] = run.y; }
    if (i0 + 1 >= R) all[1] = 0;
  }
  const uint64_t sum = static_cast<uint64_t>(all[0] + all[1]) << 32 | ((all[0] ? 1u : 0u) + (all[1] ? 1u : 0u));
  uint64_t upto = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  if (lane == 31) warp_sum[warp] = upto;
  const int base = __reduce_add_sync(0xffffffffu, warp_below[lane]);
  __syncthreads();
  uint64_t before = 0, total = 0;
  {
    const uint64_t mine = warp_sum[lane];
    uint64_t x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    before = __shfl_sync(0xffffffffu, x - mine, warp);
    total = __shfl_sync(0xffffffffu, x, 31);
  }
  const uint64_t at = before + upto - sum;
  if (i0 < R) {
    const int head = base + static_cast<int>(at >> 32), number = static_cast<int>(at & 0xffffffffu);
    heads[i0] = make_int2(head, number);
    if (i0 + 1 < R) heads[i0 + 1] = make_int2(head + static_cast<int>(all[0]), number + (all[0] ? 1 : 0));
  }
  const int end = base + static_cast<int>(total >> 32);
  if (tid == 0) {
    heads[R] = make_int2(end, 0);
    p.distinct[g] = static_cast<int>(total & 0xffffffffu);
    if (g + 1 == p.buckets) *p.valid = end;
  }
  __syncthreads();
  if (p.first) {
    for (int i = tid; i < R; i += kEsThreads) p.first[lo + i] = heads[i].x;
    if (g + 1 == p.buckets && tid == 0) p.first[p.V] = end;
  }

  // The places.
  auto put_list = [&]() {
    __syncwarp();
    for (int i = 0; i < n; i += 32) {
      const bool have = i + lane < n;
      const uint32_t entry = have ? list[i + lane] : 0;
      const unsigned id = have ? entry & ((1u << kEsIdBits) - 1u) : 0xffffffffu;
      const unsigned same = __match_any_sync(0xffffffffu, id);
      unsigned ahead = 0;
      if (have) ahead = cells[id];
      __syncwarp();
      if (have) {
        if (__ffs(same) - 1 == lane) cells[id] = static_cast<Cell>(ahead + __popc(same));
        const int2 head = heads[id];
        const int to = head.x + static_cast<int>(ahead) + __popc(same & ((1u << lane) - 1u));
        p.places[to] = make_int4(static_cast<int>(begin + (entry >> kEsIdBits)), lo + static_cast<int>(id), head.x, heads[id + 1].x);
        if (p.by_rows) p.numbers[to] = make_int2(g, head.y);
      }
      __syncwarp();
    }
  };
  if (again) {
    n = 0;
    stream(false, [&]() { put_list(); n = 0; });
  }
  put_list();
}

// Eight channels of a thread, in runs that lie side by side: of 16 bytes of the gradient, or single ones where rows start anywhere.
// (Eight at once out of the aligned words that hold them, as lookups take them, and turned round for the result: 9000 x 1001 bf16 26.3 -> 32.8 us.)
template <int kRun, int kThreads>
__device__ __forceinline__ int eg_channel(int slice, int i, int thread = static_cast<int>(threadIdx.x)) {
  return slice * (kThreads * kEgEach) + (i / kRun) * (kThreads * kRun) + thread * kRun + i % kRun;
}
template <int kType>
using EgWord = EmWord<kType, kEgEach>;
// Rows of a thread in the ring: 24 KB of a CTA of 128 threads.
template <int kType>
__host__ __device__ constexpr int eg_stages() { return 24 * 1024 / (kEgThreads * kEgEach * tab_bytes(kType)); }

// The sums, scaled, to a row of the result (added to what is there), run by run.
template <int kRun, int kThreads>
__device__ __forceinline__ void eg_write(const EgParams& p, int out_type, long long row, int slice, const float* sum,
                                         int thread = static_cast<int>(threadIdx.x)) {
#pragma unroll
  for (int i = 0; i < kEgEach; i += kRun) {
    const int h = eg_channel<kRun, kThreads>(slice, i, thread);
    if (h >= p.H) continue;
    const long long at = row * p.out_stride + h;
    float x[kRun];
#pragma unroll
    for (int c = 0; c < kRun; ++c) x[c] = __fmul_rn(sum[i + c], p.scale);
    if (p.accumulate) {
      float a[kRun];
      em_load_as<kRun>(out_type, p.out, at, a);
#pragma unroll
      for (int c = 0; c < kRun; ++c) x[c] = __fadd_rn(a[c], x[c]);
    }
    em_store_as<kRun>(out_type, p.out, at, x);
  }
}

// Zeros to the bytes from `at` to `end`, whole elements of `size` bytes: 16 at a time where these are aligned.
template <int kThreads>
__device__ __forceinline__ void eg_zeros(unsigned char* at, unsigned char* end, int size) {
  unsigned char* first = at + ((0 - reinterpret_cast<uintptr_t>(at)) & 15u);
  unsigned char* last = end - (reinterpret_cast<uintptr_t>(end) & 15u);
  if (first > last) first = last = end;                  // (less than one such)
  for (unsigned char* x = first + threadIdx.x * 16; x < last; x += kThreads * 16) *reinterpret_cast<uint4*>(x) = make_uint4(0, 0, 0, 0);
  for (unsigned char* x = at + threadIdx.x * size; x < first; x += kThreads * size) {
    if (size == 4) *reinterpret_cast<uint32_t*>(x) = 0;
    else *reinterpret_cast<uint16_t*>(x) = 0;
  }
  for (unsigned char* x = last + threadIdx.x * size; x < end; x += kThreads * size) {
    if (size == 4) *reinterpret_cast<uint32_t*>(x) = 0;
    else *reinterpret_cast<uint16_t*>(x) = 0;
  }
}

// kVec: everything is aligned.
template <int kType, bool kVec, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == kEgFewThreads ? 16 : kVec ? 7 : 4)
    embed_grad_kernel(const __grid_constant__ EgParams p, int out_type, int windows) {
  constexpr int kRun = kVec ? 16 / tab_bytes(kType) : 1, kSlice = kThreads * kEgEach;
  constexpr int kMine = kEgRanges / kThreads;            // ranges that a thread adds up
  __shared__ __align__(16) unsigned char eg_ring[kVec ? eg_stages<kType>() * kSlice * tab_bytes(kType) : 16];
  __shared__ int rows[kEgMaxWindow + kEgMaxPiece];       // of the gradient, by place from x0 on; complemented where a piece ends
  __shared__ int4 spots[kEgMaxWindow];
  __shared__ int firsts[kEgMaxWindow + 1], out_rows[kEgMaxWindow];
  __shared__ int part_sum[kThreads / 32], range_rows[kEgRanges];
  __shared__ int last_here;
  const int slice = static_cast<int>(blockIdx.x % static_cast<unsigned>(p.slices)), tid = threadIdx.x;
  const int w = static_cast<int>(blockIdx.x / static_cast<unsigned>(p.slices));
  grid_dependency_wait();
  grid_dependency_release();
  if (w >= windows) {
    // The whole table: zeros to the rows of ids that do not occur.
    const float zero[kEgEach] = {};
    const int v0 = (w - windows) * p.blank, n = min(p.blank, p.V - v0);
    for (int i = tid; i <= n; i += kThreads) firsts[i] = p.first[v0 + i];
    __syncthreads();
    const int size = tab_bytes(out_type), h0 = slice * kSlice, h1 = min(h0 + kSlice, p.H);
    // (rows without a gap between them are one stretch)
    const bool joined = !kVec && p.slices == 1 && p.out_stride == p.H;
    for (int i = 0; i < n; ++i) {
      if (firsts[i] != firsts[i + 1]) continue;
      if (kVec) {
        eg_write<kRun, kThreads>(p, out_type, v0 + i, slice, zero);
      } else {
        int last = i;
        while (joined && last + 1 < n && firsts[last + 1] == firsts[last + 2]) ++last;
        unsigned char* out = static_cast<unsigned char*>(p.out);
        eg_zeros<kThreads>(out + ((v0 + i) * p.out_stride + h0) * size, out + ((v0 + last) * p.out_stride + h1) * size, size);
        i = last;
      }
    }
    return;
  }
  // (behind the last valid place there is something to read, which is not used)
  const int w0 = w * p.window, before_S = p.S - 1;
  for (int i = tid; i < p.window && w0 + i < p.N; i += kThreads) spots[i] = p.places[w0 + i];
  // by rows: distinct ids of the first kEgRanges ranges, added up
  int in_ranges = 0, upto = 0, in_range[kMine];
  if (p.by_rows) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      in_range[i] = kMine * tid + i < p.buckets ? p.distinct[kMine * tid + i] : 0;
      in_ranges += in_range[i];
    }
    upto = in_ranges;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, upto, o);
      if ((tid & 31) >= o) upto += x;
    }
    if ((tid & 31) == 31) part_sum[tid >> 5] = upto;
  }
  const int w1 = min(w0 + p.window, *p.valid);
  if (w == 0 && slice == 0 && p.by_rows && tid < 32) {
    int n = 0;
    for (int i = tid; i < p.buckets; i += 32) n += p.distinct[i];
    n = __reduce_add_sync(0xffffffffu, n);
    if (tid == 0) *p.count_out = n;
  }
  if (w0 >= w1) return;
  __syncthreads();
  if (p.by_rows) {
    // where each range's ids begin in the result
    int at = upto - in_ranges;
    for (int i = 0; i < tid >> 5; ++i) at += part_sum[i];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      range_rows[kMine * tid + i] = at;
      at += in_range[i];
    }
  }
  // Places x0 .. x1 - 1: from the first piece that begins in the window to the end of the last one that does.
  int x0 = w0, x1 = w1;
  {
    const int in = (w0 - spots[0].z) & before_S;
    if (in != 0) x0 = min(w0 + p.S - in, spots[0].w);
    if (x0 >= w1) return;                                // (all of the window inside one piece)
    const int4 last = spots[w1 - 1 - w0];
    x1 = min(last.z + (((w1 - 1 - last.z) | before_S) + 1), last.w);
  }
  for (int i = tid; i < x1 - x0; i += kThreads) {
    // (places behind the window belong to the last piece)
    bool ends = x0 + i + 1 == x1;
    int row;
    if (x0 + i < w1) {
      const int4 here = spots[x0 + i - w0];
      row = here.x;
      ends = x0 + i + 1 == here.w || ((x0 + i + 1 - here.z) & before_S) == 0;
    } else {
      row = p.places[x0 + i].x;
    }
    rows[i] = ends ? ~row : row;
  }
  __syncthreads();

  // The first rows are on their way while the rows of the result are looked up.  Aligned ones: through a ring in shared memory, of which a
  // thread reads what it has copied itself.
  constexpr int kWords = kEgEach / kRun;                 // 16-byte words of a row that a thread takes
  const uint32_t ring = kVec ? static_cast<uint32_t>(__cvta_generic_to_shared(eg_ring)) + tid * 16 : 0;
  auto copy = [&](int x, int slot) {                     // the row at place x, into a slot of the ring
    if (x < x1) {
      const int row = rows[x - x0];
      const unsigned char* at =
          static_cast<const unsigned char*>(p.grad) + static_cast<long long>(row < 0 ? ~row : row) * p.g_stride * tab_bytes(kType);
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const int h = eg_channel<kRun, kThreads>(slice, i * kRun);
        if (h < p.H)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                       ::"r"(ring + (slot * kWords + i) * kThreads * 16), "l"(at + static_cast<long long>(h) * tab_bytes(kType)) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  constexpr int kStages = eg_stages<kType>();
  if (kVec) {
#pragma unroll 1
    for (int s = 0; s < kStages - 1; ++s) copy(x0 + s, s);
  }
  for (int k = tid; k < w1 - w0; k += kThreads) {
    int row = spots[k].y;
    if (p.by_rows) {
      // the distinct ids ahead of an id's own range, and ahead of it there
      const int2 number = p.numbers[w0 + k];
      row = range_rows[min(number.x, kEgRanges - 1)] + number.y;
#pragma unroll 4
      for (int i = kEgRanges - 1; i < number.x; ++i) row += p.distinct[i];
    }
    out_rows[k] = row;
  }
  __syncthreads();

  float sum[kEgEach] = {};
  // The piece that ends at place x: written, or put with the token's other ones.
  auto finish = [&](int x) {
    const int k = min(x, w1 - 1) - w0, begin = spots[k].z, end = spots[k].w;
    bool whole = true;
    if (end - begin > p.S) {
      const int from = begin + ((x - begin) & ~before_S);
      const long long width = static_cast<long long>(p.slices) * kSlice;
      float* mine = p.partial + (2ll * (from >> p.S_log2) + (from == begin ? 1 : 0)) * width + slice * kSlice + tid;
#pragma unroll
      for (int i = 0; i < kEgEach; ++i) { mine[i * kThreads] = sum[i]; sum[i] = 0.f; }
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        const unsigned n = static_cast<unsigned>((end - begin + before_S) >> p.S_log2);
        last_here = atomicAdd(&p.done[static_cast<long long>(begin >> p.S_log2) * p.slices + slice], 1u) == n - 1 ? 1 : 0;
      }
      __syncthreads();
      whole = last_here != 0;
      __syncthreads();
      if (whole) {
        __threadfence();
#pragma unroll 4
        for (int b = begin; b < end; b += p.S) {
          const float* y = p.partial + (2ll * (b >> p.S_log2) + (b == begin ? 1 : 0)) * width + slice * kSlice + tid;
#pragma unroll
          for (int i = 0; i < kEgEach; ++i) sum[i] = __fadd_rn(sum[i], __ldcg(y + i * kThreads));
        }
      }
    }
    if (!whole) return;
    if (p.by_rows && slice == 0 && tid == 0) p.ids_out[out_rows[k]] = static_cast<int>(spots[k].y + p.v_offset);
    eg_write<kRun, kThreads>(p, out_type, out_rows[k], slice, sum);
#pragma unroll
    for (int i = 0; i < kEgEach; ++i) sum[i] = 0.f;
  };
  if (kVec) {
    int slot = 0, before = kStages - 1;                  // of place x, and of the one before it, which is free
#pragma unroll 1
    for (int x = x0; x < x1; ++x) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
      EgWord<kType> g;
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const uint4 y = *reinterpret_cast<const uint4*>(eg_ring + ((slot * kWords + i) * kThreads + tid) * 16);
        g.w[4 * i] = y.x; g.w[4 * i + 1] = y.y; g.w[4 * i + 2] = y.z; g.w[4 * i + 3] = y.w;
      }
      const bool ends = rows[x - x0] < 0;
      copy(x + kStages - 1, before);
      before = slot;
      slot = slot + 1 == kStages ? 0 : slot + 1;
#pragma unroll
      for (int i = 0; i < kEgEach; ++i) sum[i] = __fadd_rn(sum[i], g.get(i));
      if (ends) finish(x);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
#pragma unroll 1
    for (int x = x0; x < x1; x += kEgAhead) {
      EmWord<kType, 1> g[kEgAhead][kEgEach];
      int row[kEgAhead];
#pragma unroll
      for (int u = 0; u < kEgAhead; ++u) {
        row[u] = x + u < x1 ? rows[x + u - x0] : 0;
        const unsigned char* at =
            static_cast<const unsigned char*>(p.grad) + static_cast<long long>(row[u] < 0 ? ~row[u] : row[u]) * p.g_stride * tab_bytes(kType);
#pragma unroll
        for (int i = 0; i < kEgEach; ++i) {
          const int h = eg_channel<1, kThreads>(slice, i);
          if (x + u < x1 && h < p.H) g[u][i].load(at + static_cast<long long>(h) * tab_bytes(kType));
        }
      }
#pragma unroll
      for (int u = 0; u < kEgAhead; ++u) {
        if (x + u >= x1) break;
#pragma unroll
        for (int i = 0; i < kEgEach; ++i) sum[i] = __fadd_rn(sum[i], g[u][i].get(0));
        if (row[u] < 0) finish(x + u);
      }
    }
  }
}

// Few tokens: all of it in one launch, without a workspace.  Every CTA reads all tokens and finds out, by a table in shared memory, which
// are the first of their id and which ids have more than kEfAlone rows.  A token's row in the result is, by rows, the number of first ones
// with smaller ids.  The other ids: a CTA takes every `groups`-th token, where it is the first of its id, for a share of the slices of 256
// channels; votes say where the id occurs, and a warp adds up its rows in rising r.  Those with many rows are dealt out to all CTAs by 64
// channels; eight lanes take a stretch of the rows, and the stretches are added up in their order.  Bound by latency: launch, tokens,
// table, votes, rows.  us, sorted / so, V = 32000, by rows, fp32: 64 x 4096 9.4 / 3.5, 320 x 4096 9.7 / 6.1, 512 x 4096 10.3 / 8.7, tokens by
// falling frequency 11.8 / 11.4, 512 x 1024 9.6 / 6.3, one id 13.9 / 9.2, 512 x 8192 11.7 / 11.6; beyond 512 tokens the votes and tables
// of all CTAs cost more than a sort (1024 x 4096 11.8 / 14.8).  Whole table, 64 x 4096 80.4 / 73.5.
constexpr int kEfMost = 512;           // tokens
constexpr int kEfThreads = 256, kEfWarps = 8, kEfSlots = 2 * kEfMost;
constexpr int kEfPerSm = 3;            // CTAs
constexpr int kEfAlone = 16;            // rows of an id that a warp adds up by itself
constexpr int kEfLanes = 8, kEfStretches = kEfThreads / kEfLanes;      // of an id with many rows

template <int kType, bool kVec>
__global__ void __launch_bounds__(kEfThreads, kEfPerSm) embed_grad_few_kernel(const __grid_constant__ EgParams p, int out_type, int groups,
                                                                                     int shares) {
  constexpr int kRun = kVec ? kEgEach : 1, kAhead = kType == kTabF32 || !kVec ? 4 : 8, kNone = INT32_MAX, kMine = kEfMost / kEfThreads;
  __shared__ int ids[kEfMost], distinct[kEfMost];        // rows of the table, -1: none; those of the tokens that are the first of their id
  __shared__ int keys[kEfSlots], seen[kEfSlots], times[kEfSlots];      // ids, the first tokens that have them, how many do
  __shared__ unsigned many[kEfMost / 32];                // bits: first tokens of ids with many rows
  __shared__ unsigned short list[kEfMost];               // rows of the ids that this CTA adds up
  __shared__ int at_of[kEfMost], row_of[kEfMost];        // the CTA's ids: places in the list, rows of the result
  __shared__ int n_of[kEfMost];                          // rows of the ids of the tokens that are their first
  __shared__ float part[kEfStretches][kEfLanes * kEgEach];
  __shared__ int used;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  grid_dependency_wait();
  grid_dependency_release();
  if (blockIdx.x >= static_cast<unsigned>(groups * shares)) {
    // The whole table: zeros to the rows of ids that do not occur, rows without a gap between them as one stretch.
    const int v0 = (static_cast<int>(blockIdx.x) - groups * shares) * p.blank, n = min(p.blank, p.V - v0);
    if (tid < n) n_of[tid] = 0;
    __syncthreads();
    for (int i = tid; i < p.N; i += kEfThreads) {
      bool bad;
      const int v = em_row(p.tokens, p.wide, i, p.V, p.v_offset, p.V_global, &bad);
      if (v >= v0 && v < v0 + n) n_of[v - v0] = 1;
    }
    __syncthreads();
    const int size = tab_bytes(out_type);
    unsigned char* out = static_cast<unsigned char*>(p.out);
    for (int i = 0; i < n; ++i) {
      if (n_of[i]) continue;
      int last = i;
      while (p.out_stride == p.H && last + 1 < n && !n_of[last + 1]) ++last;
      eg_zeros<kEfThreads>(out + (v0 + i) * p.out_stride * size, out + ((v0 + last) * p.out_stride + p.H) * size, size);
      i = last;
    }
    return;
  }
  const int group = static_cast<int>(blockIdx.x) / shares, share = static_cast<int>(blockIdx.x) - group * shares;
  const int slices = (p.slices + shares - 1) / shares, s0 = share * slices, s1 = min(s0 + slices, p.slices);
  int id_of[kMine], slot[kMine];
  bool bad_here = false;
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int i = tid + k * kEfThreads;
    bool bad = false;
    id_of[k] = i < p.N ? em_row(p.tokens, p.wide, i, p.V, p.v_offset, p.V_global, &bad) : -1;
    ids[i] = id_of[k];
    bad_here = bad_here || bad;
  }
  if (blockIdx.x == 0 && bad_here && p.status) atomicOr(p.status, HOLA_FLAG_BAD_TOKEN);
  if (tid == 0) used = 0;
  for (int i = tid; i < kEfSlots; i += kEfThreads) { keys[i] = -1; seen[i] = kNone; times[i] = 0; }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int id = id_of[k];
    slot[k] = static_cast<int>((static_cast<uint32_t>(id) * 2654435761u) / (0x100000000ull / kEfSlots));
    if (id < 0) continue;
    for (int had = atomicCAS(&keys[slot[k]], -1, id); had != -1 && had != id; had = atomicCAS(&keys[slot[k]], -1, id))
      slot[k] = (slot[k] + 1) & (kEfSlots - 1);          // (half of the places stay free)
    atomicMin(&seen[slot[k]], tid + k * kEfThreads);
    atomicAdd(&times[slot[k]], 1);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int i = tid + k * kEfThreads;
    const bool first = id_of[k] >= 0 && seen[slot[k]] == i;
    distinct[i] = first ? id_of[k] : kNone;
    n_of[i] = first ? times[slot[k]] : 0;
    const unsigned bits = __ballot_sync(0xffffffffu, first && times[slot[k]] > kEfAlone);
    if (lane == 0) many[i >> 5] = bits;
  }
  __syncthreads();

  // For a whole warp: the row of the result of the id of token i; its rows to the list from `at` on (-1: not).
  auto find = [&](int id, int at) {
    unsigned mask = 0;                                   // lane w: of tokens 32 w .. 32 w + 31
    int smaller = 0;
    for (int w = 0; w * 32 < p.N; ++w) {
      const unsigned same = __ballot_sync(0xffffffffu, ids[w * 32 + lane] == id);
      if (lane == w) mask = same;
      smaller += distinct[w * 32 + lane] < id ? 1 : 0;
    }
    if (at >= 0) {
      const int here = __popc(mask);
      int upto = here;
#pragma unroll
      for (int o = 1; o < kEfMost / 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
      }
      for (int to = at + upto - here; mask; mask &= mask - 1u) list[to++] = static_cast<unsigned short>(lane * 32 + __ffs(mask) - 1);
    }
    return p.by_rows ? __reduce_add_sync(0xffffffffu, smaller) : id;
  };
  // A thread's eight channels of some rows of the list, `lanes` threads to a row, summed.
  float sum[kEgEach];
  auto add_up = [&](auto lanes, int slice, int thread, int from, int to) {
#pragma unroll
    for (int c = 0; c < kEgEach; ++c) sum[c] = 0.f;
#pragma unroll 1
    for (int x = from; x < to; x += kAhead) {
      EmWord<kType, kRun> g[kAhead][kEgEach / kRun];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (x + u >= to) break;
        const unsigned char* at = static_cast<const unsigned char*>(p.grad) + list[x + u] * p.g_stride * tab_bytes(kType);
#pragma unroll
        for (int i = 0; i < kEgEach / kRun; ++i) {
          const int h = eg_channel<kRun, decltype(lanes)::value>(slice, i * kRun, thread);
          if (h < p.H) g[u][i].load(at + static_cast<long long>(h) * tab_bytes(kType));
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (x + u >= to) break;
#pragma unroll
        for (int c = 0; c < kEgEach; ++c) sum[c] = __fadd_rn(sum[c], g[u][c / kRun].get(c % kRun));
      }
    }
  };

  // Ids with many rows.
  int items = 0, word = 0, passed = 0;
  for (int w = 0; w < kEfMost / 32; ++w) items += __popc(many[w]);
  const int cuts = (p.H + kEfLanes * kEgEach - 1) / (kEfLanes * kEgEach);
  int found = -1, n = 0, row = 0;
  for (long long item = blockIdx.x; item < static_cast<long long>(items) * cuts; item += groups * shares) {
    const int which = static_cast<int>(item / cuts), cut = static_cast<int>(item - static_cast<long long>(which) * cuts);
    if (which != found) {
      for (; passed + __popc(many[word]) <= which; ++word) passed += __popc(many[word]);
      unsigned bits = many[word];
      for (int i = passed; i < which; ++i) bits &= bits - 1u;
      const int i = word * 32 + __ffs(bits) - 1;
      found = which;
      n = n_of[i];
      __syncthreads();                                   // (the list before it has been read)
      row = find(ids[i], warp == 0 ? 0 : -1);
      __syncthreads();
    }
    const int stretch = tid / kEfLanes, thread = tid % kEfLanes, each = (n + kEfStretches - 1) / kEfStretches;
    add_up(std::integral_constant<int, kEfLanes>(), cut, thread, min(stretch * each, n), min((stretch + 1) * each, n));
#pragma unroll
    for (int c = 0; c < kEgEach; ++c) part[stretch][c * kEfLanes + thread] = sum[c];
    __syncthreads();
    if (tid < kEfLanes * kEgEach) {
      float x = part[0][tid];
#pragma unroll
      for (int q = 1; q < kEfStretches; ++q) x = __fadd_rn(x, part[q][tid]);
      part[0][tid] = x;
    }
    __syncthreads();
    if (tid < kEfLanes) {
#pragma unroll
      for (int c = 0; c < kEgEach; ++c) sum[c] = part[0][c * kEfLanes + tid];
      eg_write<kRun, kEfLanes>(p, out_type, row, cut, sum, tid);
    }
    __syncthreads();
  }

  // The CTA's other ids; whose row of the result holds which id.
  const int mine = group < p.N ? (p.N - 1 - group) / groups + 1 : 0;
  for (int k = warp; k < mine; k += kEfWarps) {
    const int i = group + k * groups, id = ids[i], rows = n_of[i];
    if (rows == 0) continue;
    const bool here = rows <= kEfAlone;
    if (!here && (!p.by_rows || share != 0)) continue;
    int at = -1;
    if (here) {
      if (lane == 0) at = atomicAdd(&used, rows);
      at = __shfl_sync(0xffffffffu, at, 0);
    }
    const int to = find(id, at);
    if (p.by_rows && share == 0 && lane == 0) p.ids_out[to] = static_cast<int>(id + p.v_offset);
    if (lane == 0) { at_of[k] = at; row_of[k] = to; }
  }
  __syncthreads();
  // (a slice at a time to a warp, so that the slices of an id with several rows lie with several warps)
  const int pieces = mine * (s1 - s0);
  for (int x = warp; x < pieces; x += kEfWarps) {
    const int k = x / (s1 - s0), s = s0 + (x - k * (s1 - s0)), rows = n_of[group + k * groups];
    if (rows == 0 || rows > kEfAlone) continue;
    add_up(std::integral_constant<int, 32>(), s, lane, at_of[k], at_of[k] + rows);
    eg_write<kRun, 32>(p, out_type, row_of[k], s, sum, lane);
  }
  if (blockIdx.x == 0 && p.by_rows && warp == kEfWarps - 1) {
    int count = 0;
    for (int i = lane; i < kEfMost; i += 32) count += distinct[i] != kNone ? 1 : 0;
    count = __reduce_add_sync(0xffffffffu, count);
    if (lane == 0) *p.count_out = count;
  }
}

struct EgLayout {
  size_t places, numbers, first, distinct, valid, done, partial, total;
  size_t enough;                       // for as many tokens and for any smaller number
};

// Host: the cut of the work.  False: sizes that are not served.
bool eg_plan(long long N, int V, int H, EgParams* p, EgLayout* l) {
  if (N < 0 || N > kEgMaxTokens || V <= 0 || H <= 0 || V > 1 << 30 || H > INT32_MAX - 4096) return false;
  p->N = static_cast<int>(N); p->V = V; p->H = H;
  p->few = N <= kEfMost;
  if (p->few) {
    *l = {};
    l->total = l->enough = 256;
    p->slices = (H + 32 * kEgEach - 1) / (32 * kEgEach);
    p->blank = kEgMaxWindow;
    while (p->blank > 1 && V / p->blank < 16 * kEgPlanSms) p->blank >>= 1;
    return true;
  }
  int warps = N > 2 * kEfMost ? kEsWarps : kEsWarps / 2;
  // Ranges: one per SM where their counters fit, else as many as it takes.  (A thread adds up two ids.)
  const int cell = N <= UINT16_MAX ? 2 : 4, most = (1 << kEsIdBits) - 2;
  int ids = (V + kEgPlanSms - kEsZipf) / (kEgPlanSms - kEsZipf + 1);
  if (ids > most) ids = most;
  // (rather fewer warps than a second round of CTAs)
  while (warps > kEsWarps / 2 && EsLayout(ids, warps, kEsList, cell).total > kEsMaxShared) warps -= 4;
  while (EsLayout(ids, warps, kEsList, cell).total > kEsMaxShared) --ids;
  const int room = (kEsMaxShared - EsLayout(ids, warps, 0, cell).total) / (4 * warps) / 32 * 32;
  p->list = room < kEsMaxList ? room : kEsMaxList;
  p->warps = warps;
  p->chunk = static_cast<int>(((N + warps - 1) / warps + 31) / 32 * 32);
  p->R = ids;
  p->even = (V + ids - 1) / ids;
  p->buckets = p->even + kEsZipf - 1;
  int S = 32;                                            // (some 512 pieces, where one token is all there is)
  while (S < kEgMaxPiece && N > 512ll * S) S <<= 1;
  p->S = S;
  p->S_log2 = 0;
  while (1 << p->S_log2 < S) ++p->S_log2;
  const int slice = (H <= kEgFewThreads * kEgEach ? kEgFewThreads : kEgThreads) * kEgEach;
  p->slices = (H + slice - 1) / slice;
  p->blank = kEgMaxWindow;
  while (p->blank > 1 && static_cast<long long>(V) / p->blank * p->slices < 16ll * kEgPlanSms) p->blank >>= 1;
  int window = kEgMaxWindow;
  while (window > 4 && (N + window - 1) / window * p->slices < 16ll * kEgPlanSms) window >>= 1;
  p->window = window;
  const size_t pieces = static_cast<size_t>((N + S - 1) / S);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
  l->places = take(static_cast<size_t>(N) * 16);
  l->numbers = take(static_cast<size_t>(N) * 8);
  l->first = take((static_cast<size_t>(V) + 1) * 4);
  l->distinct = take(static_cast<size_t>(p->buckets) * 4);
  l->valid = take(4);
  const size_t lists = at;
  auto sums = [&](size_t n) {                            // what n pieces need, behind the lists
    at = lists;
    l->done = take(n * p->slices * 4);
    l->partial = take(2 * n * p->slices * slice * 4);
    return at;
  };
  // (pieces double in length where there would be more than 512, so that fewer tokens may have more of them; the lists only grow)
  const size_t by_32 = static_cast<size_t>((N + 31) / 32);
  l->enough = sums(by_32 < 512 ? by_32 : pieces < 512 ? 512 : pieces);
  l->total = sums(pieces);
  return true;
}

template <int kType>
cudaError_t launch_embed_grad_few(const EgParams& p, int out_type, bool vec, cudaStream_t stream) {
  // (a token for every warp, and as many CTAs as there is room for: a share of the slices to each)
  constexpr int kRoom = kEfPerSm * kEgPlanSms;
  const int groups = p.N > kEfWarps ? (p.N + kEfWarps - 1) / kEfWarps : 1;
  const int shares = kRoom / groups < p.slices ? kRoom / groups : p.slices;
  const long long blank = p.by_rows || p.accumulate ? 0 : (static_cast<long long>(p.V) + p.blank - 1) / p.blank;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.attrs = attr; cfg.numAttrs = 1; cfg.stream = stream;
  cfg.gridDim = dim3(static_cast<unsigned>(static_cast<long long>(groups) * shares + blank)); cfg.blockDim = dim3(kEfThreads);
  return vec ? cudaLaunchKernelEx(&cfg, embed_grad_few_kernel<kType, true>, p, out_type, groups, shares)
             : cudaLaunchKernelEx(&cfg, embed_grad_few_kernel<kType, false>, p, out_type, groups, shares);
}

template <int kType>
cudaError_t launch_embed_grad(const EgParams& p, int out_type, bool vec, cudaStream_t stream) {
  if (p.few) return launch_embed_grad_few<kType>(p, out_type, vec, stream);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.attrs = attr; cfg.numAttrs = 1; cfg.stream = stream;
  cfg.gridDim = dim3(static_cast<unsigned>(p.buckets)); cfg.blockDim = dim3(kEsThreads);
  cfg.dynamicSmemBytes = static_cast<size_t>(EsLayout(p.R, p.warps, p.list, p.N <= UINT16_MAX ? 2 : 4).total);
  const bool few_tokens = p.N <= UINT16_MAX;
  cudaError_t e;
  if (p.wide)
    e = few_tokens ? cudaLaunchKernelEx(&cfg, embed_sort_kernel<uint16_t, int64_t>, p)
                   : cudaLaunchKernelEx(&cfg, embed_sort_kernel<uint32_t, int64_t>, p);
  else
    e = few_tokens ? cudaLaunchKernelEx(&cfg, embed_sort_kernel<uint16_t, int32_t>, p)
                   : cudaLaunchKernelEx(&cfg, embed_sort_kernel<uint32_t, int32_t>, p);
  if (e != cudaSuccess) return e;
  const long long windows = (p.N + p.window - 1) / p.window;
  const long long blank = p.first ? (static_cast<long long>(p.V) + p.blank - 1) / p.blank : 0;
  const bool few = p.H <= kEgFewThreads * kEgEach;
  cfg.gridDim = dim3(static_cast<unsigned>((windows + blank) * p.slices)); cfg.blockDim = dim3(few ? kEgFewThreads : kEgThreads);
  cfg.dynamicSmemBytes = 0;
  const int n = static_cast<int>(windows);
  if (few)
    return vec ? cudaLaunchKernelEx(&cfg, embed_grad_kernel<kType, true, kEgFewThreads>, p, out_type, n)
               : cudaLaunchKernelEx(&cfg, embed_grad_kernel<kType, false, kEgFewThreads>, p, out_type, n);
  return vec ? cudaLaunchKernelEx(&cfg, embed_grad_kernel<kType, true, kEgThreads>, p, out_type, n)
             : cudaLaunchKernelEx(&cfg, embed_grad_kernel<kType, false, kEgThreads>, p, out_type, n);
}

template <typename Cell>
cudaError_t configure_sort() {
  const cudaError_t e = cudaFuncSetAttribute(embed_sort_kernel<Cell, int32_t>, cudaFuncAttributeMaxDynamicSharedMemorySize, kEsMaxShared);
  return e != cudaSuccess ? e : cudaFuncSetAttribute(embed_sort_kernel<Cell, int64_t>, cudaFuncAttributeMaxDynamicSharedMemorySize, kEsMaxShared);
}
// What the sums have on the way is in shared memory, as many CTAs of it as there is room for; where rows start anywhere, in the L1, which
// the sort has left next to nothing of (16384 aligned rows that way: 81.4 us, 70.6 with room for them).
template <int kType, int kThreads>
cudaError_t configure_sums_of() {
  const cudaError_t e = cudaFuncSetAttribute(embed_grad_kernel<kType, true, kThreads>, cudaFuncAttributePreferredSharedMemoryCarveout, 100);
  return e != cudaSuccess ? e : cudaFuncSetAttribute(embed_grad_kernel<kType, false, kThreads>, cudaFuncAttributePreferredSharedMemoryCarveout, 25);
}
template <int kType>
cudaError_t configure_sums() {
  const cudaError_t e = configure_sums_of<kType, kEgThreads>();
  return e != cudaSuccess ? e : configure_sums_of<kType, kEgFewThreads>();
}
cudaError_t configure_embedding() {
  cudaError_t e = configure_sort<uint16_t>();
  if (e == cudaSuccess) e = configure_sort<uint32_t>();
  if (e == cudaSuccess) e = configure_sums<kTabF32>();
  if (e == cudaSuccess) e = configure_sums<kTabBf16>();
  return e == cudaSuccess ? configure_sums<kTabF16>() : e;
}
