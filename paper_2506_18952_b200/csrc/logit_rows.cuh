// logit_rows.cuh - rows of logits in memory as groups of 32 bytes, and the order of their entries (inside the anonymous namespaces of
// hola_verify.cu and decode_ops.cu).

constexpr int kLpGroupBytes = 32;      // neighbouring entries that a thread loads at once

// Floats in the order of their values as unsigned whole numbers (one zero; NaN does not occur).
__device__ __forceinline__ uint32_t lp_order(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float lp_value(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ uint64_t lp_key(float x, int at) {
  return static_cast<uint64_t>(lp_order(x)) << 32 | static_cast<uint32_t>(~at);
}

// A group of neighbouring logits as loaded.
template <typename T>
struct LpGroup {
  static constexpr int kEntries = kLpGroupBytes / sizeof(T);
  uint32_t w[8];
  __device__ __forceinline__ void load(const T* p) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
  }
  // Entries 2 i and 2 i + 1.
  __device__ __forceinline__ void pair(int i, float& lo, float& hi) const {
    if (sizeof(T) == 4) {
      lo = __uint_as_float(w[(2 * i) & 7]); hi = __uint_as_float(w[(2 * i + 1) & 7]);
    } else if (std::is_same<T, __nv_bfloat16>::value) {
      lo = __uint_as_float(w[i & 7] << 16); hi = __uint_as_float(w[i & 7] & 0xffff0000u);
    } else {
      const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&w[i & 7]));
      lo = y.x; hi = y.y;
    }
  }
  __device__ __forceinline__ float entry(int i) const {
    float lo, hi;
    pair(i >> 1, lo, hi);
    return i & 1 ? hi : lo;
  }
  __device__ __forceinline__ float largest() const {     // NaN where there is one
    if (sizeof(T) == 4) {
      const float* f = reinterpret_cast<const float*>(w);
      return max3_nan(max3_nan(f[0], f[1], f[2]), max3_nan(f[3], f[4], f[5]), max3_nan(f[6], f[7], f[7]));
    }
    uint32_t m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = w[i];
#pragma unroll
    for (int n = 4; n > 0; n >>= 1)
#pragma unroll
      for (int i = 0; i < n; ++i) {
        if (std::is_same<T, __nv_bfloat16>::value) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m[i]) : "r"(m[i + n]));
        else asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(m[i]) : "r"(m[i + n]));
      }
    LpGroup<T> g;
    g.w[0] = m[0];
    float lo, hi;
    g.pair(0, lo, hi);
    return max3_nan(lo, hi, hi);
  }
};

// A row as groups that start on 32-byte boundaries: with E entries in one, group j holds entries E j - off ... E j - off + E - 1, the
// first and the last one perhaps fewer (what they lack reads as -inf).
template <typename T>
struct LpRow {
  static constexpr int E = LpGroup<T>::kEntries;
  const T* base;               // entry -off, on a 32-byte boundary (not read before entry 0)
  int off, V, groups;          // groups whole_begin .. whole_end - 1 are whole
  int whole_begin, whole_end;
  __device__ __forceinline__ LpRow(const T* row, int V_) : V(V_) {
    off = static_cast<int>((reinterpret_cast<uintptr_t>(row) & (kLpGroupBytes - 1u)) / sizeof(T));
    base = row - off;
    groups = static_cast<int>((static_cast<long long>(V_) + off + E - 1) / E);
    whole_begin = off ? 1 : 0;
    whole_end = static_cast<int>((static_cast<long long>(V_) + off) / E);
  }
  __device__ __forceinline__ bool whole(int j) const { return j >= whole_begin && j < whole_end; }
  __device__ __forceinline__ int first(int j) const { return j * E - off; }
  static __device__ __forceinline__ uint32_t none_bits() {        // -inf
    return sizeof(T) == 4 ? 0xff800000u : std::is_same<T, __nv_bfloat16>::value ? 0xff80u : 0xfc00u;
  }
  static __device__ __forceinline__ LpGroup<T> none() {
    LpGroup<T> g;
#pragma unroll
    for (int i = 0; i < 8; ++i) g.w[i] = sizeof(T) == 4 ? none_bits() : none_bits() * 0x10001u;
    return g;
  }
  __device__ __forceinline__ LpGroup<T> get(int j) const {
    if (!whole(j)) return get_ragged(j);
    LpGroup<T> g;
    g.load(base + static_cast<size_t>(j) * E);
    return g;
  }
  __device__ __noinline__ LpGroup<T> get_ragged(int j) const {
    LpGroup<T> g;
    const uint32_t none = none_bits();
#pragma unroll
    for (int i = 0; i < 8; ++i) g.w[i] = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const long long v = static_cast<long long>(j) * E - off + i;
      uint32_t bits = none;
      if (v >= 0 && v < V) {
        if (sizeof(T) == 4) bits = reinterpret_cast<const uint32_t*>(base)[v + off];
        else bits = reinterpret_cast<const uint16_t*>(base)[v + off];
      }
      if (sizeof(T) == 4) g.w[i & 7] = bits;
      else g.w[(i >> 1) & 7] |= bits << (16 * (i & 1));
    }
    return g;
  }
};
