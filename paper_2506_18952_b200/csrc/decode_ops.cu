// decode_ops.cu - sm_100a kernels and C ABI for what stands around the LM head in a decoder: a beam search's step, token embeddings and
// their gradient.  See include/hola_verify.h for the contract.
//
// Kernels
//   beam_select_kernel, beam_reorder_kernel  (beams.cuh) the best continuations of all beams of a sequence, and the beams' states in the
//       order of their parents.
//   embed_kernel                (embedding.cuh) rows of a table, the head's own storage forms among them, by token; embed_sort_kernel,
//       embed_grad_kernel, the gradient of a table by sorted tokens.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include <cooperative_groups.h>

#include <atomic>
#include <initializer_list>
#include <mutex>
#include <type_traits>

#include "../../include/hola_verify.h"

namespace cg = cooperative_groups;

namespace {

#include "device_util.cuh"
#include "logit_rows.cuh"
#include "beams.cuh"
#include "embedding.cuh"

// Whether any of these lies on no address of 32-bit words.
bool off_words(std::initializer_list<const void*> of) {
  uintptr_t all = 0;
  for (const void* x : of) all |= reinterpret_cast<uintptr_t>(x);
  return all % 4 != 0;
}

// ------------------------------------------------------------------------------------------------ bytes that operands share
// Bytes of an operand: runs that start at every index of some axes, by falling stride.
struct Bytes {
  static constexpr int kAxes = 4;
  uintptr_t at;                        // 0: no bytes
  int axes = 0;
  long long size[kAxes], stride[kAxes];
  long long extent[kAxes + 1];         // from the first byte to behind the last one of what the axes from here on span
  struct Axis { long long size, apart; };
  Bytes(const void* base, long long run) : Bytes(base, run, nullptr, 0) {}
  template <int n>
  Bytes(const void* base, long long run, const Axis (&along)[n]) : Bytes(base, run, along, n) { static_assert(n <= kAxes, "axes"); }

 private:
  Bytes(const void* base, long long run, const Axis* along, int n) : at(run > 0 ? reinterpret_cast<uintptr_t>(base) : 0) {
    for (int k = 0; k < n; ++k) {
      if (along[k].size <= 0) at = 0;
      if (along[k].size <= 1) continue;
      int i = axes++;
      for (; i > 0 && stride[i - 1] < along[k].apart; --i) { size[i] = size[i - 1]; stride[i] = stride[i - 1]; }
      size[i] = along[k].size;
      stride[i] = along[k].apart;
    }
    extent[axes] = run;
    for (int i = axes; i > 0; --i) extent[i - 1] = extent[i] + (size[i - 1] - 1) * stride[i - 1];
  }
};

// Whether a, from axis i on, and b, from axis j on, which begins d bytes behind it, share a byte: the longest stride left is taken first, of which
// only indices matter whose spans meet (one or two, where strides are larger than what they step over).  Layouts for which
// more than a few thousand pairs would have to be looked at count as if they did.
bool meet(const Bytes& a, int i, const Bytes& b, int j, long long d, int* looks) {
  if (d >= a.extent[i] || d <= -b.extent[j]) return false;
  if (i == a.axes && j == b.axes) return true;
  if (++*looks > 4096) return true;
  const long long s = i < a.axes ? a.stride[i] : -1, t = j < b.axes ? b.stride[j] : -1, step = s > t ? s : t;
  if (step == 0) return meet(a, a.axes, b, b.axes, d, looks);
  // (places of b behind those of a, in steps)
  long long first = s == step ? -(a.size[i] - 1) : 0, last = t == step ? b.size[j] - 1 : 0;
  if (s == step) ++i;
  if (t == step) ++j;
  auto down = [](long long x, long long y) { return x >= 0 ? x / y : -((y - 1 - x) / y); };
  const long long from = down(-b.extent[j] - d, step) + 1, to = down(a.extent[i] - 1 - d, step);
  for (long long k = first > from ? first : from; k <= (last < to ? last : to); ++k)
    if (meet(a, i, b, j, d + k * step, looks)) return true;
  return false;
}
bool share(const Bytes& a, const Bytes& b) {
  const long long d = static_cast<long long>(b.at - a.at);
  if (!a.at || !b.at || d >= a.extent[0] || d <= -b.extent[0]) return false;
  int looks = 0;
  return meet(a, 0, b, 0, d, &looks);
}

// The same of operands without axes.
inline bool share(const void* a, long long a_bytes, const void* b, long long b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + static_cast<uintptr_t>(b_bytes) && y < x + static_cast<uintptr_t>(a_bytes);
}

// Whether two indices of a's axes from i on have a byte in common.
bool shares_with_itself(const Bytes& a) {
  int looks = 0;
  for (int i = 0; i < a.axes; ++i)
    for (long long k = 1; k < a.size[i] && k * a.stride[i] < a.extent[i + 1]; ++k)       // (nothing to do where strides are larger than what they step over)
      if (meet(a, i + 1, a, i + 1, k * a.stride[i], &looks)) return true;
  return false;
}

}  // namespace

extern "C" {

// What the launches need to know of a device, asked for once (the first call on a device also tells the runtime how much shared memory
// the kernels use, which the calls behind it need not say again).
struct DeviceFacts {
  int sms;
  int fit[kBsMaxCluster + 1];          // see bs_cluster
};
// The current device's; null: no device that runs these kernels.
static const DeviceFacts* device_facts() {
  constexpr int kDevices = 64;
  static DeviceFacts facts[kDevices];
  static std::atomic<bool> known[kDevices];
  static std::mutex first;
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return nullptr;
  if (known[dev].load(std::memory_order_acquire)) return &facts[dev];
  std::lock_guard<std::mutex> lock(first);
  if (known[dev].load(std::memory_order_acquire)) return &facts[dev];
  DeviceFacts f = {};
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&f.sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || major != 10 || f.sms <= 0)
    return nullptr;
  if (configure_beams(f.fit) != cudaSuccess || configure_embedding() != cudaSuccess) return nullptr;
  facts[dev] = f;
  known[dev].store(true, std::memory_order_release);
  return &facts[dev];
}

hola_status hola_beam_select(const hola_beam_args* a, void* cuda_stream) {
  if (!a || a->B < 0 || a->W <= 0 || a->V <= 0 || a->n <= 0 || a->seq_stride < 0 || a->beam_stride < 0) return HOLA_ERR_INVALID_ARG;
  if (a->l_dtype < HOLA_L_F32 || a->l_dtype > HOLA_L_F16) return HOLA_ERR_INVALID_ARG;
  if (a->W > kBsMaxBeams || a->n > kBsMaxKept || a->V > kBsMaxV || a->B > INT32_MAX / kBsMaxCluster) return HOLA_ERR_UNSUPPORTED_SHAPE;
  if (a->keep_slots && a->n != a->W) return HOLA_ERR_INVALID_ARG;
  if (a->end_token < -1 || a->end_token >= a->V || (a->finished && a->end_token < 0)) return HOLA_ERR_INVALID_ARG;
  if (a->B == 0) return HOLA_OK;
  if (!a->logits || !a->logZ || !a->score || !a->score_out || !a->parent || !a->token) return HOLA_ERR_INVALID_ARG;
  const int entry = a->l_dtype == HOLA_L_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(a->logits) % entry || off_words({a->logZ, a->score, a->weight, a->score_out, a->parent, a->token, a->status_word}))
    return HOLA_ERR_INVALID_ARG;
  // A sequence is written when all of it has been read; another one's beams may lie where its candidates go, but for the same layout.
  const long long beams = static_cast<long long>(a->B) * a->W, kept = static_cast<long long>(a->B) * a->n;
  const struct { const void* at; int bytes; } in[] = {{a->score, 4}, {a->logZ, 4}, {a->weight, 4}, {a->finished, 1}},
                                              out[] = {{a->score_out, 4}, {a->finished_out, 1}, {a->parent, 4}, {a->token, 4}};
  for (const auto& x : in)
    for (const auto& y : out) {
      const bool itself = a->n == a->W && x.at == y.at && ((x.at == a->score && y.at == a->score_out) || (x.at == a->finished && y.at == a->finished_out));
      if (!itself && share(x.at, beams * x.bytes, y.at, kept * y.bytes)) return HOLA_ERR_INVALID_ARG;
    }
  const Bytes rows(a->logits, static_cast<long long>(a->V) * entry, {{a->B, a->seq_stride * entry}, {a->W, a->beam_stride * entry}});
  for (int i = 0; i < 4; ++i)
    if (share({out[i].at, kept * out[i].bytes}, rows)) return HOLA_ERR_INVALID_ARG;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < i; ++j)
      if (share(out[i].at, kept * out[i].bytes, out[j].at, kept * out[j].bytes)) return HOLA_ERR_INVALID_ARG;
  const DeviceFacts* dev = device_facts();
  if (!dev) return HOLA_ERR_NO_DEVICE;
  BsParams p = {};
  p.logits = a->logits; p.seq_stride = a->seq_stride; p.beam_stride = a->beam_stride; p.B = a->B; p.W = a->W; p.V = a->V; p.n = a->n;
  p.logZ = a->logZ; p.score = a->score; p.finished = a->finished; p.weight = a->weight; p.end_token = a->end_token;
  p.keep_slots = a->keep_slots; p.score_out = a->score_out; p.parent = a->parent; p.token = a->token; p.finished_out = a->finished_out;
  p.status = a->status_word;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = a->l_dtype == HOLA_L_F32 ? launch_beam_select<float>(p, dev->fit, stream)
                        : a->l_dtype == HOLA_L_BF16 ? launch_beam_select<__nv_bfloat16>(p, dev->fit, stream) : launch_beam_select<__half>(p, dev->fit, stream);
  return e == cudaSuccess ? HOLA_OK : HOLA_ERR_CUDA;
}

// What is read of a state, and what is written (in place: the same).
static Bytes state_read(const hola_reorder_args* a, const hola_beam_state& s) {
  return {s.src, s.run, {{a->B, s.seq_stride}, {a->W, s.beam_stride}, {s.outer[0], s.outer_stride[0]}, {s.outer[1], s.outer_stride[1]}}};
}
static Bytes state_written(const hola_reorder_args* a, const hola_beam_state& s) {
  return {s.dst, s.run, {{a->B, s.dst_seq_stride}, {s.src == s.dst ? a->W : a->n, s.dst_beam_stride}, {s.outer[0], s.dst_outer_stride[0]},
                         {s.outer[1], s.dst_outer_stride[1]}}};
}

// Every state by itself, and beside what a call reads.  in_place: -1 where there is nothing to move.
static hola_status look_at_states(const hola_reorder_args* a, bool call, int* in_place) {
  *in_place = -1;
  if (!a || a->B < 0 || a->W <= 0 || a->n <= 0 || a->count < 0 || (call && a->parent_stride < 0)) return HOLA_ERR_INVALID_ARG;
  if (a->W > kBsMaxBeams || a->n > kBsMaxBeams) return HOLA_ERR_UNSUPPORTED_SHAPE;
  if (a->B == 0 || a->count == 0) return HOLA_OK;
  if (!a->states || (call && (!a->parent || off_words({a->parent, a->used, a->status_word})))) return HOLA_ERR_INVALID_ARG;
  const Bytes parent(call ? a->parent : nullptr, a->n * 4ll, {{a->B, a->parent_stride * 4}}), used(call ? a->used : nullptr, a->B * 4ll);
  for (int i = 0; i < a->count; ++i) {
    const hola_beam_state& s = a->states[i];
    if (s.run < 0 || s.position < 0 || s.outer[0] < 0 || s.outer[1] < 0) return HOLA_ERR_INVALID_ARG;
    if (s.run == 0 || s.outer[0] == 0 || s.outer[1] == 0) continue;
    if (!s.src || !s.dst || s.seq_stride < 0 || s.beam_stride < 0 || s.outer_stride[0] < 0 || s.outer_stride[1] < 0 || s.dst_seq_stride < 0 ||
        s.dst_beam_stride < 0 || s.dst_outer_stride[0] < 0 || s.dst_outer_stride[1] < 0)
      return HOLA_ERR_INVALID_ARG;
    const bool here = s.src == s.dst;
    if (*in_place >= 0 && *in_place != static_cast<int>(here)) return HOLA_ERR_INVALID_ARG;
    *in_place = here;
    if (here && (a->n > a->W || s.seq_stride != s.dst_seq_stride || s.beam_stride != s.dst_beam_stride ||
                 s.outer_stride[0] != s.dst_outer_stride[0] || s.outer_stride[1] != s.dst_outer_stride[1]))
      return HOLA_ERR_INVALID_ARG;
    if ((a->n > 1 && s.dst_beam_stride < s.run) || (a->W > 1 && s.beam_stride < s.run)) return HOLA_ERR_INVALID_ARG;      // beams that share bytes
    const long long pieces = (s.run - 1) / br_piece(s) + 1;
    if (pieces > INT32_MAX || s.outer[0] > INT32_MAX || s.outer[1] > INT32_MAX) return HOLA_ERR_UNSUPPORTED_SHAPE;
    const double ctas = static_cast<double>(pieces) * a->B * static_cast<double>(s.outer[0]) * static_cast<double>(s.outer[1]);
    if (ctas > INT32_MAX) return HOLA_ERR_UNSUPPORTED_SHAPE;
    const Bytes to = state_written(a, s);
    if (shares_with_itself(to) || (!here && share(state_read(a, s), to)) || share(parent, to) || share(used, to)) return HOLA_ERR_INVALID_ARG;
  }
  return HOLA_OK;
}

hola_status hola_beam_states_check(const hola_reorder_args* a) {
  int in_place;
  const hola_status status = look_at_states(a, false, &in_place);
  if (status != HOLA_OK || in_place < 0) return status;
  for (int i = 0; i < a->count; ++i) {
    const Bytes to = state_written(a, a->states[i]);
    for (int j = 0; j < a->count; ++j)
      if ((j < i && share(state_written(a, a->states[j]), to)) || (j != i && !in_place && share(state_read(a, a->states[j]), to)))
        return HOLA_ERR_INVALID_ARG;
  }
  return HOLA_OK;
}

hola_status hola_beam_reorder(const hola_reorder_args* a, void* cuda_stream) {
  // (all states are looked at before the first launch)
  int in_place;
  const hola_status status = look_at_states(a, true, &in_place);
  if (status != HOLA_OK || in_place < 0) return status;
  const DeviceFacts* dev = device_facts();
  if (!dev) return HOLA_ERR_NO_DEVICE;
  const int sms = dev->sms;
  BrParams p = {};
  p.B = a->B; p.W = a->W; p.n = a->n; p.parent = a->parent; p.parent_stride = a->parent_stride; p.used = a->used; p.status = a->status_word;
  p.in_place = in_place;
  long long ctas = 0;
  for (int i = 0; i <= a->count; ++i) {
    long long more = 0, pieces = 0;
    const hola_beam_state* s = i < a->count ? &a->states[i] : nullptr;
    if (s) {
      if (s->run == 0 || s->outer[0] == 0 || s->outer[1] == 0) continue;
      pieces = (s->run - 1) / br_piece(*s) + 1;
      more = pieces * a->B * s->outer[0] * s->outer[1];
    }
    if (p.count > 0 && (!s || p.count == kBrStates || ctas + more > INT32_MAX)) {
      // (parents one after the other take a microsecond each: shared out where there are CTAs to spare)
      for (p.split = 1; p.split < a->W && 2 * p.split * ctas <= 8ll * sms; p.split <<= 1) {}
      const cudaError_t e = launch_beam_reorder(p, static_cast<unsigned>(ctas * p.split), static_cast<cudaStream_t>(cuda_stream));
      if (e != cudaSuccess) return HOLA_ERR_CUDA;
      p.count = 0;
      ctas = 0;
    }
    if (!s) break;
    BrState& o = p.s[p.count++];
    o.src = static_cast<const unsigned char*>(s->src); o.dst = static_cast<unsigned char*>(s->dst);
    o.seq = s->seq_stride; o.beam = s->beam_stride; o.outer0 = s->outer_stride[0]; o.outer1 = s->outer_stride[1];
    o.to_seq = s->dst_seq_stride; o.to_beam = s->dst_beam_stride; o.to_outer0 = s->dst_outer_stride[0]; o.to_outer1 = s->dst_outer_stride[1];
    o.run = s->run; o.position = s->position;
    o.n0 = static_cast<unsigned>(s->outer[0]); o.n1 = static_cast<unsigned>(s->outer[1]);
    o.pieces = static_cast<unsigned>(pieces); o.piece = br_piece(*s); o.first_cta = static_cast<unsigned>(ctas);
    ctas += more;
  }
  return HOLA_OK;
}

// Whether n bytes at a time can be read or written of rows of `stride` elements.
static bool in_words(const void* base, long long stride, int elem, unsigned bytes) {
  return reinterpret_cast<uintptr_t>(base) % bytes == 0 && stride * elem % bytes == 0;
}

hola_status hola_embed(const hola_embed_args* a, void* cuda_stream) {
  if (!a || a->N < 0 || a->V <= 0 || a->H <= 0 || a->row_stride < 0 || a->add_stride < 0 || a->out_stride < 0) return HOLA_ERR_INVALID_ARG;
  if (a->t_dtype < HOLA_T_F32 || a->t_dtype > HOLA_T_MIXED || a->out_dtype < HOLA_T_F32 || a->out_dtype > HOLA_T_F16) return HOLA_ERR_INVALID_ARG;
  if (a->v_offset < 0 || a->V_global < 0 || (a->V_global > 0 && static_cast<long long>(a->v_offset) + a->V > a->V_global)) return HOLA_ERR_INVALID_ARG;
  if (a->V_global == 0 && a->v_offset != 0) return HOLA_ERR_INVALID_ARG;
  const bool mixed = a->t_dtype == HOLA_T_MIXED;
  if (a->N > INT32_MAX || a->H > kEmMaxH || (mixed && a->H % 128 != 0)) return HOLA_ERR_UNSUPPORTED_SHAPE;
  if (a->N == 0) return HOLA_OK;
  if (!a->tokens || !a->out || (a->N > 1 && a->out_stride < a->H)) return HOLA_ERR_INVALID_ARG;
  if (mixed) {
    const hola_wmix* m = a->wmix;
    if (!m || !m->group_width || !m->group_row || m->rows4 < 0 || m->rows8 < 0 || m->rows16 < 0 ||
        static_cast<long long>(m->rows4) + m->rows8 + m->rows16 != a->V)
      return HOLA_ERR_INVALID_ARG;
    if ((m->rows4 > 0 && (!m->W4 || !m->shift4)) || (m->rows8 > 0 && !m->W8) || (m->rows16 > 0 && !m->W16)) return HOLA_ERR_INVALID_ARG;
  } else if (!a->table) {
    return HOLA_ERR_INVALID_ARG;
  }
  if ((mixed || a->t_dtype == HOLA_T_INT8) != (a->w_scale != nullptr)) return HOLA_ERR_INVALID_ARG;
  const int te = mixed ? 1 : tab_bytes(a->t_dtype), oe = tab_bytes(a->out_dtype);
  if (reinterpret_cast<uintptr_t>(a->tokens) % (a->wide_tokens ? 8 : 4) || reinterpret_cast<uintptr_t>(a->out) % oe ||
      reinterpret_cast<uintptr_t>(a->add) % oe || (!mixed && reinterpret_cast<uintptr_t>(a->table) % te) || off_words({a->w_scale, a->status_word}) ||
      (mixed && (reinterpret_cast<uintptr_t>(a->wmix->W16) % 2 || off_words({a->wmix->group_row}))))
    return HOLA_ERR_INVALID_ARG;
  const Bytes out(a->out, static_cast<long long>(a->H) * oe, {{a->N, a->out_stride * oe}});
  const bool itself = a->add == a->out && (a->N == 1 || a->add_stride == a->out_stride);
  const long long H = a->H;
  if ((!itself && share({a->add, H * oe, {{a->N, a->add_stride * oe}}}, out)) || share({a->tokens, a->N * (a->wide_tokens ? 8 : 4)}, out) ||
      share({a->w_scale, a->V * 4ll}, out) || (!mixed && share({a->table, H * te, {{a->V, a->row_stride * te}}}, out)))
    return HOLA_ERR_INVALID_ARG;
  if (mixed) {
    const hola_wmix& m = *a->wmix;
    const long long groups = (static_cast<long long>(a->V) + 255) / 256;
    for (const Bytes& x : {Bytes(m.W16, m.rows16 * H * 2), Bytes(m.W8, m.rows8 * H), Bytes(m.W4, m.rows4 * (H / 2)), Bytes(m.shift4, m.rows4 * (H / 128)),
                           Bytes(m.group_width, groups), Bytes(m.group_row, groups * 4)})
      if (share(x, out)) return HOLA_ERR_INVALID_ARG;
  }
  const DeviceFacts* dev = device_facts();
  if (!dev) return HOLA_ERR_NO_DEVICE;
  EmParams p = {};
  p.tokens = a->tokens; p.wide = a->wide_tokens; p.N = a->N; p.V = a->V; p.H = a->H; p.v_offset = a->v_offset;
  p.V_global = a->V_global ? a->V_global : a->V;
  p.table = a->table; p.row_stride = a->row_stride; p.w_scale = a->w_scale;
  if (mixed) p.mix = *a->wmix;
  auto end = [&](const void* base, long long rows, long long stride, int elem) {
    return base ? static_cast<const unsigned char*>(base) + ((rows - 1) * stride + a->H) * elem : nullptr;
  };
  p.table_end = end(a->table, a->V, a->row_stride, te); p.add_end = end(a->add, a->N, a->add_stride, oe);
  p.scale = a->scale; p.add = a->add; p.add_stride = a->add_stride; p.out = a->out; p.out_stride = a->out_stride; p.status = a->status_word;
  // (eight channels at a time: 8, 16 or 32 bytes)
  bool words = a->H % 8 == 0 && in_words(a->out, a->out_stride, oe, 8 * oe) && (!a->add || in_words(a->add, a->add_stride, oe, 8 * oe));
  if (mixed) words = words && in_words(p.mix.W16, 0, 1, 16) && in_words(p.mix.W8, 0, 1, 8) && in_words(p.mix.W4, 0, 1, 4);
  else words = words && in_words(a->table, a->row_stride, te, 8 * te);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const bool wide = words && a->H % 16 == 0 && oe == 2 && !mixed && te <= 2 && in_words(a->out, a->out_stride, oe, 32) &&
                    (!a->add || in_words(a->add, a->add_stride, oe, 32)) && in_words(a->table, a->row_stride, te, 16 * te);
  const cudaError_t e = wide ? launch_embed_16(p, a->t_dtype, a->out_dtype, dev->sms, stream)
                             : launch_embed_of(p, a->t_dtype, a->out_dtype, words, dev->sms, stream);
  return e == cudaSuccess ? HOLA_OK : HOLA_ERR_CUDA;
}

size_t hola_embed_grad_workspace_bytes(long long N, int V, int H) {
  EgParams p = {};
  EgLayout l;
  return eg_plan(N, V, H, &p, &l) ? l.enough : 0;
}

hola_status hola_embed_grad(const hola_embed_grad_args* a, void* cuda_stream) {
  if (!a || a->N < 0 || a->V <= 0 || a->H <= 0 || a->grad_stride < 0 || a->out_stride < 0) return HOLA_ERR_INVALID_ARG;
  if (a->g_dtype < HOLA_T_F32 || a->g_dtype > HOLA_T_F16 || a->out_dtype < HOLA_T_F32 || a->out_dtype > HOLA_T_F16) return HOLA_ERR_INVALID_ARG;
  if (a->v_offset < 0 || a->V_global < 0 || (a->V_global > 0 && static_cast<long long>(a->v_offset) + a->V > a->V_global)) return HOLA_ERR_INVALID_ARG;
  if (a->V_global == 0 && a->v_offset != 0) return HOLA_ERR_INVALID_ARG;
  const bool by_rows = a->ids_out || a->count_out;
  if (by_rows && (!a->count_out || a->accumulate)) return HOLA_ERR_INVALID_ARG;
  EgParams p = {};
  EgLayout l;
  if (!eg_plan(a->N, a->V, a->H, &p, &l)) return HOLA_ERR_UNSUPPORTED_SHAPE;
  if (a->N > 0 && (!a->tokens || !a->grad || (by_rows && (!a->ids_out || !a->out)))) return HOLA_ERR_INVALID_ARG;
  if (!by_rows && !a->out) return HOLA_ERR_INVALID_ARG;
  if (!a->workspace || reinterpret_cast<uintptr_t>(a->workspace) % 16 || a->workspace_bytes < l.total) return HOLA_ERR_INVALID_ARG;
  if ((by_rows ? a->N : static_cast<long long>(a->V)) > 1 && a->out_stride < a->H) return HOLA_ERR_INVALID_ARG;
  const int ge = tab_bytes(a->g_dtype), oe = tab_bytes(a->out_dtype);
  if (reinterpret_cast<uintptr_t>(a->tokens) % (a->wide_tokens ? 8 : 4) || reinterpret_cast<uintptr_t>(a->grad) % ge ||
      reinterpret_cast<uintptr_t>(a->out) % oe || off_words({a->ids_out, a->count_out, a->status_word}))
    return HOLA_ERR_INVALID_ARG;
  // (CTAs read tokens and rows while others write results, and the sort's lists lie in the workspace)
  const long long rows = by_rows ? a->N : a->V, width = a->H;
  const Bytes in[] = {{a->tokens, a->N * (a->wide_tokens ? 8 : 4)}, {a->grad, width * ge, {{a->N, a->grad_stride * ge}}}},
              out[] = {{a->out, width * oe, {{rows, a->out_stride * oe}}}, {a->ids_out, a->N * 4}, {a->count_out, 4},
                       {a->workspace, static_cast<long long>(l.total)}};
  for (int i = 0; i < 4; ++i) {
    for (const Bytes& x : in)
      if (share(x, out[i])) return HOLA_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (share(out[j], out[i])) return HOLA_ERR_INVALID_ARG;
  }
  const long long blank = by_rows || a->accumulate ? 0 : (static_cast<long long>(a->V) + p.blank - 1) / p.blank;       // (CTAs that write zeros)
  const long long ctas = p.few ? blank + kEfPerSm * kEgPlanSms : ((a->N + p.window - 1) / p.window + 1 + blank) * p.slices;
  if (ctas > INT32_MAX) return HOLA_ERR_UNSUPPORTED_SHAPE;
  if (!device_facts()) return HOLA_ERR_NO_DEVICE;
  p.tokens = a->tokens; p.wide = a->wide_tokens; p.v_offset = a->v_offset;
  p.V_global = a->V_global ? a->V_global : a->V;
  p.grad = a->grad; p.g_stride = a->grad_stride; p.scale = a->scale; p.out = a->out; p.out_stride = a->out_stride;
  p.accumulate = a->accumulate; p.by_rows = by_rows; p.ids_out = a->ids_out; p.count_out = a->count_out; p.status = a->status_word;
  unsigned char* ws = static_cast<unsigned char*>(a->workspace);
  p.places = reinterpret_cast<int4*>(ws + l.places); p.numbers = reinterpret_cast<int2*>(ws + l.numbers);
  p.first = by_rows || a->accumulate ? nullptr : reinterpret_cast<int*>(ws + l.first);
  p.distinct = reinterpret_cast<int*>(ws + l.distinct); p.valid = reinterpret_cast<int*>(ws + l.valid);
  p.done = reinterpret_cast<unsigned*>(ws + l.done);
  p.partial = reinterpret_cast<float*>(ws + l.partial);
  const bool words = a->H % 8 == 0 && in_words(a->grad, a->grad_stride, ge, 8 * ge) && in_words(a->out, a->out_stride, oe, 8 * oe);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = a->g_dtype == HOLA_T_F32 ? launch_embed_grad<kTabF32>(p, a->out_dtype, words, stream)
                        : a->g_dtype == HOLA_T_BF16 ? launch_embed_grad<kTabBf16>(p, a->out_dtype, words, stream)
                                                    : launch_embed_grad<kTabF16>(p, a->out_dtype, words, stream);
  return e == cudaSuccess ? HOLA_OK : HOLA_ERR_CUDA;
}

}  // extern "C"
