// Softmax attention of rows over lists of neighbours, and its gradient.  Row i (a
// frontier node) attends over the keys and values that indices[offsets[i] ..
// offsets[i+1]) name, as sampling lists them (or as a CSR graph holds them):
//
//   s_e = a q_i . k_j + b_e,   lse_i = ln sum_e exp(s_e),   o_i = sum_e exp(s_e - lse_i) v_j
//
// for each query head; `share` consecutive query heads read one key head.  One pass over
// a list: a running maximum m, the sum of exp(s - m) and the weighted values, rescaled
// when m grows.  The gradient recomputes the probabilities from the saved lse:
//
//   p_e = exp(s_e - lse_i),   ds_e = p_e (do_i . v_j - do_i . o_i),   db_e = ds_e
//   dq_i = a sum_e ds_e k_j,   dk_j = a sum_{e to j} ds_e q_i,   dv_j = sum_{e to j} p_e do_i
//
// in two steps: by rows (dq, and p and ds of every edge), then by keys over the edges
// sorted by key (dg_segments.h), which adds without atomics.
//
// About four operations per byte gathered: bound by memory, that is by the number of
// rows in flight.  So a wave holds whole vectors of several edges at once: of its lanes,
// 2^lg_g hold the vectors of one head, 2^lg_h the heads, 2^lg_e edges of a list, and
// the rest other rows.  Lists longer than a chunk are cut at multiples of the chunk
// length, a wave per chunk, and joined by a second launch.
#include <string.h>

#include "dg_segments.h"

namespace dg {
namespace {

constexpr int AT = 256;  // threads
constexpr int AW = AT / 64;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float NINF = -__builtin_inff();

struct Attend {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const int64_t *offsets;
  const int32_t *indices;
  const float *bias;   // [edges][bias_heads] or NULL
  int bias_heads;
  int64_t nq, nkv, edges;
  int heads, kv_heads, share, D;
  float scale;
  int lg_g, lg_h, lg_e;
  int64_t row_blocks;  // blocks that take rows; the others take chunks
  int64_t chunks;      // 0: no list can be longer than ch
  int ch;
  int64_t slot;        // numbers of a partial result
  float *part;         // [2 * chunks][slot]
  int32_t *status;
  // forward
  void *out;
  float *lse;
  // gradient
  const void *go, *o;
  int64_t go_stride, o_stride;
  const float *lse_in;
  float2 *pd;          // [edges][heads] p and ds
  int32_t *row_of;     // [edges]
  void *dq;
};

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

// What a lane is for.
template <typename T, int V, int RT>
struct Lane {
  Piece<V> pc;
  int es, rs;       // edge and row within the wave
  int kvh, h0;      // key head, first query head
  bool head;        // whether there is such a head
  bool ragged;      // elements of a key may be foreign
  __device__ __forceinline__ Lane(const Attend &a, int lg_e)
      : pc((int)(threadIdx.x & ((1 << a.lg_g) - 1)), a.D) {
    const int lane = threadIdx.x & 63;
    const int parts = a.share / RT;
    const int tile = blockIdx.y / parts;
    const int h = (tile << a.lg_h) + ((lane >> a.lg_g) & ((1 << a.lg_h) - 1));
    es = (lane >> (a.lg_g + a.lg_h)) & ((1 << lg_e) - 1);
    rs = lane >> (a.lg_g + a.lg_h + lg_e);
    head = h < a.kv_heads;
    kvh = min(h, a.kv_heads - 1);
    h0 = kvh * a.share + (blockIdx.y - tile * parts) * RT;
    ragged = (V << a.lg_g) != a.D;
  }
  // A row's vectors of the RT heads from h0; elements of other lanes are 0.
  __device__ __forceinline__ void heads_of(const void *p, int64_t row, int64_t stride, int D,
                                           float (&x)[RT][V]) const {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const auto r = ld_piece<T, V>(static_cast<const T *>(p) + row * stride + (h0 + t) * D, pc);
      to_floats<T, V>(r, x[t]);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (!pc.own(i) || pc.at + i >= D) x[t][i] = 0.f;
    }
  }
};

// Edges of row r (0 to 0 where the offsets are out of order or out of range).
__device__ __forceinline__ void list_of(const Attend &a, int64_t r, int64_t *start, int64_t *end) {
  const int64_t s = a.offsets[r], e = a.offsets[r + 1];
  const bool ok = s >= 0 && s <= e && e <= a.edges;
  if (!ok && a.status) atomicOr(a.status, 2);
  *start = ok ? s : 0;
  *end = ok ? e : 0;
}

// The row whose list holds edge e, found by the whole wave: 64 probes a step.  -1: none.
__device__ __forceinline__ int64_t row_at(const Attend &a, int64_t e) {
  const int lane = threadIdx.x & 63;
  if (a.offsets[0] > e) return -1;
  int64_t lo = 0, hi = a.nq + 1;  // offsets[lo] <= e, and offsets[hi] > e or hi past the end
  while (hi - lo > 1) {
    const int64_t step = (hi - lo + 63) / 64;
    const int64_t at = lo + lane * step;
    const uint64_t le = __ballot(at < hi && a.offsets[at < hi ? at : lo] <= e);
    // (out of order offsets: some row, or none)
    const int many = le == ~0ull ? 64 : __builtin_ctzll(~le);
    const int64_t next = lo + (int64_t)(many > 0 ? many - 1 : 0) * step;
    hi = min(hi, next + step);
    lo = next;
  }
  return lo < a.nq ? lo : -1;
}

// The part of a list that one wave reads at a time: U edges of each edge slot.
template <typename T, int V, int RT, int U>
struct Edges {
  Raw<T, V> k[U], v[U];
  float b[U][RT];
  bool in[U], ok[U];
  int64_t e[U];
  __device__ __forceinline__ void load(const Attend &a, const Lane<T, V, RT> &ln, int64_t base,
                                       int64_t end, int lg_e, bool *bad) {
    int32_t j[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      e[u] = base + ((int64_t)u << lg_e) + ln.es;
      in[u] = e[u] < end;
      j[u] = a.indices[min(e[u], a.edges - 1)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      ok[u] = in[u] && j[u] >= 0 && (int64_t)j[u] < a.nkv;
      *bad |= in[u] && !ok[u] && j[u] != -1;
      const int64_t row = ok[u] ? j[u] : 0;
      k[u] = ld_piece<T, V>(static_cast<const T *>(a.k) + row * a.k_stride + ln.kvh * a.D, ln.pc);
      v[u] = ld_piece<T, V>(static_cast<const T *>(a.v) + row * a.v_stride + ln.kvh * a.D, ln.pc);
    }
    if (a.bias) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int t = 0; t < RT; ++t)
          b[u][t] = a.bias[min(e[u], a.edges - 1) * a.bias_heads +
                           (a.bias_heads > 1 ? ln.h0 + t : 0)];
    }
  }
  // A key's (or value's) vector; foreign elements, which meet zeros, may not be infinite.
  __device__ __forceinline__ void floats(const Lane<T, V, RT> &ln, const Raw<T, V> &r, int D,
                                         float (&x)[V]) const {
    to_floats<T, V>(r, x);
    if (ln.ragged) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (!ln.pc.own(i) || ln.pc.at + i >= D) x[i] = 0.f;
    }
  }
  // Scores: -inf for no edge and for a masked one, whatever its key holds.
  __device__ __forceinline__ void scores(const Attend &a, const Lane<T, V, RT> &ln,
                                         const float (&q)[RT][V], float (&s)[U * RT]) const {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[V];
      floats(ln, k[u], a.D, x);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float d = q[t][0] * x[0];
#pragma unroll
        for (int i = 1; i < V; ++i) d += q[t][i] * x[i];
        s[u * RT + t] = d;
      }
    }
    group_sum(s, a.lg_g);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const float bias = a.bias ? b[u][t] : 0.f;
        s[u * RT + t] = ok[u] && bias != NINF ? s[u * RT + t] * a.scale + bias : NINF;
      }
  }
};

// ------------------------------------------------------------------ forward
template <typename T, int V, int RT>
struct State {
  float m[RT], l[RT], acc[RT][V];
};

// Attends over edges [start, end) of this lane's row, all lanes of the wave together;
// every lane of the row has the whole result.
template <typename T, int V, int RT, int U>
__device__ __forceinline__ void attend_list(const Attend &a, const Lane<T, V, RT> &ln,
                                            const float (&q)[RT][V], int64_t start, int64_t end,
                                            int lg_e, State<T, V, RT> &st, bool *bad) {
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    st.m[t] = NINF;
    st.l[t] = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) st.acc[t][i] = 0.f;
  }
  for (int64_t base = start; __ballot(base < end) != 0; base += (int64_t)U << lg_e) {
    Edges<T, V, RT, U> ed;
    ed.load(a, ln, base, end, lg_e, bad);
    float s[U * RT];
    ed.scores(a, ln, q, s);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float top = st.m[t];
#pragma unroll
      for (int u = 0; u < U; ++u) top = fmaxf(top, s[u * RT + t]);
      const float from = top == NINF ? 0.f : top;  // no edge yet
      const float f = exp_of(st.m[t] - from);
      st.m[t] = top;
      st.l[t] *= f;
#pragma unroll
      for (int i = 0; i < V; ++i) st.acc[t][i] *= f;
#pragma unroll
      for (int u = 0; u < U; ++u) s[u * RT + t] = exp_of(s[u * RT + t] - from);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[V];
      to_floats<T, V>(ed.v[u], x);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const float p = s[u * RT + t];
        st.l[t] += p;
        if (p != 0.f) {  // an edge of weight 0 adds nothing, whatever its value holds
#pragma unroll
          for (int i = 0; i < V; ++i) st.acc[t][i] += p * x[i];
        }
      }
    }
  }
  // the edge slots of a row
  const int from = a.lg_g + a.lg_h, to = from + lg_e;
  if (from == to) return;
  float top[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) top[t] = st.m[t];
  lanes_reduce<false>(top, from, to, MaxF());
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const float f = exp_of(st.m[t] - (top[t] == NINF ? 0.f : top[t]));
    st.m[t] = top[t];
    st.l[t] *= f;
#pragma unroll
    for (int i = 0; i < V; ++i) st.acc[t][i] *= f;
    lanes_reduce<false>(st.acc[t], from, to, AddF());
  }
  lanes_reduce<false>(st.l, from, to, AddF());
}

template <typename T, int V, int RT, int U>
__global__ __launch_bounds__(AT) void k_attend(Attend a) {
  bool bad = false;
  const int wave = threadIdx.x >> 6;
  float q[RT][V];
  State<T, V, RT> st;
  if ((int64_t)blockIdx.x < a.row_blocks) {
    const Lane<T, V, RT> ln(a, a.lg_e);
    const int rows = 64 >> (a.lg_g + a.lg_h + a.lg_e);
    const int64_t row = ((int64_t)blockIdx.x * AW + wave) * rows + ln.rs;
    const bool live = row < a.nq;
    int64_t start = 0, end = 0;
    if (live) list_of(a, row, &start, &end);
    const bool chunked = a.chunks && end - start > a.ch;
    if (chunked) end = start;
    ln.heads_of(a.q, live ? row : a.nq - 1, a.q_stride, a.D, q);
    attend_list<T, V, RT, U>(a, ln, q, start, end, a.lg_e, st, &bad);
    if (live && !chunked && ln.head && ln.es == 0) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const int h = ln.h0 + t;
        const float inv = st.l[t] == 0.f ? 0.f : 1.f / st.l[t];
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = st.acc[t][i] * inv;
        st_piece<false>(from_floats<T, V>(y),
                        static_cast<T *>(a.out) + (row * a.heads + h) * a.D, ln.pc);
        if ((threadIdx.x & ((1 << a.lg_g) - 1)) == 0)
          a.lse[row * a.heads + h] = st.l[t] == 0.f ? NINF : st.m[t] + logf(st.l[t]);
      }
    }
  } else {
    const int lg_e = 6 - a.lg_g - a.lg_h;
    const Lane<T, V, RT> ln(a, lg_e);
    const int64_t c = ((int64_t)blockIdx.x - a.row_blocks) * AW + wave;
    if (c >= a.chunks) return;
    const int64_t lo = c * a.ch, hi = min(lo + a.ch, a.edges);
    const int64_t r0 = row_at(a, lo), r1 = row_at(a, hi - 1);
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
      const int64_t row = side ? r1 : r0;
      if (row < 0 || (side && r1 == r0)) continue;  // the same for the wave
      int64_t start, end;
      list_of(a, row, &start, &end);
      if (end - start <= a.ch) continue;
      ln.heads_of(a.q, row, a.q_stride, a.D, q);
      attend_list<T, V, RT, U>(a, ln, q, max(start, lo), min(end, hi), lg_e, st, &bad);
      if (ln.head && ln.es == 0) {
        float *part = a.part + (2 * c + side) * a.slot;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const int h = ln.h0 + t;
          Raw<float, V> r;
          memcpy(&r.w, st.acc[t], sizeof(st.acc[t]));
          st_piece<false>(r, part + h * a.D, ln.pc);
          if ((threadIdx.x & ((1 << a.lg_g) - 1)) == 0) {
            part[a.heads * a.D + 2 * h] = st.m[t];
            part[a.heads * a.D + 2 * h + 1] = st.l[t];
          }
        }
      }
    }
  }
  if (bad && a.status) atomicOr(a.status, 1);
}

// A block per chunk and head; where a long list starts in the chunk, it joins the list's
// partial results: 1024 / 2^lg groups of lanes take every such part, a column each.
constexpr int JT = 1024;
struct LongList {
  int64_t row, first, parts;  // the first part's slot; the others are 2 (c + 1), 2 (c + 2), ..
};
__device__ __forceinline__ LongList long_list(const Attend &a, int64_t c) {
  LongList l = {-1, 0, 0};
  const int64_t lo = c * a.ch, hi = min(lo + a.ch, a.edges);
  const int64_t row = row_at(a, hi - 1);
  if (row < 0) return l;
  const int64_t start = a.offsets[row], end = a.offsets[row + 1];
  if (start < lo || end > a.edges || end - start <= a.ch) return l;
  l.row = row;
  l.first = 2 * c + (start > lo);
  l.parts = (end - 1) / a.ch - c + 1;
  return l;
}

template <typename T, bool GRAD>
__global__ __launch_bounds__(JT) void k_attend_join(Attend a, int lg) {
  __shared__ float s_m[JT / 64], s_acc[JT], s_l[JT];
  const int64_t c = blockIdx.x;
  const int h = blockIdx.y;
  const LongList l = long_list(a, c);
  if (l.row < 0) return;  // the same for the block
  const int d = threadIdx.x & ((1 << lg) - 1), g = threadIdx.x >> lg, groups = JT >> lg;
  auto part = [&](int64_t j) { return a.part + (j ? 2 * (c + j) : l.first) * a.slot; };
  float top = NINF, from = 0.f;
  if (!GRAD) {
    for (int64_t j = threadIdx.x; j < l.parts; j += JT)
      top = fmaxf(top, part(j)[a.heads * a.D + 2 * h]);
    float t[1] = {top};
    lanes_reduce<true>(t, 0, 6, MaxF());
    if ((threadIdx.x & 63) == 0) s_m[threadIdx.x >> 6] = t[0];
    __syncthreads();
    top = NINF;
#pragma unroll
    for (int i = 0; i < JT / 64; ++i) top = fmaxf(top, s_m[i]);
    from = top == NINF ? 0.f : top;
  }
  float acc = 0.f, sum = 0.f;
  for (int64_t j0 = g; j0 < l.parts; j0 += 8 * groups) {
    float x[8], m[8], ls[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float *p = part(min(j0 + u * groups, l.parts - 1));
      x[u] = p[h * a.D + min(d, a.D - 1)];
      m[u] = GRAD ? 0.f : p[a.heads * a.D + 2 * h];
      ls[u] = GRAD ? 0.f : p[a.heads * a.D + 2 * h + 1];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (j0 + u * groups >= l.parts) continue;
      const float f = GRAD ? 1.f : exp_of(m[u] - from);
      if (f != 0.f) {
        acc += f * x[u];
        sum += f * ls[u];
      }
    }
  }
  s_acc[threadIdx.x] = acc;
  s_l[threadIdx.x] = sum;
  __syncthreads();
  if (g != 0 || d >= a.D) return;
  acc = sum = 0.f;
  for (int i = 0; i < groups; ++i) {
    acc += s_acc[(i << lg) + d];
    sum += s_l[(i << lg) + d];
  }
  const int64_t at = (l.row * a.heads + h) * a.D + d;
  if (GRAD) {
    static_cast<T *>(a.dq)[at] = (T)(acc * a.scale);
  } else {
    static_cast<T *>(a.out)[at] = (T)(sum == 0.f ? 0.f : acc / sum);
    if (d == 0) a.lse[l.row * a.heads + h] = sum == 0.f ? NINF : top + logf(sum);
  }
}

// ------------------------------------------------------------------ gradient by rows
template <typename T, int V, int RT, int U>
__device__ __forceinline__ void grad_list(const Attend &a, const Lane<T, V, RT> &ln, int64_t row,
                                          int64_t start, int64_t end, int lg_e,
                                          float (&dq)[RT][V], bool *bad) {
  float q[RT][V], go[RT][V], delta[RT], lse[RT];
  ln.heads_of(a.q, row, a.q_stride, a.D, q);
  ln.heads_of(a.go, row, a.go_stride, a.D, go);
  {
    float o[RT][V];
    ln.heads_of(a.o, row, a.o_stride, a.D, o);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      delta[t] = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) delta[t] += go[t][i] * o[t][i];
      lse[t] = a.lse_in[row * a.heads + ln.h0 + t];
    }
  }
  group_sum(delta, a.lg_g);
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < V; ++i) dq[t][i] = 0.f;
  const bool writer = ln.head && (threadIdx.x & ((1 << a.lg_g) - 1)) == 0;
  for (int64_t base = start; __ballot(base < end) != 0; base += (int64_t)U << lg_e) {
    Edges<T, V, RT, U> ed;
    ed.load(a, ln, base, end, lg_e, bad);
    float s[U * RT], dp[U * RT];
    ed.scores(a, ln, q, s);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[V];
      ed.floats(ln, ed.v[u], a.D, x);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float d = go[t][0] * x[0];
#pragma unroll
        for (int i = 1; i < V; ++i) d += go[t][i] * x[i];
        dp[u * RT + t] = d;
      }
    }
    group_sum(dp, a.lg_g);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[V];
      to_floats<T, V>(ed.k[u], x);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        // a row without weight has lse = -inf and no gradient
        const float p = lse[t] == NINF ? 0.f : exp_of(s[u * RT + t] - lse[t]);
        const float ds = p == 0.f ? 0.f : p * (dp[u * RT + t] - delta[t]);
        if (p != 0.f) {
#pragma unroll
          for (int i = 0; i < V; ++i) dq[t][i] += ds * x[i];
        }
        if (writer && ed.in[u]) a.pd[ed.e[u] * a.heads + ln.h0 + t] = float2{p, ds};
      }
      if (writer && ln.kvh == 0 && ln.h0 == 0 && ed.in[u]) a.row_of[ed.e[u]] = (int32_t)row;
    }
  }
  const int from = a.lg_g + a.lg_h;
#pragma unroll
  for (int t = 0; t < RT; ++t) lanes_reduce<false>(dq[t], from, from + lg_e, AddF());
}

template <typename T, int V, int RT, int U>
__global__ __launch_bounds__(AT) void k_attend_grad_rows(Attend a) {
  bool bad = false;
  const int wave = threadIdx.x >> 6;
  float dq[RT][V];
  if ((int64_t)blockIdx.x < a.row_blocks) {
    const Lane<T, V, RT> ln(a, a.lg_e);
    const int rows = 64 >> (a.lg_g + a.lg_h + a.lg_e);
    const int64_t row = ((int64_t)blockIdx.x * AW + wave) * rows + ln.rs;
    const bool live = row < a.nq;
    int64_t start = 0, end = 0;
    if (live) list_of(a, row, &start, &end);
    const bool chunked = a.chunks && end - start > a.ch;
    if (chunked) end = start;
    grad_list<T, V, RT, U>(a, ln, live ? row : a.nq - 1, start, end, a.lg_e, dq, &bad);
    if (live && !chunked && ln.head && ln.es == 0) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = dq[t][i] * a.scale;
        st_piece<false>(from_floats<T, V>(y),
                        static_cast<T *>(a.dq) + (row * a.heads + ln.h0 + t) * a.D, ln.pc);
      }
    }
  } else {
    const int lg_e = 6 - a.lg_g - a.lg_h;
    const Lane<T, V, RT> ln(a, lg_e);
    const int64_t c = ((int64_t)blockIdx.x - a.row_blocks) * AW + wave;
    if (c >= a.chunks) return;
    const int64_t lo = c * a.ch, hi = min(lo + a.ch, a.edges);
    const int64_t r0 = row_at(a, lo), r1 = row_at(a, hi - 1);
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
      const int64_t row = side ? r1 : r0;
      if (row < 0 || (side && r1 == r0)) continue;  // the same for the wave
      int64_t start, end;
      list_of(a, row, &start, &end);
      if (end - start <= a.ch) continue;
      grad_list<T, V, RT, U>(a, ln, row, max(start, lo), min(end, hi), lg_e, dq, &bad);
      if (ln.head && ln.es == 0) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          Raw<float, V> r;
          memcpy(&r.w, dq[t], sizeof(dq[t]));
          st_piece<false>(r, a.part + (2 * c + side) * a.slot + (ln.h0 + t) * a.D, ln.pc);
        }
      }
    }
  }
  if (bad && a.status) atomicOr(a.status, 1);
}

// ------------------------------------------------------------------ gradient by keys
// A group of 2^lg lanes per chunk of the edges in the order of their keys, each lane a
// vector of one key head (vph vectors per head); blocks from sum_blocks on write the
// rows of keys without an edge as zeros.
template <typename T, int V>
__global__ __launch_bounds__(AT) void k_attend_grad_keys(Attend a, IdSort so, T *dk, T *dv, int vph,
                                                         int lg, int64_t sum_blocks) {
  constexpr int U = 4;
  const int sub = threadIdx.x & ((1 << lg) - 1), per = AT >> lg;
  const int at = (blockIdx.y << lg) + sub;
  const int kvh = min(at / vph, a.kv_heads - 1);
  const Piece<V> pc(at < a.kv_heads * vph ? at - kvh * vph : vph, a.D);
  const int64_t width = (int64_t)a.kv_heads * a.D;
  if ((int64_t)blockIdx.x >= sum_blocks) {
    const int64_t groups = ((int64_t)gridDim.x - sum_blocks) * per;
    const float zero[V] = {};
    for (int64_t r = ((int64_t)blockIdx.x - sum_blocks) * per + (threadIdx.x >> lg); r < a.nkv;
         r += groups) {
      if (so.seen[r]) continue;
      st_piece<false>(from_floats<T, V>(zero), dk + r * width + kvh * a.D, pc);
      st_piece<false>(from_floats<T, V>(zero), dv + r * width + kvh * a.D, pc);
    }
    return;
  }
  const int64_t c = (int64_t)blockIdx.x * per + (threadIdx.x >> lg);
  if (c >= so.chunks) return;
  const uint32_t limit = (uint32_t)a.nkv;
  const Chunk k = chunk_of(so.dst, so.n, so.C, c);
  const int64_t end = k.beyond ? min(k.stop + so.C, so.n) : k.stop;
  float ak[V], av[V];
  int32_t cur = -1;
  bool lead = k.lead_part;
  auto flush = [&](bool final) {
    if ((uint32_t)cur >= limit) return;
    if (lead || (final && k.trail_part)) {
      float *p = so.part + (2 * c + (lead ? 0 : 1)) * so.width + kvh * a.D;
      Raw<float, V> r;
      memcpy(&r.w, ak, sizeof(ak));
      st_piece<false>(r, p, pc);
      memcpy(&r.w, av, sizeof(av));
      st_piece<false>(r, p + width, pc);
      if (!lead && sub == 0 && blockIdx.y == 0) so.long_at[atomicAdd(so.n_long, 1)] = (int32_t)c;
    } else {
      float y[V];
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = ak[i] * a.scale;
      st_piece<false>(from_floats<T, V>(y), dk + cur * width + kvh * a.D, pc);
      st_piece<false>(from_floats<T, V>(av), dv + cur * width + kvh * a.D, pc);
    }
    lead = false;
  };
  bool done = false;
  for (int64_t i = k.begin; i < end && !done; i += U) {
    int32_t d[U], e[U], row[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t j = min(i + u, so.n - 1);
      d[u] = so.dst[j];
      e[u] = so.order[j];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) row[u] = a.row_of[e[u]];
    float xk[U][V], xv[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int x = 0; x < V; ++x) xk[u][x] = xv[u][x] = 0.f;
    for (int t = 0; t < a.share; ++t) {
      const int h = kvh * a.share + t;
      Raw<T, V> rq[U], rg[U];
      float2 w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        // (an edge of no row: its weights were not written)
        const bool ok = (uint32_t)d[u] < limit && (uint32_t)row[u] < (uint32_t)a.nq;
        const int64_t r = ok ? row[u] : 0;
        w[u] = a.pd[(int64_t)e[u] * a.heads + h];
        if (!ok) w[u] = float2{0.f, 0.f};
        rq[u] = ld_piece<T, V>(static_cast<const T *>(a.q) + r * a.q_stride + h * a.D, pc);
        rg[u] = ld_piece<T, V>(static_cast<const T *>(a.go) + r * a.go_stride + h * a.D, pc);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float y[V];
        if (w[u].x != 0.f) {
          to_floats<T, V>(rq[u], y);
#pragma unroll
          for (int x = 0; x < V; ++x) xk[u][x] += w[u].y * y[x];
          to_floats<T, V>(rg[u], y);
#pragma unroll
          for (int x = 0; x < V; ++x) xv[u][x] += w[u].x * y[x];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (done || i + u >= end || (i + u >= k.stop && d[u] != k.last)) {
        done = true;
        continue;
      }
      if (i + u == k.begin || d[u] != cur) {
        if (i + u != k.begin) flush(false);
        cur = d[u];
#pragma unroll
        for (int x = 0; x < V; ++x) {
          ak[x] = xk[u][x];
          av[x] = xv[u][x];
        }
      } else {
#pragma unroll
        for (int x = 0; x < V; ++x) {
          ak[x] += xk[u][x];
          av[x] += xv[u][x];
        }
      }
    }
  }
  if (k.begin < end) flush(true);
}

// db: ds of the edge's heads, added up where they share the bias.
__global__ __launch_bounds__(AT) void k_attend_grad_bias(Attend a, float *db) {
  const int64_t n = a.edges * a.bias_heads;
  for (int64_t i = (int64_t)blockIdx.x * AT + threadIdx.x; i < n; i += (int64_t)gridDim.x * AT) {
    if (a.bias_heads > 1) {
      db[i] = a.pd[i].y;
      continue;
    }
    float t = 0.f;
    for (int h = 0; h < a.heads; ++h) t += a.pd[i * a.heads + h].y;
    db[i] = t;
  }
}

// Rows without keys at all.
template <typename T>
__global__ __launch_bounds__(AT) void k_fill_rows(T *p, int64_t n, float value) {
  for (int64_t i = (int64_t)blockIdx.x * AT + threadIdx.x; i < n; i += (int64_t)gridDim.x * AT)
    p[i] = (T)value;
}
template <typename T>
void fill_rows(T *p, int64_t n, float value, hipStream_t s) {
  if (n < 1) return;
  const int64_t b = (n + AT - 1) / AT;
  hipLaunchKernelGGL(k_fill_rows<T>, dim3((unsigned)(b > 4096 ? 4096 : b)), dim3(AT), 0, s, p, n,
                     value);
}

// ------------------------------------------------------------------ host side
// Chunk length: about 2048 chunks, of 128 to 1024 edges.
int chunk_edges(int64_t edges) {
  int ch = 128;
  while (ch < 1024 && edges > (int64_t)ch * 2048) ch *= 2;
  return ch;
}
// Chunks of lists of up to `edges` edges, which never shrinks with the number.
int64_t most_chunks(int64_t edges) {
  const int64_t c = (edges + 1023) / 1024, few = (edges + 127) / 128;
  return few <= 2048 ? few : c > 2048 ? c : 2048;
}
size_t part_bytes(int64_t edges, int64_t slot) {
  if (edges <= chunk_edges(edges)) return 256;
  return ((size_t)(2 * most_chunks(edges)) * (size_t)slot * sizeof(float) + 255) & ~(size_t)255;
}

void set_lanes(Attend &a, int vec) {
  a.lg_g = log2_up((a.D + vec - 1) / vec);
  const int heads = log2_up(a.kv_heads);
  a.lg_h = heads < 6 - a.lg_g ? heads : 6 - a.lg_g;
  const int rest = 6 - a.lg_g - a.lg_h;
  // edge slots for a list of middling length in one round of four edges a slot
  const int want = log2_up((a.edges / a.nq + 3) / 4);
  a.lg_e = want < rest ? want : rest;
  const int rows = AW * (64 >> (a.lg_g + a.lg_h + a.lg_e));
  a.row_blocks = (a.nq + rows - 1) / rows;
  a.ch = chunk_edges(a.edges);
  a.chunks = a.edges > a.ch ? (a.edges + a.ch - 1) / a.ch : 0;
}

// Calls f(RT, U) with the query heads that a wave takes of each key head and the edges in
// flight per lane.
template <typename F>
void with_heads(int share, F f) {
  using std::integral_constant;
  if (share % 4 == 0) f(integral_constant<int, 4>(), integral_constant<int, 2>());
  else if (share % 2 == 0) f(integral_constant<int, 2>(), integral_constant<int, 4>());
  else f(integral_constant<int, 1>(), integral_constant<int, 4>());
}
dim3 attend_grid(const Attend &a, int rt) {
  const int tiles = (a.kv_heads + (1 << a.lg_h) - 1) >> a.lg_h;
  return dim3((unsigned)(a.row_blocks + (a.chunks + AW - 1) / AW),
              (unsigned)(tiles * (a.share / rt)));
}

int check_attend(const char *who, int64_t nq, int64_t nkv, int64_t edges, int32_t heads,
                 int32_t kv_heads, int32_t D, int32_t type, const void *bias, int32_t bias_heads) {
  if (nq < 0 || nq > 0x7fffffffll || nkv < 0 || nkv > 0x7fffffffll || edges < 0 ||
      edges > 0x7fffffffll || (edges > 0 && (nq == 0 || nkv == 0)))
    return set_error(DG_EINVAL, "%s: bad sizes", who);
  if (heads < 1 || kv_heads < 1 || heads % kv_heads || heads > DG_MAX_HEADS || D < 1 ||
      D > DG_MAX_HEAD_DIM)
    return set_error(DG_EINVAL, "%s: heads must be a multiple of kv_heads up to %d, D 1 to %d", who,
                     DG_MAX_HEADS, DG_MAX_HEAD_DIM);
  if (!is_wide_type(type)) return set_error(DG_EINVAL, "%s: bad type", who);
  if (bias && bias_heads != 1 && bias_heads != heads)
    return set_error(DG_EINVAL, "%s: bias_heads must be 1 or heads", who);
  return DG_OK;
}

// The sort of the edges by key.
void set_edge_sort(IdSort &so, const int32_t *indices, int64_t edges, int64_t nkv, int64_t kv_heads,
                   int64_t D) {
  memset(&so, 0, sizeof(so));
  so.ids = indices;
  so.n = edges;
  so.slots = nkv;
  so.compact = false;
  so.width = 2 * kv_heads * D;
}

}  // namespace

// ------------------------------------------------------------------ offsets of an edge list
namespace {
__global__ __launch_bounds__(AT) void k_edge_offsets(const int32_t *src, int64_t n, int64_t rows,
                                                     int64_t *offsets, int32_t *status) {
  const int64_t r0 = (int64_t)blockIdx.x * AT, r = r0 + threadIdx.x;
  // offsets[r] = first edge whose row is not below r; the block's span first
  __shared__ int64_t s_at[2];
  if (threadIdx.x < 2) {
    const int64_t want = threadIdx.x ? min(r0 + AT, rows) : r0;
    int64_t lo = 0, hi = n;
    while (lo < hi) {
      const int64_t m = (lo + hi) >> 1;
      if (src[m] < want) lo = m + 1; else hi = m;
    }
    s_at[threadIdx.x] = lo;
  }
  __syncthreads();
  if (r <= rows) {
    int64_t lo = s_at[0], hi = max(s_at[1], lo);
    while (lo < hi) {
      const int64_t m = (lo + hi) >> 1;
      if (src[m] < r) lo = m + 1; else hi = m;
    }
    offsets[r] = lo;
  }
  if (!status) return;
  bool bad = false;  // the block's share of the edges
  for (int64_t e = (int64_t)blockIdx.x * AT + threadIdx.x; e < n; e += (int64_t)gridDim.x * AT) {
    const int32_t x = src[e];
    bad |= x < 0 || (int64_t)x >= rows || (e > 0 && src[e - 1] > x);
  }
  if (bad) atomicOr(status, 2);
}
}  // namespace

}  // namespace dg

using namespace dg;

extern "C" int dg_edge_offsets(const int32_t *edge_src, int64_t num_edges, int64_t num_rows,
                               int64_t *offsets, int32_t *status, hipStream_t stream) {
  if (num_edges < 0 || num_edges > 0x7fffffffll || num_rows < 0 || num_rows > 0x7fffffffll)
    return set_error(DG_EINVAL, "dg_edge_offsets: bad sizes");
  if (!offsets || (num_edges > 0 && !edge_src))
    return set_error(DG_EINVAL, "dg_edge_offsets: null pointer argument");
  if (ranges_overlap(offsets, 8 * (num_rows + 1), edge_src, 4 * num_edges))
    return set_error(DG_EINVAL, "dg_edge_offsets: the output overlaps the input");
  hipLaunchKernelGGL(k_edge_offsets, dim3((unsigned)((num_rows + 1 + AT - 1) / AT)), dim3(AT), 0,
                     stream, edge_src, num_edges, num_rows, offsets, status);
  DG_HIP(hipGetLastError());
  return DG_OK;
}

extern "C" size_t dg_attend_edges_workspace_bytes(int64_t num_edges, int32_t heads, int32_t D) {
  if (num_edges < 0 || num_edges > 0x7fffffffll || heads < 1 || heads > DG_MAX_HEADS || D < 1 ||
      D > DG_MAX_HEAD_DIM)
    return 0;
  return part_bytes(num_edges, (int64_t)heads * (D + 2));
}

extern "C" int dg_attend_edges(const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                               const void *v, int64_t v_stride, int32_t type, int64_t nq,
                               int64_t nkv, int32_t heads, int32_t kv_heads, int32_t D,
                               const int64_t *offsets, const int32_t *indices, int64_t num_edges,
                               const float *bias, int32_t bias_heads, float scale, void *out,
                               float *lse, int32_t *status, void *ws, size_t ws_bytes,
                               hipStream_t stream) {
  DG_TRY(check_attend("dg_attend_edges", nq, nkv, num_edges, heads, kv_heads, D, type, bias,
                      bias_heads));
  if (nq == 0) return DG_OK;
  const int64_t qw = (int64_t)heads * D, kw = (int64_t)kv_heads * D, b = type_bytes(type);
  if (q_stride < qw || (num_edges > 0 && (k_stride < kw || v_stride < kw)))
    return set_error(DG_EINVAL, "dg_attend_edges: bad sizes");
  if (!q || !offsets || !out || !lse || (num_edges > 0 && (!k || !v || !indices)))
    return set_error(DG_EINVAL, "dg_attend_edges: null pointer argument");
  const int64_t ob = nq * qw * b, lb = 4 * nq * heads;
  if (ranges_overlap(out, ob, q, span_bytes(nq, qw, q_stride, b)) ||
      ranges_overlap(out, ob, k, span_bytes(nkv, kw, k_stride, b)) ||
      ranges_overlap(out, ob, v, span_bytes(nkv, kw, v_stride, b)) ||
      ranges_overlap(out, ob, lse, lb) || ranges_overlap(out, ob, indices, 4 * num_edges) ||
      ranges_overlap(out, ob, offsets, 8 * (nq + 1)) || ranges_overlap(lse, lb, bias, 4 * num_edges))
    return set_error(DG_EINVAL, "dg_attend_edges: an output overlaps an input or output");
  const size_t need = part_bytes(num_edges, (int64_t)heads * (D + 2));
  if (num_edges > chunk_edges(num_edges) && (!ws || ws_bytes < need || ((uintptr_t)ws & 255)))
    return set_error(DG_EWORKSPACE, "dg_attend_edges: workspace needs %zu bytes", need);
  Attend a;
  memset(&a, 0, sizeof(a));
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.offsets = offsets;
  a.indices = indices;
  a.bias = bias;
  a.bias_heads = bias_heads;
  a.nq = nq;
  a.nkv = nkv;
  a.edges = num_edges;
  a.heads = heads;
  a.kv_heads = kv_heads;
  a.share = heads / kv_heads;
  a.D = D;
  a.scale = scale;
  a.slot = (int64_t)heads * (D + 2);
  a.part = static_cast<float *>(ws);
  a.status = status;
  a.out = out;
  a.lse = lse;
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    if (num_edges == 0) {
      fill_rows(static_cast<T *>(out), nq * qw, 0.f, stream);
      fill_rows(lse, nq * heads, NINF, stream);
      DG_HIP(hipGetLastError());
      return (int)DG_OK;
    }
    (void)with_vec<T>(D, [&](auto v) {
      constexpr int V = decltype(v)::value;
      set_lanes(a, V);
      with_heads(a.share, [&](auto rt, auto u) {
        hipLaunchKernelGGL((k_attend<T, V, decltype(rt)::value, decltype(u)::value>),
                           attend_grid(a, decltype(rt)::value), dim3(AT), 0, stream, a);
      });
      return (int)DG_OK;
    });
    if (a.chunks)
      hipLaunchKernelGGL((k_attend_join<T, false>), dim3((unsigned)a.chunks, (unsigned)heads),
                         dim3(JT), 0, stream, a, log2_up(D));
    DG_HIP(hipGetLastError());
    return (int)DG_OK;
  });
}

namespace {
// The gradient's workspace: p and ds per edge and head, each edge's row, partial sums of
// long lists, and the sort.
struct GradRoom {
  float2 *pd;
  int32_t *row_of;
  float *part;
  size_t fixed;
};
GradRoom carve_grad(Carve &c, int64_t edges, int32_t heads, int32_t D) {
  GradRoom r;
  r.pd = c.take<float2>((size_t)edges * (size_t)heads);
  r.row_of = c.take<int32_t>((size_t)edges);
  r.part = c.take<float>(part_bytes(edges, (int64_t)heads * D) / sizeof(float));
  r.fixed = c.used;
  return r;
}
}  // namespace

extern "C" size_t dg_attend_edges_grad_workspace_bytes(int64_t num_edges, int64_t nkv,
                                                       int32_t heads, int32_t kv_heads, int32_t D) {
  if (num_edges < 0 || num_edges > 0x7fffffffll || nkv < 0 || nkv > 0x7fffffffll || heads < 1 ||
      heads > DG_MAX_HEADS || kv_heads < 1 || kv_heads > heads || D < 1 || D > DG_MAX_HEAD_DIM)
    return 0;
  Carve c(nullptr);
  const GradRoom r = carve_grad(c, num_edges, heads, D);
  IdSort so;
  set_edge_sort(so, nullptr, num_edges, nkv, kv_heads, D);
  return r.fixed + sort_room(so);
}

extern "C" int dg_attend_edges_grad(
    const void *grad_out, int64_t grad_stride, const void *q, int64_t q_stride, const void *k,
    int64_t k_stride, const void *v, int64_t v_stride, const void *out, int64_t out_stride,
    const float *lse, int32_t type, int64_t nq, int64_t nkv, int32_t heads, int32_t kv_heads,
    int32_t D, const int64_t *offsets, const int32_t *indices, int64_t num_edges,
    const float *bias, int32_t bias_heads, float scale, void *grad_q, void *grad_k, void *grad_v,
    float *grad_bias, int32_t *status, void *ws, size_t ws_bytes, hipStream_t stream) {
  DG_TRY(check_attend("dg_attend_edges_grad", nq, nkv, num_edges, heads, kv_heads, D, type, bias,
                      bias_heads));
  const int64_t qw = (int64_t)heads * D, kw = (int64_t)kv_heads * D, b = type_bytes(type);
  if ((nq > 0 && (q_stride < qw || grad_stride < qw || out_stride < qw)) ||
      (nkv > 0 && (k_stride < kw || v_stride < kw)))
    return set_error(DG_EINVAL, "dg_attend_edges_grad: bad sizes");
  if ((nq > 0 && (!grad_out || !q || !out || !lse || !offsets || !grad_q)) ||
      (nkv > 0 && (!grad_k || !grad_v)) || (num_edges > 0 && (!k || !v || !indices)))
    return set_error(DG_EINVAL, "dg_attend_edges_grad: null pointer argument");
  if (grad_bias && !bias)
    return set_error(DG_EINVAL, "dg_attend_edges_grad: grad_bias without bias");
  const struct {
    const void *p;
    int64_t n;
  } ins[] = {{grad_out, span_bytes(nq, qw, grad_stride, b)}, {q, span_bytes(nq, qw, q_stride, b)},
             {k, span_bytes(nkv, kw, k_stride, b)}, {v, span_bytes(nkv, kw, v_stride, b)},
             {out, span_bytes(nq, qw, out_stride, b)}, {lse, 4 * nq * heads},
             {indices, 4 * num_edges}, {offsets, 8 * (nq + 1)},
             {bias, 4 * num_edges * (bias_heads > 1 ? bias_heads : 1)}},
    outs[] = {{grad_q, nq * qw * b}, {grad_k, nkv * kw * b}, {grad_v, nkv * kw * b},
              {grad_bias, 4 * num_edges * (bias_heads > 1 ? bias_heads : 1)}};
  for (int i = 0; i < 4; ++i) {
    for (const auto &x : ins)
      if (ranges_overlap(outs[i].p, outs[i].n, x.p, x.n))
        return set_error(DG_EINVAL, "dg_attend_edges_grad: an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (ranges_overlap(outs[i].p, outs[i].n, outs[j].p, outs[j].n))
        return set_error(DG_EINVAL, "dg_attend_edges_grad: two outputs overlap");
  }
  if (num_edges > 0) {
    IdSort so;
    set_edge_sort(so, indices, num_edges, nkv, kv_heads, D);
    Carve size(nullptr);
    (void)carve_grad(size, num_edges, heads, D);
    carve_sort(so, size);
    if (!ws || ws_bytes < size.used || ((uintptr_t)ws & 255))
      return set_error(DG_EWORKSPACE, "dg_attend_edges_grad: workspace needs %zu bytes", size.used);
  }
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    if (num_edges == 0) {
      fill_rows(static_cast<T *>(grad_q), nq * qw, 0.f, stream);
      fill_rows(static_cast<T *>(grad_k), nkv * kw, 0.f, stream);
      fill_rows(static_cast<T *>(grad_v), nkv * kw, 0.f, stream);
      DG_HIP(hipGetLastError());
      return (int)DG_OK;
    }
    Attend a;
    memset(&a, 0, sizeof(a));
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.offsets = offsets;
    a.indices = indices;
    a.bias = bias;
    a.bias_heads = bias_heads;
    a.nq = nq;
    a.nkv = nkv;
    a.edges = num_edges;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.share = heads / kv_heads;
    a.D = D;
    a.scale = scale;
    a.slot = qw;
    a.status = status;
    a.go = grad_out;
    a.o = out;
    a.go_stride = grad_stride;
    a.o_stride = out_stride;
    a.lse_in = lse;
    a.dq = grad_q;
    Carve c(ws);
    const GradRoom r = carve_grad(c, num_edges, heads, D);
    a.pd = r.pd;
    a.row_of = r.row_of;
    a.part = r.part;
    IdSort so;
    set_edge_sort(so, indices, num_edges, nkv, kv_heads, D);
    carve_sort(so, c);
    DG_TRY(run_sort(so, nullptr, nullptr, status, stream));
    (void)with_vec<T>(D, [&](auto v) {
      constexpr int V = decltype(v)::value;
      set_lanes(a, V);
      with_heads(a.share, [&](auto rt, auto u) {
        hipLaunchKernelGGL((k_attend_grad_rows<T, V, decltype(rt)::value, decltype(u)::value>),
                           attend_grid(a, decltype(rt)::value), dim3(AT), 0, stream, a);
      });
      if (a.chunks)
        hipLaunchKernelGGL((k_attend_join<T, true>), dim3((unsigned)a.chunks, (unsigned)heads),
                           dim3(JT), 0, stream, a, log2_up(D));
      const int vph = (D + V - 1) / V;
      const RowLanes lanes = row_lanes((int64_t)kv_heads * vph);
      const int per = AT >> lanes.lg;
      const int64_t sums = (so.chunks + per - 1) / per;
      int64_t zeros = (nkv + 8 * per - 1) / (8 * per);
      if (zeros > 4096) zeros = 4096;
      hipLaunchKernelGGL((k_attend_grad_keys<T, V>),
                         dim3((unsigned)(sums + zeros), (unsigned)lanes.tiles), dim3(AT), 0,
                         stream, a, so, static_cast<T *>(grad_k), static_cast<T *>(grad_v), vph,
                         lanes.lg, sums);
      return (int)DG_OK;
    });
    if (grad_bias) {
      const int64_t blocks = (num_edges * bias_heads + AT - 1) / AT;
      hipLaunchKernelGGL(k_attend_grad_bias, dim3((unsigned)(blocks > 8192 ? 8192 : blocks)),
                         dim3(AT), 0, stream, a, grad_bias);
    }
    DG_HIP(hipGetLastError());
    const JoinOut j = {{grad_k, grad_v}, {kw, kw}, {0, kw}, {scale, 1.f}};
    return run_join(so, j, 2, (int)kw, type, stream);
  });
}
