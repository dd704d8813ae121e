// Placement policies: rows of logits over resources, one row per op and
// policy.  A group of G lanes (1 to 64) holds a row, NV resources a lane (8, or 16
// beyond 512 resources), so that up to 64 rows share a wavefront and the sums
// within a row take log2 G exchanges.  Times beside the kernels are of one MI355X,
// of calls between others: the same call again and again for some milliseconds
// slows the card down, by a third for the longest draws.
#include <algorithm>
#include <climits>

#include "policy.hpp"
#include "sim.hpp"

namespace mlsim {
namespace {

constexpr int kThreads = 256;
constexpr float kInf = __builtin_inff();
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;
constexpr uint16_t kNoPlace = 65535;

// ---- values across the lanes of a group ----

// The value of the lane O away within its 2 O: lanes whose O-lane blocks hold
// equal values (the state of a reduction before step O) get the other block's.
// Data-parallel moves up to 8, row swaps for 16 and 32: nothing goes through LDS.
template <int O>
__device__ __forceinline__ uint32_t partner(uint32_t v) {
  if constexpr (O == 1) return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true);         // quad 1 0 3 2
  else if constexpr (O == 2) return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true);    // quad 2 3 0 1
  else if constexpr (O == 4) return __builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, true);   // mirrored in 8
  else if constexpr (O == 8) return __builtin_amdgcn_mov_dpp(v, 0x140, 0xF, 0xF, true);   // mirrored in 16
  else if constexpr (O == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return (threadIdx.x & 16) ? r[0] : r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (threadIdx.x & 32) ? r[0] : r[1];
  }
}

template <int O, class F>
__device__ __forceinline__ F partner_of(F v) {
  uint32_t w[sizeof(F) / 4];
  __builtin_memcpy(w, &v, sizeof(F));
#pragma unroll
  for (unsigned i = 0; i < sizeof(F) / 4; ++i) w[i] = partner<O>(w[i]);
  __builtin_memcpy(&v, w, sizeof(F));
  return v;
}

// op over the G lanes of a group, the result in all of them.
template <int G, class F, class Op>
__device__ __forceinline__ F group_all(F v, Op op) {
  if constexpr (G > 1) v = op(v, partner_of<1>(v));
  if constexpr (G > 2) v = op(v, partner_of<2>(v));
  if constexpr (G > 4) v = op(v, partner_of<4>(v));
  if constexpr (G > 8) v = op(v, partner_of<8>(v));
  if constexpr (G > 16) v = op(v, partner_of<16>(v));
  if constexpr (G > 32) v = op(v, partner_of<32>(v));
  return v;
}

// An infinity that the compiler does not know.  The median of two values and
// it is the larger of the two (the other one where one is NaN) in one
// instruction; a maximum, or a median with a known infinity, first clears
// signalling NaN in each: 152 instructions for a merge of 96.
__device__ __forceinline__ float some_infinity() {
  float inf = kInf;
  asm("" : "+v"(inf));
  return inf;
}

template <int G>
__device__ __forceinline__ float group_max(float v) {
  const float inf = some_infinity();
  return group_all<G>(v, [=](float a, float b) { return __builtin_amdgcn_fmed3f(a, b, inf); });
}

// The largest of a group's values, passing over NaN.
template <int G, int NV>
__device__ __forceinline__ float row_max(const float (&x)[NV]) {
  const float inf = some_infinity();
  float m = x[0];
#pragma unroll
  for (int j = 1; j < NV; ++j) m = __builtin_amdgcn_fmed3f(m, x[j], inf);
  return group_max<G>(m);
}

template <int G, class F>
__device__ __forceinline__ F group_sum(F v) {
  return group_all<G>(v, [](F a, F b) { return a + b; });
}
template <int G>
__device__ __forceinline__ uint32_t group_umax(uint32_t v) {
  return group_all<G>(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// The value of lane (lane ^ X), for the X that sorting needs.
template <int X>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  if constexpr (X == 1 || X == 2 || X == 7 || X == 15 || X == 16 || X == 32)
    return partner<(X == 7 ? 4 : X == 15 ? 8 : X)>(v);
  else if constexpr (X == 3) return __builtin_amdgcn_mov_dpp(v, 0x1B, 0xF, 0xF, true);   // quad 3 2 1 0
  else if constexpr (X == 8) return __builtin_amdgcn_mov_dpp(v, 0x128, 0xF, 0xF, true);  // 16 turned by 8
  else if constexpr (X == 4) return lane_xor<3>(lane_xor<7>(v));
  else if constexpr (X == 31) return lane_xor<15>(lane_xor<16>(v));
  else return lane_xor<31>(lane_xor<32>(v));
}

// How many of a group's flags are set; a whole wavefront's through the scalar unit.
template <int G, int N>
__device__ __forceinline__ int group_count(const bool (&f)[N]) {
  int c = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) c += G == 64 ? (int)__popcll(__ballot(f[j])) : f[j];
  return G == 64 ? c : group_sum<G>(c);
}

template <class T>
__device__ __forceinline__ T from_lane(T v, int lane) {
  uint32_t w[sizeof(T) / 4];
  __builtin_memcpy(w, &v, sizeof(T));
#pragma unroll
  for (unsigned i = 0; i < sizeof(T) / 4; ++i) w[i] = __builtin_amdgcn_readlane(w[i], lane);
  __builtin_memcpy(&v, w, sizeof(T));
  return v;
}

// A compare's result that is an addition's carry, or a select's, makes two or
// three instructions an element where the compiler makes three or five.  A
// vector instruction may read such a result two others after the compare, so
// four elements take turns.

// n += (a[0 .. 3] <= b)
__device__ __forceinline__ void count_le(uint32_t &n, const float *a, float b) {
  uint64_t p, q, r;
  asm("v_cmp_le_f32 %1, %4, %8\n\tv_cmp_le_f32 %2, %5, %8\n\tv_cmp_le_f32 %3, %6, %8\n\t"
      "v_addc_co_u32 %0, %1, 0, %0, %1\n\tv_cmp_le_f32 %1, %7, %8\n\t"
      "v_addc_co_u32 %0, %2, 0, %0, %2\n\tv_addc_co_u32 %0, %3, 0, %0, %3\n\tv_addc_co_u32 %0, %1, 0, %0, %1"
      : "+&v"(n), "=&s"(p), "=&s"(q), "=&s"(r)
      : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(b));
}

// n += !(x[0 .. 3] < cutoff), and w = 0 where x < cutoff.
__device__ __forceinline__ void keep_from(uint32_t &n, float *w, const float *x, float cutoff) {
  uint64_t p, q, r;
  asm("v_cmp_nlt_f32 %5, %8, %12\n\tv_cmp_nlt_f32 %6, %9, %12\n\tv_cmp_nlt_f32 %7, %10, %12\n\t"
      "v_cndmask_b32 %1, 0, %1, %5\n\tv_addc_co_u32 %0, %5, 0, %0, %5\n\tv_cmp_nlt_f32 %5, %11, %12\n\t"
      "v_cndmask_b32 %2, 0, %2, %6\n\tv_addc_co_u32 %0, %6, 0, %0, %6\n\t"
      "v_cndmask_b32 %3, 0, %3, %7\n\tv_addc_co_u32 %0, %7, 0, %0, %7\n\t"
      "v_cndmask_b32 %4, 0, %4, %5\n\tv_addc_co_u32 %0, %5, 0, %0, %5"
      : "+&v"(n), "+&v"(w[0]), "+&v"(w[1]), "+&v"(w[2]), "+&v"(w[3]), "=&s"(p), "=&s"(q), "=&s"(r)
      : "v"(x[0]), "v"(x[1]), "v"(x[2]), "v"(x[3]), "v"(cutoff));
}

// k = 2 k + (u >= t), for four
__device__ __forceinline__ void descend(uint32_t *k, const float *u, const float *t) {
  uint64_t p, q, r;
  asm("v_cmp_ge_f32 %4, %7, %11\n\tv_cmp_ge_f32 %5, %8, %12\n\tv_cmp_ge_f32 %6, %9, %13\n\t"
      "v_addc_co_u32 %0, %4, %0, %0, %4\n\tv_cmp_ge_f32 %4, %10, %14\n\t"
      "v_addc_co_u32 %1, %5, %1, %1, %5\n\tv_addc_co_u32 %2, %6, %2, %2, %6\n\tv_addc_co_u32 %3, %4, %3, %3, %4"
      : "+&v"(k[0]), "+&v"(k[1]), "+&v"(k[2]), "+&v"(k[3]), "=&s"(p), "=&s"(q), "=&s"(r)
      : "v"(u[0]), "v"(u[1]), "v"(u[2]), "v"(u[3]), "v"(t[0]), "v"(t[1]), "v"(t[2]), "v"(t[3]));
}

// v as the data-parallel move CTRL brings it to the rows of 16 lanes in ROWS, 0 elsewhere.
template <int CTRL, int ROWS, class F>
__device__ __forceinline__ F moved(F v) {
  uint32_t w[sizeof(F) / 4];
  __builtin_memcpy(w, &v, sizeof(F));
#pragma unroll
  for (unsigned i = 0; i < sizeof(F) / 4; ++i)
    w[i] = ROWS == 0xF ? __builtin_amdgcn_mov_dpp(w[i], CTRL, 0xF, 0xF, true) : __builtin_amdgcn_update_dpp(0u, w[i], CTRL, ROWS, 0xF, false);
  __builtin_memcpy(&v, w, sizeof(F));
  return v;
}

// Sum over the lanes of a group before this one, and over all of them: shifts
// within 16 lanes (0x110 + o), then the last lane of 16 (0x142) and of 32
// (0x143) passed on.  A shift brings other groups' values too; those are dropped.
template <int G, class F>
__device__ __forceinline__ F group_before(F v, int g, F &all) {
  if constexpr (G == 1) {
    all = v;
    return F(0);
  }
  F in = v;
  auto step = [&](F t, int o) { in += g % 16 >= o ? t : F(0); };
  if constexpr (G > 1) step(moved<0x111, 0xF>(in), 1);
  if constexpr (G > 2) step(moved<0x112, 0xF>(in), 2);
  if constexpr (G > 4) step(moved<0x114, 0xF>(in), 4);
  if constexpr (G > 8) step(moved<0x118, 0xF>(in), 8);
  if constexpr (G > 16) in += moved<0x142, 0xA>(in);
  if constexpr (G > 32) in += moved<0x143, 0xC>(in);
  if constexpr (G == 2)
    all = moved<0xF5, 0xF>(in);  // quad 1 1 3 3
  else if constexpr (G == 4)
    all = moved<0xFF, 0xF>(in);  // quad 3 3 3 3
  else if constexpr (G == 64)
    all = from_lane(in, 63);
  else if constexpr (sizeof(F) == 4)
    all = group_sum<G>(v);  // as a float, another order of additions
  else
    all = __shfl(in, G - 1, G);
  F ex;
  if constexpr (G <= 16)
    ex = moved<0x111, 0xF>(in);
  else
    ex = __shfl_up(in, 1, G);
  return g ? ex : F(0);
}

// LDS of one wavefront is read and written in order; this keeps the compiler to it.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---- rows ----

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ float f16_value(uint32_t bits) {
  const uint16_t b = (uint16_t)bits;
  _Float16 h;
  __builtin_memcpy(&h, &b, 2);
  return (float)h;
}
// Both round to nearest, ties to even; NaN stays NaN.
typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
typedef _Float16 f16_pair __attribute__((ext_vector_type(2)));
typedef float f32_pair __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t half_pair(float lo, float hi, bool f16) {
  const f32_pair v = {lo, hi};
  uint32_t bits;
  if (f16) {
    const f16_pair h = __builtin_convertvector(v, f16_pair);
    __builtin_memcpy(&bits, &h, 4);
  } else {
    const bf16_pair h = __builtin_convertvector(v, bf16_pair);
    __builtin_memcpy(&bits, &h, 4);
  }
  return bits;
}
__device__ __forceinline__ float half_value(uint32_t bits, bool f16) { return f16 ? f16_value(bits) : bf16_value(bits); }

__device__ __forceinline__ float load_elem(const void *base, int32_t dtype, int64_t i) {
  if (dtype == SIM_F32) return ((const float *)base)[i];
  return half_value(((const uint16_t *)base)[i], dtype == SIM_F16);
}

// x[j] = the row's element r0 + j, -inf behind its end.  Lanes with NV elements
// take them in loads of 16 bytes, which need no alignment; only a row whose
// length NV does not divide has a lane that takes fewer, one by one.
template <int NV>
__device__ __forceinline__ void load_row(const void *base, int32_t dtype, int64_t row, int r0, int n, float (&x)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) x[j] = -kInf;
  const bool f16 = dtype == SIM_F16;
  if (r0 + NV <= n) {
    if (dtype == SIM_F32) {
      __builtin_memcpy(x, (const float *)base + row + r0, sizeof(x));
    } else {
      uint16_t h[NV];
      __builtin_memcpy(h, (const uint16_t *)base + row + r0, sizeof(h));
      // a branch for eight: else both values are made and one selected, 24
      // instructions (log-probabilities of 1024 x 6624 rows of 48: 179 us, 169 with
      // the branch); for the pieces of long rows it would part their loads (16 x
      // 20000 rows of 1001, distilled: 485 us, 604 with it)
      if (NV >= 8 && f16) {
        asm volatile("");
#pragma unroll
        for (int j = 0; j < NV; ++j) x[j] = f16_value(h[j]);
      } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) x[j] = half_value(h[j], NV < 8 && f16);
      }
    }
  }
  if (NV > 1 && n % NV && r0 < n && r0 + NV > n) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (r0 + j < n) x[j] = load_elem(base, dtype, row + r0 + j);
  }
}

// The same as they stand in memory, of 16 bits, pair by pair.
template <int NV>
__device__ __forceinline__ void load_bits(const void *base, bool f16, int64_t row, int r0, int n, uint32_t (&w)[NV / 2]) {
#pragma unroll
  for (int i = 0; i < NV / 2; ++i) w[i] = f16 ? 0xFC00FC00u : 0xFF80FF80u;  // -inf
  const uint16_t *p = (const uint16_t *)base + row + r0;
  if (r0 + NV <= n) __builtin_memcpy(w, p, sizeof(w));
  if (n % NV && r0 < n && r0 + NV > n) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (r0 + j < n) w[j / 2] = j % 2 ? (w[j / 2] & 0xFFFFu) | (uint32_t)p[j] << 16 : (w[j / 2] & 0xFFFF0000u) | p[j];
  }
}
template <int NV>
__device__ __forceinline__ void values_of(const uint32_t (&w)[NV / 2], bool f16, float (&x)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) x[j] = half_value(w[j / 2] >> 16 * (j % 2) & 0xFFFFu, f16);
}

template <int NV>
__device__ __forceinline__ void store_row(void *base, int32_t dtype, int64_t row, int r0, int n, const float (&x)[NV]) {
  if (r0 >= n) return;
  if (dtype == SIM_F32) {
    float *p = (float *)base + row + r0;
    if (r0 + NV <= n) {
      __builtin_memcpy(p, x, sizeof(x));
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (r0 + j < n) p[j] = x[j];
    }
    return;
  }
  uint16_t *p = (uint16_t *)base + row + r0;
  uint32_t w[(NV + 1) / 2];
#pragma unroll
  for (int j = 0; j < NV; j += 2) w[j / 2] = half_pair(x[j], j + 1 < NV ? x[j + 1] : 0.0f, dtype == SIM_F16);
  if (r0 + NV <= n) {
    __builtin_memcpy(p, w, NV * 2);
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (r0 + j < n) p[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
  }
}

// Rows whose order does not matter to the sums are held in pieces of V
// resources, lane after lane, so that long rows are read in whole lines: lane g
// has resource (j / V) G V + g V + j % V as its element j.
constexpr int piece(int nv) { return nv > 8 ? 4 : nv; }

template <int G, int NV>
__device__ __forceinline__ void load_spread(const void *base, int32_t dtype, int64_t row, int g, int n, float (&x)[NV]) {
  constexpr int V = piece(NV);
#pragma unroll
  for (int c = 0; c < NV / V; ++c) load_row<V>(base, dtype, row, (c * G + g) * V, n, reinterpret_cast<float (&)[V]>(x[c * V]));
}

template <int G, int NV>
__device__ __forceinline__ void store_spread(void *base, int32_t dtype, int64_t row, int g, int n, const float (&x)[NV]) {
  constexpr int V = piece(NV);
#pragma unroll
  for (int c = 0; c < NV / V; ++c) store_row<V>(base, dtype, row, (c * G + g) * V, n, reinterpret_cast<const float (&)[V]>(x[c * V]));
}

// A spread row as it stands in memory, for loads ahead of their use: what is
// loaded is first looked at by values().
template <int TYPE, int G, int NV>
struct RowWords {
  static constexpr int V = piece(NV), kPiece = TYPE == SIM_F32 ? V : V / 2;
  uint32_t w[NV / V][kPiece];

  __device__ __forceinline__ void load(const void *base, int64_t row, int g, int n) {
#pragma unroll
    for (int c = 0; c < NV / V; ++c) {
      const int r0 = (c * G + g) * V;
      if constexpr (TYPE == SIM_F32) {
        const float *p = (const float *)base + row + r0;
#pragma unroll
        for (int j = 0; j < V; ++j) w[c][j] = 0xFF800000u;  // -inf
        if (r0 + V <= n) __builtin_memcpy(w[c], p, sizeof(w[c]));
        if (n % V && r0 < n && r0 + V > n) {
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (r0 + j < n) w[c][j] = __float_as_uint(p[j]);
        }
      } else {
        load_bits<V>(base, TYPE == SIM_F16, row, r0, n, w[c]);
      }
    }
  }
  __device__ __forceinline__ void values(float (&x)[NV]) const {
#pragma unroll
    for (int c = 0; c < NV / V; ++c) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        x[c * V + j] = TYPE == SIM_F32 ? __uint_as_float(w[c][j % kPiece])
                                       : half_value(w[c][j / 2 % kPiece] >> 16 * (j % 2) & 0xFFFFu, TYPE == SIM_F16);
    }
  }
};

// f(the type) as a compile-time constant.
template <class F>
__device__ __forceinline__ void by_type(int32_t dtype, F f) {
  if (dtype == SIM_F32) f(std::integral_constant<int, SIM_F32>{});
  if (dtype == SIM_BF16) f(std::integral_constant<int, SIM_BF16>{});
  if (dtype == SIM_F16) f(std::integral_constant<int, SIM_F16>{});
}

// Which element of lane g a resource is; negative: none.
template <int G, int NV>
__device__ __forceinline__ int spread_at(int r, int g) {
  constexpr int V = piece(NV);
  const int c = r / (G * V), in = r % (G * V);
  return in / V == g ? c * V + in % V : -1;
}

// ---- settings, and which scenarios a policy has ----

// A temperature is 0 or a normal float32: 1 / T and log2 e / T are finite then.
__device__ __forceinline__ bool temperature_ok(float T) {
  return T == 0 || (T >= kLeastTemperature && T < kInf);
}

__device__ __forceinline__ float policy_temperature(const PolicyArgs &a, int p) {
  return a.settings ? a.settings[(int64_t)p * 4] : a.temperature;
}

struct Cut {
  float T;
  int k;        // at most so many
  float p, m;   // top_p, min_p
  bool ok;
};

__device__ __forceinline__ Cut policy_cut(const PolicyArgs &a, int p) {
  float T = a.temperature, k = a.top_k, tp = a.top_p, mp = a.min_p;
  if (a.settings) {
    const float *s = a.settings + (int64_t)p * 4;
    T = s[0], k = s[1], tp = s[2], mp = s[3];
  }
  Cut c;
  c.ok = temperature_ok(T) && k >= 0 && tp >= 0 && tp <= 1 && mp >= 0 && mp <= 1;
  c.k = k >= 1 ? (int)fminf(k, (float)SIM_MAX_RES) : SIM_MAX_RES;
  if (T == 0 || tp == 0) c.k = 1;
  c.T = T == 0 ? 1.0f : T;
  c.p = tp == 0 ? 1.0f : tp, c.m = mp;
  return c;
}

__device__ __forceinline__ int policy_of(const PolicyArgs &a, int64_t s) {
  return (int)(((a.phase + s) / a.block) % a.n_pol);
}

// f(beg, end) for every run of scenarios of policy p within [from, to), in rising order.
template <class F>
__device__ __forceinline__ void for_runs(const PolicyArgs &a, int p, int64_t from, int64_t to, F f) {
  if (a.period == INT64_MAX && p > 0 && a.block > INT64_MAX / p) return;  // no scenario reaches it
  int64_t t = (int64_t)p * a.block - a.phase;
  if (from > t) {
    t += (from - t) / a.period * a.period;
    if (t <= from - a.block) t += a.period;  // at INT64_MAX, t is behind every scenario then
  }
  while (t < to) {
    const int64_t beg = max(t, from), end = a.block < to - t ? t + a.block : to;
    f(beg, end);
    if (a.period >= to - t) break;
    t += a.period;
  }
}

// ---- a row's distribution ----

// One step of merging across lanes: against lane ^ X, whose elements are taken
// in reverse order if FLIP; a lane keeps the larger ones (bound = inf) or the
// smaller (-inf).
template <int X, bool FLIP, int NV>
__device__ __forceinline__ void exchange(float (&v)[NV], float bound) {
  float q[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) q[j] = __uint_as_float(lane_xor<X>(__float_as_uint(v[FLIP ? NV - 1 - j : j])));
#pragma unroll
  for (int j = 0; j < NV; ++j) v[j] = __builtin_amdgcn_fmed3f(v[j], q[j], bound);
}

template <int S, int NV>
__device__ __forceinline__ void merge_lanes(float (&v)[NV], int g) {
  exchange<S, false>(v, (g & S) ? -kInf : kInf);
  if constexpr (S > 1) merge_lanes<S / 2>(v, g);
}

// Two rows' logits of 16 bits as whole numbers in the same order, which packed
// instructions compare at once.
typedef short key_pair __attribute__((ext_vector_type(2)));

// The larger value first.
__device__ __forceinline__ void put_in_order(float &a, float &b) {
  const float hi = fmaxf(a, b), lo = fminf(a, b);
  a = hi, b = lo;
}
__device__ __forceinline__ void put_in_order(key_pair &a, key_pair &b) {
  const key_pair hi = __builtin_elementwise_max(a, b), lo = __builtin_elementwise_min(a, b);
  a = hi, b = lo;
}

// A lane's bitonic values into falling order.
template <int NV, class F>
__device__ __forceinline__ void merge_lane(F (&v)[NV]) {
#pragma unroll
  for (int s = NV / 2; s >= 1; s /= 2)
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (!(j & s)) put_in_order(v[j], v[j + s]);
}

// Merge the sorted halves of 2 L lanes: the bitonic order, all steps the same way.
template <int L, int G, int NV>
__device__ __forceinline__ void merge_up(float (&v)[NV], int g) {
  if constexpr (L < G) {
    exchange<2 * L - 1, true>(v, (g & L) ? -kInf : kInf);
    if constexpr (L > 1) merge_lanes<L / 2>(v, g);
    merge_lane(v);
    merge_up<2 * L, G>(v, g);
  }
}

// A lane's values in falling order: the odd-even merge exchanges.
template <int NV, class F>
__device__ __forceinline__ void sort_lane(F (&v)[NV]) {
#pragma unroll
  for (int p = 1; p < NV; p *= 2)
#pragma unroll
    for (int k = p; k >= 1; k /= 2)
#pragma unroll
      for (int j = k % p; j + k < NV; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < NV && (i + j) / (2 * p) == (i + j + k) / (2 * p)) put_in_order(v[i + j], v[i + j + k]);
}

// Sort a group's G * NV values, the largest into element 0 of lane 0.
template <int G, int NV>
__device__ __forceinline__ void sort_row(float (&v)[NV], int g) {
  sort_lane<NV>(v);
  merge_up<1, G>(v, g);
}

// The larger of two values, or the smaller.
__device__ __forceinline__ float larger(float a, float b, float inf) { return __builtin_amdgcn_fmed3f(a, b, inf); }
__device__ __forceinline__ key_pair larger(key_pair a, key_pair b, float) { return __builtin_elementwise_max(a, b); }
__device__ __forceinline__ float one_of(float a, float b, bool smaller, float inf) {
  return __builtin_amdgcn_fmed3f(a, b, smaller ? -inf : inf);
}
__device__ __forceinline__ key_pair one_of(key_pair a, key_pair b, bool smaller, float) {
  return smaller ? __builtin_elementwise_min(a, b) : __builtin_elementwise_max(a, b);
}
template <int X, class F>
__device__ __forceinline__ F value_of(F v) {
  return __builtin_bit_cast(F, lane_xor<X>(__builtin_bit_cast(uint32_t, v)));
}

// The NV largest of G lanes in falling order, in every lane, from the lanes' own.
template <int L, int G, int NV, class F>
__device__ __forceinline__ void merge_top(F (&v)[NV], float inf) {
  if constexpr (L < G) {
    F q[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) q[j] = value_of<2 * L - 1>(v[NV - 1 - j]);
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = larger(v[j], q[j], inf);
    merge_lane(v);
    merge_top<2 * L, G>(v, inf);
  }
}

// v[j] = v[j + (i mod End)] for the j that End divides: a select for two elements.
template <int S, int End, int NV, class F>
__device__ __forceinline__ void pick_bits(F (&v)[NV], int i) {
  if constexpr (S < End) {
    const bool odd = __builtin_amdgcn_inverse_ballot_w64(__ballot((i & S) != 0));
#pragma unroll
    for (int j = 0; j + S < NV; j += 2 * S) v[j] = odd ? v[j + S] : v[j];
    pick_bits<2 * S, End>(v, i);
  }
}

// A bitonic order of 2 S lanes, a value each, into falling order.
template <int S, class F>
__device__ __forceinline__ F merge_across(F v, int g, float inf) {
  if constexpr (S == 0)
    return v;
  else
    return merge_across<S / 2>(one_of(v, value_of<S>(v), (g & S) != 0, inf), g, inf);
}

// The element of a group's spread row that belongs to resource r: every lane picks
// the one that its holder would, and takes the holder's.
template <int G, int NV>
__device__ __forceinline__ float spread_value(const float (&x)[NV], int r) {
  constexpr int V = piece(NV);
  float v[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) v[j] = x[j];
  pick_bits<1, NV>(v, V == NV ? r : r / (G * V) * V + r % V);
  if constexpr (G == 1) return v[0];
  const int holder = (threadIdx.x & (64 - G)) + r / V % G;
  return __uint_as_float(__builtin_amdgcn_ds_bpermute(holder * 4, __float_as_uint(v[0])));
}

// Value g in falling order of a group (G >= NV lanes, sorted each), for g < NV.  The
// last merge is of two halves of the group, which hold their lists in every
// lane: a lane takes two elements of it and goes on with one.
template <int G, int NV, class F>
__device__ __forceinline__ F top_value(F (&v)[NV], int g) {
  const float inf = some_infinity();
  constexpr int H = NV / 2;
  merge_top<1, G / 2>(v, inf);
  pick_bits<1, H>(v, g);
  const F a = v[0], b = v[H];
  const F c = larger(a, value_of<G - 1>(b), inf), d = larger(b, value_of<G - 1>(a), inf);
  return merge_across<H / 2>(one_of(c, d, (g & H) != 0, inf), g, inf);
}

// The NV largest of two rows of 16-bit logits (G >= NV lanes), the one of rank g
// in lane g: numbers with the sign bit set are turned over, so that whole numbers
// are in the floats' order (-0 before 0, which is the same logit).
template <int G, int NV>
__device__ __forceinline__ void top_of_two(const uint32_t (&x)[NV / 2], const uint32_t (&y)[NV / 2], bool f16, int g, float &own_x,
                                           float &own_y) {
  auto turned = [](key_pair k) { return k ^ ((k >> (short)15) & (short)0x7FFF); };
  key_pair v[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j)
    v[j] = turned(__builtin_bit_cast(key_pair, __builtin_amdgcn_perm(y[j / 2], x[j / 2], j % 2 ? 0x07060302u : 0x05040100u)));
  sort_lane<NV>(v);
  const uint32_t own = __builtin_bit_cast(uint32_t, turned(top_value<G>(v, g)));
  own_x = g < NV ? half_value(own & 0xFFFFu, f16) : -kInf;
  own_y = g < NV ? half_value(own >> 16, f16) : -kInf;
}

// Partial sums of a row's kept weights w = exp((l - max) / T), in 64 bits.
template <int NV>
struct RowSums {
  double c[NV];  // up to and with this lane's resource j
  double total;
  int last;      // the last resource of positive weight
  bool ok;
};

template <int G, int NV>
__device__ __forceinline__ void row_sums(const float (&x)[NV], const Cut &cut, int g, RowSums<NV> &out) {
  float m = x[0];
  int bad = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    m = fmaxf(m, x[j]);
    bad |= x[j] != x[j];
  }
  m = group_max<G>(m);
  bad = group_sum<G>(bad);
  out.ok = !bad && cut.ok && m > -kInf && m < kInf;
  const double inv = 1.0 / (double)cut.T;
  auto weight = [&](float l) { return exp(((double)l - (double)m) * inv); };
  double w[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) w[j] = x[j] > -kInf ? weight(x[j]) : 0.0;
  if (cut.k < SIM_MAX_RES || cut.p < 1) {
    float s[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) s[j] = x[j];
    sort_row<G, NV>(s, g);
    bool in[NV];  // a first part of the order
#pragma unroll
    for (int j = 0; j < NV; ++j) in[j] = s[j] > -kInf && g * NV + j < cut.k;
    if (cut.p < 1) {
      double ws[NV], mass = 0, all;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        ws[j] = mass;
        mass += in[j] ? weight(s[j]) : 0.0;
      }
      const double before = group_before<G>(mass, g, all), target = (double)cut.p * all;
#pragma unroll
      for (int j = 0; j < NV; ++j) in[j] = in[j] && (ws[j] + before < target || g * NV + j == 0);
    }
    // the last logit of the kept part, and how many of its equals belong to it
    float cutoff = kInf;
#pragma unroll
    for (int j = 0; j < NV; ++j) cutoff = in[j] ? s[j] : cutoff;
    cutoff = -group_max<G>(-cutoff);
    bool eq_in[NV];
    int ties = 0, all;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      eq_in[j] = in[j] && s[j] == cutoff;
      ties += x[j] == cutoff;
    }
    const int room = group_count<G>(eq_in);
    int rank = group_before<G>(ties, g, all);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const bool tie = x[j] == cutoff;
      if (!(x[j] > cutoff || (tie && rank < room))) w[j] = 0;
      rank += tie;
    }
  }
  double sum = 0;
  int last = -1;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (w[j] < (double)cut.m) w[j] = 0;
    sum += w[j];
    out.c[j] = sum;
    if (w[j] > 0) last = g * NV + j;
  }
  const double before = group_before<G>(sum, g, out.total);
#pragma unroll
  for (int j = 0; j < NV; ++j) out.c[j] += before;
  out.last = (int)group_umax<G>((uint32_t)(last + 1)) - 1;
}

// The same in 32 bits, where `unsure` says that a choice lies within what the
// roundings can move.  An exponent (l c - mc, below) carries four of them, so a
// weight is off by 2^-24 (4 |z| + 2) of itself and a sum by the mean of that,
// where the mean |z| of a distribution over 1024 is at most ln 1024; 22
// additions, two differences and the product with u come on top: below 2^-17
// of the whole sum, of which kMargin is twice.
constexpr float kMargin = 0x1p-16f;

template <int NV>
struct RowNear {
  float c[NV];   // within the lane
  float before;  // of the lanes before
  float total;   // NaN for a row without a distribution, or one that 32 bits cannot weigh
  bool unsure;   // of the group's lanes some may say so
};

template <int G, int NV>
__device__ __forceinline__ bool keeps_few(const Cut &cut) {
  return G >= NV && cut.k <= NV;
}

// `sorted`: own is element g of the order of the first NV, and the cut takes no more.
template <int G, int NV, bool CUT>
__device__ __forceinline__ void row_near(const float (&x)[NV], const Cut &cut, int g, RowNear<NV> &out, bool sorted = false,
                                         float own = 0) {
  const float m = sorted ? group_max<G>(own) : row_max<G>(x);
  const float c = kLog2e * (1.0f / cut.T), mc = m * c;
  bool unsure = !(fabsf(mc) < 65536.0f) && m > -kInf;
  auto weight = [&](float l) { return __builtin_amdgcn_exp2f(__builtin_fmaf(l, c, -mc)); };
  const float most = weight(m);  // 1 but for the rounding of mc, in every weight alike
  float w[NV];  // NaN in a row of -inf, and where a logit is NaN; no cut drops NaN, so the total shows it
#pragma unroll
  for (int j = 0; j < NV; ++j) w[j] = weight(x[j]);
  if (CUT && (cut.k < SIM_MAX_RES || cut.p < 1)) {
    float s[NV];
    // up to NV resources kept: every lane gets them all, from a shorter merge
    const bool top = sorted || keeps_few<G, NV>(cut);
    if (!sorted) {
#pragma unroll
      for (int j = 0; j < NV; ++j) s[j] = x[j];
      sort_lane<NV>(s);
      bool done = false;
      if constexpr (G >= NV) {
        if (top) own = top_value<G>(s, g), done = true;
        own = g < NV ? own : -kInf;
      }
      if (!done) merge_up<1, G>(s, g);
    }
    float cutoff = -kInf;  // the negative of the last kept
    uint32_t kept = 0;
    // What lies behind the first k, or is -inf, adds nothing: the whole mass lies
    // before it, so it is not kept.  Nothing lies before the first.
    if (top) {
      // lane g takes element g of the order
      bool in = g < cut.k;
      if (cut.p < 1) {
        float all;
        const float off = group_before<G>(in ? weight(own) : 0.0f, g, all) - cut.p * all;
        unsure |= fabsf(off) <= kMargin * all;
        in = off < 0;
      }
      cutoff = in ? -own : cutoff;
      kept = in;
    } else {
      const int k = cut.k - g * NV;  // so many of this lane's
      if (cut.p < 1) {
        float off[NV], mass = 0, near = kInf, all;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          off[j] = mass;
          mass += j < k ? weight(s[j]) : 0.0f;
        }
        const float before = group_before<G>(mass, g, all) - cut.p * all;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          off[j] += before;
          near = fminf(near, fabsf(off[j]));
          const bool in = off[j] < 0;
          cutoff = in ? -s[j] : cutoff;
          kept += in;
        }
        unsure |= near <= kMargin * all;
      } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          cutoff = j < k ? -s[j] : cutoff;
          kept += j < k;
        }
      }
    }
    cutoff = -group_max<G>(cutoff);
    // as many at or above it as are kept, or some of its equals are not
    uint32_t above = 0;
#pragma unroll
    for (int j = 0; j < NV; j += 4) keep_from(above, w + j, x + j, cutoff);
    kept = group_sum<G>(kept + (above << 16));
    if ((kept & 0xFFFFu) != kept >> 16) {
      int ties = 0, all;
#pragma unroll
      for (int j = 0; j < NV; ++j) ties += x[j] == cutoff;
      int rank = group_before<G>(ties, g, all);
      const int room = (int)(kept & 0xFFFFu) - ((int)(kept >> 16) - all);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const bool tie = x[j] == cutoff;
        if (tie && rank >= room) w[j] = 0;
        rank += tie;
      }
    }
  }
  if (CUT && cut.m > 0) {
    const float least = cut.m * most;
    float near = kInf;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      near = fminf(near, fabsf(w[j] - least));
      w[j] = w[j] < least ? 0.0f : w[j];  // NaN stays
    }
    unsure |= near <= 0x1p-15f * least;
  }
  float sum = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    sum += w[j];
    out.c[j] = sum;
  }
  out.before = group_before<G>(sum, g, out.total);
  if (CUT && !cut.ok) out.total = __builtin_nanf("");
  out.unsure = unsure;
}

// A block's tile: 2^log_pol policies (or scenarios) by the groups left.
struct Tile {
  int log_pol;
  int per;  // op steps of a block
};

// Draws of one row in 64 bits by a whole wavefront, i0 <= i < i1 of its policy's
// scenarios: f(i) is the random number's index, or negative when there is none
// left; u and place are the row's.
template <int NV, class F>
__device__ __noinline__ void draw_sure(const PolicyArgs &a, int pol, int64_t at_row, const float *u, uint16_t *place, int i0,
                                       int i1, F scenario) {
  const int lane = threadIdx.x & 63;
  float x[NV];
  load_row<NV>(a.logits, a.dtype, at_row, lane * NV, a.n_res, x);
  RowSums<NV> row;
  row_sums<64, NV>(x, policy_cut(a, pol), lane, row);
  for (int i = i0; i < i1; ++i) {
    const int64_t s = scenario(i);
    if (s < 0) return;
    const float us = u[s];
    const double target = (double)fmaxf(us, 0.0f) * row.total;
    bool in[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) in[j] = row.c[j] <= target;
    const int n = min(group_count<64>(in), row.last);
    if (lane == 0) place[s] = row.ok && us == us ? (uint16_t)n : kNoPlace;
  }
}

// The scenario of a policy that has at most one; n_scen when it has none.
__device__ __forceinline__ int64_t only_scenario(const PolicyArgs &a, int64_t pol, int64_t n_scen) {
  const int64_t s = pol >= a.phase ? pol - a.phase : pol - a.phase + a.period;
  return s < n_scen ? s : n_scen;
}

// Where a group's row kernel stands: the policies of its tile side by side, its ops in steps of nv.
template <int G>
struct RowWalk {
  int pol, np, nv, steps;  // steps of this group; 0 without a policy
  int64_t v0;

  __device__ __forceinline__ RowWalk(const PolicyArgs &a, Tile t, uint32_t block) {
    const int grp = threadIdx.x / G;
    np = 1 << t.log_pol, nv = (kThreads / G) >> t.log_pol;
    const uint32_t pol_tiles = ((uint32_t)a.n_pol + np - 1) >> t.log_pol, v_tile = block / pol_tiles;
    const uint32_t at = ((block - v_tile * pol_tiles) << t.log_pol) + (grp & (np - 1));
    v0 = (int64_t)v_tile * nv * t.per + (grp >> t.log_pol);
    const bool live = at < (uint32_t)a.n_pol;
    pol = live ? (int)at : 0;
    steps = live ? (int)max((int64_t)0, min((int64_t)t.per, (a.n_ops - v0 + nv - 1) / nv)) : 0;
  }
};

// One scenario a row at most: a group of lanes works a row out in 32 bits and
// draws.  A draw that lies within the roundings of a border (63 borders at 64
// resources, 2^-16 of the sum to either side: two in a thousand) is done again in
// 64 bits by the whole wavefront, so that every answer is the 64-bit one.  Bound
// by vector instructions: 1024 x 6624 rows of 48 bf16 take 0.26 ms uncut and 0.41
// ms with top_k 8 and top_p 0.9 (the eight largest of two rows at once, the next
// two already loading; 316 instructions a row and wavefront, 4 clocks each, are all
// of the time; 0.54 ms with a sort for each, 3.5 ms with all sums in 64 bits and the
// cut searched bit by bit).  The registers of the 64-bit way count for the whole
// kernel: rows of over 512 resources run two wavefronts a SIMD.
template <int G, int NV, bool CUT>
__global__ __launch_bounds__(kThreads) void k_policy_sample_one(PolicyArgs a, int64_t n_scen, const float *u, int64_t ld_u,
                                                                uint16_t *place, int64_t ld_place, Tile t,
                                                                uint32_t first) {
  constexpr int kWide = G * NV > 64 ? G * NV / 64 : 1;
  const int g = threadIdx.x % G;
  const RowWalk<G> walk(a, t, first + blockIdx.x);
  const Cut cut = policy_cut(a, walk.pol);
  const int64_t s = only_scenario(a, walk.pol, n_scen);
  const int steps = s < n_scen ? walk.steps : 0;
  // unsigned: what is past the last op may wrap, and is not used
  uint64_t at_row = (uint64_t)walk.pol * a.ld_pol + (uint64_t)walk.v0 * a.ld_op, at_u = (uint64_t)walk.v0 * ld_u + s,
           at_place = (uint64_t)walk.v0 * ld_place + s;
  auto load = [&](bool act, float (&x)[NV], float &now) {
    now = act ? u[at_u] : 0.0f;
    load_row<NV>(a.logits, a.dtype, act ? (int64_t)at_row : 0, g * NV, a.n_res, x);
  };
  auto draw = [&](bool act, const float (&x)[NV], float now, bool sorted, float own) {
    RowNear<NV> row;
    row_near<G, NV, CUT>(x, cut, g, row, sorted, own);
    // sure where as many sums lie below the target's margin as below its end, and not all
    const float margin = kMargin * row.total, mid = fmaxf(now, 0.0f) * row.total - row.before, from = mid - margin, to = mid + margin;
    uint32_t below = 0, upto = 0;
#pragma unroll
    for (int j = 0; j < NV; j += 4) {
      count_le(below, row.c + j, from);
      count_le(upto, row.c + j, to);
    }
    const uint32_t n = group_sum<G>(row.unsure + (below << 10) + (upto << 21));
    const bool drawn = act && (row.total > 0 || (n & 0x3FFu)) && now == now;
    const bool redo = drawn && ((n & 0x3FFu) || (n >> 10 & 0x7FFu) != n >> 21 || n >> 21 == G * NV);
    if (act && g == 0 && !redo) place[at_place] = drawn ? (uint16_t)(n >> 21) : kNoPlace;
    for (uint64_t left = __ballot(redo && g == 0); left; left &= left - 1) {
      const int l = __builtin_ctzll(left);
      draw_sure<kWide>(PolicyArgs(a), from_lane(walk.pol, l), (int64_t)from_lane(at_row, l), u + from_lane(at_u, l),
                       place + from_lane(at_place, l), 0, 1, [](int) { return (int64_t)0; });
    }
  };
  auto next = [&] { at_row += walk.nv * a.ld_op, at_u += walk.nv * ld_u, at_place += walk.nv * ld_place; };
  int i = 0;
  if constexpr (CUT && G >= NV) {
    // two rows at a time while every group has two that keep few, the next two already loading
    auto pairs = [&](auto type) {
      constexpr bool f16 = type;
      uint32_t w[2][NV / 2];
      float now[2];
      auto load_two = [&](int i) {
        uint64_t row = at_row, of_u = at_u;
#pragma unroll
        for (int k = 0; k < 2; ++k, row += walk.nv * a.ld_op, of_u += walk.nv * ld_u) {
          const bool act = i + k < steps;
          now[k] = act ? u[of_u] : 0.0f;
          load_bits<NV>(a.logits, f16, act ? (int64_t)row : 0, g * NV, a.n_res, w[k]);
        }
      };
      load_two(0);
      while (__any(i + 1 < steps)) {
        float x[NV], y[NV], own_x, own_y;
        const float now_x = now[0], now_y = now[1];
        const bool act_x = i < steps, act_y = i + 1 < steps;
        values_of<NV>(w[0], f16, x);
        values_of<NV>(w[1], f16, y);
        top_of_two<G, NV>(w[0], w[1], f16, g, own_x, own_y);
        const uint64_t at[3] = {at_row, at_u, at_place};
        next(), next();
        i += 2;
        load_two(i);
        const uint64_t then[3] = {at_row, at_u, at_place};
        at_row = at[0], at_u = at[1], at_place = at[2];
        draw(act_x, x, now_x, true, own_x);
        next();
        draw(act_y, y, now_y, true, own_y);
        at_row = then[0], at_u = then[1], at_place = then[2];
      }
    };
    if (__all(steps == 0 || keeps_few<G, NV>(cut))) {
      if (a.dtype == SIM_F16) pairs(std::true_type{});
      if (a.dtype == SIM_BF16) pairs(std::false_type{});
    }
  }
  for (; __any(i < steps); ++i, next()) {
    float x[NV], now;
    load(i < steps, x, now);
    draw(i < steps, x, now, false, 0.0f);
  }
}

// Scenario i of a policy (negative: none left): `first` of them from `beg` on, then
// runs of `block` at t + j * period.  Lengths from 2^30 on are beyond any i.
struct PolicyScenarios {
  int64_t beg, t, period, n_scen;
  uint32_t first, block;

  __device__ __forceinline__ PolicyScenarios(const PolicyArgs &a, int pol, int64_t n) {
    n_scen = n, period = a.period, block = (uint32_t)min(a.block, (int64_t)1 << 30);
    beg = n, first = 1u << 30;
    if (a.period == INT64_MAX && pol > 0 && a.block > INT64_MAX / pol) return;  // no scenario reaches it
    t = (int64_t)pol * a.block - a.phase;
    if (t <= -a.block) t += a.period;  // at INT64_MAX, t is behind every scenario then
    beg = max(t, (int64_t)0);
    if (t < 0) first = (uint32_t)min(a.block + t, (int64_t)1 << 30);
    else first = block;
    if (a.period >= n - t && first < 1u << 30) period = 0;  // one run
  }
  __device__ __forceinline__ int64_t operator()(int i) const {
    if ((uint32_t)i < first) return beg + i < n_scen ? beg + i : -1;
    const uint32_t k = i - first, j = k / block;
    // beyond 2^41 only the next run can begin within a batch
    if (period == 0 || (j > 0 && period > (int64_t)1 << 41)) return -1;
    const int64_t s = t + (j + 1) * period + (k - j * block);
    return s < n_scen ? s : -1;
  }
};

// Some scenarios a row: a group works a row out as above, puts its partial
// sums into LDS, and every lane draws another scenario: log2 of the row's
// length steps down the sums, sure where both neighbours of the place found are
// more than the margin away (sums that the roundings put out of order are
// nearer to each other than that).  12 x 6624 rows of 48 bf16, cut, 32 draws each:
// 32 us.
template <int G, int NV, bool CUT>
__global__ __launch_bounds__(kThreads) void k_policy_sample_few(PolicyArgs a, int64_t n_scen, const float *u, int64_t ld_u,
                                                                uint16_t *place, int64_t ld_place, Tile t,
                                                                uint32_t first) {
  constexpr int kWide = G * NV > 64 ? G * NV / 64 : 1, kRow = G * NV;
  __shared__ float lds[kThreads * NV];
  const int g = threadIdx.x % G;
  float *c = lds + threadIdx.x / G * kRow;
  const RowWalk<G> walk(a, t, first + blockIdx.x);
  const Cut cut = policy_cut(a, walk.pol);
  const PolicyScenarios scenario(a, walk.pol, n_scen);
  uint64_t at_row = (uint64_t)walk.pol * a.ld_pol + (uint64_t)walk.v0 * a.ld_op, at_u = (uint64_t)walk.v0 * ld_u,
           at_place = (uint64_t)walk.v0 * ld_place;
  for (int i = 0; __any(i < walk.steps); ++i, at_row += walk.nv * a.ld_op, at_u += walk.nv * ld_u, at_place += walk.nv * ld_place) {
    const bool act = i < walk.steps;
    int64_t s = act ? scenario(g) : -1;
    float now = s >= 0 ? u[at_u + s] : 0.0f;
    float x[NV];
    load_row<NV>(a.logits, a.dtype, act ? (int64_t)at_row : 0, g * NV, a.n_res, x);
    RowNear<NV> row;
    row_near<G, NV, CUT>(x, cut, g, row);
    const bool unsure = group_umax<G>((uint32_t)row.unsure) != 0, ok = row.total > 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) c[g * NV + j] = row.c[j] + row.before;
    wave_order();
    const float margin = kMargin * row.total;
    if (unsure) s = -1;  // the whole row, below
    for (int d = g; __any(s >= 0); d += G) {
      const int64_t at = s;
      const float us = now;
      s = s >= 0 ? scenario(d + G) : -1;
      now = s >= 0 ? u[at_u + s] : 0.0f;
      const float target = fmaxf(us, 0.0f) * row.total;
      int n = 0;
#pragma unroll
      for (int h = kRow / 2; h >= 1; h /= 2) n += c[n + h - 1] <= target ? h : 0;
      const float gap = fminf(c[n] - target, n ? target - c[n - 1] : kInf);
      const bool redo = at >= 0 && ok && us == us && !(gap > margin);
      if (at >= 0 && !redo) place[at_place + at] = ok && us == us ? (uint16_t)n : kNoPlace;
      for (uint64_t left = __ballot(redo); left; left &= left - 1) {
        const int l = __builtin_ctzll(left);
        const int64_t rs = from_lane(at, l);
        draw_sure<kWide>(PolicyArgs(a), from_lane(walk.pol, l), (int64_t)from_lane(at_row, l), u + from_lane(at_u, l), place + from_lane(at_place, l),
                         0, 1, [=](int) { return rs; });
      }
    }
    for (uint64_t left = __ballot(act && unsure && g == 0); left; left &= left - 1) {
      const int l = __builtin_ctzll(left), pol = from_lane(walk.pol, l);
      draw_sure<kWide>(PolicyArgs(a), pol, (int64_t)from_lane(at_row, l), u + from_lane(at_u, l), place + from_lane(at_place, l), 0, INT32_MAX,
                       PolicyScenarios(a, pol, n_scen));
    }
    wave_order();
  }
}

// A row's weights in 32 bits, e = 2^(x c - mc) with c = log2 e / T and mc the
// rounded product of c and the maximum m: one multiply-add and the machine's
// 2^x.  What mc's rounding leaves in the exponent is the same for the whole row
// (`shift`), so that ratios do not have it.  Where mc is so large that `shift`
// might not be small, the difference is taken first.
template <int NV>
__device__ __forceinline__ void row_weights(const float (&x)[NV], float m, float c, float (&e)[NV], float &shift) {
  const float mc = m * c;
  const bool far = !(fabsf(mc) < 65536.0f);
  shift = 0;
  if (far) {
#pragma unroll
    for (int j = 0; j < NV; ++j) e[j] = x[j] == -kInf ? 0.0f : __builtin_amdgcn_exp2f((x[j] - m) * c);  // inf - inf: NaN
  } else {
    shift = __builtin_fmaf(m, c, -mc);
#pragma unroll
    for (int j = 0; j < NV; ++j) e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], c, -mc));
  }
}

// (l - m) / T from 1 / T, where l - m may be beyond the largest number: half of it
// is not, and halves are exact.
__device__ __forceinline__ float over(float l, float m, float inv) { return __builtin_fmaf(l, 0.5f, -0.5f * m) * (2 * inv); }

// log2 p: the machine's logarithm takes a subnormal number for 0.
__device__ __forceinline__ float log2_of(float p) {
  const bool low = p < 0x1p-126f;
  return __builtin_amdgcn_logf(low ? p * 0x1p32f : p) - (low ? 32.0f : 0.0f);
}

// A row's softmax in 32 bits.
template <int NV>
struct RowExp {
  float e[NV];
  float sum;     // of e; NaN for an invalid row, 0 for an empty one
  float m, inv;  // the maximum, 1 / T
  float shift;

  // log pi of a resource with logit l: (l - m) / T is off by 2^-24 of 3 |z|.
  __device__ __forceinline__ float log_sum() const { return kLn2 * (__builtin_amdgcn_logf(sum) - shift); }
  __device__ __forceinline__ float z(float l) const { return over(l, m, inv); }
};

template <int G, int NV>
__device__ __forceinline__ void row_exp(const float (&x)[NV], float T, RowExp<NV> &o) {
  o.m = row_max<G>(x);
  o.inv = 1.0f / T;
  row_weights<NV>(x, o.m, o.inv * kLog2e, o.e, o.shift);
  float s = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) s += o.e[j];
  o.sum = group_sum<G>(s);
  if (T == 0 || !temperature_ok(T)) o.sum = __builtin_nanf("");
}

// Log-probabilities row by row: a group of lanes works through a scenario's
// rows of a chunk of the ops, the next row loading meanwhile.  Memory and vector
// instructions (two thirds of them one unpacking, multiply-add, 2^x and addition an
// element) are even: 1024 x 6624 rows of 48 bf16 take 148 us, 4.5 TB/s (169
// without the load ahead).
template <int G, int NV>
__global__ __launch_bounds__(kThreads) void k_policy_logp(PolicyArgs a, int64_t n_scen, const uint16_t *place,
                                                          int64_t ld_place, double *part, Tile t, uint32_t first) {
  __shared__ double red[kThreads / G];
  const int g = threadIdx.x % G, grp = threadIdx.x / G;
  const int ns = 1 << t.log_pol, nv = (kThreads / G) >> t.log_pol;
  const int64_t scen_tiles = (n_scen + ns - 1) / ns;
  const int64_t block = first + blockIdx.x, chunk = block / scen_tiles, s0 = block % scen_tiles * ns, s = s0 + (grp & (ns - 1));
  double sum = 0;
  if (s < n_scen) {
    const int pol = policy_of(a, s);
    const float T = policy_temperature(a, pol);
    const int64_t v0 = chunk * nv * t.per + (grp >> t.log_pol);
    uint64_t at_row = (uint64_t)pol * a.ld_pol + (uint64_t)v0 * a.ld_op, at_place = (uint64_t)v0 * ld_place + s;
    const int steps = (int)min((int64_t)t.per, (a.n_ops - v0 + nv - 1) / nv);
    by_type(a.dtype, [&](auto type) {
      RowWords<type, G, NV> next;
      int to = kNoPlace;
      if (steps > 0) next.load(a.logits, at_row, g, a.n_res), to = place[at_place];
      for (int i = 0; i < steps; ++i) {
        float x[NV];
        next.values(x);
        const int to_now = to;
        at_row += nv * a.ld_op, at_place += nv * ld_place;
        if (i + 1 < steps) next.load(a.logits, at_row, g, a.n_res), to = place[at_place];
        RowExp<NV> row;
        row_exp<G, NV>(x, T, row);
        float l = spread_value<G, NV>(x, to_now);  // the place's logit
        l = to_now < a.n_res ? l : -kInf;
        sum += (double)(row.sum != row.sum ? row.sum : l == -kInf ? -kInf : row.z(l) - row.log_sum());
      }
    });
  }
  if (g == 0) red[grp] = sum;
  __syncthreads();
  if (threadIdx.x < ns) {
    const int64_t so = s0 + threadIdx.x;
    double all = 0;
    for (int i = 0; i < nv; ++i) all += red[(i << t.log_pol) + threadIdx.x];
    if (so < n_scen) part[chunk * n_scen + so] = all;
  }
}

// The smaller of two pairs of 16 bits.
__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b) {
  typedef unsigned short pair __attribute__((ext_vector_type(2)));
  pair x, y;
  __builtin_memcpy(&x, &a, 4);
  __builtin_memcpy(&y, &b, 4);
  x = __builtin_elementwise_min(x, y);
  __builtin_memcpy(&a, &x, 4);
  return a;
}

// The larger.
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
  return ~min_pair(~a, ~b);
}

// A lane's eight scenarios s .. s + 7 of [beg, end) are one load of 16 bytes, at
// any even address.  A lane that has fewer takes the last eight instead and
// shares some with the lane before; a lane that has none leaves its values as
// they are.  Only a range of under eight is read one by one, 65535 (or 0) behind
// its end.  Nothing here reads what was loaded, so several loads stay in flight.
template <int E, class I>
__device__ __forceinline__ I first_of(I s, I beg, I end) {
  return end - beg >= E ? min(s, end - E) : s;
}

template <int E, class I>
__device__ __forceinline__ void load_places(const uint16_t *p, I s, I beg, I end, uint32_t (&w)[(E + 1) / 2]) {
  if (E == 8 && end - beg >= E) {
    if (s < end) __builtin_memcpy(w, p + min(s, end - E), sizeof(w));
    return;
  }
#pragma unroll
  for (int i = 0; i < (E + 1) / 2; ++i) {
    const uint32_t lo = s + 2 * i < end ? p[s + 2 * i] : kNoPlace;
    const uint32_t hi = 2 * i + 1 < E && s + 2 * i + 1 < end ? p[s + 2 * i + 1] : kNoPlace;
    w[i] = lo | hi << 16;
  }
}

template <int N>
__device__ __forceinline__ uint32_t place_at(const uint32_t (&w)[N], int e) {
  return (w[e / 2] >> (16 * (e & 1))) & 0xFFFFu;
}

// A batch cut into pieces of at most `span` scenarios of one policy: piece t
// of run j (the scenarios up to the next change of policy).
struct Pieces {
  int64_t first, span;     // scenarios of run 0 before the batch; most scenarios of a piece
  uint32_t per_run, n;     // pieces of a run, of the batch
  int32_t pol;             // policy of run 0
};

struct Piece {
  int64_t beg, end;
  int pol;
};

__device__ __forceinline__ Piece piece_of(const PolicyArgs &a, const Pieces &ps, int64_t n_scen, uint32_t i) {
  const uint32_t j = i / ps.per_run, t = i - j * ps.per_run;
  const int64_t beg = j ? a.block - ps.first + (int64_t)(j - 1) * a.block : 0;  // j > 0: block is below the batch's end
  const int64_t len = j ? a.block : a.block - ps.first;
  const int64_t end = len < n_scen - beg ? beg + len : n_scen;
  Piece p;
  p.beg = beg + t * ps.span;
  p.end = ps.span < end - p.beg ? p.beg + ps.span : end;
  const uint32_t q = ps.pol + j % (uint32_t)a.n_pol;
  p.pol = (int)(q >= (uint32_t)a.n_pol ? q - a.n_pol : q);
  return p;
}

// Log-probabilities where many scenarios share a row.  A block takes a piece
// of up to E scenarios a thread and a chunk of the ops: it puts the logarithms
// of as many rows as it has groups of lanes into LDS, then every thread adds up
// its scenarios' entries, one 16-byte load of eight places per row.  Entry
// n_res stands for a place that is no resource.  Bound by memory (the times stand
// at logp_runs).  32 terms are added in 32 bits, the rest in 64, and a chunk's sum
// is rounded once for the join: no term is above 0, so that each rounding is off by
// 2^-24 of the whole sum at most, as the result's own is.
template <int G, int NV, int E>
__global__ __launch_bounds__(kThreads) void k_policy_logp_runs(PolicyArgs a, int64_t n_scen, const uint16_t *place,
                                                               int64_t ld_place, float *part, Pieces ps, int ops_per,
                                                               uint32_t first) {
  constexpr int kRows = kThreads / G;  // rows of one table
  constexpr int kAhead = 4;            // rows whose places are loaded together
  __shared__ float table[kRows * (G * NV + 1)];
  const int g = threadIdx.x % G, grp = threadIdx.x / G, R = a.n_res;
  const uint32_t block = first + blockIdx.x, chunk = block / ps.n;
  const Piece pc = piece_of(a, ps, n_scen, block - chunk * ps.n);
  if (pc.beg >= pc.end) return;
  const float T = policy_temperature(a, pc.pol);
  const int len = (int)(pc.end - pc.beg), s0 = threadIdx.x * E;
  const int v_end = (int)min((int64_t)a.n_ops, (chunk + 1) * (int64_t)ops_per);
  double total[E] = {};
  for (int v0 = (int)(chunk * (int64_t)ops_per); v0 < v_end; v0 += kRows) {
    const int rows = min(kRows, v_end - v0);
    uint32_t at[kAhead][(E + 1) / 2] = {};
    auto load = [&](int r) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        load_places<E>(place + (int64_t)(v0 + min(r + i, rows - 1)) * ld_place + pc.beg, s0, 0, len, at[i]);
    };
    load(0);
    if (grp < rows) {
      float x[NV];
      load_row<NV>(a.logits, a.dtype, pc.pol * a.ld_pol + (v0 + grp) * a.ld_op, g * NV, R, x);
      RowExp<NV> row;
      row_exp<G, NV>(x, T, row);
      const float ls = row.log_sum();
      float *t = table + grp * (R + 1);
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (g * NV + j < R) t[g * NV + j] = row.sum != row.sum ? row.sum : x[j] == -kInf ? -kInf : row.z(x[j]) - ls;
      if (g == 0) t[R] = row.sum != row.sum ? row.sum : -kInf;
    }
    __syncthreads();
    float sum[E] = {};  // at most 32 terms, then 64 bits
    for (int r = 0; r < rows; r += kAhead) {
      uint32_t now[kAhead][(E + 1) / 2];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
#pragma unroll
        for (int e = 0; e < (E + 1) / 2; ++e) now[i][e] = min_pair(at[i][e], (uint32_t)R * 0x10001u);
      if (r + kAhead < rows) load(r + kAhead);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (r + i >= rows) break;
        const float *t = table + (r + i) * (R + 1);
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += t[place_at(now[i], e)];
      }
      if (((r + kAhead) & 31) == 0 || r + kAhead >= rows) {
#pragma unroll
        for (int e = 0; e < E; ++e) total[e] += (double)sum[e], sum[e] = 0;
      }
    }
    __syncthreads();
  }
  float *to = part + chunk * n_scen + pc.beg + first_of<E>(s0, 0, len);
  const int have = len >= E ? s0 < len ? E : 0 : len - s0;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e < have) to[e] = (float)total[e];
}

constexpr int kJoinScen = 16;

// The chunks' sums joined in order: sixteen lanes a scenario.
template <class F>
__global__ __launch_bounds__(kThreads) void k_policy_join(const F *part, int64_t chunks, int64_t n_scen, float *logp, uint32_t first) {
  constexpr int kScen = kJoinScen, kLanes = kThreads / kScen;
  __shared__ double red[kLanes][kScen];
  const int64_t s = (int64_t)(first + blockIdx.x) * kScen + threadIdx.x % kScen;
  const int lane = threadIdx.x / kScen;
  double sum = 0;
  if (s < n_scen)
    for (int64_t c = lane; c < chunks; c += kLanes) sum += (double)part[c * n_scen + s];
  red[lane][threadIdx.x % kScen] = sum;
  __syncthreads();
  if (lane || s >= n_scen) return;
  for (int i = 1; i < kLanes; ++i) sum += red[i][threadIdx.x];
  logp[s] = (float)sum;
}

// ---- draws where many scenarios share a row ----

// The lowest u >= 0 of float32 whose product with `total`, rounded to 64 bits,
// is not below c: u >= border is then the same as u * total >= c.
__device__ __forceinline__ float border(double c, double total, double inv) {
  if (!(c > 0)) return 0;
  const float f = (float)(c * inv);
  const float up = __uint_as_float(__float_as_uint(f) + 1);
  if ((double)f * total < c) return up;
  const float down = f > 0 ? __uint_as_float(__float_as_uint(f) - 1) : 0.0f;
  return (double)down * total >= c ? down : f;
}

template <int E, class I>
__device__ __forceinline__ void load_numbers(const float *p, I s, I beg, I end, float (&u)[E]) {
  if (end - beg >= E) {
    if (s < end) __builtin_memcpy(u, p + min(s, end - E), sizeof(u));
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) u[e] = s + e < end ? p[s + e] : 0.0f;
  }
}

template <int E, class I>
__device__ __forceinline__ void store_places(uint16_t *p, I s, I beg, I end, const uint32_t (&at)[E]) {
  if (end - beg >= E) {
    typedef uint32_t words __attribute__((ext_vector_type(E / 2), aligned(2)));
    words w;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) w[i] = at[2 * i] | at[2 * i + 1] << 16;
    if (s < end) __builtin_nontemporal_store(w, (words *)(p + min(s, end - E)));
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (s + e < end) p[s + e] = (uint16_t)at[e];
  }
}

// WR wavefronts draw one row's placements for one piece.  The row's n_res - 1
// borders go to LDS as float32, in the order of a binary tree's levels (node k
// has 2k and 2k + 1 below it), so that a level's entries lie in consecutive
// banks and a draw is log2 n_res steps k = 2k + (u >= tree[k]), three vector
// instructions and one LDS read each.  Bound by memory: 20000 rows of 64, 16384
// scenarios each, take 331 us (5.9 TB/s); with steps of four instructions, and
// stores that stay in the caches, 416.
template <int NV, int WR>
__global__ __launch_bounds__(kThreads) void k_policy_sample_runs(PolicyArgs a, int64_t n_scen, const float *u,
                                                                 int64_t ld_u, uint16_t *place, int64_t ld_place,
                                                                 Pieces ps, int levels, uint32_t first) {
  constexpr int E = 8, kRows = kThreads / 64 / WR, kNodes = 64 * NV;  // E: consecutive scenarios of a lane
  __shared__ float lds[kRows * kNodes];
  __shared__ int lds_ok[kRows];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, of_row = wave % WR;
  float *tree = lds + wave / WR * kNodes;
  const uint32_t block = first + blockIdx.x, vb = block / ps.n;
  const int64_t v = (int64_t)vb * kRows + wave / WR;
  if (v >= a.n_ops) return;  // with WR > 1 a block has one row
  const Piece pc = piece_of(a, ps, n_scen, block - vb * ps.n);
  if (pc.beg >= pc.end) return;
  const float *pu = u + v * ld_u + pc.beg;
  uint16_t *pp = place + v * ld_place + pc.beg;
  const int len = (int)(pc.end - pc.beg);
  int s = (of_row * 64 + lane) * E;
  float us[E] = {};
  load_numbers<E>(pu, s, 0, len, us);
  if (of_row == 0) {
    float x[NV];
    load_row<NV>(a.logits, a.dtype, pc.pol * a.ld_pol + v * a.ld_op, lane * NV, a.n_res, x);
    RowSums<NV> row;
    row_sums<64, NV>(x, policy_cut(a, pc.pol), lane, row);
    const double inv = 1.0 / row.total;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const uint32_t i = lane * NV + j + 1;  // border i - 1: between resources i - 1 and i
      if (i < 1u << levels) {
        const int z = __builtin_ctz(i);
        tree[(1u << (levels - 1 - z)) + (i >> (z + 1))] = (int)i - 1 < row.last ? border(row.c[j], row.total, inv) : kInf;
      }
    }
    if (lane == 0) lds_ok[wave / WR] = row.ok;
  }
  if (WR > 1)
    __syncthreads();
  else
    wave_order();
  const bool ok = lds_ok[wave / WR];
  while (s - lane * E < len) {
    uint32_t k[E];
    bool nan = !ok;
    float at[E], keep[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (e & 1) nan |= __builtin_isunordered(us[e - 1], us[e]);
      keep[e] = us[e];
      at[e] = __builtin_amdgcn_fmed3f(us[e], 0.0f, 2.0f);  // above 1 all are the same
      k[e] = 1;
    }
    const int now = s;
    s += WR * 64 * E;
    load_numbers<E>(pu, s, 0, len, us);
    for (int l = 0; l < levels; ++l) {
      float t[E];
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] = tree[k[e]];
#pragma unroll
      for (int e = 0; e < E; e += 4) descend(k + e, at + e, t + e);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) k[e] -= 1u << levels;
    if (__any(nan)) {
#pragma unroll
      for (int e = 0; e < E; ++e) k[e] = ok && keep[e] == keep[e] ? k[e] : kNoPlace;
    }
    store_places<E>(pp, now, 0, len, k);
  }
}

// The gradient of a row from its softmax and what every resource received.  T
// divides last: at 2^-126 a product before it would be infinite.
template <int G, int NV>
__device__ __forceinline__ void row_grad(const RowExp<NV> &row, const float (&x)[NV], const float (&h)[NV], float (&out)[NV]) {
  float w = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) w += x[j] == -kInf ? 0.0f : h[j];
  w = group_sum<G>(w);
  const bool nan = row.sum != row.sum;
  const float k = nan ? row.sum : row.sum > 0 ? -w / row.sum : 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) out[j] = nan ? row.sum : x[j] == -kInf ? 0.0f : __builtin_fmaf(row.e[j], k, h[j]) * row.inv;
}

// Few scenarios a row (ONE: at most one): a group of lanes takes them one after
// another, the next row loading meanwhile.  Bound by memory: 1024 x 6624 rows of
// 48 bf16 take 273 us, 4.8 TB/s in and out (304 without the load ahead).
template <int G, int NV, bool ONE>
__global__ __launch_bounds__(kThreads) void k_policy_grad(PolicyArgs a, int64_t n_scen, const uint16_t *place,
                                                          int64_t ld_place, const float *weight, PolicyOut grad, Tile t,
                                                          uint32_t first) {
  const int g = threadIdx.x % G, grp = threadIdx.x / G;
  const int np = 1 << t.log_pol, nv = (kThreads / G) >> t.log_pol;
  const uint32_t block = first + blockIdx.x, pol_tiles = ((uint32_t)a.n_pol + np - 1) >> t.log_pol, v_tile = block / pol_tiles;
  const uint32_t pol = ((block - v_tile * pol_tiles) << t.log_pol) + (grp & (np - 1));
  const int64_t v0 = (int64_t)v_tile * nv * t.per + (grp >> t.log_pol);
  if (pol >= (uint32_t)a.n_pol) return;
  const float T = policy_temperature(a, (int)pol);
  uint64_t at_row = (uint64_t)pol * a.ld_pol + (uint64_t)v0 * a.ld_op, at_grad = (uint64_t)pol * grad.ld_pol + (uint64_t)v0 * grad.ld_op,
           at_place = (uint64_t)v0 * ld_place;
  const int64_t only = ONE ? only_scenario(a, pol, n_scen) : 0;
  const float w_only = ONE && only < n_scen ? weight[only] : 0.0f;
  const int steps = (int)min((int64_t)t.per, (a.n_ops - v0 + nv - 1) / nv);
  by_type(a.dtype, [&](auto type) {
    RowWords<type, G, NV> next;
    int to = kNoPlace;
    auto load = [&] {
      next.load(a.logits, at_row, g, a.n_res);
      if (ONE && only < n_scen) to = place[at_place + only];
    };
    if (steps > 0) load();
    for (int i = 0; i < steps; ++i, at_grad += nv * grad.ld_op) {
      float x[NV], h[NV], out[NV];
      next.values(x);
      const int at = ONE ? spread_at<G, NV>(to, g) : -1;
      const uint64_t at_scen = at_place;
      at_row += nv * a.ld_op, at_place += nv * ld_place;
      if (i + 1 < steps) load();
      RowExp<NV> row;
      row_exp<G, NV>(x, T, row);
      if (ONE) {
#pragma unroll
        for (int j = 0; j < NV; ++j) h[j] = j == at ? w_only : 0.0f;
      } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) h[j] = 0;
        for_runs(a, (int)pol, 0, n_scen, [&](int64_t beg, int64_t end) {
          for (int64_t s = beg; s < end; ++s) {
            const int mine = spread_at<G, NV>(place[at_scen + s], g);
            const float w = weight[s];
#pragma unroll
            for (int j = 0; j < NV; ++j) h[j] += j == mine ? w : 0.0f;
          }
        });
      }
      row_grad<G, NV>(row, x, h, out);
      store_spread<G, NV>(grad.p, type, at_grad, g, a.n_res, out);
    }
  });
}

// The largest magnitude of each policy's finite weights, for the grid below:
// peak[p][part], of the scenarios whose number in their policy lies in every
// `parts`th block of threads.
__global__ __launch_bounds__(kThreads) void k_policy_peak(PolicyArgs a, int64_t n_scen, const float *weight, uint32_t parts, float *peak,
                                                          uint32_t first) {
  __shared__ float red[kThreads / 64];
  const uint32_t block = first + blockIdx.x, pol = block / parts, threads = blockDim.x;
  const PolicyScenarios scenario(a, (int)pol, n_scen);
  float m = 0;
  for (uint32_t i = (block - pol * parts) * threads + threadIdx.x; i < n_scen; i += parts * threads) {
    const int64_t s = scenario((int)i);
    if (s < 0) break;
    const float w = fabsf(weight[s]);
    m = w < kInf ? fmaxf(m, w) : m;
  }
  m = group_max<64>(m);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x) return;
  for (uint32_t i = 1; i < threads / 64; ++i) m = fmaxf(m, red[i]);
  peak[block] = m;
}

// A block of the kernel below has four wavefronts.  Together (WR = 4) they take
// `rows` ops of a policy at once, so that a weight is loaded and rounded once for
// several rows, with `columns` columns for a row's table: at most 32 KB of LDS in
// all.  Alone (WR = 1) each takes a row of its own.
template <int NV, int WR>
struct GradShape {
  static constexpr int kGroups = 4 / WR;  // of wavefronts in a block
  static constexpr int kRows = WR == 1 || NV > 2 ? 1 : 4 / NV;
  static constexpr int kColumns = WR == 1 ? 16 / NV : NV <= 4 ? 16 : 64 / NV;
  static size_t lds(int n_res) { return (size_t)n_res * kGroups * kRows * kColumns * 8; }
};

// The gradient where many scenarios share a row.  Weights are added up by
// resource in a table of LDS of float64 for every row.  A weight is first
// rounded to a grid on which every sum of a split is exact, so that the lanes'
// order does not matter and any of them may add to any entry: with the largest
// weight of the row's policy below 2^E and fewer than 2^L scenarios, multiples of
// 2^(E + L - 53) (an error of at most 2^-38 of the largest at 16384 scenarios,
// 2^-30 at most).
// Columns keep down how many lanes meet in one entry.  (An LDS addition of
// float64 takes 9 clocks for a wavefront with 16 columns or more, 17 with 8, 20
// with 4; one of float32 takes 193, 3 a lane.)  Then a wavefront adds up a row's
// columns and goes on to its gradient.  With several splits of the batch a row's
// sums go to `part`, and the next kernel joins them.  Bound by memory: 20000 rows
// of 64, 16384 scenarios each, take 126 us with the weights' peaks, 5.3 TB/s; with
// a row a block 176, without the grid (columns for half a wavefront) 228.
template <int NV, int WR>
__global__ __launch_bounds__(kThreads) void k_policy_grad_runs(PolicyArgs a, int64_t n_scen, const uint16_t *place,
                                                               int64_t ld_place, const float *weight, const float *peak,
                                                               uint32_t parts, PolicyOut grad, double *part, uint32_t tiles,
                                                               uint32_t splits, int64_t per_split, uint32_t first) {
  using S = GradShape<NV, WR>;
  constexpr int C = S::kColumns, RB = S::kRows, E = 8;
  extern __shared__ double lds_table[];
  const int R = a.n_res, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int t = threadIdx.x % (64 * WR);  // of the group's lanes
  const uint32_t id = (first + blockIdx.x) * S::kGroups + wave / WR;
  const uint32_t tile = id / splits, k = id - tile * splits;
  if (tile >= tiles) return;  // with WR = 4 a block is one group
  const uint32_t per_pol = ((uint32_t)a.n_ops + RB - 1) / RB, pol = tile / per_pol, v0 = (tile - pol * per_pol) * RB;
  const int rows = min(RB, a.n_ops - (int)v0);
  double *table = lds_table + wave / WR * (RB * R * C);
  // a wavefront's row once the sums are there
  const int own = wave % WR;
  const uint32_t v = v0 + own;
  const bool finish = own < rows;
  float x[NV];
  if (finish && splits == 1)
    load_row<NV>(a.logits, a.dtype, pol * a.ld_pol + v * a.ld_op, lane * NV, R, x);
  for (int i = t; i < RB * R * C; i += 64 * WR) table[i] = 0;
  const float top = group_max<64>(peak[(uint64_t)pol * parts + min((uint32_t)lane, parts - 1)]);
  // adding and taking away 1.5 2^52 grid steps rounds to the grid; weights that
  // are not finite stay, and so do sums with them, in any order
  const double magic = top > 0 ? ldexp(1.5, ilogbf(top) + 64 - __clzll(per_split)) : 0.0;
  if (WR > 1)
    __syncthreads();
  else
    wave_order();
  const uint16_t *pp = place + (int64_t)v0 * ld_place;
  const int64_t from = k * per_split, to = min(n_scen, from + per_split);
  double *mine = table + lane % C;
  auto add = [&](int row, uint32_t at, double w) {
    __hip_atomic_fetch_add(mine + (row * R + at) * C, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  };
  if (a.block >= 64 * E) {
    for_runs(a, (int)pol, from, to, [&](int64_t beg, int64_t end) {
      int64_t s = beg + t * E;
      uint32_t w[RB][E / 2] = {};
      float y[E] = {};
      auto load = [&] {
#pragma unroll
        for (int i = 0; i < RB; ++i) load_places<E>(pp + min(i, rows - 1) * ld_place, s, beg, end, w[i]);
        load_numbers<E>(weight, s, beg, end, y);
      };
      load();
      while (s - t * E < end) {
        uint32_t at[RB][E / 2];
        double z[E];
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = (double)y[e] + magic - magic;
        if (__any(s + E > end) && end - beg >= E) {  // what the lane before has, or nobody
          const int not_mine = s < end ? (int)max((int64_t)0, s + E - end) : E;
#pragma unroll
          for (int e = 0; e < E; ++e) z[e] = e < not_mine ? 0.0 : z[e];
        }
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int e = 0; e < E / 2; ++e) at[i][e] = w[i][e];
        s += 64 * WR * E;
        load();
#pragma unroll
        for (int i = 0; i < RB; ++i) {
          if (i >= rows) break;
          uint32_t most = at[i][0];
#pragma unroll
          for (int e = 1; e < E / 2; ++e) most = max_pair(most, at[i][e]);
          if (__any(max(most & 0xFFFFu, most >> 16) >= (uint32_t)R)) {  // no resource, or behind the end
#pragma unroll
            for (int e = 0; e < E; ++e)
              if (place_at(at[i], e) < (uint32_t)R) add(i, place_at(at[i], e), z[e]);
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) add(i, place_at(at[i], e), z[e]);
          }
        }
      }
    });
  } else {
    // short runs: the policy's scenarios one after another over the lanes; run
    // j begins at b + j * period
    const uint32_t block = (uint32_t)a.block, step_j = 64 * WR / block, step_o = 64 * WR - step_j * block;
    int64_t b = (int64_t)pol * a.block - a.phase;
    if (from > b) b += (from - b) / a.period * a.period;
    b += t / block * a.period;
    uint32_t o = t % block;
    while (b < to) {
      const int64_t s = b + o;
      if (s >= from && s < to) {
        const double z = (double)weight[s] + magic - magic;
        for (int i = 0; i < rows; ++i) {
          const uint32_t at = pp[i * ld_place + s];
          if (at < (uint32_t)R) add(i, at, z);
        }
      }
      b += step_j * a.period;
      o += step_o;
      if (o >= block) o -= block, b += a.period;
    }
  }
  if (WR > 1)
    __syncthreads();
  else
    wave_order();
  if (!finish) return;
  const int r0 = lane * NV;
  double sum[NV];
  float h[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    sum[j] = 0;
    if (r0 + j < R) {
#pragma unroll
      for (int c = 0; c < C; ++c) sum[j] += table[(own * R + r0 + j) * C + (lane + c) % C];  // lanes in different banks
    }
    if (sum[j] != sum[j]) sum[j] = __builtin_nan("");  // of several the first stays: one for all
    h[j] = (float)sum[j];
  }
  if (splits > 1) {
    double *to_part = part + (((int64_t)k * a.n_pol + pol) * a.n_ops + v) * R;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (r0 + j < R) to_part[r0 + j] = sum[j];
    return;
  }
  const float T = policy_temperature(a, (int)pol);
  float out[NV];
  RowExp<NV> row;
  row_exp<64, NV>(x, T, row);
  row_grad<64, NV>(row, x, h, out);
  store_row<NV>(grad.p, a.dtype, pol * grad.ld_pol + v * grad.ld_op, r0, R, out);
}

// The splits' sums of every row joined in order, and its gradient.
template <int G, int NV>
__global__ __launch_bounds__(kThreads) void k_policy_grad_join(PolicyArgs a, const double *part, uint32_t splits,
                                                               uint32_t rows, PolicyOut grad, uint32_t first) {
  const int g = threadIdx.x % G, r0 = g * NV;
  const uint32_t row_id = (first + blockIdx.x) * (kThreads / G) + threadIdx.x / G;
  if (row_id >= rows) return;
  const uint32_t pol = row_id / (uint32_t)a.n_ops, v = row_id - pol * (uint32_t)a.n_ops;
  const float T = policy_temperature(a, (int)pol);
  float x[NV], h[NV], out[NV];
  load_row<NV>(a.logits, a.dtype, pol * a.ld_pol + v * a.ld_op, r0, a.n_res, x);
  double sum[NV] = {};
  for (uint32_t k = 0; k < splits; ++k) {
    const double *p = part + ((int64_t)k * rows + row_id) * a.n_res + r0;
#pragma unroll
    for (int j = 0; j < NV; ++j) sum[j] += r0 + j < a.n_res ? p[j] : 0.0;
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) h[j] = (float)sum[j];
  RowExp<NV> row;
  row_exp<G, NV>(x, T, row);
  row_grad<G, NV>(row, x, h, out);
  store_row<NV>(grad.p, a.dtype, pol * grad.ld_pol + v * grad.ld_op, r0, a.n_res, out);
}

// A group of lanes distils a row.  The teacher's entries are scattered over
// the resources in LDS (q), so that the gradient is one pass over the row; the loss
// is summed entry by entry.  An entry on a logit of -inf is not scattered: its
// gradient is 0 and it makes the loss infinite.  Entries that share a resource are
// found by writing every entry's number to its resource and reading it back;
// one lane then adds them up in order.  Bound by memory: 16 x 20000 rows of 1001
// float32 with 32 entries take 486 us, 5.4 TB/s.
template <int G, int NV>
__global__ __launch_bounds__(kThreads) void k_policy_distill(PolicyArgs a, PolicyTop top, const float *weight,
                                                             float *loss, PolicyOut grad, int64_t rows) {
  constexpr int V = piece(NV), kWords = V % 4 == 0 ? 4 : 1;
  __shared__ __align__(16) float lds_q[kThreads * NV];
  __shared__ uint16_t lds_entry[kThreads * NV];
  const int g = threadIdx.x % G, grp = threadIdx.x / G;
  float *q = lds_q + grp * (G * NV);
  uint16_t *entry = lds_entry + grp * (G * NV);
  const uint32_t n_groups = gridDim.x * (kThreads / G);
  for (int64_t row_id = (int64_t)blockIdx.x * (kThreads / G) + grp; row_id < rows; row_id += n_groups) {
    const int64_t pol = (uint64_t)row_id < 1ull << 32 ? (uint32_t)row_id / (uint32_t)a.n_ops : row_id / a.n_ops, v = row_id - pol * a.n_ops;
    const float T = policy_temperature(a, (int)pol);
    const int64_t at_row = pol * a.ld_pol + v * a.ld_op;
    const uint16_t *ids = top.res + pol * top.ld_res_pol + v * top.ld_res_op;
    const int64_t at_log = pol * top.ld_log_pol + v * top.ld_log_op;
    float x[NV];
    load_spread<G, NV>(a.logits, a.dtype, at_row, g, a.n_res, x);
    const float w = weight ? weight[row_id] : 1.0f;
    uint32_t masked = 0;  // the logits of -inf, where the weight's product with 0 is not 0
    if (!(fabsf(w) < kInf)) {
#pragma unroll
      for (int j = 0; j < NV; ++j) masked |= (uint32_t)(x[j] == -kInf) << j;
    }
#pragma unroll
    for (int j = 0; j < NV; j += kWords)
#pragma unroll
      for (int i = 0; i < kWords; ++i) q[((j / V) * G + g) * V + j % V + i] = 0;
    // f(k, resource, teacher's logit, own logit) for this lane's entries; the first is kept
    const int id0 = g < top.top ? ids[g] : kNoPlace;
    const float y0 = g < top.top ? load_elem(top.logits, a.dtype, at_log + g) : -kInf;
    const bool have0 = id0 < a.n_res && y0 != -kInf;
    const float l0 = have0 ? load_elem(a.logits, a.dtype, at_row + id0) : -kInf;
    auto entries = [&](auto f) {
      if (have0) f(g, id0, y0, l0);
      for (int k = g + G; k < top.top; k += G) {
        const int id = ids[k];
        const float y = load_elem(top.logits, a.dtype, at_log + k);
        if (id < a.n_res && y != -kInf) f(k, id, y, load_elem(a.logits, a.dtype, at_row + id));
      }
    };
    float m = -kInf;  // passes over NaN, which the sum then shows
    entries([&](int k, int id, float y, float) {
      m = fmaxf(m, y);
      entry[id] = (uint16_t)k;
    });
    m = group_max<G>(m);
    RowExp<NV> row;
    row_exp<G, NV>(x, T, row);
    const float ls = row.log_sum();
    wave_order();
    float sum = 0;
    uint32_t seen = 0;  // low half: entries, high half: those that found another's number
    entries([&](int k, int id, float y, float own) {
      const float e = __builtin_amdgcn_exp2f(over(y, m, row.inv) * kLog2e);
      sum += e;
      seen += entry[id] == k ? 1u : 0x10001u;
      if (own > -kInf) q[id] = e;
    });
    sum = group_sum<G>(sum);
    seen = group_sum<G>(seen);
    wave_order();
    if (seen >> 16 && g == 0) {
      for (int k = top.top - 1; k >= 0; --k) {
        const int id = ids[k];
        if (id >= a.n_res || load_elem(top.logits, a.dtype, at_log + k) == -kInf) continue;
        entry[id] = (uint16_t)k;  // in the end the first one's
        q[id] = 0;
      }
      for (int k = 0; k < top.top; ++k) {
        const int id = ids[k];
        if (id >= a.n_res) continue;
        const float y = load_elem(top.logits, a.dtype, at_log + k);
        if (y != -kInf && load_elem(a.logits, a.dtype, at_row + id) > -kInf)
          q[id] += __builtin_amdgcn_exp2f(over(y, m, row.inv) * kLog2e);
      }
    }
    wave_order();
    float l = 0;
    const float inv = 1.0f / sum;
    entries([&](int k, int id, float, float own) {
      if (entry[id] != k) return;
      const float p = q[id] * inv;
      if (!(own > -kInf))
        l = kInf;
      else if (p > 0)
        l += p * (kLn2 * log2_of(p) - (row.z(own) - ls));
    });
    l = group_sum<G>(l);
    const float nan = row.sum + (seen ? sum : 0.0f);  // NaN or not
    if (g == 0) loss[row_id] = nan != nan ? nan : l;
    if (grad.p) {
      const float ke = nan != nan ? nan : seen && row.sum > 0 ? w / row.sum : 0.0f, kq = seen ? -w * inv : 0.0f;
      float out[NV];
#pragma unroll
      for (int j = 0; j < NV; j += kWords)
#pragma unroll
        for (int i = 0; i < kWords; ++i)
          out[j + i] = __builtin_fmaf(row.e[j + i], ke, q[((j / V) * G + g) * V + j % V + i] * kq) * row.inv;
      if (masked && nan == nan) {
#pragma unroll
        for (int j = 0; j < NV; ++j) out[j] = masked >> j & 1 ? 0.0f : out[j];
      }
      store_spread<G, NV>(grad.p, a.dtype, pol * grad.ld_pol + v * grad.ld_op, g, a.n_res, out);
    }
    wave_order();
  }
}

// ---- launches ----

// f(G, NV) as compile-time constants: the smallest group of lanes, at eight
// resources a lane, that holds a row (sixteen a lane beyond 512).
template <class F>
int by_row(int n_res, F f) {
#define MLSIM_ROW(G, NV) f(std::integral_constant<int, G>{}, std::integral_constant<int, NV>{})
  if (n_res <= 8) return MLSIM_ROW(1, 8);
  if (n_res <= 16) return MLSIM_ROW(2, 8);
  if (n_res <= 32) return MLSIM_ROW(4, 8);
  if (n_res <= 64) return MLSIM_ROW(8, 8);
  if (n_res <= 128) return MLSIM_ROW(16, 8);
  if (n_res <= 256) return MLSIM_ROW(32, 8);
  if (n_res <= 512) return MLSIM_ROW(64, 8);
  return MLSIM_ROW(64, 16);
#undef MLSIM_ROW
}

// f(NV): the resources a lane holds of a row that a wavefront has to itself.
template <class F>
int by_wave(int n_res, F f) {
  if (n_res <= 64) return f(std::integral_constant<int, 1>{});
  if (n_res <= 128) return f(std::integral_constant<int, 2>{});
  if (n_res <= 256) return f(std::integral_constant<int, 4>{});
  if (n_res <= 512) return f(std::integral_constant<int, 8>{});
  return f(std::integral_constant<int, 16>{});
}

int row_lanes(int n_res) {
  int g = 1;
  while (g < 64 && g * 8 < n_res) g *= 2;
  return g;
}

int log2_at_least(int64_t n, int most) {
  int l = 0;
  while ((1 << l) < most && ((int64_t)1 << l) < n) ++l;
  return l;
}

int launched() { return hipGetLastError() == hipSuccess ? SIM_OK : SIM_E_HIP; }

constexpr int64_t kMaxBlocks = INT32_MAX;

// A launch holds fewer than 2^32 threads, and more are cut off without an error:
// a grid goes out in launches of up to 2^23 blocks, which are told the first.
constexpr int64_t kLaunchBlocks = 1 << 23;

template <class F>
int launch_blocks(int64_t blocks, F f) {
  for (int64_t first = 0; first < blocks; first += kLaunchBlocks) {
    f(dim3((unsigned)std::min(blocks - first, kLaunchBlocks)), (uint32_t)first);
    if (int rc = launched()) return rc;
  }
  return SIM_OK;
}

// Row kernels: up to `side` policies (logp: scenarios) side by side, the other
// groups along the ops, so that a wavefront's rows lie in few places.  Draws of
// short rows have 16 side by side, which write 32 bytes of places together, and
// so have log-probabilities of the shortest, which read them.  With 4 and 16:
// draws of 2048 x 6624 rows of 8 150 and 76 us, of 1024 x 6624 rows of 48 268 and
// 261; log-probabilities of 4096 x 6624 rows of 8 148 and 113, of 1024 x 6624 rows
// of 32 90 and 99; gradients of 1024 x 6624 rows of 32 185 and 218.
int row_tile(const PolicyArgs &a, int side, Tile &t, int64_t &blocks) {
  const int ng = kThreads / row_lanes(a.n_res);
  t.log_pol = log2_at_least(a.n_pol, std::min(side, ng));
  const int64_t np = 1 << t.log_pol, nv = ng >> t.log_pol, pol_tiles = (a.n_pol + np - 1) / np;
  t.per = (int)std::max<int64_t>(1, std::min<int64_t>(16, pol_tiles * ((a.n_ops + nv - 1) / nv) / 2048));
  blocks = pol_tiles * ((a.n_ops + nv * t.per - 1) / (nv * t.per));
  return blocks > kMaxBlocks ? SIM_E_LIMIT : SIM_OK;
}

int64_t logp_tile(const PolicyArgs &a, int64_t n_scen, Tile &t, int64_t &blocks) {
  const int ng = kThreads / row_lanes(a.n_res);
  t.log_pol = log2_at_least(n_scen, a.n_res <= 8 ? 16 : std::min(4, ng));
  const int64_t ns = 1 << t.log_pol, nv = ng >> t.log_pol, tiles = (n_scen + ns - 1) / ns;
  const int64_t steps = (a.n_ops + nv - 1) / nv;
  t.per = (int)std::min<int64_t>(steps, std::max<int64_t>(4, steps * tiles / 4096));
  const int64_t chunks = (steps + t.per - 1) / t.per;
  blocks = tiles * chunks;
  return chunks;
}

// Their number; a launch checks that it fits.
int64_t make_pieces(const PolicyArgs &a, int64_t n_scen, int64_t span, Pieces &p) {
  p.span = span;
  p.first = a.phase % a.block;
  p.pol = (int32_t)(a.phase / a.block);
  const int64_t left = a.block - p.first;
  const int64_t runs = left >= n_scen ? 1 : 1 + (n_scen - left + a.block - 1) / a.block;
  const int64_t per_run = (std::min(a.block, n_scen) + span - 1) / span;
  p.per_run = (uint32_t)std::min(per_run, kMaxBlocks);
  p.n = (uint32_t)std::min(runs * per_run, kMaxBlocks);
  return runs * per_run;
}

// Whether a row's table is worth making: the row kernel works through a whole
// row for every scenario, a table costs that twice and as much as 48 lanes more.
// 1024 scenarios of 6624 rows of 48 bf16, 4 and 8 a table: 230 and 131 us, row by
// row 127 and 124; 4096 of 8, 16 a table: 253 us, row by row 60.
bool long_runs(const PolicyArgs &a, int64_t n_scen) {
  const int64_t lanes = row_lanes(a.n_res);
  return std::min(a.block, n_scen) * lanes > 2 * lanes + 48;
}

constexpr double kPerUs = 600e3;  // wavefront instructions of all SIMDs in a microsecond

// Whether the draws go row by row by groups of lanes, or a wavefront a row and
// run: by the instructions of either, and by their latency where there are few
// rows.  A group works a row out in about 300 and takes 200 for every G draws; a
// wavefront in 64 bits in 450.  2000000 rows of 64, 63 draws each: 1010 us by
// groups, 1480 by wavefronts; 256 draws: 3650 and 1480; 17403 rows of 4, 47 draws:
// 30 us by groups (47 rounds one after another), 13 by wavefronts.
bool sample_by_rows(const PolicyArgs &a, int64_t n_scen) {
  const int64_t run = std::min(a.block, n_scen), lanes = row_lanes(a.n_res);
  const double rows = (double)a.n_pol * a.n_ops, rounds = (double)((std::max(n_scen / a.n_pol, run) + lanes - 1) / lanes);
  const double us = kPerUs;
  const double groups = std::max(rows * lanes / 64 * (300 + 200 * rounds), rounds * 0.8 * us);
  const double waves = std::max((double)a.n_ops * n_scen / std::min<int64_t>(run, 4096) * 450 * std::max<int64_t>(1, lanes / 16), 6 * us);
  return groups <= waves || (double)a.n_ops * n_scen / run > 1e9;  // blocks of a grid
}

// Whether a gradient's scenarios are added by groups of lanes in registers (38
// instructions each) or by a wavefront a row in LDS (about 480 a row, twice that for
// the longest).  2000000 rows of 64 bf16: with 16, 32 and 63 scenarios a row 393, 597
// and 1104 us by groups, 1770 to 1850 by wavefronts; 127620 rows of 149 with 57: 237
// us, and 106.
bool grad_by_rows(const PolicyArgs &a, int64_t n_scen) {
  const double lanes = row_lanes(a.n_res), rows = (double)a.n_pol * a.n_ops, long_row = a.n_res > 512 ? 2.3 : 1;
  const double scen = (double)std::max(n_scen / a.n_pol, std::min(a.block, n_scen));
  const double groups = std::max(rows * lanes / 64 * (250 * long_row + 38 * scen), scen * 0.2 * kPerUs);
  return groups <= std::max(rows * 480 * long_row, 10 * kPerUs);
}

struct LogpRuns {
  Pieces ps;
  int64_t pieces, chunks;
  int ops_per;
  bool wide;  // eight scenarios a thread
};

LogpRuns logp_runs(const PolicyArgs &a, int64_t n_scen) {
  LogpRuns l;
  const int rows = kThreads / row_lanes(a.n_res);
  l.wide = std::min(a.block, n_scen) >= 8 * 64;
  l.pieces = make_pieces(a, n_scen, (int64_t)kThreads * (l.wide ? 8 : 1), l.ps);
  // At most three blocks a CU, so that all run at once (20000 ops of 64
  // resources in 16384 scenarios take 117 us with 720 blocks, 5.6 TB/s, what a
  // plain read reaches; 127 with 632 and 138 with 1256, which leave some CUs a block
  // more to do than others), whole tables of rows or, for small batches, parts
  // of one, down to 16 rows.
  const int64_t most = l.wide ? 768 : 4096, want = most / std::min(l.pieces, most);
  const int64_t even = (a.n_ops + want - 1) / want, unit = even >= rows ? rows : std::min(16, rows);
  l.ops_per = (int)((even + unit - 1) / unit * unit);
  l.chunks = (a.n_ops + l.ops_per - 1) / l.ops_per;
  return l;
}

struct GradRuns {
  int64_t rows, splits, per_split;
  int waves;  // of a row
  // The peak of a policy's weights is found in parts of one load a thread, by the
  // scenarios that one policy may have: 1000000 in one of 1000 policies of 2 x 5
  // take 504 us, with parts by the mean 1545.
  uint32_t parts;
  int peak_threads;
  int64_t peak_bytes;
};

// Enough wavefronts to fill the chip, none with fewer than 2048 scenarios of
// the batch; no split above 2^22, which bounds the weights' grid.
GradRuns grad_runs(const PolicyArgs &a, int64_t n_scen) {
  GradRuns r;
  r.rows = (int64_t)a.n_pol * a.n_ops;
  r.waves = n_scen / a.n_pol >= 2048 ? 4 : 1;
  const int64_t fill = 4096 / std::min<int64_t>(r.rows * r.waves, 4096);
  r.splits = std::max<int64_t>(1, std::min(fill, n_scen / (r.waves * 2048)));
  r.splits = std::max(r.splits, (n_scen + (1 << 22) - 1) >> 22);
  r.per_split = ((n_scen + r.splits - 1) / r.splits + 511) / 512 * 512;
  r.splits = (n_scen + r.per_split - 1) / r.per_split;
  const int64_t most = std::max(n_scen / a.n_pol, std::min(a.block, n_scen));
  r.peak_threads = most > 64 ? kThreads : 64;
  r.parts = (uint32_t)std::min<int64_t>({64, (most + kThreads - 1) / kThreads, std::max(1, 65536 / a.n_pol)});
  r.peak_bytes = ((int64_t)a.n_pol * r.parts * 4 + 7) / 8 * 8;
  return r;
}

}  // namespace

int launch_policy_sample(const PolicyArgs &a, int64_t n_scen, const float *u, int64_t ld_u, uint16_t *place,
                         int64_t ld_place, hipStream_t st) {
  const bool cut = a.settings || a.temperature == 0 || a.top_k >= 1 || a.top_p < 1 || a.min_p > 0;
  const bool one = a.block == 1 && n_scen <= a.period;
  if (!one && !sample_by_rows(a, n_scen)) {
    Pieces ps;
    // Four wavefronts a row share one working-out of it, but wait for it: 20000
    // rows of 64, 16384 scenarios, nothing cut: 334 us, and 369 with one; 79488 cut
    // rows of 48, 4096 scenarios: 475 us, and 350 with one, whose wavefronts work out rows side by side.
    const int wr = !cut && std::min(a.block, n_scen) >= 2048 ? 4 : 1;
    const int64_t pieces = make_pieces(a, n_scen, 4096, ps), blocks = pieces * ((a.n_ops * (int64_t)wr + 3) / 4);
    if (blocks > kMaxBlocks) return SIM_E_LIMIT;
    const int levels = log2_at_least(a.n_res, SIM_MAX_RES);
    return by_wave(a.n_res, [&](auto NV) {
      return launch_blocks(blocks, [&](dim3 grid, uint32_t first) {
        if (wr == 4)
          k_policy_sample_runs<NV(), 4><<<grid, dim3(kThreads), 0, st>>>(a, n_scen, u, ld_u, place, ld_place, ps, levels, first);
        else
          k_policy_sample_runs<NV(), 1><<<grid, dim3(kThreads), 0, st>>>(a, n_scen, u, ld_u, place, ld_place, ps, levels, first);
      });
    });
  }
  Tile t;
  int64_t blocks;
  if (int rc = row_tile(a, a.n_res <= 64 ? 16 : 4, t, blocks)) return rc;
  return by_row(a.n_res, [&](auto G, auto NV) {
    auto go = [&](auto cuts) {
      return launch_blocks(blocks, [&](dim3 grid, uint32_t first) {
        if (one)
          k_policy_sample_one<G(), NV(), cuts()><<<grid, dim3(kThreads), 0, st>>>(a, n_scen, u, ld_u, place, ld_place, t, first);
        else
          k_policy_sample_few<G(), NV(), cuts()><<<grid, dim3(kThreads), 0, st>>>(a, n_scen, u, ld_u, place, ld_place, t, first);
      });
    };
    return cut ? go(std::true_type{}) : go(std::false_type{});
  });
}

int64_t policy_work(const PolicyArgs &a, int64_t n_scen) {
  int64_t logp, grad = 0;
  if (long_runs(a, n_scen)) {
    const LogpRuns l = logp_runs(a, n_scen);
    logp = l.chunks > 1 ? l.chunks * n_scen * 4 : 0;
  } else {
    Tile t;
    int64_t blocks;
    logp = logp_tile(a, n_scen, t, blocks) * n_scen * 8;
  }
  if (!grad_by_rows(a, n_scen)) {
    const GradRuns r = grad_runs(a, n_scen);
    grad = r.peak_bytes + (r.splits > 1 ? r.splits * r.rows * a.n_res * 8 : 0);
  }
  return (std::max(logp, grad) + 7) / 8 * 8;
}

int launch_policy_logp(const PolicyArgs &a, int64_t n_scen, const uint16_t *place, int64_t ld_place, float *logp,
                       void *work, hipStream_t st) {
  auto join = [&](auto *part, int64_t chunks) {
    return launch_blocks((n_scen + kJoinScen - 1) / kJoinScen, [&](dim3 grid, uint32_t first) {
      k_policy_join<<<grid, dim3(kThreads), 0, st>>>(part, chunks, n_scen, logp, first);
    });
  };
  if (long_runs(a, n_scen)) {
    const LogpRuns l = logp_runs(a, n_scen);
    const int64_t blocks = l.pieces * l.chunks;
    if (blocks > kMaxBlocks) return SIM_E_LIMIT;
    float *to = l.chunks > 1 ? (float *)work : logp;
    const int rc = by_row(a.n_res, [&](auto G, auto NV) {
      return launch_blocks(blocks, [&](dim3 grid, uint32_t first) {
        if (l.wide)
          k_policy_logp_runs<G(), NV(), 8><<<grid, dim3(kThreads), 0, st>>>(a, n_scen, place, ld_place, to, l.ps, l.ops_per, first);
        else
          k_policy_logp_runs<G(), NV(), 1><<<grid, dim3(kThreads), 0, st>>>(a, n_scen, place, ld_place, to, l.ps, l.ops_per, first);
      });
    });
    return rc || l.chunks == 1 ? rc : join((const float *)work, l.chunks);
  }
  Tile t;
  int64_t blocks;
  const int64_t chunks = logp_tile(a, n_scen, t, blocks);
  if (blocks > kMaxBlocks) return SIM_E_LIMIT;
  const int rc = by_row(a.n_res, [&](auto G, auto NV) {
    return launch_blocks(blocks, [&](dim3 grid, uint32_t first) {
      k_policy_logp<G(), NV()><<<grid, dim3(kThreads), 0, st>>>(a, n_scen, place, ld_place, (double *)work, t, first);
    });
  });
  return rc ? rc : join((const double *)work, chunks);
}

int launch_policy_grad(const PolicyArgs &a, int64_t n_scen, const uint16_t *place, int64_t ld_place,
                       const float *weight, const PolicyOut &grad, void *work, hipStream_t st) {
  if (!grad_by_rows(a, n_scen)) {
    const GradRuns r = grad_runs(a, n_scen);
    const int64_t peak_blocks = a.n_pol * (int64_t)r.parts;
    if (std::max(r.rows * r.splits, peak_blocks) > kMaxBlocks) return SIM_E_LIMIT;
    float *peak = (float *)work;
    double *part = (double *)((char *)work + r.peak_bytes);
    const uint32_t rows = (uint32_t)r.rows, splits = (uint32_t)r.splits;
    if (int rc = launch_blocks(peak_blocks, [&](dim3 grid, uint32_t first) {
          k_policy_peak<<<grid, dim3(r.peak_threads), 0, st>>>(a, n_scen, weight, r.parts, peak, first);
        }))
      return rc;
    auto go = [&](auto NV, auto WR) {
      using S = GradShape<NV(), WR()>;
      const uint32_t tiles = (uint32_t)(a.n_pol * ((a.n_ops + (int64_t)S::kRows - 1) / S::kRows));
      const int64_t blocks = ((int64_t)tiles * splits + S::kGroups - 1) / S::kGroups;
      return launch_blocks(blocks, [&](dim3 grid, uint32_t first) {
        k_policy_grad_runs<NV(), WR()><<<grid, dim3(kThreads), S::lds(a.n_res), st>>>(
            a, n_scen, place, ld_place, weight, peak, r.parts, grad, part, tiles, splits, r.per_split, first);
      });
    };
    int rc = by_wave(a.n_res, [&](auto NV) {
      return r.waves == 4 ? go(NV, std::integral_constant<int, 4>{}) : go(NV, std::integral_constant<int, 1>{});
    });
    if (rc || splits == 1) return rc;
    return by_row(a.n_res, [&](auto G, auto NV) {
      const int64_t per = kThreads / G();
      return launch_blocks((r.rows + per - 1) / per, [&](dim3 grid, uint32_t first) {
        k_policy_grad_join<G(), NV()><<<grid, dim3(kThreads), 0, st>>>(a, part, splits, rows, grad, first);
      });
    });
  }
  Tile t;
  int64_t blocks;
  if (int rc = row_tile(a, 4, t, blocks)) return rc;
  return by_row(a.n_res, [&](auto G, auto NV) {
    return launch_blocks(blocks, [&](dim3 grid, uint32_t first) {
      if (a.block == 1 && n_scen <= a.period)
        k_policy_grad<G(), NV(), true><<<grid, dim3(kThreads), 0, st>>>(a, n_scen, place, ld_place, weight, grad, t, first);
      else
        k_policy_grad<G(), NV(), false><<<grid, dim3(kThreads), 0, st>>>(a, n_scen, place, ld_place, weight, grad, t, first);
    });
  });
}

int launch_policy_distill(const PolicyArgs &a, const PolicyTop &top, const float *weight, float *loss,
                          const PolicyOut &grad, hipStream_t st) {
  const int64_t rows = (int64_t)a.n_pol * a.n_ops;
  return by_row(a.n_res, [&](auto G, auto NV) {
    const int64_t per = kThreads / G(), blocks = std::min<int64_t>((rows + per - 1) / per, 16384);
    k_policy_distill<G(), NV()><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(a, top, weight, loss, grad, rows);
    return launched();
  });
}

}  // namespace mlsim
