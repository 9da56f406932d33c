// Position rotation of query and key heads, alone or with the RMS norm of every head in the same pass,
// and the norm's backward pass.
//   pair (a, b) of a row at position p, angle t = 2 pi p turns[j]:  (s (a cos t - b sin t), s (b cos t + a sin t))
//   norm:      y = R(x r gamma),  r = (mean(x^2) + eps)^(-1/2)
//   backward:  g = R^T dy;  h = g gamma;  dx = r (h - xhat mean(h xhat)),  xhat = x r;  dgamma = sum g xhat
// Bound by HBM: every element is read once and written once (backward: two reads).  What has to stay off
// the path is the angles: p turns[j] loses whole turns in fp32 once p passes a few thousand, so it is taken in
// fp64 and reduced to a quarter turn there; a workgroup does that once per (row, pair) of its rows, into LDS, and all
// heads of those rows read the pair's cosine and sine from it.
// A head is held by a group of lanes, each with two 16-byte chunks ("slot"): in the half layout the two
// chunks whose elements turn together, so no lane needs another's elements except for the norm's sums.
#include <algorithm>

#include "vf_device.h"

namespace vf {
namespace {

constexpr int NT = 256;

struct Turns { double t[VF_ROPE_MAX_PAIRS]; };

template <typename T, int C> struct Chunk;
template <> struct Chunk<float, 4> {
  typedef vf_f32x4 Raw;
  static __device__ __forceinline__ Raw zero() { return Raw{0.f, 0.f, 0.f, 0.f}; }
  static __device__ __forceinline__ Raw load(const float* p) { return *reinterpret_cast<const Raw*>(p); }
  static __device__ __forceinline__ void open(const Raw& r, float* v) {
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = r[u];
  }
  static __device__ __forceinline__ void store(float* p, const float* v) { *reinterpret_cast<Raw*>(p) = Raw{v[0], v[1], v[2], v[3]}; }
};
template <> struct Chunk<bf16_t, 8> {
  typedef vf_u32x4 Raw;
  static __device__ __forceinline__ Raw zero() { return Raw{0u, 0u, 0u, 0u}; }
  static __device__ __forceinline__ Raw load(const bf16_t* p) { return *reinterpret_cast<const Raw*>(p); }
  static __device__ __forceinline__ void open(const Raw& w, float* v) {
#pragma unroll
    for (int u = 0; u < 4; ++u) { v[2 * u] = __uint_as_float(w[u] << 16); v[2 * u + 1] = __uint_as_float(w[u] & 0xffff0000u); }
  }
  static __device__ __forceinline__ void store(bf16_t* p, const float* v) {
    Raw w;
#pragma unroll
    for (int u = 0; u < 4; ++u) w[u] = f32x2_to_bf16x2(v[2 * u], v[2 * u + 1]);
    *reinterpret_cast<Raw*>(p) = w;
  }
};
template <typename T> struct Chunk<T, 1> {
  typedef float Raw;
  static __device__ __forceinline__ Raw zero() { return 0.f; }
  static __device__ __forceinline__ Raw load(const T* p) { return load_f(p); }
  static __device__ __forceinline__ void open(const Raw& r, float* v) { v[0] = r; }
  static __device__ __forceinline__ void store(T* p, const float* v) { store_f(p, v[0]); }
};

// The two chunks of a slot: first elements (or -1: the slot has none), the index of the first pair of each, and whether
// they turn.  together: element e of the first chunk turns with element e of the second.
struct Slot {
  int a0, a1, pair0, pair1;
  bool together;
};
template <int C>
__device__ __forceinline__ Slot slot_of(int s, int layout, int rot, int dh) {
  Slot r;
  if (layout == VF_ROPE_HALF || C == 1) {
    const int turning = rot / (2 * C);
    r.together = s < turning;
    if (r.together) {
      r.a0 = layout == VF_ROPE_HALF ? s * C : 2 * s;
      r.a1 = layout == VF_ROPE_HALF ? rot / 2 + s * C : 2 * s + 1;
      r.pair0 = s * C;
    } else {
      r.a0 = rot + 2 * C * (s - turning);
      r.a1 = r.a0 + C;
      r.pair0 = -1;
    }
    r.pair1 = -1;
  } else {
    r.together = false;
    r.a0 = 2 * C * s;
    r.a1 = r.a0 + C;
    r.pair0 = r.a0 < rot ? r.a0 / 2 : -1;
    r.pair1 = r.a1 < rot ? r.a1 / 2 : -1;
  }
  if (r.a0 >= dh) r.a0 = -1;
  if (r.a1 >= dh) r.a1 = -1;
  return r;
}

template <int C>
__device__ __forceinline__ void turn_slot(const Slot& k, const float2* cs, float* v0, float* v1) {
  if (k.together) {
#pragma unroll
    for (int e = 0; e < C; ++e) {
      const float2 c = cs[k.pair0 + e];
      const float a = v0[e], b = v1[e];
      v0[e] = a * c.x - b * c.y;
      v1[e] = b * c.x + a * c.y;
    }
    return;
  }
  if constexpr (C > 1) {
    if (k.pair0 >= 0) {
#pragma unroll
      for (int e = 0; e < C / 2; ++e) {
        const float2 c = cs[k.pair0 + e];
        const float a = v0[2 * e], b = v0[2 * e + 1];
        v0[2 * e] = a * c.x - b * c.y;
        v0[2 * e + 1] = b * c.x + a * c.y;
      }
    }
    if (k.pair1 >= 0) {
#pragma unroll
      for (int e = 0; e < C / 2; ++e) {
        const float2 c = cs[k.pair1 + e];
        const float a = v1[2 * e], b = v1[2 * e + 1];
        v1[2 * e] = a * c.x - b * c.y;
        v1[2 * e + 1] = b * c.x + a * c.y;
      }
    }
  }
}

// Cosines and sines (times scale; sine times sign) of rows row0 .. row0 + n - 1.
__device__ __forceinline__ void fill_angles(const RopeJob& j, const Turns& turns, int64_t row0, int n, float2* cs) {
  const int pairs = j.rot / 2;
  for (int i = threadIdx.x; i < n * pairs; i += NT) {
    const int r = i / pairs, k = i - r * pairs;
    const int64_t row = row0 + r;
    const int64_t pos = j.positions ? (int64_t)j.positions[row] : j.first + (j.seq_len > 0 ? row % j.seq_len : row);
    const double quarter = 4.0 * ((double)pos * turns.t[k]);
    const double whole = rint(quarter);
    float s, c;
    sincospif(0.5f * (float)(quarter - whole), &s, &c);     // |argument| <= 1/4: a quarter turn at most
    const int q = (int)(whole - 4.0 * floor(0.25 * whole));
    const float cq = q == 0 ? c : q == 1 ? -s : q == 2 ? -c : s;
    const float sq = q == 0 ? s : q == 1 ? c : q == 2 ? -s : -c;
    cs[i] = make_float2(cq * j.scale, sq * j.scale * j.sign);
  }
}

// Heads of a workgroup: blocks of `take` heads, first the query heads' blocks, then the key heads'.
struct HeadBlock { int first, count; bool key; };
__device__ __forceinline__ HeadBlock head_block(const RopeJob& j, int y) {
  HeadBlock b;
  b.key = y >= j.q_blocks;
  const int lo = b.key ? j.q_heads + (y - j.q_blocks) * j.take : y * j.take;
  b.first = lo;
  b.count = min(j.take, (b.key ? j.heads : j.q_heads) - lo);
  return b;
}

// sum over the lanes that share a head
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// A thread asks for the chunks of AHEAD heads before it works on the first of them, and for the first ones before the angles
// are taken.  (65536 rows of 16 heads of 128, bf16, half of each turned: one head after the other 116 us.)
template <typename T, int C, int NS, bool NORM>
__global__ __launch_bounds__(NT) void rope_kernel(RopeJob j, Turns turns) {
  constexpr int AHEAD = NS > 1 ? 1 : NORM ? 2 : 4;
  typedef Chunk<T, C> Ch;
  extern __shared__ float2 rope_cs[];
  const HeadBlock hb = head_block(j, blockIdx.y);
  const int lanes = 1 << j.lane_bits, me = threadIdx.x & (lanes - 1), units = NT >> j.lane_bits, unit = threadIdx.x >> j.lane_bits;
  Slot k[NS];
  float g0[NS][C], g1[NS][C];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    k[i] = slot_of<C>(me + i * lanes, j.layout, j.rot, j.dh);
    if constexpr (NORM) {
      const float* gamma = hb.key ? j.gamma_k : j.gamma_q;
#pragma unroll
      for (int e = 0; e < C; ++e) {
        g0[i][e] = gamma && k[i].a0 >= 0 ? gamma[k[i].a0 + e] : 1.f;
        g1[i][e] = gamma && k[i].a1 >= 0 ? gamma[k[i].a1 + e] : 1.f;
      }
    }
  }
  for (int64_t row0 = (int64_t)blockIdx.x * j.tile; row0 < j.rows; row0 += (int64_t)gridDim.x * j.tile) {
    const int rows = (int)min((int64_t)j.tile, j.rows - row0);
    const int items = rows * hb.count;
    const uint32_t inv = 0xffffffffu / (uint32_t)hb.count + 1;   // exact: item hb.count < 2^32
    const T* xt = static_cast<const T*>(j.x) + row0 * j.x_row + (int64_t)hb.first * j.x_head;
    T* yt = static_cast<T*>(j.y) + row0 * j.y_row + (int64_t)hb.first * j.y_head;
    for (int base = unit; base - unit < items; base += units * AHEAD) {
      typename Ch::Raw x0[AHEAD][NS], x1[AHEAD][NS];
      int r[AHEAD], h[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int item = base + u * units;
        if (u && base - unit + u * units >= items) break;  // (nothing left for any thread)
        r[u] = hb.count == 1 ? item : (int)__umulhi((uint32_t)item, inv);   // item / hb.count
        h[u] = item - r[u] * hb.count;
        const T* x = xt + r[u] * j.x_row + h[u] * j.x_head;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          x0[u][i] = item < items && k[i].a0 >= 0 ? Ch::load(x + k[i].a0) : Ch::zero();
          x1[u][i] = item < items && k[i].a1 >= 0 ? Ch::load(x + k[i].a1) : Ch::zero();
        }
      }
      if (j.rot && base == unit) {                         // (every thread's first turn)
        __syncthreads();                                   // the last tile's cosines are no longer read
        fill_angles(j, turns, row0, rows, rope_cs);
        __syncthreads();
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (u && base - unit + u * units >= items) break;
        const bool on = base + u * units < items;
        float v0[NS][C], v1[NS][C], ss = 0.f;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          Ch::open(x0[u][i], v0[i]);
          Ch::open(x1[u][i], v1[i]);
          if constexpr (NORM) {
#pragma unroll
            for (int e = 0; e < C; ++e) ss += v0[i][e] * v0[i][e] + v1[i][e] * v1[i][e];
          }
        }
        if constexpr (NORM) {
          const float rstd = 1.0f / sqrtf(lanes_sum(ss, lanes) / (float)j.dh + j.eps);
#pragma unroll
          for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int e = 0; e < C; ++e) { v0[i][e] *= rstd * g0[i][e]; v1[i][e] *= rstd * g1[i][e]; }
        }
        T* y = yt + r[u] * j.y_row + h[u] * j.y_head;
        const float2* cs = rope_cs + (on ? r[u] : 0) * (j.rot / 2);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          turn_slot<C>(k[i], cs, v0[i], v1[i]);
          if (on && k[i].a0 >= 0) Ch::store(y + k[i].a0, v0[i]);
          if (on && k[i].a1 >= 0) Ch::store(y + k[i].a1, v1[i]);
        }
      }
    }
  }
}

template <int C> __host__ __device__ __forceinline__ int unit_pitch(int dh) { return C > 1 ? dh + 4 : dh + 1; }

// Backward pass of the norm with rotation.  A workgroup walks row tiles blockIdx.x, blockIdx.x + gridDim.x, ... so that the
// partial sums of dgamma stay few; they are added in the order of the workgroups by gamma_finish_kernel.
template <typename T, int C, int NS>
__global__ __launch_bounds__(NT) void norm_bwd_kernel(RopeJob j, Turns turns) {
  typedef Chunk<T, C> Ch;
  extern __shared__ float2 rope_cs[];
  const HeadBlock hb = head_block(j, blockIdx.y);
  const int lanes = 1 << j.lane_bits, me = threadIdx.x & (lanes - 1), units = NT >> j.lane_bits, unit = threadIdx.x >> j.lane_bits;
  const float* gamma = hb.key ? j.gamma_k : j.gamma_q;
  Slot k[NS];
  float g0[NS][C], g1[NS][C], s0[NS][C], s1[NS][C];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    k[i] = slot_of<C>(me + i * lanes, j.layout, j.rot, j.dh);
#pragma unroll
    for (int e = 0; e < C; ++e) {
      g0[i][e] = gamma && k[i].a0 >= 0 ? gamma[k[i].a0 + e] : 1.f;
      g1[i][e] = gamma && k[i].a1 >= 0 ? gamma[k[i].a1 + e] : 1.f;
      s0[i][e] = s1[i][e] = 0.f;
    }
  }
  for (int64_t row0 = (int64_t)blockIdx.x * j.tile; row0 < j.rows; row0 += (int64_t)gridDim.x * j.tile) {
    const int rows = (int)min((int64_t)j.tile, j.rows - row0);
    const int items = rows * hb.count;
    const uint32_t inv = 0xffffffffu / (uint32_t)hb.count + 1;   // exact: item hb.count < 2^32
    for (int base = 0; base < items; base += units) {
      const int item = base + unit;
      const bool on = item < items;
      const int r = on ? (hb.count == 1 ? item : (int)__umulhi((uint32_t)item, inv)) : 0, h = on ? item - r * hb.count : 0;
      const int64_t row = row0 + r, head = hb.first + h;
      const T* x = static_cast<const T*>(j.x) + row * j.x_row + head * j.x_head;
      const T* dy = static_cast<const T*>(j.dy) + row * j.dy_row + head * j.dy_head;
      T* dx = static_cast<T*>(j.y) + row * j.y_row + head * j.y_head;
      typename Ch::Raw rx0[NS], rx1[NS], rd0[NS], rd1[NS];
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const bool p0 = on && k[i].a0 >= 0, p1 = on && k[i].a1 >= 0;
        rx0[i] = p0 ? Ch::load(x + k[i].a0) : Ch::zero();
        rx1[i] = p1 ? Ch::load(x + k[i].a1) : Ch::zero();
        rd0[i] = p0 ? Ch::load(dy + k[i].a0) : Ch::zero();
        rd1[i] = p1 ? Ch::load(dy + k[i].a1) : Ch::zero();
      }
      if (j.rot && base == 0) {                            // (the loads are under way meanwhile)
        __syncthreads();                                   // the last tile's cosines are no longer read
        fill_angles(j, turns, row0, rows, rope_cs);
        __syncthreads();
      }
      float x0[NS][C], x1[NS][C], d0[NS][C], d1[NS][C], ss = 0.f, hx = 0.f;
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        Ch::open(rx0[i], x0[i]);
        Ch::open(rx1[i], x1[i]);
        Ch::open(rd0[i], d0[i]);
        Ch::open(rd1[i], d1[i]);
        turn_slot<C>(k[i], rope_cs + r * (j.rot / 2), d0[i], d1[i]);
#pragma unroll
        for (int e = 0; e < C; ++e) {
          ss += x0[i][e] * x0[i][e] + x1[i][e] * x1[i][e];
          hx += d0[i][e] * g0[i][e] * x0[i][e] + d1[i][e] * g1[i][e] * x1[i][e];
        }
      }
      ss = lanes_sum(ss, lanes);
      hx = lanes_sum(hx, lanes);
      const float rstd = 1.0f / sqrtf(ss / (float)j.dh + j.eps);
      const float mean = hx * rstd / (float)j.dh;        // of h xhat
#pragma unroll
      for (int i = 0; i < NS; ++i) {
#pragma unroll
        for (int e = 0; e < C; ++e) {
          const float xh0 = x0[i][e] * rstd, xh1 = x1[i][e] * rstd;
          if (on) { s0[i][e] = fmaf(d0[i][e], xh0, s0[i][e]); s1[i][e] = fmaf(d1[i][e], xh1, s1[i][e]); }
          d0[i][e] = rstd * (d0[i][e] * g0[i][e] - xh0 * mean);
          d1[i][e] = rstd * (d1[i][e] * g1[i][e] - xh1 * mean);
        }
        if (on && k[i].a0 >= 0) Ch::store(dx + k[i].a0, d0[i]);
        if (on && k[i].a1 >= 0) Ch::store(dx + k[i].a1, d1[i]);
      }
    }
  }
  if (!j.partial) return;
  // The units' sums side by side in LDS; then 256 threads take the columns, several groups of units to a column where there are
  // fewer than 256, each group in the order of its units, and the groups in theirs.
  // (Rows of the units four banks apart: at a pitch of 64 the 16 units of a wavefront met on the same banks, 3 us of 11.)
  float* sums = reinterpret_cast<float*>(rope_cs);
  const int pitch = unit_pitch<C>(j.dh);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    float* mine = sums + unit * pitch;
    if constexpr (C > 1) {
#pragma unroll
      for (int e = 0; e < C; e += 4) {
        if (k[i].a0 >= 0) *reinterpret_cast<float4*>(mine + k[i].a0 + e) = make_float4(s0[i][e], s0[i][e + 1], s0[i][e + 2], s0[i][e + 3]);
        if (k[i].a1 >= 0) *reinterpret_cast<float4*>(mine + k[i].a1 + e) = make_float4(s1[i][e], s1[i][e + 1], s1[i][e + 2], s1[i][e + 3]);
      }
    } else {
      if (k[i].a0 >= 0) mine[k[i].a0] = s0[i][0];
      if (k[i].a1 >= 0) mine[k[i].a1] = s1[i][0];
    }
  }
  __syncthreads();
  float* out = j.partial + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * j.dh;
  const int groups = max(1, min(units, NT / j.dh)), per = (units + groups - 1) / groups;
  for (int c0 = 0; c0 < j.dh; c0 += NT) {
    const int g = groups > 1 ? (int)threadIdx.x / j.dh : 0, c = c0 + (groups > 1 ? (int)threadIdx.x - g * j.dh : (int)threadIdx.x);
    float v = 0.f;
    if (c < j.dh && g < groups) {
      const int first = g * per, last = min(units, first + per);
#pragma unroll 8
      for (int u = first; u < last; ++u) v += sums[u * pitch + c];
    }
    if (groups > 1) {                                      // (then c0 is 0: one turn)
      __syncthreads();
      if (c < j.dh && g < groups) sums[g * j.dh + c] = v;
      __syncthreads();
      if (g == 0 && c < j.dh) {
        v = 0.f;
        for (int i = 0; i < groups; ++i) v += sums[i * j.dh + c];
      }
    }
    if (g == 0 && c < j.dh) out[c] = v;
  }
}

// dgamma = alpha (sum of the partials, in order) (+ dgamma).  Workgroup (16 columns, class): 64 groups of 16 threads take
// every 64th partial, four loads under way at a time, and their sums are added in the order of the groups.  (512 partials of
// 64 columns: with 16 groups of 64 columns, one load after the other, 9.3 us.)
struct GammaFinish {
  const float* partial[2];
  int64_t count[2];
  float* out[2];
  float alpha;
  int accumulate, dh;
};
constexpr int FIN_COLS = 16, FIN_GROUPS = 64;
__global__ __launch_bounds__(FIN_COLS * FIN_GROUPS) void gamma_finish_kernel(GammaFinish f) {
  __shared__ float part[FIN_GROUPS][FIN_COLS + 1];
  const int which = blockIdx.y, t = threadIdx.x % FIN_COLS, g = threadIdx.x / FIN_COLS;
  const int c = blockIdx.x * FIN_COLS + t;
  if (!f.out[which]) return;
  float v = 0.f;
  if (c < f.dh) {
    const float* p = f.partial[which] + c;
    const int n = (int)f.count[which];
    for (int i = g; i < n; i += 4 * FIN_GROUPS) {
      float x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = i + u * FIN_GROUPS < n ? p[(int64_t)(i + u * FIN_GROUPS) * f.dh] : 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) v += x[u];
    }
  }
  part[g][t] = v;
  __syncthreads();
  if (g == 0 && c < f.dh) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < FIN_GROUPS; ++i) sum += part[i][t];
    GradOut o{f.out[which], f.alpha, f.accumulate};
    grad_store(o, c, sum);
  }
}

// Whether 16-byte chunks of C elements fit the pointers, strides and the rotated part.
bool chunks_fit(const RopeJob& j, int C, bool bwd) {
  const void* ptrs[3] = {j.x, j.y, bwd ? j.dy : nullptr};
  const int64_t strides[6] = {j.x_row, j.x_head, j.y_row, j.y_head, bwd ? j.dy_row : 0, bwd ? j.dy_head : 0};
  for (const void* p : ptrs)
    if (reinterpret_cast<uintptr_t>(p) % 16) return false;
  for (int64_t s : strides)
    if (s % C) return false;
  if (j.dh % C) return false;
  return j.layout == VF_ROPE_HALF ? j.rot % (2 * C) == 0 : j.rot % C == 0;
}

int log2_ceil(int v) {
  int b = 0;
  while ((1 << b) < v) ++b;
  return b;
}

constexpr int64_t kMaxPartials = 512;       // workgroups along the rows of the backward kernel, per block of heads
constexpr int64_t kMaxRowGroups = 1 << 20;  // ... of the other kernel
constexpr int64_t kFillGroups = 1024;       // workgroups from which the chip is taken to be full

// Lanes per head, rows per workgroup and heads per workgroup.
struct Plan { int slots, ns; dim3 grid; size_t lds; };
Plan plan_of(RopeJob& j, int C, bool bwd) {
  Plan p;
  const int turning = j.rot / (2 * C);
  p.slots = (j.layout == VF_ROPE_HALF || C == 1) ? turning + (j.dh - j.rot + 2 * C - 1) / (2 * C) : (j.dh + 2 * C - 1) / (2 * C);
  j.lane_bits = std::min(6, log2_ceil(p.slots));
  p.ns = (p.slots + (1 << j.lane_bits) - 1) >> j.lane_bits;
  const int units = NT >> j.lane_bits, k_heads = j.heads - j.q_heads;
  // as many rows as give every thread one or two angles, and all their heads
  j.tile = std::max(1, std::min(32, j.rot ? 512 / (j.rot / 2) : 8));
  j.take = std::max(j.q_heads, k_heads);
  // few rows: fewer rows, then fewer heads to a workgroup, as long as its units still have work
  auto groups = [&] {
    return ((j.rows + j.tile - 1) / j.tile) * (int64_t)((j.q_heads + j.take - 1) / j.take + (k_heads + j.take - 1) / j.take);
  };
  while (j.tile > 1 && groups() < kFillGroups && (int64_t)j.tile * j.take > units) j.tile = (j.tile + 1) / 2;
  while (j.take > units && groups() < kFillGroups) j.take = (j.take + 1) / 2;
  j.q_blocks = (j.q_heads + j.take - 1) / j.take;
  const int k_blocks = (k_heads + j.take - 1) / j.take;
  const int64_t gx = std::min((j.rows + j.tile - 1) / j.tile, bwd ? kMaxPartials : kMaxRowGroups);
  p.grid = dim3((unsigned)gx, (unsigned)(j.q_blocks + k_blocks));
  p.lds = (size_t)j.tile * (j.rot / 2) * sizeof(float2);
  if (bwd) p.lds = std::max(p.lds, (size_t)units * (C > 1 ? unit_pitch<4>(j.dh) : unit_pitch<1>(j.dh)) * sizeof(float));
  return p;
}

template <typename T, int C, int NS>
int launch_one(const RopeJob& j, const Plan& p, const Turns& t, bool norm, bool bwd, hipStream_t st) {
  if (bwd) norm_bwd_kernel<T, C, NS><<<p.grid, NT, p.lds, st>>>(j, t);
  else if (norm) rope_kernel<T, C, NS, true><<<p.grid, NT, p.lds, st>>>(j, t);
  else rope_kernel<T, C, NS, false><<<p.grid, NT, p.lds, st>>>(j, t);
  VF_LAUNCH_CHECK();
  return VF_OK;
}

template <typename T, int C>
int launch_typed(RopeJob& j, const Turns& t, bool norm, bool bwd, hipStream_t st, dim3* grid) {
  const bool wide = chunks_fit(j, C, bwd);
  const Plan p = plan_of(j, wide ? C : 1, bwd);
  *grid = p.grid;
  if (wide) return launch_one<T, C, 1>(j, p, t, norm, bwd, st);
  return p.ns == 1 ? launch_one<T, 1, 1>(j, p, t, norm, bwd, st) : launch_one<T, 1, 4>(j, p, t, norm, bwd, st);
}

int launch(int dtype, RopeJob& j, const vf_rope_plan* plan, bool norm, bool bwd, hipStream_t st, dim3* grid) {
  Turns t{};
  if (plan) std::copy(plan->turns, plan->turns + VF_ROPE_MAX_PAIRS, t.t);
  return dtype == VF_BF16 ? launch_typed<bf16_t, 8>(j, t, norm, bwd, st, grid) : launch_typed<float, 4>(j, t, norm, bwd, st, grid);
}

}  // namespace

int64_t rope_partial_floats(int64_t rows, int q_heads, int k_heads, int dh) {
  // workgroups of the backward kernel: at most kMaxPartials for each of the two classes of heads, or, where heads are
  // spread over several, less than twice kFillGroups (a halving of `take` at most doubles them)
  return std::min(rows * (q_heads + k_heads), std::max(2 * kMaxPartials, 2 * kFillGroups)) * dh;
}

int launch_rope(int dtype, RopeJob j, const vf_rope_plan* plan, bool norm, hipStream_t st) {
  dim3 grid;
  return launch(dtype, j, plan, norm, false, st, &grid);
}

int launch_norm_bwd(int dtype, RopeJob j, const vf_rope_plan* plan, float* dgamma_q, float* dgamma_k, float alpha,
                    int accumulate, hipStream_t st) {
  dim3 grid(0, 0);
  if (j.rows > 0 && j.heads > 0) VF_TRY(launch(dtype, j, plan, true, true, st, &grid));
  if (!dgamma_q && !dgamma_k) return VF_OK;
  const int64_t qn = grid.x ? (int64_t)((j.q_heads + j.take - 1) / std::max(1, j.take)) * grid.x : 0;
  GammaFinish f{};
  f.partial[0] = j.partial;
  f.partial[1] = j.partial ? j.partial + qn * j.dh : nullptr;
  f.count[0] = qn;
  f.count[1] = (int64_t)grid.x * grid.y - qn;
  f.out[0] = dgamma_q; f.out[1] = dgamma_k;
  f.alpha = alpha; f.accumulate = accumulate; f.dh = j.dh;
  gamma_finish_kernel<<<dim3((unsigned)((j.dh + FIN_COLS - 1) / FIN_COLS), 2), FIN_COLS * FIN_GROUPS, 0, st>>>(f);
  VF_LAUNCH_CHECK();
  return VF_OK;
}

}  // namespace vf
