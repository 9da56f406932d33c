// Attention of queries to keys and values of another length, forward and backward, on the matrix cores.
//   forward :  z = scale q k^T over the visible keys;  p = exp(z - lse);  o = p v      (one pass: running maximum and sum)
//   backward:  dv = p^T dO;  dp = dO v^T;  dz = p (dp - rowsum(dO o));  dq = scale dz k;  dk = scale dz^T q
// The scores are never stored: the backward kernels take p again from z and lse.
//
// Every kernel holds 32 rows per wavefront in registers as the right operand (queries, or in the dk/dv kernel keys and
// values) and streams tiles of the other side through LDS as the left operand, so that an accumulator tile has the
// held rows as its columns, one per lane (two lanes, l and l + 32, share a column): the softmax statistics are a
// scalar per lane, and the tile is at once the right operand of the product that contracts over its rows.  That
// product needs the streamed tile transposed; bf16 comes out of LDS through the transposing read, fp32 operands hold
// one element per lane and need none.  In both, the contraction's order of rows is that of the accumulator tile.
//
// The query heads that share a key head are rows of one problem (row r = query r / group of head r % group), so the keys
// are read once for all of them and the gradients of shared keys are summed in registers.
#include <algorithm>
#include <atomic>

#include "vf_device.h"

namespace vf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 256;                                     // four wavefronts
constexpr int WR = 32;                                      // held rows of a wavefront
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFar = 1048576.f;                          // log2 units from which 2^-24 of a score is no longer far below 1

// row of register r in a 32 x 32 accumulator tile
__device__ __forceinline__ int acc_row(int r, int half) { return 8 * (r >> 2) + 4 * half + (r & 3); }

template <typename T> struct Elem;
template <> struct Elem<bf16_t> {
  static constexpr int CE = 8;                              // elements of a 16-byte chunk
  static constexpr int TR = 64;                             // rows of a streamed tile
};
template <> struct Elem<float> {
  static constexpr int CE = 4;
  static constexpr int TR = 32;
};

// A streamed tile in LDS: TR rows of DP elements, unpadded; chunk c of row r lies at position c ^ f(r) of its row, f chosen
// so that 16 consecutive rows put equal chunks on 16 different 16-byte columns of the banks, and four consecutive
// rows put four neighbouring chunks on different ones (the transposing read).
template <typename T, int DP>
struct Tile {
  static constexpr int CE = Elem<T>::CE, TR = Elem<T>::TR;
  static constexpr int CH = DP / CE;                        // chunks of a row
  static constexpr int ELEMS = TR * DP;
  static_assert(CH % 4 == 0, "chunks of a row");
  static __device__ __forceinline__ int pos(int r, int c) {
    int f;
    if constexpr (CH % 16 == 0) f = ((r & 3) << 2) | ((r >> 2) & 3);
    else if constexpr (CH % 8 == 0) f = (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    else f = (r >> 2) & 3;
    return r * DP + (c ^ f) * CE;
  }
};

// The right operand held by a lane: column l % 32 of 32 rows, the whole head in steps of two chunks (half h of the
// wavefront holds chunk 2 s + h of step s).
template <typename T, int DP>
struct Held {
  static constexpr int CE = Elem<T>::CE, STEPS = DP / (2 * CE);
  u32x4 w[STEPS];
  // row: first element of the lane's row, or null for zeros; dh: elements of the head
  __device__ __forceinline__ void load(const T* row, int dh, int half) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int e = (2 * s + half) * CE;
      w[s] = u32x4{0u, 0u, 0u, 0u};
      if (row && e < dh) w[s] = *reinterpret_cast<const u32x4*>(row + e);
    }
  }
};

// acc[streamed row][held column] += tile rows row0 .. row0 + 31 times the held rows, over the head.
template <typename T, int DP>
__device__ __forceinline__ void dot_rows(f32x16& acc, const T* tile, int row0, const Held<T, DP>& b, int lane) {
  const int r = row0 + (lane & 31), half = lane >> 5;
#pragma unroll
  for (int s = 0; s < Held<T, DP>::STEPS; ++s) {
    const u32x4 a = *reinterpret_cast<const u32x4*>(tile + Tile<T, DP>::pos(r, 2 * s + half));
    if constexpr (sizeof(T) == 2) {
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b.w[s]), acc, 0, 0, 0);
    } else {
      const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b.w[s]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc, 0, 0, 0);
    }
  }
}

// Transposing read: elements (row0 + 4 half + 0..3, col0 + l % 32) and the same eight rows further down.
template <int DP>
__device__ __forceinline__ bf16x8 read_cols(const bf16_t* tile, int row0, int col0, int lane) {
  const int s = lane & 15, half = lane >> 5;
  const int r = row0 + 4 * half + (s >> 2), c = col0 + ((lane >> 4) & 1) * 16 + 4 * (s & 3);
  const bf16_t* p0 = tile + Tile<bf16_t, DP>::pos(r, c >> 3) + (c & 7);
  const bf16_t* p1 = tile + Tile<bf16_t, DP>::pos(r + 8, c >> 3) + (c & 7);
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)p0);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)p1);
  bf16x8 v;
  __builtin_memcpy(&v, &lo, 8);
  __builtin_memcpy(reinterpret_cast<char*>(&v) + 8, &hi, 8);
  return v;
}

// acc[db][head element 32 db + ..][held column] += sum over tile rows row0 .. row0 + 31 of tile[row][element] w[row][column].
// w is an accumulator tile; bf16 rounds it (the operand of a product).
template <typename T, int DP>
__device__ __forceinline__ void dot_cols(f32x16 (&acc)[DP / 32], const T* tile, int row0, const f32x16& w, int lane) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 b[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 packed;
#pragma unroll
      for (int u = 0; u < 4; ++u) packed[u] = f32x2_to_bf16x2(w[8 * s + 2 * u], w[8 * s + 2 * u + 1]);
      b[s] = __builtin_bit_cast(bf16x8, packed);
    }
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
      for (int s = 0; s < 2; ++s)
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_cols<DP>(tile, row0 + 16 * s, 32 * db, lane), b[s], acc[db], 0, 0, 0);
  } else {
    const int half = lane >> 5, m = lane & 31;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = row0 + acc_row(r, half);
#pragma unroll
      for (int db = 0; db < DP / 32; ++db) {
        const int col = 32 * db + m;
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(tile[Tile<T, DP>::pos(row, col >> 2) + (col & 3)], w[r], acc[db], 0, 0, 0);
      }
    }
  }
}

template <int N>
__device__ __forceinline__ void clear(f32x16 (&a)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) a[i][r] = 0.f;
}

// A tile on its way from memory: chunks of this thread, in registers until the buffer they go to is free.
template <typename T, int DP>
struct Stage {
  static constexpr int CE = Elem<T>::CE, CH = DP / CE, N = Elem<T>::TR * CH / NT;
  static_assert(Elem<T>::TR * CH % NT == 0, "chunks of a tile over the threads");
  u32x4 w[N];
  static __device__ __forceinline__ int row(int i) { return (i * NT + (int)threadIdx.x) / CH; }
  static __device__ __forceinline__ int chunk(int i) { return (i * NT + (int)threadIdx.x) % CH; }
  // row_ptr(r): first element of tile row r, or null for a row of zeros
  template <typename F>
  __device__ __forceinline__ void fetch(F row_ptr, int dh) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const T* p = row_ptr(row(i));
      w[i] = u32x4{0u, 0u, 0u, 0u};
      if (p && chunk(i) * CE < dh) w[i] = *reinterpret_cast<const u32x4*>(p + chunk(i) * CE);
    }
  }
  __device__ __forceinline__ void put(T* tile) const {
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(tile + Tile<T, DP>::pos(row(i), chunk(i))) = w[i];
  }
};

// One (batch, key head) problem.
struct Problem {
  int b, hk;
  int rows, q_len;            // rows = group * q_rows
  int keys;                   // k_len, clamped
};
__device__ __forceinline__ Problem problem_of(const AttnJob& j, int id) {
  Problem p;
  p.b = id / j.s.kv_heads;
  p.hk = id - p.b * j.s.kv_heads;
  p.rows = j.group * j.s.q_rows;
  p.q_len = j.q_len ? min(max(j.q_len[p.b], 0), j.s.q_rows) : j.s.q_rows;
  p.keys = j.k_len ? min(max(j.k_len[p.b], 0), j.s.k_rows) : j.s.k_rows;
  return p;
}
// query and head (among the group's) of row r
struct RowOf { int t, g; };
__device__ __forceinline__ RowOf row_of(const AttnJob& j, int r) {
  if (j.group == 1) return {r, 0};
  const int t = (int)__umulhi((uint32_t)r, j.group_inv);
  return {t, r - t * j.group};
}
template <typename T>
__device__ __forceinline__ T* at(const void* base, const vf_attn_layout& l, int b, int row, int head) {
  return const_cast<T*>(static_cast<const T*>(base)) + (int64_t)b * l.batch + (int64_t)row * l.row + (int64_t)head * l.head;
}

// Which of the keys k0 .. k0 + 63 are visible, one bit each (the same in every lane of the wavefront).
__device__ __forceinline__ uint64_t visible(const AttnJob& j, const Problem& p, int k0, int lane) {
  const int k = k0 + lane;
  bool on = k < p.keys;
  if (j.key_mask && on) on = j.key_mask[(int64_t)p.b * j.s.k_rows + k] != 0;
  return __ballot(on);
}

// max / sum over the two lanes of a column
__device__ __forceinline__ float pair_max(float v) { return fmaxf(v, __shfl_xor(v, 32, 64)); }
__device__ __forceinline__ float pair_sum(float v) { return v + __shfl_xor(v, 32, 64); }

// An accumulator over the head (elements down, held rows across), times `f`, to the lane's row.
template <typename T, int DP>
__device__ __forceinline__ void store_row(T* row, const f32x16 (&acc)[DP / 32], float f, int dh, int half) {
#pragma unroll
  for (int db = 0; db < DP / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int e = 32 * db + 8 * g + 4 * half;
      if (e >= dh) continue;
      const float a = acc[db][4 * g] * f, b = acc[db][4 * g + 1] * f, c = acc[db][4 * g + 2] * f, d = acc[db][4 * g + 3] * f;
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint2*>(row + e) = make_uint2(f32x2_to_bf16x2(a, b), f32x2_to_bf16x2(c, d));
      } else {
        *reinterpret_cast<float4*>(row + e) = make_float4(a, b, c, d);
      }
    }
}

// ---- forward ------------------------------------------------------------------------------------
template <typename T, int DP>
__global__ __launch_bounds__(NT, 2) void xattn_fwd_kernel(AttnJob j, int tiles) {
  constexpr int TR = Elem<T>::TR, KB = TR / 32, ELEMS = Tile<T, DP>::ELEMS;
  extern __shared__ __attribute__((aligned(16))) char xattn_lds[];
  T* lds = reinterpret_cast<T*>(xattn_lds);                 // [2][k, v][ELEMS]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const Problem p = problem_of(j, blockIdx.x / tiles);
  const int r = (blockIdx.x % tiles) * (4 * WR) + wave * WR + (lane & 31);
  const bool mine = r < p.rows;
  const RowOf ro = row_of(j, mine ? r : 0);
  const int head = p.hk * j.group + ro.g;
  const bool live = mine && ro.t < p.q_len;
  const int dh = j.s.d_head;
  const float c = j.s.scale * kLog2e;

  Held<T, DP> q;
  q.load(live ? at<const T>(j.q, j.s.q, p.b, ro.t, head) : nullptr, dh, half);
  f32x16 o[DP / 32];
  clear(o);
  float m = -INFINITY, l = 0.f;

  const T* kbase = at<const T>(j.k, j.s.k, p.b, 0, p.hk);
  const T* vbase = at<const T>(j.v, j.s.v, p.b, 0, p.hk);
  Stage<T, DP> ks, vs;
  auto fetch = [&](int k0, uint64_t vis) {
    ks.fetch([&](int t) { return (vis >> t) & 1 ? kbase + (int64_t)(k0 + t) * j.s.k.row : nullptr; }, dh);
    vs.fetch([&](int t) { return (vis >> t) & 1 ? vbase + (int64_t)(k0 + t) * j.s.v.row : nullptr; }, dh);
  };
  uint64_t vis = p.keys > 0 ? visible(j, p, 0, lane) : 0;
  if (p.keys > 0) fetch(0, vis);
  int buf = 0;
  for (int k0 = 0; k0 < p.keys; k0 += TR, buf ^= 1) {
    T* kt = lds + buf * 2 * ELEMS;
    T* vt = kt + ELEMS;
    ks.put(kt);
    vs.put(vt);
    const uint64_t now = vis;
    if (k0 + TR < p.keys) {
      vis = visible(j, p, k0 + TR, lane);
      fetch(k0 + TR, vis);
    }
    __syncthreads();                                        // (two buffers: the next iteration writes the other one)
    f32x16 s[KB];
    clear(s);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) dot_rows<T, DP>(s[kb], kt, 32 * kb, q, lane);
    const uint64_t all = TR == 64 ? ~0ull : 0xffffffffull;
    if ((now & all) != all) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const uint32_t bits = (uint32_t)(now >> (32 * kb)) >> (4 * half);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!((bits >> acc_row(i, 0)) & 1)) s[kb][i] = -INFINITY;
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
    const float mn = fmaxf(m, pair_max(top));
    const float ref = mn == -INFINITY ? 0.f : mn;           // no visible key so far: every p is exp2(-inf) = 0
    const float fade = __builtin_amdgcn_exp2f((m - ref) * c);
    const float base = ref * c;
    m = mn;
    // s c - base in one operation keeps the rounding of base: nothing as long as that is far below 1, and the same
    // factor for all of a row; where it is not, the difference is taken first.
    if (__any(fabsf(base) > kFar)) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = __builtin_amdgcn_exp2f((s[kb][i] - ref) * c);
    } else {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = __builtin_amdgcn_exp2f(fmaf(s[kb][i], c, -base));
    }
    float sum = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum += s[kb][i];
    l = l * fade + sum;
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] *= fade;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) dot_cols<T, DP>(o, vt, 32 * kb, s[kb], lane);
  }
  if (!mine) return;
  l = pair_sum(l);
  const bool any = live && l != 0.f;                        // (a NaN goes on)
  store_row<T, DP>(at<T>(j.o, j.s.o, p.b, ro.t, head), o, any ? 1.f / l : 0.f, dh, half);
  if (j.lse && half == 0)
    j.lse[((int64_t)p.b * j.s.q_heads + head) * j.s.q_rows + ro.t] = any ? fmaf(m, j.s.scale, logf(l)) : -INFINITY;
}

// ---- backward: dq, and lse / rowsum(dO o) of every row for the kernel behind it ---------------------
template <typename T, int DP>
__global__ __launch_bounds__(NT, 1) void xattn_dq_kernel(AttnJob j, int tiles) {
  constexpr int TR = Elem<T>::TR, KB = TR / 32, ELEMS = Tile<T, DP>::ELEMS;
  extern __shared__ __attribute__((aligned(16))) char xattn_lds[];
  T* lds = reinterpret_cast<T*>(xattn_lds);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int id = blockIdx.x / tiles;
  const Problem p = problem_of(j, id);
  const int r = (blockIdx.x % tiles) * (4 * WR) + wave * WR + (lane & 31);
  const bool mine = r < p.rows;
  const RowOf ro = row_of(j, mine ? r : 0);
  const int head = p.hk * j.group + ro.g;
  const int dh = j.s.d_head;
  const float c = j.s.scale * kLog2e;
  const float lse_in = mine && ro.t < p.q_len ? j.lse[((int64_t)p.b * j.s.q_heads + head) * j.s.q_rows + ro.t] : -INFINITY;
  const bool live = lse_in != -INFINITY;                    // a row without a visible key has p = 0 everywhere
  const float lse = live ? lse_in * kLog2e : INFINITY;

  Held<T, DP> q, g;
  q.load(live ? at<const T>(j.q, j.s.q, p.b, ro.t, head) : nullptr, dh, half);
  g.load(live ? at<const T>(j.d_o, j.s.d_o, p.b, ro.t, head) : nullptr, dh, half);
  float delta = 0.f;
  {
    Held<T, DP> out;
    out.load(live ? at<const T>(j.o, j.s.o, p.b, ro.t, head) : nullptr, dh, half);
#pragma unroll
    for (int s = 0; s < Held<T, DP>::STEPS; ++s)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if constexpr (sizeof(T) == 2) {
          delta = fmaf(__uint_as_float(out.w[s][u] << 16), __uint_as_float(g.w[s][u] << 16), delta);
          delta = fmaf(__uint_as_float(out.w[s][u] & 0xffff0000u), __uint_as_float(g.w[s][u] & 0xffff0000u), delta);
        } else {
          delta = fmaf(__uint_as_float(out.w[s][u]), __uint_as_float(g.w[s][u]), delta);
        }
      }
    delta = pair_sum(delta);
  }
  if (mine && half == 0) {
    j.row_lse[(int64_t)id * p.rows + r] = lse;
    j.row_delta[(int64_t)id * p.rows + r] = delta;
  }
  f32x16 dq[DP / 32];
  clear(dq);

  const T* kbase = at<const T>(j.k, j.s.k, p.b, 0, p.hk);
  const T* vbase = at<const T>(j.v, j.s.v, p.b, 0, p.hk);
  Stage<T, DP> ks, vs;
  auto fetch = [&](int k0, uint64_t vis) {
    ks.fetch([&](int t) { return (vis >> t) & 1 ? kbase + (int64_t)(k0 + t) * j.s.k.row : nullptr; }, dh);
    vs.fetch([&](int t) { return (vis >> t) & 1 ? vbase + (int64_t)(k0 + t) * j.s.v.row : nullptr; }, dh);
  };
  uint64_t vis = p.keys > 0 ? visible(j, p, 0, lane) : 0;
  if (p.keys > 0) fetch(0, vis);
  int buf = 0;
  for (int k0 = 0; k0 < p.keys; k0 += TR, buf ^= 1) {
    T* kt = lds + buf * 2 * ELEMS;
    T* vt = kt + ELEMS;
    ks.put(kt);
    vs.put(vt);
    const uint64_t now = vis;
    if (k0 + TR < p.keys) {
      vis = visible(j, p, k0 + TR, lane);
      fetch(k0 + TR, vis);
    }
    __syncthreads();
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      f32x16 s[1], dp[1];
      clear(s);
      clear(dp);
      dot_rows<T, DP>(s[0], kt, 32 * kb, q, lane);
      dot_rows<T, DP>(dp[0], vt, 32 * kb, g, lane);
      const uint32_t bits = (uint32_t)(now >> (32 * kb)) >> (4 * half);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float pr = __builtin_amdgcn_exp2f(fminf(fmaf(s[0][i], c, -lse), 0.f));   // (scores so far out that the rounding of lse passes 1)
        if (!((bits >> acc_row(i, 0)) & 1)) pr = 0.f;
        s[0][i] = pr * (dp[0][i] - delta);
      }
      dot_cols<T, DP>(dq, kt, 32 * kb, s[0], lane);
    }
  }
  if (mine) store_row<T, DP>(at<T>(j.dq, j.s.dq, p.b, ro.t, head), dq, j.s.scale, dh, half);
}

// ---- backward: dk and dv ------------------------------------------------------------------------------
template <typename T, int DP>
__global__ __launch_bounds__(NT, 1) void xattn_dkv_kernel(AttnJob j, int tiles) {
  constexpr int TR = Elem<T>::TR, QB = TR / 32, ELEMS = Tile<T, DP>::ELEMS;
  extern __shared__ __attribute__((aligned(16))) char xattn_lds[];
  T* lds = reinterpret_cast<T*>(xattn_lds);                 // [2][q, dO][ELEMS], then [2][lse, delta][TR]
  float* stats = reinterpret_cast<float*>(lds + 4 * ELEMS);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int id = blockIdx.x / tiles;
  const Problem p = problem_of(j, id);
  const int key = (blockIdx.x % tiles) * (4 * WR) + wave * WR + (lane & 31);
  const bool mine = key < j.s.k_rows;
  bool seen = key < p.keys;
  if (j.key_mask && seen) seen = j.key_mask[(int64_t)p.b * j.s.k_rows + key] != 0;
  const int dh = j.s.d_head;
  const float c = j.s.scale * kLog2e;

  Held<T, DP> k, v;
  k.load(seen ? at<const T>(j.k, j.s.k, p.b, key, p.hk) : nullptr, dh, half);
  v.load(seen ? at<const T>(j.v, j.s.v, p.b, key, p.hk) : nullptr, dh, half);
  f32x16 dk[DP / 32], dv[DP / 32];
  clear(dk);
  clear(dv);

  const int rows = p.q_len * j.group;                       // padding lies behind them
  Stage<T, DP> qs, gs;
  float stat = 0.f;
  auto fetch = [&](int r0) {
    auto row = [&](const void* base, const vf_attn_layout& l, int t) -> const T* {
      if (r0 + t >= rows) return nullptr;
      const RowOf ro = row_of(j, r0 + t);
      return at<const T>(base, l, p.b, ro.t, p.hk * j.group + ro.g);
    };
    qs.fetch([&](int t) { return row(j.q, j.s.q, t); }, dh);
    gs.fetch([&](int t) { return row(j.d_o, j.s.d_o, t); }, dh);
    const int t = threadIdx.x % TR;
    if (threadIdx.x < 2 * TR) {
      const float* from = threadIdx.x < TR ? j.row_lse : j.row_delta;
      stat = r0 + t < rows ? from[(int64_t)id * p.rows + r0 + t] : (threadIdx.x < TR ? INFINITY : 0.f);
    }
  };
  const bool block_seen = (blockIdx.x % tiles) * (4 * WR) < p.keys;      // else nothing but zeros to write
  const int end = block_seen ? rows : 0;
  if (end > 0) fetch(0);
  int buf = 0;
  for (int r0 = 0; r0 < end; r0 += TR, buf ^= 1) {
    T* qt = lds + buf * 2 * ELEMS;
    T* gt = qt + ELEMS;
    float* st = stats + buf * 2 * TR;
    qs.put(qt);
    gs.put(gt);
    if (threadIdx.x < 2 * TR) st[threadIdx.x] = stat;
    if (r0 + TR < end) fetch(r0 + TR);
    __syncthreads();
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      f32x16 s[1], dp[1];
      clear(s);
      clear(dp);
      dot_rows<T, DP>(s[0], qt, 32 * qb, k, lane);
      dot_rows<T, DP>(dp[0], gt, 32 * qb, v, lane);
#pragma unroll
      for (int gq = 0; gq < 4; ++gq) {
        const f32x4 lse = *reinterpret_cast<const f32x4*>(st + 32 * qb + 8 * gq + 4 * half);
        const f32x4 delta = *reinterpret_cast<const f32x4*>(st + TR + 32 * qb + 8 * gq + 4 * half);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float pr = __builtin_amdgcn_exp2f(fminf(fmaf(s[0][4 * gq + i], c, -lse[i]), 0.f));
          s[0][4 * gq + i] = pr;
          dp[0][4 * gq + i] = pr * (dp[0][4 * gq + i] - delta[i]);
        }
      }
      dot_cols<T, DP>(dv, gt, 32 * qb, s[0], lane);
      dot_cols<T, DP>(dk, qt, 32 * qb, dp[0], lane);
    }
  }
  if (!mine) return;
  // an invisible key's columns hold what its zeros gave: nothing of it is stored
  if (!seen) { clear(dk); clear(dv); }
  store_row<T, DP>(at<T>(j.dk, j.s.dk, p.b, key, p.hk), dk, j.s.scale, dh, half);
  store_row<T, DP>(at<T>(j.dv, j.s.dv, p.b, key, p.hk), dv, 1.f, dh, half);
}

// LDS above 64 KB has to be allowed for a kernel once on every device.
int allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  VF_HIP(hipGetDevice(&dev));
  const uint64_t bit = 1ull << (dev & 63);
  if (done.load(std::memory_order_relaxed) & bit) return VF_OK;
  VF_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
  if (dev < 64) done.fetch_or(bit, std::memory_order_relaxed);
  return VF_OK;
}

template <typename T, int DP>
int launch_fwd(const AttnJob& j, hipStream_t st) {
  constexpr int lds = 4 * Tile<T, DP>::ELEMS * sizeof(T);
  static std::atomic<uint64_t> ready{0};
  VF_TRY(allow_lds(reinterpret_cast<const void*>(&xattn_fwd_kernel<T, DP>), lds, ready));
  const int tiles = (j.group * j.s.q_rows + 4 * WR - 1) / (4 * WR);
  xattn_fwd_kernel<T, DP><<<j.s.batch * j.s.kv_heads * tiles, NT, lds, st>>>(j, tiles);
  VF_LAUNCH_CHECK();
  return VF_OK;
}

template <typename T, int DP>
int launch_bwd(const AttnJob& j, hipStream_t st) {
  constexpr int lds = 4 * Tile<T, DP>::ELEMS * sizeof(T), lds_kv = lds + 4 * Elem<T>::TR * sizeof(float);
  static std::atomic<uint64_t> ready_q{0}, ready_kv{0};
  VF_TRY(allow_lds(reinterpret_cast<const void*>(&xattn_dq_kernel<T, DP>), lds, ready_q));
  VF_TRY(allow_lds(reinterpret_cast<const void*>(&xattn_dkv_kernel<T, DP>), lds_kv, ready_kv));
  const int heads = j.s.batch * j.s.kv_heads;
  const int qt = (j.group * j.s.q_rows + 4 * WR - 1) / (4 * WR), kt = (j.s.k_rows + 4 * WR - 1) / (4 * WR);
  if (qt) {
    xattn_dq_kernel<T, DP><<<heads * qt, NT, lds, st>>>(j, qt);
    VF_LAUNCH_CHECK();
  }
  if (kt) {
    xattn_dkv_kernel<T, DP><<<heads * kt, NT, lds_kv, st>>>(j, kt);
    VF_LAUNCH_CHECK();
  }
  return VF_OK;
}

}  // namespace

// Backward: two floats per row (lse and rowsum(dO o)).
int64_t attn_workspace_bytes(const vf_attn_shape& s, bool backward) {
  if (!backward) return 0;
  return (int64_t)s.batch * s.q_heads * s.q_rows * 2 * (int64_t)sizeof(float);
}

int launch_attn(const AttnJob& j, void*, hipStream_t st) {
  if (!j.s.batch || !j.s.q_rows) return VF_OK;
  const bool wide = j.s.d_head > 64;
  if (j.s.dtype == VF_BF16) return wide ? launch_fwd<bf16_t, 128>(j, st) : launch_fwd<bf16_t, 64>(j, st);
  return wide ? launch_fwd<float, 128>(j, st) : launch_fwd<float, 64>(j, st);
}

int launch_attn_bwd(AttnJob j, void* workspace, hipStream_t st) {
  if (!j.s.batch || (!j.s.q_rows && !j.s.k_rows)) return VF_OK;
  j.row_lse = static_cast<float*>(workspace);
  j.row_delta = j.row_lse + (int64_t)j.s.batch * j.s.q_heads * j.s.q_rows;
  const bool wide = j.s.d_head > 64;
  if (j.s.dtype == VF_BF16) return wide ? launch_bwd<bf16_t, 128>(j, st) : launch_bwd<bf16_t, 64>(j, st);
  return wide ? launch_bwd<float, 128>(j, st) : launch_bwd<float, 64>(j, st);
}

}  // namespace vf
