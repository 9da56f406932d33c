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
#include <type_traits>

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
constexpr float kSlack = 8.f;                              // see the forward kernel
constexpr float kFar = 1048576.f;                          // log2 units from which 2^-24 of a score is no longer far below 1

// row of register r in a 32 x 32 accumulator tile
__device__ __forceinline__ int acc_row(int r, int half) { return 8 * (r >> 2) + 4 * half + (r & 3); }

template <typename T> struct Elem;
template <> struct Elem<bf16_t> {
  static constexpr int CE = 8;                              // elements of a 16-byte chunk
  static constexpr int TR = 64;                             // rows of a streamed tile, at least
};
template <> struct Elem<float> {
  static constexpr int CE = 4;
  static constexpr int TR = 32;
};
// The four wavefronts of a workgroup hold 4 / SW blocks of 32 rows; the SW wavefronts that hold the same block take
// different blocks of 32 streamed rows of a tile, and their results are joined at the end.
template <typename T, int SW> constexpr int tile_rows() { return Elem<T>::TR > 32 * SW ? Elem<T>::TR : 32 * SW; }

// A streamed tile in LDS: rows of DP elements, unpadded; chunk c of row r lies at position c ^ f(r) of its row, f chosen
// so that 16 consecutive rows put equal chunks on 16 different 16-byte columns of the banks, and four consecutive
// rows put four neighbouring chunks on different ones (the transposing read).
template <typename T, int DP>
struct Tile {
  static constexpr int CE = Elem<T>::CE;
  static constexpr int CH = DP / CE;                        // chunks of a row
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
  // Waits for the loads here: the compiler does not count the loads of tiles, and would wait for all of them at the first use
  // of w in the loop, in every iteration.
  __device__ __forceinline__ void arrive() {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) asm volatile("" : "+v"(w[s]));
  }
};

// acc[streamed row][held column] = 32 tile rows times the held rows, over the head; two such products at once (rows ra of tile ta
// with a, rows rb of tile tb with b), their operations in turn.  The operands are asked for AHEAD steps ahead of their use:
// left to itself the compiler waits for every one of them just before the instruction that takes it.
template <typename T>
__device__ __forceinline__ void step_of(f32x16& acc, u32x4 x, u32x4 y) {
  if constexpr (sizeof(T) == 2) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
  } else {
    const f32x4 u = __builtin_bit_cast(f32x4, x), v = __builtin_bit_cast(f32x4, y);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(u[e], v[e], acc, 0, 0, 0);
  }
}
template <typename T, int DP, bool TWO, int AHEAD = 4>
__device__ __forceinline__ void dot_rows(f32x16& accA, const T* ta, int ra, const Held<T, DP>& a, f32x16& accB, const T* tb, int rb,
                                         const Held<T, DP>& b, int lane) {
  constexpr int S = Held<T, DP>::STEPS, LOOK = S < AHEAD ? S : AHEAD, PAIR = TWO ? 2 : 1, OPS = PAIR * (sizeof(T) == 2 ? 1 : 4);
  const int half = lane >> 5;
  ra += lane & 31;
  rb += lane & 31;
  u32x4 x[S], y[S];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    x[s] = *reinterpret_cast<const u32x4*>(ta + Tile<T, DP>::pos(ra, 2 * s + half));
    if constexpr (TWO) y[s] = *reinterpret_cast<const u32x4*>(tb + Tile<T, DP>::pos(rb, 2 * s + half));
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) accA[i] = accB[i] = 0.f;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    step_of<T>(accA, x[s], a.w[s]);
    if constexpr (TWO) step_of<T>(accB, y[s], b.w[s]);
  }
  __builtin_amdgcn_sched_group_barrier(0x100, PAIR * LOOK, 0);     // LDS reads
#pragma unroll
  for (int s = 0; s < S - LOOK; ++s) {
    __builtin_amdgcn_sched_group_barrier(0x8, OPS, 0);             // matrix instructions
    __builtin_amdgcn_sched_group_barrier(0x100, PAIR, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x8, OPS * LOOK, 0);
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
// w is an accumulator tile; bf16 rounds it (the operand of a product).  With TWO, acc2 += the same rows times w2.
template <typename T, int DP, bool TWO = false>
__device__ __forceinline__ void dot_cols(f32x16 (&acc)[DP / 32], const T* tile, int row0, const f32x16& w, int lane,
                                         f32x16 (*acc2)[DP / 32] = nullptr, const f32x16* w2 = nullptr) {
  if constexpr (sizeof(T) == 2) {
    auto operand = [](const f32x16& v, int s) {
      u32x4 packed;
#pragma unroll
      for (int u = 0; u < 4; ++u) packed[u] = f32x2_to_bf16x2(v[8 * s + 2 * u], v[8 * s + 2 * u + 1]);
      return __builtin_bit_cast(bf16x8, packed);
    };
    bf16x8 b[2], b2[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      b[s] = operand(w, s);
      if constexpr (TWO) b2[s] = operand(*w2, s);
    }
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const bf16x8 a = read_cols<DP>(tile, row0 + 16 * s, 32 * db, lane);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b[s], acc[db], 0, 0, 0);
        if constexpr (TWO) (*acc2)[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b2[s], (*acc2)[db], 0, 0, 0);
      }
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

// Tiles go from memory straight into LDS (global_load_lds_dwordx4: the lanes of a wavefront deposit 16 bytes each, side by
// side), so a tile under way costs no registers, and a ring of STAGES buffers keeps STAGES - 1 of them under way.  The order of
// chunks in LDS is made on the memory side: a lane fetches the chunk that belongs at its place.  Rows that are padding or
// invisible and chunks behind the head come from a block of zeros: nothing that lies there in memory reaches a product.
// Loads of a wavefront complete in order, so "all but the newest n" (vmcnt) says when a tile is there.  (M0 holds a load's LDS address;
// nothing else in these kernels uses it.)
__device__ __attribute__((aligned(16))) uint32_t g_zeros[4];
__device__ uint32_t g_infinity = 0x7f800000u;

__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(const void __attribute__((address_space(3)))*)p; }
__device__ __forceinline__ void lds_load16(const void* src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(dst), "v"(src) : "memory");
}
__device__ __forceinline__ void lds_load16(const char* base, uint32_t off, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void lds_load4(const void* src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(dst), "v"(src) : "memory");
}
// all but the newest N loads there, own LDS reads done; then all wavefronts meet
template <int N>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// ... for the next tile of a ring: all but the STAGES - 2 tiles behind it, of LOADS loads each, or, at the end of the stream, all
template <int STAGES, int LOADS>
__device__ __forceinline__ void meet_for_tile(bool more) {
  if (STAGES == 2 || !more) wait_and_meet<0>();
  else wait_and_meet<(STAGES - 2) * LOADS>();
}

template <typename T, int DP, int SW>
struct Ring {
  static constexpr int CE = Elem<T>::CE, CH = DP / CE, TR = tile_rows<T, SW>(), N = TR * CH / NT;   // N: loads of a wavefront per tile
  static constexpr int ELEMS = TR * DP, BYTES = ELEMS * (int)sizeof(T);
  static constexpr int STAGES = BYTES <= 8192 ? 3 : 2;      // 48 KB (64 KB) for pairs of tiles: three (two) workgroups to a compute unit
  static constexpr int LDS = 2 * STAGES * BYTES;
  // room for the join of the wavefronts' results: 128 rows of DP + 4 floats, and their statistics
  static constexpr int JOIN_PITCH = DP + 4, JOIN = SW > 1 ? 128 * JOIN_PITCH * 4 + 128 * 12 : 0;
  static_assert(TR * CH % NT == 0, "chunks of a tile over the threads");
};

// What a workgroup does: tile `tile` of the held rows of problem `id`, a part of the streamed side from tile `first` on.
// Grid (problems, tiles, parts): neighbouring workgroups go to different XCDs, so with a multiple of 8 problems all workgroups
// that stream the same rows share an L2.  (A contiguous run of the numbers for each XCD: no faster at 2 x 16 problems of 4096 x
// 8192 x 128, and three integer divisions a workgroup cost 3 us of 12 where it has two tiles.)
struct Work { int id, tile, part, first; };
__device__ __forceinline__ Work work_of(const AttnSplit& sp) {
  return {(int)blockIdx.x, (int)blockIdx.y, (int)blockIdx.z, (int)blockIdx.z * sp.per};
}

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
  typedef const __attribute__((address_space(4))) int32_t* scalar;        // (the same for all: scalar loads)
  p.q_len = j.q_len ? min(max(((scalar)j.q_len)[p.b], 0), j.s.q_rows) : j.s.q_rows;
  p.keys = j.k_len ? min(max(((scalar)j.k_len)[p.b], 0), j.s.k_rows) : j.s.k_rows;
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

// This thread's chunks of one streamed tensor.  Row r of the problem is head r % group of row r / group (GROUPED), or row r.
// Where the rows of a tile lie within 32 bits of its first one, and every tile starts with the group's first head, a tile's
// addresses are a scalar that moves on and offsets that stay (`near`): no vector instruction for a whole tile.
template <typename T, int DP, int SW, bool GROUPED>
struct Source {
  static constexpr int N = Ring<T, DP, SW>::N, CH = Ring<T, DP, SW>::CH, TR = Ring<T, DP, SW>::TR, WORDS = (TR + 63) / 64;
  static_assert(WORDS <= 2, "words of bits");
  const char* base;             // head 0 of row 0
  int64_t row_b, head_b;        // strides in bytes
  bool near;
  uint32_t off[N];
  static __device__ __forceinline__ int row(int i) { return (i * NT + (int)threadIdx.x) / CH; }
  // first element of chunk i in its row (the exchange of places undoes itself)
  static __device__ __forceinline__ int elem(int i) { return Tile<T, DP>::pos(row(i), (i * NT + (int)threadIdx.x) % CH) - row(i) * DP; }
  __device__ __forceinline__ void init(const AttnJob& j, const T* first, const vf_attn_layout& l) {
    base = reinterpret_cast<const char*>(first);
    row_b = l.row * (int64_t)sizeof(T);
    head_b = l.head * (int64_t)sizeof(T);
    near = row_b >= 0 && (!GROUPED || head_b >= 0) && TR * row_b + (GROUPED ? j.group * head_b : 0) < (1ll << 31) && (!GROUPED || TR % j.group == 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const RowOf ro = GROUPED ? row_of(j, row(i)) : RowOf{row(i), 0};
      off[i] = (near ? (uint32_t)ro.t * (uint32_t)row_b + (uint32_t)ro.g * (uint32_t)head_b : 0) + elem(i) * (uint32_t)sizeof(T);
    }
  }
  // Which of this thread's chunks are wanted: those of rows whose bit is set, within the head.
  static __device__ __forceinline__ void wanted(const uint64_t (&rows)[WORDS], int dh, bool (&on)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (NT % CH == 0) {                         // (a load's rows lie within one word)
        const uint64_t word = rows[i * (NT / CH) / 64] >> (threadIdx.x / CH);
        on[i] = (uint32_t)(word >> (i * (NT / CH) % 64)) & 1;
      } else {
        const int r = row(i);
        on[i] = (uint32_t)((WORDS > 1 && r >= 64 ? rows[WORDS - 1] : rows[0]) >> (r & 63)) & 1;
      }
      if (dh < DP) on[i] = on[i] && elem(i) < dh;
    }
  }
  // The tile's first row
  __device__ __forceinline__ const char* start(const AttnJob& j, int r0) const { return base + (GROUPED ? row_of(j, r0) : RowOf{r0, 0}).t * row_b; }
  // Tile from row r0 on, all of it.  tile: LDS address of the tile's buffer for this wavefront
  __device__ __forceinline__ void issue(const AttnJob& j, int r0, uint32_t tile) const {
    const char* from = start(j, r0);
#pragma unroll
    for (int i = 0; i < N; ++i) lds_load16(from, off[i], tile + i * (NT * 16));
  }
  // ... the wanted chunks; zeros for the others
  __device__ __forceinline__ void issue(const AttnJob& j, int r0, const bool (&on)[N], const char* zeros, uint32_t tile) const {
    const char* from = start(j, r0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const char* p = from + off[i];
      if (!near) {
        const RowOf ro = GROUPED ? row_of(j, r0 + row(i)) : RowOf{r0 + row(i), 0};
        p = base + ro.t * row_b + ro.g * head_b + off[i];
      }
      lds_load16(on[i] ? p : zeros, tile + i * (NT * 16));
    }
  }
};
// A pair of tiles (rows r0 on of two tensors): rows as bits; whole: all of them, and the head fills its chunks.
template <typename S>
__device__ __forceinline__ void issue_pair(const AttnJob& j, const S& a, const S& b, int r0, const uint64_t (&rows)[S::WORDS], bool whole, int dh,
                                           const char* zeros, uint32_t tile_a, uint32_t tile_b) {
  if (whole && a.near && b.near) {
    a.issue(j, r0, tile_a);
    b.issue(j, r0, tile_b);
    return;
  }
  bool on[S::N];
  S::wanted(rows, dh, on);
  a.issue(j, r0, on, zeros, tile_a);
  b.issue(j, r0, on, zeros, tile_b);
}

__device__ __forceinline__ uint64_t first_bits(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }
// An address in scalar registers that is not taken again in the loops.
__device__ __forceinline__ const char* fixed_address(const void* p) {
  const char* z = static_cast<const char*>(p);
  asm volatile("" : "+s"(z));
  return z;
}

// Which of the keys k0 .. k0 + 63 are visible, one bit each.  A mask comes as such bits.  Up to kMaskWords words a workgroup makes
// them itself from the part of the mask it needs (take_mask: words[i], keys first + 64 i ...); longer ones come from
// mask_bits_kernel (k0 a multiple of 32) by scalar loads, which do not stand in the queue of the tiles' loads.
constexpr int kMaskWords = 64;
struct Mask { uint64_t* words; int first; };
__device__ __forceinline__ uint64_t visible(const AttnJob& j, const Problem& p, const Mask& m, int k0) {
  const int n = p.keys - k0;
  uint64_t bits = first_bits(n);
  if (j.key_mask && n > 0) {
    if (j.bits) {
      const __attribute__((address_space(4))) uint64_t* w = (const __attribute__((address_space(4))) uint64_t*)(j.bits + (int64_t)p.b * j.words + (k0 >> 6));
      bits &= w[0] >> (k0 & 32);
    } else {
      const uint64_t w = m.words[(k0 - m.first) >> 6] >> ((k0 - m.first) & 32);
      bits &= (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)w) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(w >> 32)) << 32;
    }
  }
  return bits;
}
__device__ __forceinline__ Mask take_mask(const AttnJob& j, const Problem& p, char* lds, int beg, int end) {
  const Mask m{reinterpret_cast<uint64_t*>(lds), beg};
  if (j.key_mask && !j.bits && beg < end) {
    const int lane = threadIdx.x & 63;
    for (int i = threadIdx.x >> 6; beg + 64 * i < end; i += NT / 64) {
      const int k = beg + 64 * i + lane;
      const uint64_t on = __ballot(k < end && j.key_mask[(int64_t)p.b * j.s.k_rows + k] != 0);
      if (lane == 0) m.words[i] = on;
    }
    __syncthreads();
  }
  return m;
}
// bits[b][w], bit i: key 64 w + i of the mask is visible.
__global__ __launch_bounds__(NT) void mask_bits_kernel(const uint8_t* __restrict__ mask, int keys, int words, int64_t n, uint64_t* __restrict__ bits) {
  const int64_t w = (int64_t)blockIdx.x * (NT / 64) + (threadIdx.x >> 6);
  if (w >= n) return;
  const int64_t b = w / words;
  const int k = (int)(w - b * words) * 64 + (threadIdx.x & 63);
  const uint64_t on = __ballot(k < keys && mask[b * keys + k] != 0);
  if ((threadIdx.x & 63) == 0) bits[w] = on;
}

// p of a score: at most 1 also where scores lie so far out that the rounding of lse passes 1.  (The bound is the instruction's own:
// clamped to [0, 1].)
__device__ __forceinline__ float weight_of(float s, float c, float lse) {
  return __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(fmaf(s, c, -lse)), 0.f, 1.f);
}

// max / sum over the two lanes of a column
__device__ __forceinline__ float other_half(float v, float* mine) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  *mine = __uint_as_float(r[0]);                            // (in both halves: the lower lane's, the upper lane's)
  return __uint_as_float(r[1]);
}
__device__ __forceinline__ float pair_max(float v) { float a; const float b = other_half(v, &a); return fmaxf(a, b); }
__device__ __forceinline__ float pair_sum(float v) { float a; const float b = other_half(v, &a); return a + b; }

// An accumulator over the head (elements down, held rows across), times `f`, to the lane's row; zeros unless `any`, whatever the
// accumulator holds.  (Cleared ahead of this instead, the loop before it keeps its accumulators elsewhere: twice the time.)
template <typename T, int DP>
__device__ __forceinline__ void store_row(T* row, const f32x16 (&acc)[DP / 32], bool any, float f, int dh, int half) {
  auto value = [&](int db, int i) { return any ? acc[db][i] * f : 0.f; };
  asm volatile("" : "+v"(half));                            // (or the loads' tests of the same elements are kept through the loop for this)
#pragma unroll
  for (int db = 0; db < DP / 32; ++db) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int g = 0; g < 4; g += 2) {
        // the halves exchange four elements each, so that a lane has eight side by side (26 x 1040 queries of 30 heads of 80,
        // 11 keys: 79 -> 69 us)
        uint32_t w[2][2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int u = 0; u < 2; ++u) w[k][u] = f32x2_to_bf16x2(value(db, 4 * (g + k) + 2 * u), value(db, 4 * (g + k) + 2 * u + 1));
        const auto lo = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
        const int e = 32 * db + 8 * (g + half);
        if (e < dh) *reinterpret_cast<uint4*>(row + e) = make_uint4(lo[0], hi[0], lo[1], hi[1]);
      }
    } else {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int e = 32 * db + 8 * g + 4 * half;
        if (e < dh) *reinterpret_cast<float4*>(row + e) = make_float4(value(db, 4 * g), value(db, 4 * g + 1), value(db, 4 * g + 2), value(db, 4 * g + 3));
      }
    }
  }
}

// a -= f b
template <int N>
__device__ __forceinline__ void remove(f32x16 (&a)[N], const f32x16 (&b)[N], float f) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) a[i][r] = fmaf(-f, b[i][r], a[i][r]);
}
// Wavefronts to a SIMD that the kernels' registers are kept down to: two wherever that spills no vector register, else one.  Two
// exceptions, both dq with four wavefronts to a block: bf16 of 128, not exact, spills 26 registers (2 x 4 x 9000 x 4 (2) x 128, backward:
// 41.1 us, with one wavefront 39.9; 20 x 8000 x 8 x 128: 45.1 and 44.7), fp32 of 64 has 58 scalar registers in vector ones (9 x 64 x 211 x 4 x 64:
// 29.7 us, with one 30.5; 4 x 40 x 1000 x 8 x 64: 40.1 and 40.8).
template <typename T, int DP> constexpr int fwd_waves() { return DP * sizeof(T) <= 384 ? 2 : 1; }
template <typename T, int DP, int SW, bool EXACT> constexpr int dq_waves() {
  return sizeof(T) == 4 ? (DP <= 64 ? 2 : 1) : !EXACT || DP <= 64 || (DP <= 96 && SW < 4) ? 2 : 1;
}
template <typename T, int DP> constexpr int dkv_waves() { return DP * sizeof(T) <= 128 ? 2 : 1; }

// Row r of the problem in part w.part's partial results.
__device__ __forceinline__ int64_t part_row(const AttnJob& j, const Problem& p, const Work& w, int r) {
  return ((int64_t)w.part * j.s.batch * j.s.kv_heads + w.id) * p.rows + r;
}
// The sum over the SW wavefronts of `rows` (128 rows of fp32 in LDS, wavefront by wavefront) in order, times factor(row): held
// row r0 + row, below `end`, goes to out(r), or, of a part, to part + r d_head.
template <typename T, int DP, int SW, typename F, typename O>
__device__ __forceinline__ void join_waves(const float* rows, F factor, int r0, int end, int dh, float* part, O out) {
  constexpr int RW = 4 / SW, PITCH = Ring<T, DP, SW>::JOIN_PITCH;
  for (int i = threadIdx.x; i < RW * WR * (DP / 4); i += NT) {
    const int row = i / (DP / 4), e = i % (DP / 4) * 4, r = r0 + row;
    if (r >= end || e >= dh) continue;
    float4 v = *reinterpret_cast<const float4*>(rows + row * PITCH + e);
#pragma unroll
    for (int k = 1; k < SW; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(rows + (k * RW * WR + row) * PITCH + e);
      v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    }
    const float f = factor(row);
    if (part) {
      *reinterpret_cast<float4*>(part + (int64_t)r * dh + e) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
    } else if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint2*>(out(r) + e) = make_uint2(f32x2_to_bf16x2(v.x * f, v.y * f), f32x2_to_bf16x2(v.z * f, v.w * f));
    } else {
      *reinterpret_cast<float4*>(out(r) + e) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
    }
  }
}
// The same for rows of queries.
template <typename T, int DP, int SW, typename F>
__device__ __forceinline__ void join_queries(const AttnJob& j, const Problem& p, const Work& w, const AttnSplit& sp, const float* rows, F factor,
                                             int r0, const void* base, const vf_attn_layout& l) {
  join_waves<T, DP, SW>(rows, factor, r0, p.rows, j.s.d_head, sp.parts > 1 ? sp.out[0] + part_row(j, p, w, 0) * j.s.d_head : nullptr, [&](int r) {
    const RowOf ro = row_of(j, r);
    return at<T>(base, l, p.b, ro.t, p.hk * j.group + ro.g);
  });
}

// ---- forward ------------------------------------------------------------------------------------
template <typename T, int DP, int SW>
__global__ __launch_bounds__(NT, (fwd_waves<T, DP>())) void xattn_fwd_kernel(AttnJob j, AttnSplit sp) {
  using R = Ring<T, DP, SW>;
  constexpr int TR = R::TR, KB = TR / 32 / SW, RW = 4 / SW, ELEMS = R::ELEMS, STAGES = R::STAGES, BYTES = R::BYTES;
  constexpr int WORDS = Source<T, DP, SW, false>::WORDS;
  constexpr uint64_t ALL = TR >= 64 ? ~0ull : (1ull << TR) - 1, MINE = KB == 2 ? ~0ull : 0xffffffffull;
  extern __shared__ __attribute__((aligned(16))) char xattn_lds[];
  T* lds = reinterpret_cast<T*>(xattn_lds);                 // [STAGES][k, v][ELEMS]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const Work w = work_of(sp);
  const Problem p = problem_of(j, w.id);
  const int block = __builtin_amdgcn_readfirstlane(wave) / RW * KB;       // first of this wavefront's blocks of a tile
  const int r0 = w.tile * (RW * WR), r = r0 + wave % RW * WR + (lane & 31);
  const int kbeg = w.first * TR, kend = min(p.keys, kbeg + sp.per * TR);
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
  float m = -INFINITY, l = 0.f, ref = 0.f, base = 0.f;
  bool far = false;

  const Mask mask = take_mask(j, p, xattn_lds + R::LDS, kbeg, kend);
  const uint32_t lds0 = lds_address(lds) + __builtin_amdgcn_readfirstlane(wave) * 1024;
  const char* const zeros = fixed_address(g_zeros);
  Source<T, DP, SW, false> ks, vs;
  ks.init(j, at<const T>(j.k, j.s.k, p.b, 0, p.hk), j.s.k);
  vs.init(j, at<const T>(j.v, j.s.v, p.b, 0, p.hk), j.s.v);
  auto issue = [&](int k0, int buf) {
    uint64_t vis[WORDS], all = ~0ull;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      vis[i] = k0 + 64 * i < kend ? visible(j, p, mask, k0 + 64 * i) : 0;
      all &= vis[i];
    }
    const bool whole = dh == DP && (all & ALL) == ALL;
    issue_pair(j, ks, vs, k0, vis, whole, dh, zeros, lds0 + buf * 2 * BYTES, lds0 + buf * 2 * BYTES + BYTES);
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i)
    if (kbeg + i * TR < kend) issue(kbeg + i * TR, i);
  q.arrive();
  auto step = [&](auto buf, int k0) {
    const T* kt = lds + buf * 2 * ELEMS;
    const T* vt = kt + ELEMS;
    const int ahead = k0 + (STAGES - 1) * TR;               // this tile is there, and nobody reads the one before it:
    meet_for_tile<STAGES, 2 * R::N>(ahead < kend);
    if (ahead < kend) issue(ahead, (buf + STAGES - 1) % STAGES);
    const uint64_t now = visible(j, p, mask, k0 + 32 * block);
    f32x16 s[KB];
    if constexpr (KB == 2) {
      dot_rows<T, DP, true>(s[0], kt, 32 * block, q, s[1], kt, 32 * block + 32, q, lane);
    } else {
      f32x16 none;
      dot_rows<T, DP, false>(s[0], kt, 32 * block, q, none, kt, 0, q, lane);
    }
    if ((now & MINE) != MINE) {
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
    // The reference m of a row's exponentials follows its maximum only when some row's has passed it by kSlack: until then no p
    // exceeds 2^kSlack and nothing is rescaled.  (2 x 16 problems of 4096 x 8192 x 128: 556 -> 540 us against always.)
    const float mt = pair_max(top);
    if (__any((mt - m) * c > kSlack)) {
      const float mn = fmaxf(m, mt);
      const float fade = __builtin_amdgcn_exp2f((m - (mn == -INFINITY ? 0.f : mn)) * c);
      m = mn;
      ref = mn == -INFINITY ? 0.f : mn;                     // no visible key so far: every p is exp2(-inf) = 0
      base = ref * c;
      far = __any(fabsf(base) > kFar);
      l *= fade;
#pragma unroll
      for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= fade;
    }
    // s c - base in one operation keeps the rounding of base: nothing as long as that is far below 1, and the same
    // factor for all of a row; where it is not, the difference is taken first.
    if (far) {
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
    l += sum;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) dot_cols<T, DP>(o, vt, 32 * (block + kb), s[kb], lane);
  };
  if constexpr (SW == 1 && STAGES == 2) {                   // (buffers known where the code is made: no address is computed in the loop)
    for (int k0 = kbeg; k0 < kend; k0 += TR) {
      step(std::integral_constant<int, 0>(), k0);
      if ((k0 += TR) >= kend) break;
      step(std::integral_constant<int, 1>(), k0);
    }
  } else {
    int buf = 0;
    for (int k0 = kbeg; k0 < kend; k0 += TR, buf = (buf + 1) % STAGES) step(buf, k0);
  }
  l = pair_sum(l);
  if (!live) l = 0.f;                                       // (its zeros times an infinite key are NaN)
  if constexpr (SW > 1) {
    // the wavefronts' maxima and sums, then their results weighed by them
    float* rows = reinterpret_cast<float*>(xattn_lds);
    float* stat = rows + 128 * R::JOIN_PITCH;               // [128][maximum, sum], then [128] factors
    const int slot = wave * WR + (lane & 31);
    __syncthreads();                                        // nobody reads a tile any more
    if (half == 0) *reinterpret_cast<float2*>(stat + 2 * slot) = make_float2(m, l);
    __syncthreads();
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int k = 0; k < SW; ++k) {
      const float2 x = *reinterpret_cast<const float2*>(stat + 2 * ((k * RW + wave % RW) * WR + (lane & 31)));
      if (x.y != 0.f) top = fmaxf(top, x.x);
    }
    if (top == -INFINITY) top = 0.f;
#pragma unroll
    for (int k = 0; k < SW; ++k) {
      const float2 x = *reinterpret_cast<const float2*>(stat + 2 * ((k * RW + wave % RW) * WR + (lane & 31)));
      if (x.y != 0.f) total = fmaf(x.y, __builtin_amdgcn_exp2f((x.x - top) * c), total);
    }
    const float mine_w = __builtin_amdgcn_exp2f((m - top) * c);      // may be 0: what is not finite stays so all the same
    const float factor = sp.parts > 1 ? 1.f : total != 0.f ? 1.f / total : 0.f;
    store_row<float, DP>(rows + slot * R::JOIN_PITCH, o, l != 0.f, mine_w, DP, half);
    if (wave < RW && half == 0) {
      stat[256 + slot] = factor;
      if (mine) {
        if (sp.parts > 1) *reinterpret_cast<float2*>(sp.stats + 2 * part_row(j, p, w, r)) = make_float2(top, total);
        else if (j.lse) j.lse[((int64_t)p.b * j.s.q_heads + head) * j.s.q_rows + ro.t] = total != 0.f ? fmaf(top, j.s.scale, logf(total)) : -INFINITY;
      }
    }
    __syncthreads();
    join_queries<T, DP, SW>(j, p, w, sp, rows, [&](int row) { return stat[256 + row]; }, r0, j.o, j.s.o);
    return;
  }
  if (!mine) return;
  if (sp.parts > 1) {                                       // a part: unnormalised, with its maximum and sum
    const int64_t row = part_row(j, p, w, r);
    if (half == 0) *reinterpret_cast<float2*>(sp.stats + 2 * row) = make_float2(m, l);
    store_row<float, DP>(sp.out[0] + row * dh, o, l != 0.f, 1.f, dh, half);
    return;
  }
  const bool any = l != 0.f;                                // (a NaN goes on)
  store_row<T, DP>(at<T>(j.o, j.s.o, p.b, ro.t, head), o, any, 1.f / l, dh, half);
  if (j.lse && half == 0)
    j.lse[((int64_t)p.b * j.s.q_heads + head) * j.s.q_rows + ro.t] = any ? fmaf(m, j.s.scale, logf(l)) : -INFINITY;
}

// ---- backward: dq, and lse / rowsum(dO o) of every row for the kernel behind it ---------------------
// rowsum(dO o) from the rounded o is off by e, and every dz by -p e: their sum, which should be 0, is -e.  The kernel behind is
// given the exact rowsum.  Here dq is off by -scale e sum(p k): nothing beside the rounding of dz when many keys share a
// row and o is small, but 0.0014 of the norm at 77 keys (0.0027 in all, 0.0023 without it).  EXACT takes sum(p k) along and
// removes it; for sources of up to 2048 keys (heads of more than 96 elements, where its registers cost the second wavefront of a
// SIMD: 512), not in parts.
template <typename T, int DP, int SW, bool EXACT>
__global__ __launch_bounds__(NT, (dq_waves<T, DP, SW, EXACT>())) void xattn_dq_kernel(AttnJob j, AttnSplit sp) {
  using R = Ring<T, DP, SW>;
  constexpr int TR = R::TR, KB = TR / 32 / SW, RW = 4 / SW, ELEMS = R::ELEMS, STAGES = R::STAGES, BYTES = R::BYTES;
  constexpr int WORDS = Source<T, DP, SW, false>::WORDS;
  constexpr uint64_t ALL = TR >= 64 ? ~0ull : (1ull << TR) - 1, MINE = KB == 2 ? ~0ull : 0xffffffffull;
  extern __shared__ __attribute__((aligned(16))) char xattn_lds[];
  T* lds = reinterpret_cast<T*>(xattn_lds);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const Work w = work_of(sp);
  const Problem p = problem_of(j, w.id);
  const int block = __builtin_amdgcn_readfirstlane(wave) / RW * KB;       // first of this wavefront's blocks of a tile
  const int r0 = w.tile * (RW * WR), r = r0 + wave % RW * WR + (lane & 31);
  const int kbeg = w.first * TR, kend = min(p.keys, kbeg + sp.per * TR);
  const bool mine = r < p.rows;
  const RowOf ro = row_of(j, mine ? r : 0);
  const int head = p.hk * j.group + ro.g;
  const int dh = j.s.d_head;
  const float c = j.s.scale * kLog2e;
  const float lse_in = mine && ro.t < p.q_len ? j.lse[((int64_t)p.b * j.s.q_heads + head) * j.s.q_rows + ro.t] : -INFINITY;
  const bool live = lse_in != -INFINITY;                    // a row without a visible key has p = 0 everywhere
  const float lse = live ? lse_in * kLog2e : INFINITY;

  f32x16 dq[DP / 32], pk[EXACT ? DP / 32 : 1];
  clear(dq);
  clear(pk);
  float rest = 0.f;                                         // sum of dz

  const Mask mask = take_mask(j, p, xattn_lds + R::LDS, kbeg, kend);
  const uint32_t lds0 = lds_address(lds) + __builtin_amdgcn_readfirstlane(wave) * 1024;
  const char* const zeros = fixed_address(g_zeros);
  Source<T, DP, SW, false> ks, vs;
  ks.init(j, at<const T>(j.k, j.s.k, p.b, 0, p.hk), j.s.k);
  vs.init(j, at<const T>(j.v, j.s.v, p.b, 0, p.hk), j.s.v);
  auto issue = [&](int k0, int buf) {
    uint64_t vis[WORDS], all = ~0ull;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      vis[i] = k0 + 64 * i < kend ? visible(j, p, mask, k0 + 64 * i) : 0;
      all &= vis[i];
    }
    const bool whole = dh == DP && (all & ALL) == ALL;
    issue_pair(j, ks, vs, k0, vis, whole, dh, zeros, lds0 + buf * 2 * BYTES, lds0 + buf * 2 * BYTES + BYTES);
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i)
    if (kbeg + i * TR < kend) issue(kbeg + i * TR, i);
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
  q.arrive();
  g.arrive();
  auto step = [&](auto buf, int k0) {
    const T* kt = lds + buf * 2 * ELEMS;
    const T* vt = kt + ELEMS;
    const int ahead = k0 + (STAGES - 1) * TR;               // this tile is there, and nobody reads the one before it:
    meet_for_tile<STAGES, 2 * R::N>(ahead < kend);
    if (ahead < kend) issue(ahead, (buf + STAGES - 1) % STAGES);
    const uint64_t now = visible(j, p, mask, k0 + 32 * block);
#pragma unroll 1
    for (int kb = 0; kb < KB; ++kb) {
      const uint32_t seen = (uint32_t)(now >> (32 * kb));
      if (seen == 0) continue;                              // (the same for the whole wavefront)
      f32x16 s, dp, pr;
      dot_rows<T, DP, true, 2>(s, kt, 32 * (block + kb), q, dp, vt, 32 * (block + kb), g, lane);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        pr[i] = weight_of(s[i], c, lse);
      }
      if (seen != 0xffffffffu) {
        const uint32_t bits = seen >> (4 * half);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!((bits >> acc_row(i, 0)) & 1)) pr[i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = pr[i] * (dp[i] - delta);
        rest += s[i];
      }
      if constexpr (EXACT) dot_cols<T, DP, true>(dq, kt, 32 * (block + kb), s, lane, &pk, &pr);
      else dot_cols<T, DP>(dq, kt, 32 * (block + kb), s, lane);
    }
  };
  if constexpr (SW == 1 && STAGES == 2) {                   // (buffers known where the code is made: no address is computed in the loop)
    for (int k0 = kbeg; k0 < kend; k0 += TR) {
      step(std::integral_constant<int, 0>(), k0);
      if ((k0 += TR) >= kend) break;
      step(std::integral_constant<int, 1>(), k0);
    }
  } else {
    int buf = 0;
    for (int k0 = kbeg; k0 < kend; k0 += TR, buf = (buf + 1) % STAGES) step(buf, k0);
  }
  rest = pair_sum(rest);
  if (!live) rest = 0.f;                                    // (as in the forward kernel)
  if constexpr (SW > 1) {
    float* rows = reinterpret_cast<float*>(xattn_lds);
    float* stat = rows + 128 * R::JOIN_PITCH;               // [128] rests
    const int slot = wave * WR + (lane & 31);
    __syncthreads();
    if (half == 0) stat[slot] = rest;
    __syncthreads();
    rest = 0.f;
#pragma unroll
    for (int k = 0; k < SW; ++k) rest += stat[(k * RW + wave % RW) * WR + (lane & 31)];
    if constexpr (EXACT) remove(dq, pk, rest);
    store_row<float, DP>(rows + slot * R::JOIN_PITCH, dq, live, 1.f, DP, half);
    __syncthreads();
    if (wave < RW && half == 0 && mine) {
      if (sp.parts > 1) *reinterpret_cast<float2*>(sp.stats + 2 * part_row(j, p, w, r)) = make_float2(rest, delta);
      else j.row_delta[(int64_t)w.id * p.rows + r] = delta + rest;
      if (w.part == 0) j.row_lse[(int64_t)w.id * p.rows + r] = lse;
    }
    const float f = sp.parts > 1 ? 1.f : j.s.scale;
    join_queries<T, DP, SW>(j, p, w, sp, rows, [&](int) { return f; }, r0, j.dq, j.s.dq);
    return;
  }
  if (!mine) return;
  if (sp.parts > 1) {
    const int64_t row = part_row(j, p, w, r);
    if (half == 0) *reinterpret_cast<float2*>(sp.stats + 2 * row) = make_float2(rest, delta);
    store_row<float, DP>(sp.out[0] + row * dh, dq, live, 1.f, dh, half);
    if (w.part == 0 && half == 0) j.row_lse[(int64_t)w.id * p.rows + r] = lse;
    return;
  }
  if constexpr (EXACT) remove(dq, pk, rest);
  if (half == 0) {
    j.row_lse[(int64_t)w.id * p.rows + r] = lse;
    j.row_delta[(int64_t)w.id * p.rows + r] = delta + rest;
  }
  store_row<T, DP>(at<T>(j.dq, j.s.dq, p.b, ro.t, head), dq, live, j.s.scale, dh, half);
}

// Keeps accumulators in the accumulation registers at this point: left to itself the compiler copies three of the eight tiles out and
// back in every step.  (2 x 2048 x 4096 x 32 (8) x 128, dq and dk/dv: 975 -> 950 us.)
template <int N>
__device__ __forceinline__ void stay(f32x16 (&a)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+a"(a[i]));
}

// ---- backward: dk and dv ------------------------------------------------------------------------------
template <typename T, int DP, int SW>
__global__ __launch_bounds__(NT, (dkv_waves<T, DP>())) void xattn_dkv_kernel(AttnJob j, AttnSplit sp) {
  using R = Ring<T, DP, SW>;
  constexpr int TR = R::TR, QB = TR / 32 / SW, RW = 4 / SW, ELEMS = R::ELEMS, STAGES = R::STAGES, BYTES = R::BYTES;
  constexpr int WORDS = Source<T, DP, SW, false>::WORDS, STAT = 64 * WORDS;   // rows of statistics of a stage
  // blocks of 32 rows of a tile: bf16 heads of 64 take them one by one and leave out what lies behind the last row; wider ones keep
  // both in one piece of code for the scheduler (16 problems of 8192 rows x 4096 keys x 128, with dq: 949 us, one by one 1015)
  constexpr bool ONE_BY_ONE = DP * sizeof(T) <= 128;
  constexpr uint64_t ALL = TR >= 64 ? ~0ull : (1ull << TR) - 1;
  extern __shared__ __attribute__((aligned(16))) char xattn_lds[];
  T* lds = reinterpret_cast<T*>(xattn_lds);                 // [STAGES][q, dO][ELEMS], then [STAGES][lse, delta][STAT]
  float* stats = reinterpret_cast<float*>(lds + 2 * STAGES * ELEMS);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const Work w = work_of(sp);
  const Problem p = problem_of(j, w.id);
  const int block = __builtin_amdgcn_readfirstlane(wave) / RW * QB;       // first of this wavefront's blocks of a tile
  const int key0 = w.tile * (RW * WR), key = key0 + wave % RW * WR + (lane & 31);
  const bool mine = key < j.s.k_rows;
  bool seen = key < p.keys;
  if (j.key_mask && seen) seen = j.key_mask[(int64_t)p.b * j.s.k_rows + key] != 0;
  const int dh = j.s.d_head;
  const float c = j.s.scale * kLog2e;

  Held<T, DP> k, v;
  f32x16 dk[DP / 32], dv[DP / 32];
  clear(dk);
  clear(dv);
  bool lost = false;                                        // a row's lse is NaN: so are its p, which weight_of bounds all the same

  const int rows = p.q_len * j.group;                       // padding lies behind them
  const uint32_t lds0 = lds_address(lds) + __builtin_amdgcn_readfirstlane(wave) * 1024, stats0 = lds_address(stats);
  const char *const zeros = fixed_address(g_zeros), *const infinity = fixed_address(&g_infinity);
  const int beg = w.first * TR, stop = min(rows, beg + sp.per * TR);
  const int end = key0 < p.keys ? stop : beg;               // (a tile without a visible key: nothing but zeros to write)
  Source<T, DP, SW, true> qs, gs;
  qs.init(j, at<const T>(j.q, j.s.q, p.b, 0, p.hk * j.group), j.s.q);
  gs.init(j, at<const T>(j.d_o, j.s.d_o, p.b, 0, p.hk * j.group), j.s.d_o);
  auto issue = [&](int r0, int buf) {
    uint64_t want[WORDS], all = ~0ull;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      want[i] = first_bits(stop - r0 - 64 * i);
      all &= want[i];
    }
    const bool whole = dh == DP && (all & ALL) == ALL;
    issue_pair(j, qs, gs, r0, want, whole, dh, zeros, lds0 + buf * 2 * BYTES, lds0 + buf * 2 * BYTES + BYTES);
    // every wavefront loads the statistics of the tile's rows (the same values to the same place: all count alike)
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      const int row = r0 + 64 * i + lane;
      const bool in = row < stop;
      const int64_t at_row = (int64_t)w.id * p.rows + row;
      const uint32_t dst = stats0 + (buf * 2 * STAT + 64 * i) * 4;
      lds_load4(in ? static_cast<const void*>(j.row_lse + at_row) : static_cast<const void*>(infinity), dst);
      lds_load4(in ? static_cast<const void*>(j.row_delta + at_row) : static_cast<const void*>(zeros), dst + STAT * 4);
    }
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i)
    if (beg + i * TR < end) issue(beg + i * TR, i);
  k.load(seen ? at<const T>(j.k, j.s.k, p.b, key, p.hk) : nullptr, dh, half);
  v.load(seen ? at<const T>(j.v, j.s.v, p.b, key, p.hk) : nullptr, dh, half);
  k.arrive();
  v.arrive();
  auto step = [&](auto buf, int r0) {
    const T* qt = lds + buf * 2 * ELEMS;
    const T* gt = qt + ELEMS;
    const float* st = stats + buf * 2 * STAT;
    const int ahead = r0 + (STAGES - 1) * TR;
    meet_for_tile<STAGES, 2 * R::N + 2 * WORDS>(ahead < end);
    if constexpr (dkv_waves<T, DP>() == 1) {
      stay(dk);
      stay(dv);
    }
    if (ahead < end) issue(ahead, (buf + STAGES - 1) % STAGES);
    // p, dz of 32 rows from their products
    auto weights = [&](f32x16& s, f32x16& dp, int row0) {
#pragma unroll
      for (int gq = 0; gq < 4; ++gq) {
        const f32x4 lse = *reinterpret_cast<const f32x4*>(st + row0 + 8 * gq + 4 * half);
        const f32x4 delta = *reinterpret_cast<const f32x4*>(st + STAT + row0 + 8 * gq + 4 * half);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float pr = weight_of(s[4 * gq + i], c, lse[i]);
          s[4 * gq + i] = pr;
          dp[4 * gq + i] = pr * (dp[4 * gq + i] - delta[i]);
        }
      }
    };
    constexpr int UNROLL = ONE_BY_ONE ? 1 : 2;
#pragma unroll UNROLL
    for (int qb = 0; qb < QB; ++qb) {
      if (ONE_BY_ONE && r0 + 32 * (block + qb) >= stop) break;
      f32x16 s, dp;
      dot_rows<T, DP, true, 6>(s, qt, 32 * (block + qb), k, dp, gt, 32 * (block + qb), v, lane);
      weights(s, dp, 32 * (block + qb));
      dot_cols<T, DP>(dv, gt, 32 * (block + qb), s, lane);
      dot_cols<T, DP>(dk, qt, 32 * (block + qb), dp, lane);
    }
#pragma unroll
    for (int i = 0; i < WORDS; ++i) lost = lost || st[64 * i + lane] != st[64 * i + lane];
  };
  int buf = 0;
  for (int r0 = beg; r0 < end; r0 += TR, buf = (buf + 1) % STAGES) step(buf, r0);
  // an invisible key's columns hold what its zeros gave: nothing of it is stored
  const bool any_lost = __any(lost);                        // (of the whole wavefront, whatever its own key)
  const float dv_by = seen && any_lost ? NAN : 1.f;
  if (!seen) { clear(dk); clear(dv); }
  if constexpr (SW > 1) {
    float* rows = reinterpret_cast<float*>(xattn_lds);
    const int64_t part = (((int64_t)w.part * j.s.batch * j.s.kv_heads + w.id) * j.s.k_rows) * dh;
    const float f = sp.parts > 1 ? 1.f : j.s.scale;
    float* slot = rows + (wave * WR + (lane & 31)) * R::JOIN_PITCH;
    __syncthreads();                                        // nobody reads a tile any more
    store_row<float, DP>(slot, dk, true, 1.f, DP, half);
    __syncthreads();
    join_waves<T, DP, SW>(rows, [&](int) { return f; }, key0, j.s.k_rows, dh, sp.parts > 1 ? sp.out[0] + part : nullptr,
                          [&](int r) { return at<T>(j.dk, j.s.dk, p.b, r, p.hk); });
    __syncthreads();
    store_row<float, DP>(slot, dv, true, dv_by, DP, half);
    __syncthreads();
    join_waves<T, DP, SW>(rows, [&](int) { return 1.f; }, key0, j.s.k_rows, dh, sp.parts > 1 ? sp.out[1] + part : nullptr,
                          [&](int r) { return at<T>(j.dv, j.s.dv, p.b, r, p.hk); });
    return;
  }
  if (!mine) return;
  if (sp.parts > 1) {
    const int64_t row = ((int64_t)w.part * j.s.batch * j.s.kv_heads + w.id) * j.s.k_rows + key;
    store_row<float, DP>(sp.out[0] + row * dh, dk, true, 1.f, dh, half);
    store_row<float, DP>(sp.out[1] + row * dh, dv, true, dv_by, dh, half);
    return;
  }
  store_row<T, DP>(at<T>(j.dk, j.s.dk, p.b, key, p.hk), dk, true, j.s.scale, dh, half);
  store_row<T, DP>(at<T>(j.dv, j.s.dv, p.b, key, p.hk), dv, true, dv_by, dh, half);
}

// ---- joining the parts -----------------------------------------------------------------------------------
// A part's rows are fp32 [part][problem][row][d_head].  32 lanes take a row, four elements each; the parts are added in their
// order.  KIND 0: forward, parts weighed by their maxima and sums; 1: dq, with the rows' delta; 2: dk and 3: dv.
template <typename T, int KIND>
__device__ __forceinline__ void join_rows(const AttnJob& j, const AttnSplit& sp, int64_t i, int e) {
  const int dh = j.s.d_head;
  const int held = KIND < 2 ? j.group * j.s.q_rows : j.s.k_rows;
  const int id = (int)((uint32_t)i / (uint32_t)held), r = (int)((uint32_t)i - (uint32_t)id * (uint32_t)held);
  const int b = id / j.s.kv_heads, hk = id - b * j.s.kv_heads;
  const int64_t step = (int64_t)j.s.batch * j.s.kv_heads * held;
  const float* part = sp.out[KIND == 3 ? 1 : 0] + i * dh + e;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  float top = -INFINITY, total = 0.f, delta = 0.f, factor = 1.f;
  if constexpr (KIND == 0) {
#pragma unroll 4
    for (int k = 0; k < sp.parts; ++k) {
      const float2 ml = *reinterpret_cast<const float2*>(sp.stats + 2 * (i + k * step));
      if (ml.y != 0.f) top = fmaxf(top, ml.x);
    }
    if (top == -INFINITY) top = 0.f;
  }
  const float c = j.s.scale * kLog2e;
#pragma unroll 4
  for (int k = 0; k < sp.parts; ++k) {                      // (four parts' loads under way together)
    float w = 1.f;
    if constexpr (KIND < 2) {
      const float2 st = *reinterpret_cast<const float2*>(sp.stats + 2 * (i + k * step));
      if constexpr (KIND == 0) {
        w = st.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((st.x - top) * c);
        total = fmaf(st.y, w, total);
      } else {
        if (k == 0) delta = st.y;
        total += st.x;
      }
    }
    const float4 v = e < dh ? *reinterpret_cast<const float4*>(part + k * step * dh) : make_float4(0.f, 0.f, 0.f, 0.f);
    sum.x = fmaf(v.x, w, sum.x); sum.y = fmaf(v.y, w, sum.y); sum.z = fmaf(v.z, w, sum.z); sum.w = fmaf(v.w, w, sum.w);
  }
  T* out;
  if constexpr (KIND < 2) {
    const RowOf ro = row_of(j, r);
    const int head = hk * j.group + ro.g;
    if constexpr (KIND == 0) {
      out = at<T>(j.o, j.s.o, b, ro.t, head);
      factor = total != 0.f ? 1.f / total : 0.f;
      if (j.lse && e == 0)
        j.lse[((int64_t)b * j.s.q_heads + head) * j.s.q_rows + ro.t] = total != 0.f ? fmaf(top, j.s.scale, logf(total)) : -INFINITY;
    } else {
      out = at<T>(j.dq, j.s.dq, b, ro.t, head);
      factor = j.s.scale;
      if (e == 0) j.row_delta[i] = delta + total;
    }
  } else {
    out = KIND == 2 ? at<T>(j.dk, j.s.dk, b, r, hk) : at<T>(j.dv, j.s.dv, b, r, hk);
    factor = KIND == 2 ? j.s.scale : 1.f;
  }
  if (e >= dh) return;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint2*>(out + e) = make_uint2(f32x2_to_bf16x2(sum.x * factor, sum.y * factor), f32x2_to_bf16x2(sum.z * factor, sum.w * factor));
  } else {
    *reinterpret_cast<float4*>(out + e) = make_float4(sum.x * factor, sum.y * factor, sum.z * factor, sum.w * factor);
  }
}
template <typename T, int KIND>
__global__ __launch_bounds__(NT) void xattn_join_kernel(AttnJob j, AttnSplit sp, int64_t rows) {
  const int64_t i = (int64_t)blockIdx.x * (NT / 32) + (threadIdx.x >> 5);
  if (i >= rows) return;
  const int e = 4 * (threadIdx.x & 31);
  if constexpr (KIND == 2) {
    if (blockIdx.y == 0) join_rows<T, 2>(j, sp, i, e);
    else join_rows<T, 3>(j, sp, i, e);
  } else {
    join_rows<T, KIND>(j, sp, i, e);
  }
}

// How the streamed side is split: among the wavefronts of a workgroup (sw: 128 / sw held rows to a workgroup, every wavefront a
// quarter or half of a tile's blocks), and into parts, whose results a kernel behind joins.  Both make more and shorter workgroups
// where few rows are held.  The choice is the one with the least estimated time, in us:
//   a workgroup alone takes kStart + tiles * chain (its steps wait for each other), and as many of them run side by side as LDS and
//   the forward kernel's registers allow (`beside` to a compute unit);  workgroups of one compute unit share its matrix units: tiles *
//   busy each.
//   Joining the wavefronts' results takes 1 us for 64 elements, parts cost kJoin and a pass over their fp32 results.
// Measured per tile (forward): bf16 heads of 64: 1.1 chain, 0.55 busy (one block of 32 rows to a wavefront instead of two: 0.75, 0.3),
// of 128: 1.8 and 1.15; fp32, bound by its matrix instructions: 2.4 and 2.1 at 64.  (192 workgroups of 7 tiles in three parts: 12.6 us
// became 11.8 + 8.4; 256 workgroups of 24 tiles with sw = 4 instead of 1: 30 us became 19; 256 of 4 tiles, 128 wide: 13 us with
// sw = 1, 15 with 2, 31 with 4.)
// Of the other kernels, dk/dv of more than 128 bytes to a head and the fp32 dq of 96 have registers for one workgroup to a unit, and
// so has the exact dq above 96 elements, which alone is counted so (`alone`), also where its keys then go in parts and the other dq
// runs.  Counting one for each that has room for one changes the choice at 32 of 600 sizes (1 to 4096 queries, 1 to 8192 keys): backward
// passes of fp32 up to 11 % slower (18 x 106 x 2202 x 6 (3) x 80: 407 -> 451 us), 6 % faster at one; of bf16 up to 14 % faster where
// it takes fewer wavefronts to a block (39 x 1468 x 1319 x 2 x 80: 388 -> 332) and up to 15 % slower where more (56 x 711 x 59 x 5 x 96: 86 -> 99).
constexpr int kUnits = 256, kMaxParts = 64;
constexpr float kStart = 5.f, kJoin = 8.f;
AttnSplit split_of(const vf_attn_shape& s, int held, int streamed, float work, bool alone) {
  const bool b = s.dtype == VF_BF16;
  const int dp = !b && s.d_head <= 32 ? 32 : s.d_head <= 64 ? 64 : s.d_head <= 96 ? 96 : 128, problems = s.batch * s.kv_heads;
  const int most = b || dp <= 64 ? 4 : 2;                   // (wider fp32 tiles for four wavefronts would not fit the LDS)
  AttnSplit best{};
  float least = 0.f;
  for (int sw = 1; sw <= most; sw *= 2) {
    const int block = 128 / sw, rows = std::max(b ? Elem<bf16_t>::TR : Elem<float>::TR, 32 * sw);
    const bool two = rows / 32 / sw == 2;                   // blocks of a wavefront
    const float wide = work * (float)dp / 64.f, chain = b ? (two ? 0.75f : 0.5f) + (two ? 0.35f : 0.25f) * wide : 0.3f + 2.1f * wide;
    const float busy = b ? (two ? 0.55f : 0.3f) * wide : 2.1f * wide;
    const int tile_bytes = rows * dp * (b ? 2 : 4), lds = (tile_bytes <= 8192 ? 6 : 4) * tile_bytes;
    const int beside = alone ? 1 : std::max(1, std::min(b ? (dp <= 64 ? 3 : 2) : (dp <= 96 ? 2 : 1), 160 * 1024 / lds));
    const float start = kStart + (sw > 1 ? (float)dp / 64.f : 0.f);
    if (sw > 1 && (held + block - 1) / block > 65535) break;    // (a dimension of the grid)
    const int tiles = std::max(1, (held + block - 1) / block), all = std::max(1, (streamed + rows - 1) / rows);
    const int64_t groups = std::max<int64_t>(1, (int64_t)problems * tiles);
    for (int m = 0; m <= 4; ++m) {                          // one part, or as many as give every compute unit m workgroups
      const int parts = m == 0 ? 1 : (int)std::min<int64_t>({(int64_t)kUnits * m / groups, (int64_t)all, (int64_t)kMaxParts});
      if (parts < 1 || (m > 0 && parts == 1)) continue;
      const int per = (all + parts - 1) / parts, n = (all + per - 1) / per;
      const int64_t wgs = groups * n, rounds = (wgs + kUnits * beside - 1) / (kUnits * beside), load = (wgs + kUnits - 1) / kUnits;
      float t = std::max((float)rounds * (start + (float)per * chain), start + (float)load * (float)per * busy);
      if (n > 1) t += kJoin + (float)n * (float)problems * (float)held * (float)s.d_head * 2e-6f;
      if (best.sw == 0 || t < least) {
        least = t;
        best.sw = sw; best.tiles = (held + block - 1) / block; best.parts = n; best.per = per;
      }
    }
  }
  return best;
}
// Sources for which dq takes sum(p k) along (see its kernel): above 96 elements that leaves one workgroup to a compute unit.
bool exact_dq(const vf_attn_shape& s) { return s.dtype == VF_BF16 && s.k_rows <= (s.d_head <= 96 ? 2048 : 512); }
// The splits of the forward and dq kernels, and of the dk/dv kernel.
AttnSplit split_rows(const vf_attn_shape& s, bool backward) {
  return split_of(s, s.q_heads / s.kv_heads * s.q_rows, s.k_rows, 1.f, backward && s.d_head > 96 && exact_dq(s));
}
AttnSplit split_keys(const vf_attn_shape& s) { return split_of(s, s.k_rows, s.q_heads / s.kv_heads * s.q_rows, 2.f, false); }
int64_t round4(int64_t floats) { return (floats + 3) & ~int64_t(3); }
// Floats of the parts of a pass over the rows (results and two statistics a row), and over the keys (dk and dv).
int64_t part_rows_floats(const vf_attn_shape& s, const AttnSplit& sp) {
  return sp.parts > 1 ? sp.parts * (int64_t)s.batch * s.q_heads * s.q_rows * (s.d_head + 2) : 0;
}
int64_t part_keys_floats(const vf_attn_shape& s, const AttnSplit& sp) {
  return sp.parts > 1 ? sp.parts * (int64_t)s.batch * s.kv_heads * s.k_rows * 2 * s.d_head : 0;
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

template <typename T, int KIND>
int launch_join(const AttnJob& j, const AttnSplit& sp, int64_t rows, hipStream_t st) {
  xattn_join_kernel<T, KIND><<<dim3((unsigned)((rows + NT / 32 - 1) / (NT / 32)), KIND == 2 ? 2 : 1), NT, 0, st>>>(j, sp, rows);
  VF_LAUNCH_CHECK();
  return VF_OK;
}

template <typename T, int DP, int SW>
int launch_fwd(const AttnJob& j, const AttnSplit& sp, hipStream_t st) {
  constexpr int lds = std::max(Ring<T, DP, SW>::LDS + kMaskWords * 8, Ring<T, DP, SW>::JOIN);
  static std::atomic<uint64_t> ready{0};
  VF_TRY(allow_lds(reinterpret_cast<const void*>(&xattn_fwd_kernel<T, DP, SW>), lds, ready));
  xattn_fwd_kernel<T, DP, SW><<<dim3(j.s.batch * j.s.kv_heads, sp.tiles, sp.parts), NT, lds, st>>>(j, sp);
  VF_LAUNCH_CHECK();
  return VF_OK;
}
template <typename T, int DP, int SW, bool EXACT>
int launch_dq_of(const AttnJob& j, const AttnSplit& sp, hipStream_t st) {
  constexpr int lds = std::max(Ring<T, DP, SW>::LDS + kMaskWords * 8, Ring<T, DP, SW>::JOIN);
  static std::atomic<uint64_t> ready{0};
  VF_TRY(allow_lds(reinterpret_cast<const void*>(&xattn_dq_kernel<T, DP, SW, EXACT>), lds, ready));
  xattn_dq_kernel<T, DP, SW, EXACT><<<dim3(j.s.batch * j.s.kv_heads, sp.tiles, sp.parts), NT, lds, st>>>(j, sp);
  VF_LAUNCH_CHECK();
  return VF_OK;
}
template <typename T, int DP, int SW>
int launch_dq(const AttnJob& j, const AttnSplit& sp, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (exact_dq(j.s) && sp.parts == 1) return launch_dq_of<T, DP, SW, true>(j, sp, st);
  }
  return launch_dq_of<T, DP, SW, false>(j, sp, st);
}
template <typename T, int DP, int SW>
int launch_dkv(const AttnJob& j, const AttnSplit& sp, hipStream_t st) {
  using R = Ring<T, DP, SW>;
  constexpr int lds = std::max(R::LDS + R::STAGES * 8 * std::max(64, R::TR), R::JOIN);
  static std::atomic<uint64_t> ready{0};
  VF_TRY(allow_lds(reinterpret_cast<const void*>(&xattn_dkv_kernel<T, DP, SW>), lds, ready));
  xattn_dkv_kernel<T, DP, SW><<<dim3(j.s.batch * j.s.kv_heads, sp.tiles, sp.parts), NT, lds, st>>>(j, sp);
  VF_LAUNCH_CHECK();
  return VF_OK;
}

// The passes over the rows (forward, dq) and over the keys, with their joins.
template <typename T, int DP>
int pass_rows(const AttnJob& j, float* ws, bool backward, hipStream_t st) {
  const int64_t rows = (int64_t)j.s.batch * j.s.q_heads * j.s.q_rows;
  AttnSplit sp = split_rows(j.s, backward);
  sp.out[0] = ws;
  sp.stats = ws + sp.parts * rows * j.s.d_head;
  if constexpr (sizeof(T) == 2 || DP <= 64) {
    if (sp.sw == 4) VF_TRY((backward ? launch_dq<T, DP, 4>(j, sp, st) : launch_fwd<T, DP, 4>(j, sp, st)));
  }
  if (sp.sw == 2) VF_TRY((backward ? launch_dq<T, DP, 2>(j, sp, st) : launch_fwd<T, DP, 2>(j, sp, st)));
  if (sp.sw == 1) VF_TRY((backward ? launch_dq<T, DP, 1>(j, sp, st) : launch_fwd<T, DP, 1>(j, sp, st)));
  if (sp.parts == 1) return VF_OK;
  return backward ? launch_join<T, 1>(j, sp, rows, st) : launch_join<T, 0>(j, sp, rows, st);
}
template <typename T, int DP>
int pass_keys(const AttnJob& j, float* ws, hipStream_t st) {
  const int64_t rows = (int64_t)j.s.batch * j.s.kv_heads * j.s.k_rows;
  AttnSplit sp = split_keys(j.s);
  sp.out[0] = ws;
  sp.out[1] = ws + sp.parts * rows * j.s.d_head;
  if constexpr (sizeof(T) == 2 || DP <= 64) {
    if (sp.sw == 4) VF_TRY((launch_dkv<T, DP, 4>(j, sp, st)));
  }
  if (sp.sw == 2) VF_TRY((launch_dkv<T, DP, 2>(j, sp, st)));
  if (sp.sw == 1) VF_TRY((launch_dkv<T, DP, 1>(j, sp, st)));
  return sp.parts > 1 ? launch_join<T, 2>(j, sp, rows, st) : VF_OK;
}
template <typename T, int DP>
int launch_bwd(const AttnJob& j, float* ws, hipStream_t st) {
  if (j.s.q_rows) VF_TRY((pass_rows<T, DP>(j, ws, true, st)));
  if (j.s.k_rows) VF_TRY((pass_keys<T, DP>(j, ws, st)));     // (its parts take the place of the rows' ones)
  return VF_OK;
}

}  // namespace

// Heads are held and streamed in widths of 64, 96 and 128 elements, filled up with zeros; fp32, which its matrix instructions bound,
// also in one of 32 (60 x 495 x 944 x 6 (3) x 32: forward 417 -> 325 us, backward 1506 -> 777).
template <typename T, typename F>
static int by_width(int d_head, F f) {
  if constexpr (sizeof(T) == 4) {
    if (d_head <= 32) return f(std::integral_constant<int, 32>());
  }
  if (d_head <= 64) return f(std::integral_constant<int, 64>());
  return d_head <= 96 ? f(std::integral_constant<int, 96>()) : f(std::integral_constant<int, 128>());
}

// The bits of a mask that no workgroup may have to make alone; backward: two floats per row (lse and rowsum(dO o)); then the parts of
// one pass at a time.
static int64_t mask_words(const vf_attn_shape& s) { return ((int64_t)s.k_rows + 63) / 64; }
static int64_t mask_floats(const vf_attn_shape& s, bool masked) {
  return masked && s.k_rows > kMaskWords * 64 ? round4(2 * s.batch * mask_words(s)) : 0;
}
int64_t attn_workspace_bytes(const vf_attn_shape& s, bool backward, bool masked) {
  if (!s.batch || (!backward && !s.q_rows)) return 0;
  const int64_t parts = part_rows_floats(s, split_rows(s, backward));
  if (!backward) return (mask_floats(s, masked) + parts) * (int64_t)sizeof(float);
  const int64_t stats = 2 * round4((int64_t)s.batch * s.q_heads * s.q_rows);
  return (mask_floats(s, masked) + stats + std::max(parts, part_keys_floats(s, split_keys(s)))) * (int64_t)sizeof(float);
}

static int make_bits(AttnJob& j, bool backward, float* ws, hipStream_t st) {
  j.words = (int)mask_words(j.s);
  const int64_t n = (int64_t)j.s.batch * j.words;
  const AttnSplit sp = split_rows(j.s, backward);
  const int tile = std::max(j.s.dtype == VF_BF16 ? Elem<bf16_t>::TR : Elem<float>::TR, 32 * sp.sw);
  if (!j.key_mask || !n || !j.s.q_rows || (int64_t)sp.per * tile <= kMaskWords * 64) return VF_OK;
  j.bits = reinterpret_cast<uint64_t*>(ws);
  mask_bits_kernel<<<(unsigned)((n + NT / 64 - 1) / (NT / 64)), NT, 0, st>>>(j.key_mask, j.s.k_rows, j.words, n, reinterpret_cast<uint64_t*>(ws));
  VF_LAUNCH_CHECK();
  return VF_OK;
}

int launch_attn(AttnJob j, void* workspace, hipStream_t st) {
  if (!j.s.batch || !j.s.q_rows) return VF_OK;
  float* ws = static_cast<float*>(workspace);
  VF_TRY(make_bits(j, false, ws, st));
  ws += mask_floats(j.s, j.key_mask);
  if (j.s.dtype == VF_BF16) return by_width<bf16_t>(j.s.d_head, [&](auto dp) { return pass_rows<bf16_t, decltype(dp)::value>(j, ws, false, st); });
  return by_width<float>(j.s.d_head, [&](auto dp) { return pass_rows<float, decltype(dp)::value>(j, ws, false, st); });
}

int launch_attn_bwd(AttnJob j, void* workspace, hipStream_t st) {
  if (!j.s.batch || (!j.s.q_rows && !j.s.k_rows)) return VF_OK;
  float* ws = static_cast<float*>(workspace);
  VF_TRY(make_bits(j, true, ws, st));
  const int64_t rows = round4((int64_t)j.s.batch * j.s.q_heads * j.s.q_rows);
  j.row_lse = ws + mask_floats(j.s, j.key_mask);
  j.row_delta = j.row_lse + rows;
  ws = j.row_delta + rows;
  if (j.s.dtype == VF_BF16) return by_width<bf16_t>(j.s.d_head, [&](auto dp) { return launch_bwd<bf16_t, decltype(dp)::value>(j, ws, st); });
  return by_width<float>(j.s.d_head, [&](auto dp) { return launch_bwd<float, decltype(dp)::value>(j, ws, st); });
}

}  // namespace vf
