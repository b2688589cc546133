// Device helpers shared by the backward and the position-bias kernels: MFMA operand types, a
// swizzled 64 x 128 bf16 tile in LDS that can be read by rows and transposed, and its loader.
//
// Register layout of v_mfma_f32_32x32x16_bf16 (lane l, r = l % 32, g = l / 32): A holds row r
// and B column r with k = 8 g + (0..7); D holds column r and, in register v, row
// 8 (v / 4) + 4 g + v % 4.  A product X^T = A B^T whose columns are "own" rows (one per lane
// pair l, l ^ 32) is therefore, rounded to bf16, the B operand of the next product over those
// register rows: registers 8 s .. 8 s + 7 are k-step s.
//
// Tile swizzle: 16-byte chunk c of row i sits in slot c ^ f(i), f(i) = 4 (i % 4) + (i / 4) % 4.
// f takes 16 values over 16 consecutive rows (row operands: 16 lanes read one chunk of 16 rows)
// and its upper two bits differ over 4 consecutive rows (transposed reads: 32 lanes read four
// chunks of 4 rows), so both kinds of read touch every bank once.
#ifndef DSATTN_ATTN_TILES_H
#define DSATTN_ATTN_TILES_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dsattn {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kD = 128;                  // head dimension
constexpr int kRowBytes = kD * 2;
constexpr int kTile = 64;                // rows of an LDS tile
constexpr int kTileElems = kTile * kD;   // 16 KiB
constexpr int kBlockBytes = 32 * kRowBytes;
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ void sched_fence() { __builtin_amdgcn_sched_barrier(0); }
__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// Sum of a value over the two lanes (l, l ^ 32) of an own row.
__device__ __forceinline__ float half_sum(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  const auto sw = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return __builtin_bit_cast(float, (uint32_t)sw[0]) + __builtin_bit_cast(float, (uint32_t)sw[1]);
}

// This lane's number, taken anew: what rare paths derive from it then holds no register of a loop
// around them, which the compiler otherwise computes it ahead of.
__device__ __forceinline__ int lane_now() {
  int x;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
  return x;
}

__device__ __forceinline__ int tile_swz(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }

// LDS byte address of p.
__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)p; }

// Operand reads take the lane's own part of the LDS byte address (row_lane, col_lane; it lies
// below kBlockBytes), the byte offset `block` of a 32-row block, and constants.  What changes from
// operand to operand is an XOR with a constant: one instruction.  Where registers are scarce,
// `block` is the same for the whole wave and part of a scalar XORed value, which leaves no vector
// register in use between the reads; scalar() keeps the compiler from splitting that XOR and
// holding the parts in some.  Otherwise (InLane) the lane's part has it already, kept opaque by
// here(), and the XOR is with a literal, which saves the scalar instructions.
__device__ __forceinline__ uint32_t scalar(uint32_t x) {
  x = __builtin_amdgcn_readfirstlane(x);
  asm volatile("" : "+s"(x));
  return x;
}
template <typename T>
__device__ __forceinline__ void here(T& x) { asm volatile("" : "+v"(x)); }
struct InLane {};
__device__ __forceinline__ uint32_t flip(uint32_t at, uint32_t block, uint32_t x) {
  return at ^ scalar(block | x);
}
__device__ __forceinline__ uint32_t flip(uint32_t at, InLane, uint32_t x) { return at ^ x; }
__device__ __forceinline__ uint32_t row_lane(int r, int g) {
  return (uint32_t)(r * kRowBytes + ((tile_swz(r) ^ g) << 4));
}
__device__ __forceinline__ uint32_t col_lane(int lane) {
  const int grp = lane >> 4, lg = lane & 15, g = grp >> 1, i = lg >> 2;
  return (uint32_t)((4 * g + i) * kRowBytes + (i << 6) +
                    (((2 * (grp & 1) + ((lg & 3) >> 1)) ^ g) << 4) + 8 * (lg & 1));
}

// Row operand, of the tiles at LDS address `tiles`: rows r of the block, k-step s (columns 16 s + 8 g + 0..7).
template <typename BLOCK>
__device__ __forceinline__ bf16x8 row_operand(uint32_t at, BLOCK block, uint32_t tiles, int s) {
  typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
  const uint32_t x = flip(at, block, (uint32_t)(s << 5)) + tiles;
  return __builtin_bit_cast(bf16x8, *(lds_u32x4*)(uintptr_t)x);
}

// Transposed operand: columns 32 db + r as rows; k-step s (0..1) of the 32-row block, the rows
// that registers 8 s .. 8 s + 7 of a D block hold.
template <typename BLOCK>
__device__ __forceinline__ bf16x8 col_operand(uint32_t at, BLOCK block, uint32_t tiles, int s, int db) {
  typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
  bf16x8 out;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const uint32_t x = flip(at, block, (uint32_t)((db << 6) | (c << 5))) + tiles +
                       8 * (2 * s + c) * kRowBytes;
    const bf16x4 y = __builtin_bit_cast(
        bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(uintptr_t)x));
#pragma unroll
    for (int i = 0; i < 4; ++i) out[4 * c + i] = y[i];
  }
  return out;
}

__device__ __forceinline__ f32x16 mfma(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Buffer resource of `rows` rows of one head: rows past the end read as zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const uint16_t* base, int rows) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, rows * kRowBytes, 0x00020000);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t word_buffer(const void* base, int words) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, words * 4, 0x00020000);
}

// Byte offset, inside a tile, of what lane `lane` of wave w fetches first: wave w copies the
// 1 KiB blocks (4 rows) u * 4 + w, lane l the slot l % 16 of row l / 16.  f depends on the row
// modulo 16 only, so one offset serves all four blocks.
__device__ __forceinline__ uint32_t tile_lane_offset(int w, int lane) {
  const int row = 4 * w + (lane >> 4);
  return (uint32_t)(row * kRowBytes + ((lane & 15) ^ tile_swz(row)) * 16);
}

// Copy rows row0 .. row0 + 63 into an LDS tile, without registers (see the swizzle above).
// Inline assembly, since the compiler cannot tell which tile such a load writes and would wait
// for all of them before any LDS read; the caller waits with tiles_ready.  M0 (the LDS base) is
// saved and restored, with the wait state that an M0 write needs before the load.
__device__ __forceinline__ void load_tile(uint16_t* tile, __amdgpu_buffer_rsrc_t rs, uint32_t off,
                                          int row0, int w) {
  const uint32_t o0 = off + (uint32_t)row0 * kRowBytes;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(tile + w * 512));
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %[sv], m0\n\t"
      "s_mov_b32 m0, %[l0]\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %[o0], %[rs], 0 offen lds\n\t"
      "s_add_u32 m0, %[l0], 0x1000\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %[o1], %[rs], 0 offen lds\n\t"
      "s_add_u32 m0, %[l0], 0x2000\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %[o2], %[rs], 0 offen lds\n\t"
      "s_add_u32 m0, %[l0], 0x3000\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %[o3], %[rs], 0 offen lds\n\t"
      "s_mov_b32 m0, %[sv]"
      : [sv] "=&s"(saved)
      : [l0] "s"(lds0), [o0] "v"(o0), [o1] "v"(o0 + 4096u), [o2] "v"(o0 + 8192u),
        [o3] "v"(o0 + 12288u), [rs] "s"(rs)
      : "memory", "scc");
}

// Copy 64 words (word0 .. word0 + 63, those outside the buffer as zeros) into LDS.
__device__ __forceinline__ void load_words(const void* dst, __amdgpu_buffer_rsrc_t rs, int word0,
                                           int lane) {
  const uint32_t o0 = (uint32_t)(word0 + lane) * 4u;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)dst);
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %[sv], m0\n\t"
      "s_mov_b32 m0, %[l0]\n\t"
      "s_nop 0\n\t"
      "buffer_load_dword %[o0], %[rs], 0 offen lds\n\t"
      "s_mov_b32 m0, %[sv]"
      : [sv] "=&s"(saved)
      : [l0] "s"(lds0), [o0] "v"(o0), [rs] "s"(rs)
      : "memory", "scc");
}

// This wave's loads have arrived and every wave is here: the loaded tiles can be read, and the
// tiles read before can be overwritten.
__device__ __forceinline__ void tiles_ready() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Distances key - query of a workgroup's 128 rows and a streamed tile: 128 + 64 - 1 of them, in
// windows of kWindow words that begin with the tile's smallest.
constexpr int kWindow = 192;

// First and last streamed tile with an open run of distances (first > last: none).  The window of
// tile t begins at distance index e0 + DIR * kTile * t; `ends` is LDS for the first and the last open
// run that any of them reaches into.
struct TileRange {
  int first, last;
};
template <int DIR>
__device__ __forceinline__ TileRange open_tiles(int (&ends)[2], const int32_t* runs, int n_runs,
                                                int n_tiles, int e0) {
  static_assert(kTile == 64, "the shifts below");
  if (threadIdx.x == 0) {
    ends[0] = n_runs;
    ends[1] = -1;
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, e1 = e0 + DIR * kTile * (n_tiles - 1);
  const int j0 = max(0, min(e0, e1) >> 5), j1 = min(n_runs - 1, (max(e0, e1) + kWindow - 2) >> 5);
  int first = n_runs, last = -1;
  for (int j = j0 + (int)(threadIdx.x & ~63u); j <= j1; j += kThreads) {
    const bool open = j + lane <= j1 && runs[min(j + lane, j1)] != -1;   // kRunClosed
    const uint64_t have = __ballot(open);
    if (have == 0) continue;
    first = min(first, j + __ffsll((unsigned long long)have) - 1);
    last = max(last, j + 63 - __clzll((long long)have));
  }
  if (lane == 0 && last >= 0) {
    atomicMin(&ends[0], first);
    atomicMax(&ends[1], last);
  }
  __syncthreads();
  first = __builtin_amdgcn_readfirstlane(ends[0]);
  last = __builtin_amdgcn_readfirstlane(ends[1]);
  if (last < 0) return TileRange{n_tiles, -1};
  // tile t reaches into run j where 32 j - (kWindow - 2) <= e0 + DIR * kTile * t <= 32 j + 31
  const int t0 = DIR > 0 ? 32 * first - (kWindow - 2) - e0 : e0 - 32 * last - 31;
  const int t1 = DIR > 0 ? 32 * last + 31 - e0 : e0 - 32 * first + (kWindow - 2);
  return TileRange{max(0, (t0 + 63) >> 6), min(n_tiles - 1, t1 >> 6)};
}

// Own-row fragments (B operands, all eight k-steps) of one row of a head; zeros where !valid.
__device__ __forceinline__ void load_row(bf16x8 (&f)[8], const uint16_t* base, int row, bool valid,
                                         int g) {
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const u32x4 x = valid ? *reinterpret_cast<const u32x4*>(base + (size_t)row * kD + 16 * s + 8 * g)
                          : u32x4{0, 0, 0, 0};
    f[s] = __builtin_bit_cast(bf16x8, x);
  }
}

// Store a^T (four D blocks, columns = own rows) times m as one row of bf16.
__device__ __forceinline__ void store_row(uint16_t* base, int row, const f32x16 (&a)[4], float m,
                                          int g) {
  uint16_t* out = base + (size_t)row * kD;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x4 h;
#pragma unroll
      for (int t = 0; t < 4; ++t) h[t] = (__bf16)(a[db][4 * i + t] * m);
      *reinterpret_cast<bf16x4*>(out + 32 * db + 8 * i + 4 * g) = h;
    }
}

// Partial sums of a wave's 32 rows lie as the lanes hold them: 16 times 1 KiB, one store each.  (By
// rows, the same stores of 16 bytes in 32 rows cost one head of 2048 rows 2 of 52 us.)  Of fewer
// rows than 32 in all there are `rows` times 16 bytes twice as often, so that single ones lie
// together.
__device__ __forceinline__ void store_part(float* slot, const f32x16 (&a)[4], int rows, int w, int lane) {
  const int r = lane & 31, n = min(rows, 32);
  if (r >= n) return;
  float* part = slot + w * 32 * kD + ((lane >> 5) * n + r) * 4;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4*>(part + (4 * db + i) * n * 8) =
          f32x4{a[db][4 * i], a[db][4 * i + 1], a[db][4 * i + 2], a[db][4 * i + 3]};
}

// What thread `id` of a join has: four columns of a row, at `offset` of each of a shared unit's parts.
struct PartPlace {
  int slot0, row, col;   // the unit's first slot, its row (0..127) and the first column
  size_t offset;
};
__device__ __forceinline__ PartPlace part_place(int id, int rows) {   // rows: of a slot, part_rows
  const int in_slot = id % (rows * (kD / 4)), n = min(rows, 32);
  const int w = in_slot / (n * 32), in_wave = in_slot % (n * 32);
  return PartPlace{id / (rows * (kD / 4)), 32 * w + in_wave % n, 4 * (in_wave / n), (size_t)in_slot * 4};
}

// Store four columns of a row of sums, times m, as bf16.
__device__ __forceinline__ void store_cols(uint16_t* out, const f32x4& x, float m) {
  bf16x4 h;
#pragma unroll
  for (int t = 0; t < 4; ++t) h[t] = (__bf16)(x[t] * m);
  *reinterpret_cast<bf16x4*>(out) = h;
}

}  // namespace
}  // namespace dsattn

#endif
