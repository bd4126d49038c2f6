// Projections of few rows with weights in 4 bits (daf_linear_mx): C = A W^T (+ bias)
// (+ residual), W as e2m1 codes with a power-of-two scale per 32 of a row, A in bf16 or
// as e4m3 codes with such scales (daf_add_rmsnorm).
//
// Codes times their scale become bf16 by one conversion instruction per two values, exactly
// below 2^128, so the products of v_mfma_f32_16x16x32_bf16 are exact within fp32's normal
// range, and sums are fp32. (The
// instruction that takes the codes and scales themselves keeps about 13 bits of a small
// term beside a large one.)
//
// Bound by the bytes of W. A workgroup passes a range of tiles of 16 rows of W; each of its
// waves keeps a part of K for all of them, with its part of A in registers, and its own
// ring in LDS to which copies of its part of the next tiles are on their way: 256 bytes of
// a row at a time, nothing of a wave waits for another's. From there lane (n, g) reads the
// 16 bytes of row n that are the 32 values with one scale at k = 32 g of a step of 128,
// four operands of 8 values; A is held in the same order of k. A tile's sums of the waves
// meet in LDS, in a fixed order, one barrier per tile.
//
// 32 rows by 37888 x 3584 (72 MB of W) take 18.6 to 19.4 us, 3.9 TB/s, where reading as many
// bytes takes 13; of the SIMDs' cycles matrix instructions are 22% and vector instructions 36%.
// In calls of 19.3, without the joins it takes 16.8, without matrix instructions 17.4, of A alone
// 5.5 (launch included). Rings beside registers: loads of W to registers in operand layout keep
// the address unit 64 cycles for 1 KiB, a copy of whole pieces of rows 16; the first version,
// with those and A read again for each tile, took 26 to 42. 1 row by 4608 x 3584 5.7 us, most of
// it launch and one chain of loads; 12 rows by 3584 x 18944 13.6 us in 5 splits, of which the
// join is 3.9 and what A takes ahead of W, with launches and join, 8.4.
#include <algorithm>

#include "step.h"

namespace daf {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma(const bf16x8 &a, const bf16x8 &b, const f32x4 &c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

// 2^(b - 127) of a scale's byte, which counts as one of 27 .. 247 (2^-100 .. 2^120), as rows in
// 8 bits and weights have them: all values of codes are then normal bf16 values, but for e4m3
// codes of 256 or more under 2^120, which are infinite; 255 is NaN
__device__ __forceinline__ float scale_of(unsigned b) {
  const unsigned e = b == 255 ? 0x7fc00000u : min(max(b, 27u), 247u) << 23;
  return __builtin_bit_cast(float, e);
}

// eight e2m1 codes (the low half of a byte first) times a scale
__device__ __forceinline__ bf16x8 widen4(unsigned w, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#else
  return bf16x8{};
#endif
}
// eight e4m3 codes times a scale
__device__ __forceinline__ bf16x8 widen8(unsigned lo, unsigned hi, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#else
  return bf16x8{};
#endif
}

__device__ __forceinline__ void lds_barrier() {  // loads and copies from memory stay in flight
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#endif
}
template <int N>
__device__ __forceinline__ void wait_copies() {  // all but the N newest of the wave's copies have arrived
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
#endif
}
// Copies of 16 (or 4) bytes per lane, from byte voff of the buffer to LDS byte lds + 16 (4)
// times the lane; zeros from beyond the buffer's end. In asm, so that the compiler does not
// wait for the copies in flight at each LDS read: wait_copies counts them. The s_nop makes
// up the wait states between a vector instruction that writes a scalar operand and this read
// of it, which the compiler does not see here.
__device__ __forceinline__ void copy16(const u32x4 &rsrc, uint32_t voff, uint32_t lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 3\n\t"
      "buffer_load_dwordx4 %1, %2, 0 offen lds"
      :
      : "s"(lds), "v"(voff), "s"(rsrc)
      : "memory", "m0");
#endif
}
__device__ __forceinline__ void copy4(const u32x4 &rsrc, uint32_t voff, uint32_t lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 3\n\t"
      "buffer_load_dword %1, %2, 0 offen lds"
      :
      : "s"(lds), "v"(voff), "s"(rsrc)
      : "memory", "m0");
#endif
}
__device__ __forceinline__ u32x4 buffer(const unsigned char *p, uint32_t bytes) {
  const uint64_t base = (uint64_t)p;
  return u32x4{(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, bytes, 0x00020000u};
}
constexpr uint32_t kNowhere = 0xf0000000u;  // beyond the end of every buffer here

// What a wave's ring holds of 16 rows: of each PIECES pieces of 16 bytes, piece c of row r at
// place c ^ swizzle(r), so that the 16 rows of a piece are in different banks; then of each
// row 4 aligned words from the one that has its first scale on, and then a fifth.
template <int PIECES>
struct Slot {
  static constexpr int COPIES = PIECES / 4, CODES = COPIES * 1024;
  static __device__ __forceinline__ int swizzle(int row) { return PIECES == 16 ? row : PIECES == 8 ? row / 2 : row / 4; }
  static __device__ __forceinline__ int row(int copy) { return (copy * 64 + (threadIdx.x & 63)) / PIECES; }
  static __device__ __forceinline__ int piece(int copy) { return (threadIdx.x & 63) % PIECES ^ swizzle(row(copy)); }
  static __device__ __forceinline__ u32x4 read(const unsigned char *slot, int row, int piece) {
    return *reinterpret_cast<const u32x4 *>(slot + (row * PIECES + (piece ^ swizzle(row))) * 16);
  }
  // the scale at byte b of a row's words
  static __device__ __forceinline__ unsigned scale(const unsigned char *slot, int row, int b) {
    return slot[CODES + (b < 16 ? row * 16 + b : 240 + row * 4 + b)];
  }
};
constexpr int kSlotBytes = 4096 + 512;  // a copy of words writes one for each of 64 lanes
// Of a wave's ring: two tiles are on their way beside the one that is read. (us: 1 row by 37888 x
// 3584 14.8, with 2 slots 17.0, with 4 15.8; 12 rows by 3584 x 18944 13.6, 13.5 and 14.7; 32 rows,
// for which 4 do not fit LDS, by 37888 x 3584 19.3 and 20.9.)
constexpr int kSlots = 3;

// The words of 16 rows' scales, `blocks` bytes a row, from block b0 of each on
struct ScaleWords {
  uint32_t at[2];  // of a lane
  int skew;        // bytes between the first word and the first scale
  int first;       // byte of the lane's row, as an operand has rows, in its first word
  __device__ __forceinline__ ScaleWords(const unsigned char *scales, int blocks, int b0) {
    const int lane = threadIdx.x & 63;
    skew = (int)((uintptr_t)scales & 3);
    auto byte = [&](int row) { return skew + row * blocks + b0; };
    at[0] = (byte(lane / 4) & ~3) + 4 * (lane % 4);
    at[1] = lane < 16 ? (byte(lane) & ~3) + 16 : kNowhere;
    first = byte(lane & 15) & 3;
  }
  // of `rows` rows from `scales` on, to LDS; words beyond the last row's are not read
  __device__ __forceinline__ void copy(const unsigned char *scales, int blocks, int rows, uint32_t ahead, uint32_t to) const {
    const u32x4 words = buffer(scales - skew, rows > 0 ? (skew + rows * blocks + 3) & ~3 : 0);
    copy4(words, at[0] + ahead, to);
    copy4(words, at[1] + (at[1] == kNowhere ? 0 : ahead), to + 256);
  }
};

template <bool MX, int MT, int STEPS>
__global__ __launch_bounds__(64 * kMxWaves, 2) void linear_mx_kernel(const MxLaunch p) {
  using S = Slot<4 * STEPS>;
  using SA = Slot<16>;  // of A 256 bytes a row: a step of bf16, two of codes
  constexpr int SLOTS = kSlots, APIECE = MX ? 2 : 1, ITEMS = (STEPS + APIECE - 1) / APIECE * MT;
  __shared__ f32x4 sums[2][kMxWaves][MT][64];
  __shared__ __align__(16) unsigned char rings[kMxWaves][SLOTS][kSlotBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int group = blockIdx.x, split = blockIdx.y;
  const int64_t m0 = (int64_t)blockIdx.z * (16 * MT);
  const int kwaves = 1 << p.kwaves_log2, kwave = wave & (kwaves - 1);
  const int nwave = wave >> p.kwaves_log2, nwaves_log2 = kMxWavesLog2 - p.kwaves_log2, nwaves = 1 << nwaves_log2;
  // this wave's steps of K
  const int part = split * kwaves + kwave;
  const int s0 = part * p.part_steps + min(part, p.longer_parts), n_steps = p.part_steps + (part < p.longer_parts);
  // the workgroup's tiles, nwaves at a time
  const int t0 = group * p.group_tiles + min(group, p.longer_groups);
  const int t1 = t0 + p.group_tiles + (group < p.longer_groups), n_tiles = (t1 - t0 + nwaves - 1) >> nwaves_log2;
  const int blocks = p.k / kBlockValues, row_bytes = p.k / 2;

  // Through the ring go, one after the other, the parts of A and the tiles; what lies beyond
  // their ends is copied from nowhere, so that every item has as many copies.
  const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)&rings[wave][0][0];
  const int arow_bytes = p.k * (MX ? 1 : 2);
  uint32_t a_at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) a_at[i] = SA::row(i) * arow_bytes + s0 * (MX ? 128 : 256) + SA::piece(i) * 16;
  const ScaleWords a_words(MX ? p.a_scales : p.w_scales, blocks, s0 * 4);
  auto fetch_a = [&](int slot, int item) {
    const int e = item % MT, ahead = item / MT * 256;  // bytes of the rows before
    const int64_t row = m0 + 16 * e, rows = min((int64_t)16, max(p.m - row, (int64_t)0));
    const u32x4 from = buffer(p.a + (rows > 0 ? row : 0) * arow_bytes, (uint32_t)rows * arow_bytes);
    const uint32_t to = ring + slot * kSlotBytes;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = s0 * (MX ? 128 : 256) + ahead + SA::piece(i) * 16 < arow_bytes;
      copy16(from, in ? a_at[i] + ahead : kNowhere, to + i * 1024);
    }
    a_words.copy(MX ? p.a_scales + (rows > 0 ? row : 0) * blocks : p.w_scales, blocks, MX ? (int)rows : 0,
                 item / MT * 8, to + SA::CODES);
  };
  uint32_t w_at[STEPS];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int at = s0 * (kMxStep / 2) + S::piece(i) * 16;  // of the row
    w_at[i] = S::piece(i) < n_steps * 4 && at < row_bytes ? (uint32_t)(S::row(i) * row_bytes + at) : kNowhere;
  }
  const ScaleWords w_words(p.w_scales, blocks, s0 * 4);
  auto fetch = [&](int slot, int i) {
    const int t = t0 + i * nwaves + nwave, rows = t < t1 ? min(16, p.n - t * 16) : 0;
    const size_t row = t < t1 ? (size_t)t * 16 : 0;
    const u32x4 codes = buffer(p.w + row * row_bytes, rows * row_bytes);
    const uint32_t to = ring + slot * kSlotBytes;
#pragma unroll
    for (int j = 0; j < STEPS; ++j) copy16(codes, w_at[j], to + j * 1024);
    w_words.copy(p.w_scales + row * blocks, blocks, rows, 0, to + S::CODES);
  };
  auto fetch_item = [&](int slot, int item) { item < ITEMS ? fetch_a(slot, item) : fetch(slot, item - ITEMS); };
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) fetch_item(i, i);

  int slot = 0;
  auto turn = [&] { slot = slot == SLOTS - 1 ? 0 : slot + 1; };
  auto before = [&] { return slot == 0 ? SLOTS - 1 : slot - 1; };
  auto slot_is_read = [&] {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#endif
  };
  auto k_of = [&](int step) { return (s0 + step) * kMxStep + g * 32; };  // of a lane
  bf16x8 a[STEPS][MT][4];
#pragma unroll
  for (int item = 0; item < ITEMS; ++item) {
    // fewer steps than 4: a tile has fewer copies than a part of A
    wait_copies<STEPS == 4 ? (SLOTS - 1) * 6 : 0>();
    const unsigned char *at = rings[wave][slot];
    const int e = item % MT, s = item / MT * APIECE;
    u32x4 x[4];
    unsigned scale[APIECE];
    if constexpr (MX) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[2 * i] = SA::read(at, n16, i * 8 + g * 2);
        x[2 * i + 1] = SA::read(at, n16, i * 8 + g * 2 + 1);
        scale[i] = SA::scale(at, n16, a_words.first + i * 4 + g);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = SA::read(at, n16, g * 4 + i);
    }
    slot_is_read();
    if (item < ITEMS - 1) fetch_item(slot, item + SLOTS);
    turn();
    if constexpr (MX) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (s + i >= STEPS) break;
        const float f = scale_of(k_of(s + i) < p.k ? scale[i] : 127u);  // past the end: codes are 0
#pragma unroll
        for (int j = 0; j < 4; ++j)
          a[s + i][e][j] = widen8(x[2 * i + j / 2][j % 2 * 2], x[2 * i + j / 2][j % 2 * 2 + 1], f);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) a[s][e][j] = __builtin_bit_cast(bf16x8, x[j]);
    }
  }

  auto store = [&](int i, int e, f32x4 x) {
    const int t = t0 + i * nwaves + nwave, n = t * 16 + g * 4;  // a lane has 4 features of a row
    const int64_t m = m0 + 16 * e + n16;
    if (t >= t1 || n >= p.n || m >= p.m) return;
    if (p.splits > 1) {
      float *to = p.part + ((size_t)split * p.m + m) * p.n + n;
      if (p.n % 4 == 0) *reinterpret_cast<f32x4 *>(to) = x;
      else
        for (int k = 0; k < 4 && n + k < p.n; ++k) to[k] = x[k];
      return;
    }
    const size_t at = (size_t)m * p.n + n;
    const __bf16 *bias = static_cast<const __bf16 *>(p.bias), *res = static_cast<const __bf16 *>(p.residual);
    __bf16 *to = static_cast<__bf16 *>(p.c) + at;
    if (p.n % 4 == 0) {
      if (bias) {
        const bf16x4 v = *reinterpret_cast<const bf16x4 *>(bias + n);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] += (float)v[k];
      }
      if (res) {
        const bf16x4 v = *reinterpret_cast<const bf16x4 *>(res + at);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] += (float)v[k];
      }
      *reinterpret_cast<bf16x4 *>(to) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
    } else {
      for (int k = 0; k < 4 && n + k < p.n; ++k) {
        float y = x[k];
        if (bias) y += (float)bias[n + k];
        if (res) y += (float)res[at + k];
        to[k] = (__bf16)y;
      }
    }
  };
  for (int i = 0; i < n_tiles; ++i) {
    wait_copies<(SLOTS - 2) * (STEPS + 2)>();
    const unsigned char *at = rings[wave][slot];
    u32x4 w[STEPS];
    unsigned scale[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      w[s] = S::read(at, n16, s * 4 + g);
      scale[s] = S::scale(at, n16, w_words.first + s * 4 + g);
    }
    slot_is_read();
    fetch(before(), i + SLOTS - 1);
    turn();
    // two sums each: a matrix instruction does not wait for the one before it
    f32x4 acc[MT] = {}, odd[MT] = {};
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
      if (s < n_steps) {
        // past the end of a row: zeros of A beside whatever lies there, but no NaN
        const float x1 = scale_of(k_of(s) < p.k ? scale[s] : 127u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x8 x = widen4(w[s][j], x1);
#pragma unroll
          for (int e = 0; e < MT; ++e) {
            f32x4 &to = j & 1 ? odd[e] : acc[e];
            to = mfma(x, a[s][e][j], to);
          }
        }
      }
#pragma unroll
    for (int e = 0; e < MT; ++e) acc[e] += odd[e];
    if (kwaves > 1) {
#pragma unroll
      for (int e = 0; e < MT; ++e) sums[i & 1][wave][e][lane] = acc[e];
      lds_barrier();
    }
#pragma unroll
    for (int e = 0; e < MT; ++e) {
      if (kwaves > 1) {  // the waves take the tiles' joins in turn
        if (kwave != ((i * MT + e) & (kwaves - 1))) continue;
        f32x4 y[kMxWaves];
#pragma unroll
        for (int k = 0; k < kMxWaves; ++k) y[k] = sums[i & 1][k < kwaves ? nwave * kwaves + k : wave][e][lane];
        acc[e] = y[0];
#pragma unroll
        for (int k = 1; k < kMxWaves; ++k)
          if (k < kwaves) acc[e] += y[k];
      }
      store(i, e, acc[e]);
    }
  }
  wait_copies<0>();  // none may arrive after the workgroup's end
}

// The sum of the splits, in their order: VEC features of a row per thread.
template <int VEC>
__global__ __launch_bounds__(256) void linear_mx_join_kernel(const MxLaunch p) {
  typedef float fv __attribute__((ext_vector_type(VEC)));
  typedef __bf16 bv __attribute__((ext_vector_type(VEC)));
  const int n = (blockIdx.y * 256 + threadIdx.x) * VEC;
  if (n >= p.n) return;
  const size_t at = (size_t)blockIdx.x * p.n + n, total = (size_t)p.m * p.n;
  constexpr int FLIGHT = 8;
  fv x = {};
  bv bias = {}, residual = {};
  if (p.bias) bias = *reinterpret_cast<const bv *>(static_cast<const __bf16 *>(p.bias) + n);
  if (p.residual) residual = *reinterpret_cast<const bv *>(static_cast<const __bf16 *>(p.residual) + at);
  for (int s0 = 0; s0 < p.splits; s0 += FLIGHT) {
    fv y[FLIGHT];
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i) y[i] = *reinterpret_cast<const fv *>(p.part + min(s0 + i, p.splits - 1) * total + at);
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i)
      if (s0 + i < p.splits) x += y[i];
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) x[i] += (float)bias[i];
#pragma unroll
  for (int i = 0; i < VEC; ++i) x[i] += (float)residual[i];
  bv y;
  for (int i = 0; i < VEC; ++i) y[i] = (__bf16)x[i];
  *reinterpret_cast<bv *>(static_cast<__bf16 *>(p.c) + at) = y;
}

template <bool MX>
void launch(const MxLaunch &p, hipStream_t st) {
  const dim3 grid(p.groups, p.splits, p.row_blocks);
  auto go = [&](auto kern) { kern<<<grid, 64 * kMxWaves, 0, st>>>(p); };
  if (p.mt == 1) p.steps == 1 ? go(linear_mx_kernel<MX, 1, 1>) : p.steps == 2 ? go(linear_mx_kernel<MX, 1, 2>) : go(linear_mx_kernel<MX, 1, 4>);
  else p.steps == 1 ? go(linear_mx_kernel<MX, 2, 1>) : p.steps == 2 ? go(linear_mx_kernel<MX, 2, 2>) : go(linear_mx_kernel<MX, 2, 4>);
}

}  // namespace

// Up to 4 steps of a wave, which with two tiles of A are 128 registers, by 8 waves: K above
// 4096 is split over workgroups, and more than 32 rows pass W again (37888 x 3584 by 32 rows
// 19.3 us, 64 28.5, 128 50.4). One workgroup per CU (their rings fill its LDS; 512 for 256 take
// 23.4 us for 19.3 by 32 rows); short K leaves waves for more tiles at once.
void plan_linear_mx(MxLaunch &p) {
  const int steps = (p.k + kMxStep - 1) / kMxStep;
  p.mt = p.m <= 16 ? 1 : 2;
  p.kwaves_log2 = steps >= 8 ? 3 : steps >= 4 ? 2 : steps >= 2 ? 1 : 0;
  const int kwaves = 1 << p.kwaves_log2, nwaves = kMxWaves / kwaves;
  p.splits = (steps + 4 * kwaves - 1) / (4 * kwaves);
  const int parts = p.splits * kwaves, most = (steps + parts - 1) / parts;
  p.part_steps = steps / parts;
  p.longer_parts = steps % parts;
  p.steps = most <= 2 ? most : 4;
  p.row_blocks = (int)((p.m + 16 * p.mt - 1) / (16 * p.mt));
  const int64_t tiles = ((int64_t)p.n + 15) / 16, turns = (tiles + nwaves - 1) / nwaves;
  p.groups = (int)std::min<int64_t>(turns, std::max<int64_t>(1, 256 / ((int64_t)p.row_blocks * p.splits)));
  p.group_tiles = (int)(tiles / p.groups);
  p.longer_groups = (int)(tiles % p.groups);
}

hipError_t launch_linear_mx(const MxLaunch &p, hipStream_t st) {
  p.a_scales ? launch<true>(p, st) : launch<false>(p, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const int vec = p.n % 4 == 0 ? 4 : 1;
  const dim3 grid((unsigned)p.m, (p.n + 256 * vec - 1) / (256 * vec));
  if (vec == 4) linear_mx_join_kernel<4><<<grid, 256, 0, st>>>(p);
  else linear_mx_join_kernel<1><<<grid, 256, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace daf
