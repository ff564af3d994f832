// Tiles of matrix products on the matrix cores: what the products grouped by
// expert, forward and backward, and those in MXFP4 have in common.
//
//   C[a, b] = sum_k A[a, k] B[b, k]
//
// A block is 4 waves, one per SIMD, 2 x 2 over a tile of 64 TA x 64 TB; a wave
// owns TA x TB tiles of 32 x 32 (v_mfma_f32_32x32x16, in MXFP4
// v_mfma_scale_f32_32x32x64: lane l holds 16 bytes of row l % 32 of either
// operand and C[8 (i / 4) + 4 (l / 32) + i % 4][l % 32]).
//
// Staging.  Both operands go to LDS by direct loads of 16 bytes a lane, in
// stages of 64 reduction steps (256 in MXFP4) and rings of 2 to 8 slots.  An
// operand whose reduction is contiguous in memory (ROWS) takes one full
// 128-byte line of each row; one whose reduction runs over the rows (COLS)
// takes 64 rows of 128 T bytes and is transposed by the fragment reads
// (ds_read_b64_tr_b16: four elements of a column).  What lies outside of the
// matrices - rows and columns past the ends, reduction steps past the last -
// is masked by the buffer's range check and arrives as zeros.
//
// Bank conflicts.  ROWS: the 16-byte chunk c of row r sits at position
// c ^ (r / 2 % 8).  COLS: 64-byte pieces are permuted by the row's last bits,
// so that the four rows that a half-wave reads 64 bytes of cover all banks.
//
// Order of the reduction.  It is free as long as both operands agree: lane
// half h takes steps 32 h + 8 s .. + 7 of the stage in step s = 0..3 (in MXFP4
// blocks of 32: block 4 h + s, whose scales are then byte s of a dword).
//
// Pipeline.  Fragments of step s + 1 are read between the products of step s;
// the barrier between stages stands before the last step's products, so that
// the next stage's first fragments are read under those.  A stage's loads are
// spread over its quarters.  They are inline assembly without register results
// (the compiler would otherwise wait for all of them before every LDS read);
// the waits are explicit counts.
#pragma once

#include <type_traits>

#include "moe_internal.h"

namespace moe {
namespace tile {

constexpr int kThreads = 256;
constexpr int kStage = 64;                        // reduction steps of 16 bits per stage

enum { F16 = 0, BF16 = 1, F4 = 2 };               // element types of the products
enum { ROWS = 0, COLS = 1, CODES = 2 };           // how an operand lies in memory

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kMasked = 1u << 31;            // an offset outside of every buffer

// 16 bytes per lane from base + off to LDS at lds + 16 * lane; zeros where
// off >= limit.  lds, base and limit are wave-uniform.  m0 holds the LDS
// address; one wait state is required between its write and the load.
__device__ inline void load_lds(uint32_t lds, const uint8_t* base, uint32_t limit, uint32_t off) {
  const uint64_t p = (uint64_t)(uintptr_t)base;
  const u32x4 d = {(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, limit, 0x00020000u};
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(lds), "v"(off), "s"(d) : "memory", "m0");
}

// All but the N newest loads of this wave are in LDS and every LDS read of it
// has returned, then the block's barrier.
template <int N>
__device__ inline void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

// A wave-uniform pointer in scalar registers.
__device__ inline const uint8_t* uniform(const void* p) {
  const uint64_t v = (uint64_t)(uintptr_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const uint8_t*>(((uint64_t)hi << 32) | lo);
}

template <class T>
__device__ inline T lds_read(const lds_u8* lds, uint32_t at) {
  return *reinterpret_cast<const __attribute__((address_space(3))) T*>(lds + at);
}
template <class T>
__device__ inline void lds_write(lds_u8* lds, uint32_t at, T v) {
  *reinterpret_cast<__attribute__((address_space(3))) T*>(lds + at) = v;
}

// One operand of a block's tile: 64 T rows (ROWS, CODES) or columns (COLS) of
// a matrix from `base` on, of which `valid` exist.
struct Operand {
  const uint8_t* base;
  uint32_t row_bytes;   // distance of the matrix's rows
  int valid;
};

// An operand's loads: per lane the source of each of a wave's 2 T loads per
// stage, relative to the stage's base.  Load i of wave w fills 1024 bytes of
// the slot from 1024 (w + 4 i) on.
template <int KIND, int T>
struct Loads {
  static constexpr int kN = 2 * T;
  static constexpr uint32_t kSlot = 8192 * T;
  uint32_t off[KIND == CODES ? 1 : kN];
  uint32_t chunk;       // ROWS, CODES: the lane's 16 bytes of each row's 128
  const uint8_t* base;
  uint32_t row_bytes;
  int row0, valid;      // CODES: the lane's row of load 0

  __device__ inline void init(const Operand& o, int wave) {
    const int l = threadIdx.x & 63;
    base = uniform(o.base);
    row_bytes = o.row_bytes;
    chunk = 16 * ((l & 7) ^ ((4 * (wave & 1) + (l >> 4)) & 7));
    row0 = 8 * wave + (l >> 3);
    valid = o.valid;
#pragma unroll
    for (int i = 0; i < (KIND == CODES ? 0 : kN); ++i) {
      const int q = wave + 4 * i;
      if (KIND == COLS) {
        const int at = 64 * q + l, row = at / (8 * T), pos = at % (8 * T);
        const int c = pos ^ piece(row);
        off[i] = 8 * c < o.valid ? (uint32_t)row * row_bytes + 16 * c : kMasked;
      } else {
        const int row = 8 * q + (l >> 3);
        off[i] = row < valid ? (uint32_t)row * row_bytes + chunk : kMasked;
      }
    }
  }
  // (a unit's loads are spread over four stages: their number is not known
  // where they are issued)
  __device__ inline uint32_t source(int i) const {
    if constexpr (KIND != CODES) return off[i];
    const int row = row0 + 32 * i;
    return row < valid ? (uint32_t)row * row_bytes + chunk : kMasked;
  }
  // COLS: what row r's chunks are permuted by (64-byte pieces: bits 2 and up)
  static __device__ inline int piece(int r) { return T % 2 ? (r & 2) << 1 : (r & 3) << 2; }

  // stage k of `steps` reduction steps in all (ROWS, CODES: bytes of a row)
  __device__ inline void load(int k, int steps, int i, uint32_t lds, uint32_t tail) const {
    if (KIND == COLS) {
      const int left = __builtin_amdgcn_readfirstlane(max(0, min(steps - kStage * k, kStage)));
      load_lds(lds, base + (int64_t)k * kStage * row_bytes, (uint32_t)left * row_bytes, source(i));
    } else {
      load_lds(lds, base + (int64_t)k * 128, 128 * k < steps ? kMasked - 1 : 0, source(i) | tail);
    }
  }
};

__device__ inline uint32_t as_u32(f16x2 v) { return __builtin_bit_cast(uint32_t, v); }

// The 8 values of a word of codes, in TYPE.
template <int TYPE>
__device__ inline u32x4 decode(uint32_t w, float s) {
  if constexpr (TYPE == F16) {
    return u32x4{as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0)),
                 as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1)),
                 as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2)),
                 as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3))};
  } else {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
    return u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                 __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
  }
}

// 2^(byte - 127) as the conversion instructions take it (they go by the
// exponent field, so infinity is the byte 255 and gives NaN; 2^-127 is a
// subnormal).
__device__ inline float scale_of(uint32_t byte) {
  return __builtin_bit_cast(float, max(byte << 23, 0x00400000u));
}

// LDS of a tile: rings of SA and SB slots (a slot of CODES holds 4 stages),
// then two slots of scales, 8 bytes per row.
template <int TYPE, int KA, int KB, int TA, int TB, int LDS>
struct Ring {
  static constexpr bool kScales = TYPE == F4 || KA == CODES;
  static constexpr uint32_t kA = 8192 * TA, kB = 8192 * TB;
  static constexpr uint32_t kScaleSlot = kScales ? 512 * (TA + (TYPE == F4 ? TB : 0)) : 0;
  static constexpr uint32_t kRoom = LDS - 2 * kScaleSlot;
  static constexpr int kBoth = (int)(kRoom / (kA + kB));
  // with scales, whose loads the compiler waits for, no load is left in
  // flight at a barrier, and deeper rings would be waited for in vain
  static constexpr int SB = kScales ? 2 : kBoth > 8 ? 8 : kBoth;
  static constexpr int SA = kScales ? 2 : SB == 2 && 3 * kA + 2 * kB <= kRoom ? 3 : SB;
  static constexpr uint32_t kBBase = SA * kA, kScaleBase = kBBase + SB * kB;
  static_assert(SB >= 2 && kScaleBase + 2 * kScaleSlot <= LDS, "LDS");
  // loads that may be in flight when a stage ends: those of the stages after
  // the next one
  static constexpr int kPending = (SA - 2) * 2 * TA + (SB - 2) * 2 * TB;
};

// The accumulators of a wave: acc[i][j] is A tile i, B tile j of its own.
template <int TA, int TB> using Acc = f32x16[TA][TB];

// Scales of an operand in MXFP4 (null otherwise): row 0's, rows of `bytes`.
struct Scales {
  const uint8_t* at;
  int bytes;
};

// acc = the tile's product over `steps` reduction steps (F4: columns).
template <int TYPE, int KA, int KB, int TA, int TB, int LDS>
__device__ __forceinline__ void product(const Operand& oa, const Operand& ob, int steps, lds_u8* lds,
                                        Acc<TA, TB>& acc, Scales as = {nullptr, 0},
                                        Scales bs = {nullptr, 0}) {
  using R = Ring<TYPE, KA, KB, TA, TB, LDS>;
  constexpr bool kF4 = TYPE == F4, kCodes = KA == CODES;
  const int l = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wa = wave >> 1, wb = wave & 1;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  // stages; bytes of a row where it is the reduction
  const int nst = kF4 ? (steps + 255) / 256 : (steps + kStage - 1) / kStage;
  const int a_steps = KA == COLS ? steps : kF4 || kCodes ? steps / 2 : steps * 2;
  const int b_steps = KB == COLS ? steps : kF4 ? steps / 2 : steps * 2;

  Loads<KA, TA> la;
  Loads<KB, TB> lb;
  la.init(oa, wave);
  lb.init(ob, wave);
  // In MXFP4 a row's last line may be partial: its missing chunks are masked
  // (both operands' chunks are the same).
  auto tail = [&](int k, int bytes) -> uint32_t {
    return (uint32_t)(128 * k) + la.chunk < (uint32_t)bytes ? 0 : kMasked;
  };
  auto load_a = [&](int k, int i, uint32_t slot) {
    la.load(k, a_steps, i, lds0 + slot * R::kA + (wave + 4 * i) * 1024,
            kF4 || kCodes ? tail(k, a_steps) : 0);
  };
  auto load_b = [&](int k, int i, uint32_t slot) {
    lb.load(k, b_steps, i, lds0 + R::kBBase + slot * R::kB + (wave + 4 * i) * 1024,
            kF4 ? tail(k, b_steps) : 0);
  };

  // Scales of 256 columns (8 bytes) of the thread's row of A, and in F4 of B:
  // from memory to registers, a unit later to LDS.  Past the row: 2^0.
  const int t = threadIdx.x;
  auto fetch = [&](const Scales& s, int row, int u) -> uint64_t {
    const uint8_t* p = s.at + (int64_t)row * s.bytes + 8 * u;
    uint64_t v = 0x7F7F7F7F7F7F7F7Full;
    if (8 * u + 8 <= s.bytes) {
      __builtin_memcpy(&v, p, 8);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (8 * u + 2 * i < s.bytes) {
          uint16_t w;
          __builtin_memcpy(&w, p + 2 * i, 2);
          v = (v & ~(0xFFFFull << (16 * i))) | (uint64_t)w << (16 * i);
        }
    }
    return v;
  };
  uint64_t sa_next = 0, sb_next = 0;
  auto fetch_scales = [&](int u) {
    if constexpr (R::kScales) {
      if (t < 64 * TA) sa_next = fetch(as, min(t, oa.valid - 1), u);
      if (kF4 && t < 64 * TB) sb_next = fetch(bs, min(t, ob.valid - 1), u);
    }
  };
  auto put_scales = [&](int u) {
    if constexpr (R::kScales) {
      const uint32_t at = R::kScaleBase + (u & 1) * R::kScaleSlot;
      if (t < 64 * TA) lds_write(lds, at + 8 * t, sa_next);
      if (kF4 && t < 64 * TB) lds_write(lds, at + 512 * TA + 8 * t, sb_next);
    }
  };

  fetch_scales(0);
  put_scales(0);
  fetch_scales(1);
  // the rings' first stages; what the first stage needs comes first
#pragma unroll
  for (int v = 0; v < (R::SA > R::SB ? R::SA : R::SB) - 1; ++v) {
    if (v < R::SB - 1) {
#pragma unroll
      for (int i = 0; i < 2 * TB; ++i) load_b(v, i, v);
    }
    if (v < R::SA - 1) {
#pragma unroll
      for (int i = 0; i < 2 * TA; ++i) load_a(v, i, v);
    }
  }
#pragma unroll
  for (int i = 0; i < TA; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

  // where the lane's fragments lie in a slot
  const int half = l >> 5, sw = (l >> 1) & 7;
  uint32_t cat[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) cat[s] = 16 * ((4 * half + s) ^ sw);
  const uint32_t arow = (uint32_t)(wa * TA * 32 + (l & 31)) * 128;
  const uint32_t brow = (uint32_t)(wb * TB * 32 + (l & 31)) * 128;
  // COLS: the lane's row within a step's four, and its 8 bytes of tile i
  const int cr = (l & 15) >> 2;
  auto col_at = [&](int T, int tile_) -> uint32_t {
    const int x = T % 2 ? cr >> 1 : cr;
    return (uint32_t)(32 * half + cr) * (128 * T) + 64 * (tile_ ^ x) + 32 * ((l >> 4) & 1) + 8 * (l & 3);
  };
  uint32_t acol[TA], bcol[TB];
#pragma unroll
  for (int i = 0; i < TA; ++i) acol[i] = KA == COLS ? col_at(TA, wa * TA + i) : 0;
#pragma unroll
  for (int j = 0; j < TB; ++j) bcol[j] = KB == COLS ? col_at(TB, wb * TB + j) : 0;

  u32x4 a[2][TA], b[2][TB], raw[kCodes ? TA : 1];
  float scale[kCodes ? TA : 1];
  uint32_t sa[kF4 ? TA : 1], sb[kF4 ? TB : 1], sa1[kF4 ? TA : 1], sb1[kF4 ? TB : 1];
  auto transposed = [&](uint32_t at, uint32_t four_rows) -> u32x4 {
    const auto p = reinterpret_cast<__attribute__((address_space(3))) s16x4*>(lds + at);
    const auto q = reinterpret_cast<__attribute__((address_space(3))) s16x4*>(lds + at + four_rows);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q);
    const u32x2 x = __builtin_bit_cast(u32x2, lo), y = __builtin_bit_cast(u32x2, hi);
    return u32x4{x.x, x.y, y.x, y.y};
  };
  auto read_a = [&](int s, int i, uint32_t slot) {
    const uint32_t at = slot * R::kA;
    if constexpr (KA == ROWS) a[s & 1][i] = lds_read<u32x4>(lds, at + arow + i * 4096 + cat[s]);
    else if constexpr (KA == COLS) a[s & 1][i] = transposed(at + acol[i] + s * 1024 * TA, 512 * TA);
    else a[s & 1][i] = decode<TYPE>(raw[i][s], scale[i]);
  };
  auto read_b = [&](int s, int j, uint32_t slot) {
    const uint32_t at = R::kBBase + slot * R::kB;
    if constexpr (KB == COLS) b[s & 1][j] = transposed(at + bcol[j] + s * 1024 * TB, 512 * TB);
    else b[s & 1][j] = lds_read<u32x4>(lds, at + brow + j * 4096 + cat[s]);
  };
  // CODES: the lane's 32 codes of stage k and their scale
  auto read_raw = [&](int k, int i, uint32_t slot) {
    if constexpr (kCodes) {
      raw[i] = lds_read<u32x4>(lds, slot * R::kA + arow + i * 4096 + 16 * ((2 * (k & 3) + half) ^ sw));
      const uint32_t at = R::kScaleBase + ((k >> 2) & 1) * R::kScaleSlot + (arow >> 4) + i * 256;
      scale[i] = scale_of(lds_read<uint8_t>(lds, at + 2 * (k & 3) + half));
    }
  };
  auto read_scales = [&](int k, uint32_t (&x)[kF4 ? TA : 1], uint32_t (&y)[kF4 ? TB : 1]) {
    if constexpr (kF4) {
      const uint32_t at = R::kScaleBase + (k & 1) * R::kScaleSlot + 4 * half;
#pragma unroll
      for (int i = 0; i < TA; ++i) x[i] = lds_read<uint32_t>(lds, at + (arow >> 4) + i * 256);
#pragma unroll
      for (int j = 0; j < TB; ++j) y[j] = lds_read<uint32_t>(lds, at + 512 * TA + (brow >> 4) + j * 256);
    }
  };
  // quarter c of the products of step s
  constexpr int kProducts = TA * TB;
  auto one = [&](auto sc, int m) {
    constexpr int s = decltype(sc)::value;
    const u32x4 x = a[s & 1][m % TA], y = b[s & 1][m / TA];
    f32x16& c = acc[m % TA][m / TA];
    if constexpr (TYPE == F16) {
      c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
    } else if constexpr (TYPE == BF16) {
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
    } else {
      const i32x8 p = {(int)x.x, (int)x.y, (int)x.z, (int)x.w, 0, 0, 0, 0};
      const i32x8 q = {(int)y.x, (int)y.y, (int)y.z, (int)y.w, 0, 0, 0, 0};
      c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p, q, c, 4, 4, s, (int)sa[m % TA], s, (int)sb[m / TA]);
    }
  };
  auto products = [&](auto sc, int c) {
#pragma unroll
    for (int m = c * kProducts / 4; m < (c + 1) * kProducts / 4; ++m) one(sc, m);
  };
  // keeps a quarter's reads and conversions between its products
  auto pin = [&](int c) {
#pragma unroll
    for (int m = c * kProducts / 4; m < (c + 1) * kProducts / 4; ++m) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);  // LDS reads
      __builtin_amdgcn_sched_group_barrier(0x002, kCodes ? 6 : 2, 0);  // VALU
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  auto next = [](uint32_t slot, int slots) { return slot + 1 == (uint32_t)slots ? 0u : slot + 1; };
  uint32_t ac = 0, bc = 0;                          // slots of stage k (CODES: of its unit)
  uint32_t al = R::SA - 1, bl = R::SB - 1;          // slots loaded next
  // Quarter c's share (of 16) of the loads issued between the barrier before
  // stage k and the one in it: B's first, whose ring is never the deeper one.
  // CODES: a quarter of a unit's per stage.
  static_assert(!kCodes || TA % 2 == 0, "whole loads per stage");
  constexpr int kAStage = kCodes ? TA / 2 : 2 * TA;
  constexpr int kAll = 2 * TB + kAStage;
  constexpr int kSpread = 12;
  auto loads = [&](int k, int c) {
#pragma unroll
    for (int i = c * kAll / kSpread; i < min((c + 1) * kAll / kSpread, kAll); ++i) {
      if (i < 2 * TB) {
        load_b(k + R::SB - 1, i, bl);
      } else if constexpr (kCodes) {
        load_a((k >> 2) + 1, (k & 3) * kAStage + i - 2 * TB, al);
      } else {
        load_a(k + R::SA - 1, i - 2 * TB, al);
      }
    }
  };
  constexpr std::integral_constant<int, 0> s0;
  constexpr std::integral_constant<int, 1> s1;
  constexpr std::integral_constant<int, 2> s2;
  constexpr std::integral_constant<int, 3> s3;
  auto step = [&](auto sc, int k) {
    constexpr int s = decltype(sc)::value;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      loads(k, 4 + 4 * s + c);
#pragma unroll
      for (int i = 0; i < TA; ++i)
        if (3 * i / TA == c) read_a(s + 1, i, ac);
#pragma unroll
      for (int j = 0; j < TB; ++j)
        if (3 * j / TB == c) read_b(s + 1, j, bc);
      products(sc, c);
      pin(c);
    }
  };

  stage_barrier<0>();
  read_scales(0, sa, sb);
#pragma unroll
  for (int i = 0; i < TA; ++i) {
    read_raw(0, i, 0);
    read_a(0, i, 0);
  }
#pragma unroll
  for (int j = 0; j < TB; ++j) read_b(0, j, 0);
  // scales one unit ahead: into LDS, whose slot the last barrier freed, and
  // the unit after it into registers
  auto scales_ahead = [&](int k) {
    if constexpr (kF4) {
      put_scales(k + 1);
      fetch_scales(k + 2);
    } else if constexpr (kCodes) {
      if ((k & 3) == 0) {
        put_scales((k >> 2) + 1);
        fetch_scales((k >> 2) + 2);
      }
    }
  };
  scales_ahead(0);
#pragma unroll
  for (int c = 0; c < 4; ++c) loads(0, c);
  for (int k = 0; k < nst; ++k) {
    step(s0, k);
    step(s1, k);
    step(s2, k);
    // every load of stage k + 1 has arrived; the slots of stage k are free
    stage_barrier<R::kPending>();
    if (!kCodes || (k & 3) == 3) {
      ac = next(ac, R::SA);
      al = next(al, R::SA);
    }
    bc = next(bc, R::SB);
    bl = next(bl, R::SB);
    scales_ahead(k + 1);
    read_scales(k + 1, sa1, sb1);
    // (after the last stage: reads that are not multiplied)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      loads(k + 1, c);
      if (c == 0) {
#pragma unroll
        for (int i = 0; i < TA; ++i) read_raw(k + 1, i, ac);
      }
#pragma unroll
      for (int i = 0; i < TA; ++i)
        if (kCodes ? 1 + i * 3 / TA == c : 3 * i / TA == c) read_a(0, i, ac);
#pragma unroll
      for (int j = 0; j < TB; ++j)
        if (3 * j / TB == c) read_b(0, j, bc);
      products(s3, c);
      pin(c);
    }
    if constexpr (kF4) {
#pragma unroll
      for (int i = 0; i < TA; ++i) sa[i] = sa1[i];
#pragma unroll
      for (int j = 0; j < TB; ++j) sb[j] = sb1[j];
    }
  }
  // the LDS must not be handed on with loads in flight
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// Stores a wave's tiles as 16-bit rows: C's b is the row, a the column, whose
// eight values go out as 16 bytes (the lane halves trade four each).
template <class T, int TA, int TB>
__device__ __forceinline__ void store_rows(Acc<TA, TB>& acc, T* out, int64_t ld, int rows, int cols) {
  typedef T x2 __attribute__((ext_vector_type(2)));
  const int l = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int a0 = (wave >> 1) * TA * 32, b0 = (wave & 1) * TB * 32;
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    const int row = b0 + 32 * j + (l & 31);
    T* to = out + (int64_t)row * ld + a0 + 8 * (l >> 5);
#pragma unroll
    for (int i = 0; i < TA; ++i) {
      if (a0 + 32 * i >= cols) continue;
      // (a tile stays where the products left it until it is converted: all of
      // them copied at once would not fit the other registers)
      if constexpr (TA * TB > 8) asm volatile("" : "+v"(acc[i][j]));
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        uint32_t v[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const x2 w = {(T)acc[i][j][8 * q + 2 * p], (T)acc[i][j][8 * q + 2 * p + 1]};
          v[p] = __builtin_bit_cast(uint32_t, w);
        }
        // lower half: columns 0..3 of both eights, upper half: 4..7
        const auto x = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
        const auto y = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
        if (row < rows)
          *reinterpret_cast<u32x4*>(to + 32 * i + 16 * q) =
              u32x4{(uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1]};
      }
    }
  }
}

}  // namespace tile
}  // namespace moe
