// Tiles of matrix products on the matrix cores: what the products grouped by
// expert, forward and backward, and those in MXFP4 have in common.
//
//   C[a, b] = sum_k A[a, k] B[b, k]
//
// A block is 4 waves, one per SIMD, 2 x 2 over a tile of 64 TA x 64 TB (Waves); a
// wave owns TA x TB tiles of 32 x 32 (v_mfma_f32_32x32x16, in MXFP4
// v_mfma_scale_f32_32x32x64: lane l holds 16 bytes of row l % 32 of either
// operand and C[8 (i / 4) + 4 (l / 32) + i % 4][l % 32]).
//
// Staging.  Both operands go to LDS by direct loads of 16 bytes a lane, in
// stages of 64 reduction steps (256 in MXFP4) and rings of 2 to 6 slots.  An
// operand whose reduction is contiguous in memory (ROWS) takes one full
// 128-byte line of each row; one whose reduction runs over the rows (COLS)
// takes 64 rows of 128 T bytes and is transposed by the fragment reads
// (ds_read_b64_tr_b16: four elements of a column).  What lies outside of the
// matrices - rows and columns past the ends, reduction steps past the last -
// is masked by the buffer's range check and arrives as zeros.  Codes beside a
// partner of 16 bits (CODES) come in units of four stages, whole lines too, and
// become 16-bit fragments after the read, as a rule each by one wave.  Weights of tiles
// of up to 128 rows, which few other tiles share, pass the caches by: 60 experts
// of 1472 x 2048 with 89 rows each took 111 us without that, 97 with it.  The rows
// of d_y that the gradient of W has in their place do not.
//
// Bank conflicts.  ROWS: the 16-byte chunk c of row r sits at position
// c ^ (r / 2 % 8), CODES likewise.  COLS: 64-byte pieces are permuted by the row's last bits,
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
//
// Blocks.  Tiles of 256 x 256 have 64 products per 16 fragments read, one wave
// per SIMD; 160 KB of LDS hold two stages and the third of one operand.  Blocks
// of 128 and 64 columns leave room for two of them on a unit, for calls whose
// large tiles would not fill the chip.  Blocks are persistent: while one tile is
// stored the next one's loads are under way.
//
// Measured: 16384 x 4096 by 16 experts' 6400 rows in fp16 774 to 863 us, 1.0 to
// 1.1 PF, the matrix cores busy 75 % of the time; their power bounds it: with
// more and more columns to sum each costs as much as at 1.35 PF, on zeros as at
// 2.06 (products alone, nothing loaded: 1.68).  In MXFP4 8192 rows take 158 to
// 177 us, 2.4 to 2.7 PF of the 6.2 that the products alone reach: a wave has no
// partner on its SIMD to fill in between two stages, and the matrix cores are
// busy 37 % (without any loads it takes 16 us less).
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
// address; one wait state is required between its write and the load.  STREAM:
// what is read once, past the caches.
template <bool STREAM = false>
__device__ inline void load_lds(uint32_t lds, const uint8_t* base, uint32_t limit, uint32_t off) {
  const uint64_t p = (uint64_t)(uintptr_t)base;
  const u32x4 d = {(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, limit, 0x00020000u};
  if constexpr (STREAM)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds"
                 :: "s"(lds), "v"(off), "s"(d) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(off), "s"(d) : "memory", "m0");
}

// 4 bytes per lane to LDS at lds + 4 * lane, likewise.
__device__ inline void load_lds4(uint32_t lds, const uint8_t* base, uint32_t limit, uint32_t off) {
  const uint64_t p = (uint64_t)(uintptr_t)base;
  const u32x4 d = {(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, limit, 0x00020000u};
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
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

// A uniform value into vector registers: what is needed once a tile would crowd
// the scalar ones out of the loop.
template <class T>
__device__ inline void set_aside(T& v) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+v"(v));
#endif
}

// (a pointer that was set aside has lost its address space)
template <class T>
__device__ inline __attribute__((address_space(1))) T* global_ptr(const void* p) {
  return (__attribute__((address_space(1))) T*)(uintptr_t)p;
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

// An operand's loads: per lane the source of each of a wave's kN loads per
// stage, relative to the stage's place, which moves on.  Load i of wave w fills
// 1024 bytes of the slot from 1024 (w + 4 i) on.
template <int KIND, int T>
struct Loads {
  static constexpr int kN = 2 * T;
  static constexpr uint32_t kSlot = 4096 * kN;
  uint32_t off[kN];
  const uint8_t* at;
  uint32_t limit;       // what of it may be read (0: nothing)
  uint32_t row_bytes;

  // ROWS, CODES: the lane's 16 bytes of each row's 128 (of every load the same)
  static __device__ inline uint32_t chunk(int wave) {
    const int l = threadIdx.x & 63;
    return 16 * ((l & 7) ^ ((4 * (wave & 1) + (l >> 4)) & 7));
  }
  // COLS: what row r's chunks are permuted by (64-byte pieces: bits 2 and up)
  static __device__ inline int piece(int r) { return T % 2 ? (r & 2) << 1 : (r & 3) << 2; }

  __device__ inline void open(const Operand& o, int wave) {
    const int l = threadIdx.x & 63;
    at = uniform(o.base);
    row_bytes = __builtin_amdgcn_readfirstlane(o.row_bytes);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int q = wave + 4 * i;
      if (KIND == COLS) {
        const int to = 64 * q + l, row = to / (8 * T), c = (to % (8 * T)) ^ piece(row);
        off[i] = 8 * c < o.valid ? (uint32_t)row * row_bytes + 16 * c : kMasked;
      } else {
        const int row = 8 * q + (l >> 3);
        off[i] = row < o.valid ? (uint32_t)row * row_bytes + chunk(wave) : kMasked;
      }
    }
  }
  // to the next stage of the same tile, or (another) just opened
  __device__ inline void advance(bool another) {
    at += another ? 0 : KIND == COLS ? (int64_t)kStage * row_bytes : 128;
  }
  // `left` reduction steps from the stage's first on (0: none are read)
  __device__ inline void bound(int left) {
    limit = __builtin_amdgcn_readfirstlane(
        KIND == COLS ? max(0, min(left, kStage)) * row_bytes : left > 0 ? kMasked - 1 : 0);
  }
  template <bool STREAM>
  __device__ inline void load(int i, uint32_t lds, uint32_t mask) const {
    load_lds<STREAM>(lds, at, limit, off[i] | mask);
  }
};

__device__ inline uint32_t as_u32(f16x2 v) { return __builtin_bit_cast(uint32_t, v); }

// The 8 values of a word of codes, in TYPE: exact in bf16, and in fp16 where it
// holds the value; others are rounded to it (a product on the matrix cores takes
// operands of one type).
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

// Scale bytes 8 u .. 8 u + 7 of a row of `bytes` (256 columns of it; the row
// lies on an even address); those past the row: 2^0.
__device__ inline uint64_t scale_unit(const uint8_t* row, int bytes, int u) {
  const uint8_t* at = row + 8 * u;
  uint64_t v = 0x7F7F7F7F7F7F7F7Full;
  if (8 * u + 8 <= bytes) {
    __builtin_memcpy(&v, at, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (8 * u + 2 * i < bytes) {
        uint16_t w;
        __builtin_memcpy(&w, at + 2 * i, 2);
        v = (v & ~(0xFFFFull << (16 * i))) | (uint64_t)w << (16 * i);
      }
  }
  return v;
}

// LDS of a tile: rings of SA and SB slots, then slots of scales.
//
// F4: two slots of 8 bytes per row, a stage's.  They come through registers
// (a row of scales may lie on any even address), and the compiler waits for
// these loads as if the others were not there: so none is left in flight at a
// barrier, and deeper rings would be waited for in vain.
//
// CODES: eight slots of three dwords per row, the 8 bytes of a unit of four
// stages and what is before or behind them up to whole dwords, by direct loads:
// dword j of all rows lies at 256 TA j.
template <int TYPE, int KA, int KB, int TA, int TB, int LDS>
struct Ring {
  static constexpr uint32_t kA = Loads<KA, TA>::kSlot, kB = Loads<KB, TB>::kSlot;
  static constexpr uint32_t kScaleSlot = TYPE == F4 ? 512 * (TA + TB) : KA == CODES ? 768 * TA : 0;
  static constexpr int kScaleSlots = TYPE == F4 ? 2 : 8;
  static constexpr uint32_t kRoom = LDS - kScaleSlots * kScaleSlot;
  static constexpr int kBoth = (int)(kRoom / (kA + kB));
  // CODES: units of A, and stages of B ahead.  A unit's loads go out when the
  // products begin the one SA - 1 before it, and these may have a stage each:
  // no more stages of B than that may be in flight behind them.
  static constexpr int kUnits = kRoom >= 3 * kA + 4 * kB ? 3 : 2;
  static constexpr int kBeside = (int)((kRoom - kUnits * kA) / kB);
  static constexpr int SB = TYPE == F4 ? 2 : KA == CODES ? (kBeside > kUnits + 1 ? kUnits + 1 : kBeside)
                            : kBoth > 6 ? 6 : kBoth;
  static constexpr int SA = KA == CODES ? kUnits : TYPE != F4 && SB < 6 && (SB + 1) * kA + SB * kB <= kRoom ? SB + 1 : SB;
  static constexpr uint32_t kBBase = SA * kA, kScaleBase = kBBase + SB * kB;
  // (a tile of one stage has a slot of scales of its own, and the queue of
  // stream() holds the tile of the products and seven behind it)
  static_assert(SA <= 6 && SB <= 6, "stages ahead");
  static_assert(SB >= 2 && kScaleBase + kScaleSlots * kScaleSlot <= LDS, "LDS");
  // stages ahead of the products that anything is fetched for
  static constexpr int kAhead = TYPE == F4 ? 2 : (SA > SB ? SA : SB) - 1;
  // loads that may be in flight when a stage ends: those of the stages after
  // the next one (CODES: B's; a unit of A has as many stages to arrive)
  static constexpr int kPending = (KA == CODES ? 0 : SA - 2) * Loads<KA, TA>::kN + (SB - 2) * Loads<KB, TB>::kN;
  // quarters (of 16 between two barriers) that the loads are spread over: all
  // of a ring of two have to arrive within these (in MXFP4 over 2, 4, 8, 12 of
  // them 186, 183, 184, 189 us for 8192 rows, 16 experts of 6400 x 4096)
  static constexpr int kSpread = SB == 2 && SA == 2 ? 4 : 12;
  // A passes the caches by: weights, of tiles of up to 128 rows; in blocks of 128
  // columns, which hold no more rows and meet an expert's others as neighbours, of
  // 64.  In the gradient of W (both operands COLS) A is d_y, which all column tiles
  // of d_W read.  Us of that gradient, whose last column tile is a small one, past
  // the caches / through them: 8 experts, 4096 rows, 4096 x 4160 191 / 179, 4096 x
  // 1088 60.3 / 56.2; 16 experts, 8192 rows, 6400 x 1088 151 / 144, 6400 x 4160
  // 554 / 569; 60 experts, 5348 rows, 2048 x 2112 both 194.
  static constexpr bool kStream = KB != COLS && TB <= (TA == 2 ? 1 : 2);
};

// The accumulators of a wave: acc[i][j] is A tile i, B tile j of its own.
template <int TA, int TB> using Acc = f32x16[TA][TB];

// Scales of an operand in MXFP4 (null otherwise): row 0's, rows of `bytes`.
struct Scales {
  const uint8_t* at;
  int bytes;
};

// How the waves share a block's tile: 2 x 2; CODES of two tiles and more 4 x 1,
// so that each is converted once.
template <int KA, int TA>
struct Waves {
  static constexpr bool kLine = KA == CODES && TA > 1;
  static constexpr int kA(int ta) { return kLine ? ta / 2 : ta; }
  static constexpr int kB(int tb) { return kLine ? 2 * tb : tb; }
  static __device__ inline int a(int wave) { return kLine ? wave : wave >> 1; }
  static __device__ inline int b(int wave) { return kLine ? 0 : wave & 1; }
};

// The products of a sequence of tiles, one after another through the same
// rings: the loads of a tile's first stages are in flight while the products
// of the last one's end and its results are stored.  Job:
//   struct Tile          uniform, trivially copied
//   bool next(Tile&)     the tile after the last one given; false: none (again
//                        and again, once it was)
//   int steps(Tile)      reduction steps (F4: columns)
//   Operand a(Tile), b(Tile);  Scales a_scales(Tile), b_scales(Tile)
//   void store(Tile, Acc&)
template <int TYPE, int KA, int KB, int TA, int TB, int LDS, class Job>
__device__ __forceinline__ void stream(Job& job, lds_u8* lds) {
  using R = Ring<TYPE, KA, KB, TA, TB, LDS>;
  typedef typename Job::Tile Tile;
  constexpr bool kF4 = TYPE == F4, kCodes = KA == CODES;
  constexpr int kNA = Loads<KA, TA>::kN, kNB = Loads<KB, TB>::kN;
  const int l = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // the wave's place, and its tiles of 32
  typedef Waves<KA, TA> W;
  constexpr int NA = W::kA(TA), NB = W::kB(TB);
  const int wa = W::a(wave), wb = W::b(wave);
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;

  // The tiles to come: eight words each in the lanes of one register, tile i in
  // lanes 8 (i % 8) and up: its stages (0: behind the last tile; a tile without
  // reduction steps takes one stage of zeros), its steps, and what the job says.
  constexpr int kWords = sizeof(Tile) / 4;
  static_assert(kWords <= 6, "a tile's words");
  int queue = 0, made = 0;
  auto put = [&](int lane, int v) { queue = l == lane ? v : queue; };
  auto make = [&]() {
    Tile tile;
    const int at = 8 * (made++ & 7);
    int n = 0, steps = 0;  // (behind the last tile no load reads anything)
    if (job.next(tile)) {
      steps = job.steps(tile);
      n = max(1, kF4 ? (steps + 255) / 256 : (steps + kStage - 1) / kStage);
      int w[kWords];
      __builtin_memcpy(w, &tile, sizeof(Tile));
#pragma unroll
      for (int i = 0; i < kWords; ++i) put(at + 2 + i, w[i]);
    }
    put(at, n);
    put(at + 1, steps);
  };
  auto tile_of = [&](int i) {
    Tile tile;
    int w[kWords];
#pragma unroll
    for (int j = 0; j < kWords; ++j) w[j] = __builtin_amdgcn_readlane(queue, 8 * (i & 7) + 2 + j);
    __builtin_memcpy(&tile, w, sizeof(Tile));
    return tile;
  };
  // Where an operand's loads are: at stage k of n of tile i (n = 0: behind the
  // last), which takes `steps` reduction steps.
  struct Place {
    int i, k, n, steps;
  };
  auto begin = [&](int i) -> Place {
    return {i, 0, __builtin_amdgcn_readlane(queue, 8 * (i & 7)),
            __builtin_amdgcn_readlane(queue, 8 * (i & 7) + 1)};
  };
  // Moves on; true: to another tile (that is there), or behind the last.
  auto move = [&](Place& p) {
    if (++p.k < p.n) return false;
    p = begin(p.n ? p.i + 1 : p.i);
    return true;
  };
#pragma unroll 1
  for (int i = 0; i < R::kAhead + 2; ++i) make();
  Place pa = begin(0), pb = pa;
  if (pa.n == 0) return;
  int tile = 0, left = pa.n, k_now = 0;             // of the products: stages left, stage
  if (kCodes) pa.n = (pa.n + 3) >> 2;               // A's stages are units
  // (of all tiles the same where codes or scales are read)
  const int columns = pa.steps;

  Loads<KA, TA> la;
  Loads<KB, TB> lb;
  la.open(job.a(tile_of(0)), wave);
  lb.open(job.b(tile_of(0)), wave);
  la.bound(pa.steps);
  lb.bound(pb.steps);
  auto move_a = [&]() {
    const bool another = move(pa);
    if (kCodes && another) pa.n = (pa.n + 3) >> 2;
    if (another && pa.n) la.open(job.a(tile_of(pa.i)), wave);
    la.advance(another);
    la.bound(pa.steps - (kF4 || kCodes ? 256 : kStage) * pa.k);
  };
  auto move_b = [&]() {
    const bool another = move(pb);
    if (another && pb.n) lb.open(job.b(tile_of(pb.i)), wave);
    lb.advance(another);
    lb.bound(pb.steps - (kF4 ? 256 : kStage) * pb.k);
  };
  // In MXFP4 a row's last line may be partial: the chunks behind it are masked
  // (of either operand, whose loads are at the same stage).
  auto load_a = [&](int i, uint32_t slot) {
    const uint32_t mask =
        (kF4 || kCodes) && (uint32_t)(128 * pa.k) + la.chunk(wave) >= (uint32_t)columns / 2 ? kMasked : 0;
    la.template load<R::kStream>(i, lds0 + slot * R::kA + (wave + 4 * i) * 1024, mask);
  };
  auto load_b = [&](int i, uint32_t slot) {
    const uint32_t mask = kF4 && (uint32_t)(128 * pb.k) + la.chunk(wave) >= (uint32_t)columns / 2 ? kMasked : 0;
    lb.template load<false>(i, lds0 + R::kBBase + slot * R::kB + (wave + 4 * i) * 1024, mask);
  };

  // F4: scales of 256 columns (8 bytes) of the thread's row of A and of B, into
  // registers; a stage later to LDS, and not touched before: that would wait for
  // them.  A row's last 8 bytes are moved into place then; past the row: 2^0.
  const int t = threadIdx.x;
  const uint8_t *sa_row = nullptr, *sb_row = nullptr;
  uint64_t sa_next = 0, sb_next = 0;
  int past = 0;                                     // bits to move by
  Place ps = pa;
  auto open_scales = [&]() {
    if constexpr (kF4) {
      const Tile x = tile_of(ps.i);
      const Scales u = job.a_scales(x), w = job.b_scales(x);
      sa_row = u.at + (int64_t)min(t, min(64 * TA, job.a(x).valid) - 1) * u.bytes;
      sb_row = w.at + (int64_t)min(t, min(64 * TB, job.b(x).valid) - 1) * w.bytes;
    }
  };
  auto fetch_scales = [&]() {
    if constexpr (kF4) {
      // (behind the last stage: the last tile's first ones again)
      const int bytes = columns / 32;
      if (bytes < 8) {
        sa_next = scale_unit(sa_row, bytes, 0);
        sb_next = scale_unit(sb_row, bytes, 0);
      } else {
        const int at = min(8 * ps.k, bytes - 8);
        past = 8 * (8 * ps.k - at);
        typedef uint64_t __attribute__((aligned(2))) any_u64;
        sa_next = *global_ptr<any_u64>(sa_row + at);
        sb_next = *global_ptr<any_u64>(sb_row + at);
      }
    }
  };
  auto move_scales = [&]() {
    if constexpr (kF4) {
      if (move(ps) && ps.n) open_scales();
    }
  };
  auto put_scales = [&](uint32_t slot) {
    const uint32_t at = R::kScaleBase + slot * R::kScaleSlot;
    if constexpr (kF4) {
      const uint64_t fill = past ? 0x7F7F7F7F7F7F7F7Full << (64 - past) : 0;
      if (64 * TA >= kThreads || t < 64 * TA) lds_write(lds, at + 8 * t, sa_next >> past | fill);
      if (64 * TB >= kThreads || t < 64 * TB) lds_write(lds, at + 512 * TA + 8 * t, sb_next >> past | fill);
    }
  };
  // CODES: the scales of the unit where A's loads are.  An odd row
  // whose scales fill no whole dwords begins two bytes earlier.
  uint32_t unit = 0, unit_read = 0;                 // slots written next, read
  auto load_unit = [&]() {
    if constexpr (kCodes) {
      if (pa.n) {
        const Tile x = tile_of(pa.i);
        const Scales s = job.a_scales(x);
        const int valid = min(job.a(x).valid, 64 * TA);
        const uint8_t* base = uniform(s.at + 8 * pa.k);
        const uint32_t limit = valid * s.bytes - 8 * pa.k;
#pragma unroll
        for (int i = 0; i < 3 * TA / 4 + (TA % 4 != 0); ++i) {
          const int piece = wave + 4 * i;            // 64 rows of a dword
          const int j = piece / TA, r = piece % TA * 64 + l;
          const uint32_t off = r < valid && j < 3 ? r * s.bytes - (r * s.bytes & 2) + 4 * j : kMasked;
          if (piece < 3 * TA) load_lds4(lds0 + R::kScaleBase + unit * R::kScaleSlot + 256 * piece, base, limit, off);
        }
        unit = (unit + 1) & 7;
      }
    }
  };

  if constexpr (kF4) {
    open_scales();
    fetch_scales();
    put_scales(0);
    move_scales();
    fetch_scales();
  }
  // the rings' first stages; what the first stage needs comes first
#pragma unroll
  for (int v = 0; v < R::kAhead; ++v) {
    if (v < R::SB - 1) {
#pragma unroll
      for (int i = 0; i < kNB; ++i) load_b(i, v);
      move_b();
    }
    if (v < R::SA - 1) {
      load_unit();
#pragma unroll
      for (int i = 0; i < kNA; ++i) load_a(i, v);
      move_a();
    }
  }
  Acc<NA, NB> acc;

  // where the lane's fragments lie in a slot
  const int half = l >> 5, sw = (l >> 1) & 7;
  uint32_t cat[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) cat[s] = 16 * ((4 * half + s) ^ sw);
  const uint32_t arow = (uint32_t)(wa * NA * 32 + (l & 31)) * 128;
  const uint32_t brow = (uint32_t)(wb * NB * 32 + (l & 31)) * 128;
  // COLS: the lane's row within a step's four, and its 8 bytes of a tile
  const int cr = (l & 15) >> 2;
  auto col_at = [&](int T, int tile_) -> uint32_t {
    const int x = T % 2 ? cr >> 1 : cr;
    return (uint32_t)(32 * half + cr) * (128 * T) + 64 * (tile_ ^ x) + 32 * ((l >> 4) & 1) + 8 * (l & 3);
  };
  uint32_t acol[NA], bcol[NB];
#pragma unroll
  for (int i = 0; i < NA; ++i) acol[i] = KA == COLS ? col_at(TA, wa * NA + i) : 0;
#pragma unroll
  for (int j = 0; j < NB; ++j) bcol[j] = KB == COLS ? col_at(TB, wb * NB + j) : 0;

  u32x4 a[2][NA], b[2][NB], raw[kCodes ? NA : 1];
  float scale[kCodes ? NA : 1];
  uint32_t sa[kF4 ? NA : 1], sb[kF4 ? NB : 1], sa1[kF4 ? NA : 1], sb1[kF4 ? NB : 1];
  auto transposed = [&](uint32_t at, uint32_t four_rows) -> u32x4 {
    const auto x = reinterpret_cast<__attribute__((address_space(3))) s16x4*>(lds + at);
    const auto y = reinterpret_cast<__attribute__((address_space(3))) s16x4*>(lds + at + four_rows);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(x);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(y);
    const u32x2 u = __builtin_bit_cast(u32x2, lo), w = __builtin_bit_cast(u32x2, hi);
    return u32x4{u.x, u.y, w.x, w.y};
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
  // CODES: the lane's 32 codes of a stage and their scale, byte `at` of the
  // row's 12
  auto read_raw = [&](int i, uint32_t slot, int k) {
    if constexpr (kCodes) {
      raw[i] = lds_read<u32x4>(lds, slot * R::kA + arow + i * 4096 + 16 * ((2 * (k & 3) + half) ^ sw));
      const int at = 2 * (k & 3) + half + ((l & 1) & (columns >> 6)) * 2;
      scale[i] = scale_of(lds_read<uint8_t>(lds, R::kScaleBase + unit_read * R::kScaleSlot + (arow >> 5) + i * 128 +
                                                     (at >> 2) * 256 * TA + (at & 3)));
    }
  };
  auto read_scales = [&](uint32_t slot, uint32_t (&x)[kF4 ? NA : 1], uint32_t (&y)[kF4 ? NB : 1]) {
    if constexpr (kF4) {
      const uint32_t at = R::kScaleBase + slot * R::kScaleSlot + 4 * half;
#pragma unroll
      for (int i = 0; i < NA; ++i) x[i] = lds_read<uint32_t>(lds, at + (arow >> 4) + i * 256);
#pragma unroll
      for (int j = 0; j < NB; ++j) y[j] = lds_read<uint32_t>(lds, at + 512 * TA + (brow >> 4) + j * 256);
    }
  };
  // quarter c of the products of step s
  constexpr int kProducts = NA * NB;
  auto one = [&](auto sc, int m) {
    constexpr int s = decltype(sc)::value;
    const u32x4 x = a[s & 1][m % NA], y = b[s & 1][m / NA];
    f32x16& c = acc[m % NA][m / NA];
    if constexpr (TYPE == F16) {
      c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
    } else if constexpr (TYPE == BF16) {
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
    } else {
      const i32x8 u = {(int)x.x, (int)x.y, (int)x.z, (int)x.w, 0, 0, 0, 0};
      const i32x8 w = {(int)y.x, (int)y.y, (int)y.z, (int)y.w, 0, 0, 0, 0};
      c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(u, w, c, 4, 4, s, (int)sa[m % NA], s, (int)sb[m / NA]);
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
  uint32_t ac = 0, bc = 0, sc = 0;                  // slots of the products' stage
  uint32_t al = R::SA - 1, bl = R::SB - 1;          // slots loaded next
  // Quarter c's share (of 16) of the loads issued between two barriers: B's
  // first, whose ring is never the deeper one.
  constexpr int kAll = kNB + (kCodes ? 0 : kNA), kSpread = R::kSpread;
  auto loads = [&](int c) {
#pragma unroll
    for (int i = c * kAll / kSpread; i < min((c + 1) * kAll / kSpread, kAll); ++i) {
      if (i < kNB) load_b(i, bl);
      else load_a(i - kNB, al);
    }
  };
  constexpr std::integral_constant<int, 0> s0;
  constexpr std::integral_constant<int, 1> s1;
  constexpr std::integral_constant<int, 2> s2;
  constexpr std::integral_constant<int, 3> s3;
  auto step = [&](auto st) {
    constexpr int s = decltype(st)::value;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      loads(4 + 4 * s + c);
#pragma unroll
      for (int i = 0; i < NA; ++i)
        if (3 * i / NA == c) read_a(s + 1, i, ac);
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if (3 * j / NB == c) read_b(s + 1, j, bc);
      products(st, c);
      pin(c);
    }
  };

  stage_barrier<0>();
  read_scales(0, sa, sb);
#pragma unroll
  for (int i = 0; i < NA; ++i) {
    read_raw(i, 0, 0);
    read_a(0, i, 0);
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) read_b(0, j, 0);
  if constexpr (kF4) {
    put_scales(1);
    move_scales();
    fetch_scales();
  }
  // CODES: the unit SA - 1 units ahead, at once when the products begin one
  auto load_ahead = [&]() {
    load_unit();
#pragma unroll
    for (int i = 0; i < kNA; ++i) load_a(i, al);
  };
  if constexpr (kCodes) load_ahead();
#pragma unroll
  for (int c = 0; c < 4; ++c) loads(c);
  do {
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
    do {
      step(s0);
      step(s1);
      step(s2);
#ifdef __HIP_DEVICE_COMPILE__
      // (a use here: the compiler would move the products behind the branches
      // below, away from their operands' reads)
      if constexpr (kF4) {
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            if constexpr (TA == 4) asm volatile("" :: "a"(acc[i][j][0]));
            else asm volatile("" :: "v"(acc[i][j][0]));
          }
      }
#endif
      // every load of the next stage has arrived; this stage's slots are free
      stage_barrier<R::kPending>();
      bc = next(bc, R::SB);
      bl = next(bl, R::SB);
      sc ^= 1;
      k_now = left > 1 ? k_now + 1 : 0;             // (of the next stage)
      move_b();
      if (!kCodes || (k_now & 3) == 0) {
        ac = next(ac, R::SA);
        al = next(al, R::SA);
        unit_read = (unit_read + 1) & 7;
        move_a();
        if (kCodes) load_ahead();
      }
      if constexpr (kF4) {
        // scales of the stage after the next into LDS, whose slot the barrier
        // freed, those of the one behind it into registers
        put_scales(sc ^ 1);
        move_scales();
        fetch_scales();
      }
      read_scales(sc, sa1, sb1);
      // (after the last stage of all: reads that are not multiplied)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        loads(c);
        if (c == 0) {
#pragma unroll
          for (int i = 0; i < NA; ++i) read_raw(i, ac, k_now);
        }
#pragma unroll
        for (int i = 0; i < NA; ++i)
          if (kCodes ? 1 + i * 3 / NA == c : 3 * i / NA == c) read_a(0, i, ac);
#pragma unroll
        for (int j = 0; j < NB; ++j)
          if (3 * j / NB == c) read_b(0, j, bc);
        products(s3, c);
        pin(c);
      }
      if constexpr (kF4) {
#pragma unroll
        for (int i = 0; i < NA; ++i) sa[i] = sa1[i];
#pragma unroll
        for (int j = 0; j < NB; ++j) sb[j] = sb1[j];
      }
    } while (--left);
    job.store(tile_of(tile), acc);
    // the next tile; what is read ahead of it has one more to go to
    const Place now = begin(++tile);
    left = now.n;
    while (made <= tile + R::kAhead + 1) make();
  } while (left);
  // the LDS must not be handed on with loads in flight, nor while another wave
  // reads it
  stage_barrier<0>();
}

// A tile stays in the accumulation registers until it is stored: all of them
// copied at once would not fit the others.  (The host's pass knows no such
// registers.)
template <int TILES>
__device__ inline void keep(f32x16& c) {
#ifdef __HIP_DEVICE_COMPILE__
  if constexpr (TILES >= 8) asm volatile("" : "+a"(c));
#endif
}

// Stores a wave's tiles as 16-bit rows: C's b is the row, a the column, whose
// eight values go out as 16 bytes (the lane halves trade four each).  The fp32
// sums are rounded here, once, to the type of the output.
template <class T, class W, int TA, int TB>
__device__ __forceinline__ void store_rows(Acc<TA, TB>& acc, T* out, int64_t ld, int rows, int cols) {
  typedef T x2 __attribute__((ext_vector_type(2)));
  const int l = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int a0 = W::a(wave) * TA * 32, b0 = W::b(wave) * TB * 32;
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    const int row = b0 + 32 * j + (l & 31);
    T* to = out + (int64_t)row * ld + a0 + 8 * (l >> 5);
#pragma unroll
    for (int i = 0; i < TA; ++i) {
      if (a0 + 32 * i >= cols) continue;
      keep<TA * TB>(acc[i][j]);
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
          *global_ptr<u32x4>(to + 32 * i + 16 * q) =
              u32x4{(uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1]};
      }
    }
  }
}

}  // namespace tile
}  // namespace moe
