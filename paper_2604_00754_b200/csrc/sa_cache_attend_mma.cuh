// Attention over the 4-bit cache on the tensor cores.  Tiles are made for 64, 128 or 256 dimensions; other head
// dimensions (multiples of 16) take the next of these (kPad): their rows are copied in 8-byte pieces, what lies
// behind a row has scale 0, and Q is 0 there.
//
// Bound by the cache's bytes (4.5 bits a value, each read once per tile of query rows), so everything
// between HBM and the multiply has to keep up with 23 bytes = 41 values per clock and SM.  A warp takes 16
// keys of each step alone, from its copies to its own running maximum, sum and rows: no barrier stands
// in the loop, the four warps of a CTA join once per segment.
// 32 sequences of 32768 keys, 32/8 heads of 128 (1.21 GB): 255-275 us, 68-73 % of the copy bandwidth, where the power cap
// holds the clock near 1755 MHz; 236 (79 %) in the first calls of a burst.  What holds it back is the work itself: per warp and 16 keys of 128 dimensions 64
// conversions, 64 products with scales, 16 matrix instructions and 160 others, the ALU half busy, three warps per
// scheduler.
//   - Copies: cp.async into a ring of the warp's own (pages are contiguous per head and side: 16-byte pieces).
//   - Scores as S^T = K Q^T: the keys are the 16 rows of mma.m16n8k16, eight query rows its columns, so that
//     a group of 8 heads or fewer wastes no row of K.  A lane's codes become fp16 by the hardware
//     conversion (two values an instruction) times their scale: exact, K never rounds.  tcgen05 would need the
//     dequantised tile in shared memory, 2 bytes a value written and read again: 164 bytes per clock and SM of
//     the 128 that shared memory gives; registers feed mma.sync directly.
//   - Sums as O^T += V^T P^T: S^T's accumulator transposed by movmatrix is the B operand, and O^T has the
//     heads in the columns that S^T has them in, so a rescaling is a product in place.  V^T's rows are dimensions and
//     its pairs are two keys: nibbles of two keys are interleaved as words, then converted.
//   - The order of dimensions within a product is free: lane c of a quad takes the c-th quarter of a key's
//     codes (one wide load), and Q's fragments are built to match.
// Rounding.  Q is scaled per row by a power of two into fp16: exact for bf16 (8 bits) wherever it is within
// 2^-31 of the row's largest; fp32 goes as two fp16 terms (22 bits and a remainder below 2^-24).  P is taken
// relative to a reference that keeps it between 2^12 and 2^15.75 at its largest (small ones stay normal in
// fp16, and the reference seldom moves); it is rounded once to 11 bits in bf16 calls, below the rounding of
// y, and goes as two terms in fp32 calls.  All sums are fp32; the matrix instruction cuts its own off, so fp32 calls
// add 16 dimensions of a score and 16 keys of a row in the instruction and the rest by rounded additions.
#pragma once

#include <type_traits>

#include "sa_cache_attend.cuh"

namespace sa {
namespace attend {

constexpr float kAim = 12.f, kMost = 15.75f;   // log2 of the largest P where the reference is set, and may be
constexpr float kNone = -3.4028235e38f;        // reference before the first key: any score is more
constexpr float kLarge = 16777216.f;           // 2^24: the rounding of a reference is 1/2 at most below it

template <int D>
struct Tile {                    // a warp's 16 keys
  static constexpr int kCodes = 8 * D, kScales = D, kBytes = 2 * (kCodes + kScales);
};

// Byte of 16-byte piece `piece` of a key's codes within a side's tile.  The pieces are permuted so that
// neither the reads of K (keys r / 2 and r / 2 + 4 with all pieces) nor those of V (four keys in a row, two
// pieces) meet in a bank.
template <int D>
__device__ __forceinline__ int tile_at(int key, int piece) {
  if (D == 64) return (key >> 2) * 128 + ((((key & 3) * 2 + piece) ^ ((key & 4))) * 16);
  if (D == 128) return (key >> 1) * 128 + ((((key & 1) * 4 + piece) ^ (key & 2) ^ (key & 4)) * 16);
  return key * 128 + ((piece ^ (2 * (key & 3)) ^ ((key >> 2) & 1)) * 16);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __half2 r = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&r);
}
// What fp16 leaves of a pair, as fp16.
__device__ __forceinline__ uint32_t rest2(float lo, float hi, uint32_t of) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&of));
  return pack2(lo - f.x, hi - f.y);
}
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const uint8_t* p) {
  if (N == 1) w[0] = *reinterpret_cast<const uint32_t*>(p);
  if (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x;
    w[N - 1] = v.y;
  }
  if (N == 4) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x;
    w[1 % N] = v.y;
    w[2 % N] = v.z;
    w[3 % N] = v.w;
  }
}

// NT tiles of eight query rows; PC fp16 terms for Q and P (1: bf16 calls, 2: fp32 calls).
template <typename T, int D, int NT, bool kPad>
struct Shape {
  static constexpr int PC = sizeof(T) == 2 ? 1 : 2;
  static constexpr int kRows = 8 * NT;
  static constexpr int kKs = D / 16;                       // 16-deep steps of the scores, tiles of the sums
  static constexpr bool kQInRegs = kKs * 2 * NT * PC <= (NT == 1 && D < 256 ? 32 : 16);   // else in shared memory
  // Units a warp takes at once (one look at the maximum, one turn of the loop), as far as registers reach,
  // and turns in its ring.
  static constexpr int kUnits = D < 256 && NT == 1 ? 2 : 1;
  static constexpr int kTurns = kUnits == 2 ? (D == 64 ? 3 : 2) : D == 64 ? 6 : D == 128 ? 4 : 3;
  static constexpr int kRing = kTurns * kUnits * Tile<D>::kBytes;
  // CTAs per SM: what registers (rows of O, Q, the tile in flight) and shared memory leave.  With 64 registers of O
  // two CTAs are as good as three in one tile of rows or better (16 x 8192 keys, 16/4 heads of 256: bf16 43.5 us
  // against 43.2, fp32 57.0 against 59.6) and as good in four (32 fp32 rows over 9 x 2500 keys of 16 heads of 64:
  // 47.5 against 47.4), not in two (four tokens over 16 x 8192 keys, 32/8 heads of 128: 67.1 against 64.2).  Some fp32
  // instances spill at that: one tile of 128 dimensions 56 bytes of a thread at three CTAs, which beat two without
  // spills (16 x 8192 keys, 32/8 heads: 54.3 against 56.7); two tiles of 256 dimensions 116, of 64 dimensions 56.
  static constexpr int kORegs = kKs * 4 * NT;
  static constexpr int kCtas = kORegs + (kQInRegs ? kKs * 2 * NT * PC : 0) <= 40 ? 4
                               : kORegs < 64 || (kORegs == 64 && NT == 2) ? 3 : 2;
  static constexpr int kQBytes = kQInRegs ? 0 : kKs * NT * PC * 32 * 8;
  static constexpr int kOPitch = D + 4;
  static constexpr int kOs = NT == 1 && D <= 128 ? kWarps : 1;   // a warp's rows side by side, or one after the other
  static constexpr int kOffQ = kWarps * kRing;
  static constexpr int kOffO = kOffQ + kQBytes;            // [kOs][kRows][kOPitch] fp32
  static constexpr int kOffMl = kOffO + kOs * kRows * kOPitch * 4;   // [kWarps][2][kRows] fp32
  static constexpr int kOffPlaces = kOffMl + kWarps * 2 * kRows * 4;  // [kWarps][64] uint2
  static constexpr int kOffPieces = kOffPlaces + kWarps * 64 * 8;     // kPad: [D] uint16
  static constexpr int kSmem = kOffPieces + (kPad ? D * 2 : 0);
};

template <typename T, int D, int NT, bool kPad>
__global__ void __launch_bounds__(32 * kWarps, Shape<T, D, NT, kPad>::kCtas) attend_mma_kernel(const Params p) {
  using S = Shape<T, D, NT, kPad>;
  constexpr int PC = S::PC, kRows = S::kRows, kKs = S::kKs, U = S::kUnits, kTurns = S::kTurns;
  extern __shared__ __align__(128) uint8_t smem[];
  const AttendArgs& a = p.a;
  const CacheView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int lr = lane >> 2, lc = lane & 3;                 // row and column of a lane in mma fragments
  const int key_k = (lr >> 1) + 4 * (lr & 1);              // key of this lane's row of S^T; the second is 8 on
  uint8_t* ring = smem + warp * S::kRing;
  const uint32_t ring_u32 = (uint32_t)__cvta_generic_to_shared(ring);
  uint2* q_s = reinterpret_cast<uint2*>(smem + S::kOffQ);
  float* o_s = reinterpret_cast<float*>(smem + S::kOffO);
  float* ml_s = reinterpret_cast<float*>(smem + S::kOffMl);
  uint2* places = reinterpret_cast<uint2*>(smem + S::kOffPlaces) + warp * 64;
  const int d = kPad ? c.d : D, groups = d / 16;
  uint16_t* pieces = reinterpret_cast<uint16_t*>(smem + S::kOffPieces);   // where an 8-byte piece of a unit goes
  if (kPad) {
    for (int x = tid; x < d; x += 32 * kWarps) {
      const int key = x / groups, y = x - key * groups;
      pieces[x] = (uint16_t)(tile_at<D>(key, y >> 1) + (y & 1) * 8);
    }
    __syncthreads();
  }
  const uint32_t page_128 = (uint32_t)(c.page_bytes / 128);   // without kPad a page is a multiple of 1152 bytes from d = 64 on

  // where this lane reads in a unit's tile: K's rows key_k (8 on: 4 D bytes on), V's keys lc and lc + 4
  const int at_k = D == 64 ? tile_at<D>(key_k, lc >> 1) + (lc & 1) * 8 : tile_at<D>(key_k, lc * (D / 128));
  const int at_k1 = at_k ^ 16;             // the next piece (D = 256)
  const int at_ks = 2 * Tile<D>::kCodes + key_k * groups + lc * (D / 64);
  const int v_piece = D == 64 ? lr >> 2 : D == 128 ? lr >> 1 : lr, v_byte = D == 64 ? (lr & 3) * 4 : D == 128 ? (lr & 1) * 8 : 0;
  const int at_v = Tile<D>::kCodes + tile_at<D>(lc, v_piece) + v_byte;
  const int at_v4 = Tile<D>::kCodes + tile_at<D>(lc + 4, v_piece) + v_byte;
  const int at_vs = 2 * Tile<D>::kCodes + Tile<D>::kScales + lc * groups + (D == 64 ? lr >> 1 : lr * (D / 128));

  grid_dependency_wait();
  grid_dependents_launch();
  int e;
  int64_t before;
  const Line line = find(p, &e, &before);
  Walk w;
  if (!start(p, line, e, before, &w)) return file_nothing(p);
  Entry& en = w.en;
  bool begins = false;
  // the portion at hand: this warp's first unit (the next is kStep on), how many, in how many turns
  int unit0, units, turns, full_hi;
  int64_t full_lo;
  uint2 ahead;
  const uint8_t *src_k, *src_v, *src_s;
  uint32_t there, slot;      // units of the last kTurns - 1 turns, the oldest on top; ring slot of the next turn
  const uint32_t dst_lane = ring_u32 + tile_at<D>(lane / (D / 32), lane % (D / 32));
  const uint32_t dst_s = ring_u32 + 2 * Tile<D>::kCodes + lane * 16;

  // places of units (K's codes in 128 bytes, K's scales in 64 bytes from the head's start of the pool; kPad: page
  // and row of it; all ones: none)
  auto fetch_place = [&](int i) -> uint2 {
    const int64_t key = (int64_t)unit0 + (int64_t)i * kStep;
    if (i >= units || key >= en.hi || key + kUnit <= en.lo) return make_uint2(~0u, ~0u);
    const uint32_t pg = c.table[(int64_t)en.slot * c.row + (key >> c.p_shift)];
    if (pg < (uint32_t)c.pages) {
      const uint32_t row = (uint32_t)key & (c.P - 1), at = pg * page_128;
      if (kPad) return make_uint2(pg, row);
      return make_uint2(at + row * (D / 2) / 128, 2 * at + row * (D / 16) / 64);
    }
    report_cache(c);
    return make_uint2(~0u, ~0u);
  };
  auto issue = [&](int turn, uint32_t to_slot) -> uint32_t {      // bits: units that are there
    uint32_t found = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = turn * U + u;
      const uint2 at = places[i & 63];
      if (i < units && at.x != ~0u) {
        found |= 1u << u;
        const uint32_t to = to_slot + u * Tile<D>::kBytes;
        if (kPad) {
          const uint8_t* k = src_k + (uint64_t)at.x * (uint32_t)c.page_bytes + at.y * (d / 2);
          for (int x = lane; x < d; x += 32) {
            copy8(ring_u32 + to + pieces[x], k + x * 8);
            copy8(ring_u32 + to + Tile<D>::kCodes + pieces[x], k + c.side + x * 8);
          }
          const uint8_t* s = src_s + (uint64_t)at.x * (uint32_t)c.page_bytes + at.y * groups;
          if (lane < groups) copy16(dst_s + to, s);
          else if (lane < 2 * groups) copy16(dst_s + to + Tile<D>::kScales - d, s + c.side - d);
          continue;
        }
        const uint8_t *k = src_k + (uint64_t)at.x * 128, *v = src_v + (uint64_t)at.x * 128;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {   // 32 pieces are 1024 / D keys: a multiple of 4, of 8 up to D = 128
          const uint32_t x = D == 256 && (j & 1) ? (dst_lane ^ 16u) : dst_lane;
          copy16(x + to + j * 512, k + j * 512);
          copy16(x + to + Tile<D>::kCodes + j * 512, v + j * 512);
        }
        if (lane < D / 8) copy16(dst_s + to, src_s + (uint64_t)at.y * 64);
      }
    }
    copies_end();
    return found;
  };
  // takes the next portion and starts its first copies; the warp has read what its ring held
  auto open = [&]() -> bool {
    if (!next(p, &w)) return false;
    unit0 = (en.first + w.k0) * kStep + warp * kUnit;
    units = w.k1 - w.k0;
    turns = (units + U - 1) / U;
    // keys below full_hi and from full_lo on are seen by every row
    full_hi = a.causal ? min(en.len + en.t0 + 1, en.hi) : en.hi;   // (lengths and T are below 2^30)
    full_lo = a.w > 0 ? (int64_t)en.len + en.t1 - a.w + 1 : 0;
    // rows of Q on their way while the places are looked up
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      if (8 * nt + lr < en.rows && (!kPad || lc * (D / 4) < d))
        asm volatile("prefetch.global.L1 [%0];" ::"l"(row_of(p, reinterpret_cast<const T*>(a.q), a.qs, en, w.h, 8 * nt + lr) +
                                                     lc * (D / 4)));
    // this lane's 16-byte pieces of a unit: D / 64 of K's codes and of V's, 512 bytes apart, and one of scales
    const uint8_t* head = c.pool + (int64_t)2 * w.h * c.side;
    src_k = head + (kPad ? 0 : lane * 16);
    src_v = src_k + c.side;
    src_s = head + c.P * (d / 2) + (kPad || lane < D / 16 ? 0 : c.side - D) + lane * 16;
    // places of units 0 .. 31 into the warp's list, of 32 .. 63 on the way
    __syncwarp();
    places[lane] = fetch_place(lane);
    ahead = fetch_place(32 + lane);
    __syncwarp();
    there = slot = 0;
#pragma unroll
    for (int i = 0; i < kTurns - 1; ++i) there = there << U | issue(i, i * U * Tile<D>::kBytes);
    return true;
  };

  bool more = open();
  while (more) {
    bool plain = true;        // no score of these rows can pass kLarge
    // Q of this lane's fragments: row 8 nt + lr, the lc-th quarter of its dimensions
    uint32_t qf[S::kQInRegs ? NT : 1][PC][S::kQInRegs ? kKs : 1][2];
    float factor[NT][2];      // log2 units per unit of a score, of the two columns 2 lc, 2 lc + 1
    if (!S::kQInRegs) __syncthreads();   // the last segment's readers are done
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = 8 * nt + lr;
      float x[D / 4];
      const T* q = row_of(p, reinterpret_cast<const T*>(a.q), a.qs, en, w.h, r < en.rows ? r : 0) + lc * (D / 4);
      if (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const bool there = !kPad || lc * (D / 4) + 8 * i < d;
          const uint4 v = there ? reinterpret_cast<const uint4*>(q)[i] : make_uint4(0, 0, 0, 0);
          const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            x[8 * i + 2 * z] = __uint_as_float(u[z] << 16);
            x[8 * i + 2 * z + 1] = __uint_as_float(u[z] & 0xffff0000u);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const bool there = !kPad || lc * (D / 4) + 4 * i < d;
          const float4 v = there ? reinterpret_cast<const float4*>(q)[i] : make_float4(0.f, 0.f, 0.f, 0.f);
          x[4 * i] = v.x;
          x[4 * i + 1] = v.y;
          x[4 * i + 2] = v.z;
          x[4 * i + 3] = v.w;
        }
      }
      uint32_t top = 0;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < D / 4; ++i) {
        top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
        sum += fabsf(x[i]);
      }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      plain &= sum * p.scale2 <= kLarge / 2688.f;      // 2688: the largest code times the largest scale
      // the row's largest becomes 2^14 .. 2^15; rows with an infinity or NaN, and zero ones, stay
      const int ex = (int)(top >> 23) - 127;
      const int up = ex == 128 || ex == -127 ? 0 : min(14 - ex, 126);
      const float by = __uint_as_float((uint32_t)(127 + up) << 23);
      // not 0: a hidden score of -infinity stays one
      const float back = fmaxf(p.scale2 * __uint_as_float((uint32_t)(127 - up) << 23), 1.2e-38f);
      factor[nt][0] = __shfl_sync(0xffffffffu, back, 8 * lc);
      factor[nt][1] = __shfl_sync(0xffffffffu, back, 8 * lc + 4);
#pragma unroll
      for (int ks = 0; ks < kKs; ++ks) {
        uint32_t f[PC][2];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const float lo = x[4 * ks + 2 * z] * by, hi = x[4 * ks + 2 * z + 1] * by;
          f[0][z] = pack2(lo, hi);
          if (PC == 2) f[PC - 1][z] = rest2(lo, hi, f[0][z]);
        }
#pragma unroll
        for (int w = 0; w < PC; ++w) {
          if (S::kQInRegs) {
            qf[nt % (S::kQInRegs ? NT : 1)][w][ks % (S::kQInRegs ? kKs : 1)][0] = f[w][0];
            qf[nt % (S::kQInRegs ? NT : 1)][w][ks % (S::kQInRegs ? kKs : 1)][1] = f[w][1];
          } else if (warp == nt % kWarps) {
            q_s[((nt * PC + w) * kKs + ks) * 32 + lane] = make_uint2(f[w][0], f[w][1]);
          }
        }
      }
    }
    if (!S::kQInRegs) __syncthreads();

    plain = __all_sync(0xffffffffu, plain);
    float m[NT][2], l[NT][2], o[kKs][NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        m[nt][x] = kNone;
        l[nt][x] = 0.f;
      }
#pragma unroll
    for (int i = 0; i < kKs; ++i)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) o[i][nt][0] = o[i][nt][1] = o[i][nt][2] = o[i][nt][3] = 0.f;

    for (int turn = 0; turn < turns; ++turn) {
      __syncwarp();            // every lane has read the slot that the next copy fills
      if ((turn & (32 / U - 1)) == 0) {
        places[(turn * U + 32 + lane) & 63] = ahead;
        ahead = fetch_place(turn * U + 64 + lane);
        __syncwarp();
      }
      const uint32_t next = slot == 0 ? (kTurns - 1) * U * Tile<D>::kBytes : slot - U * Tile<D>::kBytes;
      there = there << U | issue(turn + kTurns - 1, next);
      copies_wait<kTurns - 1>();
      __syncwarp();
      const uint8_t* tiles = ring + slot;
      slot = slot == (kTurns - 1) * U * Tile<D>::kBytes ? 0 : slot + U * Tile<D>::kBytes;
      const uint32_t here = there >> (U * (kTurns - 1)) & ((1u << U) - 1u);
      if (here == 0) continue;
      const int unit = unit0 + turn * (U * kStep);
      const bool full = plain && here == (1u << U) - 1u && unit >= full_lo && unit + (U - 1) * kStep + kUnit <= full_hi;
      // two copies of the code: where every row sees every key, no branch stands between what can overlap
      auto take = [&](auto seen_by_all) {
        constexpr bool kFull = decltype(seen_by_all)::value;
        // scores of keys key_k, key_k + 8 (rows) and query rows 2 lc, 2 lc + 1 of each tile (columns)
        float x[U][NT][4];
#pragma unroll
        for (int un = 0; un < U; ++un) {
          const uint8_t* tile = tiles + un * Tile<D>::kBytes;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) x[un][nt][0] = x[un][nt][1] = x[un][nt][2] = x[un][nt][3] = 0.f;
          constexpr int kWords = D / 32, kLoad = kWords < 4 ? kWords : 4;   // a lane's quarter of a key
          uint32_t w[2][kWords], sc[2][D == 256 ? 2 : 1];
#pragma unroll
          for (int z = 0; z < 2; ++z) {          // 8 keys on is 4 D bytes on, and the pieces lie alike
#pragma unroll
            for (int u = 0; u < kWords / kLoad; ++u) {
              uint32_t v[kLoad];
              load_words(v, tile + (u ? at_k1 : at_k) + z * 4 * D);
#pragma unroll
              for (int y = 0; y < kLoad; ++y) w[z][u * kLoad + y] = v[y];
            }
            const uint8_t* ks = tile + at_ks + z * 8 * groups;
            if (kPad) {
              uint32_t four = 0;               // the scales of this lane's quarter, 0 behind the row
#pragma unroll
              for (int g = 0; g < D / 64; ++g)
                if (lc * (D / 64) + g < groups) four |= (uint32_t)ks[g] << (8 * g);
              sc[z][0] = scales_to_half2(D == 64 ? four * 0x101u : four);
              if (D == 256) sc[z][D == 256 ? 1 : 0] = scales_to_half2(four >> 16);
            } else if (D == 64) {
              sc[z][0] = scales_to_half2(*ks * 0x101u);
            } else if (D == 128) {
              sc[z][0] = scales_to_half2(*reinterpret_cast<const uint16_t*>(ks));
            } else {
              const uint32_t four = *reinterpret_cast<const uint32_t*>(ks);
              sc[z][0] = scales_to_half2(four);
              sc[z][D == 256 ? 1 : 0] = scales_to_half2(four >> 16);
            }
          }
#pragma unroll
          for (int u = 0; u < kWords; ++u) {      // eight dimensions of this lane: two 16-deep steps
            uint32_t v[2][4];
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              codes_to_half2(w[z][u], v[z]);
              const int g = u / 2;                // its group of 16
              const uint32_t two = D == 64 ? sc[z][0] : __byte_perm(sc[z][D == 256 ? g / 2 : 0], 0, g & 1 ? 0x3232 : 0x1010);
#pragma unroll
              for (int y = 0; y < 4; ++y) v[z][y] = mul2(v[z][y], two);
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const uint32_t fa[4] = {v[0][2 * y], v[1][2 * y], v[0][2 * y + 1], v[1][2 * y + 1]};
              const int ks = 2 * u + y;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                // the tensor core cuts its sums off: 32 of them in one accumulator (256 dimensions, two terms) took up to
                // 1.1e-6 of an fp32 score, always towards 0; so each 16 dimensions have their own, and are added rounded
                float t[4] = {0.f, 0.f, 0.f, 0.f};
                float(&sum)[4] = PC == 1 ? x[un][nt] : t;
#pragma unroll
                for (int z = PC - 1; z >= 0; --z) {
                  if (S::kQInRegs) {
                    const auto& f = qf[nt % (S::kQInRegs ? NT : 1)][z][ks % (S::kQInRegs ? kKs : 1)];
                    mma(sum, fa, f[0], f[1]);
                  } else {
                    const uint2 f = q_s[((nt * PC + z) * kKs + ks) * 32 + lane];
                    mma(sum, fa, f.x, f.y);
                  }
                }
                if (PC == 2) {
#pragma unroll
                  for (int k = 0; k < 4; ++k) x[un][nt][k] += t[k];
                }
              }
            }
          }
        }
        // bit: key of the unit that some row sees; what the others have is whatever the page holds
        uint32_t shown[U];
#pragma unroll
        for (int un = 0; un < U; ++un) shown[un] = 0xffffu;
        if (!kFull) {
#pragma unroll
          for (int un = 0; un < U; ++un) {
            const int first = unit + un * kStep;
            const int below = min(max(en.lo - first, 0), kUnit), above = min(max(en.hi - first, 0), kUnit);
            shown[un] = here >> un & 1 ? (1u << above) - (1u << min(below, above)) : 0u;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const int r = 8 * nt + 2 * lc + (y & 1), key = key_k + (y & 2 ? 8 : 0);
                const int pos = en.len + (en.r0 + r) / p.G, j = first + key;
                const bool sees = (shown[un] >> key & 1) && (!a.causal || j <= pos) && (a.w <= 0 || pos - j < a.w);
                if (!sees) x[un][nt][y] = -INFINITY;
              }
          }
        }
        // Exponents relative to the reference m; lanes look at each other only where one has too much.  A score's
        // product and the difference are one rounding, which needs a reference whose own rounding is small; the
        // copy for masked tiles, which also takes rows that may have larger ones, rounds their products as the
        // reference was.
        auto exponent = [&](float score, int nt, int y) {
          if (!kFull && fabsf(m[nt][y]) > kLarge) return __fmul_rn(score, factor[nt][y]) - m[nt][y];
          return fmaf(score, factor[nt][y], -m[nt][y]);
        };
        auto top_of = [&](int nt, int y) {
          float top = -INFINITY;
#pragma unroll
          for (int un = 0; un < U; ++un) top = fmaxf(top, fmaxf(x[un][nt][y], x[un][nt][y + 2]));
          return top;
        };
        bool high = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int y = 0; y < 2; ++y) high |= exponent(top_of(nt, y), nt, y) > kMost;
        if (__any_sync(0xffffffffu, high)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              float top = top_of(nt, y);
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
              float to = fmaf(top, factor[nt][y], -kAim);
              if (!kFull) {
                const float score = __fmul_rn(top, factor[nt][y]);
                if (fabsf(score) > kLarge) to = score - (score - kAim) > kMost ? score : score - kAim;   // 12 may be less than a unit
              }
              to = fmaxf(m[nt][y], to);
              const float keep = exp2f(m[nt][y] - to);
              m[nt][y] = to;
              l[nt][y] *= keep;
#pragma unroll
              for (int z = 0; z < kKs; ++z) {
                o[z][nt][y] *= keep;
                o[z][nt][y + 2] *= keep;
              }
            }
        }
#pragma unroll
        for (int un = 0; un < U; ++un) {
          const uint8_t* tile = tiles + un * Tile<D>::kBytes;
          uint32_t pf[NT][PC][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const float p0 = exp2f(exponent(x[un][nt][0], nt, 0)), p1 = exp2f(exponent(x[un][nt][1], nt, 1));
            const float p2 = exp2f(exponent(x[un][nt][2], nt, 0)), p3 = exp2f(exponent(x[un][nt][3], nt, 1));
            l[nt][0] += p0 + p2;
            l[nt][1] += p1 + p3;
            const uint32_t top = pack2(p0, p1), low = pack2(p2, p3);
            pf[nt][0][0] = transpose8(top);
            pf[nt][0][1] = transpose8(low);
            if (PC == 2) {
              pf[nt][PC - 1][0] = transpose8(rest2(p0, p1, top));
              pf[nt][PC - 1][1] = transpose8(rest2(p2, p3, low));
            }
          }
          // sums: keys lc, lc + 4, lc + 8, lc + 12 and the lr-th eighth of the dimensions
          constexpr int kWords = D / 64;
          uint32_t w[4][kWords], sv[4];           // words of a key; its scales, one byte or (D = 256) two
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            load_words(w[z], tile + (z & 1 ? at_v4 : at_v) + (z / 2) * 4 * D);
            const uint8_t* vs = tile + at_vs + z * 4 * groups;
            if (kPad) {
              const int g = D == 64 ? lr >> 1 : lr * (D / 128);
              sv[z] = g < groups ? vs[0] : 0u;
              if (D == 256 && g + 1 < groups) sv[z] |= (uint32_t)vs[1] << 8;
            } else {
              sv[z] = D == 256 ? *reinterpret_cast<const uint16_t*>(vs) : *vs;
            }
          }
          uint32_t poisoned[D == 256 ? 2 : 1] = {};     // bit: key whose values of this lane's group are NaN
          if (!kFull) {
            bool nan = false;
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              if (!(shown[un] >> (lc + 4 * z) & 1)) sv[z] = 0;
              nan |= (sv[z] & 0x7f) == 0x7f || (sv[z] & 0x7f00) == 0x7f00;
            }
            if (__any_sync(0xffffffffu, nan)) {
              // 0 times NaN would reach the rows that do not see the key: taken out here, put in below
#pragma unroll
              for (int z = 0; z < 4; ++z)
#pragma unroll
                for (int g = 0; g < (D == 256 ? 2 : 1); ++g) {
                  const bool bad = (sv[z] >> (8 * g) & 0x7f) == 0x7f;
                  poisoned[g] |= (__ballot_sync(0xffffffffu, bad) >> (4 * lr) & 15u) << (4 * z);
                  if (bad) sv[z] &= ~(0xffu << (8 * g));
                }
            }
          }
#pragma unroll
          for (int u = 0; u < kWords; ++u) {
            const int g = D == 256 ? u / 2 : 0;
            uint32_t v[2][2][4];                  // [dimension even, odd][keys lower, upper half][pair of rows]
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const uint32_t a0 = w[2 * z][u], a1 = w[2 * z + 1][u];
              const uint32_t even = (a0 & 0x0f0f0f0fu) | ((a1 << 4) & 0xf0f0f0f0u);
              const uint32_t odd = ((a0 >> 4) & 0x0f0f0f0fu) | (a1 & 0xf0f0f0f0u);
              const uint32_t two = scales_to_half2(__byte_perm(sv[2 * z], sv[2 * z + 1], g ? 0x0051 : 0x0040));
              codes_to_half2(even, v[0][z]);
              codes_to_half2(odd, v[1][z]);
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                v[0][z][y] = mul2(v[0][z][y], two);
                v[1][z][y] = mul2(v[1][z][y], two);
              }
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const uint32_t fa[4] = {v[0][0][y], v[1][0][y], v[0][1][y], v[1][1][y]};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                float(&sum)[4] = o[4 * u + y][nt];
                if (PC == 1) {
                  mma(sum, fa, pf[nt][0][0], pf[nt][0][1]);
                } else {
                  // as the scores: over a unit the cut is nothing, over thousands of keys in one accumulator it was
                  // 3e-6 of an fp32 result; the running sum is rounded
                  float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                  for (int z = PC - 1; z >= 0; --z) mma(t, fa, pf[nt][z][0], pf[nt][z][1]);
#pragma unroll
                  for (int k = 0; k < 4; ++k) sum[k] += t[k];
                }
              }
            }
          }
          if (!kFull) {
#pragma unroll
            for (int g = 0; g < (D == 256 ? 2 : 1); ++g)
              if (poisoned[g])
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                  for (int y = 0; y < 2; ++y) {
                    const int pos = en.len + (en.r0 + 8 * nt + 2 * lc + y) / p.G, first = unit + un * kStep;
                    bool hit = false;
                    for (int key = 0; key < kUnit; ++key)
                      hit |= (poisoned[g] >> key & 1) && (!a.causal || first + key <= pos) &&
                             (a.w <= 0 || pos - (first + key) < a.w);
                    if (hit)
#pragma unroll
                      for (int z = 0; z < kKs; ++z)
                        if (D != 256 || z / 8 == g) o[z][nt][y] = o[z][nt][y + 2] = __uint_as_float(0x7fffffffu);
                  }
          }
        }
      };
      if (full) take(std::true_type());
      else take(std::false_type());
    }

    // the next segment's copies start before this one is joined
    const Entry done = en;
    const int done_h = w.h;
    const bool whole = w.k0 == 0 && w.k1 == en.n, first = w.k0 == 0;
    begins |= file_split(p, line, w);
    __syncwarp();
    more = open();

    // the warps join: maximum and sums first, then the rows, one warp after the other
    __syncthreads();           // o_s of the last segment has been read
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float sum = l[nt][y];
        sum += __shfl_xor_sync(0xffffffffu, sum, 4);
        sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        if (lr == 0) {
          ml_s[warp * 2 * kRows + 8 * nt + 2 * lc + y] = m[nt][y];
          ml_s[warp * 2 * kRows + kRows + 8 * nt + 2 * lc + y] = sum;
        }
      }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float to = kNone;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) to = fmaxf(to, ml_s[w * 2 * kRows + 8 * nt + 2 * lc + y]);
        const float keep = exp2f(m[nt][y] - to);
#pragma unroll
        for (int z = 0; z < kKs; ++z) {
          o[z][nt][y] *= keep;
          o[z][nt][y + 2] *= keep;
        }
      }
    for (int w = 0; w < (S::kOs == 1 ? kWarps : 1); ++w) {
      if (S::kOs > 1 || warp == w) {
        float* mine = o_s + (S::kOs > 1 ? warp * kRows * S::kOPitch : 0);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int z = 0; z < kKs; ++z) {
              // dimension lr * D / 8 + 2 z and the next: side by side, eighths next to each other
              float2* at = reinterpret_cast<float2*>(mine + (8 * nt + 2 * lc + y) * S::kOPitch + 16 * z + 2 * lr);
              float2 v = make_float2(o[z][nt][y], o[z][nt][y + 2]);
              if (w) {
                v.x += at->x;
                v.y += at->y;
              }
              *at = v;
            }
      }
      __syncthreads();
    }
    float* part = part_of(p, blockIdx.x, first);
    for (int i = tid; i < done.rows * D; i += 32 * kWarps) {
      const int r = i / D, x = i % D;
      if (kPad && x >= d) continue;
      float to = kNone, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) to = fmaxf(to, ml_s[w * 2 * kRows + r]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w)
        sum += exp2f(ml_s[w * 2 * kRows + r] - to) * ml_s[w * 2 * kRows + kRows + r];
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < S::kOs; ++w)
        v += o_s[(w * kRows + r) * S::kOPitch + (x % (D / 8)) / 2 * 16 + x / (D / 8) * 2 + (x & 1)];
      if (whole) {
        row_of(p, reinterpret_cast<T*>(a.y), a.ys, done, done_h, r)[x] = from_f32<T>(v * row_scale(sum, c.v_scale));
        if (x == 0 && a.lse) *lse_of(p, done, done_h, r) = row_lse(to, sum);
      } else {
        part[r * d + x] = v;
        if (x == 0) {
          part[kRows * d + r] = to;
          part[kRows * (d + 1) + r] = sum;
        }
      }
    }
  }
  if (!begins) file_nothing(p);
}

template <typename T, int D, int NT, bool kPad>
cudaError_t launch(const Params& p, cudaStream_t st) {
  using S = Shape<T, D, NT, kPad>;
  auto kernel = attend_mma_kernel<T, D, NT, kPad>;
  if (S::kSmem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e != cudaSuccess) return reported(e);
  }
  return launch_dependent(kernel, dim3(p.shares), dim3(32 * kWarps), S::kSmem, st, p);
}

// Tile of a head dimension.
inline int tile_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// Row tiles of eight that a warp takes at most: of 256 dimensions two (the sums of more would not fit the registers),
// of padded ones two (fewer kernels).
constexpr int most_tiles(int D, bool pad) { return pad || D == 256 ? 2 : 4; }

// f(D, NT) of a head dimension and a number of row tiles, as types.
template <bool kPad, typename F>
auto with_shape(int d, int nt, F&& f) {
  auto rows = [&](auto dim) {
    constexpr int kMost = most_tiles(decltype(dim)::value, kPad);
    return nt == 1   ? f(dim, std::integral_constant<int, 1>())
           : nt == 2 ? f(dim, std::integral_constant<int, 2>())
           : nt == 3 ? f(dim, std::integral_constant<int, kMost < 3 ? kMost : 3>())
                     : f(dim, std::integral_constant<int, kMost>());
  };
  const int D = tile_dim(d);
  return D == 64 ? rows(std::integral_constant<int, 64>()) : D == 128 ? rows(std::integral_constant<int, 128>())
                                                                      : rows(std::integral_constant<int, 256>());
}

cudaError_t launch_padded(const Params& p, int nt, int dtype, cudaStream_t st);
int padded_ctas(int d, int nt, int dtype);

}  // namespace attend
}  // namespace sa
