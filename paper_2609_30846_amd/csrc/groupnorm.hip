// Group normalization, channels last, with the integer Swish or without an activation
// (the statistics of each utterance and group of channels in place of a calibrated BatchNorm).
//
// For the n values z of a group (W bits; include/ipk.h has the whole definition):
//   S = sum z, Q = sum z^2, m0 = floor(S / n), r = S - n m0
//   D = Q - m0 (2 S - n m0) - floor(r^2 / n)
//   R = floor(2^55 / floor(sqrt(2^16 (floor(2^16 D / n) + eps))))
//   A_c = floor(gn_mult_c R / 2^(40-W)),  C_c = gn_bias_c + 2^(shift-1) - floor(mu A_c / 2^16)
//   h   = floor((z A_c + C_c) / 2^shift)
// |S| <= 2^42 and Q <= 2^57 for n <= 2^27 int16 values, so every term fits 64 bits; the two
// products with gn_mult and A_c are taken in two parts.  z A_c + C_c is at most 2^53 plus the
// bias in magnitude (|z - mean| <= sigma sqrt(n)), so it is exact whatever its terms' sizes.
//
// A value costs two to four bytes of traffic and about 16 integer instructions with a Swish whose multiplier has up
// to 16 bits (a 32 x 32 + 64-bit multiply-add for the normalization, another for the Swish, clamps and
// packing), 24 with a wider one (64-bit products), 7 without, so large calls are bound by memory and by issuing
// them (48 x 1000 x 1024: half of the SIMDs' cycles at 2.4 GHz, two thirds with a wide multiplier, with 3.5 waves a SIMD
// resident on average of the six that 78 registers allow), and small ones by the launch and the trip
// to memory and back.  Every value that has been read stays in registers until the
// statistics are there:
//  * one workgroup per utterance and group where a group's values fit its registers (per utterance and a
//    few groups where those are smaller than two pieces of 16 bytes): one read, one write, one launch.
//    48 x 1000 frames of 1024 int16 channels in 32 groups (500 to 1000 of them valid): 43.8 us, 4.0 TB/s of
//    the bytes it cannot do without; 16 x 375: 8.7 us; 1 x 125: 5.2 us; with Swish multipliers of 17 bits
//    50.8, 10.8 and 5.9 us;
//  * otherwise two kernels (three with many groups): partial sums of tiles of 128 bytes of channels x some frames (integer
//    sums, so their order does not matter), and the application, whose workgroups first add the
//    partial sums of their groups while their own values are on the way.  2500 frames of int8 in 16
//    groups: 3.5 + 6.1 us.
// The statistics' division by n is a multiplication by floor((2^64 - 1) / n) with one correction;
// the square root and R take six and eight steps of 64 candidates each, one per lane (about 1 us in
// all).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "ipk_internal.h"

namespace ipk {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v2s __attribute__((ext_vector_type(2)));

struct NormArgs {
  GroupNorm g;
  const void* z;
  void* x;
  int T;
  int pieces;      // 16-byte pieces of a row: of a group, or of all channels
  int rpp;         // rows of pieces per pass of the workgroup (one-kernel form)
  int units, per_xcd;
  int ns, chunks, frames;  // two-kernel form: slices of 8 pieces, frame chunks, frames per chunk
  int narrow;      // the shifted values fit 32 bits
  DivU dv_a, dv_b, dv_cg, dv_fr;
  Lengths lens;
  uint64_t recip[IPK_MAX_BATCH_INTERNAL];  // floor((2^64 - 1) / n) of each utterance
};

__device__ __forceinline__ uint64_t mulhi64(uint64_t a, uint64_t b) { return __umul64hi(a, b); }

// floor(x / n) and the remainder, `m` = floor((2^64 - 1) / n): x m / 2^64 is less than 1 below x / n
__device__ __forceinline__ uint64_t div_n(uint64_t x, uint32_t n, uint64_t m, uint64_t* rem) {
  uint64_t q = mulhi64(x, m);
  uint64_t r = x - q * n;
  if (r >= n) {
    r -= n;
    ++q;
  }
  *rem = r;
  return q;
}

// The largest lane whose candidate holds, for a test that holds on lanes 0 .. k
__device__ __forceinline__ uint32_t last_lane(bool holds) { return (uint32_t)__popcll(__ballot(holds)) - 1; }

struct Stats {
  int64_t R, mu;
};

__device__ __forceinline__ uint64_t uniform64(uint64_t v) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32)) << 32 |
         (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);
}

// R and mu of a group from its sums, the same in every lane of the wave (and in scalar registers).
__device__ __forceinline__ Stats group_stats(int64_t S, int64_t Q, uint32_t n, uint64_t m, uint32_t eps) {
  const uint32_t lane = threadIdx.x & 63;
  S = (int64_t)uniform64((uint64_t)S);
  Q = (int64_t)uniform64((uint64_t)Q);
  uint64_t rem;
  int64_t m0, r;
  if (S >= 0) {
    m0 = (int64_t)div_n((uint64_t)S, n, m, &rem);
    r = (int64_t)rem;
  } else {
    m0 = -1 - (int64_t)div_n((uint64_t)(-1 - S), n, m, &rem);
    r = (int64_t)n - 1 - (int64_t)rem;
  }
  uint64_t unused;
  const int64_t D = Q - m0 * (2 * S - (int64_t)n * m0) - (int64_t)div_n((uint64_t)(r * r), n, m, &unused);
  const uint64_t whole = div_n((uint64_t)D, n, m, &rem);
  const uint64_t v = ((whole << 16) + div_n(rem << 16, n, m, &unused) + eps) << 16;  // at most 2^62 + 2^47
  uint32_t sigma = 0;
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    const int sh = i < 5 ? 26 - 6 * i : 0;
    const uint32_t c = sigma + (lane << sh);
    sigma += last_lane((uint64_t)c * c <= v) << sh;
  }
  sigma = __builtin_amdgcn_readfirstlane(sigma);
  // sigma >= 256, so the division's first digit enters with remainder 2^7: 2^55 = 2^7 64^8
  const uint64_t p = (uint64_t)lane * sigma;
  uint64_t rest = 1 << 7, R = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    rest <<= 6;
    const uint32_t digit = last_lane(p <= rest);
    rest -= (uint64_t)digit * sigma;
    R = (R << 6) | digit;
  }
  // floor((2^17 S + n) / (2 n)) = 2^16 m0 + floor((2^17 r + n) / (2 n)), the latter's inner floor by n
  const uint64_t frac = div_n(((uint64_t)r << 17) + n, n, m, &unused) >> 1;
  return Stats{(int64_t)R, m0 * 65536 + (int64_t)frac};
}

// Channel coefficients: floor(floor(m R / 2^24) / 2^(16-W)), and mu A by 2^16, each from two parts.
template <int W>
__device__ __forceinline__ void coefficients(const Stats& s, int mult, int64_t bias, int64_t* A, int64_t* C) {
  const int64_t a = ((int64_t)mult * (int)(s.R >> 24) + (((int64_t)mult * (int)(s.R & 0xffffff)) >> 24)) >> (16 - W);
  *A = a;
  *C = bias - ((s.mu >> 16) * a + (((s.mu & 0xffff) * a) >> 16));
}

// Eq. 12's Swish of an int16 value and its requantization: -(|h| L + h q1) is -h (t^2 + 2 q1) for
// h >= 0 and h t^2 below, t = qc - min(|h|, qc): the median of qc - h, qc + h and 0.
//  FAST: |h m_sw| and t^2 + 2 |q1| stay below 2^31 and shift_sw >= 32: one 64-bit multiply-add
//  otherwise products of 64 bits, exact as the accepted constants keep h w m_sw + 2^(shift_sw-1) below 2^63
template <bool FAST>
__device__ __forceinline__ int swish(int h, const GroupNorm& g) {
  const int a = g.sw_qc - h, b = g.sw_qc + h;
  const int t = max(min(max(a, b), 0), min(a, b));
  if constexpr (FAST) {
    const int t2 = __mul24(t, t);
    const int w = h < 0 ? t2 : -2 * (int)g.sw_q1 - t2;
    const int64_t v = (int64_t)__mul24(h, g.m_sw) * w + (1ll << (g.shift_sw - 1));
    return (int)(v >> 32) >> (g.shift_sw - 32);
  } else {
    const int64_t t2 = (int64_t)t * t;
    const int64_t w = h < 0 ? t2 : -(t2 + 2 * g.sw_q1);
    const int64_t o = (h * w * g.m_sw + (1ll << (g.shift_sw - 1))) >> g.shift_sw;
    return (int)min(max(o, (int64_t)-32768), (int64_t)32767);
  }
}

enum { SW_NONE = 0, SW_FAST = 1, SW_WIDE = 2 };

template <typename TI>
constexpr int kPiece = 16 / (int)sizeof(TI);  // values of a 16-byte piece

template <typename TI>
__device__ __forceinline__ int value_of(const v4i& v, int i) {
  if constexpr (sizeof(TI) == 1) return (v[i >> 2] << (24 - 8 * (i & 3))) >> 24;
  else return (v[i >> 1] << (16 - 16 * (i & 1))) >> 16;
}

// A workgroup's channel coefficients, each computed once, by one thread, and laid out for 16-byte
// reads of the lanes of consecutive pieces: of P pieces of PC channels, channel i of piece p has
// its A (low and high word) at ((i / 4) P + p) 4 + i % 4 and its C at ((i / 2) P + p) 2 + i % 2.
// (In channel order the lanes of a read met in the same banks: reading 128 channels' coefficients then
// took 4 us of a 10 us kernel.)
template <int N>
struct Coefs {
  int lo[N], hi[N];
  int64_t C[N];
  int narrow;  // every A fits 32 bits (and the shifted values do: NormArgs::narrow)

  template <int PC>
  __device__ __forceinline__ void put(int c, int P, int64_t a, int64_t cc) {
    const int p = c / PC, i = c % PC;
    const int at = ((i >> 2) * P + p) * 4 + (i & 3);
    lo[at] = (int)a;
    hi[at] = (int)(a >> 32);
    C[((i >> 1) * P + p) * 2 + (i & 1)] = cc;
    if (a != (int)a) narrow = 0;
  }
};

typedef long long v2l __attribute__((ext_vector_type(2)));

// One piece of input values to the output values of its channels, piece p of c's P pieces.
template <typename TI, typename TO, int SW, int N>
struct Apply {
  static constexpr int PC = kPiece<TI>;
  const Coefs<N>& c;
  const int p, P;
  int64_t C[PC];
  int A[PC];

  __device__ __forceinline__ Apply(const Coefs<N>& coefs, int piece, int pieces) : c(coefs), p(piece), P(pieces) {
#pragma unroll
    for (int i = 0; i < PC; i += 4) {
      const v4i v = *(const v4i*)&c.lo[((i >> 2) * P + p) * 4];
#pragma unroll
      for (int k = 0; k < 4; ++k) A[i + k] = v[k];
    }
#pragma unroll
    for (int i = 0; i < PC; i += 2) {
      const v2l v = *(const v2l*)&c.C[((i >> 1) * P + p) * 2];
      C[i] = v[0];
      C[i + 1] = v[1];
    }
  }

  template <typename F>
  __device__ __forceinline__ void values(const v4i& v, const NormArgs& a, int (&o)[PC], F h_of) const {
#pragma unroll
    for (int i = 0; i < PC; ++i) {
      int h = h_of(i, value_of<TI>(v, i));
      if (SW != SW_NONE) h = swish<SW == SW_FAST>(min(max(h, -32767), 32767), a.g);
      o[i] = sizeof(TO) == 1 ? min(max(h, -127), 127) : h;
    }
  }
  // two values to int16, held to +-32767 (the pack saturates to -32768 .. 32767)
  static __device__ __forceinline__ int pack16(int x, int y) {
    const v2s p = __builtin_elementwise_max(__builtin_amdgcn_cvt_pk_i16(x, y), (v2s){-32767, -32767});
    return __builtin_bit_cast(int, p);
  }

  __device__ __forceinline__ void run(const v4i& v, const NormArgs& a, TO* x) const {
    int o[PC];
    const int sh = a.g.shift;
    if (c.narrow) {
      if (sh < 32)
        values(v, a, o, [&](int i, int z) {
          const uint64_t t = (uint64_t)((int64_t)z * A[i] + C[i]);
          return (int)__builtin_amdgcn_alignbit((uint32_t)(t >> 32), (uint32_t)t, sh);
        });
      else
        values(v, a, o, [&](int i, int z) { return (int)(((int64_t)z * A[i] + C[i]) >> 32) >> (sh - 32); });
    } else {
      values(v, a, o, [&](int i, int z) {
        const int64_t A64 = (int64_t)c.hi[((i >> 2) * P + p) * 4 + (i & 3)] << 32 | (uint32_t)A[i];
        const int64_t t = (z * A64 + C[i]) >> sh;
        return (int)min(max(t, (int64_t)-32768), (int64_t)32767);
      });
    }
    if constexpr (sizeof(TO) == 1) {
      uint32_t d[PC / 4];
#pragma unroll
      for (int k = 0; k < PC / 4; ++k)
        d[k] = __builtin_amdgcn_perm((uint32_t)o[4 * k + 1], (uint32_t)o[4 * k], 0x0c0c0400u) |
               __builtin_amdgcn_perm((uint32_t)o[4 * k + 3], (uint32_t)o[4 * k + 2], 0x04000c0cu);
      if constexpr (PC == 16) *(v4i*)x = (v4i){(int)d[0], (int)d[1], (int)d[2], (int)d[3]};
      else *(uint2*)x = make_uint2(d[0], d[1]);
    } else {
#pragma unroll
      for (int k = 0; k < PC / 8; ++k) {
        v4i d;
#pragma unroll
        for (int w = 0; w < 4; ++w)
          d[w] = pack16(o[8 * k + 2 * w], o[8 * k + 2 * w + 1]);
        *(v4i*)(x + 8 * k) = d;
      }
    }
  }

  __device__ __forceinline__ static void zero(TO* x) {
    constexpr int BYTES = PC * (int)sizeof(TO);
    if constexpr (BYTES == 8) {
      *(uint2*)x = make_uint2(0, 0);
    } else {
#pragma unroll
      for (int k = 0; k < BYTES / 16; ++k) *((v4i*)x + k) = (v4i){0, 0, 0, 0};
    }
  }
};

// S and Q of a piece: S in 32 bits (a lane sees fewer than 2^16 values), Q in 64; an int16 pair's
// squares reach 2^31, exact as an unsigned word
template <typename TI>
__device__ __forceinline__ void add_sums(const v4i& v, int& S, uint64_t& Q) {
  if constexpr (sizeof(TI) == 1) {
    int q = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      S = __builtin_amdgcn_sdot4(v[w], 0x01010101, S, false);
      q = __builtin_amdgcn_sdot4(v[w], v[w], q, false);
    }
    Q += (uint32_t)q;
  } else {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int word = v[w];  // (a bit cast of v[w] itself takes the vector's first element)
      const v2s p = __builtin_bit_cast(v2s, word);
      S = __builtin_amdgcn_sdot2(p, (v2s){1, 1}, S, false);
      Q += (uint32_t)__builtin_amdgcn_sdot2(p, p, 0, false);
    }
  }
}

// Sums over the lanes of a wave that agree in their low bits, STEP of them: 1, all 64 lanes, or 8, the
// eight rows of a wave of 8 pieces.  Rotations within 16 lanes (row_ror by DPP), then swaps of the
// 16-lane rows and of the halves.
template <int CTRL>
__device__ __forceinline__ uint64_t dpp64(uint64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, 0xF, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, 0xF, 0xF, false);
  return (uint64_t)hi << 32 | lo;
}
template <int STEP>
__device__ __forceinline__ uint64_t lanes_sum(uint64_t v) {
  if (STEP == 1) {
    v += dpp64<0x121>(v);
    v += dpp64<0x122>(v);
    v += dpp64<0x124>(v);
  }
  v += dpp64<0x128>(v);
  {
    const auto l = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    const auto h = __builtin_amdgcn_permlane16_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
    v = ((uint64_t)h[0] << 32 | l[0]) + ((uint64_t)h[1] << 32 | l[1]);
  }
  const auto l = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  const auto h = __builtin_amdgcn_permlane32_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
  return ((uint64_t)h[0] << 32 | l[0]) + ((uint64_t)h[1] << 32 | l[1]);
}
template <int STEP>
__device__ __forceinline__ int lanes_sum(int v) {
  if (STEP == 1) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x121, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x122, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x124, 0xF, 0xF, false);
  }
  v += __builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, false);
  const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
  v = (int)(r[0] + r[1]);
  const auto q = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  return (int)(q[0] + q[1]);
}

// --- one workgroup per utterance and group, or a few groups

constexpr int FUSED_THREADS = 512;
constexpr int FUSED_CG = 1024;    // channels of a workgroup's group at most
constexpr int FUSED_GROUPS = 16;  // groups of a workgroup at most

// SEVERAL: groups of one piece, or groups that end inside pieces: the workgroup has the fewest channels that are
// whole groups and whole pieces, or a multiple of them, in rows of up to eight pieces, one per lane
// of eight.  Otherwise it has one group of whole pieces, and each lane a piece of its rows.
template <typename TI, typename TO, int SW, int NP, bool SEVERAL>
__global__ __launch_bounds__(FUSED_THREADS) void groupnorm_fused(NormArgs a) {
  constexpr int PC = kPiece<TI>;
  __shared__ unsigned long long sums[SEVERAL ? FUSED_GROUPS : FUSED_THREADS / 64][2];
  __shared__ Stats stats[SEVERAL ? FUSED_GROUPS : 1];
  __shared__ __align__(16) Coefs<SEVERAL ? 8 * PC : FUSED_CG> coefs;
  // neighbouring groups share cache lines: consecutive ones on one XCD
  const int unit = (blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);
  if (unit >= a.units) return;
  const int b = (int)div_u((uint32_t)unit, a.dv_a), u = unit - b * (int)a.dv_a.d;
  const int L = a.lens.len[b], T = a.T, d = a.g.d, cg = (int)a.dv_cg.d;
  const int first = u * a.pieces * PC;                                // the workgroup's first channel,
  const int cw = SEVERAL ? min(a.pieces * PC, d - first) : cg;        // its channels
  const int tid = threadIdx.x;
  const int r0 = SEVERAL ? tid >> 3 : (int)div_u((uint32_t)tid, a.dv_b);
  const int col = SEVERAL ? tid & 7 : tid - r0 * a.pieces;
  const bool active = SEVERAL ? col * PC < cw : r0 < a.rpp;
  const int c0 = active ? col * PC : 0;
  const size_t base = (size_t)b * T * d + first + c0;
  v4i v[NP];
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int t = r0 + k * a.rpp;
    v[k] = active && t < L ? *(const v4i*)((const TI*)a.z + base + (size_t)t * d) : (v4i){0, 0, 0, 0};
  }
  const int cm = first + min(tid, cw - 1);
  const int mult = a.g.mult[cm];
  const int64_t bias = a.g.bias[cm];
  if (tid == 0) coefs.narrow = a.narrow;
  const uint32_t n = (uint32_t)L * (uint32_t)cg;
  if constexpr (SEVERAL) {
    if (tid < 2 * FUSED_GROUPS) sums[tid >> 1][tid & 1] = 0;
    __syncthreads();
    const bool adds = active && (tid & 63) < 8;  // for the eight rows of its wave
    if (cg == PC) {
      int S = 0;
      uint64_t Q = 0;
#pragma unroll
      for (int k = 0; k < NP; ++k) add_sums<TI>(v[k], S, Q);
      S = lanes_sum<8>(S);
      Q = lanes_sum<8>(Q);
      if (adds) {
        atomicAdd(&sums[col][0], (unsigned long long)(int64_t)S);
        atomicAdd(&sums[col][1], (unsigned long long)Q);
      }
    } else {
      // sums of each channel, or of each group where pieces are whole groups (every lane's end at once):
      // 32 bits but for the squares of int16 values
      using TQ = std::conditional_t<sizeof(TI) == 1, int, uint64_t>;
      const int step = cg < PC && !(cg & (cg - 1)) ? cg : 1;  // PC is a power of two
      int S = 0;
      TQ Q = 0;
#pragma unroll
      for (int i = 0; i < PC; ++i) {
#pragma unroll
        for (int k = 0; k < NP; ++k) {
          const int y = value_of<TI>(v[k], i);
          S += y;
          Q += (uint32_t)__mul24(y, y);
        }
        if ((i + 1) & (step - 1)) continue;
        const int Sw = lanes_sum<8>(S);
        const TQ Qw = lanes_sum<8>(Q);
        if (adds) {
          const int g = (int)div_u((uint32_t)(c0 + i), a.dv_cg);
          atomicAdd(&sums[g][0], (unsigned long long)(int64_t)Sw);
          atomicAdd(&sums[g][1], (unsigned long long)Qw);
        }
        S = 0;
        Q = 0;
      }
    }
    __syncthreads();
    const int ng = (int)div_u((uint32_t)cw, a.dv_cg);
    for (int g = tid >> 6; g < ng; g += FUSED_THREADS / 64) {
      const Stats r = group_stats((int64_t)sums[g][0], (int64_t)sums[g][1], n, a.recip[b], (uint32_t)a.g.eps);
      if ((tid & 63) == 0) stats[g] = r;
    }
  } else {
    int S = 0;
    uint64_t Q = 0;
#pragma unroll
    for (int k = 0; k < NP; ++k) add_sums<TI>(v[k], S, Q);
    // a wave's S: 64 lanes x NP pieces of at most 8 x 2^15, below 2^31
    S = lanes_sum<1>(S);
    Q = lanes_sum<1>(Q);
    if ((tid & 63) == 0) {
      sums[tid >> 6][0] = (uint64_t)(int64_t)S;
      sums[tid >> 6][1] = Q;
    }
    __syncthreads();
    if (tid < 64) {
      uint64_t St = 0, Qt = 0;
#pragma unroll
      for (int w = 0; w < FUSED_THREADS / 64; ++w) {
        St += sums[w][0];
        Qt += sums[w][1];
      }
      const Stats r = group_stats((int64_t)St, (int64_t)Qt, n, a.recip[b], (uint32_t)a.g.eps);
      if (tid == 0) stats[0] = r;
    }
  }
  __syncthreads();
  if (tid < cw) {
    const Stats r = stats[SEVERAL ? (int)div_u((uint32_t)tid, a.dv_cg) : 0];
    int64_t A, C;
    coefficients<8 * sizeof(TI)>(r, mult, bias, &A, &C);
    coefs.template put<PC>(tid, a.pieces, A, C);
    if constexpr (!SEVERAL)
      for (int c = tid + FUSED_THREADS; c < cg; c += FUSED_THREADS) {
        coefficients<8 * sizeof(TI)>(r, a.g.mult[first + c], a.g.bias[first + c], &A, &C);
        coefs.template put<PC>(c, a.pieces, A, C);
      }
  }
  __syncthreads();
  if (!active) return;
  const Apply<TI, TO, SW, SEVERAL ? 8 * PC : FUSED_CG> ap(coefs, col, a.pieces);
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int t = r0 + k * a.rpp;
    TO* x = (TO*)a.x + base + (size_t)t * d;
    if (t < L) ap.run(v[k], a, x);
    else if (t < T) ap.zero(x);
  }
}

// --- partial sums, then the application

constexpr int TILE_THREADS = 256;
constexpr int TILE_ROWS = TILE_THREADS / 8;  // rows of 8 pieces (128 bytes) per pass

// The sums of slice s of the channels and group g meet in entry g + s of a chunk's partial sums: along
// the channels the two indexes only grow, so no two overlapping pairs share an entry.
__device__ __forceinline__ uint64_t* entry_at(const NormArgs& a, int b, int chunk, int e) {
  return (uint64_t*)a.g.partial + (((size_t)b * a.chunks + chunk) * (a.ns + a.g.groups) + e) * 2;
}

template <typename TI>
__global__ __launch_bounds__(TILE_THREADS) void groupnorm_sums(NormArgs a) {
  constexpr int PC = kPiece<TI>, SLC = 8 * PC;
  __shared__ unsigned long long sums[SLC + 1][2];
  const int bc = (int)div_u(blockIdx.x, a.dv_a), s = (int)blockIdx.x - bc * a.ns;
  const int b = (int)div_u((uint32_t)bc, a.dv_b), chunk = bc - b * a.chunks;
  const int L = a.lens.len[b], d = a.g.d, cg = (int)a.dv_cg.d;
  const int t0 = chunk * a.frames, t1 = min(t0 + a.frames, L);
  if (t0 >= L) return;  // never read
  const int tid = threadIdx.x, piece = s * 8 + (tid & 7), row = tid >> 3;
  const bool in = piece < a.pieces;
  const int c0 = piece * PC;
  const int g0 = (int)div_u((uint32_t)(s * SLC), a.dv_cg);
  for (int i = tid; i < 2 * (SLC + 1); i += TILE_THREADS) sums[i >> 1][i & 1] = 0;
  __syncthreads();
  const TI* z = (const TI*)a.z + (size_t)b * a.T * d + c0;
  // the lane's rows of the chunk, four loads at a time (rows past the chunk as zeros)
  auto rows = [&](auto add) {
    for (int t = t0 + row; in && t < t1; t += 4 * TILE_ROWS) {
      v4i v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        v[k] = t + k * TILE_ROWS < t1 ? *(const v4i*)(z + (size_t)(t + k * TILE_ROWS) * d) : (v4i){0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < 4; ++k) add(v[k]);
    }
  };
  if (cg % PC == 0) {
    // a piece lies in one group; the rows of a wave are added by lane exchanges first
    int S = 0;
    uint64_t Q = 0;
    rows([&](const v4i& v) { add_sums<TI>(v, S, Q); });
    S = lanes_sum<8>(S);  // 8 lanes x 256 pieces of at most 8 x 2^15
    Q = lanes_sum<8>(Q);
    if (in && (tid & 63) < 8) {
      const int g = (int)div_u((uint32_t)c0, a.dv_cg) - g0;
      atomicAdd(&sums[g][0], (unsigned long long)(int64_t)S);
      atomicAdd(&sums[g][1], (unsigned long long)Q);
    }
  } else {
    // groups end inside pieces: sums of each channel, a lane's in 32 bits (int8: 256 squares of at most
    // 2^14) or 64
    using TQ = std::conditional_t<sizeof(TI) == 1, int, uint64_t>;
    int S[PC];
    TQ Q[PC];
#pragma unroll
    for (int i = 0; i < PC; ++i) {
      S[i] = 0;
      Q[i] = 0;
    }
    rows([&](const v4i& v) {
#pragma unroll
      for (int i = 0; i < PC; ++i) {
        const int y = value_of<TI>(v, i);
        S[i] += y;
        Q[i] += (uint32_t)__mul24(y, y);
      }
    });
#pragma unroll
    for (int i = 0; i < PC; ++i) {
      const int Si = lanes_sum<8>(S[i]);
      const TQ Qi = lanes_sum<8>(Q[i]);
      if (in && (tid & 63) < 8) {
        const int g = (int)div_u((uint32_t)(c0 + i), a.dv_cg) - g0;
        atomicAdd(&sums[g][0], (unsigned long long)(int64_t)Si);
        atomicAdd(&sums[g][1], (unsigned long long)Qi);
      }
    }
  }
  __syncthreads();
  const int last = min((s + 1) * SLC, d) - 1;
  const int ng = (int)div_u((uint32_t)last, a.dv_cg) - g0 + 1;
  for (int i = tid; i < 2 * ng; i += TILE_THREADS) entry_at(a, b, chunk, g0 + (i >> 1) + s)[i & 1] = sums[i >> 1][i & 1];
}

// R and mu of group g of utterance b, its partial sums added over chunks and slices by one wave.
template <int SLC>
__device__ __forceinline__ Stats gather_stats(const NormArgs& a, int b, int g) {
  const int L = a.lens.len[b], cg = (int)a.dv_cg.d;
  const int nch = (int)div_u((uint32_t)(L + a.frames - 1), a.dv_fr);
  const int s0 = g * cg / SLC, n_s = ((g + 1) * cg - 1) / SLC - s0 + 1;
  uint64_t S = 0, Q = 0;
  for (int k = threadIdx.x & 63; k < nch; k += 64)
    for (int j = 0; j < n_s; j += 8) {
      uint64_t e[8][2];  // eight loads at a time
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const uint64_t* p = entry_at(a, b, k, g + s0 + min(j + u, n_s - 1));
        e[u][0] = j + u < n_s ? p[0] : 0;
        e[u][1] = j + u < n_s ? p[1] : 0;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        S += e[u][0];
        Q += e[u][1];
      }
    }
  S = lanes_sum<1>(S);
  Q = lanes_sum<1>(Q);
  return group_stats((int64_t)S, (int64_t)Q, (uint32_t)L * (uint32_t)cg, a.recip[b], (uint32_t)a.g.eps);
}

// One wave per utterance and group.
template <int SLC>
__global__ __launch_bounds__(TILE_THREADS) void groupnorm_stats(NormArgs a) {
  const int unit = (int)blockIdx.x * (TILE_THREADS / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= a.units) return;
  const int b = (int)div_u((uint32_t)unit, a.dv_a), g = unit - b * (int)a.dv_a.d;
  const Stats r = gather_stats<SLC>(a, b, g);
  if ((threadIdx.x & 63) == 0) ((Stats*)a.g.stats)[unit] = r;
}

// GATHER: the workgroup forms the statistics of its groups itself, one wave each (otherwise
// groupnorm_stats has).
template <typename TI, typename TO, int SW, int NP, bool GATHER>
__global__ __launch_bounds__(TILE_THREADS) void groupnorm_apply(NormArgs a) {
  constexpr int PC = kPiece<TI>, SLC = 8 * PC;
  __shared__ Stats stats[GATHER ? SLC + 1 : 1];
  __shared__ __align__(16) Coefs<SLC> coefs;
  const int bc = (int)div_u(blockIdx.x, a.dv_a), s = (int)blockIdx.x - bc * a.ns;
  const int b = (int)div_u((uint32_t)bc, a.dv_b), t0 = (bc - b * (int)a.dv_b.d) * (NP * TILE_ROWS);
  const int L = a.lens.len[b], T = a.T, d = a.g.d;
  const int tid = threadIdx.x, piece = s * 8 + (tid & 7), row = t0 + (tid >> 3);
  const bool in = piece < a.pieces;
  const int c0 = in ? piece * PC : 0;
  const size_t base = (size_t)b * T * d + c0;
  v4i v[NP];
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int t = row + k * TILE_ROWS;
    v[k] = in && t < L ? *(const v4i*)((const TI*)a.z + base + (size_t)t * d) : (v4i){0, 0, 0, 0};
  }
  const int cm = min(s * SLC + (tid & (SLC - 1)), d - 1), gm = (int)div_u((uint32_t)cm, a.dv_cg);
  const int mult = a.g.mult[cm];
  const int64_t bias = a.g.bias[cm];
  if (tid == 0) coefs.narrow = a.narrow;
  if (t0 < L) {
    Stats r{};
    if constexpr (GATHER) {
      const int g0 = (int)div_u((uint32_t)(s * SLC), a.dv_cg);
      const int ng = (int)div_u((uint32_t)(min((s + 1) * SLC, d) - 1), a.dv_cg) - g0 + 1;
      for (int i = tid >> 6; i < ng; i += TILE_THREADS / 64) {
        const Stats gs = gather_stats<SLC>(a, b, g0 + i);
        if ((tid & 63) == 0) stats[i] = gs;
      }
      __syncthreads();
      r = stats[gm - g0];
    } else {
      r = ((const Stats*)a.g.stats)[(size_t)b * a.g.groups + gm];
      __syncthreads();
    }
    if (tid < SLC) {
      int64_t A, C;
      coefficients<8 * sizeof(TI)>(r, mult, bias, &A, &C);
      coefs.template put<PC>(tid, 8, A, C);
    }
    __syncthreads();
  }
  if (!in) return;
  const Apply<TI, TO, SW, SLC> ap(coefs, tid & 7, 8);
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int t = row + k * TILE_ROWS;
    TO* x = (TO*)a.x + base + (size_t)t * d;
    if (t < L) ap.run(v[k], a, x);
    else if (t < T) ap.zero(x);
  }
}

template <typename TI, typename TO, int SW, bool SEVERAL>
static hipError_t launch_fused(NormArgs& a, int np, hipStream_t st) {
  const dim3 grid(8 * a.per_xcd), block(FUSED_THREADS);
  if (np <= 1) hipLaunchKernelGGL((groupnorm_fused<TI, TO, SW, 1, SEVERAL>), grid, block, 0, st, a);
  else if (np <= 2) hipLaunchKernelGGL((groupnorm_fused<TI, TO, SW, 2, SEVERAL>), grid, block, 0, st, a);
  else if (np <= 4) hipLaunchKernelGGL((groupnorm_fused<TI, TO, SW, 4, SEVERAL>), grid, block, 0, st, a);
  else if (SEVERAL || np <= 8) hipLaunchKernelGGL((groupnorm_fused<TI, TO, SW, 8, SEVERAL>), grid, block, 0, st, a);
  else if constexpr (!SEVERAL) hipLaunchKernelGGL((groupnorm_fused<TI, TO, SW, 16, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

// Pieces of a row of the one-kernel form's workgroups, 0 where it does not apply.  Groups of several whole
// pieces: one group's.  Others: the largest multiple, up to eight pieces and FUSED_GROUPS groups,
// of the fewest pieces that are whole groups.
static int fused_pieces(int cg, int groups, int PC, bool* several) {
  *several = !(cg % PC == 0 && cg >= 2 * PC);
  if (!*several) return cg <= FUSED_CG ? cg / PC : 0;
  int gcd = PC;
  while (cg % gcd) gcd /= 2;
  const int least = cg / gcd, per = PC / gcd;  // those pieces, and their groups
  if (least > 8) return 0;
  const int times = std::min({8 / least, FUSED_GROUPS / per, groups / per});
  return least * times;
}

template <typename TI, typename TO, int SW>
static hipError_t launch_norm(NormArgs& a, int B, hipStream_t st) {
  constexpr int PC = kPiece<TI>, SLC = 8 * PC;
  const int d = a.g.d, T = a.T, cg = d / a.g.groups;
  a.dv_cg = make_div((uint32_t)cg);
  // One kernel with up to four pieces a lane, or up to sixteen where the workgroups fill the CUs (times with
  // multipliers of the Swish of up to 16 bits): 4 x 500 x 1024 in 32 groups (4 pieces, 128 workgroups) 8.0 us against
  // 10.4, 2 x 300 (4, 64) 6.2 against 9.0, 48 x 1000 (8, 1536) 43 against 51; but 1 x 400 in 8 groups (16, 8) 13.2 against
  // 7.9.  With several groups a workgroup,
  // where it takes the place of three launches (calls / kernels alone): up to four, or eight for int16 or
  // where the CUs are filled, beyond which more registers a lane would spill.  1 x 25 x 512 int16 in 64 groups (1 piece)
  // 6.7 / 4.3 us against 12.5 / 8.1, 1 x 256 x 256 int8 in 64 (4) 10.5 / 10.1 against 12.5 / 10.1, 64 x 500 x 512 int16
  // in 64 (8) 18.6 / 19.6 against 24.5 / 25.6, 1 x 500 x 256 int16 in 64 (8) 11.0 / 10.6 against 12.5 / 9.1; but 1 x
  // 500 x 256 int8 in 64 (8) 16.4 / 16.0 against 12.7 / 10.0 (sums of each channel then).
  bool several;
  const int pieces = fused_pieces(cg, a.g.groups, PC, &several);
  const int rpp = !pieces ? 0 : several ? FUSED_THREADS / 8 : FUSED_THREADS / pieces;
  const int np = rpp ? (T + rpp - 1) / rpp : 0, per_b = pieces ? (d / PC + pieces - 1) / pieces : 0;
  if (rpp && np <= (B * per_b < 256 ? (several && PC == 8 ? 8 : 4) : several ? 8 : 16)) {
    a.pieces = pieces;
    a.rpp = rpp;
    a.units = B * per_b;
    a.per_xcd = (a.units + 7) / 8;
    a.dv_a = make_div((uint32_t)per_b);
    a.dv_b = make_div((uint32_t)pieces);
    return several ? launch_fused<TI, TO, SW, true>(a, np, st) : launch_fused<TI, TO, SW, false>(a, np, st);
  }
  a.pieces = d / PC;
  a.ns = (d + SLC - 1) / SLC;
  a.chunks = groupnorm_chunks(B, T, a.ns, cg % PC == 0);
  a.frames = (T + a.chunks - 1) / a.chunks;
  a.dv_fr = make_div((uint32_t)a.frames);
  a.dv_a = make_div((uint32_t)a.ns);
  a.dv_b = make_div((uint32_t)a.chunks);
  hipLaunchKernelGGL(groupnorm_sums<TI>, dim3(B * a.chunks * a.ns), dim3(TILE_THREADS), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // up to four groups in a slice: their statistics in the application's workgroups, a wave each; in calls
  // whose workgroups all run at once up to eight, in two rounds, which take less time than a launch (calls / kernels alone,
  // eight int16 groups: 1 x 1000 x 512 9.5 / 8.5 us against 13.2 / 8.3, 1 x 2500 11.9 / 11.5 against 12.5 / 9.6; but 8 x
  // 1000 14.3 / 13.9 against 12.7 / 11.4; sixteen, 1 x 1000 x 256: 12.8 / 12.1 against 12.5 / 8.9)
  const long tiles1 = (long)B * ((T + TILE_ROWS - 1) / TILE_ROWS) * a.ns;
  const bool gather = cg * (tiles1 < 1024 ? 8 : 4) >= SLC;
  if (!gather) {
    a.units = B * a.g.groups;
    a.dv_a = make_div((uint32_t)a.g.groups);
    hipLaunchKernelGGL(groupnorm_stats<SLC>, dim3((a.units + 3) / 4), dim3(TILE_THREADS), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    a.dv_a = make_div((uint32_t)a.ns);
  }
  // as many rows per lane as leave every CU a workgroup or two
  auto launch = [&](auto kernel, int NP) {
    const int per = (T + NP * TILE_ROWS - 1) / (NP * TILE_ROWS);
    a.dv_b = make_div((uint32_t)per);
    hipLaunchKernelGGL(kernel, dim3(B * per * a.ns), dim3(TILE_THREADS), 0, st, a);
    return hipGetLastError();
  };
  if (gather) {
    if (tiles1 >= 4096) return launch(groupnorm_apply<TI, TO, SW, 4, true>, 4);
    if (tiles1 >= 1024) return launch(groupnorm_apply<TI, TO, SW, 2, true>, 2);
    return launch(groupnorm_apply<TI, TO, SW, 1, true>, 1);
  }
  if (tiles1 >= 4096) return launch(groupnorm_apply<TI, TO, SW, 4, false>, 4);
  if (tiles1 >= 1024) return launch(groupnorm_apply<TI, TO, SW, 2, false>, 2);
  return launch(groupnorm_apply<TI, TO, SW, 1, false>, 1);
}

template <typename TI, typename TO>
static hipError_t launch_types(NormArgs& a, int B, hipStream_t st) {
  const GroupNorm& g = a.g;
  if (!g.swish) return launch_norm<TI, TO, SW_NONE>(a, B, st);
  const int64_t q1 = g.sw_q1 < 0 ? -g.sw_q1 : g.sw_q1;
  const bool fast = g.m_sw < (1 << 16) && g.sw_qc < (1 << 15) && (int64_t)g.sw_qc * g.sw_qc + 2 * q1 < ((int64_t)1 << 31) &&
                    g.shift_sw >= 32;
  return fast ? launch_norm<TI, TO, SW_FAST>(a, B, st) : launch_norm<TI, TO, SW_WIDE>(a, B, st);
}

hipError_t launch_groupnorm(const GroupNorm& g, const void* z, const Lengths& lens, int B, int T, void* x,
                            hipStream_t st) {
  NormArgs a{};
  a.g = g;
  a.z = z;
  a.x = x;
  a.T = T;
  a.lens = lens;
  const int cg = g.d / g.groups;
  uint32_t n_max = 0;
  for (int b = 0; b < B; ++b) {
    const uint32_t n = (uint32_t)lens.len[b] * (uint32_t)cg;
    a.recip[b] = ~0ull / n;
    n_max = n > n_max ? n : n_max;
  }
  // |z A + C| <= max|gn_mult| 2^(W-1) (sqrt(n) + 1) 257/256 + max|bias|: sigma + 1 exceeds 2^16 times the
  // standard deviation and sigma is at least 256, so R is at most 257/256 of 2^39 over it, and the mean's
  // rounding adds less than the 1
  const double bound = (double)g.mult_max * (double)(1 << (8 * g.in_bytes - 1)) * (sqrt((double)n_max) + 1) * 1.01 +
                       (double)g.bias_max;
  a.narrow = bound < ldexp(1.0, 31 + g.shift) * 0.99;
  if (g.in_bytes == 1) return g.out_bytes == 1 ? launch_types<int8_t, int8_t>(a, B, st) : launch_types<int8_t, int16_t>(a, B, st);
  return g.out_bytes == 1 ? launch_types<int16_t, int8_t>(a, B, st) : launch_types<int16_t, int16_t>(a, B, st);
}

}  // namespace ipk
