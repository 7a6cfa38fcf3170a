// Linear layer of int8 tokens with a scale for each token and each output channel.
//
//   acc = sum_k q_rk w_ck,  t = floor(acc 2^p s_r / 2^32),
//   y   = clampT(floor((t mult_c + bias_c + 2^16 m_z z_rc + 2^(n-1)) / 2^n)),  n >= 32
//
// |acc 2^p| <= 2^30, so t is the high word of one 32 x 32 product and the output the high word of one
// 32 x 32 + 64-bit multiply-add (two with the residual term), shifted by n - 32.
//
// The product is the projection GEMMs' (gemm_loop.h): 32 x 32 x 32 int8 MFMA, the weights in
// fragment order straight from memory, the token tile through LDS, tiles dealt to the XCDs in
// square groups.
//
// Epilogue: a lane owns one token (one s) and 4 consecutive channels per accumulator group; the
// channels' multipliers and biases come from LDS once per 32 channels and serve all the wave's
// tokens.  Rows leave (and the residual input arrives) in pieces of 16 bytes at any address, so that
// rows of any length take them; only a last piece of fewer values goes value by value.
//  * int8: an exchange with the lane 32 away leaves 16 consecutive channels, one piece, with each
//    lane (32-byte runs of a row);
//  * int16 and int32: a wave passes each 32 channels x 32 tokens through a piece of LDS of its own, so
//    that eight lanes store a row's 128 bytes (four and 64 with an int16 residual).  In pieces of 16
//    bytes a lane, 12000 tokens x 512 -> 2048 to int32 took 46.6 us instead of 29.1, 23000 x 1024 -> 4096 to int16
//    120 instead of 111, 2500 x 1024 -> 1025 to int32 11.2 instead of 9.1 (all with outputs that stay in the
//    caches, see launch_tiles); int8 takes the same time either way.
//
// What bounds it: with many tokens the product, at the clock the chip's power holds (23000 x 4096 -> 1024 to int8
// with the residual 100 us, 1.93 POP/s, the library's int8 product of 8192^3 2.16); with K = 1024 its eight K steps
// leave first operands and epilogue in sight (6000 x 1024 -> 4096 to int16 30 us, 1.68 POP/s, 49 MB of stores; with
// the residual input, as many bytes again in 64-byte runs, 45 us); fewer tokens than fill the CUs once are
// latency (2500 x 1024 -> 1025 to int32 8.6 us: less than one wave a SIMD, eight K steps one after the other).
#include "gemm_loop.h"
#include "gemm_tiles.h"
#include "ipk_internal.h"

namespace ipk {

typedef int v4iu __attribute__((ext_vector_type(4), aligned(1)));  // a piece at any address

struct TokenLinearArgs {
  TokenLinear l;
  const int8_t* q;
  const int32_t* s;
  const void* z;
  void* y;
  int rows;
  int tiles_total, per_xcd;
  TileGrid grid;
  DivU dv_n;  // few tokens: 32-channel tiles
};

// Between a wave's writes to its piece of LDS and its lanes' reads of each other's: the hardware keeps
// a wave's LDS accesses in order, so this only holds the compiler to theirs.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// 16 bytes of a row, the first `left` values of them in it
template <typename T>
__device__ __forceinline__ v4i load_piece(const T* p, int left) {
  constexpr int PC = 16 / (int)sizeof(T);
  if (left >= PC) return *(const v4iu*)p;
  alignas(16) T v[PC] = {};
  for (int k = 0; k < left; ++k) v[k] = p[k];
  return *(const v4i*)v;
}
// PASSING: past the caches
template <typename T, bool PASSING = false>
__device__ __forceinline__ void store_piece(T* p, v4i v, int left) {
  constexpr int PC = 16 / (int)sizeof(T);
  if (left >= PC) {
    if constexpr (PASSING) __builtin_nontemporal_store((v4iu)v, (v4iu*)p);
    else *(v4iu*)p = v;
  } else {
#pragma unroll
    for (int k = 0; k < PC; ++k)
      if (k < left) p[k] = (T)(v[k * (int)sizeof(T) / 4] >> (8 * sizeof(T) * k % 32));
  }
}

__device__ __forceinline__ uint32_t pack8(int a, int b, int c, int d) {
  return __builtin_amdgcn_perm((uint32_t)b, (uint32_t)a, 0x0c0c0400u) |
         __builtin_amdgcn_perm((uint32_t)d, (uint32_t)c, 0x04000c0cu);
}
__device__ __forceinline__ uint32_t pack16(int a, int b) {
  return __builtin_amdgcn_perm((uint32_t)b, (uint32_t)a, 0x05040100u);
}
__device__ __forceinline__ void get4(uint32_t w, int (&o)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = (int)(w << (24 - 8 * e)) >> 24;
}
__device__ __forceinline__ void get4(uint2 w, int (&o)[4]) {
  o[0] = (int)(w.x << 16) >> 16;
  o[1] = (int)w.x >> 16;
  o[2] = (int)(w.y << 16) >> 16;
  o[3] = (int)w.y >> 16;
}

// The four groups' bytes of a lane's block (group g: channels 8 g + 4 (lane / 32) ..) to 16 consecutive
// channels, 16 (lane / 32) .., and back: two exchanges of the halves
__device__ __forceinline__ v4i exchange(const uint32_t (&D)[4]) {
  const auto x = __builtin_amdgcn_permlane32_swap(D[0], D[2], false, false);
  const auto y = __builtin_amdgcn_permlane32_swap(D[1], D[3], false, false);
  return (v4i){(int)x[0], (int)x[1], (int)y[0], (int)y[1]};
}
__device__ __forceinline__ void exchange(const v4i& v, uint32_t (&D)[4]) {
  const auto x = __builtin_amdgcn_permlane32_swap((uint32_t)v[0], (uint32_t)v[1], false, false);
  const auto y = __builtin_amdgcn_permlane32_swap((uint32_t)v[2], (uint32_t)v[3], false, false);
  D[0] = x[0];
  D[2] = x[1];
  D[1] = y[0];
  D[3] = y[1];
}

template <int TN, int TM, int NWAVE, int WN, typename T, bool RES, bool PASSING>
__global__ __launch_bounds__(64 * NWAVE, NWAVE == 8 ? 1 : 2) void token_linear(TokenLinearArgs a) {
  constexpr int LIM = (int)((1u << (8 * sizeof(T) - 1)) - 1);
  constexpr int WM = NWAVE / WN, WTN = TN / WN, WTM = TM / WM, FN = WTN / 32, FM = WTM / 32;
  constexpr int E = (int)sizeof(T);
  constexpr bool STAGED = E > 1;
  // blocks of 32 channels that pass through LDS together (two blocks' constants and the residual
  // input at once would not fit the registers)
  constexpr int SB = E == 2 && !RES ? FN : 1;
  // the token tiles of the K loop, and after it the waves' stages of 32 tokens: rows of SB blocks and 16
  // bytes more, so that neighbouring rows lie in other banks
  constexpr int PITCH = SB * 32 * E + 16, STAGE = STAGED ? 32 * PITCH : 0;
  constexpr int TILES = 2 * TM * BK, LDS = TILES > NWAVE * STAGE ? TILES : NWAVE * STAGE;
  __shared__ __align__(16) int8_t smem[LDS];
  int8_t(&sx)[2][TM * BK] = *(int8_t(*)[2][TM * BK])smem;
  __shared__ __align__(16) int smult[TN];
  __shared__ __align__(16) long long sbias[TN];

  const int lin = blockIdx.x;
  const int tile = (lin & 7) * a.per_xcd + (lin >> 3);
  if (tile >= a.tiles_total) return;
  const int K = a.l.K, N = a.l.N, rows = a.rows;
  const int Kw = (K + 31) & ~31, Nw = (N + 31) & ~31;
  const TilePos pos = tile_at(a.grid, tile);
  const int n0 = pos.nt * TN, t0 = pos.mt * TM;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave % WN, wm = wave / WN;
  const int col = lane & 31, half = lane >> 5;
  const int tw0 = t0 + wm * WTM;

  // the tile's constants and the wave's token scales, requested ahead of the first operands
  const int c = min(n0 + min(tid, TN - 1), Nw - 1);
  const int rm = a.l.mult[c];
  const long long rb = a.l.bias[c];
  int sc[FM];
#pragma unroll
  for (int j = 0; j < FM; ++j) sc[j] = a.s[min(tw0 + j * 32 + col, rows - 1)];

  const __amdgpu_buffer_rsrc_t wres = __builtin_amdgcn_make_buffer_rsrc((void*)a.l.w, (short)0, Nw * Kw, BUF_WORD3);
  const __amdgpu_buffer_rsrc_t xres = __builtin_amdgcn_make_buffer_rsrc((void*)(a.q + (size_t)t0 * K), (short)0,
                                                                        min(rows - t0, TM) * K, BUF_WORD3);
  v16i acc[FN][FM];
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int j = 0; j < FM; ++j) acc[i][j] = (v16i){};
  gemm_kloop<TN, TM, NWAVE, WN, false>(sx, wres, xres, K, Kw, Nw, lane, wm, loop_place(tid, K, n0 + wn * WTN), acc, [&]() {
    if (tid < TN) {
      smult[tid] = rm;
      sbias[tid] = rb;
    }
  });

  const int pre = a.l.pre, post = a.l.shift - 32;
  if (STAGED) __syncthreads();  // the token tiles are done with
  // a stage's 16-byte pieces: the lane's row pr and piece pc of the first of the passes over its rows
  constexpr int CH = 2 * E * SB, RP = STAGED ? 64 / CH : 32;
  const int pr = STAGED ? lane / CH : col, pc = STAGED ? lane % CH : half;
  int8_t* stage = smem + wave * STAGE;
#pragma unroll
  for (int i0 = 0; i0 < FN; i0 += SB) {
    const int nl = wn * WTN + i0 * 32;  // first channel of these blocks, tile-local
    if (n0 + nl >= N) continue;
    const int c0 = n0 + nl + pc * (16 / E);  // first channel of this lane's piece
    const int left = N - c0;
    int m[SB][16];
    long long b[SB][16];
#pragma unroll
    for (int k = 0; k < SB; ++k)
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          m[k][4 * g + e] = smult[nl + k * 32 + g * 8 + half * 4 + e];
          b[k][4 * g + e] = sbias[nl + k * 32 + g * 8 + half * 4 + e];
        }
#pragma unroll
    for (int j = 0; j < FM; ++j) {
      const int tj = tw0 + j * 32;
      uint32_t Z[4];  // int8: the residual's bytes of each group
      if constexpr (RES && STAGED) {
#pragma unroll
        for (int p = 0; p < 32 / RP; ++p) {
          const int r = p * RP + pr;
          if (tj + r < rows)
            *(v4i*)(stage + r * PITCH + pc * 16) = load_piece<T>((const T*)a.z + (size_t)(tj + r) * N + c0, left);
        }
        wave_order();
      } else if constexpr (RES) {
        const v4i z = tj + col < rows ? load_piece<T>((const T*)a.z + (size_t)(tj + col) * N + c0, left) : (v4i){0, 0, 0, 0};
        exchange(z, Z);
      }
      uint32_t D[4];
#pragma unroll
      for (int k = 0; k < SB; ++k)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          int8_t* at = stage + col * PITCH + (k * 32 + g * 8 + half * 4) * E;
          int o[4], zv[4];
          if constexpr (RES && STAGED) get4(*(const uint2*)at, zv);
          else if constexpr (RES) get4(Z[g], zv);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = __mulhi(acc[i0 + k][j][4 * g + e] << pre, sc[j]);
            long long v = (long long)t * m[k][4 * g + e] + b[k][4 * g + e];
            if constexpr (RES) v += (long long)(zv[e] << 16) * a.l.m_z;
            o[e] = min(max((int)(v >> 32) >> post, -LIM), LIM);
          }
          if constexpr (E == 4) *(v4i*)at = (v4i){o[0], o[1], o[2], o[3]};
          else if constexpr (E == 2) *(uint2*)at = make_uint2(pack16(o[0], o[1]), pack16(o[2], o[3]));
          else D[g] = pack8(o[0], o[1], o[2], o[3]);
        }
      if constexpr (STAGED) {
        wave_order();
#pragma unroll
        for (int p = 0; p < 32 / RP; ++p) {
          const int r = p * RP + pr;
          if (tj + r < rows)
            store_piece<T, PASSING>((T*)a.y + (size_t)(tj + r) * N + c0, *(const v4i*)(stage + r * PITCH + pc * 16),
                                    left);
        }
        wave_order();
      } else {
        const v4i out = exchange(D);
        if (tj + col < rows) store_piece<T>((T*)a.y + (size_t)(tj + col) * N + c0, out, left);
      }
    }
  }
}

// Few tokens: a workgroup of eight waves computes 32 channels x 32 tokens, of which the first 8 XR are
// loaded, the waves sharing out the contraction in steps of 128 bytes.  A wave's weights come straight
// from memory, its token rows in whole cache lines through a piece of LDS of its own, so no barrier is
// needed until the waves' sums meet in LDS.  (As fragments straight from memory, 32 bytes of each row at a
// time, the rows' loads bound the kernel: 125 x 4096 -> 1024 7.2 us instead of 5.2.)  Then each thread
// adds the eight sums of four channels of a token and finishes them.  What bounds it is latency: the
// launch, one trip to memory, two barriers; 1 token x 4096 -> 4096 reads its 16 MB of weights in 4.1 us.
constexpr int FEW_WAVES = 8;

template <int XR, typename T, bool RES>
__global__ __launch_bounds__(64 * FEW_WAVES) void token_linear_few(TokenLinearArgs a) {
  constexpr int LIM = (int)((1u << (8 * sizeof(T) - 1)) - 1);
  constexpr int PITCH = 36;    // dwords of a token's 32 channels: neighbouring rows in other banks
  constexpr int XT = 32 * BK, PT = FEW_WAVES * 32 * PITCH * 4;
  __shared__ __align__(16) int8_t smem[FEW_WAVES * XT > PT ? FEW_WAVES * XT : PT];
  const int mt = (int)div_u(blockIdx.x, a.dv_n), nt = (int)blockIdx.x - mt * (int)a.dv_n.d;
  const int K = a.l.K, N = a.l.N, rows = a.rows;
  const int KS = (K + 31) >> 5, n0 = nt * 32, t0 = mt * 32;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const __amdgpu_buffer_rsrc_t wres =
      __builtin_amdgcn_make_buffer_rsrc((void*)(a.l.w + (size_t)nt * KS * 1024), (short)0, KS * 1024, BUF_WORD3);
  const __amdgpu_buffer_rsrc_t xres = __builtin_amdgcn_make_buffer_rsrc((void*)(a.q + (size_t)t0 * K), (short)0,
                                                                        min(rows - t0, 32) * K, BUF_WORD3);
  const int steps = (K + BK - 1) / BK, per = (steps + FEW_WAVES - 1) / FEW_WAVES;
  const int k0 = wave * per, k1 = min(k0 + per, steps);
  int8_t* sx = smem + wave * XT;
  const int frow = lane >> 3, fchunk = lane & 7;
  v16i acc = (v16i){};
  // B steps, all their loads requested at once (no load is sent that is not needed: also one that
  // reads nothing holds up the CU's load path)
  auto batch = [&](int k, auto count) {
    constexpr int B = decltype(count)::value;
    v4i wf[B][4], xf[B][XR];
#pragma unroll
    for (int i = 0; i < B; ++i) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        wf[i][u] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(wres, lane * 16, min((k + i) * 4 + u, KS - 1) * 1024, 0);
      // bytes past a row's end read as zeros, so that weights there (the last slice again) do not
      // matter; what stands for a token that is not there reaches its own outputs alone
      const int kb = (k + i) * BK + fchunk * 16;
#pragma unroll
      for (int r = 0; r < XR; ++r)
        xf[i][r] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(xres, kb < K ? (frow + 8 * r) * K + kb : 0x7f000000, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < B; ++i) {
#pragma unroll
      for (int r = 0; r < XR; ++r) *(v4i*)(sx + lds_off(frow + 8 * r, fchunk)) = xf[i][r];
      wave_order();
#pragma unroll
      for (int u = 0; u < 4; ++u)
        acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[i][u], *(const v4i*)(sx + lds_off(col, 2 * u + half)), acc, 0, 0, 0);
      wave_order();
    }
  };
  // this thread's four outputs and their constants
  const int tok = tid >> 3, c0 = n0 + (tid & 7) * 4;
  const bool mine = tok < 32 && t0 + tok < rows && c0 < N;
  int m[4], sc = 0;
  long long b[4];
  if (mine) {
    sc = a.s[t0 + tok];
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // padded to a multiple of 32 channels
      m[e] = a.l.mult[c0 + e];
      b[e] = a.l.bias[c0 + e];
    }
  }
  int k = k0;
  for (; k + 4 <= k1; k += 4) batch(k, std::integral_constant<int, 4>{});
  if (k + 2 <= k1) {
    batch(k, std::integral_constant<int, 2>{});
    k += 2;
  }
  if (k < k1) batch(k, std::integral_constant<int, 1>{});
  __syncthreads();
  int(*part)[32][PITCH] = (int(*)[32][PITCH])smem;
#pragma unroll
  for (int g = 0; g < 4; ++g)
    *(v4i*)&part[wave][col][g * 8 + half * 4] = (v4i){acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
  __syncthreads();
  if (!mine) return;
  v4i sum = (v4i){};
#pragma unroll
  for (int w = 0; w < FEW_WAVES; ++w) sum += *(const v4i*)&part[w][tok][(tid & 7) * 4];
  const size_t at = (size_t)(t0 + tok) * N + c0;
  T* y = (T*)a.y + at;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (c0 + e >= N) break;
    const int t = __mulhi(sum[e] << a.l.pre, sc);
    long long v = (long long)t * m[e] + b[e];
    if (RES) v += (long long)((int)((const T*)a.z)[at + e] << 16) * a.l.m_z;
    y[e] = (T)min(max((int)(v >> 32) >> (a.l.shift - 32), -LIM), LIM);
  }
}

template <typename T, bool RES>
static hipError_t launch_few(TokenLinearArgs& a, uint32_t nt, uint32_t mt, hipStream_t st) {
  a.dv_n = make_div(nt);
  const dim3 grid(nt * mt), block(64 * FEW_WAVES);
  if (a.rows <= 8) hipLaunchKernelGGL((token_linear_few<1, T, RES>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((token_linear_few<4, T, RES>), grid, block, 0, st, a);
  return hipGetLastError();
}

template <int I, typename T, bool RES>
static hipError_t launch_tiles(TokenLinearArgs& a, hipStream_t st) {
  constexpr TileShape s = kTiles[I];
  constexpr int NWAVE = s.tm == 256 ? 8 : 4;
  a.grid = tile_grid(1, a.rows, a.l.N, s.tn, s.tm);
  a.tiles_total = a.grid.tiles_n * a.grid.tiles_m;
  a.per_xcd = (a.tiles_total + 7) / 8;
  const dim3 grid(8 * a.per_xcd), block(64 * NWAVE);
  // Outputs of 16 and 32 bits leave past the caches, not to push the operands out of them, where their rows
  // are whole cache lines and they are more than the caches would keep for the next call.  Calls alone,
  // past the caches and not, in us: 6000 x 1024 -> 4096 to int16 32.2 / 34.2, 23000 x 1024 -> 4096 113 / 120, 4200 x
  // 1024 -> 1024 to int32 11.2 / 12.7; also where a wave's run is half a line, as in int16 with the residual input (6000 x
  // 1024 -> 4096 44.9 / 58.5, 23000 x 4096 -> 1024 116 / 117) and in int16 from tiles of 64 and 128 channels (3000 x
  // 1024 -> 2048 12.0 / 13.5, 17000 x 256 -> 256 6.4 / 6.9): 1 to 26 % in each of 39 calls of 8 MiB and more.  But 23000
  // x 256 -> 300 to int32, rows of 9.4 lines, 17.1 / 11.4, and int8 rows, runs of 32 bytes, 23000 x 4096 -> 1024 103 / 100.
  // A call that reads them next pays some of it back: with the token quantization 7 % less to 5 % more time for both
  // (less in 28 of 39; 6000 x 1024 -> 4096 44.5 / 44.9), with a group norm 3 % less to 8 % more (more in 17 of 26;
  // 71.4 / 68.7, and 41.1 / 41.3 for 6000 x 4096 -> 1024); below 8 MiB it is more (500 x 1024 -> 1024 to int16 and
  // quantization 6.6 / 6.4).
  const size_t row_bytes = (size_t)a.l.N * sizeof(T);
  const bool passing = row_bytes % 128 == 0 && (uintptr_t)a.y % 128 == 0 && row_bytes * a.rows >= ((size_t)8 << 20);
  if constexpr (sizeof(T) > 1)
    if (passing) {
      hipLaunchKernelGGL((token_linear<s.tn, s.tm, NWAVE, s.tn == 64 ? 2 : 4, T, RES, true>), grid, block, 0, st, a);
      return hipGetLastError();
    }
  hipLaunchKernelGGL((token_linear<s.tn, s.tm, NWAVE, s.tn == 64 ? 2 : 4, T, RES, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

template <typename T, bool RES>
static hipError_t launch_shape(TokenLinearArgs& a, hipStream_t st) {
  // as long as each CU gets one of their workgroups: 1 token x 1024 -> 1024 2.7 us against 3.6 us in tiles,
  // 1 x 4096 -> 1024 3.5 against 7.1, 125 x 4096 -> 1024 (128 workgroups) 5.2 against 7.6, 250 x 4096 -> 1024
  // (256) 5.7 against 7.7; above, 250 x 2048 -> 2048 (512) 5.8 against 5.4.  (Sixteen waves a workgroup are
  // slower by 0.2 - 0.3 us up to K = 4096.)
  const uint32_t nt = (uint32_t)(a.l.N + 31) / 32, mt = (uint32_t)(a.rows + 31) / 32;
  if ((uint64_t)nt * mt <= kGemmCUs) return launch_few<T, RES>(a, nt, mt, st);
  const GemmDims dims{1, a.rows, a.l.N};
  switch (pick_shape(&dims, 1, a.l.K, 32, EPI_TOKEN)) {
    case 0: return launch_tiles<0, T, RES>(a, st);
    case 1: return launch_tiles<1, T, RES>(a, st);
    case 2: return launch_tiles<2, T, RES>(a, st);
    case 3: return launch_tiles<3, T, RES>(a, st);
    case 4: return launch_tiles<4, T, RES>(a, st);
    default: return launch_tiles<5, T, RES>(a, st);
  }
}

hipError_t launch_token_linear(const TokenLinear& l, const int8_t* q, const int32_t* s, int rows, const void* z,
                               void* y, hipStream_t st) {
  TokenLinearArgs a{};
  a.l = l;
  a.q = q;
  a.s = s;
  a.z = z;
  a.y = y;
  a.rows = rows;
  if (l.out_bytes == 4) return launch_shape<int32_t, false>(a, st);
  if (l.out_bytes == 2) return z ? launch_shape<int16_t, true>(a, st) : launch_shape<int16_t, false>(a, st);
  return z ? launch_shape<int8_t, true>(a, st) : launch_shape<int8_t, false>(a, st);
}

}  // namespace ipk
