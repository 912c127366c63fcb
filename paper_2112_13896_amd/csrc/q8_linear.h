// y[t][n] = (sum_k x[t][k] w[n][k]) * (sx[t] * sw[n]) + bias[n] for int8 x and
// w: the sum in int32 (exact: k <= 131,072), one rounding to y's type.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "q8_places.h"
#include "q8_rows.h"

namespace cs {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

struct Q8Linear {
  const int8_t* x;
  int64_t ldx;
  const float* sx;
  int64_t rows;
  int k;
  const int8_t* w;
  int64_t ldw;
  const float* sw;
  int d_out;
  const float* bias;
  void* y;
  int64_t ldy;
  int y_vec;           // rows of y start on 16 bytes
};

// 16 codes of a row from element e on; those past k read as 0.  The row starts
// on 16 bytes.  `inner`: it is not the matrix's last, so that its bytes up to a
// multiple of 16 are the matrix's own and can be loaded.
__device__ __forceinline__ i32x4 codes16(const int8_t* row, int e, int k, bool inner) {
  i32x4 v = {0, 0, 0, 0};
  if (e >= k) return v;
  if (inner || e + 16 <= k) {
    v = *reinterpret_cast<const i32x4*>(row + e);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int keep = k - e - 4 * i;                      // bytes of the dword before k
      if (keep < 4) v[i] = keep <= 0 ? 0 : v[i] & (int)((1u << (8 * keep)) - 1);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (e + i < k) v[i / 4] |= (int)((uint32_t)(uint8_t)row[e + i] << (8 * (i % 4)));
  }
  return v;
}

// The same of a row that starts anywhere.
__device__ __forceinline__ i32x4 codes16_any(const int8_t* row, int e, int k) {
  i32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (e + i < k) v[i / 4] |= (int)((uint32_t)(uint8_t)row[e + i] << (8 * (i % 4)));
  return v;
}

// linear_q8_any: rows that start anywhere.  A 64 x 64 tile of y to a
// workgroup of four wavefronts, 32 x 32 each, 64 codes of k a step through
// registers and LDS, 16 bytes a thread and operand put together from single
// ones, which is what bounds it (the simplest kernel that is right for any row;
// padding rows to 16 bytes, as quantise_rows does, avoids it).
template <typename T>
__global__ __launch_bounds__(256) void linear_q8_any(Q8Linear a) {
  constexpr int kLd = 64 + 16;                             // a row's bytes in LDS, padded
  __shared__ __align__(16) int8_t lx[64 * kLd], lw[64 * kLd];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int64_t t0 = (int64_t)workgroup() * 64;
  const int n0 = blockIdx.z * 64;
  const int sr = tid / 4, sc = tid % 4 * 16;               // the piece this thread stages
  const int64_t xt = min(t0 + sr, a.rows - 1);
  const int wn = min(n0 + sr, a.d_out - 1);
  const int8_t* xr = a.x + xt * a.ldx;
  const int8_t* wr = a.w + (int64_t)wn * a.ldw;
  const int tr = wave / 2 * 32, nc = wave % 2 * 32;
  const int fr = lane % 32, fk = lane / 32 * 16;
  i32x16 acc = {};
  for (int k0 = 0; k0 < a.k; k0 += 64) {
    const i32x4 vx = codes16_any(xr, k0 + sc, a.k);
    const i32x4 vw = codes16_any(wr, k0 + sc, a.k);
    __syncthreads();
    *reinterpret_cast<i32x4*>(lx + sr * kLd + sc) = vx;
    *reinterpret_cast<i32x4*>(lw + sr * kLd + sc) = vw;
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < 64; kk += 32)
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(
          *reinterpret_cast<const i32x4*>(lx + (tr + fr) * kLd + kk + fk),
          *reinterpret_cast<const i32x4*>(lw + (nc + fr) * kLd + kk + fk), acc, 0, 0, 0);
  }
  const int n = n0 + nc + lane % 32;
  if (n >= a.d_out) return;
  const float s = a.sw[n], b = a.bias ? a.bias[n] : 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int64_t t = t0 + tr + 8 * (i / 4) + 4 * (lane / 32) + i % 4;
    if (t < a.rows)
      static_cast<T*>(a.y)[t * a.ldy + n] = (T)fmaf((float)acc[i], a.sx[t] * s, b);
  }
}

// linear_q8_tile: a BM x BN tile of y to a workgroup, WM x WN of it to a
// wavefront in 32 x 32 products, 128 codes of k a step.  Codes go from memory
// straight into LDS, 16 bytes a lane, NB - 1 steps ahead of the products, with
// NB buffers and one barrier a step.  A row's eight 16-byte chunks are permuted
// (chunk_turn) so that the sixteen lanes served together when a column of
// chunks is read meet all 64 banks (with row % 8 alone, every such read took
// half as long again); as LDS receives a wavefront's load in lane order, the
// permutation is made in the addresses it loads from.  Rows past the end
// repeat the last one and are not stored; the codes past the last whole 128 go
// through registers, zeros after k.
// The products are w times x: a lane then holds four neighbouring channels of
// one token, which go through LDS (free by then), 32 tokens of a wavefront at a
// time, to be stored as whole rows of its tile, 16 bytes a lane (with two-byte
// stores and each row's scale loaded beside them, a tile's end took as long as
// a third of its products: 315 us for the case below).
// 256 x 256 with eight wavefronts, two buffers (128 KB): 8,192 x 4,096 x 8,192
// in 286 us, 252 at best, 1.9-2.2 POP/s (a library int8 product of that size: 2.4-2.5).  Matrix
// instructions issue half of the time; of a step of 128 codes a fifth is the
// wait for its loads, and a tile's start and end, which nothing overlaps, are a
// fifth of the whole.  64 x 64, four wavefronts, four buffers: 777 x 1,500 x 1,001 in
// 10 us, 0.3 us a step, which is the latency of twelve dependent steps.
struct TileOrder {
  uint32_t tiles_m, tiles_n, per_xcd, more;                // tiles / 8, tiles % 8
};

// The tile of a workgroup: workgroups go to the eight XCDs in turn, and each
// XCD (its L2) takes consecutive tiles, in columns of four rows of tiles.
__device__ __forceinline__ void place_tile(const TileOrder& o, uint32_t id, int* tm, int* tn) {
  const uint32_t x = id % 8, i = id / 8;
  const uint32_t tile = x * o.per_xcd + min(x, o.more) + i;
  const uint32_t band = 4 * o.tiles_n;
  const uint32_t b = tile / band, in = tile - b * band;
  const uint32_t rows = min(4u, o.tiles_m - 4 * b);
  *tn = (int)(in / rows);
  *tm = (int)(4 * b + in - *tn * rows);
}

typedef __attribute__((address_space(1))) const void gvoid;
typedef __attribute__((address_space(3))) void lvoid;

template <int ROWS, int THREADS>
__device__ __forceinline__ void codes_to_lds(const int8_t* base,
                                             const uint32_t (&off)[ROWS * 8 / THREADS], int k0,
                                             int8_t* lds) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
  for (int p = 0; p < ROWS * 8 / THREADS; ++p)
    __builtin_amdgcn_global_load_lds((gvoid*)(base + k0 + off[p]),
                                     (lvoid*)(lds + (p * THREADS + wave * 64) * 16), 16, 0, 0);
}

// All but the last N of this wavefront's loads have landed, its LDS reads are
// done, and so are the other wavefronts'.
template <int N>
__device__ __forceinline__ void landed() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <typename T, int BM, int BN, int WM, int WN, int NB>
__global__ __launch_bounds__(BM / WM * (BN / WN) * 64, 2) void linear_q8_tile(Q8Linear a,
                                                                             TileOrder order) {
  constexpr int NW = BN / WN, THREADS = BM / WM * NW * 64;
  constexpr int MT = WM / 32, NT = WN / 32;
  constexpr int PX = BM * 8 / THREADS, PW = BN * 8 / THREADS;
  // (variables of their own: the compiler then knows that a load into one is not read in another)
  __shared__ __align__(16) int8_t lx0[BM * 128], lx1[BM * 128], lw0[BN * 128], lw1[BN * 128];
  __shared__ __align__(16) int8_t lx2[NB > 2 ? BM * 128 : 16], lw2[NB > 2 ? BN * 128 : 16];
  __shared__ __align__(16) int8_t lx3[NB > 2 ? BM * 128 : 16], lw3[NB > 2 ? BN * 128 : 16];
  static_assert(NB == 2 || NB == 4, "");
  __shared__ __align__(16) float l_sw[BN], l_bias[BN];
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  int tm, tn;
  place_tile(order, blockIdx.x, &tm, &tn);
  const int64_t t0 = (int64_t)tm * BM;
  const int n0 = tn * BN;
  const int8_t* xb = a.x + t0 * a.ldx;
  const int8_t* wb = a.w + (int64_t)n0 * a.ldw;
  const int xrows = (int)min<int64_t>(BM, a.rows - t0), wrows = min(BN, a.d_out - n0);
  // the row and chunk that the 16-byte piece of a buffer holds
  uint32_t xo[PX], wo[PW];
#pragma unroll
  for (int p = 0; p < PX; ++p) {
    const int piece = p * THREADS + tid, row = TilePlaces::row(piece);
    xo[p] = (uint32_t)min(row, xrows - 1) * (uint32_t)a.ldx + TilePlaces::chunk(piece) * 16;
  }
#pragma unroll
  for (int p = 0; p < PW; ++p) {
    const int piece = p * THREADS + tid, row = TilePlaces::row(piece);
    wo[p] = (uint32_t)min(row, wrows - 1) * (uint32_t)a.ldw + TilePlaces::chunk(piece) * 16;
  }
  const int mr = wave / NW * WM, nr = wave % NW * WN;
  const int fr = lane % 32, fh = lane / 32;
  i32x16 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[m][n][i] = 0;
  // The next 32 codes' operands are read under this 32's products, one read to a product: left
  // to itself the compiler reads all of them just before their use.
  auto multiply = [&](const int8_t* lx, const int8_t* lw) {
    i32x4 fx[2][MT], fw[2][NT];
    auto read = [&](int s) {
      const int at = TilePlaces::at(fr, s, fh);
#pragma unroll
      for (int m = 0; m < MT; ++m)
        fx[s & 1][m] = *reinterpret_cast<const i32x4*>(lx + (mr + 32 * m) * 128 + at);
#pragma unroll
      for (int n = 0; n < NT; ++n)
        fw[s & 1][n] = *reinterpret_cast<const i32x4*>(lw + (nr + 32 * n) * 128 + at);
    };
    read(0);
    __builtin_amdgcn_sched_group_barrier(0x100, MT + NT, 0);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s < 3) read(s + 1);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          acc[m][n] =
              __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[s & 1][n], fx[s & 1][m], acc[m][n], 0, 0, 0);
      if (s < 3) {
#pragma unroll
        for (int i = 0; i < MT * NT; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          if (i < MT + NT) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
      } else {
        __builtin_amdgcn_sched_group_barrier(0x008, MT * NT, 0);
      }
    }
  };
  for (int i = tid; i < BN; i += THREADS) {
    const int o = min(n0 + i, a.d_out - 1);
    l_sw[i] = a.sw[o];
    l_bias[i] = a.bias ? a.bias[o] : 0.0f;
  }
  float sx[MT];                                            // of the lane's tokens
#pragma unroll
  for (int m = 0; m < MT; ++m) sx[m] = a.sx[min<int64_t>(t0 + mr + 32 * m + fr, a.rows - 1)];
  const int whole = a.k / 128;
  // step s's codes into buffer B; past the last step its codes again, into a buffer that nobody
  // reads any more, so that every step counts as many loads
  auto fetch = [&](auto buffer, int s) {
    constexpr int B = decltype(buffer)::value;
    const int k0 = min(s, whole - 1) * 128;
    codes_to_lds<BM, THREADS>(xb, xo, k0, B == 0 ? lx0 : B == 1 ? lx1 : B == 2 ? lx2 : lx3);
    codes_to_lds<BN, THREADS>(wb, wo, k0, B == 0 ? lw0 : B == 1 ? lw1 : B == 2 ? lw2 : lw3);
  };
  auto step = [&](auto buffer, int s) {
    constexpr int B = decltype(buffer)::value;
    landed<(NB - 2) * (PX + PW)>();
    fetch(std::integral_constant<int, (B + NB - 1) % NB>{}, s + NB - 1);
    multiply(B == 0 ? lx0 : B == 1 ? lx1 : B == 2 ? lx2 : lx3,
             B == 0 ? lw0 : B == 1 ? lw1 : B == 2 ? lw2 : lw3);
  };
  if (whole > 0) {
    fetch(std::integral_constant<int, 0>{}, 0);
    if constexpr (NB > 2) {
      fetch(std::integral_constant<int, 1>{}, 1);
      fetch(std::integral_constant<int, 2>{}, 2);
    }
  }
  for (int s = 0; s < whole; s += NB) {
    step(std::integral_constant<int, 0>{}, s);
    if (s + 1 >= whole) break;
    step(std::integral_constant<int, 1>{}, s + 1);
    if constexpr (NB > 2) {
      if (s + 2 >= whole) break;
      step(std::integral_constant<int, 2>{}, s + 2);
      if (s + 3 >= whole) break;
      step(std::integral_constant<int, 3>{}, s + 3);
    }
  }
  landed<0>();
  if (a.k % 128 != 0) {
    const int k0 = whole * 128;
#pragma unroll
    for (int p = 0; p < PX; ++p) {
      const int piece = p * THREADS + tid, row = min(TilePlaces::row(piece), xrows - 1);
      *reinterpret_cast<i32x4*>(lx0 + piece * 16) =
          codes16(xb + (int64_t)row * a.ldx, k0 + TilePlaces::chunk(piece) * 16, a.k,
                  t0 + row + 1 < a.rows);
    }
#pragma unroll
    for (int p = 0; p < PW; ++p) {
      const int piece = p * THREADS + tid, row = min(TilePlaces::row(piece), wrows - 1);
      *reinterpret_cast<i32x4*>(lw0 + piece * 16) =
          codes16(wb + (int64_t)row * a.ldw, k0 + TilePlaces::chunk(piece) * 16, a.k,
                  n0 + row + 1 < a.d_out);
    }
    __syncthreads();
    multiply(lx0, lw0);
  }
  __syncthreads();                                         // the last operands have been read
  constexpr int kRow = WN * (int)sizeof(T) + 16;           // a token's bytes in LDS, padded
  constexpr int kShare = THREADS / 64 / 4;                 // wavefronts to a buffer
  static_assert(kShare * 32 * kRow <= BM * 128 && kShare * 32 * kRow <= BN * 128, "");
  const int buf = wave / kShare;
  int8_t* out =
      (buf == 0 ? lx0 : buf == 1 ? lx1 : buf == 2 ? lw0 : lw1) + wave % kShare * 32 * kRow;
  constexpr int E = 16 / sizeof(T), kPieces = WN / E;      // elements of 16 bytes, pieces of a row
  typedef T t4 __attribute__((ext_vector_type(4)));
  const int nvalid = a.d_out - n0 - nr;                    // channels of the wavefront's tile
#pragma unroll
  for (int m = 0; m < MT; ++m) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int ch = 32 * n + 8 * y + 4 * fh;
        const f32x4 sw = *reinterpret_cast<const f32x4*>(l_sw + nr + ch);
        const f32x4 bias = *reinterpret_cast<const f32x4*>(l_bias + nr + ch);
        t4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          v[i] = (T)fmaf((float)acc[m][n][4 * y + i], sx[m] * sw[i], bias[i]);
        *reinterpret_cast<t4*>(out + fr * kRow + ch * sizeof(T)) = v;
      }
    wave_lds_order();
#pragma unroll
    for (int p = lane; p < 32 * kPieces; p += 64) {
      const int tok = p / kPieces, e = p % kPieces * E;
      const int64_t t = t0 + mr + 32 * m + tok;
      if (t >= a.rows) continue;
      T* y = static_cast<T*>(a.y) + t * a.ldy + n0 + nr + e;
      const u32x4 v = *reinterpret_cast<const u32x4*>(out + tok * kRow + e * sizeof(T));
      if (a.y_vec && e + E <= nvalid) {
        *reinterpret_cast<u32x4*>(y) = v;
      } else {
        T el[E];
        __builtin_memcpy(el, &v, 16);
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (e + i < nvalid) y[i] = el[i];
      }
    }
    wave_lds_order();
  }
}

// linear_q8_few: few tokens, where reading w is the work.  16 output channels
// to a workgroup of NW wavefronts, which take 128 codes of k in turn: a lane
// loads 32 bytes of a row of w (the four lanes of a row 128 bytes together),
// kept in flight four such steps deep, and multiplies them with RT tiles of 16
// tokens, read the same way (the order of k inside a product only has to agree).
// The wavefronts' int32 sums meet in LDS.  XT int8_t: tokens in codes.  A
// float XT: every workgroup quantises the tokens itself, into LDS, while its
// first loads of w are under way; that is one launch instead of two.
// Bound by latency where w is small (1 x 512 x 512, quantised here: 4.4 us) and by
// reading w where it is not (1 x 8,192 x 8,192: 15.6 us, 4.3 TB/s).
constexpr int kFewSteps = 4;

template <typename T, typename XT, int RT, int NW>
__global__ __launch_bounds__(NW * 64) void linear_q8_few(Q8Linear a) {
  constexpr bool kFloats = sizeof(XT) > 1;
  extern __shared__ __align__(16) int8_t l_x[];            // floats: [rows][kpad] codes
  __shared__ int l_sum[NW][RT][16][17];
  __shared__ uint32_t l_max[16];
  __shared__ float l_sx[16];
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int r = lane % 16, h = lane / 16;
  const int n0 = blockIdx.x * 16, steps = (a.k + 127) / 128, kpad = steps * 128;
  const int8_t* wr = a.w + (int64_t)min(n0 + r, a.d_out - 1) * a.ldw;
  const bool w_inner = n0 + r + 1 < a.d_out;
  i32x4 w[kFewSteps][2];
  auto load_w = [&](int s0) {
#pragma unroll
    for (int i = 0; i < kFewSteps; ++i) {
      const int s = s0 + i * NW, e = s * 128 + 32 * h;
      if (s >= steps) continue;
#pragma unroll
      for (int y = 0; y < 2; ++y)
        w[i][y] = s + 1 < steps ? *reinterpret_cast<const i32x4*>(wr + e + 16 * y)
                                : codes16(wr, e + 16 * y, a.k, w_inner);
    }
  };
  load_w(wave);
  if constexpr (kFloats) {
    // quantise_rows' arithmetic; whole wavefronts share a row's vectors of eight
    const XT* x = reinterpret_cast<const XT*>(a.x);
    const bool vec = (reinterpret_cast<uintptr_t>(x) & 15) == 0 &&
                     (a.rows == 1 || a.ldx * sizeof(XT) % 16 == 0);
    const int rows = (int)a.rows, nv = kpad / 8;
    // rows below NW: NW / rows wavefronts to a row; else a wavefront to every NW-th row
    const int per = max(1, NW / rows), first = wave / per, stride = NW / per;
    auto fetch = [&](int row, int v, float (&f)[8]) {
      const XT* p = x + row * a.ldx + 8 * v;
      if (vec && 8 * v + 8 <= a.k) load8(p, f);
      else load8_some(p, a.k - 8 * v, f);
    };
    const int l0 = wave % per * 64 + lane, lanes = per * 64;
    if (tid < 16) l_max[tid] = 0;
    __syncthreads();
    for (int row = first; row < rows; row += stride) {
      uint32_t top = 0;
      for (int v = l0; v < nv; v += lanes) {
        float f[8];
        fetch(row, v, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, abs_bits(f[i]));
      }
      top = wave_max_u32(top);
      if (lane == 0) atomicMax(&l_max[row], top);
    }
    __syncthreads();
    for (int row = first; row < rows; row += stride) {
      const RowScale rs = row_scale(l_max[row]);
      if (l0 == 0) l_sx[row] = rs.s;
      for (int v = l0; v < nv; v += lanes) {
        float f[8];
        fetch(row, v, f);
        *reinterpret_cast<u32x2*>(l_x + row * kpad + 8 * v) = row_codes8(f, rs);
      }
    }
    __syncthreads();
  }
  i32x4 acc[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[t] = i32x4{0, 0, 0, 0};
  for (int s0 = wave; s0 < steps; s0 += kFewSteps * NW) {
    if (s0 != wave) load_w(s0);
#pragma unroll
    for (int i = 0; i < kFewSteps; ++i) {
      const int s = s0 + i * NW, e = s * 128 + 32 * h;
      if (s >= steps) continue;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const int row = min(16 * t + r, (int)a.rows - 1);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          i32x4 x;
          if constexpr (kFloats)
            x = *reinterpret_cast<const i32x4*>(l_x + row * kpad + e + 16 * y);
          else if (s + 1 < steps)
            x = *reinterpret_cast<const i32x4*>(a.x + row * a.ldx + e + 16 * y);
          else
            x = codes16(a.x + row * a.ldx, e + 16 * y, a.k, row + 1 < a.rows);
          acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i][y], x, acc[t], 0, 0, 0);
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) l_sum[wave][t][r][4 * h + i] = acc[t][i];
  __syncthreads();
  for (int i = tid; i < RT * 256; i += NW * 64) {
    const int row = i / 16, n = i % 16, o = n0 + n;
    if (row >= a.rows || o >= a.d_out) continue;
    int sum = 0;
#pragma unroll
    for (int v = 0; v < NW; ++v) sum += l_sum[v][row / 16][row % 16][n];
    const float sx = kFloats ? l_sx[row % 16] : a.sx[row];
    static_cast<T*>(a.y)[row * a.ldy + o] =
        (T)fmaf((float)sum, sx * a.sw[o], a.bias ? a.bias[o] : 0.0f);
  }
}

}  // namespace cs
