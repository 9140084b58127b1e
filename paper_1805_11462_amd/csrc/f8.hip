// Matrix product in 8-bit floating point (e4m3) with a power of two for every block of 128 columns of a row.
//
// A block whose largest finite entry is a = f 2^p (1 <= f < 2) is stored as q = e4m3(x 2^-e), rounded to nearest even, with
// e = p - 8 where f <= 1.75 and p - 7 else: the smallest power that brings a to 448, e4m3's largest value, or less. An entry is
// off by at most half an e4m3 step, 2^-4 of its value, down to 2^-13 of the block's largest (2^-10 2^e below). A power of two
// costs no accuracy against a scale of full precision (the steps of a floating-point type move with it), and the
// matrix instruction takes it as an operand: v_mfma_scale_f32_16x16x128_f8f6f4 multiplies one 128-column block of 16 rows of either
// side and scales it by 2^(ex + ew) of its rows and columns, at twice the rate of the 16-bit ones. But it aligns the 128 products
// to the largest before it adds them and drops what falls below some 17 bits: sums of normal values are off by 1.5e-5 of their
// rms (measured; 16x16x32_fp8_fp8 the same), which 16-bit results do not see (their own rounding is up to 2^-8 or 2^-11) and fp32 results do.
// Those multiply the same e4m3 values as bf16, exact with their powers included (v_cvt_scalef32_pk_bf16_fp8), in
// v_mfma_f32_16x16x32_bf16: 2e-8 to 1e-7.
//
// Operands lie in fragment blocks of 16 rows x 128 columns, 2 KB: lane l of a wave holds row l % 16, columns 32 (l / 16) .. + 31,
// its first 16 bytes at 16 l of the first kilobyte, the others at 16 l of the second. (The instruction's own order of the columns
// does not matter as long as both operands have the same.) Consecutive blocks go down the rows, so that what a tile of rows needs
// of one block of columns is one stretch of memory (along the columns, the stretches of a tile lie a power of two apart for
// many sizes and meet in few of the L2's channels: 8192-cubed took 467 us). Then, behind all blocks, the powers (biased
// by 127), one byte per row and block: blocks 4 j .. 4 j + 3 of a row are a dword, which the instruction picks its byte
// from, the dwords of all rows side by side, then those of the next four blocks.

#include <type_traits>

#include "answer.h"
#include "common.h"
#include "gemm_device.h"
#include "types.h"

namespace onmt {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kF8One = 127;                    // biased power of blocks that hold nothing
constexpr float kF8Most = 0x1.ep127f;          // larger entries count as this, the last value before 2^128: all stay finite

// The power of two of a block whose largest entry is a.
__device__ __forceinline__ int f8_exp(float a) {
  if (!(a > 0.f)) return 0;
  int ex;
  const float m = frexpf(a, &ex);              // a = m 2^ex, m in [0.5, 1)
  return max(ex - 9 + (m > 0.875f ? 1 : 0), -kF8One);
}

// 32 entries times 2^-e as e4m3, entry i in byte i % 4 of word i / 4.
__device__ __forceinline__ void f8_round(const float (&x)[32], int e, i32x4& lo, i32x4& hi) {
  i32x4 q[2];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(ldexpf(x[4 * i], -e), ldexpf(x[4 * i + 1], -e), w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(ldexpf(x[4 * i + 2], -e), ldexpf(x[4 * i + 3], -e), w, true);
    q[i >> 2][i & 3] = w;
  }
  lo = q[0];
  hi = q[1];
}

// Entries k0 .. k0 + 31 of a row of `cols` columns, zeros past them, clamped to finite values.
template <class T>
__device__ __forceinline__ void load32(const T* row, int k0, int cols, float (&v)[32]) {
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = 0.f;
  if (k0 + 32 <= cols) {
#pragma unroll
    for (int i = 0; i < 32; i += kVec<T>) load_vec(row + k0 + i, &v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (k0 + i < cols) v[i] = to_float(row[k0 + i]);
  }
}

// A wave's fragment block from its entries: lo, hi, and the power of the lane's row.
__device__ __forceinline__ int f8_block(float (&v)[32], i32x4& lo, i32x4& hi) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    v[i] = v[i] > kF8Most ? kF8Most : v[i] < -kF8Most ? -kF8Most : v[i];   // NaN stays
    a = fmaxf(a, fabsf(v[i]));                                             // and does not count
  }
  a = fmaxf(a, __shfl_xor(a, 16, kWave));
  a = fmaxf(a, __shfl_xor(a, 32, kWave));
  const int e = f8_exp(a);
  f8_round(v, e, lo, hi);
  return e;
}

// One wave per fragment block.
template <class T>
__global__ __launch_bounds__(256) void k_f8_pack(const T* __restrict__ x, int64_t ld, int rows, int cols, F8Mat out, int nblocks) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (b >= nblocks) return;
  const int rb = b % out.rblocks, kb = b / out.rblocks;
  const int r = rb * 16 + (lane & 15), g = lane >> 4;
  float v[32];
  load32(x + (int64_t)min(r, rows - 1) * ld, kb * kF8Block + 32 * g, r < rows ? cols : 0, v);
  i32x4 lo, hi;
  const int e = f8_block(v, lo, hi);
  char* d = out.data + (size_t)b * kF8Frag + lane * 16;
  *(i32x4*)d = lo;
  *(i32x4*)(d + kF8Frag / 2) = hi;
  if (g == 0) {
    uint8_t* s = (uint8_t*)(out.exps + ((size_t)(kb / 4) * out.rblocks + rb) * 16 + lane);
    s[kb & 3] = (uint8_t)(kF8One + e);
    if (kb == out.kblocks - 1)
      for (int j = (kb & 3) + 1; j < 4; ++j) s[j] = kF8One;
  }
}

__global__ __launch_bounds__(256) void k_f8_unpack(F8Mat w, int rows, int cols, float* __restrict__ out, int64_t ld) {
  const int quads = (cols + 3) / 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)rows * quads; i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i / quads), c = (int)(i % quads) * 4;
    const int rb = r / 16, kb = c / kF8Block, g = c % kF8Block / 32, o = c % 32;
    const int word = *(const int*)(w.data + ((size_t)kb * w.rblocks + rb) * kF8Frag + (o >= 16 ? kF8Frag / 2 : 0) +
                                   (r % 16 + 16 * g) * 16 + o % 16);
    const int e = (int)(((const uint8_t*)(w.exps + ((size_t)(kb / 4) * w.rblocks + rb) * 16 + r % 16))[kb & 3]) - kF8One;
    const float v[4] = {__builtin_amdgcn_cvt_f32_fp8(word, 0), __builtin_amdgcn_cvt_f32_fp8(word, 1),
                        __builtin_amdgcn_cvt_f32_fp8(word, 2), __builtin_amdgcn_cvt_f32_fp8(word, 3)};
    for (int j = 0; j < 4 && c + j < cols; ++j) out[(int64_t)r * ld + c + j] = ldexpf(v[j], e);
  }
}

// ------------------------------------------------------------------------------------------------- products
// The weights are the instruction's row operand: lane (i16, g) ends up with columns 4 g .. + 3 of row i16 of a 16 x 16 tile.

// A lane's 32 values as bf16, times 2^(biased - 127): the operands of four 32-column products.
struct Wide8 {
  bf16x8 q[4];
};
__device__ __forceinline__ Wide8 f8_widen(const i32x8& f, int biased) {
  const float s = __builtin_bit_cast(float, biased << 23);
  Wide8 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    i32x4 p;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      p[2 * h] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * i + h], s, false));
      p[2 * h + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * i + h], s, true));
    }
    w.q[i] = __builtin_bit_cast(bf16x8, p);
  }
  return w;
}

__device__ __forceinline__ i32x8 f8_frag(const char* p) {
  const i32x4 a = *(const i32x4*)p, b = *(const i32x4*)(p + kF8Frag / 2);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// c[x][y] += products of one 128-column block: rows' fragments a[x] and weights' w[y], byte J of their powers.
template <bool EXACT, int J, int TM, int TN>
__device__ __forceinline__ void f8_multiply(f32x4 (&c)[TM][TN], const i32x8 (&a)[TM], const int (&ea)[TM], const i32x8 (&w)[TN],
                                            const int (&ew)[TN]) {
  if constexpr (EXACT) {
    Wide8 ww[TN];
#pragma unroll
    for (int y = 0; y < TN; ++y) ww[y] = f8_widen(w[y], ew[y] >> (8 * J) & 255);
#pragma unroll
    for (int x = 0; x < TM; ++x) {
      const Wide8 aw = f8_widen(a[x], ea[x] >> (8 * J) & 255);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int y = 0; y < TN; ++y) c[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ww[y].q[i], aw.q[i], c[x][y], 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
      for (int y = 0; y < TN; ++y)
        c[x][y] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[y], a[x], c[x][y], 0, 0, J, ew[y], J, ea[x]);
  }
}

template <class T, int N>
struct Packed {
  typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// Four biases from column n on, zeros past N.
__device__ __forceinline__ f32x4 bias4(const float* __restrict__ bias, int N, int n) {
  f32x4 b{0.f, 0.f, 0.f, 0.f};
  if (bias) {
    if (n + 4 <= N) {
      b = *(const Packed<float, 4>::type*)(bias + n);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n + j < N) b[j] = bias[n + j];
    }
  }
  return b;
}

// Few rows (up to 16 TM): the weights' stream is the bound (25.6 MB at 50000 x 500), so each wave loads those of its own 16
// columns straight into registers, four blocks at a time and the next four before it multiplies. The workgroup rounds all rows
// to 8 bits itself, into LDS, while its first weights are on their way: a launch less, and every workgroup reads the rows from
// the caches.
template <class X, class T, int TM>
__global__ __launch_bounds__(256) void k_f8_few(const X* __restrict__ x, int64_t ldx, F8Mat w, int M, int N, int cols,
                                                const float* __restrict__ bias, T* __restrict__ out, int64_t ld) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  constexpr bool EXACT = sizeof(T) == 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g = lane >> 4;
  const int kb = w.kblocks, kq = w.kquads(), nrb = w.rblocks;
  const int nb = min(blockIdx.x * 4 + wave, nrb - 1);
  const char* wp = w.data + (size_t)nb * kF8Frag + lane * 16;
  const int* we = w.exps + (size_t)nb * 16 + i16;
  i32x8 f[2][4];
  int ew[2];
  auto load = [&](int q, i32x8 (&r)[4], int& e) {
    e = we[(size_t)min(q, kq - 1) * nrb * 16];
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = f8_frag(wp + (size_t)min(4 * q + j, kb - 1) * nrb * kF8Frag);
  };
  load(0, f[0], ew[0]);
  const f32x4 b4 = bias4(bias, N, nb * 16 + 4 * g);
  // rows: fragment blocks [kb][TM], then the powers [TM][kq][16] as in a packed matrix; for fp32 results the values as bf16, each
  // lane's four quarters in a kilobyte each (widened once here and not by every wave: 64 rows of 500 by 50000 28.7 us so)
  constexpr int BLK = EXACT ? 2 * kF8Frag : kF8Frag;
  int* le = (int*)(lds + (size_t)kb * TM * BLK);
  for (int b = wave; b < kb * TM; b += 4) {
    const int rb = b % TM, k = b / TM, r = rb * 16 + i16;
    float v[32];
    load32(x + (int64_t)min(r, M - 1) * ldx, k * kF8Block + 32 * g, r < M ? cols : 0, v);
    i32x4 lo, hi;
    const int e = f8_block(v, lo, hi);
    char* d = lds + (size_t)b * BLK + lane * 16;
    if constexpr (EXACT) {
      const Wide8 q = f8_widen(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), kF8One + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) *(bf16x8*)(d + i * 1024) = q.q[i];
      continue;
    }
    *(i32x4*)d = lo;
    *(i32x4*)(d + kF8Frag / 2) = hi;
    if (g == 0) ((uint8_t*)(le + (rb * kq + k / 4) * 16 + i16))[k & 3] = (uint8_t)(kF8One + e);
  }
  __syncthreads();
  f32x4 c[TM][1];
#pragma unroll
  for (int t = 0; t < TM; ++t) c[t][0] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto quad = [&](int q, const i32x8 (&r)[4], int e) {
    int ea[TM];
#pragma unroll
    for (int t = 0; t < TM; ++t) ea[t] = EXACT ? 0 : le[(t * kq + q) * 16 + i16];
    auto step = [&](auto j) {
      constexpr int J = decltype(j)::value;
      const int k = 4 * q + J;
      if (k >= kb) return;
      const char* row = lds + (size_t)k * TM * BLK + lane * 16;
      if constexpr (EXACT) {
        const Wide8 b = f8_widen(r[J], e >> (8 * J) & 255);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int t = 0; t < TM; ++t)
            c[t][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.q[i], *(const bf16x8*)(row + t * BLK + i * 1024), c[t][0], 0, 0, 0);
      } else {
        i32x8 a[TM];
#pragma unroll
        for (int t = 0; t < TM; ++t) a[t] = f8_frag(row + t * BLK);
        const i32x8 b[1] = {r[J]};
        const int eb[1] = {e};
        f8_multiply<EXACT, J, TM, 1>(c, a, ea, b, eb);
      }
    };
    step(Const<0>{});
    step(Const<1>{});
    step(Const<2>{});
    step(Const<3>{});
  };
  for (int q = 0; q < kq; q += 2) {
    if (q + 1 < kq) load(q + 1, f[1], ew[1]);
    quad(q, f[0], ew[0]);
    if (q + 1 < kq) {
      if (q + 2 < kq) load(q + 2, f[0], ew[0]);
      quad(q + 1, f[1], ew[1]);
    }
  }
  if (blockIdx.x * 4 + wave >= nrb) return;
  const int n = nb * 16 + 4 * g;
#pragma unroll
  for (int t = 0; t < TM; ++t) {
    const int m = t * 16 + i16;
    if (m >= M) break;
    const f32x4 v = c[t][0] + b4;
    T* p = out + (int64_t)m * ld + n;
    if (n + 4 <= N) {
      typename Packed<T, 4>::type o;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = from_float<T>(v[j]);
      *(typename Packed<T, 4>::type*)p = o;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n + j < N) p[j] = from_float<T>(v[j]);
    }
  }
}

// A workgroup's tiles: bands of `band` row tiles, column tiles outer, so that what a band's rows and a few column tiles hold fits
// an XCD's L2. Workgroups are dealt round-robin to the XCDs; each XCD has a contiguous range of tiles, which its
// workgroups take in turn.
struct F8Tiles {
  int nm, nn, band, per, first, last;
  __device__ __forceinline__ F8Tiles(int nm_, int nn_, int band_) : nm(nm_), nn(nn_), band(band_), per((int)gridDim.x / 8) {
    const int n = nm * nn, xcd = blockIdx.x & 7;
    first = xcd * (n / 8) + min(xcd, n % 8);
    last = first + n / 8 + (xcd < n % 8 ? 1 : 0);
  }
  // The first row and column blocks of tile t.
  __device__ __forceinline__ void at(int t, int rb, int cb, int& rb0, int& cb0) const {
    const int b0 = t / (band * nn) * band, bh = min(band, nm - b0);
    t -= b0 * nn;
    rb0 = (b0 + t % bh) * rb;
    cb0 = t / bh * cb;
  }
};

// Many rows: 16 WM TM x 16 WN TN tiles of WM x WN waves, both operands through LDS in two stages of one 128-column block, moved
// there by LDS-destination loads: a stage's loads are issued right behind the barrier that frees its buffer and are in flight
// while the other stage is multiplied. A workgroup takes several tiles (SLOTS per 8 XCDs share them) and goes on to the next one's
// first stage while it multiplies a tile's last, so that only the first tile waits for memory and a tile's stores drain
// behind the next one's products (6400 x 1000 by 50000 fp16: 449 us with a workgroup per tile).
template <int TM_, int TN_, int WM_, int WN_, int SLOTS_>
struct F8Tile {
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, NT = 64 * WM * WN, SLOTS = SLOTS_;
  static constexpr int RB = WM * TM, CB = WN * TN, BM = 16 * RB, BN = 16 * CB;
  static constexpr int STG = (RB + CB) * kF8Frag, EXP = 1024, LDS = 2 * STG + 4 * EXP;
  static constexpr int LPW = 2 * (RB + CB) / (WM * WN);          // 1 KB loads per wave and stage
  static_assert(LPW * WM * WN == 2 * (RB + CB) && RB <= 16 && CB <= 16, "whole loads");
};

template <class C, class T>
__global__ __launch_bounds__(C::NT) void k_f8_wide(F8Mat x, F8Mat w, int M, int N, const float* __restrict__ bias,
                                                   T* __restrict__ out, int64_t ld, int nm, int nn, int band, F8Partials part) {
  constexpr bool EXACT = sizeof(T) == 4;
  constexpr int TM = C::TM, TN = C::TN, W = C::WM * C::WN;
  __shared__ __attribute__((aligned(16))) char lds[C::LDS];
  char* exps = lds + 2 * C::STG;                 // [four blocks' parity][rows, columns][16 blocks][16]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g = lane >> 4, wm = wave % C::WM, wn = wave / C::WM;
  const int kb = x.kblocks;

  struct Where {
    int rb0, cb0, nra, nca;
  };
  const F8Tiles tiles(nm, nn, band);
  const int per = tiles.per, last = tiles.last;
  auto where = [&](int t) {
    Where p;
    tiles.at(t, C::RB, C::CB, p.rb0, p.cb0);
    p.nra = min(C::RB, x.rblocks - p.rb0);
    p.nca = min(C::CB, w.rblocks - p.cb0);
    return p;
  };

  // load i of this wave moves half (w + W i) & 1 of block (w + W i) / 2 of the stage; row blocks past the operand's last
  // re-read that (they are never stored). Every fourth stage brings the powers of its block and the next three.
  auto issue = [&](const Where& p, int st, int buf, int quad) {
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(x.data + ((size_t)st * x.rblocks + p.rb0) * kF8Frag, p.nra * kF8Frag);
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(w.data + ((size_t)st * w.rblocks + p.cb0) * kF8Frag, p.nca * kF8Frag);
    char* base = lds + buf * C::STG;
#pragma unroll
    for (int i = 0; i < C::LPW; ++i) {
      const int q = wave + W * i, b = q >> 1;
      const uint32_t half = (q & 1) * (kF8Frag / 2);
      if (b < C::RB) dma16(rx, base + q * (kF8Frag / 2), lane * 16u, (uint32_t)min(b, p.nra - 1) * kF8Frag + half);
      else dma16(rw, base + q * (kF8Frag / 2), lane * 16u, (uint32_t)min(b - C::RB, p.nca - 1) * kF8Frag + half);
    }
    if ((st & 3) == 0 && wave < 2) {             // reads zeros past the tile's rows
      const F8Mat& o = wave ? w : x;
      const int b0 = wave ? p.cb0 : p.rb0, nb = wave ? p.nca : p.nra;
      dma16(make_rsrc(o.exps + ((size_t)(st / 4) * o.rblocks + b0) * 16, nb * 64), exps + ((quad & 1) * 2 + wave) * C::EXP, lane * 16u, 0);
    }
  };
  auto barrier = [&] {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  int t = tiles.first + (int)(blockIdx.x >> 3);
  if (t >= last) return;
  Where at = where(t);
  int buf = 0, quad = 0;
  issue(at, 0, 0, 0);
  __builtin_amdgcn_s_waitcnt(waitcnt_stage(0));
  for (;;) {
    const bool more = t + per < last;
    const Where next = more ? where(t + per) : at;
    f32x4 c[TM][TN];
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
      for (int b = 0; b < TN; ++b) c[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int n0 = (at.cb0 + wn * TN) * 16;
    int ea[TM], ew[TN];                            // powers of this block (low byte) and the next ones of its four
    for (int st = 0; st < kb; ++st, buf ^= 1) {
      // this wave's loads of stage st have landed (those of a tile's first stage before the stores of the tile before); behind
      // the barrier everyone's have, and nobody reads the other buffer
      if (st == 0) __builtin_amdgcn_s_waitcnt(waitcnt_stage(63));
      else __builtin_amdgcn_s_waitcnt(waitcnt_stage(0));
      barrier();
      const bool wrap = st + 1 >= kb;
      const int q = quad;
      if (wrap || (st & 3) == 3) ++quad;
      if (!wrap || more) issue(wrap ? next : at, wrap ? 0 : st + 1, buf ^ 1, quad);
      if ((st & 3) == 0) {
        const char* e = exps + (q & 1) * 2 * C::EXP + i16 * 4;
#pragma unroll
        for (int a = 0; a < TM; ++a) ea[a] = *(const int*)(e + (wm * TM + a) * 64);
#pragma unroll
        for (int b = 0; b < TN; ++b) ew[b] = *(const int*)(e + C::EXP + (wn * TN + b) * 64);
      } else {
#pragma unroll
        for (int a = 0; a < TM; ++a) ea[a] >>= 8;
#pragma unroll
        for (int b = 0; b < TN; ++b) ew[b] >>= 8;
      }
      const char* base = lds + buf * C::STG + lane * 16;
      i32x8 wf[TN], af[TM];
#pragma unroll
      for (int b = 0; b < TN; ++b) wf[b] = f8_frag(base + (C::RB + wn * TN + b) * kF8Frag);
#pragma unroll
      for (int a = 0; a < TM; ++a) af[a] = f8_frag(base + (wm * TM + a) * kF8Frag);
      f8_multiply<EXACT, 0, TM, TN>(c, af, ea, wf, ew);
      if constexpr (!EXACT) {       // rows' fragments one ahead of the products that take them
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * TN + 4, 0);
#pragma unroll
        for (int a = 0; a < TM; ++a) {
          __builtin_amdgcn_sched_group_barrier(0x008, TN, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
      }
    }
    // The tile's results through the buffer that was multiplied last, half of every wave's rows at a time: 256 or 512 bytes of a row leave
    // together, where the accumulators' own layout has 8 or 16 bytes of 16 rows per store. Chunks of 16 bytes are swizzled by
    // the row against bank conflicts. The next tile's first stage is waited for here, so that nothing has to wait for the stores.
    constexpr int VEC = kVec<T>, CH = C::BN / VEC, RPI = kWave / CH;      // chunks per row, rows per store
    constexpr int ROWS = C::BM / 2;                                       // per pass
    static_assert(TN == 4 && ROWS * CH * 16 <= C::STG && ROWS % (RPI * W) == 0, "half a tile in a buffer");
    f32x4 add[TN];
#pragma unroll
    for (int b = 0; b < TN; ++b) add[b] = bias4(bias, N, n0 + 16 * b + 4 * g);
    __builtin_amdgcn_s_waitcnt(waitcnt_stage(0));
    char* mid = lds + (buf ^ 1) * C::STG;
    const int n = at.cb0 * 16 + lane % CH * VEC;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
      __builtin_amdgcn_s_waitcnt(waitcnt_stage(63));
      barrier();
#pragma unroll
      for (int a = 0; a < TM / 2; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b) {
          const f32x4 v = c[pass * (TM / 2) + a][b] + add[b];
          typedef T quarter __attribute__((ext_vector_type(4)));
          quarter o;
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] = from_float<T>(v[j]);
          const int r = wm * (8 * TM) + 16 * a + i16, k = wn * 64 + 16 * b + 4 * g;
          *(quarter*)(mid + (r * CH + ((k / VEC) ^ (r & 7))) * 16 + k % VEC * (int)sizeof(T)) = o;
        }
      __builtin_amdgcn_s_waitcnt(waitcnt_stage(63));
      barrier();
#pragma unroll
      for (int it = 0; it < ROWS / RPI / W; ++it) {
        const int r = (it * W + wave) * RPI + lane / CH;
        const int m = at.rb0 * 16 + r / (8 * TM) * (16 * TM) + pass * (8 * TM) + r % (8 * TM);
        typedef T vec __attribute__((ext_vector_type(VEC)));
        const vec v = *(const vec*)(mid + (r * CH + ((lane % CH) ^ (r & 7))) * 16);
        if constexpr (EXACT && C::BN == 128) {   // half a wave holds the row's 128 columns
          if (part.max) {
            const float ninf = -__builtin_inff();
            float z[VEC], top = ninf, sum = 0.f;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
              z[j] = n + j < N ? v[j] : ninf;
              top = fmaxf(top, z[j]);
            }
            top = half_max(top);
#pragma unroll
            for (int j = 0; j < VEC; ++j) sum += top > ninf ? __expf(z[j] - top) : 0.f;
            sum = group_sum<32>(sum);
            if ((lane & 31) == 31 && m < M) {
              part.max[(size_t)m * part.ntiles + at.cb0 / 8] = top;
              part.sum[(size_t)m * part.ntiles + at.cb0 / 8] = sum;
            }
          }
        }
        if (m < M) {
          T* p = out + (int64_t)m * ld + n;
          if (n + VEC <= N) {
            __builtin_nontemporal_store((typename Packed<T, VEC>::type)v, (typename Packed<T, VEC>::type*)p);
          } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
              if (n + j < N) p[j] = v[j];
          }
        }
      }
    }
    if (!more) return;
    t += per;
    at = next;
  }
}

// ------------------------------------------------------------------------------------------------- launches
// f(a null pointer of the type)
template <class F>
static hipError_t f8_type(int dtype, F&& f) {
  if (dtype == kF32) f((float*)nullptr);
  else if (dtype == kBF16) f((bf16_t*)nullptr);
  else f((f16_t*)nullptr);
  return hipGetLastError();
}
#define ONMT_TYPE(p) std::remove_pointer_t<decltype(p)>

hipError_t f8_pack(const void* x, int dtype, int64_t ld, int rows, int cols, const F8Mat& out, hipStream_t st) {
  const int nb = (rows + 15) / 16 * out.kblocks;
  return f8_type(dtype, [&](auto* t) {
    using X = ONMT_TYPE(t);
    hipLaunchKernelGGL(k_f8_pack<X>, dim3((nb + 3) / 4), dim3(256), 0, st, (const X*)x, ld, rows, cols, out, nb);
  });
}

hipError_t f8_unpack(const F8Mat& w, int rows, int cols, float* out, int64_t ld, hipStream_t st) {
  const int64_t nb = ((int64_t)rows * ((cols + 3) / 4) + 255) / 256;
  hipLaunchKernelGGL(k_f8_unpack, dim3((unsigned)(nb < 65536 ? nb : 65536)), dim3(256), 0, st, w, rows, cols, out, ld);
  return hipGetLastError();
}

// LDS of a workgroup of k_f8_few for 16 tm rows, and the row tiles that it takes: 1, 2 or 4, 0 if the rows are too many for it. It is
// level with the wide tiles or ahead of them wherever it can run (us, few against wide: 16 x 500 by 50000 fp32 8.5 and
// 15.9, 64 rows 17.1 and 17.1, 17 x 1000 by 50000 fp32 23.2 and 22.7, 64 x 1024 by 32000 bf16 13.3 and 13.4, 16 x 64 by 1000 4.7 and 8.9).
constexpr size_t kFewLds = 64 << 10;
static size_t few_lds(int tm, int cols, bool exact) {
  return (exact ? 2 : 1) * f8_data_bytes(16 * tm, cols) + f8_exp_bytes(16 * tm, cols);
}
static int few_rows(int M, int cols, bool exact) {
  const int tm = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  return M <= 64 && few_lds(tm, cols, exact) <= kFewLds ? tm : 0;
}

template <class X, class T, int TM>
static void launch_few(const void* x, int64_t ldx, int M, const F8Mat& w, int N, int cols, const float* bias, void* out, int64_t ld,
                       hipStream_t st) {
  const int bytes = (int)few_lds(TM, cols, sizeof(T) == 4);
  hipLaunchKernelGGL((k_f8_few<X, T, TM>), dim3((N + 63) / 64), dim3(256), bytes, st, (const X*)x, ldx, w, M, N, cols, bias,
                     (T*)out, ld);
}

template <class C, class T>
static void launch_wide(const F8Mat& x, int M, const F8Mat& w, int N, const float* bias, void* out, int64_t ld, const F8Partials& part,
                        hipStream_t st) {
  const int nm = (M + C::BM - 1) / C::BM, nn = (N + C::BN - 1) / C::BN;
  const int slots = min(C::SLOTS, (nm * nn + 7) / 8 * 8);         // whole rounds of the XCDs
  hipLaunchKernelGGL((k_f8_wide<C, T>), dim3(slots), dim3(C::NT), 0, st, x, w, M, N, bias, (T*)out, ld, nm, nn, 8, part);
}

size_t f8_linear_ws(int M, int cols) { return few_rows(M, cols, true) ? 0 : f8_data_bytes(M, cols) + f8_exp_bytes(M, cols); }

hipError_t f8_linear(const void* x, int dtype, int64_t ldx, int M, const F8Mat& w, int N, int cols, const float* bias, void* out,
                     int out_dtype, int64_t ld, void* ws, hipStream_t st, F8Partials* part) {
  const F8Partials p = part ? *part : F8Partials{};
  if (part) *part = F8Partials{};
  if (const int tm = few_rows(M, cols, out_dtype == kF32))
    return f8_type(dtype, [&](auto* tx) {
      f8_type(out_dtype, [&](auto* to) {
        using X = ONMT_TYPE(tx);
        using T = ONMT_TYPE(to);
        (tm == 1 ? launch_few<X, T, 1> : tm == 2 ? launch_few<X, T, 2> : launch_few<X, T, 4>)(x, ldx, M, w, N, cols, bias, out, ld, st);
      });
    });
  const F8Mat xm = f8_mat(ws, M, cols);
  const hipError_t e = f8_pack(x, dtype, ldx, M, cols, xm, st);
  if (e != hipSuccess) return e;
  // 128 x 128 tiles, two workgroups per CU; 256 x 256 for 16-bit results of many rows, whose 8-bit products would else wait for LDS
  // (256 x 500 by 50000 fp16 24 us with the small tiles, 22 with the large; 20480 x 1024 by 4096 bf16 119 and 106; 128 rows of
  // 500 by 50000 bf16 14.4 and 18)
  return f8_type(out_dtype, [&](auto* to) {
    using T = ONMT_TYPE(to);
    if constexpr (sizeof(T) == 2)
      if (M > 192) return launch_wide<F8Tile<8, 4, 2, 4, 256>, T>(xm, M, w, N, bias, out, ld, p, st);
    launch_wide<F8Tile<4, 4, 2, 2, 512>, T>(xm, M, w, N, bias, out, ld, p, st);
    if (part && sizeof(T) == 4) *part = p;
  });
}

}  // namespace onmt
