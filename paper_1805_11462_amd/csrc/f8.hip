// Matrix product in 8-bit floating point (e4m3) with a power of two for every block of 128 columns of a row.
//
// A block whose largest finite entry is a = f 2^p (1 <= f < 2) is stored as q = e4m3(x 2^-e), rounded to nearest even, with
// e = p - 8 where f <= 1.75 and p - 7 else: the smallest power that brings a to 448, e4m3's largest value, or less. An entry is
// off by at most half an e4m3 step, 2^-4 of its value, down to 2^-14 of the block's largest (2^-10 2^e below). A power of two
// costs no accuracy against a scale of full precision (the steps of a floating-point type move with it), and the
// matrix instruction takes it as an operand: v_mfma_scale_f32_16x16x128_f8f6f4 multiplies one 128-column block of 16 rows of either
// side and scales it by 2^(ex + ew) of its rows and columns, at twice the rate of the 16-bit ones. But it aligns the 128 products
// to the largest before it adds them and drops what falls below some 17 bits: sums of normal values are off by 1.5e-5 of their
// rms (measured; 16x16x32_fp8_fp8 the same), which 16-bit results do not see (their own rounding is 2^-9 or 2^-12) and fp32 results do.
// Those multiply the same e4m3 values as bf16, exact with their powers included (v_cvt_scalef32_pk_bf16_fp8), in
// v_mfma_f32_16x16x32_bf16: 2e-8 to 1e-7.
//
// Operands lie in fragment blocks of 16 rows x 128 columns, 2 KB: lane l of a wave holds row l % 16, columns 32 (l / 16) .. + 31,
// its first 16 bytes at 16 l of the first kilobyte, the others at 16 l of the second. (The instruction's own order of the columns
// does not matter as long as both operands have the same.) Consecutive blocks along the columns; then, behind all blocks,
// the powers (biased by 127), one byte per row and block: the four blocks 4 j .. 4 j + 3 of a row are a dword, which the
// instruction picks its byte from, the dwords of 16 rows side by side.

#include "common.h"
#include "kernels.h"
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

// Four e4m3 values times 2^(biased - 127) as bf16.
__device__ __forceinline__ int2 f8_widen(int w, int biased) {
  const float s = __builtin_bit_cast(float, biased << 23);
  return make_int2(__builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false)),
                   __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)));
}

// One wave per fragment block. WIDE: the values as bf16 with their powers, in blocks of twice the size: 16 bytes per lane and
// quarter of the lane's 32 columns, a kilobyte per quarter; no powers.
template <class T, bool WIDE>
__global__ __launch_bounds__(256) void k_f8_pack(const T* __restrict__ x, int64_t ld, int rows, int cols, F8Mat out, int nblocks) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (b >= nblocks) return;
  const int rb = b / out.kblocks, kb = b % out.kblocks;
  const int r = rb * 16 + (lane & 15), g = lane >> 4;
  const int k0 = kb * kF8Block + 32 * g;
  float v[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = 0.f;
  if (r < rows) {
    const T* p = x + (int64_t)r * ld + k0;
    if (k0 + 32 <= cols) {
#pragma unroll
      for (int i = 0; i < 32; i += kVec<T>) load_vec(p + i, &v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (k0 + i < cols) v[i] = to_float(p[i]);
    }
  }
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    v[i] = v[i] > kF8Most ? kF8Most : v[i] < -kF8Most ? -kF8Most : v[i];   // NaN stays
    a = fmaxf(a, fabsf(v[i]));                                             // and does not count
  }
  a = fmaxf(a, __shfl_xor(a, 16, kWave));
  a = fmaxf(a, __shfl_xor(a, 32, kWave));
  const int e = f8_exp(a);
  i32x4 lo, hi;
  f8_round(v, e, lo, hi);
  if constexpr (WIDE) {
    char* d = out.data + (size_t)b * (2 * kF8Frag) + lane * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const i32x4& h = i < 2 ? lo : hi;
      const int2 p = f8_widen(h[2 * (i & 1)], kF8One + e), q = f8_widen(h[2 * (i & 1) + 1], kF8One + e);
      *(i32x4*)(d + i * 1024) = i32x4{p.x, p.y, q.x, q.y};
    }
    return;
  }
  char* d = out.data + (size_t)b * kF8Frag + lane * 16;
  *(i32x4*)d = lo;
  *(i32x4*)(d + kF8Frag / 2) = hi;
  if (g == 0) {
    const int kq = out.kquads();
    uint8_t* s = (uint8_t*)(out.exps + ((size_t)rb * kq + kb / 4) * 16 + lane);
    s[kb & 3] = (uint8_t)(kF8One + e);
    if (kb == out.kblocks - 1)
      for (int j = (kb & 3) + 1; j < 4; ++j) s[j] = kF8One;
  }
}

__global__ __launch_bounds__(256) void k_f8_unpack(F8Mat w, int rows, int cols, float* __restrict__ out, int64_t ld) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int quads = (cols + 3) / 4;
  const int64_t row = i / quads;
  if (row >= rows) return;
  const int r = (int)row, c = (int)(i % quads) * 4;
  const int rb = r / 16, kb = c / kF8Block, g = c % kF8Block / 32, o = c % 32;
  const int word = *(const int*)(w.data + ((size_t)rb * w.kblocks + kb) * kF8Frag + (o >= 16 ? kF8Frag / 2 : 0) +
                                 (r % 16 + 16 * g) * 16 + o % 16);
  const int e = (int)(((const uint8_t*)(w.exps + ((size_t)rb * w.kquads() + kb / 4) * 16 + r % 16))[kb & 3]) - kF8One;
  const float v[4] = {__builtin_amdgcn_cvt_f32_fp8(word, 0), __builtin_amdgcn_cvt_f32_fp8(word, 1),
                      __builtin_amdgcn_cvt_f32_fp8(word, 2), __builtin_amdgcn_cvt_f32_fp8(word, 3)};
  for (int j = 0; j < 4 && c + j < cols; ++j) out[(int64_t)r * ld + c + j] = ldexpf(v[j], e);
}

template <int J>
__device__ __forceinline__ f32x4 mfma_f8(const i32x8& w, const i32x8& x, const f32x4& c, int we, int xe) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 0, 0, J, we, J, xe);
}

__device__ __forceinline__ i32x8 f8_frag(const char* p) {
  const i32x4 a = *(const i32x4*)p, b = *(const i32x4*)(p + kF8Frag / 2);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// One wave per 16 rows x 16 TN columns. The weights are the instruction's row operand: lane (i16, g) ends up with columns
// 4 g .. + 3 of row i16.
constexpr int kTN = 4;

template <class T>
__global__ __launch_bounds__(256) void k_f8_linear(F8Mat x, F8Mat w, int M, int N, const float* __restrict__ bias,
                                                   T* __restrict__ out, int64_t ld, int nm, int ntiles) {
  constexpr bool WIDE = sizeof(T) == 4;
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= ntiles) return;
  const int mb = t % nm, nb0 = t / nm * kTN, nrb = (N + 15) / 16;
  const int kb = x.kblocks, kq = x.kquads();
  const int i16 = lane & 15, g = lane >> 4;
  const char* xp = x.data + (size_t)mb * kb * (WIDE ? 2 * kF8Frag : kF8Frag) + lane * 16;
  const int* xe = x.exps + (size_t)mb * kq * 16 + i16;
  const char* wp[kTN];
  const int* we[kTN];
  f32x4 c[kTN];
#pragma unroll
  for (int y = 0; y < kTN; ++y) {
    const size_t rb = min(nb0 + y, nrb - 1);
    wp[y] = w.data + rb * kb * kF8Frag + lane * 16;
    we[y] = w.exps + rb * kq * 16 + i16;
    c[y] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  for (int q = 0; q < kq; ++q) {
    const int ex = WIDE ? 0 : xe[q * 16];
    int ew[kTN];
#pragma unroll
    for (int y = 0; y < kTN; ++y) ew[y] = we[y][q * 16];
    auto step = [&](auto j) {
      constexpr int J = decltype(j)::value;
      const int k = 4 * q + J;
      if (k >= kb) return;
      if constexpr (WIDE) {
        bf16x8 a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = *(const bf16x8*)(xp + (size_t)k * (2 * kF8Frag) + i * 1024);
#pragma unroll
        for (int y = 0; y < kTN; ++y) {
          const i32x8 b = f8_frag(wp[y] + (size_t)k * kF8Frag);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int2 p = f8_widen(b[2 * i], ew[y] >> (8 * J) & 255), r = f8_widen(b[2 * i + 1], ew[y] >> (8 * J) & 255);
            c[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, i32x4{p.x, p.y, r.x, r.y}), a[i], c[y], 0,
                                                           0, 0);
          }
        }
      } else {
        const i32x8 a = f8_frag(xp + (size_t)k * kF8Frag);
#pragma unroll
        for (int y = 0; y < kTN; ++y) c[y] = mfma_f8<J>(f8_frag(wp[y] + (size_t)k * kF8Frag), a, c[y], ew[y], ex);
      }
    };
    step(Const<0>{});
    step(Const<1>{});
    step(Const<2>{});
    step(Const<3>{});
  }
  const int m = mb * 16 + i16;
  if (m >= M) return;
#pragma unroll
  for (int y = 0; y < kTN; ++y) {
    const int n = (nb0 + y) * 16 + 4 * g;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n + j < N) out[(int64_t)m * ld + n + j] = from_float<T>(c[y][j] + (bias ? bias[n + j] : 0.f));
  }
}

template <class T>
static hipError_t pack(const void* x, int64_t ld, int rows, int cols, bool wide, const F8Mat& out, hipStream_t st) {
  const int nb = (rows + 15) / 16 * out.kblocks;
  const auto kernel = wide ? k_f8_pack<T, true> : k_f8_pack<T, false>;
  hipLaunchKernelGGL(kernel, dim3((nb + 3) / 4), dim3(256), 0, st, (const T*)x, ld, rows, cols, out, nb);
  return hipGetLastError();
}

static hipError_t pack_any(const void* x, int dtype, int64_t ld, int rows, int cols, bool wide, const F8Mat& out, hipStream_t st) {
  return dtype == kF32 ? pack<float>(x, ld, rows, cols, wide, out, st)
         : dtype == kBF16 ? pack<bf16_t>(x, ld, rows, cols, wide, out, st)
                          : pack<f16_t>(x, ld, rows, cols, wide, out, st);
}

hipError_t f8_pack(const void* x, int dtype, int64_t ld, int rows, int cols, const F8Mat& out, hipStream_t st) {
  return pack_any(x, dtype, ld, rows, cols, false, out, st);
}

hipError_t f8_unpack(const F8Mat& w, int rows, int cols, float* out, int64_t ld, hipStream_t st) {
  const int64_t n = (int64_t)rows * ((cols + 3) / 4);
  hipLaunchKernelGGL(k_f8_unpack, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, w, rows, cols, out, ld);
  return hipGetLastError();
}

template <class T>
static hipError_t linear(const F8Mat& x, const F8Mat& w, int M, int N, const float* bias, void* out, int64_t ld, hipStream_t st) {
  const int nm = (M + 15) / 16, nt = nm * ((N + 16 * kTN - 1) / (16 * kTN));
  hipLaunchKernelGGL(k_f8_linear<T>, dim3((nt + 3) / 4), dim3(256), 0, st, x, w, M, N, bias, (T*)out, ld, nm, nt);
  return hipGetLastError();
}

size_t f8_linear_ws(int M, int cols) { return 2 * f8_data_bytes(M, cols); }

hipError_t f8_linear(const void* x, int dtype, int64_t ldx, int M, const F8Mat& w, int N, int cols, const float* bias, void* out,
                     int out_dtype, int64_t ld, void* ws, hipStream_t st) {
  const F8Mat xm = f8_mat(ws, M, cols);
  const hipError_t e = pack_any(x, dtype, ldx, M, cols, out_dtype == kF32, xm, st);
  if (e != hipSuccess) return e;
  return out_dtype == kF32 ? linear<float>(xm, w, M, N, bias, out, ld, st)
         : out_dtype == kBF16 ? linear<bf16_t>(xm, w, M, N, bias, out, ld, st)
                              : linear<f16_t>(xm, w, M, N, bias, out, ld, st);
}

}  // namespace onmt
