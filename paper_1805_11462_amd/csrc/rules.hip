// Rules on logits: penalties for repeated tokens, biases, bans of repeated n-grams and grammar masks, then the softmax.
//
// For token v of a row with logit x (fp32 whatever the logits' type; every operation rounded by itself, so that equal logits under
// equal rules stay equal): with c > 0 occurrences of v in the row's history x = x > 0 ? x / rho : x rho, then (x - c f) - p; the
// last entry of the row's bias list that names v is added; a token that would repeat an n-gram of the history, or whose mask bit
// is 0, gets -inf whatever it was.
//
// A workgroup takes 4096 consecutive tokens of a row and every wave 1024 of them, 16 per lane, in 16-byte accesses. The rules
// name tokens, not places: occurrences are counted in LDS, one word per token of the slice (integer atomics, so their
// order does not matter; the top bit marks an n-gram's end), and of a bias list each token keeps its last entry's index (atomic
// maximum). The logits are loaded before that and wait in registers. What bounds it is memory: each logit is read once
// (twice for whole log-probabilities, the second time from the caches where the batch fits them) and each output written once.

#include "common.h"
#include "kernels.h"
#include "types.h"

namespace onmt {

constexpr int kSlice = 4096, kThreads = 256, kPerLane = 16;
static_assert(kSlice == kThreads * kPerLane && kRuleTile == kWave * kPerLane, "a wave's tokens are a tile");
constexpr int kNoId = 0x7fffffff;
constexpr uint32_t kEnds = 0x80000000u;        // top bit of a count: the token would end a repeated n-gram

// The lane's tokens: position i of vector u (kVec<T> tokens each) is base + u * (64 kVec<T>) + i.
template <class T>
struct Tokens {
  static constexpr int VEC = kVec<T>, NV = kPerLane / VEC;
  int slice0, base;
  __device__ __forceinline__ explicit Tokens(int slice)
      : slice0(slice * kSlice), base(slice0 + (threadIdx.x >> 6) * kRuleTile + (threadIdx.x & 63) * VEC) {}
  __device__ __forceinline__ int at(int u) const { return base + u * kWave * VEC; }
};

// One token's penalties and bias, every operation rounded by itself.
__device__ __forceinline__ float penalized(float z, float times, bool rep, float rho, float freq, float pres) {
#pragma clang fp contract(off)
  if (rep) z = z > 0.f ? z / rho : z * rho;
  return (z - times * freq) - pres;
}

// v = the lane's logits of row `row` under the rules, -inf past V. lds: 4096 words of counts (with a history), then 4096 of
// bias entries (with biases).
template <class T>
__device__ __forceinline__ void ruled(const LogitRules& q, const T* x, int V, int row, const Tokens<T>& tk,
                                      uint32_t* lds, float (&v)[kPerLane]) {
  constexpr int VEC = Tokens<T>::VEC, NV = Tokens<T>::NV;
  const float ninf = -__builtin_inff();
  const int tid = threadIdx.x;
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int t = tk.at(u);
    if (t + VEC <= V) {
      load_vec(x + t, &v[u * VEC]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[u * VEC + i] = t + i < V ? to_float(x[t + i]) : ninf;
    }
  }
  uint32_t* cnt = lds;
  int* which = (int*)(lds + (q.history ? kSlice : 0));
  if (q.history || q.n_bias) {
    if (q.history)
      for (int i = tid; i < kSlice / 4; i += kThreads) ((uint4*)cnt)[i] = make_uint4(0, 0, 0, 0);
    if (q.n_bias)
      for (int i = tid; i < kSlice / 4; i += kThreads) ((int4*)which)[i] = make_int4(-1, -1, -1, -1);
    __syncthreads();
    const int width = min(kSlice, V - tk.slice0);
    if (q.history) {
      const int32_t* h = q.history + (int64_t)row * q.history_stride;
      const int n = min(max(q.history_len[row], 0), q.max_history);
      const int g = q.ngram;
      for (int j = tid; j < n; j += kThreads) {
        const int id = h[j], o = id - tk.slice0;
        if (id < tk.slice0 || o >= width) continue;
        atomicAdd(&cnt[o], 1u);
        if (g > 0 && j >= g - 1) {
          bool same = true;
          for (int i = 1; i < g && same; ++i) same = h[j - i] == h[n - i];
          if (same) atomicOr(&cnt[o], kEnds);
        }
      }
    }
    if (q.n_bias) {
      const int32_t* ids = q.bias_ids + (int64_t)row * q.bias_stride;
      for (int j = tid; j < q.n_bias; j += kThreads) {
        const int id = ids[j], o = id - tk.slice0;
        if (id >= tk.slice0 && o < width) atomicMax(&which[o], j);
      }
    }
    __syncthreads();
    const float rho = q.repetition ? q.repetition[row] : 1.f;
    const float pres = q.presence ? q.presence[row] : 0.f;
    const float freq = q.frequency ? q.frequency[row] : 0.f;
    const float* bias = q.n_bias ? q.bias + (int64_t)row * q.bias_stride : nullptr;
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int o = tk.at(u) - tk.slice0 + i;
        float z = v[u * VEC + i];
        if (q.history) {
          const uint32_t c = cnt[o];
          if (c) {
            z = penalized(z, (float)(c & ~kEnds), q.repetition != nullptr, rho, freq, pres);
          }
          if (q.n_bias && which[o] >= 0) z = z + bias[which[o]];
          if (c & kEnds) z = ninf;
        } else if (which[o] >= 0) {
          z = z + bias[which[o]];
        }
        v[u * VEC + i] = tk.at(u) + i < V ? z : ninf;
      }
  }
  if (q.mask) {
    const int mr = q.mask_row ? q.mask_row[row] : row;
    if (mr >= 0) {
      const uint32_t* bits = q.mask + (int64_t)min(mr, q.n_masks - 1) * q.mask_stride;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int t = tk.at(u);
        const uint32_t word = t < V && mr < q.n_masks ? bits[t >> 5] >> (t & 31) : 0u;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (!((word >> i) & 1u)) v[u * VEC + i] = ninf;
      }
    }
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_rules_logits(LogitRules q, const T* x, int64_t ld, int V, int slices,
                                                           T* out, int64_t ld_out) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  const int row = blockIdx.x / slices;
  const Tokens<T> tk(blockIdx.x % slices);
  float v[kPerLane];
  ruled(q, x + (int64_t)row * ld, V, row, tk, lds, v);
  T* o = out + (int64_t)row * ld_out;
#pragma unroll
  for (int u = 0; u < tk.NV; ++u) {
    const int t = tk.at(u);
    if (t + tk.VEC <= V) {
      store_vec(o + t, &v[u * tk.VEC]);
    } else {
#pragma unroll
      for (int i = 0; i < tk.VEC; ++i)
        if (t + i < V) o[t + i] = from_float<T>(v[u * tk.VEC + i]);
    }
  }
}

// Rows' partials: a tile's largest value and the sum of exp(v - that) (NaN where one is; a +inf makes it NaN too). K > 0: the
// tile's top K, larger first, smaller id on ties, by one wave: theta, the K-th largest of the lanes' maxima, is at most the tile's
// K-th largest value, found bit by bit with ballots; the values that reach it, K or a few more, are ranked against
// each other, one per lane. Tiles with more of them than lanes (ties) take K rounds of an argmax.
template <class T, bool LISTS>
__global__ __launch_bounds__(kThreads) void k_rules_partials(LogitRules q, const T* __restrict__ x, int64_t ld, int V, int slices,
                                                             int ntiles, int K, float* __restrict__ pmax,
                                                             float* __restrict__ psum, float* __restrict__ pval,
                                                             int32_t* __restrict__ pid) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  __shared__ float sv[kThreads / kWave][kWave];
  __shared__ int si[kThreads / kWave][kWave];
  const int row = blockIdx.x / slices, slice = blockIdx.x % slices;
  const Tokens<T> tk(slice);
  constexpr int VEC = Tokens<T>::VEC;
  const float ninf = -__builtin_inff();
  float v[kPerLane];
  ruled(q, x + (int64_t)row * ld, V, row, tk, lds, v);
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int tile = slice * (kSlice / kRuleTile) + w;
  if (tile >= ntiles) return;
  float m = ninf;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) m = fmaxf(m, v[i]);
  const float top = wave_max(m), shift = top > ninf ? top : 0.f;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) s += __expf(v[i] - shift);
  s = wave_sum(s);
  const size_t o = (size_t)row * ntiles + tile;
  if (lane == 0) {
    pmax[o] = top;
    psum[o] = s;
  }
  if constexpr (LISTS) {
    auto id_of = [&](int i) { return tk.at(i / VEC) + i % VEC; };
    uint32_t key = __builtin_bit_cast(uint32_t, m), th = 0;
    key ^= key >> 31 ? 0xffffffffu : 0x80000000u;
    for (int b = 31; b >= 0; --b) {
      const uint32_t t = th | 1u << b;
      if (__popcll(__ballot(key >= t)) >= K) th = t;
    }
    th ^= th >> 31 ? 0x80000000u : 0xffffffffu;
    const float theta = __builtin_bit_cast(float, th);
    const unsigned long long below = lane == 0 ? 0ull : (~0ull >> (64 - lane));
    int n = 0;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
      const bool keep = v[i] >= theta && v[i] > ninf;
      const unsigned long long who = __ballot(keep);
      if (who) {
        const int pos = n + __popcll(who & below);
        if (keep && pos < kWave) {
          sv[w][pos] = v[i];
          si[w][pos] = id_of(i);
        }
        n += __popcll(who);
      }
    }
    __builtin_amdgcn_wave_barrier();
    float lv = ninf;
    int li = kNoId;
    if (n <= kWave) {
      const float a = lane < n ? sv[w][lane] : ninf;
      const int id = lane < n ? si[w][lane] : kNoId;
      int r = 0;
      for (int d = 0; d < n; ++d) r += before(readlane_f(a, d), readlane_i(id, d), a, id) ? 1 : 0;
      __builtin_amdgcn_wave_barrier();
      if (lane < n && r < K) {
        sv[w][r] = a;
        si[w][r] = id;
      }
      __builtin_amdgcn_wave_barrier();
      if (lane < min(n, K)) {
        lv = sv[w][lane];
        li = si[w][lane];
      }
    } else {
      float pv = __builtin_inff();
      int pi = -1;
      for (int k = 0; k < K; ++k) {
        float bv = ninf;
        int bi = kNoId;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i)
          if (v[i] > ninf && before(pv, pi, v[i], id_of(i)) && before(v[i], id_of(i), bv, bi)) {
            bv = v[i];
            bi = id_of(i);
          }
#pragma unroll
        for (int d = kWave / 2; d > 0; d >>= 1) {
          const float ov = __shfl_xor(bv, d, kWave);
          const int oi = __shfl_xor(bi, d, kWave);
          if (before(ov, oi, bv, bi)) {
            bv = ov;
            bi = oi;
          }
        }
        if (lane == k) {
          lv = bv;
          li = bi;
        }
        pv = bv;
        pi = bi;
      }
    }
    if (lane < K) {
      pval[o * K + lane] = lv;
      pid[o * K + lane] = li;
    }
  }
}

// log-probabilities: the logits under the rules again, less the row's logsumexp, which every wave forms from the partials.
template <class T>
__global__ __launch_bounds__(kThreads) void k_rules_log_probs(LogitRules q, const T* x, int64_t ld, int V, int slices, int ntiles,
                                                              const float* __restrict__ pmax, const float* __restrict__ psum,
                                                              float* logp, int64_t ld_out, float* __restrict__ lse_out) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  const int row = blockIdx.x / slices;
  const Tokens<T> tk(blockIdx.x % slices);
  constexpr int VEC = Tokens<T>::VEC, NV = Tokens<T>::NV;
  const float ninf = -__builtin_inff();
  const int lane = threadIdx.x & 63;
  float v[kPerLane];
  ruled(q, x + (int64_t)row * ld, V, row, tk, lds, v);
  float m = ninf, s = 0.f;
  for (int t = lane; t < ntiles; t += kWave) m = fmaxf(m, pmax[(size_t)row * ntiles + t]);
  m = wave_max(m);
  const float shift = m > ninf ? m : 0.f;
  for (int t = lane; t < ntiles; t += kWave) s += psum[(size_t)row * ntiles + t] * __expf(pmax[(size_t)row * ntiles + t] - shift);
  const float lse = shift + logf(wave_sum(s));
  if (lse_out && tk.slice0 == 0 && threadIdx.x == 0) lse_out[row] = lse;
  float* o = logp + (int64_t)row * ld_out;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) v[i] = v[i] == ninf ? ninf : v[i] - lse;
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int t = tk.at(u);
    if (t + VEC <= V) {
#pragma unroll
      for (int i = 0; i < VEC; i += 4) store_vec(o + t + i, &v[u * VEC + i]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (t + i < V) o[t + i] = v[u * VEC + i];
    }
  }
}

static unsigned lds_bytes(const LogitRules& r) { return ((r.history != nullptr) + (r.n_bias > 0)) * kSlice * 4; }
static int slices_of(int V) { return (V + kSlice - 1) / kSlice; }
static int tiles_of(int V) { return (V + kRuleTile - 1) / kRuleTile; }

template <class F>
static hipError_t by_type(int dtype, F&& f) {
  if (dtype == kF32) f((float*)nullptr);
  else if (dtype == kBF16) f((bf16_t*)nullptr);
  else f((f16_t*)nullptr);
  return hipGetLastError();
}

hipError_t rules_logits(const LogitRules& r, const LogitMat& m, void* out, int64_t ld_out, hipStream_t st) {
  const int sl = slices_of(m.V);
  return by_type(m.dtype, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    hipLaunchKernelGGL(k_rules_logits<T>, dim3(m.N * sl), dim3(kThreads), lds_bytes(r), st, r, (const T*)m.x, m.ld, m.V, sl,
                       (T*)out, ld_out);
  });
}

hipError_t rules_partials(const LogitRules& r, const LogitMat& m, int K, float* pmax, float* psum, float* pval, int32_t* pid,
                          hipStream_t st) {
  const int sl = slices_of(m.V), nt = tiles_of(m.V);
  return by_type(m.dtype, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    const auto kernel = K > 0 ? k_rules_partials<T, true> : k_rules_partials<T, false>;
    hipLaunchKernelGGL(kernel, dim3(m.N * sl), dim3(kThreads), lds_bytes(r), st, r, (const T*)m.x, m.ld, m.V, sl, nt, K, pmax,
                       psum, pval, pid);
  });
}

hipError_t rules_log_probs(const LogitRules& r, const LogitMat& m, const float* pmax, const float* psum, float* logp,
                           int64_t ld_out, float* lse, hipStream_t st) {
  const int sl = slices_of(m.V), nt = tiles_of(m.V);
  return by_type(m.dtype, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    hipLaunchKernelGGL(k_rules_log_probs<T>, dim3(m.N * sl), dim3(kThreads), lds_bytes(r), st, r, (const T*)m.x, m.ld, m.V, sl,
                       nt, pmax, psum, logp, ld_out, lse);
  });
}

}  // namespace onmt
