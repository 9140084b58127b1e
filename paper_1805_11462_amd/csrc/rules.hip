// Rules on logits: penalties for repeated tokens, biases, bans of repeated n-grams and grammar masks, then the softmax.
//
// For token v of a row with logit x (fp32 whatever the logits' type; every operation rounded by itself, so that equal logits under
// equal rules stay equal): with c > 0 occurrences of v in the row's history x = x > 0 ? x / rho : x rho, then (x - c f) - p; the
// last entry of the row's bias list that names v is added; a token that would repeat an n-gram of the history, or whose mask bit
// is 0, gets -inf whatever it was.
//
// A workgroup takes 4096 consecutive tokens of a row (8192 in large batches; the whole row where its registers hold one) and
// every wave 1024 of them, 16 per lane, in 16-byte accesses. The rules name tokens, not places, and few of them: the
// occurrences of a history's tokens in the slice are counted in LDS (integer atomics, so their order does not matter), the
// first to touch a token lists it, and one thread per listed token then forms
// its new logit, which the lane that holds the token fetches where a bitmap says so. Bias lists go the same way with an atomic
// maximum of entry indices. (Every lane looking up a count for each of its 16 tokens, divisions and all, took
// 322 us at 2560 x 50000 bf16 where memory alone takes 50.) The logits are loaded before that and wait in registers. What
// bounds it is memory: each logit is read once (twice for log-probabilities of rows past a workgroup's registers, the second
// time from the caches where the batch fits them) and each output written once.

#include <algorithm>
#include <cstddef>
#include <type_traits>

#include "answer.h"
#include "common.h"
#include "types.h"

namespace onmt {

constexpr int kThreads = 256;
constexpr int kNoId = 0x7fffffff;
// The lane's PER tokens: position i of vector u (VEC tokens each) is base + u * (64 VEC) + i. A wave's tokens are a tile, a
// workgroup's a slice.
template <int PER_, int VEC_, int THREADS_ = kThreads>
struct Tokens {
  static constexpr int PER = PER_, VEC = VEC_, THREADS = THREADS_, NV = PER / VEC, TILE = PER * kWave, SLICE = PER * THREADS;
  int slice0, base;
  __device__ __forceinline__ explicit Tokens(int slice)
      : slice0(slice * SLICE), base(slice0 + (threadIdx.x >> 6) * TILE + (threadIdx.x & 63) * VEC) {}
  __device__ __forceinline__ int at(int u) const { return base + u * kWave * VEC; }
};

template <class T, int VEC>
__device__ __forceinline__ void load_some(const T* p, float* v) {
  typedef T vec __attribute__((ext_vector_type(VEC), aligned(sizeof(T))));
  const vec x = *(const vec*)p;
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = (float)x[i];
}

// One token's penalties, every operation rounded by itself.
__device__ __forceinline__ float penalized(float z, float times, bool rep, float rho, float freq, float pres) {
#pragma clang fp contract(off)
  if (rep) z = z > 0.f ? z / rho : z * rho;
  return (z - times * freq) - pres;
}

// The largest value of a row of 16 lanes that holds the same in every row, in every lane.
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, dpp_move<0x111, 0xf>(v, v));
  v = fmaxf(v, dpp_move<0x112, 0xf>(v, v));
  v = fmaxf(v, dpp_move<0x114, 0xf>(v, v));
  v = fmaxf(v, dpp_move<0x118, 0xf>(v, v));
  return readlane_f(v, 15);
}

// Takes the lanes that hold `theta` out of c; how many they were.
__device__ __forceinline__ int taken(float& c, float theta) {
  const bool is = c == theta;
  c = is ? -__builtin_inff() : c;
  return __popcll(__ballot(is));
}

// Workgroup barrier for what lies in LDS only: loads from memory stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// What a workgroup knows about the tokens its rules name: for each a word (occurrences in the low half, last bias entry + 1 in
// the high half; then the new logit), a list of them, bits of them, and bits of the tokens that would end a repeated n-gram.
enum { kNoLists = 0, kLongLists = 1, kShortLists = 2 };
constexpr int kListed = 1024;

// Long lists: a word per token of the slice; the list holds up to kListed of the touched ones (more: every token's bit is looked at).
// Small enough for eight workgroups of 4096 tokens per CU, which hide each other's trips to memory.
template <int PER, int LISTS, int THREADS = kThreads>
struct RuleLds {
  static constexpr int SLICE = PER * THREADS, WORDS = SLICE / 32;
  uint32_t word[SLICE];
  uint16_t list[kListed];
  uint32_t touched[WORDS];
  uint32_t ends[WORDS];
  int n;
};

// Short lists, of at most kListed entries together: a word per touched token, found through a slot per token of the slice, which
// needs no clearing and half the room: workgroups of 8192 tokens, six per CU.
template <int PER, int THREADS>
struct RuleLds<PER, kShortLists, THREADS> {
  static constexpr int SLICE = PER * THREADS, WORDS = SLICE / 32;
  uint16_t slot[SLICE];
  uint32_t word[kListed];
  uint16_t list[kListed];
  uint32_t touched[WORDS];
  uint32_t ends[WORDS];
  int n;
};

// The first to touch token o lists it.
template <int PER, int THREADS>
__device__ __forceinline__ void touch(RuleLds<PER, kLongLists, THREADS>& s, int o) {
  const uint32_t bit = 1u << (o & 31);
  if (atomicOr(&s.touched[o >> 5], bit) & bit) return;
  const int at = atomicAdd(&s.n, 1);
  if (at < kListed) s.list[at] = (uint16_t)o;
}
template <int PER, int THREADS>
__device__ __forceinline__ void touch(RuleLds<PER, kShortLists, THREADS>& s, int o) {
  const uint32_t bit = 1u << (o & 31);
  if (atomicOr(&s.touched[o >> 5], bit) & bit) return;
  const int at = atomicAdd(&s.n, 1);               // below kListed: every entry touches one token
  s.list[at] = (uint16_t)o;
  s.slot[o] = (uint16_t)at;
  s.word[at] = 0;
}
template <int PER, int THREADS>
__device__ __forceinline__ uint32_t& word_of(RuleLds<PER, kLongLists, THREADS>& s, int o) { return s.word[o]; }
template <int PER, int THREADS>
__device__ __forceinline__ uint32_t& word_of(RuleLds<PER, kShortLists, THREADS>& s, int o) { return s.word[s.slot[o]]; }

// v = the lane's logits of row `row` under the rules, -inf past V. s: used where there is a history or a bias list. Everything
// whose address is known at the start is loaded there (the first entries of the lists too), so that one trip to memory is
// exposed instead of one per rule (2560 x 50000 bf16 with every rule: 236 us before).
template <class T, int LISTS, int PER, int VEC, int THREADS>
__device__ __forceinline__ void ruled(const LogitRules& q, const T* x, int V, int row, const Tokens<PER, VEC, THREADS>& tk,
                                      RuleLds<PER, LISTS, THREADS>& s, float (&v)[PER]) {
  constexpr int NV = PER / VEC, SLICE = PER * THREADS;
  const float ninf = -__builtin_inff();
  const int tid = threadIdx.x, width = min(SLICE, V - tk.slice0);
  const bool penalties = LISTS && q.history && (q.repetition || q.presence || q.frequency);
  const bool ngrams = LISTS && q.history && q.ngram > 0;
  const int32_t* h = q.history + (int64_t)row * q.history_stride;
  const int32_t* ids = q.bias_ids + (int64_t)row * q.bias_stride;
  const int n = LISTS && q.history ? min(max(q.history_len[row], 0), q.max_history) : 0, g = q.ngram;
  const int mr = q.mask ? (q.mask_row ? q.mask_row[row] : row) : -1;
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int t = tk.at(u);
    if (t + VEC <= V) {
      load_some<T, VEC>(x + t, &v[u * VEC]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[u * VEC + i] = t + i < V ? to_float(x[t + i]) : ninf;
    }
  }
  int hid = -1, prev = 0, bid = -1;
  if constexpr (LISTS) {
    if (q.history && tid < q.max_history) hid = h[tid];
    if (ngrams && g > 1 && tid > 0 && tid < q.max_history) prev = h[tid - 1];
    if (tid < q.n_bias) bid = ids[tid];
  }
  uint32_t on[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int t = tk.at(u);
    on[u] = ~0u;
    if (mr >= 0) on[u] = t < V && mr < q.n_masks ? q.mask[(int64_t)mr * q.mask_stride + (t >> 5)] >> (t & 31) : 0u;
  }
  // the bits of vector u's tokens
  auto bits_of = [&](const uint32_t* b, int u) {
    const int o = tk.at(u) - tk.slice0;
    return b[o >> 5] >> (o & 31) & ((1u << VEC) - 1);
  };
  if constexpr (LISTS) {
    if constexpr (LISTS == kLongLists)
#pragma unroll
      for (int i = 0; i < PER / 4; ++i) ((uint4*)s.word)[tid + i * THREADS] = make_uint4(0, 0, 0, 0);
    static_assert(RuleLds<PER, LISTS, THREADS>::WORDS <= THREADS);
    if (tid < s.WORDS) s.touched[tid] = s.ends[tid] = 0;
    if (tid == 0) s.n = 0;
    // f(token within the slice, entry) for every entry of a list; ahead: the thread's first entry
    auto each = [&](const int32_t* list, int ahead, int n, auto&& f) {
      auto entry = [&](int id, int j) {
        const int o = id - tk.slice0;
        if (id >= tk.slice0 && o < width && j < n) f(o, j);
      };
      entry(ahead, tid);
      for (int j0 = THREADS; j0 < n; j0 += 4 * THREADS) {      // four loads in flight
        int id[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int j = j0 + tid + a * THREADS;
          id[a] = j < n ? list[j] : -1;
        }
#pragma unroll
        for (int a = 0; a < 4; ++a) entry(id[a], j0 + tid + a * THREADS);
      }
    };
    lds_barrier();
    if constexpr (LISTS == kShortLists) {            // slots first, then what is counted in them
      if (penalties) each(h, hid, n, [&](int o, int) { touch(s, o); });
      if (q.n_bias) each(ids, bid, q.n_bias, [&](int o, int) { touch(s, o); });
      lds_barrier();
    }
    if (q.n_bias) {
      each(ids, bid, q.n_bias, [&](int o, int j) {
        if constexpr (LISTS == kLongLists) touch(s, o);
        atomicMax(&word_of(s, o), (uint32_t)(j + 1) << 16);
      });
      lds_barrier();
    }
    if (q.history) {
      const int last = n > 0 ? h[n - 1] : 0;
      each(h, hid, n, [&](int o, int j) {
        if (penalties) {
          if constexpr (LISTS == kLongLists) touch(s, o);
          atomicAdd(&word_of(s, o), 1u);
        }
        if (ngrams && j >= g - 1 && (g == 1 || (j == tid ? prev : h[j - 1]) == last)) {
          bool same = true;
          for (int i = 2; i < g && same; ++i) same = h[j - i] == h[n - i];
          if (same) atomicOr(&s.ends[o >> 5], 1u << (o & 31));
        }
      });
      lds_barrier();
    }
    if (penalties || q.n_bias) {
      const float rho = penalties && q.repetition ? q.repetition[row] : 1.f;
      const float pres = penalties && q.presence ? q.presence[row] : 0.f;
      const float freq = penalties && q.frequency ? q.frequency[row] : 0.f;
      const float* bias = q.bias + (int64_t)row * q.bias_stride;
      const bool listed = LISTS == kShortLists || s.n <= kListed;
      for (int i = tid; i < (listed ? s.n : SLICE); i += THREADS) {
        const int o = listed ? s.list[i] : i;
        if (!listed && !(s.touched[o >> 5] >> (o & 31) & 1)) continue;
        uint32_t& at = LISTS == kShortLists ? s.word[i] : s.word[o];
        const uint32_t w = at, c = w & 0xffff, j = w >> 16;
        float z = to_float(x[tk.slice0 + o]);
        const float b = j ? bias[j - 1] : 0.f;
        if (c) z = penalized(z, (float)c, q.repetition != nullptr, rho, freq, pres);
        if (j) z += b;
        at = __builtin_bit_cast(uint32_t, z);
      }
      lds_barrier();
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const uint32_t b = bits_of(s.touched, u);
        if (b) {
          const int o = tk.at(u) - tk.slice0;
#pragma unroll
          for (int i = 0; i < VEC; i += 4) {
            uint32_t w[4];
            if constexpr (LISTS == kShortLists) {    // slots of other tokens hold anything
              const uint2 q = *(const uint2*)&s.slot[o + i];
              w[0] = s.word[q.x & (kListed - 1)];
              w[1] = s.word[q.x >> 16 & (kListed - 1)];
              w[2] = s.word[q.y & (kListed - 1)];
              w[3] = s.word[q.y >> 16 & (kListed - 1)];
            } else {
              const uint4 q = *(const uint4*)&s.word[o + i];
              w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
              v[u * VEC + i + k] = b >> (i + k) & 1 ? __builtin_bit_cast(float, w[k]) : v[u * VEC + i + k];
          }
        }
      }
    }
  }
  // what is forbidden, -inf: x = (x & keep) | (-inf & ~keep) with each bit spread over a word
  if (ngrams || mr >= 0) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const uint32_t b = ngrams ? on[u] & ~bits_of(s.ends, u) : on[u];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const uint32_t keep = (uint32_t)((int)(b << (31 - i)) >> 31);
        v[u * VEC + i] = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, v[u * VEC + i]) & keep) | (0xff800000u & ~keep));
      }
    }
  }
}

template <class T, int PER, int LISTS>
__global__ __launch_bounds__(kThreads) void k_rules_logits(LogitRules q, const T* x, int64_t ld, int V, int slices,
                                                           T* out, int64_t ld_out) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int row = blockIdx.x / slices;
  const Tokens<PER, kVec<T>> tk(blockIdx.x % slices);
  float v[PER];
  ruled<T, LISTS>(q, x + (int64_t)row * ld, V, row, tk, *(RuleLds<PER, LISTS>*)lds, v);
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

// What the first pass leaves of each tile of a row: largest value and sum of exp, and (K > 0) a list of the candidates for the
// row's K largest, as (value, id).
struct RulePartials {
  uint2* list;
  float* max;                   // [N, ntiles]
  float* sum;
  int* count;
  int ntiles, K;
};

// Entries of a tile's list: as many values as may pass its bound, or the K largest.
__host__ __device__ inline int list_cap(int K) { return 4 * K < 32 ? 4 * K : 32; }

// The lane's share of a wave's maximum and, with that in every lane, the sum of exp(v - maximum) (NaN where one is; a +inf makes
// it NaN too).
template <int PER>
__device__ __forceinline__ float lane_max(const float (&v)[PER]) {
  float m = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < PER; ++i) m = fmaxf(m, v[i]);
  return m;
}
template <int PER>
__device__ __forceinline__ float sum_exp(const float (&v)[PER], float top) {
  const float shift = top > -__builtin_inff() ? top : 0.f;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) s += __expf(v[i] - shift);
  return wave_sum(s);
}

// Lists the values of a wave's tile that can be among the row's K largest, at most list_cap(K); how many they are. m: the
// lane's largest. theta, the K-th largest of the maxima of 16 groups of four lanes (K > 8: of the 64 lanes), is at most the
// tile's K-th largest value: those that reach it, K or a few more, are listed in no order. Tiles with more of them (ties)
// list the K largest, by K rounds of an argmax. Ranking belongs to the row's merge. (2560 x 50000 bf16 at K = 5: theta bit by
// bit with ballots and lists ranked here took 331 scalar and 357 vector instructions per wave, and either unit was as long in
// it as the memory.)
template <int PER, int VEC, int THREADS>
__device__ __forceinline__ int list_top(const float (&v)[PER], float m, int K, const Tokens<PER, VEC, THREADS>& tk, uint2* list) {
  const float ninf = -__builtin_inff();
  const int lane = threadIdx.x & 63, cap = list_cap(K);
  auto id_of = [&](int i) { return tk.at(i / VEC) + i % VEC; };
  int n = 0;
  float theta = ninf;
  if (K <= 8) {
    float c = fmaxf(m, __shfl_xor(m, 16, kWave));
    c = fmaxf(c, __shfl_xor(c, 32, kWave));      // every row of 16 lanes holds the 16 groups' maxima
    for (int k = 0; k < 4 * K; k += taken(c, theta)) theta = row_max(c);
  } else {
    float c = m;
    for (int k = 0; k < K; k += taken(c, theta)) theta = wave_max(c);
  }
  theta = fmaxf(theta, -3.402823466e38f);        // -inf is no candidate
  const unsigned long long below = lane == 0 ? 0ull : (~0ull >> (64 - lane));
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const bool keep = v[i] >= theta;
    const unsigned long long who = __ballot(keep);
    if (who) {
      const int pos = n + __popcll(who & below);
      if (keep && pos < cap) list[pos] = make_uint2(__builtin_bit_cast(uint32_t, v[i]), (uint32_t)id_of(i));
      n += __popcll(who);
    }
  }
  if (n > cap) {
    float pv = __builtin_inff();
    int pi = -1;
    for (n = 0; n < K; ++n) {
      float bv = ninf;
      int bi = kNoId;
#pragma unroll
      for (int i = 0; i < PER; ++i)
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
      if (lane == 0) list[n] = make_uint2(__builtin_bit_cast(uint32_t, bv), (uint32_t)bi);
      pv = bv;
      pi = bi;
    }
  }
  return n;
}

// Rows' partials: a tile's largest value and sum of exp and, TOP, its list.
template <class T, int PER, int LISTS, bool TOP>
__global__ __launch_bounds__(kThreads) void k_rules_partials(LogitRules q, const T* __restrict__ x, int64_t ld, int V, int slices,
                                                             RulePartials p) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int row = blockIdx.x / slices, slice = blockIdx.x % slices;
  constexpr int VEC = kVec<T>;
  const Tokens<PER, VEC> tk(slice);
  const float ninf = -__builtin_inff();
  float v[PER];
  ruled<T, LISTS>(q, x + (int64_t)row * ld, V, row, tk, *(RuleLds<PER, LISTS>*)lds, v);
  const int lane = threadIdx.x & 63;
  const int tile = slice * (kThreads / kWave) + (threadIdx.x >> 6);
  if (tile >= p.ntiles) return;
  const float m = lane_max(v), top = wave_max(m), s = sum_exp(v, top);
  const size_t o = (size_t)row * p.ntiles + tile;
  int n = 0;
  if constexpr (TOP) n = list_top(v, m, p.K, tk, p.list + o * list_cap(p.K));
  if (lane == 0) {
    p.max[o] = top;
    p.sum[o] = s;
    if (TOP) p.count[o] = n;
  }
}

// A row's partials, lane l those of tiles l + 64 j: loaded at once, those past the first kAhead per lane where they are needed.
struct RowTiles {
  static constexpr int kAhead = 4;
  const float *mx, *sm;
  int ntiles;
  float m[kAhead], s[kAhead];
  __device__ __forceinline__ RowTiles(const RulePartials& p, int row)
      : mx(p.max + (size_t)row * p.ntiles), sm(p.sum + (size_t)row * p.ntiles), ntiles(p.ntiles) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int t = lane + j * kWave;
      m[j] = t < ntiles ? mx[t] : -__builtin_inff();
      s[j] = t < ntiles ? sm[t] : 0.f;
    }
  }
  // The largest value of the lane's tiles.
  __device__ __forceinline__ float lane_max() const {
    float r = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
    for (int t = (threadIdx.x & 63) + kAhead * kWave; t < ntiles; t += kWave) r = fmaxf(r, mx[t]);
    return r;
  }
  // The row's logsumexp, in every lane; lmax: lane_max().
  __device__ __forceinline__ float lse(float lmax) const {
    const float top = wave_max(lmax), shift = top > -__builtin_inff() ? top : 0.f;
    float r = 0.f;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) r += s[j] * __expf(m[j] - shift);
    for (int t = (threadIdx.x & 63) + kAhead * kWave; t < ntiles; t += kWave) r += sm[t] * __expf(mx[t] - shift);
    return shift + logf(wave_sum(r));
  }
};

// One wave per row: the lists of the tiles whose maximum reaches the K-th largest tile maximum hold the row's K largest values;
// those that reach it too are ranked against each other. Where ties make that too many, K rounds of an argmax over all lists.
constexpr int kMergeWaves = 1, kMergeTiles = 256, kMergeCands = 256;

__global__ __launch_bounds__(kMergeWaves * kWave) void k_rules_merge(RulePartials p, int N, float* __restrict__ out,
                                                                     int32_t* __restrict__ out_id, float* __restrict__ out_lse) {
  __shared__ int qt[kMergeWaves][kMergeTiles];
  __shared__ uint2 sv[kMergeWaves][kMergeCands];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int row = blockIdx.x * kMergeWaves + w;
  if (row >= N) return;
  const float ninf = -__builtin_inff();
  const int K = p.K, cap = list_cap(K);
  const RowTiles tiles(p, row);
  const float* mx = tiles.mx;
  const int* cnt = p.count + (size_t)row * p.ntiles;
  const uint2* lists = p.list + (size_t)row * p.ntiles * cap;
  float c = tiles.lane_max(), theta = ninf;
  const float lse = tiles.lse(c);
  for (int k = 0; k < K; k += taken(c, theta)) theta = wave_max(c);
  const unsigned long long below = lane == 0 ? 0ull : (~0ull >> (64 - lane));
  int nq = 0, n = 0;
  auto qualify = [&](int t, float m) {
    const bool q = m >= theta && m > ninf;
    const unsigned long long who = __ballot(q);
    const int pos = nq + __popcll(who & below);
    if (q && pos < kMergeTiles) qt[w][pos] = t;
    nq += __popcll(who);
  };
#pragma unroll
  for (int j = 0; j < RowTiles::kAhead; ++j)
    if (j * kWave < p.ntiles) qualify(lane + j * kWave, tiles.m[j]);
  for (int t0 = RowTiles::kAhead * kWave; t0 < p.ntiles; t0 += kWave)
    qualify(t0 + lane, t0 + lane < p.ntiles ? mx[t0 + lane] : ninf);
  __builtin_amdgcn_wave_barrier();
  if (nq <= kMergeTiles)
    for (int s0 = 0; s0 < nq * cap && n <= kMergeCands; s0 += kWave) {
      const int e = s0 + lane, t = e < nq * cap ? qt[w][e / cap] : 0;
      uint2 a = make_uint2(0xff800000u, 0);
      if (e < nq * cap && e % cap < cnt[t]) a = lists[(size_t)t * cap + e % cap];
      const float v = __builtin_bit_cast(float, a.x);
      const bool keep = v >= theta && v > ninf;
      const unsigned long long who = __ballot(keep);
      const int pos = n + __popcll(who & below);
      if (keep && pos < kMergeCands) sv[w][pos] = a;
      n += __popcll(who);
    }
  __builtin_amdgcn_wave_barrier();
  float* o = out + (size_t)row * K;
  int32_t* oi = out_id + (size_t)row * K;
  if (nq <= kMergeTiles && n <= kMergeCands) {
    for (int c0 = lane; c0 < n; c0 += kWave) {
      const uint2 a = sv[w][c0];
      const float v = __builtin_bit_cast(float, a.x);
      int r = 0;
      for (int d = 0; d < n; ++d) r += before(__builtin_bit_cast(float, sv[w][d].x), (int)sv[w][d].y, v, (int)a.y) ? 1 : 0;
      if (r < K) {
        o[r] = v - lse;
        oi[r] = (int)a.y;
      }
    }
    if (lane >= n && lane < K) {
      o[lane] = ninf;
      oi[lane] = kNoId;
    }
  } else {
    float pv = __builtin_inff();
    int pi = -1;
    for (int k = 0; k < K; ++k) {
      float bv = ninf;
      int bi = kNoId;
      for (int e = lane; e < p.ntiles * cap; e += kWave) {
        if (e % cap >= cnt[e / cap]) continue;
        const uint2 a = lists[e];
        const float v = __builtin_bit_cast(float, a.x);
        if (v > ninf && before(pv, pi, v, (int)a.y) && before(v, (int)a.y, bv, bi)) {
          bv = v;
          bi = (int)a.y;
        }
      }
#pragma unroll
      for (int d = kWave / 2; d > 0; d >>= 1) {
        const float ov = __shfl_xor(bv, d, kWave);
        const int od = __shfl_xor(bi, d, kWave);
        if (before(ov, od, bv, bi)) {
          bv = ov;
          bi = od;
        }
      }
      if (lane == 0) {
        o[k] = bi == kNoId ? ninf : bv - lse;
        oi[k] = bi;
      }
      pv = bv;
      pi = bi;
    }
  }
  if (out_lse && lane == 0) out_lse[row] = lse;
}

// log-probabilities: the logits under the rules again, less the row's logsumexp, which every wave forms from the partials.
template <class T, int PER, int LISTS>
__global__ __launch_bounds__(kThreads) void k_rules_log_probs(LogitRules q, const T* x, int64_t ld, int V, int slices,
                                                              RulePartials p, float* logp, int64_t ld_out,
                                                              float* __restrict__ lse_out) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int row = blockIdx.x / slices;
  constexpr int VEC = 4, NV = PER / VEC;       // 16-byte stores
  const Tokens<PER, VEC> tk(blockIdx.x % slices);
  const float ninf = -__builtin_inff();
  const RowTiles tiles(p, row);
  float v[PER];
  ruled<T, LISTS>(q, x + (int64_t)row * ld, V, row, tk, *(RuleLds<PER, LISTS>*)lds, v);
  const float lse = tiles.lse(tiles.lane_max());
  if (lse_out && tk.slice0 == 0 && threadIdx.x == 0) lse_out[row] = lse;
  float* o = logp + (int64_t)row * ld_out;
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = v[i] == ninf ? ninf : v[i] - lse;
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int t = tk.at(u);
    if (t + VEC <= V) {
      store_vec(o + t, &v[u * VEC]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (t + i < V) o[t + i] = v[u * VEC + i];
    }
  }
}

// Where a workgroup holds the whole row in registers, one launch does it all and reads every logit once. Log-probabilities of
// 512 x 32000 bf16 with penalties and biases 21 us against 39 in two passes (24.7 against 47 fp32 logits; 17 against 24 without
// rules), 5.4 against 5.2 for a single row without rules. Rows of 50000 would leave one workgroup per CU, whose waves then wait
// for each other: 43 us against 54 at 512 of them, but 16 against 14 at 64 and 131 against 137 at 1280, so those take two passes.
constexpr int kRowThreads = 1024, kMaxRow = 32 * kRowThreads;

// What the waves of a row tell each other, in the rules' LDS when those are through; cand: room for every wave's list.
template <int THREADS>
struct RowLds {
  static constexpr int WAVES = THREADS / kWave, CANDS = WAVES * 32;
  float max[WAVES], sum[WAVES];
  int count[WAVES];
  int n;
  uint2 list[CANDS], cand[CANDS];
};

// The row's logsumexp from its waves' largest values and sums; wmax: lane l's that of wave l.
template <int THREADS>
__device__ __forceinline__ float row_lse(const RowLds<THREADS>& s, float wmax) {
  const int lane = threadIdx.x & 63;
  const float top = wave_max(wmax), shift = top > -__builtin_inff() ? top : 0.f;
  return shift + logf(wave_sum(lane < s.WAVES ? s.sum[lane] * __expf(wmax - shift) : 0.f));
}

template <class T, int PER, int LISTS, int THREADS>
__global__ __launch_bounds__(THREADS, LISTS == kLongLists && PER > 16 ? 4 : 8) void k_rules_row_log_probs(
    LogitRules q, const T* x, int64_t ld, int V, float* logp, int64_t ld_out, float* __restrict__ lse_out) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  constexpr int VEC = 4, NV = PER / VEC;
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const Tokens<PER, VEC, THREADS> tk(0);
  const float ninf = -__builtin_inff();
  float v[PER];
  ruled<T, LISTS>(q, x + (int64_t)row * ld, V, row, tk, *(RuleLds<PER, LISTS, THREADS>*)lds, v);
  RowLds<THREADS>& s = *(RowLds<THREADS>*)lds;
  const float m = wave_max(lane_max(v)), sum = sum_exp(v, m);
  if (LISTS) lds_barrier();
  if (lane == 0) {
    s.max[threadIdx.x >> 6] = m;
    s.sum[threadIdx.x >> 6] = sum;
  }
  lds_barrier();
  const float lse = row_lse(s, lane < s.WAVES ? s.max[lane] : ninf);
  if (lse_out && threadIdx.x == 0) lse_out[row] = lse;
  float* o = logp + (int64_t)row * ld_out;
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = v[i] == ninf ? ninf : v[i] - lse;
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int t = tk.at(u);
    if (t + VEC <= V) {
      store_vec(o + t, &v[u * VEC]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (t + i < V) o[t + i] = v[u * VEC + i];
    }
  }
}

// The K largest: every wave lists its candidates, those of them that reach the K-th largest wave maximum are ranked. At 16 tokens
// per lane; with 32 the listing runs out of registers (512 x 32000 bf16 with penalties and biases 52 us against 24 in two launches).
template <class T, int PER, int LISTS, int THREADS>
__global__ __launch_bounds__(THREADS, 8) void k_rules_row_top(
    LogitRules q, const T* __restrict__ x, int64_t ld, int V, int K, float* __restrict__ out, int32_t* __restrict__ out_id,
    float* __restrict__ lse_out) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const Tokens<PER, kVec<T>, THREADS> tk(0);
  const float ninf = -__builtin_inff();
  float v[PER];
  ruled<T, LISTS>(q, x + (int64_t)row * ld, V, row, tk, *(RuleLds<PER, LISTS, THREADS>*)lds, v);
  RowLds<THREADS>& s = *(RowLds<THREADS>*)lds;
  const float m = lane_max(v), top = wave_max(m), sum = sum_exp(v, top);
  if (LISTS) lds_barrier();
  const int mine = list_top(v, m, K, tk, &s.list[w * 32]);
  if (lane == 0) {
    s.max[w] = top;
    s.sum[w] = sum;
    s.count[w] = mine;
  }
  if (tid == 0) s.n = 0;
  lds_barrier();
  const float wmax = lane < s.WAVES ? s.max[lane] : ninf, lse = row_lse(s, wmax);
  float c = wmax, theta = ninf;
  for (int k = 0; k < K; k += taken(c, theta)) theta = wave_max(c);
  if (tid < s.CANDS && tid % 32 < s.count[tid / 32]) {
    const uint2 a = s.list[tid];
    if (__builtin_bit_cast(float, a.x) >= theta) s.cand[atomicAdd(&s.n, 1)] = a;      // in any order: ranks follow from value and id
  }
  lds_barrier();
  const int n = s.n;
  float* o = out + (size_t)row * K;
  int32_t* oi = out_id + (size_t)row * K;
  if (tid < n) {
    const uint2 a = s.cand[tid];
    const float z = __builtin_bit_cast(float, a.x);
    int rank = 0;
    for (int d = 0; d < n; ++d) rank += before(__builtin_bit_cast(float, s.cand[d].x), (int)s.cand[d].y, z, (int)a.y) ? 1 : 0;
    if (rank < K) {
      o[rank] = z - lse;
      oi[rank] = (int)a.y;
    }
  } else if (tid < K) {
    o[tid] = ninf;
    oi[tid] = kNoId;
  }
  if (lse_out && tid == 0) lse_out[row] = lse;
}

static int lists_of(const LogitRules& r) {
  if (!r.history && r.n_bias == 0) return kNoLists;
  return (r.history ? r.max_history : 0) + r.n_bias <= kListed ? kShortLists : kLongLists;
}

// Tokens per lane: 16, or 32 where that leaves several rounds of workgroups and pays: it halves what a tile costs beside its
// logits (2560 x 50000 bf16, K = 5, no lists: 65 us against 81, every rule: 127 against 139), but not where there are neither lists
// nor candidates (logits alone 94 us against 89), nor with long lists, whose LDS it doubles (173 us against 137), nor at fewer
// rows (320 x 50000 fp32 with penalties 26.0 us against 24.8).
static int per_lane(const LogitRules& r, int N, int V, int K) {
  const int64_t slices = (V + 32 * kThreads - 1) / (32 * kThreads) * (int64_t)N;
  const int lists = lists_of(r);
  return slices >= 4096 && lists != kLongLists && (K > 0 || lists == kShortLists) ? 32 : 16;
}

// f(a null pointer of the logits' type, tokens per lane and the kind of lists as types, slices, LDS bytes)
template <class F>
static hipError_t by_type(const LogitRules& r, const LogitMat& m, int K, F&& f) {
  auto run = [&](auto* t, auto per, auto lists) {
    constexpr int P = decltype(per)::value, L = decltype(lists)::value;
    f(t, per, lists, (m.V + P * kThreads - 1) / (P * kThreads), L ? (int)sizeof(RuleLds<P, L>) : 0);
  };
  auto g = [&](auto* t) {
    const bool wide = per_lane(r, m.N, m.V, K) == 32;
    switch (lists_of(r)) {
      case kNoLists:
        return wide ? run(t, Const<32>{}, Const<kNoLists>{}) : run(t, Const<16>{}, Const<kNoLists>{});
      case kShortLists:
        if (wide) return run(t, Const<32>{}, Const<kShortLists>{});
    }
    return run(t, Const<16>{}, Const<kLongLists>{});
  };
  if (m.dtype == kF32) g((float*)nullptr);
  else if (m.dtype == kBF16) g((bf16_t*)nullptr);
  else g((f16_t*)nullptr);
  return hipGetLastError();
}

static size_t partials_layout(int N, int V, int K, int per, char* base, RulePartials* p) {
  const int tile = per * kWave, nt = (V + tile - 1) / tile;
  const size_t n = (size_t)N * nt, list = n * list_cap(K) * sizeof(uint2);      // the 8-byte entries first
  if (p) *p = RulePartials{(uint2*)base, (float*)(base + list), (float*)(base + list) + n, (int*)(base + list) + 2 * n, nt, K};
  return list + n * (K > 0 ? 12 : 8);
}

size_t rules_ws(int N, int V, int K) { return partials_layout(N, V, K, 16, nullptr, nullptr); }

#define ONMT_TYPES(t, per, lists)                         \
  using T = std::remove_pointer_t<decltype(t)>;           \
  constexpr int P = decltype(per)::value;                 \
  constexpr int L = decltype(lists)::value

hipError_t rules_logits(const LogitRules& r, const LogitMat& m, void* out, int64_t ld_out, hipStream_t st) {
  return by_type(r, m, 0, [&](auto* t, auto per, auto lists, int sl, int lds) {
    ONMT_TYPES(t, per, lists);
    hipLaunchKernelGGL((k_rules_logits<T, P, L>), dim3(m.N * sl), dim3(kThreads), lds, st, r, (const T*)m.x, m.ld, m.V, sl,
                       (T*)out, ld_out);
  });
}

// The first pass, and where it left its results in ws.
static hipError_t partials(const LogitRules& r, const LogitMat& m, int K, void* ws, RulePartials* p, hipStream_t st) {
  partials_layout(m.N, m.V, K, per_lane(r, m.N, m.V, K), (char*)ws, p);
  return by_type(r, m, K, [&](auto* t, auto per, auto lists, int sl, int lds) {
    ONMT_TYPES(t, per, lists);
    const auto kernel = K > 0 ? k_rules_partials<T, P, L, true> : k_rules_partials<T, P, L, false>;
    hipLaunchKernelGGL(kernel, dim3(m.N * sl), dim3(kThreads), lds, st, r, (const T*)m.x, m.ld, m.V, sl, *p);
  });
}

// f(a null pointer of the logits' type, tokens per lane, the kind of lists and threads as types, LDS bytes) for rows of at most
// kMaxRow logits, the smallest workgroup that holds one.
template <class F>
static hipError_t by_row(const LogitRules& r, const LogitMat& m, F&& f) {
  auto run = [&](auto* t, auto per, auto lists, auto threads) {
    constexpr int P = decltype(per)::value, L = decltype(lists)::value, D = decltype(threads)::value;
    const int rules = L ? (int)sizeof(RuleLds<P, L, D>) : 0;
    f(t, per, lists, threads, std::max(rules, (int)sizeof(RowLds<D>)));
  };
  auto h = [&](auto* t, auto per, auto threads) {
    switch (lists_of(r)) {
      case kNoLists: return run(t, per, Const<kNoLists>{}, threads);
      case kShortLists: return run(t, per, Const<kShortLists>{}, threads);
    }
    return run(t, per, Const<kLongLists>{}, threads);
  };
  auto g = [&](auto* t) {
    if (m.V <= 16 * kThreads) h(t, Const<16>{}, Const<kThreads>{});
    else if (m.V <= 16 * kRowThreads) h(t, Const<16>{}, Const<kRowThreads>{});
    else h(t, Const<32>{}, Const<kRowThreads>{});
  };
  if (m.dtype == kF32) g((float*)nullptr);
  else if (m.dtype == kBF16) g((bf16_t*)nullptr);
  else g((f16_t*)nullptr);
  return hipGetLastError();
}

hipError_t rules_top(const LogitRules& r, const LogitMat& m, int K, void* ws, float* out, int32_t* ids, float* lse,
                     hipStream_t st) {
  // One launch for rows of a small workgroup (8 x 1000 fp32 4.6 us against 6.8, with short lists 7.7 against 9.4), and for those of
  // a large one while every row has a CU (64 x 16384 bf16 6.9 against 8.2; but 1280 rows 22 against 20: the rows' ranking has
  // nothing to hide behind).
  if (m.V <= 16 * kThreads || (m.V <= 16 * kRowThreads && m.N <= 256))
    return by_row(r, m, [&](auto* t, auto per, auto lists, auto threads, int lds) {
      ONMT_TYPES(t, per, lists);
      constexpr int D = decltype(threads)::value;
      if constexpr (P == 16)
        hipLaunchKernelGGL((k_rules_row_top<T, P, L, D>), dim3(m.N), dim3(D), lds, st, r, (const T*)m.x, m.ld, m.V, K, out, ids,
                           lse);
    });
  RulePartials p;
  const hipError_t e = partials(r, m, K, ws, &p, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_rules_merge, dim3((m.N + kMergeWaves - 1) / kMergeWaves), dim3(kMergeWaves * kWave), 0, st, p, m.N, out,
                     ids, lse);
  return hipGetLastError();
}

hipError_t rules_log_probs(const LogitRules& r, const LogitMat& m, void* ws, float* logp, int64_t ld_out, float* lse,
                           hipStream_t st) {
  if (m.V <= kMaxRow)
    return by_row(r, m, [&](auto* t, auto per, auto lists, auto threads, int lds) {
      ONMT_TYPES(t, per, lists);
      constexpr int D = decltype(threads)::value;
      hipLaunchKernelGGL((k_rules_row_log_probs<T, P, L, D>), dim3(m.N), dim3(D), lds, st, r, (const T*)m.x, m.ld, m.V, logp, ld_out,
                         lse);
    });
  RulePartials p;
  const hipError_t e = partials(r, m, 0, ws, &p, st);
  if (e != hipSuccess) return e;
  return by_type(r, m, 0, [&](auto* t, auto per, auto lists, int sl, int lds) {
    ONMT_TYPES(t, per, lists);
    hipLaunchKernelGGL((k_rules_log_probs<T, P, L>), dim3(m.N * sl), dim3(kThreads), lds, st, r, (const T*)m.x, m.ld, m.V, sl, p,
                       logp, ld_out, lse);
  });
}

}  // namespace onmt
