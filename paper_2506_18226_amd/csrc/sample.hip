// The next token of every row of logits (adsa_sample): temperature, top-k, top-p and min-p, from a random number that the caller brings.
//
//  k_sample<EB, NT, VEC>: a workgroup takes a row, and reads it again in every pass over it.
//  What is kept of a row is always the front of its descending order, so it is known by its last one: (z, index), and a logit is in if its z is
//  larger, or the same and its index no larger.  That last one is found without sorting: logits are counted, and their weights summed, by
//  kBins steps of z below the largest; the bin in which a limit falls is looked at logit by logit.  A bin that holds more than kList of them (many
//  equal ones) is narrowed bit by bit instead.
//  Weights are whole numbers of 2^-44 of the largest one's: their sums do not depend on an order, and what is less than half of that is nothing.  They are formed in 64
//  bits, since a token is decided by where a random number falls among up to 2^18 of them: with weights good to 2^-24 every thousandth row of a large
//  vocabulary would get its neighbour.
#include <type_traits>

#include "adsa_device.h"

namespace adsa {
namespace {

typedef unsigned long long u64;

struct SampleArgs {
  const char* logits;
  const float* uniform;
  int32_t* token;
  float* logprob;              // or NULL
  const adsa_seq* seqs;        // or NULL
  const float *temperatures, *top_ps, *min_ps;       // or NULL
  const int32_t* top_ks;
  long long stride_b;
  int n_rows, vocab, guided, top_k;
  float guidance, temperature, top_p, min_p;
};

constexpr int kBins = 1024, kList = 1024;
constexpr float kReach = 31.25f;         // e^-31.25 < 2^-45: what is further below the largest (in temperatures) weighs nothing
constexpr double kOne = 17592186044416.0;            // 2^44

__device__ __forceinline__ uint32_t order_of(float z) {            // ascending as z is; -0 and +0 are equal
  const uint32_t u = __float_as_uint(z + 0.0f);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

// exp((z - top) / T) in 64 bits, by 2^(j / 32) from a table and a polynomial: off by some 2^-51 of it.
struct Weigh {
  const double* table;         // 2^(j / 32), LDS
  double inv;                  // 32 log2(e) / T
  float top;
  __device__ __forceinline__ double share(float z, int* steps) const {     // share * 2^(steps / 32)
    const double x = z == top ? 0.0 : fmax(((double)z - (double)top) * inv, -2048.0);
    const double n = __builtin_rint(x), r = (x - n) * (0.69314718055994530942 / 32.0);
    *steps = (int)n;
    return table[*steps & 31] * fma(r, fma(r, fma(r, fma(r, fma(r, 1.0 / 120.0, 1.0 / 24.0), 1.0 / 6.0), 0.5), 1.0), 1.0);
  }
  __device__ __forceinline__ double exact(float z) const {
    int n;
    const double s = share(z, &n);
    return __builtin_ldexp(s, n >> 5);
  }
  static __device__ __forceinline__ u64 whole(double w) {                  // rounded to a whole number of 2^-44
    return (u64)__double_as_longlong(fma(w, kOne, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
  }
  __device__ __forceinline__ u64 operator()(float z) const { return whole(exact(z)); }
};

template <int X, typename T>
__device__ __forceinline__ T from_below(T x, T none) {            // of lane - X
  const T y = __shfl_up(x, X);
  return (int)(threadIdx.x % kWave) >= X ? y : none;
}
template <typename T>
__device__ __forceinline__ T wave_scan(T x) {
  x += from_below<1>(x, (T)0); x += from_below<2>(x, (T)0); x += from_below<4>(x, (T)0);
  x += from_below<8>(x, (T)0); x += from_below<16>(x, (T)0); x += from_below<32>(x, (T)0);
  return x;
}
template <typename T>
__device__ __forceinline__ T wave_sum(T x) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

template <int NT>
struct SampleShared {
  static constexpr int NW = NT / kWave;
  double table[32];
  u64 weight[kBins];           // of a bin, then of it and those before
  u64 list_weight[kList];
  u64 wave_weight[2][NW];
  uint32_t count[kBins];
  uint32_t list_key[kList];
  int list_index[kList];
  uint32_t wave_count[2][NW];
  float wave_top[NW];
  u64 above_weight;            // what comes before the bin that a limit falls in
  uint32_t above_count, n_list;
  int bin, last_index, token;
  uint32_t last_key;
  float token_z;
};

// Where a row's candidates end: the last one in descending order.  Nothing set: key 0, and every index.
struct Last {
  uint32_t key;
  int index;
  __device__ __forceinline__ bool holds(uint32_t k, int i) const { return k > key || (k == key && i <= index); }
};

template <int EB, int NT, bool VEC>
__global__ __launch_bounds__(NT) void k_sample(SampleArgs A) {
  constexpr int NW = NT / kWave;
  __shared__ SampleShared<NT> sh;
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), r = blockIdx.x, V = A.vocab;
  const bool guided = A.guided != 0;
  if (A.seqs) {
    const ADSA_GLOBAL adsa_seq& sq = ((const ADSA_GLOBAL adsa_seq*)A.seqs)[r];
    if (sq.step < 0 || sq.status != 0) {             // (a pair goes by its conditional row)
      if (tid == 0) {
        A.token[r] = -1;
        if (guided) A.token[A.n_rows + r] = -1;
        if (A.logprob) A.logprob[r] = 0.0f;
      }
      return;
    }
  }
  if (tid < 32) sh.table[tid] = exp2((double)tid / 32.0);
  for (int i = tid; i < kBins; i += NT) { sh.weight[i] = 0; sh.count[i] = 0; }
  const float T = A.temperatures ? A.temperatures[r] : A.temperature, top_p = A.top_ps ? A.top_ps[r] : A.top_p, min_p = A.min_ps ? A.min_ps[r] : A.min_p;
  const int top_k = A.top_ks ? A.top_ks[r] : A.top_k;
  const gchar* const row = (const gchar*)A.logits + (long long)r * A.stride_b;
  const gchar* const partner = row + (long long)A.n_rows * A.stride_b;
  // ---- logits: a wave takes consecutive ones, a group 256 of them, a lane 4
  const int groups = (V + NT * 4 - 1) / (NT * 4), first = wave * groups * 256 + lane * 4;
  auto read4 = [&](const gchar* from, int i, float (&f)[4]) {
    if constexpr (VEC) {
      if (i < V) {                                   // (V is a multiple of 4)
        if constexpr (EB == 4) {
          const uint4 x = load16(from + (long long)i * 4);
          f[0] = __uint_as_float(x.x); f[1] = __uint_as_float(x.y); f[2] = __uint_as_float(x.z); f[3] = __uint_as_float(x.w);
        } else {
          const u32x2 x = *(const ADSA_GLOBAL u32x2*)(from + (long long)i * 2);
          f[0] = __uint_as_float(x.x << 16); f[1] = __uint_as_float(x.x & 0xFFFF0000u); f[2] = __uint_as_float(x.y << 16); f[3] = __uint_as_float(x.y & 0xFFFF0000u);
        }
      } else f[0] = f[1] = f[2] = f[3] = -INFINITY;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int at = min(i + e, V - 1);
        const float x = EB == 4 ? ((const gfloat*)from)[at] : __uint_as_float((uint32_t)((const ADSA_GLOBAL uint16_t*)from)[at] << 16);
        f[e] = i + e < V ? x : -INFINITY;
      }
    }
  };
  auto read_group = [&](int g, float (&z)[4]) {
    const int i = first + g * 256;
    read4(row, i, z);
    if (guided) {
      float u[4];
      read4(partner, i, u);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma clang fp contract(off)
        const double c = z[e], f = u[e], step = c - f, far = (double)A.guidance * step;
        z[e] = i + e < V ? (float)(f + far) : -INFINITY;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = z[e] != z[e] ? -INFINITY : z[e];
  };
  // f(logit, index) for each of the thread's, in ascending order
  auto each_logit = [&](auto f) {
    for (int g = 0; g < groups; ++g) {
      float z[4];
      read_group(g, z);
#pragma unroll
      for (int e = 0; e < 4; ++e) f(z[e], first + g * 256 + e);
    }
  };
  // ---- the largest
  float top = -INFINITY;
  each_logit([&](float z, int) { top = fmaxf(top, z); });
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) sh.wave_top[wave] = top;
  if (tid == 0) { sh.token = V; sh.n_list = 0; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) top = fmaxf(top, sh.wave_top[w]);
  auto finish = [&](int token, float logprob) {
    A.token[r] = token;
    if (guided) A.token[A.n_rows + r] = token;
    if (A.logprob) A.logprob[r] = logprob;
  };
  if (top == -INFINITY) {
    if (tid == 0) finish(-1, -INFINITY);
    return;
  }
  if (!(T > 0.0f)) {
    int at = V;
    each_logit([&](float z, int i) { at = z == top ? min(at, i) : at; });
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) at = min(at, __shfl_xor(at, d));
    if (lane == 0) atomicMin(&sh.token, at);
    __syncthreads();
    if (tid == 0) finish(sh.token, 0.0f);
    return;
  }
  const Weigh weigh = {sh.table, 46.166241308446830 / (double)T, top};                 // 32 log2(e)
  const float reach = fminf(kReach * T, 1e38f), per_bin = (float)kBins / reach;
  auto below = [&](float z) { return z == top ? 0.0f : top - z; };
  auto live = [&](float z) { return below(z) <= reach; };
  auto bin_of = [&](float z) { return min((int)(below(z) * per_bin), kBins - 1); };
  const bool by_count = top_k > 0 && top_k < V, by_sum = top_p < 1.0f;
  Last last = {0u, 0x7FFFFFFF};
  // sums of a count and a weight over the workgroup
  int turn = 0;
  auto block_sum = [&](uint32_t n, u64 w, uint32_t* all_n, u64* all_w) {
    n = wave_sum(n);
    w = wave_sum(w);
    if (lane == 0) { sh.wave_count[turn][wave] = n; sh.wave_weight[turn][wave] = w; }
    __syncthreads();
    *all_n = 0;
    *all_w = 0;
#pragma unroll
    for (int k = 0; k < NW; ++k) { *all_n += sh.wave_count[turn][k]; *all_w += sh.wave_weight[turn][k]; }
    turn ^= 1;                                       // (the next sum writes elsewhere: one barrier each)
  };
  if (by_count || by_sum) {
    each_logit([&](float z, int) {
      if (live(z)) {
        const int b = bin_of(z);
        atomicAdd(&sh.count[b], 1u);
        atomicAdd(&sh.weight[b], weigh(z));
      }
    });
    __syncthreads();
    // running sums over the bins, PB of them a thread
    constexpr int PB = kBins / NT > 1 ? kBins / NT : 1;
    uint32_t n[PB], n_sum = 0;
    u64 w[PB], w_sum = 0;
    const bool scans = tid * PB < kBins;
#pragma unroll
    for (int k = 0; k < PB; ++k) {
      n[k] = scans ? sh.count[tid * PB + k] : 0u;
      w[k] = scans ? sh.weight[tid * PB + k] : 0ull;
      n_sum += n[k];
      w_sum += w[k];
    }
    const uint32_t n_up = wave_scan(n_sum);
    const u64 w_up = wave_scan(w_sum);
    if (lane == kWave - 1) { sh.wave_count[0][wave] = n_up; sh.wave_weight[0][wave] = w_up; }
    __syncthreads();
    uint32_t n_at = n_up - n_sum, n_live = 0;
    u64 w_at = w_up - w_sum, total = 0;
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      if (k < wave) { n_at += sh.wave_count[0][k]; w_at += sh.wave_weight[0][k]; }
      n_live += sh.wave_count[0][k];
      total += sh.wave_weight[0][k];
    }
    turn = 1;
    // The last one before which fewer than `most` logits lie (by_n), or less than `enough` of weight, among those that `last` holds.  The bin in which
    // that falls is found from the running sums; its own logits, few as a rule, are ranked against each other.
    auto cut = [&](bool by_n, uint32_t most, u64 enough) {
      uint32_t nb = n_at;
      u64 wb = w_at;
      __syncthreads();                               // (the list and the words below have been read)
      if (tid == 0) sh.n_list = 0;
#pragma unroll
      for (int k = 0; k < PB; ++k) {
        const bool here = by_n ? nb < most && most <= nb + n[k] : wb < enough && enough <= wb + w[k];
        if (here) { sh.bin = tid * PB + k; sh.above_count = nb; sh.above_weight = wb; }
        nb += n[k];
        wb += w[k];
      }
      __syncthreads();
      const int bin = sh.bin;
      const uint32_t above_n = sh.above_count;
      const u64 above_w = sh.above_weight;
      const uint32_t in_bin = sh.count[bin];
      if (in_bin <= (uint32_t)kList) {               // (uniform)
        each_logit([&](float z, int i) {
          if (live(z) && bin_of(z) == bin && last.holds(order_of(z), i)) {
            const uint32_t at = atomicAdd(&sh.n_list, 1u);
            sh.list_key[at] = order_of(z);
            sh.list_index[at] = i;
            sh.list_weight[at] = weigh(z);
          }
        });
        __syncthreads();
        const int m = (int)sh.n_list;
        for (int i = tid; i < m; i += NT) {
          const Last me = {sh.list_key[i], sh.list_index[i]};
          uint32_t before_n = above_n;
          u64 before_w = above_w;
          for (int j = 0; j < m; ++j)
            if (j != i && me.holds(sh.list_key[j], sh.list_index[j])) { ++before_n; before_w += sh.list_weight[j]; }
          const bool ends = by_n ? before_n == most - 1 : before_w < enough && enough <= before_w + sh.list_weight[i];
          if (ends) { sh.last_key = me.key; sh.last_index = me.index; }
        }
        __syncthreads();
      } else {
        // the largest key from which on there is enough, then, among its logits, the lowest index up to which
        const Last held_by = last;
        uint32_t key = 0, cn;
        u64 cw;
        for (int bit = 31; bit >= 0; --bit) {
          const uint32_t from = key | 1u << bit;
          uint32_t c = 0;
          u64 s = 0;
          each_logit([&](float z, int i) {
            const uint32_t k = order_of(z);
            if (live(z) && k >= from && held_by.holds(k, i)) { ++c; s += weigh(z); }
          });
          block_sum(c, s, &cn, &cw);
          if (by_n ? cn >= most : cw >= enough) key = from;
        }
        int index = -1;                              // fewer than enough up to here
        uint32_t c = 0;
        u64 s = 0;
        each_logit([&](float z, int i) {
          const uint32_t k = order_of(z);
          if (live(z) && k > key && held_by.holds(k, i)) { ++c; s += weigh(z); }
        });
        uint32_t on;
        u64 ow;
        block_sum(c, s, &on, &ow);
        for (int bit = 17; bit >= 0; --bit) {
          const int upto = index + (1 << bit);
          c = 0;
          s = 0;
          each_logit([&](float z, int i) {
            const uint32_t k = order_of(z);
            if (live(z) && k == key && i <= upto && held_by.holds(k, i)) { ++c; s += weigh(z); }
          });
          block_sum(c, s, &cn, &cw);
          if (!(by_n ? on + cn >= most : ow + cw >= enough)) index = upto;
        }
        __syncthreads();
        if (tid == 0) { sh.last_key = key; sh.last_index = index + 1; }
        __syncthreads();
      }
      last.key = sh.last_key;
      last.index = sh.last_index;
    };
    if (by_count && (uint32_t)top_k < n_live) {
      cut(true, (uint32_t)top_k, 0);
      if (by_sum) {
        uint32_t c = 0, all;
        u64 s = 0;
        each_logit([&](float z, int i) {
          if (live(z) && last.holds(order_of(z), i)) { ++c; s += weigh(z); }
        });
        block_sum(c, s, &all, &total);
      }
    }
    if (by_sum) {
      const double share = (double)fmaxf(top_p, 0.0f) * (double)total;
      u64 enough = (u64)share;
      if ((double)enough < share) ++enough;          // as few as reach it
      cut(false, 0, enough < 1 ? 1 : enough > total ? total : enough);
    }
  }
  // ---- the candidates' whole weight, by waves, and where the random number falls
  const double least = min_p > 0.0f ? (double)fminf(min_p, 1.0f) : 0.0;
  auto weight_of = [&](float z, int i) -> u64 {
    if (!live(z) || !last.holds(order_of(z), i)) return 0;
    const double w = weigh.exact(z);
    return w >= least ? Weigh::whole(w) : 0;
  };
  u64 mine = 0;
  each_logit([&](float z, int i) { mine += weight_of(z, i); });
  mine = wave_sum(mine);
  __syncthreads();
  if (lane == 0) sh.wave_weight[0][wave] = mine;
  __syncthreads();
  u64 all = 0;
#pragma unroll
  for (int k = 0; k < NW; ++k) all += sh.wave_weight[0][k];
  const float u = A.uniform[r];
  const double at = (u >= 0.0f ? (double)fminf(u, 0.99999994f) : 0.0) * (double)all;
  u64 target = (u64)at;
  target = target < all ? target : all - 1;
  u64 before = 0;
#pragma unroll
  for (int k = 0; k < NW; ++k)
    if (k < wave) before += sh.wave_weight[0][k];
  if (target < before || target - before >= mine) return;            // (uniform in the wave: the one it falls in goes on)
  u64 left = target - before;
  auto find = [&](float (&z)[4], int g) {            // whether it is in group g
    const int i = first + g * 256;
    u64 w[4], sum = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) { w[e] = weight_of(z[e], i + e); sum += w[e]; }
    const u64 upto = wave_scan(sum), group = __shfl(upto, kWave - 1);
    if (left >= group) { left -= group; return false; }
    u64 from = upto - sum;
    if (left >= from && left < upto) {
      int e = 0;
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (e == k && left - from >= w[k]) { from += w[k]; ++e; }
      const float ze = e == 0 ? z[0] : e == 1 ? z[1] : e == 2 ? z[2] : z[3];
      const double d = ze == top ? 0.0 : ((double)ze - (double)top) / (double)T;
      finish(i + e, (float)(d - log((double)all * (1.0 / kOne))));
    }
    return true;
  };
  for (int g = 0; g < groups; ++g) {
    float z[4];
    read_group(g, z);
    if (find(z, g)) break;
  }
}

template <int EB, int NT>
hipError_t launch_n(const SampleArgs& A, bool vec, hipStream_t st) {
  if (vec) k_sample<EB, NT, true><<<dim3((unsigned)A.n_rows), NT, 0, st>>>(A);
  else k_sample<EB, NT, false><<<dim3((unsigned)A.n_rows), NT, 0, st>>>(A);
  return hipGetLastError();
}

template <int EB>
hipError_t launch_e(const SampleArgs& A, hipStream_t st) {
  const bool vec = A.vocab % 4 == 0 && reinterpret_cast<uintptr_t>(A.logits) % (4 * EB) == 0 && A.stride_b % (4 * EB) == 0;
  return A.vocab <= 4096 ? launch_n<EB, 256>(A, vec, st) : launch_n<EB, 1024>(A, vec, st);
}

}  // namespace

hipError_t launch_sample(const adsa_sampling& s, const adsa_seq* seqs, const void* logits, const float* uniform, int32_t* token, float* logprob, hipStream_t st) {
  SampleArgs A = {};
  A.logits = (const char*)logits; A.uniform = uniform; A.token = token; A.logprob = logprob; A.seqs = seqs;
  A.temperatures = s.temperatures; A.top_ps = s.top_ps; A.min_ps = s.min_ps; A.top_ks = s.top_ks;
  A.stride_b = (s.row_stride ? s.row_stride : s.vocab) * (s.dtype == ADSA_F32 ? 4 : 2);
  A.n_rows = s.n_rows; A.vocab = s.vocab; A.guided = s.guided; A.top_k = s.top_k;
  A.guidance = s.guidance; A.temperature = s.temperature; A.top_p = s.top_p; A.min_p = s.min_p;
  return s.dtype == ADSA_F32 ? launch_e<4>(A, st) : launch_e<2>(A, st);
}

}  // namespace adsa
