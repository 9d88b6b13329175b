// The next token of every row of logits (adsa_sample): temperature, top-k, top-p and min-p, from a random number that the caller brings.
//
//  k_sample<EB, NT, BINS, VEC>: a workgroup takes a row.  It reads it once and keeps it in LDS as far as that goes (28672 logits); what is beyond is read again in every pass.
//  What is kept of a row by top-k and top-p is the front of its descending order, so it is known by its last one: (z, index), and a logit is in if its z is
//  larger, or the same and its index no larger.  That last one is found without sorting: logits are counted, and their weights summed, by
//  BINS steps of z below the largest; running sums over the bins say in which bin a limit falls, and that bin's logits, some dozens, are listed in one more
//  pass and ranked against each other.  Where they are more than kList (many equal ones), the last one is found bit by bit instead.
//  Weights are whole numbers of 2^-44 of the largest one's: their sums do not depend on an order, and what is less than half of that is nothing.  They are formed in 64
//  bits, since a token is decided by where a random number falls among up to 2^18 of them: with weights good to 2^-24 every thousandth row of a large
//  vocabulary would get its neighbour.
//  The passes: the largest; bins (rows with top-k or top-p); a list for each limit; the candidates' weight by runs of 1024; the run that the random number falls in.
//  What bounds it: memory for the first pass, from then on what the vector unit issues, about 18 instructions a weight, twice a logit.
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
  int n_rows, vocab, guided, top_k, held;            // held: groups of a wave that stay in LDS
  float guidance, temperature, top_p, min_p;
};

constexpr int kGroup = 4 * kWave;        // logits of a group: 4 consecutive ones to a lane
constexpr int kRun = 4;                  // groups of a run, whose weight is kept
constexpr int kList = 512;
constexpr float kReach = 31.25f;         // e^-31.25 < 2^-45: what is further below the largest (in temperatures) weighs nothing
constexpr double kOne = 17592186044416.0;            // 2^44

__device__ __forceinline__ uint32_t order_of(float z) {            // ascending as z is; -0 and +0 are equal
  const uint32_t u = __float_as_uint(z + 0.0f);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

// The weight of a live logit (see k_sample): exp((z - top) / T) * 2^44, by 2^(j / 32) from a table and a polynomial of degree 5, off by some 2^-49 of it, rounded
// to a whole number.  Sums' low bits do the rounding: x + kRound holds the nearest whole number of x in its low bits, and w + 2^52 that of w.
struct Weigh {
  static constexpr double kRound = 6755399441055744.0;             // 1.5 * 2^52
  const double* table;         // 2^(44 + j / 32), LDS
  double inv, top;             // 32 log2(e) / T; the largest logit
  __device__ __forceinline__ u64 operator()(float z) const {
    constexpr double a = 0.69314718055994530942 / 32.0;            // ln(2) / 32
    const double d = (double)z - top, t = fma(d, inv, kRound), r = fma(d, inv, kRound - t);
    const int steps = (int)(uint32_t)__double_as_longlong(t);
    const double p = fma(r, fma(r, fma(r, fma(r, fma(r, a * a * a * a * a / 120.0, a * a * a * a / 24.0), a * a * a / 6.0), a * a / 2.0), a), 1.0);
    const u64 power = (u64)__double_as_longlong(table[steps & 31]) + ((u64)(uint32_t)(steps >> 5) << 52);         // (2^-2 at least: an exponent that there is)
    return (u64)__double_as_longlong(fma(__longlong_as_double((long long)power), p, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
  }
};

// x of the lane that CTRL names, 0 where there is none; of the rows of lanes in ROWS only
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, true); }
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 moved(u64 x) { return (u64)moved<CTRL, ROWS>((uint32_t)(x >> 32)) << 32 | moved<CTRL, ROWS>((uint32_t)x); }
// running sums over the wave: within rows of 16, then the row before, then the lower half
template <typename T>
__device__ __forceinline__ T wave_scan(T x) {
  x += moved<0x111, 0xF>(x); x += moved<0x112, 0xF>(x); x += moved<0x114, 0xF>(x); x += moved<0x118, 0xF>(x);          // row_shr
  x += moved<0x142, 0xA>(x);                         // row_bcast:15 to rows 1 and 3
  x += moved<0x143, 0xC>(x);                         // row_bcast:31 to rows 2 and 3
  return x;
}
__device__ __forceinline__ uint32_t lane_of(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }
__device__ __forceinline__ u64 lane_of(u64 x, int lane) { return (u64)lane_of((uint32_t)(x >> 32), lane) << 32 | lane_of((uint32_t)x, lane); }
template <typename T>
__device__ __forceinline__ T wave_sum(T x) { return lane_of(wave_scan(x), kWave - 1); }

template <int NT, int BINS>
struct SampleShared {
  static constexpr int NW = NT / kWave;
  double table[32];
  u64 weight[BINS];            // of a bin
  u64 list_weight[kList];
  u64 run_weight[NT / kRun];
  u64 wave_weight[2][NW];
  u64 above_weight, left;      // weight before the bin that a limit falls in; of a run before the random number
  uint32_t count[BINS];
  uint32_t list_key[kList];
  int list_index[kList];
  uint32_t wave_count[2][NW];
  float wave_top[NW], wave_least[NW];
  uint32_t above_count, n_list, last_key;
  int bin, last_index, token, run;
};

// Where a row's candidates end: the last one in descending order.  Nothing set: key 0, and every index.
struct Last {
  uint32_t key;
  int index;
  __device__ __forceinline__ bool holds(uint32_t k, int i) const { return k > key || (k == key && i <= index); }
};

template <int EB, int NT, int BINS, bool VEC>
__global__ __launch_bounds__(NT) void k_sample(SampleArgs A) {
  constexpr int NW = NT / kWave;
  extern __shared__ __align__(16) float s_held[];    // [group of a wave][NT][4]
  __shared__ SampleShared<NT, BINS> sh;
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
  const float T = A.temperatures ? A.temperatures[r] : A.temperature, top_p = A.top_ps ? A.top_ps[r] : A.top_p, min_p = A.min_ps ? A.min_ps[r] : A.min_p;
  const float u = A.uniform[r];
  const int top_k = A.top_ks ? A.top_ks[r] : A.top_k;
  const gchar* const row = (const gchar*)A.logits + (long long)r * A.stride_b;
  const gchar* const partner = row + (long long)A.n_rows * A.stride_b;
  // ---- logits: a wave takes consecutive ones, group by group
  const int groups = (V + NT * 4 - 1) / (NT * 4), runs = (groups + kRun - 1) / kRun, held = min(A.held, groups), first = wave * groups * kGroup + lane * 4;
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
  auto read_group = [&](int g, float (&z)[4]) {      // from memory
    const int i = first + g * kGroup;
    read4(row, i, z);
    if (guided) {
      float f4[4];
      read4(partner, i, f4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma clang fp contract(off)
        const double c = z[e], f = f4[e], step = c - f, far = (double)A.guidance * step;
        z[e] = i + e < V ? (float)(f + far) : -INFINITY;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = z[e] != z[e] ? -INFINITY : z[e];
  };
  // ---- the largest, and the least that is finite
  float top = -INFINITY, least_z = INFINITY;
#pragma unroll 4
  for (int g = 0; g < groups; ++g) {
    float z[4];
    read_group(g, z);
    if (g < held) *reinterpret_cast<float4*>(s_held + (g * NT + tid) * 4) = make_float4(z[0], z[1], z[2], z[3]);
    top = fmaxf(fmaxf(top, fmaxf(z[0], z[1])), fmaxf(z[2], z[3]));
#pragma unroll
    for (int e = 0; e < 4; ++e) least_z = fminf(least_z, z[e] == -INFINITY ? INFINITY : z[e]);
  }
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) { top = fmaxf(top, __shfl_xor(top, d)); least_z = fminf(least_z, __shfl_xor(least_z, d)); }
  if (lane == 0) { sh.wave_top[wave] = top; sh.wave_least[wave] = least_z; }
  if (tid < 32) sh.table[tid] = exp2((double)tid / 32.0) * kOne;
  for (int i = tid; i < BINS; i += NT) { sh.weight[i] = 0; sh.count[i] = 0; }
  if (tid == 0) { sh.token = V; sh.n_list = 0; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) { top = fmaxf(top, sh.wave_top[w]); least_z = fminf(least_z, sh.wave_least[w]); }
  auto finish = [&](int token, float logprob) {
    A.token[r] = token;
    if (guided) A.token[A.n_rows + r] = token;
    if (A.logprob) A.logprob[r] = logprob;
  };
  if (top == -INFINITY) {
    if (tid == 0) finish(-1, -INFINITY);
    return;
  }
  const bool infinite = top == INFINITY;             // then only the infinities are candidates: as 0, and the others as -infinity
  top = infinite ? 0.0f : top;
  auto group_of = [&](int g, float (&z)[4]) {
    if (g < held) {
      const float4 x = *reinterpret_cast<const float4*>(s_held + (g * NT + tid) * 4);
      z[0] = x.x; z[1] = x.y; z[2] = x.z; z[3] = x.w;
    } else read_group(g, z);
    if (infinite) {
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = z[e] == INFINITY ? 0.0f : -INFINITY;
    }
  };
  // f(logit, index) for each of the thread's, in ascending order
  auto each_logit = [&](auto f) {
#pragma unroll 2
    for (int g = 0; g < groups; ++g) {
      float z[4];
      group_of(g, z);
#pragma unroll
      for (int e = 0; e < 4; ++e) f(z[e], first + g * kGroup + e);
    }
  };
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
  const double inv = 46.166241308446828384 / (double)T;                    // 32 log2(e) / T
  const Weigh weigh = {sh.table, inv, (double)top};
  const float reach = fminf(kReach * T, 1e38f), range = fminf(reach, infinite ? 1.0f : top - least_z), per_bin = range > 0.0f ? (float)BINS / range : 0.0f;
  auto live = [&](float z) { return top - z <= reach; };
  auto bin_of = [&](float below) { return min((int)(below * per_bin), BINS - 1); };            // below the largest
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
  auto enough_of = [&](u64 total) {                  // the least whole number that reaches top_p's share, 1 at least
    const double share = (double)fmaxf(top_p, 0.0f) * (double)total;
    u64 e = (u64)share;
    if ((double)e < share) ++e;
    return e < 1 ? (u64)1 : e > total ? total : e;
  };
  if (by_count || by_sum) {
    each_logit([&](float z, int) {
      const float below = top - z;
      if (below <= reach) {
        const int b = bin_of(below);
        atomicAdd(&sh.count[b], 1u);
        if (by_sum) atomicAdd(&sh.weight[b], weigh(z));
      }
    });
    __syncthreads();
    // running sums over the bins, PB of them a thread
    constexpr int PB = BINS / NT;
    static_assert(PB * NT == BINS, "whole bins");
    uint32_t n[PB], n_sum = 0;
    u64 w[PB], w_sum = 0;
#pragma unroll
    for (int k = 0; k < PB; ++k) {
      n[k] = sh.count[tid * PB + k];
      w[k] = sh.weight[tid * PB + k];
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
    // (what can be in the bin lies between `from` and `to`, a bin's width to either side: two comparisons for nearly all)
    const float width = range / (float)BINS;
    auto in_bin = [&](float z, int bin) {
      const float below = top - z, from = ((float)bin - 1.0f) * width, to = bin == BINS - 1 || per_bin == 0.0f ? INFINITY : ((float)bin + 2.0f) * width;
      return below >= from && below < to && below <= reach && bin_of(below) == bin;
    };
    // The last one up to which there are `most` logits, or `enough` of weight, among those that `last` holds.
    auto cut = [&](bool by_n, uint32_t most, u64 enough) {
      {
        uint32_t nb = n_at;
        u64 wb = w_at;
#pragma unroll
        for (int k = 0; k < PB; ++k) {
          if (by_n ? nb < most && most <= nb + n[k] : wb < enough && enough <= wb + w[k]) { sh.bin = tid * PB + k; sh.above_count = nb; sh.above_weight = wb; sh.n_list = 0; }
          nb += n[k];
          wb += w[k];
        }
      }
      __syncthreads();
      const int bin = sh.bin;
      if (sh.count[bin] <= (uint32_t)kList) {        // (uniform)
        each_logit([&](float z, int i) {
          if (in_bin(z, bin) && last.holds(order_of(z), i)) {
            const uint32_t at = atomicAdd(&sh.n_list, 1u);
            sh.list_key[at] = order_of(z);
            sh.list_index[at] = i;
            if (by_sum) sh.list_weight[at] = weigh(z);
          }
        });
        __syncthreads();
        // a wave ranks an entry: its lanes are the entries that may come before it (or are it)
        const int m = (int)sh.n_list;
        for (int i = wave; i < m; i += NW) {
          const Last me = {sh.list_key[i], sh.list_index[i]};
          uint32_t rank = sh.above_count;
          u64 upto = 0;
          for (int j0 = 0; j0 < m; j0 += kWave) {
            const int j = j0 + lane;
            const bool in = j < m && me.holds(sh.list_key[min(j, m - 1)], sh.list_index[min(j, m - 1)]);
            rank += (uint32_t)__popcll(__ballot(in));
            if (!by_n) upto += in ? sh.list_weight[j] : 0;
          }
          bool ends = rank == most;
          if (!by_n) {
            upto = sh.above_weight + wave_sum(upto);
            ends = upto >= enough && upto - sh.list_weight[i] < enough;
          }
          if (ends && lane == 0) { sh.last_key = me.key; sh.last_index = me.index; }
        }
        __syncthreads();
        last = {sh.last_key, sh.last_index};
        return;
      }
      // Many equal logits: the largest key from which on there is enough, then, among that key's logits, the lowest index up to which.
      const Last held_by = last;
      auto sum = [&](auto in, uint32_t* all_n, u64* all_w) {
        uint32_t c = 0;
        u64 x = 0;
        each_logit([&](float z, int i) {
          const uint32_t k = order_of(z);
          if (live(z) && held_by.holds(k, i) && in(k, i)) { ++c; x += by_n ? 0 : weigh(z); }
        });
        block_sum(c, x, all_n, all_w);
      };
      uint32_t key = 0, cn, on;
      u64 cw, ow;
      for (int bit = 31; bit >= 0; --bit) {
        const uint32_t from = key | 1u << bit;
        sum([&](uint32_t k, int) { return k >= from; }, &cn, &cw);
        if (by_n ? cn >= most : cw >= enough) key = from;
      }
      sum([&](uint32_t k, int) { return k > key; }, &on, &ow);
      int index = -1;                                // not enough up to here
      for (int bit = 17; bit >= 0; --bit) {
        const int upto = index + (1 << bit);
        sum([&](uint32_t k, int i) { return k == key && i <= upto; }, &cn, &cw);
        if (!(by_n ? on + cn >= most : ow + cw >= enough)) index = upto;
      }
      last = {key, index + 1};
    };
    if (by_count && (uint32_t)top_k < n_live) {
      cut(true, (uint32_t)top_k, 0);
      if (by_sum) {                                  // the sum that top_p is a share of: whole bins, and what is left of the one that top-k ends in
        const int bin = sh.bin;
        const u64 above = sh.above_weight;
        uint32_t none;
        u64 mine = 0;
        if (sh.count[bin] <= (uint32_t)kList) {      // (listed, without those that are left out: any entry's weight counts if it is held)
          const int m = (int)sh.n_list;
          for (int j = tid; j < m; j += NT) {
            if (last.holds(sh.list_key[j], sh.list_index[j])) mine += sh.list_weight[j];
          }
        } else {
          each_logit([&](float z, int i) {
            if (in_bin(z, bin) && last.holds(order_of(z), i)) mine += weigh(z);
          });
        }
        block_sum(0, mine, &none, &total);
        total += above;
      }
    }
    if (by_sum) cut(false, 0, enough_of(total));
    __syncthreads();
  }
  // ---- the candidates' weight by runs, and the run that the random number falls in
  const u64 least = min_p > 0.0f ? (u64)ceil((double)fminf(min_p, 1.0f) * kOne) : 0;
  auto weight_of = [&](float z, int i) -> u64 {
    if (!live(z) || !last.holds(order_of(z), i)) return 0;
    const u64 w = weigh(z);
    return w >= least ? w : 0;
  };
  for (int run = 0; run < runs; ++run) {
    u64 sum = 0;
#pragma unroll 2
    for (int g = run * kRun; g < min((run + 1) * kRun, groups); ++g) {
      float z[4];
      group_of(g, z);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += weight_of(z[e], first + g * kGroup + e);
    }
    sum = wave_sum(sum);
    if (lane == 0) sh.run_weight[wave * runs + run] = sum;
  }
  __syncthreads();
  {
    const u64 mine = tid < NW * runs ? sh.run_weight[tid] : 0, upto = wave_scan(mine);
    if (lane == kWave - 1) sh.wave_weight[0][wave] = upto;
    __syncthreads();
    u64 before = upto - mine, all = 0;
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      before += k < wave ? sh.wave_weight[0][k] : 0;
      all += sh.wave_weight[0][k];
    }
    u64 target = (u64)((u >= 0.0f ? (double)fminf(u, 0.99999994f) : 0.0) * (double)all);
    target = target < all ? target : all - 1;
    if (target >= before && target - before < mine) { sh.run = tid; sh.left = target - before; sh.above_weight = all; }
    __syncthreads();
  }
  // ---- its own logits
  if (wave != sh.run / runs) return;
  u64 left = sh.left;
  for (int g = sh.run % runs * kRun; g < groups; ++g) {
    const int i = first + g * kGroup;
    float z[4];
    group_of(g, z);
    u64 w[4], sum = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) { w[e] = weight_of(z[e], i + e); sum += w[e]; }
    const u64 upto = wave_scan(sum), whole = lane_of(upto, kWave - 1);
    if (left >= whole) {
      left -= whole;
      continue;
    }
    u64 from = upto - sum;
    if (left >= from && left < upto) {
      int e = 0;
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (e == k && left - from >= w[k]) { from += w[k]; ++e; }
      const float ze = e == 0 ? z[0] : e == 1 ? z[1] : e == 2 ? z[2] : z[3];
      finish(i + e, (float)(((double)ze - (double)top) / (double)T - log((double)sh.above_weight * (1.0 / kOne))));
    }
    break;
  }
}

// Threads, bins and logits in LDS by the vocabulary: bins as many as leave some 200 logits of a row's densest part to one, LDS beside them for logits.
template <int NT, int BINS>
constexpr int kHeld = (160 * 1024 - 256 - (int)sizeof(SampleShared<NT, BINS>)) / (NT * 16);       // groups of a wave

template <int EB, int NT, int BINS>
hipError_t launch_n(SampleArgs A, bool vec, hipStream_t st) {
  A.held = (A.vocab + NT * 4 - 1) / (NT * 4);
  const int most = kHeld<NT, BINS>;
  A.held = A.held < most ? A.held : most;
  const size_t lds = (size_t)A.held * NT * 16;
  if (vec) k_sample<EB, NT, BINS, true><<<dim3((unsigned)A.n_rows), NT, lds, st>>>(A);
  else k_sample<EB, NT, BINS, false><<<dim3((unsigned)A.n_rows), NT, lds, st>>>(A);
  return hipGetLastError();
}

template <int EB>
hipError_t launch_e(const SampleArgs& A, hipStream_t st) {
  const bool vec = A.vocab % 4 == 0 && reinterpret_cast<uintptr_t>(A.logits) % (4 * EB) == 0 && A.stride_b % (4 * EB) == 0;
  if (A.vocab <= 4096) return launch_n<EB, 256, 1024>(A, vec, st);
  if (A.vocab <= 65536) return launch_n<EB, 1024, 2048>(A, vec, st);
  return launch_n<EB, 1024, 8192>(A, vec, st);
}

}  // namespace

hipError_t sample_prepare_kernels() {
  hipError_t e = hipSuccess;
  auto allow = [&](auto kernel, int bytes) {
    if (e == hipSuccess) e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  auto both = [&](auto eb, auto nt, auto bins) {
    constexpr int EB = decltype(eb)::value, NT = decltype(nt)::value, BINS = decltype(bins)::value;
    allow(k_sample<EB, NT, BINS, true>, kHeld<NT, BINS> * NT * 16);
    allow(k_sample<EB, NT, BINS, false>, kHeld<NT, BINS> * NT * 16);
  };
  auto sizes = [&](auto eb) {
    using std::integral_constant;
    both(eb, integral_constant<int, 256>(), integral_constant<int, 1024>());
    both(eb, integral_constant<int, 1024>(), integral_constant<int, 2048>());
    both(eb, integral_constant<int, 1024>(), integral_constant<int, 8192>());
  };
  sizes(std::integral_constant<int, 2>());
  sizes(std::integral_constant<int, 4>());
  return e;
}

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
