// Attention of many query rows over one set of keys, on the matrix cores (gfx950): prompts over the caches they have just entered
// (adsa_prefill), and decode steps of sequences that share a prompt (adsa_attend_shared).
//
//  k_prompt, k_prompt_finish: a tile of (token, query head) rows of one (sequence, cache head) against the slots up to its last row's.
//  k_prompt_mass: the probability every slot received, a second pass over the scores with each row's normaliser known: a workgroup owns
//    its slots and takes the rows in order, so no atomics and one order of summation.
//  k_shared, k_shared_finish: tiles of a group's (member, query head) rows against parts of the group's prompt, and each sequence's own
//    list (the rows are then the query heads of a cache head), all as workgroups of one launch; the second kernel joins the parts.
//
// All of them turn around one tile product.  Scores are formed transposed, S^T = K Q^T (a 32x32 block: A = 32 keys, B = 32 rows), so a lane
// holds 16 scores of ONE row (its column, lane % 32): maxima and sums are sums over registers and one exchange of the wave's halves,
// and P^T is, register by register, the B operand of O^T = V^T P^T; the order of keys that this fixes within an instruction
// is met on the other side by how V^T is fetched, bf16 by transposing LDS loads, so P never goes through memory.
// Scores are held in fp32 and in units of log 2 (exp2 is the hardware's); so are sums, maxima and outputs until the end.  P enters the second
// product in the cache's type: for bf16 as one value and what that leaves of it as another, 16 bits together, as exact as adsa_attend, for half as many products again.  us
// with one | with two: 64 sequences x 64 heads over 8 x 128 with four prompts 51.6 | 56.2 (capped 53.7 | 61.8, with distances 66.8 | 70.7), 64 x 18 heads over 9 x 64 with lists
// of 553 31.7 | 32.9, 3 x 2..7 tokens x 20 x 64 behind 2011 slots 12.2 either way, 16 x 1..9 x 24 x 64 behind 700 16.1 | 16.4.  Prompts of many rows (k_prompt_many) are bound by their
// products and round P to one bf16, by 2^-8 of it at most, as much as the output's own rounding, unless ADSA_FLAG_SPLIT_P asks for two: 2 x 4352 x 32 x 128 364 | 511 us, lowered
// with distance 487 | 699, by documents 131 | 160, capped ragged prompts of 64 heads over 8 226 | 271, 32 x 120 x 24 x 64 14.2 | 16.9.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "adsa_device.h"

namespace adsa {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.4028234663852886e38f;     // the maximum of a row that has seen no key: z - kLowest is never NaN

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
#define ADSA_LDS __attribute__((address_space(3)))
typedef ADSA_LDS char lchar;

// A pointer that all lanes hold alike, in scalar registers.
template <typename T>
__device__ __forceinline__ T* scalar(T* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint32_t lower = (uint32_t)__builtin_amdgcn_readfirstlane((int)x), upper = (uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32));
  return reinterpret_cast<T*>((uint64_t)upper << 32 | lower);          // (halves without a sign)
}

// f(0) .. f(N - 1), each a constant of the program
template <typename F, int... I>
__device__ __forceinline__ void each(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
template <int N, typename F>
__device__ __forceinline__ void each(F f) { each(f, std::make_integer_sequence<int, N>()); }

template <int EB>
__device__ __forceinline__ void store4(gchar* p, float a, float b, float c, float d) {
  if constexpr (EB == 4) *(ADSA_GLOBAL u32x4*)p = u32x4{__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d)};
  else *(ADSA_GLOBAL u32x2*)p = u32x2{pack2_bf16(a, b), pack2_bf16(c, d)};
}

// What a bf16 pair leaves of two fp32 values, as another pair: the two hold 16 bits of each.  (A dot product with -1 and 0 takes one of a pair.  The
// constants come in registers: the compiler writes -1 in one half as the inline constant -1.0, which gave wrong results.)
__device__ __forceinline__ uint32_t rest2_bf16(uint32_t pair, float a, float b) {
  const bf16x2 x = __builtin_bit_cast(bf16x2, pair);
  uint32_t lower = 0x0000BF80u, upper = 0xBF800000u;
  asm("" : "+s"(lower));
  asm("" : "+s"(upper));
  return pack2_bf16(__builtin_amdgcn_fdot2_f32_bf16(x, __builtin_bit_cast(bf16x2, lower), a, false),
                    __builtin_amdgcn_fdot2_f32_bf16(x, __builtin_bit_cast(bf16x2, upper), b, false));
}

// What is done to scores before the softmax.
struct Mods {
  const float* slopes;         // per query head, or NULL
  const int32_t* doc;          // [n_seq][doc_stride], or NULL
  long long doc_stride;
  float cap_in, cap_out;       // softmax scale / cap, cap * log2(e); cap_out 0: no cap
  bool wide;                   // a cap so far off that scores near 0 need more than capped<2> keeps of them (bf16)
  float scale_log2;            // softmax scale * log2(e)
};

// The keys of a workgroup, one (sequence, cache head): entries [begin, end) of a list of slots, or the slots themselves.
struct Keys {
  const gchar* k;              // row of slot 0
  const gchar* v;
  long long stride_b;
  const gint* list;
  const gint* pos;             // of slots (slopes)
  const gint* doc;             // of slots
  gfloat* logits;              // own lists: scores of row 0 of the tile, log2 units; the next row's lg_stride on
  int lg_stride, lg_rows;
  int begin, end, last_slot, skip;     // skip: a slot that is not attended
  int pos0;                    // positions are taken from here (slopes): fp32 holds near ones whole, whatever the absolute ones are
};

// A lane's row: what it sees are keys below `limit` (of its document).
struct Row {
  int limit, pos, doc;         // pos: from the keys' pos0
  float slope;                 // log2 units
};

template <int EB, int D> struct Layout {
  static constexpr int RB = D * EB, CPR = RB / 16;         // bytes and 16-byte pieces of a row
  // A row's pieces are permuted so that the 16 lanes of an LDS access that read the same piece of 16 rows (K), or 4 rows' pieces of
  // 16 columns (V), meet all banks.
  static __device__ __forceinline__ int swz_k(int row) { return CPR == 8 ? (row >> 1) & 7 : row & 15; }
  static __device__ __forceinline__ int swz_v(int row) {
    return EB == 4 ? ((row >> 2) & 1) << 3 : CPR == 8 ? ((row >> 1) & 1) << 2 : (row & 3) << 2;
  }
};

__device__ __forceinline__ uint4 lds16(const lchar* p) {
  const u32x4 v = *(const ADSA_LDS u32x4*)p;
  return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ void put16(lchar* p, const uint4& x) { *(ADSA_LDS u32x4*)p = u32x4{x.x, x.y, x.z, x.w}; }

__device__ __forceinline__ bool bf16_bad(uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }
__device__ __forceinline__ uint32_t bf16_finite(uint32_t w) {            // infinities and NaN as 0
  if ((w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
  if ((w & 0x7F800000u) == 0x7F800000u) w &= 0xFFFFu;
  return w;
}
// whether one of N 16-byte pieces of bf16 values holds an infinity or a NaN
template <int N>
__device__ __forceinline__ bool bf16_bad_among(const uint4 (&r)[N]) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  u16x2 most = {0, 0};
  auto meet = [&](uint32_t w) { most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu)); };
#pragma unroll
  for (int i = 0; i < N; ++i) { meet(r[i].x); meet(r[i].y); meet(r[i].z); meet(r[i].w); }
  return most.x >= 0x7F80 || most.y >= 0x7F80;
}
// ones (bf16) where w's values are +infinity or -infinity; a NaN counts as both
__device__ __forceinline__ uint32_t ones_at(uint32_t w, bool negative) {
  auto hit = [&](uint32_t h) { return (h & 0x7FFFu) > 0x7F80u || h == (negative ? 0xFF80u : 0x7F80u); };
  return (hit(w & 0xFFFFu) ? 0x3F80u : 0u) | (hit(w >> 16) ? 0x3F800000u : 0u);
}
__device__ __forceinline__ bool f32_bad(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }

// Capped score: fp32 sum q.k -> log2 units.  bf16: tanh t = 1 - 2 / (e^2t + 1), three instructions of which two are transcendental.  What it is off
// by does not shrink with t: about 2^-22 of the cap, 6e-5 of a score's unit at kWideCap, which bf16 probabilities (2^-9) and lse hide.
constexpr float kWideCap = 256.0f;
template <int EB>
__device__ __forceinline__ float capped(float s, const Mods& mods) {
  if constexpr (EB == 4) return mods.cap_out * tanhf(s * mods.cap_in);
  return fmaf(-2.0f * mods.cap_out, __builtin_amdgcn_rcpf(fast_exp2(s * (mods.cap_in * (2.0f * kLog2e))) + 1.0f), mods.cap_out);
}
// ... beyond kWideCap: within 2^-20 of the score itself, by tanh's series (to t^11; the next term is 1e-8 of t at 0.35) and, further out, by
// (1 - e^-2t) / (1 + e^-2t).
__device__ __forceinline__ float capped_wide(float s, const Mods& mods) {
  const float t = s * mods.cap_in, a = fabsf(t), x = t * t, u = fast_exp2(a * (-2.0f * kLog2e));
  const float near = fmaf(x, fmaf(x, fmaf(x, fmaf(x, fmaf(x, -1382.0f / 155925.0f, 62.0f / 2835.0f), -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f) * t;
  const float far = copysignf((1.0f - u) * __builtin_amdgcn_rcpf(1.0f + u), t);
  return mods.cap_out * (a < 0.35f ? near : far);
}
template <int EB>
__device__ __forceinline__ float capped_any(float s, const Mods& mods) {
  if constexpr (EB == 2)
    if (mods.wide) return capped_wide(s, mods);
  return capped<EB>(s, mods);
}

// Two waves share a SIMD's registers, but for fp32 rows of 128, whose steps alone take half of one's.  (Within 256 registers products are formed in
// those the vector unit works on, too; beyond, scores and outputs would be copied between the two kinds.)
template <int EB, int D> constexpr int kWavesPerSimd = EB == 4 && D == 128 ? 1 : 2;

template <int EB, int D, int WK> struct Shape {
  static constexpr int kThreads = WK * kWave, kRows = 32;      // rows of a workgroup's tile
  static constexpr int TK = WK * 32;                   // keys of a step
  static constexpr int kMeta = 2 * TK * Layout<EB, D>::RB;             // LDS: K, V, then per key: position (float), document, flag
  static constexpr int kStep = kMeta + 3 * TK * 4;
  static constexpr int kMerge = WK * (D / 32) * 16 * kWave * 4 + 2 * WK * kWave * 4;       // over the same memory, behind the loop
  static constexpr int kLds = kStep > kMerge ? kStep : kMerge;
};

// The attention of a workgroup's 32 rows (a lane's q pieces in qf) over its keys, which its waves split: each stages the 32 rows of a step that it
// alone reads, so nobody waits for anybody in the loop (its own lanes' hand-over apart).  Afterwards m, l (of the lane's row, both halves of the wave alike) and the wave's
// share of the unnormalised outputs: acc[r], r in [0, D / 32 * 16 / WK), are the elements of register r + wk * (...) of the D / 32
// transposed 32x32 blocks.
// ALL: every row sees every key of the list or prompt, so none can hold what must not reach a row.  What stands in for others (past the end, or
// for the query token) counts as 0 in V: its probability is 0, but 0 times an infinity is not.
template <int EB, int D, int WK, bool MOD, bool LIST, bool ALL>
struct Tile {
  using L = Layout<EB, D>;
  using S = Shape<EB, D, WK>;
  static constexpr int KT = 32, TK = S::TK, CPR = L::CPR, RB = L::RB, DT = D / 32;
  static constexpr int RPT = kWave / CPR, NL = KT / RPT;                // rows per round of a wave; rounds
  static constexpr int kMine = DT * 16 / WK;                            // output registers of a lane after the waves' merge
  static constexpr bool SPLIT = EB == 2;                                // probabilities in two bf16, which hold 16 bits of them
  static_assert(NL * RPT == KT && kMine % 4 == 0, "whole rounds");

  const Mods& mods;
  const Keys& keys;
  lchar* const lds;
  const int tid, lane, col, half, wk;
  uint4 qf[CPR / 2];
  Row row;
  f32x16 acc[DT];
  float m, l;
  bool bad;                    // V held infinities or NaN where not every row sees them (SPLIT: anywhere; times what is left of a probability they
                               // may be anything)
  bool bad_here;               // SPLIT: in the wave's staged rows
  // the next step's rows on their way
  uint4 kr[NL], vr[NL];
  int slot_next[NL], meta_next, stand_in;        // LIST: entries of the step after it
  int meta_slot;
  int meta_pos;
  int meta_doc;

  __device__ __forceinline__ Tile(const Mods& mods_, const Keys& keys_, lchar* lds_)
      : mods(mods_), keys(keys_), lds(lds_), tid(threadIdx.x), lane(threadIdx.x % kWave), col(lane % 32), half(lane / 32),
        wk(__builtin_amdgcn_readfirstlane(tid / kWave)) {}

  // row number i of the thread among a step's, and the one whose position, document and flag it brings (if `brings`)
  __device__ __forceinline__ int staged(int i) const { return wk * KT + lane / CPR + i * RPT; }
  __device__ __forceinline__ bool brings() const { return lane < KT; }
  __device__ __forceinline__ int brought() const { return wk * KT + lane; }

  __device__ __forceinline__ void load_q(const gchar* q_row) {
#pragma unroll
    for (int s = 0; s < CPR / 2; ++s) qf[s] = load16(q_row + (2 * s + half) * 16);
  }

  // LIST: entries are asked for a step before the rows they name, and looked at only when those are (a look waits for whatever was asked for before it,
  // the rows of the step ahead among it).  Instead of the slot that is not attended (rows of the cache that hold nothing yet must not reach the sums,
  // not even times 0): another one of the list.
  __device__ __forceinline__ int entry(int key) const { return keys.list[min(key, keys.end - 1)]; }
  __device__ __forceinline__ int slot_of(int entry) const { return min(max(entry == keys.skip ? stand_in : entry, 0), keys.last_slot); }
  __device__ __forceinline__ void load_slots(int base) {
    if constexpr (LIST) {
#pragma unroll
      for (int i = 0; i < NL; ++i) slot_next[i] = entry(base + staged(i));
      int first = base + wk * KT;                    // (a sum with the lane that is kept would be spilled, and its reload waits for the rows asked for)
      asm volatile("" : "+s"(first));
      if (brings()) meta_next = entry(first + lane);
    }
  }
  __device__ __forceinline__ void load_rows(int base) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int slot = LIST ? slot_of(slot_next[i]) : min(base + staged(i), keys.end - 1);
      const long long off = (long long)slot * keys.stride_b + (tid % CPR) * 16;
      kr[i] = load16(keys.k + off);
      vr[i] = load16(keys.v + off);
    }
    if (brings()) {
      if constexpr (LIST) meta_slot = meta_next;
      if constexpr (MOD) {
        const int slot = LIST ? slot_of(meta_next) : min(base + brought(), keys.end - 1);
        meta_pos = mods.slopes ? keys.pos[slot] : keys.pos0;       // (not touched before store_rows: a touch waits for the rows)
        meta_doc = keys.doc ? keys.doc[slot] : 0;
      }
    }
  }
  __device__ __forceinline__ void store_rows(int base) {
    if constexpr (SPLIT) bad_here = __ballot(bf16_bad_among(vr)) != 0;
    if (ALL && base + wk * KT + KT > keys.end) {     // (uniform: the wave's last step)
      int past = base + staged(0) - keys.end;
      asm volatile("" : "+v"(past));                 // (formed here: no registers in the loop)
#pragma unroll
      for (int i = 0; i < NL; ++i)
        if (past + i * RPT >= 0) vr[i] = make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int r = staged(i), c = tid % CPR;
      put16(lds + r * RB + ((c ^ L::swz_k(r)) << 4), kr[i]);
      put16(lds + TK * RB + r * RB + ((c ^ L::swz_v(r)) << 4), vr[i]);
    }
    if (brings()) {
      ADSA_LDS int* const meta = (ADSA_LDS int*)(lds + S::kMeta) + brought();
      if constexpr (MOD) { meta[0] = __float_as_int((float)(meta_pos - keys.pos0)); meta[TK] = meta_doc; }
      if constexpr (LIST) meta[2 * TK] = meta_slot == keys.skip;
    }
  }

  // The lane's piece of V^T for 32 elements (block dt) and 16 keys (t) of the 32 from row r0 on, bf16: element j of a lane of half h belongs to
  // key 16 t + 8 (j / 4) + 4 h + j % 4, where the score register 8 t + j has it.  A transposing load gives lane i of 16 column i of
  // 4 rows of 16 elements, of which lane 4 r + c addresses 4 elements of row r from column 4 c on.
  __device__ __forceinline__ u32x4 value_piece(int r0, int dt, int t) const {
    const int vrow = r0 + half * 4 + (lane % 16) / 4, vcol = ((lane / 16) & 1) * 16 + (lane % 4) * 4;
    const lchar* const at = lds + TK * RB + (vrow + 16 * t) * RB + (vcol % 8) * 2 + (((dt * 4 + vcol / 8) ^ L::swz_v(vrow)) << 4);
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ADSA_LDS i16x4*)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ADSA_LDS i16x4*)(at + 8 * RB));
    const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
    return u32x4{a.x, a.y, b.x, b.y};
  }
  // fp32: element dt * 32 + lane % 32 of the key that score register i of this half belongs to
  __device__ __forceinline__ float value(int r0, int i, int dt) const {
    const int key = r0 + (i / 4) * 8 + half * 4 + i % 4;
    return *(const ADSA_LDS float*)(lds + TK * RB + key * RB + (((dt * 8 + col / 4) ^ L::swz_v(key)) << 4) + (col % 4) * 4);
  }
  // O^T += V^T P^T over the 32 keys from row r0 of the step
  __device__ __forceinline__ void add_values(int r0, const float* p) {
    if constexpr (EB == 2) {
      bf16x8 pb[2], pr[2];                           // pr (SPLIT): what pb leaves of the probabilities
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        u32x4 w, rest = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = pack2_bf16(p[8 * t + 2 * i], p[8 * t + 2 * i + 1]);
          if constexpr (SPLIT) rest[i] = rest2_bf16(w[i], p[8 * t + 2 * i], p[8 * t + 2 * i + 1]);
        }
        pb[t] = __builtin_bit_cast(bf16x8, w);
        pr[t] = __builtin_bit_cast(bf16x8, rest);
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const u32x4 w = value_piece(r0, dt, t);
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), pb[t], acc[dt], 0, 0, 0);
          if constexpr (SPLIT) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), pr[t], acc[dt], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(value(r0, i, dt), p[i], acc[dt], 0, 0, 0);
        }
    }
  }
  // whether V of these 32 keys holds an infinity or a NaN
  __device__ __forceinline__ bool values_bad(int r0) const {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 32 * CPR / kWave; ++i) {
      const uint4 w = lds16(lds + TK * RB + r0 * RB + (i * kWave + lane) * 16);
      if constexpr (EB == 2) bad |= bf16_bad(w.x) || bf16_bad(w.y) || bf16_bad(w.z) || bf16_bad(w.w);
      else bad |= f32_bad(__uint_as_float(w.x)) || f32_bad(__uint_as_float(w.y)) || f32_bad(__uint_as_float(w.z)) || f32_bad(__uint_as_float(w.w));
    }
    return __ballot(bad) != 0;
  }
  // ... and what those give the rows that see their key: where V holds +infinity (and where -infinity, NaN counting as both) the
  // product of ones there with ones for p > 0 says which rows have one among their keys.
  __device__ __forceinline__ void add_bad_values(int r0, const float* p) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int negative = 0; negative < 2; ++negative) {
        f32x16 r = {};
        if constexpr (EB == 2) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const u32x4 w = value_piece(r0, dt, t);
            u32x4 x;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = (p[8 * t + 2 * i] > 0.0f ? 0x3F80u : 0u) | (p[8 * t + 2 * i + 1] > 0.0f ? 0x3F800000u : 0u);
            const u32x4 o = {ones_at(w.x, negative), ones_at(w.y, negative), ones_at(w.z, negative), ones_at(w.w, negative)};
            r = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, o), __builtin_bit_cast(bf16x8, x), r, 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float a = value(r0, i, dt);
            const bool hit = a != a || a == (negative ? -INFINITY : INFINITY);
            r = __builtin_amdgcn_mfma_f32_32x32x2f32(hit ? 1.0f : 0.0f, p[i] > 0.0f ? 1.0f : 0.0f, r, 0, 0, 0);
          }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] += r[i] > 0.0f ? (negative ? -INFINITY : INFINITY) : 0.0f;
        __builtin_amdgcn_sched_barrier(0);           // (one after the other: registers matter here, time does not)
      }
  }
  __device__ __forceinline__ void clear_bad_values(int r0) const {           // (the rows are the wave's own)
#pragma unroll 1
    for (int i = 0; i < 32 * CPR / kWave; ++i) {
      lchar* const at = lds + TK * RB + r0 * RB + (i * kWave + lane) * 16;
      uint4 w = lds16(at);
      if constexpr (EB == 2) w = make_uint4(bf16_finite(w.x), bf16_finite(w.y), bf16_finite(w.z), bf16_finite(w.w));
      else {
        auto tidy = [](uint32_t x) { return f32_bad(__uint_as_float(x)) ? 0u : x; };
        w = make_uint4(tidy(w.x), tidy(w.y), tidy(w.z), tidy(w.w));
      }
      put16(at, w);
    }
  }

  // scores of one step's keys of this wave, to be multiplied by score_scale(); masked: some row does not see all of them
  __device__ __forceinline__ float score_scale() const { return MOD ? 1.0f : mods.scale_log2; }
  __device__ __forceinline__ f32x16 scores(int base, bool masked) const {
    const int r0 = wk * KT;
    f32x16 s = {};
    const lchar* const krow = lds + (r0 + col) * RB;
    const int sw = L::swz_k(r0 + col);
#pragma unroll
    for (int c = 0; c < CPR / 2; ++c) {
      const uint4 a = lds16(krow + (((2 * c + half) ^ sw) << 4));
      if constexpr (EB == 2) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, qf[c]), s, 0, 0, 0);
      else {
        const uint32_t ka[4] = {a.x, a.y, a.z, a.w}, qa[4] = {qf[c].x, qf[c].y, qf[c].z, qf[c].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(ka[e]), __uint_as_float(qa[e]), s, 0, 0, 0);
      }
    }
    const ADSA_LDS int* const meta = (const ADSA_LDS int*)(lds + S::kMeta) + r0;
    auto key_of = [&](int i) { return (i / 4) * 8 + half * 4 + i % 4; };      // of the lane's score number i
    if constexpr (MOD) {
      if (EB == 2 && mods.wide) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[i] = capped_wide(s[i], mods);
          __builtin_amdgcn_sched_barrier(0);         // (registers matter here)
        }
      } else if (mods.cap_out != 0.0f) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = capped<EB>(s[i], mods);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] *= mods.scale_log2;
      }
      if (mods.slopes) {
        const float here = (float)row.pos;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(-row.slope, fabsf(here - __int_as_float(meta[key_of(i)])), s[i]);
      }
    }
    if (masked) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        bool seen = base + r0 + key_of(i) < row.limit;
        if constexpr (LIST) seen &= meta[2 * TK + key_of(i)] == 0;
        if constexpr (MOD)
          if (keys.doc) seen &= meta[TK + key_of(i)] == row.doc;
        s[i] = seen ? s[i] : -INFINITY;
      }
    }
    return s;
  }
  __device__ __forceinline__ void fold(int base, bool masked) {
    const int r0 = wk * KT;
    const float scale = score_scale();
    const f32x16 s = scores(base, masked);
    if constexpr (LIST) {
      if (keys.logits && col < keys.lg_rows) {       // four at a time: a row's padding to a multiple of 4 may get something, too
        gfloat* const at = keys.logits + (size_t)col * keys.lg_stride;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const int k = base + r0 + i * 2 + half * 4;
          if (k < keys.end) store4<4>((gchar*)(at + k), s[i] * scale, s[i + 1] * scale, s[i + 2] * scale, s[i + 3] * scale);
        }
      }
    }
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);     // (no asm here: a product's result takes wait states that the compiler counts)
    mx = xor_max<32>(mx) * scale;
    if (__ballot(mx > m) != 0) {                     // some row's maximum rose: bring every row's state to its new one
      const float m_new = max2(m, mx), corr = fast_exp2(m - m_new);
      m = m_new;
      l *= corr;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] *= corr;
    }
    float p[16], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = fast_exp2(fmaf(s[i], scale, -m));
      sum += p[i];
    }
    l += sum;
    if (SPLIT ? bad_here : !ALL && masked && values_bad(r0)) {                 // as 0 for now
      clear_bad_values(r0);
      wave_lds_sync();
      bad = true;
    }
    add_values(r0, p);
  }
  // Infinities and NaN of V that not every row of their step saw, or (SPLIT) any (rare): another pass over the keys, behind the loop, whose registers have no room for it.
  __device__ __forceinline__ void fold_bad(int base, bool masked) {
    const int r0 = wk * KT;
    if ((!SPLIT && !masked) || !values_bad(r0)) return;
    const f32x16 s = scores(base, masked);
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = fast_exp2(fmaf(s[i], score_scale(), -m));
    add_bad_values(r0, p);
  }

  __device__ __forceinline__ void run() {
    m = kLowest;
    l = 0.0f;
    bad = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x16{};
    // keys that all rows of the wave see, and that none sees any more
    int lo = row.limit, hi = row.limit;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) { lo = min(lo, __shfl_xor(lo, x)); hi = max(hi, __shfl_xor(hi, x)); }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    int doc_lo = 0x7FFFFFFF, doc_hi = -1;            // of the wave's rows
    if constexpr (MOD)
      if (keys.doc) {
        if (row.doc >= 0) doc_lo = doc_hi = row.doc;
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) { doc_lo = min(doc_lo, __shfl_xor(doc_lo, x)); doc_hi = max(doc_hi, __shfl_xor(doc_hi, x)); }
      }
    // what the wave is to do about a staged step: nothing, fold it, and whether some row does not see all of it
    auto examine = [&](int first, bool* masked) {
      bool wanted = first < hi;
      *masked = first + KT > lo;
      if constexpr (MOD)
        if (keys.doc && wanted) {                    // documents of the rows among the step's? only the rows' one?
          const int d = ((const ADSA_LDS int*)(lds + S::kMeta))[TK + wk * KT + lane % KT];
          wanted = __ballot(d >= doc_lo && d <= doc_hi) != 0;
          *masked |= __ballot(d != doc_lo || d != doc_hi) != 0;
        }
      if constexpr (LIST) {
        if (keys.skip >= 0) {
          int at = lane;
          asm volatile("" : "+v"(at));               // (as in store_rows)
          const uint64_t hit = __ballot(at < KT && ((const ADSA_LDS int*)(lds + S::kMeta))[2 * TK + wk * KT + at % KT] != 0);
          *masked |= hit != 0;
          if (hit != 0) {                            // (a list names a slot once)
            int piece = lane;
            uint32_t zero = 0;
            asm volatile("" : "+v"(piece), "+v"(zero));          // (as in store_rows)
            if (piece < CPR) put16(lds + TK * RB + (wk * KT + __builtin_ctzll(hit)) * RB + piece * 16, make_uint4(zero, zero, zero, zero));
            wave_lds_sync();
          }
        }
      }
      return wanted;
    };
    bool masked;
    if constexpr (LIST) {
      stand_in = keys.list[keys.begin];
      if (stand_in == keys.skip) stand_in = keys.list[min(keys.begin + 1, keys.end - 1)];
      stand_in = __builtin_amdgcn_readfirstlane(stand_in);
    }
    load_slots(keys.begin);
    load_rows(keys.begin);
    load_slots(keys.begin + TK);
    const int end = min(hi, keys.end);               // (from here on keys are others')
    for (int base = keys.begin; base + wk * KT < end; base += TK) {
      wave_lds_sync();                               // (the step before has been read)
      store_rows(base);
      wave_lds_sync();
      if (base + TK < keys.end) {
        load_rows(base + TK);
        load_slots(base + 2 * TK);
      }
      if (examine(base + wk * KT, &masked)) fold(base, masked);
    }
    if constexpr (!ALL || SPLIT)
      if (bad)                                       // (uniform)
        for (int base = keys.begin; base + wk * KT < end; base += TK) {
          load_slots(base);
          load_rows(base);
          wave_lds_sync();
          store_rows(base);
          wave_lds_sync();
          if (examine(base + wk * KT, &masked)) fold_bad(base, masked);
        }
    l = xor_sum<32>(l);
    {                                                // the waves' states meet in LDS
      ADSA_LDS float* const a = (ADSA_LDS float*)lds;
      ADSA_LDS float* const ml = a + WK * DT * 16 * kWave;
      __syncthreads();
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) a[((wk * DT + dt) * 16 + i) * kWave + lane] = acc[dt][i];
      ml[wk * kWave + lane] = m;
      ml[(WK + wk) * kWave + lane] = l;
      __syncthreads();
      float w[WK], M = kLowest, sum = 0.0f;
#pragma unroll
      for (int k = 0; k < WK; ++k) M = fmaxf(M, ml[k * kWave + lane]);
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        w[k] = fast_exp2(ml[k * kWave + lane] - M);
        sum = fmaf(ml[(WK + k) * kWave + lane], w[k], sum);
      }
      m = M;
      l = sum;
#pragma unroll
      for (int r = 0; r < kMine; ++r) {
        float x = 0.0f;
#pragma unroll
        for (int k = 0; k < WK; ++k) x = fmaf(a[(k * DT * 16 + wk * kMine + r) * kWave + lane], w[k], x);
        acc[r / 16][r % 16] = x;
      }
    }
  }
  // first of the 4 consecutive elements that registers r .. r + 3 of the wave's share hold
  __device__ __forceinline__ int element(int r) const {
    const int i = wk * kMine + r;
    return i / 16 * 32 + i % 16 / 4 * 8 + half * 4;
  }
};


// Many rows of a bf16 prompt: W waves of 32 rows each, keys in steps of 32, two steps to a tile of K and V in LDS.
//
// What bounds it: a step is 2 x D / 16 products of 32x32x16, 32 cycles of the SIMD's matrix core each, and about 100 vector instructions
// (16 exponentials at half the rate, their arguments, sums, maxima, conversions), as many cycles again, so neither may wait for the other.
// So a wave takes whatever is independent at one time: the scores of step j + 1 and the outputs of step j - 1 on the matrix core, the softmax of
// step j on the vector unit, laid out alternately by hand (a product, then its share of the vector work), since the
// compiler left alone puts all of one kind before the other.
// A row's maximum is looked for only where a lane's sum of P passes 2^20 (the first keys', a row's first ones behind a mask, and next to never
// after that), so no score waits for the others of its step; P is as exact at 2^20 as at 1.  It is followed where it has grown by more than 2^8.
// MODS: kPlain, kCapped (by a tanh, nothing else), kAny (distances, documents or both, without a branch for either) or kAnyCapped (the same, capped; also caps
// beyond kWideCap; the cap is looked for at every score, which leaves little of the alternation).
enum : int { kPlain, kCapped, kAny, kAnyCapped };
// SPLIT: probabilities in two bf16, which hold 16 bits of them, and half as many products again.  DOCS: keys may have documents.
template <int D, int W, int MODS, bool SPLIT, bool DOCS>
struct Flow {
  static constexpr bool MOD = MODS >= kAny;          // keys' positions and documents are wanted (0 where there are none)
  using L = Layout<2, D>;
  static constexpr int CPR = L::CPR, RB = L::RB, DT = D / 32, KC = D / 16, VC = DT * 2, NC = KC + VC;
  static constexpr int kThreads = W * kWave, kRows = W * 32, TK = 64;
  static constexpr int RPT = kThreads / CPR, NL = TK / RPT;
  static constexpr int kV = 2 * TK * RB, kMeta = 2 * kV, kFlag = kMeta + (MOD ? 3 * 2 * TK * 4 : 0), kLds = kFlag + 16;      // two tiles of K, of V; positions and documents of three;
                                                     // whether a tile of V holds infinities or NaN
  static constexpr float kGrowth = 8.0f, kMost = 1048576.0f;

  const Mods& mods;
  const Keys& keys;
  lchar* const lds;
  const int tid, lane, col, half, wave;
  uint4 qf[KC];
  Row row;
  f32x16 acc[DT], s;
  static constexpr int PW = SPLIT ? 16 : 8;
  uint32_t p[PW];          // probabilities of the step before, two to a word (SPLIT: then what those leave of them)
  float m, l;
  uint4 kr[NL], vr[NL];
  int meta_pos, meta_doc;
  // LDS offsets: the lane's pieces of the tile of K and of V that are read, the thread's of those that are written.  Each changes buffers
  // with every tile (K's two lie TK * RB apart, an offset's bit of that value says which; so do V's).
  // FEW: registers are short (what is asked for ahead would be spilled, which waits for it), and offsets are formed from the first one's, of whose
  // bits they differ in some.  us without | with: 64 x 8 tokens x 64 heads over 8 x 128 behind 2000 slots, lowered with distance, 213 | 141.
  static constexpr bool FEW = (MOD || SPLIT) && D == 128;
  static constexpr int KA = FEW ? 1 : KC, VA = FEW ? 1 : DT, RA = FEW ? 1 : NL;
  int k_at[KA], v_at[VA], k_to, v_to;
  uint32_t row_at[RA];         // offsets of the thread's rows of a tile from its first

  __device__ __forceinline__ Flow(const Mods& mods_, const Keys& keys_, lchar* lds_)
      : mods(mods_), keys(keys_), lds(lds_), tid(threadIdx.x), lane(threadIdx.x % kWave), col(lane % 32), half(lane / 32),
        wave(__builtin_amdgcn_readfirstlane(tid / kWave)) {
#pragma unroll
    for (int i = 0; i < RA; ++i) row_at[i] = (uint32_t)((tid / CPR + i * RPT) * (int)keys.stride_b + (tid % CPR) * 16);
#pragma unroll
    for (int c = 0; c < KA; ++c) k_at[c] = col * RB + (((2 * c + half) ^ L::swz_k(col)) << 4);
    const int vrow = half * 4 + (lane % 16) / 4, vcol = ((lane / 16) & 1) * 16 + (lane % 4) * 4;       // (see Tile::add_values)
#pragma unroll
    for (int dt = 0; dt < VA; ++dt) v_at[dt] = kV + TK * RB + vrow * RB + (vcol % 8) * 2 + (((dt * 4 + vcol / 8) ^ L::swz_v(vrow)) << 4);
    const int r = tid / CPR;                         // (rows RPT further on are permuted alike)
    static_assert(RPT % 16 == 0, "swizzles repeat");
    k_to = r * RB + (((tid % CPR) ^ L::swz_k(r)) << 4);
    v_to = kV + r * RB + (((tid % CPR) ^ L::swz_v(r)) << 4);
  }
  __device__ __forceinline__ void change_buffers() {
#pragma unroll
    for (int c = 0; c < KA; ++c) k_at[c] ^= TK * RB;
#pragma unroll
    for (int dt = 0; dt < VA; ++dt) v_at[dt] ^= TK * RB;
    k_to ^= TK * RB;
    v_to ^= TK * RB;
  }
  __device__ __forceinline__ void load_q(const gchar* q_row) {
#pragma unroll
    for (int c = 0; c < KC; ++c) qf[c] = load16(q_row + (2 * c + half) * 16);
  }

  // rows of a tile on their way: 32-bit offsets from the tile's first row, which hold for every tile but a last, shorter one
  __device__ __forceinline__ void load_tile(const gchar* from, int base, uint4 (&r)[NL]) {
    const gchar* const first = from + (long long)base * keys.stride_b;
    const int last = keys.end - 1 - base;
    if (last >= TK - 1) {
#pragma unroll
      for (int i = 0; i < NL; ++i) r[i] = FEW ? load16(first + (long long)(i * RPT) * keys.stride_b + row_at[0]) : load16(first + row_at[i % RA]);
    } else {
#pragma unroll
      for (int i = 0; i < NL; ++i) r[i] = load16(first + (uint32_t)(min(tid / CPR + i * RPT, last) * (int)keys.stride_b + (tid % CPR) * 16));
    }
  }
  __device__ __forceinline__ void store_k(int third) {
#pragma unroll
    for (int i = 0; i < NL; ++i) put16(lds + k_to + i * RPT * RB, kr[i]);
    if constexpr (MOD)
      if (tid < TK) {
        ADSA_LDS int* const meta = (ADSA_LDS int*)(lds + kMeta) + third * 2 * TK;
        meta[tid] = __float_as_int((float)(meta_pos - keys.pos0));
        if constexpr (DOCS) meta[TK + tid] = meta_doc;
      }
  }
  // check: some row does not see all of the tile (SPLIT: infinities and NaN of V times what is left of a probability may be anything, so all are looked at)
  __device__ __forceinline__ void store_v(int t, bool check) {
#pragma unroll
    for (int i = 0; i < NL; ++i) put16(lds + v_to + i * RPT * RB, vr[i]);
    if (SPLIT || check) {
      if (__ballot(bf16_bad_among(vr)) != 0) *(ADSA_LDS int*)(lds + kFlag + t % 4 * 4) = t + 1;
    }
  }
  __device__ __forceinline__ void load_meta(int base) {
    if constexpr (MOD)
      if (tid < TK) {
        const int slot = min(base + tid, keys.end - 1);
        meta_pos = mods.slopes ? keys.pos[slot] : keys.pos0;       // (not touched before store_k: a touch waits for the rows)
        if constexpr (DOCS) meta_doc = keys.doc ? keys.doc[slot] : 0;
      }
  }

  __device__ __forceinline__ uint4 k_piece(int sub, int c) const { return lds16(lds + (FEW ? k_at[0] ^ c << 5 : k_at[c % KA]) + sub * 32 * RB); }
  __device__ __forceinline__ u32x4 v_piece(int sub, int i) const {
    const lchar* const at = lds + (FEW ? v_at[0] ^ i / 2 << 6 : v_at[i / 2 % VA]) + (sub * 32 + 16 * (i % 2)) * RB;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ADSA_LDS i16x4*)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ADSA_LDS i16x4*)(at + 8 * RB));
    const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
    return u32x4{a.x, a.y, b.x, b.y};
  }
  __device__ __forceinline__ bf16x8 p_piece(int t) const { return __builtin_bit_cast(bf16x8, u32x4{p[4 * t], p[4 * t + 1], p[4 * t + 2], p[4 * t + 3]}); }

  // Infinities and NaN among tile t's rows of V (rare) must not reach rows that do not see them.
  __device__ __forceinline__ bool values_bad(int t) const { return *(const ADSA_LDS int*)(lds + kFlag + t % 4 * 4) == t + 1; }
  // ... and what those give the rows that see their key: where V holds +infinity (and where -infinity, NaN counting as both) the
  // product of ones there with ones for p > 0 says which rows have one among their keys.
  __device__ __forceinline__ void add_bad_values(int sub) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int negative = 0; negative < 2; ++negative) {
        f32x16 r = {};
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const u32x4 w = v_piece(sub, dt * 2 + t);
          u32x4 x = {p[4 * t], p[4 * t + 1], p[4 * t + 2], p[4 * t + 3]};
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = ((x[i] & 0xFFFFu) ? 0x3F80u : 0u) | ((x[i] >> 16) ? 0x3F800000u : 0u);
          const u32x4 o = {ones_at(w.x, negative), ones_at(w.y, negative), ones_at(w.z, negative), ones_at(w.w, negative)};
          r = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, o), __builtin_bit_cast(bf16x8, x), r, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] += r[i] > 0.0f ? (negative ? -INFINITY : INFINITY) : 0.0f;
        __builtin_amdgcn_sched_barrier(0);           // (one after the other: registers matter here, time does not)
      }
  }

  // pieces of the two steps' work
  // positions and documents of the keys of the lane's scores 4 q .. 4 q + 3
  __device__ __forceinline__ u32x4 quad(const ADSA_LDS int* meta, int q) const { return *(const ADSA_LDS u32x4*)(meta + q * 8 + half * 4); }
  // cap and distance of score number i (WIDE: a cap beyond kWideCap)
  template <bool WIDE = false>
  __device__ __forceinline__ void bend(int i, const u32x4& pos) {
    if constexpr (WIDE) s[i] = capped_wide(s[i], mods);
    else if (MODS == kCapped || (MODS == kAnyCapped && mods.cap_out != 0.0f)) s[i] = capped<2>(s[i], mods);
    else s[i] *= mods.scale_log2;
    if constexpr (MOD) s[i] = fmaf(-row.slope, fabsf((float)row.pos - __uint_as_float(pos[i % 4])), s[i]);
  }
  __device__ __forceinline__ void hide(int i, int base, const u32x4& doc) {       // if the row does not see its key, one of those from `base` on
    bool seen = base + (i / 4) * 8 + half * 4 + i % 4 < row.limit;
    if constexpr (DOCS) seen &= (int)doc[i % 4] == row.doc;
    s[i] = seen ? s[i] : -INFINITY;
  }
  __device__ __forceinline__ float score_scale() const { return MODS != kPlain ? 1.0f : mods.scale_log2; }
  // The step's maximum; where it has grown, what the state so far has to be multiplied by.
  __device__ __forceinline__ bool maximum(float* corr) {
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);   // (no asm here: a product's result takes wait states that the compiler counts)
    mx = xor_max<32>(mx) * score_scale();
    const bool grows = mx > m + kGrowth;
    const float m_new = grows ? mx : m;
    *corr = fast_exp2(m - m_new);
    m = m_new;
    return grows;
  }
  __device__ __forceinline__ float probability(int i) const { return fast_exp2(fmaf(s[i], score_scale(), -m)); }
  __device__ __forceinline__ float probabilities(uint32_t (&to)[PW]) const {           // their sum
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float a = probability(i), d = probability(i + 1);
      sum += a;
      sum += d;
      to[i / 2] = pack2_bf16(a, d);
      if constexpr (SPLIT) to[8 + i / 2] = rest2_bf16(to[i / 2], a, d);
    }
    return sum;
  }
  __device__ __forceinline__ void rescale(float corr) {
    l *= corr;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[dt][i] *= corr;
  }
  __device__ __forceinline__ f32x16 score_product(const uint4& k, int c, const f32x16& x) const {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, qf[c]), x, 0, 0, 0);
  }
  __device__ __forceinline__ void output_product(const u32x4& v, int i) {
    acc[i / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), p_piece(i % 2), acc[i / 2], 0, 0, 0);
    if constexpr (SPLIT) acc[i / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), p_piece(2 + i % 2), acc[i / 2], 0, 0, 0);
  }

  // One step (HIDE: of keys that not every row sees): the scores of K's rows (half SUB of the tile), the softmax of the scores s of the step
  // before, the outputs of its predecessor's p with V's rows, alternately.
  template <int SUB, bool HIDE>
  __device__ __forceinline__ void step(int base, const ADSA_LDS int* meta) {
    f32x16 next = {};
    uint32_t pn[PW];
    float even = 0.0f, sum = 0.0f;
    constexpr int kAhead = D == 64 || (MOD && SPLIT) ? 2 : 3;        // pieces fetched ahead of their product (as registers allow)
    uint4 kp[KC];
    u32x4 vp[VC];
    auto fetch = [&](auto at) {
      constexpr int c = decltype(at)::value;
      if constexpr (c < KC) kp[c] = k_piece(SUB, c);
      else if constexpr (c < NC) vp[c - KC] = v_piece(SUB, c - KC);
    };
    u32x4 pos[4] = {}, doc[4] = {};
    auto fetch_quad = [&](auto q) {
      constexpr int i = decltype(q)::value;
      if constexpr (MOD && i < 4) {
        pos[i] = quad(meta, i);
        if constexpr (HIDE && DOCS) doc[i] = quad(meta + TK, i);
      }
    };
    each<kAhead>(fetch);
    fetch_quad(std::integral_constant<int, 0>());
    each<NC>([&](auto at) {
      constexpr int c = decltype(at)::value, i0 = 16 * c / NC, n = 16 * (c + 1) / NC - i0;
      fetch(std::integral_constant<int, c + kAhead>());
      if constexpr (c < KC) next = score_product(kp[c], c, next);
      else output_product(vp[c - KC], c - KC);
      // this chunk's share of the softmax
      if constexpr (i0 % 4 == 0) fetch_quad(std::integral_constant<int, i0 / 4 + 1>());
      each<n>([&](auto o) {
        constexpr int i = i0 + decltype(o)::value;
        if constexpr (MODS != kPlain) bend(i, pos[i / 4]);
        if constexpr (HIDE) hide(i, base, doc[i / 4]);
        const float x = probability(i);
        sum += x;
        if constexpr (i % 2 == 0) even = x;
        else {
          pn[i / 2] = pack2_bf16(even, x);
          if constexpr (SPLIT) pn[8 + i / 2] = rest2_bf16(pn[i / 2], even, x);
        }
        if constexpr (i % 2 == 0) asm volatile("" : "+v"(even), "+v"(sum));            // (here, not where p is used)
        else if constexpr (SPLIT) asm volatile("" : "+v"(pn[i / 2]), "+v"(pn[8 + i / 2]), "+v"(sum));
        else asm volatile("" : "+v"(pn[i / 2]), "+v"(sum));
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    if (__ballot(sum > kMost) != 0) {
      float corr;
      maximum(&corr);
      rescale(corr);
      sum = probabilities(pn);
    }
    l += sum;
    s = next;
#pragma unroll
    for (int i = 0; i < PW; ++i) p[i] = pn[i];
  }

  // The same one after the other: first and last steps (which lack a part), and keys that not every row sees.
  __device__ __forceinline__ void outputs(int sub, bool tidy) {
    if (tidy) add_bad_values(sub);
#pragma unroll
    for (int i = 0; i < VC; ++i) {
      u32x4 w = v_piece(sub, i);
      if (tidy) w = u32x4{bf16_finite(w.x), bf16_finite(w.y), bf16_finite(w.z), bf16_finite(w.w)};
      output_product(w, i);
    }
  }
  __device__ __forceinline__ void scores(int sub) {
    s = f32x16{};
#pragma unroll
    for (int c = 0; c < KC; ++c) s = score_product(k_piece(sub, c), c, s);
  }
  __device__ __forceinline__ void softmax(int base, const ADSA_LDS int* meta) {
    const bool hidden = hides(base);
    auto bend_all = [&](auto wide) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        bend<decltype(wide)::value>(i, MOD ? quad(meta, i / 4) : u32x4{});
        if (decltype(wide)::value) __builtin_amdgcn_sched_barrier(0);                  // (registers matter here)
      }
    };
    if constexpr (MODS == kAnyCapped) {
      if (mods.wide) bend_all(std::true_type());
      else bend_all(std::false_type());
    } else if constexpr (MODS != kPlain) bend_all(std::false_type());
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const u32x4 none = {};
      if (hidden) hide(i, base, DOCS ? quad(meta + TK, i / 4) : none);
    }
    float corr;
    const bool grown = maximum(&corr);
    if (__ballot(grown) != 0) rescale(corr);
    l += probabilities(p);
  }

  // (as a Tile's: outputs r .. r + 3 of the lane are elements from element(r) on)
  static constexpr int kMine = DT * 16, wk = 0;
  __device__ __forceinline__ int element(int r) const { return r / 16 * 32 + r % 16 / 4 * 8 + half * 4; }

  int lo, hi;                  // keys that all rows of the wave see, and from which on none does
  __device__ __forceinline__ bool hides(int first) const {            // whether some row does not see all of the 32 keys from `first` on
    bool x = first + 32 > lo;
    if constexpr (DOCS) x |= keys.doc != nullptr;
    return x;
  }
  // Tile number t (of `mine` that this wave's rows see): the scores of steps 2t and 2t + 1, the softmax of 2t - 1 and 2t, the outputs of 2t - 2
  // and 2t - 1; so K's tile t and V's tile t - 1 are read.
  __device__ __forceinline__ const ADSA_LDS int* meta_of(int t) const { return (const ADSA_LDS int*)(lds + kMeta) + t % 3 * 2 * TK; }
  __device__ __forceinline__ void tile(int t, int mine, bool tidy) {
    if (t > mine || mine == 0) return;
    const int base = keys.begin + t * TK;
    for (int sub = 0; sub < 2; ++sub) {
      if (t > 0) {
        outputs(sub, tidy);
        if (sub == 0) softmax(base - 32, meta_of(t + 2) + 32);
      }
      if (t < mine) {
        if (sub == 1) softmax(base, meta_of(t));
        scores(sub);
      }
    }
  }
  // least: no row of the workgroup sees fewer keys
  __device__ __forceinline__ void run(int least) {
    m = kLowest;
    l = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x16{};
    if (keys.begin >= keys.end) return;              // (a part without keys: there is no row to load)
    lo = hi = row.limit;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) { lo = min(lo, __shfl_xor(lo, x)); hi = max(hi, __shfl_xor(hi, x)); }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    const int tiles = (keys.end - keys.begin + TK - 1) / TK, mine = max(0, (min(hi, keys.end) - keys.begin + TK - 1) / TK);
    // tiles 1 .. open - 1 have no key that some row does not see
    const int open = DOCS && keys.doc ? 1 : min(mine, max(0, lo - 32 - keys.begin) / TK + 1);
    const int checked = DOCS && keys.doc ? 0 : max(0, least - keys.begin) / TK;      // the first tile that some row of the workgroup does not see all of
    if (tid < 4) ((ADSA_LDS int*)(lds + kFlag))[tid] = 0;
    load_tile(keys.k, keys.begin, kr);
    load_meta(keys.begin);
    store_k(0);
    k_to ^= TK * RB;
    __syncthreads();
    load_tile(keys.v, keys.begin, vr);
    if (tiles > 1) { load_tile(keys.k, keys.begin + TK, kr); load_meta(keys.begin + TK); }
    // Between two barriers, tile t's K and tile t - 1's V are read, and tile t + 1's K and tile t's V written, into the other buffers.
    auto next_tile = [&](int t) {
      if (t + 1 < tiles) store_k((t + 1) % 3);
      store_v(t, t >= checked);
      __syncthreads();
      change_buffers();
      if (t + 2 < tiles) { load_tile(keys.k, keys.begin + (t + 2) * TK, kr); load_meta(keys.begin + (t + 2) * TK); }
      if (t + 1 < tiles) load_tile(keys.v, keys.begin + (t + 1) * TK, vr);
    };
    tile(0, mine, false);
    next_tile(0);
    int t = 1;
    const bool wide = MODS == kAnyCapped && mods.wide;                                 // (rare: one after the other throughout)
    for (; t < open && !wide && !(SPLIT && values_bad(t - 1)); ++t) {
      step<0, false>(0, meta_of(t + 2) + 32);
      step<1, false>(0, meta_of(t));
      next_tile(t);
    }
    for (; t < mine && !wide && !values_bad(t - 1); ++t) {
      const int base = keys.begin + t * TK;
      step<0, true>(base - 32, meta_of(t + 2) + 32);
      step<1, true>(base, meta_of(t));
      next_tile(t);
    }
    for (; t <= tiles; ++t) {
      tile(t, mine, values_bad(t - 1));
      if (t < tiles) next_tile(t);
    }
    l = xor_sum<32>(l);
  }
};

// ---------------------------------------------------------------------------------------------------- prompts
struct PromptArgs {
  adsa_seq* seqs;
  const int32_t* begin;
  const int32_t* slot0;
  const char* q;
  char* out;
  float* lse;
  float* part_ml;
  float* part_acc;
  float* norm;                 // NULL: no attention mass wanted
  Mods mods;
  long long slot_stride_b, head_stride_b;
  int n_seq, n_tokens, max_len, h, G, cap, mask, tiles, chunks, advance;
  uint32_t inv_G;              // ceil(2^32 / G) for G > 1: row / G is the upper half of a product (rows are less than 2^17, G at most 16)
  __device__ __forceinline__ int token_of(int row) const { return G == 1 ? row : (int)__umulhi((uint32_t)row, inv_G); }
};

// A sequence's new tokens: where they stand in the packed rows and in the cache.
struct Prompt {
  int from, len, slot0, prefix, status;      // status: 0, or why the record does not fit (one without new tokens does)
};
__device__ __forceinline__ Prompt prompt_of(const PromptArgs& A, int b) {
  const ADSA_GLOBAL adsa_seq& sq = ((const ADSA_GLOBAL adsa_seq*)A.seqs)[b];
  Prompt pr;
  pr.from = ((const gint*)A.begin)[b];
  pr.len = ((const gint*)A.begin)[b + 1] - pr.from;
  pr.slot0 = ((const gint*)A.slot0)[b];
  pr.status = sq.status;
  const int n_res = sq.n_res;
  pr.prefix = A.mask == ADSA_MASK_PREFIX ? sq.n_keep_prefix : 0;
  if (pr.from < 0 || pr.len < 0 || pr.len > A.n_tokens || pr.from > A.n_tokens - pr.len) pr.len = 0;        // (begin[] is not what it should be)
  if (pr.status == 0 && pr.len > 0 && (n_res < 0 || n_res > A.cap || pr.slot0 < 0 || pr.len > A.max_len || pr.slot0 > n_res - pr.len)) pr.status = ADSA_SEQ_BAD_STATE;
  return pr;
}
// keys below this are seen by the token in slot s
__device__ __forceinline__ int limit_of(const Prompt& pr, int s) {
  return s < pr.prefix ? max(s + 1, min(pr.prefix, pr.slot0 + pr.len)) : s + 1;
}

// (pair of sequence and cache head, unit) of a workgroup: workgroups are dealt round robin to the 8 dies, so pairs are dealt by eights and a
// pair's units, which read the same K and V, follow each other on one die.
__device__ __forceinline__ void pair_of(unsigned id, unsigned units, int* pair, int* unit) {
  const unsigned y = id / 8;
  *pair = (int)(y / units * 8 + id % 8);
  *unit = (int)(y % units);
}

// What a workgroup of k_prompt / k_prompt_many is to do; false: nothing (left).
struct Job {
  Prompt pr;
  Keys keys;
  int b, head, chunk, row0, rows;
};
template <int EB, int D, int ROWS, int THREADS>
__device__ __forceinline__ bool job_of(const PromptArgs& A, Job& J) {
  int pair, unit;
  pair_of(blockIdx.x, (unsigned)(A.tiles * A.chunks), &pair, &unit);
  if (pair >= A.n_seq * A.h) return false;
  J.b = pair / A.h;
  J.head = pair % A.h;
  J.chunk = unit % A.chunks;
  const int tile = A.tiles - 1 - unit / A.chunks, tid = threadIdx.x, hq = A.h * A.G;       // (the longest rows first)
  ADSA_GLOBAL adsa_seq& sq = ((ADSA_GLOBAL adsa_seq*)A.seqs)[J.b];
  J.pr = prompt_of(A, J.b);
  if (J.pr.status != 0) {                            // zeros, by the workgroups of the sequence together
    if (J.chunk != 0) return false;
    if (J.head == 0 && tile == 0 && tid == 0 && sq.status == 0) sq.status = J.pr.status;
    for (long long r = tile; r < J.pr.len; r += A.tiles) {
      const size_t at = ((size_t)(J.pr.from + r) * hq + J.head * A.G);
      for (int o = tid; o < A.G * D * EB / 4; o += THREADS) ((gint*)(A.out + at * D * EB))[o] = 0;
      for (int o = tid; o < A.G; o += THREADS) {
        ((gfloat*)A.lse)[at + o] = 0.0f;
        if (A.chunks > 1) ((gfloat*)A.part_ml)[(at + o) * A.chunks * 2 + 1] = -1.0f;           // (k_prompt_finish leaves the row alone)
      }
    }
    return false;
  }
  J.rows = J.pr.len * A.G;
  J.row0 = tile * ROWS;
  if (J.row0 >= J.rows) return false;
  if (A.advance && J.head == 0 && tile == 0 && J.chunk == 0 && tid == 0) sq.step = sq.step + 1;
  Keys& keys = J.keys;
  keys.k = (const gchar*)sq.k + J.head * A.head_stride_b;
  keys.v = (const gchar*)sq.v + J.head * A.head_stride_b;
  keys.stride_b = A.slot_stride_b;
  keys.list = nullptr;
  keys.pos = (const gint*)sq.pos;
  keys.doc = A.mods.doc ? (const gint*)A.mods.doc + J.b * A.mods.doc_stride : nullptr;
  keys.pos0 = A.mods.slopes ? keys.pos[J.pr.slot0 + J.row0 / A.G] : 0;
  keys.logits = nullptr;
  keys.skip = -1;
  // what the tile's last row sees (a row of the prefix may see more than later rows)
  const int end = min(J.row0 + ROWS, J.rows), last_slot = J.pr.slot0 + (end + A.G - 1) / A.G - 1, first_slot = J.pr.slot0 + J.row0 / A.G;
  const int n = max(limit_of(J.pr, last_slot), limit_of(J.pr, first_slot));
  int first = 0, last = n;
  if (keys.doc) {                                    // (uniform) only from the first to the last slot of a document that the tile's rows belong to
    // (each wave to one number by itself: lanes' atomics on one word are done one lane after the other, 7 us of a launch where this takes 1)
    constexpr int NW = THREADS / kWave;
    __shared__ int s_doc[4][NW];                     // least and greatest of the rows' documents, first and last slot of one among them; a wave's
    const int lane = tid % kWave, wave = tid / kWave, slots = last_slot - first_slot + 1;
    auto spread = [&](int lo, int hi, int at) {      // both over the workgroup
#pragma unroll
      for (int x = 1; x < kWave; x <<= 1) { lo = min(lo, __shfl_xor(lo, x)); hi = max(hi, __shfl_xor(hi, x)); }
      if (lane == 0) { s_doc[at][wave] = lo; s_doc[at + 1][wave] = hi; }
      __syncthreads();
#pragma unroll
      for (int w = 0; w < NW; ++w) { lo = min(lo, s_doc[at][w]); hi = max(hi, s_doc[at + 1][w]); }
      return int2{lo, hi};
    };
    int lo = 0x7FFFFFFF, hi = -1;
    for (int i = tid; i < slots; i += THREADS) {
      const int d = keys.doc[first_slot + i];
      if (d >= 0) { lo = min(lo, d); hi = max(hi, d); }
    }
    const int2 docs = spread(lo, hi, 0);
    lo = 0x7FFFFFFF, hi = -1;
    for (int i = tid; i < n; i += THREADS) {
      const int d = keys.doc[i];
      if (d >= docs.x && d <= docs.y) { lo = min(lo, i); hi = i; }
    }
    const int2 at = spread(lo, hi, 2);
    first = at.y < 0 ? 0 : at.x / 32 * 32;
    last = at.y < 0 ? min(n, 1) : at.y + 1;          // (none: one key, which nobody sees)
  }
  const int m = last - first, per = A.chunks == 1 ? m : ((m + A.chunks - 1) / A.chunks + 31) / 32 * 32;
  keys.begin = min(last, first + J.chunk * per);
  keys.end = min(last, keys.begin + per);
  return true;
}
// Row number r of the job (past the last one: that one again): its place among the packed rows, and what it sees.
template <bool MOD>
__device__ __forceinline__ size_t row_of(const PromptArgs& A, const Job& J, int r, Row& row) {
  const int rr = min(r, J.rows - 1), token = rr / A.G, qh = J.head * A.G + rr % A.G, slot = J.pr.slot0 + token;
  row.limit = min(limit_of(J.pr, slot), J.keys.end);   // (a step past the end of a part repeats its last key)
  row.pos = 0;
  row.doc = 0;
  row.slope = 0.0f;
  if constexpr (MOD) {
    if (A.mods.slopes) { row.pos = J.keys.pos[slot] - J.keys.pos0; row.slope = ((const gfloat*)A.mods.slopes)[qh] * kLog2e; }
    if (J.keys.doc) {
      row.doc = J.keys.doc[slot];
      if (row.doc < 0) row.limit = 0;
    }
  }
  return (size_t)(J.pr.from + token) * (A.h * A.G) + qh;
}
__device__ __forceinline__ void store_part(const PromptArgs& A, const Job& J, size_t at, float m, float l) {
  gfloat* const ml = (gfloat*)A.part_ml + (at * A.chunks + J.chunk) * 2;
  ml[0] = m;
  ml[1] = l;
}
__device__ __forceinline__ float inverse(float l) { return l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l; }       // (a NaN stays one)
__device__ __forceinline__ void store_lse(const PromptArgs& A, size_t at, float m, float l) {
  ((gfloat*)A.lse)[at] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
  if (A.norm) ((gfloat*)A.norm)[at] = l == 0.0f ? INFINITY : m + __log2f(l);           // (exp2(z - norm): 0 for a row that sees nothing)
}

// Few rows, or fp32: a Tile.  Bound by dependent trips where keys are few (3 x 2..7 tokens x 20 heads x 64 behind 2011 slots: 10.6 us for 31 MB), by HBM where they are
// many (16 x 1..9 x 24 x 64 behind 700: 15 us, 4.5 TB/s), in fp32 by the matrix core (8 x 900..1000 x 16 x 64: 203 us, 73 TFLOP/s of whole and part-seen blocks).
// (Caps, distances and documents of bf16 rows of 128 spill 14 words, two reloaded in the loop; fp32 rows of 64 six, outside it.)
template <int EB, int D, int WK, bool MOD>
__global__ __launch_bounds__(WK * kWave, (kWavesPerSimd<EB, D>)) void k_prompt(PromptArgs A) {
  using T = Tile<EB, D, WK, MOD, false, false>;
  using S = typename T::S;
  extern __shared__ __align__(16) char s_lds[];
  Job J;
  if (!job_of<EB, D, S::kRows, S::kThreads>(A, J)) return;
  T t(A.mods, J.keys, (lchar*)s_lds);
  const int r = J.row0 + t.col;
  const size_t at = row_of<MOD>(A, J, r, t.row);
  t.load_q((const gchar*)A.q + at * (D * EB));
  t.run();
  if (r >= J.rows) return;
  const bool parts = A.chunks > 1;
  const float inv = parts ? 1.0f : inverse(t.l);
  gfloat* const acc = (gfloat*)A.part_acc + (at * A.chunks + J.chunk) * D;
  gchar* const out = (gchar*)A.out + at * (D * EB);
#pragma unroll
  for (int i = 0; i < T::kMine; i += 4) {
    const f32x16& x = t.acc[i / 16];
    const int j = i % 16;
    if (parts) store4<4>((gchar*)(acc + t.element(i)), x[j], x[j + 1], x[j + 2], x[j + 3]);
    else store4<EB>(out + t.element(i) * EB, x[j] * inv, x[j + 1] * inv, x[j + 2] * inv, x[j + 3] * inv);
  }
  if (t.half == 0 && t.wk == 0) {
    if (parts) store_part(A, J, at, t.m, t.l);
    else store_lse(A, at, t.m, t.l);
  }
}

template <int D, int W, int MODS, bool SPLIT> using PromptFlow = Flow<D, W, MODS, SPLIT, (MODS >= kAny)>;
// Many rows of a bf16 cache: a Flow.  4 x 4352 x 32 x 128 causal 690-710 us (0.89 PFLOP/s), 4 x 4352 x 24 x 64 312 us (0.74), capped ragged prompts of 64 heads over 8
// 226-231 us (0.53; vector unit 58 % of the time and matrix core 24, so the two add up there: prompts of some 580 keys are few tiles a workgroup, and the first
// and last are not interleaved), 2 x 4352 x 32 x 128 lowered with distance 488 us (0.64).  At head size 128 distances and documents need more than the 256 registers: 18 words are spilled (35 with a cap), and
// some reloaded in the loops; plain and capped forms spill 4 outside theirs.  Three waves a SIMD at head size 64, but for distances and documents (16 x 300..600 x 24 x 64 with
// three | two 92 | 59 us: spills).
template <int D, int W, int MODS, bool SPLIT>
__global__ __launch_bounds__(W * kWave, D == 64 && MODS < kAny && !SPLIT ? 3 : 2) void k_prompt_many(PromptArgs A) {
  using F = PromptFlow<D, W, MODS, SPLIT>;
  extern __shared__ __align__(16) char s_lds[];
  Job J;
  if (!job_of<2, D, F::kRows, F::kThreads>(A, J)) return;
  F f(A.mods, J.keys, (lchar*)s_lds);
  const int r = J.row0 + f.wave * 32 + f.col;
  const size_t at = row_of<F::MOD>(A, J, r, f.row);
  f.load_q((const gchar*)A.q + at * (D * 2));
  f.run(min(J.keys.end, limit_of(J.pr, J.pr.slot0 + J.row0 / A.G)));       // (the first row's limit is the least: the prefix's are no less than the first's)
  if (r >= J.rows) return;
  if (A.chunks > 1) {
    gfloat* const acc = (gfloat*)A.part_acc + (at * A.chunks + J.chunk) * D;
#pragma unroll
    for (int dt = 0; dt < F::DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; i += 4) store4<4>((gchar*)(acc + dt * 32 + i * 2 + f.half * 4), f.acc[dt][i], f.acc[dt][i + 1], f.acc[dt][i + 2], f.acc[dt][i + 3]);
    if (f.half == 0) store_part(A, J, at, f.m, f.l);
    return;
  }
  const float inv = inverse(f.l);
  gchar* const out = (gchar*)A.out + at * (D * 2);
#pragma unroll
  for (int dt = 0; dt < F::DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; i += 8) {                // the halves of the wave trade 4 elements each: 8 in a row for both
      const f32x16& x = f.acc[dt];
      const u32x2 u = __builtin_amdgcn_permlane32_swap(pack2_bf16(x[i] * inv, x[i + 1] * inv), pack2_bf16(x[i + 4] * inv, x[i + 5] * inv), false, false);
      const u32x2 v = __builtin_amdgcn_permlane32_swap(pack2_bf16(x[i + 2] * inv, x[i + 3] * inv), pack2_bf16(x[i + 6] * inv, x[i + 7] * inv), false, false);
      store16(out + (dt * 32 + i * 2 + f.half * 8) * 2, make_uint4(u.x, v.x, u.y, v.y));
    }
  if (f.half == 0) store_lse(A, at, f.m, f.l);
}

// Split keys: a wave joins the parts of one row.  Nothing it loads depends on anything but its arguments (bound by one trip to memory): 16 bytes of a
// part's outputs to a lane, 64 * 4 / D parts side by side, and every part's maximum and sum to a lane of its own.  3.3 us for 8 parts of 260 rows of 64.
template <int EB, int D>
__global__ __launch_bounds__(256) void k_prompt_finish(PromptArgs A) {
  constexpr int LPR = D / 4, kSide = kWave / LPR, kBatch = 4;
  const int lane = threadIdx.x % kWave, side = lane / LPR, e = lane % LPR * 4, C = A.chunks;
  const size_t at = (size_t)blockIdx.x * (256 / kWave) + threadIdx.x / kWave;
  if (at >= (size_t)A.n_tokens * A.h * A.G || at >= (size_t)((const gint*)A.begin)[A.n_seq] * A.h * A.G) return;
  const gfloat* const ml = (const gfloat*)A.part_ml + (at * C + min(lane, C - 1)) * 2;
  const gfloat* const acc = (const gfloat*)A.part_acc + at * C * D + e;
  u32x4 part[kBatch];
  auto fetch = [&](int c0) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) part[i] = *(const ADSA_GLOBAL u32x4*)(acc + (size_t)min(c0 + i * kSide + side, C - 1) * D);
  };
  fetch(0);
  const float m = ml[0], l = ml[1];
  if (__shfl(l, 0) < 0.0f) return;                   // (a sequence that is not attended: zeros already)
  float M = m;
#pragma unroll
  for (int x = 1; x < kMaxChunks; x <<= 1) M = fmaxf(M, __shfl_xor(M, x));             // (lanes past the last part repeat it)
  const float w = lane < C ? fast_exp2(m - M) : 0.0f;
  float L = lane < C ? l * w : 0.0f, x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  L = row_sum<16>(L);
  for (int c0 = 0; c0 < C; c0 += kBatch * kSide) {
    if (c0 > 0) fetch(c0);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int c = c0 + i * kSide + side;
      const float f = __shfl(w, min(c, kMaxChunks));   // (0 past the last part)
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = f != 0.0f ? fmaf(__uint_as_float(part[i][k]), f, x[k]) : x[k];
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (kSide == 4) x[k] = xor_sum<16>(x[k]);
    x[k] = xor_sum<32>(x[k]);
  }
  L = __shfl(L, 0);
  const float inv = inverse(L);
  if (side == 0) store4<EB>((gchar*)A.out + (at * D + e) * EB, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  if (lane == 0) store_lse(A, at, M, L);
}

// score[head][slot] += sum over rows of the probability they gave the slot.  A wave keeps NB x 32 slots' K rows as the A operand and meets the rows
// from the first that can see the slots on, 32 at a time; a lane's column is a row, whose normaliser (m + log2 l) it holds, and its registers
// are slots, which it sums up over its rows: lanes meet once, at the end.  The products of a block of rows run beside the exponentials of
// the one before.  Two blocks of slots share a fetch of q rows (with one, LDS takes as long as the products).  4 x 4352 x 32 x 128: 400-430 us, 0.74 PFLOP/s,
// the vector unit busy 54 % of the time and the matrix core 34.
template <int EB, int D, bool MOD> struct Mass {      // (slots' positions and documents, or fp32 rows, take the second block's registers)
  static constexpr int NB = EB == 2 && !MOD ? 2 : 1, kKeys = 4 * 32 * NB, kRows = 64, kTile = kRows * Layout<EB, D>::RB;
  static constexpr int kLds = 2 * kTile;
};
template <int EB, int D, bool MOD>
__global__ __launch_bounds__(256, EB == 2 ? 2 : 1) void k_prompt_mass(PromptArgs A, int key_tiles) {
  using L = Layout<EB, D>;
  using M = Mass<EB, D, MOD>;
  constexpr int CPR = L::CPR, RB = L::RB, RPT = 256 / CPR, NL = M::kRows / RPT, KC = CPR / 2, NB = M::NB;
  extern __shared__ __align__(16) char s_lds[];
  lchar* const lds = (lchar*)s_lds;
  int pair, tile;
  pair_of(blockIdx.x, (unsigned)key_tiles, &pair, &tile);
  if (pair >= A.n_seq * A.h) return;
  const int b = pair / A.h, head = pair % A.h, tid = threadIdx.x, lane = tid % kWave, col = lane % 32, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave), hq = A.h * A.G;
  const Prompt pr = prompt_of(A, b);
  const int n = pr.slot0 + pr.len, rows = pr.len * A.G, key0 = tile * M::kKeys, mine = key0 + wave * 32 * NB;
  if (pr.status != 0 || pr.len == 0 || key0 >= n) return;
  const ADSA_GLOBAL adsa_seq& sq = ((const ADSA_GLOBAL adsa_seq*)A.seqs)[b];
  const gint* const pos = (const gint*)sq.pos;
  const gint* const doc = MOD && A.mods.doc ? (const gint*)A.mods.doc + b * A.mods.doc_stride : nullptr;
  const int pos0 = MOD && A.mods.slopes ? pos[key0] : 0;       // (see Keys)
  uint4 kf[NB][KC];
#pragma unroll
  for (int x = 0; x < NB; ++x) {
    const gchar* const krow = (const gchar*)sq.k + head * A.head_stride_b + (long long)min(mine + x * 32 + col, n - 1) * A.slot_stride_b;
#pragma unroll
    for (int c = 0; c < KC; ++c) kf[x][c] = load16(krow + (2 * c + half) * 16);
  }
  // of the slots that this lane's registers stand for
  auto slot_of = [&](int x, int i) { return min(mine + x * 32 + (i / 4) * 8 + half * 4 + i % 4, n - 1); };
  float kpos[NB][16];
  int kdoc[NB][16];
  if constexpr (MOD) {
#pragma unroll
    for (int x = 0; x < NB; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        kpos[x][i] = A.mods.slopes ? (float)(pos[slot_of(x, i)] - pos0) : 0.0f;
        kdoc[x][i] = doc ? doc[slot_of(x, i)] : 0;
      }
  }
  // the first row that sees the tile: the token of its first slot, or any where the prefix sees itself
  const int row0 = (key0 < pr.prefix ? 0 : max(0, key0 - pr.slot0)) * A.G, steps = (rows - row0 + M::kRows - 1) / M::kRows;
  uint4 qr[NL];
  const gchar* const q_first = (const gchar*)A.q + ((size_t)pr.from * hq + head * A.G) * RB;         // of the sequence, for this cache head
  auto load = [&](int t) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int r = min(row0 + t * M::kRows + tid / CPR + i * RPT, rows - 1), token = A.token_of(r);
      qr[i] = load16(q_first + ((uint64_t)(uint32_t)token * (uint32_t)(hq * RB) + (uint32_t)((r - token * A.G) * RB + (tid % CPR) * 16)));
    }
  };
  auto store = [&](int t) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int r = tid / CPR + i * RPT;
      put16(lds + (t & 1) * M::kTile + r * RB + (((tid % CPR) ^ L::swz_k(r)) << 4), qr[i]);
    }
  };
  // a lane's row of a block: its normaliser, and what it sees (nothing: past the last row)
  struct Column {
    float norm, slope, pos;
    int limit, doc;
  };
  const gfloat* const norm_first = (const gfloat*)A.norm + (size_t)pr.from * hq + head * A.G;
  auto column = [&](int t, int u) {
    const int r = row0 + t * M::kRows + u * 32 + col, rr = min(r, rows - 1), token = A.token_of(rr), g = rr - token * A.G, qh = head * A.G + g, s = pr.slot0 + token;
    Column x;
    x.norm = norm_first[(uint64_t)(uint32_t)token * (uint32_t)hq + (uint32_t)g];
    x.limit = r < rows ? limit_of(pr, s) : 0;
    x.slope = MOD && A.mods.slopes ? ((const gfloat*)A.mods.slopes)[qh] * kLog2e : 0.0f;
    x.pos = MOD && A.mods.slopes ? (float)(pos[s] - pos0) : 0.0f;
    x.doc = MOD && doc ? doc[s] : 0;
    if (MOD && doc && x.doc < 0) x.limit = 0;
    return x;
  };
  f32x16 s0[NB], s1[NB];       // scores of a step's first and second block of rows
  float sum[NB][16];
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[x][i] = 0.0f;
  const float scale = MOD ? 1.0f : A.mods.scale_log2;
  auto product = [&](f32x16 (&next)[NB], int x, int c, const uint4& q) {
    const f32x16 z = {};
    const f32x16& to = c == 0 ? z : next[x];
    if constexpr (EB == 2) next[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[x][c]), __builtin_bit_cast(bf16x8, q), to, 0, 0, 0);
    else {
      f32x16 y = to;
      const uint32_t ka[4] = {kf[x][c].x, kf[x][c].y, kf[x][c].z, kf[x][c].w}, qa[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) y = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(ka[e]), __uint_as_float(qa[e]), y, 0, 0, 0);
      next[x] = y;
    }
  };
  auto count = [&](const f32x16 (&s)[NB], int e, const Column& y) {         // score number e of the lane's NB * 16
    const int x = e / 16, i = e % 16;
    sum[x][i] += fast_exp2(fmaf(s[x][i], scale, -y.norm));
  };
  // what comes before the exponentials where not all is seen, or scores are changed
  auto prepare = [&](f32x16 (&s)[NB], Column& y) {
    if constexpr (MOD) {
      auto each_score = [&](auto f) {
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[x][i] = f(s[x][i], kpos[x][i]);
      };
      if (EB == 2 && A.mods.wide) each_score([&](float z, float) { return capped_wide(z, A.mods); });
      else if (A.mods.cap_out != 0.0f) each_score([&](float z, float) { return capped<EB>(z, A.mods); });
      else each_score([&](float z, float) { return z * A.mods.scale_log2; });
      if (A.mods.slopes) each_score([&](float z, float p) { return fmaf(-y.slope, fabsf(y.pos - p), z); });
    }
    const int last = mine + NB * 32;
    if ((MOD && doc) || __ballot(y.limit < last) != 0) {
      const float spoils = y.norm != y.norm ? y.norm : 0.0f;                 // a row whose normaliser is NaN gives that to the slots it sees, and to no others
      y.norm = y.norm != y.norm ? 0.0f : y.norm;
#pragma unroll
      for (int x = 0; x < NB; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          bool seen = mine + x * 32 + (i / 4) * 8 + half * 4 + i % 4 < y.limit;
          if constexpr (MOD)
            if (doc) seen &= kdoc[x][i] == y.doc;
          s[x][i] = seen ? s[x][i] + spoils : -INFINITY;
        }
    }
  };
  // the products of block u of step t beside the exponentials of the block before (LAST: there is one)
  auto block = [&](f32x16 (&next)[NB], int t, int u, auto last, f32x16 (&s)[NB], Column& y) {
    constexpr bool kLast = decltype(last)::value;
    if constexpr (kLast) prepare(s, y);
    const lchar* const qrow = lds + (t & 1) * M::kTile + (u * 32 + col) * RB;
    const int sw = L::swz_k(col);
    uint4 q[KC];
    auto fetch = [&](auto at) {
      constexpr int c = decltype(at)::value;
      if constexpr (c < KC) q[c] = lds16(qrow + (((2 * c + half) ^ sw) << 4));
    };
    each<2>(fetch);
    each<KC>([&](auto at) {
      constexpr int c = decltype(at)::value;
      fetch(std::integral_constant<int, c + 2>());
#pragma unroll
      for (int x = 0; x < NB; ++x) product(next, x, c, q[c]);
      if constexpr (kLast) {
        constexpr int e0 = NB * 16 * c / KC, e1 = NB * 16 * (c + 1) / KC;
        each<e1 - e0>([&](auto o) { count(s, e0 + decltype(o)::value, y); });
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  load(0);
  store(0);
  Column y0 = column(0, 0), y1;
  if (steps > 1) load(1);
  __syncthreads();
  block(s0, 0, 0, std::false_type(), s1, y0);
  for (int t = 0; t < steps; ++t) {
    y1 = column(t, 1);
    block(s1, t, 1, std::true_type(), s0, y0);
    if (t + 1 < steps) {
      store(t + 1);                                  // (the buffer's rows were read before the barrier below, a step ago)
      y0 = column(t + 1, 0);
      if (t + 2 < steps) load(t + 2);
      __syncthreads();
      block(s0, t + 1, 0, std::true_type(), s1, y1);
    }
  }
  prepare(s1, y1);
#pragma unroll
  for (int e = 0; e < NB * 16; ++e) count(s1, e, y1);
  // the 32 lanes of a half meet
  gfloat* const score = (gfloat*)sq.score + (size_t)head * A.cap;
#pragma unroll
  for (int x = 0; x < NB; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float v = row_sum<16>(sum[x][i]);
      v = xor_sum<16>(v);
      const int slot = mine + x * 32 + (i / 4) * 8 + half * 4 + i % 4;
      if (col == i && slot < n) score[slot] = score[slot] + v;
    }
}

// ---------------------------------------------------------------------------------------------------- shared prompts
struct SharedArgs {
  adsa_seq* seqs;
  const adsa_seq* prompts;
  const int32_t* members;
  const char* q;
  const char* k_new;
  const char* v_new;
  const int32_t* sel_idx;
  const int32_t* sel_cnt;
  char* out;
  float* lse;
  float* logits;
  float* part_ml;
  float* part_acc;
  Mods mods;
  long long slot_stride_b, head_stride_b, prompt_slot_stride_b, prompt_head_stride_b;
  int n_seq, n_groups, h, G, cap, sel_cap, lg_stride, max_prompt, max_members;
  int prompt_tiles, prompt_chunks, own_chunks, prompt_blocks;
  int accumulate, append, advance, new_f32;
};

// A group's members and its prompt's slots; n < 0: not what they should be.
struct Group {
  int first, end, n;
};
__device__ __forceinline__ Group group_at(const SharedArgs& A, int g) {
  Group gr;
  gr.first = ((const gint*)A.members)[g];
  gr.end = ((const gint*)A.members)[g + 1];
  const ADSA_GLOBAL adsa_seq& pr = ((const ADSA_GLOBAL adsa_seq*)A.prompts)[g];
  gr.n = pr.n_res;
  if (pr.status != 0 || gr.n < 0 || gr.n > A.max_prompt || gr.first < 0 || gr.end > A.n_seq || gr.end < gr.first || gr.end - gr.first > A.max_members) gr.n = -1;
  return gr;
}

// One query head over a part of its sequence's own list: nothing is shared, so there is no matrix product; bound by the rows' way from HBM.
// 16 bytes of a row per lane, 64 / (row bytes / 16) tokens ("a unit") per load of a wave; kRing units of K and V are on their way at any time, and
// a unit's registers are refilled as soon as it is folded into its lanes' softmax states.  Entries that are not attended read the query's
// row instead (whatever the cache holds there must not reach the sums, not even times 0).  32 x 24 heads x 553 tokens x 64, with prompts of 120: 20.4-22 us for 114 MB.
template <int EB, int D, int NW, bool MOD>
__device__ __forceinline__ void own_list(const Mods& mods, const Keys& keys, const gchar* q_row, float slope, int q_pos, gfloat* part_ml, gfloat* part_acc, lchar* lds) {
  constexpr int EPL = Elems<EB>::N, LPR = D / EPL, RPW = kWave / LPR, kRing = 8;
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), dl = lane % LPR, ts = lane / LPR;
  const gchar* const mine = q_row + dl * 16;
  const Elems<EB> q(load16(mine), MOD ? 1.0f : mods.scale_log2);
  const int units = (keys.end - keys.begin + RPW - 1) / RPW, n = units > wave ? (units - wave + NW - 1) / NW : 0;      // of this wave
  const int first = keys.begin + wave * RPW + ts;      // the lane's entry in the wave's first unit
  uint4 kr[kRing], vr[kRing];
  int ent[kRing], next[kRing], pos[kRing];
  auto entry = [&](int i) { return keys.list[min(first + i * NW * RPW, keys.end - 1)]; };
  auto load = [&](int u, int i) {
    const int slot = min(max(next[u], 0), keys.last_slot);
    const bool on = first + i * NW * RPW < keys.end && next[u] != keys.skip;
    ent[u] = on ? slot : -1;
    const long long off = (long long)slot * keys.stride_b + dl * 16;
    kr[u] = load_stream16(on ? keys.k + off : mine);
    vr[u] = load_stream16(on ? keys.v + off : mine);
    if (MOD && mods.slopes) pos[u] = keys.pos[slot];
  };
#pragma unroll
  for (int u = 0; u < kRing; ++u) next[u] = entry(u);
#pragma unroll
  for (int u = 0; u < kRing; ++u) {
    load(u, u);
    next[u] = entry(u + kRing);
  }
  float m = kLowest, l = 0.0f, acc[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) acc[e] = 0.0f;
  for (int i0 = 0; i0 < n; i0 += kRing)
#pragma unroll
    for (int u = 0; u < kRing; ++u) {
      if (i0 + u >= n) break;                        // (uniform)
      float z = row_sum<LPR>(q.dot(kr[u]));
      if constexpr (MOD) {
        z = mods.cap_out != 0.0f ? capped_any<EB>(z, mods) : z * mods.scale_log2;
        if (mods.slopes) z = fmaf(-slope, fabsf((float)(q_pos - pos[u])), z);
      } else z = Elems<EB>::scaled(z, mods.scale_log2);
      z = ent[u] >= 0 ? z : -INFINITY;
      const int j = first + (i0 + u) * NW * RPW;
      if (keys.logits && dl == 0 && j < keys.end) keys.logits[j] = z;
      const float m_new = fmaxf(m, z), corr = fast_exp2(m - m_new), p = fast_exp2(z - m_new);
      m = m_new;
      l = fmaf(l, corr, p);
      float v[EPL];
      Elems<EB>::unpack(vr[u], v);
#pragma unroll
      for (int e = 0; e < EPL; ++e) acc[e] = fmaf(acc[e], corr, p * v[e]);
      load(u, i0 + u + kRing);
      next[u] = entry(i0 + u + 2 * kRing);
    }
  // the wave's groups of lanes, then its waves
  float M = m;
#pragma unroll
  for (int x = LPR; x < kWave; x <<= 1) M = x == 8 ? xor_max<8>(M) : x == 16 ? xor_max<16>(M) : xor_max<32>(M);
  const float w = fast_exp2(m - M);
  l *= w;
#pragma unroll
  for (int x = LPR; x < kWave; x <<= 1) l = x == 8 ? xor_sum<8>(l) : x == 16 ? xor_sum<16>(l) : xor_sum<32>(l);
  ADSA_LDS float* const s_acc = (ADSA_LDS float*)lds;
  ADSA_LDS float* const s_ml = s_acc + NW * D;
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    float x = acc[e] * w;
#pragma unroll
    for (int y = LPR; y < kWave; y <<= 1) x = y == 8 ? xor_sum<8>(x) : y == 16 ? xor_sum<16>(x) : xor_sum<32>(x);
    if (ts == 0) s_acc[wave * D + dl * EPL + e] = x;
  }
  if (lane == 0) { s_ml[wave] = M; s_ml[NW + wave] = l; }
  __syncthreads();
  if (tid < D) {
    float top = kLowest, sum = 0.0f, x = 0.0f;
#pragma unroll
    for (int k = 0; k < NW; ++k) top = fmaxf(top, s_ml[k]);
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      const float f = fast_exp2(s_ml[k] - top);
      sum = fmaf(s_ml[NW + k], f, sum);
      x = fmaf(s_acc[k * D + tid], f, x);
    }
    part_acc[tid] = x;
    if (tid == 0) { part_ml[0] = top; part_ml[1] = sum; }
  }
}

template <int D, int W, int MODS> using SharedFlow = Flow<D, W, MODS, true, false>;
// Tiles of prompts come first, since they take longest.  64 sequences x 64 heads over 8 x 128, lists of 200..577, four prompts of 2100..4352: 51 us for 159 MB (37 and 28 alone).
// BIG: prompts are met by 128 rows at a time (bf16; groups of more than 32 rows), else by 32 rows and as many waves that split the keys.
// MODS: what is done to scores, as a Flow has it (a Tile tells plain from anything else).
// Three waves a SIMD where 64 elements of 32 rows leave registers for them (64 x 18 heads over 9 x 64, lists of 553: two | three 38.6 | 32.9 us).
template <int EB, int D, int WK, int MODS, bool ONE, bool BIG>
__global__ __launch_bounds__(WK * kWave, (EB == 2 && D == 64 && !BIG ? 3 : kWavesPerSimd<EB, D>)) void k_shared(SharedArgs A) {
  constexpr bool MOD = MODS != kPlain;
  extern __shared__ __align__(16) char s_lds[];
  const int hq = A.h * A.G, C = A.prompt_chunks + A.own_chunks;
  Keys keys;
  keys.doc = nullptr;
  keys.logits = nullptr;
  keys.skip = -1;
  keys.pos0 = 0;
  auto store = [&](auto& t, size_t at, int part) {
    gfloat* const acc = (gfloat*)A.part_acc + (at * C + part) * D;
    using T = std::decay_t<decltype(t)>;
#pragma unroll
    for (int i = 0; i < T::kMine; i += 4)
      store4<4>((gchar*)(acc + t.element(i)), t.acc[i / 16][i % 16], t.acc[i / 16][i % 16 + 1], t.acc[i / 16][i % 16 + 2], t.acc[i / 16][i % 16 + 3]);
    if (t.half == 0 && t.wk == 0) {
      gfloat* const ml = (gfloat*)A.part_ml + (at * C + part) * 2;
      ml[0] = t.m;
      ml[1] = t.l;
    }
  };
  auto nothing = [&](size_t at, int part) {          // (joined with weight 0, its outputs not read)
    gfloat* const ml = (gfloat*)A.part_ml + (at * C + part) * 2;
    ml[0] = kLowest;
    ml[1] = 0.0f;
  };
  auto query_pos = [&](int b) {
    const ADSA_GLOBAL adsa_seq& sq = ((const ADSA_GLOBAL adsa_seq*)A.seqs)[b];
    return sq.grid_origin + sq.step - 1;
  };
  if ((int)blockIdx.x < A.prompt_blocks) {           // a tile of a group's rows over a part of its prompt
    int unit, tile;
    pair_of(blockIdx.x, (unsigned)A.prompt_tiles, &unit, &tile);
    if (unit >= A.n_groups * A.h * A.prompt_chunks) return;
    const int chunk = unit % A.prompt_chunks, head = unit / A.prompt_chunks % A.h, g = unit / A.prompt_chunks / A.h;
    const Group gr = group_at(A, g);
    const int rows = (gr.end - gr.first) * A.G;
    constexpr int kRows = BIG ? 128 : 32;
    if (gr.n < 0 || tile * kRows >= rows) return;
    const ADSA_GLOBAL adsa_seq& pr = ((const ADSA_GLOBAL adsa_seq*)A.prompts)[g];
    keys.k = (const gchar*)pr.k + head * A.prompt_head_stride_b;
    keys.v = (const gchar*)pr.v + head * A.prompt_head_stride_b;
    keys.stride_b = A.prompt_slot_stride_b;
    keys.list = nullptr;
    keys.pos = scalar((const gint*)pr.pos);
    const int per = ((gr.n + A.prompt_chunks - 1) / A.prompt_chunks + 31) / 32 * 32;
    keys.begin = min(gr.n, chunk * per);
    keys.end = min(gr.n, keys.begin + per);
    auto attend = [&](auto& t, int r) {
      const int rr = min(r, rows - 1), b = gr.first + rr / A.G, qh = head * A.G + rr % A.G;
      const size_t at = (size_t)b * hq + qh;
      t.row = {keys.end, MOD && A.mods.slopes ? query_pos(b) - keys.pos0 : 0, 0, MOD && A.mods.slopes ? ((const gfloat*)A.mods.slopes)[qh] * kLog2e : 0.0f};
      t.load_q((const gchar*)A.q + at * (D * EB));
      if constexpr (BIG) t.run(keys.end);
      else t.run();
      if (r < rows) store(t, at, chunk);
    };
    if (keys.begin >= keys.end) {
      for (int r = tile * kRows + threadIdx.x; r < min(rows, (tile + 1) * kRows); r += WK * kWave) nothing((size_t)(gr.first + r / A.G) * hq + head * A.G + r % A.G, chunk);
      return;
    }
    if (MOD && A.mods.slopes) keys.pos0 = keys.pos[keys.begin];
    if constexpr (BIG) {
      SharedFlow<D, WK, MODS> t(A.mods, keys, (lchar*)s_lds);
      attend(t, tile * kRows + t.wave * 32 + t.col);
    } else {
      Tile<EB, D, WK, MOD, false, true> t(A.mods, keys, (lchar*)s_lds);
      attend(t, tile * kRows + t.col);
    }
    return;
  }
  // one sequence's own list
  const int id = (int)blockIdx.x - A.prompt_blocks, chunk = id % A.own_chunks, head = id / A.own_chunks % A.h, b = id / A.own_chunks / A.h;
  const ADSA_GLOBAL adsa_seq& sq = ((const ADSA_GLOBAL adsa_seq*)A.seqs)[b];
  if (sq.status != 0 || sq.step < 0) return;
  const int cnt = min(max(((const gint*)A.sel_cnt)[b], 0), A.sel_cap);
  keys.k = (const gchar*)sq.k + head * A.head_stride_b;
  keys.v = (const gchar*)sq.v + head * A.head_stride_b;
  keys.stride_b = A.slot_stride_b;
  keys.list = (const gint*)A.sel_idx + (size_t)b * A.sel_cap;
  keys.pos = scalar((const gint*)sq.pos);
  keys.last_slot = A.cap - 1;
  const int pending = A.append ? sq.pending_slot : -1;
  keys.skip = pending >= 0 && pending < A.cap ? pending : -1;
  const int per = ((cnt + A.own_chunks - 1) / A.own_chunks + 31) / 32 * 32;
  keys.begin = min(cnt, chunk * per);
  keys.end = min(cnt, keys.begin + per);
  const size_t at0 = (size_t)b * hq + head * A.G;
  keys.logits = A.accumulate ? (gfloat*)A.logits + at0 * A.lg_stride : nullptr;
  if constexpr (ONE) {
    if (keys.begin >= keys.end) {
      if (threadIdx.x == 0) nothing(at0, A.prompt_chunks + chunk);
      return;
    }
    const size_t part = at0 * C + A.prompt_chunks + chunk;
    const bool far = MOD && A.mods.slopes;
    own_list<EB, D, WK, MOD>(A.mods, keys, (const gchar*)A.q + at0 * (D * EB), far ? ((const gfloat*)A.mods.slopes)[head] * kLog2e : 0.0f, far ? query_pos(b) : 0,
                             (gfloat*)A.part_ml + part * 2, (gfloat*)A.part_acc + part * D, (lchar*)s_lds);
    return;
  }
  keys.lg_stride = A.lg_stride;
  keys.lg_rows = A.G;
  Tile<EB, D, WK, MOD, true, true> t(A.mods, keys, (lchar*)s_lds);
  const size_t at = at0 + min(t.col, A.G - 1);
  // (a part that holds the query token alone has no other row to stand in for it)
  if (keys.begin >= keys.end || (keys.end - keys.begin == 1 && keys.list[keys.begin] == keys.skip)) {
    if ((int)threadIdx.x < A.G) nothing(at, A.prompt_chunks + chunk);
    return;
  }
  const int qh = head * A.G + min(t.col, A.G - 1);
  keys.pos0 = MOD && A.mods.slopes ? query_pos(b) : 0;
  t.row = {keys.end, 0, 0, MOD && A.mods.slopes ? ((const gfloat*)A.mods.slopes)[qh] * kLog2e : 0.0f};
  t.load_q((const gchar*)A.q + at * (D * EB));
  t.run();
  if (t.col < A.G) store(t, at, A.prompt_chunks + chunk);
}

// Joins the parts of a (sequence, cache head)'s rows with the query token, whose row enters the cache, and updates the scores.  Bound by the trips
// that depend on each other (record, parts, list and scores' logits; scores and the group's record), so everything leaves as soon as its address is known.
// 5.2 us for 768 rows of one head, 10 for 512 x 8 heads with their scores, 7 without.
constexpr int kMaxParts = 2 * kMaxChunks;
template <int EB, int D, bool ONE>
__global__ __launch_bounds__(256) void k_shared_finish(SharedArgs A) {
  constexpr int NT = 256, E = D / kWave, kMaxG = ONE ? 1 : 16, kEarly = 3, kAcc = 4, kLg = ONE ? 1 : 8, kQ = ONE ? 1 : 2;
  __shared__ float s_w[kMaxG][kMaxParts + 1], s_l[kMaxG][kMaxParts], s_lse[kMaxG], s_new[kMaxG], s_inv[kMaxG];
  __shared__ __attribute__((aligned(16))) float s_v[D];
  __shared__ int s_has;
  const int b = blockIdx.x / A.h, head = blockIdx.x % A.h, tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int G = ONE ? 1 : A.G, hq = A.h * G, C = A.prompt_chunks + A.own_chunks;
  const size_t at0 = (size_t)b * hq + head * G, row = ((size_t)b * A.h + head) * D;
  ADSA_GLOBAL adsa_seq& sq = ((ADSA_GLOBAL adsa_seq*)A.seqs)[b];
  const gint* const list = (const gint*)A.sel_idx + (size_t)b * A.sel_cap;
  // ---- what depends on the arguments only
  const int status = sq.status, step = sq.step, pending = sq.pending_slot;
  gfloat* const score = (gfloat*)sq.score + (size_t)head * A.cap;
  int cnt = ((const gint*)A.sel_cnt)[b], g = -1;
  for (int i = 0; i < A.n_groups; i += kWave)          // the sequence's group: the last that begins at or before it
    g += __popcll(__ballot(i + lane < A.n_groups && ((const gint*)A.members)[min(i + lane, A.n_groups - 1)] <= b));
  int slot[kEarly];
  float old[kEarly], lg[kEarly][kLg];
#pragma unroll
  for (int k = 0; k < kEarly; ++k) {
    slot[k] = list[min(tid + k * NT, A.sel_cap - 1)];
    if (A.accumulate) {
#pragma unroll
      for (int h = 0; h < kLg; ++h) lg[k][h] = ((const gfloat*)A.logits)[(at0 + min(h, G - 1)) * A.lg_stride + min(tid + k * NT, A.sel_cap - 1)];
    }
  }
  for (int o = tid; o < G * C; o += NT) {
    const gfloat* const ml = (const gfloat*)A.part_ml + (at0 * C + o) * 2;
    s_w[o / C][o % C] = ml[0];
    s_l[o / C][o % C] = ml[1];
  }
  // the parts' outputs: 4 elements of a query head per thread, the first parts at once
  const int items = G * (D / 4), oh = tid / (D / 4), oe = tid % (D / 4) * 4;
  auto part_of = [&](int h, int c) { return *(const ADSA_GLOBAL u32x4*)((const gfloat*)A.part_acc + ((at0 + h) * C + c) * D + oe); };
  u32x4 parts[kAcc];
  if (tid < items) {
#pragma unroll
    for (int c = 0; c < kAcc; ++c) parts[c] = part_of(oh, min(c, C - 1));
  }
  float kn[E], vn[E], qn[kQ][E];
  auto q_of = [&](int h, int e) {
    const size_t o = (at0 + h) * D + e * kWave + lane;
    return EB == 4 ? ((const gfloat*)A.q)[o] : __uint_as_float((uint32_t)((const ADSA_GLOBAL uint16_t*)A.q)[o] << 16);
  };
  if (A.append) {
#pragma unroll
    for (int k = 0; k < kQ; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) qn[k][e] = q_of(min(wave + k * (NT / kWave), G - 1), e);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const size_t o = row + e * kWave + lane;
      if (EB == 4 || A.new_f32) {
        kn[e] = ((const gfloat*)A.k_new)[o];
        vn[e] = ((const gfloat*)A.v_new)[o];
        if constexpr (EB == 2) {
          kn[e] = __uint_as_float(f32_to_bf16_rne(kn[e]) << 16);
          vn[e] = __uint_as_float(f32_to_bf16_rne(vn[e]) << 16);
        }
      } else {
        kn[e] = __uint_as_float((uint32_t)((const ADSA_GLOBAL uint16_t*)A.k_new)[o] << 16);
        vn[e] = __uint_as_float((uint32_t)((const ADSA_GLOBAL uint16_t*)A.v_new)[o] << 16);
      }
    }
  }
  // ---- what depends on that: scores so far, the group's record
  const bool live = status == 0 && step >= 0;
  cnt = min(max(cnt, 0), A.sel_cap);
#pragma unroll
  for (int k = 0; k < kEarly; ++k) {
    old[k] = 0.0f;
    if (A.accumulate && live && tid + k * NT < cnt) old[k] = score[min(max(slot[k], 0), A.cap - 1)];
  }
  const Group gr = group_at(A, max(g, 0));
  const bool fits = gr.n >= 0 && gr.first <= b && b < gr.end;
  if (!live || !fits) {
    if (live && head == 0 && tid == 0) sq.status = ADSA_SEQ_BAD_STATE;
    for (int o = tid; o < G * D * EB / 4; o += NT) ((gint*)(A.out + at0 * D * EB))[o] = 0;
    for (int o = tid; o < G; o += NT) ((gfloat*)A.lse)[at0 + o] = 0.0f;
    return;
  }
  const int new_slot = A.append && pending >= 0 && pending < A.cap ? pending : -1;
  bool mine = false;
#pragma unroll
  for (int k = 0; k < kEarly; ++k) mine |= tid + k * NT < cnt && slot[k] == new_slot;
  for (int j = tid + kEarly * NT; j < cnt; j += NT) mine |= list[j] == new_slot;
  if (tid == 0) s_has = 0;
  __syncthreads();
  if (new_slot >= 0) {
    if (mine) s_has = 1;
    if (wave == 0) {                                 // the query token's row enters the cache
      gchar* const kc = (gchar*)sq.k + head * A.head_stride_b + new_slot * A.slot_stride_b;
      gchar* const vc = (gchar*)sq.v + head * A.head_stride_b + new_slot * A.slot_stride_b;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if constexpr (EB == 4) { ((gfloat*)kc)[e * kWave + lane] = kn[e]; ((gfloat*)vc)[e * kWave + lane] = vn[e]; }
        else {
          ((ADSA_GLOBAL uint16_t*)kc)[e * kWave + lane] = (uint16_t)(__float_as_uint(kn[e]) >> 16);
          ((ADSA_GLOBAL uint16_t*)vc)[e * kWave + lane] = (uint16_t)(__float_as_uint(vn[e]) >> 16);
        }
        s_v[e * kWave + lane] = vn[e];
      }
    }
    auto meet = [&](int h, auto q) {                 // its score with a query head
      float z = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) z = fmaf(q(e), kn[e], z);
      z = row_sum<32>(z);
      z = xor_sum<32>(z);
      z = A.mods.cap_out != 0.0f ? capped_any<EB>(z, A.mods) : z * A.mods.scale_log2;      // (its distance to itself is 0)
      if (lane == 0) s_new[h] = z;
    };
#pragma unroll
    for (int k = 0; k < kQ; ++k)
      if (wave + k * (NT / kWave) < G) meet(wave + k * (NT / kWave), [&](int e) { return qn[k][e]; });
    for (int h = wave + kQ * (NT / kWave); h < G; h += NT / kWave) meet(h, [&](int e) { return q_of(h, e); });
  }
  __syncthreads();
  const bool has = new_slot >= 0 && s_has != 0;
  if (tid < G) {
    float M = has ? s_new[tid] : kLowest;
    for (int c = 0; c < C; ++c) M = fmaxf(M, s_w[tid][c]);
    const float pn = has ? fast_exp2(s_new[tid] - M) : 0.0f;
    float sum = pn;
    for (int c = 0; c < C; ++c) {
      const float w = s_l[tid][c] == 0.0f ? 0.0f : fast_exp2(s_w[tid][c] - M);
      s_w[tid][c] = w;
      sum = fmaf(s_l[tid][c], w, sum);
    }
    s_w[tid][C] = pn;
    s_inv[tid] = sum == 0.0f ? 0.0f : 1.0f / sum;
    s_lse[tid] = sum == 0.0f ? INFINITY : M + __log2f(sum);            // (no finite score: no slot gains anything)
    ((gfloat*)A.lse)[at0 + tid] = sum == 0.0f ? -INFINITY : s_lse[tid] * kLn2;
  }
  __syncthreads();
  for (int o = tid; o < items; o += NT) {
    const int h = o / (D / 4);                       // (NT is a multiple of D / 4: the same elements in every round)
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = has ? s_w[h][C] * s_v[oe + e] : 0.0f;
    auto add = [&](int c, const u32x4& part) {
      const float w = s_w[h][c];
      const bool there = s_l[h][c] != 0.0f;          // (else nothing was stored)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = there ? fmaf(__uint_as_float(part[e]), w, x[e]) : x[e];
    };
#pragma unroll
    for (int c = 0; c < kAcc; ++c)
      if (c < C) add(c, o == tid ? parts[c] : part_of(h, c));
    for (int c = kAcc; c < C; ++c) add(c, part_of(h, c));
    store4<EB>((gchar*)A.out + ((at0 + h) * D + oe) * EB, x[0] * s_inv[h], x[1] * s_inv[h], x[2] * s_inv[h], x[3] * s_inv[h]);
  }
  if (A.accumulate) {
    auto logit = [&](int j, int h) { return ((const gfloat*)A.logits)[(at0 + h) * A.lg_stride + j]; };
    auto chance = [&](int raw, int h, float z) { return fast_exp2((raw == new_slot && new_slot >= 0 ? s_new[h] : z) - s_lse[h]); };
    auto slot_of = [&](int raw) { return min(max(raw, 0), A.cap - 1); };
#pragma unroll
    for (int k = 0; k < kEarly; ++k)
      if (tid + k * NT < cnt) {
        float gain = 0.0f;
#pragma unroll
        for (int h = 0; h < kLg; ++h)
          if (h < G) gain += chance(slot[k], h, lg[k][h]);
        for (int h = kLg; h < G; ++h) gain += chance(slot[k], h, logit(tid + k * NT, h));
        score[slot_of(slot[k])] = old[k] + gain;
      }
    for (int j = tid + kEarly * NT; j < cnt; j += NT) {
      const int raw = list[j];
      const float before = score[slot_of(raw)];
      float gain = 0.0f;
      for (int h = 0; h < G; ++h) gain += chance(raw, h, logit(j, h));
      score[slot_of(raw)] = before + gain;
    }
  }
  if (A.advance && head == 0 && tid == 0) sq.step = step + 1;
}

Mods make_mods(const adsa_params& p, const adsa_mods& m) {
  const float scale = p.softmax_scale > 0.0f ? p.softmax_scale : 1.0f / sqrtf((float)p.head_dim);
  Mods o;
  o.slopes = m.slopes;
  o.doc = m.doc;
  o.doc_stride = m.doc_stride;
  o.cap_in = m.softcap > 0.0f ? scale / m.softcap : 0.0f;
  o.cap_out = m.softcap > 0.0f ? m.softcap * kLog2e : 0.0f;
  o.wide = p.dtype == ADSA_BF16 && m.softcap > kWideCap;
  o.scale_log2 = scale * kLog2e;
  return o;
}
bool modded(const Mods& m) { return m.slopes || m.doc || m.cap_out != 0.0f; }

// Waves that split the keys of 32 rows.
template <int EB, int D> constexpr int kKeyWaves = EB == 4 && D == 128 ? 2 : 4;


// Rows of a k_prompt_many workgroup: 4 waves' 32 each.  us with 4 | 8 waves: 4 x 4352 x 32 x 128 with its mass 1127 | 1102, lowered with distance 2 x 4352 x 32 x 128 495 | 470,
// by documents 135 | 144, capped ragged prompts of 64 over 8 heads 226 | 242, 16 x 300..600 x 24 x 64 lowered with distance 59 | 76.
constexpr int kRowWaves = 4;

template <int EB, int D, bool MOD>
hipError_t prompt_launches(const PromptArgs& A, const PromptPlan& plan, bool split, hipStream_t st) {
  const unsigned pairs = (unsigned)((A.n_seq * A.h + 7) / 8 * 8);
  constexpr int KW = kKeyWaves<EB, D>;
  const dim3 grid(pairs * (unsigned)(plan.tiles * plan.chunks));
  if (!plan.flow) k_prompt<EB, D, KW, MOD><<<grid, KW * kWave, Shape<EB, D, KW>::kLds, st>>>(A);
  else {
    if constexpr (EB == 2) {
      auto launch = [&](auto mods, auto two) {
        constexpr int M = decltype(mods)::value;
        constexpr bool kSplit = decltype(two)::value;
        k_prompt_many<D, kRowWaves, M, kSplit><<<grid, kRowWaves * kWave, PromptFlow<D, kRowWaves, M, kSplit>::kLds, st>>>(A);
      };
      auto many = [&](auto mods) { split ? launch(mods, std::true_type()) : launch(mods, std::false_type()); };
      if constexpr (!MOD) many(std::integral_constant<int, kPlain>());
      else if (A.mods.slopes || A.mods.doc || A.mods.wide) {
        if (A.mods.cap_out != 0.0f) many(std::integral_constant<int, kAnyCapped>());
        else many(std::integral_constant<int, kAny>());
      } else many(std::integral_constant<int, kCapped>());
    }
  }
  if (plan.chunks > 1) {
    const size_t rows = (size_t)A.n_tokens * A.h * A.G;
    k_prompt_finish<EB, D><<<dim3((unsigned)((rows + 3) / 4)), 256, 0, st>>>(A);
  }
  if (A.norm) {
    const int key_tiles = (A.cap + Mass<EB, D, MOD>::kKeys - 1) / Mass<EB, D, MOD>::kKeys;
    k_prompt_mass<EB, D, MOD><<<dim3(pairs * (unsigned)key_tiles), 256, Mass<EB, D, MOD>::kLds, st>>>(A, key_tiles);
  }
  return hipGetLastError();
}

template <int EB, int D, int MODS, bool BIG>
constexpr int shared_lds = [] {
  const int own = Shape<EB, D, kKeyWaves<EB, D>>::kLds;
  if constexpr (BIG) return std::max(own, SharedFlow<D, 4, MODS>::kLds);
  else return own;
}();

template <int EB, int D, bool MOD>
hipError_t shared_launches(const SharedArgs& A, const SharedPlan& plan, hipStream_t st) {
  constexpr int KW = kKeyWaves<EB, D>;
  const dim3 grid((unsigned)(A.prompt_blocks + A.n_seq * A.h * A.own_chunks));
  auto launch = [&](auto mods, auto big) {
    constexpr int M = decltype(mods)::value;
    constexpr bool kBig = decltype(big)::value;
    if (A.G == 1) k_shared<EB, D, KW, M, true, kBig><<<grid, KW * kWave, shared_lds<EB, D, M, kBig>, st>>>(A);
    else k_shared<EB, D, KW, M, false, kBig><<<grid, KW * kWave, shared_lds<EB, D, M, kBig>, st>>>(A);
  };
  using std::integral_constant;
  constexpr int kAll = MOD ? kAnyCapped : kPlain;
  bool done = false;
  if constexpr (EB == 2)
    if (plan.big) {
      done = true;
      if (MOD && !A.mods.slopes && !A.mods.wide) launch(integral_constant<int, MOD ? kCapped : kPlain>(), std::true_type());
      else if (MOD && A.mods.cap_out == 0.0f) launch(integral_constant<int, MOD ? kAny : kPlain>(), std::true_type());
      else launch(integral_constant<int, kAll>(), std::true_type());
    }
  if (!done) launch(integral_constant<int, kAll>(), std::false_type());
  if (A.G == 1) k_shared_finish<EB, D, true><<<dim3((unsigned)(A.n_seq * A.h)), 256, 0, st>>>(A);
  else k_shared_finish<EB, D, false><<<dim3((unsigned)(A.n_seq * A.h)), 256, 0, st>>>(A);
  return hipGetLastError();
}

template <int EB, int D, bool MOD>
hipError_t allow_lds() {
  constexpr int KW = kKeyWaves<EB, D>;
  hipError_t e = hipSuccess;
  auto allow = [&](auto kernel, int bytes) {
    if (e == hipSuccess) e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  allow(k_prompt<EB, D, KW, MOD>, Shape<EB, D, KW>::kLds);
  allow(k_prompt_mass<EB, D, MOD>, Mass<EB, D, MOD>::kLds);
  auto shared = [&](auto mods, auto big) {
    constexpr int M = decltype(mods)::value;
    constexpr bool kBig = decltype(big)::value;
    allow(k_shared<EB, D, KW, M, true, kBig>, shared_lds<EB, D, M, kBig>);
    allow(k_shared<EB, D, KW, M, false, kBig>, shared_lds<EB, D, M, kBig>);
  };
  using std::integral_constant;
  shared(integral_constant<int, MOD ? kAnyCapped : kPlain>(), std::false_type());
  if constexpr (EB == 2) {
    auto many = [&](auto mods) {
      constexpr int M = decltype(mods)::value;
      allow(k_prompt_many<D, kRowWaves, M, false>, PromptFlow<D, kRowWaves, M, false>::kLds);
      allow(k_prompt_many<D, kRowWaves, M, true>, PromptFlow<D, kRowWaves, M, true>::kLds);
    };
    auto both = [&](auto mods) { many(mods); shared(mods, std::true_type()); };
    if constexpr (!MOD) both(integral_constant<int, kPlain>());
    else {
      both(integral_constant<int, kCapped>());
      both(integral_constant<int, kAny>());
      both(integral_constant<int, kAnyCapped>());
    }
  }
  return e;
}

template <typename F>
hipError_t by_type(const adsa_params& p, bool mod, F f) {
  const bool f32 = p.dtype == ADSA_F32, wide = p.head_dim == 128;
  using std::integral_constant;
  auto with = [&](auto eb, auto d) { return mod ? f(eb, d, std::true_type()) : f(eb, d, std::false_type()); };
  if (f32) return wide ? with(integral_constant<int, 4>(), integral_constant<int, 128>()) : with(integral_constant<int, 4>(), integral_constant<int, 64>());
  return wide ? with(integral_constant<int, 2>(), integral_constant<int, 128>()) : with(integral_constant<int, 2>(), integral_constant<int, 64>());
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
int query_group(const adsa_params& p) { return p.q_per_kv > 1 ? p.q_per_kv : 1; }

}  // namespace

hipError_t prompt_prepare_kernels() {
  for (int dtype : {ADSA_F32, ADSA_BF16})
    for (int d : {64, 128})
      for (bool mod : {false, true}) {
        adsa_params p = {};
        p.dtype = dtype;
        p.head_dim = d;
        const hipError_t e = by_type(p, mod, [](auto eb, auto hd, auto m) { return allow_lds<decltype(eb)::value, decltype(hd)::value, decltype(m)::value>(); });
        if (e != hipSuccess) return e;
      }
  return hipSuccess;
}

PromptPlan make_prompt_plan(const adsa_params& p, const adsa_tokens& t) {
  const long long rows = (long long)t.max_len * query_group(p), pairs = (long long)p.n_seq * p.n_heads;
  PromptPlan plan;
  auto groups = [&](int tile) { return pairs * ((rows + tile - 1) / tile); };
  const bool near = p.kv_slot_stride * 2 * 64 < (1ll << 31);       // (k_prompt_many reaches a tile's rows with 32-bit offsets from its first)
  // Tiles of 32 rows, whose 4 waves split the keys, or of 128, whose waves share them (bf16).  The host does not know how many keys there are, so the
  // capacity stands for them, and a short prompt in a long cache takes the long ones' form (1 x 400 x 24 x 64 in 512 | 600 slots 7.8 | 16).  us with 128 | 32 rows a tile:
  // short caches that leave CUs idle, 1 x 400 x 24 heads x 64 12.5 | 7.7, 4 x 120 7.9 | 6.2; 64 rows and less, of which 128 leave half empty, behind
  // 2000 slots 2 x 60 x 24 x 64 19.4 | 14.0, behind 700 slots 16 x 60 x 24 x 64 29 | 18.4.  Elsewhere K and V are read too often: 32 x 60 x 24 x 64
  // 10.6 | 13.4, 16 x 60 x 32 x 128 behind 700 47 | 52, 2 x 1000 x 32 x 128 41 | 110.
  const bool idle = groups(128) <= 256, half = rows <= 64 && (idle || (p.head_dim == 64 && p.cap > 512));
  plan.flow = p.dtype == ADSA_BF16 && near && rows > 32 && !half && !(idle && p.cap <= 512);
  plan.rows = plan.flow ? 128 : 32;
  plan.tiles = (int)((rows + plan.rows - 1) / plan.rows);
  // Keys are split where tiles alone leave CUs idle.  (Two parts where 256 tiles fill them: 16 x 1..9 x 24 x 64 behind 700 slots 15.4 -> 21.3 us.)
  const long long n = groups(plan.rows), most = plan.flow ? (p.cap + 511) / 512 : (p.cap + 255) / 256;
  plan.chunks = n > 256 ? 1 : (int)std::clamp<long long>(std::min<long long>((plan.flow ? 256 : 512) / n, most), 1, kMaxChunks);
  return plan;
}

PromptWorkspace make_prompt_workspace(const adsa_params& p, const adsa_tokens& t, const PromptPlan& plan) {
  const size_t rows = (size_t)t.n_tokens * p.n_heads * query_group(p);
  PromptWorkspace w;
  w.part_ml_off = 0;
  w.part_acc_off = w.part_ml_off + (plan.chunks > 1 ? up256(rows * plan.chunks * 8) : 0);
  w.norm_off = w.part_acc_off + (plan.chunks > 1 ? up256(rows * plan.chunks * p.head_dim * 4) : 0);
  w.total = w.norm_off + (p.score_mode == ADSA_SCORE_ATTN_MASS ? up256(rows * 4) : 0);
  w.total = std::max<size_t>(w.total, 256);
  return w;
}

SharedPlan make_shared_plan(const adsa_params& p, const adsa_shared& s) {
  SharedPlan plan;
  const int rows = s.max_members * query_group(p);
  plan.big = p.dtype == ADSA_BF16 && rows > 32 && s.kv_slot_stride * 2 * 64 < (1ll << 31);       // (see make_prompt_plan)
  plan.prompt_tiles = (rows + (plan.big ? 127 : 31)) / (plan.big ? 128 : 32);
  auto parts = [](long long groups, int longest) {
    return (int)std::clamp<long long>(std::min<long long>((512 + groups - 1) / groups, (longest + 127) / 128), 1, kMaxChunks);
  };
  plan.prompt_chunks = parts((long long)s.n_groups * p.n_heads * plan.prompt_tiles * 4, s.max_prompt);
  plan.own_chunks = parts((long long)p.n_seq * p.n_heads, p.sel_cap);
  return plan;
}

SharedWorkspace make_shared_workspace(const adsa_params& p, const SharedPlan& plan) {
  const size_t rows = (size_t)p.n_seq * p.n_heads * query_group(p), parts = (size_t)(plan.prompt_chunks + plan.own_chunks);
  SharedWorkspace w;
  w.lg_stride = (p.sel_cap + 3) / 4 * 4;
  w.logits_off = 0;
  w.part_ml_off = up256(rows * w.lg_stride * 4);
  w.part_acc_off = w.part_ml_off + up256(rows * parts * 8);
  w.total = w.part_acc_off + up256(rows * parts * p.head_dim * 4);
  return w;
}

hipError_t launch_prefill(const adsa_params& p, const adsa_tokens& t, const adsa_mods& mods, const PromptPlan& plan, adsa_seq* seqs, const void* q, void* out,
                          float* lse, char* ws, const PromptWorkspace& w, bool accumulate, bool advance, bool split, hipStream_t st) {
  PromptArgs A = {};
  A.seqs = seqs; A.begin = t.begin; A.slot0 = t.slot0; A.q = (const char*)q; A.out = (char*)out; A.lse = lse;
  A.part_ml = (float*)(ws + w.part_ml_off);
  A.part_acc = (float*)(ws + w.part_acc_off);
  A.norm = accumulate ? (float*)(ws + w.norm_off) : nullptr;
  A.mods = make_mods(p, mods);
  A.slot_stride_b = p.kv_slot_stride * elem_bytes(p);
  A.head_stride_b = p.kv_head_stride * elem_bytes(p);
  A.n_seq = p.n_seq; A.n_tokens = t.n_tokens; A.max_len = t.max_len; A.h = p.n_heads; A.G = query_group(p); A.cap = p.cap; A.mask = mods.mask;
  A.tiles = plan.tiles; A.chunks = plan.chunks; A.advance = advance ? 1 : 0;
  A.inv_G = A.G > 1 ? (uint32_t)(((1ull << 32) + A.G - 1) / A.G) : 0;
  return by_type(p, modded(A.mods), [&](auto eb, auto d, auto m) {
    return prompt_launches<decltype(eb)::value, decltype(d)::value, decltype(m)::value>(A, plan, split, st);
  });
}

hipError_t launch_attend_shared(const adsa_params& p, const adsa_shared& s, const adsa_mods& mods, const SharedPlan& plan, adsa_seq* seqs, const void* q,
                                const void* k_new, const void* v_new, const int32_t* sel_idx, const int32_t* sel_cnt, void* out, float* lse, char* ws,
                                const SharedWorkspace& w, bool accumulate, bool append, bool advance, bool new_f32, hipStream_t st) {
  SharedArgs A = {};
  A.seqs = seqs; A.prompts = s.prompts; A.members = s.members; A.q = (const char*)q; A.k_new = (const char*)k_new; A.v_new = (const char*)v_new;
  A.sel_idx = sel_idx; A.sel_cnt = sel_cnt; A.out = (char*)out; A.lse = lse;
  A.logits = (float*)(ws + w.logits_off);
  A.part_ml = (float*)(ws + w.part_ml_off);
  A.part_acc = (float*)(ws + w.part_acc_off);
  A.mods = make_mods(p, mods);
  A.mods.doc = nullptr;
  const int eb = elem_bytes(p);
  A.slot_stride_b = p.kv_slot_stride * eb; A.head_stride_b = p.kv_head_stride * eb;
  A.prompt_slot_stride_b = s.kv_slot_stride * eb; A.prompt_head_stride_b = s.kv_head_stride * eb;
  A.n_seq = p.n_seq; A.n_groups = s.n_groups; A.h = p.n_heads; A.G = query_group(p); A.cap = p.cap; A.sel_cap = p.sel_cap; A.lg_stride = w.lg_stride;
  A.max_prompt = s.max_prompt; A.max_members = s.max_members;
  A.prompt_tiles = plan.prompt_tiles; A.prompt_chunks = plan.prompt_chunks; A.own_chunks = plan.own_chunks;
  A.prompt_blocks = (s.n_groups * p.n_heads * plan.prompt_chunks + 7) / 8 * 8 * plan.prompt_tiles;
  A.accumulate = accumulate; A.append = append; A.advance = advance; A.new_f32 = new_f32;
  return by_type(p, modded(A.mods), [&](auto eb_, auto d, auto m) {
    return shared_launches<decltype(eb_)::value, decltype(d)::value, decltype(m)::value>(A, plan, st);
  });
}

}  // namespace adsa
