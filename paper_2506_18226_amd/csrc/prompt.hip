// The kernels of prompts over dense caches and of decode steps that share a prompt.  (What they are made of, and their figures, is in prompt_device.h.)
//
//  k_prompt, k_prompt_many, k_prompt_finish: a tile of (token, query head) rows of one (sequence, cache head) against the slots up to its last row's.
//  k_prompt_mass: the probability every slot received, a second pass over the scores with each row's normaliser known: a workgroup owns
//    its slots and takes the rows in order, so no atomics and one order of summation.
//  k_shared, k_shared_finish: tiles of a group's (member, query head) rows against parts of the group's prompt, and each sequence's own
//    list (the rows are then the query heads of a cache head), all as workgroups of one launch; the second kernel joins the parts.
#include "prompt_device.h"

namespace adsa {
namespace {

template <int EB, int D, int WK, bool MOD>
__global__ __launch_bounds__(WK * kWave, (kWavesPerSimd<EB, D>)) void k_prompt(PromptArgs A) { prompt_tile<EB, D, WK, MOD, false>(A); }
template <int D, int W, int MODS, bool SPLIT>
__global__ __launch_bounds__(W * kWave, (kFlowWaves<D, MODS, SPLIT>)) void k_prompt_many(PromptArgs A) { prompt_flow<D, W, MODS, SPLIT, false>(A); }
template <int EB, int D, bool MOD>
__global__ __launch_bounds__(256, EB == 2 ? 2 : 1) void k_prompt_mass(PromptArgs A, int key_tiles) { prompt_mass<EB, D, MOD, false>(A, key_tiles); }

struct DenseKernels {
  static constexpr bool kPaged = false;
  template <int EB, int D, int WK, bool MOD> static auto tile() { return k_prompt<EB, D, WK, MOD>; }
  template <int D, int W, int MODS, bool SPLIT> static auto flow() { return k_prompt_many<D, W, MODS, SPLIT>; }
  template <int EB, int D, bool MOD> static auto mass() { return k_prompt_mass<EB, D, MOD>; }
};

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
  allow_prompt_lds<DenseKernels, EB, D, MOD>(allow);
  auto shared = [&](auto mods, auto big) {
    constexpr int M = decltype(mods)::value;
    constexpr bool kBig = decltype(big)::value;
    allow(k_shared<EB, D, KW, M, true, kBig>, shared_lds<EB, D, M, kBig>);
    allow(k_shared<EB, D, KW, M, false, kBig>, shared_lds<EB, D, M, kBig>);
  };
  using std::integral_constant;
  shared(integral_constant<int, MOD ? kAnyCapped : kPlain>(), std::false_type());
  if constexpr (EB == 2) {
    auto big = [&](auto mods) { shared(mods, std::true_type()); };
    if constexpr (!MOD) big(integral_constant<int, kPlain>());
    else {
      big(integral_constant<int, kCapped>());
      big(integral_constant<int, kAny>());
      big(integral_constant<int, kAnyCapped>());
    }
  }
  return e;
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

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
  return paged_prompt_prepare_kernels();
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
  fill_prompt_args(A, p, t, mods, plan, seqs, q, out, lse, ws, w, accumulate, advance);
  return by_type(p, modded(A.mods), [&](auto eb, auto d, auto m) {
    return prompt_launches<DenseKernels, decltype(eb)::value, decltype(d)::value, decltype(m)::value>(A, plan, split, st);
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
