// Rotary positions with up to three axes, for the query token of every sequence (adsa_rotate) and for new tokens on their way into
// the caches (adsa_append).
//
//  k_rotate<EB, D, IN32, NEAR, APPEND>: a workgroup takes a few tokens and some of their rows (heads of q, then of k, then of v).
//    The angle of (token, pair) is one number for all heads: sum over the axes of coordinate * frequency, in 64 bits, brought to a
//    fraction of a turn there; its sine and cosine go to LDS once and every head's rows are turned with them.
//    A thread turns 8 pairs: 16 bytes of bf16 on either side of the row (NEAR false), or 32 bytes in a row (NEAR).
//    Bound by HBM (9216 tokens x 96 rows x 128: 90 us, 5 TB/s; 4352 x 72 x 64: 16.6 us, 4.8 TB/s), few tokens by two trips that depend on each other (3.4 us).
#include <algorithm>
#include <type_traits>

#include "adsa_device.h"
#include "adsa_partition.h"

namespace adsa {
namespace {

constexpr int kRotThreads = 256;

struct RotateArgs {
  const char* q;
  const char* k;
  const char* v;
  char* q_out;
  char* k_out;                     // rotate only
  adsa_seq* seqs;
  const double* freq;              // NULL: nothing is turned
  const int32_t* coords;           // NULL: from positions
  const int32_t* begin;            // append only
  const int32_t* slot0;
  const int32_t* pos0;
  long long q_stride_b, k_stride_b, v_stride_b, slot_stride_b, head_stride_b;
  int n_tokens, n_seq, max_len, hq, h, cap, total, score_rows, n_axes, advance;
  int tags_at;                     // place of the step tags in adsa_seq.vcos_u (fused V-cosine ranking), else 0
  int tokens_here, parts;          // tokens per workgroup; workgroups that share a token's rows
  int text[3], origin[3], row[3], col[3];
  GridWidth grid;
};
struct PagedRotateArgs : RotateArgs {
  PageArgs pages;
};

// What a workgroup knows of a token.
struct Token {
  gchar* k;                        // row of head 0 in the caches (append)
  gchar* v;
  int pos, origin;                 // absolute position; that of image token 0
  int ok;                          // rows are wanted (else zeros, and nothing enters the caches)
};

template <int D>
struct RotateShared {
  float2 turn[kRotThreads];        // (cos, sin) of [token][pair]
  Token token[kRotThreads / (D / 2)];
};

// 8 values at p
template <bool F32>
__device__ __forceinline__ void load8(const gchar* p, float* f) {
  const uint4 a = load16(p);
  if constexpr (F32) {
    const uint4 b = load16(p + 16);
    f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y); f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
    f[4] = __uint_as_float(b.x); f[5] = __uint_as_float(b.y); f[6] = __uint_as_float(b.z); f[7] = __uint_as_float(b.w);
  } else {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
}
template <int EB>
__device__ __forceinline__ void store8(gchar* p, const float* f) {
  if constexpr (EB == 4) {
    store16(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
    store16(p + 16, make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
  } else {
    store16(p, make_uint4(pack2_bf16(f[0], f[1]), pack2_bf16(f[2], f[3]), pack2_bf16(f[4], f[5]), pack2_bf16(f[6], f[7])));
  }
}

// Sequence of packed token t: the last b with begin[b] <= t.
__device__ __forceinline__ int sequence_of(const gint* begin, int n_seq, int t) {
  int lo = 0, hi = n_seq;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (begin[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// The new token t of adsa_append: where its rows go, or that its sequence's record does not fit.  The thread with `writes` also brings
// pos, score and, for a sequence's first token, the record up to date.  The other workgroups of the sequence may be reading the
// record meanwhile: what decides here is either not written by this launch, or decides the same way before and after (n_res >= slot0
// holds for the old n_res and for slot0 + len; a status that is set belongs to a record that everybody finds unfit).
// no_page (pages): the sequence's new slots that lack a page.  rows: where the rows of a slot's head 0 lie.
template <typename Rows>
__device__ __forceinline__ Token append_token(const RotateArgs& A, int t, bool writes, bool no_page, Rows rows) {
  Token tk = {nullptr, nullptr, 0, 0, 0};
  const gint* const begin = (const gint*)A.begin;
  const int b = sequence_of(begin, A.n_seq, t), from = begin[b], len = begin[b + 1] - from, j = t - from;
  if (j < 0 || j >= len) return tk;                            // (begin[] is not what it should be: nobody's token)
  ADSA_GLOBAL adsa_seq& sq = ((ADSA_GLOBAL adsa_seq*)A.seqs)[b];
  const int status = sq.status, n_res = sq.n_res, slot0 = ((const gint*)A.slot0)[b], P = sq.grid_origin;
  int reject = 0;
  if (n_res < 0 || n_res > A.cap || slot0 < 0 || slot0 > n_res || len > A.max_len || sq.hole != 0) reject = ADSA_SEQ_BAD_STATE;
  else if (len > A.cap - slot0) reject = ADSA_SEQ_CACHE_FULL;
  long long pos0 = 0;
  if (reject == 0) {
    pos0 = A.pos0 ? ((const gint*)A.pos0)[b] : slot0 > 0 ? (long long)((const gint*)sq.pos)[slot0 - 1] + 1 : 0;
    if (pos0 < 0 || pos0 + len > 0x7FFFFFFF || pos0 + len - P > A.total) reject = ADSA_SEQ_BAD_STATE;
  }
  if (reject == 0 && no_page) reject = ADSA_SEQ_CACHE_FULL;
  if (status != 0 || reject != 0) {
    if (writes && status == 0 && j == 0) sq.status = reject;
    return tk;
  }
  const int slot = slot0 + j;
  rows(b, slot, tk);
  tk.pos = (int)pos0 + j;
  tk.origin = P;
  tk.ok = 1;
  if (writes) {
    ((gint*)sq.pos)[slot] = tk.pos;
    gfloat* const score = (gfloat*)sq.score + slot;
    for (int r = 0; r < A.score_rows; ++r) score[(size_t)r * A.cap] = 0.0f;
    if (j == 0) {
      const long long image = pos0 + len - P;                  // image tokens up to the last new one
      sq.n_res = slot0 + len;
      sq.step = (image > 0 ? (int)image : 0) + A.advance;
      sq.compacted = 0;
      sq.pending_slot = -1;
      if (A.tags_at != 0 && sq.vcos_u) {
        gfloat* const tags = (gfloat*)sq.vcos_u + A.tags_at;
        for (int i = 0; i < kVcosTags; ++i) tags[i] = 0.0f;
      }
    }
  }
  return tk;
}

// Pages: whether the new tokens t0 .. t0 + n_here - 1 belong to sequences whose new slots all have a page, a bit each.  Every workgroup looks at all of
// a sequence's new pages, so all decide alike (slots that cannot be are append_token's to refuse).
template <typename Shared>
__device__ __forceinline__ void find_pages(const PagedRotateArgs& A, int t0, int n_here, Shared& no_page) {
  const gint* const begin = (const gint*)A.begin;
  if (threadIdx.x < n_here) no_page[threadIdx.x] = 0;
  __syncthreads();
  int b = -1;
  for (int i = 0; i < n_here; ++i) {                 // (uniform)
    const int before = b;
    b = sequence_of(begin, A.n_seq, t0 + i);
    const int slot0 = ((const gint*)A.slot0)[b], len = begin[b + 1] - begin[b];
    if (b == before) {                               // as the token before: looked at below
      continue;
    }
    if (slot0 < 0 || len < 1 || len > A.cap || slot0 > A.cap - len) continue;
    const gint* const table = (const gint*)A.pages.table + (size_t)b * A.pages.table_stride;
    bool bad = false;
    for (int e = (slot0 >> A.pages.shift) + (int)threadIdx.x; e <= (slot0 + len - 1) >> A.pages.shift; e += kRotThreads) bad |= (uint32_t)table[e] >= (uint32_t)A.pages.n_pages;
    if (bad) no_page[i] = 1;                         // (whoever stores stores the same)
  }
  __syncthreads();
}

template <int EB, int D, bool IN32, bool NEAR, bool APPEND, bool PAGED = false>
__global__ __launch_bounds__(kRotThreads) void k_rotate(std::conditional_t<PAGED, PagedRotateArgs, RotateArgs> A) {
  constexpr int kPairs = D / 2, IB = IN32 ? 4 : EB, kPieces = kPairs / 8;
  __shared__ RotateShared<D> sh;
  const int tid = threadIdx.x, t0 = (int)(blockIdx.x / (unsigned)A.parts) * A.tokens_here, part = (int)(blockIdx.x % (unsigned)A.parts);
  const int n_here = min(A.tokens_here, A.n_tokens - t0);
  // rows: q heads, k heads, then (append) v heads; a thread takes 8 pairs of a row, as two vectors of 8 elements, from ea and eb on
  const int q_rows = A.q ? A.hq : 0, rows = q_rows + (APPEND ? 2 : 1) * A.h;
  const int first = rows * part / A.parts, mine = rows * (part + 1) / A.parts - first, work = n_here * mine * kPieces;
  const int piece = tid % kPieces, ea = NEAR ? piece * 16 : piece * 8, eb = NEAR ? ea + 8 : ea + kPairs;       // (kRotThreads is a multiple of kPieces)
  int i = tid / kPieces / mine, r = tid / kPieces - i * mine;        // the thread's token and row of its part
  struct Place {
    bool is_q, is_v;
    int head;
  };
  auto place = [&](int row) { return Place{row < q_rows, row >= q_rows + A.h, row < q_rows ? row : row >= q_rows + A.h ? row - q_rows - A.h : row - q_rows}; };
  float a[8], b[8];
  auto fetch = [&](int i, int r) {
    const Place p = place(first + r);
    const long long t = t0 + i;
    const gchar* const in = (p.is_q ? (const gchar*)A.q + t * A.q_stride_b : p.is_v ? (const gchar*)A.v + t * A.v_stride_b : (const gchar*)A.k + t * A.k_stride_b) + p.head * (D * IB);
    load8<IB == 4>(in + ea * IB, a);
    load8<IB == 4>(in + eb * IB, b);
  };
  // ---- on their way together: the thread's first piece, its token and its pair's frequencies
  if (tid < work) fetch(i, r);
  const int ai = tid / kPairs, pair = tid % kPairs;                  // the angle that this thread forms
  const bool turns_one = A.freq && tid < n_here * kPairs;
  double f[3] = {0.0, 0.0, 0.0};
  if (turns_one) {
#pragma unroll
    for (int x = 0; x < 3; ++x)
      if (x < A.n_axes) f[x] = ((const ADSA_GLOBAL double*)A.freq)[x * kPairs + pair];
  }
  if constexpr (PAGED) {
    __shared__ int s_no_page[kRotThreads / kPairs];
    find_pages(A, t0, n_here, s_no_page);
    if (tid < n_here) {
      const gint* const begin = (const gint*)A.begin;
      int first = tid;                               // the first token here of the same sequence
      const int b = sequence_of(begin, A.n_seq, t0 + tid);
      first = max(0, begin[b] - t0);
      sh.token[tid] = append_token(A, t0 + tid, part == 0, s_no_page[min(first, tid)] != 0, [&](int seq, int slot, Token& tk) {
        const long long page = ((const gint*)A.pages.table)[(size_t)seq * A.pages.table_stride + (slot >> A.pages.shift)];
        const long long off = page * A.pages.page_stride_b + (slot & ((1 << A.pages.shift) - 1)) * A.slot_stride_b;
        tk.k = (gchar*)A.pages.k + off;
        tk.v = (gchar*)A.pages.v + off;
      });
    }
  } else if (tid < n_here) {
    const int t = t0 + tid;
    if constexpr (APPEND)
      sh.token[tid] = append_token(A, t, part == 0, false, [&](int b, int slot, Token& tk) {
        const ADSA_GLOBAL adsa_seq& sq = ((const ADSA_GLOBAL adsa_seq*)A.seqs)[b];
        tk.k = (gchar*)sq.k + slot * A.slot_stride_b;
        tk.v = (gchar*)sq.v + slot * A.slot_stride_b;
      });
    else {
      const ADSA_GLOBAL adsa_seq& sq = ((const ADSA_GLOBAL adsa_seq*)A.seqs)[t];
      const int step = sq.step;
      sh.token[tid] = {nullptr, nullptr, sq.grid_origin + step - 1, sq.grid_origin, step >= 0 && step <= A.total && sq.status == 0};
    }
  }
  __syncthreads();
  if (turns_one) {
    double c[3] = {0.0, 0.0, 0.0};
    if (A.coords) {
#pragma unroll
      for (int x = 0; x < 3; ++x)
        if (x < A.n_axes) c[x] = ((const gint*)A.coords)[(size_t)(t0 + ai) * A.n_axes + x];
    } else if (sh.token[ai].ok) {
      const int pos = sh.token[ai].pos, origin = sh.token[ai].origin;
      int col = 0, row = 0;
      if (pos >= origin) row = A.grid.row(pos - origin, &col);
#pragma unroll
      for (int x = 0; x < 3; ++x)
        c[x] = pos < origin ? (double)A.text[x] * pos : (double)A.origin[x] * origin + (double)A.row[x] * row + (double)A.col[x] * col;
    }
    double angle = 0.0;
#pragma unroll
    for (int x = 0; x < 3; ++x) angle = fma(c[x], f[x], angle);      // (axes that are not there have 0)
    double turns = angle * 0.15915494309189533577;                   // 1 / (2 pi)
    turns = 2.0 * (turns - rint(turns));                             // half turns, -1 .. 1
    const float x = (float)turns, d = (float)(turns - x) * 3.14159265358979f;
    float s, co;
    sincospif(x, &s, &co);
    sh.turn[tid] = make_float2(fmaf(-s, d, co), fmaf(co, d, s));
  }
  __syncthreads();
  for (int w = tid; w < work; w += kRotThreads) {
    const Token tk = sh.token[i];
    const Place p = place(first + r);
    float x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { x[e] = tk.ok ? a[e] : 0.0f; y[e] = tk.ok ? b[e] : 0.0f; }
    const float2* const turn = sh.turn + i * kPairs + piece * 8;
    gchar* out;
    if (p.is_q) out = (gchar*)A.q_out + ((size_t)(t0 + i) * A.hq + p.head) * (D * EB);
    else if constexpr (APPEND) out = (p.is_v ? tk.v : tk.k) + p.head * A.head_stride_b;
    else out = (gchar*)A.k_out + ((size_t)(t0 + i) * A.h + p.head) * (D * EB);
    // the next piece leaves before this one is stored (which nobody else reads or writes)
    r += kRotThreads / kPieces;
    while (r >= mine) { r -= mine; ++i; }
    if (w + kRotThreads < work) fetch(i, r);
    if (A.freq && !p.is_v && tk.ok) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 cs = turn[e];
        float& u = NEAR ? (e < 4 ? x[2 * e] : y[2 * e - 8]) : x[e];
        float& v = NEAR ? (e < 4 ? x[2 * e + 1] : y[2 * e - 7]) : y[e];
        const float u0 = u, v0 = v;
        u = u0 * cs.x - v0 * cs.y;
        v = v0 * cs.x + u0 * cs.y;
      }
    }
    if (APPEND && !tk.ok && !p.is_q) continue;
    store8<EB>(out + ea * EB, x);
    store8<EB>(out + eb * EB, y);
  }
}

template <bool APPEND, bool PAGED = false>
hipError_t launch(const adsa_params& p, std::conditional_t<PAGED, PagedRotateArgs, RotateArgs>& A, const adsa_rope* rope, bool in_f32, hipStream_t st) {
  const int D = p.head_dim, eb = elem_bytes(p), ib = in_f32 ? 4 : eb, pairs = D / 2;
  A.h = p.n_heads;
  A.hq = p.n_heads * (p.q_per_kv > 1 ? p.q_per_kv : 1);
  A.cap = p.cap;
  A.n_seq = p.n_seq;
  A.total = p.grid_h * p.grid_w;
  A.grid = {p.grid_w, 1.0f / (float)p.grid_w};
  A.slot_stride_b = p.kv_slot_stride * eb;
  A.head_stride_b = p.kv_head_stride * eb;
  if constexpr (PAGED) { A.slot_stride_b = A.pages.slot_stride_b; A.head_stride_b = A.pages.head_stride_b; }
  auto stride = [&](long long elements, int heads) { return (elements ? elements : (long long)heads * D) * ib; };
  A.q_stride_b = stride(A.q_stride_b, A.hq);
  A.k_stride_b = stride(A.k_stride_b, A.h);
  A.v_stride_b = stride(A.v_stride_b, A.h);
  if (rope) {
    A.freq = rope->freq;
    A.n_axes = rope->n_axes;
    for (int a = 0; a < ADSA_MAX_AXES; ++a) { A.text[a] = rope->text[a]; A.origin[a] = rope->origin[a]; A.row[a] = rope->row[a]; A.col[a] = rope->col[a]; }
  }
  // Few tokens: a token per workgroup, and its rows in as many parts as there are 256-thread pieces of them, so that every thread
  // has one piece of work behind the angles.  Many: about six pieces a thread, the next on its way while one is turned.  us at one token a
  // workgroup | two | four | eight, 4352 tokens of 24 + 2 x 24 heads x 64: 22 | 18.8 | 16.9 | 18.0 (80 MB); 9216 of 32 + 2 x 32 x 128: - | 93 | 101 | - (453 MB).
  const int rows = (A.q ? A.hq : 0) + (APPEND ? 2 : 1) * A.h;
  A.tokens_here = std::clamp(std::min(A.n_tokens / 512, 6 * kRotThreads / (rows * (pairs / 8))), 1, kRotThreads / pairs);
  A.parts = A.tokens_here == 1 ? std::clamp(rows * (pairs / 8) / kRotThreads, 1, 8) : 1;
  const dim3 grid((unsigned)((A.n_tokens + A.tokens_here - 1) / A.tokens_here * A.parts));
  const bool near = rope && rope->pairing == ADSA_PAIR_NEIGHBOURS;
#define ADSA_ROTATE(EB, IN32, NEAR)                                                                    \
  (D == 64 ? k_rotate<EB, 64, IN32, NEAR, APPEND, PAGED><<<grid, kRotThreads, 0, st>>>(A) : k_rotate<EB, 128, IN32, NEAR, APPEND, PAGED><<<grid, kRotThreads, 0, st>>>(A))
  if (eb == 4) { if (near) ADSA_ROTATE(4, true, true); else ADSA_ROTATE(4, true, false); }
  else if (in_f32) { if (near) ADSA_ROTATE(2, true, true); else ADSA_ROTATE(2, true, false); }
  else { if (near) ADSA_ROTATE(2, false, true); else ADSA_ROTATE(2, false, false); }
#undef ADSA_ROTATE
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const adsa_params& p, const adsa_rope& rope, const adsa_seq* seqs, const int32_t* coords, const void* q, const void* k,
                         int64_t q_stride, int64_t k_stride, void* q_out, void* k_out, bool in_f32, hipStream_t st) {
  RotateArgs A = {};
  A.q = (const char*)q; A.k = (const char*)k; A.q_out = (char*)q_out; A.k_out = (char*)k_out;
  A.seqs = const_cast<adsa_seq*>(seqs);
  A.coords = coords;
  A.q_stride_b = q_stride; A.k_stride_b = k_stride;
  A.n_tokens = p.n_seq;
  return launch<false>(p, A, &rope, in_f32, st);
}

static void fill_append_args(RotateArgs& A, const adsa_params& p, const adsa_tokens& t, adsa_seq* seqs, const void* q, const void* k, const void* v, void* q_out,
                             bool advance) {
  A.q = (const char*)q; A.k = (const char*)k; A.v = (const char*)v; A.q_out = (char*)q_out;
  A.seqs = seqs;
  A.coords = t.coords; A.begin = t.begin; A.slot0 = t.slot0; A.pos0 = t.pos0;
  A.q_stride_b = t.q_stride; A.k_stride_b = t.k_stride; A.v_stride_b = t.v_stride;
  A.n_tokens = t.n_tokens; A.max_len = t.max_len;
  A.score_rows = score_rows(p);
  A.advance = advance ? 1 : 0;
  A.tags_at = p.score_mode == ADSA_SCORE_VCOS_FUSED ? p.n_heads * p.head_dim : 0;
}

hipError_t launch_append(const adsa_params& p, const adsa_tokens& t, const adsa_rope* rope, adsa_seq* seqs, const void* q, const void* k, const void* v,
                         void* q_out, bool in_f32, bool advance, hipStream_t st) {
  RotateArgs A = {};
  fill_append_args(A, p, t, seqs, q, k, v, q_out, advance);
  return launch<true>(p, A, rope, in_f32, st);
}

hipError_t launch_append_paged(const adsa_params& p, const PageArgs& pages, const adsa_tokens& t, const adsa_rope* rope, adsa_seq* seqs, const void* q,
                               const void* k, const void* v, void* q_out, bool in_f32, bool advance, hipStream_t st) {
  PagedRotateArgs A = {};
  fill_append_args(A, p, t, seqs, q, k, v, q_out, advance);
  A.pages = pages;
  return launch<true, true>(p, A, rope, in_f32, st);
}

}  // namespace adsa
