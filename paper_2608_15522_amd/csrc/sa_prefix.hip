// Attention of a batch over keys and values kept in pages (sa_prefix_attention): the
// sequences of a group may share their first pages, whose keys are then read once for
// all of the group's queries.
//
// O = softmax(scale Q K^T) V over the keys of a sequence.  With the keys cut into parts
// i, each with its running max m_i (log2 units), sum l_i = sum 2^(x - m_i) and
// unnormalised row O_i = sum 2^(x - m_i) v, the whole is
//   M = max m_i,  O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i,
// so the shared keys can be taken against the queries of all sequences of the group at
// once and the sequences' own keys one sequence at a time.
//
// Segments.  Per key head: the shared keys of each group against the rows of all its
// sequences (kShared; only where a sequence has few rows), then each sequence's other
// keys against its own rows.  The rows of (sequence, key head) are its Hq / Hkv heads
// times S queries, which lie one behind the other in Q; in its own segment they are taken
// query by query, as many as it has, so that the rows of a tile see nearly the same keys
// under a causal mask.  A segment is row tiles times 64-key tiles; all of them, head by head, laid
// end to end are the call's units of work, cut into runs that differ by a unit at most, one
// per workgroup slot of the chip, unless whole row tiles are better (plan_of).  The lengths
// are read on the device, so a captured call follows them; every workgroup finds its run by
// the same prefix sums over the segments.  A row tile that runs share leaves partial rows,
// which prefix_combine_kernel joins in key order, so results do not depend on timing.
#include <float.h>

#include "sa_device.h"
#include "sa_internal.h"

namespace sa {
namespace {

typedef __attribute__((address_space(3))) uint16_t lds_u16_t;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4_t;

constexpr int kTile = 64;         // keys per unit of work
constexpr int kMaxWaves = 8;      // waves of a workgroup: 4, or 8 of the forms of few rows
constexpr int kSegs = kMaxAttendSegs;

// The running max is raised when a score exceeds it by 2^8, as in the other attention
// kernels: weights stay below 2^8, exact after the division by the row sum.
constexpr float kRescaleSlack = 8.0f;
constexpr float kSlackWeight = 1.f / 256.f;  // 2^-kRescaleSlack

// Units of work of a row tile: one for each 64-key tile, and `cost` for what it takes
// whatever its keys (finding its pages, the first copies' latency, its epilogue).  A cut
// leaves at least kSnap tiles on either side, or moves to the row tile's end.  64 samples
// of 4 query heads a key head (8 of them) over 16384 shared tokens and up to 2000 of their
// own at d 128 take 86 us with costs of 4 (128 rows) and 6 (32 rows), 83 to 87 with 2 to 4 of
// either; 4 groups of 8 such samples 87, and 89 to 92.
constexpr int kSnap = 2;
constexpr int kRunMin = 5;  // least units of a run

// A divisor d that the host knows: with l the bits of d - 1 and m = 2^(31+l) / d rounded
// down, plus 1, floor(x / d) = floor(x m / 2^(31+l)) for 0 <= x < 2^31, since m d exceeds
// 2^(31+l) by at most 2^l.
struct Div {
  int d;
  uint32_t m;
  int l;
  __device__ __forceinline__ int by(int x) const {
    return static_cast<int>(__umulhi(static_cast<uint32_t>(x) << 1, m) >> l);
  }
};
Div divisor(int d) {
  int l = 0;
  while ((1ll << l) < d) ++l;
  return {d, static_cast<uint32_t>((1ull << (31 + l)) / static_cast<uint32_t>(d) + 1), l};
}

struct Args {
  const void* q;
  const void* kp;
  const void* vp;
  void* o;
  float* lse;
  const int32_t* table;
  const int32_t* seq_len;
  const int32_t* shared_len;  // NULL: nothing shared
  const int32_t* q_len;       // NULL: S queries each
  int B, G, N;                // sequences, groups (0: no shared segments), sequences a group
  int Hkv, R, S, RS;          // key heads, query heads a key head, queries, R * S
  Div by_N, by_S, by_R, by_RS, by_B, by_tiles;  // by_tiles: B * nrto
  int n_pages, lp, max_pages, causal;
  int TRp, TRo;               // rows of a row tile: shared segments, own segments
  int lTRp, lTRo;             // their logarithms
  int TR;                     // the larger of the two: rows of a partial row tile's place
  int cp, co;                 // cost of a row tile: shared segments, own segments
  Log2Scale c;
  int* shared_out;            // [G] shared tokens that the call takes once
  int2* parts;                // [row tiles] first slot, parts (0: none, 1: the whole tile)
  int cols;                   // XCDs that share a head's row tiles (tile_of)
  int longer;                 // of these, those that take by_longer.d row tiles; the others
  Div by_longer, by_least;    // by_least.d
  int nrtp, nrto;             // row tiles of a segment (an own one with S queries)
  float* full;                // [2][B * Hq * S][D] partial rows of whole row tiles
  float2* full_ml;            // [2][B * Hq * S]
  float* piece;               // [2 slots][TR][D] partial rows of shared row tiles
  float2* piece_ml;           // [2 slots][TR]
};

__device__ __forceinline__ int seq_tokens(const Args& a, int b) {
  const long long cap = static_cast<long long>(a.max_pages) << a.lp;
  const int len = a.seq_len[b];
  return len < 0 ? 0 : static_cast<int>(len < cap ? len : cap);
}
// What the queries' positions count from: a length beyond the table row leaves out the tokens
// that have no page, and the newest queries stay where they are.
__device__ __forceinline__ int seq_end(const Args& a, int b) { return max(a.seq_len[b], 0); }
__device__ __forceinline__ int seq_queries(const Args& a, int b) {
  return a.q_len != nullptr ? min(max(a.q_len[b], 0), a.S) : a.S;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// x / y for 0 <= x < 2^30, 0 < y, inv = 1.f / y, and quotients below 2^21: x, y, inv and the
// product are each rounded by 2^-24 relatively, so the product is off by less than one.  The
// kernel's start is bound by cold instruction fetches, and an integer division is some thirty
// of them.
__device__ __forceinline__ int div_small(int x, int y, float inv) {
  int q = static_cast<int>(static_cast<float>(x) * inv);
  q -= q * y > x;
  q += x - q * y >= y;
  return q;
}

__device__ __forceinline__ int group_of(const Args& a, int b) { return a.by_N.by(b); }
// Query of a row within (sequence, key head), as they lie in Q.
__device__ __forceinline__ int query_of(const Args& a, int in) {
  return in - a.by_S.by(in) * a.S;
}

// An address that is the same in every lane, as the copies need it, for certain.
template <typename P>
__device__ __forceinline__ const P* uniform(const P* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint64_t lo = static_cast<uint32_t>(uniform(static_cast<int>(x)));
  const uint64_t hi = static_cast<uint32_t>(uniform(static_cast<int>(x >> 32)));
  return reinterpret_cast<const P*>(hi << 32 | lo);
}

// Prefix sums of the segments' units of one head, the sequences' lengths, and the shared
// tokens of each group: whole pages, at most what every sequence with a key has and
// (causal) what its first query sees.
struct Schedule {
  alignas(16) int off[kSegs + 1];
  int wave_tot[kMaxWaves];
  int len[kSegs];
  int nq[kSegs];  // queries
  int sh[kSegs / 2];
  int most;  // units of the longest row tile
};

__device__ __forceinline__ int row_units(int cost, int keys) {
  return cost + ceil_div(keys, kTile);
}

// Queries and row tiles of sequence b.
__device__ __forceinline__ int queries_of(const Args& a, const Schedule& s, int b) {
  return a.q_len == nullptr ? a.S : s.nq[b];
}
__device__ __forceinline__ int own_tiles(const Args& a, const Schedule& s, int b) {
  return a.q_len == nullptr ? a.nrto : (a.R * s.nq[b] + a.TRo - 1) >> a.lTRo;
}

// Tokens of sequence b behind the shared ones.
template <bool GROUPS>
__device__ __forceinline__ int own_keys(const Args& a, const Schedule& s, int b) {
  return GROUPS ? max(s.len[b] - s.sh[group_of(a, b)], 0) : s.len[b];
}

template <int W, bool GROUPS>
__device__ void build_schedule(const Args& a, Schedule& s) {
  constexpr int NT = W * kWave;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if constexpr (GROUPS)
    for (int g = tid; g < a.G; g += NT) s.sh[g] = 0x7fffffff;
  if (tid == 0) s.most = 0;
  __syncthreads();
  for (int b = tid; b < a.B; b += NT) {
    const int len = seq_tokens(a, b), nq = seq_queries(a, b);
    s.len[b] = len;
    s.nq[b] = nq;
    if (!GROUPS) atomicMax(&s.most, row_units(a.co, len));
    if (GROUPS && len > 0)
      atomicMin(&s.sh[group_of(a, b)],
                a.causal ? max(min(seq_end(a, b) - max(nq - 1, 0), len), 0) : len);
  }
  __syncthreads();
  if constexpr (GROUPS) {
    for (int g = tid; g < a.G; g += NT) {
      // no sequence of the group has a key: nothing to share
      const int v = s.sh[g] == 0x7fffffff ? 0 : min(s.sh[g], max(a.shared_len[g], 0));
      s.sh[g] = v >> a.lp << a.lp;
    }
    __syncthreads();
  }
  const int groups = GROUPS ? a.G : 0, n = groups + a.B, each = ceil_div(n, NT);
  const int i0 = min(tid * each, n), i1 = min(i0 + each, n);
  auto units = [&](int i) {
    if (i < groups) return s.sh[i] == 0 ? 0 : a.nrtp * row_units(a.cp, s.sh[i]);
    const int b = i - groups;
    return own_tiles(a, s, b) * row_units(a.co, own_keys<GROUPS>(a, s, b));
  };
  int sum = 0;
  for (int i = i0; i < i1; ++i) sum += units(i);
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(incl, o, 64);
    if (lane >= o) incl += u;
  }
  if (lane == 63) s.wave_tot[wave] = incl;
  __syncthreads();
  int at = incl - sum;
#pragma unroll
  for (int w = 0; w < W; ++w)
    if (w < wave) at += s.wave_tot[w];
  for (int i = i0; i < i1; ++i) {
    s.off[i] = at;
    at += units(i);
  }
  if (i1 == n && i0 < n) s.off[n] = at;
  __syncthreads();
}

// What one workgroup does at a time: 64-key tiles [t0, t1) of a row tile of a segment.
struct Job {
  int h;            // key head
  int b0;           // kShared: first sequence of the group; else the sequence
  int rows;         // rows of the segment: kShared RS a sequence, else R a query
  int nq;           // not kShared: the sequence's queries
  int row0;         // first row of the tile
  int pos0, pos1;   // key positions of the segment
  const int32_t* pages;  // table row that they are read through
  int t0, t1;
  bool shared;
  bool whole;       // all tiles of the row tile
  int piece;        // place of the partial rows if not
};

// Row rho of a segment: sequence, row within (sequence, key head), query, whether the
// segment has it, and whether it holds a query.
struct Row {
  int b, in, query;
  bool inside, real;
};
__device__ __forceinline__ Row row_of(const Args& a, const Job& j, int rho) {
  Row r;
  r.inside = rho < j.rows;
  rho = r.inside ? rho : j.rows - 1;
  if (j.shared) {
    const int k = a.by_RS.by(rho);
    r.b = j.b0 + k;
    r.in = rho - k * a.RS;
    r.query = query_of(a, r.in);
    r.real = r.inside && r.query < seq_queries(a, r.b);
  } else {
    r.b = j.b0;
    r.query = a.by_R.by(rho);
    r.in = (rho - r.query * a.R) * a.S + r.query;
    r.real = r.inside;
  }
  return r;
}
__device__ __forceinline__ size_t row_index(const Args& a, int h, const Row& r) {
  return (static_cast<size_t>(r.b) * a.Hkv + h) * a.RS + r.in;
}

// 64 table entries ahead of a sweep over ascending positions, one a lane, the next 64
// on their way: a page number is then a lane read.
struct PageCursor {
  const int32_t* pages;
  int max_pages, n_pages, lp;
  int base, cur, next;
  __device__ __forceinline__ int load(int i) const {
    i += threadIdx.x & 63;
    return i < max_pages ? pages[i] : -1;
  }
  __device__ __forceinline__ void start(const Args& a, const int32_t* p, int pos) {
    pages = p;
    max_pages = a.max_pages;
    n_pages = a.n_pages;
    lp = a.lp;
    base = __builtin_amdgcn_readfirstlane(pos >> lp);
    cur = load(base);
    next = load(base + 64);
  }
  // Row of the pool (in tokens of one head, page 0 for an entry that is no page) that
  // holds position pos, pos being at most 64 pages behind the last one asked for.
  __device__ __forceinline__ size_t row(int pos, int h, int Hkv) {
    pos = uniform(pos);
    h = uniform(h);
    int i = __builtin_amdgcn_readfirstlane(pos >> lp) - base;
    if (i >= 64) {
      base += 64;
      i -= 64;
      cur = next;
      next = load(base + 64);
    }
    int p = __builtin_amdgcn_readlane(cur, i);
    p = p >= 0 && p < n_pages ? p : 0;
    return (((static_cast<size_t>(p) * Hkv + h) << lp) + (pos & ((1 << lp) - 1)));
  }
  // Whether an entry between the cursor's start and position `end` is no page: its keys are
  // left out.  The entries that start() loads, and what lies behind them.
  __device__ __forceinline__ bool bad(int end) const {
    const int last = ceil_div(end, 1 << lp), lane = threadIdx.x & 63;
    auto none = [&](int i, int p) { return i < last && (p < 0 || p >= n_pages); };
    bool b = none(base + lane, cur) || none(base + 64 + lane, next);
    for (int i = base + 128; i < last; i += 64) b = b || none(i + lane, load(i));
    return __any(b);
  }
};

__device__ __forceinline__ bool bad_page(const Args& a, const int32_t* pages, int pos) {
  const int i = pos >> a.lp;
  if (i >= a.max_pages) return true;
  const int p = pages[i];
  return p < 0 || p >= a.n_pages;
}

__device__ __forceinline__ float max_halves(float x) {
  const auto pr = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x),
                                                   false, false);
  return fmaxf(x, fmaxf(__uint_as_float(pr[0]), __uint_as_float(pr[1])));
}
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }  // lgkmcnt(0)

// Last key position that a row sees, plus one.
__device__ __forceinline__ int row_end(const Args& a, const Job& j, const Row& r) {
  if (!a.causal || j.shared) return j.pos1;
  return min(j.pos1, seq_end(a, r.b) - j.nq + r.query + 1);
}

__device__ __forceinline__ float natural_lse(float m, float l) {
  return l == 0.f ? -INFINITY
                  : static_cast<float>(static_cast<double>(m) * 0.6931471805599453 +
                                       static_cast<double>(logf(l)));
}

// ---- rows out ---------------------------------------------------------------------------
// Four channels of a row and its (m, l), m in log2 units: to O and lse if the row tile is
// whole and nothing is to be joined to it, else to the row's place among the partial rows.
template <int D, typename T>
__device__ __forceinline__ void store_row(const Args& a, size_t at, int c4, f32x4 num, float m,
                                          float l) {
  const float inv = l != 0.f ? 1.f / l : 0.f;  // a row without a key is zeros
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + at * D + 4 * c4) =
        u32x2{pack_bf16x2(num[0] * inv, num[1] * inv), pack_bf16x2(num[2] * inv, num[3] * inv)};
  else
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + at * D + 4 * c4) =
        f32x4{num[0] * inv, num[1] * inv, num[2] * inv, num[3] * inv};
  if (a.lse != nullptr && c4 == 0) a.lse[at] = natural_lse(m, l);
}
template <int D, typename T>
__device__ __forceinline__ void put_row(const Args& a, const Job& j, int jr, int c4, f32x4 num,
                                        float m, float l) {
  const Row r = row_of(a, j, j.row0 + jr);
  if (j.whole && a.G == 0) {
    if (r.real) store_row<D, T>(a, row_index(a, j.h, r), c4, num, m, l);
    return;
  }
  size_t at = static_cast<size_t>(j.piece) * a.TR + jr;
  if (j.whole)
    at = (j.shared ? 0 : static_cast<size_t>(a.B) * a.Hkv * a.RS) + row_index(a, j.h, r);
  *reinterpret_cast<f32x4*>((j.whole ? a.full : a.piece) + at * D + 4 * c4) = num;
  if (c4 == 0) (j.whole ? a.full_ml : a.piece_ml)[at] = make_float2(m, l);
}

// Joins the waves' partial rows of a row tile, in wave order.  A wave's rows lie in its
// own LDS buffers (BYTES each), slot c4 of row r at join_slot(r, c4).
constexpr int kJoinRows = 32;
template <int D>
__device__ __forceinline__ int join_slot(int r, int c4) {
  return r * D * 4 + ((c4 ^ r) & (D / 4 - 1)) * 16;
}
template <int D, int W, int BYTES, typename T>
__device__ __forceinline__ void join_waves(const Args& a, const Job& j, int rows,
                                           const char* lds_all, const float2* lds_ml) {
  __syncthreads();
  constexpr int TPR = D / 4;
  for (int u = threadIdx.x; u < rows * TPR; u += W * kWave) {
    const int jr = u / TPR, c4 = u % TPR;
    float M = -FLT_MAX, den = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w)
      if (lds_ml[w * kJoinRows + jr].y != 0.f) M = fmaxf(M, lds_ml[w * kJoinRows + jr].x);
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float2 ml = lds_ml[w * kJoinRows + jr];
      const float f = ml.y != 0.f ? fast_exp2(ml.x - M) : 0.f;
      const f32x4 x = *reinterpret_cast<const f32x4*>(lds_all + w * BYTES + join_slot<D>(jr, c4));
      den = fmaf(f, ml.y, den);
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] = fmaf(f, x[e], num[e]);
    }
    put_row<D, T>(a, j, jr, c4, num, M, den);
  }
  __syncthreads();  // the buffers may be filled again
}

// The thread's number, found anew for every job: what is derived from it would otherwise be
// computed once for all jobs and kept in scratch memory (45 registers' worth).
__device__ __forceinline__ int my_thread() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// ---- bf16, few rows ---------------------------------------------------------------------
// 32 rows to a workgroup; its waves take 32-key pieces in turn, each through 16 KB (d = 128)
// of LDS of its own, so the loop has no barrier, and join their rows at the end.  Bound by
// HBM: each key row is used for 32 rows at most.  A wave has one buffer for K and one for
// V, refilled by LDS DMA as soon as it is used up: K of the next piece is on its way during
// the softmax and P V, V during the next piece's Q K^T.
constexpr int kPiece = 32;
// lds_dma16 of data that is read once (nontemporal).
__device__ __forceinline__ void lds_dma16_once(const char* sbase, uint32_t voff,
                                               uint32_t lds_addr) {
  asm volatile(
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, %1 nt"
      :
      : "v"(voff), "s"(sbase), "s"(lds_addr)
      : "memory", "m0");
}
template <int D, int W>
__device__ void attend_few(const Args& a, const Job& j, char* lds_all, float2* lds_ml) {
  constexpr int KC = D / 16, DT = D / 32, NI = kPiece * D * 2 / 1024;
  constexpr int BUF = kPiece * D * 2;  // bytes
  const int tid = my_thread(), lane = tid & 63, g = lane >> 5, n = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char* lds = lds_all + wave * 2 * BUF;
  const uint32_t lds_k = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(lds_void_t*)lds);
  const uint32_t lds_v = lds_k + BUF;

  const Row row = row_of(a, j, j.row0 + n);
  const uint16_t* q = static_cast<const uint16_t*>(a.q);
  const int run0 = j.pos0 + kTile * j.t0, run1 = min(j.pos1, j.pos0 + kTile * j.t1);
  const int first = run0 + kPiece * wave;
  // loads that do not wait for one another go out together: table entries, Q
  PageCursor cur;
  cur.start(a, j.pages, min(first, max(run1 - 1, 0)));
  u32x4 qf[KC];
#pragma unroll
  for (int kc = 0; kc < KC; ++kc)
    qf[kc] = row.inside ? ldg16(q + row_index(a, j.h, row) * D + 16 * kc + 8 * g)
                        : u32x4{0u, 0u, 0u, 0u};
  const bool bad = cur.bad(run1);
  const int end = row_end(a, j, row);

  // DMA: 1 KB = 16 rows of one 32-channel plane; lane l's source is the 16-byte slot that
  // the swizzle keeps at slot l % 4 of row l / 4.
  const uint32_t voff = static_cast<uint32_t>((lane >> 2) * (D * 2) +
                                              16 * ((lane & 3) ^ plane_swz(lane >> 2)));
  const int k_off0 = n * 64 + 16 * ((0 + g) ^ plane_swz(n));
  const int k_off1 = n * 64 + 16 * ((2 + g) ^ plane_swz(n));
  const int grp = lane >> 4, gi = lane & 15;
  const int tr_key = 4 * (grp >> 1) + (gi >> 2);
  const int tr_byte = 32 * (grp & 1) + 8 * (gi & 3);
  const int v_off0 = tr_key * 64 + 16 * ((tr_byte >> 4) ^ plane_swz(tr_key)) + (tr_byte & 15);
  const int v_off1 = (8 + tr_key) * 64 + 16 * ((tr_byte >> 4) ^ plane_swz(8 + tr_key)) +
                     (tr_byte & 15);

  size_t off[2];  // byte offsets of the piece's two 16-row groups, the same in K and V
  auto look = [&](int pos) {
#pragma unroll
    for (int u = 0; u < 2; ++u) off[u] = cur.row(pos + 16 * u, j.h, a.Hkv) * (D * 2);
  };
  // Own keys behind shared ones are read once, by this job, and leave the caches to the
  // shared ones (nt): 64 samples of 4 query heads over 16384 shared tokens and up to 2000 of
  // their own: 94 to 86 us; 16 of 6 queries each over 4992 and up to 700: 46 to 40.  Without
  // shared keys 26 to 28 (64 sequences of up to 1000).
  const bool once = j.pos0 > 0;
  auto issue = [&](const void* pool, uint32_t to) {
    const char* p = static_cast<const char*>(pool);
    if (once) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        lds_dma16_once(uniform(p + off[i & 1]), voff + 64 * (i >> 1),
                       to + (i >> 1) * 2048 + (i & 1) * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        lds_dma16(uniform(p + off[i & 1]), voff + 64 * (i >> 1),
                  to + (i >> 1) * 2048 + (i & 1) * 1024);
    }
  };

  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = zero16();
  float m = -FLT_MAX, lsum = 0.f;
  const float c = a.c.hi + a.c.lo;
  if (first < run1) {
    look(first);
    issue(a.kp, lds_k);
    issue(a.vp, lds_v);
  }
  for (int pos = first; pos < run1; pos += kPiece * W) {
    const bool more = pos + kPiece * W < run1;
    const bool masked = bad || pos + kPiece > run1 || (a.causal && !j.shared);
    wait_vm<NI>();  // K; V's copies are behind it
    __builtin_amdgcn_sched_barrier(0);
    f32x16 s = zero16();
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const u32x4 ka = *reinterpret_cast<const u32x4*>(lds + (kc >> 1) * 2048 +
                                                       ((kc & 1) ? k_off1 : k_off0));
      s = mfma32x32x16(ka, qf[kc], s);
    }
    wait_lds();  // the reads of K are done
    __builtin_amdgcn_sched_barrier(0);
    if (more) {
      look(pos + kPiece * W);
      issue(a.kp, lds_k);
    }
    bool none[2] = {false, false};  // the piece's 16-key groups without a page
    if (masked) {
      if (bad) {
        none[0] = bad_page(a, j.pages, pos);
        none[1] = bad_page(a, j.pages, pos + 16);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = crow(i, g);
        if (pos + key >= end || none[key >> 4]) s[i] = -INFINITY;
      }
    }
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = max_halves(mx) * c;
    if (__any(mx > m + kRescaleSlack)) {
      const float m_new = fmaxf(m, mx);
      const float alpha = fast_exp2(m - m_new);
      m = m_new;
      lsum *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] *= alpha;
    }
    // the row sum in fp32, the weights of P V rounded to bf16 (its operand type): half a
    // step of 2^-8 each, averaged over the keys
    uint32_t pb[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p0 = fast_exp2(fmaf(s[2 * i], c, -m));
      const float p1 = fast_exp2(fmaf(s[2 * i + 1], c, -m));
      lsum += p0 + p1;
      pb[i] = pack_bf16x2(p0, p1);
    }
    if (more)
      wait_vm<NI>();  // V; the next K's copies are behind it
    else
      wait_dma();
    __builtin_amdgcn_sched_barrier(0);
    if (masked) {
      // rows of V that no row of the workgroup sees may hold anything, NaN too: zeros
      const int rr = lane >> 1;  // a row's halves of every plane
      const bool gone = pos + rr >= run1 || (rr < 16 ? none[0] : none[1]);
      if (gone) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          char* z = lds + BUF + dt * 2048 + rr * 64 + (lane & 1) * 32;
          *reinterpret_cast<u32x4*>(z) = u32x4{0u, 0u, 0u, 0u};
          *reinterpret_cast<u32x4*>(z + 16) = u32x4{0u, 0u, 0u, 0u};
        }
      }
      wait_lds();
      __builtin_amdgcn_sched_barrier(0);
    }
    const lds_u16_t* Vb = (const lds_u16_t*)(lds + BUF);
#pragma unroll
    for (int mm = 0; mm < 2; ++mm) {
      const u32x4 b = {pb[4 * mm], pb[4 * mm + 1], pb[4 * mm + 2], pb[4 * mm + 3]};
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const lds_u16_t* base = Vb + (dt * 2048 + mm * 1024) / 2;
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4_t*)(base + v_off0 / 2)));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4_t*)(base + v_off1 / 2)));
        acc[dt] = mfma32x32x16(u32x4{lo.x, lo.y, hi.x, hi.y}, b, acc[dt]);
      }
    }
    wait_lds();  // the reads of V are done
    __builtin_amdgcn_sched_barrier(0);
    if (more) issue(a.vp, lds_v);
  }

  // the wave's rows in its own buffers, 16-byte slots swizzled by row
  const int rows = min(32, j.rows - j.row0);
  const float ltot = lsum + swap_halves(lsum);
  if (n < rows) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg)
        *reinterpret_cast<f32x4*>(lds + join_slot<D>(n, 8 * dt + 2 * rg + g)) =
            f32x4{acc[dt][4 * rg], acc[dt][4 * rg + 1], acc[dt][4 * rg + 2], acc[dt][4 * rg + 3]};
    if (g == 0) lds_ml[wave * kJoinRows + n] = make_float2(m, ltot);
  }
  join_waves<D, W, 2 * BUF, uint16_t>(a, j, rows, lds_all, lds_ml);
}

// ---- bf16, many rows --------------------------------------------------------------------
// 128 rows to a workgroup, 32 a wave; 64-key tiles of K and V go through double-buffered
// LDS that the waves share, by LDS DMA: wave w copies the tile's 16-key group w, which lies
// in one page.  Bound by the matrix cores.  The products, the softmax and the order of the
// steady-state loop are those of the block-sparse kernel (sa_attn.hip): S(t+1) = K Q^T runs
// under the exponentials of tile t, the row max of S(t+1) under P(t) V.  K is copied two
// tiles ahead, V one.
constexpr int kManyRows = 128;
template <int D>
__device__ void attend_many(const Args& a, const Job& j, char* lds) {
  constexpr int KC = D / 16, DT = D / 32;
  constexpr int NI = D / 32;                 // DMA instructions a wave and tile
  constexpr int TILE = kTile * D * 2;        // bytes of a tile of K or V
  const int tid = my_thread(), lane = tid & 63, g = lane >> 5, n = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // the lane's row: found again where it is needed, since the loop needs every register
  auto my_row = [&]() { return row_of(a, j, j.row0 + 32 * wave + n); };
  u32x4 qf[KC];
  {
    const Row row = my_row();
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + row_index(a, j.h, row) * D + 8 * g;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
      qf[kc] = row.inside ? ldg16(q + 16 * kc) : u32x4{0u, 0u, 0u, 0u};
  }
  const int run0 = j.pos0 + kTile * j.t0, run1 = min(j.pos1, j.pos0 + kTile * j.t1);
  int most = run1, least = run1;       // the furthest and the nearest end of the tile's rows
  if (a.causal && !j.shared) {
    const int q0 = seq_end(a, j.b0) - j.nq + 1, last = min(j.row0 + kManyRows, j.rows) - 1;
    most = min(run1, q0 + a.by_R.by(last));
    least = min(run1, q0 + a.by_R.by(j.row0));
  }
  PageCursor cur;  // from the same page in every wave, so that all find the same
  cur.start(a, j.pages, run0);
  const bool bad = cur.bad(run1);
  const int T = most > run0 ? ceil_div(most - run0, kTile) : 0;
  // leading tiles that every row sees whole
  const int T_full = bad || least <= run0 ? 0 : min((least - run0) / kTile, T);

  // DMA: 1 KB = 16 rows of one 32-channel plane; lane l's source is the 16-byte slot that
  // the swizzle keeps at slot l % 4 of row l / 4
  const uint32_t voff = static_cast<uint32_t>((lane >> 2) * (D * 2) +
                                              16 * ((lane & 3) ^ plane_swz(lane >> 2)));
  const int k_off0 = n * 64 + 16 * ((0 + g) ^ plane_swz(n));
  const int k_off1 = n * 64 + 16 * ((2 + g) ^ plane_swz(n));
  const int grp = lane >> 4, gi = lane & 15;
  const int tr_key = 4 * (grp >> 1) + (gi >> 2);
  const int tr_byte = 32 * (grp & 1) + 8 * (gi & 3);
  const int v_off0 = tr_key * 64 + 16 * ((tr_byte >> 4) ^ plane_swz(tr_key)) + (tr_byte & 15);
  const int v_off1 = (8 + tr_key) * 64 + 16 * ((tr_byte >> 4) ^ plane_swz(8 + tr_key)) +
                     (tr_byte & 15);

  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(lds_void_t*)lds);
  // byte addresses of the wave's group in the buffers of tile t
  auto kdst = [&](int t) { return lds0 + (t & 1) * TILE + wave * 1024; };
  auto vdst = [&](int t) { return lds0 + (2 + (t & 1)) * TILE + wave * 1024; };
  auto kbuf = [&](int t) -> const char* { return lds + (t & 1) * TILE; };
  auto vbuf = [&](int t) -> char* { return lds + (2 + (t & 1)) * TILE; };
  const char* kp = static_cast<const char*>(a.kp);
  const char* vp = static_cast<const char*>(a.vp);
  // byte offset of the wave's group of tile t, the same in K and V
  auto look = [&](int t) { return cur.row(run0 + kTile * t + 16 * wave, j.h, a.Hkv) * (D * 2); };

  auto qk = [&](int t, f32x16& s0, f32x16& s1) {
    const char* Kb = kbuf(t);
    s0 = zero16();
    s1 = zero16();
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const int off = (kc & 1) ? k_off1 : k_off0;
      const u32x4 a0 = *reinterpret_cast<const u32x4*>(Kb + (kc >> 1) * 4096 + off);
      const u32x4 a1 = *reinterpret_cast<const u32x4*>(Kb + (kc >> 1) * 4096 + 2048 + off);
      s0 = mfma32x32x16(a0, qf[kc], s0);
      s1 = mfma32x32x16(a1, qf[kc], s1);
    }
  };
  auto none = [&](int t, int group) {  // a 16-key group without a page
    return bad && bad_page(a, j.pages, run0 + kTile * t + 16 * group);
  };
  auto mask = [&](int t, f32x16& s0, f32x16& s1) {
    const int left = row_end(a, j, my_row()) - (run0 + kTile * t);
    bool gone[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) gone[u] = none(t, u);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = crow(i, g);
      if (key >= left || gone[(8 * (i >> 2)) >> 4]) s0[i] = -INFINITY;
      if (32 + key >= left || gone[2 + ((8 * (i >> 2)) >> 4)]) s1[i] = -INFINITY;
    }
  };
  auto tile_max = [&](const f32x16& s0, const f32x16& s1) {
    float mx = s0[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s0[i]);
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s1[i]);
    return mx;
  };

  // rows of V that no row of the workgroup sees may hold anything, NaN too: zeros
  auto clear = [&](int t) {
    const int rr = 16 * wave + (lane >> 2);
    if (run0 + kTile * t + rr >= most || none(t, wave)) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        *reinterpret_cast<u32x4*>(vbuf(t) + i * 4096 + rr * 64 + (lane & 3) * 16) =
            u32x4{0u, 0u, 0u, 0u};
    }
    wait_lds();
  };
  // A wave without rows copies its share of the tiles and computes nothing: one sequence of 24
  // rows in a last row tile leaves three waves idle.
  const bool idle = j.row0 + 32 * wave >= j.rows;

  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = zero16();
  float m = -FLT_MAX, lsum = 0.f;
  const float c = a.c.hi + a.c.lo;
  f32x16 sc0 = zero16(), sc1 = zero16(), sn_0, sn_1;
  float mx_cur = -INFINITY;
  size_t off1 = 0;  // of the next tile
  if (T > 0) {
    const size_t off0 = look(0);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      lds_dma16(uniform(kp + off0) + 64 * i, voff, kdst(0) + i * 4096);
      lds_dma16(uniform(vp + off0) + 64 * i, voff, vdst(0) + i * 4096);
    }
    off1 = off0;
    if (T > 1) {
      off1 = look(1);
#pragma unroll
      for (int i = 0; i < NI; ++i) lds_dma16(uniform(kp + off1) + 64 * i, voff, kdst(1) + i * 4096);
    }
    wait_dma();
    __syncthreads();
    if (!idle) {
      qk(0, sc0, sc1);
      if (T_full < 1) mask(0, sc0, sc1);
      mx_cur = tile_max(sc0, sc1);
      wait_lds();
    }
    __syncthreads();  // every wave has read K(0) before iteration 0 refills its buffer
  }
  auto rescale = [&]() {
    const float mx = max_halves(mx_cur) * c;
    if (__any(mx > m + kRescaleSlack)) {
      const float m_new = fmaxf(m, mx);
      const float alpha = fast_exp2(m - m_new);
      m = m_new;
      lsum *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] *= alpha;
    }
  };
  auto vread = [&](const lds_u16_t* Vb, int jj) {
    const lds_u16_t* base = Vb + ((jj % DT) * 4096 + (jj / DT) * 1024) / 2;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_s16x4_t*)(base + v_off0 / 2)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_s16x4_t*)(base + v_off1 / 2)));
    return u32x4{lo.x, lo.y, hi.x, hi.y};
  };
  // Any tile t: P(t), S(t+1) with its mask, P(t) V(t).  Past the last tile its copies are
  // repeated into the free buffers.
  auto iteration = [&](int t) {
    const size_t off2 = t + 2 < T ? look(t + 2) : off1;
    if (t >= T_full) clear(t);
    __syncthreads();
    rescale();
    f32x16 sn0, sn1;
    qk(t + 1, sn0, sn1);  // on stale data in the last iteration, and then not used
    if (t + 1 >= T_full && t + 1 < T) mask(t + 1, sn0, sn1);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      lds_dma16(uniform(kp + off2) + 64 * i, voff, kdst(t) + i * 4096);
      lds_dma16(uniform(vp + off1) + 64 * i, voff, vdst(t + 1) + i * 4096);
    }
    uint32_t pb[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p0 = fast_exp2(fmaf(sc0[2 * i], c, -m));
      const float p1 = fast_exp2(fmaf(sc0[2 * i + 1], c, -m));
      const float p2 = fast_exp2(fmaf(sc1[2 * i], c, -m));
      const float p3 = fast_exp2(fmaf(sc1[2 * i + 1], c, -m));
      lsum += (p0 + p1) + (p2 + p3);
      pb[i] = pack_bf16x2(p0, p1);
      pb[8 + i] = pack_bf16x2(p2, p3);
    }
    const lds_u16_t* Vb = (const lds_u16_t*)vbuf(t);
#pragma unroll
    for (int jj = 0; jj < 4 * DT; ++jj) {
      const int mm = jj / DT;
      const u32x4 b = {pb[4 * mm], pb[4 * mm + 1], pb[4 * mm + 2], pb[4 * mm + 3]};
      acc[jj % DT] = mfma32x32x16(vread(Vb, jj), b, acc[jj % DT]);
    }
    mx_cur = tile_max(sn0, sn1);
    sc0 = sn0;
    sc1 = sn1;
    off1 = off2;
    wait_dma();
    __syncthreads();
  };
  // Steady state: tiles t and t + 1 need no mask.  The issue order is fixed by scheduling
  // barriers so that every MFMA is followed by a share of the VALU work: in the Q K^T phase
  // one bf16 pair of P(t) per MFMA, in three stages a step apart (FMAs, exponentials,
  // packing); in the P V phase the row max of S(t+1).  Operand reads run two MFMAs ahead,
  // and the copies are spread over the Q K^T phase.
  auto main_iter = [&](int t, f32x16& c0, f32x16& c1, f32x16& n0, f32x16& n1) {
    const size_t off2 = t + 2 < T ? look(t + 2) : off1;
    const char* kbase = uniform(kp + off2);
    const char* vbase = uniform(vp + off1);
    off1 = off2;
    rescale();
    const char* Kb = kbuf(t + 1);
    const lds_u16_t* Vb = (const lds_u16_t*)vbuf(t);
    const uint32_t kd = kdst(t), vd = vdst(t + 1);
    auto kread = [&](int kc, u32x4* dst) {
      const int off = (kc & 1) ? k_off1 : k_off0;
      dst[0] = *reinterpret_cast<const u32x4*>(Kb + (kc >> 1) * 4096 + off);
      dst[1] = *reinterpret_cast<const u32x4*>(Kb + (kc >> 1) * 4096 + 2048 + off);
    };
    __builtin_amdgcn_s_setprio(1);
    constexpr int NA = 2 * KC;          // MFMAs
    constexpr int PPA = 16 / NA;        // bf16 pairs of P per MFMA
    u32x4 ka[3][2];
    uint32_t pb[16];
    kread(0, ka[0]);
    kread(1, ka[1]);
    n0 = zero16();
    n1 = zero16();
    float fx[2][PPA][2], ex[2][PPA][2];
    auto stage_fma = [&](int st) {
#pragma unroll
      for (int u = 0; u < PPA; ++u) {
        const int pk = st * PPA + u;
        const f32x16& src = pk < 8 ? c0 : c1;
        const int e = 2 * (pk & 7);
        fx[st & 1][u][0] = fmaf(src[e], c, -m);
        fx[st & 1][u][1] = fmaf(src[e + 1], c, -m);
      }
    };
    auto stage_exp = [&](int st) {
#pragma unroll
      for (int u = 0; u < PPA; ++u) {
        ex[st & 1][u][0] = fast_exp2(fx[st & 1][u][0]);
        ex[st & 1][u][1] = fast_exp2(fx[st & 1][u][1]);
        lsum += ex[st & 1][u][0] + ex[st & 1][u][1];
      }
    };
    auto stage_pack = [&](int st) {
#pragma unroll
      for (int u = 0; u < PPA; ++u)
        pb[st * PPA + u] = pack_bf16x2(ex[st & 1][u][0], ex[st & 1][u][1]);
    };
    stage_fma(0);
#pragma unroll
    for (int st = 0; st < NA; ++st) {
      const int kc = st >> 1;
      if ((st & 1) == 0 && kc + 2 < KC) kread(kc + 2, ka[(kc + 2) % 3]);
      if (st & 1)
        n1 = mfma32x32x16(ka[kc % 3][1], qf[kc], n1);
      else
        n0 = mfma32x32x16(ka[kc % 3][0], qf[kc], n0);
      if (st > 0) stage_pack(st - 1);
      stage_exp(st);
      if (st + 1 < NA) stage_fma(st + 1);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        if (i * NA / NI == st) lds_dma16(kbase + 64 * i, voff, kd + i * 4096);
        if (i * NA / NI + NA / (2 * NI) == st) lds_dma16(vbase + 64 * i, voff, vd + i * 4096);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    stage_pack(NA - 1);
    __builtin_amdgcn_s_setprio(0);
    constexpr int NB = 4 * DT;          // MFMAs
    constexpr int VB = 16 / NB > 0 ? 16 / NB : 1;  // pairs of the row max per MFMA
    u32x4 va[3];
    va[0] = vread(Vb, 0);
    va[1] = vread(Vb, 1);
    float mxn = -INFINITY;
#pragma unroll
    for (int jj = 0; jj < NB; ++jj) {
      if (jj + 2 < NB) va[(jj + 2) % 3] = vread(Vb, jj + 2);
      const int mm = jj / DT, dt = jj % DT;
      const u32x4 b = {pb[4 * mm], pb[4 * mm + 1], pb[4 * mm + 2], pb[4 * mm + 3]};
      acc[dt] = mfma32x32x16(va[jj % 3], b, acc[dt]);
#pragma unroll
      for (int u = 0; u < VB; ++u) {
        const int e = jj * VB + u;  // pair e: elements 2e, 2e+1 of n0 (e < 8) or n1
        const f32x16& src = e < 8 ? n0 : n1;
        mxn = fmaxf(mxn, src[2 * (e & 7)]);
        mxn = fmaxf(mxn, src[2 * (e & 7) + 1]);
        asm volatile("" : "+v"(mxn));  // keeps this share of the max in its slot
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    mx_cur = mxn;
    wait_dma();
    __syncthreads();
  };

  const int T_main = T_full == T ? T : (T_full > 1 ? T_full - 1 : 0);
  if (idle) {
    for (int t = 0; t < T; ++t) {
      const size_t off2 = t + 2 < T ? look(t + 2) : off1;
      if (t >= T_main) {
        if (t >= T_full) clear(t);
        __syncthreads();
      }
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        lds_dma16(uniform(kp + off2) + 64 * i, voff, kdst(t) + i * 4096);
        lds_dma16(uniform(vp + off1) + 64 * i, voff, vdst(t + 1) + i * 4096);
      }
      off1 = off2;
      wait_dma();
      __syncthreads();
    }
    return;
  }
  int t = 0;
  for (; t + 1 < T_main; t += 2) {
    main_iter(t, sc0, sc1, sn_0, sn_1);
    main_iter(t + 1, sn_0, sn_1, sc0, sc1);
  }
  if (t < T_main) {
    main_iter(t, sc0, sc1, sn_0, sn_1);
    sc0 = sn_0;
    sc1 = sn_1;
    ++t;
  }
  for (; t < T; ++t) iteration(t);

  const float ltot = lsum + swap_halves(lsum);
  const int jr = 32 * wave + n;
  if (j.row0 + jr >= j.rows) return;
  const Row row = my_row();
  if (j.whole && a.G == 0) {
    if (!row.real) return;
    const float inv = ltot != 0.f ? 1.f / ltot : 0.f;
    const size_t at = row_index(a, j.h, row);
    uint16_t* orow = static_cast<uint16_t*>(a.o) + at * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int rp = 0; rp < 2; ++rp) {
        // the lane's channels 16rp + 4g .. +3 and 16rp + 8 + 4g .. +3 of group dt,
        // exchanged with the lane of the other half: 8 in a row
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = pack_bf16x2(acc[dt][8 * rp + 2 * i] * inv, acc[dt][8 * rp + 2 * i + 1] * inv);
        const auto e0 = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
        const auto e1 = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
        stg16(orow + 32 * dt + 16 * rp + 8 * g, u32x4{e0[0], e1[0], e0[1], e1[1]});
      }
    if (g == 0 && a.lse != nullptr) a.lse[at] = natural_lse(m, ltot);
    return;
  }
  size_t at = static_cast<size_t>(j.piece) * a.TR + jr;
  if (j.whole)
    at = (j.shared ? 0 : static_cast<size_t>(a.B) * a.Hkv * a.RS) + row_index(a, j.h, row);
  float* po = (j.whole ? a.full : a.piece) + at * D;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int rg = 0; rg < 4; ++rg)
      *reinterpret_cast<f32x4*>(po + 32 * dt + 8 * rg + 4 * g) =
          f32x4{acc[dt][4 * rg], acc[dt][4 * rg + 1], acc[dt][4 * rg + 2], acc[dt][4 * rg + 3]};
  if (g == 0) (j.whole ? a.full_ml : a.piece_ml)[at] = make_float2(m, ltot);
}

// ---- fp32 -------------------------------------------------------------------------------
// 16 rows to a workgroup; its waves take 16-key pieces in turn: K through LDS buffers of
// their own (RowTile16), V in registers, both one piece ahead, products in fp32
// (v_mfma_f32_16x16x4_f32):
//   S^T = K Q^T    lane (n, gk) = (l % 16, l / 16) holds channels 16i + 4gk + e of Q[n]
//                  and K[n]; the result leaves it with keys 4gk .. 4gk + 3 of query n;
//   O^T += V^T P^T with k slot gk of step r standing for key 4gk + r, and row i of channel
//                  tile (dq, e) for channel 64dq + 4i + e.
// Weights are taken down by 2^-8, the slack of the running max, so that none exceeds 1.  Under a
// causal mask every row tile goes through all keys of its segment, also those that none of its
// rows sees (the form of many rows stops at the last that one does).
constexpr int kF32Keys = 16;
template <int D, int W>
__device__ void attend_f32(const Args& a, const Job& j, char* lds_all, float2* lds_ml) {
  constexpr int KI = D / 16, DQ = D / 64;
  using KTile = RowTile16<D>;
  const int tid = my_thread(), lane = tid & 63, n = lane & 15, gk = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char* lds = lds_all + wave * 2 * KTile::kBytes;
  const Row row = row_of(a, j, j.row0 + n);
  const float* q = static_cast<const float*>(a.q);
  const int run0 = j.pos0 + kTile * j.t0, run1 = min(j.pos1, j.pos0 + kTile * j.t1);
  const int first = run0 + kF32Keys * wave;
  PageCursor cur;
  cur.start(a, j.pages, min(first, max(run1 - 1, 0)));
  f32x4 qf[KI];
#pragma unroll
  for (int i = 0; i < KI; ++i)
    qf[i] = row.inside ? ldg_f32x4(q + row_index(a, j.h, row) * D + 16 * i + 4 * gk)
                       : f32x4{0.f, 0.f, 0.f, 0.f};
  const bool bad = cur.bad(run1);
  const int end = row_end(a, j, row);
  KTile kt;
  kt.init(lds, lane);
  struct Piece {
    f32x4 v[4][DQ];
  };
  auto load = [&](int pos, int buf, Piece& x) {
    const size_t at = cur.row(pos, j.h, a.Hkv) * D;
    kt.copy(uniform(static_cast<const float*>(a.kp) + at), 0, kF32Keys, buf);
    const float* v = static_cast<const float*>(a.vp) + at;
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int dq = 0; dq < DQ; ++dq)
        x.v[s][dq] = ldg_f32x4(v + (4 * gk + s) * D + 4 * n + 64 * dq);
  };
  f32x4 acc[DQ][4];
#pragma unroll
  for (int dq = 0; dq < DQ; ++dq)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[dq][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -FLT_MAX, lsum = 0.f;
  constexpr int STEP = kF32Keys * W;
  auto step = [&](int pos, int buf, Piece& x, Piece& nx) {
    wait_dma();
    __builtin_amdgcn_sched_barrier(0);
    f32x4 kf[KI];
    kt.read(buf, kf);
    if (pos + STEP < run1) load(pos + STEP, buf ^ 1, nx);
    __builtin_amdgcn_sched_barrier(0);
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KI; ++i)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        s0 = mfma16x16x4_f32(kf[i][e], qf[i][e], s0);
        s1 = mfma16x16x4_f32(kf[i][e + 1], qf[i][e + 1], s1);
      }
    float s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = s0[e] + s1[e];
    if (bad || pos + kF32Keys > run1 || (a.causal && !j.shared)) {
      const bool none = bad && bad_page(a, j.pages, pos);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = pos + 4 * gk + e;
        if (key >= end || none) s[e] = -INFINITY;
        // rows of V that no row of the workgroup sees may hold anything, NaN too
        if (key >= run1 || none)
#pragma unroll
          for (int dq = 0; dq < DQ; ++dq) x.v[e][dq] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
    const float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])) * a.c.hi;
    if (__any(mx > m + kRescaleSlack)) {
      float m_new = fmaxf(m, mx);
      m_new = fmaxf(m_new, __shfl_xor(m_new, 16, 64));
      m_new = fmaxf(m_new, __shfl_xor(m_new, 32, 64));
      const float alpha = fast_exp2(m - m_new);
      m = m_new;
      lsum *= alpha;
#pragma unroll
      for (int dq = 0; dq < DQ; ++dq)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[dq][e] *= alpha;
    }
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = kSlackWeight * fast_exp2(log2_score(s[e], a.c, m));
    lsum += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int dq = 0; dq < DQ; ++dq)
#pragma unroll
        for (int w = 0; w < 4; ++w)
          acc[dq][w] = mfma16x16x4_f32(x.v[e][dq][w], p[e], acc[dq][w]);
  };
  Piece xa, xb;
  if (first < run1) {
    load(first, 0, xa);
    int pos = first;
    for (; pos + STEP < run1; pos += 2 * STEP) {
      step(pos, 0, xa, xb);
      step(pos + STEP, 1, xb, xa);
    }
    if (pos < run1) step(pos, 0, xa, xb);
  }
  lsum += __shfl_xor(lsum, 16, 64);
  lsum += __shfl_xor(lsum, 32, 64);
  const int rows = min(16, j.rows - j.row0);
  wait_lds();
  if (n < rows) {
    // acc[dq][e][s] is channel 64dq + 16gk + 4s + e of query n
#pragma unroll
    for (int dq = 0; dq < DQ; ++dq)
#pragma unroll
      for (int s = 0; s < 4; ++s)
        *reinterpret_cast<f32x4*>(lds + join_slot<D>(n, 16 * dq + 4 * gk + s)) =
            f32x4{acc[dq][0][s], acc[dq][1][s], acc[dq][2][s], acc[dq][3][s]};
    // 2^-8 goes back into the reference, exactly
    if (gk == 0) lds_ml[wave * kJoinRows + n] = make_float2(m + kRescaleSlack, lsum);
  }
  join_waves<D, W, 2 * KTile::kBytes, float>(a, j, rows, lds_all, lds_ml);
}

// Bytes of LDS that the waves' buffers take: 16 KB a wave at d = 128 for either type.
template <int D, int W>
constexpr int attend_lds() {
  return W * 128 * D;
}

// ---- the runs ---------------------------------------------------------------------------
// Run c of n begins at unit c * total / n (at c * kRunMin in a small call), or at a row
// tile's end where that would leave less than kSnap tiles on either side.
struct Runs {
  int total, n;  // n <= 512 runs
  bool small;    // of kRunMin units each
};
__device__ __forceinline__ Runs runs_of(int total, int slots) {
  const bool small = total < slots * kRunMin;
  return {total, small ? ceil_div(total, kRunMin) : slots, small};
}
__device__ __forceinline__ int run_begin(const Runs& r, int c) {
  return r.small ? min(c * kRunMin, r.total)
                 : static_cast<int>(static_cast<long long>(r.total) * c / r.n);
}
// The last run that begins at unit x or before.
__device__ __forceinline__ int run_at(const Runs& r, int x) {
  int c = static_cast<int>(static_cast<float>(x) *
                           (r.small ? 1.f / kRunMin : r.n / static_cast<float>(r.total)));
  while (c > 0 && run_begin(r, c) > x) --c;
  while (c + 1 < r.n && run_begin(r, c + 1) <= x) ++c;
  return c;
}
// Where a cut at unit k of a row tile goes.
__device__ __forceinline__ int cut_at(int cost, int per, int k) {
  if (k >= cost + kSnap && k <= per - kSnap) return k;
  return k < cost + kSnap ? 0 : per;
}

// Where unit u lies: its head, segment, row tile, the units of the row tile before it, and
// those of the row tile.
struct Place {
  int h, seg, rt, k, per;
};
template <bool GROUPS>
__device__ __forceinline__ Place place_of(const Args& a, const Schedule& s, int per_head,
                                          float inv_head, int u) {
  const int lane = threadIdx.x & 63, groups = GROUPS ? a.G : 0, n = groups + a.B;
  Place p;
  p.h = uniform(div_small(u, per_head, inv_head));
  const int in = u - p.h * per_head;
  int before = 0;  // segments that start at or before `in`: the last of them is not empty
  for (int i = 0; i < n; i += 64)
    before += __popcll(__ballot(i + lane < n && s.off[i + lane] <= in));
  p.seg = uniform(before) - 1;
  const bool shared = p.seg < groups;
  const int b = p.seg - groups;
  if (GROUPS && shared)
    p.per = row_units(a.cp, uniform(s.sh[p.seg]));
  else
    p.per = row_units(a.co, uniform(own_keys<GROUPS>(a, s, b)));
  const int x = in - uniform(s.off[p.seg]);
  p.rt = uniform(div_small(x, p.per, 1.f / static_cast<float>(p.per)));
  p.k = x - p.rt * p.per;
  return p;
}

// How the row tiles reach the workgroups.  kWhole: one row tile a workgroup, every one
// written out at once.  kRuns: as above, without shared segments; if no sequence's rows take
// much longer than the mean and there are as many row tiles as slots, each slot first takes
// whole row tiles, in rounds of all slots of an XCD, and only the rest is cut: the workgroups
// of a round go through a head's keys side by side, so that these come from the XCD's L2.  16
// heads of 4 x 1024 queries over 16000 keys (a whole row tile a slot) run at 920 TFLOP/s, 20
// heads cut into equal runs at 740.  5 x 1024 queries, 16 heads, d 128, over 8000 keys in the
// mean, the longest 1.0, 1.2, 1.3 and 1.5 times that: 404, 390, 373 and 370 us in runs, 321, 347,
// 359 and 376 in rounds; 130 single tokens, 4 heads, over 3000: 148, 153, 152 and 153 in runs,
// 148, 155, 160 and 171 in rounds.  kGroups: runs over shared and own segments.  Each is a kernel
// of its own, since a short call waits for its instructions as long as for its data: 4 sequences
// of 316 tokens, 8 heads of d 64, 6.4 us in a kernel of kWhole alone, 7.8 in one of all three.
enum Split { kWhole, kRuns, kGroups };
constexpr float kUneven = 1.25f;  // the longest row tile to the mean, for rounds at most

// Row tile t of a call without shared segments: head by head, the last rows first (under a
// causal mask they see the most keys), sequence by sequence.  With a.cols > 1 XCDs to a head
// (kWhole) each takes every a.cols-th row tile, so that they have as many keys to see (6
// causal prompts of 701 queries each, 16 heads over 4, d 64: 39 to 34 us behind 512 tokens
// each, 43 to 38 behind 512 to 1014).
struct Tile {
  int h, b, rt;
};
template <bool WHOLE>
__device__ __forceinline__ Tile tile_of(const Args& a, int t) {
  Tile x;
  x.h = a.by_tiles.by(t);
  const int in = t - x.h * a.by_tiles.d;
  int q = a.by_B.by(in);
  x.b = in - q * a.B;
  if (WHOLE && a.cols > 1) {
    const int cut = a.longer * a.by_longer.d;
    if (q < cut) {
      const int c = a.by_longer.by(q);
      q = (q - c * a.by_longer.d) * a.cols + c;
    } else {
      const int c = a.by_least.by(q - cut);
      q = (q - cut - c * a.by_least.d) * a.cols + c + a.longer;
    }
  }
  x.rt = a.nrto - 1 - q;
  return x;
}

// In kWhole a CU has one or two row tiles at a time, so the longest ones decide.  An XCD's row
// tiles are ranked by the keys that they see, the most first, and the second half of those
// that run together the other way round: its longest one shares its CU with its shortest.
// 64 sequences of up to 1000 tokens, 4 heads a key head (8 of them), d 128: 36 to 31 us; 80 of
// them 41 to 38; with more than kMostRanked row tiles an XCD it loses what the order of the
// heads keeps in the L2 (causal prompts, 132 of them: 48 to 50).  Returns this workgroup's tile
// of [t0, t0 + n).
constexpr int kCusXcd = 32, kMostRanked = 128;
template <int W>
__device__ int ranked_tile(const Args& a, Schedule& s, int t0, int n, int in_xcd) {
  const int i = threadIdx.x;
  uint32_t mine = 0;
  if (i < n) {
    const Tile x = tile_of<true>(a, t0 + i);
    const int nq = seq_queries(a, x.b), row0 = x.rt << a.lTRo, rows = a.R * nq;
    int keys = row0 < rows ? seq_tokens(a, x.b) : 0;
    if (a.causal && row0 < rows) {
      const int last = min(row0 + a.TRo, rows) - 1;
      keys = max(min(keys, seq_end(a, x.b) - nq + a.by_R.by(last) + 1), 0);
    }
    mine = static_cast<uint32_t>(ceil_div(keys, kTile)) << 8 | static_cast<uint32_t>(255 - i);
  }
  uint32_t* all = reinterpret_cast<uint32_t*>(s.off);
  if (i < 256) all[i] = mine;
  __syncthreads();
  int rank = 0;
  for (int k = 0; k < n; k += 4) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(all + k);
    rank += (x.x > mine) + (x.y > mine) + (x.z > mine) + (x.w > mine);
  }
  if (i < n) s.len[rank] = t0 + i;
  __syncthreads();
  const int first = min(n, 2 * kCusXcd);
  return s.len[in_xcd < kCusXcd || in_xcd >= first ? in_xcd : first - 1 - (in_xcd - kCusXcd)];
}

// W waves a workgroup: with eight, two workgroups' worth of buffers and waves work on one
// row tile.
template <int D, typename T, bool MANY_SHARED, bool MANY_OWN, int W, Split SPLIT>
__global__ void __launch_bounds__(W * kWave) __attribute__((amdgpu_waves_per_eu(2, 2)))
prefix_attention_kernel(const Args a) {
  static_assert(W == 4 || !(MANY_SHARED || MANY_OWN), "the form of many rows has four waves");
  __shared__ __attribute__((aligned(1024))) char lds[attend_lds<D, W>()];
  __shared__ float2 lds_ml[W * kJoinRows];
  __shared__ Schedule s;
  const int lane = threadIdx.x & 63;
  const int xcd = blockIdx.x & 7, in_xcd = blockIdx.x >> 3, slots_xcd = gridDim.x >> 3;
  // consecutive runs on one XCD, so that row tiles of a head share their keys in its L2
  const int slot = xcd * slots_xcd + in_xcd;
  const int nt = a.Hkv * a.B * a.nrto;
  constexpr bool whole = SPLIT == kWhole, GROUPS = SPLIT == kGroups;
  const int groups = GROUPS ? a.G : 0;
  bool rounds = false;
  int per_head = 1, total = 0;
  float inv_head = 1.f;
  if constexpr (!whole) {
    build_schedule<W, GROUPS>(a, s);
    per_head = uniform(s.off[groups + a.B]);
    total = per_head * a.Hkv;
    inv_head = 1.f / static_cast<float>(per_head);
    if constexpr (GROUPS) {
      if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < a.G; i += W * kWave) a.shared_out[i] = s.sh[i];
    } else {
      rounds = nt >= static_cast<int>(gridDim.x) &&
               uniform(s.most) <= kUneven * static_cast<float>(total) / static_cast<float>(nt);
    }
  }
  // Rounds: row tiles [t, end) of the XCD, slots_xcd at a time.  What remains then, less than
  // one row tile a slot, is kept a row tile a lane (slots_xcd is at most 64): units `per_l`,
  // `upto` with those of the lanes before.
  int t = slot, end = nt, rest = 0, per_l = 0, upto = 0;
  if constexpr (whole) {
    const int n = min(slots_xcd, nt - xcd * slots_xcd);
    if (in_xcd >= n) return;
    if (n > kCusXcd && n <= kMostRanked)
      t = uniform(ranked_tile<W>(a, s, xcd * slots_xcd, n, in_xcd));
  }
  if (rounds) {
    t = static_cast<int>(static_cast<long long>(nt) * xcd / kXcds);
    end = static_cast<int>(static_cast<long long>(nt) * (xcd + 1) / kXcds);
    rest = t + (end - t) / slots_xcd * slots_xcd;
    if (rest + lane < end) {
      const Tile x = tile_of<whole>(a, rest + lane);
      if (x.rt < own_tiles(a, s, x.b)) per_l = row_units(a.co, s.len[x.b]);
    }
    upto = per_l;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(upto, o, 64);
      if (lane >= o) upto += v;
    }
    total = uniform(__shfl(upto, 63, 64));
    t += in_xcd;
  }
  // The run: units [u, stop) of the call or, after the rounds, of the XCD's rest, both ends
  // moved to where row tiles may be cut.
  const int my = rounds ? in_xcd : slot;
  const Runs runs = runs_of(total, rounds ? slots_xcd : gridDim.x);
  int u = 0, stop = 0;
  bool moved = true;  // u
  if (!whole && my < runs.n && total > 0) {
    u = uniform(run_begin(runs, my));
    stop = my + 1 < runs.n ? uniform(run_begin(runs, my + 1)) : total;
    moved = false;
  }
  for (;;) {
    Place p;
    int take = 0, last = 0;  // slots behind this one that hold parts of a row tile begun here
    if (!GROUPS && t < (rounds ? rest : whole ? end : 0)) {
      const Tile x = tile_of<whole>(a, uniform(t));
      p = Place{x.h, x.b, x.rt, 0, row_units(a.co, whole ? 0 : s.len[x.b])};
      take = p.per;
      t = whole ? end : t + slots_xcd;
    } else {
      if (u >= stop) break;
      if (rounds) {
        const int i = uniform(__popcll(__ballot(upto <= u)));
        p.per = __builtin_amdgcn_readlane(per_l, i);
        p.k = u - (__builtin_amdgcn_readlane(upto, i) - p.per);
        const Tile y = tile_of<whole>(a, rest + i);
        p.h = y.h;
        p.seg = y.b;
        p.rt = y.rt;
      } else if constexpr (!whole) {
        p = place_of<GROUPS>(a, s, per_head, inv_head, u);
      }
      const int cost = p.seg < groups ? a.cp : a.co;
      if (!moved) {
        moved = true;
        const int k = cut_at(cost, p.per, p.k);
        u = uniform(u + k - p.k);
        if (k > p.k) continue;  // another row tile
        p.k = k;
      }
      take = uniform(min(stop - u + p.k, p.per));
      if (take < p.per) take = uniform(cut_at(cost, p.per, take));
      take -= p.k;
      if (take == 0) break;  // the next run takes the row tile from its start
      // those whose runs begin inside the row tile
      if (p.k + take < p.per && p.k == 0) last = run_at(runs, u + p.per - kSnap) - my;
      u = p.k + take < p.per ? stop : u + take;
    }
    const int cost = p.seg < groups ? a.cp : a.co;
    Job j;
    int tile;  // the row tile's number in `parts`
    j.h = p.h;
    j.shared = p.seg < groups;
    if (GROUPS && j.shared) {
      j.b0 = p.seg * a.N;
      j.rows = a.N * a.RS;
      j.row0 = p.rt << a.lTRp;
      j.nq = 0;
      j.pos0 = 0;
      j.pos1 = uniform(s.sh[p.seg]);
      int rep = j.b0;  // the group's first sequence with a key
      while (rep + 1 < j.b0 + a.N && s.len[rep] == 0) ++rep;
      j.pages = a.table + static_cast<size_t>(uniform(rep)) * a.max_pages;
      tile = (p.seg * a.Hkv + p.h) * a.nrtp + p.rt;
    } else {
      j.b0 = p.seg - groups;
      const int len = whole ? seq_tokens(a, j.b0) : s.len[j.b0];
      j.nq = uniform(whole ? seq_queries(a, j.b0) : queries_of(a, s, j.b0));
      j.rows = a.R * j.nq;
      j.row0 = p.rt << a.lTRo;
      if (j.row0 >= j.rows) continue;  // a row tile of rows that hold no query
      j.pos0 = GROUPS ? uniform(min(s.sh[group_of(a, j.b0)], len)) : 0;
      j.pos1 = uniform(len);
      j.pages = a.table + static_cast<size_t>(j.b0) * a.max_pages;
      tile = groups * a.Hkv * a.nrtp + (j.b0 * a.Hkv + p.h) * a.nrto + p.rt;
    }
    j.t0 = uniform(max(p.k - cost, 0));
    j.t1 = uniform(whole ? ceil_div(j.pos1, kTile) : max(p.k + take - cost, 0));
    j.whole = take == p.per;
    j.piece = 2 * slot + (p.k > 0 ? 0 : 1);
    if (!whole && p.k == 0 && threadIdx.x == 0)
      a.parts[tile] = make_int2(slot, j.pos1 == j.pos0 ? 0 : last + 1);
    if constexpr (sizeof(T) == 4) {
      attend_f32<D, W>(a, j, lds, lds_ml);
    } else if constexpr (MANY_SHARED == MANY_OWN || !GROUPS) {
      if constexpr (MANY_OWN)
        attend_many<D>(a, j, lds);
      else
        attend_few<D, W>(a, j, lds, lds_ml);
    } else {
      if (j.shared)
        attend_many<D>(a, j, lds);
      else
        attend_few<D, W>(a, j, lds, lds_ml);
    }
  }
}

// Joins the partial rows of every row that has some: those of the shared keys, then those
// of its own, in key order.  Workgroup (x, h, b) takes `chunk` rows of a (sequence, key
// head), in the order of its own segment; PG groups of D / 4 threads share a row, each taking
// every PG-th part, four parts' loads at a time, and their sums are joined in group order.
// Latency-bound: lengths and parts, then the rows (64 samples of 32 heads with 18 parts each
// 6.4 us; 10.7 MB of them).
constexpr int kCombineThreads = 256;
template <int D, typename T, int PG>
__global__ void __launch_bounds__(kCombineThreads)
prefix_combine_kernel(const Args a, int chunk) {
  constexpr int TPR = D / 4, RA = kCombineThreads / (TPR * PG);  // rows at once
  __shared__ f32x4 sum_num[PG > 1 ? kCombineThreads : 1];
  __shared__ float2 sum_ml[PG > 1 ? RA * PG : 1];
  const int tid = threadIdx.x;
  const int c4 = tid % TPR, pg = tid / TPR % PG, ra = tid / (TPR * PG);
  const int b = blockIdx.z, h = blockIdx.y, pair = b * a.Hkv + h;
  const int first_row = blockIdx.x * chunk, last_row = min(first_row + chunk, a.RS);
  const int2* own = a.parts + a.G * a.Hkv * a.nrtp + pair * a.nrto;
  // one row tile, and written already unless it is cut
  if (a.G == 0 && chunk <= a.TRo && own[first_row >> a.lTRo].y <= 1) return;
  // Three loads, pinned so that none waits for another; shared_out has any int without groups.
  const int g = a.G > 0 ? group_of(a, b) : 0;
  int q_raw = (a.q_len != nullptr ? a.q_len : a.seq_len)[b], len = a.seq_len[b];
  int taken = a.shared_out[g];
  asm("" : "+s"(q_raw), "+s"(len), "+s"(taken));
  const bool shared = a.G > 0 && len > 0 && taken > 0;
  const int own_rows = a.R * (a.q_len != nullptr ? min(max(q_raw, 0), a.S) : a.S);
  // What a part chooses between, pinned: the compiler would choose between the arguments'
  // addresses and load the chosen one for each part, a latency of its own.
  ptrdiff_t piece = a.piece - a.full, piece_ml = a.piece_ml - a.full_ml;
  int mask_shared = a.TRp - 1, mask_own = a.TRo - 1;
  asm("" : "+s"(piece), "+s"(piece_ml), "+s"(mask_shared), "+s"(mask_own));
  const size_t rows = static_cast<size_t>(a.B) * a.Hkv * a.RS;
  for (int r0 = first_row; r0 < last_row; r0 += RA) {
    const int at_own = min(r0 + ra, a.RS - 1);
    const bool real = r0 + ra < last_row && at_own < own_rows;
    const int query = a.by_R.by(at_own);
    const int in = (at_own - query * a.R) * a.S + query;
    const size_t row = static_cast<size_t>(pair) * a.RS + in;
    const int2 po = own[at_own >> a.lTRo];
    const int rho = (b - g * a.N) * a.RS + in;  // among the group's rows
    const int2 ps = shared ? a.parts[(g * a.Hkv + h) * a.nrtp + (rho >> a.lTRp)] : make_int2(0, 0);
    const int np = ps.y + po.y;
    const bool mine = real && (a.G > 0 || po.y > 1);  // else it is written already
    const int in_shared = rho & mask_shared, in_own = at_own & mask_own;
    float M = -FLT_MAX, den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    if (mine) {
      auto part = [&](int i, f32x4* x) {
        const bool of_shared = i < ps.y;
        const int2 p = of_shared ? ps : po;
        const int k = of_shared ? i : i - ps.y;  // part k of the row tile
        const bool whole = p.y == 1;
        const size_t place = static_cast<size_t>(2) * (p.x + k) + (k == 0 ? 1 : 0);
        const size_t at = whole ? (of_shared ? 0 : rows) + row
                                : place * a.TR + (of_shared ? in_shared : in_own);
        *x = ldg_f32x4(a.full + (whole ? 0 : piece) + at * D + 4 * c4);
        return a.full_ml[(whole ? 0 : piece_ml) + at];
      };
      for (int i0 = pg; i0 < np; i0 += 4 * PG) {
        f32x4 x[4];
        float2 ml[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) ml[e] = part(min(i0 + e * PG, np - 1), &x[e]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (i0 + e * PG >= np || ml[e].y == 0.f) continue;
          const float m = fmaxf(M, ml[e].x), fa = fast_exp2(M - m), fb = fast_exp2(ml[e].x - m);
          M = m;
          den = fmaf(fb, ml[e].y, fa * den);
#pragma unroll
          for (int w = 0; w < 4; ++w) num[w] = fmaf(fb, x[e][w], fa * num[w]);
        }
      }
    }
    if constexpr (PG > 1) {
      sum_num[tid] = num;
      if (c4 == 0) sum_ml[ra * PG + pg] = make_float2(M, den);
      __syncthreads();
      if (pg == 0) {
#pragma unroll
        for (int w = 1; w < PG; ++w) {
          const float2 ml = sum_ml[ra * PG + w];
          if (ml.y == 0.f) continue;
          const f32x4 x = sum_num[tid + w * TPR];
          const float m = fmaxf(M, ml.x), fa = fast_exp2(M - m), fb = fast_exp2(ml.x - m);
          M = m;
          den = fmaf(fb, ml.y, fa * den);
#pragma unroll
          for (int e = 0; e < 4; ++e) num[e] = fmaf(fb, x[e], fa * num[e]);
        }
      }
      __syncthreads();
    }
    if (mine && pg == 0) store_row<D, T>(a, row, c4, num, M, den);
  }
}

// How a call is cut up, by its row tiles and by the keys that a table row has room for: the
// lengths are on the device, so a table wider than its sequences is cut up as for longer ones
// (6 causal prompts of up to 701 queries, d 64: whole row tiles, 28 us, or with a table four
// times as wide runs, 36; 4 x 1 token over 316, 8 heads: 11, and 13 sixteen times as wide).
// Every row tile whole, in a workgroup of its own, saves finding the runs and the joining
// kernel (some 5 us); a workgroup of eight waves reads one row tile's keys at up to twice the
// rate of one of four, where there is a CU for each.  Row tiles of few rows, sequences of 1 to
// n tokens, and of n each (us: whole with 4 waves, runs with 4, whole with 8, runs with 8):
//   bf16, d 128,  24 row tiles, 1-2000    18  20  14  17        1-4000   36  21  28  19
//                160            1-2000    22  26  21  25          4000   59  70  67  69
//                272            1-2000    31  37  33  36          4000  144 111 141 110
//                384            1-4000    78  87  78  82          4000  150 151 153 147
//                512            1-4000    95 110 106 104          8000  345 352 348 353
//                576            1-4000   105 122 116 116          8000  433 401 446 398
//   bf16, d 64,  160            1-4000    30  25  21  26          4000   40  37  32  38
//                512            1-4000    52  60  57  60          4000   92  97  95  98
//   fp32, d 128,  24            1-1000    24  28  23  21        1-4000   81  30  74  24
//                192            1-1500    38           39          1500   55           69
//                272            1-2000    64  69  64  66          2000  129 114 134 115
//                512            1-4000   182 199 195 193          4000  350 354 349 354
struct Plan {
  Split split;
  int waves;
};
Plan plan_of(const Args& a, const PrefixCall& p, bool bf16, int d) {
  const bool many_own = a.TRo == kManyRows, many = many_own || (a.G > 0 && a.TRp == kManyRows);
  const long long tiles = static_cast<long long>(a.Hkv) * a.B * a.nrto;
  const long long keys = static_cast<long long>(p.max_pages) * p.page;
  const int row = d * (bf16 ? 2 : 4);
  bool whole;
  if (a.G > 0) {
    // reading shared tokens for each sequence: only for so few keys that the caches make up
    // for it.  8 key heads, whole against shared: 64 sequences of 960 + up to 900 tokens at
    // d 128 32 against 44 us, of 1920 + up to 900 42 against 46, of 3840 + up to 64 45 against
    // 29; with 24 key heads, d 64, 448 + up to 400 29 against 38, 960 + up to 900 64 against 55.
    // fp32, one token, 8 key heads, d 64: 16 sequences of 960 + up to 64 14.5 against 15.3, of
    // 1920 + up to 64 23 against 15.5 (18 in four waves); 64 of 448 + up to 64 16.0 against
    // 18.8, of 960 + up to 64 25 against 19; d 128: 16 of 448 + up to 64 14.5 against 18.2, of
    // 960 + up to 64 24.5 against 20.7.
    whole = bf16 ? keys <= 2048 && tiles * keys * d <= 1 << 27
                 : keys * d <= 1 << 17 && tiles * keys * d <= 1 << 25;
  } else if (many_own) {
    // 2048 queries at d 128, whole against runs (us): a workgroup that is alone on its CU goes
    // through its keys at half the card's rate, one of several rounds waits for the longest of
    // each, and runs cost some 20 us of their own and read a head's keys at different places.
    //   row tiles             128        256        384        640
    //   2048 keys           36   43    42   59    60   79   104  105
    //   4096                65   56    75   87   106  120   195  177
    //   8192               123   84   140  143   200  206   385  318
    //   causal, 4096        67   52    73   82    93  110   148  160
    //   causal, 8192       124   79   139  138   187  198   332  300
    // and 16 to 64 row tiles of 256 rows 28 to 29 against 30 to 35 with 1500 keys, 34 to 36
    // against 30 to 36 with 2000.
    whole = keys <= 1536 || (tiles >= kPrefixSlots / 4 && keys <= 2048) ||
            (tiles >= kPrefixSlots / 2 && (p.causal ? keys <= 4096 || keys <= 2ll * p.S
                                                    : keys <= 4096 && tiles <= kPrefixSlots));
  } else if (tiles <= kPrefixSlots / 2) {
    whole = !bf16 ? keys * d <= 1 << 16 || (tiles >= kPrefixSlots / 4 && keys <= 1024) ||
                        (tiles >= 192 && keys <= 1536)
                  : keys <= 2048 || (row < 256 && tiles >= kPrefixSlots / 4 && keys <= 4096);
  } else {  // the nearer they come to a row tile a slot, the better
    whole = keys <= (tiles >= 384 ? 4096 : bf16 ? 2048 : 1536) ||
            (tiles >= 448 && tiles <= kPrefixSlots && keys <= 8192);
  }
  // With eight times as many row tiles as slots these even out by themselves, if no sequence is
  // much longer than the others: the longest row tile is one workgroup.  512 sequences of 8
  // heads, d 128, whole against runs: 1000 tokens each 360 and 370 us, 1 to 2000 367 and 375, one
  // of 20000 478 and 389, one of 100000 1294 and 445; 4 x 16384 queries, 8 heads, d 64, 16384
  // keys 2273 and 2279, causal 1171 and 1233; 64 x 1024 queries, 8 heads, d 128, 1024 to 4096
  // keys 1187 and 1118, causal 1005 and 950.
  whole = whole || (a.G == 0 && tiles >= 8 * kPrefixSlots);
  // Workgroups without 128-row tiles have eight waves: whole row tiles up to half the CUs (all
  // with short rows), runs but for many row tiles of short rows or few keys.  Four waves against
  // eight, us, sequences of 1 to n tokens:
  //   whole, n = 1000 (fp32 500)      row tiles   64        128       256       320
  //     bf16, d 128                           13.3 12.5  13.7 13.1  16.1 16.7  19.8 21.8
  //     bf16, d 64                             9.6  9.6  11.2  9.5  11.8 10.5  13.2 14.8
  //     fp32, d 128                           15.0 15.7  15.4 16.3  17.6 19.0  21.5 22.3
  //     fp32, d 64                             9.6  9.6  10.2 10.2  11.1 11.8  13.0 15.7
  //   runs, n = 4000 (fp32 2000)      row tiles   48        96        128       512
  //     bf16, d 128                           22.5 20.1  29.0 28.9  36.7 36.2   106  102
  //     bf16, d 64                            17.6 15.8  19.4 19.0  20.9 21.4    59   58
  //     fp32, d 128                           29.0 22.4  32.2 28.8  38.0 37.8   109  107
  //     fp32, d 64                            19.3 16.5  20.5 19.5  21.7 21.5    59   59
  const bool few = !many || (whole && !many_own);
  const bool eight =
      few && (whole ? tiles * row <= 1 << 15
                    : tiles <= 64 || (row >= 256 && (tiles <= kPrefixSlots / 2 || keys > 1024)));
  return {whole ? kWhole : a.G > 0 ? kGroups : kRuns, eight ? 8 : 4};
}

}  // namespace

void launch_prefix_attention(const PrefixCall& p, int dtype, int d, char* ws, hipStream_t s) {
  const PrefixWs w = prefix_ws_layout(p.B, p.Hq, p.Hkv, p.S, d, dtype, p.n_groups);
  Args a{};
  a.q = p.q;
  a.kp = p.k_pages;
  a.vp = p.v_pages;
  a.o = p.o;
  a.lse = p.lse;
  a.table = p.page_table;
  a.seq_len = p.seq_len;
  a.shared_len = p.shared_len;
  a.q_len = p.q_len;
  a.B = p.B;
  a.G = w.groups;
  a.N = w.groups > 0 ? p.B / w.groups : 0;
  a.Hkv = p.Hkv;
  a.R = p.Hq / p.Hkv;
  a.S = p.S;
  a.RS = a.R * p.S;
  a.by_N = divisor(a.N > 0 ? a.N : 1);
  a.by_S = divisor(a.S);
  a.by_R = divisor(a.R);
  a.by_RS = divisor(a.RS);
  a.n_pages = p.n_pages;
  a.lp = __builtin_ctz(static_cast<unsigned>(p.page));
  a.max_pages = p.max_pages;
  a.causal = p.causal;
  a.TRp = w.shared_rows;
  a.TRo = w.own_rows;
  a.lTRp = __builtin_ctz(static_cast<unsigned>(a.TRp));
  a.lTRo = __builtin_ctz(static_cast<unsigned>(a.TRo));
  a.TR = w.piece_rows;
  const auto cost = [&](int rows) { return rows == kManyRows ? 4 : 6; };
  a.cp = cost(a.TRp);
  a.co = cost(a.TRo);
  a.c = log2_scale(p.scale);
  a.shared_out = reinterpret_cast<int*>(ws + w.shared);
  a.parts = reinterpret_cast<int2*>(ws + w.parts);
  a.nrtp = w.groups > 0 ? ceil_div(a.N * a.RS, a.TRp) : 0;
  a.nrto = ceil_div(a.RS, a.TRo);
  a.by_B = divisor(a.B);
  a.by_tiles = divisor(a.B * a.nrto);
  a.full = reinterpret_cast<float*>(ws + w.full);
  a.full_ml = reinterpret_cast<float2*>(ws + w.full_ml);
  a.piece = reinterpret_cast<float*>(ws + w.piece);
  a.piece_ml = reinterpret_cast<float2*>(ws + w.piece_ml);
  // threads that share a row in the joining kernel: eight times as many where a row tile may
  // be cut into 16 parts and more
  const long tiles = a.G > 0 ? static_cast<long>(a.G) * a.Hkv * a.nrtp
                             : static_cast<long>(a.B) * a.Hkv * a.nrto;
  const bool share = kPrefixSlots / tiles >= 16;
  const int at_once = kCombineThreads / (d / 4) / (share ? 8 : 1);
  const int chunk = a.G == 0 && !share ? (a.TRo < 32 ? a.TRo : 32) : at_once;
  const dim3 cgrid(ceil_div(a.RS, chunk), a.Hkv, a.B);
  const Plan plan = plan_of(a, p, dtype == 0, d);
  const Split split = plan.split;
  const bool wide = plan.waves == 8;
  if (split != kGroups) a.G = 0;  // the joining kernel looks for what the split left
  a.cols = split == kWhole && a.Hkv < kXcds ? ceil_div(kXcds, a.Hkv) : 1;
  a.longer = a.nrto % a.cols;
  a.by_longer = divisor(a.nrto / a.cols + 1);
  a.by_least = divisor(a.nrto >= a.cols ? a.nrto / a.cols : 1);
  const int slots = wide ? kPrefixSlots / 2 : kPrefixSlots;
  const int wgs = split == kWhole ? kXcds * ceil_div(a.Hkv * a.B * a.nrto, kXcds) : slots;
#define SA_PREFIX(D, T, P, O, W)                                                              \
  do {                                                                                        \
    if (split == kWhole) {                                                                    \
      hipLaunchKernelGGL((prefix_attention_kernel<D, T, O, O, W, kWhole>), dim3(wgs),         \
                         dim3(W * kWave), 0, s, a);                                           \
      break;                                                                                  \
    }                                                                                         \
    if (split == kRuns)                                                                       \
      hipLaunchKernelGGL((prefix_attention_kernel<D, T, O, O, W, kRuns>), dim3(wgs),          \
                         dim3(W * kWave), 0, s, a);                                           \
    else                                                                                      \
      hipLaunchKernelGGL((prefix_attention_kernel<D, T, P, O, W, kGroups>), dim3(wgs),        \
                         dim3(W * kWave), 0, s, a);                                           \
    if (share)                                                                                \
      hipLaunchKernelGGL((prefix_combine_kernel<D, T, 8>), cgrid, dim3(kCombineThreads), 0, s, \
                         a, chunk);                                                           \
    else                                                                                      \
      hipLaunchKernelGGL((prefix_combine_kernel<D, T, 1>), cgrid, dim3(kCombineThreads), 0, s, \
                         a, chunk);                                                           \
  } while (0)
#define SA_PREFIX_D(D)                          \
  do {                                          \
    if (dtype != 0 && wide)                     \
      SA_PREFIX(D, float, false, false, 8);     \
    else if (dtype != 0)                        \
      SA_PREFIX(D, float, false, false, 4);     \
    else if (wide)                              \
      SA_PREFIX(D, uint16_t, false, false, 8);  \
    else if (a.TRo == kManyRows)                \
      SA_PREFIX(D, uint16_t, true, true, 4);    \
    else if (a.TRp == kManyRows)                \
      SA_PREFIX(D, uint16_t, true, false, 4);   \
    else                                        \
      SA_PREFIX(D, uint16_t, false, false, 4);  \
  } while (0)
  if (d == 128)
    SA_PREFIX_D(128);
  else
    SA_PREFIX_D(64);
#undef SA_PREFIX_D
#undef SA_PREFIX
}

}  // namespace sa
