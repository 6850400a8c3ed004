// C entry points of the paged keys and values: argument validation, workspace sizing
// and dispatch, as in sa_api.hip.
#include <math.h>

#include "../../include/sa.h"
#include "sa_checks.h"
#include "sa_device.h"
#include "sa_internal.h"

using namespace sa::host;

namespace {

constexpr long long kMaxCapacity = 1ll << 30;  // tokens of a sequence: positions in 32 bits

bool page_size(int page) { return page == 16 || page == 32 || page == 64 || page == 128; }

// Sizes that describe a cache.
int check_cache(const char* fn, int B, int max_pages, int n_pages, int page, int most) {
  if (B < 1 || max_pages < 1 || n_pages < 1)
    return fail(SA_ERR_INVALID_ARG, "%s: B=%d max_pages=%d n_pages=%d must all be >= 1", fn, B,
                max_pages, n_pages);
  if (B > most)
    return fail(SA_ERR_UNSUPPORTED, "%s: B=%d exceeds %d", fn, B, most);
  if (!page_size(page))
    return fail(SA_ERR_UNSUPPORTED, "%s: page=%d not in {16, 32, 64, 128}", fn, page);
  if (static_cast<long long>(max_pages) * page > kMaxCapacity)
    return fail(SA_ERR_UNSUPPORTED, "%s: max_pages=%d pages of %d tokens exceed %lld tokens", fn,
                max_pages, page, kMaxCapacity);
  return SA_OK;
}

// The planning kernels go through the owner counts in steps of 16384 pages, in 32 bits.
constexpr int kMaxPages = 1 << 30;

int check_table(const char* fn, const int32_t* page_table, const int32_t* page_ref,
                int n_pages) {
  if (n_pages > kMaxPages)
    return fail(SA_ERR_UNSUPPORTED, "%s: n_pages=%d exceeds %d", fn, n_pages, kMaxPages);
  SA_TRY(check_tensor(fn, "page_table", page_table, true, 4));
  SA_TRY(check_tensor(fn, "page_ref", page_ref, true, 4));
  return SA_OK;
}

// Head, row and type checks of the calls that read or write K and V.
int check_rows(const char* fn, int H, int S, int d, int dtype) {
  if (H < 1 || S < 1) return fail(SA_ERR_INVALID_ARG, "%s: H=%d S=%d must be >= 1", fn, H, S);
  if (S > sa::kMaxTokens)
    return fail(SA_ERR_UNSUPPORTED, "%s: S=%d exceeds %d", fn, S, sa::kMaxTokens);
  if (dtype != SA_BF16 && dtype != SA_F32)
    return fail(SA_ERR_UNSUPPORTED, "%s: dtype %d is neither SA_BF16 nor SA_F32", fn, dtype);
  if (d != 64 && d != 128)
    return fail(SA_ERR_UNSUPPORTED, "%s: head dim d=%d not in {64, 128}", fn, d);
  return SA_OK;
}

constexpr long long kMaxRows = 0x7fffffff;

bool prefix_sizes_ok(int B, int Hq, int Hkv, int S, int d, int dtype, int n_groups) {
  return B >= 1 && Hkv >= 1 && Hq >= Hkv && Hq % Hkv == 0 && S >= 1 && S <= sa::kMaxTokens &&
         (d == 64 || d == 128) && (dtype == SA_BF16 || dtype == SA_F32) && n_groups >= 0 &&
         n_groups <= B && (n_groups == 0 || B % n_groups == 0) &&
         static_cast<long long>(B) + n_groups <= sa::kMaxAttendSegs &&
         static_cast<long long>(B) * Hkv <= sa::kMaxPairs &&
         static_cast<long long>(B) * Hq <= kMaxRows / S;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y ? na > y - x : nb > x - y;  // an end may lie behind the last address
}

// Bytes of a pool; Hkv and n_pages may be any ints.
int pool_bytes(const char* fn, int n_pages, int Hkv, int page, size_t row_bytes, size_t* bytes) {
  const size_t heads = static_cast<size_t>(n_pages) * Hkv;  // below 2^62
  if (__builtin_mul_overflow(heads, page * row_bytes, bytes))
    return fail(SA_ERR_UNSUPPORTED, "%s: n_pages=%d pages of Hkv=%d heads are too large", fn,
                n_pages, Hkv);
  return SA_OK;
}

}  // namespace

extern "C" {

int sa_pages_reserve(int32_t* page_table, int32_t* seq_len, int32_t* page_ref,
                     const int32_t* n_new, int B, int max_pages, int n_pages, int page,
                     int32_t* missing, void* stream) {
  const char* fn = "sa_pages_reserve";
  SA_TRY(check_cache(fn, B, max_pages, n_pages, page, sa::kMaxSequences));
  SA_TRY(check_table(fn, page_table, page_ref, n_pages));
  SA_TRY(check_tensor(fn, "seq_len", seq_len, true, 4));
  SA_TRY(check_tensor(fn, "n_new", n_new, true, 4));
  SA_TRY(check_tensor(fn, "missing", missing, true, 4));
  sa::launch_pages_reserve(page_table, seq_len, page_ref, n_new, B, max_pages, n_pages, page,
                           missing, static_cast<hipStream_t>(stream));
  return check_launch(fn);
}

int sa_pages_write(const void* k, const void* v, void* k_pages, void* v_pages,
                   const int32_t* page_table, const int32_t* seq_len, const int32_t* n_new,
                   const int32_t* missing, int B, int Hkv, int S, int d, int dtype, int n_pages,
                   int page, int max_pages, void* stream) {
  const char* fn = "sa_pages_write";
  SA_TRY(check_cache(fn, B, max_pages, n_pages, page, sa::kMaxSequences));
  SA_TRY(check_rows(fn, Hkv, S, d, dtype));
  if (static_cast<long long>(B) * Hkv > kMaxRows / S)
    return fail(SA_ERR_UNSUPPORTED, "%s: B=%d Hkv=%d S=%d is too large", fn, B, Hkv, S);
  SA_TRY(check_tensor(fn, "k", k, true, 16));
  SA_TRY(check_tensor(fn, "v", v, true, 16));
  SA_TRY(check_tensor(fn, "k_pages", k_pages, true, 16));
  SA_TRY(check_tensor(fn, "v_pages", v_pages, true, 16));
  SA_TRY(check_tensor(fn, "page_table", page_table, true, 4));
  SA_TRY(check_tensor(fn, "seq_len", seq_len, true, 4));
  SA_TRY(check_tensor(fn, "n_new", n_new, false, 4));
  SA_TRY(check_tensor(fn, "missing", missing, false, 4));
  const int row_bytes = d * (dtype == SA_BF16 ? 2 : 4);
  const size_t rows = static_cast<size_t>(B) * Hkv * S * row_bytes;
  size_t pool;
  SA_TRY(pool_bytes(fn, n_pages, Hkv, page, row_bytes, &pool));
  if (overlap(k_pages, pool, v_pages, pool))
    return fail(SA_ERR_INVALID_ARG, "%s: k_pages and v_pages overlap", fn);
  if (overlap(k, rows, k_pages, pool) || overlap(v, rows, k_pages, pool) ||
      overlap(k, rows, v_pages, pool) || overlap(v, rows, v_pages, pool))
    return fail(SA_ERR_INVALID_ARG, "%s: k or v overlaps the pages", fn);
  sa::launch_pages_write(k, v, k_pages, v_pages, page_table, seq_len, n_new, missing, B, Hkv, S,
                         row_bytes, max_pages, n_pages, page, static_cast<hipStream_t>(stream));
  return check_launch(fn);
}

int sa_pages_fork(int32_t* page_table, int32_t* seq_len, int32_t* page_ref, const int32_t* src,
                  const int32_t* dst, int n, int B, int max_pages, int n_pages, int page,
                  int32_t* copy_src, int32_t* copy_dst, int32_t* missing, void* stream) {
  const char* fn = "sa_pages_fork";
  SA_TRY(check_cache(fn, B, max_pages, n_pages, page, sa::kMaxSequences));
  if (n < 1 || n > B)
    return fail(SA_ERR_INVALID_ARG, "%s: n=%d outside [1, B=%d]", fn, n, B);
  SA_TRY(check_table(fn, page_table, page_ref, n_pages));
  SA_TRY(check_tensor(fn, "seq_len", seq_len, true, 4));
  SA_TRY(check_tensor(fn, "src", src, true, 4));
  SA_TRY(check_tensor(fn, "dst", dst, true, 4));
  SA_TRY(check_tensor(fn, "copy_src", copy_src, true, 4));
  SA_TRY(check_tensor(fn, "copy_dst", copy_dst, true, 4));
  SA_TRY(check_tensor(fn, "missing", missing, true, 4));
  sa::launch_pages_fork(page_table, seq_len, page_ref, src, dst, n, B, max_pages, n_pages, page,
                        copy_src, copy_dst, missing, static_cast<hipStream_t>(stream));
  return check_launch(fn);
}

int sa_pages_free(int32_t* page_table, int32_t* seq_len, int32_t* page_ref, const int32_t* seqs,
                  int n, int B, int max_pages, int n_pages, int page, void* stream) {
  const char* fn = "sa_pages_free";
  SA_TRY(check_cache(fn, B, max_pages, n_pages, page, sa::kMaxSequences));
  if (n < 1 || n > sa::kMaxSequences)
    return fail(SA_ERR_INVALID_ARG, "%s: n=%d outside [1, %d]", fn, n, sa::kMaxSequences);
  SA_TRY(check_table(fn, page_table, page_ref, n_pages));
  SA_TRY(check_tensor(fn, "seq_len", seq_len, true, 4));
  SA_TRY(check_tensor(fn, "seqs", seqs, true, 4));
  sa::launch_pages_free(page_table, seq_len, page_ref, seqs, n, B, max_pages, n_pages, page,
                        static_cast<hipStream_t>(stream));
  return check_launch(fn);
}

int sa_pages_compact(int32_t* page_table, int32_t* page_ref, int B, int max_pages, int n_pages,
                     int32_t* move_src, int32_t* move_dst, int32_t* counts, void* stream) {
  const char* fn = "sa_pages_compact";
  SA_TRY(check_cache(fn, B, max_pages, n_pages, 16, sa::kMaxSequences));  // reads no tokens
  SA_TRY(check_table(fn, page_table, page_ref, n_pages));
  SA_TRY(check_tensor(fn, "move_src", move_src, n_pages > 1, 4));
  SA_TRY(check_tensor(fn, "move_dst", move_dst, n_pages > 1, 4));
  SA_TRY(check_tensor(fn, "counts", counts, true, 4));
  sa::launch_pages_compact(page_table, page_ref, B, max_pages, n_pages, move_src, move_dst, counts,
                           static_cast<hipStream_t>(stream));
  return check_launch(fn);
}

int sa_pages_copy(void* pools, int n_pools, int n_pages, size_t page_bytes, const int32_t* src,
                  const int32_t* dst, int n, void* stream) {
  const char* fn = "sa_pages_copy";
  if (n_pools < 1 || n_pages < 1)
    return fail(SA_ERR_INVALID_ARG, "%s: n_pools=%d n_pages=%d must be >= 1", fn, n_pools,
                n_pages);
  if (page_bytes < 16 || page_bytes % 16 != 0 || page_bytes > 1ull << 31)
    return fail(SA_ERR_INVALID_ARG, "%s: page_bytes=%zu must be a multiple of 16 from 16 to 2^31",
                fn, page_bytes);
  if (n < 0) return fail(SA_ERR_INVALID_ARG, "%s: n=%d must be >= 0", fn, n);
  SA_TRY(check_tensor(fn, "pools", pools, true, 16));
  SA_TRY(check_tensor(fn, "src", src, n > 0, 4));
  SA_TRY(check_tensor(fn, "dst", dst, n > 0, 4));
  if (n == 0) return ok();
  sa::launch_pages_copy(pools, n_pools, n_pages, page_bytes, src, dst, n,
                        static_cast<hipStream_t>(stream));
  return check_launch(fn);
}

size_t sa_prefix_attention_workspace(int B, int Hq, int Hkv, int S, int d, int dtype,
                                     int n_groups) {
  if (!prefix_sizes_ok(B, Hq, Hkv, S, d, dtype, n_groups)) return 0;
  return sa::prefix_ws_layout(B, Hq, Hkv, S, d, dtype, n_groups).total;
}

int sa_prefix_attention(const void* q, const void* k_pages, const void* v_pages, void* o,
                        float* lse, const int32_t* page_table, const int32_t* seq_len,
                        const int32_t* shared_len, const int32_t* q_len, int B, int Hq, int Hkv,
                        int S, int d, int dtype, float scale, int causal, int n_groups,
                        int n_pages, int page, int max_pages, void* ws, size_t ws_bytes,
                        void* stream) {
  const char* fn = "sa_prefix_attention";
  SA_TRY(check_cache(fn, B, max_pages, n_pages, page, sa::kMaxAttendSegs));
  SA_TRY(check_rows(fn, Hkv, S, d, dtype));
  if (Hq < Hkv || Hq % Hkv != 0)
    return fail(SA_ERR_INVALID_ARG, "%s: Hq=%d is no multiple of Hkv=%d", fn, Hq, Hkv);
  if (n_groups < 0 || n_groups > B || (n_groups > 0 && B % n_groups != 0))
    return fail(SA_ERR_INVALID_ARG, "%s: n_groups=%d does not divide B=%d", fn, n_groups, B);
  if ((shared_len != nullptr) != (n_groups > 0))
    return fail(SA_ERR_INVALID_ARG, "%s: shared_len must be NULL iff n_groups=%d is 0", fn,
                n_groups);
  if (B + n_groups > sa::kMaxAttendSegs)
    return fail(SA_ERR_UNSUPPORTED, "%s: B + n_groups = %d exceeds %d", fn, B + n_groups,
                sa::kMaxAttendSegs);
  if (static_cast<long long>(B) * Hq > kMaxRows / S)
    return fail(SA_ERR_UNSUPPORTED, "%s: B=%d Hq=%d S=%d is too large", fn, B, Hq, S);
  if (static_cast<long long>(B) * Hkv > sa::kMaxPairs)
    return fail(SA_ERR_UNSUPPORTED, "%s: B*Hkv=%lld exceeds %d", fn,
                static_cast<long long>(B) * Hkv, sa::kMaxPairs);
  if (sa::prefix_units(B, Hq, Hkv, S, d, dtype, n_groups,
                       static_cast<long long>(max_pages) * page) > 0x3fffffff)
    return fail(SA_ERR_UNSUPPORTED,
                "%s: B=%d Hq=%d S=%d over up to %lld tokens each is too large for one call", fn, B,
                Hq, S, static_cast<long long>(max_pages) * page);
  if (causal != 0 && causal != 1)
    return fail(SA_ERR_INVALID_ARG, "%s: causal=%d must be 0 or 1", fn, causal);
  if (!(scale > 0.f) || !isfinite(scale))
    return fail(SA_ERR_INVALID_ARG, "%s: scale=%g must be finite and > 0", fn,
                static_cast<double>(scale));
  SA_TRY(check_tensor(fn, "q", q, true, 16));
  SA_TRY(check_tensor(fn, "k_pages", k_pages, true, 16));
  SA_TRY(check_tensor(fn, "v_pages", v_pages, true, 16));
  SA_TRY(check_tensor(fn, "o", o, true, 16));
  SA_TRY(check_tensor(fn, "lse", lse, false, 4));
  SA_TRY(check_tensor(fn, "page_table", page_table, true, 4));
  SA_TRY(check_tensor(fn, "seq_len", seq_len, true, 4));
  SA_TRY(check_tensor(fn, "q_len", q_len, false, 4));
  const size_t e = dtype == SA_BF16 ? 2 : 4;
  const size_t rows = static_cast<size_t>(B) * Hq * S * d * e;
  size_t pool;
  SA_TRY(pool_bytes(fn, n_pages, Hkv, page, d * e, &pool));
  if (overlap(o, rows, q, rows) || overlap(o, rows, k_pages, pool) ||
      overlap(o, rows, v_pages, pool))
    return fail(SA_ERR_INVALID_ARG, "%s: o overlaps an input", fn);
  SA_TRY(check_ws(fn, ws, ws_bytes,
                  sa::prefix_ws_layout(B, Hq, Hkv, S, d, dtype, n_groups).total));
  const sa::PrefixCall p{q, k_pages, v_pages, o, lse, page_table, seq_len, shared_len, q_len,
                         B, Hq, Hkv, S, n_groups, n_pages, page, max_pages, causal, scale};
  sa::launch_prefix_attention(p, dtype, d, static_cast<char*>(ws),
                              static_cast<hipStream_t>(stream));
  return check_launch(fn);
}

}  // extern "C"
