// twk_cache_api.cu -- the C ABI of the operators around the pass (declared in include/twinkv.h):
// argument checks and launches of the norms with rotation, of the 4-bit pages and of the attention
// over them.
#include <cmath>

#include "twinkv.h"
#include "twk_cache.cuh"
#include "twk_cache_internal.h"

using namespace twk;

namespace {

constexpr int64_t kMaxUnits = 65535;   // units run on grid.y
constexpr int64_t kMaxRows = 1 << 20;  // positions of a unit, as for the audit
constexpr int kMaxAppend = kPage;
constexpr int kMaxTokens = 64;         // query tokens of an attention call

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

bool dim_ok(int d) { return d == 64 || d == 128; }

int page_bytes(int d) { return d == 128 ? PageLayout<128>::kBytes : PageLayout<64>::kBytes; }

// strides in elements that keep every row on a 16-byte boundary
template <typename... S>
bool rows_aligned(bool f32, S... strides)
{
    const int64_t step = f32 ? 4 : 8;
    return (... && (strides % step == 0));
}

bool pool_ok(const twinkv_pool& p)
{
    return dim_ok(p.d) && p.pages && aligned16(p.pages) && p.n_pages >= 1;
}

bool table_ok(const int32_t* table, int32_t max_pages)
{
    return table && aligned4(table) && max_pages >= 1 && max_pages <= kMaxRows / kPage;
}

Pages pages_of(const twinkv_pool& pool, const int32_t* table, int32_t max_pages)
{
    return {static_cast<uint8_t*>(pool.pages), pool.n_pages, table, max_pages};
}

twinkv_status check_ws(void* ws, size_t bytes, size_t need)
{
    if (need == 0) return TWINKV_ERR_INVALID_ARG;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) != 0 || bytes < need)
        return TWINKV_ERR_WORKSPACE;
    return TWINKV_OK;
}

// 0 where the sizes are beyond the call's limits.  Pages are counted in 32 bits: 65535 row parts of
// 16384 pages are fewer than 2^31.
size_t attend_bytes(const twinkv_queries& s, int d)
{
    if (!dim_ok(d) || s.B < 1 || s.H < 1 || s.Hq < 1 || s.n < 1 || s.Hq % s.H != 0) return 0;
    if (s.n > kMaxTokens || s.Hq / s.H > 256) return 0;
    const int64_t units = static_cast<int64_t>(s.B) * s.H;
    if (units > kMaxUnits) return 0;
    const int rows = s.Hq / s.H * s.n;
    if (units * ((rows + 15) / 16) > kMaxUnits) return 0;
    return attend_workspace(static_cast<int>(units), rows, s.n, d);
}

}  // namespace

extern "C" {

size_t twinkv_cache_page_bytes(int32_t d) { return dim_ok(d) ? page_bytes(d) : 0; }

size_t twinkv_cache_move_workspace(int32_t units, int32_t N)
{
    if (units < 1 || units > kMaxUnits || N < 1 || N > kMaxRows) return 0;
    return up256(static_cast<size_t>(units) * N * 4);
}

size_t twinkv_cache_attend_workspace(twinkv_queries s, int32_t d)
{
    return attend_bytes(s, d);
}

twinkv_status twinkv_qk_norm_rope(const void* q, const void* k, twinkv_heads s, const void* wq,
                                  const void* wk, float eps, const float* cos_sin,
                                  const int32_t* positions, void* out_q, void* out_k,
                                  int32_t* out_status, void* stream)
{
    if (s.tokens < 1 || s.heads_q < 0 || s.heads_k < 0 || s.heads_q + s.heads_k < 1 ||
        s.heads_q > 65535 || s.heads_k > 65535 || s.rows < 1 || !dim_ok(s.d) ||
        (s.dtype != TWINKV_BF16 && s.dtype != TWINKV_F32))
        return TWINKV_ERR_INVALID_ARG;
    if (!std::isfinite(eps) || eps < 0.0f) return TWINKV_ERR_INVALID_ARG;
    if ((s.heads_q > 0 && (!q || !out_q)) || (s.heads_k > 0 && (!k || !out_k)))
        return TWINKV_ERR_INVALID_ARG;
    if (!cos_sin || !positions || !aligned4(positions) || !aligned4(out_status))
        return TWINKV_ERR_INVALID_ARG;
    const bool f32 = s.dtype == TWINKV_F32;
    if (!aligned16(q) || !aligned16(k) || !aligned16(wq) || !aligned16(wk) ||
        !aligned16(cos_sin) || !aligned16(out_q) || !aligned16(out_k) ||
        !rows_aligned(f32, s.q_token, s.q_head, s.k_token, s.k_head, s.out_q_token, s.out_q_head,
                      s.out_k_token, s.out_k_head))
        return TWINKV_ERR_INVALID_ARG;
    int sms = 0;
    const twinkv_status r = device_facts(&sms);
    if (r != TWINKV_OK) return r;
    RopeArgs a{};
    a.q = q;
    a.k = k;
    a.q_token = s.q_token;
    a.q_head = s.q_head;
    a.k_token = s.k_token;
    a.k_head = s.k_head;
    a.out_q = out_q;
    a.out_k = out_k;
    a.oq_token = s.out_q_token;
    a.oq_head = s.out_q_head;
    a.ok_token = s.out_k_token;
    a.ok_head = s.out_k_head;
    a.wq = wq;
    a.wk = wk;
    a.cos_sin = cos_sin;
    a.positions = positions;
    a.out_status = out_status;
    a.tokens = s.tokens;
    a.heads_q = s.heads_q;
    a.heads_k = s.heads_k;
    a.d = s.d;
    a.rows = s.rows;
    a.eps = eps;
    return cuda_result(launch_rope(a, f32, sms, static_cast<cudaStream_t>(stream)));
}

twinkv_status twinkv_cache_pack(const void* keys, const void* values, twinkv_shape s,
                                const uint8_t* retained_mask, twinkv_pool pool,
                                const int32_t* table, int32_t max_pages, int32_t* out_lens,
                                int32_t* out_status, void* workspace, size_t workspace_bytes,
                                void* stream)
{
    if (!keys || !values || !aligned16(keys) || !aligned16(values) || !out_lens ||
        !aligned4(out_lens) || !aligned4(out_status))
        return TWINKV_ERR_INVALID_ARG;
    if (!pool_ok(pool) || !table_ok(table, max_pages) || s.d != pool.d ||
        (s.dtype != TWINKV_BF16 && s.dtype != TWINKV_F32))
        return TWINKV_ERR_INVALID_ARG;
    if (s.L < 1 || s.H < 1 || s.N < 1 || s.N > kMaxRows) return TWINKV_ERR_INVALID_ARG;
    const int64_t units = static_cast<int64_t>(s.L) * s.H;
    if (units > kMaxUnits) return TWINKV_ERR_INVALID_ARG;
    twinkv_status r = TWINKV_OK;
    if (retained_mask)
        r = check_ws(workspace, workspace_bytes,
                     twinkv_cache_move_workspace(static_cast<int32_t>(units), s.N));
    if (r != TWINKV_OK) return r;
    int sms = 0;
    if ((r = device_facts(&sms)) != TWINKV_OK) return r;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    IndexArgs x{};
    x.mask = retained_mask;
    x.units = static_cast<int>(units);
    x.N = x.limit_most = s.N;
    x.dst_table = table;
    x.dst_max_pages = max_pages;
    x.n_pages = pool.n_pages;
    x.index = static_cast<int*>(workspace);
    x.out_lens = out_lens;
    x.out_status = out_status;
    if ((r = cuda_result(launch_index(x, st))) != TWINKV_OK) return r;
    PackArgs a{};
    a.keys = keys;
    a.values = values;
    a.units = x.units;
    a.N = s.N;
    a.index = retained_mask ? x.index : nullptr;
    a.lens = out_lens;
    a.to = pages_of(pool, table, max_pages);
    a.out_status = out_status;
    return cuda_result(launch_pack(a, s.d, s.dtype == TWINKV_F32, st));
}

twinkv_status twinkv_cache_append(const void* keys, const void* values, twinkv_rows s,
                                  const int32_t* positions, twinkv_pool pool,
                                  const int32_t* table, int32_t max_pages, const int32_t* lens,
                                  int32_t* out_lens, int32_t* out_status, void* stream)
{
    if (!keys || !values || !positions || !lens || !out_lens || !aligned16(keys) ||
        !aligned16(values) || !aligned4(positions) || !aligned4(lens) || !aligned4(out_lens) ||
        !aligned4(out_status))
        return TWINKV_ERR_INVALID_ARG;
    if (!pool_ok(pool) || !table_ok(table, max_pages) ||
        (s.dtype != TWINKV_BF16 && s.dtype != TWINKV_F32))
        return TWINKV_ERR_INVALID_ARG;
    if (s.B < 1 || s.H < 1 || s.n < 1 || static_cast<int64_t>(s.B) * s.H > kMaxUnits)
        return TWINKV_ERR_INVALID_ARG;
    if (s.n > kMaxAppend) return TWINKV_ERR_UNSUPPORTED;
    const bool f32 = s.dtype == TWINKV_F32;
    if (!rows_aligned(f32, s.k_batch, s.k_token, s.k_head, s.v_batch, s.v_token, s.v_head))
        return TWINKV_ERR_INVALID_ARG;
    int sms = 0;
    const twinkv_status r = device_facts(&sms);
    if (r != TWINKV_OK) return r;
    AppendArgs a{};
    a.keys = keys;
    a.values = values;
    a.k_batch = s.k_batch;
    a.k_token = s.k_token;
    a.k_head = s.k_head;
    a.v_batch = s.v_batch;
    a.v_token = s.v_token;
    a.v_head = s.v_head;
    a.B = s.B;
    a.H = s.H;
    a.n = s.n;
    a.positions = positions;
    a.to = pages_of(pool, table, max_pages);
    a.lens = lens;
    a.out_lens = out_lens;
    a.out_status = out_status;
    return cuda_result(launch_append(a, pool.d, f32, static_cast<cudaStream_t>(stream)));
}

twinkv_status twinkv_cache_compact(twinkv_pool pool, const int32_t* table, int32_t max_pages,
                                   const int32_t* lens, int32_t units, const uint8_t* keep,
                                   int32_t N, const int32_t* new_table, int32_t new_max_pages,
                                   int32_t* out_lens, int32_t* out_status, void* workspace,
                                   size_t workspace_bytes, void* stream)
{
    if (!pool_ok(pool) || !table_ok(table, max_pages) || !table_ok(new_table, new_max_pages) ||
        !lens || !out_lens || !aligned4(lens) || !aligned4(out_lens) || !aligned4(out_status))
        return TWINKV_ERR_INVALID_ARG;
    if (units < 1 || units > kMaxUnits || N < 1 || N > kMaxRows || lens == out_lens)
        return TWINKV_ERR_INVALID_ARG;
    twinkv_status r = TWINKV_OK;
    if (keep)
        r = check_ws(workspace, workspace_bytes, twinkv_cache_move_workspace(units, N));
    if (r != TWINKV_OK) return r;
    int sms = 0;
    if ((r = device_facts(&sms)) != TWINKV_OK) return r;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    IndexArgs x{};
    x.mask = keep;
    x.limit = lens;
    x.units = units;
    x.N = N;
    x.limit_most = static_cast<int>(
        std::min<int64_t>(N, static_cast<int64_t>(max_pages) * kPage));
    x.src_table = table;
    x.src_max_pages = max_pages;
    x.dst_table = new_table;
    x.dst_max_pages = new_max_pages;
    x.n_pages = pool.n_pages;
    x.index = static_cast<int*>(workspace);
    x.out_lens = out_lens;
    x.out_status = out_status;
    if ((r = cuda_result(launch_index(x, st))) != TWINKV_OK) return r;
    CompactArgs a{};
    a.from = pages_of(pool, table, max_pages);
    a.to = pages_of(pool, new_table, new_max_pages);
    a.units = units;
    a.N = N;
    a.index = keep ? x.index : nullptr;
    a.lens = out_lens;
    return cuda_result(launch_compact(a, pool.d, st));
}

twinkv_status twinkv_cache_read(twinkv_pool pool, const int32_t* table, int32_t max_pages,
                                const int32_t* lens, int32_t units, int32_t rows, int32_t last,
                                void* out_keys, void* out_values, int32_t* out_positions,
                                int32_t* out_status, void* stream)
{
    if (!pool_ok(pool) || !table_ok(table, max_pages) || !lens || !aligned4(lens) || !out_keys ||
        !out_values || !aligned16(out_keys) || !aligned16(out_values) ||
        !aligned4(out_positions) || !aligned4(out_status))
        return TWINKV_ERR_INVALID_ARG;
    if (units < 1 || units > kMaxUnits || rows < 1 || rows > kMaxRows)
        return TWINKV_ERR_INVALID_ARG;
    int sms = 0;
    const twinkv_status r = device_facts(&sms);
    if (r != TWINKV_OK) return r;
    ReadArgs a{};
    a.from = pages_of(pool, table, max_pages);
    a.lens = lens;
    a.units = units;
    a.rows = rows;
    a.last = last != 0;
    a.out_keys = static_cast<uint16_t*>(out_keys);
    a.out_values = static_cast<uint16_t*>(out_values);
    a.out_positions = out_positions;
    a.out_status = out_status;
    return cuda_result(launch_read(a, pool.d, static_cast<cudaStream_t>(stream)));
}

twinkv_status twinkv_cache_attend(const void* q, twinkv_queries s, float scale, int32_t window,
                                  int32_t n_sink, twinkv_pool pool, const int32_t* table,
                                  int32_t max_pages, const int32_t* lens, void* out,
                                  float* out_lse, int32_t* out_status, void* workspace,
                                  size_t workspace_bytes, void* stream)
{
    if (!q || !out || !lens || !aligned16(q) || !aligned16(out) || !aligned4(lens) ||
        !aligned4(out_lse) || !aligned4(out_status))
        return TWINKV_ERR_INVALID_ARG;
    if (!pool_ok(pool) || !table_ok(table, max_pages)) return TWINKV_ERR_INVALID_ARG;
    if (!std::isfinite(scale) || scale <= 0.0f || window < 0 || n_sink < 0)
        return TWINKV_ERR_INVALID_ARG;
    if (s.B < 1 || s.H < 1 || s.Hq < 1 || s.n < 1 || s.Hq % s.H != 0 ||
        !rows_aligned(false, s.q_batch, s.q_token, s.q_head))
        return TWINKV_ERR_INVALID_ARG;
    const size_t need = attend_bytes(s, pool.d);
    if (need == 0) return TWINKV_ERR_UNSUPPORTED;
    twinkv_status r = check_ws(workspace, workspace_bytes, need);
    if (r != TWINKV_OK) return r;
    int sms = 0;
    if ((r = device_facts(&sms)) != TWINKV_OK) return r;
    AttendArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.q_batch = s.q_batch;
    a.q_token = s.q_token;
    a.q_head = s.q_head;
    a.B = s.B;
    a.H = s.H;
    a.G = s.Hq / s.H;
    a.n = s.n;
    a.d = pool.d;
    a.scale = scale;
    a.window = window;
    a.n_sink = n_sink;
    a.from = pages_of(pool, table, max_pages);
    a.lens = lens;
    a.out = static_cast<uint16_t*>(out);
    a.out_lse = out_lse;
    a.out_status = out_status;
    a.ws = workspace;
    return cuda_result(launch_attend(a, sms, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
