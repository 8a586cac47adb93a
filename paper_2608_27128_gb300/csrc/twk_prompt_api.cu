// twk_prompt_api.cu -- the C ABI of the operators that make a retained set (declared in
// include/twinkv.h): argument checks and launches of the attention over prompts, of its weights per
// key, over prompts and over pages, and of the eviction by accumulated weight.
#include <cmath>

#include "twinkv.h"
#include "twk_cache.cuh"
#include "twk_prompt_internal.h"

using namespace twk;

namespace {

constexpr int kMaxPacked = 1 << 24;    // rows of q or k
constexpr int kMaxRows = 1 << 20;      // positions of a unit, as for the audit
constexpr int kMaxUnits = 65535;
constexpr int kMaxGroup = 128;         // query heads per KV head over prompts

// above 0, and a float32 as a multiple of log 2 too
bool scale_ok(float scale) { return std::isfinite(scale) && scale > 0.0f && scale < 0x1p127f; }

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// of a dimension of n: rows on 16-byte boundaries, apart from each other, within a copy's reach
bool stride_ok(int64_t stride, int n)
{
    return n == 1 || (stride > 0 && stride % 8 == 0 && stride < (int64_t{1} << 38));
}

twinkv_status check_ws(void* ws, size_t bytes, size_t need)
{
    if (!ws || !aligned(ws, 256) || bytes < need) return TWINKV_ERR_WORKSPACE;
    return TWINKV_OK;
}

twinkv_status sizes_ok(const twinkv_prompt& s)
{
    if ((s.d != 64 && s.d != 128) || s.B < 1 || s.H < 1 || s.Hq < 1 || s.Hq % s.H != 0 ||
        s.tokens < 1 || s.keys < 1)
        return TWINKV_ERR_INVALID_ARG;
    if (s.tokens > kMaxPacked || s.keys > kMaxPacked || s.B > kMaxUnits || s.Hq > kMaxUnits ||
        s.Hq / s.H > kMaxGroup)
        return TWINKV_ERR_UNSUPPORTED;
    return TWINKV_OK;
}

twinkv_status prompt_ok(const void* q, const void* k, const twinkv_prompt& s,
                        const twinkv_sequences& seqs, float scale, int32_t window, int32_t n_sink,
                        const int32_t* out_status)
{
    if (!q || !k || !aligned(q, 16) || !aligned(k, 16) || !aligned(out_status, 4) ||
        !aligned(seqs.offsets, 4) || !aligned(seqs.lens, 4) || !aligned(seqs.k_offsets, 4) ||
        !aligned(seqs.k_lens, 4))
        return TWINKV_ERR_INVALID_ARG;
    const twinkv_status r = sizes_ok(s);
    if (r != TWINKV_OK) return r;
    if (!seqs.offsets && s.B != 1) return TWINKV_ERR_INVALID_ARG;
    if (!stride_ok(s.q_token, s.tokens) || !stride_ok(s.q_head, s.Hq) ||
        !stride_ok(s.k_token, s.keys) || !stride_ok(s.k_head, s.H))
        return TWINKV_ERR_INVALID_ARG;
    if (!scale_ok(scale) || window < 0 || n_sink < 0)
        return TWINKV_ERR_INVALID_ARG;
    return TWINKV_OK;
}

PromptArgs args_of(const void* q, const void* k, const twinkv_prompt& s,
                   const twinkv_sequences& seqs, float scale, int32_t window, int32_t n_sink,
                   int32_t* out_status, void* ws)
{
    PromptArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.s = s;
    a.seqs = seqs;
    a.G = s.Hq / s.H;
    a.tile_tokens = 128 / a.G;
    a.scale = scale;
    // beyond every position they are alike, and sums with positions stay in 32 bits
    a.window = window < 2 * kMaxPacked ? window : 2 * kMaxPacked;
    a.n_sink = n_sink < 2 * kMaxPacked ? n_sink : 2 * kMaxPacked;
    a.out_status = out_status;
    a.ws = ws;
    return a;
}

}  // namespace

extern "C" {

size_t twinkv_prompt_attend_workspace(twinkv_prompt s)
{
    return sizes_ok(s) == TWINKV_OK ? up256(prompt_attend_workspace(s)) : 0;
}

size_t twinkv_prompt_weights_workspace(twinkv_prompt s)
{
    return sizes_ok(s) == TWINKV_OK ? up256(prompt_weights_workspace(s)) : 0;
}

size_t twinkv_cache_weights_workspace(twinkv_queries s, int32_t d)
{
    if (twinkv_cache_attend_workspace(s, d) == 0) return 0;
    return up256(static_cast<size_t>(s.B) * s.H * (1 + s.n) * 4);
}

twinkv_status twinkv_prompt_attend(const void* q, const void* k, const void* v, twinkv_prompt s,
                                   twinkv_sequences seqs, float scale, int32_t window,
                                   int32_t n_sink, void* out, float* out_lse, int32_t* out_status,
                                   void* workspace, size_t workspace_bytes, void* stream)
{
    twinkv_status r = prompt_ok(q, k, s, seqs, scale, window, n_sink, out_status);
    if (r != TWINKV_OK) return r;
    // rows are read while others are written
    if (out == q || out == k || out == v) return TWINKV_ERR_INVALID_ARG;
    if (!v || !out || !aligned(v, 16) || !aligned(out, 16) || !aligned(out_lse, 4) ||
        !stride_ok(s.v_token, s.keys) || !stride_ok(s.v_head, s.H))
        return TWINKV_ERR_INVALID_ARG;
    r = check_ws(workspace, workspace_bytes, twinkv_prompt_attend_workspace(s));
    if (r != TWINKV_OK) return r;
    int sms = 0;
    WaitFacts w;
    if ((r = device_facts(&sms)) != TWINKV_OK || (r = wait_facts(&w)) != TWINKV_OK) return r;
    PromptArgs a = args_of(q, k, s, seqs, scale, window, n_sink, out_status, workspace);
    a.v = static_cast<const uint16_t*>(v);
    a.out = static_cast<uint16_t*>(out);
    a.out_lse = out_lse;
    return cuda_result(launch_prompt_attend(a, sms, w, static_cast<cudaStream_t>(stream)));
}

twinkv_status twinkv_prompt_weights(const void* q, const void* k, const float* lse,
                                    twinkv_prompt s, twinkv_sequences seqs, float scale,
                                    int32_t window, int32_t n_sink, int32_t last,
                                    const float* score, float* out_score, int32_t* out_status,
                                    void* workspace, size_t workspace_bytes, void* stream)
{
    twinkv_status r = prompt_ok(q, k, s, seqs, scale, window, n_sink, out_status);
    if (r != TWINKV_OK) return r;
    if (!lse || !out_score || !aligned(lse, 4) || !aligned(score, 4) || !aligned(out_score, 4) ||
        last < 0)
        return TWINKV_ERR_INVALID_ARG;
    r = check_ws(workspace, workspace_bytes, twinkv_prompt_weights_workspace(s));
    if (r != TWINKV_OK) return r;
    int sms = 0;
    WaitFacts w;
    if ((r = device_facts(&sms)) != TWINKV_OK || (r = wait_facts(&w)) != TWINKV_OK) return r;
    PromptArgs a = args_of(q, k, s, seqs, scale, window, n_sink, out_status, workspace);
    a.lse = lse;
    a.last = last;
    a.score = score;
    a.out_score = out_score;
    return cuda_result(launch_prompt_weights(a, sms, w, static_cast<cudaStream_t>(stream)));
}

twinkv_status twinkv_cache_weights(const void* q, const float* lse, twinkv_queries s, float scale,
                                   int32_t window, int32_t n_sink, twinkv_pool pool,
                                   const int32_t* table, int32_t max_pages, const int32_t* lens,
                                   const float* score, float* out_score, int32_t N,
                                   int32_t* out_status, void* workspace, size_t workspace_bytes,
                                   void* stream)
{
    if (!q || !lse || !lens || !score || !out_score || !aligned(q, 16) || !aligned(lse, 4) ||
        !aligned(lens, 4) || !aligned(score, 4) || !aligned(out_score, 4) ||
        !aligned(out_status, 4))
        return TWINKV_ERR_INVALID_ARG;
    if ((pool.d != 64 && pool.d != 128) || !pool.pages || !aligned(pool.pages, 16) ||
        pool.n_pages < 1 || !table || !aligned(table, 4) || max_pages < 1 ||
        max_pages > kMaxRows / kPage)
        return TWINKV_ERR_INVALID_ARG;
    if (!scale_ok(scale) || window < 0 || n_sink < 0 || N < 1 ||
        N > kMaxRows)
        return TWINKV_ERR_INVALID_ARG;
    if (s.B < 1 || s.H < 1 || s.Hq < 1 || s.n < 1 || s.Hq % s.H != 0 || s.q_batch % 8 ||
        s.q_token % 8 || s.q_head % 8)
        return TWINKV_ERR_INVALID_ARG;
    const size_t need = twinkv_cache_weights_workspace(s, pool.d);
    if (need == 0) return TWINKV_ERR_UNSUPPORTED;
    twinkv_status r = window > 0 ? check_ws(workspace, workspace_bytes, need) : TWINKV_OK;
    if (r != TWINKV_OK) return r;
    int sms = 0;
    if ((r = device_facts(&sms)) != TWINKV_OK) return r;
    CacheWeightsArgs p{};
    p.a.q = static_cast<const uint16_t*>(q);
    p.a.q_batch = s.q_batch;
    p.a.q_token = s.q_token;
    p.a.q_head = s.q_head;
    p.a.B = s.B;
    p.a.H = s.H;
    p.a.G = s.Hq / s.H;
    p.a.n = s.n;
    p.a.d = pool.d;
    p.a.scale = scale;
    p.a.window = window;
    p.a.n_sink = n_sink;
    p.a.from = {static_cast<uint8_t*>(pool.pages), pool.n_pages, table, max_pages};
    p.a.lens = lens;
    p.a.out_status = out_status;
    p.a.ws = workspace;
    p.lse = lse;
    p.score = score;
    p.out_score = out_score;
    p.N = N;
    return cuda_result(launch_cache_weights(p, sms, static_cast<cudaStream_t>(stream)));
}

twinkv_status twinkv_weight_policy(const float* score, int32_t units, int32_t N,
                                   const int32_t* lens, const int32_t* budget, int32_t n_sink,
                                   int32_t n_recent, uint8_t* out_mask, float* out_score,
                                   int32_t* out_status, void* stream)
{
    if (!score || !budget || !out_mask || !aligned(score, 4) || !aligned(lens, 4) ||
        !aligned(budget, 4) || !aligned(out_score, 4) || !aligned(out_status, 4) ||
        score == out_score)
        return TWINKV_ERR_INVALID_ARG;
    if (units < 1 || units > kMaxUnits || N < 1 || N > kMaxRows || n_sink < 0 || n_recent < 0)
        return TWINKV_ERR_INVALID_ARG;
    int sms = 0;
    const twinkv_status r = device_facts(&sms);
    if (r != TWINKV_OK) return r;
    WeightPolicyArgs a{};
    a.score = score;
    a.units = units;
    a.N = N;
    a.lens = lens;
    a.budget = budget;
    a.n_sink = n_sink;
    a.n_recent = n_recent;
    a.out_mask = out_mask;
    a.out_score = out_score;
    a.out_status = out_status;
    return cuda_result(launch_weight_policy(a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
