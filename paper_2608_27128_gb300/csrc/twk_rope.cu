// twk_rope.cu -- norms of queries and keys per head, with the position rotation in the same pass:
// what turns a layer's projections into queries and into the post-RoPE keys that the cache stores
// and the audit reads (arXiv 2608.27128, Sec. 3.2).
//
// Per token and head, with x the D values of the head:
//     y = x / sqrt(mean(x^2) + eps) * w              (without w: y = x)
//     out[j]       = y[j] cos_j - y[j + D/2] sin_j
//     out[j + D/2] = y[j] sin_j + y[j + D/2] cos_j    j < D/2,
// cos and sin from the row of the token's position in a float32 table.  Sums, norm and rotation
// in float32, rounded once at the store.
//
// Bound by memory: each value is read and written once.  A lane holds eight values of the head's
// first half and the eight they rotate with, in 16-byte loads, so D / 16 lanes hold a head and a
// warp 512 / D of them; the squares are summed with shuffles over those lanes.  A warp stays with
// one token, so that the lanes read their cosines and sines once for all of its heads.
#include "twk_cache.cuh"
#include "twk_cache_internal.h"
#include "twk_ptx.cuh"

namespace twk {
namespace {

constexpr int kRopeThreads = 128;

template <typename T>
struct Eight;

template <>
struct Eight<uint16_t> {
    uint4 v;
    __device__ void load(const uint16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ void get(float (&x)[8]) const
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo(w[i]);
            x[2 * i + 1] = bf16_hi(w[i]);
        }
    }
    __device__ static void put(uint16_t* p, const float (&x)[8])
    {
        uint4 o;
        o.x = bf16_pair(x[0], x[1]);
        o.y = bf16_pair(x[2], x[3]);
        o.z = bf16_pair(x[4], x[5]);
        o.w = bf16_pair(x[6], x[7]);
        *reinterpret_cast<uint4*>(p) = o;
    }
};

template <>
struct Eight<float> {
    float4 a, b;
    __device__ void load(const float* p)
    {
        a = reinterpret_cast<const float4*>(p)[0];
        b = reinterpret_cast<const float4*>(p)[1];
    }
    __device__ void get(float (&x)[8]) const
    {
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
        x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    }
    __device__ static void put(float* p, const float (&x)[8])
    {
        reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
};

template <typename T, int D>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeArgs a, int splits)
{
    constexpr int kLanes = D / 16;           // lanes of a head
    constexpr int kHeads = 32 / kLanes;      // heads of a warp
    const int lane = threadIdx.x % 32, l = lane % kLanes;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * (kRopeThreads / 32) + threadIdx.x / 32;
    const int token = static_cast<int>(item / splits), split = static_cast<int>(item % splits);
    if (token >= a.tokens) return;
    const int heads = a.heads_q + a.heads_k;
    const int pos = a.positions[token];
    const bool bad = pos < 0 || pos >= a.rows;
    if (a.out_status && split == 0 && lane == 0) a.out_status[token] = bad ? 1 : 0;
    // a token without a row of the table: values, cosines and sines are 0, and there is no norm
    float cs[8], sn[8];
    {
        Eight<float> c = {}, s = {};
        if (!bad) {
            const float* row = a.cos_sin + static_cast<int64_t>(pos) * D + 8 * l;
            c.load(row);
            s.load(row + D / 2);
        }
        c.get(cs);
        s.get(sn);
    }
    // the next heads' values are loaded before the present ones are used
    auto load = [&](int h, Eight<T>& u, Eight<T>& v) {
        if (bad || h >= heads) return;
        const T* src = h < a.heads_q
                           ? static_cast<const T*>(a.q) + token * a.q_token + h * a.q_head
                           : static_cast<const T*>(a.k) + token * a.k_token +
                                 (h - a.heads_q) * a.k_head;
        u.load(src + 8 * l);
        v.load(src + D / 2 + 8 * l);
    };
    const int step = splits * kHeads;
    int h = split * kHeads + lane / kLanes;
    Eight<T> u = {}, v = {};
    load(h, u, v);
    for (int h0 = split * kHeads; h0 < heads; h0 += step, h += step) {
        float x[8], y[8];
        u.get(x);
        v.get(y);
        load(h + step, u, v);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], fmaf(y[i], y[i], sum));
#pragma unroll
        for (int m = 1; m < kLanes; m *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, m);
        if (h >= heads) continue;
        const bool is_q = h < a.heads_q;
        const T* w = static_cast<const T*>(is_q ? a.wq : a.wk);
        if (w && !bad) {
            const float r = rsqrtf(sum * (1.0f / D) + a.eps);
            float wx[8], wy[8];
            Eight<T> s, c;
            s.load(w + 8 * l);
            c.load(w + D / 2 + 8 * l);
            s.get(wx);
            c.get(wy);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] *= r * wx[i];
                y[i] *= r * wy[i];
            }
        }
        T* dst = is_q ? static_cast<T*>(a.out_q) + token * a.oq_token + h * a.oq_head
                      : static_cast<T*>(a.out_k) + token * a.ok_token +
                            (h - a.heads_q) * a.ok_head;
        float p[8], q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = x[i] * cs[i] - y[i] * sn[i];
            q[i] = x[i] * sn[i] + y[i] * cs[i];
        }
        Eight<T>::put(dst + 8 * l, p);
        Eight<T>::put(dst + D / 2 + 8 * l, q);
    }
}

template <typename T, int D>
cudaError_t launch(const RopeArgs& a, int sms, cudaStream_t st)
{
    constexpr int kHeads = 512 / D;
    const int groups = (a.heads_q + a.heads_k + kHeads - 1) / kHeads;
    // A token's heads are split over several warps while that leaves warps without work.
    const int64_t room = static_cast<int64_t>(sms) * 48;
    int splits = groups;
    if (static_cast<int64_t>(a.tokens) * groups > room)
        splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(groups, room / a.tokens)));
    const int64_t warps = static_cast<int64_t>(a.tokens) * splits;
    const int64_t blocks = (warps + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
    rope_kernel<T, D><<<static_cast<unsigned>(blocks), kRopeThreads, 0, st>>>(a, splits);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, bool f32, int sms, cudaStream_t st)
{
    if (a.d == 128) return f32 ? launch<float, 128>(a, sms, st) : launch<uint16_t, 128>(a, sms, st);
    return f32 ? launch<float, 64>(a, sms, st) : launch<uint16_t, 64>(a, sms, st);
}

}  // namespace twk
