// cp_norm_rope: norm of the heads' queries and keys, position rotation and cache append in one pass (see the header).
//
// HBM-bound: a row of (Hq + 2 Hkv) heads is read once and written once, K and V a second time into the cache.  Sixteen
// lanes hold a head's 128 elements, eight each (one 16-byte load and store), so a wavefront takes four heads a step;
// the sum of squares is four exchanges within the 16 lanes (through LDS 668 us where these take 650).  131072 tokens, 32/8
// heads: 3.76 GB in 650 us, 5.8 TB/s, what a copy reaches; 32 tokens, 64/8 heads: 4.2 us, a launch and one chain of loads.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include <cmath>

#include "cp_checks.h"
#include "cp_device.h"
#include "cp_norm_rope.h"

namespace {

constexpr int kWaves = 4; // per workgroup

struct RopeParams {
    const uint16_t *x[3]; // q, k, v
    uint16_t *out[3];
    const void *weight[2];
    uint16_t *kv_pages;
    const int32_t *positions;
    const int32_t *block_table;
    const int32_t *prefix_lens;
    const int32_t *extend_lens;
    int32_t stride[3]; // elements between rows
    int32_t heads[3];  // 0: left out
    int32_t steps[3];  // of four heads
    int32_t units;     // wavefronts per token
    int32_t batch, max_pages, T, Hkv;
    int32_t half, interleaved, weights_fp32;
    float eps, scale;
    uint64_t turns[kD / 2]; // inv_freq / (2 pi) in units of 2^-64
};

__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// Sum over the 16 lanes of a head, in every one of them: lanes exchanged within fours, then fours and eights turned around.
template <int kControl>
__device__ __forceinline__ float added(float x)
{
    return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), kControl, 0xf, 0xf, false));
}
__device__ __forceinline__ float head_sum(float x)
{
    x = added<0xb1>(x);     // quad_perm 1, 0, 3, 2
    x = added<0x4e>(x);     // quad_perm 2, 3, 0, 1
    x = added<0x124>(x);    // row_ror:4
    return added<0x128>(x); // row_ror:8
}

__device__ __forceinline__ void unpack(u32x4 raw, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(raw[i]);
        x[2 * i + 1] = bf16_hi(raw[i]);
    }
}

// Eight weights as they lie in memory: bf16 in the first four words, fp32 in all.
struct Weights {
    u32x4 lo, hi;
};
__device__ __forceinline__ Weights load_weights(const RopeParams &p, const void *from, int chunk)
{
    Weights w{u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
    if (!from) return w;
    if (p.weights_fp32) {
        w.lo = reinterpret_cast<const u32x4 *>(from)[2 * chunk];
        w.hi = reinterpret_cast<const u32x4 *>(from)[2 * chunk + 1];
    } else {
        w.lo = reinterpret_cast<const u32x4 *>(from)[chunk];
    }
    return w;
}
__device__ __forceinline__ void unpack(const RopeParams &p, const void *from, Weights w, float (&x)[8])
{
    if (!from) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 1.f;
    } else if (p.weights_fp32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = __uint_as_float(w.lo[i]);
            x[4 + i] = __uint_as_float(w.hi[i]);
        }
    } else {
        unpack(w.lo, x);
    }
}

// 1 / sqrt(mean of the squares + eps) of the 16 lanes' 8 elements each.  `before`: what the elements have to be multiplied by
// first, 1 unless their squares or eps leave the range of fp32, as those of finite bf16 values can: above it, or where the
// products below 2^-126, which the dot product takes for 0, make up more than 2^-29 of the mean.
__device__ __forceinline__ float inverse_rms(u32x4 raw, float eps, float &before)
{
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf16x2 x = __builtin_bit_cast(bf16x2, (uint32_t)raw[i]);
        sum = __builtin_amdgcn_fdot2_f32_bf16(x, x, sum, false);
    }
    sum = head_sum(sum);
    float mean = fmaf(sum, 1.f / kD, eps);
    const bool high = fmaxf(sum, mean) > 3.0e38f;
    before = high ? 0x1p-70f : mean < 0x1p-90f ? 0x1p60f : 1.f;
    if (before != 1.f) {
        float x[8], scaled = 0.f;
        unpack(raw, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) scaled = fmaf(x[i] * before, x[i] * before, scaled);
        mean = fmaf(head_sum(scaled), 1.f / kD, eps * before * before);
    }
    return __builtin_amdgcn_rsqf(mean);
}

// The element of an array of the arguments that a wavefront's step is of; an index that is no constant would have the compiler
// copy the arguments to memory.
template <typename T>
__device__ __forceinline__ T of_kind(const T (&x)[3], int kind)
{
    const T q = x[0], k = x[1], v = x[2];
    return kind == 0 ? q : kind == 1 ? k : v;
}

// A wavefront takes kSteps steps of four heads of one token; all loads are under way before the first is used.  Rows go past the
// L2 in both directions: what is read is not read again, and what is written is read by other XCDs, whose L2 is another (131072
// tokens, 32/8 heads 696 -> 668 us, 1024 10.2 -> 7.8).
template <int kSteps>
__global__ __launch_bounds__(kWaves * 64) void norm_rope_kernel(const RopeParams p)
{
    __shared__ f32x2 table[kWaves][kD / 2]; // cos and sin of the wavefront's position
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int sub = lane >> 4, chunk = lane & 15; // head of a step, 16-byte piece of its row
    const int id = (int)blockIdx.x * kWaves + wave; // the host keeps the number of them below 2^31
    const int t = id / p.units;
    if (t >= p.T) return;
    const int unit = id - t * p.units;

    // Everything that does not wait for another load: the lengths, the first heads, the weights, the lane's frequency.
    const int len0 = lane < p.batch ? p.extend_lens[lane] : 0;
    const int cached0 = lane < p.batch ? p.prefix_lens[lane] : 0;
    const int step0 = unit * kSteps; // steps go through q's heads, then k's, then v's
    const int k0 = p.steps[0], v0 = k0 + p.steps[1], end = v0 + p.steps[2];
    u32x4 raw[kSteps];
    int kind[kSteps], head[kSteps]; // 3: none
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int at = step0 + s;
        kind[s] = (at >= k0) + (at >= v0) + (at >= end);
        head[s] = (at - (at >= v0 ? v0 : at >= k0 ? k0 : 0)) * 4 + sub;
        raw[s] = u32x4{0, 0, 0, 0};
        if (kind[s] < 3 && head[s] < of_kind(p.heads, kind[s]))
            raw[s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(
                of_kind(p.x, kind[s]) + (int64_t)t * of_kind(p.stride, kind[s]) + head[s] * kD + chunk * 8));
    }
    // the element that makes a pair with one of this lane's lies in this lane (interleaved) or half / 8 lanes away
    const bool turned = chunk * 8 < 2 * p.half, second = turned && !p.interleaved && chunk * 8 >= p.half;
    const int away = !turned || p.interleaved ? 0 : second ? -(p.half >> 3) : p.half >> 3;
    const bool has_q = step0 < k0, has_k = step0 < v0 && step0 + kSteps > k0;
    Weights own[2], pair[2];
    if (has_q) {
        own[0] = load_weights(p, p.weight[0], chunk);
        pair[0] = load_weights(p, p.weight[0], chunk + away);
    }
    if (has_k) {
        own[1] = load_weights(p, p.weight[1], chunk);
        pair[1] = load_weights(p, p.weight[1], chunk + away);
    }
    const uint64_t speed = p.turns[lane];
    int position = p.positions ? p.positions[t] : 0;

    // the token's request
    int r = 0, tok = 0, cu = 0;
    for (int base = 0; base < p.batch; base += 64) {
        const int rr = base + lane;
        const int e = base == 0 ? len0 : rr < p.batch ? p.extend_lens[rr] : 0;
        const int pl = base == 0 ? cached0 : rr < p.batch ? p.prefix_lens[rr] : 0;
        const int incl = wave_scan(e);
        const int total = __builtin_amdgcn_readlane(incl, 63);
        if (t - cu < total) {
            const int first = __builtin_ctzll(__builtin_amdgcn_ballot_w64(incl > t - cu));
            r = base + first;
            tok = __builtin_amdgcn_readlane(pl - incl + e, first) + t - cu;
            break;
        }
        cu += total;
    }
    int64_t page = 0;
    if (p.kv_pages) page = p.block_table[(int64_t)r * p.max_pages + (tok >> 4)];
    if (!p.positions) position = tok;
    // x' = x * cos + y * sin with the sign of the sine that the element has, y: the other element of its pair.  The weights go in
    // with the factors: a row costs two products an element.
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        cs[i] = 1.f;
        sn[i] = 0.f;
    }
    if (p.half && (has_q || has_k)) {
        // the fraction of a turn, as a signed number; the instructions take turns, and are off by 2^-23 at most
        const float z = (float)(int32_t)(((uint64_t)(int64_t)position * speed) >> 32) * 0x1p-32f;
        table[wave][lane] = f32x2{__builtin_amdgcn_cosf(z) * p.scale, __builtin_amdgcn_sinf(z) * p.scale};
        __builtin_amdgcn_wave_barrier();
        if (turned) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f32x2 v = table[wave][p.interleaved ? chunk * 4 + i / 2 : chunk * 8 + i - (second ? p.half : 0)];
                cs[i] = v[0];
                sn[i] = (p.interleaved ? i % 2 == 1 : second) ? v[1] : -v[1];
            }
        }
    }
    float a[2][8], b[2][8];
    auto factors = [&](int k) {
        float w[8], wp[8];
        unpack(p, p.weight[k], own[k], w);
        unpack(p, p.weight[k], pair[k], wp);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            a[k][i] = cs[i] * w[i];
            b[k][i] = sn[i] * (p.interleaved ? w[i ^ 1] : wp[i]);
        }
    };
    if (has_q) factors(0);
    if (has_k) factors(1);
    uint16_t *const slot = p.kv_pages ? p.kv_pages + (page * 2 * p.Hkv * kPS + (tok & 15)) * (int64_t)kD + chunk * 8 : nullptr;

    auto finish = [&](u32x4 &raw, int k) { // a row of q or k
        float before = 1.f;
        const float rs = p.weight[k] ? inverse_rms(raw, p.eps, before) : 1.f;
        float x[8], y[8];
        unpack(raw, x);
        if (p.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
        } else {
            u32x4 other;
#pragma unroll
            for (int i = 0; i < 4; ++i) other[i] = __shfl(raw[i], lane + away, 64);
            unpack(other, y);
        }
        if (__builtin_amdgcn_ballot_w64(before != 1.f) != 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] *= before;
                y[i] *= before;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bf16x2 both;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int at = 2 * i + e;
                both[e] = (__bf16)(rs * (turned ? fmaf(x[at], a[k][at], y[at] * b[k][at]) : x[at] * a[k][at]));
            }
            raw[i] = __builtin_bit_cast(uint32_t, both);
        }
    };
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        if (kind[s] >= 3) break;
        if (kind[s] == 0) finish(raw[s], 0);
        else if (kind[s] == 1) finish(raw[s], 1);
        const int heads = of_kind(p.heads, kind[s]);
        if (head[s] >= heads) continue;
        uint16_t *const out = of_kind(p.out, kind[s]);
        if (out) __builtin_nontemporal_store(raw[s], reinterpret_cast<u32x4 *>(out + ((int64_t)t * heads + head[s]) * kD + chunk * 8));
        if (slot && kind[s] > 0)
            __builtin_nontemporal_store(raw[s], reinterpret_cast<u32x4 *>(slot + (int64_t)((kind[s] - 1) * p.Hkv + head[s]) * kPS * kD));
    }
}

// Up to this many steps in all a wavefront takes one: the time is the chain from its first load to its last store (32 tokens, 64/8
// heads 3.7 us, with four steps 5.3; 1024 tokens, 32/8 heads, 12288 steps 10.8 and 9.9).
constexpr int64_t kFewSteps = 8192;

// freq / (2 pi) in units of 2^-64, without its whole turns: the double's 53 bits times the first 128 of 1 / (2 pi), which is
// 0.28BE60DB9391054A 7F09D5F47D4D3770... in hexadecimal.  |freq| <= 2^20.
uint64_t turns_of(double freq)
{
    uint64_t bits;
    memcpy(&bits, &freq, sizeof(bits));
    const int exponent = (int)(bits >> 52 & 0x7ff); // of a number that is not denormal; one that is turns nothing
    if (exponent == 0) return 0;
    const uint64_t digits = (bits & ((1ull << 52) - 1)) | 1ull << 52; // |freq| = digits * 2^(exponent - 1075)
    // digits * 2^128 / (2 pi) in three words, the lowest left out
    const unsigned __int128 low = (unsigned __int128)digits * 0x7F09D5F47D4D3770u, high = (unsigned __int128)digits * 0x28BE60DB9391054Au;
    const unsigned __int128 words = high + (uint64_t)(low >> 64); // digits / (2 pi) in units of 2^-64
    const int shift = exponent - 1075;                            // <= -32
    const uint64_t turns = shift <= -128 ? 0 : (uint64_t)(words >> -shift);
    return freq < 0 ? 0 - turns : turns;
}

bool stride_ok(int64_t stride, int heads)
{
    return stride == 0 || (stride >= (int64_t)heads * kD && stride % 8 == 0 && stride <= INT32_MAX);
}

} // namespace

extern "C" int cp_qk_norm_rope(const void *q, const void *k, const void *v, const void *q_weight, const void *k_weight,
                               const int32_t *positions, const int32_t *block_table, const int32_t *prefix_lens,
                               const int32_t *extend_lens, void *q_out, void *k_out, void *v_out, void *kv_pages,
                               void *stream, const cp_shape *shape, const cp_norm_rope *rope)
{
    const int st = cp::validate_shape(shape);
    if (st != CP_OK) return st;
    if (!rope) return CP_ERR_NULL;
    if (rope->rotary_dim < 0 || rope->rotary_dim > kD || rope->rotary_dim % 16 != 0) return CP_ERR_SHAPE;
    if (rope->rotary_dim > 0 && !rope->h_inv_freq) return CP_ERR_NULL;
    if ((rope->interleaved | rope->weights_fp32) & ~1) return CP_ERR_SHAPE;
    if (!(rope->eps > 0.f) || !std::isfinite(rope->eps) || !std::isfinite(rope->rotary_scale)) return CP_ERR_SHAPE;
    const int Hq = shape->num_q_heads, Hkv = shape->num_kv_heads;
    const int heads[3] = {Hq, Hkv, Hkv};
    const int64_t strides[3] = {rope->q_stride, rope->k_stride, rope->v_stride};
    const void *const in[3] = {q, k, v};
    void *const out[3] = {q_out, k_out, v_out};
    if (Hq > INT32_MAX / kD) return CP_ERR_SHAPE; // elements of a row
    for (int i = 0; i < 3; ++i)
        if (!stride_ok(strides[i], heads[i])) return CP_ERR_SHAPE;
    for (int f = 0; f < rope->rotary_dim / 2; ++f)
        if (!(std::fabs(rope->h_inv_freq[f]) <= 0x1p20)) return CP_ERR_SHAPE;
    if (!prefix_lens || !extend_lens) return CP_ERR_NULL;
    if (shape->total_extend == 0) return CP_OK;
    if (kv_pages && (!k || !v || !block_table)) return CP_ERR_NULL;
    for (int i = 0; i < 3; ++i) {
        if (!in[i] ? out[i] != nullptr : !out[i] && !(i > 0 && kv_pages)) return CP_ERR_NULL;
        if (!aligned_to(in[i], 16) || !aligned_to(out[i], 16)) return CP_ERR_ALIGN;
        if (in[i] && in[i] == out[i] && strides[i] != 0 && strides[i] != (int64_t)heads[i] * kD) return CP_ERR_SHAPE;
    }
    if (!aligned_to(q_weight, 16) || !aligned_to(k_weight, 16) || !aligned_to(kv_pages, 16) || !aligned_to(positions, 4) ||
        !aligned_to(block_table, 4) || !aligned_to(prefix_lens, 4) || !aligned_to(extend_lens, 4))
        return CP_ERR_ALIGN;
    if (kv_pages && cp::debug_checks_on()) {
        const int chk = cp_check_tables(block_table, prefix_lens, extend_lens, stream, shape, nullptr);
        if (chk != CP_OK) return chk;
    }

    RopeParams p;
    int64_t steps = 0;
    for (int i = 0; i < 3; ++i) {
        p.x[i] = static_cast<const uint16_t *>(in[i]);
        p.out[i] = static_cast<uint16_t *>(out[i]);
        p.stride[i] = (int32_t)(strides[i] ? strides[i] : (int64_t)heads[i] * kD);
        p.heads[i] = in[i] ? heads[i] : 0;
        p.steps[i] = (p.heads[i] + 3) / 4;
        steps += p.steps[i];
    }
    if (steps == 0) return CP_OK;
    p.weight[0] = q_weight;
    p.weight[1] = k_weight;
    p.kv_pages = static_cast<uint16_t *>(kv_pages);
    p.positions = positions;
    p.block_table = block_table;
    p.prefix_lens = prefix_lens;
    p.extend_lens = extend_lens;
    const int per_wave = steps * shape->total_extend <= kFewSteps ? 1 : 4;
    p.units = (int32_t)((steps + per_wave - 1) / per_wave);
    p.batch = shape->batch;
    p.max_pages = shape->max_pages_per_req;
    p.T = shape->total_extend;
    p.Hkv = Hkv;
    p.half = rope->rotary_dim / 2;
    p.interleaved = rope->interleaved;
    p.weights_fp32 = rope->weights_fp32;
    p.eps = rope->eps;
    p.scale = rope->rotary_scale;
    for (int f = 0; f < kD / 2; ++f) p.turns[f] = f < p.half ? turns_of(rope->h_inv_freq[f]) : 0;
    const int64_t groups = ((int64_t)p.T * p.units + kWaves - 1) / kWaves;
    if (groups > cp::kMostThreads / (kWaves * 64)) return CP_ERR_SHAPE;
    const dim3 grid((unsigned)groups), block(kWaves * 64);
    if (per_wave == 1) hipLaunchKernelGGL(norm_rope_kernel<1>, grid, block, 0, static_cast<hipStream_t>(stream), p);
    else hipLaunchKernelGGL(norm_rope_kernel<4>, grid, block, 0, static_cast<hipStream_t>(stream), p);
    return hipGetLastError() == hipSuccess ? CP_OK : CP_ERR_LAUNCH;
}
