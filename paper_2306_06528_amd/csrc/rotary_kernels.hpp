// Norms of queries and keys, head by head, with the rotation by position in the same pass, forward and backward.  A team of L lanes holds a head, 16 bytes a lane, from its one load to its
// one store; memory bounds both passes.  A workgroup has some tokens of one particle: their angles are formed in 64 bits once for all heads (kTokens tokens at a time, to LDS), and the weights
// and their gradients stay in registers.  In the half layout a value's partner is another lane's: the team's values change lanes in its part of LDS.
#pragma once
#include "attention_common.hpp"

namespace svgd {

constexpr int kTokens = 8, kRotaryBlock = 256;
constexpr int kMaxPairs = SVGD_ROTARY_MAX_DIM / 2;

struct RotaryArgs {
    int heads, kv, dim, pairs, interleaved;
    int length;
    int64_t tokens; // batch length: of a particle
    const double *frequencies;
    const int64_t *positions;
    int64_t positions_stride;
    float eps;
    Params q_weight, k_weight;
    int blocks;  // workgroups per particle
    int64_t per; // tokens of each
};

// cos and sin of position frequency: reduced to [-pi, pi] in 64 bits, and what rounding that to 32 bits leaves out put back to first order.
__device__ __forceinline__ void turn_of(int64_t position, double frequency, float &c, float &s)
{
    const double angle = (double)position * frequency;
    const double turns = rint(angle * 0.15915494309189535);
    double r = fma(-turns, 6.283185307179586, angle);
    r = fma(-turns, 2.4492935982947064e-16, r);
    const float hi = (float)r, lo = (float)(r - (double)hi);
    float s0, c0;
    sincosf(hi, &s0, &c0);
    s = s0 + lo * c0;
    c = c0 - lo * s0;
}

template <int L> __device__ __forceinline__ float head_sum(float v)
{
    if constexpr (L <= 16) {
        return row_sum<L>(v);
    } else {
        v = row_sum(v);
        const unsigned u = __float_as_uint(v);
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        if constexpr (L == 64) {
            const unsigned w = __float_as_uint(v);
            const auto q = __builtin_amdgcn_permlane32_swap(w, w, false, false);
            v = __uint_as_float(q[0]) + __uint_as_float(q[1]);
        }
        return v;
    }
}

// Turns the lane's values, c on, by the angles in cs and sn, with sign -1 back.  slot: the team's part of LDS, 16 bytes aligned.
template <int VEC>
__device__ __forceinline__ void turn(const RotaryArgs &a, float (&y)[VEC], int c, float *slot, const float *cs, const float *sn, float sign)
{
    if (a.pairs == 0) return;
    if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
            const int j = (c + e) >> 1;
            if (j < a.pairs) {
                const float co = cs[j], si = sign * sn[j], p = y[e], q = y[e + 1];
                y[e] = p * co - q * si;
                y[e + 1] = q * co + p * si;
            }
        }
        return;
    }
    wave_sync();
#pragma unroll
    for (int e = 0; e < VEC; e += 4) *reinterpret_cast<f32x4 *>(slot + c + e) = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
    wave_sync();
    if (a.pairs % VEC == 0) {
        if (c < 2 * a.pairs) {
            const bool first = c < a.pairs;
            const int j = first ? c : c - a.pairs, other = first ? c + a.pairs : c - a.pairs;
            const float way = first ? -sign : sign;
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
                const f32x4 p = *reinterpret_cast<const f32x4 *>(slot + other + e), co = *reinterpret_cast<const f32x4 *>(cs + j + e), si = *reinterpret_cast<const f32x4 *>(sn + j + e);
#pragma unroll
                for (int f = 0; f < 4; ++f) y[e + f] = y[e + f] * co[f] + way * p[f] * si[f];
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const bool first = c + e < a.pairs;
            if (c + e < 2 * a.pairs) {
                const int j = first ? c + e : c + e - a.pairs, other = first ? c + e + a.pairs : c + e - a.pairs;
                y[e] = y[e] * cs[j] + (first ? -sign : sign) * slot[other] * sn[j];
            }
        }
    }
}

// Angles of the tokens first .. first + kTokens - 1 (those before `last`) to LDS.
__device__ __forceinline__ void angles(const RotaryArgs &a, int64_t first, int64_t last, float (&cs)[kTokens][kMaxPairs], float (&sn)[kTokens][kMaxPairs])
{
    if (a.pairs == 0) return;
    const int count = last - first < kTokens ? (int)(last - first) : kTokens;
    for (int k = threadIdx.x; k < count * a.pairs; k += kRotaryBlock) {
        const int i = k / a.pairs, j = k - i * a.pairs;
        const int64_t token = first + i, b = token / a.length, t = token - b * a.length;
        turn_of(a.positions[b * a.positions_stride + t], a.frequencies[j], cs[i][j], sn[i][j]);
    }
}

template <class T, int L>
__global__ __launch_bounds__(kRotaryBlock) void rotary_forward_kernel(RotaryArgs a, Heads<const T> q, Heads<const T> k, Heads<T> q_out, Heads<T> k_out)
{
    constexpr int VEC = 16 / sizeof(T), kTeams = kRotaryBlock / L;
    __shared__ __attribute__((aligned(16))) float cs[kTokens][kMaxPairs], sn[kTokens][kMaxPairs], slots[kTeams][L * VEC];
    const int particle = blockIdx.x / a.blocks, team = threadIdx.x / L, c = threadIdx.x % L * VEC;
    const int64_t first = (blockIdx.x - particle * a.blocks) * a.per, last = first + a.per < a.tokens ? first + a.per : a.tokens;
    const bool norm = a.q_weight.p != nullptr;
    const float inverse = 1.f / (float)a.dim;
    for (int64_t token0 = first; token0 < last; token0 += kTokens) {
        __syncthreads(); // (the angles before these have been read)
        angles(a, token0, last, cs, sn);
        __syncthreads();
        const int count = last - token0 < kTokens ? (int)(last - token0) : kTokens;
#pragma unroll 1
        for (int kind = 0; kind < 2; ++kind) {
            const Heads<const T> &from = kind ? k : q;
            const Heads<T> &to = kind ? k_out : q_out;
            const Params &weight = kind ? a.k_weight : a.q_weight;
            const int heads = kind ? a.kv : a.heads;
            float w[VEC];
            if (norm) load_pack<float, VEC>(weight.p + particle * weight.stride + c, a.dim - c, w);
            for (int item = team; item < count * heads; item += kTeams) {
                const int i = item / heads, h = item - i * heads;
                const int64_t token = token0 + i;
                const int b = (int)(token / a.length), t = (int)(token - (int64_t)b * a.length);
                float y[VEC];
                load_pack<T, VEC>(from.at(particle, b, h) + t * from.token + c, a.dim - c, y);
                if (norm) {
                    float square = 0.f;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) square += y[e] * y[e];
                    const float rstd = 1.f / sqrtf(head_sum<L>(square) * inverse + a.eps);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) y[e] = y[e] * rstd * w[e];
                }
                turn<VEC>(a, y, c, slots[team], cs[i], sn[i], 1.f);
                if (c < a.dim) store_pack<T, VEC>(to.at(particle, b, h) + t * to.token + c, a.dim - c, y);
            }
        }
    }
}

// partial: the workgroups' sums of the weights' gradients, [particle][workgroup][queries', keys'][dim]; null: not wanted
template <class T, int L>
__global__ __launch_bounds__(kRotaryBlock) void rotary_backward_kernel(RotaryArgs a, Heads<const T> dq_out, Heads<const T> dk_out, Heads<const T> q, Heads<const T> k, Heads<T> dq, Heads<T> dk,
                                                                       float *partial)
{
    constexpr int VEC = 16 / sizeof(T), kTeams = kRotaryBlock / L;
    __shared__ __attribute__((aligned(16))) float cs[kTokens][kMaxPairs], sn[kTokens][kMaxPairs], slots[kTeams][L * VEC];
    const int particle = blockIdx.x / a.blocks, team = threadIdx.x / L, c = threadIdx.x % L * VEC;
    const int64_t first = (blockIdx.x - particle * a.blocks) * a.per, last = first + a.per < a.tokens ? first + a.per : a.tokens;
    const bool norm = a.q_weight.p != nullptr;
    const float inverse = 1.f / (float)a.dim;
    float dw[2][VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[0][e] = dw[1][e] = 0.f;
    for (int64_t token0 = first; token0 < last; token0 += kTokens) {
        __syncthreads();
        angles(a, token0, last, cs, sn);
        __syncthreads();
        const int count = last - token0 < kTokens ? (int)(last - token0) : kTokens;
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
            const Heads<const T> &dy = kind ? dk_out : dq_out, &from = kind ? k : q;
            const Heads<T> &to = kind ? dk : dq;
            const Params &weight = kind ? a.k_weight : a.q_weight;
            const int heads = kind ? a.kv : a.heads;
            float w[VEC];
            if (norm) load_pack<float, VEC>(weight.p + particle * weight.stride + c, a.dim - c, w);
            for (int item = team; item < count * heads; item += kTeams) {
                const int i = item / heads, h = item - i * heads;
                const int64_t token = token0 + i;
                const int b = (int)(token / a.length), t = (int)(token - (int64_t)b * a.length);
                float g[VEC], x[VEC];
                load_pack<T, VEC>(dy.at(particle, b, h) + t * dy.token + c, a.dim - c, g);
                if (norm) load_pack<T, VEC>(from.at(particle, b, h) + t * from.token + c, a.dim - c, x);
                turn<VEC>(a, g, c, slots[team], cs[i], sn[i], -1.f);
                if (norm) {
                    float square = 0.f, mean = 0.f;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        square += x[e] * x[e];
                        mean += g[e] * w[e] * x[e];
                    }
                    const float rstd = 1.f / sqrtf(head_sum<L>(square) * inverse + a.eps);
                    mean = head_sum<L>(mean) * inverse * rstd; // of a xhat
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float xhat = x[e] * rstd;
                        dw[kind][e] += g[e] * xhat;
                        g[e] = rstd * (g[e] * w[e] - xhat * mean);
                    }
                }
                if (to.p && c < a.dim) store_pack<T, VEC>(to.at(particle, b, h) + t * to.token + c, a.dim - c, g);
            }
        }
    }
    if (!partial) return;
    // the teams' sums, in their order
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < VEC; ++e) slots[team][c + e] = dw[kind][e];
        __syncthreads();
        for (int d = threadIdx.x; d < a.dim; d += kRotaryBlock) {
            float sum = 0.f;
            for (int m = 0; m < kTeams; ++m) sum += slots[m][d];
            partial[((int64_t)blockIdx.x * 2 + kind) * a.dim + d] = sum;
        }
    }
}

} // namespace svgd
