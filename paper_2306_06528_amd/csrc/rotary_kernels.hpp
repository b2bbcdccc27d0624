// Norms of queries and keys, head by head, with the rotation by position in the same pass, forward and backward.  A team of L lanes holds a
// head, 16 bytes a lane, from its one load to its one store; memory bounds both passes.  A workgroup has some tokens of one particle: their
// angles are formed in 64 bits once for all heads (kTokens tokens at a time, to LDS), and the weights and their gradients stay in
// registers.  In the half layout a value's partner is another lane's: the team's values change lanes in its part of LDS. 8 x 2 x 4,096 x 20
// heads of 128 bf16: forward 157 us (671 MB, 4.3 TB/s), backward 234 (1,007 MB, 4.3 TB/s); 8 x 8 x 197 x 12 heads of 64, in the memory-side
// cache: 16.7 and 26.5, bound by the formation of angles, 64-bit, and by the latency of a team's loads, one head ahead.
#pragma once
#include "attention_common.hpp"

namespace svgd {

constexpr int kTokens = 8, kRotaryBlock = 256;
constexpr int kMaxPairs = SVGD_ROTARY_MAX_DIM / 2;

struct RotaryArgs {
    int dim, pairs, interleaved;
    int length;
    int64_t tokens; // batch length: of a particle
    const double *frequencies;
    const int64_t *positions;
    int64_t positions_stride;
    float eps;
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

// What a pass reads and writes of queries (0) and of keys (1): read from the kernel's arguments by number, so that only one of them takes
// scalar registers at a time.
template <class T> struct RotaryKind {
    Heads<const T> x, dy; // backward; forward x alone
    Heads<T> to;
    Params weight;
    int heads;
};
template <class T> struct RotaryKinds {
    RotaryKind<T> of[2];
};

// A lane's 16 bytes of a head as they come from memory, 0 behind the head's end.  WHOLE: heads end with such a piece.
template <class T, bool WHOLE> struct HeadPiece {
    static constexpr int VEC = 16 / sizeof(T);
    typename Pack<T, VEC>::raw v;
    __device__ __forceinline__ void load(const T *head, int c, int dim)
    {
        if constexpr (WHOLE) {
            v = *reinterpret_cast<const typename Pack<T, VEC>::type *>(head + (c < dim ? c : 0));
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = head[c + e < dim ? c + e : 0];
        }
    }
    __device__ __forceinline__ void get(float (&y)[VEC], int c, int dim) const
    {
#pragma unroll
        for (int e = 0; e < VEC; ++e) y[e] = (WHOLE ? c : c + e) < dim ? (float)v[e] : 0.f;
    }
    static __device__ __forceinline__ void store(T *head, int c, int dim, const float (&y)[VEC])
    {
        if (c < dim) store_pack<T, VEC>(head + c, WHOLE ? VEC : dim - c, y);
    }
};

// The heads of `count` tokens from token0 on, dealt to the teams one after the other.  From one of a team's to its next one it is `tokens`
// tokens and `more` heads, and at the end of a token's heads or of a sequence a step back: pointers are moved on by sums (as products of 64
// bits addresses took a third of the instructions).
struct HeadTurn {
    int items, heads, length, teams, item, tokens, more;
    int i, t, h; // the token's number among them, of its sequence; head
    int b;
    __device__ __forceinline__ HeadTurn(const RotaryArgs &a, int64_t token0, int count, int heads_, int team, int teams_)
        : items(count * heads_), heads(max(heads_, 1)), length(a.length), teams(teams_), item(team)
    {
        tokens = teams / heads;
        more = teams - tokens * heads;
        i = (uint32_t)item / (uint32_t)heads;
        h = item - i * heads;
        const int64_t token = token0 + i;
        b = (int)(token / length);
        t = (int)(token - (int64_t)b * length);
    }
    __device__ __forceinline__ bool any() const { return item < items; }
};
template <class P> struct HeadPointer {
    P *p;
    int64_t step, carry, wrap;
    __device__ __forceinline__ HeadPointer(P *base, const Heads<P> &s, const HeadTurn &at)
        : p(base + at.b * s.batch + at.t * s.token + at.h * s.head), step(at.tokens * s.token + at.more * s.head), carry(s.token - at.heads * s.head), wrap(s.batch - at.length * s.token)
    {
    }
};
template <class... Ps> __device__ __forceinline__ void next_head(HeadTurn &at, HeadPointer<Ps> &...ps)
{
    at.item += at.teams;
    at.i += at.tokens;
    at.t += at.tokens;
    at.h += at.more;
    ((ps.p += ps.step), ...);
    if (at.h >= at.heads) {
        at.h -= at.heads;
        ++at.i;
        ++at.t;
        ((ps.p += ps.carry), ...);
    }
    while (at.t >= at.length) { // (mostly not once; with a single head in sequences of one token as often as there are teams)
        at.t -= at.length;
        ((ps.p += ps.wrap), ...);
    }
}

template <class T, int L, bool WHOLE> __global__ __launch_bounds__(kRotaryBlock) void rotary_forward_kernel(RotaryArgs a, RotaryKinds<T> kinds)
{
    constexpr int VEC = 16 / sizeof(T), kTeams = kRotaryBlock / L;
    __shared__ __attribute__((aligned(16))) float cs[kTokens][kMaxPairs], sn[kTokens][kMaxPairs], slots[kTeams][L * VEC];
    const int particle = blockIdx.x / a.blocks, team = threadIdx.x / L, c = threadIdx.x % L * VEC;
    const int64_t first = (blockIdx.x - particle * a.blocks) * a.per, last = first + a.per < a.tokens ? first + a.per : a.tokens;
    const float inverse = 1.f / (float)a.dim;
    for (int64_t token0 = first; token0 < last; token0 += kTokens) {
        __syncthreads(); // (the angles before these have been read)
        angles(a, token0, last, cs, sn);
        __syncthreads();
        const int count = last - token0 < kTokens ? (int)(last - token0) : kTokens;
#pragma unroll 1
        for (int kind = 0; kind < 2; ++kind) {
            const RotaryKind<T> &k = kinds.of[kind];
            const bool norm = k.weight.p != nullptr;
            float w[VEC];
            if (norm) load_pack<float, VEC>(k.weight.p + particle * k.weight.stride + c, a.dim - c, w);
            // (the next head is on its way while one is worked on)
            HeadTurn at(a, token0, count, k.heads, team, kTeams);
            HeadPointer<const T> from(k.x.p + particle * k.x.particle, k.x, at);
            HeadPointer<T> to(k.to.p + particle * k.to.particle, k.to, at);
            HeadPiece<T, WHOLE> next;
            if (at.any()) next.load(from.p, c, a.dim);
            while (at.any()) {
                float y[VEC];
                next.get(y, c, a.dim);
                const int i = at.i;
                T *const out = to.p;
                next_head(at, from, to);
                if (at.any()) next.load(from.p, c, a.dim);
                if (norm) {
                    float square = 0.f;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) square += y[e] * y[e];
                    const float rstd = __builtin_amdgcn_rsqf(head_sum<L>(square) * inverse + a.eps);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) y[e] = y[e] * rstd * w[e];
                }
                turn<VEC>(a, y, c, slots[team], cs[i], sn[i], 1.f);
                HeadPiece<T, WHOLE>::store(out, c, a.dim, y);
            }
        }
    }
}

// partial: the workgroups' sums of the weights' gradients, [particle][workgroup][queries', keys'][dim]; null: not wanted
template <class T, int L, bool WHOLE> __global__ __launch_bounds__(kRotaryBlock) void rotary_backward_kernel(RotaryArgs a, RotaryKinds<T> kinds, float *partial)
{
    constexpr int VEC = 16 / sizeof(T), kTeams = kRotaryBlock / L;
    __shared__ __attribute__((aligned(16))) float cs[kTokens][kMaxPairs], sn[kTokens][kMaxPairs], slots[kTeams][L * VEC];
    const int particle = blockIdx.x / a.blocks, team = threadIdx.x / L, c = threadIdx.x % L * VEC;
    const int64_t first = (blockIdx.x - particle * a.blocks) * a.per, last = first + a.per < a.tokens ? first + a.per : a.tokens;
    const float inverse = 1.f / (float)a.dim;
    float dw[2][VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[0][e] = dw[1][e] = 0.f;
    for (int64_t token0 = first; token0 < last; token0 += kTokens) {
        __syncthreads();
        angles(a, token0, last, cs, sn);
        __syncthreads();
        const int count = last - token0 < kTokens ? (int)(last - token0) : kTokens;
#pragma unroll 1
        for (int kind = 0; kind < 2; ++kind) {
            const RotaryKind<T> &k = kinds.of[kind];
            const bool norm = k.weight.p != nullptr, store = k.to.p != nullptr;
            float w[VEC], d[VEC];
            if (norm) load_pack<float, VEC>(k.weight.p + particle * k.weight.stride + c, a.dim - c, w);
#pragma unroll
            for (int e = 0; e < VEC; ++e) d[e] = kind ? dw[1][e] : dw[0][e];
            HeadTurn at(a, token0, count, k.heads, team, kTeams);
            HeadPointer<const T> from(k.x.p + particle * k.x.particle, k.x, at), dy(k.dy.p + particle * k.dy.particle, k.dy, at);
            HeadPointer<T> to(k.to.p + particle * k.to.particle, k.to, at);
            HeadPiece<T, WHOLE> next_g, next_x;
            const auto fetch = [&] {
                if (!at.any()) return;
                next_g.load(dy.p, c, a.dim);
                if (norm) next_x.load(from.p, c, a.dim);
            };
            fetch();
            while (at.any()) {
                float g[VEC], x[VEC];
                next_g.get(g, c, a.dim);
                if (norm) next_x.get(x, c, a.dim);
                const int i = at.i;
                T *const out = to.p;
                next_head(at, from, dy, to);
                fetch();
                turn<VEC>(a, g, c, slots[team], cs[i], sn[i], -1.f);
                if (norm) {
                    float square = 0.f, mean = 0.f;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        square += x[e] * x[e];
                        mean += g[e] * w[e] * x[e];
                    }
                    const float rstd = __builtin_amdgcn_rsqf(head_sum<L>(square) * inverse + a.eps);
                    mean = head_sum<L>(mean) * inverse * rstd; // of a xhat
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float xhat = x[e] * rstd;
                        d[e] += g[e] * xhat;
                        g[e] = rstd * (g[e] * w[e] - xhat * mean);
                    }
                }
                if (store) HeadPiece<T, WHOLE>::store(out, c, a.dim, g);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                dw[0][e] = kind ? dw[0][e] : d[e];
                dw[1][e] = kind ? d[e] : dw[1][e];
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
