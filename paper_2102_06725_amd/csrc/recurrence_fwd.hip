// recurrence_fwd.hip -- forward pass of the gated linear recurrence.
#include "recurrence.hpp"

namespace nnconv {

namespace {

// Few tokens: a lane walks them all.
template <class T>
__global__ __launch_bounds__(64) void recurrence_fwd_short_kernel(const RecParams p) {
    const int lane = threadIdx.x;
    const Lane L(blockIdx.x * COLS + 2 * lane, p.c);
    for (int64_t n = blockIdx.y; n < p.n; n += gridDim.y) {
        const int len = length_of(p, (int)n);
        float h[2] = {0.f, 0.f}, bias[2] = {0.f, 0.f};
        if (p.h0) {
            h[0] = p.h0[n * p.c + L.k0];
            h[1] = p.h0[n * p.c + L.k1];
        }
        if (p.bias) {
            bias[0] = p.bias[L.k0] * -LOG2E;
            bias[1] = p.bias[L.k1] * -LOG2E;
        }
        const int64_t at = n * p.t * p.ld;
        const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
        const uint16_t *g = p.g ? (const uint16_t *)p.g + at : nullptr;
        uint16_t *y = (uint16_t *)p.y + n * p.t * p.ldy;
        if (p.saved && p.t > 0) {  // t <= SAVE: one state
            put2(p.saved + n * p.c, L, h[0], h[1]);
        }
        for (int t = 0; t < p.t; ++t) {
            float o[2] = {0.f, 0.f};
            if (t < len) {
                float xv[2], fv[2], gv[2];
                unpack<T>(load2(x + t * p.ld, L), xv);
                unpack<T>(load2(f + t * p.ld, L), fv);
                if (g) unpack<T>(load2(g + t * p.ld, L), gv);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float a, b;
                    gate(fv[k], bias[k], a, b);
                    h[k] = a * h[k] + b * xv[k];
                    o[k] = g ? h[k] * (gv[k] * sigma(gv[k])) : h[k];
                }
            }
            void *const row[1] = {y + t * p.ldy};
            store2<T, 1>(row, L, false, &o);
        }
        if (p.ht) put2(p.ht + n * p.c, L, h[0], h[1]);
    }
}

// The pair of a chunk, walked token by token with the arithmetic of the kernel below.
template <class T, int W, int S>
__device__ void walk_fwd(const RecParams &p, int64_t n, const Lane &L, int lo, int len,
                         const float bias[2], float A[2], float H[2]) {
    const int64_t at = n * p.t * p.ld;
    const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
    A[0] = A[1] = 1.f;
    H[0] = H[1] = 0.f;
    for (int w = 0; w < W; ++w) {
        float a1[2] = {1.f, 1.f}, h1[2] = {0.f, 0.f};
        for (int t = lo + w * S; t < min(lo + w * S + S, len); ++t) {
            float xv[2], fv[2];
            unpack<T>(load2(x + t * p.ld, L), xv);
            unpack<T>(load2(f + t * p.ld, L), fv);
            for (int k = 0; k < 2; ++k) {
                float a, b;
                gate(fv[k], bias[k], a, b);
                h1[k] = __builtin_fmaf(a, h1[k], b * xv[k]);
                a1[k] *= a;
            }
        }
        a1[0] = fmaxf(a1[0], A_MIN);
        a1[1] = fmaxf(a1[1], A_MIN);
        compose(A, H, a1, h1);
    }
}

// A chunk.  Fewer waves than the most: the only one.
template <class T, bool G, int W, int S, int NG>
__global__ __launch_bounds__(64 * W, 4) void recurrence_fwd_kernel(const RecParams p, const RecGrid q) {
    static_assert(SAVE % S == 0, "saved states lie at a team's first token");
    constexpr bool U = NG == 1;
    constexpr int TEAMS = W * NG, CHUNK = TEAMS * S;
    const Team<NG> team;
    const int w = team.w;
    const int col = blockIdx.x % q.cols, rest = blockIdx.x / q.cols;
    const int n = rest % p.n, chunk = rest / p.n;
    const Lane L(2 * (col * team.LANES + team.c), p.c);
    const int len = length_of(p, n);
    const int t0 = chunk * CHUNK + team.r * S, last = len > 0 ? len - 1 : 0;
    const int64_t at = (int64_t)n * p.t * p.ld;
    const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
    const uint16_t *g = G ? (const uint16_t *)p.g + at : nullptr;
    uint32_t xr[S], fr[S], gr[S];
    const bool whole = t0 + S <= len;           // every token takes part
    const bool full = (col + 1) * 2 * team.LANES <= p.c;  // every channel exists
    int64_t o = (int64_t)min(t0, last) * p.ld;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        xr[s] = load2<U>(x + o, L);
        fr[s] = load2<U>(f + o, L);
        o += t0 + s < last ? p.ld : 0;
    }
    float bias[2] = {0.f, 0.f};
    if (p.bias) {
        bias[0] = p.bias[L.k0] * -LOG2E;
        bias[1] = p.bias[L.k1] * -LOG2E;
    }
    float a[S][2], u[S][2], A[2] = {1.f, 1.f}, H[2] = {0.f, 0.f};
#pragma unroll
    for (int s = 0; s < S; ++s) {
        float xv[2], fv[2];
        unpack<T>(xr[s], xv);
        unpack<T>(fr[s], fv);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float b;
            gate(fv[k], bias[k], a[s][k], b);
            u[s][k] = b * xv[k];
        }
    }
    if (!whole)
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (t0 + s >= len) {
                    a[s][k] = 1.f;
                    u[s][k] = 0.f;
                }
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            H[k] = __builtin_fmaf(a[s][k], H[k], u[s][k]);
            A[k] *= a[s][k];
        }
    A[0] = fmaxf(A[0], A_MIN);
    A[1] = fmaxf(A[1], A_MIN);
    float h[2] = {0.f, 0.f};
    if (!q.words && p.h0) {  // before the barrier: ht, which another wave writes, may lie on it
        h[0] = p.h0[(int64_t)n * p.c + L.k0];
        h[1] = p.h0[(int64_t)n * p.c + L.k1];
    }
    __shared__ f32x4 part[W * 64];
    part[threadIdx.x] = f32x4{A[0], H[0], A[1], H[1]};
    __syncthreads();
    if (G) {  // not needed before the state is there: on their way during the wait
        o = (int64_t)min(t0, last) * p.ld;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            gr[s] = load2<U>(g + o, L);
            o += t0 + s < last ? p.ld : 0;
        }
    }
    // what the teams in front make of the chunk's first state
    float pa[2] = {1.f, 1.f}, ph[2] = {0.f, 0.f};
    for (int v = 0; v < w * NG + NG - 1; ++v) {
        if (v >= team.r) continue;
        const f32x4 e = part[team.of(v)];
        const float ea[2] = {e[0], e[2]}, eh[2] = {e[1], e[3]};
        compose(pa, ph, ea, eh);
    }
    if constexpr (W == FWD_WAVES) if (q.words) {
        float ca[2] = {pa[0], pa[1]}, ch[2] = {ph[0], ph[1]};
        compose(ca, ch, A, H);
        if (NG > 1)  // the last team's is the chunk's
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                ca[k] = __shfl(ca[k], 64 - team.LANES + team.c);
                ch[k] = __shfl(ch[k], 64 - team.LANES + team.c);
            }
        carry_in<W>(q, n, p.c, chunk, L, team.first_of_wave(), w, W - 1, ca, ch, [&](int place, float *a2, float *h2) {
            walk_fwd<T, TEAMS, S>(p, n, L, place * CHUNK, len, bias, a2, h2);
        }, h);
    }
    h[0] = pa[0] * h[0] + ph[0];
    h[1] = pa[1] * h[1] + ph[1];
    if (p.saved && t0 % SAVE == 0 && t0 < p.t) {
        float *to = p.saved + ((int64_t)n * ((p.t + SAVE - 1) / SAVE) + t0 / SAVE) * p.c;
        put2(to, L, h[0], h[1]);
    }
    uint16_t *y = (uint16_t *)p.y + (int64_t)n * p.t * p.ldy;
    y += (int64_t)t0 * p.ldy;
    auto finish = [&](auto checked) {
#pragma unroll
        for (int s = 0; s < S; ++s, y += p.ldy) {
            const int t = t0 + s;
            float o[2], gv[2];
            if (G) unpack<T>(gr[s], gv);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                h[k] = a[s][k] * h[k] + u[s][k];
                o[k] = G ? h[k] * (gv[k] * sigma(gv[k])) : h[k];
                if (checked && t >= len) o[k] = 0.f;
            }
            void *const row[1] = {y};
            if (!checked || t < p.t) store2<T, 1, U>(row, L, !checked, &o);
        }
    };
    if (team.all(whole) && full)
        finish(std::false_type{});
    else
        finish(std::true_type{});
    if (p.ht && chunk == q.chunks - 1 && team.r == TEAMS - 1) put2(p.ht + (int64_t)n * p.c, L, h[0], h[1]);
}

// ---- one channel: no pairs to load, a lane per sequence walks its tokens ---------

template <class T>
__global__ __launch_bounds__(64) void recurrence_fwd_single_kernel(const RecParams p) {
    const int64_t n = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (n >= p.n) return;
    const int len = length_of(p, (int)n);
    const float bias = p.bias ? p.bias[0] * -LOG2E : 0.f;
    float h = p.h0 ? p.h0[n] : 0.f;
    const uint16_t *x = (const uint16_t *)p.x + n * p.t * p.ld, *f = (const uint16_t *)p.f + n * p.t * p.ld;
    const uint16_t *g = p.g ? (const uint16_t *)p.g + n * p.t * p.ld : nullptr;
    uint16_t *y = (uint16_t *)p.y + n * p.t * p.ldy;
    for (int64_t t = 0; t < p.t; ++t) {
        if (p.saved && t % SAVE == 0) p.saved[n * ((p.t + SAVE - 1) / SAVE) + t / SAVE] = h;
        float o = 0.f;
        if (t < len) {
            float a, b;
            gate(from16<T>(f[t * p.ld]), bias, a, b);
            h = a * h + b * from16<T>(x[t * p.ld]);
            o = h;
            if (g) {
                const float gv = from16<T>(g[t * p.ld]);
                o = h * (gv * sigma(gv));
            }
        }
        y[t * p.ldy] = (uint16_t)to16<T>(o);
    }
    if (p.ht) p.ht[n] = h;
}

}  // namespace

void launch_recurrence_fwd_chunks(int dtype, const RecParams &p, const RecGrid &q, uint32_t blocks, hipStream_t st) {
    with_kind(dtype, p.g != nullptr, [&](auto t, auto g) {
        auto go = [&](auto waves, auto teams) {
            hipLaunchKernelGGL((recurrence_fwd_kernel<decltype(t), decltype(g)::value, decltype(waves)::value, TOKENS, decltype(teams)::value>),
                               dim3(blocks), dim3(64 * decltype(waves)::value), 0, st, p, q);
        };
        auto several = [&](auto teams) {
            if (q.waves == 1) go(Int<1>{}, teams); else go(Int<FWD_WAVES>{}, teams);
        };
        if (q.teams == 8) return several(Int<8>{});
        if (q.teams == 4) return several(Int<4>{});
        if (q.teams == 2) return several(Int<2>{});
        if (q.waves == 2) return go(Int<2>{}, Int<1>{});
        if (q.waves == 4) return go(Int<4>{}, Int<1>{});
        several(Int<1>{});
    });
}

void launch_recurrence_fwd_short(int dtype, const RecParams &p, hipStream_t st) {
    with_kind(dtype, true, [&](auto t, auto) {
        hipLaunchKernelGGL((recurrence_fwd_short_kernel<decltype(t)>), short_grid(p), dim3(64), 0, st, p);
    });
}

void launch_recurrence_fwd_single(int dtype, const RecParams &p, hipStream_t st) {
    with_kind(dtype, true, [&](auto t, auto) {
        hipLaunchKernelGGL((recurrence_fwd_single_kernel<decltype(t)>), dim3((uint32_t)(((int64_t)p.n + 63) / 64)), dim3(64), 0, st, p);
    });
}

}  // namespace nnconv
