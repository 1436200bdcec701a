// recurrence_bwd.hip -- backward pass of the gated linear recurrence.
#include "recurrence.hpp"

namespace nnconv {

namespace {

// With own_t = dy_t g_t sigma(g_t), the gradient of h_t is d_t = own_t + r_t, where r_t flows
// in from the right: r_(t-1) = a_t d_t.  So r obeys the same kind of recurrence from the last
// token on, with a_t and a_t own_t.

// r in front of a token; not fused with the product that own is, so that every place that
// computes it gets the same bits.
__device__ __forceinline__ float before_token(float a, float own, float r) {
#pragma clang fp contract(off)
    return a * (own + r);
}

template <class T, bool G>
struct Grad {
    float a[2], b[2], x[2], own[2], dg[2];  // dg without the factor h_t

    __device__ __forceinline__ void make(uint32_t xq, uint32_t fq, uint32_t gq, uint32_t dyq, const float bias[2]) {
        float fv[2], gv[2], dy[2];
        unpack<T>(xq, x);
        unpack<T>(fq, fv);
        unpack<T>(dyq, dy);
        if (G) unpack<T>(gq, gv);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            gate(fv[k], bias[k], a[k], b[k]);
            own[k] = dy[k];
            dg[k] = 0.f;
            if (G) {
                const float s = sigma(gv[k]), sg = gv[k] * s;
                own[k] = dy[k] * sg;
                dg[k] = dy[k] * (s + sg * (1.f - s));
            }
        }
    }

    // A token past the length: the state passes through, nothing else happens.
    __device__ __forceinline__ void pass() {
        a[0] = a[1] = 1.f;
        b[0] = b[1] = x[0] = x[1] = own[0] = own[1] = dg[0] = dg[1] = 0.f;
    }
};

// Few tokens: a lane walks them all, forward for the states (t <= SHORT_T of them, in LDS) and
// back.
template <class T, bool G>
__global__ __launch_bounds__(64) void recurrence_bwd_short_kernel(const RecParams p) {
    __shared__ float hs[SHORT_T][2][64];
    const int lane = threadIdx.x;
    const Lane L(blockIdx.x * COLS + 2 * lane, p.c);
    float bias[2] = {0.f, 0.f};
    if (p.bias) {
        bias[0] = p.bias[L.k0] * -LOG2E;
        bias[1] = p.bias[L.k1] * -LOG2E;
    }
    for (int64_t n = blockIdx.y; n < p.n; n += gridDim.y) {
        const int len = length_of(p, (int)n);
        float r[2] = {0.f, 0.f}, total[2] = {0.f, 0.f};
        if (p.dht) {
            r[0] = p.dht[n * p.c + L.k0];
            r[1] = p.dht[n * p.c + L.k1];
        }
        const int64_t at = n * p.t * p.ld;
        const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
        const uint16_t *g = G ? (const uint16_t *)p.g + at : nullptr;
        const uint16_t *dy = (const uint16_t *)p.dy + n * p.t * p.ldy;
        uint16_t *dx = (uint16_t *)p.dx + at, *df = (uint16_t *)p.df + at;
        uint16_t *dg = G ? (uint16_t *)p.dg + at : nullptr;
        if (len > 0) {
            float h[2] = {p.saved[n * p.c + L.k0], p.saved[n * p.c + L.k1]};
            for (int t = 0; t < len; ++t) {
                float xv[2], fv[2];
                unpack<T>(load2(x + t * p.ld, L), xv);
                unpack<T>(load2(f + t * p.ld, L), fv);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float a, b;
                    gate(fv[k], bias[k], a, b);
                    hs[t][k][lane] = h[k];
                    h[k] = a * h[k] + b * xv[k];
                }
            }
        }
        for (int t = p.t - 1; t >= 0; --t) {
            float out[3][2] = {{0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}};  // dx, df, dg
            if (t < len) {
                Grad<T, G> e;
                e.make(load2(x + t * p.ld, L), load2(f + t * p.ld, L),
                       G ? load2(g + t * p.ld, L) : 0u, load2(dy + t * p.ldy, L), bias);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float before = hs[t][k][lane], d = e.own[k] + r[k];
                    out[0][k] = d * e.b[k];
                    out[1][k] = d * (before - e.x[k]) * (e.a[k] * e.b[k]);
                    if (G) out[2][k] = e.dg[k] * (e.a[k] * before + e.b[k] * e.x[k]);
                    r[k] = e.a[k] * d;
                    total[k] += out[1][k];
                }
            }
            void *const row[3] = {dx + t * p.ld, df + t * p.ld, dg + t * p.ld};
            store2<T, G ? 3 : 2>(row, L, false, out);
        }
        if (p.dh0) put2(p.dh0 + n * p.c, L, r[0], r[1]);
        if (p.part) put2(p.part + n * p.c, L, total[0], total[1]);
    }
}

// The pair of a chunk for r, walked from its last token on with the arithmetic of the kernel
// below.
template <class T, bool G, int W, int S>
__device__ void walk_bwd(const RecParams &p, int64_t n, const Lane &L, int lo, int len,
                         const float bias[2], float A[2], float R[2]) {
    const int64_t at = n * p.t * p.ld;
    const uint16_t *f = (const uint16_t *)p.f + at;
    const uint16_t *g = G ? (const uint16_t *)p.g + at : nullptr;
    const uint16_t *dy = (const uint16_t *)p.dy + n * p.t * p.ldy;
    A[0] = A[1] = 1.f;
    R[0] = R[1] = 0.f;
    for (int w = W - 1; w >= 0; --w) {
        float a1[2] = {1.f, 1.f}, r1[2] = {0.f, 0.f};
        const int first = lo + w * S;
        for (int t = first; t < min(first + S, len); ++t)
            for (int k = 0; k < 2; ++k) {  // the product in the order of the tokens
                float fv[2], a, b;
                unpack<T>(load2(f + t * p.ld, L), fv);
                gate(fv[k], bias[k], a, b);
                a1[k] *= a;
            }
        for (int t = min(first + S, len) - 1; t >= first; --t) {
            Grad<T, G> e;
            e.make(0u, load2(f + t * p.ld, L), G ? load2(g + t * p.ld, L) : 0u,
                   load2(dy + t * p.ldy, L), bias);
            for (int k = 0; k < 2; ++k) r1[k] = before_token(e.a[k], e.own[k], r1[k]);
        }
        a1[0] = fmaxf(a1[0], A_MIN);
        a1[1] = fmaxf(a1[1], A_MIN);
        compose(A, R, a1, r1);
    }
}

// A chunk.  Fewer waves than the most: the only one.
template <class T, bool G, int W, int S, int NG>
__global__ __launch_bounds__(64 * W, 2) void recurrence_bwd_kernel(const RecParams p, const RecGrid q) {
    static_assert((W < BWD_WAVES || (W * S) % SAVE == 0) && SAVE % S == 0, "chunks are whole saved stretches");
    constexpr int RUN = SAVE / S;  // teams that start from one saved state
    constexpr bool U = NG == 1;
    constexpr int TEAMS = W * NG, CHUNK = TEAMS * S;
    const Team<NG> team;
    const int w = team.w;
    const int col = blockIdx.x % q.cols, rest = blockIdx.x / q.cols;
    const int n = rest % p.n, place = rest / p.n, chunk = q.chunks - 1 - place;  // the last one first
    const Lane L(2 * (col * team.LANES + team.c), p.c);
    const int len = length_of(p, n);
    const int t0 = chunk * CHUNK + team.r * S, last = len > 0 ? len - 1 : 0;
    const int64_t at = (int64_t)n * p.t * p.ld;
    const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
    const uint16_t *g = G ? (const uint16_t *)p.g + at : nullptr;
    const uint16_t *dy = (const uint16_t *)p.dy + (int64_t)n * p.t * p.ldy;
    uint32_t xr[S], fr[S], gr[S], dr[S];
    const bool whole = t0 + S <= len;           // every token takes part
    const bool full = (col + 1) * 2 * team.LANES <= p.c;  // every channel exists
    int64_t o = (int64_t)min(t0, last) * p.ld;
    dy += (int64_t)min(t0, last) * p.ldy;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        xr[s] = load2<U>(x + o, L);
        fr[s] = load2<U>(f + o, L);
        gr[s] = G ? load2<U>(g + o, L) : 0u;
        dr[s] = load2<U>(dy, L);
        o += t0 + s < last ? p.ld : 0;
        dy += t0 + s < last ? p.ldy : 0;
    }
    float h[2] = {0.f, 0.f}, bias[2] = {0.f, 0.f};
    const int run0 = t0 - team.r % RUN * S;  // first token of the saved stretch
    if (run0 < p.t) {
        const float *from = p.saved + ((int64_t)n * ((p.t + SAVE - 1) / SAVE) + run0 / SAVE) * p.c;
        h[0] = from[L.k0];
        h[1] = from[L.k1];
    }
    if (p.bias) {
        bias[0] = p.bias[L.k0] * -LOG2E;
        bias[1] = p.bias[L.k1] * -LOG2E;
    }
    Grad<T, G> e[S];
    float A[2] = {1.f, 1.f}, H[2] = {0.f, 0.f}, R[2] = {0.f, 0.f};
#pragma unroll
    for (int s = 0; s < S; ++s) {
        e[s].make(xr[s], fr[s], gr[s], dr[s], bias);
        if (!whole && t0 + s >= len) e[s].pass();
    }
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            H[k] = e[s].a[k] * H[k] + e[s].b[k] * e[s].x[k];
            A[k] *= e[s].a[k];
        }
#pragma unroll
    for (int s = S - 1; s >= 0; --s)
#pragma unroll
        for (int k = 0; k < 2; ++k) R[k] = before_token(e[s].a[k], e[s].own[k], R[k]);
    A[0] = fmaxf(A[0], A_MIN);
    A[1] = fmaxf(A[1], A_MIN);
    float r[2] = {0.f, 0.f};
    if (!q.words && p.dht) {  // before the barrier: dh0, which another wave writes, may lie on it
        r[0] = p.dht[(int64_t)n * p.c + L.k0];
        r[1] = p.dht[(int64_t)n * p.c + L.k1];
    }
    __shared__ f32x4 part[W * 64];
    __shared__ float part_r[2][W * 64];
    part[threadIdx.x] = f32x4{A[0], H[0], A[1], H[1]};
    part_r[0][threadIdx.x] = R[0];
    part_r[1][threadIdx.x] = R[1];
    __syncthreads();
    for (int k = 0; k < RUN - 1; ++k) {
        const int v = team.r - team.r % RUN + k;
        if (v >= team.r) continue;
        const f32x4 m = part[team.of(v)];
        h[0] = m[0] * h[0] + m[1];
        h[1] = m[2] * h[1] + m[3];
    }
    // what the teams behind make of the gradient that flows into the chunk
    float pa[2] = {1.f, 1.f}, pr[2] = {0.f, 0.f};
    for (int v = TEAMS - 1; v > w * NG; --v) {
        if (v <= team.r) continue;
        const f32x4 m = part[team.of(v)];
        const float ma[2] = {m[0], m[2]}, mr[2] = {part_r[0][team.of(v)], part_r[1][team.of(v)]};
        compose(pa, pr, ma, mr);
    }
    if constexpr (W == BWD_WAVES) if (q.words) {
        float ca[2] = {pa[0], pa[1]}, cr[2] = {pr[0], pr[1]};
        compose(ca, cr, A, R);
        if (NG > 1)  // the first team's is the chunk's
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                ca[k] = __shfl(ca[k], team.c);
                cr[k] = __shfl(cr[k], team.c);
            }
        carry_in<W>(q, n, p.c, place, L, team.first_of_wave(), w, 0, ca, cr, [&](int at2, float *a2, float *r2) {
            walk_bwd<T, G, TEAMS, S>(p, n, L, (q.chunks - 1 - at2) * CHUNK, len, bias, a2, r2);
        }, r);
    }
    r[0] = pa[0] * r[0] + pr[0];
    r[1] = pa[1] * r[1] + pr[1];
    float before[S][2];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            before[s][k] = h[k];
            h[k] = e[s].a[k] * h[k] + e[s].b[k] * e[s].x[k];
        }
    uint16_t *dx = (uint16_t *)p.dx + at, *df = (uint16_t *)p.df + at;
    uint16_t *dg = G ? (uint16_t *)p.dg + at : nullptr;
    float total[2] = {0.f, 0.f};
    o = (int64_t)(t0 + S - 1) * p.ld;
    auto finish = [&](auto checked) {
#pragma unroll
        for (int s = S - 1; s >= 0; --s, o -= p.ld) {
            const int t = t0 + s;
            float out[3][2];  // dx, df, dg
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Grad<T, G> &m = e[s];
                const float d = m.own[k] + r[k];
                out[0][k] = d * m.b[k];
                out[1][k] = d * (before[s][k] - m.x[k]) * (m.a[k] * m.b[k]);
                out[2][k] = m.dg[k] * (m.a[k] * before[s][k] + m.b[k] * m.x[k]);
                if (checked && t >= len) out[0][k] = out[1][k] = out[2][k] = 0.f;
                r[k] = m.a[k] * d;
                total[k] += out[1][k];
            }
            void *const row[3] = {dx + o, df + o, dg + o};
            if (!checked || t < p.t) store2<T, G ? 3 : 2, U>(row, L, !checked, out);
        }
    };
    if (team.all(whole) && full)
        finish(std::false_type{});
    else
        finish(std::true_type{});
    if (p.dh0 && chunk == 0 && team.r == 0) put2(p.dh0 + (int64_t)n * p.c, L, r[0], r[1]);
    if (p.part) {
        __syncthreads();
        part_r[0][threadIdx.x] = total[0];
        part_r[1][threadIdx.x] = total[1];
        __syncthreads();
        if (w != 0 || !team.first_of_wave()) return;
        for (int v = 1; v < TEAMS; ++v) {
            total[0] += part_r[0][team.of(v)];
            total[1] += part_r[1][team.of(v)];
        }
        float *to = p.part + ((int64_t)n * q.chunks + chunk) * p.c;
        put2(to, L, total[0], total[1]);
    }
}

template <class T>
__global__ __launch_bounds__(64) void recurrence_bwd_single_kernel(const RecParams p) {
    __shared__ float hs[SAVE][64];
    const int lane = threadIdx.x;
    const int64_t n = (int64_t)blockIdx.x * 64 + lane;
    if (n >= p.n) return;
    const int len = length_of(p, (int)n);
    const float bias = p.bias ? p.bias[0] * -LOG2E : 0.f;
    const int64_t at = n * p.t * p.ld, stretches = (p.t + SAVE - 1) / SAVE;
    const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
    const uint16_t *g = p.g ? (const uint16_t *)p.g + at : nullptr;
    const uint16_t *dy = (const uint16_t *)p.dy + n * p.t * p.ldy;
    uint16_t *dx = (uint16_t *)p.dx + at, *df = (uint16_t *)p.df + at;
    uint16_t *dg = p.g ? (uint16_t *)p.dg + at : nullptr;
    float r = p.dht ? p.dht[n] : 0.f, total = 0.f;
    for (int64_t k = stretches - 1; k >= 0; --k) {
        const int64_t lo = k * SAVE, hi = lo + SAVE < p.t ? lo + SAVE : p.t;
        float h = p.saved[n * stretches + k], part = 0.f;
        for (int64_t t = lo; t < hi && t < len; ++t) {
            float a, b;
            hs[t - lo][lane] = h;
            gate(from16<T>(f[t * p.ld]), bias, a, b);
            h = a * h + b * from16<T>(x[t * p.ld]);
        }
        for (int64_t t = hi - 1; t >= lo; --t) {
            float vx = 0.f, vf = 0.f, vg = 0.f;
            if (t < len) {
                float a, b;
                gate(from16<T>(f[t * p.ld]), bias, a, b);
                const float xv = from16<T>(x[t * p.ld]), before = hs[t - lo][lane];
                float own = from16<T>(dy[t * p.ldy]);
                if (g) {
                    const float gv = from16<T>(g[t * p.ld]), s = sigma(gv), sg = gv * s;
                    vg = own * (s + sg * (1.f - s)) * (a * before + b * xv);
                    own *= sg;
                }
                const float d = own + r;
                vx = d * b;
                vf = d * (before - xv) * (a * b);
                r = a * d;
                part += vf;
            }
            dx[t * p.ld] = (uint16_t)to16<T>(vx);
            df[t * p.ld] = (uint16_t)to16<T>(vf);
            if (dg) dg[t * p.ld] = (uint16_t)to16<T>(vg);
        }
        total += part;
    }
    if (p.dh0) p.dh0[n] = r;
    if (p.part) p.part[n] = total;
}

}  // namespace

void launch_recurrence_bwd_chunks(int dtype, const RecParams &p, const RecGrid &q, uint32_t blocks, hipStream_t st) {
    with_kind(dtype, p.g != nullptr, [&](auto t, auto g) {
        auto go = [&](auto waves, auto teams) {
            hipLaunchKernelGGL((recurrence_bwd_kernel<decltype(t), decltype(g)::value, decltype(waves)::value, TOKENS, decltype(teams)::value>),
                               dim3(blocks), dim3(64 * decltype(waves)::value), 0, st, p, q);
        };
        auto several = [&](auto teams) {
            if (q.waves == 1) go(Int<1>{}, teams); else go(Int<BWD_WAVES>{}, teams);
        };
        if (q.teams == 8) return several(Int<8>{});
        if (q.teams == 4) return several(Int<4>{});
        if (q.teams == 2) return several(Int<2>{});
        if (q.waves == 2) return go(Int<2>{}, Int<1>{});
        several(Int<1>{});
    });
}

void launch_recurrence_bwd_short(int dtype, const RecParams &p, hipStream_t st) {
    with_kind(dtype, p.g != nullptr, [&](auto t, auto g) {
        hipLaunchKernelGGL((recurrence_bwd_short_kernel<decltype(t), decltype(g)::value>), short_grid(p), dim3(64), 0, st, p);
    });
}

void launch_recurrence_bwd_single(int dtype, const RecParams &p, hipStream_t st) {
    with_kind(dtype, true, [&](auto t, auto) {
        hipLaunchKernelGGL((recurrence_bwd_single_kernel<decltype(t)>), dim3((uint32_t)(((int64_t)p.n + 63) / 64)), dim3(64), 0, st, p);
    });
}

}  // namespace nnconv
