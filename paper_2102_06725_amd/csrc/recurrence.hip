// recurrence.hip -- gated linear recurrence: how a call is split, and its launches.
#include "recurrence.hpp"

namespace nnconv {

namespace {

// Before each split call: every word empty but the states in front of the first places.
__global__ __launch_bounds__(256) void recurrence_words_kernel(const RecGrid q, int64_t n, int32_t c,
                                                               const float *init) {
    const int64_t plain = n * q.chunks * c, total = plain + n * q.groups * c;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        uint64_t v = NO_WORD;
        if (i >= plain) {
            const int64_t row = (i - plain) / c;
            if (row % q.groups == 0) v = word(0.f, init ? init[row / q.groups * c + (i - plain - row * c)] : 0.f);
        }
        q.words[i] = v;  // the states follow the words
    }
}

// Teams of a wave: as many as leave each the lanes for all channels.  (One team throughout:
// forward of 54 x 1511 x 16, ragged, 20.6 us, 17.2 with eight; forward and backward of 2 x
// 38104 x 40 75 us, 61 with two.)
int teams_of(const RecParams &p) { return p.c <= 16 ? 8 : p.c <= 32 ? 4 : p.c <= 64 ? 2 : 1; }

// Waves of a workgroup: no more than the tokens need.  (Eight throughout: forward of 4096 x 16
// x 1152 401 us, one wave 113; backward 470 and 184.)
int waves_of(const RecParams &p, bool backward) {
    const int most = backward ? BWD_WAVES : FWD_WAVES, each = TOKENS * teams_of(p);
    if (teams_of(p) > 1) return p.t <= each ? 1 : most;
    int w = 1;
    while (w < most && w * each < p.t) w *= 2;
    return w;
}

int64_t chunks_of(const RecParams &p, bool backward) {
    const int64_t k = waves_of(p, backward) * TOKENS * teams_of(p);
    return p.t <= SHORT_T || p.c == 1 ? 1 : ((int64_t)p.t + k - 1) / k;
}

// Places in groups of 2^gs: about as many groups, whose states are handed on one after the
// other, as places in one, whose pairs each place reads.  (Groups of 16 throughout: backward of
// 8 x 2048 x 1152 4 us slower.  Groups of at most 16: forward of 1 x 65536 x 256 47 us, 42 with
// 32.)
RecGrid grid_of(const RecParams &p, bool backward) {
    RecGrid q{};
    const int64_t chunks = chunks_of(p, backward);
    q.waves = waves_of(p, backward);
    q.teams = teams_of(p);
    q.cols = (p.c + COLS - 1) / COLS;  // one where a wave is several teams
    q.chunks = (int32_t)chunks;
    while (1 << q.gs < GROUP && chunks >> 2 * q.gs > 1) ++q.gs;
    q.groups = (int32_t)((chunks + (1 << q.gs) - 1) >> q.gs);
    return q;
}

int64_t word_count(const RecParams &p, bool backward) {
    const RecGrid q = grid_of(p, backward);
    return q.chunks > 1 ? (int64_t)p.n * ((int64_t)q.chunks + q.groups) * p.c : 0;
}

// Workgroups of one launch at most: work items of a launch are counted in 32 bits.
constexpr int64_t MOST_BLOCKS = 1 << 22;
constexpr int32_t MOST_TOKENS = 1 << 29;

// The sequences from n0 on, n of them.
RecParams some(const RecParams &p, bool backward, int64_t n0, int64_t n) {
    RecParams s = p;
    const int64_t in = n0 * p.t * p.ld * 2, out = n0 * p.t * p.ldy * 2, state = n0 * p.c;
    const int64_t stretches = (p.t + SAVE - 1) / SAVE;
    auto move = [](auto &q, int64_t bytes) {
        if (q) q = (std::remove_reference_t<decltype(q)>)((uintptr_t)q + bytes);
    };
    s.n = (int32_t)n;
    for (const void **q : {&s.x, &s.f, &s.g}) move(*q, in);
    for (void **q : {&s.dx, &s.df, &s.dg}) move(*q, in);
    move(s.y, out);
    move(s.dy, out);
    move(s.lengths, n0 * 4);
    for (const float **q : {&s.h0, &s.dht}) move(*q, state * 4);
    for (float **q : {&s.ht, &s.dh0}) move(*q, state * 4);
    move(s.saved, state * stretches * 4);
    move(s.part, state * chunks_of(p, backward) * 4);
    return s;
}

hipError_t launch(int dtype, const RecParams &p, bool backward, hipStream_t st) {
    if (p.n <= 0) return hipSuccess;
    if (p.c == 1) {
        (backward ? launch_recurrence_bwd_single : launch_recurrence_fwd_single)(dtype, p, st);
        return hipGetLastError();
    }
    if (p.t <= SHORT_T) {
        (backward ? launch_recurrence_bwd_short : launch_recurrence_fwd_short)(dtype, p, st);
        return hipGetLastError();
    }
    RecGrid q = grid_of(p, backward);
    const int64_t each = (int64_t)q.chunks * q.cols, most = each < MOST_BLOCKS ? MOST_BLOCKS / each : 1;
    for (int64_t n0 = 0; n0 < p.n; n0 += most) {
        const RecParams s = some(p, backward, n0, p.n - n0 < most ? p.n - n0 : most);
        if (q.chunks > 1) {  // launches follow each other: they share the words
            q.words = (uint64_t *)p.ws;
            q.states = q.words + (int64_t)s.n * q.chunks * p.c;
            const int64_t nb = (word_count(s, backward) + 255) / 256;
            hipLaunchKernelGGL(recurrence_words_kernel, dim3((uint32_t)(nb < 2048 ? nb : 2048)), dim3(256), 0, st, q,
                               (int64_t)s.n, p.c, backward ? s.dht : s.h0);
        }
        (backward ? launch_recurrence_bwd_chunks : launch_recurrence_fwd_chunks)(dtype, s, q, (uint32_t)(each * s.n), st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

// One sequence's workgroups have to fit a launch, and its tokens' numbers 32 bits, also those of
// a last workgroup's places past the end.
bool recurrence_fits(const RecParams &p) {
    if (p.t > MOST_TOKENS) return false;
    const RecGrid f = grid_of(p, false), b = grid_of(p, true);
    return (int64_t)f.chunks * f.cols <= MOST_BLOCKS && (int64_t)b.chunks * b.cols <= 2 * MOST_BLOCKS;
}

int64_t recurrence_bwd_parts(const RecParams &p) { return p.n * chunks_of(p, true); }

// Words first (8-byte aligned), then, backward, the partial sums of dbias.
size_t recurrence_words_bytes(const RecParams &p, bool backward) {
    return sizeof(uint64_t) * (size_t)word_count(p, backward);
}

size_t recurrence_ws(const RecParams &p, bool backward) {
    const size_t words = recurrence_words_bytes(p, backward);
    if (!backward) return words;
    const int64_t parts = recurrence_bwd_parts(p);
    return words + sizeof(float) * (size_t)((parts + colsum_extra(parts)) * p.c);
}

hipError_t launch_recurrence_fwd(int dtype, const RecParams &p, hipStream_t st) {
    return launch(dtype, p, false, st);
}

hipError_t launch_recurrence_bwd(int dtype, const RecParams &p, hipStream_t st) {
    return launch(dtype, p, true, st);
}

}  // namespace nnconv
