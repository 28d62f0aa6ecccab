// Drafted tokens verified against the target's probabilities with given random numbers, and the token that follows them.  Row 0 of a sequence is the token
// that is there already, the rows behind it are its drafted tokens, a chain or a tree (a row's parent is in front of it).  From the root on, the children of the node
// that has been reached are tried in order: with the node's probabilities p, child x with the random number u is accepted where
//     u q(x) < p(x)         in a chain whose tokens were drawn from the probabilities q,
//     u (1 - sum of p over the node's children refused so far) < p(x)     where tokens are proposed for certain,
// and the token that follows the last one accepted is drawn, by the root's random number, from the weights
//     w = max(p - q, 0)  or  p without the refused children,
// as the first x whose sum of w up to it exceeds u times all of them.  Each accepted token then has the target's distribution: what a refusal leaves out of it, the
// last draw makes up for.
//
// Products, differences and sums are fp64: a difference is rounded to 2^-53 of itself, and with 131072 tokens a sum has passed fewer than 40 roundings, so that a border and the sum that is
// held against it are off by less than 2^-47 of all.  The choice then is that of the exact sums but where a border is that near a token's, two draws in 10^9 at most.
//
// One row (two in a chain) of each sequence is read whole, which is what bounds it; the walk before that is a chain of three loads, and every workgroup makes it again
// by itself: a launch of its own would take longer.  64 chains of eight drafted tokens, 131072 fp32 probabilities a row, 67 MB: 13 to 14.5 us for the sums, 4.6 to 5.1 TB/s, 3 to 4 for the
// draw, which is three rounds of dependent loads; 12 trees of 48 with 32011: 5.2 and 3 to 4, the walk's and the draw's chains.  But where no weight is left, which takes probabilities that do
// not add up to 1, a draw's threads sum pieces of the target's row by themselves: a call then takes 90 us with 32011 tokens, 111 with 131072, 12.5 ms with 2^24.
#include "agzo_internal.h"

namespace agzo {

namespace {

constexpr int VF_WG = 256, VF_PIECE = 512, VF_LEAST = 8 * VF_WG, VF_MOST_SEGMENTS = 256;      // VF_PIECE: tokens that a wave takes at a time, each with a sum of its own

__device__ __forceinline__ float vf_get(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float vf_get(const bf16_t* p, int64_t i) { return bf16_to_f32(p[i]); }
// (negative values and NaN count as 0)
__device__ __forceinline__ double vf_mass(float x) { return x > 0.f ? (double)x : 0.0; }

__device__ __forceinline__ double vf_readlane(double x, int lane) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), lane), __builtin_amdgcn_readlane(__double2loint(x), lane));
}

// Where a sequence's walk ends: at a row, a chain's row refused there (0: none), how many rows accepted
struct VfEnd { int at, refused, count; };

// By one wave, 64 rows at a time, which is right since a node's children stand behind it.  write: the accepted rows are stored too
template <typename T>
__device__ __forceinline__ VfEnd vf_walk(const VerifyArgs& a, int64_t r0, int rows, bool write) {
    const T *p = static_cast<const T*>(a.p), *q = static_cast<const T*>(a.q);
    const int lane = threadIdx.x & 63;
    VfEnd e{0, 0, 0};
    double left = 1.0;
    for (int b = 0; b < rows; b += 64) {
        const int row = b + lane;
        const bool there = row > 0 && row < rows;
        const int tok = there ? a.tokens[r0 + row] : -1;
        const int up = !there ? -1 : a.parents ? a.parents[r0 + row] : row - 1;
        const int parent = up >= 0 && up < row ? up : -1;
        const bool known = parent >= 0 && tok >= 0 && tok < a.vocab;
        const double target = known ? vf_mass(vf_get(p, (r0 + parent) * a.ldp + tok)) : 0.0;
        const double draft = known && q ? vf_mass(vf_get(q, (r0 + row) * a.ldq + tok)) : 0.0;
        const double u = there ? (double)a.uniforms[r0 + row] : 0.0;
        int tried = b - 1;
        while (true) {
            const uint64_t next = __builtin_amdgcn_ballot_w64(parent == e.at && row > max(tried, e.at));
            if (!next) break;
            const int i = __builtin_ctzll(next), x = __builtin_amdgcn_readlane(tok, i);
            double mass = vf_readlane(target, i);
            tried = b + i;
            if (!q) {
                // a token that a sibling before has been refused with has nothing left
                bool again = __builtin_amdgcn_ballot_w64(parent == e.at && row < tried && tok == x) != 0;
                for (int c = 0; c < b && !again; c += 64) {
                    const bool sibling = c + lane > e.at && a.parents && a.parents[r0 + c + lane] == e.at && a.tokens[r0 + c + lane] == x;
                    again = __builtin_amdgcn_ballot_w64(sibling) != 0;
                }
                if (again) mass = 0.0;
            }
            const double of = q ? vf_readlane(draft, i) : left;
            if (mass > 0.0 && vf_readlane(u, i) * of < mass) {
                if (write && lane == 0) {
                    a.out_tokens[r0 + e.count] = x;
                    a.out_rows[r0 + e.count] = tried;
                }
                e.at = tried;
                e.refused = 0;
                ++e.count;
                left = 1.0;
            } else {
                left -= mass;
                e.refused = tried;
            }
        }
    }
    return e;
}

// bits of the tokens first .. first + n that children of `at` have: all of them were refused
__device__ __forceinline__ void vf_refused(const VerifyArgs& a, int64_t r0, int rows, int at, int64_t first, int n, uint32_t* bits) {
    for (int row = at + 1 + (int)threadIdx.x; row < rows; row += VF_WG) {
        const int up = a.parents ? a.parents[r0 + row] : row - 1;
        const int64_t x = (int64_t)a.tokens[r0 + row] - first;
        if (up == at && x >= 0 && x < n) atomicOr(&bits[x >> 5], 1u << (x & 31));
    }
}

// eight values of a row from i on (0 behind its end)
__device__ __forceinline__ void vf_eight(const float* p, int64_t i, int64_t end, float (&f)[8]) {
    typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
    if (i + 8 <= end) {
        const vec x = *reinterpret_cast<const vec*>(p + i), y = *reinterpret_cast<const vec*>(p + i + 4);
#pragma unroll
        for (int u = 0; u < 4; ++u) { f[u] = x[u]; f[4 + u] = y[u]; }
    } else {
#pragma unroll
        for (int u = 0; u < 8; ++u) f[u] = i + u < end ? p[i + u] : 0.f;
    }
}
__device__ __forceinline__ void vf_eight(const bf16_t* p, int64_t i, int64_t end, float (&f)[8]) {
    typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
    if (i + 8 <= end) {
        const vec x = *reinterpret_cast<const vec*>(p + i);
#pragma unroll
        for (int u = 0; u < 4; ++u) { f[2 * u] = __uint_as_float(x[u] << 16); f[2 * u + 1] = __uint_as_float(x[u] & 0xFFFF0000u); }
    } else {
#pragma unroll
        for (int u = 0; u < 8; ++u) f[u] = i + u < end ? bf16_to_f32(p[i + u]) : 0.f;
    }
}

// weights of eight tokens, the first one `in` of its segment
__device__ __forceinline__ void vf_weights(const float (&p)[8], const float (&q)[8], uint32_t gone, double (&w)[8]) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const double d = vf_mass(p[u]) - vf_mass(q[u]);
        w[u] = d > 0.0 && !((gone >> u) & 1) ? d : 0.0;
    }
}

template <int CTRL>
__device__ __forceinline__ double vf_dpp(double x) {
    return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, 0xF, 0xF, true), __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, 0xF, 0xF, true));
}
// sums over the lanes up to each (row_shr 1, 2, 4, 8 within 16 lanes; what comes from outside them is 0)
__device__ __forceinline__ double vf_upto(double x) {
    x += vf_dpp<0x111>(x);
    x += vf_dpp<0x112>(x);
    x += vf_dpp<0x114>(x);
    x += vf_dpp<0x118>(x);
    const double a = vf_readlane(x, 15), b = a + vf_readlane(x, 31), c = b + vf_readlane(x, 47);
    const int row = (threadIdx.x & 63) >> 4;
    return x + (row == 0 ? 0.0 : row == 1 ? a : row == 2 ? b : c);
}
__device__ __forceinline__ double vf_total(double x) { return vf_readlane(vf_upto(x), 63); }

// What the walk leaves for the draw (in one place: a load that waits for another one is a microsecond)
struct VfReached { int at, refused, count, rows; int64_t r0; float u; int unused; };
struct VfState { double* sums; VfReached* reached; int pieces; };      // [n_seq][pieces]: sums of the weights; [n_seq]
__device__ __forceinline__ void vf_rows(const VerifyArgs& a, int seq, int64_t& r0, int& rows) {
    r0 = min(max((int64_t)a.cu[seq], (int64_t)0), a.n);
    rows = (int)(min(max((int64_t)a.cu[seq + 1], r0), a.n) - r0);
}

template <typename T>
__global__ __launch_bounds__(VF_WG) void verify_sums_kernel(VerifyArgs a, VfState s, int segment) {
    extern __shared__ uint32_t vf_bits[];
    const int seq = blockIdx.y, seg = blockIdx.x;
    int64_t r0;
    int rows;
    vf_rows(a, seq, r0, rows);
    if (rows == 0) {
        if (seg == 0 && threadIdx.x == 0) {
            a.n_accepted[seq] = 0;
            s.reached[seq] = VfReached{0, 0, 0, 0, 0, 0.f, 0};
        }
        return;
    }
    const VfEnd e = vf_walk<T>(a, r0, rows, seg == 0 && threadIdx.x < 64);
    if (seg == 0) {
        if (threadIdx.x == 0) {
            a.n_accepted[seq] = e.count;
            s.reached[seq] = VfReached{e.at, e.refused, e.count, rows, r0, a.uniforms[r0], 0};
        }
        // (the entry behind the accepted ones is the draw's)
        for (int i = e.count + (int)threadIdx.x; i < rows; i += VF_WG) {
            if (i > e.count) a.out_tokens[r0 + i] = -1;
            a.out_rows[r0 + i] = -1;
        }
    }
    const T *p = static_cast<const T*>(a.p) + (r0 + e.at) * a.ldp, *q = a.q && e.refused ? static_cast<const T*>(a.q) + (r0 + e.refused) * a.ldq : nullptr;
    const int64_t first = (int64_t)seg * segment, end = min(first + segment, a.vocab);
    const bool marked = !a.q && e.refused;
    if (marked) {
        for (int i = threadIdx.x; i < segment / 32; i += VF_WG) vf_bits[i] = 0;
        __syncthreads();
        vf_refused(a, r0, rows, e.at, first, segment, vf_bits);
        lds_barrier();
    }
    for (int64_t i = first + 8 * threadIdx.x; i - 8 * (threadIdx.x & 63) < end; i += 8 * VF_WG) {      // (a wave's lanes together)
        float f[8], g[8] = {};
        vf_eight(p, i, end, f);
        if (q) vf_eight(q, i, end, g);
        double w[8];
        vf_weights(f, g, marked ? vf_bits[(i - first) >> 5] >> ((i - first) & 31) : 0, w);
        const double sum = vf_total(((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7])));
        if ((threadIdx.x & 63) == 0) s.sums[(int64_t)seq * s.pieces + i / VF_PIECE] = sum;
    }
}

// Sums of the threads up to each, this one among them, and of all
__device__ __forceinline__ double vf_scan(double x, double* red, double& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    x = vf_upto(x);
    if (lane == 63) red[wave] = x;
    lds_barrier();
    for (int i = 0; i < wave; ++i) x += red[i];
    all = ((red[3] + red[0]) + red[1]) + red[2];      // (as the last thread has it)
    return x;
}
// The first thread with `first`, VF_WG if none has, and the last one with `last`, -1 if none.  (By ballots: atomics of 256 threads on one place in LDS were 7 of the draw's 11 us)
__device__ __forceinline__ void vf_ends(bool first, bool last, int2* red, int& from, int& to) {
    const uint64_t f = __builtin_amdgcn_ballot_w64(first), l = __builtin_amdgcn_ballot_w64(last);
    const int wave = threadIdx.x / 64;
    if ((threadIdx.x & 63) == 0) red[wave] = make_int2(f ? 64 * wave + __builtin_ctzll(f) : VF_WG, l ? 64 * wave + 63 - __builtin_clzll(l) : -1);
    lds_barrier();
    from = min(min(red[0].x, red[1].x), min(red[2].x, red[3].x));
    to = max(max(red[0].y, red[1].y), max(red[2].y, red[3].y));
}

// The draw: the piece that the border lies in, then the token in it, two to a thread
template <typename T>
__global__ __launch_bounds__(VF_WG) void verify_draw_kernel(VerifyArgs a, VfState s) {
    static_assert(VF_WG == 256 && VF_PIECE == 2 * VF_WG, "four waves, two tokens a thread");
    __shared__ double red[3][VF_WG / 64];
    __shared__ int2 ends[3][VF_WG / 64];
    __shared__ double before;
    __shared__ int piece;
    __shared__ uint32_t bits[VF_PIECE / 32];
    const int seq = blockIdx.x, t = threadIdx.x;
    const VfReached e = s.reached[seq];
    // a thread's run of pieces
    const int per = (s.pieces + VF_WG - 1) / VF_WG, from = min(t * per, s.pieces), to = min(from + per, s.pieces);
    const double* sums = s.sums + (int64_t)seq * s.pieces;
    double mine = 0.0;
    for (int i = from; i < to; ++i) mine += sums[i];
    if (e.rows == 0) return;
    const int64_t r0 = e.r0;
    const T* p = static_cast<const T*>(a.p) + (r0 + e.at) * a.ldp;
    if (t < VF_PIECE / 32) bits[t] = 0;
    double all;
    double upto = vf_scan(mine, red[0], all), border = (double)e.u * all;
    int found, last;
    vf_ends(mine > 0.0 && upto > border, mine > 0.0, ends[0], found, last);
    // (nothing left, as where the probabilities do not add up to 1: the target's own, whose sums nobody has made)
    const bool own = last < 0;
    auto own_sum = [&](int i) {
        double x = 0.0;
        for (int64_t j = (int64_t)i * VF_PIECE; j < min((int64_t)(i + 1) * VF_PIECE, a.vocab); ++j) x += vf_mass(vf_get(p, j));
        return x;
    };
    if (own) {
        mine = 0.0;
        for (int i = from; i < to; ++i) mine += own_sum(i);
        upto = vf_scan(mine, red[1], all);
        border = (double)e.u * all;
        vf_ends(mine > 0.0 && upto > border, mine > 0.0, ends[1], found, last);
        if (last < 0) {                       // no token has any probability
            if (t == 0) a.out_tokens[r0 + e.count] = -1;
            return;
        }
    }
    // (a border at the end or behind it: the last token that has any weight)
    const bool behind = found == VF_WG;
    if (t == (behind ? last : found)) {
        double so_far = upto - mine;
        int pick = -1;
        for (int i = from; i < to; ++i) {
            const double x = own ? own_sum(i) : per == 1 ? mine : sums[i];
            if (x > 0.0 && (behind || pick < 0 || !(so_far > border))) { pick = i; before = so_far; }
            so_far += x;
        }
        piece = pick;
    }
    lds_barrier();
    const T* q = a.q && e.refused && !own ? static_cast<const T*>(a.q) + (r0 + e.refused) * a.ldq : nullptr;
    const int64_t first = (int64_t)piece * VF_PIECE, at = first + 2 * t;
    double w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool there = at + i < a.vocab;
        const double d = there ? vf_mass(vf_get(p, at + i)) - (q ? vf_mass(vf_get(q, at + i)) : 0.0) : 0.0;
        w[i] = d > 0.0 ? d : 0.0;
    }
    if (!a.q && e.refused && !own) {
        vf_refused(a, r0, e.rows, e.at, first, VF_PIECE, bits);
        lds_barrier();
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if ((bits[(2 * t + i) >> 5] >> ((2 * t + i) & 31)) & 1) w[i] = 0.0;
    }
    const double x = w[0] + w[1], run = before + vf_scan(x, red[2], all);
    vf_ends(!behind && x > 0.0 && run > border, x > 0.0, ends[2], found, last);
    // (sums in another order than the piece's: a border within 2^-50 of its end may be behind all of them)
    const bool at_end = found == VF_WG;
    if (t != (at_end ? last : found)) return;
    const bool second = w[0] > 0.0 && w[1] > 0.0 ? at_end || !(run - w[1] > border) : w[1] > 0.0;
    a.out_tokens[r0 + e.count] = (int)(at + second);
}

// no sequence has a row: none is accepted
__global__ __launch_bounds__(VF_WG) void verify_none_kernel(int32_t* n_accepted, int n_seq) {
    const int i = blockIdx.x * VF_WG + threadIdx.x;
    if (i < n_seq) n_accepted[i] = 0;
}

int verify_segment(int n_seq, int64_t vocab) {
    // enough workgroups to keep every compute unit's loads in flight, of no fewer tokens than a workgroup takes at a time
    int64_t size = VF_LEAST;
    while ((vocab + size - 1) / size > VF_MOST_SEGMENTS || (n_seq * ((vocab + size - 1) / size) > 1024 && size < 16 * VF_LEAST)) size *= 2;
    return (int)size;
}

template <typename T>
hipError_t launch_verify_typed(const VerifyArgs& a, void* workspace, hipStream_t st) {
    const int segment = verify_segment(a.n_seq, a.vocab), segments = (int)((a.vocab + segment - 1) / segment), pieces = (int)((a.vocab + VF_PIECE - 1) / VF_PIECE);
    const VfState s{reinterpret_cast<double*>(static_cast<VfReached*>(workspace) + a.n_seq), static_cast<VfReached*>(workspace), pieces};
    const size_t smem = a.q ? 0 : segment / 8;
    hipLaunchKernelGGL(verify_sums_kernel<T>, dim3(segments, a.n_seq), dim3(VF_WG), smem, st, a, s, segment);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(verify_draw_kernel<T>, dim3(a.n_seq), dim3(VF_WG), 0, st, a, s);
    return hipGetLastError();
}

}  // namespace

size_t verify_workspace_bytes(int n_seq, int64_t vocab) { return (size_t)n_seq * ((vocab + VF_PIECE - 1) / VF_PIECE * sizeof(double) + sizeof(VfReached)); }

hipError_t launch_verify(const VerifyArgs& a, bool f32, void* workspace, hipStream_t st) {
    if (a.n_seq == 0) return hipSuccess;
    if (a.n == 0) {
        hipLaunchKernelGGL(verify_none_kernel, dim3((a.n_seq + VF_WG - 1) / VF_WG), dim3(VF_WG), 0, st, a.n_accepted, a.n_seq);
        return hipGetLastError();
    }
    return f32 ? launch_verify_typed<float>(a, workspace, st) : launch_verify_typed<bf16_t>(a, workspace, st);
}

}  // namespace agzo
