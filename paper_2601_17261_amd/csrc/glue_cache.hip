// Rotation of queries and keys by the token's position in its layouts, the way of new tokens into a cache of keys and values in pages, and the accepted
// tokens of a tree moved together there.  A head's first `rot` values are turned in pairs,
//     y_a = m (x_a cos t f_p - x_b sin t f_p),   y_b = m (x_b cos t f_p + x_a sin t f_p),     p = 0 .. rot/2,  (a, b) = (p, p + rot/2) or (2 p, 2 p + 1),
// t the position, f_p = theta^(-2p/rot) (k_p + (1 - k_p) / factor), k_p = 1 where a frequency is kept and 0 where it is that of a `factor` times longer
// context.  The gradient is the turn by the opposite angle, times m too.
// All of it is one pass over memory, bound by HBM where tokens are many and by the chain of loads (a token's sequence, its page, its row) where they are few.
#include "paged.h"

namespace agzo {

namespace {

constexpr int RC_WG = 256;

__device__ __forceinline__ void rc_widen(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void rc_load(const bf16_t* p, float (&f)[8]) { rc_widen(*reinterpret_cast<const uint4*>(p), f); }
__device__ __forceinline__ void rc_load(const float* p, float (&f)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void rc_store(bf16_t* p, const float (&f)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
__device__ __forceinline__ void rc_store(float* p, const float (&f)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}

// m cos and m sin of `count` tokens' angles, [token][rot / 2].  A pair's frequency is worked out once for all of a workgroup's tokens, in fp64 as its product with
// the position: in fp32 an angle is off by position * 2^-24, 0.01 at positions of 10^5
__device__ __forceinline__ void rc_angles(float2* cs, const RopeArgs& r, const int32_t* positions, int count, float sign) {
    const int half = r.rot / 2;
    const int wide = half <= 32 ? 32 : half <= 64 ? 64 : 128, p = threadIdx.x & (wide - 1);
    if (p >= half) return;
    const double f = exp2(-2.0 * p / r.rot * r.log2_theta);
    const double keep = fmin(1.0, fmax(0.0, r.keep_from + r.keep_by * (r.by_turns ? f : (double)p)));
    const double turns_of_one = f * (keep + (1.0 - keep) * r.inv_factor) * 0.15915494309189533577;
    for (int t = threadIdx.x / wide; t < count; t += RC_WG / wide) {
        const double turns = (double)positions[t] * turns_of_one;      // without the whole ones
        float sn, c;
        sincospif(2.f * (float)(turns - rint(turns)), &sn, &c);
        cs[t * half + p] = make_float2(c * r.magnitude, sn * r.magnitude * sign);
    }
}

// 16 values of a head, j-th of head_dim / 16 such: eight pairs where they are turned.  Where the two eights start
__device__ __forceinline__ void rc_at(int j, int rot, bool inter, int& a, int& b) {
    const bool split = !inter && j < rot / 16;
    a = split ? 8 * j : 16 * j;
    b = split ? rot / 2 + 8 * j : 16 * j + 8;
}
__device__ __forceinline__ void rc_turn(float (&a)[8], float (&b)[8], const float2* ang, bool inter) {
    if (inter) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float& x = i < 4 ? a[2 * i] : b[2 * i - 8];
            float& y = i < 4 ? a[2 * i + 1] : b[2 * i - 7];
            const float u = x, w = y;
            x = fmaf(u, ang[i].x, -w * ang[i].y);
            y = fmaf(w, ang[i].x, u * ang[i].y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float u = a[i], w = b[i];
            a[i] = fmaf(u, ang[i].x, -w * ang[i].y);
            b[i] = fmaf(w, ang[i].x, u * ang[i].y);
        }
    }
}

template <typename T>
struct RopeSide { const T* x; int64_t ldx; T* y; int64_t ldy; int heads; };

// A token a workgroup: 16384 tokens of 40 heads of 128 in 60 us, 5.5 TB/s, and in 63, 65, 69 with two, four and eight
template <typename T>
__global__ __launch_bounds__(RC_WG) void rope_kernel(RopeSide<T> q, RopeSide<T> k, const int32_t* __restrict__ positions, RopeArgs r, float sign, int head_dim, QuickDiv by_lanes) {
    extern __shared__ float2 rc_cs[];
    const int64_t t = blockIdx.x;
    const int lanes = (int)by_lanes.d, heads = q.heads + k.heads;
    rc_angles(rc_cs, r, positions + t, 1, sign);
    lds_barrier();
    for (int item = threadIdx.x; item < heads * lanes; item += RC_WG) {
        const int h = by_lanes(item), j = item - h * lanes;
        const bool is_q = h < q.heads;
        const T* x = is_q ? q.x + t * q.ldx + (int64_t)h * head_dim : k.x + t * k.ldx + (int64_t)(h - q.heads) * head_dim;
        T* y = is_q ? q.y + t * q.ldy + (int64_t)h * head_dim : k.y + t * k.ldy + (int64_t)(h - q.heads) * head_dim;
        const bool turned = j < r.rot / 16;
        if (!turned && x == y) continue;                  // (in place)
        int ia, ib;
        rc_at(j, r.rot, r.interleaved, ia, ib);
        float a[8], b[8];
        rc_load(x + ia, a);
        rc_load(x + ib, b);
        if (turned) rc_turn(a, b, rc_cs + 8 * j, r.interleaved);
        rc_store(y + ia, a);
        rc_store(y + ib, b);
    }
}

constexpr int64_t kRopeTokens = 1 << 23;      // of a launch: one of 2^32 threads and more is cut off without a word

template <typename T>
hipError_t launch_rope_typed(const RopeArgs& r, const RopeTensor& q, const RopeTensor& k, const int32_t* positions, int64_t n, int head_dim, bool back, hipStream_t st) {
    if (n == 0 || q.heads + k.heads == 0) return hipSuccess;
    auto from = [](const RopeTensor& a, int64_t t) { return RopeSide<T>{static_cast<const T*>(a.x) + t * a.ldx, a.ldx, static_cast<T*>(a.y) + t * a.ldy, a.ldy, a.heads}; };
    for (int64_t t = 0; t < n; t += kRopeTokens) {
        hipLaunchKernelGGL(rope_kernel<T>, dim3((unsigned)std::min(n - t, kRopeTokens)), dim3(RC_WG), r.rot / 2 * sizeof(float2), st, from(q, t), from(k, t), positions + t, r, back ? -1.f : 1.f,
                           head_dim, QuickDiv(head_dim / 16));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- into the cache --------------------------------------------------------------------------------------------
constexpr int RC_MOST = 2;      // tokens of a workgroup, where they are many.  (16384 tokens, 403 MB: 80, 79 and 81 us with one, two and four, 5.1 TB/s; 81 where
// an item's values are only asked for when its turn has come)

// HD / 16 lanes a head; queries to their rows, keys and values to their pages
template <int HD, bool NORM>
__global__ __launch_bounds__(RC_WG) void cache_append_kernel(PagedCache c, RopeArgs r, CacheAppend a, int per_wg, QuickDiv by_page, QuickDiv by_heads) {
    constexpr int LANES = HD / 16;
    extern __shared__ float2 rc_cs[];
    __shared__ int64_t k_at[RC_MOST], v_at[RC_MOST];
    __shared__ int pos[RC_MOST];
    __shared__ __align__(16) float gain[2][HD];      // of queries and keys.  (In registers, 32 of them, three workgroups fewer fit on a compute unit)
    const int64_t tok0 = (int64_t)blockIdx.x * per_wg;
    const int count = (int)min((int64_t)per_wg, a.n - tok0), heads = a.n_heads + 2 * c.n_kv, items = count * heads;
    const int j = threadIdx.x % LANES;
    int ia, ib;
    rc_at(j, r.rot, r.interleaved, ia, ib);
    // A head's values, eight from ia and eight from ib on, of an item, which is a token's head: asked for while the item before is worked on, the first one's before the look-ups
    struct Data { uint4 a, b; };
    auto load = [&](int th) __attribute__((always_inline)) {
        const int t = by_heads(th), h = th - t * heads;
        const int64_t tok = tok0 + t;
        const bf16_t* x = h < a.n_heads ? a.q + tok * a.ldq + (int64_t)h * HD
                        : h < a.n_heads + c.n_kv ? a.k + tok * a.ldk + (int64_t)(h - a.n_heads) * HD : a.v + tok * a.ldv + (int64_t)(h - a.n_heads - c.n_kv) * HD;
        return Data{*reinterpret_cast<const uint4*>(x + ia), *reinterpret_cast<const uint4*>(x + ib)};
    };
    int th = threadIdx.x / LANES;
    Data next = load(min(th, items - 1));
    for (int t = threadIdx.x / 64; t < count; t += RC_WG / 64) {
        const int tok = (int)tok0 + t;
        PagedSeq s{};
        const int seq = paged_find(c, a.cu_q, (int)a.n, tok, s);
        const int place = s.nk - s.nq + tok - s.q0;
        int64_t page = 0;
        int slot = 0;
        const bool stored = seq >= 0 && paged_slot(c, by_page, seq, place, page, slot);
        if ((threadIdx.x & 63) == 0) {
            // (-2: of no sequence, -1: without a place)
            k_at[t] = seq < 0 ? -2 : stored ? page * c.k_page + slot * c.k_row : -1;
            v_at[t] = page * c.v_page + slot * c.v_row;
            pos[t] = a.positions ? a.positions[tok] : place;
        }
    }
    if (NORM)
        for (int i = threadIdx.x; i < 2 * HD; i += RC_WG) {
            const float* of = i < HD ? a.q_gain : a.k_gain;
            gain[i / HD][i % HD] = of ? of[i % HD] : 1.f;
        }
    lds_barrier();
    if (r.rot > 0) rc_angles(rc_cs, r, pos, count, 1.f);
    lds_barrier();
    const bool turned = j < r.rot / 16;
    for (; th < items; th += RC_WG / LANES) {
        const Data x = next;
        next = load(min(th + RC_WG / LANES, items - 1));
        const int t = by_heads(th), h = th - t * heads;
        const int64_t at = k_at[t], tok = tok0 + t;
        const bool is_q = h < a.n_heads, is_k = !is_q && h < a.n_heads + c.n_kv;
        if (at == -2 || (at == -1 && !is_q)) continue;
        const int kh = is_k ? h - a.n_heads : h - a.n_heads - c.n_kv;
        bf16_t* y = is_q ? a.q_out + tok * a.ldqo + (int64_t)h * HD : is_k ? c.k + at + kh * c.k_head : c.v + v_at[t] + kh * c.v_head;
        if (!is_q && !is_k) {                             // values: as they are
            *reinterpret_cast<uint4*>(y + ia) = x.a;
            *reinterpret_cast<uint4*>(y + ib) = x.b;
            continue;
        }
        float f[8], g[8];
        rc_widen(x.a, f);
        rc_widen(x.b, g);
        if (NORM) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(f[i], f[i], fmaf(g[i], g[i], ss));
#pragma unroll
            for (int off = LANES / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
            const float scale = rsqrtf(ss * (1.f / HD) + a.eps);
            float ga[8], gb[8];
            rc_load(gain[is_q ? 0 : 1] + ia, ga);
            rc_load(gain[is_q ? 0 : 1] + ib, gb);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[i] *= scale * ga[i];
                g[i] *= scale * gb[i];
            }
        }
        if (turned) rc_turn(f, g, rc_cs + t * (r.rot / 2) + 8 * j, r.interleaved);
        rc_store(y + ia, f);
        rc_store(y + ib, g);
    }
}

// ---- accepted tokens together ------------------------------------------------------------------------------------
// A workgroup has one sequence and 256 of its rows' 16-byte pieces, each thread one piece of every row: a thread reads four rows ahead of what it
// writes.  Entry j goes to place j + 1 and comes from a place behind that one or from it, so that no thread writes a piece that it has yet to read.  One tree's take 2.2 us, 256 trees' 3.9:
// the chain of loads from an entry to its row
__global__ __launch_bounds__(RC_WG) void cache_keep_kernel(PagedCache c, const int32_t* __restrict__ cu_q, int64_t n, const int32_t* __restrict__ rows,
                                                           const int32_t* __restrict__ n_kept, int head_dim, QuickDiv by_page, QuickDiv by_pieces) {
    __shared__ int64_t k_from[64], k_to[64], v_from[64], v_to[64];
    __shared__ int moves;
    const int seq = blockIdx.x;
    const PagedSeq s = paged_seq(c, cu_q, (int)n, seq);
    const int kept = min(n_kept[seq], s.nq - 1), base = s.nk - s.nq, pieces = (int)by_pieces.d;
    const int piece = blockIdx.y * RC_WG + threadIdx.x, per_tensor = c.n_kv * pieces;
    const bool is_k = piece < per_tensor, there = piece < 2 * per_tensor;
    const int in = is_k ? piece : piece - per_tensor, head = by_pieces(in), at = 8 * (in - head * pieces);
    bf16_t* x = is_k ? c.k + head * c.k_head + at : c.v + head * c.v_head + at;
    const int64_t* from = is_k ? k_from : v_from;
    const int64_t* to = is_k ? k_to : v_to;
    for (int j0 = 0; j0 < kept; j0 += 64) {
        if (threadIdx.x < 64) {
            const int j = j0 + (int)threadIdx.x;
            int64_t p0 = 0, p1 = 0;
            int s0 = 0, s1 = 0;
            bool moved = j < kept;
            if (moved) {
                const int row = rows[s.q0 + j];
                moved = row > j + 1 && row < s.nq && paged_slot(c, by_page, seq, base + row, p0, s0) && paged_slot(c, by_page, seq, base + j + 1, p1, s1);
            }
            // (one behind the other: those that stay would be branches around each load, and a wait for it)
            const uint64_t m = __builtin_amdgcn_ballot_w64(moved);
            const int at = __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
            if (moved) {
                k_from[at] = p0 * c.k_page + s0 * c.k_row;
                v_from[at] = p0 * c.v_page + s0 * c.v_row;
                k_to[at] = p1 * c.k_page + s1 * c.k_row;
                v_to[at] = p1 * c.v_page + s1 * c.v_row;
            }
            if (threadIdx.x == 0) moves = __builtin_popcountll(m);
        }
        lds_barrier();
        const int some = there ? moves : 0;
        typedef uint32_t vec __attribute__((ext_vector_type(4)));
        for (int i = 0; i < some; i += 4) {
            vec v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const vec*>(x + from[min(i + u, some - 1)]);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u < some) *reinterpret_cast<vec*>(x + to[i + u]) = v[u];
        }
        lds_barrier();
    }
}

}  // namespace

hipError_t launch_rope(const RopeArgs& r, bool f32, const RopeTensor& q, const RopeTensor& k, const int32_t* positions, int64_t n, int head_dim, bool back, hipStream_t st) {
    return f32 ? launch_rope_typed<float>(r, q, k, positions, n, head_dim, back, st) : launch_rope_typed<bf16_t>(r, q, k, positions, n, head_dim, back, st);
}

hipError_t launch_cache_append(const PagedCache& c, int head_dim, const RopeArgs& r, const CacheAppend& a, hipStream_t st) {
    if (a.n == 0 || c.n_seq == 0) return hipSuccess;
    const int per = a.n >= 1024 ? RC_MOST : 1;
    const dim3 blocks((unsigned)((a.n + per - 1) / per));
    const size_t smem = (size_t)per * (r.rot / 2) * sizeof(float2);
    const QuickDiv by_page(c.page_size), by_heads(a.n_heads + 2 * c.n_kv);
    auto* f = head_dim == 128 ? (a.norm ? cache_append_kernel<128, true> : cache_append_kernel<128, false>)
                              : (a.norm ? cache_append_kernel<64, true> : cache_append_kernel<64, false>);
    hipLaunchKernelGGL(f, blocks, dim3(RC_WG), smem, st, c, r, a, per, by_page, by_heads);
    return hipGetLastError();
}

hipError_t launch_cache_keep(const PagedCache& c, int head_dim, const int32_t* cu_q, int64_t n, const int32_t* rows, const int32_t* n_kept, hipStream_t st) {
    if (n == 0 || c.n_seq == 0) return hipSuccess;
    const int pieces = 2 * c.n_kv * head_dim / 8;
    hipLaunchKernelGGL(cache_keep_kernel, dim3((unsigned)c.n_seq, (unsigned)((pieces + RC_WG - 1) / RC_WG)), dim3(RC_WG), 0, st, c, cu_q, n, rows, n_kept, head_dim,
                       QuickDiv(c.page_size), QuickDiv(head_dim / 8));
    return hipGetLastError();
}

}  // namespace agzo
