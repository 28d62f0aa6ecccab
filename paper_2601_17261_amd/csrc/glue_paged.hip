// Attention of new tokens over a cache of keys and values in pages, with grouped heads: a sequence's new tokens are its last places,
//     o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i k_j - lse_i),  lse_i = log sum_j exp(scale q_i k_j),
// j over the keys in front of the new tokens, and of those the ones up to i, or the ones that i's bits of a tree name.
//
// A row is a (query, head) pair, row r of a sequence and key head being head r mod G of query r / G (G heads to a key head), so that a tile of rows is full whether it
// holds many queries or one with its group's heads.  Products are v_mfma_f32_32x32x16_bf16, made transposed: a lane holds for one row the scores of the
// positions 8 (e / 4) + 4 (lane / 32) + e % 4 of a block of 32 keys, and its probabilities go into the second product as they are, whose other operand is read
// from LDS with a transposition.  Keys and values reach LDS through registers, 16 rows to a group, so that where a page's size is a multiple of 16 (WHOLE) a
// group has one page, found by a scalar load; else every lane looks its rows' pages up.  Pages are looked up a tile ahead of the loads that they lead to.
//
// Lengths are on the device, so how the work is shared out is worked out there too, by every workgroup alike: all row tiles' key tiles together over the workgroups
// that are wanted is a share, and what has more keys than that is made in equal shares of them, joined by a second launch.  However uneven the
// lengths are, no workgroup has more than a share, and few rows on many keys (single tokens, trees) fill the device.
//
// What a masked place holds takes part in nothing: scores there are replaced, and where a workgroup's results are not finite it goes over its tiles once more with
// care, with such values taken out, and what the visible ones amount to found by a product of two indicators.
#include <atomic>

#include "packed_tiles.h"
#include "paged.h"

namespace agzo {

namespace {

constexpr int PG_WAVES = 4, PG_ROWS = 32 * PG_WAVES, PG_KEYS = PK_T;      // rows of a workgroup, keys of a tile

struct PgOut { float* part; float2* part_ml; int slots, target, least; QuickDiv by_kv, by_group, by_page; };

// One workgroup's work: a tile of rows of a sequence, and the tiles [from, to) of its keys that it goes over, had every row seen all.  slot: where its sums go, -1: it
// is not shared out
struct PgUnit { PagedSeq s; int seq, tile, share, per, slot; };

__device__ __forceinline__ float pg_total(float x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// Tiles of keys of a share: those of all row tiles over the workgroups of a key head that are wanted, `least` at least.  (In fp32: the same in every workgroup, which is
// all that is asked of it)
template <int ROWS, int KEYS>
__device__ __forceinline__ int pg_share(const PagedCache& c, const PagedAttention& a, const PgOut& o, int G) {
    float work = 0.f;
    for (int b = 0; b < c.n_seq; b += 64) {
        const int lane = threadIdx.x & 63;
        const PagedSeq s = paged_seq(c, a.cu_q, (int)a.total_q, min(b + lane, c.n_seq - 1));
        const int rows = (int)(((uint32_t)s.nq * (uint32_t)G + (ROWS - 1)) / ROWS), keys = (s.nk + KEYS - 1) / KEYS;
        work += pg_total(b + lane < c.n_seq ? (float)rows * (float)keys : 0.f);
    }
    return (int)fminf(1073741824.f, fmaxf((float)o.least, ceilf(work / (float)o.target)));
}

// shares of a sequence with so many tiles of keys, and tiles of each
__device__ __forceinline__ int pg_shares(int keys, int chunk, int& per) {
    const int shares = max(1, (keys + chunk - 1) / chunk);
    per = max(1, (keys + shares - 1) / shares);
    return shares;
}

// Unit number t of all sequences' units
template <int ROWS, int KEYS>
__device__ __forceinline__ bool pg_find(const PagedCache& c, const PagedAttention& a, const PgOut& o, int t, int G, PgUnit& u) {
    const int lane = threadIdx.x & 63, chunk = pg_share<ROWS, KEYS>(c, a, o, G);
    int slots = 0;
    for (int b = 0; b < c.n_seq; b += 64) {
        const PagedSeq s = paged_seq(c, a.cu_q, (int)a.total_q, min(b + lane, c.n_seq - 1));
        const int rows = b + lane < c.n_seq ? (int)(((uint32_t)s.nq * (uint32_t)G + (ROWS - 1)) / ROWS) : 0;
        int per;
        const int shares = pg_shares((s.nk + KEYS - 1) / KEYS, chunk, per), count = rows * shares, split = shares > 1 ? count : 0;
        const int sum = pk_scan(count), splits = pk_scan(split), total = __builtin_amdgcn_readlane(sum, 63);
        if (t < total) {
            const int src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(sum > t));
            const int in = t - __builtin_amdgcn_readlane(sum - count, src), tiles = __builtin_amdgcn_readlane(rows, src);
            u.seq = b + src;
            u.s = PagedSeq{__builtin_amdgcn_readlane(s.q0, src), __builtin_amdgcn_readlane(s.nq, src), __builtin_amdgcn_readlane(s.nk, src)};
            u.per = __builtin_amdgcn_readlane(per, src);
            u.share = in / tiles;
            // (a prompt's last rows see most: they come first)
            u.tile = tiles - 1 - (in - u.share * tiles);
            u.slot = __builtin_amdgcn_readlane(split, src) > 0 ? slots + __builtin_amdgcn_readlane(splits - split, src) + u.share * tiles + u.tile : -1;
            return true;
        }
        t -= total;
        slots += __builtin_amdgcn_readlane(splits, 63);
    }
    return false;
}

// The 32 keys from kb on that new token q of a sequence sees, a bit for each
__device__ __forceinline__ uint32_t pg_seen(const PagedAttention& a, const PagedSeq& s, int q, int kb) {
    const int before = s.nk - s.nq, rel = kb - before;      // the first one's number among the new tokens
    auto low = [](int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; };
    if (!a.tree) return low(q - rel + 1);
    const uint32_t* row = a.tree + (int64_t)(s.q0 + q) * a.ld_tree;
    auto word = [&](int i) { return i >= 0 && i < a.words ? row[i] : 0u; };
    const int at = rel >> 5, sh = rel & 31;                 // (rounded down)
    const uint32_t bits = (rel <= -32 ? 0u : word(at) >> sh) | (sh ? word(at + 1) << (32 - sh) : 0u);
    return (bits | low(-rel)) & low(s.nk - kb);
}

// whether new token q sees no key at all
__device__ __forceinline__ bool pg_empty(const PagedAttention& a, const PagedSeq& s, int q) {
    const int before = s.nk - s.nq;
    if (!a.tree) return q + before < 0;
    if (before > 0) return false;
    uint32_t any = 0;
    for (int kb = 0; kb < s.nk; kb += 32) any |= pg_seen(a, s, q, kb);
    return any == 0;
}

// 16 keys' rows on their way to LDS, by one wave: the keys kg, .. (those past the sequence's last one repeat it)
template <int HD, bool WHOLE>
struct PgGroup {
    static constexpr int N = HD / 32, ROWS = 16 / N;        // loads, rows of a load
    uint4 data[N];
    struct Pages { int id[WHOLE ? 1 : N]; };
    static __device__ __forceinline__ int row_of_lane() {
        int lane = (int)threadIdx.x;
        asm volatile("" : "+v"(lane));
        return (lane & 63) / (HD / 8);
    }
    static __device__ __forceinline__ Pages pages(const PagedCache& c, const QuickDiv& by_page, const int32_t* table, int kg, int nk) {
        Pages p;
        if (WHOLE) {
            p.id[0] = table[by_page(min(kg, nk - 1))];
        } else {
            const int r = row_of_lane();
#pragma unroll
            for (int i = 0; i < N; ++i) p.id[WHOLE ? 0 : i] = table[by_page(min(kg + r + ROWS * i, nk - 1))];
        }
        return p;
    }
    // base: the tensor at the key head.  (Ids that are no page's are taken as the nearest)
    __device__ __forceinline__ void load(const PagedCache& c, const QuickDiv& by_page, const bf16_t* base, int64_t page_ld, int64_t row_ld, const Pages& p, int kg, int nk) {
        const int r = row_of_lane(), most = (int)c.n_pages - 1;
        const int chunk = ((int)(threadIdx.x % (HD / 8)) ^ pk_swz<HD>(r)) << 4;
        if (WHOLE) {
            const int first = min(kg, nk - 1), slot = first - by_page(first) * c.page_size, left = nk - 1 - first;
            const int64_t page = min(max(p.id[0], 0), most);
            const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(base + page * page_ld + slot * row_ld), 0, (int)0xFFFFFFFFu, 0x00020000);
#pragma unroll
            for (int i = 0; i < N; ++i)
                data[i] = pk_load16(rsrc, (int)(__umul24((uint32_t)min(r + ROWS * i, left), (uint32_t)(2 * row_ld)) + (uint32_t)(chunk ^ (pk_swz<HD>(ROWS * i) << 4))), 0);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int key = min(kg + r + ROWS * i, nk - 1), slot = key - by_page(key) * c.page_size;
                const int64_t page = min(max(p.id[WHOLE ? 0 : i], 0), most);
                const char* at = reinterpret_cast<const char*>(base + page * page_ld + slot * row_ld) + (chunk ^ (pk_swz<HD>(ROWS * i) << 4));
                data[i] = *reinterpret_cast<const uint4*>(at);
            }
        }
    }
    // to rows 16 g .. of a tile
    __device__ __forceinline__ void store(char* tile, int g) const {
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<uint4*>(tile + (g * N + i) * 1024 + (threadIdx.x & 63) * 16) = data[i];
    }
};

// ones and zeros of 32 bits of keys, as a lane's fragments of two times 16 positions
__device__ __forceinline__ void pg_fragments(uint32_t seen, PkFrag* f) {
    const uint32_t m = seen >> (4 * ((threadIdx.x >> 5) & 1));
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int at = 16 * s + (w >> 1) * 8 + (w & 1) * 2;
            f[s].w[w] = ((m >> at) & 1 ? 0x3F80u : 0u) | ((m >> (at + 1)) & 1 ? 0x3F800000u : 0u);
        }
}

// ---- many rows ---------------------------------------------------------------------------------------------------
// Four waves of 32 rows against tiles of 64 keys that they share, two tiles of K and V in LDS, two workgroups to a compute unit, which fill each other's
// waits: the shape of attention over packed sequences, for the same reasons.
// fine: the probabilities go into the second product in two bf16 parts (16 bits).  For few rows on many keys, whose time is the keys' reading: their sums are of few large
// probabilities often, whose roundings no others' balance.
// true: stored nothing, the tiles have to be gone over with care
template <int HD, bool WHOLE, bool fine, bool careful>
__device__ __forceinline__ bool pg_forward(const PagedCache& c, const PagedAttention& a, const PgOut& o, pk_lchar lds) {
    char* smem = (char*)lds;
    const int lds_at = (int)(uint32_t)(uintptr_t)lds;
    constexpr int TILE = PG_KEYS * HD * 2, KS = HD / 16, DB = HD / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hi = lane >> 5;
    // the key heads side by side: an XCD (workgroup number mod 8) then has few of them
    const int G = (int)o.by_group.d, unit = (int)blockIdx.x, at = o.by_kv(unit), kvh = unit - at * c.n_kv;
    PgUnit u;
    if (!pg_find<PG_ROWS, PG_KEYS>(c, a, o, at, G, u)) return false;
    const PagedSeq s_ = u.s;
    if (u.slot >= o.slots) return false;      // (offsets that do not grow: more of it than there is room for)
    const int R = s_.nq * G, row0 = u.tile * PG_ROWS + wave * 32, shift = s_.nk - s_.nq;
    // The lane's row: its query, its head.  (Worked out where they are needed, from a lane number that the compiler does not know again: kept through the loop they
    // are spilled)
    struct Row { int q, head; bool mine; };
    auto row_of_lane = [&]() __attribute__((always_inline)) {
        int lane_ = (int)threadIdx.x & 31;
        asm volatile("" : "+v"(lane_));
        const int row = min(row0 + lane_, R - 1), q = o.by_group(row);
        return Row{q, kvh * G + row - q * G, row0 + lane_ < R};
    };
    // the last key that all of the wave's rows see, the last that one of them may, and the last that one of the workgroup's may
    const int wfirst = a.tree ? shift - 1 : o.by_group(min(row0, R - 1)) + shift;
    const int wlast = row0 >= R ? -1 : a.tree ? s_.nk - 1 : o.by_group(min(row0 + 31, R - 1)) + shift;
    const int last = a.tree ? s_.nk - 1 : o.by_group(min((u.tile + 1) * PG_ROWS - 1, R - 1)) + shift;
    const int tiles = last < 0 ? 0 : last / PG_KEYS + 1;
    const int j0 = u.share * u.per, j1 = min(tiles, j0 + u.per);
    // (a share that none of the row tile sees.  The first one is there for rows that see nothing at all)
    if (j0 >= j1 && u.share > 0) return false;
    const bf16_t* Kh = c.k + kvh * c.k_head;
    const bf16_t* Vh = c.v + kvh * c.v_head;
    const int32_t* table = c.table + (int64_t)u.seq * c.ld_table;
    typedef PgGroup<HD, WHOLE> Group;
    Group lk, lv;
    typename Group::Pages next;
    auto find = [&](int j) __attribute__((always_inline)) { next = Group::pages(c, o.by_page, table, j * PG_KEYS + 16 * wave, s_.nk); };
    auto request = [&](int j) __attribute__((always_inline)) {
        lk.load(c, o.by_page, Kh, c.k_page, c.k_row, next, j * PG_KEYS + 16 * wave, s_.nk);
        lv.load(c, o.by_page, Vh, c.v_page, c.v_row, next, j * PG_KEYS + 16 * wave, s_.nk);
    };
    auto arrive = [&](int j) __attribute__((always_inline)) {
        lk.store(smem + (j & 1) * (2 * TILE), wave);
        lv.store(smem + (j & 1) * (2 * TILE) + TILE, wave);
    };
    const PkOffsets<HD> off;
    PkFrag qf[KS];
    auto begin = [&]() __attribute__((always_inline)) {
        if (j0 >= j1) return;
        find(j0);
        request(j0);
        const Row r = row_of_lane();
        const bf16_t* qsrc = a.q + (int64_t)(s_.q0 + r.q) * a.ldq + (int64_t)r.head * HD + 8 * hi;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks].u = *reinterpret_cast<const uint4*>(qsrc + 16 * ks);
        find(min(j0 + 1, j1 - 1));
        __builtin_amdgcn_s_waitcnt(0x0F70);
    };
    const float sc = a.scale * PK_LOG2E;
    // sums are rescaled when a maximum has grown by more than 2^8 times: what they and the probabilities are relative to need not be the maximum itself
    const float slack = 8.f / sc;
    pk_floatx16 acc[DB];
    float top, topsc, l;
    auto one_tile = [&](int j) __attribute__((always_inline)) {
        const int kb = j * PG_KEYS;
        if (kb > wlast) return;                                          // (wave-uniform)
        const char* kt = smem + (j & 1) * (2 * TILE);
        const PkOffsets<HD> of(off, lds_at + (j & 1) * (2 * TILE));
        PkFrag f[4];
        auto read_k = [&](int i) __attribute__((always_inline)) { f[i & 3].v = of.row(i & 1, i >> 1); };
        auto read_v = [&](int i) __attribute__((always_inline)) { pk_read_trans<HD>(of, TILE + (i / DB) * 16 * HD * 2, i % DB, f[i & 3]); };
        const pk_floatx16 zero = {};
        pk_floatx16 s[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) read_k(i);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
            s[i & 1] = pk_mfma(f[i & 3], qf[i >> 1], i < 2 ? zero : s[i & 1]);
            if (i + 4 < 2 * KS) read_k(i + 4);
            else read_v(i + 4 - 2 * KS);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        const bool mask = kb + PG_KEYS - 1 > wfirst;                     // (wave-uniform)
        if (mask) {
            const int q = row_of_lane().q;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t m = pg_seen(a, s_, q, kb + 32 * h) >> (4 * hi);
#pragma unroll
                for (int e = 0; e < 16; ++e) s[h][e] = m & (1u << pk_pos(e)) ? s[h][e] : -INFINITY;
            }
        }
        float mx = s[0][0];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[h][e]);
        mx = pk_max_halves(mx);
        if (__any(mx > top + slack)) {
            const float grown = fmaxf(top, mx), to = grown == -INFINITY ? 0.f : grown * sc;
            const float alpha = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(topsc - to);
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
            top = grown;
            topsc = to;
        }
        PkFrag pf[4], pl[4];
        // (rounded to bf16 for the second product, whose sums are fp32; their sum is taken before that)
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][e & 15], sc, -topsc)), p1 = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][(e & 15) + 1], sc, -topsc));
            l += p0 + p1;
            const uint32_t w = pack_bf16x2(p0, p1);
            pf[e >> 3].w[(e & 7) >> 1] = w;
            if (fine) pl[e >> 3].w[(e & 7) >> 1] = pack_bf16x2(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xFFFF0000u));
        }
        if (careful) {
            const int q = row_of_lane().q;
            PkFrag seen[4];
            pg_fragments(pg_seen(a, s_, q, kb), seen);
            pg_fragments(pg_seen(a, s_, q, kb + 32), seen + 2);
            pk_second_careful<HD, true, fine>(kt + TILE, pf, pl, seen, acc);
            return;
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < 4 * DB; ++i) {
            acc[i % DB] = pk_mfma(f[i & 3], pf[i / DB], acc[i % DB]);
            if (fine) acc[i % DB] = pk_mfma(f[i & 3], pl[i / DB], acc[i % DB]);
            if (i + 4 < 4 * DB) read_v(i + 4);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
    };
#pragma unroll
    for (int d = 0; d < DB; ++d) pk_zero(acc[d]);
    top = -INFINITY; topsc = 0.f; l = 0.f;
    begin();
    if (j0 < j1) arrive(j0);
    for (int j = j0; j < j1; ++j) {
        lds_barrier();
        if (j + 1 < j1) {
            request(j + 1);
            find(min(j + 2, j1 - 1));
        }
        one_tile(j);
        if (j + 1 < j1) arrive(j + 1);
    }
    if (!careful && __syncthreads_or(row_of_lane().mine && pk_not_finite(acc))) return true;
    l = pk_sum_halves(l);
    const Row r = row_of_lane();
    if (u.slot >= 0) {
        if (!r.mine) return false;
        const int64_t to = ((int64_t)u.slot * c.n_kv + kvh) * PG_ROWS + wave * 32 + (lane & 31);
        float* part = o.part + to * HD + 4 * hi;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4*>(part + 32 * db + 8 * g) = make_float4(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]);
        if (hi == 0) o.part_ml[to] = make_float2(top == -INFINITY && l == 0.f ? -INFINITY : topsc, l);
        return false;
    }
    const bool empty = pg_empty(a, s_, r.q);
    const int64_t tok = s_.q0 + r.q;
    pk_store<HD>(acc, empty ? 0.f : 1.f / l, a.out + tok * a.ldo + (int64_t)r.head * HD, r.mine);
    if (a.lse && r.mine && hi == 0) a.lse[tok * a.n_heads + r.head] = empty ? -INFINITY : (topsc + log2f(l)) * PK_LN2;
    return false;
}
// (a function that is called: its registers are not the kernel's)
template <int HD, bool WHOLE, bool fine>
__device__ __noinline__ void pg_forward_again(PagedCache c, PagedAttention a, PgOut o, pk_lchar lds) { (void)pg_forward<HD, WHOLE, fine, true>(c, a, o, lds); }
template <int HD, bool WHOLE, bool fine>
__global__ __launch_bounds__(64 * PG_WAVES) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_kernel(PagedCache c, PagedAttention a, PgOut o) {
    extern __shared__ __align__(1024) char pg_dynamic[];
    if (pg_forward<HD, WHOLE, fine, false>(c, a, o, (pk_lchar)pg_dynamic)) pg_forward_again<HD, WHOLE, fine>(c, a, o, (pk_lchar)pg_dynamic);
}

// ---- shares joined -----------------------------------------------------------------------------------------------
// HD / 4 lanes a row, 256 / (HD / 4) rows of one unit's: a workgroup for every row tile's rows, of sequences that are not shared out none
template <int HD, int ROWS, int KEYS>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedCache c, PagedAttention a, PgOut o) {
    constexpr int LANES = HD / 4;
    const int G = (int)o.by_group.d;
    const int64_t rows = a.total_q * a.n_heads, at_row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES;
    // (the lanes of a wave have one token's heads or two tokens': the sequence is looked for by all of them)
    const int64_t row = min(at_row, rows - 1);
    const int tok = (int)(row / a.n_heads), head = (int)(row - (int64_t)tok * a.n_heads), j = threadIdx.x % LANES;
    const int chunk = pg_share<ROWS, KEYS>(c, a, o, G);
    PagedSeq s{};
    int seq = -1, slot = 0, per = 1, shares = 1;
    int before = 0;
    for (int b = 0; b < c.n_seq; b += 64) {
        const int lane = threadIdx.x & 63;
        const PagedSeq mine = paged_seq(c, a.cu_q, (int)a.total_q, min(b + lane, c.n_seq - 1));
        const int n_rows = b + lane < c.n_seq ? (int)(((uint32_t)mine.nq * (uint32_t)G + (ROWS - 1)) / ROWS) : 0;
        int its_per;
        const int its_shares = pg_shares((mine.nk + KEYS - 1) / KEYS, chunk, its_per), split = its_shares > 1 ? n_rows * its_shares : 0;
        const int splits = pk_scan(split);
#pragma unroll
        for (int w = 0; w < 64 / LANES; ++w) {
            const int t = __builtin_amdgcn_readlane(tok, w * LANES);
            const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(b + lane < c.n_seq && mine.q0 <= t));
            if (n == 0) continue;
            const int q0 = __builtin_amdgcn_readlane(mine.q0, n - 1), nq = __builtin_amdgcn_readlane(mine.nq, n - 1), nk = __builtin_amdgcn_readlane(mine.nk, n - 1);
            const int at = before + __builtin_amdgcn_readlane(splits - split, n - 1), p = __builtin_amdgcn_readlane(its_per, n - 1), sh = __builtin_amdgcn_readlane(its_shares, n - 1);
            if (lane / LANES == w) { s = PagedSeq{q0, nq, nk}; seq = b + n - 1; slot = at; per = p; shares = sh; }
        }
        before += __builtin_amdgcn_readlane(splits, 63);
    }
    if (at_row >= rows || seq < 0 || tok - s.q0 >= s.nq || shares == 1) return;
    const int kvh = o.by_group(head), q = tok - s.q0, R = s.nq * G, in = q * G + head - kvh * G, tile = in / ROWS, tiles = (R + ROWS - 1) / ROWS;
    // the shares that its row tile sees something of
    const int last = a.tree ? s.nk - 1 : o.by_group(min((tile + 1) * ROWS - 1, R - 1)) + s.nk - s.nq;
    const int used = last < 0 ? 1 : (last / KEYS + per) / per;
    if (slot + (used - 1) * tiles + tile >= o.slots) return;
    auto at = [&](int i) __attribute__((always_inline)) { return ((int64_t)(slot + i * tiles + tile) * c.n_kv + kvh) * ROWS + in - tile * ROWS; };
    // maxima and sums by share in the lanes of the row; a share that the row sees nothing of has no part
    float top = -INFINITY, l = 0.f;
    for (int s0 = 0; s0 < used; s0 += LANES) top = fmaxf(top, s0 + j < used ? o.part_ml[at(s0 + j)].x : -INFINITY);
#pragma unroll
    for (int w = LANES / 2; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < used; s0 += LANES) {
        const float2 m = o.part_ml[at(min(s0 + j, used - 1))];
        const float f = s0 + j >= used ? 0.f : m.y != m.y ? NAN : m.x != -INFINITY ? __builtin_amdgcn_exp2f(m.x - top) : 0.f;
        l += f == 0.f ? 0.f : f * m.y;
        const int n = min(LANES, used - s0);
        for (int i = 0; i < n; i += 4) {
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const float4*>(o.part + at(min(s0 + i + k, used - 1)) * HD + 4 * j);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float w = __shfl(f, i + k, LANES);              // (0 from the last share on)
                if (w != 0.f) { x.x = fmaf(w, v[k].x, x.x); x.y = fmaf(w, v[k].y, x.y); x.z = fmaf(w, v[k].z, x.z); x.w = fmaf(w, v[k].w, x.w); }
            }
        }
    }
#pragma unroll
    for (int w = LANES / 2; w > 0; w >>= 1) l += __shfl_xor(l, w);
    const bool empty = pg_empty(a, s, q);
    const float inv = empty ? 0.f : 1.f / l;
    *reinterpret_cast<uint2*>(a.out + (int64_t)tok * a.ldo + (int64_t)head * HD + 4 * j) = make_uint2(pack_bf16x2(x.x * inv, x.y * inv), pack_bf16x2(x.z * inv, x.w * inv));
    if (a.lse && j == 0) a.lse[row] = empty ? -INFINITY : (top + log2f(l)) * PK_LN2;
}

// ---- launches ----------------------------------------------------------------------------------------------------
// Workgroups wanted for each key head, and the fewest tiles of keys that a share has (it costs a workgroup's start, its sums and a launch that joins them)
constexpr int PG_WANTED = 512, PG_LEAST = 8;

struct PgPlan { int64_t units, row_tiles; int target, slots; };
PgPlan pg_plan(const PagedCache& c, const PagedAttention& a, int rows, int keys, int wanted, int least) {
    PgPlan p{};
    const int64_t G = a.n_heads / c.n_kv, most_keys = ((int64_t)c.max_pages * c.page_size + keys - 1) / keys;
    p.row_tiles = a.total_q * G / rows + std::min<int64_t>(c.n_seq, a.total_q);
    p.target = std::max(1, (wanted + c.n_kv - 1) / c.n_kv);
    // What is shared out has more tiles of keys than a share, so at most twice as many units as tiles / share; a share is all tiles / target at least
    // (the 64 more are for sums in fp32).  And no sequence has more than its room
    p.slots = most_keys <= least ? 0 : (int)std::min<int64_t>(2 * p.target + 64, p.row_tiles * ((most_keys + least - 1) / least));
    p.units = (p.row_tiles + p.slots) * c.n_kv;
    return p;
}

// so much LDS for a kernel, once on each device
template <typename F>
hipError_t pg_lds(F* f, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (e != hipSuccess || (done.load(std::memory_order_relaxed) & bit)) return e;
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(f), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

template <int HD, bool WHOLE, bool fine>
hipError_t pg_launch(const PagedCache& c, const PagedAttention& a, const PgOut& o, int64_t units, hipStream_t st) {
    constexpr int SMEM = 4 * PG_KEYS * HD * 2;
    static std::atomic<uint64_t> done{0};
    const hipError_t e = pg_lds(paged_kernel<HD, WHOLE, fine>, SMEM, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((paged_kernel<HD, WHOLE, fine>), dim3((unsigned)units), dim3(64 * PG_WAVES), SMEM, st, c, a, o);
    return hipGetLastError();
}

template <int HD>
hipError_t pg_launch_forward(const PagedCache& c, const PagedAttention& a, void* workspace, hipStream_t st) {
    const PgPlan p = pg_plan(c, a, PG_ROWS, PG_KEYS, PG_WANTED, PG_LEAST);
    const int64_t G = a.n_heads / c.n_kv, part_rows = (int64_t)p.slots * c.n_kv * PG_ROWS;
    float* part = static_cast<float*>(workspace);
    const PgOut o{part, reinterpret_cast<float2*>(part + part_rows * HD), p.slots, p.target, p.slots > 0 ? PG_LEAST : 1 << 30, QuickDiv(c.n_kv), QuickDiv((int)G), QuickDiv(c.page_size)};
    const int64_t blocks = (a.total_q * a.n_heads * (HD / 4) + 255) / 256;
    if (p.units >= kPackedUnits || blocks >= kPackedUnits) return hipErrorInvalidValue;
    const bool whole = c.page_size % 16 == 0, fine = a.total_q * G <= 512 * (int64_t)c.n_seq;
    const hipError_t e = whole ? (fine ? pg_launch<HD, true, true>(c, a, o, p.units, st) : pg_launch<HD, true, false>(c, a, o, p.units, st))
                               : (fine ? pg_launch<HD, false, true>(c, a, o, p.units, st) : pg_launch<HD, false, false>(c, a, o, p.units, st));
    if (e != hipSuccess || p.slots == 0) return e;
    hipLaunchKernelGGL((paged_join_kernel<HD, PG_ROWS, PG_KEYS>), dim3((unsigned)blocks), dim3(256), 0, st, c, a, o);
    return hipGetLastError();
}

}  // namespace

int64_t paged_units(const PagedCache& c, const PagedAttention& a) {
    const PgPlan p = pg_plan(c, a, PG_ROWS, PG_KEYS, PG_WANTED, PG_LEAST);
    return std::max(p.units, (a.total_q * a.n_heads * 32 + 255) / 256);
}
size_t paged_workspace_bytes(const PagedCache& c, const PagedAttention& a, int head_dim) {
    const PgPlan p = pg_plan(c, a, PG_ROWS, PG_KEYS, PG_WANTED, PG_LEAST);
    return (size_t)p.slots * c.n_kv * PG_ROWS * (head_dim * sizeof(float) + sizeof(float2));
}

hipError_t launch_paged_attention(const PagedCache& c, const PagedAttention& a, int head_dim, void* workspace, hipStream_t st) {
    if (a.total_q == 0 || c.n_seq == 0) return hipSuccess;
    return head_dim == 128 ? pg_launch_forward<128>(c, a, workspace, st) : pg_launch_forward<64>(c, a, workspace, st);
}

}  // namespace agzo
