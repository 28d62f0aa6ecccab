// Attention of new tokens over a cache of keys and values in pages, with grouped heads: a sequence's new tokens are its last places,
//     o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i k_j - lse_i),  lse_i = log sum_j exp(scale q_i k_j),
// j over the keys in front of the new tokens, and of those the ones up to i, or the ones that i's bits of a tree name.
//
// A row is a (query, head) pair, row r of a sequence and key head being head r mod G of query r / G (G heads to a key head), so that a tile of rows is full whether it
// holds many queries or one with its group's heads.  Products are made transposed: a lane's scores are one row's, and its probabilities go into the second product as
// they are, whose other operand is read from LDS with a transposition.  Where 128 or 256 rows are taken together they are v_mfma_f32_32x32x16_bf16, and a lane has the positions
// 8 (e / 4) + 4 (lane / 32) + e % 4 of a block of 32 keys; of 16 rows they are v_mfma_f32_16x16x32_bf16.  Keys and values reach LDS through registers, for 256 rows straight from
// memory, 16 rows to a group, so that where a page's size is a multiple of 16 (WHOLE) a group has one page, found by a scalar load; else every lane looks its rows' pages up.  Pages are
// looked up a tile ahead of the loads that they lead to.
//
// Lengths are on the device, so how the work is shared out is worked out there too, by every workgroup alike, and however uneven they are no workgroup has more than
// its share: few rows on many keys (single tokens, trees) fill the device.  What several workgroups have of a row tile a second launch joins.
//
// What a masked place holds takes part in nothing: scores there are replaced, and where a workgroup's results are not finite it goes over its tiles once more with
// care, with such values taken out of the products and added where they are seen.
#include <atomic>
#include <type_traits>

#include "packed_tiles.h"
#include "paged.h"
#include "paged_work.h"

namespace agzo {

namespace {

constexpr int PG_WAVES = 4;

// What a launch is told: the workgroups of each key head that there are places for at once, the keys of a row tile that a piece has at least, and the keys that go over in
// the time that sharing out costs (a piece's start, its sums, the launch that joins them)
struct PgCut { PagedSeq s; int tile, parts, slot, unused[2]; };      // a row tile that several workgroups have parts of, and the first one's slot; parts < 2: none
struct PgOut { float* part; float2* part_ml; PgCut* cuts; int places, least, cost; QuickDiv by_kv, by_group, by_page; };

// ---- who does what -----------------------------------------------------------------------------------------------
// Row tiles are one workgroup's each where that is about as soon done, or equal parts of each are, else the work of all of them in a row is cut into equal pieces, one to
// each place: a workgroup then has the end of one row tile, perhaps whole ones, and the beginning of another.  (64 single tokens on 200000 keys: 219 us with shares of each
// sequence for its own, 193 so.  Sums over the lanes by __shfl_up were most of a workgroup's start, 6 us)
// keys that go over in the time that a row tile's start and end take.  (Without them 15 of a prompt's short first row tiles went to one workgroup, and 2500 tokens of
// three prompts took 356 us for 293.)  Fewer where memory is busy: with few rows a piece's start is 4 to 5 us, in which a workgroup goes over 350 keys by itself and 80 among
// 512 that share the memory's rate.  (256 throughout: 64 single tokens on 200000 keys 159 us for 156; 64 throughout: trees on 5600 keys 19.1 us for 16.8)
// (256 rows: 2500 tokens of three prompts 275 us with 256, 250 with 448, 255 with 640)
constexpr int pg_start(int rows, bool busy) { return rows < 128 && busy ? 64 : rows > 128 ? 448 : 256; }
constexpr int PG_BUSY = 1024;      // ... from so many keys a workgroup on

template <int ROWS>
__device__ __forceinline__ PgWork pg_work_of(const PagedAttention& a, const PagedSeq& s, int G, bool there, int start) { return pg_work(there ? s.nq : 0, s.nk, G, ROWS, a.tree != nullptr, start); }

__device__ __forceinline__ int64_t pg_lane(int64_t x, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, lane));
}
template <int CTRL>
__device__ __forceinline__ int64_t pg_dpp(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, 0xF, 0xF, true) << 32 | (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true));
}
// sums over the lanes up to each (row_shr 1, 2, 4, 8 within 16 lanes; what comes from outside them is 0)
__device__ __forceinline__ int64_t pg_scan(int64_t x) {
    x += pg_dpp<0x111>(x);
    x += pg_dpp<0x112>(x);
    x += pg_dpp<0x114>(x);
    x += pg_dpp<0x118>(x);
    const int64_t a = pg_lane(x, 15), b = a + pg_lane(x, 31), c = b + pg_lane(x, 47);
    const int row = (threadIdx.x & 63) >> 4;
    return x + (row == 0 ? 0 : row == 1 ? a : row == 2 ? b : c);
}
// the largest of the lanes' (none below 0)
__device__ __forceinline__ int pg_max(int x) {
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true));
    return max(max(__builtin_amdgcn_readlane(x, 15), __builtin_amdgcn_readlane(x, 31)), max(__builtin_amdgcn_readlane(x, 47), __builtin_amdgcn_readlane(x, 63)));
}

// Where a piece of the work lies: a row tile, the part [from, to) of its work `all`; slot: where its sums go, -1: it is the whole row tile
struct PgUnit { PagedSeq s; int seq, tile, from, to, all, slot; };
__device__ __forceinline__ int pg_uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// (the same in all lanes, and known to be)
__device__ __forceinline__ PgUnit pg_uniform(const PgUnit& u) {
    return PgUnit{PagedSeq{pg_uniform(u.s.q0), pg_uniform(u.s.nq), pg_uniform(u.s.nk)}, pg_uniform(u.seq), pg_uniform(u.tile), pg_uniform(u.from), pg_uniform(u.to), pg_uniform(u.all),
                  pg_uniform(u.slot)};
}

// A workgroup's pieces of work, one after the other
template <int ROWS>
struct PgWalk {
    int64_t pos, end, start;      // work in front of what is left, and behind it; start: in front of sequence seq's row tile `tile`
    int64_t total, each;          // of all sequences; of a piece
    int seq, tile, index, pieces, start_cost;
    int parts, part;              // where each workgroup has one part of a row tile: of how many, which.  parts = 0: it is not so
    bool whole, first;
    PagedSeq s;
    PgWork w;

    // work in front of a piece
    __device__ __forceinline__ int64_t begin_of(int i) const { return min(i * each, total); }
    // its place: workgroup `index` of a key head's.  false: there is nothing for it
    __device__ __forceinline__ bool begin(const PagedCache& c, const PagedAttention& a, const PgOut& o, int index_, int G) {
        const int lane = threadIdx.x & 63;
        start_cost = 0;          // (not known yet)
        auto load = [&](int b, PagedSeq& its, PgWork& work) __attribute__((always_inline)) {
            its = paged_seq(c, a.cu_q, (int)a.total_q, min(b + lane, c.n_seq - 1));
            work = pg_work_of<ROWS>(a, its, G, b + lane < c.n_seq, start_cost);
        };
        PagedSeq its;
        PgWork work;
        int64_t sum = 0;          // of the first 64, which need no second look
        int tiles = 0, longest = 0, shortest = 0x7FFFFFFF;
        total = 0;
        for (int b = 0; b < c.n_seq; b += 64) {
            load(b, its, work);
            sum = pg_scan(pg_before(work, work.tiles));
            total += pg_lane(sum, 63);
            tiles += pk_total(work.tiles);
            longest = max(longest, pg_max(work.tiles ? pg_of(work, work.tiles - 1) : 0));
            shortest = min(shortest, 0x7FFFFFFF - pg_max(work.tiles ? 0x7FFFFFFF - work.first : 0));
        }
        start_cost = pg_start(ROWS, total >= (int64_t)o.places * PG_BUSY);
        const int64_t keys = total;
        total += (int64_t)start_cost * tiles;
        longest += start_cost;
        shortest += start_cost;
        sum += (int64_t)start_cost * pk_scan(work.tiles);
        work.first += start_cost;
        index = index_;
        first = true;
        // How long row tiles take one workgroup each: the longest, or the rounds that they go in, whose last one is short where row tiles are unlike (the heavy ones come
        // first).  2^52: what is worked out in fp64 is exact
        pieces = (int)min((int64_t)o.places, total / max(o.least, 1) + 1);
        const float share = (float)total / (float)pieces, rounds = (float)tiles / (float)o.places;
        const float alike = (float)shortest / (float)longest, alone = (float)total / (float)o.places * (1.f + alike * (ceilf(rounds) / rounds - 1.f));
        whole = fmaxf((float)longest, tiles > o.places ? alone : 0.f) <= share + (float)o.cost || o.places < 2 || total >= (1LL << 52);
        each = (int64_t)((double)total / pieces) + 1;
        parts = 0;
        int src = -1;
        if (whole) {
            if (index >= tiles) return false;
            pos = index;
            end = pos + 1;
        } else if (c.n_seq <= 64 && tiles < o.places) {
            // Every row tile in equal parts, so many that all of them have places, where such a part is little more than an even share: no workgroup then has a second piece to start.  (32
            // single tokens with 32 heads on one key head, 200000 keys, in both launches 44.6 us and 39.8 so, four trees of 17 tokens on 42000 keys 32.6 and 28.9, two prompts' pieces on 1700 keys
            // 23.3 and 20.4; what the choice costs where row tiles stay whole: 0.3 us for single tokens, 0.8 for more rows)
            const int most = work.tiles ? pg_of(work, work.tiles - 1) - start_cost : 0;      // keys of a sequence's longest
            const float even = (float)keys / (float)pieces;
            float size = fmaxf(even, (float)o.least);
            int k = 1, all = 0;
            for (int i = 0; i < 12; ++i, size *= 1.1f) {
                k = max((int)ceilf((float)most / size), 1);
                all = pk_total(work.tiles * k);
                if (all <= o.places) break;
            }
            if (all <= o.places && (float)pg_max((int)((float)most / (float)k)) <= even + (float)start_cost) {
                if (index >= all) return false;
                const int upto = pk_scan(work.tiles * k);
                src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > index));
                parts = __builtin_amdgcn_readlane(k, src);
                const int in = index - __builtin_amdgcn_readlane(upto - work.tiles * k, src);
                tile = (int)(((float)in + 0.5f) / (float)parts);
                part = in - tile * parts;
            }
        }
        if (!whole && parts == 0) {
            pos = begin_of(index);
            end = begin_of(index + 1);
            if (index >= pieces || pos >= end) return false;
        }
        if (whole && tiles > o.places && c.n_seq <= 64) {
            // level by level: a sequence's last row tile, which sees most, is as many levels high as it has row tiles, the next one a level less
            const int own = work.tiles;
            int low = 0, high = pg_max(own);
            while (low < high) {
                const int mid = (low + high) >> 1;
                if (pk_total(max(own - mid, 0)) <= index) high = mid;
                else low = mid + 1;
            }
            const int place = index - pk_total(max(own - low, 0));
            const uint64_t m = __builtin_amdgcn_ballot_w64(own >= low);
            const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
            src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(own >= low && before == place));
            tile = low - 1;
        }
        if (src >= 0) {
            take(its, src, 0, a, G);
            return true;
        }
        int64_t before = 0;
        for (int b = 0; b < c.n_seq; b += 64) {
            if (c.n_seq > 64) load(b, its, work);
            const int64_t own = whole ? (int64_t)work.tiles : pg_before(work, work.tiles);
            if (whole) sum = pk_scan(work.tiles);
            else if (c.n_seq > 64) sum = pg_scan(own);
            const uint64_t m = __builtin_amdgcn_ballot_w64(before + sum > pos);
            if (m) {
                const int src = __builtin_ctzll(m);
                take(its, src, b, a, G);
                const int64_t in = pos - before - (pg_lane(sum, src) - pg_lane(own, src));
                if (whole) {
                    tile = w.tiles - 1 - (int)in;
                    return true;
                }
                // the last row tile that begins at or in front of it
                int low = 0, high = w.tiles - 1;
                while (low < high) {
                    const int mid = (low + high + 1) >> 1;
                    if (pg_before(w, mid) <= in) low = mid;
                    else high = mid - 1;
                }
                tile = low;
                start = pos - (in - pg_before(w, low));
                return true;
            }
            before += pg_lane(sum, 63);
        }
        return false;
    }
    __device__ __forceinline__ void take(const PagedSeq& its, int src, int b, const PagedAttention& a, int G) {
        seq = b + src;
        s = PagedSeq{__builtin_amdgcn_readlane(its.q0, src), __builtin_amdgcn_readlane(its.nq, src), __builtin_amdgcn_readlane(its.nk, src)};
        w = pg_work_of<ROWS>(a, s, G, true, start_cost);
    }
    __device__ __forceinline__ PgUnit unit() const {
        PgUnit u;
        u.s = s;
        u.seq = seq;
        u.tile = tile;
        u.all = pg_of(w, tile);
        if (parts) {
            const int size = (int)((float)u.all / (float)parts) + (u.all >> 22) + 1;      // (fp32: parts times it are all)
            u.from = (int)min((int64_t)u.all, (int64_t)part * size);
            u.to = (int)min((int64_t)u.all, (int64_t)u.from + size);
            u.slot = parts == 1 ? -1 : 2 * index;
            return u;
        }
        u.from = whole ? 0 : (int)(pos - start);
        u.to = whole ? u.all : (int)min((int64_t)u.all, end - start);
        u.slot = u.from == 0 && u.to == u.all ? -1 : 2 * index + (first ? 0 : 1);
        return u;
    }
    // on to the next one
    __device__ __forceinline__ bool next(const PagedCache& c, const PagedAttention& a, int G) {
        if (whole || parts || start + pg_of(w, tile) >= end) return false;
        start += pg_of(w, tile);
        pos = start;
        first = false;
        if (++tile < w.tiles) return true;
        tile = 0;
        while (++seq < c.n_seq) {
            s = paged_seq(c, a.cu_q, (int)a.total_q, __builtin_amdgcn_readfirstlane(seq));
            w = pg_work_of<ROWS>(a, s, G, true, start_cost);
            if (w.tiles > 0) return true;
        }
        return false;
    }
};
// What a wave knows of the walk, in LDS while it goes over a piece: some forty scalar registers, which would be spilled otherwise.  (111 reloads in the kernel of 128 rows, 60 so; a piece's
// end waits for them: four trees on 600 keys 13.8 us and 13.1)
template <int ROWS>
__device__ __forceinline__ void pg_put(const PgWalk<ROWS>& w, uint32_t* at) {
    union { PgWalk<ROWS> walk; uint32_t word[sizeof(PgWalk<ROWS>) / 4]; } u;
    u.walk = w;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(PgWalk<ROWS>) / 4); ++i) at[i] = u.word[i];
}
template <int ROWS>
__device__ __forceinline__ void pg_get(PgWalk<ROWS>& w, const uint32_t* at) {
    union { PgWalk<ROWS> walk; uint32_t word[sizeof(PgWalk<ROWS>) / 4]; } u;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(PgWalk<ROWS>) / 4); ++i) u.word[i] = (uint32_t)__builtin_amdgcn_readfirstlane((int)at[i]);
    w = u.walk;
}
// A workgroup's entry for the launch that joins: the row tile that it has the beginning of and not the end, its last one.  (Worked out once more there it is 3 us)
template <int ROWS>
__device__ __forceinline__ void pg_leave(const PgOut& o, const PgWalk<ROWS>* walk, const PgUnit* u, int index, int kvh) {
    if (kvh != 0 || threadIdx.x != 0 || index >= o.places || o.places < 2) return;
    PgCut cut{};
    if (u && u->from == 0 && u->to < u->all) {
        cut.s = u->s;
        cut.tile = u->tile;
        cut.slot = u->slot;
        cut.parts = max(walk->parts, 1);
        const int64_t past = walk->start + u->all;
        while (walk->parts == 0 && index + cut.parts < walk->pieces && walk->begin_of(index + cut.parts) < past) ++cut.parts;
    }
    o.cuts[index] = cut;
}
// of a row tile's `tiles` tiles of keys those that a piece of its work has
__device__ __forceinline__ int pg_cut(int tiles, int part, int all) {
    return part >= all ? tiles : part <= 0 ? 0 : min(tiles, (int)ceil((double)tiles * part / all));
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
            // (a scalar load: a vector one's wait would be one for the tile's loads in front of it too)
            typedef const __attribute__((address_space(4))) int32_t* scalar;
            p.id[0] = ((scalar)(uintptr_t)table)[by_page(min(kg, nk - 1))];
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
                typedef uint32_t vec __attribute__((ext_vector_type(4)));
                const vec v = *reinterpret_cast<const vec*>(at);
                data[i] = make_uint4(v[0], v[1], v[2], v[3]);
            }
        }
    }
    // ... straight to LDS, at byte `to` on.  (Written out, for what the compiler does not see it does not wait for; so the wait states are written out too: five from a scalar register that
    // a vector instruction writes, a spilled one's reload say, to a load that reads it, one from m0)
    static __device__ __forceinline__ void direct(const PagedCache& c, const QuickDiv& by_page, const bf16_t* base, int64_t page_ld, int64_t row_ld, const Pages& p, int kg, int nk, int to) {
        static_assert(WHOLE, "one page");
        const int r = row_of_lane(), most = (int)c.n_pages - 1;
        const int chunk = ((int)(threadIdx.x % (HD / 8)) ^ pk_swz<HD>(r)) << 4;
        const int first = min(kg, nk - 1), slot = first - by_page(first) * c.page_size, left = nk - 1 - first;
        const int64_t page = min(max(p.id[0], 0), most);
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(base + page * page_ld + slot * row_ld), 0, (int)0xFFFFFFFFu, 0x00020000);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = (int)(__umul24((uint32_t)min(r + ROWS * i, left), (uint32_t)(2 * row_ld)) + (uint32_t)(chunk ^ (pk_swz<HD>(ROWS * i) << 4)));
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(to + i * 1024), "v"(at), "s"(rsrc) : "memory", "m0");
        }
    }
    // to rows 16 g .. of a tile
    __device__ __forceinline__ void store(char* tile, int g) const {
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<uint4*>(tile + (g * N + i) * 1024 + (threadIdx.x & 63) * 16) = data[i];
    }
};

// (the same in all lanes: a scalar register's)
__device__ __forceinline__ float pg_uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// whether any of a workgroup's lanes has it; a barrier, before which LDS has been read.  (Not __syncthreads_or(), which counts in LDS)
template <int WAVES>
__device__ __forceinline__ bool pg_any(bool x, int* flags) {
    const uint64_t m = __builtin_amdgcn_ballot_w64(x);
    if ((threadIdx.x & 63) == 0) flags[threadIdx.x >> 6] = m != 0;
    lds_barrier();
    int of = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) of |= flags[i];
    return __builtin_amdgcn_readfirstlane(of) != 0;
}

// ---- with care ---------------------------------------------------------------------------------------------------
// f x: what is not finite is so however small its weight, also where that is less than fp32 has
__device__ __forceinline__ bool pg_finite(float x) { return fabsf(x) <= __FLT_MAX__; }
__device__ __forceinline__ float pg_weighed(float f, float x) { return f == 0.f && !pg_finite(x) ? x : f * x; }
// y + f x
__device__ __forceinline__ float pg_weighed(float f, float x, float y) {
    const float r = fmaf(f, x, y);
    return pg_finite(r) ? r : y + pg_weighed(f, x);
}
// Values that are not finite, in a tile of KEYS values in LDS: in which keys there are any
template <int HD, int KEYS>
__device__ __forceinline__ uint64_t pg_bad_keys(const char* tile) {
    constexpr int LANES = HD / 8, ROWS = 64 / LANES;
    uint64_t keys = 0;
#pragma unroll 1
    for (int i = 0; i < KEYS / ROWS; ++i) {
        const uint4 v = *reinterpret_cast<const uint4*>(tile + i * 1024 + (threadIdx.x & 63) * 16);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        bool bad = false;
#pragma unroll
        for (int x = 0; x < 4; ++x) bad = bad || (w[x] & 0x7F80u) == 0x7F80u || (w[x] & 0x7F800000u) == 0x7F800000u;
        const uint64_t m = __builtin_amdgcn_ballot_w64(bad);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) keys |= (uint64_t)((m >> (r * LANES)) & ((1ull << LANES) - 1) ? 1 : 0) << (i * ROWS + r);
    }
    return keys;
}
// ... added to the sums of the rows that see them: infinities and NaN as they are, whatever their probability
template <int HD>
__device__ __forceinline__ void pg_add_bad(const char* tile, uint64_t keys, uint64_t seen, pk_floatx16 (&acc)[HD / 32]) {
    const int hi = (threadIdx.x >> 5) & 1;
#pragma unroll 1
    for (; keys; keys &= keys - 1) {
        const int r = __builtin_ctzll(keys);
        const bool sees = (seen >> r) & 1;
#pragma unroll
        for (int db = 0; db < HD / 32; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint2 v = *reinterpret_cast<const uint2*>(tile + r * (HD * 2) + (((4 * db + g) ^ pk_swz<HD>(r)) << 4) + 8 * hi);
                const uint32_t x[4] = {v.x << 16, v.x & 0xFFFF0000u, v.y << 16, v.y & 0xFFFF0000u};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (sees && (x[i] & 0x7F800000u) == 0x7F800000u) acc[db][4 * g + i] += __uint_as_float(x[i]);
            }
    }
}
__device__ __forceinline__ void pg_clean(PkFrag& f) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if ((f.w[w] & 0x7F80u) == 0x7F80u) f.w[w] &= 0xFFFF0000u;
        if ((f.w[w] & 0x7F800000u) == 0x7F800000u) f.w[w] &= 0xFFFFu;
    }
}
// the second product with them taken out, its fragments of 16 positions `at` on
template <int HD>
__device__ __forceinline__ void pg_second_clean(const PkOffsets<HD>& o, int at, const PkFrag (&p)[4], const PkFrag (&low)[4], pk_floatx16 (&acc)[HD / 32]) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int db = 0; db < HD / 32; ++db) {
            PkFrag f;
            pk_read_trans<HD>(o, at + s * 16 * HD * 2, db, f);
            pg_clean(f);
            acc[db] = pk_mfma(f, p[s], acc[db]);
            acc[db] = pk_mfma(f, low[s], acc[db]);
        }
}

// ---- many rows ---------------------------------------------------------------------------------------------------
// Whether a sequence's probabilities go into the second product in two bf16 parts (16 bits) and not in one: a single token's, which are few large ones often, and those of as few rows as
// the kernel of few rows is for.  By the sequence's own rows, so that what it is beside does not change its bits' number
__device__ __forceinline__ bool pg_two_parts(const PagedSeq& s, int G) { return s.nq <= 1 || s.nq * G <= 16; }

constexpr int PG_ROWS = 32 * PG_WAVES, PG_KEYS = PK_T;      // rows of a workgroup, keys of a tile
// Four waves of 32 rows against tiles of 64 keys that they share, two tiles of K and V in LDS, two workgroups to a compute unit, which fill each other's
// waits: the shape of attention over packed sequences, for the same reasons.  16 trees of 30 tokens with 4 heads on each of 8 key heads, 100000 keys, 415 MB, take 109 us in both
// launches, 3.8 TB/s; 2500 tokens behind and among 20001 keys, 235 GFLOP, 300 in this one, matrix cores busy 46 % of the time, vector instructions 49 %, mostly in turn.
// (Products of 16 x 16 x 32: 319 us for 283 with the join.  A second 256 workgroups with less work, or with priority: no gain, or a loss)
// The probabilities are rounded to bf16 for the second product, but for pg_two_parts.  In two parts throughout a result is off by 0.0017 of its norm and not 0.0023; 2500 tokens on 20001 keys in
// pages of 20 then take 480 us and not 368, 900 on 1700 keys 34 and not 29, trees of 17 on 42000 keys 47.5 and not 42.  (32 single tokens with 96 heads on two key heads, which have
// them: 35.6 and not 33.)  The second part's products are a pass over the values of their own: beside the first part's, a branch at each, tiles without them take 3 % longer, and with a
// copy of the whole pass for them registers are reloaded in the loop (16 trees of 30 tokens 156 us and not 109)
// true: stored nothing, the tiles have to be gone over with care
template <int HD, bool WHOLE, bool careful>
__device__ __forceinline__ bool pg_forward(const PagedCache& c, const PagedAttention& a, const PgOut& o, const PgUnit& u, int kvh, pk_lchar lds) {
    char* smem = (char*)lds;
    const int lds_at = (int)(uint32_t)(uintptr_t)lds;
    constexpr int TILE = PG_KEYS * HD * 2, KS = HD / 16, DB = HD / 32;
    static_assert(PG_KEYS == 16 * PG_WAVES, "16 keys are a wave's to load");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hi = lane >> 5;
    const int G = (int)o.by_group.d;
    const PagedSeq s_ = u.s;
    const bool fine = careful || pg_two_parts(s_, G);
    // (which of the 32 rows are a wave's: the other way round in the second 256 workgroups, of which a compute unit has one beside one of the first, so that tiles with few
    // rows keep all four SIMDs busy together: trees of 48 tokens, 192 rows in tiles of 128 and 64, 102.6 -> 97.3 us)
    const int block = (blockIdx.x >> 8) & 1 ? PG_WAVES - 1 - wave : wave;
    const int R = s_.nq * G, row0 = u.tile * PG_ROWS + block * 32, shift = s_.nk - s_.nq;
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
    const int j0 = pg_cut(tiles, u.from, u.all), j1 = pg_cut(tiles, u.to, u.all);
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
        const int tile_at = (j & 1) * (2 * TILE);
        const PkOffsets<HD> of(off.rows, off.trans[0], lds_at + tile_at);
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
            int lane_ = (int)threadIdx.x;                                // (as for rows)
            asm volatile("" : "+v"(lane_));
            const int hi_ = (lane_ >> 5) & 1;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t m = pg_seen(a, s_, q, kb + 32 * h) >> (4 * hi_);
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
                for (int e = 0; e < 16; ++e) acc[d][e] = careful ? pg_weighed(alpha, acc[d][e]) : acc[d][e] * alpha;
            top = grown;
            topsc = to;
        }
        PkFrag pf[4], pl[4];
        // (rounded to bf16 for the second product, whose sums are fp32; their sum is taken before that.  What that leaves is the second part)
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][e & 15], sc, -topsc)), p1 = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][(e & 15) + 1], sc, -topsc));
            l += p0 + p1;
            pf[e >> 3].w[(e & 7) >> 1] = pack_bf16x2(p0, p1);
            s[e >> 4][e & 15] = p0;
            s[e >> 4][(e & 15) + 1] = p1;
        }
        if (fine)
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                const uint32_t w = pf[e >> 3].w[(e & 7) >> 1];
                pl[e >> 3].w[(e & 7) >> 1] = pack_bf16x2(s[e >> 4][e & 15] - __uint_as_float(w << 16), s[e >> 4][(e & 15) + 1] - __uint_as_float(w & 0xFFFF0000u));
            }
        if (careful) {
            const int q = row_of_lane().q;
            const uint64_t seen = (uint64_t)pg_seen(a, s_, q, kb + 32) << 32 | pg_seen(a, s_, q, kb);
            pg_second_clean<HD>(of, TILE, pf, pl, acc);
            const char* values = smem + tile_at + TILE;
            pg_add_bad<HD>(values, pg_bad_keys<HD, PG_KEYS>(values), seen, acc);
            return;
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < 4 * DB; ++i) {
            acc[i % DB] = pk_mfma(f[i & 3], pf[i / DB], acc[i % DB]);
            if (i + 4 < 4 * DB) read_v(i + 4);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (fine) {                                                      // (workgroup-uniform)
#pragma unroll
            for (int i = 0; i < 4; ++i) read_v(i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 4 * DB; ++i) {
                acc[i % DB] = pk_mfma(f[i & 3], pl[i / DB], acc[i % DB]);
                if (i + 4 < 4 * DB) read_v(i + 4);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
    };
#pragma unroll
    for (int d = 0; d < DB; ++d) pk_zero(acc[d]);
    top = -INFINITY; topsc = 0.f; l = 0.f;
    begin();
    lds_barrier();                       // (of the piece before)
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
    __shared__ int flags[PG_WAVES];
    if (!careful && pg_any<PG_WAVES>(row_of_lane().mine && pk_not_finite(acc), flags)) return true;
    l = pk_sum_halves(l);
    const Row r = row_of_lane();
    if (u.slot >= 0) {
        if (!r.mine) return false;
        const int64_t to = ((int64_t)u.slot * c.n_kv + kvh) * PG_ROWS + block * 32 + (lane & 31);
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
template <int HD, bool WHOLE>
__global__ __launch_bounds__(64 * PG_WAVES) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_kernel(PagedCache c, PagedAttention a, PgOut o) {
    extern __shared__ __align__(1024) char pg_dynamic[];
    // the key heads side by side: an XCD (workgroup number mod 8) then has few of them
    const int at = o.by_kv((int)blockIdx.x), kvh = (int)blockIdx.x - at * c.n_kv, G = (int)o.by_group.d;
    __shared__ uint32_t walks[PG_WAVES][sizeof(PgWalk<PG_ROWS>) / 4];
    uint32_t* const saved = walks[threadIdx.x >> 6];
    PgWalk<PG_ROWS> walk;
    if (!walk.begin(c, a, o, at, G)) {
        pg_leave<PG_ROWS>(o, nullptr, nullptr, at, kvh);
        return;
    }
    while (true) {
        const PgUnit u = pg_uniform(walk.unit());
        pg_put(walk, saved);
        if (pg_forward<HD, WHOLE, false>(c, a, o, u, kvh, (pk_lchar)pg_dynamic)) (void)pg_forward<HD, WHOLE, true>(c, a, o, u, kvh, (pk_lchar)pg_dynamic);
        pg_get(walk, saved);
        if (walk.next(c, a, G)) continue;
        pg_leave<PG_ROWS>(o, &walk, &u, at, kvh);
        return;
    }
}

// ---- more rows on long caches --------------------------------------------------------------------------------------
// Eight waves of 32 rows against tiles of 64 keys, one workgroup to a compute unit.  Of a SIMD's two waves one makes products, a tile's second and the next tile's first, while the other
// has its exponentials: the second four waves are half a tile behind, and a barrier ends each half.  Tiles go straight from memory to LDS, K's asked for by the first four waves and V's by the
// others, three tiles ahead in rings of four (HD = 128: 96 KB on their way; a tile's place is free again before its next one is asked for, since both halves have read it a barrier
// before).  How far loads are is waited for by their number: the compiler does not see them, and would wait for all of them in front of each read of LDS.
// Against 128 rows with tiles through registers: 2500 tokens behind and among 20001 keys 312 -> 277 us in both launches (260 to 285 by card), 850 TFLOP/s, 4096 tokens of one prompt
// 161 -> 148, trees of 48 tokens on 60000 keys 88 -> 75, of 64 on 100000 155 -> 129: keys are read by half as many row tiles.  One tile by itself takes 1.7 us and not 1.4, so that short
// caches are not for it (15 prompts' pieces on 3100 keys 17.6 -> 20.6 us, two on 1700 keys 29 -> 33).  Matrix cores are busy 51 % of the time and vector instructions 51 %: the two halves
// do not fill each other, waves wait 28 % of theirs for loads, LDS and barriers and 29 % to issue.  With heads of 64 trees lose by it, 52 -> 59
constexpr int PG_WIDE = 8;
template <int HD, bool fine, bool careful>
__device__ __forceinline__ bool pg_wide(const PagedCache& c, const PagedAttention& a, const PgOut& o, const PgUnit& u, int kvh, pk_lchar lds) {
    char* smem = (char*)lds;
    const int lds_at = (int)(uint32_t)(uintptr_t)lds;
    constexpr int ROWS = 32 * PG_WIDE, TILE = PG_KEYS * HD * 2, KS = HD / 16, DB = HD / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hi = lane >> 5, late = wave >> 2, part16 = wave & 3;
    const int G = (int)o.by_group.d;
    const PagedSeq s_ = u.s;
    const int R = s_.nq * G, row0 = u.tile * ROWS + wave * 32, shift = s_.nk - s_.nq;
    struct Row { int q, head; bool mine; };
    auto row_of_lane = [&]() __attribute__((always_inline)) {
        int lane_ = (int)threadIdx.x & 31;
        asm volatile("" : "+v"(lane_));
        const int row = min(row0 + lane_, R - 1), q = o.by_group(row);
        return Row{q, kvh * G + row - q * G, row0 + lane_ < R};
    };
    const int wfirst = a.tree ? shift - 1 : o.by_group(min(row0, R - 1)) + shift;
    const int wlast = row0 >= R ? -1 : a.tree ? s_.nk - 1 : o.by_group(min(row0 + 31, R - 1)) + shift;
    const int last = a.tree ? s_.nk - 1 : o.by_group(min((u.tile + 1) * ROWS - 1, R - 1)) + shift;
    const int tiles = last < 0 ? 0 : last / PG_KEYS + 1;
    const int j0 = pg_cut(tiles, u.from, u.all), j1 = pg_cut(tiles, u.to, u.all);
    const bf16_t* base = late ? c.v + kvh * c.v_head : c.k + kvh * c.k_head;
    const int64_t page_ld = late ? c.v_page : c.k_page, row_ld = late ? c.v_row : c.k_row;
    const int32_t* table = c.table + (int64_t)u.seq * c.ld_table;
    typedef PgGroup<HD, true> Group;
    typename Group::Pages next;
    constexpr int N = Group::N;
    auto find = [&](int j) __attribute__((always_inline)) { next = Group::pages(c, o.by_page, table, j * PG_KEYS + 16 * part16, s_.nk); };
    // tile j asked for, into its place of four
    auto request = [&](int j, const typename Group::Pages& p) __attribute__((always_inline)) {
        Group::direct(c, o.by_page, base, page_ld, row_ld, p, j * PG_KEYS + 16 * part16, s_.nk, lds_at + (4 * late + (j & 3)) * TILE + part16 * (N * 1024));
    };
    const PkOffsets<HD> off;
    PkFrag qf[KS];
    lds_barrier();                       // (of the piece before)
    if (j0 < j1) {
        // (the first pages' numbers together: each is a load that the next step waits for)
        typename Group::Pages first[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            find(min(j0 + i, j1 - 1));
            first[i] = next;
        }
        find(min(j0 + 3, j1 - 1));
        const Row r = row_of_lane();
        const bf16_t* qsrc = a.q + (int64_t)(s_.q0 + r.q) * a.ldq + (int64_t)r.head * HD + 8 * hi;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks].u = *reinterpret_cast<const uint4*>(qsrc + 16 * ks);
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (j0 + i < j1) request(j0 + i, first[i]);
    }
    const float sc = pg_uniform(a.scale * PK_LOG2E), slack = pg_uniform(8.f / sc);
    pk_floatx16 acc[DB], s[2];
    PkFrag pf[4], pl[4];
    float top = -INFINITY, topsc = 0.f, l = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d) pk_zero(acc[d]);
    PkFrag f[4];
    // both products: the second of tile j - 1, the first of tile j
    auto matrix = [&](int j) __attribute__((always_inline)) {
        const bool second = j > j0 && (j - 1) * PG_KEYS <= wlast, first = j < j1 && j * PG_KEYS <= wlast;
        if (second) {
            const PkOffsets<HD> of(off, lds_at + (4 + ((j - 1) & 3)) * TILE);
            auto read_v = [&](int i) __attribute__((always_inline)) { pk_read_trans<HD>(of, (i / DB) * 16 * HD * 2, i % DB, f[i & 3]); };
            if (careful) {
                const int q = row_of_lane().q, kb = (j - 1) * PG_KEYS;
                const uint64_t seen = (uint64_t)pg_seen(a, s_, q, kb + 32) << 32 | pg_seen(a, s_, q, kb);
                pg_second_clean<HD>(of, 0, pf, pl, acc);
                const char* values = smem + (4 + ((j - 1) & 3)) * TILE;
                pg_add_bad<HD>(values, pg_bad_keys<HD, PG_KEYS>(values), seen, acc);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) read_v(i);
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
            }
        }
        if (first) {
            const PkOffsets<HD> of(off, lds_at + (j & 3) * TILE);
            auto read_k = [&](int i) __attribute__((always_inline)) { f[i & 3].v = of.row(i & 1, i >> 1); };
            const pk_floatx16 zero = {};
#pragma unroll
            for (int i = 0; i < 4; ++i) read_k(i);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < 2 * KS; ++i) {
                s[i & 1] = pk_mfma(f[i & 3], qf[i >> 1], i < 2 ? zero : s[i & 1]);
                if (i + 4 < 2 * KS) read_k(i + 4);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
        } else {
            pk_zero(s[0]);
            pk_zero(s[1]);
        }
    };
    auto softmax = [&](int j) __attribute__((always_inline)) {
        const int kb = j * PG_KEYS;
        if (kb > wlast) {
#pragma unroll
            for (int i = 0; i < 4; ++i) pf[i].u = pl[i].u = make_uint4(0, 0, 0, 0);
            return;
        }
        if (kb + PG_KEYS - 1 > wfirst) {                     // (wave-uniform)
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
                for (int e = 0; e < 16; ++e) acc[d][e] = careful ? pg_weighed(alpha, acc[d][e]) : acc[d][e] * alpha;
            top = grown;
            topsc = to;
        }
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][e & 15], sc, -topsc)), p1 = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][(e & 15) + 1], sc, -topsc));
            l += p0 + p1;
            const uint32_t w = pack_bf16x2(p0, p1);
            pf[e >> 3].w[(e & 7) >> 1] = w;
            if (fine) pl[e >> 3].w[(e & 7) >> 1] = pack_bf16x2(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xFFFF0000u));
        }
    };
    // tile j has: up to two behind it, of N loads, may still be on their way
    auto landed = [&](int j) __attribute__((always_inline)) {
        if (j + 2 < j1) __builtin_amdgcn_s_waitcnt(0x0F70 | (2 * N));
        else if (j + 1 < j1) __builtin_amdgcn_s_waitcnt(0x0F70 | N);
        else __builtin_amdgcn_s_waitcnt(0x0F70);
    };
    landed(j0);
    if (late) lds_barrier();
    for (int j = j0; j < j1; ++j) {
        lds_barrier();
        matrix(j);
        __builtin_amdgcn_sched_barrier(0);
        lds_barrier();
        if (j + 3 < j1) {
            request(j + 3, next);
            find(min(j + 4, j1 - 1));
        }
        softmax(j);
        __builtin_amdgcn_sched_barrier(0);
        landed(j + 1);
    }
    lds_barrier();
    matrix(j1);
    if (!late) lds_barrier();
    __shared__ int flags[PG_WIDE];
    if (!careful && pg_any<PG_WIDE>(row_of_lane().mine && pk_not_finite(acc), flags)) return true;
    l = pk_sum_halves(l);
    const Row r = row_of_lane();
    if (u.slot >= 0) {
        if (!r.mine) return false;
        const int64_t to = ((int64_t)u.slot * c.n_kv + kvh) * ROWS + wave * 32 + (lane & 31);
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
template <int HD>
__global__ __launch_bounds__(64 * PG_WIDE) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_wide_kernel(PagedCache c, PagedAttention a, PgOut o) {
    extern __shared__ __align__(1024) char pg_dynamic[];
    const int at = o.by_kv((int)blockIdx.x), kvh = (int)blockIdx.x - at * c.n_kv, G = (int)o.by_group.d;
    __shared__ uint32_t walks[PG_WIDE][sizeof(PgWalk<32 * PG_WIDE>) / 4];
    uint32_t* const saved = walks[threadIdx.x >> 6];
    PgWalk<32 * PG_WIDE> walk;
    if (!walk.begin(c, a, o, at, G)) {
        pg_leave<32 * PG_WIDE>(o, nullptr, nullptr, at, kvh);
        return;
    }
    while (true) {
        const PgUnit u = pg_uniform(walk.unit());
        pg_put(walk, saved);
        // (trees of 48 tokens on 60000 keys with two parts throughout: 88 us and not 75)
        const bool again = pg_two_parts(u.s, G) ? pg_wide<HD, true, false>(c, a, o, u, kvh, (pk_lchar)pg_dynamic) : pg_wide<HD, false, false>(c, a, o, u, kvh, (pk_lchar)pg_dynamic);
        if (again) (void)pg_wide<HD, true, true>(c, a, o, u, kvh, (pk_lchar)pg_dynamic);
        pg_get(walk, saved);
        if (walk.next(c, a, G)) continue;
        pg_leave<32 * PG_WIDE>(o, &walk, &u, at, kvh);
        return;
    }
}

// ---- few rows ----------------------------------------------------------------------------------------------------
// 16 rows and less (a single token's heads of a group, small trees): the time is the keys' reading.  Four waves that each go over tiles of 32 keys of their own, every
// fourth of a workgroup's, without a barrier: a tile waits in registers (HD = 128: 16 KB a wave, 128 KB a compute unit in flight from two workgroups, where 32 KB keep
// memory busy), goes through the wave's own LDS, and the next one is asked for before its products.  The waves' sums are joined at the end.
// 16 rows, in instructions of 16 x 16 x 32: lane n + 16 g has row n's scores of the keys 4 g + i and 16 + 4 g + i, and of its sums the dims 16 db + 4 g + i.
// (32 x 32 x 16 for 16 rows too are 96 registers more, and what is then spilled into the loop makes it wait for the next tile's loads.)  The probabilities go into the second
// product in two bf16 parts (16 bits): a row's sums are of few large probabilities often, whose roundings no others' balance.
// 64 single tokens on 200000 keys, 820 MB: 147 to 151 us, 5.4 to 5.6 TB/s, where a kernel that only reads such pages gets 6.2
constexpr int PG_FEW_KEYS = 32;
typedef float pg_floatx4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ pg_floatx4 pg_mfma16(const PkFrag& a, const PkFrag& b, const pg_floatx4& c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0); }
// over the lanes of a row
__device__ __forceinline__ float pg_max_row(float x) { x = pk_max_halves(x); return fmaxf(x, __shfl_xor(x, 16)); }
__device__ __forceinline__ float pg_sum_row(float x) { x = pk_sum_halves(x); return x + __shfl_xor(x, 16); }

// true: stored nothing, the tiles have to be gone over with care
template <int HD, bool WHOLE, bool careful>
__device__ __forceinline__ bool pg_few(const PagedCache& c, const PagedAttention& a, const PgOut& o, const PgUnit& u, int kvh, pk_lchar lds) {
    constexpr int ROWS = 16, TILE = PG_FEW_KEYS * HD * 2, KS = HD / 32, DB = HD / 16, PITCH = HD + 4;
    static_assert(2 * ROWS * (PITCH + 2) * 4 <= PG_WAVES * 2 * TILE, "two waves' sums in LDS");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, n16 = lane & 15;
    char* smem = (char*)lds + wave * (2 * TILE);
    const int lds_at = (int)(uint32_t)(uintptr_t)lds + wave * (2 * TILE);
    const int G = (int)o.by_group.d;
    const PagedSeq s_ = u.s;
    const int R = s_.nq * G, row0 = u.tile * ROWS, shift = s_.nk - s_.nq;
    struct Row { int q, head; bool mine; };
    auto row_of_lane = [&]() __attribute__((always_inline)) {
        int lane_ = (int)threadIdx.x & 15;
        asm volatile("" : "+v"(lane_));
        const int row = min(row0 + lane_, R - 1), q = o.by_group(row);
        return Row{q, kvh * G + row - q * G, row0 + lane_ < R};
    };
    // the last key that all rows see, and the last that one of them may
    const int all_see = a.tree ? shift - 1 : o.by_group(row0) + shift;
    const int last = a.tree ? s_.nk - 1 : o.by_group(min(row0 + ROWS - 1, R - 1)) + shift;
    const int tiles = last < 0 ? 0 : last / PG_FEW_KEYS + 1;
    const int j0 = pg_cut(tiles, u.from, u.all) + wave, j1 = pg_cut(tiles, u.to, u.all);
    const bf16_t* Kh = c.k + kvh * c.k_head;
    const bf16_t* Vh = c.v + kvh * c.v_head;
    const int32_t* table = c.table + (int64_t)u.seq * c.ld_table;
    typedef PgGroup<HD, WHOLE> Group;
    Group lk[2], lv[2];
    typename Group::Pages next[2];
    auto find = [&](int j) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) next[h] = Group::pages(c, o.by_page, table, j * PG_FEW_KEYS + 16 * h, s_.nk);
    };
    auto request = [&](int j) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) lk[h].load(c, o.by_page, Kh, c.k_page, c.k_row, next[h], j * PG_FEW_KEYS + 16 * h, s_.nk);
#pragma unroll
        for (int h = 0; h < 2; ++h) lv[h].load(c, o.by_page, Vh, c.v_page, c.v_row, next[h], j * PG_FEW_KEYS + 16 * h, s_.nk);
    };
    // byte offsets in a tile of what a lane reads: chunk g of row n16 (chunk 4 ks + g: ^ ks << 6; rows 16 further on: + 16 rows' bytes), and with transposition the
    // four rows 4 g .., dims 0 .. 16 (16 db ..: ^ db << 5)
    const int vrow = 4 * g + (n16 >> 2);
    int at_k = lds_at + n16 * (HD * 2) + ((g ^ pk_swz<HD>(n16)) << 4), at_v = lds_at + TILE + vrow * (HD * 2) + ((((n16 & 3) >> 1) ^ pk_swz<HD>(vrow)) << 4) + (n16 & 1) * 8;
    auto read_k = [&](int h, int ks) __attribute__((always_inline)) {
        typedef const __attribute__((address_space(3))) pk_bf16x8* ptr;
        PkFrag f;
        f.v = *(ptr)(uintptr_t)(uint32_t)((at_k ^ (ks << 6)) + h * 16 * HD * 2);
        return f;
    };
    auto read_v = [&](int db) __attribute__((always_inline)) {
        union { pk_bf16x4 v; uint2 u; } lo, hi;
        lo.v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((pk_trptr)(uintptr_t)(uint32_t)(at_v ^ (db << 5)));
        hi.v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((pk_trptr)(uintptr_t)(uint32_t)((at_v ^ (db << 5)) + 16 * HD * 2));
        PkFrag f;
        f.u = make_uint4(lo.u.x, lo.u.y, hi.u.x, hi.u.y);
        return f;
    };
    PkFrag qf[KS];
    const float sc = a.scale * PK_LOG2E, slack = 8.f / sc;
    pg_floatx4 acc[DB];
    float top, topsc, l;
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = pg_floatx4{0.f, 0.f, 0.f, 0.f};
    top = -INFINITY; topsc = 0.f; l = 0.f;
    if (j0 < j1) {
        find(j0);
        request(j0);
        const Row r = row_of_lane();
        const bf16_t* qsrc = a.q + (int64_t)(s_.q0 + r.q) * a.ldq + (int64_t)r.head * HD + 8 * g;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks].u = *reinterpret_cast<const uint4*>(qsrc + 32 * ks);
        find(min(j0 + PG_WAVES, j1 - 1));
    }
    lds_barrier();                       // (the sums of the piece before)
    for (int j = j0; j < j1; j += PG_WAVES) {
        const int kb = j * PG_FEW_KEYS;
#pragma unroll
        for (int h = 0; h < 2; ++h) lk[h].store(smem, h);
#pragma unroll
        for (int h = 0; h < 2; ++h) lv[h].store(smem + TILE, h);
        if (j + PG_WAVES < j1) {
            request(j + PG_WAVES);
            find(min(j + 2 * PG_WAVES, j1 - 1));
        }
        __builtin_amdgcn_sched_barrier(0);
        // (a wave's own accesses to LDS are in order)
        asm volatile("" : "+v"(at_k), "+v"(at_v));
        pg_floatx4 s[2];
        PkFrag fk[4] = {read_k(0, 0), read_k(1, 0), read_k(0, 1), read_k(1, 1)};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
            const int ks = i >> 1, h = i & 1;
            s[h] = pg_mfma16(fk[i & 3], qf[ks], ks == 0 ? pg_floatx4{0.f, 0.f, 0.f, 0.f} : s[h]);
            if (i + 4 < 2 * KS) fk[i & 3] = read_k(h, ks + 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        PkFrag pf, pl;
        if (kb + PG_FEW_KEYS - 1 > all_see) {                    // (wave-uniform)
            const uint32_t m = pg_seen(a, s_, row_of_lane().q, kb) >> (4 * g);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[h][e] = m & (1u << (16 * h + e)) ? s[h][e] : -INFINITY;
        }
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        mx = pg_max_row(mx);
        // sums are rescaled when a maximum has grown by more than 2^8 times: what they and the probabilities are relative to need not be the maximum itself
        if (__any(mx > top + slack)) {
            const float grown = fmaxf(top, mx), to = grown == -INFINITY ? 0.f : grown * sc;
            const float alpha = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(topsc - to);
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[d][e] = careful ? pg_weighed(alpha, acc[d][e]) : acc[d][e] * alpha;
            top = grown;
            topsc = to;
        }
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][e & 3], sc, -topsc)), p1 = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][(e & 3) + 1], sc, -topsc));
            l += p0 + p1;
            const uint32_t w = pack_bf16x2(p0, p1);
            pf.w[e >> 1] = w;
            pl.w[e >> 1] = pack_bf16x2(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xFFFF0000u));
        }
        // (Read ahead so far: left to itself the compiler reads all first, into registers that are not there.  Two sums at a time: an instruction whose sum the one
        // before makes waits for it)
        auto second = [&](bool clean) __attribute__((always_inline)) {
            PkFrag f[4] = {read_v(0), read_v(1), read_v(2), read_v(3)};
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int db = 0; db < DB; db += 2) {
                PkFrag &f0 = f[db & 3], &f1 = f[(db + 1) & 3];
                if (clean) {
                    pg_clean(f0);
                    pg_clean(f1);
                }
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    acc[db] = pg_mfma16(f0, part ? pl : pf, acc[db]);
                    acc[db + 1] = pg_mfma16(f1, part ? pl : pf, acc[db + 1]);
                }
                if (db + 4 < DB) {
                    f0 = read_v(db + 4);
                    f1 = read_v(db + 5);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        if (!careful) {
            second(false);
        } else {
            second(true);
            const char* tile = smem + TILE;
#pragma unroll 1
            for (uint64_t keys = pg_bad_keys<HD, PG_FEW_KEYS>(tile); keys; keys &= keys - 1) {
                const int r = __builtin_ctzll(keys);
                const bool sees = (pg_seen(a, s_, row_of_lane().q, kb) >> r) & 1;
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const uint2 v = *reinterpret_cast<const uint2*>(tile + r * (HD * 2) + (((2 * db + (g >> 1)) ^ pk_swz<HD>(r)) << 4) + 8 * (g & 1));
                    const uint32_t x[4] = {v.x << 16, v.x & 0xFFFF0000u, v.y << 16, v.y & 0xFFFF0000u};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (sees && (x[i] & 0x7F800000u) == 0x7F800000u) acc[db][i] += __uint_as_float(x[i]);
                }
            }
        }
    }
    float z = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) z = fmaf(acc[d][e], 0.f, z);
    __shared__ int flags[PG_WAVES];
    if (!careful && pg_any<PG_WAVES>(row_of_lane().mine && !(z == 0.f), flags)) return true;
    // The waves' sums, the second two to the first two and the second to the first: what they are relative to, -inf: no part, their exponentials' sum, the sums
    float* const sums = (float*)(char*)lds;
    float* const rel = sums + 2 * ROWS * PITCH;
    l = pg_sum_row(l);
    float base = top == -INFINITY && l == 0.f ? -INFINITY : topsc;
#pragma unroll
    for (int half = 2; half > 0; half >>= 1) {
        lds_barrier();
        if (wave >= half && wave < 2 * half) {
            const int row = (wave - half) * ROWS + n16;
#pragma unroll
            for (int db = 0; db < DB; ++db) *reinterpret_cast<pg_floatx4*>(sums + row * PITCH + 16 * db + 4 * g) = acc[db];
            if (g == 0) {
                rel[row * 2] = base;
                rel[row * 2 + 1] = l;
            }
        }
        lds_barrier();
        if (wave < half) {
            const int row = wave * ROWS + n16;
            const float other = rel[row * 2], other_l = rel[row * 2 + 1], both = fmaxf(base, other);
            const float f = base == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(base - both), g_ = other == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(other - both);
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const pg_floatx4 x = *reinterpret_cast<const pg_floatx4*>(sums + row * PITCH + 16 * db + 4 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[db][i] = careful ? pg_weighed(f, acc[db][i], pg_weighed(g_, x[i])) : fmaf(acc[db][i], f, x[i] * g_);
            }
            l = fmaf(l, f, other_l * g_);
            base = both;
        }
    }
    if (wave != 0) return false;
    const Row r = row_of_lane();
    if (!r.mine) return false;
    if (u.slot >= 0) {
        const int64_t to = ((int64_t)u.slot * c.n_kv + kvh) * ROWS + n16;
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<pg_floatx4*>(o.part + to * HD + 16 * db + 4 * g) = acc[db];
        if (g == 0) o.part_ml[to] = make_float2(base, l);
        return false;
    }
    const bool empty = pg_empty(a, s_, r.q);
    const int64_t tok = s_.q0 + r.q;
    const float f = empty ? 0.f : 1.f / l;
    bf16_t* to = a.out + tok * a.ldo + (int64_t)r.head * HD + 4 * g;
#pragma unroll
    for (int db = 0; db < DB; ++db)
        *reinterpret_cast<uint2*>(to + 16 * db) = make_uint2(pack_bf16x2(acc[db][0] * f, acc[db][1] * f), pack_bf16x2(acc[db][2] * f, acc[db][3] * f));
    if (a.lse && g == 0) a.lse[tok * a.n_heads + r.head] = empty ? -INFINITY : (base + log2f(l)) * PK_LN2;
    return false;
}
template <int HD, bool WHOLE>
__global__ __launch_bounds__(64 * PG_WAVES) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_few_kernel(PagedCache c, PagedAttention a, PgOut o) {
    extern __shared__ __align__(1024) char pg_dynamic[];
    const int at = o.by_kv((int)blockIdx.x), kvh = (int)blockIdx.x - at * c.n_kv, G = (int)o.by_group.d;
    __shared__ uint32_t walks[PG_WAVES][sizeof(PgWalk<16>) / 4];
    uint32_t* const saved = walks[threadIdx.x >> 6];
    PgWalk<16> walk;
    if (!walk.begin(c, a, o, at, G)) {
        pg_leave<16>(o, nullptr, nullptr, at, kvh);
        return;
    }
    while (true) {
        const PgUnit u = pg_uniform(walk.unit());
        pg_put(walk, saved);
        if (pg_few<HD, WHOLE, false>(c, a, o, u, kvh, (pk_lchar)pg_dynamic)) (void)pg_few<HD, WHOLE, true>(c, a, o, u, kvh, (pk_lchar)pg_dynamic);
        pg_get(walk, saved);
        if (walk.next(c, a, G)) continue;
        pg_leave<16>(o, &walk, &u, at, kvh);
        return;
    }
}

// ---- pieces joined -----------------------------------------------------------------------------------------------
// What workgroups have left of row tiles that others go on with: the parts joined by HD / 4 lanes a row, a row to each, and four parts on their way at a time, or eight.  It reads what the first
// launch has just written, fp32 sums: 64 MB where all 512 places have a beginning and an end of 128 rows.  (16 rows of 128 a workgroup, one after the other: trees on 60000 keys
// 93.5 us in both launches and not 91; four parts at a time throughout: 48 heads on two key heads, single tokens on 100000 keys 39.5 and not 38.6; eight: a prompt's piece 285 and not 283)
constexpr int pg_join_rows(int head_dim) { return 1024 / head_dim; }
template <int HD, int ROWS>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedCache c, PagedAttention a, PgOut o) {
    constexpr int LANES = HD / 4;
    const int p0 = o.by_kv((int)blockIdx.x), kvh = (int)blockIdx.x - p0 * c.n_kv, G = (int)o.by_group.d;
    const PgCut cut = o.cuts[p0];
    const int parts = cut.parts, first_slot = cut.slot;
    if (parts < 2) return;
    const PagedSeq s = cut.s;
    const int R = s.nq * G, j = threadIdx.x % LANES;
    const int r = blockIdx.y * pg_join_rows(HD) + threadIdx.x / LANES;
    const int in = cut.tile * ROWS + r;
    if (in >= R) return;
    const int q = o.by_group(in), head = kvh * G + in - q * G;
    auto at = [&](int i) __attribute__((always_inline)) { return ((int64_t)(i == 0 ? first_slot : 2 * (p0 + i)) * c.n_kv + kvh) * ROWS + r; };
    // maxima and sums by part in the lanes of the row; a part that the row sees nothing of has none, its weight is -1 here
    float top = -INFINITY, l;
    for (int s0 = 0; s0 < parts; s0 += LANES) top = fmaxf(top, s0 + j < parts ? o.part_ml[at(s0 + j)].x : -INFINITY);
#pragma unroll
    for (int x = LANES / 2; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    float4 x;
    auto join = [&](auto careful) __attribute__((always_inline)) {
        x = make_float4(0.f, 0.f, 0.f, 0.f);
        l = 0.f;
        for (int s0 = 0; s0 < parts; s0 += LANES) {
            const float2 m = o.part_ml[at(min(s0 + j, parts - 1))];
            const float f = s0 + j >= parts ? -1.f : m.y != m.y ? NAN : m.x != -INFINITY ? __builtin_amdgcn_exp2f(m.x - top) : -1.f;
            l += f <= 0.f ? 0.f : f * m.y;
            const int n = min(LANES, parts - s0);
            auto add = [&](int i, auto count) __attribute__((always_inline)) {
                constexpr int N = decltype(count)::value;
                float4 v[N];
#pragma unroll
                for (int k = 0; k < N; ++k) v[k] = *reinterpret_cast<const float4*>(o.part + at(min(s0 + i + k, parts - 1)) * HD + 4 * j);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float f_ = __shfl(f, i + k, LANES);              // (-1 from the last part on)
                    if (f_ < 0.f) continue;
                    if (decltype(careful)::value) x = make_float4(pg_weighed(f_, v[k].x, x.x), pg_weighed(f_, v[k].y, x.y), pg_weighed(f_, v[k].z, x.z), pg_weighed(f_, v[k].w, x.w));
                    else x = make_float4(fmaf(f_, v[k].x, x.x), fmaf(f_, v[k].y, x.y), fmaf(f_, v[k].z, x.z), fmaf(f_, v[k].w, x.w));
                }
            };
            if (parts <= 4) add(0, std::integral_constant<int, 4>());
            else
                for (int i = 0; i < n; i += 8) add(i, std::integral_constant<int, 8>());
        }
    };
    join(std::false_type());
    // (by the lanes of a row together: they read its maxima and sums from each other)
    if (__builtin_amdgcn_ballot_w64(!(pg_finite(x.x) && pg_finite(x.y) && pg_finite(x.z) && pg_finite(x.w)))) join(std::true_type());
#pragma unroll
    for (int y = LANES / 2; y > 0; y >>= 1) l += __shfl_xor(l, y);
    const bool empty = pg_empty(a, s, q);
    const float inv = empty ? 0.f : 1.f / l;
    const int64_t tok = s.q0 + q;
    *reinterpret_cast<uint2*>(a.out + tok * a.ldo + (int64_t)head * HD + 4 * j) = make_uint2(pack_bf16x2(x.x * inv, x.y * inv), pack_bf16x2(x.z * inv, x.w * inv));
    if (a.lse && j == 0) a.lse[tok * a.n_heads + head] = empty ? -INFINITY : (top + log2f(l)) * PK_LN2;
}

// ---- launches ----------------------------------------------------------------------------------------------------
// two workgroups to each of 256 compute units, or one of twice the waves
constexpr int PG_PLACES = 512, PG_LEAST = 256, PG_LONG = 2048;      // PG_LONG: room of a sequence from which on 256 rows are taken together

struct PgLaunch { int rows; int64_t units, slots; int places, cost; };
PgLaunch pg_launch_of(const PagedCache& c, const PagedAttention& a) {
    PgLaunch p{};
    const int64_t G = a.n_heads / c.n_kv;
    // By the rows of a sequence in the mean.  (The kernel of few rows with two blocks of 16, for up to 32: single tokens with 32 heads on one key head, 200000 keys, 56 us and 44 with
    // the other, trees of 6 tokens with 4 heads on a key head 192 and 176; with 16 rows in the mean 90 in the one of few and 98 in the other, with 4 rows 156 and 170)
    const int64_t mean = (a.total_q * G + c.n_seq - 1) / std::max(1, c.n_seq);
    p.rows = mean <= 16 ? 16 : mean <= 128 || c.page_size % 16 || (int64_t)c.max_pages * c.page_size < PG_LONG ? 128 : 256;
    const int64_t tiles = a.total_q * G / p.rows + std::min<int64_t>(c.n_seq, a.total_q);
    // What sharing out costs is a second piece's start, storing sums and the launch that joins them: 8 to 10 us in all.  (384 and 256 keys: 15 prompts' pieces on 3100 keys 38 us for
    // 19, trees of 44 tokens on 1400 keys 18.7 for 14.9, the first tokens of four conversations 11.5 for 10.0; 1536 and 1024: two prompts' on 1700 keys 31 for 23.)  No sequence has
    // more keys than its room: with less than that nothing is shared out
    p.cost = p.rows >= 128 ? 1024 : 768;
    p.places = (int64_t)c.max_pages * c.page_size <= p.cost ? 1 : std::max(1, (PG_PLACES / (p.rows > 128 ? 2 : 1) + c.n_kv - 1) / c.n_kv);
    p.slots = p.places < 2 ? 0 : 2LL * p.places * c.n_kv;
    p.units = std::max<int64_t>(tiles, p.places) * c.n_kv;
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

template <int HD, bool WHOLE>
hipError_t pg_launch(const PagedCache& c, const PagedAttention& a, const PgOut& o, int64_t units, hipStream_t st) {
    constexpr int SMEM = 4 * PG_KEYS * HD * 2;
    static std::atomic<uint64_t> done{0};
    const hipError_t e = pg_lds(paged_kernel<HD, WHOLE>, SMEM, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((paged_kernel<HD, WHOLE>), dim3((unsigned)units), dim3(64 * PG_WAVES), SMEM, st, c, a, o);
    return hipGetLastError();
}
template <int HD>
hipError_t pg_launch_wide(const PagedCache& c, const PagedAttention& a, const PgOut& o, int64_t units, hipStream_t st) {
    constexpr int SMEM = 8 * PG_KEYS * HD * 2;
    static std::atomic<uint64_t> done{0};
    const hipError_t e = pg_lds(paged_wide_kernel<HD>, SMEM, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_wide_kernel<HD>, dim3((unsigned)units), dim3(64 * PG_WIDE), SMEM, st, c, a, o);
    return hipGetLastError();
}
template <int HD, bool WHOLE>
hipError_t pg_launch_few(const PagedCache& c, const PagedAttention& a, const PgOut& o, int64_t units, hipStream_t st) {
    constexpr int SMEM = PG_WAVES * 2 * PG_FEW_KEYS * HD * 2;
    static std::atomic<uint64_t> done{0};
    const hipError_t e = pg_lds((paged_few_kernel<HD, WHOLE>), SMEM, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((paged_few_kernel<HD, WHOLE>), dim3((unsigned)units), dim3(64 * PG_WAVES), SMEM, st, c, a, o);
    return hipGetLastError();
}

template <int HD>
hipError_t pg_launch_forward(const PagedCache& c, const PagedAttention& a, void* workspace, hipStream_t st) {
    const PgLaunch p = pg_launch_of(c, a);
    const int64_t G = a.n_heads / c.n_kv;
    float* part = static_cast<float*>(workspace);
    float2* part_ml = reinterpret_cast<float2*>(part + p.slots * p.rows * HD);
    const PgOut o{part, part_ml, reinterpret_cast<PgCut*>(part_ml + p.slots * p.rows), p.places, PG_LEAST, p.cost, QuickDiv(c.n_kv), QuickDiv((int)G), QuickDiv(c.page_size)};
    if (paged_units(c, a) >= kPackedUnits) return hipErrorInvalidValue;
    const bool whole = c.page_size % 16 == 0;
    const hipError_t e = p.rows == 16 ? (whole ? pg_launch_few<HD, true>(c, a, o, p.units, st) : pg_launch_few<HD, false>(c, a, o, p.units, st))
                                      : p.rows == 256 ? pg_launch_wide<HD>(c, a, o, p.units, st)
                                      : whole ? pg_launch<HD, true>(c, a, o, p.units, st) : pg_launch<HD, false>(c, a, o, p.units, st);
    if (e != hipSuccess || p.places < 2) return e;
    const dim3 borders((unsigned)((p.places - 1) * c.n_kv), p.rows / pg_join_rows(HD));
    if (p.rows == 16) hipLaunchKernelGGL((paged_join_kernel<HD, 16>), borders, dim3(256), 0, st, c, a, o);
    else if (p.rows == 256) hipLaunchKernelGGL((paged_join_kernel<HD, 256>), borders, dim3(256), 0, st, c, a, o);
    else hipLaunchKernelGGL((paged_join_kernel<HD, 128>), borders, dim3(256), 0, st, c, a, o);
    return hipGetLastError();
}

}  // namespace

int64_t paged_units(const PagedCache& c, const PagedAttention& a) {
    const PgLaunch p = pg_launch_of(c, a);
    return p.rows > 128 ? 2 * p.units : p.units;      // (of 256 threads)
}
size_t paged_workspace_bytes(const PagedCache& c, const PagedAttention& a, int head_dim) {
    const PgLaunch p = pg_launch_of(c, a);
    return p.slots == 0 ? 0 : (size_t)p.slots * p.rows * (head_dim * sizeof(float) + sizeof(float2)) + p.places * sizeof(PgCut);
}

hipError_t launch_paged_attention(const PagedCache& c, const PagedAttention& a, int head_dim, void* workspace, hipStream_t st) {
    if (a.total_q == 0 || c.n_seq == 0) return hipSuccess;
    return head_dim == 128 ? pg_launch_forward<128>(c, a, workspace, st) : pg_launch_forward<64>(c, a, workspace, st);
}

}  // namespace agzo
