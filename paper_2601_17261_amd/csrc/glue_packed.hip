// Attention over packed sequences of different lengths, with grouped heads: a sequence's queries are its last positions, its keys all of them,
//     o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i k_j - lse_i),  lse_i = log sum_j exp(scale q_i k_j),  j <= i + (keys - queries) if causal,
// and back, with delta_i = do_i o_i:
//     dv_j = sum_i p_ij do_i,  ds_ij = p_ij (do_i v_j - delta_i),  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,
// the sums over i going through all heads of j's group too.
//
// Rows.  The heads of a group see the same keys, so a row is a (query, head) pair, row r of a sequence and key head being head r mod G of query
// r / G (G heads to a group).  A tile of rows is full whether it holds many queries or a single one with its group's heads, and no
// sum of the gradients crosses workgroups.
//
// All products are v_mfma_f32_32x32x16_bf16 over tiles of 32 and are made transposed: a lane holds, for ONE row (forward, dq) or ONE key (dk, dv),
// column lane % 32 of the instruction, the scores of positions 8 (e / 4) + 4 (lane / 32) + e % 4 of the other side.  So what belongs to a row is
// a lane's scalar, and the eight values of each 16 positions that a lane holds go into the second product as they are, whose other
// operand is read from LDS with a transposition in the same order of positions.
//
// What a masked place holds takes part in nothing: scores there are replaced, not added to.  Only the second products multiply a
// masked place's values, by 0, of which a value that is not finite makes a NaN.  Where a workgroup's results are not finite it goes over
// its tiles once more with care: masked tiles then have such values taken out, and what the visible ones amount to is found by a product of two
// indicators.
#include <atomic>
#include <type_traits>

#include "packed_tiles.h"

namespace agzo {

namespace {

// One sequence's places in the packed tensors, and a tile of it
struct PkTile { int tile, share, q0, k0, nq, nk; };

// Tile number t of all sequences' tiles, UNIT rows (BY_KEYS: keys) each; with chunk > 0 a row tile is one for every `chunk` tiles of 64 keys that its sequence has.
// The tiles that see most (BY_KEYS: that are seen most) of up to 64 sequences come first: a sequence's last row tile (its first tile of keys) is as many
// levels high as it has tiles, the next one a level less, and tiles are numbered level by level.  (Sequence by sequence a long one may start
// last: a training pass of 8192 tokens in eight of up to 1923 took 444 us, so 338.  From 65 sequences on, and with chunk > 0, it is sequence by sequence all the
// same.)  Offsets are taken as far as they lie inside the tensors and grow
template <int UNIT, bool BY_KEYS>
__device__ __forceinline__ bool pk_find(const PackedArgs& a, int t, int G, int chunk, PkTile& out) {
    const int lane = threadIdx.x & 63, total_q = (int)a.total_q, total_k = (int)a.total_k;
    for (int b = 0; b < a.n_seq; b += 64) {
        const int s = min(b + lane, a.n_seq - 1);
        int q0 = a.cu_q[s], q1 = a.cu_q[s + 1], k0 = a.cu_k[s], k1 = a.cu_k[s + 1];
        q0 = min(max(q0, 0), total_q);   q1 = min(max(q1, q0), total_q);
        k0 = min(max(k0, 0), total_k);   k1 = min(max(k1, k0), total_k);
        if (!BY_KEYS && a.k_len) k1 = k0 + min(max(a.k_len[s], 0), k1 - k0);
        const int own = b + lane >= a.n_seq ? 0 : (int)(((BY_KEYS ? (uint32_t)(k1 - k0) : (uint32_t)(q1 - q0) * (uint32_t)G) + (UNIT - 1)) / UNIT);
        // (a row tile without keys is one all the same: its rows are written)
        const int count = chunk > 0 ? own * max(1, ((k1 - k0 + PK_T - 1) / PK_T + chunk - 1) / chunk) : own;
        const int sum = pk_scan(count);
        const int total = __builtin_amdgcn_readlane(sum, 63);
        if (t < total) {
            int src, tile;
            if (chunk == 0 && a.n_seq <= 64) {
                // the lowest level with at most t tiles above it
                int low = 0, high = total;
                while (low < high) {
                    const int mid = (low + high) >> 1;
                    if (pk_total(max(own - mid, 0)) <= t) high = mid;
                    else low = mid + 1;
                }
                const int place = t - pk_total(max(own - low, 0));
                const uint64_t m = __builtin_amdgcn_ballot_w64(own >= low);
                const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
                src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(own >= low && before == place));
                tile = BY_KEYS ? __builtin_amdgcn_readlane(own, src) - low : low - 1;
            } else {
                src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(sum > t));
                tile = t - __builtin_amdgcn_readlane(sum - count, src);
                if (!BY_KEYS && chunk == 0) tile = __builtin_amdgcn_readlane(own, src) - 1 - tile;
            }
            const int rows = __builtin_amdgcn_readlane(own, src);
            out.share = chunk > 0 ? tile / rows : 0;
            out.tile = tile - out.share * rows;
            out.q0 = __builtin_amdgcn_readlane(q0, src);
            out.k0 = __builtin_amdgcn_readlane(k0, src);
            out.nq = __builtin_amdgcn_readlane(q1, src) - out.q0;
            out.nk = __builtin_amdgcn_readlane(k1, src) - out.k0;
            return true;
        }
        t -= total;
    }
    return false;
}

// 64 rows on their way to a tile in LDS, by the four waves of a workgroup: the rows from `base` on, `ld` values apart; rows past `left` repeat the
// last one.  (Through registers: behind direct loads to LDS the compiler lets every read with transposition wait for all that are in flight)
// (A wave's loads are 1024 bytes each, whose rows differ in the low bits of r / 4 alone, and with them the places of chunks)
template <int HD>
struct PkLoader {
    static constexpr int N = PK_T * HD * 2 / 4096, ROWS = 1024 / (HD * 2);      // loads of a wave, rows of a load
    static_assert(ROWS * N == 16 && (HD == 128 || HD == 64), "swz() of the rows of load i");
    uint4 data[N];
    __device__ __forceinline__ void load(const bf16_t* base, int64_t ld, int left) {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(base), 0, (int)0xFFFFFFFFu, 0x00020000);
        // (one way for tiles inside a sequence and at its end: loads on two ways are moved where these meet, and waited for.  Rows are below 2^6, their bytes 2^23)
        int lane_ = (int)threadIdx.x;
        asm volatile("" : "+v"(lane_));
        const int lane = lane_ & 63, r = 16 * (lane_ >> 6) + lane / (HD / 8), chunk = ((lane % (HD / 8)) ^ pk_swz<HD>(r)) << 4;
#pragma unroll
        for (int i = 0; i < N; ++i)
            data[i] = pk_load16(rsrc, (int)(__umul24((uint32_t)min(r + ROWS * i, left - 1), (uint32_t)(2 * ld)) + (uint32_t)(chunk ^ (pk_swz<HD>(ROWS * i) << 4))), 0);
    }
    __device__ __forceinline__ void store(char* tile) const {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<uint4*>(tile + (wave * N + i) * 1024 + lane * 16) = data[i];
    }
};

// ones where positions kb + .. <= limit, as the fragments of 64 positions
__device__ __forceinline__ void pk_seen(int kb, int limit, PkFrag (&f)[4]) {
    const int rel = limit - kb - 4 * (int)((threadIdx.x >> 5) & 1);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int at = 16 * s + (w >> 1) * 8 + (w & 1) * 2;
            f[s].w[w] = (at <= rel ? 0x3F80u : 0u) | (at + 1 <= rel ? 0x3F800000u : 0u);
        }
}

constexpr int PK_WAVES = 4, PK_ROWS = 32 * PK_WAVES;

// ---- forward ---------------------------------------------------------------------------------------------------
// Four waves of 32 rows against tiles of 64 keys that they share, two tiles of K and V in LDS, two workgroups to a compute unit, which fill each other's
// waits.  A tile is 32 matrix instructions a wave (HD = 128, 1024 cycles) beside some 1200 cycles of other vector instructions and 32 KB of LDS reads.
// chunk > 0: a row tile's keys are dealt out, `chunk` tiles of them a share to a workgroup, which leaves its sums, maximum and sum of exponentials for pk_join_kernel
// fine: the probabilities go into the second product in two bf16 parts.  For few rows beside the keys, whose time is the keys' reading: their sums are of few large
// probabilities often, whose roundings no others' balance (single rows were off by 0.0021 to 0.0028 of their norm, and are by the 0.0017 of
// the result's own rounding; 64 on 200000 keys: 175 us for 171)
struct PkForwardOut { bf16_t* out; int64_t ldo; float* lse; float* part; float2* part_ml; int chunk; };
// true: stored nothing, the tiles have to be gone over with care
template <int HD, bool fine, bool careful>
__device__ __forceinline__ bool pk_forward(const PackedArgs& a, const PkForwardOut& to_, pk_lchar lds) {
    char* pk_smem = (char*)lds;
    const int lds_at = (int)(uint32_t)(uintptr_t)lds;
    constexpr int TILE = PK_T * HD * 2, KS = HD / 16, DB = HD / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hi = lane >> 5;
    // the key heads side by side: an XCD (workgroup number mod 8) then has few of them
    const int G = PkDiv(a.n_kv)(a.n_heads), unit = (int)blockIdx.x, at = PkDiv(a.n_kv)(unit), kvh = unit - at * a.n_kv;
    PkTile t;
    if (!pk_find<PK_ROWS, false>(a, at, G, to_.chunk, t)) return false;
    const PkDiv by_group(G);
    const int R = t.nq * G, row0 = t.tile * PK_ROWS + wave * 32, shift = t.nk - t.nq;
    // The lane's row: its query, its head, the last key that it sees.  (Worked out where they are needed, from a lane number that the compiler does not know
    // again: kept through the loop they are spilled, and a wait for a reload is one for the next tile's loads too)
    struct Row { int64_t tok; int head, limit; bool mine; };
    auto row_of_lane = [&]() __attribute__((always_inline)) {
        int lane_ = (int)threadIdx.x & 31;
        asm volatile("" : "+v"(lane_));
        const int row = min(row0 + lane_, R - 1), q = by_group(row);
        return Row{t.q0 + q, kvh * G + row - q * G, a.causal ? q + shift : t.nk - 1, row0 + lane_ < R};
    };
    auto limit_of = [&]() __attribute__((always_inline)) { return row_of_lane().limit; };
    // the first and last of the wave's rows, and the last of the workgroup's
    const int wfirst = a.causal ? by_group(min(row0, R - 1)) + shift : t.nk - 1;
    const int wlast = row0 >= R ? -1 : a.causal ? by_group(min(row0 + 31, R - 1)) + shift : t.nk - 1;
    const int last = a.causal ? by_group(min((t.tile + 1) * PK_ROWS - 1, R - 1)) + shift : t.nk - 1;
    const int tiles = last < 0 ? 0 : last / PK_T + 1;
    const int j0 = to_.chunk > 0 ? t.share * to_.chunk : 0, j1 = to_.chunk > 0 ? min(tiles, j0 + to_.chunk) : tiles;
    // (a share that none of the row tile sees.  The first one is there for rows that see nothing at all)
    if (j0 >= j1 && t.share > 0) return false;
    const bf16_t* Kh = a.k + (int64_t)t.k0 * a.ldk + kvh * HD;
    const bf16_t* Vh = a.v + (int64_t)t.k0 * a.ldv + kvh * HD;
    PkLoader<HD> lk, lv;
    auto request = [&](int j) __attribute__((always_inline)) {
        lk.load(Kh + (int64_t)j * PK_T * a.ldk, a.ldk, t.nk - j * PK_T);
        lv.load(Vh + (int64_t)j * PK_T * a.ldv, a.ldv, t.nk - j * PK_T);
    };
    auto arrive = [&](int j) __attribute__((always_inline)) {
        lk.store(pk_smem + (j & 1) * (2 * TILE));
        lv.store(pk_smem + (j & 1) * (2 * TILE) + TILE);
    };
    const PkOffsets<HD> off;
    PkFrag qf[KS];
    // the first tile and the queries (once more for a pass with care: kept for it they would be spilled, and a wait for a reload in the loop is one for the next
    // tile's loads too).  Waited for here: what is left to the loop to wait for, it waits for in every round, and with it for the next tile's loads
    auto begin = [&]() __attribute__((always_inline)) {
        if (j0 >= j1) return;
        request(j0);
        const Row r = row_of_lane();
        const bf16_t* qsrc = a.q + r.tok * a.ldq + (int64_t)r.head * HD + 8 * hi;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks].u = *reinterpret_cast<const uint4*>(qsrc + 16 * ks);
        __builtin_amdgcn_s_waitcnt(0x0F70);
    };
    const float sc = a.scale * PK_LOG2E;
    // sums are rescaled when a maximum has grown by more than 2^8 times: what they and the probabilities are relative to need not be the maximum itself
    const float slack = 8.f / sc;
    pk_floatx16 acc[DB];
    float top, topsc, l;
    auto one_tile = [&](int j) __attribute__((always_inline)) {
            const int kb = j * PK_T;
            if (kb > wlast) return;                                          // (wave-uniform)
            const char* kt = pk_smem + (j & 1) * (2 * TILE);
            // (operands are read four instructions ahead: left to itself the compiler reads right before each instruction)
            const PkOffsets<HD> o(off, lds_at + (j & 1) * (2 * TILE));
            PkFrag f[4];
            auto read_k = [&](int i) __attribute__((always_inline)) { f[i & 3].v = o.row(i & 1, i >> 1); };
            auto read_v = [&](int i) __attribute__((always_inline)) { pk_read_trans<HD>(o, TILE + (i / DB) * 16 * HD * 2, i % DB, f[i & 3]); };
            const pk_floatx16 zero = {};
            pk_floatx16 s[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) read_k(i);
            __builtin_amdgcn_sched_barrier(0);
            // (of a SIMD's two waves the one that has matrix instructions to issue goes first, beside the other's maxima and exponentials.  16001 tokens: 1022 us, 1079
            // without; 1038 with the exponentials among the second product's instructions)
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < 2 * KS; ++i) {
                s[i & 1] = pk_mfma(f[i & 3], qf[i >> 1], i < 2 ? zero : s[i & 1]);
                if (i + 4 < 2 * KS) read_k(i + 4);
                else read_v(i + 4 - 2 * KS);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
            const bool mask = kb + PK_T - 1 > wfirst;                        // (wave-uniform)
            if (mask) {
                const int rel = limit_of() - kb - 4 * hi;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[h][e] = 32 * h + pk_pos(e) <= rel ? s[h][e] : -INFINITY;
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
            auto two = [&](int e) __attribute__((always_inline)) {              // probabilities e and e + 1 of the lane's 32
                const float p0 = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][e & 15], sc, -topsc)), p1 = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][(e & 15) + 1], sc, -topsc));
                l += p0 + p1;
                const uint32_t w = pack_bf16x2(p0, p1);
                pf[e >> 3].w[(e & 7) >> 1] = w;
                if (fine) pl[e >> 3].w[(e & 7) >> 1] = pack_bf16x2(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xFFFF0000u));
            };
            if (careful && mask) {
#pragma unroll
                for (int e = 0; e < 32; e += 2) two(e);
                PkFrag seen[4];
                pk_seen(kb, limit_of(), seen);
                pk_second_careful<HD, true, fine>(kt + TILE, pf, pl, seen, acc);
                return;
            }
            // (heads of 64, whose tiles are half the matrix instructions beside as many exponentials: those of 16 keys beside the second product of the 16 before
            // them; 8192 tokens forward and back 213 us, 222 like heads of 128)
            constexpr bool beside = HD == 64;
#pragma unroll
            for (int e = 0; e < (beside ? 8 : 32); e += 2) two(e);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < 4 * DB; ++i) {
                acc[i % DB] = pk_mfma(f[i & 3], pf[i / DB], acc[i % DB]);
                if (fine) acc[i % DB] = pk_mfma(f[i & 3], pl[i / DB], acc[i % DB]);
                if (i + 4 < 4 * DB) read_v(i + 4);
                if (beside && i < 3 * DB) {
#pragma unroll
                    for (int e = 0; e < 8 / DB; e += 2) two(8 + i * (8 / DB) + e);
                }
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
        if (j + 1 < j1) request(j + 1);
        one_tile(j);
        if (j + 1 < j1) arrive(j + 1);
    }
    if (!careful && __syncthreads_or(row_of_lane().mine && pk_not_finite(acc))) return true;
    l = pk_sum_halves(l);
    const Row r = row_of_lane();
    if (to_.part) {
        if (!r.mine) return false;
        const int64_t at = (int64_t)t.share * a.total_q * a.n_heads + r.tok * a.n_heads + r.head;
        float* to = to_.part + at * HD + 4 * hi;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4*>(to + 32 * db + 8 * g) = make_float4(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]);
        if (hi == 0) to_.part_ml[at] = make_float2(top == -INFINITY && l == 0.f ? -INFINITY : topsc, l);
        return false;
    }
    const bool empty = r.limit < 0;
    pk_store<HD>(acc, empty ? 0.f : 1.f / l, to_.out + r.tok * to_.ldo + (int64_t)r.head * HD, r.mine);
    if (to_.lse && r.mine && hi == 0) to_.lse[r.tok * a.n_heads + r.head] = empty ? -INFINITY : (topsc + log2f(l)) * PK_LN2;
    return false;
}
// (a function that is called: its registers are not the kernel's)
template <int HD, bool fine>
__device__ __noinline__ void pk_forward_again(PackedArgs a, PkForwardOut to, pk_lchar lds) { (void)pk_forward<HD, fine, true>(a, to, lds); }
template <int HD, bool fine>
__global__ __launch_bounds__(64 * PK_WAVES) __attribute__((amdgpu_waves_per_eu(2, 2))) void pk_forward_kernel(PackedArgs a, PkForwardOut to) {
    extern __shared__ __align__(1024) char pk_dynamic[];
    if (pk_forward<HD, fine, false>(a, to, (pk_lchar)pk_dynamic)) pk_forward_again<HD, fine>(a, to, (pk_lchar)pk_dynamic);
}

// Shares of the keys joined: HD / 4 lanes a row.  Rows of no sequence are left alone: their partial sums are what the workspace held
template <int HD>
__global__ __launch_bounds__(256) void pk_join_kernel(PackedArgs a, const float* __restrict__ part, const float2* __restrict__ ml, int chunk,
                                                      bf16_t* __restrict__ out, int64_t ldo, float* __restrict__ lse) {
    constexpr int LANES = HD / 4;
    const int64_t rows = a.total_q * a.n_heads, at_row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES, row = min(at_row, rows - 1);
    const bool there = at_row < rows;
    const int j = threadIdx.x % LANES;
    const int64_t tok = row / a.n_heads;
    // which sequence the token is of: the last one that starts at or before it.  (By all lanes for both of the wave's rows at most: halves one after the
    // other were six loads that wait for each other)
    int lo = -1;
    const int tok0 = __builtin_amdgcn_readfirstlane((int)tok), tok1 = __builtin_amdgcn_readlane((int)tok, 63);
    for (int b = 0; b < a.n_seq; b += 64) {
        const int s = b + (int)(threadIdx.x & 63), start = s < a.n_seq ? a.cu_q[s] : 0x7FFFFFFF;
        if (LANES == 16) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(start <= __builtin_amdgcn_readlane((int)tok, 16 * g)));
                lo += (int)((threadIdx.x & 63) >> 4) == g ? n : 0;
            }
        } else {
            const int n0 = __builtin_popcountll(__builtin_amdgcn_ballot_w64(start <= tok0)), n1 = __builtin_popcountll(__builtin_amdgcn_ballot_w64(start <= tok1));
            lo += (threadIdx.x & 63) < 32 ? n0 : n1;
        }
    }
    if (!there || lo < 0) return;
    const int q0 = min(max(a.cu_q[lo], 0), (int)a.total_q), q1 = min(max(a.cu_q[lo + 1], q0), (int)a.total_q);
    if (tok < q0 || tok >= q1) return;
    const int k0 = min(max(a.cu_k[lo], 0), (int)a.total_k), room = min(max(a.cu_k[lo + 1], k0), (int)a.total_k) - k0;
    const int nk = a.k_len ? min(max(a.k_len[lo], 0), room) : room;
    const int G = a.n_heads / a.n_kv, nq = q1 - q0, at = (int)(tok - q0), head = (int)(row - tok * a.n_heads);
    const bool empty = (a.causal ? at + nk - nq : nk - 1) < 0;
    // the shares of its row tile
    const int in = at * G + head % G, end = min((in / PK_ROWS + 1) * PK_ROWS, nq * G) - 1, last = a.causal ? end / G + nk - nq : nk - 1;
    const int shares = last < 0 ? 1 : (last / PK_T + chunk) / chunk;
    // maxima and sums by share in the lanes of the row; a share that the row sees nothing of has no part
    float top = -INFINITY, l = 0.f;
    for (int s0 = 0; s0 < shares; s0 += LANES) top = fmaxf(top, s0 + j < shares ? ml[(s0 + j) * rows + row].x : -INFINITY);
#pragma unroll
    for (int w = LANES / 2; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < shares; s0 += LANES) {
        const float2 m = ml[min(s0 + j, shares - 1) * rows + row];
        const float f = s0 + j >= shares ? 0.f : m.y != m.y ? NAN : m.x != -INFINITY ? __builtin_amdgcn_exp2f(m.x - top) : 0.f;
        l += f == 0.f ? 0.f : f * m.y;
        const int n = min(LANES, shares - s0);
        for (int s = 0; s < n; s += 4) {
            float4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const float4*>(part + (min(s0 + s + u, shares - 1) * rows + row) * HD + 4 * j);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float w = __shfl(f, s + u, LANES);              // (0 from the last share on)
                if (w != 0.f) { o.x = fmaf(w, v[u].x, o.x); o.y = fmaf(w, v[u].y, o.y); o.z = fmaf(w, v[u].z, o.z); o.w = fmaf(w, v[u].w, o.w); }
            }
        }
    }
#pragma unroll
    for (int w = LANES / 2; w > 0; w >>= 1) l += __shfl_xor(l, w);
    const float inv = empty ? 0.f : 1.f / l;
    *reinterpret_cast<uint2*>(out + tok * ldo + (int64_t)head * HD + 4 * j) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
    if (lse && j == 0) lse[row] = empty ? -INFINITY : (top + log2f(l)) * PK_LN2;
}

// ---- backward --------------------------------------------------------------------------------------------------
// Per row -lse / scale and -delta, delta = do . o, each as three bf16 (24 bits): what the scores and do v^T are to be corrected by, as further values
// of the rows of q and do that are multiplied by ones.  (0 for rows that see nothing.)  The kernel of dq makes them for both
__device__ __forceinline__ uint2 pk_split3(float f) {
    bf16_t h, m, l;
    split3_bf16(f, h, m, l);
    return make_uint2((uint32_t)h | (uint32_t)m << 16, l);
}
__device__ __forceinline__ float pk_join3(uint32_t a, uint32_t b) {
    return (__uint_as_float(a << 16) + __uint_as_float(a & 0xFFFF0000u)) + __uint_as_float(b << 16);
}
struct PkBackward { const bf16_t *out, *dout; int64_t ldo, lddo; const float* lse; uint4* rowinfo; bf16_t* dq; int64_t lddq; bf16_t* dk; int64_t lddk; bf16_t* dv; int64_t lddv; float* part; };

// dq: the forward's shape, with do beside q in registers, and K read with and without transposition
template <int HD, bool careful>
__device__ __forceinline__ bool pk_dq(const PackedArgs& a, const PkBackward& g, pk_lchar lds) {
    char* pk_smem = (char*)lds;
    const int lds_at = (int)(uint32_t)(uintptr_t)lds;
    constexpr int TILE = PK_T * HD * 2, KS = HD / 16, DB = HD / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hi = lane >> 5;
    const int G = PkDiv(a.n_kv)(a.n_heads), unit = (int)blockIdx.x, at = PkDiv(a.n_kv)(unit), kvh = unit - at * a.n_kv;
    PkTile t;
    if (!pk_find<PK_ROWS, false>(a, at, G, 0, t)) return false;
    const PkDiv by_group(G);
    const int R = t.nq * G, row0 = t.tile * PK_ROWS + wave * 32, shift = t.nk - t.nq;
    // The lane's row: its query, its head, the last key that it sees.  (Worked out where they are needed, from a lane number that the compiler does not know
    // again: kept through the loop they are spilled, and a wait for a reload is one for the next tile's loads too)
    struct Row { int64_t tok; int head, limit; bool mine; };
    auto row_of_lane = [&]() __attribute__((always_inline)) {
        int lane_ = (int)threadIdx.x & 31;
        asm volatile("" : "+v"(lane_));
        const int row = min(row0 + lane_, R - 1), q = by_group(row);
        return Row{t.q0 + q, kvh * G + row - q * G, a.causal ? q + shift : t.nk - 1, row0 + lane_ < R};
    };
    auto limit_of = [&]() __attribute__((always_inline)) { return row_of_lane().limit; };
    // the first and last of the wave's rows, and the last of the workgroup's
    const int wfirst = a.causal ? by_group(min(row0, R - 1)) + shift : t.nk - 1;
    const int wlast = row0 >= R ? -1 : a.causal ? by_group(min(row0 + 31, R - 1)) + shift : t.nk - 1;
    const int last = a.causal ? by_group(min((t.tile + 1) * PK_ROWS - 1, R - 1)) + shift : t.nk - 1;
    const int tiles = last < 0 ? 0 : last / PK_T + 1;
    const bf16_t* Kh = a.k + (int64_t)t.k0 * a.ldk + kvh * HD;
    const bf16_t* Vh = a.v + (int64_t)t.k0 * a.ldv + kvh * HD;
    PkLoader<HD> lk, lv;
    auto request = [&](int j) __attribute__((always_inline)) {
        lk.load(Kh + (int64_t)j * PK_T * a.ldk, a.ldk, t.nk - j * PK_T);
        lv.load(Vh + (int64_t)j * PK_T * a.ldv, a.ldv, t.nk - j * PK_T);
    };
    auto arrive = [&](int j) __attribute__((always_inline)) {
        lk.store(pk_smem + (j & 1) * (2 * TILE));
        lv.store(pk_smem + (j & 1) * (2 * TILE) + TILE);
    };
    const PkOffsets<HD> off;
    PkFrag qf[KS], df[KS];
    const float sc = a.scale * PK_LOG2E;
    float2 info;                                                              // lse log2 e, delta
    // (as in the forward.  Heads of 128 are out of registers all the same: an LDS offset is reloaded in every tile behind the request of the next one, whose loads
    // the wait for it is for too)
    auto begin = [&]() __attribute__((always_inline)) {
        if (tiles > 0) request(0);
        const Row r = row_of_lane();
        const bf16_t* qsrc = a.q + r.tok * a.ldq + (int64_t)r.head * HD + 8 * hi;
        const bf16_t* dsrc = g.dout + r.tok * g.lddo + (int64_t)r.head * HD + 8 * hi;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[ks].u = *reinterpret_cast<const uint4*>(qsrc + 16 * ks);
            df[ks].u = *reinterpret_cast<const uint4*>(dsrc + 16 * ks);
        }
        uint4 parts, *const to = g.rowinfo + r.tok * a.n_heads + r.head;
        if constexpr (careful) {
            parts = *to;
        } else {
            const bf16_t* osrc = g.out + r.tok * g.ldo + (int64_t)r.head * HD + 8 * hi;
            const float lse = g.lse[r.tok * a.n_heads + r.head];
            PkFrag of[KS];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) of[ks].u = *reinterpret_cast<const uint4*>(osrc + 16 * ks);
            float s = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    s = fmaf(__uint_as_float(of[ks].w[w] << 16), __uint_as_float(df[ks].w[w] << 16), s);
                    s = fmaf(__uint_as_float(of[ks].w[w] & 0xFFFF0000u), __uint_as_float(df[ks].w[w] & 0xFFFF0000u), s);
                }
            const uint2 l = pk_split3(lse == -INFINITY ? 0.f : -lse / a.scale), d = pk_split3(-pk_sum_halves(s));
            parts = make_uint4(l.x, l.y, d.x, d.y);
            if (r.mine && hi == 0) *to = parts;
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);
        info = make_float2(-sc * pk_join3(parts.x, parts.y), -pk_join3(parts.z, parts.w));
    };
    pk_floatx16 acc[DB];
    auto one_tile = [&](int j) __attribute__((always_inline)) {
            const int kb = j * PK_T;
            if (kb > wlast) return;
            const char* kt = pk_smem + (j & 1) * (2 * TILE);
            const bool mask = kb + PK_T - 1 > wfirst;
            // (operands two pairs of instructions ahead; see the forward)
            // dS in two bf16 parts (16 bits): the keys of a head share directions, dS of a row sums to 0, so that its roundings are large beside what is left of
            // the sum: in one part dq was off by 0.0028 of its norm, and is by 0.0020 (0.0017 is its own rounding).  8192 tokens forward and back: 338 us, 320 in one
            PkFrag fk[2], fv[2], ft[2], pf[4], pl[4];
            const PkOffsets<HD> o(off, lds_at + (j & 1) * (2 * TILE));
            auto read_rows = [&](int i) __attribute__((always_inline)) {
                fk[i & 1].v = o.row(i / KS, i % KS);
                fv[i & 1].v = o.row(i / KS, i % KS, TILE);
            };
            auto read_trans = [&](int i) __attribute__((always_inline)) { pk_read_trans<HD>(o, (i / DB) * 16 * HD * 2, i % DB, ft[i & 1]); };
            const pk_floatx16 zero = {};
            read_rows(0);
            read_rows(1);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pk_floatx16 s, dp;
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const int i = h * KS + ks;
                    s = pk_mfma(fk[i & 1], qf[ks], ks == 0 ? zero : s);
                    dp = pk_mfma(fv[i & 1], df[ks], ks == 0 ? zero : dp);
                    if (i + 2 < 2 * KS) read_rows(i + 2);
                    // the second product of the 32 keys before
                    if (h == 1 && !careful) {
#pragma unroll
                        for (int u = 0; u < 2 * DB / KS; ++u) {
                            const int n = ks * (2 * DB / KS) + u;
                            acc[n % DB] = pk_mfma(ft[n & 1], pf[n / DB], acc[n % DB]);
                            acc[n % DB] = pk_mfma(ft[n & 1], pl[n / DB], acc[n % DB]);
                            read_trans(n + 2);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (h == 0 && !careful) { read_trans(0); read_trans(1); }
                float ds[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) ds[e] = __builtin_amdgcn_exp2f(fmaf(s[e], sc, -info.x)) * (dp[e] - info.y);
                if (mask) {
                    // (the only key that a row sees has the probability 1 whatever its score)
                    const int limit = limit_of(), rel = limit == 0 ? -1 : limit - kb - 4 * hi;
#pragma unroll
                    for (int e = 0; e < 16; ++e) ds[e] = 32 * h + pk_pos(e) <= rel ? ds[e] : 0.f;
                }
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const uint32_t w = pack_bf16x2(ds[e], ds[e + 1]);
                    pf[2 * h + (e >> 3)].w[(e & 7) >> 1] = w;
                    pl[2 * h + (e >> 3)].w[(e & 7) >> 1] = pack_bf16x2(ds[e] - __uint_as_float(w << 16), ds[e + 1] - __uint_as_float(w & 0xFFFF0000u));
                }
            }
            if constexpr (careful) {
                if (mask) {
                    pk_second_careful<HD, false, true>(kt, pf, pl, pl, acc);
                    return;
                }
                read_trans(0);
                read_trans(1);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = careful ? 0 : 2 * DB; n < 4 * DB; ++n) {
                acc[n % DB] = pk_mfma(ft[n & 1], pf[n / DB], acc[n % DB]);
                acc[n % DB] = pk_mfma(ft[n & 1], pl[n / DB], acc[n % DB]);
                if (n + 2 < 4 * DB) read_trans(n + 2);
                __builtin_amdgcn_sched_barrier(0);
            }
    };
#pragma unroll
    for (int d = 0; d < DB; ++d) pk_zero(acc[d]);
    begin();
    if (tiles > 0) arrive(0);
    // Delta of rows that see one tile of keys at most, exactly: with out's and the probabilities' roundings in it the differences do - delta of few keys are off by
    // 2^-8 of themselves (dq of sequences of some five tokens by 0.0045 of its norm, so by 0.0017), and here it is 32 instructions more.  For dk and dv too, and
    // for a pass with care, which reads it
    if (!careful && tiles == 1) {
        __syncthreads();
        if (wlast >= 0) {
            const PkOffsets<HD> o(off, lds_at);
            const int rel = limit_of() - 4 * hi;
            float rest = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pk_floatx16 s = {}, dp = {};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    PkFrag kf, vf;
                    kf.v = o.row(h, ks);
                    vf.v = o.row(h, ks, TILE);
                    s = pk_mfma(kf, qf[ks], s);
                    dp = pk_mfma(vf, df[ks], dp);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) rest += 32 * h + pk_pos(e) <= rel ? __builtin_amdgcn_exp2f(fmaf(s[e], sc, -info.x)) * (dp[e] - info.y) : 0.f;
            }
            rest = pk_sum_halves(rest);
            info.y += rest;
            const Row r = row_of_lane();
            if (r.mine && hi == 0 && r.limit >= 0) {
                const uint2 v = pk_split3(-info.y);
                uint2* to = reinterpret_cast<uint2*>(g.rowinfo + r.tok * a.n_heads + r.head) + 1;
                *to = v;
            }
        }
    }
    for (int j = 0; j < tiles; ++j) {
        lds_barrier();
        if (j + 1 < tiles) request(j + 1);
        one_tile(j);
        if (j + 1 < tiles) arrive(j + 1);
    }
    if (!careful && __syncthreads_or(row_of_lane().mine && pk_not_finite(acc))) return true;
    const Row r = row_of_lane();
    pk_store<HD>(acc, a.scale, g.dq + r.tok * g.lddq + (int64_t)r.head * HD, r.mine);
    return false;
}
template <int HD>
__device__ __noinline__ void pk_dq_again(PackedArgs a, PkBackward g, pk_lchar lds) { (void)pk_dq<HD, true>(a, g, lds); }
template <int HD>
__global__ __launch_bounds__(64 * PK_WAVES) __attribute__((amdgpu_waves_per_eu(2, 2))) void pk_dq_kernel(PackedArgs a, PkBackward g) {
    extern __shared__ __align__(1024) char pk_dynamic[];
    if (pk_dq<HD, false>(a, g, (pk_lchar)pk_dynamic)) pk_dq_again<HD>(a, g, (pk_lchar)pk_dynamic);
}

// dk, dv: four waves of 32 keys, K and V in registers, against tiles of 64 rows of q and do that they share.  Sums, operands and scores are some 300
// registers: one wave to a SIMD.  What belongs to a row comes in through the products, as a further step of 16 dims of which three are used: read row by
// row in the instruction's layout it was 24 KB of LDS reads a tile and wave beside 64 KB of operands
template <int HD, bool careful>
__device__ __forceinline__ bool pk_dkv(const PackedArgs& a, const PkBackward& g, pk_lchar lds) {
    char* pk_smem = (char*)lds;
    const int lds_at = (int)(uint32_t)(uintptr_t)lds;
    const bf16_t* dout = g.dout;
    const int64_t lddo = g.lddo;
    constexpr int TILE = PK_T * HD * 2, KS = HD / 16, DB = HD / 32;
    uint4* infos = reinterpret_cast<uint4*>(pk_smem + 4 * TILE);              // two stages of a tile's rows
    int* limits = reinterpret_cast<int*>(infos + 2 * PK_T);                   // ... and the last key that they see
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hi = lane >> 5;
    const int G = PkDiv(a.n_kv)(a.n_heads), at = PkDiv(a.n_kv)((int)blockIdx.x), kvh = (int)blockIdx.x - at * a.n_kv;
    PkTile t;
    if (!pk_find<PK_ROWS, true>(a, at, G, 0, t)) return false;
    const int R = t.nq * G, shift = t.nk - t.nq;
    const int key0 = t.tile * PK_ROWS, wkey = key0 + wave * 32;
    const int key = min(wkey + (lane & 31), t.nk - 1);
    const bool mine = wkey + (lane & 31) < t.nk;
    const int from = a.causal ? max(key0 - shift, 0) * G : 0, all = (R - from + PK_T - 1) / PK_T;      // (below R, if there are any: key0 < nk)
    // this share's of the row tiles
    const int j0 = (int)((int64_t)all * blockIdx.y / gridDim.y), tiles = (int)((int64_t)all * (blockIdx.y + 1) / gridDim.y) - j0, row0 = from + j0 * PK_T;
    const PkDiv query_of(G);
    // a tile's rows on their way; rows past the end repeat the last one
    constexpr int N = PK_T * HD * 2 / 4096, ROWS = 1024 / (HD * 2);
    const bf16_t* Qh = a.q + (int64_t)t.q0 * a.ldq + (int64_t)kvh * G * HD;
    const bf16_t* Dh = dout + (int64_t)t.q0 * lddo + (int64_t)kvh * G * HD;
    uint4 qd[N], dd[N], next = make_uint4(0, 0, 0, 0);
    int next_limit = -1;
    // Where the next tile starts: its first row's query and head, and the lane's rows relative to that query: head and byte offsets.  A tile on, 64 rows are
    // so many queries and heads, with a query more where the heads pass G
    const int step_q = query_of(PK_T), step_h = PK_T - step_q * G, ldq2 = (int)(2 * a.ldq), ldd2 = (int)(2 * lddo);
    int at_q, at_h, lane_h[N], lane_q[N], lane_d[N];
    auto start_rows = [&]() __attribute__((always_inline)) {
        at_q = query_of(row0);
        at_h = row0 - at_q * G;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = ROWS * (N * wave + i) + lane / (HD / 8), q = query_of(at_h + r), chunk = ((lane % (HD / 8)) ^ pk_swz<HD>(r)) << 4;
            lane_h[i] = at_h + r - q * G;
            lane_q[i] = q * ldq2 + lane_h[i] * (HD * 2) + chunk;
            lane_d[i] = q * ldd2 + lane_h[i] * (HD * 2) + chunk;
        }
    };
    auto request = [&](int j) __attribute__((always_inline)) {
        const int base = row0 + j * PK_T;
        const auto rq = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(Qh + at_q * a.ldq), 0, (int)0xFFFFFFFFu, 0x00020000);
        const auto rd = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(Dh + at_q * lddo), 0, (int)0xFFFFFFFFu, 0x00020000);
        // (one way for all tiles, as in PkLoader)
        const int left = R - base, end_q = query_of(R - 1), end_h = R - 1 - end_q * G;
        const int end_at_q = (end_q - at_q) * ldq2 + end_h * (HD * 2), end_at_d = (end_q - at_q) * ldd2 + end_h * (HD * 2);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = ROWS * (N * wave + i) + lane / (HD / 8), chunk = ((lane % (HD / 8)) ^ pk_swz<HD>(r)) << 4;
            qd[i] = pk_load16(rq, r < left ? lane_q[i] : end_at_q + chunk, 0);
            dd[i] = pk_load16(rd, r < left ? lane_d[i] : end_at_d + chunk, 0);
        }
        if (wave == 0) {
            const int r = min(base + lane, R - 1), q = query_of(r);
            next = g.rowinfo[(int64_t)(t.q0 + q) * a.n_heads + kvh * G + (r - q * G)];
            next_limit = base + lane >= R ? -1 : a.causal ? q + shift : t.nk - 1;
        }
        // on to the tile behind
        at_q += step_q;
        at_h += step_h;
        const bool over = at_h >= G;
        at_q += over ? 1 : 0;
        at_h -= over ? G : 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int h = lane_h[i] + step_h, back = h >= G ? HD * 2 * G : 0, more = (h >= G ? 1 : 0) - (over ? 1 : 0);
            lane_h[i] = h >= G ? h - G : h;
            const int by = step_h * (HD * 2) - back;
            lane_q[i] += by + (more > 0 ? ldq2 : more < 0 ? -ldq2 : 0);
            lane_d[i] += by + (more > 0 ? ldd2 : more < 0 ? -ldd2 : 0);
        }
    };
    auto arrive = [&](int j) __attribute__((always_inline)) {
        char* stage = pk_smem + (j & 1) * (2 * TILE) + wave * (N * 1024) + lane * 16;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            *reinterpret_cast<uint4*>(stage + i * 1024) = qd[i];
            *reinterpret_cast<uint4*>(stage + TILE + i * 1024) = dd[i];
        }
        if (wave == 0) {
            infos[(j & 1) * PK_T + lane] = next;
            limits[(j & 1) * PK_T + lane] = next_limit;
        }
    };
    const PkOffsets<HD> off;
    PkFrag kf[KS], vf[KS], ones;
    const bf16_t* ksrc = a.k + (int64_t)(t.k0 + key) * a.ldk + kvh * HD + 8 * hi;
    const bf16_t* vsrc = a.v + (int64_t)(t.k0 + key) * a.ldv + kvh * HD + 8 * hi;
    auto begin = [&]() __attribute__((always_inline)) {                       // (as in the forward)
        if (tiles <= 0) return;
        start_rows();
        request(0);
        asm volatile("" : "+v"(ksrc), "+v"(vsrc));
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            kf[ks].u = *reinterpret_cast<const uint4*>(ksrc + 16 * ks);
            vf[ks].u = *reinterpret_cast<const uint4*>(vsrc + 16 * ks);
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);
    };
    ones.u = hi ? make_uint4(0, 0, 0, 0) : make_uint4(0x3F803F80u, 0x3F80u, 0, 0);
    const float sc = a.scale * PK_LOG2E;
    pk_floatx16 ak[DB], av[DB];
    // A tile in an order of its own, which the compiler is kept to: with one wave to a SIMD nothing else fills the waits, and left to itself the compiler reads
    // operands right before each instruction.  Operands are read four instructions ahead; the first 32 rows' scores; the others' beside the first ones'
    // exponentials; the second products of the first beside the others' exponentials; the rest.  MASK: not all of its rows see all keys of the wave
    auto tile = [&](auto MASK, int j) __attribute__((always_inline)) {
        constexpr bool mask = decltype(MASK)::value, apart = careful && mask;
        const int* limit = limits + (j & 1) * PK_T + 4 * hi;
        int4 last[2];
        auto read_last = [&](int h, int g4) __attribute__((always_inline)) { last[g4 & 1] = *reinterpret_cast<const int4*>(limit + 32 * h + 8 * g4); };
        const PkOffsets<HD> o(off, lds_at + (j & 1) * (2 * TILE));
        const uint4* info = infos + (j & 1) * PK_T;
        PkFrag fq[4], fd[4], xl[2], xd[2], pf[4], df[4];
        const pk_floatx16 zero = {};
        pk_floatx16 s[2], dp[2];
        float p_[2], d_[2];
        auto read_rows = [&](int i) __attribute__((always_inline)) {
            fq[i & 3].v = o.row(i / KS, i % KS);
            fd[i & 3].v = o.row(i / KS, i % KS, TILE);
        };
        // second products: for each 16 rows the DB groups of dims of dv, then those of dk
        auto read_trans = [&](int i) __attribute__((always_inline)) {
            const int slab = i / (2 * DB), k = i % (2 * DB);
            pk_read_trans<HD>(o, (k < DB ? TILE : 0) + slab * 16 * HD * 2, k % DB, fq[i & 3]);
        };
        auto element = [&](int h, int e) __attribute__((always_inline)) {
            p_[e & 1] = __builtin_amdgcn_exp2f(s[h][e] * sc);
            d_[e & 1] = dp[h][e] * p_[e & 1];
            if constexpr (mask) {
                if (e % 4 == 0 && e < 12) read_last(h, e / 4 + 1);
                const int4 l4 = last[(e >> 2) & 1];
                const int l = (e & 3) == 0 ? l4.x : (e & 3) == 1 ? l4.y : (e & 3) == 2 ? l4.z : l4.w;
                const bool seen = wkey + (lane & 31) <= l;
                p_[e & 1] = seen ? p_[e & 1] : 0.f;
                // (the only key that a row sees has the probability 1 whatever its score)
                d_[e & 1] = seen && l > 0 ? d_[e & 1] : 0.f;
            }
            // (in one bf16 part each: dk and dv are off by 0.0024 and 0.0023 of their norms, of which 0.0017 is their own rounding.  Second parts would be half as many
            // matrix instructions again, and registers that there are none of)
            if (e & 1) {
                pf[2 * h + (e >> 3)].w[(e & 7) >> 1] = pack_bf16x2(p_[0], p_[1]);
                df[2 * h + (e >> 3)].w[(e & 7) >> 1] = pack_bf16x2(d_[0], d_[1]);
            }
        };
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 in = info[32 * h + (lane & 31)];
            xl[h].u = make_uint4(in.x, in.y, 0, 0);
            xd[h].u = make_uint4(in.z, in.w, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) read_rows(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
            const int h = i / KS, ks = i % KS;
            if (ks == 0) {
                if constexpr (mask) {
                    if (h == 1) read_last(0, 0);
                }
                s[h] = pk_mfma(xl[h], ones, zero);
                dp[h] = pk_mfma(xd[h], ones, zero);
                __builtin_amdgcn_sched_barrier(0);
            }
            s[h] = pk_mfma(fq[i & 3], kf[ks], s[h]);
            dp[h] = pk_mfma(fd[i & 3], vf[ks], dp[h]);
            if (i + 4 < 2 * KS) read_rows(i + 4);
            else if (!apart) read_trans(i + 4 - 2 * KS);
            if (h == 1) {
#pragma unroll
                for (int e = 0; e < 16 / KS; ++e) element(0, ks * (16 / KS) + e);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (mask) read_last(1, 0);
        if constexpr (apart) {
#pragma unroll
            for (int e = 0; e < 16; ++e) element(1, e);
            const char* qt = pk_smem + (j & 1) * (2 * TILE);
            PkFrag seen[4];
#pragma unroll
            for (int s4 = 0; s4 < 4; ++s4)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int at = 16 * s4 + (w >> 1) * 8 + (w & 1) * 2;
                    seen[s4].w[w] = (wkey + (lane & 31) <= limit[at] ? 0x3F80u : 0u) | (wkey + (lane & 31) <= limit[at + 1] ? 0x3F800000u : 0u);
                }
            pk_second_careful<HD, true, false>(qt + TILE, pf, pf, seen, av);
            pk_second_careful<HD, false, false>(qt, df, df, df, ak);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8 * DB; ++i) {
            const int slab = i / (2 * DB), k = i % (2 * DB);
            if (k < DB) av[k] = pk_mfma(fq[i & 3], pf[slab], av[k]);
            else ak[k - DB] = pk_mfma(fq[i & 3], df[slab], ak[k - DB]);
            if (i + 4 < 8 * DB) read_trans(i + 4);
            if (i < 4 * DB) {
#pragma unroll
                for (int e = 0; e < 4 / DB; ++e) element(1, i * (4 / DB) + e);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto one_tile = [&](int j) __attribute__((always_inline)) {
        const int base = row0 + j * PK_T;
        const int low = a.causal ? query_of(base) + shift : t.nk - 1, high = a.causal ? query_of(min(base + PK_T - 1, R - 1)) + shift : t.nk - 1;   // the rows' first and last limit
        if (high < wkey) return;                                              // (wave-uniform)
        if (low >= wkey + 31 && base + PK_T <= R) tile(std::false_type(), j);
        else tile(std::true_type(), j);
    };
#pragma unroll
    for (int d = 0; d < DB; ++d) { pk_zero(ak[d]); pk_zero(av[d]); }
    begin();
    if (tiles > 0) arrive(0);
    for (int j = 0; j < tiles; ++j) {
        lds_barrier();
        if (j + 1 < tiles) request(j + 1);
        one_tile(j);
        // (the sums stay in accumulation registers: where the ways through a tile meet, the compiler takes them to ordinary ones and back, 256 instructions)
#pragma unroll
        for (int d = 0; d < DB; ++d) asm volatile("" : "+a"(ak[d]), "+a"(av[d]));
        if (j + 1 < tiles) arrive(j + 1);
    }
    if (!careful && __syncthreads_or(mine && (pk_not_finite(ak) || pk_not_finite(av)))) return true;
    if (g.part) {
        float* to = g.part + ((((int64_t)blockIdx.y * a.total_k + t.k0 + key) * a.n_kv + kvh) * 2) * HD + 4 * hi;
        if (mine) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int g4 = 0; g4 < 4; ++g4) {
                    *reinterpret_cast<float4*>(to + 32 * db + 8 * g4) = make_float4(ak[db][4 * g4], ak[db][4 * g4 + 1], ak[db][4 * g4 + 2], ak[db][4 * g4 + 3]);
                    *reinterpret_cast<float4*>(to + HD + 32 * db + 8 * g4) = make_float4(av[db][4 * g4], av[db][4 * g4 + 1], av[db][4 * g4 + 2], av[db][4 * g4 + 3]);
                }
        }
        return false;
    }
    pk_store<HD>(av, 1.f, g.dv + (int64_t)(t.k0 + key) * g.lddv + (int64_t)kvh * HD, mine);
    pk_store<HD>(ak, a.scale, g.dk + (int64_t)(t.k0 + key) * g.lddk + (int64_t)kvh * HD, mine);
    return false;
}
template <int HD>
__device__ __noinline__ void pk_dkv_again(PackedArgs a, PkBackward g, pk_lchar lds) { (void)pk_dkv<HD, true>(a, g, lds); }
template <int HD>
__global__ __launch_bounds__(64 * PK_WAVES) __attribute__((amdgpu_waves_per_eu(1, 1))) void pk_dkv_kernel(PackedArgs a, PkBackward g) {
    extern __shared__ __align__(1024) char pk_dynamic[];
    if (pk_dkv<HD, false>(a, g, (pk_lchar)pk_dynamic)) pk_dkv_again<HD>(a, g, (pk_lchar)pk_dynamic);
}

// The shares' sums of dk and dv added in order, HD / 4 lanes a row of dk and of dv
template <int HD>
__global__ __launch_bounds__(256) void pk_dkv_join_kernel(PackedArgs a, PkBackward g, int shares) {
    constexpr int LANES = HD / 2;
    const int64_t rows = a.total_k * a.n_kv, row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES;
    if (row >= rows) return;
    const int64_t tok = row / a.n_kv;
    if (tok < a.cu_k[0] || tok >= a.cu_k[a.n_seq]) return;                    // a row of no sequence
    const int j = threadIdx.x % LANES;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < shares; i += 8) {
        float4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const float4*>(g.part + (min(i + u, shares - 1) * rows + row) * (2 * HD) + 4 * j);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i + u < shares) { s.x += v[u].x; s.y += v[u].y; s.z += v[u].z; s.w += v[u].w; }
    }
    const bool k = j < LANES / 2;
    const float f = k ? a.scale : 1.f;
    bf16_t* to = (k ? g.dk + tok * g.lddk : g.dv + tok * g.lddv) + (row - tok * a.n_kv) * HD + 4 * (j % (LANES / 2));
    *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(s.x * f, s.y * f), pack_bf16x2(s.z * f, s.w * f));
}

// an upper bound of the row (key) tiles of all sequences, whatever their lengths
int64_t pk_units(int64_t total, int n_seq, int n_kv) { return (total / PK_ROWS + std::min<int64_t>(n_seq, total)) * n_kv; }

// Tiles of 64 keys a share, 0: row tiles are not shared out.  They are where rows are few beside the keys (single new tokens: a sequence is a
// workgroup for each key head then, whatever its length) or where row tiles are fewer than the compute units: for about two shares to each of two workgroups on a
// compute unit, of 8 tiles and more (a share costs a workgroup's start, its sums and a launch that joins them), 128 of a sequence at most and 256 MB of sums.
// Lengths are on the device: work is reckoned from their mean, and sequences of 16 tiles and more in the mean are taken to be uneven.  (Where a
// cache's rooms are mostly empty, or one long sequence is among many short ones, shares are too few for it.)  64 sequences of 200000
// keys together, up to 16760: 426 us without, 175 so, 186 with one share to each
bool pk_few_rows(const PackedArgs& a) { return a.total_q * (a.n_heads / a.n_kv) * 8 <= a.total_k; }
int pk_chunk(const PackedArgs& a, int head_dim) {
    const int64_t G = a.n_heads / a.n_kv, units = pk_units(a.total_q * G, a.n_seq, a.n_kv), rows = a.total_q * a.n_heads;
    if (units < 1 || a.total_k < 1) return 0;
    const int64_t all = (a.total_k + PK_T - 1) / PK_T, mean = (a.total_k / std::max(1, a.n_seq) + PK_T - 1) / PK_T;
    if (mean < 16 || !(pk_few_rows(a) || units < 256)) return 0;
    const int64_t chunk = std::max<int64_t>({8, (units * mean + 1023) / 1024, (all + 127) / 128, all * rows * head_dim * 4 / (1LL << 28)});
    return (int)std::min<int64_t>(chunk, 1 << 20);
}
int64_t pk_most_shares(const PackedArgs& a, int chunk) { return ((a.total_k + PK_T - 1) / PK_T + chunk - 1) / chunk; }

// Shares of the rows that a tile of keys is multiplied with: few tiles of keys take several workgroups each, for about one to a compute unit, of four tiles of 64
// rows and more in the mean.  1001 tokens of eight heads on one: 301 us without, 37 so
int pk_dkv_shares(const PackedArgs& a) {
    const int64_t G = a.n_heads / a.n_kv, units = pk_units(a.total_k, a.n_seq, a.n_kv);
    if (units < 1) return 1;
    const int64_t rows = a.total_q * G / std::max(1, a.n_seq) / PK_T;
    return (int)std::max<int64_t>(1, std::min<int64_t>(256 / units, rows / 4));
}

// so much LDS for a kernel, once on each device
template <typename F>
hipError_t pk_lds(F* f, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (e != hipSuccess || (done.load(std::memory_order_relaxed) & bit)) return e;
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(f), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

template <int HD>
hipError_t pk_launch_forward(const PackedArgs& a, bf16_t* out, int64_t ldo, float* lse, void* workspace, hipStream_t st) {
    constexpr int SMEM = 4 * PK_T * HD * 2;
    static std::atomic<uint64_t> done{0}, done_fine{0};
    const bool fine = a.total_q <= a.n_seq || pk_few_rows(a);      // (single rows, of however few keys)
    const hipError_t attr = fine ? pk_lds(pk_forward_kernel<HD, true>, SMEM, done_fine) : pk_lds(pk_forward_kernel<HD, false>, SMEM, done);
    if (attr != hipSuccess) return attr;
    const int G = a.n_heads / a.n_kv, chunk = pk_chunk(a, HD);
    const int64_t rows = a.total_q * a.n_heads, blocks = (rows * (HD / 4) + 255) / 256;
    int64_t units = pk_units(a.total_q * G, a.n_seq, a.n_kv);
    float* part = nullptr;
    float2* ml = nullptr;
    if (chunk > 0) {
        const int64_t shares = pk_most_shares(a, chunk);
        part = static_cast<float*>(workspace);
        ml = reinterpret_cast<float2*>(part + shares * rows * HD);
        // (the row tiles and, for each share of a sequence more, as many as a sequence may have; numbers behind the last leave at once)
        units += shares * (a.total_q * G / PK_ROWS + 1) * a.n_kv;
    }
    if (units >= kPackedUnits || (chunk > 0 && blocks >= kPackedUnits)) return hipErrorInvalidValue;
    const PkForwardOut to{out, ldo, lse, part, ml, chunk};
    if (fine) hipLaunchKernelGGL((pk_forward_kernel<HD, true>), dim3((unsigned)units), dim3(64 * PK_WAVES), SMEM, st, a, to);
    else hipLaunchKernelGGL((pk_forward_kernel<HD, false>), dim3((unsigned)units), dim3(64 * PK_WAVES), SMEM, st, a, to);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || chunk == 0) return e;
    hipLaunchKernelGGL(pk_join_kernel<HD>, dim3((unsigned)blocks), dim3(256), 0, st, a, part, ml, chunk, out, ldo, lse);
    return hipGetLastError();
}

template <int HD>
hipError_t pk_launch_backward(const PackedArgs& a, const PackedGrad& g, void* workspace, hipStream_t st) {
    constexpr int SMEM = 4 * PK_T * HD * 2, SMEM_KV = SMEM + 2 * PK_T * 20;
    static std::atomic<uint64_t> done_q{0}, done_kv{0};
    const hipError_t attr_q = pk_lds(pk_dq_kernel<HD>, SMEM, done_q), attr_kv = pk_lds(pk_dkv_kernel<HD>, SMEM_KV, done_kv);
    if (attr_q != hipSuccess) return attr_q;
    if (attr_kv != hipSuccess) return attr_kv;
    const int64_t rows = a.total_q * a.n_heads, G = a.n_heads / a.n_kv;
    const int64_t dq_units = pk_units(a.total_q * G, a.n_seq, a.n_kv), kv_units = pk_units(a.total_k, a.n_seq, a.n_kv);
    if (dq_units >= kPackedUnits || kv_units >= kPackedUnits) return hipErrorInvalidValue;
    uint4* info = static_cast<uint4*>(workspace);
    const int shares = pk_dkv_shares(a);
    const int64_t kv_rows = a.total_k * a.n_kv, kv_blocks = (kv_rows * (HD / 2) + 255) / 256;
    float* part = shares > 1 ? reinterpret_cast<float*>(info + rows) : nullptr;
    const PkBackward b{g.out, g.dout, g.ldo, g.lddo, g.lse, info, g.dq, g.lddq, g.dk, g.lddk, g.dv, g.lddv, part};
    hipError_t e = hipSuccess;
    if (rows > 0) {
        hipLaunchKernelGGL(pk_dq_kernel<HD>, dim3((unsigned)dq_units), dim3(64 * PK_WAVES), SMEM, st, a, b);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.total_k > 0) {
        hipLaunchKernelGGL(pk_dkv_kernel<HD>, dim3((unsigned)kv_units, (unsigned)shares), dim3(64 * PK_WAVES), SMEM_KV, st, a, b);
        e = hipGetLastError();
        if (e != hipSuccess || !part) return e;
        hipLaunchKernelGGL(pk_dkv_join_kernel<HD>, dim3((unsigned)kv_blocks), dim3(256), 0, st, a, b, shares);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int64_t packed_units(const PackedArgs& a) { return std::max(pk_units(a.total_q * (a.n_heads / a.n_kv), a.n_seq, a.n_kv), pk_units(a.total_k, a.n_seq, a.n_kv)); }
size_t packed_forward_workspace_bytes(const PackedArgs& a, int head_dim) {
    const int chunk = pk_chunk(a, head_dim);
    return chunk == 0 ? 0 : (size_t)pk_most_shares(a, chunk) * a.total_q * a.n_heads * (head_dim * sizeof(float) + sizeof(float2));
}
size_t packed_backward_workspace_bytes(const PackedArgs& a, int head_dim) {
    const int shares = pk_dkv_shares(a);
    return (size_t)a.total_q * a.n_heads * sizeof(uint4) + (shares == 1 ? 0 : (size_t)shares * a.total_k * a.n_kv * 2 * head_dim * sizeof(float));
}

hipError_t launch_packed_forward(const PackedArgs& a, int head_dim, bf16_t* out, int64_t ldo, float* lse, void* workspace, hipStream_t st) {
    if (a.total_q == 0 || a.n_seq == 0) return hipSuccess;
    return head_dim == 128 ? pk_launch_forward<128>(a, out, ldo, lse, workspace, st) : pk_launch_forward<64>(a, out, ldo, lse, workspace, st);
}

hipError_t launch_packed_backward(const PackedArgs& a, int head_dim, const PackedGrad& g, void* workspace, hipStream_t st) {
    if (a.n_seq == 0) return hipSuccess;
    return head_dim == 128 ? pk_launch_backward<128>(a, g, workspace, st) : pk_launch_backward<64>(a, g, workspace, st);
}

}  // namespace agzo
