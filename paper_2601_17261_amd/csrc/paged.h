// A cache of keys and values in pages, as its kernels see it.
#pragma once
#include "agzo_internal.h"

namespace agzo {

// x / d for 0 <= x < 2^31: the quotient by a multiplication is at most one short
struct QuickDiv {
    uint32_t d, m;
    QuickDiv() = default;
    explicit QuickDiv(int by) : d((uint32_t)by), m((uint32_t)(0x100000000ull / (uint32_t)by - (by == 1))) {}
    __device__ __forceinline__ int operator()(int x) const {
        uint32_t q = __umulhi((uint32_t)x, m);
        q += (uint32_t)x - q * d >= d;
        return (int)q;
    }
};

// One sequence's new tokens q0 .. q0 + nq, and how many keys it has, they among them.  (nk < nq: the first nq - nk of them have no place)
struct PagedSeq { int q0, nq, nk; };

__device__ __forceinline__ PagedSeq paged_seq(const PagedCache& c, const int32_t* cu_q, int total_q, int s) {
    PagedSeq r;
    r.q0 = min(max(cu_q[s], 0), total_q);
    r.nq = min(max(cu_q[s + 1], r.q0), total_q) - r.q0;
    r.nk = min(max(c.k_len[s], 0), c.max_pages * c.page_size);
    return r;
}

// The sequence that a token is of, by all lanes of a wave for one token: the last one that starts at or before it.  -1: none
__device__ __forceinline__ int paged_find(const PagedCache& c, const int32_t* cu_q, int total_q, int tok, PagedSeq& r) {
    const int lane = threadIdx.x & 63;
    int seq = -1;
    for (int b = 0; b < c.n_seq; b += 64) {
        const int s = min(b + lane, c.n_seq - 1);
        const PagedSeq mine = paged_seq(c, cu_q, total_q, s);
        const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(b + lane < c.n_seq && mine.q0 <= tok));
        if (n == 0) continue;
        seq = b + n - 1;
        r.q0 = __builtin_amdgcn_readlane(mine.q0, n - 1);
        r.nq = __builtin_amdgcn_readlane(mine.nq, n - 1);
        r.nk = __builtin_amdgcn_readlane(mine.nk, n - 1);
    }
    return seq >= 0 && tok - r.q0 < r.nq ? seq : -1;
}

// Where a sequence's place lies: its page and the slot in it.  false: nowhere
__device__ __forceinline__ bool paged_slot(const PagedCache& c, const QuickDiv& by_page, int seq, int place, int64_t& page, int& slot) {
    if (place < 0 || place >= c.max_pages * c.page_size) return false;
    const int p = by_page(place);
    slot = place - p * c.page_size;
    page = c.table[(int64_t)seq * c.ld_table + p];
    return page >= 0 && page < c.n_pages;
}

}  // namespace agzo
