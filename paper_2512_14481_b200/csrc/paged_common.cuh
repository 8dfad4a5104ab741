// Shared by the paged-cache kernels: the launch parameters, the lookup of a sequence, the division of an attention
// call's work among its thread blocks, and the conversion of int8 and 4-bit codes.
#pragma once

#include "common.cuh"

namespace sasq {

int* paged_status_ptr();    // device address of the paged kernels' sticky status word; nullptr if it cannot be had

// What both operators know about the cache and the batch (all sizes validated on the host).
struct PagedParams {
    void* k;
    void* v;
    const float* k_scale;
    const float* v_scale;
    long long page_stride, token_stride, head_stride;     // elements
    long long num_pages;
    const int* page_table;
    const int* seq_lens;
    const int* q_starts;
    long long table_stride;
    int batch, max_pages, total_q;
    int page_shift;             // log2(page_size)
    int kv_heads;
    int kind;                   // sasq_kv_kind_t
    int* status;
};

// Host checks common to both operators; fills the shared parameters.
int paged_check(const sasq_kv_cache_t* c, const sasq_kv_batch_t* b, int dt, PagedParams* p);

namespace {

// A sequence's new tokens and keys as the device arrays give them, cut to what is safe to touch.
struct Sequence {
    int first, new_len, len;
    int given_len;              // seq_lens' own value: positions follow from it, not from the cut length
};
__device__ __forceinline__ Sequence load_sequence(const PagedParams& p, int b) {
    Sequence s;
    const int q0 = p.q_starts[b], q1 = p.q_starts[b + 1];
    int len = p.seq_lens[b];
    const long long room = (long long)p.max_pages << p.page_shift;
    const bool bad = q0 < 0 || q1 < q0 || q1 > p.total_q || len < 0 || len > room;
    if (bad) atomicMax(p.status, (int)SASQ_ERR_BAD_INDEX);
    s.first = q0;
    s.new_len = (q0 < 0 || q1 < q0 || q1 > p.total_q) ? 0 : q1 - q0;
    s.len = len < 0 ? 0 : (len > room ? (int)room : len);
    s.given_len = len;
    return s;
}

// ---------------------------------------------------------------------------------------------------------------------
// Work of an attention call.  The rows of one KV head are (new token, query head of the group) pairs, token first; a
// fixed number of consecutive rows of a sequence and KV head are an item, and an item's keys are walked in units of KT.
// The units of all items, laid end to end (sequence, KV head, item, key), are cut into equal stretches, one per thread
// block: every block has the same amount of work whatever the lengths are, a block walks whole items in the middle of its stretch
// and at most two part items at its ends.  Beginning and ending an item costs as much as COST units, which stand before
// the item's own in the row: without them a block that gets many short items is the tail.  Part items leave (O, m, l) in
// the workspace, and a second launch joins them.
// A split by whole items alone would leave most SMs idle for few long sequences, and a fixed number of splits per item
// makes the longest sequence of a ragged batch the tail.
// ---------------------------------------------------------------------------------------------------------------------
struct Item {
    int b, h, i;              // sequence, KV head, row tile
    Sequence s;
    int units;                // of the whole item
    int t0, t1;               // this block's units
    long long first;          // where the item begins in the row of all
};

template <int KT, int COST>
struct Schedule {
    int rows;                 // of an item
    int group, causal, heads;

    __device__ __forceinline__ int tiles(const Sequence& s) const { return (s.new_len * group + rows - 1) / rows; }
    // keys that the rows of tile i can see at most
    __device__ __forceinline__ int key_limit(const Sequence& s, int i) const {
        if (!causal) return s.len;
        return max(0, s.len - s.new_len + (min((i + 1) * rows, s.new_len * group) - 1) / group + 1);
    }
    // an item without keys still counts one unit: its rows have to be written
    __device__ __forceinline__ int units(const Sequence& s, int i) const {
        const int n = (key_limit(s, i) + KT - 1) / KT;
        return n < 1 ? 1 : n;
    }
    // length of an item, and of a sequence's items of one KV head, in the row
    __device__ __forceinline__ int cost(const Sequence& s, int i) const { return units(s, i) + COST; }
    __device__ __forceinline__ long long head_cost(const Sequence& s) const {
        const int n = tiles(s);
        if (n == 0) return 0;
        if (!causal) return (long long)n * cost(s, 0);
        long long sum = 0;
        for (int i = 0; i < n; ++i) sum += cost(s, i);
        return sum;
    }
};

// Where block c's stretch begins when a row of `total` units goes to n blocks.
__device__ __forceinline__ long long block_begin(long long total, int c, int n) {
    if (total < (1 << 20)) return (unsigned)total * (unsigned)c / (unsigned)n;      // c, n < 4096
    return total * c / n;
}
// The block that has unit x.
__device__ __forceinline__ int block_of(long long total, long long x, int n) {
    if (total < (1 << 20)) return (int)((((unsigned)x + 1) * (unsigned)n + (unsigned)total - 1) / (unsigned)total) - 1;
    return (int)(((x + 1) * n + total - 1) / total) - 1;
}

// Where a block's stretch begins.
struct Start {
    long long total;          // length of the row of all items
    long long begin, end;     // this block's
    long long offset;         // of `begin` in sequence b
    int b;                    // -1: nothing to do
    int blocks;               // blocks that have work
};

// A whole warp calls this; every lane gets the answer.  Each lane adds up a run of sequences: no barrier, and one round
// trip to memory for up to 32 sequences.
template <int KT, int COST>
__device__ __forceinline__ Start find_start(const PagedParams& p, const Schedule<KT, COST>& sch, int max_blocks) {
    const int lane = threadIdx.x & 31;
    const int per = (p.batch + 31) >> 5;
    const int b0 = lane * per, b1 = min(b0 + per, p.batch);
    long long mine = 0;
    for (int b = b0; b < b1; ++b) mine += sch.head_cost(load_sequence(p, b)) * sch.heads;
    long long incl = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const long long other = __shfl_up_sync(0xFFFFFFFFu, incl, off);
        if (lane >= off) incl += other;
    }
    Start st;
    st.total = __shfl_sync(0xFFFFFFFFu, incl, 31);
    st.blocks = st.total < 1 ? 1 : st.total < max_blocks ? (int)st.total : max_blocks;
    const int c = blockIdx.x;
    st.begin = c < st.blocks ? block_begin(st.total, c, st.blocks) : st.total;
    st.end = c < st.blocks ? block_begin(st.total, c + 1, st.blocks) : st.total;
    // the lane in whose run the stretch begins walks its sequences
    long long at = incl - mine;
    const unsigned hit = __ballot_sync(0xFFFFFFFFu, st.begin >= at && st.begin < incl);
    st.b = -1;
    st.offset = 0;
    if (hit != 0) {
        const int owner = __ffs(hit) - 1;
        if (lane == owner) {
            for (int b = b0; b < b1; ++b) {
                const long long n = per == 1 ? mine : sch.head_cost(load_sequence(p, b)) * sch.heads;
                if (st.begin < at + n) {
                    st.b = b;
                    st.offset = st.begin - at;
                    break;
                }
                at += n;
            }
        }
        st.b = __shfl_sync(0xFFFFFFFFu, st.b, owner);
        st.offset = __shfl_sync(0xFFFFFFFFu, st.offset, owner);
    }
    return st;
}

// Walks the items of a block's stretch; every thread keeps its own copy.
template <int KT, int COST>
struct Walk {
    Schedule<KT, COST> sch;
    Item it;
    long long at, end;        // where the walk stands in the row, and the stretch's end
    int n_tiles;
    bool split;

    // The item's units in [at, end), which begins `rest` behind the item's begin: false when there are none.
    __device__ __forceinline__ bool cut(int rest) {
        it.units = sch.units(it.s, it.i);
        it.first = at - rest;
        it.t0 = max(rest - COST, 0);
        it.t1 = it.units;
        if (split) it.t1 = max((int)min((long long)it.units, end - it.first - COST), 0);
        return it.t1 > it.t0 && (split || rest == 0);
    }
    // split == false: items are not cut, an item belongs to the block in whose stretch it begins
    __device__ __forceinline__ bool begin(const PagedParams& p, const Schedule<KT, COST>& s, const Start& st, bool may_split) {
        sch = s;
        split = may_split;
        at = st.begin;
        end = st.end;
        if (st.b < 0 || at >= end) return false;
        it.b = st.b;
        it.s = load_sequence(p, it.b);
        n_tiles = sch.tiles(it.s);
        const long long per_head = sch.head_cost(it.s);
        it.h = st.offset < (1ll << 32) && per_head < (1ll << 32) ? (int)((unsigned)st.offset / (unsigned)per_head)
                                                               : (int)(st.offset / per_head);
        long long rest = st.offset - it.h * per_head;
        it.i = 0;
        for (;;) {
            const int n = sch.cost(it.s, it.i);
            if (rest < n) break;
            rest -= n;
            ++it.i;
        }
        return cut((int)rest) || next(p);
    }
    __device__ __forceinline__ bool next(const PagedParams& p) {
        do {
            at = it.first + it.units + COST;
            if (at >= end) return false;
            if (++it.i == n_tiles) {
                it.i = 0;
                if (++it.h == sch.heads) {
                    it.h = 0;
                    do {
                        if (++it.b >= p.batch) return false;  // cannot happen while at < end
                        it.s = load_sequence(p, it.b);
                        n_tiles = sch.tiles(it.s);
                    } while (n_tiles == 0);
                }
            }
        } while (!cut(0));
        return true;
    }
    // the block that has the item's last unit
    __device__ __forceinline__ int last_block(const Start& st) const {
        return block_of(st.total, it.first + COST + it.units - 1, st.blocks);
    }
};

// What the joining launch has to know of an item that starts in block c and ends in another (last < 0: there is none).
struct PartItem {
    int last;                 // the block that has the item's end
    int h;
    int first_row;            // of the item, among the (token, group head) rows of its sequence
    int rows;
    int first_token;          // of the sequence, in q
    int tile_rows;            // rows that each row tile of the item uses
    int pad[2];
};

// ---------------------------------------------------------------------------------------------------------------------
// int8 codes -> pairs of 16-bit floats, exactly.
//   bf16: with b the code's byte, 0x4300 | (b & 0x7F) stands for 128 + (b & 0x7F) and 0x4300 | (b & 0x80) for 128 or 256,
//         and their difference is the code (two's complement: low seven bits less 128 times the sign bit);
//   f16:  u = b ^ 0x80 = code + 128, 0x6400 | u stands for 1024 + u, less 1152.
// `which` picks bytes (0, 1) or (2, 3) of the word.
// ---------------------------------------------------------------------------------------------------------------------
template <bool BF, int which>
__device__ __forceinline__ uint32_t codes_to_pair(uint32_t w) {
    if constexpr (BF) {
        const uint32_t t = __byte_perm(w, 0x43434343u, which == 0 ? 0x4140 : 0x4342);
        const uint32_t a = t & 0xFF7FFF7Fu, s = t & 0xFF80FF80u;
        const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&s));
        return *reinterpret_cast<const uint32_t*>(&d);
    } else {
        const uint32_t t = __byte_perm(w ^ 0x80808080u, 0x64646464u, which == 0 ? 0x4140 : 0x4342);
        const uint32_t s = 0x64806480u;
        const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&t), *reinterpret_cast<const __half2*>(&s));
        return *reinterpret_cast<const uint32_t*>(&d);
    }
}

// A 4-bit cache's factor as it is used: rounded to bf16.  A code times it has at most 3 + 8 = 11 significant bits, which f16
// holds, so that the tensor cores can take the product as an exact operand.
__device__ __forceinline__ float factor4(float s) { return __bfloat162float(__float2bfloat16_rn(s)); }

// 4-bit codes as f16, without arithmetic: a nibble that is alone in the low byte of a 16-bit half is a subnormal number, 2^-24
// times the nibble (low nibble of the byte) or 2^-20 times (high nibble).  The code's sign bit is flipped on the way (`flip`), so
// the nibble stands for u = code + 8.  The bits to flip come as kernel parameters: a logic instruction takes one immediate, and
// of a mask and another constant the compiler makes two instructions (measured).
struct Flips {
    uint32_t low, high;
};
constexpr Flips kFlips{0x00080008u, 0x00800080u}, kHalfFlips{0x64086408u, 0x64806480u};    // the latter with the exponent of 1024
__device__ __forceinline__ uint32_t nibbles_low(uint32_t w, const Flips& f) {
    uint32_t d;
    asm("lop3.b32 %0, %1, 0x000F000F, %2, 0x6A;" : "=r"(d) : "r"(w), "r"(f.low));      // (w & mask) ^ flip
    return d;
}
__device__ __forceinline__ uint32_t nibbles_high(uint32_t w, const Flips& f) {
    uint32_t d;
    asm("lop3.b32 %0, %1, 0x00F000F0, %2, 0x6A;" : "=r"(d) : "r"(w), "r"(f.high));
    return d;
}

// 2^x by the hardware's approximation (2^-inf = 0)
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace
}  // namespace sasq
