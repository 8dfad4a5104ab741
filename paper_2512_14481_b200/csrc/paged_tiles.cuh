// Attention for many query rows per KV head (prompts, chunks): 256 rows an item, on the tensor cores (tcgen05).
#pragma once

#include "paged_rows.cuh"
#include "tcgen05.cuh"

namespace sasq {
namespace ptx {

__device__ __forceinline__ void tma_load_4d(uint32_t smem_dst, const CUtensorMap* m, uint64_t* bar, int x, int y, int z, int w) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(smem_dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t smem_dst, const CUtensorMap* m, uint64_t* bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]: 16-bit A, two elements per 32-bit column
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
        "}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_st_32x32(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
          "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]),
          "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]),
          "r"(v[30]), "r"(v[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
          "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Descriptor of an operand whose contraction index runs along the ROWS of the same 128-byte-swizzled tile (MN-major):
// 64 elements of the other index per 128-byte row, 8 rows per 1024-byte group (stride byte offset), the next 64 elements
// `lead` bytes further (leading byte offset).
__device__ __forceinline__ uint64_t smem_desc_mn_major_sw128(uint32_t smem_addr, uint32_t lead) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(lead >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
constexpr uint32_t kIdescBTransposed = 1u << 16;     // instruction descriptor: B is MN-major

}  // namespace ptx

namespace {

// An item is two row tiles, each the tokens whose heads fit 128 MMA rows: 128 / group tokens, so that a row tile is one
// box of q (of a group of five heads 125 rows are used).
constexpr int kTileKeys = 128;            // keys of a unit
// With a 4-bit cache bf16 queries meet K as f16: a warp for each row tile brings them there.
template <bool BF, int KIND>
constexpr bool kQueriesConverted = BF && KIND == SASQ_KV_INT4;
// Readers of the item queue: the softmax warps, the MMA lane, and whoever fetches K and V, and converts queries
template <bool BF, int KIND>
constexpr int kReaders = 8 + 1 + (KIND == SASQ_KV_16BIT ? 2 : 8) + (kQueriesConverted<BF, KIND> ? 2 : 0);
// Warps 0-3 and 4-7: softmax of either row tile; 8: MMA; 9: K and V; 10: Q and the items; 11: V's tails.  With an int8 or 4-bit cache
// warps 12-19 fetch and convert K and V, and 9 and 11 are idle, or convert the queries.
constexpr int kConvertThreads = 256;
template <int KIND>
constexpr int kTileThreads = KIND == SASQ_KV_16BIT ? 384 : 384 + kConvertThreads;
constexpr int kMmaWarp = 8, kLoadWarp = 9, kQueryWarp = 10, kTailWarp = 11, kConvertWarp = 12;
// Registers of a thread.  384 threads get 168 each, enough for every role.  640 get 96 at launch, of which the four-warp
// groups without a row of logits give some to the softmax: 2 x 128 + 64 + 2 x 80 = 5 x 96.  (The 4-bit cache converted by four warps, the
// softmax at 160 registers: 372 us instead of 353 for a chunk of 1024 tokens over 15000 keys.)
constexpr int kSoftmaxRegs = 128, kOtherRegs = 64, kConvertRegs = 80;

template <int D>
struct TileShape {
    static constexpr int kHalves = D / 64;                     // 128-byte columns of a tile
    static constexpr int kSlotBytes = kTileKeys * D * 2;
    static constexpr int kSlots = D == 128 ? 5 : 8;
    static constexpr int kQBytes = 128 * D * 2;                // of one row tile
};

// An item as its readers need it.
struct TileItem {
    int valid;                // 0: the block's work ends here
    int b, h, len;            // sequence, KV head, keys
    int before;               // keys before the first new token
    int first_token;          // of the sequence, in q
    int first_row, rows;      // of the item, and of its sequence: (token, head) pairs
    int limit;                // keys that its last row sees
    int t0, tiles;            // units of this block: the first, and how many
    int fold;                 // 0, or: the item has rows for one row tile only, and both work on them, the first on
                              // units t0 ... t0 + fold - 1 and the second on the others
    int begin[2], end[2];     // units of either row tile
    int whole;                // the block has all units of the item
    int last;                 // the block that has its last unit
};
constexpr int kItems = 4;     // items in the queue

// Unit i of an item in the order in which K and V are fetched.
__device__ __forceinline__ int unit_of(const TileItem& it, int i) {
    return it.fold == 0 ? it.t0 + i : it.t0 + (i >> 1) + (i & 1) * it.fold;
}

struct TileTail {
    TileItem items[kItems];
    uint64_t item_full[kItems], item_empty[kItems];
    uint64_t kv_full[8], kv_empty[8], raw_full[8];   // raw_full: a V tile whose last rows are still to be cleared
    uint64_t q_full[2], q_empty[2];
    uint64_t s_full[2], p_full[2][2], o_full[2];            // p_full: either half of the unit's keys
    uint64_t drain, meet[4];
    float2 other[128];        // reference and sum of the second row tile's rows, for the first
    uint64_t unit_empty[2];      // converted queries: the softmax warps have read row_exponent
    uint8_t row_exponent[2][128];    // of the power of two that a row was divided by, biased as a float's, of either row tile
    uint32_t tmem_base;
    volatile int abort_flag;
};

template <int D>
constexpr size_t kTileSmem = 1024 + 2 * (size_t)TileShape<D>::kQBytes + (size_t)TileShape<D>::kSlots * TileShape<D>::kSlotBytes + sizeof(TileTail);
static_assert(kTileSmem<128> <= 227 * 1024 && kTileSmem<64> <= 227 * 1024, "a block's shared memory");

// Bounded wait of one thread: false if the phase did not complete in time or another role gave up.
__device__ __forceinline__ bool tile_wait(uint64_t* bar, uint32_t parity, TileTail* tail, const AttendParams& p) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    int polls = 0;
    while (!ptx::mbar_try_wait(bar, parity)) {
        if (p.wait_limit <= 0 || (++polls & 63) == 0) {
            if (tail->abort_flag) return false;
            if (clock64() - t0 > p.wait_limit) {
                tail->abort_flag = 1;
                atomicMax(p.c.status, (int)SASQ_ERR_TIMEOUT);
                return false;
            }
        }
    }
    return true;
}

// units that beginning and ending an item costs (12 sequences of 1 to 300 new tokens over up to 2500 keys, 40 heads: 159.7 us
// with 0, 128.4 with 1, 124.7 with 2, 125.7 with 4, 130.0 with 6)
constexpr int kTileItemCost = 2;
using TileSchedule = Schedule<kTileKeys, kTileItemCost>;
using TileWalk = Walk<kTileKeys, kTileItemCost>;

// end of the units of an item, in this block, that row tile x takes part in (it.t0 or less: none)
__device__ __forceinline__ int tile_end(const TileSchedule& sch, const Item& it, int x) {
    const int half = sch.rows >> 1;
    const int rows = it.s.new_len * sch.group, first = it.i * sch.rows + half * x;
    if (first >= rows) return 0;
    const int lim = sch.causal ? it.s.len - it.s.new_len + (min(first + half, rows) - 1) / sch.group + 1 : it.s.len;
    return min(it.t1, (lim + kTileKeys - 1) / kTileKeys);
}

// A role's place in the queue of items that one warp walks for all; a whole warp, or one lane, holds a reader.
struct ItemReader {
    TileTail* tail;
    const AttendParams& p;
    int n;
    bool ok, more;
    // waits for item n; `more` says whether there is one
    template <bool WARP>
    __device__ __forceinline__ void fetch() {
        ok = tile_wait(&tail->item_full[n & (kItems - 1)], n / kItems & 1u, tail, p);
        if (WARP) ok = __all_sync(0xFFFFFFFFu, ok);
        more = ok && tail->items[n & (kItems - 1)].valid != 0;
    }
    __device__ __forceinline__ const TileItem& item() const { return tail->items[n & (kItems - 1)]; }
    // done with item n; one thread per reader arrives
    template <bool WARP>
    __device__ __forceinline__ void leave(bool arrives) {
        if (WARP) __syncwarp();
        if (arrives) ptx::mbar_arrive(&tail->item_empty[n & (kItems - 1)]);
        ++n;
    }
};

__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// 16 codes of a key as 16-bit floats into row r of a swizzled tile: two chunks of 8, of which lanes with `turn` store the
// second first.  V meets P in f16 whatever the queries' type is (five instructions for four codes, to bf16 eight).
template <bool BF>
__device__ __forceinline__ void store_codes(uint8_t* tile, int r, int chunk, int turn, const uint4& v) {
    uint8_t* const row = tile + r * 128;
    const uint2 lo = turn ? make_uint2(v.z, v.w) : make_uint2(v.x, v.y);
    const uint2 hi = turn ? make_uint2(v.x, v.y) : make_uint2(v.z, v.w);
    *reinterpret_cast<uint4*>(row + (((chunk + turn) ^ (r & 7)) << 4)) =
        make_uint4(codes_to_pair<BF, 0>(lo.x), codes_to_pair<BF, 1>(lo.x), codes_to_pair<BF, 0>(lo.y), codes_to_pair<BF, 1>(lo.y));
    *reinterpret_cast<uint4*>(row + (((chunk + (turn ^ 1)) ^ (r & 7)) << 4)) =
        make_uint4(codes_to_pair<BF, 0>(hi.x), codes_to_pair<BF, 1>(hi.x), codes_to_pair<BF, 0>(hi.y), codes_to_pair<BF, 1>(hi.y));
}

// A head's 4-bit key factors are divided by this power of two on their way to f16 (the largest becomes 2^11 ... 2^12, so that
// codes times factors fit, and are exact as long as a factor is no smaller than 2^-28 of it); from the bits of the largest.
__device__ __forceinline__ uint32_t head_unit(uint32_t largest) {
    return min(max(largest & 0x7F800000u, 13u << 23), 253u << 23) - (11u << 23);
}

// 32 4-bit codes of a key as f16 into row r of a swizzled tile: four chunks of 8, of which lanes with `turn` store the second two
// first.  K is multiplied by its factors (exact: 11 bits).  A chunk's channels lie as they come out of a word, 0 4 1 5 2 6 3 7: so do
// converted queries', and the result's until it is stored; queries that were copied meet keys in NATURAL order.
template <bool KEYS, bool NATURAL>
__device__ __forceinline__ void store_codes4(uint8_t* tile, int r, int chunk, int turn, const uint4& v, const Flips& flips,
                                             const __half2* factor) {
    uint8_t* const row = tile + r * 128;
    const uint32_t words[4] = {turn ? v.z : v.x, turn ? v.w : v.y, turn ? v.x : v.z, turn ? v.y : v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = words[i], y = w >> 8;
        // 1024 + u and 1024 + 16 u, u = code + 8: of channels (0, 4), (1, 5), (2, 6), (3, 7)
        uint32_t u[4];
        asm("lop3.b32 %0, %1, 0x000F000F, %2, 0x6A;" : "=r"(u[0]) : "r"(w), "r"(flips.low));
        asm("lop3.b32 %0, %1, 0x00F000F0, %2, 0x6A;" : "=r"(u[1]) : "r"(w), "r"(flips.high));
        asm("lop3.b32 %0, %1, 0x000F000F, %2, 0x6A;" : "=r"(u[2]) : "r"(y), "r"(flips.low));
        asm("lop3.b32 %0, %1, 0x00F000F0, %2, 0x6A;" : "=r"(u[3]) : "r"(y), "r"(flips.high));
        uint32_t c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t off = 0x64086408u, sixteenth = 0x2C002C00u, minus72 = 0xD480D480u;      // 1032, 1/16, -72
            __half2 x = *reinterpret_cast<const __half2*>(&u[e]);
            x = e & 1 ? __hfma2(x, *reinterpret_cast<const __half2*>(&sixteenth), *reinterpret_cast<const __half2*>(&minus72))
                      : __hsub2(x, *reinterpret_cast<const __half2*>(&off));
            if (KEYS) x = __hmul2(x, factor[4 * i + e]);
            c[e] = *reinterpret_cast<const uint32_t*>(&x);
        }
        *reinterpret_cast<uint4*>(row + (((chunk + (i ^ (turn << 1))) ^ (r & 7)) << 4)) =
            NATURAL ? make_uint4(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410), __byte_perm(c[0], c[1], 0x7632),
                                 __byte_perm(c[2], c[3], 0x7632))
                    : make_uint4(c[0], c[1], c[2], c[3]);
    }
}

// The warps that fill the ring from an int8 or 4-bit cache (`me` of kConvertThreads): K and V of each unit in turn, in the layout
// that the 16-bit copies leave: keys along the rows, 128-byte swizzle.  Keys behind the sequence's last are zeros.
// 4-bit, a chunk of 1024 tokens over 15000 keys, 32/8 heads of 128: f16 queries 294 us, bf16 ones 350 us, 744 TFLOP/s (int8 codes
// 304 us, a 16-bit cache 233 us).  Each of a KV head's 16 items converts the same codes again, beside a softmax at 128 registers a
// thread.  In the bf16 form neither the conversion of the codes nor their loads bound it (without either the time stays); what
// converted queries cost it has not been taken apart.
template <int D, bool BF, int KIND>
__device__ __forceinline__ void convert_tiles(const AttendParams& p, int me, uint8_t* ring, TileTail* tail) {
    using Shape = TileShape<D>;
    constexpr bool INT4 = KIND == SASQ_KV_INT4;
    constexpr int kWords = INT4 ? D / 32 : D / 16; // 16-byte words of a key's codes
    constexpr int kKeys = kConvertThreads / kWords;        // keys of a step
    constexpr int kSteps = kTileKeys / kKeys;
    const int word = me % kWords, first = me / kWords, lane = me & 31;
    const int page_mask = (1 << p.c.page_shift) - 1;
    // the word's two (4-bit: four) chunks of 8 elements; half a row's lanes store the second half first, which spreads them over
    // the banks
    uint8_t* const column = ring + (INT4 ? word >> 1 : word >> 2) * kTileKeys * 128;
    const int chunk = INT4 ? 4 * (word & 1) : 2 * (word & 3), turn = INT4 ? word >> 1 & 1 : word >> 2 & 1;
    // 4-bit: K's factors of the word's channels, (0, 4), (1, 5), (2, 6), (3, 7) of each eight, as store_codes4 wants them
    __half2 factor[INT4 ? 16 : 1];
    auto load_factors = [&](int h) {
        const float4* f4 = reinterpret_cast<const float4*>(p.c.k_scale + h * D + 32 * word);
        float f[32];
        uint32_t seen = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 v = __ldg(f4 + (i ^ turn << 2));          // in the order of the stores
            f[4 * i] = factor4(v.x), f[4 * i + 1] = factor4(v.y), f[4 * i + 2] = factor4(v.z), f[4 * i + 3] = factor4(v.w);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) seen = max(seen, __float_as_uint(f[i]) & 0x7FFFFFFFu);
#pragma unroll
        for (int o = 1; o < kWords; o <<= 1) seen = max(seen, __shfl_xor_sync(0xFFFFFFFFu, seen, o));
        const float down = 1.0f / __uint_as_float(head_unit(seen));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = 8 * (i >> 2) + (i & 3);
            factor[INT4 ? i : 0] = __floats2half2_rn(f[at] * down, f[at + 4] * down);
        }
    };
    ItemReader items{tail, p, 0, true, false};
    bool ok = true, more;
    TileItem it{};
    int i = 0, t = 0;
    const int* table = nullptr;
    auto next = [&] {                              // the next unit
        for (++i; i >= it.tiles; i = 0) {
            items.template fetch<true>();
            ok = ok && items.ok;
            more = items.more;
            if (!more) return;
            it = items.item();
            table = p.c.page_table + it.b * p.c.table_stride;
            items.template leave<true>(lane == 0);
            if (it.tiles > 0) {
                i = 0;
                break;
            }
        }
        t = unit_of(it, i);
    };
    // a lane looks up the page of 16 keys of the unit; the others ask it
    auto look_up = [&] {
        const int key = t * kTileKeys + 16 * (lane & 7);
        return more && key < it.len ? __ldg(table + (key >> p.c.page_shift)) : -1;
    };
    auto load = [&](const void* base, int entry, uint4 (&v)[kSteps]) {
        auto bytes = [](long long elements) { return INT4 ? elements >> 1 : elements; };
        const char* head = static_cast<const char*>(base) + bytes(it.h * p.c.head_stride) + word * 16;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int key = t * kTileKeys + i * kKeys + first;
            const int page = __shfl_sync(0xFFFFFFFFu, entry, (i * kKeys + first) >> 4);
            const bool in = key < it.len && page >= 0 && page < p.c.num_pages;
            v[i] = in ? ldg_stream16(head + bytes(page * p.c.page_stride + (key & page_mask) * p.c.token_stride)) : make_uint4(0, 0, 0, 0);
        }
    };
    int slot = 0;
    uint32_t phase = 0;
    auto store = [&](const uint4 (&v)[kSteps], bool values) {
        ok = ok && tile_wait(&tail->kv_empty[slot], phase ^ 1u, tail, p);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) return;
        uint8_t* const tile = column + (size_t)slot * Shape::kSlotBytes;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if constexpr (INT4) {
                if (values) store_codes4<false, false>(tile, i * kKeys + first, chunk, turn, v[i], p.half_flips, factor);
                else store_codes4<true, !kQueriesConverted<BF, KIND>>(tile, i * kKeys + first, chunk, turn, v[i], p.half_flips, factor);
            } else if (values) store_codes<false>(tile, i * kKeys + first, chunk, turn, v[i]);
            else store_codes<BF>(tile, i * kKeys + first, chunk, turn, v[i]);
        }
        ptx::fence_proxy_async_smem();
        ptx::mbar_arrive(&tail->kv_full[slot]);
        if (++slot == Shape::kSlots) { slot = 0; phase ^= 1u; }
    };
    // The next unit's keys travel while this one's values are converted, its values while its keys are; its page
    // entries come half a unit earlier.
    uint4 k[kSteps], v[kSteps];
    next();
    int entry = look_up();
    if (more) load(p.c.k, entry, k);
    int head = more ? it.h : 0;                    // whose factors are in place
    if (INT4 && more) load_factors(head);
    while (more && ok) {
        if (t * kTileKeys + 16 * (lane & 7) < it.len && (entry < 0 || entry >= p.c.num_pages))
            atomicMax(p.c.status, (int)SASQ_ERR_BAD_INDEX);
        load(p.c.v, entry, v);
        next();
        entry = look_up();
        store(k, false);
        if (more) load(p.c.k, entry, k);
        if (INT4 && more && it.h != head) load_factors(head = it.h);
        if (ok) store(v, true);
    }
}

// The warp that brings the bf16 queries of row tile x to shared memory as f16, channels in the order of K's, each row divided by a
// power of two (its largest becomes 2^14 ... 2^15: exact as long as an element is no smaller than 2^-31 of it).
template <int D>
__device__ __forceinline__ void convert_queries(const AttendParams& p, int x, uint8_t* q_tile, TileTail* tail) {
    constexpr int kLanes = D / 8, kRows = 32 / kLanes, kAhead = 8;           // lanes of a row, rows of a step, steps under way
    const int lane = threadIdx.x & 31, word = lane % kLanes, sub = lane / kLanes;
    const int tokens = 128 / p.group;
    uint8_t* const column = q_tile + (word >> 3) * 128 * 128;
    ItemReader items{tail, p, 0, true, false};
    bool ok = true;
    for (uint32_t filled = 0; ok; items.template leave<true>(lane == 0)) {
        items.template fetch<true>();
        ok = items.ok;
        if (!items.more) break;
        const TileItem& it = items.item();
        if (it.end[x] == it.begin[x]) continue;
        ok = tile_wait(&tail->q_empty[x], (filled & 1u) ^ 1u, tail, p) && tile_wait(&tail->unit_empty[x], (filled & 1u) ^ 1u, tail, p);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) continue;
        const int token0 = it.first_token + it.first_row / p.group + (it.fold != 0 ? 0 : x * tokens);
        // the rows behind the sequence's last stay as they are: they move no row's reference, and nothing of them is stored
        const int rows = min(tokens * p.group, it.rows - it.first_row - (it.fold != 0 ? 0 : x * tokens * p.group));
        auto fetch = [&](int r) {
            const int t = r / p.group;
            return r < rows && token0 + t < p.c.total_q
                       ? *reinterpret_cast<const uint4*>(p.q + (long long)(token0 + t) * p.q_stride + (long long)(it.h * p.group + r - t * p.group) * D + 8 * word)
                       : make_uint4(0, 0, 0, 0);
        };
        for (int first = sub; first - sub < rows; first += kRows * kAhead) {
            uint4 v[kAhead];
#pragma unroll
            for (int e = 0; e < kAhead; ++e) v[e] = fetch(first + kRows * e);
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                const uint32_t w[4] = {v[e].x, v[e].y, v[e].z, v[e].w};
                uint32_t seen = 0, h[4];                                      // NaN compares as the largest
#pragma unroll
                for (int i = 0; i < 4; ++i) seen = max(seen, max((w[i] << 16) & 0x7FFF0000u, w[i] & 0x7FFF0000u));
#pragma unroll
                for (int o = 1; o < kLanes; o <<= 1) seen = max(seen, __shfl_xor_sync(0xFFFFFFFFu, seen, o));
                const uint32_t top = min(max(seen & 0x7F800000u, 15u << 23), 253u << 23);
                const float up = __uint_as_float((268u << 23) - top);         // 2^14 over the power of two at or below the largest
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = widen2<true>(w[i]);
                    h[i] = narrow2<false>(f.x * up, f.y * up);
                }
                const int r = first + kRows * e;
                if (r < rows) {
                    *reinterpret_cast<uint4*>(column + r * 128 + (((word & 7) ^ (r & 7)) << 4)) =
                        make_uint4(__byte_perm(h[0], h[2], 0x5410), __byte_perm(h[0], h[2], 0x7632), __byte_perm(h[1], h[3], 0x5410),
                                   __byte_perm(h[1], h[3], 0x7632));
                    if (word == 0) tail->row_exponent[x][r] = (uint8_t)((top >> 23) - 14u);
                }
            }
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&tail->q_full[x]);
        ++filled;
    }
}

template <int KIND, bool MORE, int N>
__device__ __forceinline__ void registers_to() {
    if constexpr (KIND != SASQ_KV_16BIT) {
        if constexpr (MORE) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
    }
}

// Two row tiles x = 0, 1 share every K and V tile.  Per unit and row tile:
//   S = Q K^T       (MMA, both operands in shared memory, S in TMEM)
//   P = 2^(scale S - m), row sums, P back to TMEM over S as 16-bit pairs     (one thread per row, 4 warps per row tile)
//   O += P V        (MMA, P in TMEM, V in shared memory with the keys along its rows, O in TMEM)
// While the softmax warps of one row tile work, the MMAs of the other run.  S of the next unit is asked for right behind
// the PV that frees it, across items too: the next item's queries are fetched as soon as the last QK has read the old
// ones, so that its first S is there when the softmax warps have stored the old item's rows.
// Bound by that alternation: 256 rows x 128 keys take 2050 clocks of MMAs and 2048 of exponentials, and a step takes about
// 3500 (8192 causal tokens, 32 heads of 128, bf16: 511 us, 1076 TFLOP/s in short bursts; 619 us, 888 TFLOP/s, one call after
// another under the power cap, at 1.4 to 1.65 GHz).
template <int D, bool BF, int KIND>
__global__ void __launch_bounds__(kTileThreads<KIND>, 1)
paged_tiles_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttendParams p) {
    using Shape = TileShape<D>;
    constexpr bool INT8 = KIND == SASQ_KV_INT8, INT4 = KIND == SASQ_KV_INT4, kCodes = KIND != SASQ_KV_16BIT;
    constexpr bool kConvertsQ = kQueriesConverted<BF, KIND>;
    constexpr bool PBF = BF && !kCodes, SBF = BF && !INT4;     // the second and the first product's type; else f16
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* q_smem = smem;
    uint8_t* ring = smem + 2 * Shape::kQBytes;
    TileTail* tail = reinterpret_cast<TileTail*>(ring + (size_t)Shape::kSlots * Shape::kSlotBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int s = 0; s < Shape::kSlots; ++s) {
            ptx::mbar_init(&tail->kv_full[s], kCodes ? kConvertThreads : 1);
            ptx::mbar_init(&tail->kv_empty[s], 1);
            ptx::mbar_init(&tail->raw_full[s], 1);
        }
        for (int x = 0; x < 2; ++x) {
            ptx::mbar_init(&tail->q_full[x], 1);
            ptx::mbar_init(&tail->q_empty[x], 1);
            if constexpr (kConvertsQ) ptx::mbar_init(&tail->unit_empty[x], 4);      // (elsewhere it costs: 16-bit mixed batch 128.5 us against 125.5)
            ptx::mbar_init(&tail->s_full[x], 1);
            ptx::mbar_init(&tail->p_full[x][0], 128);
            ptx::mbar_init(&tail->p_full[x][1], 128);
            ptx::mbar_init(&tail->o_full[x], 1);
        }
        ptx::mbar_init(&tail->drain, 1);
        for (int i = 0; i < 4; ++i) ptx::mbar_init(&tail->meet[i], 64);
        for (int i = 0; i < kItems; ++i) {
            ptx::mbar_init(&tail->item_full[i], 1);
            ptx::mbar_init(&tail->item_empty[i], kReaders<BF, KIND>);
        }
        tail->abort_flag = 0;
        ptx::mbar_init_fence();
        ptx::prefetch_tensormap(&map_q);
        if constexpr (!kCodes) {
            ptx::prefetch_tensormap(&map_k);
            ptx::prefetch_tensormap(&map_v);
        }
    }
    if (warp == kMmaWarp) {
        ptx::tmem_alloc(&tail->tmem_base, 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = tail->tmem_base;
    pdl_launch_dependents();
    pdl_wait();

    const TileSchedule sch{p.item_rows, p.group, p.causal, p.c.kv_heads};
    if (tid == 0) p.part_items[blockIdx.x].last = -1;
    bool ok = true;
    // whole warps wait together: a role goes on, or gives up, as a warp
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        ok = ok && tile_wait(bar, parity, tail, p);
        ok = __all_sync(0xFFFFFFFFu, ok);
        return ok;
    };

    if (warp == kLoadWarp) {
        registers_to<KIND, false, kOtherRegs>();
        if constexpr (kConvertsQ) convert_queries<D>(p, 0, q_smem, tail);
        // ---------------- K and V of each unit, in turn, a lane per page ----------------
        int slot = 0;
        uint32_t phase = 0;
        const int box = min(1 << p.c.page_shift, kTileKeys);
        const int boxes = kTileKeys / box;
        const int page_mask = (1 << p.c.page_shift) - 1;
        ItemReader items{tail, p, 0, true, false};
        for (; !kCodes && ok; items.template leave<true>(lane == 0)) {
            items.template fetch<true>();
            ok = items.ok;
            if (!items.more) break;
            const TileItem it = items.item();
            // a unit's page entries are asked for while the unit before waits for its slots
            const int* table = p.c.page_table + it.b * p.c.table_stride;
            auto look_up = [&](int i) {
                const int key = unit_of(it, i) * kTileKeys + lane * box;
                return i < it.tiles && lane < boxes && key < it.len ? __ldg(table + (key >> p.c.page_shift)) : -1;
            };
            int next_entry = look_up(0);
            for (int i = 0; i < it.tiles && ok; ++i) {
                const int t = unit_of(it, i);
                const int key = t * kTileKeys + lane * box;
                const int entry = next_entry;
                next_entry = look_up(i + 1);
                int page = (int)p.c.num_pages;                  // outside the cache: the copy fills in zeros
                if (lane < boxes && key < it.len) {
                    if (entry < 0 || entry >= p.c.num_pages) atomicMax(p.c.status, (int)SASQ_ERR_BAD_INDEX);
                    else page = entry;
                }
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    if (!wait(&tail->kv_empty[slot], phase ^ 1u)) break;
                    // a V tile that ends behind the sequence's last key goes to the warp that clears its tail first
                    uint64_t* full = kv == 1 && it.len - t * kTileKeys < kTileKeys ? &tail->raw_full[slot] : &tail->kv_full[slot];
                    if (lane == 0) ptx::mbar_arrive_expect_tx(full, Shape::kSlotBytes);
                    __syncwarp();
                    if (lane < boxes) {
                        const uint32_t dst = ptx::smem_u32(ring) + slot * Shape::kSlotBytes + lane * box * 128;
#pragma unroll
                        for (int half = 0; half < Shape::kHalves; ++half)
                            ptx::tma_load_4d(dst + half * kTileKeys * 128, kv == 0 ? &map_k : &map_v, full, half * 64, key & page_mask, it.h,
                                             page);
                    }
                    __syncwarp();
                    if (++slot == Shape::kSlots) { slot = 0; phase ^= 1u; }
                }
            }
        }
        // Copies still in flight must land before the block's shared memory goes away: at once, unless a role gave up.
        // (A tile with a tail to clear may then never be announced; the limit is far above a copy's flight.)
        if (lane == 0 && !kCodes) {
            for (int s = 0; s < Shape::kSlots; ++s) {
                const long long t0 = clock64();
                const uint32_t par = s < slot ? phase : (phase ^ 1u);
                while (!ptx::mbar_try_wait(&tail->kv_full[s], par))
                    if (clock64() - t0 > (1LL << 24)) break;
            }
        }
        __syncwarp();
    } else if (warp == kQueryWarp) {
        registers_to<KIND, false, kOtherRegs>();
        // ---------------- the block's items, for everyone, and their Q ----------------
        uint32_t filled[2] = {0, 0};                            // times that each row tile's queries were asked for
        const int tokens = 128 / p.group;
        const Start st = find_start(p.c, sch, p.max_blocks);
        TileWalk walk;
        int n = 0;
        for (bool more = walk.begin(p.c, sch, st, p.split != 0);; more = walk.next(p.c), ++n) {
            const int at = n & (kItems - 1);
            if (!wait(&tail->item_empty[at], (n / kItems & 1u) ^ 1u)) break;
            const Item& w = walk.it;
            TileItem it;
            it.valid = more;
            if (more) {
                if (INT8 && lane == 0 && (scale_is_bad(__ldg(p.c.k_scale + w.h)) || scale_is_bad(__ldg(p.c.v_scale + w.h))))
                    atomicMax(p.c.status, (int)SASQ_ERR_BAD_SCALE);
                if (INT4)
                    for (int d = lane; d < D; d += 32)
                        if (scale_is_bad(factor4(__ldg(p.c.k_scale + w.h * D + d))) || scale_is_bad(factor4(__ldg(p.c.v_scale + w.h * D + d))))
                            atomicMax(p.c.status, (int)SASQ_ERR_BAD_SCALE);
                it.b = w.b;
                it.h = w.h;
                it.len = w.s.len;
                it.before = w.s.len - w.s.new_len;
                it.first_token = w.s.first;
                it.first_row = w.i * sch.rows;
                it.rows = w.s.new_len * p.group;
                it.limit = sch.key_limit(w.s, w.i);
                it.t0 = w.t0;
                it.begin[0] = it.begin[1] = w.t0;
                it.end[0] = max(w.t0, tile_end(sch, w, 0));
                it.end[1] = max(w.t0, tile_end(sch, w, 1));
                it.tiles = max(it.end[0], it.end[1]) - w.t0;
                it.fold = it.first_row + (sch.rows >> 1) >= it.rows && it.tiles > 1 ? (it.tiles + 1) >> 1 : 0;
                if (it.fold != 0) {
                    it.begin[1] = w.t0 + it.fold;
                    it.end[1] = it.end[0];
                    it.end[0] = it.begin[1];
                }
                it.whole = w.t0 == 0 && w.t1 == w.units;
                it.last = walk.last_block(st);
            }
            if (lane == 0) {
                tail->items[at] = it;
                ptx::mbar_arrive(&tail->item_full[at]);
            }
            __syncwarp();
            if (!more) break;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (kConvertsQ || !ok || it.end[x] == it.begin[x]) continue;
                if (!wait(&tail->q_empty[x], (filled[x] & 1u) ^ 1u)) continue;
                ++filled[x];
                if (lane == 0) {
                    ptx::mbar_arrive_expect_tx(&tail->q_full[x], (uint32_t)(tokens * p.group * D * 2));
#pragma unroll
                    for (int half = 0; half < Shape::kHalves; ++half)
                        ptx::tma_load_3d(ptx::smem_u32(q_smem) + x * Shape::kQBytes + half * 128 * 128, &map_q, &tail->q_full[x], half * 64,
                                         it.h * p.group, it.first_token + it.first_row / p.group + (it.fold != 0 ? 0 : x * tokens));
                }
                __syncwarp();
            }
            if (!ok) break;
        }
        if (lane == 0) {
            for (int x = 0; x < 2; ++x) {
                const long long t0 = clock64();
                while (filled[x] != 0 && !ptx::mbar_try_wait(&tail->q_full[x], (filled[x] & 1u) ^ 1u))
                    if (clock64() - t0 > (1LL << 24)) break;
            }
        }
        __syncwarp();
    } else if (warp == kMmaWarp) {
        registers_to<KIND, false, kOtherRegs>();
        // ---------------- MMAs, all by one lane (which lets the descriptors live in uniform registers) ----------------
        if (ptx::elect_one()) {
            constexpr uint32_t idesc_s = ptx::idesc_f16(128, kTileKeys, SBF);
            constexpr uint32_t idesc_o = ptx::idesc_f16(128, D, PBF) | ptx::kIdescBTransposed;
            uint32_t q_phase = 0, p_phase = 0;                        // a bit per row tile
            const uint64_t q_desc = ptx::smem_desc_k_major_sw128(ptx::smem_u32(q_smem));
            const uint64_t k_desc = ptx::smem_desc_k_major_sw128(ptx::smem_u32(ring));
            const uint64_t v_desc = ptx::smem_desc_mn_major_sw128(ptx::smem_u32(ring), kTileKeys * 128);
            // Steps: a unit for both row tiles, or (fold) a unit for each.  K and V tiles pass through the ring in the order
            // of the units, K before V; `at` is the step's first tile among all of the block's.
            struct Step {
                int j, n[2], steps, fold;
                uint32_t at;
                bool more;
            };
            ItemReader items{tail, p, 0, true, false};
            auto enter = [&](Step& u) {
                for (;;) {
                    items.template fetch<false>();
                    ok = ok && items.ok;
                    u.more = items.more;
                    if (!u.more) return;
                    const TileItem& it = items.item();
                    u.j = 0;
                    u.n[0] = it.end[0] - it.begin[0];
                    u.n[1] = it.end[1] - it.begin[1];
                    u.steps = max(u.n[0], u.n[1]);
                    u.fold = it.fold != 0;
                    items.template leave<false>(true);
                    if (u.steps > 0) return;
                }
            };
            auto arrived = [&](uint32_t tile) {
                ok = ok && tile_wait(&tail->kv_full[tile % Shape::kSlots], tile / Shape::kSlots & 1u, tail, p);
                return ok;
            };
            auto free_slot = [&](uint32_t tile) { ptx::mma_commit(&tail->kv_empty[tile % Shape::kSlots]); };
            // S of row tile x for step u
            auto qk = [&](const Step& u, int x) {
                const uint32_t tile = u.at + (u.fold ? 2 * x : 0);
                if (u.j == 0) {
                    ok = ok && tile_wait(&tail->q_full[x], q_phase >> x & 1u, tail, p);
                    if (!ok) return;
                    q_phase ^= 1u << x;
                    ptx::tc_fence_after_sync();
                }
                const uint64_t a = q_desc + (uint64_t)(x * (Shape::kQBytes >> 4));
                const uint64_t b = k_desc + (uint64_t)(tile % Shape::kSlots * (Shape::kSlotBytes >> 4));
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint64_t at = (uint64_t)(((k >> 2) * 128 * 128 + (k & 3) * 32) >> 4);
                    ptx::mma_f16_ss(tmem + x * 128, a + at, b + at, idesc_s, k != 0);
                }
                ptx::mma_commit(&tail->s_full[x]);
                if (u.j + 1 == u.n[x]) ptx::mma_commit(&tail->q_empty[x]);
                if (u.fold) free_slot(tile);
            };
            Step u;
            u.at = 0;
            enter(u);
            if (u.more) {
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (u.j < u.n[x] && arrived(u.at + (u.fold ? 2 * x : 0))) {
                        ptx::tc_fence_after_sync();
                        qk(u, x);
                    }
                if (!u.fold) free_slot(u.at);
            }
            while (u.more && ok) {
                const Step now = u;
                u.at += now.fold && now.j < now.n[1] ? 4 : 2;
                if (++u.j == u.steps) enter(u);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    // the tiles that this row tile needs (the second row tile's are the first's, unless folded), before P: then
                    // nothing stands between PV and the next QK
                    const bool k_next = u.more && u.j < u.n[x];
                    if (now.j < now.n[x] && (x == 0 || now.fold || now.j >= now.n[0])) arrived(now.at + (now.fold ? 2 * x : 0) + 1);
                    if (k_next && (x == 0 || u.fold || u.j >= u.n[0])) arrived(u.at + (u.fold ? 2 * x : 0));
                    if (!ok) break;
                    ptx::tc_fence_after_sync();
                    if (now.j < now.n[x]) {
                        const uint32_t tile = now.at + (now.fold ? 2 * x : 0) + 1;
                        // the first half's keys are multiplied while the softmax warps work on the second's
                        const uint64_t b = v_desc + (uint64_t)(tile % Shape::kSlots * (Shape::kSlotBytes >> 4));
#pragma unroll
                        for (int part = 0; part < 2; ++part) {
                            ok = ok && tile_wait(&tail->p_full[x][part], p_phase >> x & 1u, tail, p);
                            if (!ok) break;
                            ptx::tc_fence_after_sync();
#pragma unroll
                            for (int k = 4 * part; k < 4 * part + 4; ++k)
                                ptx::mma_f16_ts(tmem + 256 + x * D, tmem + x * 128 + 8 * k, b + (uint64_t)(k * 2048 >> 4), idesc_o,
                                                now.j != 0 || k != 0);
                        }
                        p_phase ^= 1u << x;
                        ptx::mma_commit(&tail->o_full[x]);
                        if (now.fold) free_slot(tile);
                    }
                    if (k_next && ok) qk(u, x);
                }
                if (!now.fold) free_slot(now.at + 1);
                if (u.more && !u.fold) free_slot(u.at);
            }
            // MMAs still running must end before shared memory and TMEM go away
            ptx::mma_commit(&tail->drain);
            const long long t0 = clock64();
            while (!ptx::mbar_try_wait(&tail->drain, 0))
                if (clock64() - t0 > (1LL << 24)) break;
        }
        __syncwarp();
    } else if (warp == kTailWarp) {
        registers_to<KIND, false, kOtherRegs>();
        if constexpr (kConvertsQ) convert_queries<D>(p, 1, q_smem + Shape::kQBytes, tail);
        // ---------------- rows of V behind a sequence's last key ----------------
        // Whatever they hold is multiplied by P = 0, and must be finite.  The copy of such a tile is announced here, and
        // the MMAs learn of it when the rows are zero.
        int slot = 1;                                               // of the unit's V: slots go K, V, K, V, ...
        uint32_t phases = 0;                                        // a bit per slot
        ItemReader items{tail, p, 0, true, false};
        for (; !kCodes && ok; items.template leave<true>(lane == 0)) {
            items.template fetch<true>();
            ok = items.ok;
            if (!items.more) break;
            const TileItem it = items.item();
            for (int i = 0; i < it.tiles; ++i) {
                const int t = unit_of(it, i);
                const int valid = it.len - t * kTileKeys;
                if (valid < kTileKeys) {
                    if (!wait(&tail->raw_full[slot], phases >> slot & 1u)) break;
                    phases ^= 1u << slot;
                    uint8_t* v = ring + (size_t)slot * Shape::kSlotBytes + valid * 128;
                    for (int y = lane; y < (kTileKeys - valid) * 8; y += 32)
#pragma unroll
                        for (int half = 0; half < Shape::kHalves; ++half)
                            *reinterpret_cast<uint4*>(v + half * kTileKeys * 128 + y * 16) = make_uint4(0, 0, 0, 0);
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&tail->kv_full[slot]);
                }
                slot = (slot + 2) % Shape::kSlots;
            }
        }
    } else if (kCodes && warp >= kConvertWarp) {
        // ---------------- int8 or 4-bit cache: K and V of each unit, converted on the way to shared memory ----------------
        // 16 codes a thread and step; the next tile's codes travel while this one's are converted.
        registers_to<KIND, false, kConvertRegs>();
        if constexpr (kCodes) convert_tiles<D, BF, KIND>(p, tid - 32 * kConvertWarp, ring, tail);
    } else {
        registers_to<KIND, true, kSoftmaxRegs>();
        // ---------------- softmax: row tile x, one row per thread ----------------
        const int x = warp >> 2, quad = warp & 3;
        const int half = sch.rows >> 1;
        const int row = quad * 32 + lane;                          // of the row tile
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const uint32_t s_addr = tmem + lane_base + x * 128, o_addr = tmem + lane_base + 256 + x * D;
        uint32_t s_phase = 0;                                      // parity of the unit whose S is waited for
        // the two row tiles' warps that share lanes of TMEM meet where they work on the same rows
        uint32_t meet_phase = 0;
        auto meet = [&] {
            ptx::tc_fence_before_sync();
            ptx::mbar_arrive(&tail->meet[quad]);
            if (!wait(&tail->meet[quad], meet_phase)) return false;
            meet_phase ^= 1u;
            ptx::tc_fence_after_sync();
            return true;
        };
        uint32_t q_fills = 0;                                      // converted queries: times that this row tile's came
        ItemReader items{tail, p, 0, true, false};
        for (; ok; items.template leave<true>(lane == 0)) {
            items.template fetch<true>();
            ok = items.ok;
            if (!items.more) break;
            const TileItem& it = items.item();
            const bool fold = it.fold != 0;
            const int t0 = it.begin[x], t_end = it.end[x];
            const bool any = t0 < t_end;                           // this row tile sees keys of this block's units
            const int item_row = it.first_row + (fold ? 0 : x * half) + row;      // among the sequence's rows
            const bool valid = row < half && item_row < it.rows;
            int row_limit = it.limit;
            if (p.causal && valid) row_limit = it.before + item_row / p.group + 1;
            float signed_scale = INT8 ? p.scale * __ldg(p.c.k_scale + it.h) : p.scale;
            if constexpr (INT4) {                                  // what K's factors, and the row's queries, were divided by
                uint32_t largest = 0;
#pragma unroll
                for (int d = lane; d < D; d += 32) largest = max(largest, __float_as_uint(factor4(__ldg(p.c.k_scale + it.h * D + d))) & 0x7FFFFFFFu);
                float unit = __uint_as_float(head_unit(__reduce_max_sync(0xFFFFFFFFu, largest)));
                if (kConvertsQ && any) {
                    if (!wait(&tail->q_full[x], q_fills & 1u)) break;
                    unit *= __uint_as_float((uint32_t)tail->row_exponent[x][row] << 23);
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&tail->unit_empty[x]);
                    ++q_fills;
                }
                signed_scale *= unit;                              // (one by one a far scale and unit may leave a subnormal number)
            }
            // A scale of zero, or one that vanished in the product with the factor, would turn masked logits, -inf, into NaN; the
            // smallest number there is gives the same equal weights.
            const float scale = signed_scale == 0.0f ? __uint_as_float(1u) : fabsf(signed_scale);
            const uint32_t flip = signed_scale < 0.0f ? 0x80000000u : 0u;    // maxima are then of the negated logits
            float m = -INFINITY;                                   // reference, in powers of two
            uint64_t sum2 = 0;                                     // two partial sums of P
            for (int t = t0; t < t_end; ++t) {
                if (!wait(&tail->s_full[x], s_phase)) break;
                s_phase ^= 1u;
                ptx::tc_fence_after_sync();
                const int seen = row_limit - t * kTileKeys;
                const bool cut = __any_sync(0xFFFFFFFFu, seen < kTileKeys);
                // The row is read in halves, the second one twice: for its maximum before the first half, and for its
                // exponentials behind it.  128 logits and what is made of them do not fit a thread's registers.  With the
                // int8 (and the 4-bit) cache the three steps share their code: the converting warps need the instruction cache too
                // (measured on a 1024-token chunk over 15000 keys: int8 350 -> 323 us, 16-bit 227 -> 246 us).
                constexpr int kSteps = kCodes ? 1 : 3;
                float most = -INFINITY;
#pragma unroll kSteps
                for (int step = 0; step < 3; ++step) {
                    const int part = step == 1 ? 0 : 1;
                    uint32_t s[2][32];
                    ptx::tmem_ld_32x32(s_addr + part * 64, s[0]);
                    ptx::tmem_ld_32x32(s_addr + part * 64 + 32, s[1]);
                    ptx::tmem_ld_wait();
                    if (flip != 0) {
#pragma unroll
                        for (int e = 0; e < 64; ++e) s[e >> 5][e & 31] ^= 0x80000000u;
                    }
                    if (cut) {
                        const int left = seen - part * 64;
#pragma unroll
                        for (int e = 0; e < 64; ++e)
                            if (e >= left) s[e >> 5][e & 31] = 0xFF800000u;      // -inf
                    }
                    if (step < 2) {
                        float top[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t* w = s[c >> 1] + 16 * (c & 1);
                            top[c] = fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
#pragma unroll
                            for (int e = 2; e < 16; e += 2) top[c] = max3(top[c], __uint_as_float(w[e]), __uint_as_float(w[e + 1]));
                        }
                        most = fmaxf(most, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
                    }
                    if (step == 0) continue;
                    if (step == 1) {
                        most *= scale;
                        // rows that no query owns hold what shared memory held, or others' queries: they have no vote
                        if (__any_sync(0xFFFFFFFFu, valid && most > m + (kRescaleAt + kHeadroom<!PBF>))) {
                            const float m_new = fmaxf(m, most - kHeadroom<!PBF>);
                            const float f = m_new == -INFINITY ? 1.0f : exp2_approx(m - m_new);
                            m = m_new;
                            const float2 old = unpack2(sum2);
                            sum2 = pack2(old.x * f, old.y * f);
                            if (t > t0) {     // S(t) was asked for behind the second product of t - 1, which is done as well
#pragma unroll 1
                                for (int c = 0; c < D; c += 16) {
                                    uint32_t o[16];
                                    ptx::tmem_ld_32x16(o_addr + c, o);
                                    ptx::tmem_ld_wait();
#pragma unroll
                                    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                    ptx::tmem_st_32x16(o_addr + c, o);
                                }
                            }
                        }
                    }
                    const float ref = m == -INFINITY ? 0.0f : m;
                    const uint64_t scale2 = pack2(scale, scale), ref2 = pack2(-ref, -ref);
                    uint32_t pk[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const float2 z = unpack2(fma2(pack2(__uint_as_float(s[e >> 4][2 * e & 31]), __uint_as_float(s[e >> 4][(2 * e & 31) + 1])),
                                                      scale2, ref2));
                        const float p0 = exp2_approx(z.x), p1 = exp2_approx(z.y);
                        sum2 = add2(sum2, pack2(p0, p1));
                        pk[e] = narrow2<PBF>(p0, p1);
                    }
                    ptx::tmem_st_32x32(s_addr + part * 32, pk);
                    ptx::tmem_st_wait();
                    ptx::tc_fence_before_sync();
                    ptx::mbar_arrive(&tail->p_full[x][part]);
                }
            }
            if (!ok) break;
            // ---- the item's rows
            if (any) {
                if (!wait(&tail->o_full[x], s_phase ^ 1u)) break;
                ptx::tc_fence_after_sync();
            }
            const float2 sums = unpack2(sum2);
            float sum = sums.x + sums.y;
            float f0 = 1.0f, f1 = 0.0f;                            // weights of the two row tiles' O
            if (fold) {
                if (x == 1) tail->other[row] = make_float2(m, sum);
                if (!meet()) break;                                // both O are complete
                if (x == 1) {
                    if (!meet()) break;                            // and have been read
                    continue;
                }
                const float2 o = tail->other[row];
                const float m_new = fmaxf(m, o.x), ref = m_new == -INFINITY ? 0.0f : m_new;
                f0 = exp2_approx(m - ref);
                f1 = exp2_approx(o.x - ref);
                m = m_new;
                sum = sum * f0 + o.y * f1;
            }
            const bool whole = it.whole;
            const float inv = sum != 0.0f ? (INT8 ? __ldg(p.c.v_scale + it.h) : 1.0f) / sum : 0.0f;
            const float times = INT4 ? 1.0f : inv;                 // (4-bit: already taken)
            const int tok = item_row / p.group;
            const int head = it.h * p.group + item_row - tok * p.group;
            const long long token = it.first_token + tok;
            const long long part_row = (long long)(2 * blockIdx.x + (it.t0 == 0 ? 1 : 0)) * 256 + x * 128 + row;
            // A thread stores its own row in 16-byte pieces.  Turning 4 x 4 pieces among four lanes first, so that a store
            // covers 64 bytes of a row, cost more instructions (cold in the caches, once an item) than it saved stores:
            // 47.5 against 43.9 us for seven-token drafts of 16 sequences.
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                uint32_t o[32];
                if (any) {
                    ptx::tmem_ld_32x32(o_addr + c, o);
                    ptx::tmem_ld_wait();
                    if (fold) {
                        uint32_t o1[32];
                        ptx::tmem_ld_32x32(o_addr + D + c, o1);
                        ptx::tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            o[e] = __float_as_uint(__uint_as_float(o[e]) * f0 + __uint_as_float(o1[e]) * f1);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = 0;
                }
                if constexpr (INT4) {                              // channels in their order; a whole item's averages meet V's factors
                    const float4* f4 = reinterpret_cast<const float4*>(p.c.v_scale + it.h * D + c);
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        const float4 a = __ldg(f4 + e / 4), b = __ldg(f4 + e / 4 + 1);
                        const float f[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                        uint32_t v[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            v[k] = o[e + (k & 3) * 2 + (k >> 2)];
                            if (whole) v[k] = __float_as_uint(__uint_as_float(v[k]) * inv * factor4(f[k]));
                        }
#pragma unroll
                        for (int k = 0; k < 8; ++k) o[e + k] = v[k];
                    }
                }
                if (valid && whole) {
                    uint4* dst = reinterpret_cast<uint4*>(p.out + token * p.out_stride + (long long)head * D + c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            w[k] = sum != 0.0f ? narrow2<BF>(__uint_as_float(o[8 * e + 2 * k]) * times, __uint_as_float(o[8 * e + 2 * k + 1]) * times) : 0u;
                        dst[e] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                } else if (valid) {
                    uint4* dst = reinterpret_cast<uint4*>(p.part_o + part_row * D + c);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dst[e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                }
            }
            if (valid && whole && p.lse != nullptr)
                p.lse[token * p.heads + head] = sum != 0.0f ? (m + log2f(sum)) * 0.6931471805599453f : -INFINITY;
            if (valid && !whole) p.part_ml[part_row] = make_float2(m, sum);
            if (!whole && it.t0 == 0 && tid == 0) {
                PartItem pi;
                pi.last = it.last;
                pi.h = it.h;
                pi.first_row = it.first_row;
                pi.rows = min(sch.rows, it.rows - it.first_row);
                pi.first_token = it.first_token;
                pi.tile_rows = half;
                p.part_items[blockIdx.x] = pi;
            }
            ptx::tc_fence_before_sync();                           // O has been read: the next item's first PV may overwrite it
            if (fold && !meet()) break;
        }
    }

    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, 512);
    }
}

}  // namespace
}  // namespace sasq
