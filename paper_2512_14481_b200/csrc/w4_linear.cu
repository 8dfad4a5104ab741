// Linear layers with 4-bit weights and group factors for few tokens, and the quantizer that makes such weights.
//
//   y[t, n] = narrow( sum_g s[n, g] * sum_{k in group g} x[t, k] c[n, k]  (+ bias[n]) )
//
// Bound by the weights: half a byte each, read once.  The products run on mma.sync with 16 rows of weights on its wide side and
// the tokens on the other, so that a weight goes from its byte to the operand in registers, where its group's factor can be
// applied to the group's sum.  More than 16 tokens go to the tensor cores' fifth generation instead (w4_batch.cuh).
//
// Replayed from a graph, weights out of DRAM, bf16, groups of 128: one token of 4096 x 4096 5.1 us (floor 1.3: launch, two round
// trips to memory, the meeting of the sums), of 22016 x 4096 10.2 us (4.6 TB/s, 71 % of a plain copy's rate); 7 tokens of 11008 x
// 4096 12.0 us, 16 of 4096 x 4096 11.0 us; 7 of 5120 x 13824, groups of 64, 18.5 us (from 3 tokens on the codes' conversion and
// the tokens' way to shared memory count).
#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "tcgen05.cuh"

namespace sasq {
namespace {

struct W4Params {
    const uint16_t* x;          // [T, K]
    const uint8_t* w;           // [N, K / 2]
    const uint16_t* ws;         // [N, K / G]
    const uint16_t* bias;       // [N] or nullptr
    uint16_t* y;                // [T, N]
    int T, N, K, groups;
    int x_rows;                 // tokens of a block at most
    int split, split_log;       // blocks of a cluster (1, 2, 4 or 8), each with a share of the columns' windows
    // Cluster c has tiles_each row tiles from c * tiles_each on, and one more if c < tiles_more; so have a cluster's blocks
    // windows.  (Divisions cost a warp hundreds of instructions before its first load: the host makes them.)
    int tiles_each, tiles_more, windows_each, windows_more;
    int pass_tiles;             // tiles whose sums a block holds at once
    int parts, part_windows;    // a block's windows are taken in parts whose tokens fit shared memory
    int sc_whole;               // a row's factors are whole windows
    int* status;                // of waits that ran out, and their limit in clocks
    long long wait_limit;
};

// 16 bytes from global to shared memory without a register
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds4(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}

// (a & mask) ^ c
template <uint32_t MASK>
__device__ __forceinline__ uint32_t and_xor(uint32_t a, uint32_t c) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(d) : "r"(a), "n"(MASK), "r"(c));
    return d;
}

// Exponent and flipped sign of a low and a high nibble, for codes8.  They come as kernel parameters: a logic instruction takes
// one immediate, and of a mask and a constant the compiler makes two instructions (measured).
struct Bits {
    uint32_t low, high;
};
template <bool BF>
constexpr Bits kBits = BF ? Bits{0x43084308u, 0x43084308u} : Bits{0x64086408u, 0x64806480u};

// Eight codes of a word as 16-bit floats, by the exponent that makes a nibble the low bits of a mantissa (a known way of weight-only
// kernels; the numbers follow from the formats): pairs (0, 4), (2, 6) in lo and (1, 5), (3, 7) in hi.  With the sign bit flipped a nibble
// is u = code + 8.  bf16: 128 + u, less 136.  f16: 1024 + u, less 1032; one nibble further up 1024 + 16 u, which a fused
// multiply-add brings to the code.  5 instructions of the logic pipe, which runs at half the others' rate, for f16, 7 for bf16.
template <bool BF>
__device__ __forceinline__ void codes8(uint32_t w, const Bits& bits, uint32_t (&lo)[2], uint32_t (&hi)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        lo[i] = and_xor<0x000F000Fu>(w >> (8 * i), bits.low);
        if constexpr (BF) {
            hi[i] = and_xor<0x000F000Fu>(w >> (8 * i + 4), bits.low);
            const __nv_bfloat162 bias = __halves2bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308));
            const __nv_bfloat162 a = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&lo[i]), bias);
            const __nv_bfloat162 b = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&hi[i]), bias);
            lo[i] = *reinterpret_cast<const uint32_t*>(&a);
            hi[i] = *reinterpret_cast<const uint32_t*>(&b);
        } else {
            hi[i] = and_xor<0x00F000F0u>(w >> (8 * i), bits.high);
            const uint32_t off = 0x64086408u, sixteenth = 0x2C002C00u, minus72 = 0xD480D480u;
            const __half2 a = __hsub2(*reinterpret_cast<const __half2*>(&lo[i]), *reinterpret_cast<const __half2*>(&off));
            const __half2 b = __hfma2(*reinterpret_cast<const __half2*>(&hi[i]), *reinterpret_cast<const __half2*>(&sixteenth),
                                      *reinterpret_cast<const __half2*>(&minus72));
            lo[i] = *reinterpret_cast<const uint32_t*>(&a);
            hi[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
    }
}

// d = a b + c (FIRST) or d += a b, in 16-bit floats and in signed bytes
template <bool BF, bool FIRST>
__device__ __forceinline__ void mma_float(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (FIRST) d[0] = d[1] = d[2] = d[3] = 0.0f;
    if constexpr (BF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
constexpr uint32_t kMagic = 0x4B400000u;                   // 1.5 * 2^23
constexpr uint32_t kSumStart = kMagic - (22u << 23);       // 1.5 * 2: sums of digits count in 2^-22
template <bool FIRST>
__device__ __forceinline__ void mma_s8(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (FIRST)
        asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "r"(kSumStart));
    else
        asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A lane's N weight words of one row and window from their slot: word s * (G / 32) + i is its i-th of group s.  Chunk c of 16
// bytes of a row lies at c ^ turn.
template <int G, int N>
__device__ __forceinline__ void window_words(uint32_t row_base, int turn, int j, uint32_t (&w)[N]) {
    if constexpr (G == 128) {
#pragma unroll
        for (int s = 0; s < N / 4; ++s) {
            const uint4 v = lds16(row_base + (((4 * s + j) ^ turn) << 4));
            w[4 * s] = v.x;
            w[4 * s + 1] = v.y;
            w[4 * s + 2] = v.z;
            w[4 * s + 3] = v.w;
        }
    } else if constexpr (G == 64) {
#pragma unroll
        for (int s = 0; s < N / 2; ++s) {
            const uint2 v = lds8(row_base + (((2 * s + (j >> 1)) ^ turn) << 4) + 8 * (j & 1));
            w[2 * s] = v.x;
            w[2 * s + 1] = v.y;
        }
    } else {
#pragma unroll
        for (int s = 0; s < N; ++s) w[s] = lds4(row_base + ((s ^ turn) << 4) + 4 * j);
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Two ways to the products.
//
// DIGITS (one or two tokens): as 16-bit floats 8 codes cost 5 to 7 instructions of the logic pipe and 4 others.  As signed bytes, 16
// times the code, they are a shift and two masks, and one s8 product of m16n8k32 takes twice as many of them.  So x becomes
// integers: in a window of 256 columns a token's values are multiples of a power of two, 2^-21 of that at or below the window's
// largest, whose digits to the base 256, from -128 to 127, are three columns of the product: digit l of token t is column 2 l + t.  A group's
// sums are exact integers of at most 2^21; they start at the bits of the float 1.5 * 2, so that the float they end as is that plus
// the sum times 2^-22.
// FLOATS (up to 16 tokens): exact products of 16-bit floats in fp32 sums, 32 rows at a time, so that what is read
// of x from shared memory serves twice.
//
// TOKENS: 2 for digits; 8 or 16.
// ---------------------------------------------------------------------------------------------------------------------
template <int TOKENS, int STAGES, int G>
struct W4Shape {
    static constexpr bool kDigits = TOKENS == 2;
    // Floats' sums and operands take 128 registers: 16 warps of one block share the tokens that two blocks of 8 would each bring
    // (12 tokens of 11008 x 4096: 14.3 us against 16.0).
    static constexpr int kWarps = kDigits ? 8 : 16, kThreads = 32 * kWarps;
    static constexpr int kPerSm = kWarps <= 8 ? 2 : 1;     // blocks of an SM by their registers
    static constexpr int kRows = kDigits ? 16 : 32;        // of a tile
    static constexpr int kWindow = kDigits ? 256 : 128;    // columns of a step
    static constexpr int kRowBytes = kWindow / 2;
    static constexpr int kSlot = kRows * kRowBytes;        // a window of a tile: 2 KB
    static constexpr int kRing = kWarps * STAGES * kSlot;
    static constexpr int kTiles = kDigits ? 1 : TOKENS / 8;        // 8-column blocks of the product
    static constexpr int kTable = kDigits ? 32 : 0;        // bytes of a window's units, one for each column
    static constexpr int kTokenBytes = kDigits ? 3 * 256 : 256;    // of a token's window
    static constexpr int kPiece = kRows + 4;               // floats of a piece's token: neighbouring ones lie in different banks
    static size_t x_bytes(int tokens, int windows) { return (size_t)windows * (tokens * kTokenBytes + kTable); }
    // The sums of whole tiles, the piece of a tile that a warp's run begins with, and whose pieces there are; the piece that a
    // run ends with takes the place of its ring.
    static size_t sum_bytes(int tokens, int tiles) { return ((size_t)tokens * (kRows * tiles + 4 + kWarps * kPiece) + 2 * kWarps) * sizeof(float); }
    static_assert(TOKENS * kPiece * sizeof(float) <= (size_t)STAGES * kSlot, "a piece fits a warp's ring");
};

// A block has some row tiles and (in a cluster) a share of the columns' windows.  The windows of all its tiles, laid end to end,
// are cut into equal runs, one for each warp: a warp walks on through a tile's windows, and its sums change hands only where a
// tile or its run ends.  The tokens lie in shared memory, and each warp streams its weights through a ring of its own
// (STAGES - 1 windows under way): no barrier until the sums of all the block's rows meet.
template <int TOKENS, int STAGES, bool BF, int G>
__global__ void __launch_bounds__(W4Shape<TOKENS, STAGES, G>::kThreads, W4Shape<TOKENS, STAGES, G>::kPerSm) w4_linear_kernel(const __grid_constant__ W4Params p, const __grid_constant__ Bits bits_) {
    using Shape = W4Shape<TOKENS, STAGES, G>;
    constexpr bool kDigits = Shape::kDigits;
    constexpr int kWindow = Shape::kWindow, kRows = Shape::kRows, kRowBytes = Shape::kRowBytes;
    constexpr int GW = kWindow / G, WG = G / 32;           // groups of a window, words of a lane in a group
    constexpr int NT = Shape::kTiles, MT = kRows / 16, WK = Shape::kWarps;
    constexpr uint32_t kSlot = Shape::kSlot;
    extern __shared__ __align__(128) uint8_t smem[];
    const Bits bits = bits_;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, j = lane & 3;
    const int rank = p.split > 1 ? (int)ptx::cluster_ctarank() : 0;
    const int cluster = blockIdx.x >> p.split_log;
    const int tokens = p.T;
    const int tile_begin = cluster * p.tiles_each + min(cluster, p.tiles_more), tile_end = tile_begin + p.tiles_each + (cluster < p.tiles_more);
    const int begin = rank * p.windows_each + min(rank, p.windows_more), end = begin + p.windows_each + (rank < p.windows_more);
    const int half_k = p.K >> 1;                           // bytes of a weight row
    const int sum_pitch = kRows * p.pass_tiles + 4;        // floats: neighbouring tokens lie in different banks
    const uint32_t ring = ptx::smem_u32(smem) + warp * STAGES * kSlot;
    float* const sums = reinterpret_cast<float*>(smem + Shape::kRing);
    float* const pieces = sums + p.x_rows * sum_pitch;     // [warp][token] of Shape::kPiece: the first ones
    int* const piece_tile = reinterpret_cast<int*>(pieces + WK * p.x_rows * Shape::kPiece);
    // warp w's first or last piece
    auto piece_of = [&](int w, int last) {
        return last ? reinterpret_cast<float*>(smem + (size_t)w * STAGES * kSlot) : pieces + w * p.x_rows * Shape::kPiece;
    };
    const uint32_t table = ptx::smem_u32(piece_tile + 2 * WK);                 // digits: a window's units, [8]
    const uint32_t x_base = table + p.part_windows * Shape::kTable;            // [window][digit][token], or [window][token], of 256 bytes
    const uint32_t x_window = p.x_rows * Shape::kTokenBytes;
    pdl_launch_dependents();

    // A warp's run: `left` windows from window `at` of tile `tile` on, of `windows` that a tile has in the part from `first`.
    struct Run {
        int tile, at, left, windows, first;
    };
    auto run_of = [&](int pass, int part) {
        Run r;
        r.first = begin + part * p.part_windows;
        r.windows = max(min(p.part_windows, end - r.first), 0);
        const unsigned all = (unsigned)(min(p.pass_tiles, tile_end - pass) * r.windows);   // (what fits shared memory: below 2^20)
        const unsigned u = all * warp / WK;
        r.left = (int)(all * (warp + 1) / WK - u);
        r.tile = r.windows > 0 ? (int)(u / (unsigned)r.windows) : 0;
        r.at = (int)u - r.tile * r.windows;
        r.tile += pass;
        return r;
    };

    // Copies of weights.  Whatever the group, the rows that a warp reads together lie in different banks.
    auto turn = [](int row) { return kDigits ? (row & 1) << 2 | (row & 2) | (row >> 2 & 1) : row >> 1 & 3; };
    constexpr int kChunks = kRowBytes / 16, kStep = 32 / kChunks;              // a copy takes kStep rows, four copies a slot
    const int w_row = lane / kChunks, w_chunk = lane % kChunks;
    uint32_t w_place[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) w_place[r] = (w_row + kStep * r) * kRowBytes + ((w_chunk ^ turn(w_row + kStep * r)) << 4);
    Run ld = run_of(tile_begin, 0);
    uint32_t load_at = ring, load_row[4] = {0, 0, 0, 0};
    const uint8_t* load_w = p.w;
    auto enter_load = [&] {
        const int first = ld.tile * kRows;
        load_w = p.w + (long long)first * half_k;
        // rows behind the last are read from the last one's place: their products are not stored
#pragma unroll
        for (int r = 0; r < 4; ++r) load_row[r] = (uint32_t)min(w_row + kStep * r, p.N - 1 - first) * (uint32_t)half_k;
    };
    auto load = [&] {
        if (ld.left > 0) {
            // columns behind the last are read from the last one's place, and meet zeros
            const uint8_t* src = load_w + min((ld.first + ld.at) * kRowBytes + 16 * w_chunk, half_k - 16);
#pragma unroll
            for (int r = 0; r < 4; ++r) copy16(load_at + w_place[r], src + load_row[r]);
            load_at = load_at + kSlot == ring + STAGES * kSlot ? ring : load_at + kSlot;
            if (++ld.at == ld.windows) {
                ld.at = 0;
                ++ld.tile;
                if (ld.left > 1) enter_load();
            }
            --ld.left;
        }
        copies_end_group();
    };
    auto load_first = [&] {
        if (ld.left > 0) enter_load();
#pragma unroll 1
        for (int s = 0; s < STAGES - 1; ++s) load();
    };
    // weights may be read at once, tokens when the kernels before this one are done
    load_first();
    pdl_wait();

    // The tokens of a part.  A lane has eight columns, chunk c of a window: group s, lane jj, word ii.
    auto stage_x = [&](int part) {
        constexpr int kLanes = kWindow / 8, kPairs = 32 / kLanes;              // lanes of a (window, token), those of a warp
        const int from = begin + part * p.part_windows, windows = min(from + p.part_windows, end) - from;
        const int c = lane % kLanes, s = c / (G / 8), jj = c % (G / 8) / WG, q = s * WG + c % WG;
        struct Pair {
            int w, t;
        };
        const int hop_w = WK * kPairs / tokens, hop_t = WK * kPairs - hop_w * tokens;      // from a warp's pairs to its next
        auto hop = [&](Pair& a) {
            a.w += hop_w;
            if ((a.t += hop_t) >= tokens) {
                a.t -= tokens;
                ++a.w;
            }
        };
        auto fetch = [&](const Pair& a) {
            const int col = (from + a.w) * kWindow + 8 * c;
            return a.w < windows && col < p.K ? *reinterpret_cast<const uint4*>(p.x + (long long)a.t * p.K + col) : make_uint4(0, 0, 0, 0);
        };
        constexpr int kAhead = kDigits ? 2 : 4;            // loads that travel while one is taken apart
        Pair now, ahead;
        now.w = (warp * kPairs + lane / kLanes) / tokens;
        now.t = warp * kPairs + lane / kLanes - now.w * tokens;
        ahead = now;
        uint4 next[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            next[e] = fetch(ahead);
            hop(ahead);
        }
        // (a register under way can't be moved without waiting for it: the loads take turns with theirs)
        bool more = true;
#pragma unroll 1
        while (more) {
#pragma unroll
            for (int turn_of = 0; turn_of < kAhead; ++turn_of) {
                more = __any_sync(0xFFFFFFFFu, now.w < windows);
                if (!more) break;
                const uint32_t raw[4] = {next[turn_of].x, next[turn_of].y, next[turn_of].z, next[turn_of].w};
                const int w = now.w, t = now.t;
                hop(now);
                next[turn_of] = fetch(ahead);
                hop(ahead);
                if constexpr (kDigits) {
                    // Words 2q and 2q + 1 of lanes jj = 0 ... 3 lie side by side, and every other column of the product has
                    // neighbouring pairs the other way round, in other banks.
                    float f[8];
                    uint32_t seen = 0;                         // NaN compares as the largest
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 a = widen2<BF>(raw[e]);
                        f[2 * e] = a.x;
                        f[2 * e + 1] = a.y;
                        seen = max(seen, max(__float_as_uint(a.x) & 0x7FFFFFFFu, __float_as_uint(a.y) & 0x7FFFFFFFu));
                    }
                    seen = __reduce_max_sync(0xFFFFFFFFu, seen);
                    // the largest becomes 2^21 ... 2^22
                    const uint32_t top = max(seen & 0x7F800000u, 26u << 23);
                    const float up = __uint_as_float((275u << 23) - top);
                    uint32_t d[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        d[e] = __float_as_uint(fmaf(f[e], up, __uint_as_float(kMagic))) - kMagic + 0x00808080u;
                    auto gather = [](uint32_t a, uint32_t b, uint32_t c4, uint32_t d4, uint32_t (&to)[3]) {
                        const uint32_t ab = __byte_perm(a, b, 0x5140), cd = __byte_perm(c4, d4, 0x5140);
                        to[0] = __byte_perm(ab, cd, 0x5410) ^ 0x80808080u;
                        to[1] = __byte_perm(ab, cd, 0x7632) ^ 0x80808080u;
                        to[2] = __byte_perm(__byte_perm(a, b, 0x0062), __byte_perm(c4, d4, 0x0062), 0x5410) ^ 0x80808080u;
                    };
                    uint32_t even[3], odd[3];                  // digits of columns 0, 2, 4, 6 and of 1, 3, 5, 7
                    gather(d[0], d[2], d[4], d[6], even);
                    gather(d[1], d[3], d[5], d[7], odd);
                    const uint32_t place = (q >> 1) * 64 + jj * 16 + (q & 1) * 8;
#pragma unroll
                    for (int l = 0; l < 3; ++l) {
                        const int row = l * p.x_rows + t;
                        const uint32_t to = x_base + w * x_window + row * 256 + (place ^ ((row & 1) << 6));
                        asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(to), "r"(even[l]), "r"(odd[l]) : "memory");
                    }
                    // What the lowest digit stands for, less 16 times the code, times the 2^22 that sums of digits lack; a window with
                    // infinities or NaN: NaN; columns that stand for nothing (others' digits): 0
                    const float unit = seen >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __uint_as_float(top - (3u << 23));
                    const int l = lane >> 1, tt = lane & 1;
                    if (lane < 8 && (tt == t || (tt >= tokens && t == 0)))
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(table + w * Shape::kTable + lane * 4), "f"(l < 3 && tt == t ? unit : 0.0f) : "memory");
                } else if (w < windows) {
                    // the pairs that come out of a word together: (0, 4), (2, 6), (1, 5), (3, 7).  Every other token has
                    // neighbouring words the other way round, in other banks.
                    const uint32_t to = x_base + w * x_window + t * 256 + ((q * 64 + jj * 16) ^ ((t & 1) << 6));
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(__byte_perm(raw[0], raw[2], 0x5410)),
                                 "r"(__byte_perm(raw[1], raw[3], 0x5410)), "r"(__byte_perm(raw[0], raw[2], 0x7632)),
                                 "r"(__byte_perm(raw[1], raw[3], 0x7632)) : "memory");
                }
            }
        }
    };

    // where this lane's columns of the product lie in a window, by the parity of the word or pair of words
    uint32_t x_near[NT], x_far[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int row = kDigits ? min(g >> 1, 2) * p.x_rows + min(g & 1, tokens - 1) : min(8 * nt + g, tokens - 1);
        x_near[nt] = x_base + row * 256 + 16 * j + (row & 1) * 64;
        x_far[nt] = x_base + row * 256 + 16 * j + 64 - (row & 1) * 64;
    }
    auto store = [&](int pass, int t, int row, float v) {
        const int n_row = kRows * pass + row;
        if (n_row >= p.N) return;
        if (p.bias != nullptr) v += widen1<BF>(p.bias[n_row]);
        p.y[(long long)t * p.N + n_row] = narrow1<BF>(v);
    };
    uint32_t at = ring;                                    // the slot that is read next
    for (int pass = tile_begin; pass < tile_end; pass += p.pass_tiles) {
        const int rows = kRows * min(p.pass_tiles, tile_end - pass);
        // every token and row once among the threads of `of` blocks; with many tokens a warp takes 32 rows of one at a time
        auto each_row = [&](int block, int of, auto&& f) {
            if constexpr (kDigits) {
                for (int t = 0; t < tokens; ++t)
                    for (int row = block * Shape::kThreads + tid; row < rows; row += of * Shape::kThreads) f(t, row);
            } else {
                for (int t = 0, row = 32 * (block * WK + warp) + lane;; row += 32 * WK * of) {
                    for (; row - lane >= rows && t < tokens; ++t) row -= rows;
                    if (t >= tokens) break;
                    f(t, row);
                }
            }
        };
        for (int part = 0; part < p.parts; ++part) {
            Run r = run_of(pass, part);
            const int windows = r.windows;
            // factors of the next window, as they are stored: pairs (or one)
            constexpr int kPacked = GW / 2 > 0 ? GW / 2 : 1;
            uint32_t next_sc[2 * MT][kPacked];
            const uint16_t* sc_tile = p.ws;
            uint32_t sc_row[2 * MT];
            auto load_sc = [&](int window) {
                const int first = (r.first + window) * GW;
#pragma unroll
                for (int e = 0; e < 2 * MT; ++e) {
                    const uint16_t* src = sc_tile + sc_row[e];
                    if constexpr (GW == 1) {
                        next_sc[e][0] = __ldg(src + first);
                    } else if (p.sc_whole) {               // a window's factors are one aligned word
                        if constexpr (GW == 2) {
                            next_sc[e][0] = __ldg(reinterpret_cast<const uint32_t*>(src + first));
                        } else if constexpr (GW == 4) {
                            const uint2 v = __ldg(reinterpret_cast<const uint2*>(src + first));
                            next_sc[e][0] = v.x;
                            next_sc[e][1] = v.y;
                        } else {
                            const uint4 v = __ldg(reinterpret_cast<const uint4*>(src + first));
                            next_sc[e][0] = v.x;
                            next_sc[e][1] = v.y;
                            next_sc[e][kPacked > 2 ? 2 : 0] = v.z;
                            next_sc[e][kPacked > 3 ? 3 : 0] = v.w;
                        }
                    } else {
#pragma unroll
                        for (int s = 0; s < GW / 2; ++s)
                            next_sc[e][s] = __ldg(src + min(first + 2 * s, p.groups - 1)) | (uint32_t)__ldg(src + min(first + 2 * s + 1, p.groups - 1)) << 16;
                    }
                }
            };
            auto enter_sc = [&](int tile, int window) {
                const int first = tile * kRows;
                sc_tile = p.ws + (long long)first * p.groups;
#pragma unroll
                for (int e = 0; e < 2 * MT; ++e) sc_row[e] = (uint32_t)min(8 * e + g, p.N - 1 - first) * (uint32_t)p.groups;
                load_sc(window);
            };
            if (r.left > 0) enter_sc(r.tile, r.at);
            __syncthreads();                               // the part before has been read
            if (part > 0 || pass > tile_begin) {
                ld = r;
                load_first();
            }
            if (lane < 2) piece_tile[2 * warp + lane] = -1;
            if (p.parts > 1 || pass == tile_begin) stage_x(part);
            __syncthreads();
            while (r.left > 0) {
                const int steps = min(r.left, r.windows - r.at);
                r.left -= steps;
                float tot[MT][NT][4];
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) tot[m][nt][0] = tot[m][nt][1] = tot[m][nt][2] = tot[m][nt][3] = 0.0f;
                uint32_t x_at = r.at * x_window, table_at = table + r.at * Shape::kTable + 8 * j;
#pragma unroll 1
                for (int n = 0; n < steps; ++n) {
                    float sc[2 * MT][GW];
#pragma unroll
                    for (int e = 0; e < 2 * MT; ++e) {
                        if constexpr (GW == 1) {
                            sc[e][0] = widen1<BF>((uint16_t)next_sc[e][0]);
                        } else {
#pragma unroll
                            for (int s = 0; s < GW / 2; ++s) {
                                const float2 v = widen2<BF>(next_sc[e][s]);
                                sc[e][2 * s] = v.x;
                                sc[e][2 * s + 1] = v.y;
                            }
                        }
                    }
                    if (n + 1 < steps) load_sc(r.at + n + 1);
                    else if (r.left > 0) enter_sc(r.tile + 1, 0);
                    copies_wait<STAGES - 2>();
                    __syncwarp();
                    load();
                    constexpr int kWords = kWindow / 32;
                    uint32_t wv[2 * MT][kWords];
#pragma unroll
                    for (int e = 0; e < 2 * MT; ++e) window_words<G>(at + (8 * e + g) * kRowBytes, turn(8 * e + g), j, wv[e]);
                    at = at + kSlot == ring + STAGES * kSlot ? ring : at + kSlot;
                    if constexpr (kDigits) {
                        // Nothing on the way passes fp32's end: a window's sums are below 2^22 2^-22 times its largest factor, a unit
                        // is at most 2^124, and digit j's power of 256 comes behind all windows.  (A sum times a factor below 2^-104
                        // may be a subnormal number, off by 2^-150.)
                        float win[4];
                        int acc[4];
#pragma unroll
                        for (int h = 0; h < 4; ++h) {      // two words of a lane
                            const uint4 b = lds16((h & 1 ? x_far[0] : x_near[0]) + x_at + (h >> 1) * 128);
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const int q = 2 * h + i, s = q / WG;
                                const uint32_t a[4] = {wv[0][q] << 4 & 0xF0F0F0F0u, wv[1][q] << 4 & 0xF0F0F0F0u, wv[0][q] & 0xF0F0F0F0u,
                                                       wv[1][q] & 0xF0F0F0F0u};
                                if (q % WG == 0) mma_s8<true>(acc, a, i == 0 ? b.x : b.z, i == 0 ? b.y : b.w);
                                else mma_s8<false>(acc, a, i == 0 ? b.x : b.z, i == 0 ? b.y : b.w);
                                if (q % WG == WG - 1) {
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const float v = __int_as_float(acc[e]) - __uint_as_float(kSumStart);
                                        win[e] = s == 0 ? v * sc[e >> 1][s] : fmaf(v, sc[e >> 1][s], win[e]);
                                    }
                                }
                            }
                        }
                        const uint2 f = lds8(table_at);
#pragma unroll
                        for (int e = 0; e < 4; ++e) tot[0][0][e] = fmaf(win[e], __uint_as_float(e & 1 ? f.y : f.x), tot[0][0][e]);
                        table_at += Shape::kTable;
                    } else {
                        float acc[MT][NT][4];
#pragma unroll
                        for (int q = 0; q < kWords; ++q) {
                            uint32_t lo[MT][4], hi[MT][4];
#pragma unroll
                            for (int m = 0; m < MT; ++m) {
                                uint32_t l0[2], l1[2], h0[2], h1[2];
                                codes8<BF>(wv[2 * m][q], bits, l0, h0);
                                codes8<BF>(wv[2 * m + 1][q], bits, l1, h1);
                                lo[m][0] = l0[0], lo[m][1] = l1[0], lo[m][2] = l0[1], lo[m][3] = l1[1];
                                hi[m][0] = h0[0], hi[m][1] = h1[0], hi[m][2] = h0[1], hi[m][3] = h1[1];
                            }
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                const uint4 b = lds16((q & 1 ? x_far[nt] : x_near[nt]) + x_at + (q >> 1) * 128);
#pragma unroll
                                for (int m = 0; m < MT; ++m) {
                                    if (q % WG == 0) mma_float<BF, true>(acc[m][nt], lo[m], b.x, b.y);
                                    else mma_float<BF, false>(acc[m][nt], lo[m], b.x, b.y);
                                    mma_float<BF, false>(acc[m][nt], hi[m], b.z, b.w);
                                    if (q % WG == WG - 1) {
#pragma unroll
                                        for (int e = 0; e < 4; ++e)
                                            tot[m][nt][e] = fmaf(acc[m][nt][e], sc[2 * m + (e >> 1)][q / WG], tot[m][nt][e]);
                                    }
                                }
                            }
                        }
                    }
                    x_at += x_window;
                }
                if constexpr (kDigits) {                   // the digits' columns meet, among the four lanes of a row
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        tot[0][0][e] *= __uint_as_float((127u + 8u * j) << 23);
                        tot[0][0][e] += __shfl_xor_sync(0xFFFFFFFFu, tot[0][0][e], 1);
                        tot[0][0][e] += __shfl_xor_sync(0xFFFFFFFFu, tot[0][0][e], 2);
                    }
                }
                const bool whole = steps == windows, last = r.left == 0;           // else the end of a tile, or its beginning or middle
                if (!whole && last) {
                    copies_wait<0>();
                    __syncwarp();
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int t = 8 * nt + 2 * j + e;
                        if (t < tokens) {
                            float* const to = whole ? sums + t * sum_pitch + kRows * (r.tile - pass) + g : piece_of(warp, last) + t * Shape::kPiece + g;
#pragma unroll
                            for (int m = 0; m < MT; ++m)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    float* const cell = to + 16 * m + 8 * h;
                                    *cell = whole && part > 0 ? *cell + tot[m][nt][e + 2 * h] : tot[m][nt][e + 2 * h];
                                }
                        }
                    }
                if (!whole && lane == 0) piece_tile[2 * warp + last] = r.tile - pass;
                r.at = 0;
                ++r.tile;
            }
            // the pieces of tiles meet, in the warps' order; behind the last part the tiles go out, or to the cluster
            __syncthreads();
            int tile_of[2 * WK];
#pragma unroll
            for (int k = 0; k < 2 * WK; ++k) tile_of[k] = piece_tile[k];
            const bool out = p.split == 1 && part + 1 == p.parts;
            each_row(0, 1, [&](int t, int row) {
                float* const cell = sums + t * sum_pitch + row;
                const int mine = t * Shape::kPiece + row % kRows;
                float v = 0.0f;
                bool cut = windows == 0;
#pragma unroll
                for (int k = 0; k < 2 * WK; ++k)
                    if (tile_of[k] == row / kRows) {
                        v += piece_of(k >> 1, k & 1)[mine];
                        cut = true;
                    }
                if (!cut) v = *cell;
                else if (part > 0) v += *cell;
                if (out) store(pass, t, row, v);
                else if (cut) *cell = v;
            });
        }
        if (p.split > 1) {
            ptx::cluster_sync_all();
            each_row(rank, p.split, [&](int t, int row) {
                const uint32_t here = ptx::smem_u32(&sums[t * sum_pitch + row]);
                float v = 0.0f;
                for (int k = 0; k < p.split; ++k) {
                    uint32_t peer;
                    float part;
                    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer) : "r"(here), "r"(k));
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part) : "r"(peer));
                    v += part;
                }
                store(pass, t, row, v);
            });
            ptx::cluster_sync_all();                       // nobody goes on, or leaves, while its sums are being read
        }
    }
}

// A warp per group: its largest magnitude, the factor as the linear uses it, the codes.
template <bool BF, int G>
__global__ void __launch_bounds__(256) quantize_w4_kernel(const float* __restrict__ w, uint8_t* __restrict__ codes, uint16_t* __restrict__ scale,
                                                          long long n_groups) {
    constexpr int V = G / 32;
    const int lane = threadIdx.x & 31;
    for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < n_groups; i += (long long)gridDim.x * 8) {
        float v[V], m = 0.0f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            v[e] = w[i * G + lane * V + e];
            m = fmaxf(m, fabsf(v[e]));
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, off));
        uint16_t s16 = narrow1<BF>(BF ? __fdiv_rn(m, 7.0f) : fminf(__fdiv_rn(m, 7.0f), 65504.0f));
        float s = widen1<BF>(s16);
        if (scale_is_bad(s)) {                             // an empty group, or one too small or too large for a factor
            s = 1.0f;
            s16 = narrow1<BF>(1.0f);
        }
        const float inv = __fdiv_rn(1.0f, s);
        uint32_t c[V];
#pragma unroll
        for (int e = 0; e < V; ++e) c[e] = (uint32_t)(int)fminf(fmaxf(rintf(__fmul_rn(v[e], inv)), -8.0f), 7.0f) & 15u;
        if constexpr (V == 1) {
            const uint32_t next = __shfl_down_sync(0xFFFFFFFFu, c[0], 1);
            if ((lane & 1) == 0) codes[i * 16 + (lane >> 1)] = (uint8_t)(c[0] | next << 4);
        } else if constexpr (V == 2) {
            codes[i * 32 + lane] = (uint8_t)(c[0] | c[1] << 4);
        } else {
            reinterpret_cast<uint16_t*>(codes)[i * 32 + lane] = (uint16_t)(c[0] | c[1] << 4 | c[2] << 8 | c[3] << 12);
        }
        if (lane == 0) scale[i] = s16;
    }
}

constexpr int kMaxSmem = 227 * 1024, kSmSmem = 228 * 1024;     // of a block, and of an SM (each block takes 1 KB more)
int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

__global__ void __launch_bounds__(512, 1) cluster_room_kernel() {}

// Clusters of `split` blocks, `per_sm` of them on an SM by their shared memory, that the device holds at once: fewer than the
// blocks alone would allow, for a cluster stays within a part of the chip (B200: 33 clusters of 8 at two an SM, not 37).
int cluster_slots(int split, int per_sm, int threads, int sms) {
    if (split == 1) return sms * per_sm;
    static std::atomic<int> known[64][9][4];               // (threads do not matter: shared memory decides)
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 1;
    std::atomic<int>& k = known[dev & 63][split][per_sm & 3];
    if (k.load() == 0) {
        int n = 0;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)(split * sms));
        cfg.blockDim = dim3((unsigned)threads);
        cfg.dynamicSmemBytes = kSmSmem / per_sm - 1024;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)split;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaFuncSetAttribute(cluster_room_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, cluster_room_kernel, &cfg) != cudaSuccess || n < 1)
            n = 1;
        k.store(n);
    }
    return k.load();
}

// How a call is cut: blocks of a cluster, what a block holds at once.  Cost in clocks of an SM's sub-partition: a warp's windows, at
// the pace of an SM's warps together or of one alone; its share of bringing the tokens to shared memory; the ends.  The clocks are
// rough and set by hand.  Against every split and number of blocks an SM, forced, for 1, 2, 7 and 16 tokens of seven matrices: within
// 1.5 % of the best in 15 of 28 cases, within 6 % in 25, at worst 18 % behind (2 tokens of 6144 x 4096, groups of 64: 8.45 us, one
// block an SM and no cluster 7.14).
struct W4Plan {
    int split, pass_tiles, parts, part_windows, clusters;
    size_t smem;
};
template <int TOKENS, int STAGES, int G>
W4Plan plan_w4(int tiles_all, int windows_all, int x_rows, int sms) {
    using Shape = W4Shape<TOKENS, STAGES, G>;
    W4Plan best{};
    long long least = -1;
    for (int split = 1; split <= 8 && split <= windows_all; split *= 2) {
        const int windows = ceil_div(windows_all, split);
        for (int per_sm = Shape::kPerSm; per_sm >= 1; --per_sm) {
            const long long room = kSmSmem / per_sm - 1024 - Shape::kRing;
            const int slots = cluster_slots(split, per_sm, Shape::kThreads, sms);
            const int clusters = tiles_all < slots ? tiles_all : slots;
            const int tiles = ceil_div(tiles_all, clusters);
            // sums of the block's rows get up to half of the room, tokens the rest
            int passes = 1;
            while (ceil_div(tiles, passes) > 1 && (long long)Shape::sum_bytes(x_rows, ceil_div(tiles, passes)) > room / 2) ++passes;
            const int pass = ceil_div(tiles, passes);
            const long long x_room = room - (long long)Shape::sum_bytes(x_rows, pass);
            if (x_room < (long long)Shape::x_bytes(x_rows, 1)) continue;
            const int fit = (int)(x_room / (long long)Shape::x_bytes(x_rows, 1)), part = fit < windows ? fit : windows;
            const int parts = ceil_div(windows, part);
            const long long run = (long long)passes * parts * (ceil_div((long long)pass * part, Shape::kWarps) + 1);
            const long long busy = per_sm * Shape::kWarps / 8 * (Shape::kDigits ? 400 : TOKENS == 8 ? 700 : 800);
            const long long step = busy > 900 ? busy : 900;
            const long long staged = (long long)ceil_div((long long)windows * x_rows, Shape::kWarps) * (parts > 1 ? passes : 1);
            const long long cost = run * step + staged * per_sm * Shape::kWarps / 8 * (Shape::kDigits ? 400 : 60) + passes * (split > 1 ? 3000 : 500) +
                                   (parts > 1 ? (long long)passes * parts * 1500 : 0);
            if (least >= 0 && cost >= least) continue;
            least = cost;
            best = W4Plan{split, pass, parts, part, clusters, Shape::kRing + Shape::sum_bytes(x_rows, pass) + Shape::x_bytes(x_rows, part)};
        }
    }
    return best;
}

template <int TOKENS, int STAGES, bool BF, int G>
cudaError_t launch_w4(W4Params p, int sms, cudaStream_t st) {
    using Shape = W4Shape<TOKENS, STAGES, G>;
    const int tiles = ceil_div(p.N, Shape::kRows), windows = ceil_div(p.K, Shape::kWindow);
    p.x_rows = p.T;
    p.sc_whole = p.K % Shape::kWindow == 0;
    // a decode loop asks for the same few shapes again and again: the last ones' plans are kept, by their sizes
    struct Known {
        int tiles, windows, x_rows, sms;
        W4Plan plan;
    };
    static thread_local Known known[8];
    Known& k = known[(unsigned)(tiles * 31 + windows * 7 + p.x_rows) % 8];
    if (k.tiles != tiles || k.windows != windows || k.x_rows != p.x_rows || k.sms != sms)
        k = Known{tiles, windows, p.x_rows, sms, plan_w4<TOKENS, STAGES, G>(tiles, windows, p.x_rows, sms)};
    p.split = k.plan.split;
    for (p.split_log = 0; 1 << p.split_log < p.split; ++p.split_log) {}
    p.tiles_each = tiles / k.plan.clusters;
    p.tiles_more = tiles % k.plan.clusters;
    p.windows_each = windows / p.split;
    p.windows_more = windows % p.split;
    p.pass_tiles = k.plan.pass_tiles;
    p.parts = k.plan.parts;
    p.part_windows = k.plan.part_windows;

    static std::atomic<unsigned long long> ready{0};       // devices whose shared-memory limit has been raised
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!(ready.load() >> (dev & 63) & 1)) {
        e = cudaFuncSetAttribute(w4_linear_kernel<TOKENS, STAGES, BF, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
        if (e != cudaSuccess) return e;
        ready.fetch_or(1ull << (dev & 63));
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(k.plan.clusters * p.split));
    cfg.blockDim = dim3(Shape::kThreads);
    cfg.dynamicSmemBytes = k.plan.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0] = pdl_attribute();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, w4_linear_kernel<TOKENS, STAGES, BF, G>, p, kBits<BF>);
}

}  // namespace
}  // namespace sasq

#include "w4_batch.cuh"

namespace sasq {
namespace {

template <bool BF, int G>
cudaError_t launch_tokens(const W4Params& p, int sms, cudaStream_t st) {
    // windows of a ring: as many as leave the tokens their room
    if (p.T <= 2) return launch_w4<2, 4, BF, G>(p, sms, st);
    if (p.T <= 8) return launch_w4<8, 3, BF, G>(p, sms, st);
    // (in turns of 16: 17 tokens of 4096 x 4096 14.8 us, here 9.6; 64 of 11008 x 4096 43.8 and 25.8, 32 of them 24.8 and 23.4; 61 of
    // 6144 x 4096, groups of 32, 29.3 and 23.4; 16 tokens of 4096 x 4096 10.4 and 10.3, 12 of 11008 x 4096 14.3 and above 23)
    if (p.T <= 16) return launch_w4<16, 2, BF, G>(p, sms, st);
    return p.T <= 32 ? launch_w4_batch<32, BF, G>(p, sms, st) : launch_w4_batch<64, BF, G>(p, sms, st);
}
template <bool BF>
cudaError_t launch_group(const W4Params& p, int group, int sms, cudaStream_t st) {
    return group == 128  ? launch_tokens<BF, 128>(p, sms, st)
           : group == 64 ? launch_tokens<BF, 64>(p, sms, st)
                         : launch_tokens<BF, 32>(p, sms, st);
}

}  // namespace
}  // namespace sasq

extern "C" {

int sasq_w4_linear(const void* x, const uint8_t* w, const void* w_scale, const void* bias, void* y, int64_t T, int64_t N, int64_t K,
                   int64_t group, int dt, void* stream) {
    using namespace sasq;
    if ((dt != SASQ_F16 && dt != SASQ_BF16) || T < 0 || N <= 0 || K <= 0) return SASQ_ERR_INVALID_ARG;
    if (w == nullptr || w_scale == nullptr || !aligned16(w) || !aligned16(w_scale) || !aligned16(bias)) return SASQ_ERR_INVALID_ARG;
    if (T > 0 && (x == nullptr || y == nullptr || !aligned16(x) || !aligned16(y) || x == y)) return SASQ_ERR_INVALID_ARG;
    if ((group != 32 && group != 64 && group != 128) || K % group != 0) return SASQ_ERR_UNSUPPORTED;
    if (T > (1 << 19) || N > (1 << 30) || K > (1 << 24)) return SASQ_ERR_UNSUPPORTED;
    if (T == 0) return SASQ_OK;
    const int sms = device_sm_count_if_sm100();
    if (sms <= 0) return SASQ_ERR_UNSUPPORTED;
    W4Params p{};
    p.x = static_cast<const uint16_t*>(x);
    p.w = w;
    p.ws = static_cast<const uint16_t*>(w_scale);
    p.bias = static_cast<const uint16_t*>(bias);
    p.y = static_cast<uint16_t*>(y);
    p.T = (int)T;
    p.N = (int)N;
    p.K = (int)K;
    p.groups = (int)(K / group);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dt == SASQ_BF16 ? launch_group<true>(p, (int)group, sms, st) : launch_group<false>(p, (int)group, sms, st);
    return e == cudaSuccess ? SASQ_OK : SASQ_ERR_CUDA;
}

int sasq_quantize_weight_w4(const float* w, uint8_t* w_int, void* w_scale, int64_t N, int64_t K, int64_t group, int dt, void* stream) {
    using namespace sasq;
    if ((dt != SASQ_F16 && dt != SASQ_BF16) || N < 0 || K <= 0) return SASQ_ERR_INVALID_ARG;
    if (N > 0 && (w == nullptr || w_int == nullptr || w_scale == nullptr || !aligned16(w) || !aligned16(w_int) || !aligned16(w_scale)))
        return SASQ_ERR_INVALID_ARG;
    if ((group != 32 && group != 64 && group != 128) || K % group != 0) return SASQ_ERR_UNSUPPORTED;
    if (N > (1 << 30) || K > (1 << 24)) return SASQ_ERR_UNSUPPORTED;
    if (N == 0) return SASQ_OK;
    const int sms = device_sm_count_if_sm100();
    if (sms <= 0) return SASQ_ERR_UNSUPPORTED;
    const long long n = N * (K / group);
    const int blocks = (int)(n / 8 + 1 < 16LL * sms ? n / 8 + 1 : 16LL * sms);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto go = [&](auto* kernel) { kernel<<<blocks, 256, 0, st>>>(w, w_int, static_cast<uint16_t*>(w_scale), n); };
    if (dt == SASQ_BF16)
        group == 128 ? go(quantize_w4_kernel<true, 128>) : group == 64 ? go(quantize_w4_kernel<true, 64>) : go(quantize_w4_kernel<true, 32>);
    else
        group == 128 ? go(quantize_w4_kernel<false, 128>) : group == 64 ? go(quantize_w4_kernel<false, 64>) : go(quantize_w4_kernel<false, 32>);
    return cudaGetLastError() == cudaSuccess ? SASQ_OK : SASQ_ERR_CUDA;
}

}  // extern "C"
