// Linear layers with 4-bit weights and group factors for few tokens, and the quantizer that makes such weights.
//
//   y[t, n] = narrow( sum_g s[n, g] * sum_{k in group g} x[t, k] c[n, k]  (+ bias[n]) )
//
// Bound by the weights: half a byte each, read once.  The products run on mma.sync m16n8k16 with 16 rows of weights on its
// wide side and 8 tokens on the other: one token wastes 7/8 of an instruction whose rate is no limit, and a weight goes from
// its byte to the operand in registers, where its group's factor can be applied to the group's fp32 sum.
#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "tcgen05.cuh"

namespace sasq {
namespace {

#ifndef FEW_STAGES
#define FEW_BLOCKS 2
#define FEW_STAGES 4
#endif
struct W4Params {
    const uint16_t* x;          // [T, K]
    const uint8_t* w;           // [N, K / 2]
    const uint16_t* ws;         // [N, K / G]
    const uint16_t* bias;       // [N] or nullptr
    uint16_t* y;                // [T, N]
    int T, N, K, groups;
    int tiles;                  // of 16 rows
    int windows;                // of 128 columns
    int x_rows;                 // tokens of a block at most
    int split;                  // blocks of a cluster (1, 2, 4 or 8), each with a share of the windows
    int split_log;
    // cluster c has tiles_each tiles from c * tiles_each on and one more if c < tiles_more; so have a cluster's blocks windows.
    // (Divisions cost a warp hundreds of instructions before its first load: the host makes them.)
    int tiles_each, tiles_more, windows_each, windows_more;
    int wk;                     // warps that share a tile's windows: 1, 2, 4 or 8
    int pass_tiles;             // tiles whose sums a block holds at once
    int parts, part_windows;    // a block's windows are taken in parts whose tokens fit shared memory
};

constexpr int kWindow = 128;    // columns of a step: 64 bytes of a weight row

__device__ __forceinline__ void mma_w4(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool bf) {
    if (bf)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

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

// d = a b + c, where c is the same for the rows of a token
__device__ __forceinline__ void mma_w4_from(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float c0, float c1, bool bf) {
    if (bf)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%10,%11};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%10,%11};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
}

// (a & mask) ^ c
template <uint32_t MASK>
__device__ __forceinline__ uint32_t and_xor(uint32_t a, uint32_t c) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(d) : "r"(a), "n"(MASK), "r"(c));
    return d;
}

// Eight codes of a word as 16-bit floats: pairs (0, 4), (2, 6) in lo and (1, 5), (3, 7) in hi.  With the sign bit flipped a nibble
// is u = code + 8.  BIAS: bf16 128 + u; f16, as subnormal numbers, u 2^-24 in lo and u 2^-20 in hi.  Otherwise the codes:
// bf16 takes 136 off; f16 makes 1024 + u and takes 1032 off, one nibble further up 1024 + 16 u, which a fused multiply-add brings to the
// code.  5 instructions of the logic pipe, which runs at half the others' rate and sets the pace, for f16, 7 for bf16.
// The constants that meet a mask come as kernel parameters: a logic instruction takes one immediate, and of two the compiler
// makes two instructions (measured).
struct Bits {
    uint32_t low, high;         // exponent and flipped sign of a low and a high nibble
};
template <bool BF, bool BIAS>
constexpr Bits kBits = BF ? Bits{0x43084308u, 0x43084308u} : BIAS ? Bits{0x00080008u, 0x00800080u} : Bits{0x64086408u, 0x64806480u};
template <bool BF, bool BIAS>
__device__ __forceinline__ void nibbles8(uint32_t w, const Bits& bits, uint32_t (&lo)[2], uint32_t (&hi)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        lo[i] = and_xor<0x000F000Fu>(w >> (8 * i), bits.low);
        if constexpr (BF) hi[i] = and_xor<0x000F000Fu>(w >> (8 * i + 4), bits.low);
        else hi[i] = and_xor<0x00F000F0u>(w >> (8 * i), bits.high);
        if constexpr (!BIAS && BF) {
            const __nv_bfloat162 bias = __halves2bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308));
            const __nv_bfloat162 a = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&lo[i]), bias);
            const __nv_bfloat162 b = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&hi[i]), bias);
            lo[i] = *reinterpret_cast<const uint32_t*>(&a);
            hi[i] = *reinterpret_cast<const uint32_t*>(&b);
        } else if constexpr (!BIAS) {
            const uint32_t off = 0x64086408u, sixteenth = 0x2C002C00u, minus72 = 0xD480D480u;
            const __half2 a = __hsub2(*reinterpret_cast<const __half2*>(&lo[i]), *reinterpret_cast<const __half2*>(&off));
            const __half2 b = __hfma2(*reinterpret_cast<const __half2*>(&hi[i]), *reinterpret_cast<const __half2*>(&sixteenth),
                                      *reinterpret_cast<const __half2*>(&minus72));
            lo[i] = *reinterpret_cast<const uint32_t*>(&a);
            hi[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
    }
}

// A lane's N weight words of one row and window from their slot: word s * (G / 32) + i is its i-th of group s.
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

// The tokens' columns of this block lie in shared memory, already in the order in which nibbles come out of a word, and each warp
// streams its own windows of weights (STAGES - 1 under way) through a ring of its own, 32 rows at a time: no barrier until the
// sums of all the block's rows meet.  p.wk warps share a tile's windows, the others take other tiles.  NT blocks of 8 tokens.
// One block of tokens: the weights' operands keep their bias (code + 8, bf16: + 136), and a group's sum starts at minus the bias
// times the sum of the group's x, which is the third operand of its first product.  More: the conversion hides behind the
// products, and the codes are taken as they are.
template <int NT, int STAGES, bool BF, int G>
struct W4Shape {
    static constexpr bool kBias = NT == 1;
    static constexpr int kWarps = 8, kThreads = 32 * kWarps;
    static constexpr int kSlot = 32 * 64;                  // bytes: a window of 32 rows
    static constexpr int kRing = kWarps * STAGES * kSlot;
    static constexpr int kOff = BF ? 4 : 8;                // bytes of a sum's start: f16 has one for either kind of nibble
    static size_t x_bytes(int tokens, int windows) {
        return (size_t)windows * ((size_t)tokens * 256 + (kBias ? kWindow / G * 8 * kOff : 0));
    }
    static size_t sum_bytes(int wk, int tokens, int tiles) { return (size_t)wk * tokens * (16 * tiles + 4) * sizeof(float); }
};

// What a warp works on, in order: up to two of its tiles of 16 rows, over a part of the columns.
struct W4Job {
    int pass, part, tile, end;                             // first tile of the pass; part of the columns; tile, and the warp's last
};

template <int NT, int STAGES, bool BF, int G>
__global__ void __launch_bounds__(256, NT <= 2 ? 2 : 1) w4_linear_kernel(const __grid_constant__ W4Params p, const __grid_constant__ Bits bits_) {
    using Shape = W4Shape<NT, STAGES, BF, G>;
    constexpr bool kBias = Shape::kBias, kTwo = kBias && !BF;   // kTwo: low and high nibbles have sums of their own
    constexpr int GW = kWindow / G, WG = G / 32;           // groups of a window, words of a lane in a group
    constexpr uint32_t kSlot = Shape::kSlot;
    constexpr int kOff = Shape::kOff;
    extern __shared__ __align__(128) uint8_t smem[];
    const Bits bits = bits_;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, j = lane & 3;
    const int wk = warp % p.wk, wr = warp / p.wk, row_warps = Shape::kWarps / p.wk;
    const int rank = p.split > 1 ? (int)ptx::cluster_ctarank() : 0;
    const int cluster = blockIdx.x >> p.split_log;
    const int t0 = blockIdx.y * 8 * NT;                    // tokens of this block
    const int tokens = min(8 * NT, p.T - t0);
    const int row_begin = cluster * p.tiles_each + min(cluster, p.tiles_more), row_end = row_begin + p.tiles_each + (cluster < p.tiles_more);
    const int begin = rank * p.windows_each + min(rank, p.windows_more), end = begin + p.windows_each + (rank < p.windows_more);
    const int half_k = p.K >> 1;                           // bytes of a weight row
    const int sum_pitch = 16 * p.pass_tiles + 4;           // floats: neighbouring tokens lie in different banks
    const uint32_t ring = ptx::smem_u32(smem) + warp * STAGES * kSlot;
    float* const sums = reinterpret_cast<float*>(smem + Shape::kRing);
    const uint32_t off_base = ptx::smem_u32(sums + p.wk * p.x_rows * sum_pitch);
    const uint32_t x_base = off_base + (kBias ? p.part_windows * GW * 8 * kOff : 0);
    pdl_launch_dependents();

    // this warp's tiles of a pass, and its windows of a part: part_begin + wk, + p.wk, ...
    auto enter_pass = [&](W4Job& job, int pass) {
        const int tiles = min(p.pass_tiles, row_end - pass);
        job.pass = pass;
        job.part = 0;
        job.tile = pass + tiles * wr / row_warps;
        job.end = pass + tiles * (wr + 1) / row_warps;
    };
    auto part_begin = [&](int part) { return begin + part * p.part_windows; };
    auto mine_of = [&](int part) { return (min(part_begin(part) + p.part_windows, end) - part_begin(part) - wk + p.wk - 1) / p.wk; };

    // where the copies of weights stand: the jobs that have tiles and windows, one after another
    W4Job load_job;
    enter_pass(load_job, row_begin);
    int load_n = 0, load_mine = 0, load_byte = 0;
    uint32_t load_at = ring;
    uint32_t load_row[4];                                  // of this lane's rows, bytes behind the tile's first
    const uint8_t* load_tile = p.w;
    bool load_two = false;
    const uint32_t w_place = g * 64 + ((j ^ (g >> 1 & 3)) << 4);
    auto enter_load = [&] {
        while (load_job.pass < row_end) {
            load_mine = mine_of(load_job.part);
            if (load_job.tile < load_job.end && load_mine > 0) {
                load_n = 0;
                load_two = load_job.tile + 1 < load_job.end;
                load_tile = p.w + (long long)load_job.tile * 16 * half_k;
                load_byte = (part_begin(load_job.part) + wk) * 64 + 16 * j;
                // rows behind the last are read from the last one's place: their products are not stored
#pragma unroll
                for (int r = 0; r < 4; ++r) load_row[r] = (uint32_t)min(8 * r + g, p.N - 1 - 16 * load_job.tile) * (uint32_t)half_k;
                return;
            }
            const int pass = load_job.pass, part = load_job.part + 1;
            enter_pass(load_job, pass);
            load_job.part = part;
            if (part >= p.parts) enter_pass(load_job, pass + p.pass_tiles);
        }
    };
    auto load_w = [&] {
        if (load_job.pass < row_end) {
            const uint8_t* src = load_tile + min(load_byte, half_k - 16);      // columns behind the last will meet zeros
            copy16(load_at + w_place, src + load_row[0]);
            copy16(load_at + w_place + 512, src + load_row[1]);
            if (load_two) {
                copy16(load_at + w_place + 1024, src + load_row[2]);
                copy16(load_at + w_place + 1536, src + load_row[3]);
            }
            load_byte += 64 * p.wk;
            load_at = load_at + kSlot == ring + STAGES * kSlot ? ring : load_at + kSlot;
            if (++load_n == load_mine) {
                load_job.tile += 2;
                enter_load();
            }
        }
        copies_end_group();
    };
    // weights may be read at once, tokens when the kernels before this one are done
    enter_load();
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) load_w();
    pdl_wait();

    // Chunk c of eight columns is group s, lane jj, word ii, and lies where lanes jj = 0 ... 3 read side by side, which every
    // other token does 64 bytes further on, in other banks.  Half a warp has a window of a token; four at a time travel.
    auto stage_x = [&](int part) {
        const int from = part_begin(part), pairs = (min(from + p.part_windows, end) - from) * tokens;
        const int c = lane & 15, s = c / (G / 8), jj = c % (G / 8) / WG, ii = c % WG;
        const uint32_t place = (s * WG + ii) * 64 + jj * 16;
        constexpr int kBatch = 4;
        for (int first = 2 * warp; first < pairs; first += 2 * Shape::kWarps * kBatch) {
            uint4 v[kBatch];
            int w[kBatch], t[kBatch];
#pragma unroll
            for (int e = 0; e < kBatch; ++e) {
                const int i = min(first + 2 * Shape::kWarps * e + (lane >> 4), pairs - 1);
                w[e] = i / tokens;
                t[e] = i - w[e] * tokens;
                const int col = (from + w[e]) * kWindow + 8 * c;
                v[e] = col < p.K ? *reinterpret_cast<const uint4*>(p.x + (long long)(t0 + t[e]) * p.K + col) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < kBatch; ++e) {
                const uint32_t to = x_base + (w[e] * p.x_rows + t[e]) * 256 + (place ^ ((t[e] & 1) << 6));
                asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(__byte_perm(v[e].x, v[e].z, 0x5410)),
                             "r"(__byte_perm(v[e].y, v[e].w, 0x5410)), "r"(__byte_perm(v[e].x, v[e].z, 0x7632)),
                             "r"(__byte_perm(v[e].y, v[e].w, 0x7632)) : "memory");
                if constexpr (kBias) {
                    const float2 a = widen2<BF>(v[e].x), b = widen2<BF>(v[e].y), d = widen2<BF>(v[e].z), f = widen2<BF>(v[e].w);
                    float even = (a.x + b.x) + (d.x + f.x), odd = (a.y + b.y) + (d.y + f.y);
                    if (BF) even += odd;
#pragma unroll
                    for (int o = 1; o < G / 8; o <<= 1) {
                        even += __shfl_xor_sync(0xFFFFFFFFu, even, o);
                        if (!BF) odd += __shfl_xor_sync(0xFFFFFFFFu, odd, o);
                    }
                    if (c % (G / 8) == 0) {
                        const uint32_t off = off_base + ((w[e] * GW + s) * 8 + t[e]) * kOff;
                        if (BF) asm volatile("st.shared.f32 [%0], %1;" ::"r"(off), "f"(-136.0f * even) : "memory");
                        else asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(off), "f"(even * -4.76837158203125e-7f), "f"(odd * -7.62939453125e-6f) : "memory");
                    }
                }
            }
        }
    };

    uint32_t at = ring;                                    // the slot that is read next
    // factors of the next window, as they are stored
    uint16_t next_sc[2][2][GW];
    uint32_t sc_row[2][2];
    const uint16_t* sc_tile = p.ws;
    auto load_sc = [&](int window) {
#pragma unroll
        for (int s = 0; s < GW; ++s) {
            const uint16_t* src = sc_tile + min(window * GW + s, p.groups - 1);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int r = 0; r < 2; ++r) next_sc[m][r][s] = __ldg(src + sc_row[m][r]);
        }
    };
    auto enter_sc = [&](int tile, int part) {
        sc_tile = p.ws + (long long)tile * 16 * p.groups;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < 2; ++r) sc_row[m][r] = (uint32_t)min(16 * m + 8 * r + g, p.N - 1 - 16 * tile) * (uint32_t)p.groups;
        load_sc(part_begin(part) + wk);
    };

    // a job's windows, for one or two tiles
    auto work = [&](auto mt, const W4Job& job) {
        constexpr int MT = decltype(mt)::value;
        float tot[MT][NT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) tot[m][nt][0] = tot[m][nt][1] = tot[m][nt][2] = tot[m][nt][3] = 0.0f;
        const int mine = mine_of(job.part);
        uint32_t x_at = x_base + wk * p.x_rows * 256 + 16 * j, off_at = off_base + wk * GW * 8 * kOff + 2 * j * kOff;
        for (int n = 0; n < mine; ++n) {
            float sc[MT][2][GW];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int s = 0; s < GW; ++s) sc[m][r][s] = widen1<BF>(next_sc[m][r][s]);
            if (n + 1 < mine) load_sc(part_begin(job.part) + wk + (n + 1) * p.wk);
            else if (job.tile + MT < job.end) enter_sc(job.tile + MT, job.part);
            copies_wait<STAGES - 2>();
            __syncwarp();
            load_w();
            uint32_t wv[MT][2][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 2; ++r) window_words<G>(at + (16 * m + 8 * r + g) * 64, g >> 1 & 3, j, wv[m][r]);
            at = at + kSlot == ring + STAGES * kSlot ? ring : at + kSlot;
#pragma unroll
            for (int s = 0; s < GW; ++s) {
                float acc[MT][NT][4], high[kTwo ? MT : 1][NT][4], off[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if constexpr (kTwo) {
                    const uint4 o = lds16(off_at + s * 8 * kOff);       // low and high of token 2j, then of 2j + 1
                    off[0] = __uint_as_float(o.x);
                    off[2] = __uint_as_float(o.y);
                    off[1] = __uint_as_float(o.z);
                    off[3] = __uint_as_float(o.w);
                } else if constexpr (kBias) {
                    const uint2 o = lds8(off_at + s * 8 * kOff);
                    off[0] = __uint_as_float(o.x);
                    off[1] = __uint_as_float(o.y);
                }
#pragma unroll
                for (int i = 0; i < WG; ++i) {
                    uint32_t lo[MT][4], hi[MT][4];
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        uint32_t l0[2], l1[2], h0[2], h1[2];
                        nibbles8<BF, kBias>(wv[m][0][s * WG + i], bits, l0, h0);
                        nibbles8<BF, kBias>(wv[m][1][s * WG + i], bits, l1, h1);
                        lo[m][0] = l0[0], lo[m][1] = l1[0], lo[m][2] = l0[1], lo[m][3] = l1[1];
                        hi[m][0] = h0[0], hi[m][1] = h1[0], hi[m][2] = h0[1], hi[m][3] = h1[1];
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const int t = min(8 * nt + g, tokens - 1);
                        const uint4 b = lds16(x_at + t * 256 + (((s * WG + i) << 6) ^ ((t & 1) << 6)));
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            if (i == 0) mma_w4_from(acc[m][nt], lo[m], b.x, b.y, off[0], off[1], BF);
                            else mma_w4(acc[m][nt], lo[m], b.x, b.y, BF);
                            if constexpr (kTwo) {
                                if (i == 0) mma_w4_from(high[m][nt], hi[m], b.z, b.w, off[2], off[3], BF);
                                else mma_w4(high[m][nt], hi[m], b.z, b.w, BF);
                            } else {
                                mma_w4(acc[m][nt], hi[m], b.z, b.w, BF);
                            }
                        }
                    }
                }
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float sum = kTwo ? fmaf(high[kTwo ? m : 0][nt][e], 0.0625f, acc[m][nt][e]) : acc[m][nt][e];
                            tot[m][nt][e] = fmaf(sum, sc[m][e >> 1][s], tot[m][nt][e]);
                        }
            }
            x_at += p.wk * p.x_rows * 256;
            off_at += p.wk * GW * 8 * kOff;
        }
        constexpr float kUnit = kTwo ? 16777216.0f : 1.0f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (8 * nt + 2 * j + e < tokens) {
                    float* const to = sums + (wk * p.x_rows + 8 * nt + 2 * j + e) * sum_pitch + 16 * (job.tile - job.pass) + g;
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float v = tot[m][nt][e + 2 * r] * kUnit;
                            float* const cell = to + 16 * m + 8 * r;
                            *cell = job.part == 0 ? v : *cell + v;
                        }
                }
    };

    for (int pass = row_begin; pass < row_end; pass += p.pass_tiles) {
        W4Job job;
        for (int part = 0; part < p.parts; ++part) {
            enter_pass(job, pass);
            job.part = part;
            if (job.tile < job.end && mine_of(part) > 0) enter_sc(job.tile, part);
            if (p.parts > 1 || pass == row_begin) {
                __syncthreads();                           // (the part before has been read)
                stage_x(part);
                __syncthreads();
            }
            for (; job.tile + 1 < job.end; job.tile += 2) work(std::integral_constant<int, 2>{}, job);
            if (job.tile < job.end) work(std::integral_constant<int, 1>{}, job);
        }
        const int tiles = min(p.pass_tiles, row_end - pass);
        // the warps' (and the cluster's) sums meet in a fixed order
        const int rows = 16 * tiles;
        auto store = [&](int t, int row, float v) {
            const int n_row = 16 * pass + row;
            if (n_row >= p.N) return;
            if (p.bias != nullptr) v += widen1<BF>(p.bias[n_row]);
            p.y[(long long)(t0 + t) * p.N + n_row] = narrow1<BF>(v);
        };
        __syncthreads();
        for (int i = tid; i < tokens * rows; i += Shape::kThreads) {
            const int t = i / rows, row = i - t * rows;
            float v = sums[t * sum_pitch + row];
            for (int k = 1; k < p.wk; ++k) v += sums[(k * p.x_rows + t) * sum_pitch + row];
            if (p.split == 1) store(t, row, v);
            else sums[t * sum_pitch + row] = v;
        }
        if (p.split > 1) {
            ptx::cluster_sync_all();
            for (int i = rank * Shape::kThreads + tid; i < tokens * rows; i += p.split * Shape::kThreads) {
                const int t = i / rows, row = i - t * rows;
                const uint32_t here = ptx::smem_u32(&sums[t * sum_pitch + row]);
                float v = 0.0f;
                for (int k = 0; k < p.split; ++k) {
                    uint32_t peer;
                    float part;
                    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer) : "r"(here), "r"(k));
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part) : "r"(peer));
                    v += part;
                }
                store(t, row, v);
            }
            ptx::cluster_sync_all();                       // nobody goes on, or leaves, while its sums are being read
        } else {
            __syncthreads();
        }
    }
    copies_wait<0>();
}

// ---------------------------------------------------------------------------------------------------------------------
// Up to 8 tokens.  16-bit products would need every code as a 16-bit float, 5 to 7 instructions of the logic pipe for 8 codes.
// As signed bytes, 16 times the code, 8 codes are a shift and two masks, and one s8 product of m16n8k32 takes twice as many
// of them.  So x becomes integers: in a window of 256 columns a token's values are multiples of a power of two, 2^-22 of the
// window's largest, whose digits to the base 256, from -128 to 127, are three columns of the product.  A group's sums are exact
// integers of at most 2^21; they start at the bits of the float 1.5 * 2^23, so that the float they end as is that plus the sum.
// TP: tokens rounded up to 2, 4 or 8.  Digit l of token t is column l * TP + t of 8 * kTiles.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int kFewWindow = 256;                            // columns of a step: 128 bytes of a weight row

template <int TP, int STAGES, int G>
struct FewShape {
    static constexpr int kWarps = 8;
    static constexpr int kTiles = (3 * TP + 7) / 8;        // blocks of 8 columns
    static constexpr int kSlot = 16 * 128;                 // bytes: a window of 16 rows
    static constexpr int kRing = kWarps * STAGES * kSlot;
    static constexpr int kTable = 8 * kTiles * 4;          // bytes of a window's factors
    static size_t x_bytes(int tokens, int windows) { return (size_t)windows * (3 * tokens * 256 + kTable); }
    static size_t sum_bytes(int tokens, int tiles) { return (size_t)kWarps * tokens * (16 * tiles + 4) * sizeof(float); }
};

constexpr uint32_t kMagic = 0x4B400000u;                   // 1.5 * 2^23

__device__ __forceinline__ void mma_s8(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// d = a b + c
__device__ __forceinline__ void mma_s8_from(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, uint32_t c) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "r"(c));
}

// A block has some tiles of 16 rows and (in a cluster) a share of the columns' windows.  The windows of all its tiles, laid end to
// end, are cut into equal runs, one for each warp: a warp walks on through a tile's windows, and its sums change hands only where
// a tile or its run ends.  The tokens' digits lie in shared memory, and each warp streams its weights through a ring of its own
// (STAGES - 1 windows under way): no barrier until the sums of all the block's rows meet.
template <int TP, int STAGES, bool BF, int G>
__global__ void __launch_bounds__(256, FEW_BLOCKS) w4_few_kernel(const __grid_constant__ W4Params p) {
    using Shape = FewShape<TP, STAGES, G>;
    constexpr int GW = kFewWindow / G, WG = G / 32;        // groups of a window, words of a lane in a group
    constexpr int NT = Shape::kTiles, WK = Shape::kWarps;
    constexpr uint32_t kSlot = Shape::kSlot;
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, j = lane & 3;
    const int rank = p.split > 1 ? (int)ptx::cluster_ctarank() : 0;
    const int cluster = blockIdx.x >> p.split_log;
    const int tile_begin = cluster * p.tiles_each + min(cluster, p.tiles_more), tile_end = tile_begin + p.tiles_each + (cluster < p.tiles_more);
    const int begin = rank * p.windows_each + min(rank, p.windows_more), end = begin + p.windows_each + (rank < p.windows_more);
    const int half_k = p.K >> 1;                           // bytes of a weight row
    const int sum_pitch = 16 * p.pass_tiles + 4;           // floats: neighbouring tokens lie in different banks
    const uint32_t ring = ptx::smem_u32(smem) + warp * STAGES * kSlot;
    float* const sums = reinterpret_cast<float*>(smem + Shape::kRing);
    const uint32_t table = ptx::smem_u32(sums + WK * p.T * sum_pitch);         // a window's factors: [8 * NT]
    const uint32_t x_base = table + p.part_windows * Shape::kTable;            // [window][digit][token] of 256 bytes
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

    // Copies of weights.  Chunk c of 16 bytes of a row lies at c ^ turn(row): whatever the group, the rows that a warp reads
    // together lie in different banks.
    auto turn = [](int row) { return (row & 1) << 2 | (row & 2) | (row >> 2 & 1); };
    const int w_row = lane >> 3, w_chunk = lane & 7;       // a copy takes 4 rows
    const uint32_t w_place[2] = {(uint32_t)(w_row * 128 + ((w_chunk ^ turn(w_row)) << 4)), (uint32_t)((w_row + 4) * 128 + ((w_chunk ^ turn(w_row + 4)) << 4))};
    int load_pass = tile_begin, load_part = 0;
    Run ld = run_of(load_pass, load_part);
    uint32_t load_at = ring, load_row[4] = {0, 0, 0, 0};
    const uint8_t* load_w = p.w;
    auto enter_load = [&] {
        load_w = p.w + (long long)ld.tile * 16 * half_k;
        // rows behind the last are read from the last one's place: their products are not stored
#pragma unroll
        for (int r = 0; r < 4; ++r) load_row[r] = (uint32_t)min(w_row + 4 * r, p.N - 1 - 16 * ld.tile) * (uint32_t)half_k;
    };
    auto settle = [&] {                                    // on to the next part or pass with work
        while (ld.left == 0 && load_pass < tile_end) {
            if (++load_part == p.parts) {
                load_part = 0;
                load_pass += p.pass_tiles;
            }
            if (load_pass < tile_end) {
                ld = run_of(load_pass, load_part);
                if (ld.left > 0) enter_load();
            }
        }
    };
    auto load = [&] {
        if (ld.left > 0) {
            const uint8_t* src = load_w + min((ld.first + ld.at) * 128 + 16 * w_chunk, half_k - 16);   // columns behind the last will meet zeros
#pragma unroll
            for (int r = 0; r < 4; ++r) copy16(load_at + w_place[r & 1] + (r >> 1) * 1024, src + load_row[r]);
            load_at = load_at + kSlot == ring + STAGES * kSlot ? ring : load_at + kSlot;
            --ld.left;
            if (++ld.at == ld.windows) {
                ld.at = 0;
                ++ld.tile;
                if (ld.left > 0) enter_load();
            }
            settle();
        }
        copies_end_group();
    };
    // weights may be read at once, tokens when the kernels before this one are done
    if (ld.left > 0) enter_load();
    settle();
#pragma unroll 1
    for (int s = 0; s < STAGES - 1; ++s) load();
    pdl_wait();

    // A warp has a window of a token, a lane eight columns: chunk c is group s, lane jj, word ii.  Words 2q and 2q + 1 of lanes
    // jj = 0 ... 3 lie side by side, and every other column of the product has neighbouring pairs the other way round, in other
    // banks.
    auto stage_x = [&](int part) {
        const int from = begin + part * p.part_windows, windows = min(from + p.part_windows, end) - from;
        const int c = lane, s = c / (G / 8), jj = c % (G / 8) / WG, q = s * WG + c % WG;
        const uint32_t place = (q >> 1) * 64 + jj * 16 + (q & 1) * 8;
        const int hop_w = WK / p.T, hop_t = WK - hop_w * p.T;                  // from a warp's (window, token) to its next
        struct Pair {
            int w, t;
        };
        auto hop = [&](Pair& a) {
            a.w += hop_w;
            if ((a.t += hop_t) >= p.T) {
                a.t -= p.T;
                ++a.w;
            }
        };
        auto fetch = [&](const Pair& a) {
            const int col = (from + a.w) * kFewWindow + 8 * c;
            return a.w < windows && col < p.K ? *reinterpret_cast<const uint4*>(p.x + (long long)a.t * p.K + col) : make_uint4(0, 0, 0, 0);
        };
        Pair now, ahead;
        now.w = warp / p.T;
        now.t = warp - now.w * p.T;
        ahead = now;
        hop(ahead);
        uint4 next[2] = {fetch(now), fetch(ahead)};        // two travel while one is taken apart
#pragma unroll 1
        for (; now.w < windows; hop(now)) {
            const uint32_t raw[4] = {next[0].x, next[0].y, next[0].z, next[0].w};
            const int w = now.w, t = now.t;
            hop(ahead);
            next[0] = next[1];
            next[1] = fetch(ahead);
            float f[8];
            uint32_t seen = 0;                             // NaN compares as the largest
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
                d[e] = (__float_as_uint(fmaf(f[e], up, __uint_as_float(kMagic))) - kMagic + 0x00808080u) ^ 0x00808080u;
            uint32_t even[3], odd[3];                      // digits of columns 0, 2, 4, 6 and of 1, 3, 5, 7
            auto gather = [](uint32_t a, uint32_t b, uint32_t c4, uint32_t d4, uint32_t (&to)[3]) {
                const uint32_t ab = __byte_perm(a, b, 0x5140), cd = __byte_perm(c4, d4, 0x5140);
                to[0] = __byte_perm(ab, cd, 0x5410);
                to[1] = __byte_perm(ab, cd, 0x7632);
                to[2] = __byte_perm(__byte_perm(a, b, 0x0062), __byte_perm(c4, d4, 0x0062), 0x5410);
            };
            gather(d[0], d[2], d[4], d[6], even);
            gather(d[1], d[3], d[5], d[7], odd);
#pragma unroll
            for (int l = 0; l < 3; ++l) {
                const int row = l * p.T + t;
                const uint32_t to = x_base + (w * 3 * p.T + row) * 256 + (place ^ ((row & 1) << 6));
                asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(to), "r"(even[l]), "r"(odd[l]) : "memory");
            }
            // factors: of the digit, less 16 times the code; a window with infinities or NaN: NaN; columns that stand for nothing
            // (others' digits): 0
            const float unit = seen >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __uint_as_float(top - (25u << 23));
            const int l = lane / TP, tt = lane % TP;
            if (lane < 8 * NT && (tt == t || (tt >= p.T && t == 0)))
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(table + w * Shape::kTable + lane * 4),
                             "f"(l < 3 && tt == t ? unit * __uint_as_float((127u + 8u * l) << 23) : 0.0f) : "memory");
        }
    };

    uint32_t at = ring;                                    // the slot that is read next
    // where this lane's columns of the product lie in a window
    uint32_t x_near[NT], x_far[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int col = 8 * nt + g, l = min(col / TP, 2), t = min(col % TP, p.T - 1);
        x_near[nt] = x_base + (l * p.T + t) * 256 + 16 * j + ((l * p.T + t) & 1) * 64;
        x_far[nt] = x_base + (l * p.T + t) * 256 + 16 * j + 64 - ((l * p.T + t) & 1) * 64;
    }
    for (int pass = tile_begin; pass < tile_end; pass += p.pass_tiles) {
        const int rows = 16 * min(p.pass_tiles, tile_end - pass);
        for (int part = 0; part < p.parts; ++part) {
            Run r = run_of(pass, part);
            uint16_t next_sc[2][GW];                       // factors of the next window, as they are stored
            const uint16_t* sc_row[2];
            auto load_sc = [&](int window) {
#pragma unroll
                for (int s = 0; s < GW; ++s) {
                    const int group = min((r.first + window) * GW + s, p.groups - 1);
                    next_sc[0][s] = __ldg(sc_row[0] + group);
                    next_sc[1][s] = __ldg(sc_row[1] + group);
                }
            };
            auto enter_sc = [&](int tile, int window) {
                sc_row[0] = p.ws + (long long)min(16 * tile + g, p.N - 1) * p.groups;
                sc_row[1] = p.ws + (long long)min(16 * tile + g + 8, p.N - 1) * p.groups;
                load_sc(window);
            };
            if (r.left > 0) enter_sc(r.tile, r.at);
            if (part == 0)
                for (int i = lane; i < p.T * sum_pitch; i += 32) sums[warp * p.T * sum_pitch + i] = 0.0f;
            if (p.parts > 1 || pass == tile_begin) {
                __syncthreads();                           // (the part before has been read)
                stage_x(part);
                __syncthreads();
            }
            __syncwarp();
            while (r.left > 0) {
                const int steps = min(r.left, r.windows - r.at);
                r.left -= steps;
                float tot[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) tot[nt][0] = tot[nt][1] = tot[nt][2] = tot[nt][3] = 0.0f;
                uint32_t x_at = r.at * 3 * p.T * 256, table_at = table + r.at * Shape::kTable + 8 * j;
#pragma unroll 1
                for (int n = 0; n < steps; ++n) {
                    float sc[2][GW];
#pragma unroll
                    for (int s = 0; s < GW; ++s) {
                        sc[0][s] = widen1<BF>(next_sc[0][s]);
                        sc[1][s] = widen1<BF>(next_sc[1][s]);
                    }
                    if (n + 1 < steps) load_sc(r.at + n + 1);
                    else if (r.left > 0) enter_sc(r.tile + 1, 0);
                    copies_wait<STAGES - 2>();
                    __syncwarp();
                    load();
                    uint32_t wv[2][8];
                    window_words<G>(at + g * 128, turn(g), j, wv[0]);
                    window_words<G>(at + (g + 8) * 128, turn(g), j, wv[1]);
                    at = at + kSlot == ring + STAGES * kSlot ? ring : at + kSlot;
                    float win[NT][4];
                    int acc[NT][4];
#pragma unroll
                    for (int h = 0; h < 4; ++h) {          // two words of a lane
                        uint4 b[NT];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) b[nt] = lds16((h & 1 ? x_far[nt] : x_near[nt]) + x_at + (h >> 1) * 128);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int q = 2 * h + i, s = q / WG;
                            const uint32_t a[4] = {wv[0][q] << 4 & 0xF0F0F0F0u, wv[1][q] << 4 & 0xF0F0F0F0u, wv[0][q] & 0xF0F0F0F0u,
                                                   wv[1][q] & 0xF0F0F0F0u};
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                if (q % WG == 0) mma_s8_from(acc[nt], a, i == 0 ? b[nt].x : b[nt].z, i == 0 ? b[nt].y : b[nt].w, kMagic);
                                else mma_s8(acc[nt], a, i == 0 ? b[nt].x : b[nt].z, i == 0 ? b[nt].y : b[nt].w);
                                if (q % WG == WG - 1) {
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const float v = __int_as_float(acc[nt][e]) - __uint_as_float(kMagic);
                                        win[nt][e] = s == 0 ? v * sc[e >> 1][s] : fmaf(v, sc[e >> 1][s], win[nt][e]);
                                    }
                                }
                            }
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint2 f = lds8(table_at + 8 * nt * 4);
#pragma unroll
                        for (int e = 0; e < 4; ++e) tot[nt][e] = fmaf(win[nt][e], __uint_as_float(e & 1 ? f.y : f.x), tot[nt][e]);
                    }
                    x_at += 3 * p.T * 256;
                    table_at += Shape::kTable;
                }
                // the digits' columns meet: in this lane's registers, and among the four lanes of a row
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = tot[0][e];
#pragma unroll
                    for (int nt = 1; nt < NT; ++nt) v[e] += tot[nt][e];
                    if (TP == 2) v[e] += __shfl_xor_sync(0xFFFFFFFFu, v[e], 1);
                    if (TP <= 4) v[e] += __shfl_xor_sync(0xFFFFFFFFu, v[e], 2);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int t = 2 * j + e;
                    if (t < p.T) {
                        float* const to = sums + (warp * p.T + t) * sum_pitch + 16 * (r.tile - pass) + g;
                        to[0] += v[e];
                        to[8] += v[e + 2];
                    }
                }
                r.at = 0;
                ++r.tile;
            }
        }
        // the warps' (and the cluster's) sums meet in a fixed order
        auto store = [&](int t, int row, float v) {
            const int n_row = 16 * pass + row;
            if (n_row >= p.N) return;
            if (p.bias != nullptr) v += widen1<BF>(p.bias[n_row]);
            p.y[(long long)t * p.N + n_row] = narrow1<BF>(v);
        };
        __syncthreads();
        for (int t = 0; t < p.T; ++t)
            for (int row = tid; row < rows; row += 256) {
                float v = sums[t * sum_pitch + row];
#pragma unroll
                for (int k = 1; k < WK; ++k) v += sums[(k * p.T + t) * sum_pitch + row];
                if (p.split == 1) store(t, row, v);
                else sums[t * sum_pitch + row] = v;
            }
        if (p.split > 1) {
            ptx::cluster_sync_all();
            for (int t = 0; t < p.T; ++t)
            for (int row = rank * 256 + tid; row < rows; row += p.split * 256) {
                const uint32_t here = ptx::smem_u32(&sums[t * sum_pitch + row]);
                float v = 0.0f;
                for (int k = 0; k < p.split; ++k) {
                    uint32_t peer;
                    float part;
                    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer) : "r"(here), "r"(k));
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part) : "r"(peer));
                    v += part;
                }
                store(t, row, v);
            }
            ptx::cluster_sync_all();                       // nobody goes on, or leaves, while its sums are being read
        } else if (pass + p.pass_tiles < tile_end) {
            __syncthreads();
        }
    }
    copies_wait<0>();
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

// Starts `kernel` on `clusters` x `chunks` clusters of p.split blocks; raises its limit of shared memory once a device.
template <typename Kernel, typename... More>
cudaError_t start(std::atomic<unsigned long long>* ready, const W4Params& p, int clusters, int chunks, int threads, size_t smem,
                  cudaStream_t st, Kernel kernel, const More&... more) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!(ready->load() >> (dev & 63) & 1)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
        if (e != cudaSuccess) return e;
        ready->fetch_or(1ull << (dev & 63));
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(clusters * p.split), (unsigned)chunks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0] = pdl_attribute();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, p, more...);
}

// How a call is cut: blocks of a cluster, warps that share a tile, what a block holds at once.  Cost, in clocks of an SM's
// sub-partition: the busiest warp's windows of 16 rows at the pace of an SM's warps together, bringing the tokens to shared memory,
// and meeting in a cluster.
struct W4Plan {
    int split, wk, pass_tiles, parts, part_windows, clusters, per_sm;
    size_t smem;
};
void cut_w4(W4Params* p, const W4Plan& plan) {
    p->split = plan.split;
    for (p->split_log = 0; 1 << p->split_log < plan.split; ++p->split_log) {}
    p->tiles_each = p->tiles / plan.clusters;
    p->tiles_more = p->tiles % plan.clusters;
    p->windows_each = p->windows / plan.split;
    p->windows_more = p->windows % plan.split;
}
template <int NT, int STAGES, bool BF, int G>
W4Plan plan_w4(int tiles_all, int windows_all, int x_rows, int chunks, int sms) {
    using Shape = W4Shape<NT, STAGES, BF, G>;
    constexpr int kWindowClocks = NT == 1 ? 220 : NT == 2 ? 260 : 380;
    W4Plan best{};
    long long least = -1;
    for (int split = 1; split <= 8 && split <= windows_all; split *= 2) {
        const int windows = ceil_div(windows_all, split);
        for (int per_sm = NT <= 2 ? 2 : 1; per_sm >= 1; --per_sm) {
            const long long room = kSmSmem / per_sm - 1024 - Shape::kRing;
            const int slots = sms * per_sm / split / chunks;
            const int clusters = tiles_all < slots ? tiles_all : slots < 1 ? 1 : slots;
            const int tiles = ceil_div(tiles_all, clusters);
            for (int wk = 1; wk <= Shape::kWarps; wk *= 2) {
                const int row_warps = Shape::kWarps / wk;
                // sums of the block's rows get up to a third of the room, tokens the rest
                int passes = 1;
                while (ceil_div(tiles, passes) > 1 && (long long)Shape::sum_bytes(wk, x_rows, ceil_div(tiles, passes)) > room / 3) ++passes;
                const int pass = ceil_div(tiles, passes);
                const long long x_room = room - (long long)Shape::sum_bytes(wk, x_rows, pass);
                if (x_room < (long long)Shape::x_bytes(x_rows, 1)) continue;
                int part = (int)(x_room / (long long)Shape::x_bytes(x_rows, 1));
                part = part > windows ? windows : part;
                const int parts = ceil_div(windows, part);
                part = ceil_div(ceil_div(windows, parts), wk) * wk <= part ? ceil_div(ceil_div(windows, parts), wk) * wk : part;
                part = part > windows ? windows : part;
                const int real_parts = ceil_div(windows, part);
                const long long per_tile = (long long)(real_parts - 1) * ceil_div(part, wk) + ceil_div(windows - (real_parts - 1) * part, wk);
                const long long staged = (long long)windows * x_rows * (real_parts > 1 ? passes : 1);
                const long long cost = per_sm * (passes * ceil_div(pass, row_warps) * per_tile * 2 * kWindowClocks + staged * 4) +
                                       passes * (split > 1 ? 2000 : 400) + (real_parts > 1 ? passes * real_parts * 1500 : 0);
                if (least >= 0 && cost >= least) continue;
                least = cost;
                best = W4Plan{split, wk, pass, real_parts, part, clusters, per_sm,
                              Shape::kRing + Shape::sum_bytes(wk, x_rows, pass) + Shape::x_bytes(x_rows, part)};
            }
        }
    }
    return best;
}

template <int NT, int STAGES, bool BF, int G>
cudaError_t launch_w4(W4Params p, int sms, cudaStream_t st) {
    static std::atomic<unsigned long long> ready{0};       // devices whose shared-memory limit has been raised
    const int chunks = ceil_div(p.T, 8 * NT);
    p.tiles = ceil_div(p.N, 16);
    p.windows = ceil_div(p.K, kWindow);
    p.x_rows = p.T < 8 * NT ? p.T : 8 * NT;
    // a decode loop asks for the same few shapes again and again: the last ones' plans are kept, by their sizes
    struct Known {
        int tiles, windows, x_rows, chunks, sms;
        W4Plan plan;
    };
    static thread_local Known known[8];
    Known& k = known[(unsigned)(p.tiles * 31 + p.windows * 7 + p.x_rows) % 8];
    if (k.tiles != p.tiles || k.windows != p.windows || k.x_rows != p.x_rows || k.chunks != chunks || k.sms != sms)
        k = Known{p.tiles, p.windows, p.x_rows, chunks, sms, plan_w4<NT, STAGES, BF, G>(p.tiles, p.windows, p.x_rows, chunks, sms)};
    cut_w4(&p, k.plan);
    p.wk = k.plan.wk;
    p.pass_tiles = k.plan.pass_tiles;
    p.parts = k.plan.parts;
    p.part_windows = k.plan.part_windows;
    return start(&ready, p, k.plan.clusters, chunks, 256, k.plan.smem, st, w4_linear_kernel<NT, STAGES, BF, G>, kBits<BF, NT == 1>);
}

template <int TP, int STAGES, int G>
W4Plan plan_few(int tiles_all, int windows_all, int tokens, int sms) {
    using Shape = FewShape<TP, STAGES, G>;
    W4Plan best{};
    long long least = -1;
    for (int split = 1; split <= 8 && split <= windows_all; split *= 2) {
        const int windows = ceil_div(windows_all, split);
        for (int per_sm = FEW_BLOCKS; per_sm >= 1; --per_sm) {
            const long long room = kSmSmem / per_sm - 1024 - Shape::kRing;
            const int slots = sms * per_sm / split;
            const int clusters = tiles_all < slots ? tiles_all : slots < 1 ? 1 : slots;
            const int tiles = ceil_div(tiles_all, clusters);
            // sums of the block's rows get up to a third of the room, tokens the rest
            int passes = 1;
            while (ceil_div(tiles, passes) > 1 && (long long)Shape::sum_bytes(tokens, ceil_div(tiles, passes)) > room / 3) ++passes;
            const int pass = ceil_div(tiles, passes);
            const long long x_room = room - (long long)Shape::sum_bytes(tokens, pass);
            if (x_room < (long long)Shape::x_bytes(tokens, 1)) continue;
            int part = (int)(x_room / (long long)Shape::x_bytes(tokens, 1));
            part = part >= windows ? windows : part;
            const int parts = ceil_div(windows, part);
            // clocks: a warp's windows, at the pace of an SM's warps together or of one alone; its tokens; the ends
            const long long run = (long long)passes * parts * (ceil_div((long long)pass * part, Shape::kWarps) + 1);
            const long long step = per_sm * 2 * (150 + 45 * Shape::kTiles) > 900 ? per_sm * 2 * (150 + 45 * Shape::kTiles) : 900;
            const long long staged = (long long)ceil_div((long long)windows * tokens, Shape::kWarps) * (parts > 1 ? passes : 1);
            const long long cost = run * step + staged * (per_sm * 200 > 300 ? per_sm * 200 : 300) + passes * (split > 1 ? 3000 : 500) +
                                   (parts > 1 ? (long long)passes * parts * 1500 : 0);
            if (least >= 0 && cost >= least) continue;
            least = cost;
            best = W4Plan{split, Shape::kWarps, pass, parts, part, clusters, per_sm,
                          Shape::kRing + Shape::sum_bytes(tokens, pass) + Shape::x_bytes(tokens, part)};
        }
    }
    return best;
}

template <int TP, int STAGES, bool BF, int G>
cudaError_t launch_few(W4Params p, int sms, cudaStream_t st) {
    static std::atomic<unsigned long long> ready{0};       // devices whose shared-memory limit has been raised
    p.tiles = ceil_div(p.N, 16);
    p.windows = ceil_div(p.K, kFewWindow);
    const W4Plan plan = plan_few<TP, STAGES, G>(p.tiles, p.windows, p.T, sms);
    cut_w4(&p, plan);
    p.pass_tiles = plan.pass_tiles;
    p.parts = plan.parts;
    p.part_windows = plan.part_windows;
    return start(&ready, p, plan.clusters, 1, 256, plan.smem, st, w4_few_kernel<TP, STAGES, BF, G>);
}

template <bool BF, int G>
cudaError_t launch_tokens(const W4Params& p, int sms, cudaStream_t st) {
    if (p.T <= 2) return launch_few<2, FEW_STAGES, BF, G>(p, sms, st);
    if (p.T <= 4) return launch_few<4, FEW_STAGES, BF, G>(p, sms, st);
    if (p.T <= 8) return launch_few<8, FEW_STAGES, BF, G>(p, sms, st);
    if (p.T <= 16) return launch_w4<2, 3, BF, G>(p, sms, st);
    return launch_w4<4, 3, BF, G>(p, sms, st);
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
    if (T > (1 << 20) || N > (1 << 30) || K > (1 << 24)) return SASQ_ERR_UNSUPPORTED;
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
