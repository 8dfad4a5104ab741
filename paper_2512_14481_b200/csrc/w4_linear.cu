// Linear layers with 4-bit weights and group factors for few tokens, and the quantizer that makes such weights.
//
//   y[t, n] = narrow( sum_g s[n, g] * sum_{k in group g} x[t, k] c[n, k]  (+ bias[n]) )
//
// Bound by the weights: half a byte each, read once.  The products run on mma.sync m16n8k16 with 16 rows of weights on its
// wide side and 8 tokens on the other: one token wastes 7/8 of an instruction whose rate is no limit, and a weight goes from
// its byte to the operand in registers, where its group's factor can be applied to the group's fp32 sum.
#include <atomic>

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
    int tiles;                  // row tiles
    int windows;                // of 128 columns
    int x_rows;                 // token rows of a slot
    int split;                  // blocks of a cluster, each with a share of the windows
};

constexpr int kWindow = 128;    // columns of a step: 64 bytes of a weight row
constexpr int kXPitch = 320;    // bytes from a token's window to the next token's: neighbours lie in different banks

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

// 16 bytes from global to shared memory without a register; `there` == false writes zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
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

// Eight codes of a word -> the pairs (0, 4), (1, 5), (2, 6), (3, 7) as exact 16-bit floats.  With the sign bit flipped a nibble
// is u = code + 8.  bf16: 0x4300 | u stands for 128 + u, less 136.  f16: 0x6400 | u is 1024 + u, less 1032; one nibble further
// up it is 1024 + 16 u, which one fused multiply-add brings to the code without a shift.
template <bool BF>
__device__ __forceinline__ void unpack8(uint32_t w, uint32_t (&p)[4]) {
    if constexpr (BF) {
        const uint32_t off = 0x43084308u;
        const uint32_t bias = 0x43084308u;                 // 136
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t t = ((w >> (4 * i)) & 0x000F000Fu) ^ off;
            const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&t), *reinterpret_cast<const __nv_bfloat162*>(&bias));
            p[i] = *reinterpret_cast<const uint32_t*>(&d);
        }
    } else {
        const uint32_t bias = 0x64086408u, sixteenth = 0x2C002C00u, minus72 = 0xD480D480u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t v = w >> (8 * i);
            const uint32_t lo = (v & 0x000F000Fu) ^ 0x64086408u, hi = (v & 0x00F000F0u) ^ 0x64806480u;
            const __half2 a = __hsub2(*reinterpret_cast<const __half2*>(&lo), *reinterpret_cast<const __half2*>(&bias));
            const __half2 b = __hfma2(*reinterpret_cast<const __half2*>(&hi), *reinterpret_cast<const __half2*>(&sixteenth),
                                      *reinterpret_cast<const __half2*>(&minus72));
            p[2 * i] = *reinterpret_cast<const uint32_t*>(&a);
            p[2 * i + 1] = *reinterpret_cast<const uint32_t*>(&b);
        }
    }
}

// NT blocks of 8 tokens; a warp has MT blocks of 16 rows; WR warps lie side by side on the rows and WK on the columns.
template <int NT, int MT, int WR, int WK, int STAGES>
struct W4Shape {
    static constexpr int kRows = 16 * MT * WR;             // of a tile
    static constexpr int kThreads = 32 * WR * WK;
    static constexpr int kSumPitch = kRows + 4;            // floats from a token's sums to the next token's
    static size_t slot(int x_rows) { return kRows * 64 + (size_t)x_rows * kXPitch; }
    static size_t smem(int x_rows) { return WK * STAGES * slot(x_rows) + (size_t)WK * 8 * NT * kSumPitch * sizeof(float); }
};

// A block walks row tiles; its windows of 128 columns go to the WK warps in turn, and each warp (or the WR warps that share
// a window's tokens) keeps STAGES - 1 windows of weights and tokens under way, across tiles too.
template <int NT, int MT, int WR, int WK, int STAGES, bool BF, int G>
__global__ void __launch_bounds__(32 * WR * WK, NT == 1 ? 2 : 1) w4_linear_kernel(const __grid_constant__ W4Params p) {
    using Shape = W4Shape<NT, MT, WR, WK, STAGES>;
    constexpr int R = Shape::kRows, RP = Shape::kSumPitch;
    constexpr int GW = kWindow / G, WG = G / 32;           // groups of a window, words of a lane in a group
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, j = lane & 3;
    const int wr = warp % WR, wk = warp / WR;
    const int rank = p.split > 1 ? (int)ptx::cluster_ctarank() : 0;
    const int first_tile = blockIdx.x / p.split, tile_step = gridDim.x / p.split;
    const int t0 = blockIdx.y * 8 * NT;                    // tokens of this block
    const int tokens = min(8 * NT, p.T - t0);
    const uint32_t slot_bytes = R * 64 + p.x_rows * kXPitch;
    const uint32_t ring = ptx::smem_u32(smem) + wk * STAGES * slot_bytes;
    float* const sums = reinterpret_cast<float*>(smem + (size_t)WK * STAGES * slot_bytes);
    // this block's windows, and how many of them are this warp's: windows begin + wk, + WK, ...
    const int begin = (int)((long long)p.windows * rank / p.split), end = (int)((long long)p.windows * (rank + 1) / p.split);
    const int mine = (end - begin - wk + WK - 1) / WK;
    pdl_launch_dependents();

    auto sync = [&] {
        if constexpr (WR == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + wk), "n"(32 * WR) : "memory");
    };
    // where the copies stand
    int load_tile = first_tile, load_n = 0, load_slot = 0;
    auto load_w = [&](uint32_t slot, int tile, int n) {
        const int byte = (begin + wk + n * WK) * 64 + 16 * j;
        const bool in = byte < (p.K >> 1);
#pragma unroll
        for (int r = 0; r < 2 * MT; ++r) {                 // 8 rows at a time of this warp's
            const int row = 16 * MT * wr + 8 * r + g;
            const int n_row = tile * R + row;
            copy16(slot + row * 64 + ((j ^ (row >> 1 & 3)) << 4), p.w + (long long)min(n_row, p.N - 1) * (p.K >> 1) + (in ? byte : 0), in && n_row < p.N);
        }
    };
    auto load_x = [&](uint32_t slot, int n) {
        const int col = (begin + wk + n * WK) * kWindow;
        for (int i = lane + 32 * wr; i < tokens * 16; i += 32 * WR) {
            const int t = i >> 4, c = i & 15;              // chunk of eight columns: group s, lane jj, word ii
            const int s = c / (G / 8), jj = c % (G / 8) / WG, ii = c % WG;
            const bool in = col + 8 * c < p.K;
            copy16(slot + R * 64 + t * kXPitch + ((s * WG + ii) * 4 + jj) * 16, p.x + (long long)(t0 + t) * p.K + (in ? col + 8 * c : 0), in);
        }
    };
    auto advance = [&] {
        if (++load_n >= mine) {
            load_n = 0;
            load_tile += tile_step;
        }
        if (++load_slot == STAGES) load_slot = 0;
    };
    auto loads_left = [&] { return mine > 0 && load_tile < p.tiles; };

    // weights may be read at once, tokens when the kernels before this one are done
    {
        int tile = load_tile, n = load_n;
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s)
            if (mine > 0 && tile < p.tiles) {
                load_w(ring + s * slot_bytes, tile, n);
                if (++n >= mine) {
                    n = 0;
                    tile += tile_step;
                }
            }
    }
    pdl_wait();
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        if (loads_left()) {
            load_x(ring + s * slot_bytes, load_n);
            advance();
        }
        copies_end_group();
    }

    int slot = 0;
    for (int tile = first_tile; tile < p.tiles; tile += tile_step) {
        float tot[MT][NT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) tot[m][nt][e] = 0.0f;
        for (int n = 0; n < mine; ++n) {
            const int window = begin + wk + n * WK;
            float sc[MT][2][GW];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int s = 0; s < GW; ++s) {
                        const int row = tile * R + 16 * MT * wr + 16 * m + 8 * r + g, group = window * GW + s;
                        sc[m][r][s] = row < p.N && group < p.groups ? widen1<BF>(__ldg(p.ws + (long long)row * p.groups + group)) : 0.0f;
                    }
            copies_wait<STAGES - 2>();
            sync();
            if (loads_left()) {
                const uint32_t to = ring + load_slot * slot_bytes;
                load_w(to, load_tile, load_n);
                load_x(to, load_n);
                advance();
            }
            copies_end_group();

            const uint32_t at = ring + slot * slot_bytes;
            if (++slot == STAGES) slot = 0;
            uint32_t wv[MT][2][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int row = 16 * MT * wr + 16 * m + 8 * r + g;
                    const uint32_t base = at + row * 64, turn = row >> 1 & 3;
                    if constexpr (G == 128) {
                        const uint4 v = lds16(base + ((j ^ turn) << 4));
                        wv[m][r][0] = v.x;
                        wv[m][r][1] = v.y;
                        wv[m][r][2] = v.z;
                        wv[m][r][3] = v.w;
                    } else if constexpr (G == 64) {
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const uint2 v = lds8(base + (((2 * s + (j >> 1)) ^ turn) << 4) + 8 * (j & 1));
                            wv[m][r][2 * s] = v.x;
                            wv[m][r][2 * s + 1] = v.y;
                        }
                    } else {
#pragma unroll
                        for (int s = 0; s < 4; ++s) wv[m][r][s] = lds4(base + ((s ^ turn) << 4) + 4 * j);
                    }
                }
            uint32_t x_at[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) x_at[nt] = at + R * 64 + min(8 * nt + g, p.x_rows - 1) * kXPitch + 16 * j;
#pragma unroll
            for (int s = 0; s < GW; ++s) {
                float acc[MT][NT][4];
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[m][nt][e] = 0.0f;
#pragma unroll
                for (int i = 0; i < WG; ++i) {
                    uint32_t a[MT][2][4];
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        uint32_t p0[4], p1[4];
                        unpack8<BF>(wv[m][0][s * WG + i], p0);
                        unpack8<BF>(wv[m][1][s * WG + i], p1);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            a[m][h][0] = p0[2 * h];
                            a[m][h][1] = p1[2 * h];
                            a[m][h][2] = p0[2 * h + 1];
                            a[m][h][3] = p1[2 * h + 1];
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint4 b = lds16(x_at[nt] + (s * WG + i) * 64);
                        const uint32_t b04 = __byte_perm(b.x, b.z, 0x5410), b15 = __byte_perm(b.x, b.z, 0x7632);
                        const uint32_t b26 = __byte_perm(b.y, b.w, 0x5410), b37 = __byte_perm(b.y, b.w, 0x7632);
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            mma_w4(acc[m][nt], a[m][0], b04, b15, BF);
                            mma_w4(acc[m][nt], a[m][1], b26, b37, BF);
                        }
                    }
                }
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) tot[m][nt][e] = fmaf(acc[m][nt][e], sc[m][e >> 1][s], tot[m][nt][e]);
            }
        }
        // the warps' (and the cluster's) sums meet in a fixed order
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sums[(wk * 8 * NT + 8 * nt + 2 * j + (e & 1)) * RP + 16 * MT * wr + 16 * m + 8 * (e >> 1) + g] = tot[m][nt][e];
        auto store = [&](int t, int row, float v) {
            const int n_row = tile * R + row;
            if (n_row >= p.N) return;
            if (p.bias != nullptr) v += widen1<BF>(p.bias[n_row]);
            p.y[(long long)(t0 + t) * p.N + n_row] = narrow1<BF>(v);
        };
        __syncthreads();
        if (p.split == 1) {
            for (int i = tid; i < tokens * R; i += Shape::kThreads) {
                const int t = i / R, row = i % R;
                float v = sums[t * RP + row];
#pragma unroll
                for (int k = 1; k < WK; ++k) v += sums[(k * 8 * NT + t) * RP + row];
                store(t, row, v);
            }
            __syncthreads();
        } else {
            for (int i = tid; i < tokens * R; i += Shape::kThreads) {
                const int t = i / R, row = i % R;
                float v = sums[t * RP + row];
#pragma unroll
                for (int k = 1; k < WK; ++k) v += sums[(k * 8 * NT + t) * RP + row];
                sums[t * RP + row] = v;
            }
            ptx::cluster_sync_all();
            for (int i = rank * Shape::kThreads + tid; i < tokens * R; i += p.split * Shape::kThreads) {
                const int t = i / R, row = i % R;
                const uint32_t at = ptx::smem_u32(&sums[t * RP + row]);
                float v = 0.0f;
                for (int k = 0; k < p.split; ++k) {
                    uint32_t peer;
                    float part;
                    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer) : "r"(at), "r"(k));
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part) : "r"(peer));
                    v += part;
                }
                store(t, row, v);
            }
            ptx::cluster_sync_all();                       // nobody goes on while its sums are being read
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

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

template <int NT, int MT, int WR, int WK, int STAGES, bool BF, int G>
cudaError_t launch_w4(W4Params p, int sms, cudaStream_t st) {
    using Shape = W4Shape<NT, MT, WR, WK, STAGES>;
    static std::atomic<unsigned long long> ready{0};       // devices whose shared-memory limit has been raised
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!(ready.load() >> (dev & 63) & 1)) {
        e = cudaFuncSetAttribute(w4_linear_kernel<NT, MT, WR, WK, STAGES, BF, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape::smem(8 * NT));
        if (e != cudaSuccess) return e;
        ready.fetch_or(1ull << (dev & 63));
    }
    p.tiles = ceil_div(p.N, Shape::kRows);
    p.windows = ceil_div(p.K, kWindow);
    p.x_rows = p.T < 8 * NT ? p.T : 8 * NT;
    const size_t smem = Shape::smem(p.x_rows);
    const int per_sm = NT == 1 && smem <= 113 * 1024 ? 2 : 1;
    const int chunks = ceil_div(p.T, 8 * NT);
    // few tiles: a tile's columns are shared by the blocks of a cluster
    p.split = 1;
    while (p.split < 8 && p.tiles * chunks * p.split * 2 <= sms * per_sm && p.windows >= 2 * p.split * WK) p.split *= 2;
    const int slots = sms * per_sm / p.split / chunks;
    const int clusters = p.tiles < slots ? p.tiles : slots < 1 ? 1 : slots;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(clusters * p.split), (unsigned)chunks);
    cfg.blockDim = dim3(Shape::kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0] = pdl_attribute();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, w4_linear_kernel<NT, MT, WR, WK, STAGES, BF, G>, p);
}

template <bool BF, int G>
cudaError_t launch_tokens(const W4Params& p, int sms, cudaStream_t st) {
    if (p.T <= 8) return launch_w4<1, 2, 1, 8, 4, BF, G>(p, sms, st);
    if (p.T <= 16) return launch_w4<2, 2, 2, 4, 4, BF, G>(p, sms, st);
    return launch_w4<4, 2, 4, 2, 4, BF, G>(p, sms, st);
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
