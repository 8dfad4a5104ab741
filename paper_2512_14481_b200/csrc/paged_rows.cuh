// Attention for few query rows per KV head (decode steps, drafts): at most 8 * NB rows an item.
#pragma once

#include "paged_common.cuh"

namespace sasq {

struct AttendParams {
    PagedParams c;
    const uint16_t* q;
    uint16_t* out;
    float* lse;                 // [total_q][heads] or nullptr
    long long q_stride, out_stride;
    int heads, group;           // query heads, query heads per KV head
    float scale;                // softmax_scale * log2(e)
    int causal;
    int split;                  // items may be cut among blocks (the joining launch follows)
    int max_blocks;
    int item_rows;              // rows of an item
    int tile_bound;             // few-row kernel in clusters: row tiles of a sequence and KV head, by the host's bound
    PartItem* part_items;       // [max_blocks]
    float2* part_ml;            // [2 * max_blocks][R]: maximum (log2 units) and sum
    float* part_o;              // [2 * max_blocks][R][D]
    long long wait_limit;
};

namespace {

// Blocks of 16 keys of a warp's step: with 8 rows as many bytes are under way whatever the cache holds (16 rows' sums leave
// no registers for that), and keys of a unit: a step of four warps.
template <int NB, bool INT8>
constexpr int kRowsSub = INT8 && NB == 1 ? 2 : 1;
template <int NB, bool INT8>
constexpr int kRowsUnit = 64 * kRowsSub<NB, INT8>;
constexpr int kClusterBlocks = 8;
// units that beginning and ending an item costs (64 ragged sequences of 30 to 4500 keys, 32/8 heads: 112.4 us with 0,
// 101.9 with 2, 103.8 with 4, 107.0 with 6)
constexpr int kRowsItemCost = 2;
// A row's reference moves once a logit passes what it was set for by this many powers of two.
constexpr float kRescaleAt = 8.0f;
// It is set this many powers of two below the row's maximum.  Probabilities that the second product takes as f16 then use
// that type's range: at most 2^15, and off by 2^-32 of the row's maximum where they are too small for f16's normal numbers
// (2^-25 with a reference at the maximum: of 2^20 faint keys beside a loud one, together 3 % of the row's sum, nothing
// would be left).  bf16 has fp32's range.
template <bool F16>
constexpr float kHeadroom = F16 ? 7.0f : 0.0f;

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool bf) {
    if (bf)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// the same shared-memory location in block `rank` of the cluster
__device__ __forceinline__ uint32_t peer_address(const void* p, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float peer_load(uint32_t address) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(address));
    return v;
}
__device__ __forceinline__ float4 peer_load4(uint32_t address) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(address));
    return v;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint4 ldg_stream16(const void* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint2 ldg_stream8(const void* p) {
    uint2 v;
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}

// Blocks that an SM holds: as many as the registers of the fragments leave room for.  At this bound the variants for 8 rows
// over int8 codes spill 4 to 20 bytes a thread, outside the loop over the keys (2072 local loads in a launch of 1776 warps).
template <int D, int NB, bool INT8>
constexpr int kRowsBlocksPerSm = NB == 2 ? 2 : D == 128 ? 3 : 4;

// Both products are taken transposed, keys (then dimensions) on the 16-row side of m16n8k16 and query rows on its
// 8-column side, so that one query row wastes 7/8 of the instruction and not 15/16, and neither K nor V passes through
// shared memory: a contraction may run over its index in any order, so a lane simply takes the 16 bytes of a key that
// it loaded as its fragment of the next two or four instructions, and the queries are laid out to match.  For V, pairs
// of keys are interleaved with byte permutes.  Every warp has its own 16 keys of each stretch, its own running
// maximum, sum and accumulators; the warps meet once, at the end of the item.
// Bound by DRAM: 64 ragged sequences of 30 to 4500 keys, 32/8 heads, bf16, 594 MB: 101 us, 5.9 TB/s, 91 % of a plain copy's
// rate; 328 MB of int8 codes: 71 us, 4.6 TB/s, where the codes' conversion counts as well.
//
// CLUSTER: a cluster of eight blocks has an item to itself, each block an eighth of its units, and the blocks' sums meet
// through distributed shared memory: no scan of the batch, no second launch.
template <int D, int NB, bool BF, bool INT8, bool CLUSTER, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, WARPS == 4 ? kRowsBlocksPerSm<D, NB, INT8> : 1) paged_rows_kernel(const __grid_constant__ AttendParams p) {
    constexpr int R = 8 * NB, kThreads = 32 * WARPS;
    // The products' 16-bit type: codes become f16 in five instructions for four and bf16 in eight, so with an int8 cache
    // both products are f16.  A bf16 query row is brought into f16's range by a power of two; elements below 2^-14 of the
    // row's largest then lose bits that are worth less than 2^-25 of it.
    constexpr bool PBF = BF && !INT8;
    constexpr int SUB = kRowsSub<NB, INT8>, kUnit = kRowsUnit<NB, INT8>;
    constexpr int kStride = 16 * SUB * WARPS;               // keys from a warp's step to its next
    constexpr int kWords = INT8 ? D / 64 : D / 32;          // 16-byte words of a key that a lane takes
    constexpr int kSteps = D / 16;                          // k16 steps of S, and 16-row blocks of O
    constexpr int VW = D / 8 * (INT8 ? 1 : 2) / 4;          // 32-bit words of a V row that a lane takes: D / 8 elements

    __shared__ float sm_m[WARPS][R], sm_l[WARPS][R];
    __shared__ float2 block_ml[R];                            // CLUSTER: the block's references and sums
    __shared__ alignas(16) float sm_o[WARPS][R][D];         // read back four at a time

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, j = lane & 3;
    pdl_launch_dependents();
    pdl_wait();
    const Schedule<kUnit, kRowsItemCost> sch{R, p.group, p.causal, p.c.kv_heads};
    const int rank = blockIdx.x % kClusterBlocks;             // CLUSTER: of the block in its cluster
    Walk<kUnit, kRowsItemCost> walk;
    Start st;
    bool more;
    if constexpr (CLUSTER) {
        // cluster id = (sequence, KV head, first row tile); the tiles behind the host's bound come round again
        const int id = blockIdx.x / kClusterBlocks, per_seq = p.c.kv_heads * p.tile_bound;
        walk.it.b = id / per_seq;
        walk.it.h = id % per_seq / p.tile_bound;
        walk.it.i = id % p.tile_bound;
        walk.it.s = load_sequence(p.c, walk.it.b);
        walk.n_tiles = sch.tiles(walk.it.s);
        more = walk.it.i < walk.n_tiles;
    } else {
        st = find_start(p.c, sch, p.max_blocks);
        if (tid == 0) p.part_items[blockIdx.x].last = -1;
        more = walk.begin(p.c, sch, st, p.split != 0);
    }
    while (more) {
        if constexpr (CLUSTER) {
            walk.it.units = sch.units(walk.it.s, walk.it.i);
            walk.it.t0 = (int)((long long)walk.it.units * rank / kClusterBlocks);
            walk.it.t1 = (int)((long long)walk.it.units * (rank + 1) / kClusterBlocks);
        }
        const Item it = walk.it;
        const int rows_all = it.s.new_len * p.group;
        const int first_row = it.i * R;
        const int rows = min(R, rows_all - first_row);
        const int limit = sch.key_limit(it.s, it.i);
        const float scale = INT8 ? p.scale * __ldg(p.c.k_scale + it.h) : p.scale;
        if (INT8 && tid == 0 && (scale_is_bad(__ldg(p.c.k_scale + it.h)) || scale_is_bad(__ldg(p.c.v_scale + it.h))))
            atomicMax(p.c.status, (int)SASQ_ERR_BAD_SCALE);

        // queries: the fragment of row g of each block of 8 rows, in the order of the keys' words
        uint32_t qf[NB][2 * kSteps];
        int row_limit[NB][2];                                // keys that rows 2j, 2j + 1 see
        float row_scale[NB][2];                              // and what turns their products into powers of two
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int r = first_row + nb * 8 + g;
            const bool valid = r < rows_all;
            const int tok = valid ? r / p.group : 0;
            const uint16_t* qr = p.q + (long long)(it.s.first + tok) * p.q_stride +
                                 (long long)(it.h * p.group + (valid ? r - tok * p.group : 0)) * D;
#pragma unroll
            for (int w = 0; w < 2 * kSteps / 4; ++w) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (valid) {
                    // int8: a lane's 16 codes of a key's word feed 16 elements, here in two halves
                    const int at = INT8 ? 16 * (j + 4 * (w >> 1)) + 8 * (w & 1) : 8 * (j + 4 * w);
                    v = *reinterpret_cast<const uint4*>(qr + at);
                }
                qf[nb][4 * w] = v.x;
                qf[nb][4 * w + 1] = v.y;
                qf[nb][4 * w + 2] = v.z;
                qf[nb][4 * w + 3] = v.w;
            }
            float unit = 1.0f;                               // of row g's f16 queries
            if constexpr (BF && INT8) {
                float big = 0.0f;
#pragma unroll
                for (int w = 0; w < 2 * kSteps; ++w) {
                    const float2 f = widen2<true>(qf[nb][w]);
                    big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
                }
                big = fmaxf(big, __shfl_xor_sync(0xFFFFFFFFu, big, 1));
                big = fmaxf(big, __shfl_xor_sync(0xFFFFFFFFu, big, 2));
                // the power of two at or below the largest, kept where its reciprocal is a normal number
                const uint32_t top = min(max(__float_as_uint(big) & 0x7F800000u, 0x01000000u), 0x7E000000u);
                unit = __uint_as_float(top);
                const float inv = __uint_as_float(0x7F000000u - top);
#pragma unroll
                for (int w = 0; w < 2 * kSteps; ++w) {
                    const float2 f = widen2<true>(qf[nb][w]);
                    qf[nb][w] = narrow2<false>(f.x * inv, f.y * inv);
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) row_scale[nb][e] = scale * __shfl_sync(0xFFFFFFFFu, unit, 4 * (2 * j + e));
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int rr = first_row + nb * 8 + 2 * j + e;
                const int lim = p.causal ? it.s.len - it.s.new_len + rr / p.group + 1 : it.s.len;
                row_limit[nb][e] = min(lim, limit);
            }
        }

        float o[kSteps][NB][4];
        float m[NB][2], l[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m[nb][0] = m[nb][1] = -INFINITY;
            l[nb][0] = l[nb][1] = 0.0f;
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[k][nb][e] = 0.0f;
        }

        const int elem = INT8 ? 1 : 2;
        const int* table = p.c.page_table + it.b * p.c.table_stride;
        const char* kbase = static_cast<const char*>(p.c.k) + it.h * p.c.head_stride * elem;
        const char* vbase = static_cast<const char*>(p.c.v) + it.h * p.c.head_stride * elem;
        const int page_mask = (1 << p.c.page_shift) - 1;
        const int last_key = min(it.t1 * kUnit, limit);
        int key = it.t0 * kUnit + warp * 16 * SUB;           // of this warp's step

        // byte offset of key `at` of the sequence, or -1 when there is none or its page lies outside the cache
        auto place = [&](int at) -> long long {
            if (at >= last_key) return -1;
            const int page = __ldg(table + (at >> p.c.page_shift));
            if (page < 0 || page >= p.c.num_pages) {
                atomicMax(p.c.status, (int)SASQ_ERR_BAD_INDEX);
                return -1;
            }
            return (page * p.c.page_stride + (at & page_mask) * p.c.token_stride) * elem;
        };
        uint4 kws[SUB][2][kWords];                            // keys g and g + 8
        auto load_k = [&](int at, long long off, uint4 (&kw)[2][kWords]) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const bool in = off >= 0 && at + g + 8 * r < last_key;
                const char* row = kbase + off + (long long)(g + 8 * r) * p.c.token_stride * elem;
#pragma unroll
                for (int w = 0; w < kWords; ++w)
                    kw[r][w] = in ? ldg_stream16(row + 16 * (j + 4 * w)) : make_uint4(0, 0, 0, 0);
            }
        };
        uint32_t vws[SUB][4][VW];                             // keys 2j, 2j + 1, 2j + 8, 2j + 9
        auto load_v = [&](int at, long long off, uint32_t (&vw)[4][VW]) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int kk = 2 * j + (r & 1) + 8 * (r >> 1);
                const bool in = off >= 0 && at + kk < last_key;
                const char* row = vbase + off + (long long)kk * p.c.token_stride * elem;
                if constexpr (VW == 2) {
                    const uint2 v = in ? ldg_stream8(row + 8 * g) : make_uint2(0, 0);
                    vw[r][0] = v.x;
                    vw[r][1] = v.y;
                } else {
#pragma unroll
                    for (int w = 0; w < VW / 4; ++w) {
                        const uint4 v = in ? ldg_stream16(row + 16 * (g + 8 * w)) : make_uint4(0, 0, 0, 0);
                        vw[r][4 * w] = v.x;
                        vw[r][4 * w + 1] = v.y;
                        vw[r][4 * w + 2] = v.z;
                        vw[r][4 * w + 3] = v.w;
                    }
                }
            }
        };

        long long off[SUB], off_next[SUB];
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            off[u] = place(key + 16 * u);
            load_k(key + 16 * u, off[u], kws[u]);
        }
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            load_v(key + 16 * u, off[u], vws[u]);
            off_next[u] = place(key + kStride + 16 * u);
        }
        while (key < last_key) {
            // S^T of the step's keys: rows are keys, columns query rows
            float s[SUB][NB][4];
            const int key_now = key, key_next = key + kStride;
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[u][nb][e] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWords; ++w) {
                    const uint32_t k0[4] = {kws[u][0][w].x, kws[u][0][w].y, kws[u][0][w].z, kws[u][0][w].w};
                    const uint32_t k1[4] = {kws[u][1][w].x, kws[u][1][w].y, kws[u][1][w].z, kws[u][1][w].w};
                    if constexpr (INT8) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t a[4] = {codes_to_pair<false, 0>(k0[e]), codes_to_pair<false, 0>(k1[e]),
                                                   codes_to_pair<false, 1>(k0[e]), codes_to_pair<false, 1>(k1[e])};
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb)
                                mma_16816(s[u][nb], a, qf[nb][8 * w + 2 * e], qf[nb][8 * w + 2 * e + 1], PBF);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t a[4] = {k0[2 * e], k1[2 * e], k0[2 * e + 1], k1[2 * e + 1]};
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb)
                                mma_16816(s[u][nb], a, qf[nb][4 * w + 2 * e], qf[nb][4 * w + 2 * e + 1], PBF);
                        }
                    }
                }
                // the next step's keys travel under this step's softmax
                off[u] = off_next[u];
                load_k(key_next + 16 * u, off[u], kws[u]);
                off_next[u] = place(key_next + kStride + 16 * u);
            }

            // running reference and sum in powers of two; a row's reference m only moves when a logit has passed it by
            // enough, so that most steps need neither the shuffles nor the rescaling (P stays below
            // 2^(kRescaleAt + kHeadroom))
            bool moves = false;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int at = key_now + 16 * u + g + 8 * (e >> 1);
                        s[u][nb][e] = at < row_limit[nb][e & 1] ? s[u][nb][e] * row_scale[nb][e & 1] : -INFINITY;
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) moves |= fmaxf(s[u][nb][e], s[u][nb][e + 2]) > m[nb][e] + (kRescaleAt + kHeadroom<!PBF>);
                }
            if (__any_sync(0xFFFFFFFFu, moves)) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float t = fmaxf(s[0][nb][e], s[0][nb][e + 2]);
#pragma unroll
                        for (int u = 1; u < SUB; ++u) t = fmaxf(t, fmaxf(s[u][nb][e], s[u][nb][e + 2]));
                        t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 4));
                        t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 8));
                        t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 16));
                        const float m_new = fmaxf(m[nb][e], t - kHeadroom<!PBF>);
                        const float f = m_new == -INFINITY ? 1.0f : exp2_approx(m[nb][e] - m_new);
                        m[nb][e] = m_new;
                        l[nb][e] *= f;
#pragma unroll
                        for (int k = 0; k < kSteps; ++k) {
                            o[k][nb][e] *= f;
                            o[k][nb][e + 2] *= f;
                        }
                    }
            }
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                uint32_t pf[NB][2];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    float pr[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float ref = m[nb][e & 1] == -INFINITY ? 0.0f : m[nb][e & 1];
                        pr[e] = exp2_approx(s[u][nb][e] - ref);
                        l[nb][e & 1] += pr[e];
                    }
                    pf[nb][0] = transpose_8x8(narrow2<PBF>(pr[0], pr[1]));
                    pf[nb][1] = transpose_8x8(narrow2<PBF>(pr[2], pr[3]));
                }

                // O^T += V^T P^T: rows are dimensions, the contraction is over 16 keys
                const uint32_t (&vw)[4][VW] = vws[u];
                if constexpr (INT8) {
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        const uint32_t x0 = __byte_perm(vw[0][w], vw[1][w], 0x5140), x1 = __byte_perm(vw[0][w], vw[1][w], 0x7362);
                        const uint32_t y0 = __byte_perm(vw[2][w], vw[3][w], 0x5140), y1 = __byte_perm(vw[2][w], vw[3][w], 0x7362);
                        const uint32_t a0[4] = {codes_to_pair<false, 0>(x0), codes_to_pair<false, 1>(x0), codes_to_pair<false, 0>(y0),
                                                codes_to_pair<false, 1>(y0)};
                        const uint32_t a1[4] = {codes_to_pair<false, 0>(x1), codes_to_pair<false, 1>(x1), codes_to_pair<false, 0>(y1),
                                                codes_to_pair<false, 1>(y1)};
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            mma_16816(o[2 * w][nb], a0, pf[nb][0], pf[nb][1], PBF);
                            mma_16816(o[2 * w + 1][nb], a1, pf[nb][0], pf[nb][1], PBF);
                        }
                    }
                } else {
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        const uint32_t a[4] = {__byte_perm(vw[0][w], vw[1][w], 0x5410), __byte_perm(vw[0][w], vw[1][w], 0x7632),
                                               __byte_perm(vw[2][w], vw[3][w], 0x5410), __byte_perm(vw[2][w], vw[3][w], 0x7632)};
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) mma_16816(o[w][nb], a, pf[nb][0], pf[nb][1], PBF);
                    }
                }
                load_v(key_next + 16 * u, off[u], vws[u]);
            }
            key = key_next;
        }

        // the warps' sums meet in shared memory
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float t = l[nb][e];
                t += __shfl_xor_sync(0xFFFFFFFFu, t, 4);
                t += __shfl_xor_sync(0xFFFFFFFFu, t, 8);
                t += __shfl_xor_sync(0xFFFFFFFFu, t, 16);
                const int r = nb * 8 + 2 * j + e;
                if (g == 0) {
                    sm_m[warp][r] = m[nb][e];
                    sm_l[warp][r] = t;
                }
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    // block k holds, of lane group g, the dimensions at and at + 1
                    const int at = INT8 ? (D / 8) * g + 2 * k : 8 * (g + 8 * (k >> 2)) + 2 * (k & 3);
                    *reinterpret_cast<float2*>(&sm_o[warp][r][at]) = make_float2(o[k][nb][e], o[k][nb][e + 2]);
                }
            }
        __syncthreads();
        const bool whole = !CLUSTER && it.t0 == 0 && it.t1 == it.units;
        const int slot = 2 * blockIdx.x + (it.t0 == 0 ? 1 : 0);
        const float vs = INT8 ? __ldg(p.c.v_scale + it.h) : 1.0f;
        // four elements of the item's result
        auto write = [&](int r, int d, float m, float sum, const float (&acc)[4]) {
            const float inv = sum != 0.0f ? vs / sum : 0.0f;      // 0: a row without keys; NaN is not one
            const int row = first_row + r, tok = row / p.group;
            const int head = it.h * p.group + row - tok * p.group;
            const long long t = it.s.first + tok;
            *reinterpret_cast<uint2*>(p.out + t * p.out_stride + (long long)head * D + d) =
                make_uint2(narrow2<BF>(acc[0] * inv, acc[1] * inv), narrow2<BF>(acc[2] * inv, acc[3] * inv));
            if (d == 0 && p.lse != nullptr)
                p.lse[t * p.heads + head] = sum != 0.0f ? (m + log2f(sum)) * 0.6931471805599453f : -INFINITY;
        };
        for (int x = tid * 4; x < rows * D; x += kThreads * 4) {
            const int r = x / D, d = x % D;
            float mm = sm_m[0][r];
#pragma unroll
            for (int w = 1; w < WARPS; ++w) mm = fmaxf(mm, sm_m[w][r]);
            const float ref = mm == -INFINITY ? 0.0f : mm;
            float sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float f = exp2_approx(sm_m[w][r] - ref);
                const float4 v = *reinterpret_cast<const float4*>(&sm_o[w][r][d]);
                sum += f * sm_l[w][r];
                acc[0] += f * v.x;
                acc[1] += f * v.y;
                acc[2] += f * v.z;
                acc[3] += f * v.w;
            }
            if constexpr (CLUSTER) {
                // only this thread has to do with these elements: the block's sum takes the place of the first warp's
                *reinterpret_cast<float4*>(&sm_o[0][r][d]) = make_float4(acc[0], acc[1], acc[2], acc[3]);
                if (d == 0) block_ml[r] = make_float2(mm, sum);
            } else if (whole) {
                write(r, d, mm, sum, acc);
            } else {
                *reinterpret_cast<float4*>(p.part_o + ((long long)slot * R + r) * D + d) = make_float4(acc[0], acc[1], acc[2], acc[3]);
                if (d == 0) p.part_ml[(long long)slot * R + r] = make_float2(mm, sum);
            }
        }
        if constexpr (CLUSTER) {
            cluster_barrier();
            // every block joins its share of the elements
            for (int x = (rank * kThreads + tid) * 4; x < rows * D; x += kClusterBlocks * kThreads * 4) {
                const int r = x / D, d = x % D;
                float m8[kClusterBlocks], l8[kClusterBlocks];
                float4 v[kClusterBlocks];
                float mm = -INFINITY;
#pragma unroll
                for (int k = 0; k < kClusterBlocks; ++k) {
                    m8[k] = peer_load(peer_address(&block_ml[r].x, k));
                    l8[k] = peer_load(peer_address(&block_ml[r].y, k));
                    v[k] = peer_load4(peer_address(&sm_o[0][r][d], k));
                }
#pragma unroll
                for (int k = 0; k < kClusterBlocks; ++k) mm = fmaxf(mm, m8[k]);
                const float ref = mm == -INFINITY ? 0.0f : mm;
                float sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < kClusterBlocks; ++k) {
                    const float f = exp2_approx(m8[k] - ref);
                    sum += f * l8[k];
                    acc[0] += f * v[k].x;
                    acc[1] += f * v[k].y;
                    acc[2] += f * v[k].z;
                    acc[3] += f * v[k].w;
                }
                write(r, d, mm, sum, acc);
            }
            cluster_barrier();                                 // nobody leaves, or goes on, while its sums are being read
            walk.it.i += p.tile_bound;
            more = walk.it.i < walk.n_tiles;
            continue;
        }
        if (!whole && it.t0 == 0 && tid == 0) {
            PartItem pi;
            pi.last = walk.last_block(st);
            pi.h = it.h;
            pi.first_row = first_row;
            pi.rows = rows;
            pi.first_token = it.s.first;
            pi.tile_rows = R;
            p.part_items[blockIdx.x] = pi;
        }
        __syncthreads();                                       // the next item reuses the shared memory
        more = walk.next(p.c);
    }
}

// Joins the parts of the item that began in block x and ended in a later one.  The parts lie in the second slot of block x
// and in the first slots of the blocks after it.  R rows of a slot, in row tiles of TILE of which an item may use fewer.
// WIDE: a block per row, its eight warps taking the parts in turn (few rows, long keys: up to hundreds of parts); else a
// warp per row (many rows, two or three parts).  The order of additions is fixed either way.
template <int R, int TILE, int D, bool BF, bool WIDE>
__global__ void __launch_bounds__(256) paged_join_kernel(const __grid_constant__ AttendParams p) {
    constexpr int N = D / 32;                                  // elements of a lane
    __shared__ float warp_m[8], warp_sum[8];
    __shared__ alignas(16) float warp_o[8][WIDE ? D : 4];
    pdl_launch_dependents();
    pdl_wait();
    const int c = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const PartItem pi = p.part_items[c];
    if (pi.last < 0) return;
    const float vs = p.c.v_scale != nullptr ? __ldg(p.c.v_scale + pi.h) : 1.0f;
    constexpr int kStep = WIDE ? 8 : 1;                        // parts from one of a warp to its next
    for (int r = WIDE ? blockIdx.y : blockIdx.y * 8 + warp; r < R; r += WIDE ? gridDim.y : gridDim.y * 8) {
        const int item_row = r / TILE * pi.tile_rows + r % TILE;
        if (r % TILE >= pi.tile_rows || item_row >= pi.rows) continue;
        auto slot_of = [&](int k) { return (long long)(k == c ? 2 * c + 1 : 2 * k) * R + r; };
        const int first = WIDE ? c + warp : c;
        float m = -INFINITY;
        for (int k = first + kStep * lane; k <= pi.last; k += kStep * 32) m = fmaxf(m, p.part_ml[slot_of(k)].x);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, off));
        float ref = m == -INFINITY ? 0.0f : m;
        float sum = 0.0f, acc[N];
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = 0.0f;
        auto add = [&](float f, float s, const float* src) {
            sum += f * s;
            if constexpr (N == 4) {
                const float4 v = *reinterpret_cast<const float4*>(src);
                acc[0] += f * v.x;
                acc[1] += f * v.y;
                acc[2] += f * v.z;
                acc[3] += f * v.w;
            } else {
                const float2 v = *reinterpret_cast<const float2*>(src);
                acc[0] += f * v.x;
                acc[1] += f * v.y;
            }
        };
#pragma unroll 4
        for (int k = first; k <= pi.last; k += kStep) {
            const long long s = slot_of(k);
            const float2 ml = p.part_ml[s];
            add(exp2_approx(ml.x - ref), ml.y, p.part_o + s * D + lane * N);
        }
        if constexpr (WIDE) {
            if (lane == 0) {
                warp_m[warp] = m;
                warp_sum[warp] = sum;
            }
#pragma unroll
            for (int e = 0; e < N; ++e) warp_o[warp][lane * N + e] = acc[e];
            __syncthreads();
            if (warp == 0) {
                m = warp_m[0];
#pragma unroll
                for (int w = 1; w < 8; ++w) m = fmaxf(m, warp_m[w]);
                ref = m == -INFINITY ? 0.0f : m;
                sum = 0.0f;
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] = 0.0f;
#pragma unroll
                for (int w = 0; w < 8; ++w) add(exp2_approx(warp_m[w] - ref), warp_sum[w], &warp_o[w][lane * N]);
            }
            __syncthreads();
            if (warp != 0) continue;
        }
        const float inv = sum != 0.0f ? vs / sum : 0.0f;
        const int row = pi.first_row + item_row, tok = row / p.group;
        const int head = pi.h * p.group + row - tok * p.group;
        const long long t = pi.first_token + tok;
        uint32_t* dst = reinterpret_cast<uint32_t*>(p.out + t * p.out_stride + (long long)head * D + lane * N);
#pragma unroll
        for (int e = 0; e < N / 2; ++e) dst[e] = narrow2<BF>(acc[2 * e] * inv, acc[2 * e + 1] * inv);
        if (lane == 0 && p.lse != nullptr)
            p.lse[t * p.heads + head] = sum != 0.0f ? (m + log2f(sum)) * 0.6931471805599453f : -INFINITY;
    }
}

}  // namespace
}  // namespace sasq
