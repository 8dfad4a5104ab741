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

constexpr int kTileRows = 256;            // rows of an item: two MMA tiles of 128
constexpr int kTileKeys = 128;            // keys of a unit
constexpr int kTileThreads = 384;         // warps 0-3 and 4-7: softmax of either row tile; 8: MMA; 9: loads; 10, 11 idle
// registers a thread: 168 at launch (384 x 168 of the SM's 65,536), then moved from the last four warps to the softmax,
// which holds a row of 128 logits: 208 + 208 + 88 = 3 x 168
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;
constexpr int kMmaWarp = 8, kLoadWarp = 9;

template <int D>
struct TileShape {
    static constexpr int kHalves = D / 64;                     // 128-byte columns of a tile
    static constexpr int kSlotBytes = kTileKeys * D * 2;
    static constexpr int kSlots = D == 128 ? 5 : 8;
    static constexpr int kQBytes = 128 * D * 2;                // of one row tile
};

struct TileTail {
    uint64_t kv_full[8], kv_empty[8];
    uint64_t q_full[2], s_full[2], p_full[2], o_full[2];
    uint64_t drain;
    long long scratch[kTileThreads / 32];
    Start found;
    uint32_t tmem_base;
    volatile int abort_flag;
};

template <int D>
constexpr size_t kTileSmem = 1024 + 2 * (size_t)TileShape<D>::kQBytes + (size_t)TileShape<D>::kSlots * TileShape<D>::kSlotBytes + sizeof(TileTail);

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

// tiles of 128 keys that row tile x (0 or 1) of an item takes part in
__device__ __forceinline__ int tile_count(const Schedule<kTileRows, kTileKeys>& sch, const Item& it, int x) {
    const long long rows = (long long)it.s.new_len * sch.group;
    const long long first = (long long)it.i * kTileRows + 128 * x;
    if (first >= rows) return 0;
    if (!sch.causal) return (it.s.len + kTileKeys - 1) / kTileKeys;
    const long long last = (first + 128 < rows ? first + 128 : rows) - 1;
    const long long lim = (long long)it.s.len - it.s.new_len + last / sch.group + 1;
    return lim <= 0 ? 0 : (int)((lim + kTileKeys - 1) / kTileKeys);
}

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

// Two row tiles X = 0, 1 of 128 rows share every K and V tile.  Per unit and row tile:
//   S = Q K^T       (MMA, both operands in shared memory, S in TMEM)
//   P = 2^(scale S - m), row sums, P back to TMEM over S as 16-bit pairs     (one thread per row, 4 warps per row tile)
//   O += P V        (MMA, P in TMEM, V in shared memory with the keys along its rows, O in TMEM)
// While the softmax warps of one row tile work, the MMAs of the other run.
template <int D, bool BF>
__global__ void __launch_bounds__(kTileThreads, 1)
paged_tiles_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const __grid_constant__ AttendParams p) {
    using Shape = TileShape<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* q_smem = smem;
    uint8_t* ring = smem + 2 * Shape::kQBytes;
    TileTail* tail = reinterpret_cast<TileTail*>(ring + (size_t)Shape::kSlots * Shape::kSlotBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int s = 0; s < Shape::kSlots; ++s) {
            ptx::mbar_init(&tail->kv_full[s], 1);
            ptx::mbar_init(&tail->kv_empty[s], 1);
        }
        for (int x = 0; x < 2; ++x) {
            ptx::mbar_init(&tail->q_full[x], 128);
            ptx::mbar_init(&tail->s_full[x], 1);
            ptx::mbar_init(&tail->p_full[x], 128);
            ptx::mbar_init(&tail->o_full[x], 1);
        }
        ptx::mbar_init(&tail->drain, 1);
        tail->abort_flag = 0;
        ptx::mbar_init_fence();
        ptx::prefetch_tensormap(&map_k);
        ptx::prefetch_tensormap(&map_v);
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

    const Schedule<kTileRows, kTileKeys> sch{p.group, p.causal, p.c.kv_heads, p.c.batch};
    const Start st = find_start<kTileThreads, kTileRows, kTileKeys>(p.c, sch, p.max_blocks, p.min_units, tail->scratch, &tail->found);
    if (tid == 0) p.part_items[blockIdx.x].last = -1;
    Walk<kTileRows, kTileKeys> walk;
    bool more = walk.begin(p.c, sch, st, p.split != 0);

    if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == kLoadWarp) {
        // ---------------- loads: K and V of each unit, in turn, a lane per page ----------------
        int slot = 0;
        uint32_t phase = 0;
        bool ok = true;
        const int box = min(1 << p.c.page_shift, kTileKeys);
        const int boxes = kTileKeys / box;
        const int page_mask = (1 << p.c.page_shift) - 1;
        for (; more && ok; more = walk.next(p.c)) {
            const Item& it = walk.it;
            const int* table = p.c.page_table + it.b * p.c.table_stride;
            const int t_end = min(it.t1, max(tile_count(sch, it, 0), tile_count(sch, it, 1)));
            for (int t = it.t0; t < t_end && ok; ++t) {
                const int key = t * kTileKeys + lane * box;
                int page = (int)p.c.num_pages;                  // outside the cache: the copy fills in zeros
                if (lane < boxes && key < it.s.len) {
                    const int entry = __ldg(table + (key >> p.c.page_shift));
                    if (entry < 0 || entry >= p.c.num_pages) atomicMax(p.c.status, (int)SASQ_ERR_BAD_INDEX);
                    else page = entry;
                }
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    ok = ok && tile_wait(&tail->kv_empty[slot], phase ^ 1u, tail, p);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    if (lane == 0) ptx::mbar_arrive_expect_tx(&tail->kv_full[slot], Shape::kSlotBytes);
                    __syncwarp();
                    if (lane < boxes) {
                        const uint32_t dst = ptx::smem_u32(ring) + slot * Shape::kSlotBytes + lane * box * 128;
#pragma unroll
                        for (int half = 0; half < Shape::kHalves; ++half)
                            ptx::tma_load_4d(dst + half * kTileKeys * 128, kv == 0 ? &map_k : &map_v, &tail->kv_full[slot], half * 64,
                                             key & page_mask, it.h, page);
                    }
                    __syncwarp();
                    if (++slot == Shape::kSlots) { slot = 0; phase ^= 1u; }
                }
            }
        }
        // gave up: copies still in flight must land before the block's shared memory goes away
        if (!ok && lane == 0) {
            for (int s = 0; s < Shape::kSlots; ++s) {
                const long long t0 = clock64();
                const uint32_t par = s < slot ? phase : (phase ^ 1u);
                while (!ptx::mbar_try_wait(&tail->kv_full[s], par))
                    if (clock64() - t0 > (1LL << 24)) break;
            }
        }
        __syncwarp();
    } else if (warp == kMmaWarp) {
        // ---------------- MMAs ----------------
        constexpr uint32_t idesc_s = ptx::idesc_f16(128, kTileKeys, BF);
        constexpr uint32_t idesc_o = ptx::idesc_f16(128, D, BF) | ptx::kIdescBTransposed;
        int slot = 0;
        uint32_t phase = 0, q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
        bool ok = true;
        auto advance = [&] { if (++slot == Shape::kSlots) { slot = 0; phase ^= 1u; } };
        const uint32_t ring_addr = ptx::smem_u32(ring), q_addr = ptx::smem_u32(q_smem);
        auto qk = [&](int x, int k_slot) {                        // issued by one lane
            const uint64_t a = ptx::smem_desc_k_major_sw128(q_addr + x * Shape::kQBytes);
            const uint64_t b = ptx::smem_desc_k_major_sw128(ring_addr + k_slot * Shape::kSlotBytes);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uint64_t at = (uint64_t)(((k >> 2) * 128 * 128 + (k & 3) * 32) >> 4);
                ptx::mma_f16_ss(tmem + x * 128, a + at, b + at, idesc_s, k != 0);
            }
            ptx::mma_commit(&tail->s_full[x]);
        };
        auto pv = [&](int x, int v_slot, bool first) {
            const uint64_t b = ptx::smem_desc_mn_major_sw128(ring_addr + v_slot * Shape::kSlotBytes, kTileKeys * 128);
#pragma unroll
            for (int k = 0; k < kTileKeys / 16; ++k)
                ptx::mma_f16_ts(tmem + 256 + x * D, tmem + x * 128 + 8 * k, b + (uint64_t)(k * 2048 >> 4), idesc_o, !(first && k == 0));
            ptx::mma_commit(&tail->o_full[x]);
        };
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            ok = ok && tile_wait(bar, parity, tail, p);
            ok = __all_sync(0xFFFFFFFFu, ok);
            return ok;
        };
        for (; more && ok; more = walk.next(p.c)) {
            const Item& it = walk.it;
            const int n0 = tile_count(sch, it, 0), n1 = tile_count(sch, it, 1);
            const int t_end = min(it.t1, max(n0, n1));
            if (it.t0 >= t_end) continue;
#pragma unroll
            for (int x = 0; x < 2; ++x)
                if (it.t0 < (x == 0 ? n0 : n1)) {
                    if (!wait(&tail->q_full[x], q_phase[x])) break;
                    q_phase[x] ^= 1u;
                }
            if (!ok) break;
            ptx::tc_fence_after_sync();
            if (!wait(&tail->kv_full[slot], phase)) break;
            if (ptx::elect_one()) {
                if (it.t0 < n0) qk(0, slot);
                if (it.t0 < n1) qk(1, slot);
                ptx::mma_commit(&tail->kv_empty[slot]);
            }
            __syncwarp();
            advance();
            for (int t = it.t0; t < t_end; ++t) {
                const int v_slot = slot;
                if (!wait(&tail->kv_full[v_slot], phase)) break;
                // rows of V behind the sequence's last key: whatever they hold is multiplied by P = 0, and must be finite
                const int valid = it.s.len - t * kTileKeys;
                if (valid < kTileKeys) {
                    uint8_t* v = ring + (size_t)v_slot * Shape::kSlotBytes;
                    for (int x = lane; x < (kTileKeys - valid) * 8 * Shape::kHalves; x += 32) {
                        const int half = x / ((kTileKeys - valid) * 8), y = x % ((kTileKeys - valid) * 8);
                        *reinterpret_cast<uint4*>(v + half * kTileKeys * 128 + valid * 128 + y * 16) = make_uint4(0, 0, 0, 0);
                    }
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                }
                advance();
                const int k_slot = slot;
                const bool next = t + 1 < t_end;
                if (next) {
                    if (!wait(&tail->kv_full[k_slot], phase)) break;
                    advance();
                }
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int n = x == 0 ? n0 : n1;
                    if (t < n) {
                        if (!wait(&tail->p_full[x], p_phase[x])) break;
                        p_phase[x] ^= 1u;
                        ptx::tc_fence_after_sync();
                        if (ptx::elect_one()) {
                            pv(x, v_slot, t == it.t0);
                            if (next && t + 1 < n) qk(x, k_slot);
                        }
                        __syncwarp();
                    }
                    if (x == 1 && ptx::elect_one()) {
                        ptx::mma_commit(&tail->kv_empty[v_slot]);
                        if (next) ptx::mma_commit(&tail->kv_empty[k_slot]);
                    }
                    __syncwarp();
                }
                if (!ok) break;
            }
            if (!ok) break;
        }
        if (!ok) {                        // MMAs still running must end before shared memory and TMEM go away
            if (ptx::elect_one()) {
                ptx::mma_commit(&tail->drain);
                const long long t0 = clock64();
                while (!ptx::mbar_try_wait(&tail->drain, 0))
                    if (clock64() - t0 > (1LL << 24)) break;
            }
            __syncwarp();
        }
    } else if (warp < 8) {
        // ---------------- softmax: row tile x, one row per thread ----------------
        const int x = warp >> 2, quad = warp & 3;
        const int row = quad * 32 + lane;                          // of the row tile
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const uint32_t s_addr = tmem + lane_base + x * 128, o_addr = tmem + lane_base + 256 + x * D;
        uint32_t s_phase = 0, o_phase = 0;                         // o_phase: parity of the last PV asked for
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            ok = ok && tile_wait(bar, parity, tail, p);
            ok = __all_sync(0xFFFFFFFFu, ok);
            return ok;
        };
        for (; more && ok; more = walk.next(p.c)) {
            const Item& it = walk.it;
            const int rows_all = it.s.new_len * p.group;
            const int tile_row = it.i * kTileRows + x * 128;       // first row of the row tile, among the sequence's
            const int n = tile_count(sch, it, x);
            const int t_end = min(it.t1, n);
            const bool any = it.t0 < t_end;                        // this row tile sees keys of this block's units
            // queries into the swizzled tile, 16 bytes a lane, two rows of D = 128 (four of D = 64) at a time.  Every MMA
            // that read the last ones has been waited for.
            if (any) {
                constexpr int kChunks = D / 8, kAtOnce = 32 / kChunks;
                const int chunk = lane % kChunks, sub = lane / kChunks;
                uint8_t* dst = q_smem + x * Shape::kQBytes + (chunk >> 3) * 128 * 128;
                const bool flip = p.scale < 0.0f;
#pragma unroll 4
                for (int i = 0; i < 32 / kAtOnce; ++i) {
                    const int r = quad * 32 + i * kAtOnce + sub;
                    const int rr = tile_row + r;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (rr < rows_all) {
                        const int tok = rr / p.group;
                        v = *reinterpret_cast<const uint4*>(p.q + (long long)(it.s.first + tok) * p.q_stride +
                                                            (long long)(it.h * p.group + rr - tok * p.group) * D + chunk * 8);
                        if (flip) {
                            v.x ^= 0x80008000u;
                            v.y ^= 0x80008000u;
                            v.z ^= 0x80008000u;
                            v.w ^= 0x80008000u;
                        }
                    }
                    *reinterpret_cast<uint4*>(dst + r * 128 + (((chunk & 7) ^ (r & 7)) * 16)) = v;
                }
                ptx::fence_proxy_async_smem();
                ptx::mbar_arrive(&tail->q_full[x]);
            }

            const float scale = fabsf(p.scale);
            const int limit = sch.key_limit(it.s, it.i);
            int row_limit = limit;
            if (p.causal && tile_row + row < rows_all) row_limit = it.s.len - it.s.new_len + (tile_row + row) / p.group + 1;
            float m = -INFINITY;                                   // reference, in powers of two
            uint64_t sum2 = 0;                                     // two partial sums of P
            for (int t = it.t0; t < t_end; ++t) {
                if (!wait(&tail->s_full[x], s_phase)) break;
                s_phase ^= 1u;
                ptx::tc_fence_after_sync();
                uint32_t s[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) ptx::tmem_ld_32x32(s_addr + c * 32, s[c]);
                ptx::tmem_ld_wait();
                const int seen = row_limit - t * kTileKeys;
                if (__any_sync(0xFFFFFFFFu, seen < kTileKeys)) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (c * 32 + e >= seen) s[c][e] = 0xFF800000u;      // -inf
                }
                float top[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    top[c] = __uint_as_float(s[c][0]);
#pragma unroll
                    for (int e = 1; e < 32; ++e) top[c] = fmaxf(top[c], __uint_as_float(s[c][e]));
                }
                const float tile_max = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * scale;
                if (__any_sync(0xFFFFFFFFu, tile_max > m + kRescaleAt)) {
                    const float m_new = fmaxf(m, tile_max);
                    const float f = m_new == -INFINITY ? 1.0f : exp2_approx(m - m_new);
                    m = m_new;
                    const float2 old = unpack2(sum2);
                    sum2 = pack2(old.x * f, old.y * f);
                    if (t > it.t0) {
                        if (!wait(&tail->o_full[x], o_phase ^ 1u)) break;
                        ptx::tc_fence_after_sync();
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            uint32_t o[32];
                            ptx::tmem_ld_32x32(o_addr + c, o);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            ptx::tmem_st_32x32(o_addr + c, o);
                        }
                    }
                }
                const float ref = m == -INFINITY ? 0.0f : m;
                const uint64_t scale2 = pack2(scale, scale), ref2 = pack2(-ref, -ref);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t pk[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const int col = c * 64 + 2 * e;
                        const float2 z = unpack2(fma2(pack2(__uint_as_float(s[col >> 5][col & 31]), __uint_as_float(s[col >> 5][(col & 31) + 1])),
                                                      scale2, ref2));
                        const float p0 = exp2_approx(z.x), p1 = exp2_approx(z.y);
                        sum2 = add2(sum2, pack2(p0, p1));
                        pk[e] = narrow2<BF>(p0, p1);
                    }
                    ptx::tmem_st_32x32(s_addr + c * 32, pk);
                }
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                ptx::mbar_arrive(&tail->p_full[x]);
                o_phase ^= 1u;
            }
            if (!ok) break;
            // ---- the item's rows
            if (any) {
                if (!wait(&tail->o_full[x], o_phase ^ 1u)) break;
                ptx::tc_fence_after_sync();
            }
            const float2 sums = unpack2(sum2);
            const float sum = sums.x + sums.y;
            const bool whole = it.t0 == 0 && it.t1 == it.units;
            const int slot = 2 * blockIdx.x + (it.t0 == 0 ? 1 : 0);
            const bool valid = tile_row + row < rows_all;
            const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
            const int tok = (tile_row + row) / p.group;
            const int head = it.h * p.group + (tile_row + row) - tok * p.group;
            const long long token = it.s.first + tok;
            const long long part_row = (long long)slot * kTileRows + x * 128 + row;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                uint32_t o[32];
                if (any) {
                    ptx::tmem_ld_32x32(o_addr + c, o);
                    ptx::tmem_ld_wait();
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = 0;
                }
                if (valid && whole) {
                    uint4* dst = reinterpret_cast<uint4*>(p.out + token * p.out_stride + (long long)head * D + c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            w[k] = sum > 0.0f ? narrow2<BF>(__uint_as_float(o[8 * e + 2 * k]) * inv, __uint_as_float(o[8 * e + 2 * k + 1]) * inv) : 0u;
                        dst[e] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                } else if (valid) {
                    uint4* dst = reinterpret_cast<uint4*>(p.part_o + part_row * D + c);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dst[e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                }
            }
            if (valid && whole && p.lse != nullptr)
                p.lse[token * p.heads + head] = sum > 0.0f ? (m + log2f(sum)) * 0.6931471805599453f : -INFINITY;
            if (valid && !whole) p.part_ml[part_row] = make_float2(m, sum);
            if (!whole && it.t0 == 0 && tid == 0) {
                PartItem pi;
                pi.last = block_of(st.total, it.first_unit + it.units - 1, st.blocks);
                pi.h = it.h;
                pi.first_row = it.i * kTileRows;
                pi.rows = min(kTileRows, rows_all - it.i * kTileRows);
                pi.first_token = it.s.first;
                p.part_items[blockIdx.x] = pi;
            }
            ptx::tc_fence_before_sync();                           // O has been read: the next item's first PV may overwrite it
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
