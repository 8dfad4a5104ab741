// The 4-bit linear for more than 16 tokens, on the tensor cores (tcgen05); included by w4_linear.cu.
#pragma once

namespace sasq {

int* paged_status_ptr();           // device address of a sticky status word; nullptr if it cannot be had
long long debug_wait_limit();      // sasq_debug_set_wait_limit's setting

namespace {

// D = A B^T: A is 128 rows of codes as 16-bit floats, B up to 64 tokens, a step 128 columns.  The codes are exact operands, and so
// are the tokens; a group's sums leave the tensor core for a buffer of their own in TMEM, from where a thread for each row takes
// them times the row's factor into its fp32 sums.  A cluster's blocks share a tile's columns, and their sums meet in shared memory.
//
// 64 tokens of 11008 x 4096, groups of 128: 26.0 us, 222 TFLOP/s; 61 of 6144 x 4096, groups of 32: 23.5 us; 4096 of 4096 x 4096: 350
// us, 393 TFLOP/s.  Bound by waits between the roles more than by instructions, which fill half of the busy SMs' issue slots (8.5
// million warp instructions in the second case, on 96 SMs): every group is a round trip of products, commit, load and arrival, a
// tile begins and ends with a block, and equal shares of a tile leave SMs without one.  Without the loads of codes, tokens and
// factors the first case would take 16 us, without the conversion (some 220 instructions a thread and window) too 14.
//
// Warps 0-7 bring codes and tokens to a ring of shared memory (128-byte swizzle, K-major); then four warps for each 32 tokens, which
// add up; the last one issues the products.
template <int TOKENS>
struct W4Batch {
    static constexpr int kRows = 128, kWindow = 128, kStages = 4;
    static constexpr int kABytes = kRows * kWindow * 2, kXBytes = TOKENS * kWindow * 2, kSlot = kABytes + kXBytes;
    static constexpr int kConvertWarps = 8, kAddWarps = TOKENS / 8, kThreads = 32 * (kConvertWarps + kAddWarps + 1);
    static constexpr int kBuffers = 4;                     // of group sums, TOKENS columns of TMEM each
    static constexpr int kSmem = kStages * kSlot + 1024;   // with room to align
    static_assert(TOKENS * (kRows + 1) * 4 <= kStages * kSlot, "the sums take the ring's place");
};
struct W4BatchBars {
    uint64_t full[4], empty[4];                            // of the ring
    uint64_t sums_full[4], sums_empty[4];                  // of the buffers
    uint64_t drain;
    uint32_t tmem_base;
    volatile int abort_flag;
};

// 16 bytes that this block reads once
__device__ __forceinline__ uint4 load_once16(const void* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

template <int TOKENS, bool BF, int G>
__global__ void __launch_bounds__(W4Batch<TOKENS>::kThreads, 1)
w4_batch_kernel(const __grid_constant__ W4Params p, const __grid_constant__ Bits bits_) {
    using Shape = W4Batch<TOKENS>;
    constexpr int kStages = Shape::kStages, kWindow = Shape::kWindow, kRows = Shape::kRows, kBuffers = Shape::kBuffers, GW = kWindow / G;
    constexpr int kMmaWarp = Shape::kConvertWarps + Shape::kAddWarps;
    extern __shared__ uint8_t smem_raw[];
    __shared__ W4BatchBars bars;
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = p.split > 1 ? (int)ptx::cluster_ctarank() : 0;
    const int n0 = blockIdx.x / p.split * kRows, t0 = blockIdx.y * TOKENS, tokens = min(TOKENS, p.T - t0);
    const int begin = rank * p.windows_each + min(rank, p.windows_more), windows = p.windows_each + (rank < p.windows_more);
    const int half_k = p.K >> 1;
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(&bars.full[s], 32 * Shape::kConvertWarps);
            ptx::mbar_init(&bars.empty[s], 1);
        }
        for (int b = 0; b < kBuffers; ++b) {
            ptx::mbar_init(&bars.sums_full[b], 1);
            ptx::mbar_init(&bars.sums_empty[b], Shape::kAddWarps);
        }
        ptx::mbar_init(&bars.drain, 1);
        bars.abort_flag = 0;
        ptx::mbar_init_fence();
    }
    if (warp == kMmaWarp) {
        ptx::tmem_alloc(&bars.tmem_base, kBuffers * TOKENS);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = bars.tmem_base;
    pdl_launch_dependents();
    // bounded: false if the phase did not complete in time or another role gave up
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (ptx::mbar_try_wait(bar, parity)) return true;
        const long long since = clock64();
        int polls = 0;
        while (!ptx::mbar_try_wait(bar, parity))
            if (p.wait_limit <= 0 || (++polls & 63) == 0) {
                if (bars.abort_flag) return false;
                if (clock64() - since > p.wait_limit) {
                    bars.abort_flag = 1;
                    atomicMax(p.status, (int)SASQ_ERR_TIMEOUT);
                    return false;
                }
            }
        return true;
    };
    float sums[32];                                        // warps that add: of a row, 32 tokens
    const int quad = warp & 3, part = (warp - Shape::kConvertWarps) >> 2, row = 32 * quad + lane;

    if (warp < Shape::kConvertWarps) {
        const Bits bits = bits_;
        constexpr int kAhead = 4;                          // windows of codes under way
        // codes: 16 bytes, 32 columns, of rows tid / 4 and tid / 4 + 64.  Half the lanes store a row's words the other way round,
        // which spreads them over the banks.
        const int chunk = tid & 3, turn = chunk >> 1;
        const uint8_t* w_row[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) w_row[i] = p.w + (long long)min(n0 + (tid >> 2) + 64 * i, p.N - 1) * half_k;
        auto load_w = [&](int w, uint4 (&v)[2]) {
            if (w >= windows) return;
            // columns behind the last are read from the last one's place, and meet zeros
            const int at = min((begin + w) * (kWindow / 2) + 16 * chunk, half_k - 16);
#pragma unroll
            for (int i = 0; i < 2; ++i) v[i] = load_once16(w_row[i] + at);
        };
        // tokens: 16 bytes, eight columns, of every sixteenth token, copied to their place two windows ahead.  Tokens and
        // columns behind the last are zeros (nothing is read for them: with the last token in their place every block reads its
        // lines again and again, 33 tokens of 11008 x 4096: 32.8 us).
        constexpr int kX = TOKENS / 16, kXAhead = 2;
        const int x_chunk = tid & 15, x_row = tid >> 4;
        const uint16_t* const x_from = p.x + (long long)t0 * p.K + 8 * x_chunk;
        const uint32_t x_to = ptx::smem_u32(smem) + Shape::kABytes + (x_chunk >> 3) * (TOKENS * 128) + x_row * 128 + (((x_chunk & 7) ^ (x_row & 7)) << 4);
        bool ok = true;
        auto copy_x = [&](int w) {
            if (w < windows) {
                const int s = w % kStages, col = (begin + w) * kWindow;
                ok = ok && wait(&bars.empty[s], (w / kStages & 1u) ^ 1u);
#pragma unroll
                for (int i = 0; i < kX; ++i) {
                    const uint32_t bytes = col + 8 * x_chunk < p.K && x_row + 16 * i < tokens ? 16u : 0u;
                    const uint16_t* from = bytes != 0 ? x_from + (long long)(x_row + 16 * i) * p.K + col : p.x;
                    if (ok)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(x_to + s * Shape::kSlot + i * 16 * 128), "l"(from), "r"(bytes) : "memory");
                }
            }
            copies_end_group();
        };
        uint4 wv[kAhead][2];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            wv[a][0] = wv[a][1] = make_uint4(0, 0, 0, 0);
            load_w(a, wv[a]);
        }
        // weights may be read at once, tokens when the kernels before this one are done
        pdl_wait();
#pragma unroll
        for (int w = 0; w < kXAhead; ++w) copy_x(w);
        // (a register under way can't be moved without waiting for it: the windows take turns with theirs)
#pragma unroll 1
        for (int w0 = 0; w0 < windows && ok; w0 += kAhead) {
#pragma unroll
            for (int turn_of = 0; turn_of < kAhead; ++turn_of) {
                const int w = w0 + turn_of;
                if (w >= windows) break;
                copy_x(w + kXAhead);                       // (the slot of window w was free then)
                if (!ok) break;
                uint8_t* const a = smem + w % kStages * Shape::kSlot + turn * (kRows * 128);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = (tid >> 2) + 64 * i;
                    const uint4 v = wv[turn_of][i];
                    const uint32_t words[4] = {turn ? v.z : v.x, turn ? v.w : v.y, turn ? v.x : v.z, turn ? v.y : v.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t lo[2], hi[2];
                        codes8<BF>(words[k], bits, lo, hi);
                        const int at = 4 * (chunk & 1) + (k ^ (turn << 1));
                        *reinterpret_cast<uint4*>(a + r * 128 + ((at ^ (r & 7)) << 4)) =
                            make_uint4(__byte_perm(lo[0], hi[0], 0x5410), __byte_perm(lo[1], hi[1], 0x5410), __byte_perm(lo[0], hi[0], 0x7632),
                                       __byte_perm(lo[1], hi[1], 0x7632));
                    }
                }
                load_w(w + kAhead, wv[turn_of]);
                copies_wait<kXAhead>();
                ptx::fence_proxy_async_smem();
                ptx::mbar_arrive(&bars.full[w % kStages]);
            }
        }
        copies_wait<0>();                                  // none lands after the block has gone
    } else if (warp < kMmaWarp) {
        pdl_wait();
#pragma unroll
        for (int t = 0; t < 32; ++t) sums[t] = 0.0f;
        const uint16_t* const factors = p.ws + (long long)min(n0 + row, p.N - 1) * p.groups;
        constexpr int kAhead = GW == 4 ? 2 : 4;            // windows of factors under way
        uint32_t next[kAhead][(GW + 1) / 2];               // pairs, or one
        auto load_factors = [&](int w, uint32_t (&to)[(GW + 1) / 2]) {
            const int first = (begin + w) * GW;
            if (GW > 1 && p.sc_whole) {                    // a window's factors are one aligned word
                if (w >= windows) return;
                if constexpr (GW == 4) {
                    const uint2 v = __ldg(reinterpret_cast<const uint2*>(factors + first));
                    to[0] = v.x;
                    to[1] = v.y;
                } else {
                    to[0] = __ldg(reinterpret_cast<const uint32_t*>(factors + first));
                }
            } else {
#pragma unroll
                for (int s = 0; s < GW; s += 2) {
                    to[s / 2] = __ldg(factors + min(first + s, p.groups - 1));
                    if (GW > 1) to[s / 2] |= (uint32_t)__ldg(factors + min(first + s + 1, p.groups - 1)) << 16;
                }
            }
        };
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            next[a][0] = next[a][(GW - 1) / 2] = 0;
            load_factors(a, next[a]);
        }
        bool ok = true;
        uint32_t n = 0;                                    // groups so far
#pragma unroll 1
        for (int w0 = 0; w0 < windows && ok; w0 += kAhead) {
#pragma unroll
            for (int turn = 0; turn < kAhead; ++turn) {
                const int w = w0 + turn;
                if (w >= windows || !ok) break;
                float f[GW];
#pragma unroll
                for (int s = 0; s < GW; ++s) f[s] = widen1<BF>((uint16_t)(next[turn][s / 2] >> 16 * (s & 1)));
                load_factors(w + kAhead, next[turn]);
#pragma unroll
                for (int s = 0; s < GW; ++s, ++n) {
                    ok = ok && wait(&bars.sums_full[n % kBuffers], n / kBuffers & 1u);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    ptx::tc_fence_after_sync();
                    uint32_t v[32];
                    ptx::tmem_ld_32x32(tmem + ((uint32_t)(32 * quad) << 16) + n % kBuffers * TOKENS + 32 * part, v);
                    ptx::tmem_ld_wait();
                    ptx::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&bars.sums_empty[n % kBuffers]);
                    if ((begin + w) * GW + s < p.groups) { // those behind the last have no factor
#pragma unroll
                        for (int t = 0; t < 32; ++t) sums[t] = fmaf(__uint_as_float(v[t]), f[s], sums[t]);
                    }
                }
            }
        }
        // all products are done: the sums take the ring's place
        if (ok && p.split > 1) {
            float* const to = reinterpret_cast<float*>(smem) + 32 * part * (kRows + 1) + row;
#pragma unroll
            for (int t = 0; t < 32; ++t) to[t * (kRows + 1)] = sums[t];
        }
        if (ok && p.split == 1 && n0 + row < p.N) {
            const float bias = p.bias != nullptr ? widen1<BF>(p.bias[n0 + row]) : 0.0f;
            uint16_t* const to = p.y + (long long)(t0 + 32 * part) * p.N + n0 + row;
#pragma unroll
            for (int t = 0; t < 32; ++t)
                if (32 * part + t < tokens) to[(long long)t * p.N] = narrow1<BF>(sums[t] + bias);
        }
    } else {
        pdl_wait();
        if (ptx::elect_one()) {
            constexpr uint32_t idesc = ptx::idesc_f16(kRows, TOKENS, BF);
            const uint64_t desc = ptx::smem_desc_k_major_sw128(ptx::smem_u32(smem));
            bool ok = true;
            uint32_t n = 0;
#pragma unroll 1
            for (int w = 0; w < windows && ok; ++w) {
                const int slot = w % kStages;
                ok = wait(&bars.full[slot], w / kStages & 1u);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                const uint64_t a = desc + (uint64_t)(slot * Shape::kSlot >> 4), b = a + (uint64_t)(Shape::kABytes >> 4);
#pragma unroll
                for (int s = 0; s < GW; ++s, ++n) {
                    ok = ok && wait(&bars.sums_empty[n % kBuffers], (n / kBuffers & 1u) ^ 1u);
                    if (!ok) break;
                    ptx::tc_fence_after_sync();
#pragma unroll
                    for (int i = 0; i < G / 16; ++i) {
                        const int k = s * (G / 16) + i;
                        ptx::mma_f16_ss(tmem + n % kBuffers * TOKENS, a + (uint64_t)(((k >> 2) * kRows * 128 + (k & 3) * 32) >> 4),
                                        b + (uint64_t)(((k >> 2) * TOKENS * 128 + (k & 3) * 32) >> 4), idesc, i != 0);
                    }
                    ptx::mma_commit(&bars.sums_full[n % kBuffers]);
                }
                if (ok) ptx::mma_commit(&bars.empty[slot]);
            }
            // products still running must end before shared memory and TMEM go away
            ptx::mma_commit(&bars.drain);
            const long long since = clock64();
            while (!ptx::mbar_try_wait(&bars.drain, 0))
                if (clock64() - since > (1LL << 24)) break;
        }
        __syncwarp();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, kBuffers * TOKENS);
    }
    if (p.split > 1) {
        __syncwarp();
        ptx::cluster_sync_all();
        // the cluster's tokens are dealt to its blocks, a warp 32 rows of one at a time
        for (int i = rank * (Shape::kThreads / 32) + warp; i < tokens * (kRows / 32); i += p.split * (Shape::kThreads / 32)) {
            const int t = i >> 2, r = 32 * (i & 3) + lane;
            const uint32_t here = ptx::smem_u32(smem) + (uint32_t)(t * (kRows + 1) + r) * 4;
            float v = 0.0f;
            for (int k = 0; k < p.split; ++k) {
                float one;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(one) : "r"(ptx::mapa_u32(here, (uint32_t)k)));
                v += one;
            }
            if (n0 + r < p.N) {
                if (p.bias != nullptr) v += widen1<BF>(p.bias[n0 + r]);
                p.y[(long long)(t0 + t) * p.N + n0 + r] = narrow1<BF>(v);
            }
        }
        __syncwarp();
        ptx::cluster_sync_all();                           // nobody leaves while its sums are being read
    }
}

template <int TOKENS, bool BF, int G>
cudaError_t launch_w4_batch(W4Params p, int sms, cudaStream_t st) {
    using Shape = W4Batch<TOKENS>;
    const int chunks = ceil_div(p.T, TOKENS), tiles = ceil_div(p.N, Shape::kRows), windows = ceil_div(p.K, Shape::kWindow);
    // Blocks of a cluster: rounds of the device times a block's steps, of which beginning and ending take about eight
    long long least = -1;
    for (int split = 1; split <= 8 && split <= windows; ++split) {
        const int slots = cluster_slots(split, 1, 512, sms);
        const long long cost = (long long)ceil_div((long long)tiles * chunks, slots) * (ceil_div(windows, split) + 8 + (split > 1 ? 3 : 0));
        if (least >= 0 && cost >= least) continue;
        least = cost;
        p.split = split;
    }
    p.windows_each = windows / p.split;
    p.windows_more = windows % p.split;
    p.sc_whole = p.K % Shape::kWindow == 0;
    p.wait_limit = debug_wait_limit();
    p.status = paged_status_ptr();
    if (p.status == nullptr) return cudaErrorUnknown;
    static std::atomic<unsigned long long> ready{0};       // devices whose shared-memory limit has been raised
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!(ready.load() >> (dev & 63) & 1)) {
        e = cudaFuncSetAttribute(w4_batch_kernel<TOKENS, BF, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::kSmem);
        if (e != cudaSuccess) return e;
        ready.fetch_or(1ull << (dev & 63));
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles * p.split), (unsigned)chunks);
    cfg.blockDim = dim3(Shape::kThreads);
    cfg.dynamicSmemBytes = Shape::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0] = pdl_attribute();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, w4_batch_kernel<TOKENS, BF, G>, p, kBits<BF>);
}

}  // namespace
}  // namespace sasq
