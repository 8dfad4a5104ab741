// Rotary positions on q and k, and k and v appended to the paged cache, in one pass over the three.
//
// Pure movement: every element of q, k and v is read once and written once, in 16-byte words, with four multiplies per
// rotated pair on the way.  Bound by DRAM for prompts (7815 tokens, 40 + 80 heads of 128, fp16: 80 us, 482 MB, 6.0 TB/s, 93 %
// of a plain copy's rate) and by the launch for single tokens (2.8 us replayed from a graph).  4096 tokens into an int8 cache
// (32 + 16 heads of 128, interleaved pairs, tokens first): 28.7 us, 94 MB, 3.3 TB/s; single tokens 3.4 us.  4815 tokens into a
// 4-bit cache (40 + 16 heads of 128, a factor for each channel): 34.5 us, 124 MB, 3.6 TB/s, bound by instructions; single
// tokens 3.7 us.
#include "paged_common.cuh"

namespace sasq {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppend4Threads = 64;           // of many tokens into a 4-bit cache

struct AppendParams {
    PagedParams c;
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    uint16_t* q_out;
    long long q_stride, k_stride, v_stride, q_out_stride;
    int q_heads;                // 0 when q is absent
    int dim, rot, interleaved;
    const float* cos_sin;
    long long max_positions;
    int head_step;              // heads that a block's threads take at a time
    int heads_per_block;        // gridDim.y blocks share a token's heads
};

// code of Eq. 1 (b = 8) of an fp32 value
__device__ __forceinline__ uint32_t code8(float x, float inv) {
    const float r = rintf(__fmul_rn(x, inv));
    return (uint32_t)(uint8_t)(int8_t)(int)fminf(fmaxf(r, -128.0f), 127.0f);
}

template <bool BF>
__device__ __forceinline__ void widen8(const uint4& w, float (&f)[8]) {
    const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = widen2<BF>(a[i]);
        f[2 * i] = t.x;
        f[2 * i + 1] = t.y;
    }
}
template <bool BF>
__device__ __forceinline__ uint4 narrow8(const float (&f)[8]) {
    return make_uint4(narrow2<BF>(f[0], f[1]), narrow2<BF>(f[2], f[3]), narrow2<BF>(f[4], f[5]), narrow2<BF>(f[6], f[7]));
}
__device__ __forceinline__ uint2 codes8(const float (&f)[8], float inv) {
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = code8(f[i], inv);
    return make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
}

// The same with b = 4 for eight channels with a factor each, the first in the word's low bits; `bad` collects whether Eq. 1 can
// use the factors.  -8 and 7 are integers, so a value may be cut to them before it is rounded: adding 1.5 * 2^23 rounds it, and
// with 8 more its low bits are the code + 8, which eight multiplications by 16 put together and one flip of their top bits turns
// into codes.
__device__ __forceinline__ uint32_t codes4(const float (&f)[8], const float* scale, bool* bad) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(scale)), b = __ldg(reinterpret_cast<const float4*>(scale) + 1);
    const float s[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    constexpr uint32_t kRound = 0x4B400000u;                 // 1.5 * 2^23
    uint32_t w = 0;
#pragma unroll
    for (int i = 7; i >= 0; --i) {
        const float inv = __frcp_rn(factor4(s[i]));
        *bad |= !(fabsf(inv) > 0.0f && fabsf(inv) < __uint_as_float(0x7F800000u));      // a factor of 0, infinity or NaN, or too small
        const float c = fminf(fmaxf(__fmul_rn(f[i], inv), -8.0f), 7.0f);
        w = w * 16u + (__float_as_uint(__fadd_rn(c, __uint_as_float(kRound + 8u))) - kRound);
    }
    return w ^ 0x88888888u;
}

// A thread owns a "unit" of a head, two 8-element words that the rotation mixes: words u and u + rot / 16 for half-split
// pairs, 2u and 2u + 1 for interleaved ones and behind the rotated part.  Its cosines and sines serve every head that
// it walks (heads h, h + head_step, ...), so they are read once per token and block.  A block has one token.
template <bool BF, int KIND>
__global__ void __launch_bounds__(kAppendThreads) rope_kv_append_kernel(const __grid_constant__ AppendParams p) {
    constexpr bool INT8 = KIND == SASQ_KV_INT8, INT4 = KIND == SASQ_KV_INT4;
    const int units = p.dim >> 4;
    const int u = threadIdx.x % units, slot = threadIdx.x / units;
    pdl_launch_dependents();
    pdl_wait();
    const int t = blockIdx.x;
    const int kv = p.c.kv_heads;
    const int total_heads = p.q_heads + 2 * kv;
    const int h_begin = blockIdx.y * p.heads_per_block;
    const int h_end = min(h_begin + p.heads_per_block, total_heads);
    const bool idle = slot >= p.head_step;

    // 4-bit: the first head's words travel while the token's page is looked up, and a head's while the one before is turned
    [[maybe_unused]] uint4 next0, next1;
    [[maybe_unused]] auto fetch = [&](int h) {
        if (idle || h >= h_end) return;
        const int which = h < p.q_heads ? 0 : h < p.q_heads + kv ? 1 : 2, step = which != 2 && u < (p.rot >> 4) && !p.interleaved ? p.rot >> 4 : 0;
        const uint16_t* src = which == 0 ? p.q + t * p.q_stride : which == 1 ? p.k + t * p.k_stride : p.v + t * p.v_stride;
        const uint4* words = reinterpret_cast<const uint4*>(src + (long long)(which == 0 ? h : which == 1 ? h - p.q_heads : h - p.q_heads - kv) * p.dim);
        next0 = words[step != 0 ? u : 2 * u];
        next1 = words[step != 0 ? u + step : 2 * u + 1];
    };

    // the token's sequence: how many sequences end at or before it, counted by a warp at a time
    const int lane = threadIdx.x & 31;
    int b = 0;
    for (int base = 0; base < p.c.batch; base += 32) {
        const bool past = base + lane < p.c.batch && p.c.q_starts[base + lane + 1] <= t;
        b += __popc(__ballot_sync(0xFFFFFFFFu, past));
    }
    if (b >= p.c.batch || idle) return;          // padding behind the last sequence
    const Sequence s = load_sequence(p.c, b);
    if (t < s.first || t >= s.first + s.new_len) return;
    if constexpr (INT4) fetch(h_begin + slot);   // rows of padding are not read
    // from the length as given: a token that the table has no room for is skipped, it does not move to another's place
    const long long place = (long long)s.given_len - s.new_len + (t - s.first);
    bool there = place >= 0 && place < (long long)p.c.max_pages << p.c.page_shift;      // (reported by load_sequence)
    const int pos = (int)place;
    if (there && p.rot > 0 && pos >= p.max_positions) {
        atomicMax(p.c.status, (int)SASQ_ERR_BAD_INDEX);
        there = false;
    }
    long long row = 0;                           // element offset of the token's place, without the head
    if (there) {
        const int page = p.c.page_table[b * p.c.table_stride + (pos >> p.c.page_shift)];
        if (page < 0 || page >= p.c.num_pages) {
            atomicMax(p.c.status, (int)SASQ_ERR_BAD_INDEX);
            there = false;
        } else {
            row = page * p.c.page_stride + (pos & ((1 << p.c.page_shift) - 1)) * p.c.token_stride;
        }
    }
    const int pairs = p.rot >> 1;                // rotated pairs of a head
    const bool turns = u < (p.rot >> 4);
    const int w0 = (turns && !p.interleaved) ? u : 2 * u;
    const int w1 = (turns && !p.interleaved) ? u + (p.rot >> 4) : 2 * u + 1;
    float co[8], si[8];
    if (turns && there) {
        const float4* c4 = reinterpret_cast<const float4*>(p.cos_sin + (long long)pos * p.rot + 8 * u);
        const float4* s4 = reinterpret_cast<const float4*>(p.cos_sin + (long long)pos * p.rot + pairs + 8 * u);
        const float4 c0 = __ldg(c4), c1 = __ldg(c4 + 1), s0 = __ldg(s4), s1 = __ldg(s4 + 1);
        co[0] = c0.x; co[1] = c0.y; co[2] = c0.z; co[3] = c0.w; co[4] = c1.x; co[5] = c1.y; co[6] = c1.z; co[7] = c1.w;
        si[0] = s0.x; si[1] = s0.y; si[2] = s0.z; si[3] = s0.w; si[4] = s1.x; si[5] = s1.y; si[6] = s1.z; si[7] = s1.w;
    }

    constexpr int kUnroll = INT4 ? 1 : 4;
#pragma unroll kUnroll
    for (int h = h_begin + slot; h < h_end; h += p.head_step) {
        const int which = h < p.q_heads ? 0 : h < p.q_heads + kv ? 1 : 2;
        const int hh = which == 0 ? h : which == 1 ? h - p.q_heads : h - p.q_heads - kv;
        const uint16_t* src = which == 0 ? p.q + t * p.q_stride : which == 1 ? p.k + t * p.k_stride : p.v + t * p.v_stride;
        const bool turn = turns && which != 2;
        const int a0 = which == 2 ? 2 * u : w0, a1 = which == 2 ? 2 * u + 1 : w1;
        uint4 x0, x1;
        if constexpr (INT4) {
            x0 = next0;
            x1 = next1;
            fetch(h + p.head_step);
        } else {
            const uint4* words = reinterpret_cast<const uint4*>(src + (long long)hh * p.dim);
            x0 = words[a0];
            x1 = words[a1];
        }
        if (which != 0 && !there) continue;
        float f0[8], f1[8];
        if (turn || (KIND != SASQ_KV_16BIT && which != 0)) {
            widen8<BF>(x0, f0);
            widen8<BF>(x1, f1);
        }
        if (turn && there) {
            if (!p.interleaved) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float a = f0[i], c = f1[i];
                    f0[i] = __fsub_rn(__fmul_rn(a, co[i]), __fmul_rn(c, si[i]));
                    f1[i] = __fadd_rn(__fmul_rn(c, co[i]), __fmul_rn(a, si[i]));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float* f = i < 4 ? f0 : f1;
                    const float a = f[2 * (i & 3)], c = f[2 * (i & 3) + 1];
                    f[2 * (i & 3)] = __fsub_rn(__fmul_rn(a, co[i]), __fmul_rn(c, si[i]));
                    f[2 * (i & 3) + 1] = __fadd_rn(__fmul_rn(c, co[i]), __fmul_rn(a, si[i]));
                }
            }
            if (KIND == SASQ_KV_16BIT || which == 0) {
                x0 = narrow8<BF>(f0);
                x1 = narrow8<BF>(f1);
            }
        }
        if (which == 0) {
            if (!there) x0 = x1 = make_uint4(0, 0, 0, 0);
            uint4* dst = reinterpret_cast<uint4*>(p.q_out + t * p.q_out_stride + (long long)hh * p.dim);
            dst[a0] = x0;
            dst[a1] = x1;
        } else {
            const long long at = row + hh * p.c.head_stride;
            void* base = which == 1 ? p.c.k : p.c.v;
            if constexpr (INT8) {
                const float sc = __ldg((which == 1 ? p.c.k_scale : p.c.v_scale) + hh);
                if (scale_is_bad(sc)) atomicMax(p.c.status, (int)SASQ_ERR_BAD_SCALE);
                const float inv = __fdiv_rn(1.0f, sc);
                uint2* dst = reinterpret_cast<uint2*>(static_cast<int8_t*>(base) + at);
                dst[a0] = codes8(f0, inv);
                dst[a1] = codes8(f1, inv);
            } else if constexpr (INT4) {
                const float* sc = (which == 1 ? p.c.k_scale : p.c.v_scale) + hh * p.dim;
                uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(base) + (at >> 1));
                bool bad = false;
                dst[a0] = codes4(f0, sc + 8 * a0, &bad);
                dst[a1] = codes4(f1, sc + 8 * a1, &bad);
                if (bad) atomicMax(p.c.status, (int)SASQ_ERR_BAD_SCALE);
            } else {
                uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + at);
                dst[a0] = x0;
                dst[a1] = x1;
            }
        }
    }
}

}  // namespace

int paged_check(const sasq_kv_cache_t* c, const sasq_kv_batch_t* b, int dt, PagedParams* p) {
    if (c == nullptr || b == nullptr || (dt != SASQ_F16 && dt != SASQ_BF16)) return SASQ_ERR_INVALID_ARG;
    if (c->kind != SASQ_KV_16BIT && c->kind != SASQ_KV_INT8 && c->kind != SASQ_KV_INT4) return SASQ_ERR_INVALID_ARG;
    if (c->num_pages < 0 || c->num_kv_heads <= 0 || c->head_dim <= 0 || b->batch < 0 || b->total_q < 0 || b->max_pages < 0 ||
        b->max_q_len < 0 || b->max_seq_len < 0 || b->reserved != 0)
        return SASQ_ERR_INVALID_ARG;
    if (b->batch > 0 && (b->page_table == nullptr || b->seq_lens == nullptr || b->q_starts == nullptr ||
                         b->page_table_stride < b->max_pages))
        return SASQ_ERR_INVALID_ARG;
    const uintptr_t ints = reinterpret_cast<uintptr_t>(b->page_table) | reinterpret_cast<uintptr_t>(b->seq_lens) |
                           reinterpret_cast<uintptr_t>(b->q_starts);
    if (ints & 3u) return SASQ_ERR_INVALID_ARG;
    if (c->num_pages > 0 && (c->k == nullptr || c->v == nullptr || !aligned16(c->k) || !aligned16(c->v)))
        return SASQ_ERR_INVALID_ARG;
    const int per_word = c->kind == SASQ_KV_INT4 ? 32 : c->kind == SASQ_KV_INT8 ? 16 : 8;      // elements in 16 bytes
    if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return SASQ_ERR_INVALID_ARG;
    if (c->page_stride % per_word != 0 || c->token_stride % per_word != 0 || c->head_stride % per_word != 0)
        return SASQ_ERR_INVALID_ARG;
    const bool factors = c->k_scale != nullptr && c->v_scale != nullptr;
    if (c->kind != SASQ_KV_16BIT ? !factors : (c->k_scale != nullptr || c->v_scale != nullptr)) return SASQ_ERR_INVALID_ARG;
    // 4-bit: a factor per channel, read in 16-byte words
    const uintptr_t odd = (reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale));
    if (odd & (c->kind == SASQ_KV_INT4 ? 15u : 3u)) return SASQ_ERR_INVALID_ARG;
    int shift = 4;
    while (shift < 8 && (1 << shift) != c->page_size) ++shift;
    if ((1 << shift) != c->page_size) return SASQ_ERR_UNSUPPORTED;
    if (c->num_pages > 0x7FFFFFFF || ((long long)b->max_pages << shift) > (1 << 30)) return SASQ_ERR_UNSUPPORTED;
    p->k = c->k;
    p->v = c->v;
    p->k_scale = c->k_scale;
    p->v_scale = c->v_scale;
    p->page_stride = c->page_stride;
    p->token_stride = c->token_stride;
    p->head_stride = c->head_stride;
    p->num_pages = c->num_pages;
    p->page_table = b->page_table;
    p->seq_lens = b->seq_lens;
    p->q_starts = b->q_starts;
    p->table_stride = b->page_table_stride;
    p->batch = b->batch;
    p->max_pages = b->max_pages;
    p->total_q = b->total_q;
    p->page_shift = shift;
    p->kv_heads = c->num_kv_heads;
    p->kind = c->kind;
    return SASQ_OK;
}

}  // namespace sasq

extern "C" int sasq_rope_kv_append(const sasq_kv_cache_t* cache, const sasq_kv_batch_t* batch, const void* q, const void* k,
                                   const void* v, void* q_out, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                   int64_t q_out_stride, int num_q_heads, const float* cos_sin, int64_t max_positions,
                                   int rot_dim, int interleaved, int dt, void* stream) {
    using namespace sasq;
    AppendParams p{};
    const int rc = paged_check(cache, batch, dt, &p.c);
    if (rc != SASQ_OK) return rc;
    if (num_q_heads < 0 || rot_dim < 0 || max_positions < 0) return SASQ_ERR_INVALID_ARG;
    const bool has_q = q != nullptr;
    if (has_q != (q_out != nullptr) || (has_q && num_q_heads == 0)) return SASQ_ERR_INVALID_ARG;
    const int64_t row_kv = (int64_t)cache->num_kv_heads * cache->head_dim, row_q = (int64_t)num_q_heads * cache->head_dim;
    if (batch->total_q > 0) {
        if (k == nullptr || v == nullptr || !aligned16(k) || !aligned16(v) || !aligned16(q) || !aligned16(q_out))
            return SASQ_ERR_INVALID_ARG;
        if (k_stride < row_kv || v_stride < row_kv || k_stride % 8 != 0 || v_stride % 8 != 0) return SASQ_ERR_INVALID_ARG;
        if (has_q && (q_stride < row_q || q_out_stride < row_q || q_stride % 8 != 0 || q_out_stride % 8 != 0))
            return SASQ_ERR_INVALID_ARG;
        // in place a row has to stay where it is: with another stride rows would be written that are still to be read
        if (has_q && q == q_out && q_stride != q_out_stride && batch->total_q > 1) return SASQ_ERR_INVALID_ARG;
        if (rot_dim > 0 && (cos_sin == nullptr || !aligned16(cos_sin))) return SASQ_ERR_INVALID_ARG;
    }
    if (cache->head_dim % 16 != 0 || cache->head_dim > 256 || rot_dim % 16 != 0 || rot_dim > cache->head_dim)
        return SASQ_ERR_UNSUPPORTED;
    if (cache->kind == SASQ_KV_INT4 && cache->head_dim % 32 != 0) return SASQ_ERR_UNSUPPORTED;
    if (batch->total_q == 0 || batch->batch == 0) return SASQ_OK;
    const int sms = device_sm_count_if_sm100();
    if (sms <= 0) return SASQ_ERR_UNSUPPORTED;
    p.c.status = paged_status_ptr();
    if (p.c.status == nullptr) return SASQ_ERR_CUDA;
    p.q = static_cast<const uint16_t*>(q);
    p.k = static_cast<const uint16_t*>(k);
    p.v = static_cast<const uint16_t*>(v);
    p.q_out = static_cast<uint16_t*>(q_out);
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.q_out_stride = q_out_stride;
    p.q_heads = has_q ? num_q_heads : 0;
    p.dim = cache->head_dim;
    p.rot = rot_dim;
    p.interleaved = interleaved != 0;
    p.cos_sin = cos_sin;
    p.max_positions = max_positions;
    // Codes of 4 bits cost more instructions than DRAM's time covers, those before a thread's first head among them: with many
    // tokens a thread takes more heads of one (4815 tokens of 40 + 16 heads of 128, fp16: 34.5 us with 64 threads a block,
    // 36.5 with 128, 46.6 with 256).  Few tokens leave no choice but more threads.
    const int threads = cache->kind == SASQ_KV_INT4 && batch->total_q >= 2 * sms ? kAppend4Threads : kAppendThreads;
    p.head_step = threads / (p.dim >> 4);
    const int heads = p.q_heads + 2 * p.c.kv_heads;
    // few tokens: their heads spread over more blocks, so that a thread has one unit; many: one block per token, whose
    // threads keep their cosines and sines over all heads
    const int steps = (heads + p.head_step - 1) / p.head_step;
    const int ways = batch->total_q >= 2 * sms ? 1 : steps;
    p.heads_per_block = (steps + ways - 1) / ways * p.head_step;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)batch->total_q, (unsigned)((heads + p.heads_per_block - 1) / p.heads_per_block));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr = pdl_attribute();
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    auto go = [&](auto* bf16_kernel, auto* f16_kernel) { return cudaLaunchKernelEx(&cfg, dt == SASQ_BF16 ? bf16_kernel : f16_kernel, p); };
    const cudaError_t e = cache->kind == SASQ_KV_INT4 ? go(rope_kv_append_kernel<true, SASQ_KV_INT4>, rope_kv_append_kernel<false, SASQ_KV_INT4>)
                          : cache->kind == SASQ_KV_INT8 ? go(rope_kv_append_kernel<true, SASQ_KV_INT8>, rope_kv_append_kernel<false, SASQ_KV_INT8>)
                                                        : go(rope_kv_append_kernel<true, SASQ_KV_16BIT>, rope_kv_append_kernel<false, SASQ_KV_16BIT>);
    return e == cudaSuccess ? SASQ_OK : SASQ_ERR_CUDA;
}
