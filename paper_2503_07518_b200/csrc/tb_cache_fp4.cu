// Maintenance of a 4-bit cache (TB_FP4, see tb_fp4.cuh): new rows are scaled and rounded as they enter, keys are projected
// from the rows as they are held.
#include <type_traits>

#include "tb_fp4.cuh"
#include "tb_internal.h"

namespace tb {

// A thread quantises one block of 16 channels: 32 bytes in, 8 bytes of codes and a scale byte out; 16 neighbours share a
// (token, head).  A block belongs to one (layer, sequence).  512 bytes read and 144 written per token and head: 424,000 of them in 52 us, 5.4 TB/s
// (82% of the copy bandwidth), the conversions taking 63% of the ALU's cycles; bound by the launch for a decode token.  With one 32-byte access
// per thread instead of two of 16 and no division; before, 64 us; two blocks of channels in flight per thread instead of four, 7% slower.
constexpr int kQuantThreads = 256;
constexpr int kQuantUnroll = 4;
constexpr int kQuantPairs = kQuantThreads / 16 * kQuantUnroll;        // (token, head) pairs of a block

__global__ void __launch_bounds__(kQuantThreads) append_fp4_kernel(Geom gm, UnitTable ut, AppendTable at, int total_new,
                                                                   const __nv_bfloat16* __restrict__ k_new, const __nv_bfloat16* __restrict__ v_new,
                                                                   unsigned char* __restrict__ kv, int32_t* __restrict__ len_dev,
                                                                   uint32_t* __restrict__ counter, int32_t* __restrict__ status,
                                                                   unsigned char* __restrict__ res_rows, int res_sinks, int res_window) {
    const int ll = blockIdx.y;
    int s = 0;
    for (int step = kMaxLaunchSeq / 2; step > 0; step >>= 1)       // the last sequence that starts at or before this block
        if (s + step < ut.n_seq && at.blk_off[s + step] <= (int)blockIdx.x) s += step;
    const int n_s = at.tok_off[s + 1] - at.tok_off[s];
    pdl_wait();                                        // (see append_kernel)
    pdl_launch_dependents();
    const int base = unit_len(gm, ut, ll, s);
    const unsigned n_pair = (unsigned)n_s * gm.Hkv, j = threadIdx.x & 15;        // pair = (token, head), as in the source
    const unsigned first = (blockIdx.x - at.blk_off[s]) * kQuantPairs + (threadIdx.x >> 4);
    if (base + n_s <= gm.max_seq_len && first < n_pair) {
        const size_t unit0 = ((size_t)(ut.layer_begin + ll) * gm.max_batch + ut.seq_id[s]) * gm.Hkv;
        const size_t src0 = ((size_t)ll * total_new + at.tok_off[s]) * gm.Hkv;
        const unsigned hkv = gm.Hkv;
        const bool wide = (((uintptr_t)k_new | (uintptr_t)v_new) & 31) == 0;
        uint32_t w[kQuantUnroll][8];
#pragma unroll
        for (int i = 0; i < kQuantUnroll; ++i) {
            const unsigned pair = first + i * (kQuantThreads / 16);
            if (pair >= n_pair) break;
            load_32_bytes((j < 8 ? k_new : v_new) + (src0 + pair) * 128 + (j & 7) * 16, wide, w[i]);
        }
#pragma unroll
        for (int i = 0; i < kQuantUnroll; ++i) {
            const unsigned pair = first + i * (kQuantThreads / 16), tok = pair / hkv, h = pair - tok * hkv;
            if (pair >= n_pair) break;
            uint2 codes;
            uint32_t scale;
            fp4_encode(w[i], codes, scale);
            const int pos = base + (int)tok;
            auto write = [&](unsigned char* row) {
                *reinterpret_cast<uint2*>(row + j * 8 + (j < 8 ? 0 : kFp4VCodes - 64)) = codes;
                row[kFp4KScales + j] = (unsigned char)scale;
            };
            write(kv + ((unit0 + h) * gm.max_seq_len + pos) * kFp4Row);
            if (res_rows) {                            // resident copies, as append_kernel keeps them
                int slot = -1;
                if (pos < res_sinks) slot = pos;
                else if (res_window > 0 && pos >= base + n_s - res_window) slot = res_sinks + pos % res_window;
                if (slot >= 0) write(res_rows + ((unit0 + h) * (size_t)(res_sinks + res_window) + slot) * kFp4Row);
            }
        }
    }
    append_finish(gm, ut, at, len_dev, counter, status);
}

cudaError_t launch_append_fp4(const tb_ctx* c, const UnitTable& ut, const int* n_new, const int* tok_off, int total_new,
                              const void* k, const void* v, cudaStream_t s) {
    AppendTable at;
    for (int i = 0; i <= ut.n_seq; ++i) at.tok_off[i] = tok_off[i];
    const Geom& gm = c->geom;
    at.blk_off[0] = 0;
    for (int i = 0; i < ut.n_seq; ++i) at.blk_off[i + 1] = at.blk_off[i] + (int)(((long long)n_new[i] * gm.Hkv + kQuantPairs - 1) / kQuantPairs);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)at.blk_off[ut.n_seq], ut.layer_count, 1);
    cfg.blockDim = dim3(kQuantThreads, 1, 1), cfg.dynamicSmemBytes = 0, cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see pdl_wait()
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr, cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, append_fp4_kernel, gm, ut, at, total_new, (const __nv_bfloat16*)k, (const __nv_bfloat16*)v,
                              (unsigned char*)c->kv, c->st.len, c->st.misc_counter, c->st.status, (unsigned char*)c->res_rows, c->res_sinks,
                              c->res_window);
}

// ---------------------------------------------------------------------------------------------
// Rows as values: a thread turns 8 bytes of codes and a scale into 16 bf16 channels (exact), kReadUnroll of them in flight.  Bound by
// DRAM: 144 bytes in, 512 out, 424,000 rows in 43 us (6.4 TB/s).
constexpr int kReadUnroll = 4;
constexpr int kReadPairs = kQuantThreads / 16 * kReadUnroll;

__global__ void __launch_bounds__(kQuantThreads) read_fp4_kernel(Geom gm, UnitTable ut, ReadTable rt, const unsigned char* __restrict__ kv,
                                                                 __nv_bfloat16* __restrict__ k_out, __nv_bfloat16* __restrict__ v_out) {
    const int ll = blockIdx.z, s = blockIdx.y;
    const unsigned n_pair = (unsigned)(rt.tok_off[s + 1] - rt.tok_off[s]) * gm.Hkv, j = threadIdx.x & 15, hkv = gm.Hkv;
    const size_t unit0 = ((size_t)(ut.layer_begin + ll) * gm.max_batch + ut.seq_id[s]) * gm.Hkv;
    const size_t dst0 = ((size_t)ll * rt.tok_off[ut.n_seq] + rt.tok_off[s]) * gm.Hkv;
    const bool wide = (((uintptr_t)k_out | (uintptr_t)v_out) & 31) == 0;
    for (unsigned first = blockIdx.x * kReadPairs + (threadIdx.x >> 4); first < n_pair; first += gridDim.x * kReadPairs) {
        uint2 codes[kReadUnroll];
        uint32_t scale[kReadUnroll];
#pragma unroll
        for (int i = 0; i < kReadUnroll; ++i) {
            const unsigned pair = first + i * (kQuantThreads / 16), tok = pair / hkv, h = pair - tok * hkv;
            if (pair >= n_pair) break;
            const unsigned char* row = kv + ((unit0 + h) * gm.max_seq_len + rt.pos_begin[s] + tok) * kFp4Row;
            codes[i] = __ldg(reinterpret_cast<const uint2*>(row + j * 8 + (j < 8 ? 0 : kFp4VCodes - 64)));
            scale[i] = __ldg(row + kFp4KScales + j);
        }
#pragma unroll
        for (int i = 0; i < kReadUnroll; ++i) {
            const unsigned pair = first + i * (kQuantThreads / 16);
            if (pair >= n_pair) break;
            const uint32_t sp = fp4_scale_pair<0>(scale[i]);
            uint32_t f[8];
            fp4_unpack(codes[i].x, f[0], f[1], f[2], f[3]);
            fp4_unpack(codes[i].y, f[4], f[5], f[6], f[7]);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = f16x2_to_bf16x2(mul_f16x2(f[e], sp));
            store_32_bytes((j < 8 ? k_out : v_out) + (dst0 + pair) * 128 + (j & 7) * 16, wide, f);
        }
    }
}

cudaError_t launch_read_fp4(const tb_ctx* c, const UnitTable& ut, const ReadTable& rt, int max_tokens, void* k, void* v, cudaStream_t s) {
    const Geom& gm = c->geom;
    const long long blocks = ((long long)max_tokens * gm.Hkv + kReadPairs - 1) / kReadPairs;
    dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536), ut.n_seq, ut.layer_count);
    read_fp4_kernel<<<grid, kQuantThreads, 0, s>>>(gm, ut, rt, (const unsigned char*)c->kv, (__nv_bfloat16*)k, (__nv_bfloat16*)v);
    return cudaGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Key projection from 4-bit rows on the tensor cores (mma.sync m16n8k16, bf16 x bf16 -> fp32): 16 tokens x 128 channels times
// the head's [128][d'] matrix.  The contraction may take the channels in any order, so a lane's share of a row
// is 16 contiguous bytes: lane (gid, tig) holds channels 32 tig .. 32 tig + 31 of rows gid and gid + 8, two scale blocks, and k-step ks
// takes its channels 32 tig + 4 ks + (0, 1 | 2, 3).  The rows of W_K are fetched in the same order, its columns placed so that a lane ends with
// consecutive outputs of its two tokens.
// Codes become f16 pairs and are scaled there, exactly.  W_K is bf16; a warp that walks brings its matrix to f16 too, by a power of two that puts
// the largest element in [2^13, 2^14): exact for elements down to 2^-30 of it.  Where one is smaller, and for few tokens, the keys are turned
// into bf16 instead, also exactly, which costs three instructions per pair (1M rows x d' 32: 53 us like that, 43 on f16).  The products and the
// order of their sums are the same, and so are the results; one rounding, at the end.
// kWalk: a block keeps the matrix in registers and walks over the tokens, each warp a tile of 16 at a time with the next kProjAhead on their
// way.  Otherwise (few tokens per unit, or one key stream per layer, which sums the heads' projections) it is read from shared memory,
// two tiles at a time, and twice as many blocks are resident.  One key stream per layer brings a head's matrix into shared memory for every 128
// tokens, behind two barriers, which bounds it: 4 layers of 32768 tokens of 8 heads, d' 32, 72 us (bf16 rows 51; a stream per head 39).
// Bound by DRAM: of a row's 144 bytes 96 are asked for (three sectors), but memory is read 64 bytes at a time and that is all of it, so 144 in and
// 2 d' out: 1M rows, d' 32, 218 MB in 41 us (5.3 TB/s); rows prefetched into registers 46, 64 tokens and a matrix per block 99.
constexpr int kProjFp4Threads = 128;
constexpr int kProjAhead = 6;
constexpr int kProjRow = 80;                           // bytes of a row that a tile needs: K codes and both halves' scales

// W_K into shared memory, [channel][DP] with a pad of 16 bytes per row; output j = 2 NT t + 2 n + e stands in column 8 n + 2 t + e.
template <int DP>
__device__ __forceinline__ void stage_projection(const __nv_bfloat16* __restrict__ W, unsigned char* Ws) {
    constexpr int NT = DP / 8, kWPitch = DP * 2 + 16;
    for (int i = threadIdx.x; i < 128 * NT; i += kProjFp4Threads) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(W) + i);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        unsigned char* row = Ws + (i / NT) * kWPitch;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = (i % NT) * 8 + 2 * e;
            *reinterpret_cast<uint32_t*>(row + (((j % (2 * NT)) / 2) * 8 + (j / (2 * NT)) * 2) * 2) = w[e];
        }
    }
}
// B fragments of k-step ks and column tiles 2 np, 2 np + 1: matrices (k 0..7, tile 2 np), (k 8..15, same), (k 0..7, tile 2 np + 1), (k 8..15, same);
// row r of the first kind is channel 32 (r / 2) + 4 ks + r % 2, of the second two more.
template <int DP>
__device__ __forceinline__ void projection_fragment(uint32_t ws, int ks, int np, uint32_t (&b)[4]) {
    const int lane = threadIdx.x & 31, mi = lane >> 3, r8 = lane & 7;
    const int ch = 32 * (r8 >> 1) + 4 * ks + (r8 & 1) + 2 * (mi & 1);
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(b[0]), "=r"(b[1]), "=r"(b[2]), "=r"(b[3])
                 : "r"(ws + ch * (DP * 2 + 16) + (np * 16 + (mi >> 1) * 8) * 2));
}
struct KeyTile {                                       // a lane's share of 16 rows: of rows gid and gid + 8
    uint4 code[2];
    uint32_t scale[2];
    __device__ __forceinline__ void load(const unsigned char* rows, int t0, int end) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const unsigned char* row = rows + (size_t)min(t0 + (lane >> 2) + 8 * i, end - 1) * kFp4Row;     // rows past the range repeat the last one
            code[i] = __ldcs(reinterpret_cast<const uint4*>(row + (lane & 3) * 16));
            scale[i] = __ldcs(reinterpret_cast<const unsigned short*>(row + kFp4KScales + (lane & 3) * 2));
        }
    }
    // the same through a stage of 16 rows in shared memory: asked for, then taken
    static __device__ __forceinline__ void ask(uint32_t stage, const unsigned char* rows, int t0, int end) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int item = i * 32 + lane, row = item / 5, chunk = item - row * 5;
            if (item < 80)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(stage + item * 16), "l"(rows + (size_t)min(t0 + row, end - 1) * kFp4Row + chunk * 16) : "memory");
        }
    }
    __device__ __forceinline__ void take(const unsigned char* stage) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const unsigned char* row = stage + ((lane >> 2) + 8 * i) * kProjRow;
            code[i] = *reinterpret_cast<const uint4*>(row + (lane & 3) * 16);
            scale[i] = *reinterpret_cast<const unsigned short*>(row + kFp4KScales + (lane & 3) * 2);
        }
    }
    // A fragments of k-steps 2 j and 2 j + 1, in f16 or bf16
    template <bool kF16>
    __device__ __forceinline__ void fragments(int j, uint32_t (&a)[2][4]) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t w = j == 0 ? code[i].x : j == 1 ? code[i].y : j == 2 ? code[i].z : code[i].w;
            const uint32_t s = j < 2 ? fp4_scale_pair<0>(scale[i]) : fp4_scale_pair<1>(scale[i]);
            uint32_t f[4];
            fp4_unpack(w, f[0], f[1], f[2], f[3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t x = mul_f16x2(f[e], s);
                a[e >> 1][2 * (e & 1) + i] = kF16 ? x : f16x2_to_bf16x2(x);
            }
        }
    }
};
template <bool kF16>
__device__ __forceinline__ void mma_acc(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (kF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The accumulators of 16 tokens, rounded: lane (gid, tig) has outputs 2 NT tig .. of tokens t0 + gid and t0 + gid + 8.
template <int DP>
__device__ __forceinline__ void store_projection(__nv_bfloat16* out, int t0, int end, const float (&acc)[DP / 8][4], float scale = 1.f) {
    constexpr int NT = DP / 8;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int t = t0 + (lane >> 2) + 8 * i;
        uint32_t w[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(acc[n][2 * i] * scale, acc[n][2 * i + 1] * scale);
            w[n] = *reinterpret_cast<const uint32_t*>(&v);
        }
        if (t >= end) continue;
        __nv_bfloat16* dst = out + (size_t)t * DP + (lane & 3) * 2 * NT;
        if constexpr (NT == 4) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
    }
}

template <int DP, bool kWalk>
__global__ void __launch_bounds__(kProjFp4Threads, kWalk ? 3 : 6) project_fp4_kernel(Geom gm, UnitTable ut, ProjectTable pt, const unsigned char* __restrict__ kv,
                                                                      const __nv_bfloat16* __restrict__ Wall, __nv_bfloat16* __restrict__ kimp,
                                                                      int32_t* __restrict__ len_proj_dev, uint32_t* __restrict__ counter) {
    constexpr int D = 128, NT = DP / 8;
    __shared__ __align__(16) unsigned char Ws[D * (DP * 2 + 16)];
    __shared__ __align__(16) unsigned char ring[kWalk ? kProjFp4Threads / 32 * kProjAhead * 16 * kProjRow : 16];
    const int ll = blockIdx.z / ut.n_seq, s = blockIdx.z % ut.n_seq, h = blockIdx.y;
    const int layer = ut.layer_begin + ll, warp = threadIdx.x >> 5;
    // The (first) matrix is fetched beside the predecessor's tail: tb_set_projection's copy is no kernel, so it was complete when the predecessor
    // began.  Rows, and lengths read on the device, may be the predecessor's.
    stage_projection<DP>(Wall + ((size_t)layer * gm.Hkv + (kWalk ? h : h * (gm.Hkv / gm.Hi))) * D * DP, Ws);
    pdl_wait();
    pdl_launch_dependents();
    int begin, end;
    project_range(gm, ut, pt, ll, s, begin, end);
    const size_t pair = (size_t)layer * gm.max_batch + ut.seq_id[s];
    const uint32_t ws = smem_u32(Ws);
    __nv_bfloat16* out = kimp + (pair * gm.Hi + h) * gm.max_seq_len * DP;
    // (a launch under device lengths is sized for the longest range that can be: blocks beyond it have nothing to do)
    if constexpr (kWalk) {
        const int step = gridDim.x * (kProjFp4Threads / 32) * 16;
        const int first = begin + (blockIdx.x * (kProjFp4Threads / 32) + warp) * 16;
        if (begin + (int)blockIdx.x * (kProjFp4Threads / 32) * 16 < end) {             // (the same for all of the block)
            const unsigned char* rows = kv + (pair * gm.Hkv + h) * gm.max_seq_len * kFp4Row;
            const unsigned char* stages = ring + warp * kProjAhead * 16 * kProjRow;
            const uint32_t stages_u32 = smem_u32(stages);
            // (a group per tile, empty or not: all but the newest kProjAhead - 1 have landed when one is taken)
#pragma unroll
            for (int i = 0; i < kProjAhead; ++i) {
                if ((long long)first + (long long)i * step < end) KeyTile::ask(stages_u32 + i * 16 * kProjRow, rows, first + i * step, end);
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
            __syncthreads();
            uint32_t b[8][NT / 2][4];
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
#pragma unroll
                for (int np = 0; np < NT / 2; ++np) projection_fragment<DP>(ws, ks, np, b[ks][np]);
            // the matrix in f16, if that is exact (every warp holds all of it: they agree)
            uint32_t top2 = 0;
#pragma unroll
            for (int i = 0; i < 8 * NT * 2; ++i) top2 = __vmaxu2(top2, b[i / (2 * NT)][i / 4 % (NT / 2)][i % 4] & 0x7fff7fffu);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, o));
            const uint32_t e = min(max(max(top2 & 0xffffu, top2 >> 16) >> 7, 14u), 253u);
            const float up = __uint_as_float((267u - e) << 23), down = __uint_as_float((e - 13u) << 23);
            bool exact = max(top2 & 0xffffu, top2 >> 16) <= 0x7f7fu;
#pragma unroll
            for (int i = 0; i < 8 * NT * 2; ++i) {
                const uint32_t w = b[i / (2 * NT)][i / 4 % (NT / 2)][i % 4];
                const __half2 h = __floats2half2_rn(bf16_lo(w) * up, bf16_hi(w) * up);
                const float2 f = __half22float2(h);
                exact &= f.x == bf16_lo(w) * up && f.y == bf16_hi(w) * up;
            }
            exact = __all_sync(0xffffffffu, exact);
            if (exact) {
#pragma unroll
                for (int i = 0; i < 8 * NT * 2; ++i) {
                    uint32_t& w = b[i / (2 * NT)][i / 4 % (NT / 2)][i % 4];
                    const __half2 h = __floats2half2_rn(bf16_lo(w) * up, bf16_hi(w) * up);
                    w = *reinterpret_cast<const uint32_t*>(&h);
                }
            }
            auto walk = [&](auto f16) {
                constexpr bool kF16 = decltype(f16)::value;
                int stage = 0;
                for (long long t0 = first; t0 < end; t0 += step) {
                    asm volatile("cp.async.wait_group %0;" ::"n"(kProjAhead - 1) : "memory");
                    __syncwarp();
                    KeyTile now;
                    now.take(stages + stage * 16 * kProjRow);
                    __syncwarp();
                    if (t0 + (long long)kProjAhead * step < end) KeyTile::ask(stages_u32 + stage * 16 * kProjRow, rows, (int)t0 + kProjAhead * step, end);
                    asm volatile("cp.async.commit_group;" ::: "memory");
                    stage = stage + 1 == kProjAhead ? 0 : stage + 1;
                    float acc[NT][4];
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t a[2][4];
                        now.fragments<kF16>(j, a);
#pragma unroll
                        for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
                            for (int n = 0; n < NT; ++n) mma_acc<kF16>(acc[n], a[k2], b[2 * j + k2][n / 2][2 * (n & 1)], b[2 * j + k2][n / 2][2 * (n & 1) + 1]);
                    }
                    store_projection<DP>(out, (int)t0, end, acc, kF16 ? down : 1.f);
                }
                asm volatile("cp.async.wait_group 0;" ::: "memory");
            };
            if (exact) walk(std::true_type{});
            else walk(std::false_type{});
        }
    } else {
        // (one key stream per layer: the heads' projections are summed in the accumulators, heads in ascending order)
        const int n_sum = gm.Hkv / gm.Hi;
        int staged = h * n_sum;                        // whose matrix is in shared memory
        constexpr int kTiles = 2, kTokens = kProjFp4Threads / 32 * 16 * kTiles;
        for (int t0 = begin + blockIdx.x * kTokens; t0 < end; t0 += gridDim.x * kTokens) {
            const int tw = t0 + warp * 16 * kTiles;
            float acc[kTiles][NT][4];
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.f;
            for (int hk = h * n_sum; hk < (h + 1) * n_sum; ++hk) {
                const unsigned char* rows = kv + (pair * gm.Hkv + hk) * gm.max_seq_len * kFp4Row;
                KeyTile tile[kTiles];
#pragma unroll
                for (int i = 0; i < kTiles; ++i) tile[i].load(rows, min(tw + 16 * i, end - 1), end);
                __syncthreads();                                       // the previous matrix has been read, or the first one written
                if (hk != staged) {
                    stage_projection<DP>(Wall + ((size_t)layer * gm.Hkv + hk) * D * DP, Ws);
                    staged = hk;
                    __syncthreads();
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t a[kTiles][2][4];
#pragma unroll
                    for (int i = 0; i < kTiles; ++i) tile[i].fragments<false>(j, a[i]);
#pragma unroll
                    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
                        for (int np = 0; np < NT / 2; ++np) {
                            uint32_t b[4];
                            projection_fragment<DP>(ws, 2 * j + k2, np, b);
#pragma unroll
                            for (int i = 0; i < kTiles; ++i) {
                                mma_acc<false>(acc[i][2 * np], a[i][k2], b[0], b[1]);
                                mma_acc<false>(acc[i][2 * np + 1], a[i][k2], b[2], b[3]);
                            }
                        }
                }
            }
#pragma unroll
            for (int i = 0; i < kTiles; ++i) store_projection<DP>(out, tw + 16 * i, end, acc[i]);
        }
    }
    project_finish(gm, ut, pt, len_proj_dev, counter);
}

cudaError_t launch_project_fp4(const tb_ctx* c, const UnitTable& ut, const ProjectTable& pt, int max_range, cudaStream_t s) {
    const Geom& gm = c->geom;
    const int units = gm.Hi * ut.layer_count * ut.n_seq;
    const bool walk = gm.Hi == gm.Hkv && max_range > 32 * (kProjFp4Threads / 32);
    const int tokens = (walk ? 16 : 32) * (kProjFp4Threads / 32);      // of a block's pass
    int bx = (max_range + tokens - 1) / tokens;
    const int most = (walk ? 3 : 6) * c->sm_count / units;             // what is resident at once: a block goes on with the rest
    if (bx > most) bx = most > 0 ? most : 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(bx, gm.Hi, ut.layer_count * ut.n_seq);
    cfg.blockDim = dim3(kProjFp4Threads, 1, 1), cfg.dynamicSmemBytes = 0, cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see pdl_wait()
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr, cfg.numAttrs = 1;
    auto launch = [&](auto kernel) {
        return cudaLaunchKernelEx(&cfg, kernel, gm, ut, pt, (const unsigned char*)c->kv, (const __nv_bfloat16*)c->st.W, (__nv_bfloat16*)c->kimp, c->st.len_proj,
                                  c->st.misc_counter + 1);
    };
    if (gm.dp == 32) return walk ? launch(project_fp4_kernel<32, true>) : launch(project_fp4_kernel<32, false>);
    return walk ? launch(project_fp4_kernel<16, true>) : launch(project_fp4_kernel<16, false>);
}

}  // namespace tb
