// Maintenance of a 4-bit cache (TB_FP4, see tb_fp4.cuh): new rows are scaled and rounded as they enter, keys are projected
// from the rows as they are held.
#include "tb_fp4.cuh"
#include "tb_internal.h"

namespace tb {

// A thread quantises one block of 16 channels: 32 bytes in, 8 bytes of codes and a scale byte out; 16 neighbours share a
// (token, head).  A block belongs to one (layer, sequence).  Bound by DRAM bandwidth for prompts (512 bytes read, 144 written per
// token and head) and by the launch for a decode token.
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
        uint32_t w[kQuantUnroll][8];
#pragma unroll
        for (int i = 0; i < kQuantUnroll; ++i) {
            const unsigned pair = first + i * (kQuantThreads / 16);
            if (pair >= n_pair) break;
            const uint4* src = reinterpret_cast<const uint4*>((j < 8 ? k_new : v_new) + (src0 + pair) * 128 + (j & 7) * 16);
            const uint4 a = __ldcs(src), b = __ldcs(src + 1);
            w[i][0] = a.x, w[i][1] = a.y, w[i][2] = a.z, w[i][3] = a.w, w[i][4] = b.x, w[i][5] = b.y, w[i][6] = b.z, w[i][7] = b.w;
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
// Rows as values: a thread turns 8 bytes of codes and a scale into 16 bf16 channels (exact).
__global__ void __launch_bounds__(kQuantThreads) read_fp4_kernel(Geom gm, UnitTable ut, ReadTable rt, const unsigned char* __restrict__ kv,
                                                                 __nv_bfloat16* __restrict__ k_out, __nv_bfloat16* __restrict__ v_out) {
    const int ll = blockIdx.z, s = blockIdx.y;
    const int n_s = rt.tok_off[s + 1] - rt.tok_off[s];
    const unsigned n_pair = (unsigned)n_s * gm.Hkv, j = threadIdx.x & 15;
    const size_t unit0 = ((size_t)(ut.layer_begin + ll) * gm.max_batch + ut.seq_id[s]) * gm.Hkv;
    const size_t dst0 = ((size_t)ll * rt.tok_off[ut.n_seq] + rt.tok_off[s]) * gm.Hkv;
    const unsigned hkv = gm.Hkv;
    for (unsigned pair = blockIdx.x * (kQuantThreads / 16) + (threadIdx.x >> 4); pair < n_pair; pair += gridDim.x * (kQuantThreads / 16)) {
        const unsigned tok = pair / hkv, h = pair - tok * hkv;
        const unsigned char* row = kv + ((unit0 + h) * gm.max_seq_len + rt.pos_begin[s] + tok) * kFp4Row;
        const uint2 codes = *reinterpret_cast<const uint2*>(row + j * 8 + (j < 8 ? 0 : kFp4VCodes - 64));
        const uint32_t scale = fp4_scale_pair<0>(row[kFp4KScales + j]);
        uint32_t f[8];
        fp4_unpack(codes.x, f[0], f[1], f[2], f[3]);
        fp4_unpack(codes.y, f[4], f[5], f[6], f[7]);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f16x2_to_bf16x2(mul_f16x2(f[i], scale));
        uint4* dst = reinterpret_cast<uint4*>((j < 8 ? k_out : v_out) + (dst0 + pair) * 128 + (j & 7) * 16);
        dst[0] = make_uint4(f[0], f[1], f[2], f[3]);
        dst[1] = make_uint4(f[4], f[5], f[6], f[7]);
    }
}

cudaError_t launch_read_fp4(const tb_ctx* c, const UnitTable& ut, const ReadTable& rt, int max_tokens, void* k, void* v, cudaStream_t s) {
    const Geom& gm = c->geom;
    const long long blocks = ((long long)max_tokens * gm.Hkv + kQuantThreads / 16 - 1) / (kQuantThreads / 16);
    dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536), ut.n_seq, ut.layer_count);
    read_fp4_kernel<<<grid, kQuantThreads, 0, s>>>(gm, ut, rt, (const unsigned char*)c->kv, (__nv_bfloat16*)k, (__nv_bfloat16*)v);
    return cudaGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Key projection from 4-bit rows on the tensor cores (mma.sync m16n8k16, bf16 x bf16 -> fp32): 16 tokens x 128 channels times
// the head's [128][d'] matrix.  The contraction may take the channels in any order, so a lane's share of a row
// is 16 contiguous bytes: lane (gid, tig) holds channels 32 tig .. 32 tig + 31 of rows gid and gid + 8, two scale blocks, and k-step ks
// takes its channels 32 tig + 4 ks + (0, 1 | 2, 3).  The rows of W_K are fetched in the same order.
// Codes become f16 pairs, are scaled there and turned into bf16, all exactly; one rounding, of the result.
constexpr int kProjFp4Threads = 128;

template <int DP>
__global__ void __launch_bounds__(kProjFp4Threads) project_fp4_kernel(Geom gm, UnitTable ut, ProjectTable pt, const unsigned char* __restrict__ kv,
                                                                      const __nv_bfloat16* __restrict__ Wall, __nv_bfloat16* __restrict__ kimp,
                                                                      int32_t* __restrict__ len_proj_dev, uint32_t* __restrict__ counter) {
    constexpr int D = 128, NT = DP / 8;
    constexpr int kWPitch = DP * 2 + 16;
    constexpr int kTokens = kProjFp4Threads / 32 * 16;                 // tokens per pass of the block
    __shared__ __align__(16) unsigned char Ws[D * kWPitch];
    const int ll = blockIdx.z / ut.n_seq, s = blockIdx.z % ut.n_seq, h = blockIdx.y;
    const int layer = ut.layer_begin + ll;
    int begin, end;
    project_range(gm, ut, pt, ll, s, begin, end);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
    const int mi = lane >> 3, r8 = lane & 7;
    const int n_sum = gm.Hkv / gm.Hi;
    const size_t pair = (size_t)layer * gm.max_batch + ut.seq_id[s];
    const uint32_t ws_u32 = smem_u32(Ws);
    // (a launch under device lengths is sized for the longest range that can be: blocks beyond it have nothing to do)
    for (int t0 = begin + blockIdx.x * kTokens; t0 < end; t0 += gridDim.x * kTokens) {
        const int tA = t0 + warp * 16 + gid, tB = tA + 8;
        float acc[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
        for (int hs = 0; hs < n_sum; ++hs) {
            const int hk = h * n_sum + hs;
            __syncthreads();                                           // the previous matrix has been read
            const unsigned char* wbase = reinterpret_cast<const unsigned char*>(Wall + ((size_t)layer * gm.Hkv + hk) * D * DP);
            for (int i = tid; i < D * NT; i += kProjFp4Threads)
                *reinterpret_cast<uint4*>(Ws + (i / NT) * kWPitch + (i % NT) * 16) = __ldg(reinterpret_cast<const uint4*>(wbase) + i);
            __syncthreads();
            const unsigned char* rows = kv + (pair * gm.Hkv + hk) * gm.max_seq_len * kFp4Row;
            uint4 code[2];
            uint32_t sc[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const unsigned char* row = rows + (size_t)min(i ? tB : tA, end - 1) * kFp4Row;    // rows past the range repeat the last one
                code[i] = *reinterpret_cast<const uint4*>(row + tig * 16);
                sc[i] = *reinterpret_cast<const unsigned short*>(row + kFp4KScales + tig * 2);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {                              // eight channels of the lane: two k-steps
                uint32_t a[2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t w = j == 0 ? code[i].x : j == 1 ? code[i].y : j == 2 ? code[i].z : code[i].w;
                    const uint32_t scale = j < 2 ? fp4_scale_pair<0>(sc[i]) : fp4_scale_pair<1>(sc[i]);
                    fp4_unpack(w, a[i][0], a[i][1], a[i][2], a[i][3]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[i][e] = f16x2_to_bf16x2(mul_f16x2(a[i][e], scale));
                }
#pragma unroll
                for (int k2 = 0; k2 < 2; ++k2) {
                    const int ks = 2 * j + k2;
#pragma unroll
                    for (int np = 0; np < NT / 2; ++np) {
                        // matrices: (k 0..7, outputs np * 16 + 0..7), (k 8..15, same), (k 0..7, outputs + 8), (k 8..15, + 8); row r
                        // of the first kind is channel 32 (r / 2) + 4 ks + r % 2, of the second two more
                        uint32_t b0, b1, b2, b3;
                        const int ch = 32 * (r8 >> 1) + 4 * ks + (r8 & 1) + 2 * (mi & 1);
                        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                                     : "=r"(b0), "=r"(b1), "=r"(b2), "=r"(b3)
                                     : "r"(ws_u32 + ch * kWPitch + (np * 16 + (mi >> 1) * 8) * 2));
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            float* d = acc[2 * np + q];
                            asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                                         : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                                         : "r"(a[0][2 * k2]), "r"(a[1][2 * k2]), "r"(a[0][2 * k2 + 1]), "r"(a[1][2 * k2 + 1]), "r"(q ? b2 : b0), "r"(q ? b3 : b1));
                        }
                    }
                }
            }
        }
        __nv_bfloat16* out = kimp + (pair * gm.Hi + h) * gm.max_seq_len * DP;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int j = n * 8 + tig * 2;
            if (tA < end) *reinterpret_cast<__nv_bfloat162*>(out + (size_t)tA * DP + j) = __floats2bfloat162_rn(acc[n][0], acc[n][1]);
            if (tB < end) *reinterpret_cast<__nv_bfloat162*>(out + (size_t)tB * DP + j) = __floats2bfloat162_rn(acc[n][2], acc[n][3]);
        }
    }
    project_finish(gm, ut, pt, len_proj_dev, counter);
}

cudaError_t launch_project_fp4(const tb_ctx* c, const UnitTable& ut, const ProjectTable& pt, int max_range, cudaStream_t s) {
    const Geom& gm = c->geom;
    dim3 grid((max_range + 63) / 64, gm.Hi, ut.layer_count * ut.n_seq);
    const unsigned char* kvp = (const unsigned char*)c->kv;
    const __nv_bfloat16* wp = (const __nv_bfloat16*)c->st.W;
    if (gm.dp == 32) project_fp4_kernel<32><<<grid, kProjFp4Threads, 0, s>>>(gm, ut, pt, kvp, wp, (__nv_bfloat16*)c->kimp, c->st.len_proj, c->st.misc_counter + 1);
    else project_fp4_kernel<16><<<grid, kProjFp4Threads, 0, s>>>(gm, ut, pt, kvp, wp, (__nv_bfloat16*)c->kimp, c->st.len_proj, c->st.misc_counter + 1);
    return cudaGetLastError();
}

}  // namespace tb
