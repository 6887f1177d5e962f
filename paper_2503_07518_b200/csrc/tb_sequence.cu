// Cached sequences as wholes: copying one into other slots (parallel samples, beams, a shared prompt) and dropping tokens of one in
// place (rejected drafts, a branch that keeps part of its context).  Rows are moved as bytes, whatever their type.
#include "tb_common.cuh"
#include "tb_internal.h"

namespace tb {

namespace {

// The streams of rows that a (layer, sequence) holds: one per KV head in the K|V cache, then one per head of the projected keys.
struct RowStream {
    uint4* base;          // of the cache's first unit
    int heads, h, chunks; // units per (layer, sequence); this one; 16-byte chunks of a row
    __device__ __forceinline__ RowStream(const Geom& gm, void* kv, void* kimp, int stream) {
        const bool rows = stream < gm.Hkv;
        base = reinterpret_cast<uint4*>(rows ? kv : kimp);
        heads = rows ? gm.Hkv : gm.Hi, h = rows ? stream : stream - gm.Hkv;
        chunks = (rows ? gm.row_bytes : gm.dp * (gm.dtype == TB_BF16 ? 2 : 4)) / 16;
    }
    __device__ __forceinline__ uint4* unit(const Geom& gm, int layer, int seq) const {
        return base + (((size_t)layer * gm.max_batch + seq) * heads + h) * gm.max_seq_len * chunks;
    }
};

}  // namespace

// A unit's rows are contiguous, so a copy is one run of bytes per unit, read once and written to every slot; a block takes 32 KB of it.
// Bound by DRAM: 16384 4-bit tokens of 8 heads and 8 layers to eight slots (1.96 GB) 317 us, 94% of the copy bandwidth; 348 with a couple
// of waves of blocks that walk over the rest.
constexpr int kForkThreads = 256;
constexpr int kForkUnroll = 8;

__global__ void __launch_bounds__(kForkThreads) fork_kernel(Geom gm, UnitTable ut, ForkArgs a, void* __restrict__ kv, void* __restrict__ kimp,
                                                            int32_t* __restrict__ lists, int32_t* __restrict__ counts,
                                                            int32_t* __restrict__ len_dev, int32_t* __restrict__ len_proj_dev,
                                                            uint32_t* __restrict__ counter) {
    const int layer = ut.layer_begin + blockIdx.z, stream = blockIdx.y;
    int n = unit_len(gm, ut, blockIdx.z, 0);
    if (a.n_tokens >= 0) n = min(n, a.n_tokens);
    if (stream < gm.Hkv + gm.Hi) {
        const RowStream rs(gm, kv, kimp, stream);
        const uint4* src = rs.unit(gm, layer, a.src);
        const size_t total = (size_t)n * rs.chunks, step = (size_t)gridDim.x * kForkThreads * kForkUnroll;
        for (size_t at = (size_t)blockIdx.x * kForkThreads * kForkUnroll + threadIdx.x; at < total; at += step) {
            uint4 v[kForkUnroll];
#pragma unroll
            for (int i = 0; i < kForkUnroll; ++i)
                if (at + i * kForkThreads < total) v[i] = src[at + i * kForkThreads];
            for (int d = 0; d < a.n_dst; ++d) {
                uint4* dst = rs.unit(gm, layer, a.dst[d]);
#pragma unroll
                for (int i = 0; i < kForkUnroll; ++i)
                    if (at + i * kForkThreads < total) dst[at + i * kForkThreads] = v[i];
            }
        }
    } else if (a.n_tokens < 0) {                       // the stored lists
        const size_t unit = ((size_t)layer * gm.max_batch + a.src) * gm.Hl;
        for (int h = blockIdx.x; h < gm.Hl; h += gridDim.x) {
            const int cnt = counts[unit + h], m = max(0, min(cnt, gm.idx_cap));
            for (int d = 0; d < a.n_dst; ++d) {
                const size_t to = ((size_t)layer * gm.max_batch + a.dst[d]) * gm.Hl + h;
                for (int i = threadIdx.x; i < m; i += kForkThreads) lists[to * gm.idx_cap + i] = lists[(unit + h) * gm.idx_cap + i];
                if (threadIdx.x == 0) counts[to] = cnt;
            }
        }
    }
    if (!ut.use_dev_len || !last_block_arrives(counter, gridDim.x * gridDim.y * gridDim.z)) return;
    for (int i = threadIdx.x; i < ut.layer_count * a.n_dst; i += kForkThreads) {
        const size_t row = (size_t)(ut.layer_begin + i / a.n_dst) * gm.max_batch;
        const int L = len_dev[row + a.src], P = len_proj_dev[row + a.src], most = a.n_tokens < 0 ? L : min(L, a.n_tokens);
        len_dev[row + a.dst[i % a.n_dst]] = most, len_proj_dev[row + a.dst[i % a.n_dst]] = min(P, most);
    }
}

cudaError_t launch_fork(const tb_ctx* c, const UnitTable& ut, const ForkArgs& a, cudaStream_t s) {
    const Geom& gm = c->geom;
    const int streams = gm.Hkv + gm.Hi + (a.n_tokens < 0 ? 1 : 0);
    const long long chunks = (long long)a.max_tokens * (gm.row_bytes / 16);
    long long bx = (chunks + kForkThreads * kForkUnroll - 1) / (kForkThreads * kForkUnroll);
    if (bx < 1) bx = 1;
    dim3 grid((unsigned)bx, streams, ut.layer_count);
    fork_kernel<<<grid, kForkThreads, 0, s>>>(gm, ut, a, c->kv, c->kimp, c->st.idx, c->st.cnt, c->st.len, c->st.len_proj, c->st.misc_counter + 2);
    return cudaGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Row begin + j becomes row keep[j], in place.  Kept positions ascend, so keep[j] >= begin + j: a row only ever moves down,
// onto rows that are read with it or were read before it.  A block takes one unit's rows in order, a tile at a time: all threads
// have read tile t (and, behind the barrier, know it) before any writes it, and what tile t writes lies below all that later tiles
// read, so the next tile's rows are on their way before this one's are written.  Columns of a row do not depend on one another: where
// there are too few units to fill the chip, a unit is cut into slices of columns, a block each.  A few rows per unit (accepted drafts) are a
// warp's work instead (kGroup threads; 1024 units of 8 rows: 3.5 us behind the launch before, 6 with a block each).
// Bound by DRAM: copying 32768 bf16 tokens of 8 heads and 4 layers and keeping 15565 of them (1.78 GB) takes 300 us, 91% of the copy bandwidth;
// 383 when entries were fetched with their rows, 1290 with a block per unit.
// Entries that do not ascend or lie outside [begin, length) are reported and their rows left alone (the order above holds for
// any entry >= begin + j, and others are not followed).
// Lengths read on the device may differ from what the host checked.  A layer of a sequence is then left as it is, whole, where it is shorter than the
// counts say (kStatusBadIndex), or where the projected tokens end among those it may keep (kStatusUnprojected: a projected length is a prefix
// and could not say which of the kept rows have their keys).
__device__ __forceinline__ bool compact_partial(const Geom& gm, const UnitTable& ut, const CompactArgs& a, int ll, int s, int L) {
    if (!ut.use_dev_len || a.n_keep[s] == 0) return false;
    const int P = ut.len_proj_dev[(size_t)(ut.layer_begin + ll) * gm.max_batch + ut.seq_id[s]];
    return P > a.begin[s] && P < L;
}
constexpr int kCompactThreads = 256;
constexpr int kCompactUnroll = 8;

template <int kGroup>
__global__ void __launch_bounds__(kCompactThreads, 2) compact_kernel(Geom gm, UnitTable ut, CompactArgs a, void* __restrict__ kv, void* __restrict__ kimp,
                                                                     int32_t* __restrict__ len_dev, int32_t* __restrict__ len_proj_dev,
                                                                     uint32_t* __restrict__ counter, int32_t* __restrict__ status) {
    const int n_kv = gm.Hkv * a.kv_slices, n_streams = n_kv + gm.Hi * a.imp_slices;
    const int group = blockIdx.x * (kCompactThreads / kGroup) + threadIdx.x / kGroup, me = threadIdx.x % kGroup;
    const bool there = group < n_streams * ut.layer_count * ut.n_seq;  // (the last block's groups may be more than are left)
    const int z = there ? group / n_streams : 0, y = there ? group % n_streams : 0;
    const int ll = z / ut.n_seq, s = z % ut.n_seq;
    const int stream = y < n_kv ? y / a.kv_slices : gm.Hkv + (y - n_kv) / a.imp_slices;
    const int slices = y < n_kv ? a.kv_slices : a.imp_slices, slice = y < n_kv ? y % slices : (y - n_kv) % slices;
    const RowStream rs(gm, kv, kimp, stream);
    pdl_wait();                                        // (see append_kernel)
    pdl_launch_dependents();
    const int begin = a.begin[s], L = unit_len(gm, ut, ll, s);
    const bool partial = compact_partial(gm, ut, a, ll, s, L);
    // (the sequence that is too short is reported with the bad entries, behind the loop: decided here with the other one, the loop took 9% longer)
    const int n = there && begin + a.n_keep[s] <= L && !partial ? a.n_keep[s] : 0;
    bool bad = begin + a.n_keep[s] > L;
    const int wide = rs.chunks / slices, rows = kGroup / wide;        // chunks of the slice; rows that the group moves side by side
    const int row0 = me / wide;
    const bool works = row0 < rows;
    uint4* unit = rs.unit(gm, ut.layer_begin + ll, ut.seq_id[s]) + slice * wide + (me - row0 * wide);
    const int32_t* keep = a.keep + (size_t)s * a.stride;
    const int tile = rows * kCompactUnroll;
    int from[kCompactUnroll];                          // rows of the tile that is on its way: -1 = stays
    int entry[kCompactUnroll], before[kCompactUnroll]; // entries of the one behind it, and those before them
    uint4 v[kCompactUnroll];
    auto fetch = [&](int j0) {
#pragma unroll
        for (int i = 0; i < kCompactUnroll; ++i) {
            const int j = j0 + row0 + i * rows;
            // (not through the read-only path: the predecessor may have written them while this kernel was already there)
            if (works && j < n) entry[i] = __ldcg(keep + j), before[i] = j ? __ldcg(keep + j - 1) : -1;
        }
    };
    auto load = [&](int j0) {
#pragma unroll
        for (int i = 0; i < kCompactUnroll; ++i) {
            const int j = j0 + row0 + i * rows;
            from[i] = -1;
            if (works && j < n) {
                const bool ok = entry[i] >= begin + j && entry[i] < L && before[i] < entry[i];
                bad |= !ok;
                if (ok && entry[i] > begin + j) from[i] = entry[i], v[i] = __ldcg(unit + (size_t)entry[i] * rs.chunks);
            }
        }
    };
    fetch(0);
    load(0);
    fetch(tile);
    for (int j0 = 0; j0 < n; j0 += tile) {
        uint4 w[kCompactUnroll];
        unsigned moves = 0;
#pragma unroll
        for (int i = 0; i < kCompactUnroll; ++i) w[i] = v[i], moves |= (unsigned)(from[i] >= 0) << i;
        load(j0 + tile);
        fetch(j0 + 2 * tile);
        if constexpr (kGroup == 32) __syncwarp();
        else __syncthreads();
#pragma unroll
        for (int i = 0; i < kCompactUnroll; ++i)
            if (moves >> i & 1) unit[(size_t)(begin + j0 + row0 + i * rows) * rs.chunks] = w[i];
    }
    if (bad) atomicExch(status, kStatusBadIndex);
    if (partial && there && me == 0) atomicExch(status, kStatusUnprojected);
    if (!ut.use_dev_len || !last_block_arrives(counter, gridDim.x * gridDim.y * gridDim.z)) return;
    for (int i = threadIdx.x; i < ut.layer_count * ut.n_seq; i += kCompactThreads) {
        const int s2 = i % ut.n_seq, want = a.begin[s2] + a.n_keep[s2];
        const size_t pair = (size_t)(ut.layer_begin + i / ut.n_seq) * gm.max_batch + ut.seq_id[s2];
        const int len = min(len_dev[pair], want);
        if (compact_partial(gm, ut, a, i / ut.n_seq, s2, len_dev[pair])) continue;
        len_dev[pair] = len;
        if (len_proj_dev[pair] > len) len_proj_dev[pair] = len;
    }
}

cudaError_t launch_compact(const tb_ctx* c, const UnitTable& ut, const CompactArgs& a_in, cudaStream_t s) {
    const Geom& gm = c->geom;
    CompactArgs a = a_in;
    const int kv_chunks = gm.row_bytes / 16, imp_chunks = gm.dp * (gm.dtype == TB_BF16 ? 2 : 4) / 16, units = ut.layer_count * ut.n_seq;
    a.kv_slices = a.imp_slices = 1;
    // up to two of a warp's tiles: a warp each, its rows at most 32 chunks wide; up to two of a block's are not worth cutting
    const long long kv_work = (long long)a.max_keep * kv_chunks;
    const bool warps = kv_work <= 2 * 32 * kCompactUnroll;
    if (warps) {
        a.kv_slices = (kv_chunks + 31) / 32;
    } else if (kv_work > 2 * kCompactThreads * kCompactUnroll) {
        for (int wide = 64; wide >= 2; wide /= 2) {
            a.kv_slices = !gm.fp4 ? (kv_chunks + wide - 1) / wide : wide >= 9 ? 1 : wide >= 3 ? 3 : 9;
            a.imp_slices = (imp_chunks + wide - 1) / wide;
            if (units * (gm.Hkv * a.kv_slices + gm.Hi * a.imp_slices) >= 2 * c->sm_count) break;
        }
    }
    const int groups = units * (gm.Hkv * a.kv_slices + gm.Hi * a.imp_slices), per_block = warps ? kCompactThreads / 32 : 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((groups + per_block - 1) / per_block, 1, 1);
    cfg.blockDim = dim3(kCompactThreads, 1, 1), cfg.dynamicSmemBytes = 0, cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see pdl_wait()
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr, cfg.numAttrs = 1;
    auto launch = [&](auto kernel) {
        return cudaLaunchKernelEx(&cfg, kernel, gm, ut, a, c->kv, c->kimp, c->st.len, c->st.len_proj, c->st.misc_counter + 3, c->st.status);
    };
    return warps ? launch(compact_kernel<32>) : launch(compact_kernel<kCompactThreads>);
}

// ---------------------------------------------------------------------------------------------
// Resident rows (offloaded KV) of sequences whose rows have moved: the first res_sinks tokens and the res_window most recent ones.
__global__ void __launch_bounds__(256) refresh_resident_kernel(Geom gm, UnitTable ut, const uint4* __restrict__ kv, uint4* __restrict__ res, int sinks, int window) {
    const int ll = blockIdx.z / ut.n_seq, s = blockIdx.z % ut.n_seq, chunks = gm.row_bytes / 16;
    const int L = unit_len(gm, ut, ll, s);
    const size_t unit = (((size_t)(ut.layer_begin + ll) * gm.max_batch + ut.seq_id[s]) * gm.Hkv + blockIdx.y);
    const int n_sink = min(sinks, L), w_begin = max(n_sink, L - window), n = n_sink + L - w_begin;
    const uint4* src = kv + unit * gm.max_seq_len * chunks;
    uint4* dst = res + unit * (size_t)(sinks + window) * chunks;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < (long long)n * chunks; i += (long long)gridDim.x * blockDim.x) {
        const int row = (int)(i / chunks), t = row < n_sink ? row : w_begin + row - n_sink;
        const int slot = t < sinks ? t : sinks + t % window;
        dst[(size_t)slot * chunks + i % chunks] = src[(size_t)t * chunks + i % chunks];
    }
}

cudaError_t launch_refresh_resident(const tb_ctx* c, const UnitTable& ut, cudaStream_t s) {
    const Geom& gm = c->geom;
    const long long chunks = ((long long)c->res_sinks + c->res_window) * (gm.row_bytes / 16);
    dim3 grid((unsigned)(chunks < 256 * 64 ? (chunks + 255) / 256 : 64), gm.Hkv, ut.layer_count * ut.n_seq);
    refresh_resident_kernel<<<grid, 256, 0, s>>>(gm, ut, (const uint4*)c->kv, (uint4*)c->res_rows, c->res_sinks, c->res_window);
    return cudaGetLastError();
}

}  // namespace tb
