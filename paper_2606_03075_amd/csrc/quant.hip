// The paged cache in 8 bits: the retained rows quantised as they are written, and rows read back.
//
// Both are HBM streams.  compact_pages_kernel is compact_kernel with a different store: a row of head_dim
// bf16 is read by head_dim/8 lanes with 16-byte loads, the lanes agree on its largest magnitude by row
// swaps on the vector units, and each writes 8 codes; the row's first lane writes its exponent byte.
// read_pages_kernel goes the other way, from pages of any kind to contiguous bf16 rows.
#include <algorithm>
#include <climits>

#include "tgvkv_quant.h"
#include "tgvkv_shape.h"

namespace tgvkv {
namespace {

constexpr int kThreads = 256;

template <int D, int KIND>
__global__ __launch_bounds__(kThreads) void compact_pages_kernel(Shape s, Pages pg, const uint16_t* __restrict__ k,
                                                                 const uint16_t* __restrict__ v,
                                                                 const int32_t* __restrict__ idx,
                                                                 const int32_t* __restrict__ budgets,
                                                                 const int64_t* __restrict__ idx_off, int nsplit,
                                                                 const int32_t* __restrict__ unit_order) {
    constexpr int CPR = D / 8;
    constexpr int RPP = kThreads / CPR;
    int bid = blockIdx.x;
    const int split = bid % nsplit;
    bid /= nsplit;
    const int kvh = bid % s.Hkv;
    const int bl = unit_order != nullptr ? min(max(unit_order[bid / s.Hkv], 0), s.B * s.L - 1) : bid / s.Hkv;
    const int bsz = budgets[bl];
    const long long ioff = idx_off[bl] + (s.head_mode == 0 ? 0 : (long long)kvh * bsz);
    const int per = (bsz + nsplit - 1) / nsplit;
    const int r_beg = min(split * per, bsz), r_end = min(r_beg + per, bsz);
    const int cc = threadIdx.x % CPR, rl = threadIdx.x / CPR;
    const size_t src0 = ((size_t)bl * s.Hkv + kvh) * (size_t)s.N * D + cc * 8;
    // the lanes of a row take the same branch, so the row's maximum is taken among active lanes
    for (int r = r_beg + rl; r < r_end; r += RPP) {
        const int pos = min(max(idx[ioff + r], 0), s.N - 1);
        const u32x4 kr = load16_stream(k + src0 + (size_t)pos * D), vr = load16_stream(v + src0 + (size_t)pos * D);
        const size_t row = pool_row(pg, s.Hkv, kvh, table_page(pg, bl, r), r);
        const uint32_t ke = exp_byte<KIND>(group_max<CPR>(amax8(kr))), ve = exp_byte<KIND>(group_max<CPR>(amax8(vr)));
        *reinterpret_cast<u32x2*>(pg.k + row * D + cc * 8) = encode8<KIND>(kr, ke);
        *reinterpret_cast<u32x2*>(pg.v + row * D + cc * 8) = encode8<KIND>(vr, ve);
        if (cc == 0) {
            pg.k_exp[row] = (uint8_t)ke;
            pg.v_exp[row] = (uint8_t)ve;
        }
    }
}

template <int D, int KIND>
__global__ __launch_bounds__(kThreads) void read_pages_kernel(Shape s, Pages pg, const int32_t* __restrict__ first,
                                                              const int32_t* __restrict__ count,
                                                              const int64_t* __restrict__ seg_off, int nsplit,
                                                              uint16_t* __restrict__ kc, uint16_t* __restrict__ vc) {
    constexpr int CPR = D / 8;
    constexpr int RPP = kThreads / CPR;
    int bid = blockIdx.x;
    const int split = bid % nsplit;
    bid /= nsplit;
    const int kvh = bid % s.Hkv, bl = bid / s.Hkv;
    const int64_t s0 = seg_off[bl], cap = seg_off[bl + 1] - s0;
    const int f = first != nullptr ? max(first[bl], 0) : 0;
    const int rows = (int)min((int64_t)max(count[bl], 0), cap);
    const int per = (rows + nsplit - 1) / nsplit;
    const int r_beg = min(split * per, rows), r_end = min(r_beg + per, rows);
    const int cc = threadIdx.x % CPR, rl = threadIdx.x / CPR;
    const size_t dst0 = ((size_t)s0 * s.Hkv + (size_t)kvh * cap) * D + cc * 8;
    for (int r = r_beg + rl; r < r_end; r += RPP) {
        const size_t row = pool_row(pg, s.Hkv, kvh, table_page(pg, bl, f + r), f + r);
        const size_t at = (row * D + cc * 8) * code_bytes(KIND);
        u32x4 kr, vr;
        if constexpr (KIND == kCacheBf16) {
            kr = load16_stream(pg.k + at);
            vr = load16_stream(pg.v + at);
        } else {
            kr = decode8<KIND>(*reinterpret_cast<const u32x2*>(pg.k + at));
            vr = decode8<KIND>(*reinterpret_cast<const u32x2*>(pg.v + at));
            const float ks = exp_scale(pg.k_exp[row]), vs = exp_scale(pg.v_exp[row]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                kr[i] = scale2bf16(kr[i], ks);
                vr[i] = scale2bf16(vr[i], vs);
            }
        }
        store16(kc + dst0 + (size_t)r * D, kr);
        store16(vc + dst0 + (size_t)r * D, vr);
    }
}

// Workgroups per (sequence, layer, KV head), as compaction's.
int row_splits(const Shape& s, int64_t rows_total) {
    const long long units = (long long)s.B * s.L * s.Hkv;
    if (units <= 0 || rows_total <= 0) return 1;
    const long long avg_rows = rows_total / ((long long)s.B * s.L);
    const long long n = std::min<long long>(2048 / units, avg_rows / 64);
    return (int)std::max<long long>(1, std::min<long long>(n, 16));
}

}  // namespace

hipError_t launch_compact_pages(const Shape& s, const Pages& pg, const uint16_t* k, const uint16_t* v,
                                const int32_t* idx, const int32_t* budgets, const int64_t* idx_off, int64_t rows_total,
                                const int32_t* unit_order, hipStream_t st) {
    if (rows_total <= 0 || s.B * s.L == 0) return hipSuccess;
    const int nsplit = row_splits(s, rows_total);
    const dim3 grid((unsigned)((long long)s.B * s.L * s.Hkv * nsplit));
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, s, pg, k, v, idx, budgets, idx_off, nsplit, unit_order);
    };
    if (pg.kind == kCacheFp8) {
        if (s.D == 128) launch(compact_pages_kernel<128, kCacheFp8>);
        else launch(compact_pages_kernel<64, kCacheFp8>);
    } else {
        if (s.D == 128) launch(compact_pages_kernel<128, kCacheInt8>);
        else launch(compact_pages_kernel<64, kCacheInt8>);
    }
    return hipGetLastError();
}

hipError_t launch_read_pages(const Shape& s, const Pages& pg, const int32_t* first, const int32_t* count,
                             const int64_t* seg_off, uint16_t* kc, uint16_t* vc, hipStream_t st) {
    if (s.B * s.L == 0) return hipSuccess;
    const long long units = (long long)s.B * s.L * s.Hkv;
    const int nsplit = (int)std::max<long long>(1, std::min<long long>(2048 / units, 16));
    const dim3 grid((unsigned)(units * nsplit));
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, s, pg, first, count, seg_off, nsplit, kc, vc);
    };
    if (s.D == 128) {
        if (pg.kind == kCacheBf16) launch(read_pages_kernel<128, kCacheBf16>);
        else if (pg.kind == kCacheFp8) launch(read_pages_kernel<128, kCacheFp8>);
        else launch(read_pages_kernel<128, kCacheInt8>);
    } else {
        if (pg.kind == kCacheBf16) launch(read_pages_kernel<64, kCacheBf16>);
        else if (pg.kind == kCacheFp8) launch(read_pages_kernel<64, kCacheFp8>);
        else launch(read_pages_kernel<64, kCacheInt8>);
    }
    return hipGetLastError();
}

}  // namespace tgvkv
