// The paged cache in 8 bits: the retained rows quantised as they are written, and rows read back.
//
// Both are HBM streams.  compact_pages_kernel is compact_kernel with a different store, and for tables of any width
// (rows behind the table's are not stored): a row of head_dim bf16 is read by head_dim/8 lanes with 16-byte loads, the lanes agree on its largest magnitude by lane swaps
// on the vector units, and each writes 8 codes; the row's first lane writes its exponent byte.
// read_pages_kernel goes the other way, from pages of any kind to contiguous bf16 rows.  Each thread keeps
// kPasses rows' K and V in flight (one row at a time was bound by latency: 298 us to store and 384 us to read
// 1.2 M rows of 128, layers of 120 to 2979 rows), and page ids are looked up in LDS.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "tgvkv_quant.h"
#include "tgvkv_shape.h"

namespace tgvkv {
namespace {

constexpr int kThreads = 256;
constexpr int kPasses = 8;
constexpr int kMaxRowGroups = 16384;

template <int D, int KIND>
__global__ __launch_bounds__(kThreads) void compact_pages_kernel(Shape s, Pages pg, const uint16_t* __restrict__ k,
                                                                 const uint16_t* __restrict__ v,
                                                                 const int32_t* __restrict__ idx,
                                                                 const int32_t* __restrict__ budgets,
                                                                 const int64_t* __restrict__ idx_off, int nsplit,
                                                                 const int32_t* __restrict__ unit_order) {
    extern __shared__ uint32_t lds_pages[];
    constexpr int CPR = D / 8;           // lanes per row
    constexpr int RPP = kThreads / CPR;  // rows per pass
    int bid = blockIdx.x;
    const int split = bid % nsplit;
    bid /= nsplit;
    const int kvh = bid % s.Hkv;
    const int bl = unit_order != nullptr ? min(max(unit_order[bid / s.Hkv], 0), s.B * s.L - 1) : bid / s.Hkv;
    const int bsz = budgets[bl];
    const long long ioff = idx_off[bl] + (s.head_mode == 0 ? 0 : (long long)kvh * bsz);
    const int held = (int)min((long long)bsz, (long long)pg.max_pages << pg.shift);  // rows that the table can name
    const int per = (held + nsplit - 1) / nsplit;
    const int r_beg = min(split * per, held), r_end = min(r_beg + per, held);
    if (r_beg >= r_end) return;  // uniform, before any barrier
    const int cc = threadIdx.x % CPR, rl = threadIdx.x / CPR;
    const size_t src0 = ((size_t)bl * s.Hkv + kvh) * (size_t)s.N * D + cc * 8;
    // positions come from tgvkv_select; clamped so a corrupt index can never read outside the slice.  Rows behind the
    // last repeat it and are not stored.
    int pos[kPasses];
    auto positions = [&](int r0) {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) pos[i] = min(max(idx[ioff + min(r0 + i * RPP + rl, r_end - 1)], 0), s.N - 1);
    };
    positions(r_beg);
    PageRows pages;
    pages.init<kThreads>(s, pg, bl, kvh, r_beg, r_end, lds_pages);
    __syncthreads();
    for (int r0 = r_beg; r0 < r_end; r0 += RPP * kPasses) {
        u32x4 kr[kPasses], vr[kPasses];
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            kr[i] = load16_stream(k + src0 + (size_t)pos[i] * D);
            vr[i] = load16_stream(v + src0 + (size_t)pos[i] * D);
        }
        positions(r0 + RPP * kPasses);
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int r = r0 + i * RPP + rl;
            if constexpr (KIND == kCacheBf16) {
                if (r < r_end) {
                    const size_t at = (pages.row(r) * D + cc * 8) * 2;
                    store16(pg.k + at, kr[i]);
                    store16(pg.v + at, vr[i]);
                }
            } else {
                // every lane takes part in the row's maximum
                const uint32_t ke = exp_byte<KIND>(group_max<CPR>(amax8(kr[i]))), ve = exp_byte<KIND>(group_max<CPR>(amax8(vr[i])));
                if (r < r_end) {
                    const size_t row = pages.row(r);
                    *reinterpret_cast<u32x2*>(pg.k + row * D + cc * 8) = encode8<KIND>(kr[i], ke);
                    *reinterpret_cast<u32x2*>(pg.v + row * D + cc * 8) = encode8<KIND>(vr[i], ve);
                    if (cc == 0) {
                        pg.k_exp[row] = (uint8_t)ke;
                        pg.v_exp[row] = (uint8_t)ve;
                    }
                }
            }
        }
    }
}

template <int D, int KIND, int THREADS>
__global__ __launch_bounds__(THREADS) void read_pages_kernel(Shape s, Pages pg, const int32_t* __restrict__ first,
                                                              const int32_t* __restrict__ count,
                                                              const int64_t* __restrict__ seg_off, int64_t out_rows,
                                                              int nsplit, uint16_t* __restrict__ kc, uint16_t* __restrict__ vc) {
    extern __shared__ uint32_t lds_pages[];
    constexpr int CPR = D / 8;
    constexpr int RPP = THREADS / CPR;
    int bid = blockIdx.x;
    const int split = bid % nsplit;
    bid /= nsplit;
    const int kvh = bid % s.Hkv, bl = bid / s.Hkv;
    const int64_t s0 = seg_off[bl], cap = seg_off[bl + 1] - s0;
    if (s0 < 0 || cap < 0 || s0 + cap > out_rows) return;  // a segment that the output does not hold
    const int f = first != nullptr ? max(first[bl], 0) : 0;
    // rows that the table can name
    const long long most = ((long long)pg.max_pages << pg.shift) - f;
    const int rows = (int)max(min(min((long long)max(count[bl], 0), (long long)cap), most), 0ll);
    const int per = (rows + nsplit - 1) / nsplit;
    const int r_beg = min(split * per, rows), r_end = min(r_beg + per, rows);
    if (r_beg >= r_end) return;  // uniform, before any barrier
    const int cc = threadIdx.x % CPR, rl = threadIdx.x / CPR;
    PageRows pages;
    pages.init<THREADS>(s, pg, bl, kvh, f + r_beg, f + r_end, lds_pages);
    __syncthreads();
    const size_t dst0 = ((size_t)s0 * s.Hkv + (size_t)kvh * cap) * D + cc * 8;
    auto move = [&](auto passes, int r0) {
        constexpr int N = decltype(passes)::value;
        u32x4 kr[N], vr[N];
        uint32_t ke[N], ve[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {  // rows behind the last repeat it and are not stored
            const size_t row = pages.row(f + min(r0 + i * RPP + rl, r_end - 1)), at = (row * D + cc * 8) * code_bytes(KIND);
            if constexpr (KIND == kCacheBf16) {
                kr[i] = load16_stream(pg.k + at);
                vr[i] = load16_stream(pg.v + at);
            } else {
                const u32x2 kc8 = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(pg.k + at));
                const u32x2 vc8 = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(pg.v + at));
                kr[i][0] = kc8[0], kr[i][1] = kc8[1], vr[i][0] = vc8[0], vr[i][1] = vc8[1];
                ke[i] = pg.k_exp[row];
                ve[i] = pg.v_exp[row];
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = r0 + i * RPP + rl;
            if (r >= r_end) continue;
            if constexpr (KIND != kCacheBf16) {
                kr[i] = values8<KIND>(u32x2{kr[i][0], kr[i][1]}, exp_scale(ke[i]));
                vr[i] = values8<KIND>(u32x2{vr[i][0], vr[i][1]}, exp_scale(ve[i]));
            }
            store16(kc + dst0 + (size_t)r * D, kr[i]);
            store16(vc + dst0 + (size_t)r * D, vr[i]);
        }
    };
    int r0 = r_beg;
    for (; r_end - r0 > RPP; r0 += RPP * kPasses) move(std::integral_constant<int, kPasses>(), r0);
    if (r0 < r_end) move(std::integral_constant<int, 1>(), r0);  // a chunk's few rows, or the last ones
}

// Workgroups per (sequence, layer, KV head): about one per 64 rows of the mean segment.  Segments differ in
// length by an order of magnitude, and small shares even that out (1.2 M rows in 4096 units of 120 to 2979: 200 us
// with 4 each, 300 with one), but workgroups without rows are not free: 16384 of them take 40 us.
int row_splits(const Shape& s, int64_t rows_total) {
    const long long units = (long long)s.B * s.L * s.Hkv, mean = rows_total / std::max<long long>((long long)s.B * s.L, 1);
    return (int)std::max<long long>(1, std::min<long long>({kMaxRowGroups / std::max<long long>(units, 1), mean / 64, 16}));
}

}  // namespace

hipError_t launch_compact_pages(const Shape& s, const Pages& pg, const uint16_t* k, const uint16_t* v,
                                const int32_t* idx, const int32_t* budgets, const int64_t* idx_off, int64_t rows_total,
                                const int32_t* unit_order, hipStream_t st) {
    if (rows_total <= 0 || s.B * s.L == 0) return hipSuccess;
    const int nsplit = row_splits(s, rows_total);
    const dim3 grid((unsigned)((long long)s.B * s.L * s.Hkv * nsplit));
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), lds_pages_bytes(pg), st, s, pg, k, v, idx, budgets, idx_off, nsplit, unit_order);
    };
    if (pg.kind == kCacheFp8) {
        if (s.D == 128) launch(compact_pages_kernel<128, kCacheFp8>);
        else launch(compact_pages_kernel<64, kCacheFp8>);
    } else if (pg.kind == kCacheInt8) {
        if (s.D == 128) launch(compact_pages_kernel<128, kCacheInt8>);
        else launch(compact_pages_kernel<64, kCacheInt8>);
    } else {  // tables too narrow for compact_kernel, which takes every row to have a page
        if (s.D == 128) launch(compact_pages_kernel<128, kCacheBf16>);
        else launch(compact_pages_kernel<64, kCacheBf16>);
    }
    return hipGetLastError();
}

hipError_t launch_read_pages(const Shape& s, const Pages& pg, const int32_t* first, const int32_t* count,
                             const int64_t* seg_off, int64_t out_rows, uint16_t* kc, uint16_t* vc, hipStream_t st) {
    if (out_rows <= 0 || s.B * s.L == 0) return hipSuccess;
    const int nsplit = row_splits(s, out_rows);
    const dim3 grid((unsigned)((long long)s.B * s.L * s.Hkv * nsplit));
    auto launch = [&](auto kernel, int threads) {
        hipLaunchKernelGGL(kernel, grid, dim3(threads), lds_pages_bytes(pg), st, s, pg, first, count, seg_off, out_rows,
                           nsplit, kc, vc);
    };
    // segments of a few rows (what a step or a chunk appended) are work for one wave: 4096 of one row take 4.8 us, in four
    // waves each 7.2; 2^24 workgroups of four waves are more threads than a launch numbers
    auto pick = [&](auto d, auto kind) {
        constexpr int D = decltype(d)::value, KIND = decltype(kind)::value;
        if (out_rows <= (int64_t)s.B * s.L * (8 * 64 / D) || grid.x >= 1u << 24) launch(read_pages_kernel<D, KIND, 64>, 64);
        else launch(read_pages_kernel<D, KIND, kThreads>, kThreads);
    };
    auto pick_kind = [&](auto d) {
        if (pg.kind == kCacheBf16) pick(d, std::integral_constant<int, kCacheBf16>());
        else if (pg.kind == kCacheFp8) pick(d, std::integral_constant<int, kCacheFp8>());
        else pick(d, std::integral_constant<int, kCacheInt8>());
    };
    if (s.D == 128) pick_kind(std::integral_constant<int, 128>());
    else pick_kind(std::integral_constant<int, 64>());
    return hipGetLastError();
}

}  // namespace tgvkv
