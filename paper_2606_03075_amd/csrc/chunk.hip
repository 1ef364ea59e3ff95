// Attention of a chunk of new tokens over the paged cache.
//
// A sequence at step s brings c new tokens.  In every layer their keys and values become rows
// f .. f + c - 1 of the segment, f = b_l + s, and token i attends to rows n <= f + i (Eq. (2) over the
// pruned cache of Eq. (3)-(4)): c decode steps in one call.  The c tokens of the G query heads that share
// a KV head are c G query rows against the same keys, row r = i G + g, which is what the matrix cores want:
//   S^T = K Q^T   32 keys x 16 rows per step: lane l holds row l % 16, keys 4 (l / 16) + {0..3} and + 16;
//   online softmax per row: a lane's 8 values, then two row swaps across the lane quarters;
//   O^T += V^T P  with the probabilities where the first product left them: the key order of the second
//                 product's sum is free, so slot j of a lane quarter is the key that the quarter holds; V^T
//                 comes from row-major V rows in LDS by transposing reads.  O's columns are rows of the
//                 softmax, so a new maximum rescales a lane's values by the lane's own factor.
// With 32-bit results the probabilities enter as two bf16 parts (16 significant bits), two products; with
// bf16 results as one, whose 2^-9 is of the size of the result's own rounding.
//
// K and V rows reach LDS as bf16 whatever the pages hold: an 8-bit code times its row's power of two is a
// bf16, so the arithmetic behind the staging is the same for every kind.  LDS rows are padded so that both
// kinds of read are free of bank conflicts: K rows by 16 bytes (16 rows at one column), V rows by 32 (the
// transposing read takes 32 bytes of 8 rows at a time).
//
// Two kernels:
//   few_kernel   up to 32 query rows (drafted tokens, single tokens): a stream of the cache.  Every wave holds all
//                rows and takes every fourth block of 32 keys, staged in LDS of its own, no barrier; the
//                new rows are one more block, quantised and written to the pages on the way.
//   rows_kernel  more: a wave holds 16 NT rows of its own and the workgroup's keys are staged for all.
//
// A value that is not finite in a new token's V would reach earlier tokens through 0 * inf; such elements
// are staged as 0 and added to the rows that see them at the end (rare: one flag is looked at).
#include <algorithm>
#include <atomic>
#include <chrono>
#include <climits>

#include "tgvkv_quant.h"
#include "tgvkv_shape.h"

namespace tgvkv {
namespace {

constexpr int kThreads = 256;
constexpr int kCUs = 256;

// One segment's part in the call: its first new row and its new tokens, 0 where it takes no part (an idle
// or exhausted sequence, or a table row too narrow for the rows).
struct Part {
    int first, count;
};
__device__ __forceinline__ Part part_of(const Shape& s, const Pages& pg, const Chunk& ck, int bl) {
    const int b = bl / s.L;
    const int st = ck.steps[b], c = ck.n_new != nullptr ? ck.n_new[b] : ck.chunk;
    const int bsz = max(ck.budgets[bl], 0);
    const bool ok = st >= 0 && c >= 1 && c <= ck.chunk && (long long)st + c <= ck.reserve &&
                    (long long)bsz + st + c <= ((long long)pg.max_pages << pg.shift);
    return ok ? Part{bsz + st, c} : Part{0, 0};
}

// The new rows into the pages, for rows_kernel on 8-bit pages (its many row tiles then read codes).
template <int D, int KIND>
__global__ __launch_bounds__(kThreads) void append_kernel(Shape s, Pages pg, Chunk ck) {
    constexpr int CPR = D / 8;
    constexpr int RPP = kThreads / CPR;
    const int bl = blockIdx.x;
    const Part part = part_of(s, pg, ck, bl);
    const int cc = threadIdx.x % CPR;
    // rows in the inputs' order: token by token, KV head by KV head
    const int rows = part.count * s.Hkv;
    for (int r = blockIdx.y * RPP + threadIdx.x / CPR; r < rows; r += gridDim.y * RPP) {
        const int i = r / s.Hkv, kvh = r % s.Hkv, n = part.first + i;
        const size_t src = ((size_t)bl * ck.chunk * s.Hkv + r) * D + cc * 8;
        const u32x4 kr = load16(ck.k_new + src), vr = load16(ck.v_new + src);
        const int page = table_page(pg, bl, n);
        const uint32_t ke = exp_byte<KIND>(group_max<CPR>(amax8(kr))), ve = exp_byte<KIND>(group_max<CPR>(amax8(vr)));
        if (page >= 0 && page < pg.n_pages) {  // a row without a page is not written
            const size_t row = pool_row(pg, s.Hkv, kvh, page, n);
            *reinterpret_cast<u32x2*>(pg.k + row * D + cc * 8) = encode8<KIND>(kr, ke);
            *reinterpret_cast<u32x2*>(pg.v + row * D + cc * 8) = encode8<KIND>(vr, ve);
            if (cc == 0) {
                pg.k_exp[row] = (uint8_t)ke;
                pg.v_exp[row] = (uint8_t)ve;
            }
        }
    }
}

template <int D>
constexpr int kKRow = D * 2 + 16;  // LDS bytes of a staged K row
template <int D>
constexpr int kVRow = D * 2 + 32;  // and of a V row

// A lane's 16 bytes of bf16 with what is not finite set to 0; true if there was any.
__device__ __forceinline__ bool drop_non_finite(u32x4& r) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool lo = (r[i] & 0x7F80u) == 0x7F80u, hi = (r[i] & 0x7F800000u) == 0x7F800000u;
        any |= lo | hi;
        r[i] = (lo ? 0u : r[i] & 0xFFFFu) | (hi ? 0u : r[i] & 0xFFFF0000u);
    }
    return any;
}

// 16 NT query rows of one (segment, KV head) in a wave, row 16 nt + l % 16 in lane l.
template <int D, int NT, bool FINE>
struct QueryRows {
    bf16x8 qf[NT][D / 32];  // B operand of S^T: 8 dims of the lane's quarter per step
    f32x4 o[NT][D / 16];    // O^T: dims 16 db + 4 (l / 16) + {0..3}
    float m[NT], l[NT];     // running maximum (base-2 logits) and the lane quarter's share of the sum
    int lim[NT];            // last visible row

    // Rows r0 .. of the c G rows; rows behind the last are zeros and see what the last one sees.
    __device__ __forceinline__ void load(const Shape& s, const Chunk& ck, const Part& part, int bl, int kvh, int r0) {
        const int c = threadIdx.x & 15, qq = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = r0 + nt * 16 + c, rows = part.count * s.G;
            const bool in = r < rows;
            const int i = min(r, rows - 1) / s.G, g = min(r, rows - 1) % s.G;
            const uint16_t* qp = ck.q + (((size_t)bl * ck.chunk + i) * s.H + kvh * s.G + g) * D + qq * 8;
            const u32x4 z = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) qf[nt][ks] = as_bf16x8(in ? load16(qp + ks * 32) : z);
            lim[nt] = part.first + i;
            m[nt] = kNegInf;
            l[nt] = 0.f;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) o[nt][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    __device__ __forceinline__ void settle_rows() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) settle(qf[nt][ks]);
    }

    // One step over the 32 staged rows n0 ..; MASK: only those up to lim count, and below `end`.
    template <bool MASK>
    __device__ __forceinline__ void step(const char* kst, const char* vst, int n0, int end, float scale2) {
        const int c = threadIdx.x & 15, qq = (threadIdx.x & 63) >> 4;
        f32x4 a[2][NT];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) a[b][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) {
            const bf16x8 k0 = as_bf16x8(load16(kst + c * kKRow<D> + ks * 64 + qq * 16));
            const bf16x8 k1 = as_bf16x8(load16(kst + (16 + c) * kKRow<D> + ks * 64 + qq * 16));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                a[0][nt] = mfma16x16x32(k0, qf[nt][ks], a[0][nt]);
                a[1][nt] = mfma16x16x32(k1, qf[nt][ks], a[1][nt]);
            }
        }
        bf16x8 ph[NT], pl[FINE ? NT : 1];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float z[8], mb = kNegInf;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                z[j] = a[j / 4][nt][j % 4];
                if (MASK) {
                    const int n = n0 + 16 * (j / 4) + 4 * qq + j % 4;
                    z[j] = n <= lim[nt] && n < end ? z[j] : kNegInf;
                }
                mb = fmaxf(mb, z[j]);
            }
            mb = max_xor32(max_xor16(mb)) * scale2;
            if (__builtin_amdgcn_ballot_w64(mb > m[nt]) != 0) {  // some row's maximum grew (uniform branch)
                const float mn = fmaxf(m[nt], mb), sc = mn == kNegInf ? 1.f : fast_exp2(m[nt] - mn);
                l[nt] *= sc;
#pragma unroll
                for (int db = 0; db < D / 16; ++db) o[nt][db] *= sc;
                m[nt] = mn;
            }
            const float mu = m[nt] == kNegInf ? 0.f : m[nt];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p = fast_exp2(__builtin_fmaf(z[j], scale2, -mu));
                l[nt] += p;
                ph[nt][j] = (__bf16)p;
                if (FINE) pl[nt][j] = (__bf16)(p - (float)ph[nt][j]);
            }
        }
        const char* vp = vst + (4 * qq + (c >> 2)) * kVRow<D> + (c & 3) * 8;
#pragma unroll
        for (int db = 0; db < D / 16; ++db) {
            const s16x4 v0 = lds_read_tr16(vp + db * 32), v1 = lds_read_tr16(vp + 16 * kVRow<D> + db * 32);
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            const bf16x8 vv = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                o[nt][db] = mfma16x16x32(vv, ph[nt], o[nt][db]);
                if (FINE) o[nt][db] = mfma16x16x32(vv, pl[nt], o[nt][db]);
            }
        }
    }

    // The lane quarters' shares of the sums together.
    __device__ __forceinline__ void close() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) l[nt] = sum_xor32(sum_xor16(l[nt]));
    }

    // Adds the non-finite values of V rows n0 .. n1 - 1 that a row sees: those of the new tokens in bf16, or, with
    // 8-bit pages, rows of the exponent byte 255.
    template <int KIND>
    __device__ __forceinline__ void add_non_finite(const Shape& s, const Pages& pg, const Chunk& ck, const Part& part, int bl,
                                                   int kvh, int n0, int n1) {
        const int qq = (threadIdx.x & 63) >> 4;
        for (int n = n0; n < n1; ++n) {
            const uint16_t* v = ck.v_new + (((size_t)bl * ck.chunk + n - part.first) * s.Hkv + kvh) * D + 4 * qq;
            uint32_t row_max = 0;
            if constexpr (KIND != kCacheBf16) {
                for (int e = 0; e < D; e += 8) row_max = max(row_max, amax8(load16(v - 4 * qq + e)));
            }
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(v + 16 * db);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t x = j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16;
                    if constexpr (KIND != kCacheBf16) x = row_max >= 0x7F80u ? 0x7FC00000u : 0u;
                    const bool odd = (x & 0x7F800000u) == 0x7F800000u;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        if (odd && n <= lim[nt]) o[nt][db][j] += __uint_as_float(x);
                }
            }
        }
    }
};

// 8 values of a new row as later steps will read them, and the row into its page.
template <int D, int KIND>
__device__ __forceinline__ u32x4 append8(const Pages& pg, uint8_t* pool, uint8_t* exps, size_t row, int cc, bool in, u32x4 r) {
    if constexpr (KIND == kCacheBf16) {
        if (in) store16(pool + (row * D + cc * 8) * 2, r);
        return r;
    } else {
        const uint32_t e = exp_byte<KIND>(group_max<D / 8>(amax8(r)));
        const u32x2 codes = encode8<KIND>(r, e);
        if (in) {
            *reinterpret_cast<u32x2*>(pool + row * D + cc * 8) = codes;
            if (cc == 0) exps[row] = (uint8_t)e;
        }
        const float sc = exp_scale(e);
        const u32x2 a = values4<KIND>(codes[0], sc), b = values4<KIND>(codes[1], sc);
        return u32x4{a[0], a[1], b[0], b[1]};
    }
}

// Rows of a segment's pages: the first pool row of every page of rows [n0, n1), in LDS.  A pool's rows are
// numbered in 32 bits (2^32 of the smallest rows, in two pools, are more memory than the GPU has).
struct PageRows {
    const uint32_t* base;
    int p0, shift;
    __device__ __forceinline__ void init(const Shape& s, const Pages& pg, int bl, int kvh, int n0, int n1, uint32_t* lds) {
        shift = pg.shift;
        p0 = n0 >> shift;
        base = lds;
        const int p1 = n1 > n0 ? ((n1 - 1) >> shift) + 1 : p0;
        for (int i = p0 + (int)threadIdx.x; i < p1; i += kThreads)
            lds[i - p0] = (uint32_t)pool_row(pg, s.Hkv, kvh, pg.table[(size_t)bl * pg.max_pages + i], 0);
    }
    __device__ __forceinline__ size_t row(int n) const { return base[(n >> shift) - p0] + (uint32_t)(n & ((1 << shift) - 1)); }
};

// One lane's share of `ROWS` rows' K or V on its way from the pages to LDS.  LANES lanes work together, each on 16
// bytes of a row at a time: 8 bf16, or 16 codes.
template <int D, int KIND, int ROWS, int LANES>
struct Staged {
    static constexpr int CH = D * code_bytes(KIND) / 16;  // 16-byte pieces per row
    static constexpr int N = ROWS * CH / LANES;
    u32x4 x[N];
    uint32_t e[KIND == kCacheBf16 ? 1 : N];

    __device__ __forceinline__ static int row_of(int it, int lane) { return (it * LANES + lane) / CH; }

    __device__ __forceinline__ void from_page(int it, int lane, const uint8_t* pool, const uint8_t* exps, size_t row) {
        x[it] = load16_stream(pool + (row * CH + (it * LANES + lane) % CH) * 16);
        if constexpr (KIND != kCacheBf16) e[it] = exps[row];
    }
    // To LDS rows of `stride` bytes, as bf16.
    __device__ __forceinline__ void store(int it, int lane, char* lds, int stride) {
        char* p = lds + row_of(it, lane) * stride + (it * LANES + lane) % CH * (KIND == kCacheBf16 ? 16 : 32);
        if constexpr (KIND == kCacheBf16) {
            store16(p, x[it]);
        } else {
            const float sc = exp_scale(e[it]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x2 a = values4<KIND>(x[it][2 * h], sc), b = values4<KIND>(x[it][2 * h + 1], sc);
                store16(p + 16 * h, u32x4{a[0], a[1], b[0], b[1]});
            }
        }
    }
};

// Results of a row: f32 or bf16.
template <bool FINE>
__device__ __forceinline__ void store_out(const Chunk& ck, size_t at, float v) {
    if constexpr (FINE) reinterpret_cast<float*>(ck.out)[at] = v;
    else reinterpret_cast<__bf16*>(ck.out)[at] = (__bf16)v;
}

// Splits of a unit's keys over workgroups, joined in the same launch: each workgroup of a unit leaves its
// partial and then a mark, the call's number, and the one that finds every mark joins the partials in split order and
// clears the marks.  No workgroup waits.  Partials and marks are GPU-scope atomic accesses, which
// go through to memory, so that a finished store is visible on every XCD.  The workspace's first contents
// do not matter: a mark counts only if it is this call's number, 64 bits that differ between calls; a
// replayed graph brings its number again, but every call leaves its marks cleared.
struct KeySplits {
    unsigned long long* marks;  // [units][most]
    float* part;                // [units][most][rows][D + 2]
    unsigned long long call;
    int most;
};
constexpr int kMaxKeySplits = 32;
constexpr int kSplitRows = 256;  // a split has at least so many rows

__device__ __forceinline__ void store_shared(float* p, float v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float load_shared(const float* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int D, int KIND, int NT, bool FINE>
__global__ __launch_bounds__(kThreads) void few_kernel(Shape s, Pages pg, Chunk ck, KeySplits sp) {
    constexpr int KB = 32;               // keys per block
    constexpr int ROWS = 16 * NT;
    constexpr int CPR = D / 8;           // 16-byte pieces of a bf16 row
    constexpr int STAGE = KB * (kKRow<D> + kVRow<D>);
    constexpr int MERGE = 4 * ROWS * (D + 2) * (int)sizeof(float);
    __shared__ __align__(16) char smem[4 * STAGE > MERGE ? 4 * STAGE : MERGE];
    extern __shared__ uint32_t lds_pages[];
    __shared__ int found;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int split = blockIdx.x % sp.most, slot = blockIdx.x / sp.most;
    const int kvh = slot % s.Hkv;
    const int bl = ck.unit_order != nullptr ? min(max(ck.unit_order[slot / s.Hkv], 0), s.B * s.L - 1) : slot / s.Hkv;
    const Part part = part_of(s, pg, ck, bl);
    if (part.count == 0) return;
    const int f = part.first, c = part.count, rows = c * s.G;
    const int nsplit = min(max((f + kSplitRows - 1) / kSplitRows, 1), sp.most);
    if (split >= nsplit) return;
    const int per = ((f + KB - 1) / KB + nsplit - 1) / nsplit * KB;
    const int t0 = min(split * per, f), t1 = min(t0 + per, f);
    PageRows pages;
    pages.init(s, pg, bl, kvh, t0, t1, lds_pages);
    __syncthreads();

    char* kst = smem + wave * STAGE;
    char* vst = kst + KB * kKRow<D>;
    Staged<D, KIND, KB, 64> ka, va;
    // rows behind the last repeat it (they count nothing), so every load is issued
    auto issue = [&](int n0) {
#pragma unroll
        for (int it = 0; it < ka.N; ++it) {
            const size_t row = pages.row(min(n0 + ka.row_of(it, lane), t1 - 1));
            ka.from_page(it, lane, pg.k, pg.k_exp, row);
            va.from_page(it, lane, pg.v, pg.v_exp, row);
        }
    };
    int n0 = t0 + KB * wave;
    if (n0 < t1) issue(n0);
    QueryRows<D, NT, FINE> qr;
    qr.load(s, ck, part, bl, kvh, 0);
    qr.settle_rows();

    // the new rows, a block of their own: to the pages, and attended as the pages hold them
    if (split == nsplit - 1 && wave == 3) {
        const int cc = lane % CPR;
        bool odd = false;
#pragma unroll 4
        for (int it = 0; it < KB * CPR / 64; ++it) {
            const int i = it * (64 / CPR) + lane / CPR, n = f + min(i, c - 1);
            const size_t src = (((size_t)bl * ck.chunk + min(i, c - 1)) * s.Hkv + kvh) * D + cc * 8;
            u32x4 kr = load16(ck.k_new + src), vr = load16(ck.v_new + src);
            const int page = table_page(pg, bl, n);
            const bool in = i < c && page >= 0 && page < pg.n_pages;  // a row without a page is not written
            const size_t row = pool_row(pg, s.Hkv, kvh, page, n);
            kr = append8<D, KIND>(pg, pg.k, pg.k_exp, row, cc, in, kr);
            vr = append8<D, KIND>(pg, pg.v, pg.v_exp, row, cc, in, vr);
            odd |= drop_non_finite(vr);
            store16(kst + i * kKRow<D> + cc * 16, kr);
            store16(vst + i * kVRow<D> + cc * 16, vr);
        }
        asm volatile("" ::: "memory");
        qr.template step<true>(kst, vst, f, f + c, s.scale2);
        if (__builtin_amdgcn_ballot_w64(odd) != 0) qr.template add_non_finite<KIND>(s, pg, ck, part, bl, kvh, f, f + c);
        asm volatile("" ::: "memory");
    }
    for (; n0 < t1; n0 += 4 * KB) {
        asm volatile("" ::: "memory");  // this wave's reads of the previous block were issued before
#pragma unroll
        for (int it = 0; it < ka.N; ++it) {
            ka.store(it, lane, kst, kKRow<D>);
            va.store(it, lane, vst, kVRow<D>);
        }
        if (n0 + 4 * KB < t1) issue(n0 + 4 * KB);
        asm volatile("" ::: "memory");
        if (n0 + KB <= t1) qr.template step<false>(kst, vst, n0, t1, s.scale2);
        else qr.template step<true>(kst, vst, n0, t1, s.scale2);
    }
    qr.close();

    // the waves' partials through LDS
    __syncthreads();  // every wave is done with its stage
    const int c16 = lane & 15, qq = lane >> 4;
    float* wm = reinterpret_cast<float*>(smem);  // [4][ROWS]
    float* wl = wm + 4 * ROWS;
    float* wacc = wl + 4 * ROWS;  // [4][ROWS][D]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = nt * 16 + c16;
        if (qq == 0) {
            wm[wave * ROWS + r] = qr.m[nt];
            wl[wave * ROWS + r] = qr.l[nt];
        }
#pragma unroll
        for (int db = 0; db < D / 16; ++db)
            *reinterpret_cast<f32x4*>(wacc + (size_t)(wave * ROWS + r) * D + 16 * db + 4 * qq) = qr.o[nt][db];
    }
    __syncthreads();
    float* mine = sp.part + ((size_t)slot * sp.most + split) * ROWS * (D + 2);
    for (int x = tid; x < rows * D; x += kThreads) {
        const int r = x / D, e = x % D;
        float M = kNegInf;
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, wm[w * ROWS + r]);
        const float mu = M == kNegInf ? 0.f : M;
        float num = 0.f, den = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float sc = fast_exp2(wm[w * ROWS + r] - mu);
            num += sc * wacc[(size_t)(w * ROWS + r) * D + e];
            den += sc * wl[w * ROWS + r];
        }
        if (nsplit == 1) {
            store_out<FINE>(ck, (((size_t)bl * ck.chunk + r / s.G) * s.H + kvh * s.G + r % s.G) * D + e, num / den);
        } else {
            store_shared(mine + r * (D + 2) + 2 + e, num);
            if (e == 0) {
                store_shared(mine + r * (D + 2), M);
                store_shared(mine + r * (D + 2) + 1, den);
            }
        }
    }
    if (nsplit == 1) return;

    wait_vmem_ordered();  // this thread's part of the partial has reached memory ...
    __syncthreads();      // ... and every thread's has, before the mark
    unsigned long long* marks = sp.marks + (size_t)slot * sp.most;
    if (tid < 64) {
        if (tid == 0) __hip_atomic_store(marks + split, sp.call, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        wait_vmem_ordered();  // the mark has reached memory before the others' are read
        const bool here = tid >= nsplit ||
                          __hip_atomic_load(marks + tid, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == sp.call;
        const bool all = __ballot(!here) == 0;
        if (tid == 0) found = all;
    }
    __syncthreads();
    if (!found) return;
    const float* base = sp.part + (size_t)slot * sp.most * ROWS * (D + 2);
    for (int x = tid; x < rows * nsplit; x += kThreads) {  // maxima and sums to LDS
        const int r = x / nsplit, i = x % nsplit;
        const float* p = base + ((size_t)i * ROWS + r) * (D + 2);
        wm[r * kMaxKeySplits + i] = load_shared(p);
        wm[(ROWS + r) * kMaxKeySplits + i] = load_shared(p + 1);
    }
    __syncthreads();
    for (int x = tid; x < rows * D; x += kThreads) {
        const int r = x / D, e = x % D;
        float M = kNegInf;
        for (int i = 0; i < nsplit; ++i) M = fmaxf(M, wm[r * kMaxKeySplits + i]);
        const float mu = M == kNegInf ? 0.f : M;
        float num = 0.f, den = 0.f;
        for (int i0 = 0; i0 < nsplit; i0 += 8) {
            float a[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                a[u] = load_shared(base + ((size_t)min(i0 + u, nsplit - 1) * ROWS + r) * (D + 2) + 2 + e);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (i0 + u < nsplit) {
                    const float sc = fast_exp2(wm[r * kMaxKeySplits + i0 + u] - mu);
                    num += sc * a[u];
                    den += sc * wm[(ROWS + r) * kMaxKeySplits + i0 + u];
                }
            }
        }
        store_out<FINE>(ck, (((size_t)bl * ck.chunk + r / s.G) * s.H + kvh * s.G + r % s.G) * D + e, num / den);
    }
    if (tid < nsplit) __hip_atomic_store(marks + tid, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A workgroup per (segment, KV head, 64 NT query rows).
template <int D, int KIND, int NT, bool FINE>
__global__ __launch_bounds__(kThreads) void rows_kernel(Shape s, Pages pg, Chunk ck, int tiles) {
    constexpr int KT = 64;  // keys per tile
    __shared__ __align__(16) char kst[KT * kKRow<D>];
    __shared__ __align__(16) char vst[KT * kVRow<D>];
    __shared__ int odd_seen;
    extern __shared__ uint32_t lds_pages[];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // the row tiles of a unit follow one another on one XCD (workgroups go to the 8 XCDs in turn), whose L2 then
    // holds the unit's keys
    const int units = s.B * s.L * s.Hkv;
    const int x = blockIdx.x / 8, slot = x / tiles * 8 + blockIdx.x % 8, tile = x % tiles;
    if (slot >= units) return;
    const int kvh = slot % s.Hkv;
    const int bl = ck.unit_order != nullptr ? min(max(ck.unit_order[slot / s.Hkv], 0), s.B * s.L - 1) : slot / s.Hkv;
    const Part part = part_of(s, pg, ck, bl);
    const int rows = part.count * s.G, r_beg = tile * 64 * NT;
    if (r_beg >= rows) return;
    const int f = part.first, r_end = min(r_beg + 64 * NT, rows);
    const int end = f + (r_end - 1) / s.G + 1;  // rows that the workgroup's last token sees
    const int paged = KIND == kCacheBf16 ? f : end;  // rows read from the pages; the rest from the inputs
    PageRows pages;
    pages.init(s, pg, bl, kvh, 0, paged, lds_pages);
    if (tid == 0) odd_seen = 0;
    __syncthreads();

    Staged<D, KIND, KT, kThreads> ka, va;
    auto issue = [&](int n0) {
#pragma unroll
        for (int it = 0; it < ka.N; ++it) {
            const int n = min(n0 + ka.row_of(it, tid), end - 1);
            if (KIND == kCacheBf16 && n >= f) {
                const size_t row = ((size_t)bl * ck.chunk + n - f) * s.Hkv + kvh;
                ka.from_page(it, tid, reinterpret_cast<const uint8_t*>(ck.k_new), nullptr, row);
                va.from_page(it, tid, reinterpret_cast<const uint8_t*>(ck.v_new), nullptr, row);
            } else {
                const size_t row = pages.row(n);
                ka.from_page(it, tid, pg.k, pg.k_exp, row);
                va.from_page(it, tid, pg.v, pg.v_exp, row);
            }
        }
    };
    issue(0);
    QueryRows<D, NT, FINE> qr;
    const int w0 = r_beg + wave * 16 * NT;  // the wave's first row
    qr.load(s, ck, part, bl, kvh, w0);
    qr.settle_rows();
    // the wave's rows see at least the rows below `all`, and none from `none` on
    const int all = f + min(w0, rows - 1) / s.G + 1, none = f + min(w0 + 16 * NT - 1, rows - 1) / s.G + 1;
    const bool live = w0 < rows;

    for (int n0 = 0; n0 < end; n0 += KT) {
        __syncthreads();  // the tile's rows have been read
        const bool fresh = n0 + KT > f;
        if (KIND == kCacheBf16 && fresh) {
            bool odd = false;
#pragma unroll
            for (int it = 0; it < va.N; ++it) {
                if (n0 + va.row_of(it, tid) >= f) odd |= drop_non_finite(va.x[it]);
            }
            if (odd) odd_seen = 1;
        }
        if constexpr (KIND != kCacheBf16) {
            bool odd = false;
#pragma unroll
            for (int it = 0; it < va.N; ++it) {
                if (n0 + va.row_of(it, tid) >= f && va.e[it] == 255u) {
                    va.e[it] = 0;
                    odd = true;
                }
            }
            if (odd) odd_seen = 1;
        }
#pragma unroll
        for (int it = 0; it < ka.N; ++it) {
            ka.store(it, tid, kst, kKRow<D>);
            va.store(it, tid, vst, kVRow<D>);
        }
        if (n0 + KT < end) issue(n0 + KT);
        __syncthreads();
        if (live) {
#pragma unroll
            for (int b = 0; b < KT; b += 32) {
                if (n0 + b >= none) continue;
                if (n0 + b + 32 <= all) qr.template step<false>(kst + b * kKRow<D>, vst + b * kVRow<D>, n0 + b, end, s.scale2);
                else qr.template step<true>(kst + b * kKRow<D>, vst + b * kVRow<D>, n0 + b, end, s.scale2);
            }
        }
    }
    qr.close();
    __syncthreads();
    if (odd_seen) qr.template add_non_finite<KIND>(s, pg, ck, part, bl, kvh, f, end);

    const int c16 = lane & 15, qq = lane >> 4;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = w0 + nt * 16 + c16;
        if (r >= rows) continue;
        const float inv = 1.f / qr.l[nt];
        const size_t at = (((size_t)bl * ck.chunk + r / s.G) * s.H + kvh * s.G + r % s.G) * D + 4 * qq;
#pragma unroll
        for (int db = 0; db < D / 16; ++db) {
            const f32x4 v = qr.o[nt][db] * inv;
            if constexpr (FINE) {
                *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(ck.out) + at + 16 * db) = v;
            } else {
                const bf16x4 w = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
                *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(ck.out) + at + 16 * db) = w;
            }
        }
    }
    // the new rows into the pages: those of the tokens whose first query row is here
    if constexpr (KIND == kCacheBf16) {
        constexpr int CPR = D / 8;
        const int i_end = (r_end - 1) / s.G + 1;
        for (int i = (r_beg + s.G - 1) / s.G + tid / CPR; i < i_end; i += kThreads / CPR) {
            const int page = table_page(pg, bl, f + i);
            if (page < 0 || page >= pg.n_pages) continue;
            const size_t row = pool_row(pg, s.Hkv, kvh, page, f + i), src = ((size_t)bl * ck.chunk + i) * s.Hkv + kvh;
            const int e = tid % CPR * 8;
            store16(pg.k + (row * D + e) * 2, load16(ck.k_new + src * D + e));
            store16(pg.v + (row * D + e) * 2, load16(ck.v_new + src * D + e));
        }
    }
}

constexpr int kFewRows = 32;  // query rows of a unit up to which few_kernel takes them

int few_tiles(const Shape& s, int32_t chunk) { return (int)(((long long)chunk * s.G + 15) / 16); }

// Splits that few_kernel may give a unit's keys.
int key_splits(const Shape& s, int32_t chunk) {
    const long long units = (long long)s.B * s.L * s.Hkv;
    if (units <= 0 || (long long)chunk * s.G > kFewRows) return 1;
    return (int)std::max<long long>(1, std::min<long long>(2 * kCUs / units, kMaxKeySplits));
}

size_t partial_floats(const Shape& s, int32_t chunk, int most) {
    return most > 1 ? (size_t)s.B * s.L * s.Hkv * most * 16 * few_tiles(s, chunk) * (s.D + 2) : 0;
}

template <int D, int KIND, bool FINE>
hipError_t launch_chunk_d(const Shape& s, const Pages& pg, const Chunk& ck, hipStream_t st) {
    const long long units = (long long)s.B * s.L * s.Hkv, rows = (long long)ck.chunk * s.G;
    const size_t lds = sizeof(uint32_t) * (size_t)pg.max_pages;
    if (rows <= kFewRows) {
        KeySplits sp{nullptr, nullptr, 0, key_splits(s, ck.chunk)};
        if (sp.most > 1) {
            static std::atomic<unsigned long long> next{
                (unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() * 0x9E3779B97F4A7C15ull};
            do sp.call = next.fetch_add(1, std::memory_order_relaxed); while (sp.call == 0);
            sp.part = ck.ws;
            sp.marks = reinterpret_cast<unsigned long long*>(ck.ws + partial_floats(s, ck.chunk, sp.most));
        }
        const dim3 grid((unsigned)(units * sp.most));
        if (few_tiles(s, ck.chunk) == 1)
            hipLaunchKernelGGL((few_kernel<D, KIND, 1, FINE>), grid, dim3(kThreads), lds, st, s, pg, ck, sp);
        else
            hipLaunchKernelGGL((few_kernel<D, KIND, 2, FINE>), grid, dim3(kThreads), lds, st, s, pg, ck, sp);
        return hipGetLastError();
    }
    if constexpr (KIND != kCacheBf16) {
        constexpr int RPP = kThreads / (D / 8);
        const int parts = (int)std::min<long long>(((long long)ck.chunk * s.Hkv + RPP - 1) / RPP, 256);
        hipLaunchKernelGGL((append_kernel<D, KIND>), dim3(s.B * s.L, parts), dim3(kThreads), 0, st, s, pg, ck);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int nt = rows <= 64 ? 1 : 2;
    const int tiles = (int)((rows + 64 * nt - 1) / (64 * nt));
    const dim3 grid((unsigned)((units + 7) / 8 * 8 * tiles));
    if (nt == 1) hipLaunchKernelGGL((rows_kernel<D, KIND, 1, FINE>), grid, dim3(kThreads), lds, st, s, pg, ck, tiles);
    else hipLaunchKernelGGL((rows_kernel<D, KIND, 2, FINE>), grid, dim3(kThreads), lds, st, s, pg, ck, tiles);
    return hipGetLastError();
}

template <int D, int KIND>
hipError_t launch_chunk_k(const Shape& s, const Pages& pg, const Chunk& ck, hipStream_t st) {
    return ck.out_bf16 ? launch_chunk_d<D, KIND, false>(s, pg, ck, st) : launch_chunk_d<D, KIND, true>(s, pg, ck, st);
}

}  // namespace

size_t chunk_workspace(const Shape& s, int32_t chunk) {
    const int most = key_splits(s, chunk);
    if (most <= 1) return 0;
    return sizeof(float) * partial_floats(s, chunk, most) + sizeof(unsigned long long) * (size_t)s.B * s.L * s.Hkv * most;
}

hipError_t launch_chunk(const Shape& s, const Pages& pg, const Chunk& ck, hipStream_t st) {
    if ((long long)s.B * s.L == 0) return hipSuccess;
    if (s.D == 128) {
        if (pg.kind == kCacheBf16) return launch_chunk_k<128, kCacheBf16>(s, pg, ck, st);
        if (pg.kind == kCacheFp8) return launch_chunk_k<128, kCacheFp8>(s, pg, ck, st);
        return launch_chunk_k<128, kCacheInt8>(s, pg, ck, st);
    }
    if (pg.kind == kCacheBf16) return launch_chunk_k<64, kCacheBf16>(s, pg, ck, st);
    if (pg.kind == kCacheFp8) return launch_chunk_k<64, kCacheFp8>(s, pg, ck, st);
    return launch_chunk_k<64, kCacheInt8>(s, pg, ck, st);
}

}  // namespace tgvkv
