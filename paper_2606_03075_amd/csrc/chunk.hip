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
// With 32-bit results the probabilities enter as three bf16 parts, all of their 24 bits (errors of 2e-7 against 64 bits;
// two parts left 2e-6, and three take 0 to 2 % longer where the cache is read, 8 % where products bound the
// call); with bf16 results as one, off by 2^-8 at most like the result itself (2.3e-3 against 64 bits, where a result in
// 32 bits rounded once has 1.7e-3, as two parts have: 2.66 ms for 2.10 with 1000 tokens of the video shape, 169 us for 141
// with 48 on e4m3 pages.  A caller who wants the one rounding takes 32-bit results and rounds them).
//
// An 8-bit code times its row's power of two is a bf16, so the products take bf16 whatever the pages hold.
//
// Two kernels (measured on MI355X):
//   few_kernel   up to 32 query rows (drafted tokens, single tokens): a stream of the cache.  Every wave holds all
//                rows and takes every fourth block of 32 keys, staged in LDS of its own, no barrier; codes stay codes
//                in LDS (half of it: three workgroups per CU instead of two).  The new rows are one more block,
//                quantised and written to the pages on the way.  4096 units of 215 rows of e4m3, one query row each:
//                57 us, 4.1 TB/s; the loads alone take 43.  Bound by instruction issue (78 % busy) and the units' set-up.
//   rows_kernel  more: a wave holds 16 NT rows of its own, and 64 keys at a time are staged as bf16 for the workgroup.
//                1000 tokens of 4 sequences, 28 layers, 28/4 heads of 128, bf16 results: 2.10 ms, 750 TFLOP/s, in a steady
//                run (in a short one from a cold start 2.1 to 2.25).  Bound by what two waves per SIMD overlap of LDS
//                waits, exponentials and products.
//
// A value that is not finite in a new token's V would reach earlier tokens through 0 * inf; such elements
// are staged as 0 and added to the rows that see them at the end (rare: one flag is looked at), after the last
// rescaling: a factor or a probability too small for 32 bits times an infinity is a NaN, where the sum is infinite.
// Those of retained rows, which all of the chunk's rows see, are looked for only where a sum came out not finite,
// and take its place: an infinity counts as one whatever its probability.
#include <algorithm>
#include <atomic>
#include <chrono>
#include <climits>

#include "tgvkv_quant.h"
#include "tgvkv_shape.h"

namespace tgvkv {
namespace {

constexpr int kThreads = 256;

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

// Token and head of query row r = i G + g: r / G by a multiplication (exact below 2^28, and a segment's rows end at 2^24).
__device__ __forceinline__ int token_of(const Shape& s, const Chunk& ck, int r) {
    return s.G == 1 ? r : (int)__umulhi((unsigned)r, ck.inv_g);
}
// First element of query row r in q and out.
__device__ __forceinline__ size_t query_at(const Shape& s, const Chunk& ck, int bl, int kvh, int r, int D) {
    const int i = token_of(s, ck, r);
    return (((size_t)bl * ck.chunk + i) * s.H + kvh * s.G + (r - i * s.G)) * D;
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

// LDS rows of a block of keys.  bf16: K rows padded by 16 bytes (a read takes one column of 16 rows), V rows by 32
// (a transposing read takes 32 bytes of 8 rows).  Codes: both by 16, and the upper 16 V rows 16 further.
template <int D, bool CODES>
struct Block {
    static constexpr int K = CODES ? D + 16 : D * 2 + 16;
    static constexpr int V = CODES ? D + 16 : D * 2 + 32;
    __device__ static int k_at(int row) { return row * K; }
    __device__ static int v_at(int row) { return row * V + (CODES && row >= 16 ? 16 : 0); }
    static constexpr int kBytes = 32 * K, vBytes = 32 * V + (CODES ? 16 : 0);  // of 32 rows
};

// Whether a lane's 16 bytes of bf16 hold a value that is not finite, and the bytes with such values set to 0.
__device__ __forceinline__ bool non_finite(const u32x4& r) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 e = {0, 0};  // the larger exponent fields, half by half
#pragma unroll
    for (int i = 0; i < 4; ++i) e = __builtin_elementwise_max(e, __builtin_bit_cast(u16x2, r[i] & 0x7F807F80u));
    return e[0] == 0x7F80u || e[1] == 0x7F80u;
}
__device__ __forceinline__ void drop_non_finite(u32x4& r) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        r[i] = ((r[i] & 0x7F80u) == 0x7F80u ? 0u : r[i] & 0xFFFFu) | ((r[i] & 0x7F800000u) == 0x7F800000u ? 0u : r[i] & 0xFFFF0000u);
}

// A weighted sum taken to another reference: an infinity stays one, also where the factor has no 32 bits left.
__device__ __forceinline__ float rescaled(float sum, float factor) { return __builtin_isfinite(sum) ? sum * factor : sum; }

// For sched_barrier: vector and scalar arithmetic may cross, matrix and LDS instructions stay in order.
constexpr int kAluMayCross = 0x2 | 0x4;

// 16 NT query rows of one (segment, KV head) in a wave, row 16 nt + l % 16 in lane l.  Keys come as bf16 rows in LDS
// (CODED = kCacheBf16) or as codes of that kind with their rows' powers of two beside them.  PARTS: bf16 parts of
// a probability in the product with V.
template <int D, int NT, int PARTS, int CODED>
struct QueryRows {
    static constexpr bool CODES = CODED != kCacheBf16;
    using B = Block<D, CODES>;
    bf16x8 qf[NT][D / 32];  // B operand of S^T: 8 dims of the lane's quarter per step
    f32x4 o[NT][D / 16];    // O^T: dims 16 db + 4 (l / 16) + {0..3}
    float m[NT], l[NT];     // reference of the exponents (base-2 logits, see raise) and the lane quarter's share of the sum
    int lim[NT];            // last visible row

    // First of the 8 dims of step ks in lane quarter qq.  A read of 16 codes feeds two steps.
    __device__ static int dim_of(int ks, int qq) { return CODES ? 64 * (ks / 2) + 16 * qq + 8 * (ks % 2) : 32 * ks + 8 * qq; }

    // Rows r0 .. of the c G rows; rows behind the last are zeros and see what the last one sees.
    __device__ __forceinline__ void load(const Shape& s, const Chunk& ck, const Part& part, int bl, int kvh, int r0) {
        const int c = threadIdx.x & 15, qq = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = r0 + nt * 16 + c, rows = part.count * s.G;
            const bool in = r < rows;
            const uint16_t* qp = ck.q + query_at(s, ck, bl, kvh, min(r, rows - 1), D);
            const u32x4 z = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) qf[nt][ks] = as_bf16x8(in ? load16(qp + dim_of(ks, qq)) : z);
            lim[nt] = part.first + token_of(s, ck, min(r, rows - 1));
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

    // Logits (unscaled) of 16 NB staged K rows: a[b][nt][j] is row 16 b + 4 (l / 16) + j's.
    template <int NB>
    __device__ __forceinline__ void logits(const char* kst, f32x4 (&a)[NB][NT]) const {
        const int c = threadIdx.x & 15, qq = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) a[b][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
        const char* kp = kst + B::k_at(c) + qq * 16;
        if constexpr (CODES) {
#pragma unroll
            for (int k2 = 0; k2 < D / 64; ++k2)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const u32x4 w = load16(kp + B::k_at(16 * b) + k2 * 64);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const bf16x8 kf = as_bf16x8(decode8<CODED>(u32x2{w[2 * h], w[2 * h + 1]}));
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) a[b][nt] = mfma16x16x32(kf, qf[nt][2 * k2 + h], a[b][nt]);
                    }
                }
        } else {
            // the next step's fragments are read before this step's products, and the compiler keeps it so
            u32x4 kf[2][NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) kf[0][b] = load16(kp + B::k_at(16 * b));
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) {
                if (ks + 1 < D / 32) {
#pragma unroll
                    for (int b = 0; b < NB; ++b) kf[(ks + 1) & 1][b] = load16(kp + B::k_at(16 * b) + (ks + 1) * 64);
                }
                __builtin_amdgcn_sched_barrier(kAluMayCross);
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) a[b][nt] = mfma16x16x32(as_bf16x8(kf[ks & 1][b]), qf[nt][ks], a[b][nt]);
                __builtin_amdgcn_sched_barrier(kAluMayCross);
            }
        }
    }

    // MASK: rows n0 + .. above lim, or from `end` on, get -inf.  Then the rows' references: a row's reference is kSlack above
    // the largest logit that moved it, so the probabilities stay at most 1, most steps move nothing, and what they lie
    // below 1 costs no precision in floating point.
    template <bool MASK, int NB>
    __device__ __forceinline__ void raise(f32x4 (&a)[NB][NT], int n0, int end, float scale2) {
        const int qq = (threadIdx.x & 63) >> 4;
        constexpr float kSlack = 8.f;
        float mb[NT];
        bool grew = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mb[nt] = kNegInf;
            const int last = min(lim[nt], end - 1) - n0 - 4 * qq;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (MASK) a[b][nt][j] = 16 * b + j <= last ? a[b][nt][j] : kNegInf;
                    mb[nt] = fmaxf(mb[nt], a[b][nt][j]);
                }
            mb[nt] = max_xor32(max_xor16(mb[nt])) * scale2;
            grew |= mb[nt] > m[nt];
        }
        if (__builtin_amdgcn_ballot_w64(grew) != 0) {  // uniform branch
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float mn = mb[nt] > m[nt] ? mb[nt] + kSlack : m[nt], sc = mn == kNegInf ? 1.f : fast_exp2(m[nt] - mn);
                l[nt] *= sc;
#pragma unroll
                for (int db = 0; db < D / 16; ++db) o[nt][db] *= sc;
                m[nt] = mn;
            }
        }
    }

    // The probabilities of 32 rows (a[0], a[1]) and their product with the staged V rows.  vsc: with codes, the rows' powers of two.
    __device__ __forceinline__ void weigh(const f32x4* a0, const f32x4* a1, const char* vst, const f32x4* vsc, float scale2) {
        const int c = threadIdx.x & 15, qq = (threadIdx.x & 63) >> 4;
        bf16x8 pp[PARTS][NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float mu = m[nt] == kNegInf ? 0.f : m[nt];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float p = fast_exp2(__builtin_fmaf(j < 4 ? a0[nt][j % 4] : a1[nt][j % 4], scale2, -mu));
                l[nt] += p;
                if constexpr (CODES) p *= vsc[j / 4][j % 4];
                pp[0][nt][j] = (__bf16)p;
#pragma unroll
                for (int x = 1; x < PARTS; ++x) {
                    p -= (float)pp[x - 1][nt][j];
                    pp[x][nt][j] = (__bf16)p;
                }
            }
        }
        // keys of a lane's slots: 4 qq + {0..3}, 16 + 4 qq + {0..3}
        const char* vp = CODES ? vst + B::v_at((c >> 1) < 4 ? 4 * qq + (c >> 1) : 12 + 4 * qq + (c >> 1)) + (c & 1) * 8
                               : vst + B::v_at(4 * qq + (c >> 2)) + (c & 3) * 8;
        if constexpr (CODES) {
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
                const bf16x8 vv = as_bf16x8(decode8<CODED>(__builtin_bit_cast(u32x2, lds_read_tr8(vp + db * 16))));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int x = 0; x < PARTS; ++x) o[nt][db] = mfma16x16x32(vv, pp[x][nt], o[nt][db]);
            }
        } else {
            // fragments of two column blocks at a time, read two pairs ahead
            constexpr int N2 = D / 32;
            s16x4 vf[3][2][2];
            auto read = [&](int g) {
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    vf[g % 3][d][0] = lds_read_tr16(vp + (2 * g + d) * 32);
                    vf[g % 3][d][1] = lds_read_tr16(vp + 16 * B::V + (2 * g + d) * 32);
                }
            };
            read(0);
            read(1);
#pragma unroll
            for (int g = 0; g < N2; ++g) {
                if (g + 2 < N2) read(g + 2);
                __builtin_amdgcn_sched_barrier(kAluMayCross);
#pragma unroll
                for (int x = 0; x < PARTS; ++x)
#pragma unroll
                    for (int d = 0; d < 2; ++d) {
                        typedef short s16x8 __attribute__((ext_vector_type(8)));
                        const bf16x8 vv = __builtin_bit_cast(
                            bf16x8, (s16x8)__builtin_shufflevector(vf[g % 3][d][0], vf[g % 3][d][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) o[nt][2 * g + d] = mfma16x16x32(vv, pp[x][nt], o[nt][2 * g + d]);
                    }
                __builtin_amdgcn_sched_barrier(kAluMayCross);
            }
        }
    }

    // One step over the 32 staged rows n0 ..  scales: with codes, the rows' powers of two, 32 of K and 32 of V.
    template <bool MASK>
    __device__ __forceinline__ void step(const char* kst, const char* vst, const float* scales, int n0, int end, float scale2) {
        const int qq = (threadIdx.x & 63) >> 4;
        f32x4 a[2][NT], vsc[2];
        logits<2>(kst, a);
        if constexpr (CODES) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const f32x4 ksc = *reinterpret_cast<const f32x4*>(scales + 16 * b + 4 * qq);
                vsc[b] = *reinterpret_cast<const f32x4*>(scales + 32 + 16 * b + 4 * qq);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) a[b][nt][j] *= ksc[j];
            }
        }
        raise<MASK, 2>(a, n0, end, scale2);
        weigh(a[0], a[1], vst, vsc, scale2);
    }

    // The lane quarters' shares of the sums together.
    __device__ __forceinline__ void close() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) l[nt] = sum_xor32(sum_xor16(l[nt]));
    }

    // Whether a weighted sum of the wave is not finite: 0 times it is a NaN then.
    __device__ __forceinline__ bool any_non_finite() const {
        float x = 0.f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
#pragma unroll
                for (int j = 0; j < 4; ++j) x = __builtin_fmaf(o[nt][db][j], 0.f, x);
        return __builtin_amdgcn_ballot_w64(x != x) != 0;
    }

    // With bf16 pages: the sums over rows that hold an infinity or a NaN, from the blocks of 32 rows n_beg, n_beg + step ..
    // below n_end.  Every query row sees these rows, so such a dim's sum is that of its non-finite values, where the
    // products made a NaN of every infinity (its probability's lower parts are 0 or negative, and a row that repeats the last
    // has the probability 0).  Only called where a sum is not finite, which is rare.
    __device__ __forceinline__ void sum_non_finite(const Pages& pg, const PageRows& pages, int n_beg, int n_end, int step) {
        constexpr int CH = D / 8, N = 32 * CH / 64;  // 16-byte pieces per row, and of 32 rows per lane
        const int lane = threadIdx.x & 63, qq = lane >> 4;
        uint32_t dims = 0;  // bit 4 db + j
        static_assert(D / 4 <= 32, "a bit for each of the lane's dims");
#pragma unroll 1
        for (uint32_t add = 0;; add = ~0u) {
#pragma unroll 1
            for (int n0 = n_beg; n0 < n_end; n0 += step) {
                bool here = false;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const size_t row = pages.row(min(n0 + (i * 64 + lane) / CH, n_end - 1));
                    here |= non_finite(load16(pg.v + (row * D + lane % CH * 8) * 2));
                }
                if (__builtin_amdgcn_ballot_w64(here) == 0) continue;
#pragma unroll 1
                for (int n = n0; n < min(n0 + 32, n_end); ++n) {
                    const uint8_t* v = pg.v + (pages.row(n) * D + 4 * qq) * 2;
#pragma unroll
                    for (int db = 0; db < D / 16; ++db) {
                        const u32x2 w = *reinterpret_cast<const u32x2*>(v + 32 * db);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t x = j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16;
                            // masks in vector registers: 32 conditions in scalar ones spill
                            const uint32_t odd = (x & 0x7F800000u) == 0x7F800000u ? ~0u : 0u;
                            dims |= odd & 1u << (4 * db + j);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) o[nt][db][j] += __uint_as_float(x & odd & add);
                        }
                    }
                }
            }
            if (add != 0) return;
            if (__builtin_amdgcn_ballot_w64(dims != 0) == 0) return;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint32_t drop = (uint32_t)((int)(dims << (31 - 4 * db - j)) >> 31);
                        o[nt][db][j] = __uint_as_float(__float_as_uint(o[nt][db][j]) & ~drop);
                    }
            }
        }
    }

    // Adds the non-finite values of V rows n0 .. n1 - 1 that a row sees: those of the new tokens in bf16, or, with
    // 8-bit pages, rows of the exponent byte 255.
    template <int KIND>
    __device__ __forceinline__ void add_non_finite(const Shape& s, const Chunk& ck, const Part& part, int bl,
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

// One lane's share of `ROWS` rows' K or V on its way from the pages.  LANES lanes work together, each on 16
// bytes of a row at a time: 8 bf16, or 16 codes.
template <int D, int KIND, int ROWS, int LANES>
struct Staged {
    static constexpr int CH = D * code_bytes(KIND) / 16;  // 16-byte pieces per row
    static constexpr int N = ROWS * CH / LANES;
    u32x4 x[N];
    __device__ __forceinline__ static int row_of(int it, int lane) { return (it * LANES + lane) / CH; }
    __device__ __forceinline__ static int piece_of(int it, int lane) { return (it * LANES + lane) % CH; }
};

// Results of a row: f32 or bf16.
template <int PARTS>
__device__ __forceinline__ void store_out(const Chunk& ck, size_t at, float v) {
    if constexpr (PARTS > 1) reinterpret_cast<float*>(ck.out)[at] = v;
    else reinterpret_cast<__bf16*>(ck.out)[at] = (__bf16)v;
}

// Shares of the keys.  An item is the work of one (segment, KV head, row tile).  Segments differ in length
// by an order of magnitude, and a call may have few of them, so a long item is cut into shares of S rows: its first share
// has the item's own workgroup, the others take the call's `extras` workgroups, which come first in
// the grid.  S = the call's rows over its extras, so that these suffice whatever the lengths are, and at least
// kShareRows.  A workgroup finds its share from the segments' lengths (a scan of at most kScanSegments; an item of
// up to kShareRows needs none).  Calls of more items have no extras and every item is whole.
//
// The shares of an item are joined in the same launch: each leaves its partial (maximum, sum, weighted sum per
// row) and then a mark, the call's number; the one that finds every mark joins the partials in order and clears
// the marks.  No workgroup waits.  Partials and marks are GPU-scope atomic accesses, which go through to memory, so
// that a finished store is visible on every XCD.  The workspace's first contents do not matter: a mark counts
// only if it is this call's number, 64 bits that differ between calls; a replayed graph brings its number again,
// but every call leaves its marks cleared.
struct Shares {
    unsigned long long* marks;  // [2 extras]
    float* part;                // [2 extras][rows][D + 2]
    unsigned long long call;
    int extras;
};
constexpr int kShareRows = 256;
constexpr int kMaxShares = 16;  // of an item
constexpr int kScanSegments = 2048;

struct Item {
    int bl, kvh, tile;
    int share, shares, rows;  // its share, shares of the item, rows per share
    int slot0;                // slots of the item: slot0 + {0 .. shares - 2} its extras, extras + slot0 its first share
    __device__ int slot(int i, int extras) const { return i == 0 ? extras + slot0 : slot0 + i - 1; }
};

__device__ __forceinline__ int rows_per_share(int len, int least) {
    return max(least, ((len + kMaxShares - 1) / kMaxShares + 63) / 64 * 64);
}

// The item and share of a workgroup; false: none.  `unit`, `tile`: its own item where it is not an extra.  Called by
// all threads, with the same arguments.
__device__ __forceinline__ bool take_share(const Shape& s, const Pages& pg, const Chunk& ck, const Shares& sh, int tiles,
                                           int units, int unit, int tile, Item& it) {
    __shared__ unsigned long long total_w[4];
    __shared__ int extra_w[4], found[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool extra = (int)blockIdx.x < sh.extras;
    if (!extra) {
        if (unit >= units) return false;
        it.kvh = unit % s.Hkv;
        it.bl = ck.unit_order != nullptr ? min(max(ck.unit_order[unit / s.Hkv], 0), s.B * s.L - 1) : unit / s.Hkv;
        it.tile = tile;
        it.share = 0;
        it.shares = 1;
        it.slot0 = 0;
        const Part part = part_of(s, pg, ck, it.bl);
        it.rows = part.first + part.count;
        if (part.count == 0) return false;
        if (sh.extras == 0 || it.rows <= kShareRows) return true;
    }
    // every thread has the segments of its own run
    const int n = s.B * s.L, per = (n + kThreads - 1) / kThreads, heads = s.Hkv * tiles;
    const int i0 = min(tid * per, n), i1 = min(i0 + per, n);
    auto read_length = [&](int i) {
        const Part p = part_of(s, pg, ck, i);
        return p.first + p.count;
    };
    const int length0 = i0 < i1 ? read_length(i0) : 0;  // the only one of up to 256 segments
    auto length = [&](int i) { return i == i0 ? length0 : read_length(i); };
    unsigned long long total = 0;
    for (int i = i0; i < i1; ++i) total += (unsigned)length(i);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
    if (lane == 0) total_w[wave] = total;
    if (tid == 0) found[0] = -1;
    __syncthreads();
    total = (total_w[0] + total_w[1] + total_w[2] + total_w[3]) * (unsigned)heads;
    const int least = (int)min((total / (unsigned)sh.extras + 64) / 64 * 64, 1ull << 30);
    const int rows0 = max(kShareRows, least);
    int mine = 0;  // extras of the thread's run
    for (int i = i0; i < i1; ++i) {
        const int len = length(i);
        if (len > rows0) mine += ((len - 1) / rows_per_share(len, rows0)) * heads;
    }
    int before = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(before, o);
        if (lane >= o) before += y;
    }
    if (lane == 63) extra_w[wave] = before;
    __syncthreads();
    before -= mine;
    for (int w = 0; w < wave; ++w) before += extra_w[w];
    for (int i = i0; i < i1; ++i) {
        const int len = length(i);
        const int k = len > rows0 ? (len - 1) / rows_per_share(len, rows0) : 0;
        const int x = (int)blockIdx.x - before;
        if (extra ? x >= 0 && x < k * heads : i == it.bl) {
            found[0] = i;
            found[1] = k + 1;
            found[2] = before;
            found[3] = rows_per_share(len, rows0);
        }
        before += k * heads;
    }
    __syncthreads();
    if (found[0] < 0) return false;
    it.shares = found[1];
    it.rows = found[3];
    if (extra) {
        const int x = (int)blockIdx.x - found[2], k = it.shares - 1;
        it.bl = found[0];
        it.kvh = x / k / tiles;
        it.tile = x / k % tiles;
        it.share = 1 + x % k;
    }
    it.slot0 = found[2] + (it.kvh * tiles + it.tile) * (it.shares - 1);
    return true;
}

__device__ __forceinline__ void store_shared(float* p, float v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float load_shared(const float* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Called by all threads of a workgroup after they wrote its share's partial of `rows` rows (of at most ROWS); the last
// to come joins them.  ml: LDS of 2 ROWS kMaxShares floats.  r0: the tile's first query row.
template <int D, int ROWS, int PARTS>
__device__ __forceinline__ void join_shares(const Shape& s, const Chunk& ck, const Shares& sh, const Item& it, int rows, int r0,
                                            float* ml) {
    __shared__ int all_here;
    const int tid = threadIdx.x, n = it.shares;
    wait_vmem_ordered();  // this thread's part of the partial has reached memory ...
    __syncthreads();      // ... and every thread's has, before the mark
    if (tid < 64) {
        if (tid == 0)
            __hip_atomic_store(sh.marks + it.slot(it.share, sh.extras), sh.call, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        wait_vmem_ordered();  // the mark has reached memory before the others' are read
        const bool here = tid >= n || __hip_atomic_load(sh.marks + it.slot(min(tid, n - 1), sh.extras), __ATOMIC_RELAXED,
                                                        __HIP_MEMORY_SCOPE_AGENT) == sh.call;
        const bool all = __ballot(!here) == 0;
        if (tid == 0) all_here = all;
    }
    __syncthreads();
    if (!all_here) return;
    for (int x = tid; x < rows * n; x += kThreads) {  // maxima and sums to LDS
        const int r = x / n, i = x % n;
        const float* p = sh.part + ((size_t)it.slot(i, sh.extras) * ROWS + r) * (D + 2);
        ml[r * kMaxShares + i] = load_shared(p);
        ml[(ROWS + r) * kMaxShares + i] = load_shared(p + 1);
    }
    __syncthreads();
    for (int x = tid; x < rows * D; x += kThreads) {
        const int r = x / D, e = x % D;
        float a[kMaxShares], M = kNegInf;
#pragma unroll
        for (int i = 0; i < kMaxShares; ++i)
            a[i] = load_shared(sh.part + ((size_t)it.slot(min(i, n - 1), sh.extras) * ROWS + r) * (D + 2) + 2 + e);
        for (int i = 0; i < n; ++i) M = fmaxf(M, ml[r * kMaxShares + i]);
        const float mu = M == kNegInf ? 0.f : M;
        float num = 0.f, den = 0.f;
#pragma unroll
        for (int i = 0; i < kMaxShares; ++i) {
            if (i < n) {
                const float sc = fast_exp2(ml[r * kMaxShares + i] - mu);
                num += rescaled(a[i], sc);
                den += sc * ml[(ROWS + r) * kMaxShares + i];
            }
        }
        store_out<PARTS>(ck, query_at(s, ck, it.bl, it.kvh, r0 + r, D) + e, num / den);
    }
    if (tid < n)
        __hip_atomic_store(sh.marks + it.slot(tid, sh.extras), 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int D, int KIND, int NT, int PARTS>
__global__ __launch_bounds__(kThreads, KIND != kCacheBf16 && NT == 1 ? 3 : 2) void few_kernel(Shape s, Pages pg, Chunk ck, Shares sh) {
    constexpr bool CODES = KIND != kCacheBf16;
    using B = Block<D, CODES>;
    constexpr int KB = 32;  // keys per block
    constexpr int ROWS = 16 * NT;
    constexpr int CPR = D / 8;  // 16-byte pieces of a bf16 row
    constexpr int STAGE = (B::kBytes + B::vBytes + (CODES ? 64 * (int)sizeof(float) : 0) + 15) / 16 * 16;
    constexpr int MERGE = 4 * ROWS * (D + 2) * (int)sizeof(float);
    static_assert(MERGE >= 2 * ROWS * kMaxShares * (int)sizeof(float), "room to join the shares");
    __shared__ __align__(16) char smem[4 * STAGE > MERGE ? 4 * STAGE : MERGE];
    extern __shared__ uint32_t lds_pages[];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Item it;
    const int units = s.B * s.L * s.Hkv;
    if (!take_share(s, pg, ck, sh, 1, units, (int)blockIdx.x - sh.extras, 0, it)) return;
    const int bl = it.bl, kvh = it.kvh;
    const Part part = part_of(s, pg, ck, bl);
    const int f = part.first, c = part.count, rows = c * s.G;
    const bool last_share = it.share == it.shares - 1;  // takes the new rows
    const int t0 = min(it.share * it.rows, f), t1 = it.shares == 1 ? f : min(t0 + it.rows, f);
    PageRows pages;
    pages.init<kThreads>(s, pg, bl, kvh, t0, t1, lds_pages);
    __syncthreads();

    char* kst = smem + wave * STAGE;
    char* vst = kst + B::kBytes;
    float* scales = reinterpret_cast<float*>(kst + (B::kBytes + B::vBytes + 15) / 16 * 16);
    Staged<D, KIND, KB, 64> ka, va;
    uint32_t ex = 0;  // codes: exponent byte of K row `lane`, or of V row `lane` - 32
    // A load instruction of the wave takes RPI rows.  Where they are one page's, their address is one scalar (the lanes'
    // own offsets never change); else, and at the end, each lane looks its row up.  Rows behind the last repeat it
    // (they count nothing), so every load is issued.
    constexpr int RPI = 64 / ka.CH;
    const bool wide_pages = (1 << pg.shift) >= RPI;
    const uint32_t lane_at = lane * 16;
    auto issue = [&](int n0) {
        if (wide_pages && n0 + KB <= t1) {
#pragma unroll
            for (int i = 0; i < ka.N; ++i) {
                const size_t at = pages.uniform_row(n0 + i * RPI) * (ka.CH * 16);
                ka.x[i] = load16_stream(pg.k + at + lane_at);
                va.x[i] = load16_stream(pg.v + at + lane_at);
            }
        } else {
#pragma unroll
            for (int i = 0; i < ka.N; ++i) {
                const size_t at = pages.row(min(n0 + ka.row_of(i, lane), t1 - 1)) * (ka.CH * 16) + ka.piece_of(i, lane) * 16;
                ka.x[i] = load16_stream(pg.k + at);
                va.x[i] = load16_stream(pg.v + at);
            }
        }
        if constexpr (CODES) ex = (lane < 32 ? pg.k_exp : pg.v_exp)[pages.row(min(n0 + (lane & 31), t1 - 1))];
    };
    const int blocks = (t1 - t0 + KB - 1) / KB;
    int n0 = t0 + KB * wave;
    if (n0 < t1) issue(n0);
    QueryRows<D, NT, PARTS, KIND> qr;
    qr.load(s, ck, part, bl, kvh, 0);
    qr.settle_rows();

    // the new rows, a block of their own for the wave that would take the next one: to the pages, and attended as
    // the pages hold them
    bool odd = false;  // a new value that is not finite
    if (last_share && wave == (blocks & 3)) {
        const int cc = lane % CPR;
        for (int i0 = 0; i0 < KB; i0 += 64 / CPR) {
            const int i = i0 + lane / CPR;
            u32x4 kr = {0u, 0u, 0u, 0u}, vr = {0u, 0u, 0u, 0u};
            uint32_t ke = 0, ve = 0;
            if (i0 < c) {
                if (i < c) {
                    const size_t src = (((size_t)bl * ck.chunk + i) * s.Hkv + kvh) * D + cc * 8;
                    kr = load16(ck.k_new + src);
                    vr = load16(ck.v_new + src);
                }
                const int page = i < c ? table_page(pg, bl, f + i) : -1;
                const bool in = page >= 0 && page < pg.n_pages;  // a row without a page is not written
                const size_t row = pool_row(pg, s.Hkv, kvh, page, f + i);
                if constexpr (CODES) {
                    ke = exp_byte<KIND>(group_max<CPR>(amax8(kr)));
                    ve = exp_byte<KIND>(group_max<CPR>(amax8(vr)));
                    const u32x2 kc = encode8<KIND>(kr, ke), vc = encode8<KIND>(vr, ve);
                    kr[0] = kc[0], kr[1] = kc[1], vr[0] = vc[0], vr[1] = vc[1];
                    if (in) {
                        *reinterpret_cast<u32x2*>(pg.k + row * D + cc * 8) = kc;
                        *reinterpret_cast<u32x2*>(pg.v + row * D + cc * 8) = vc;
                        if (cc == 0) {
                            pg.k_exp[row] = (uint8_t)ke;
                            pg.v_exp[row] = (uint8_t)ve;
                        }
                    }
                    odd |= ve == 255u;
                    if (ve == 255u) ve = 0;  // its values are 0 here
                } else {
                    if (in) {
                        store16(pg.k + (row * D + cc * 8) * 2, kr);
                        store16(pg.v + (row * D + cc * 8) * 2, vr);
                    }
                    const bool here = non_finite(vr);
                    odd |= here;
                    if (__builtin_amdgcn_ballot_w64(here) != 0 && here) drop_non_finite(vr);  // uniform branch
                }
            }
            if constexpr (CODES) {
                *reinterpret_cast<u32x2*>(kst + B::k_at(i) + cc * 8) = u32x2{kr[0], kr[1]};
                *reinterpret_cast<u32x2*>(vst + B::v_at(i) + cc * 8) = u32x2{vr[0], vr[1]};
                if (cc == 0) {
                    scales[i] = exp_scale(ke);
                    scales[32 + i] = exp_scale(ve);
                }
            } else {
                store16(kst + B::k_at(i) + cc * 16, kr);
                store16(vst + B::v_at(i) + cc * 16, vr);
            }
        }
        asm volatile("" ::: "memory");
        qr.template step<true>(kst, vst, scales, f, f + c, s.scale2);
        asm volatile("" ::: "memory");
    }
    for (; n0 < t1; n0 += 4 * KB) {
        asm volatile("" ::: "memory");  // this wave's reads of the previous block were issued before
#pragma unroll
        for (int i = 0; i < ka.N; ++i) {
            store16(kst + B::k_at(ka.row_of(i, lane)) + ka.piece_of(i, lane) * 16, ka.x[i]);
            store16(vst + B::v_at(ka.row_of(i, lane)) + ka.piece_of(i, lane) * 16, va.x[i]);
        }
        if constexpr (CODES) scales[lane] = exp_scale(ex);
        if (n0 + 4 * KB < t1) issue(n0 + 4 * KB);
        asm volatile("" ::: "memory");
        if (n0 + KB <= t1) qr.template step<false>(kst, vst, scales, n0, t1, s.scale2);
        else qr.template step<true>(kst, vst, scales, n0, t1, s.scale2);
    }
    qr.close();
    if constexpr (!CODES) {
        if (qr.any_non_finite()) qr.sum_non_finite(pg, pages, t0 + KB * wave, t1, 4 * KB);
    }
    if (__builtin_amdgcn_ballot_w64(odd) != 0) qr.template add_non_finite<KIND>(s, ck, part, bl, kvh, f, f + c);

    // the waves' partials through LDS
    __syncthreads();  // every wave is done with its stage
    const int c16 = lane & 15, qq = lane >> 4;
    float* wm = reinterpret_cast<float*>(smem);  // [4][ROWS]
    float* wl = wm + 4 * ROWS;
    float* wacc = wl + 4 * ROWS;  // [4][ROWS][D]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = nt * 16 + c16;
        if (r >= rows) continue;
        if (qq == 0) {
            wm[wave * ROWS + r] = qr.m[nt];
            wl[wave * ROWS + r] = qr.l[nt];
        }
#pragma unroll
        for (int db = 0; db < D / 16; ++db)
            *reinterpret_cast<f32x4*>(wacc + (size_t)(wave * ROWS + r) * D + 16 * db + 4 * qq) = qr.o[nt][db];
    }
    __syncthreads();
    float* mine = sh.part + (size_t)it.slot(it.share, sh.extras) * ROWS * (D + 2);
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
            num += rescaled(wacc[(size_t)(w * ROWS + r) * D + e], sc);
            den += sc * wl[w * ROWS + r];
        }
        if (it.shares == 1) {
            store_out<PARTS>(ck, query_at(s, ck, bl, kvh, r, D) + e, num / den);
        } else {
            store_shared(mine + r * (D + 2) + 2 + e, num);
            if (e == 0) {
                store_shared(mine + r * (D + 2), M);
                store_shared(mine + r * (D + 2) + 1, den);
            }
        }
    }
    if (it.shares > 1) join_shares<D, ROWS, PARTS>(s, ck, sh, it, rows, 0, wm);
}

// 16 bytes of a row's staged piece to LDS as bf16: 8 bf16, or 16 codes times their row's power of two.
template <int KIND>
__device__ __forceinline__ void put_bf16(char* p, const u32x4& x, float sc) {
    if constexpr (KIND == kCacheBf16) {
        store16(p, x);
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            store16(p + 16 * h, values8<KIND>(u32x2{x[2 * h], x[2 * h + 1]}, sc));
            __builtin_amdgcn_sched_barrier(0);  // few values in registers at a time
        }
    }
}

constexpr int kStreamChunk = 32;

// A workgroup per (segment, KV head, 64 NT query rows), and per share of its keys.
template <int D, int KIND, int NT, int PARTS>
__global__ __launch_bounds__(kThreads, NT == 1 ? 3 : 2) void rows_kernel(Shape s, Pages pg, Chunk ck, Shares sh, int tiles) {
    using B = Block<D, false>;
    constexpr int KT = 64;  // keys per tile
    constexpr int ROWS = 64 * NT;
    constexpr int STAGE = KT * (B::K + B::V), JOIN = 2 * ROWS * kMaxShares * (int)sizeof(float);
    static_assert(STAGE >= JOIN, "room to join the shares");
    __shared__ __align__(16) char smem[STAGE];
    __shared__ int odd_seen;
    extern __shared__ uint32_t lds_pages[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // the row tiles of a unit follow one another on one XCD (workgroups go to the 8 XCDs in turn), whose L2 then
    // holds the unit's keys
    const int units = s.B * s.L * s.Hkv, own = (int)blockIdx.x - sh.extras, x8 = own / 8;
    Item it;
    if (!take_share(s, pg, ck, sh, tiles, units, x8 / tiles * 8 + (own & 7), x8 % tiles, it)) return;
    const int bl = it.bl, kvh = it.kvh;
    const Part part = part_of(s, pg, ck, bl);
    const int rows = part.count * s.G, r_beg = it.tile * ROWS;
    if (r_beg >= rows) return;
    const int f = part.first, r_end = min(r_beg + ROWS, rows);
    const int seen = f + (r_end - 1) / s.G + 1;  // rows that the workgroup's last token sees
    const int t0 = it.shares == 1 ? 0 : min(it.share * it.rows, seen), t1 = it.shares == 1 ? seen : min(t0 + it.rows, seen);
    const int paged = KIND == kCacheBf16 ? f : seen;  // rows read from the pages; the rest from the inputs
    PageRows pages;
    pages.init<kThreads>(s, pg, bl, kvh, t0, min(t1, paged), lds_pages);
    if (tid == 0) odd_seen = 0;
    __syncthreads();

    Staged<D, KIND, KT, kThreads> ka, va;
    uint32_t ke[ka.N], ve[ka.N];  // codes: the rows' exponent bytes
    // Rows behind the last repeat it (they count nothing), so every load is issued.  With bf16 pages new rows come from
    // the inputs, at a stride of their own: addresses first, by the kind of tile (uniform branches), then the loads.
    const size_t new_row = (size_t)s.Hkv * D * 2;
    const size_t new0 = (((size_t)bl * ck.chunk - f) * s.Hkv + kvh) * D * 2;  // row n is at new0 + n new_row
    auto issue = [&](int n0) {
        const uint8_t *kp[ka.N], *vp[ka.N];
        if (KIND == kCacheBf16 && n0 >= f) {
#pragma unroll
            for (int i = 0; i < ka.N; ++i) {
                const size_t at = new0 + (size_t)min(n0 + ka.row_of(i, tid), t1 - 1) * new_row;
                kp[i] = reinterpret_cast<const uint8_t*>(ck.k_new) + at;
                vp[i] = reinterpret_cast<const uint8_t*>(ck.v_new) + at;
            }
        } else {
#pragma unroll
            for (int i = 0; i < ka.N; ++i) {
                const size_t row = pages.row(min(n0 + ka.row_of(i, tid), min(t1, paged) - 1));
                kp[i] = pg.k + row * (D * code_bytes(KIND));
                vp[i] = pg.v + row * (D * code_bytes(KIND));
                if constexpr (KIND != kCacheBf16) {
                    ke[i] = pg.k_exp[row];
                    ve[i] = pg.v_exp[row];
                }
            }
            if (KIND == kCacheBf16 && n0 + KT > f) {
#pragma unroll
                for (int i = 0; i < ka.N; ++i) {
                    const int n = min(n0 + ka.row_of(i, tid), t1 - 1);
                    const size_t at = new0 + (size_t)n * new_row;
                    kp[i] = n >= f ? reinterpret_cast<const uint8_t*>(ck.k_new) + at : kp[i];
                    vp[i] = n >= f ? reinterpret_cast<const uint8_t*>(ck.v_new) + at : vp[i];
                }
            }
        }
        // Where the call is a read of the retained rows, once (one row tile per unit, few tokens), they are streamed: 5 tokens of
        // 7 heads on the video shape 67 us against 75.  Several tiles find the keys in L2, and with more tokens, whose
        // rows are read again to be written to the pages, plain loads are faster: 64 tokens of one head on the LLaVA-NeXT shape
        // 185 us against 199.  Only these two were measured.  With 33 to 64 query rows (NT = 1) the limit lies between them:
        // up to 31 tokens means two heads or more per KV head, 33 and more means one.
        if (NT == 1 && ck.chunk < kStreamChunk) {
            asm volatile("; streamed");  // the compiler would merge the two branches' loads, and drop the hint
#pragma unroll
            for (int i = 0; i < ka.N; ++i) {
                ka.x[i] = load16_global<true>(kp[i] + ka.piece_of(i, tid) * 16);
                va.x[i] = load16_global<true>(vp[i] + ka.piece_of(i, tid) * 16);
            }
            asm volatile("; streamed");
        } else {
#pragma unroll
            for (int i = 0; i < ka.N; ++i) {
                ka.x[i] = load16_global<false>(kp[i] + ka.piece_of(i, tid) * 16);
                va.x[i] = load16_global<false>(vp[i] + ka.piece_of(i, tid) * 16);
            }
        }
    };
    if (t0 < t1) issue(t0);
    QueryRows<D, NT, PARTS, kCacheBf16> qr;
    const int w0 = r_beg + wave * 16 * NT;  // the wave's first row
    qr.load(s, ck, part, bl, kvh, w0);
    qr.settle_rows();
    // the wave's rows see all rows below `all`, and none from `none` on
    const int all = f + min(w0, rows - 1) / s.G + 1, none = w0 < rows ? f + min(w0 + 16 * NT - 1, rows - 1) / s.G + 1 : 0;

    // the loaded tile n0 into LDS
    auto put = [&](int n0, char* st) {
        if (n0 + KT > f) {
            bool odd = false;
#pragma unroll
            for (int i = 0; i < va.N; ++i) {
                if constexpr (KIND == kCacheBf16) {
                    const bool here = n0 + va.row_of(i, tid) >= f && non_finite(va.x[i]);
                    odd |= here;
                    if (__builtin_amdgcn_ballot_w64(here) != 0 && here) drop_non_finite(va.x[i]);  // uniform branch
                } else if (n0 + va.row_of(i, tid) >= f && ve[i] == 255u) {
                    ve[i] = 0;
                    odd = true;
                }
            }
            if (odd) odd_seen = 1;
        }
#pragma unroll
        for (int i = 0; i < ka.N; ++i) {
            const int row = ka.row_of(i, tid), at = ka.piece_of(i, tid) * (KIND == kCacheBf16 ? 16 : 32);
            put_bf16<KIND>(st + B::k_at(row) + at, ka.x[i], KIND == kCacheBf16 ? 1.f : exp_scale(ke[i]));
            put_bf16<KIND>(st + KT * B::K + B::v_at(row) + at, va.x[i], KIND == kCacheBf16 ? 1.f : exp_scale(ve[i]));
        }
    };
    for (int n0 = t0; n0 < t1; n0 += KT) {
        __syncthreads();  // the tile before this one has been read
        put(n0, smem);
        if (n0 + KT < t1) issue(n0 + KT);
        __syncthreads();
        if (n0 >= none) continue;
        f32x4 a[4][NT];
        qr.template logits<4>(smem, a);
        if (n0 + KT <= min(all, t1)) qr.template raise<false, 4>(a, n0, t1, s.scale2);
        else qr.template raise<true, 4>(a, n0, t1, s.scale2);
        qr.weigh(a[0], a[1], smem + KT * B::K, nullptr, s.scale2);
        qr.weigh(a[2], a[3], smem + KT * B::K + 32 * B::V, nullptr, s.scale2);
    }
    qr.close();
    if constexpr (KIND == kCacheBf16) {
        if (qr.any_non_finite()) qr.sum_non_finite(pg, pages, t0, min(t1, f), 32);
    }
    __syncthreads();
    if (odd_seen) qr.template add_non_finite<KIND>(s, ck, part, bl, kvh, max(f, t0), t1);

    const int c16 = lane & 15, qq = lane >> 4;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = w0 + nt * 16 + c16;
        if (r >= rows) continue;
        if (it.shares == 1) {
            const float inv = 1.f / qr.l[nt];
            const size_t at = query_at(s, ck, bl, kvh, r, D) + 4 * qq;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
                const f32x4 v = qr.o[nt][db] * inv;
                if constexpr (PARTS > 1) {
                    *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(ck.out) + at + 16 * db) = v;
                } else {
                    const bf16x4 w = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
                    *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(ck.out) + at + 16 * db) = w;
                }
            }
        } else {
            float* p = sh.part + ((size_t)it.slot(it.share, sh.extras) * ROWS + r - r_beg) * (D + 2);
            if (qq == 0) {
                store_shared(p, qr.m[nt]);
                store_shared(p + 1, qr.l[nt]);
            }
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
#pragma unroll
                for (int j = 0; j < 4; ++j) store_shared(p + 2 + 16 * db + 4 * qq + j, qr.o[nt][db][j]);
        }
    }
    // the new rows into the pages: those of the tokens whose first query row is here
    if constexpr (KIND == kCacheBf16) {
        constexpr int CPR = D / 8;
        const int i_end = it.share == 0 ? (r_end - 1) / s.G + 1 : 0;
        for (int i = (r_beg + s.G - 1) / s.G + tid / CPR; i < i_end; i += kThreads / CPR) {
            const int page = table_page(pg, bl, f + i);
            if (page < 0 || page >= pg.n_pages) continue;
            const size_t row = pool_row(pg, s.Hkv, kvh, page, f + i), src = ((size_t)bl * ck.chunk + i) * s.Hkv + kvh;
            const int e = tid % CPR * 8;
            store16(pg.k + (row * D + e) * 2, load16(ck.k_new + src * D + e));
            store16(pg.v + (row * D + e) * 2, load16(ck.v_new + src * D + e));
        }
    }
    if (it.shares > 1) join_shares<D, ROWS, PARTS>(s, ck, sh, it, r_end - r_beg, r_beg, reinterpret_cast<float*>(smem));
}

// Workgroups for further shares, in calls of up to so many items.  Few extras make long shares, and each costs its
// scan whether there is a share for it or not: five tokens on the video shape (896 items, layers of 139 to 5449 rows)
// 82 us with 256, 62 with 384, 60 with 448, 67 with 512, 76 with 1024; single tokens there on 8-bit pages 67, 54, 54,
// 54 and 62 us.  The number was chosen on this one shape, whatever a call's items.  More items than kItemsOfExtras even
// out in part, longest first: a step from 2016 to 2128 items of such layers (18 and 19 sequences) takes five tokens
// from 110 to 167 us, single tokens on bf16 pages from 90 to 93 and on int8 pages from 63 to 78; without unit_order,
// 161 to 251, 105 to 143 and 83 to 125.
constexpr int kExtras = 448, kItemsOfExtras = 2048;

// How a call is dealt out.
struct Plan {
    bool few;        // few_kernel
    int nt, tiles;   // 16-row blocks per wave; row tiles per unit
    int extras;      // workgroups for the further shares of long items
    int part_rows;   // query rows of a partial
};

Plan plan_chunk(const Shape& s, int32_t chunk) {
    const long long units = (long long)s.B * s.L * s.Hkv, rows = (long long)chunk * s.G;
    Plan p;
    p.few = rows <= 32;
    p.nt = p.few ? (rows <= 16 ? 1 : 2) : (rows <= 64 ? 1 : 2);
    p.tiles = p.few ? 1 : (int)((rows + 64 * p.nt - 1) / (64 * p.nt));
    p.part_rows = (p.few ? 16 : 64) * p.nt;
    const long long items = units * p.tiles;
    p.extras = items > 0 && items <= kItemsOfExtras && (long long)s.B * s.L <= kScanSegments ? kExtras : 0;
    return p;
}

// Workgroups of few_kernel, or of rows_kernel with the units' row tiles in groups of 8 units.
long long attention_workgroups(const Shape& s, const Plan& p) {
    const long long units = (long long)s.B * s.L * s.Hkv;
    return p.extras + (p.few ? units : (units + 7) / 8 * 8 * p.tiles);
}

size_t partial_floats(const Shape& s, const Plan& p) { return (size_t)2 * p.extras * p.part_rows * (s.D + 2); }

// A number that no other call of the process has; never 0.
unsigned long long call_number() {
    static std::atomic<unsigned long long> next{
        (unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() * 0x9E3779B97F4A7C15ull};
    unsigned long long call;
    do call = next.fetch_add(1, std::memory_order_relaxed); while (call == 0);
    return call;
}

template <int D, int KIND, int PARTS>
hipError_t launch_chunk_d(const Shape& s, const Pages& pg, const Chunk& ck, hipStream_t st) {
    const Plan p = plan_chunk(s, ck.chunk);
    const size_t lds = lds_pages_bytes(pg);
    const dim3 grid((unsigned)attention_workgroups(s, p));
    Shares sh{nullptr, nullptr, 0, p.extras};
    if (p.extras > 0) {
        sh.call = call_number();
        sh.part = ck.ws;
        sh.marks = reinterpret_cast<unsigned long long*>(ck.ws + partial_floats(s, p));
    }
    if (p.few) {
        if (p.nt == 1) hipLaunchKernelGGL((few_kernel<D, KIND, 1, PARTS>), grid, dim3(kThreads), lds, st, s, pg, ck, sh);
        else hipLaunchKernelGGL((few_kernel<D, KIND, 2, PARTS>), grid, dim3(kThreads), lds, st, s, pg, ck, sh);
        return hipGetLastError();
    }
    if constexpr (KIND != kCacheBf16) {
        constexpr int RPP = kThreads / (D / 8);
        const int parts = (int)std::min<long long>(((long long)ck.chunk * s.Hkv + RPP - 1) / RPP, 256);
        hipLaunchKernelGGL((append_kernel<D, KIND>), dim3(s.B * s.L, parts), dim3(kThreads), 0, st, s, pg, ck);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.nt == 1)
        hipLaunchKernelGGL((rows_kernel<D, KIND, 1, PARTS>), grid, dim3(kThreads), lds, st, s, pg, ck, sh, p.tiles);
    else
        hipLaunchKernelGGL((rows_kernel<D, KIND, 2, PARTS>), grid, dim3(kThreads), lds, st, s, pg, ck, sh, p.tiles);
    return hipGetLastError();
}

constexpr int kFineParts = 3;  // bf16 parts of a probability with 32-bit results: all of its 24 bits

template <int D, int KIND>
hipError_t launch_chunk_k(const Shape& s, const Pages& pg, const Chunk& ck, hipStream_t st) {
    return ck.out_bf16 ? launch_chunk_d<D, KIND, 1>(s, pg, ck, st) : launch_chunk_d<D, KIND, kFineParts>(s, pg, ck, st);
}

}  // namespace

int64_t chunk_workgroups(const Shape& s, int32_t chunk) { return attention_workgroups(s, plan_chunk(s, chunk)); }

size_t chunk_workspace(const Shape& s, int32_t chunk) {
    const Plan p = plan_chunk(s, chunk);
    return sizeof(float) * partial_floats(s, p) + sizeof(unsigned long long) * 2 * (size_t)p.extras;
}

// The largest of the chunks up to `chunk`.  A partial's rows step up behind 16, 32 and 64 query rows, and among chunks of
// the same the first has the fewest items: where it has no extras, none has.
size_t chunk_workspace_up_to(const Shape& s, int32_t chunk) {
    size_t most = 0;
    for (const int32_t rows : {0, 16, 32, 64})
        if (rows / s.G + 1 <= chunk) most = std::max(most, chunk_workspace(s, rows / s.G + 1));
    return most;
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
