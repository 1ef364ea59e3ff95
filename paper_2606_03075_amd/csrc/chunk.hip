// Attention of a chunk of new tokens over the paged cache.
//
// A sequence at step s brings c new tokens.  In every layer their keys and values become rows
// f .. f + c - 1 of the segment, f = b_l + s, and token i attends to rows n <= f + i (Eq. (2) over the
// pruned cache of Eq. (3)-(4)): c decode steps in one call.  append_kernel writes the rows into the pages
// (quantised, where the pages hold 8 bits); attention then reads the pages only, so a token sees the
// values that every later step will see.
#include <algorithm>
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
        const bool in = page >= 0 && page < pg.n_pages;  // a row without a page is not written
        const size_t row = pool_row(pg, s.Hkv, kvh, page, n);
        if constexpr (KIND == kCacheBf16) {
            if (in) {
                store16(pg.k + (row * D + cc * 8) * 2, kr);
                store16(pg.v + (row * D + cc * 8) * 2, vr);
            }
        } else {
            const uint32_t ke = exp_byte<KIND>(group_max<CPR>(amax8(kr)));
            const uint32_t ve = exp_byte<KIND>(group_max<CPR>(amax8(vr)));
            if (in) {
                *reinterpret_cast<u32x2*>(pg.k + row * D + cc * 8) = encode8<KIND>(kr, ke);
                *reinterpret_cast<u32x2*>(pg.v + row * D + cc * 8) = encode8<KIND>(vr, ve);
                if (cc == 0) {
                    pg.k_exp[row] = (uint8_t)ke;
                    pg.v_exp[row] = (uint8_t)ve;
                }
            }
        }
    }
}

// A wave per (segment, new token, query head): 64 keys at a time, a key per lane for the logits, D/64 dims
// per lane for the weighted sum.
template <int D, int KIND, bool OUT_BF16>
__global__ __launch_bounds__(kThreads) void chunk_kernel(Shape s, Pages pg, Chunk ck) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __shared__ float qs[4][D];
    const long long w = (long long)blockIdx.x * 4 + wave;
    const int h = (int)(w % s.H), i = (int)(w / s.H % ck.chunk);
    const int bl = (int)min(w / s.H / ck.chunk, (long long)s.B * s.L - 1);
    const Part part = part_of(s, pg, ck, bl);
    const bool live = w / s.H / ck.chunk < (long long)s.B * s.L && i < part.count;
    const size_t at = (((size_t)bl * ck.chunk + i) * s.H + h) * D;
    for (int e = lane; e < D; e += 64) qs[wave][e] = live ? bf16_bits_to_float(ck.q[at + e]) * s.scale2 : 0.f;
    __syncthreads();
    if (!live) return;
    const int kvh = h / s.G, len = part.first + i + 1;
    float m = kNegInf, l = 0.f, acc[D / 64] = {};
    for (int n0 = 0; n0 < len; n0 += 64) {
        const int n = min(n0 + lane, len - 1);
        const size_t row = pool_row(pg, s.Hkv, kvh, table_page(pg, bl, n), n);
        float z = 0.f;
        for (int e = 0; e < D; e += 8) {
            u32x4 kr;
            if constexpr (KIND == kCacheBf16) kr = load16(pg.k + (row * D + e) * 2);
            else kr = decode8<KIND>(*reinterpret_cast<const u32x2*>(pg.k + row * D + e));
            for (int j = 0; j < 4; ++j) {
                z += qs[wave][e + 2 * j] * __uint_as_float(kr[j] << 16);
                z += qs[wave][e + 2 * j + 1] * __uint_as_float(kr[j] & 0xFFFF0000u);
            }
        }
        float vs = 1.f;
        if constexpr (KIND != kCacheBf16) {
            z *= exp_scale(pg.k_exp[row]);
            vs = exp_scale(pg.v_exp[row]);
        }
        if (n0 + lane >= len) z = kNegInf;
        float mb = z;
        for (int o = 32; o > 0; o >>= 1) mb = fmaxf(mb, __shfl_xor(mb, o));
        const float mn = fmaxf(m, mb), mu = mn == kNegInf ? 0.f : mn, sc = fast_exp2(m - mu);
        const float p = fast_exp2(z - mu);  // every logit -inf: sums of 0, and 0 / 0 as in the formula
        float ps = p;
        for (int o = 32; o > 0; o >>= 1) ps += __shfl_xor(ps, o);
        l = l * sc + ps;
        m = mn;
        for (int x = 0; x < D / 64; ++x) acc[x] *= sc;
        const float pv = p * vs;
        for (int u = 0; u < min(64, len - n0); ++u) {
            const float pu = __shfl(pv, u);
            const size_t ru = (size_t)__shfl((long long)row, u);
            for (int x = 0; x < D / 64; ++x) {
                const int e = x * 64 + lane;
                float vv;
                if constexpr (KIND == kCacheBf16) vv = bf16_bits_to_float(reinterpret_cast<const uint16_t*>(pg.v)[ru * D + e]);
                else if constexpr (KIND == kCacheInt8) vv = (float)(int8_t)pg.v[ru * D + e];
                else vv = __builtin_amdgcn_cvt_f32_fp8((int)pg.v[ru * D + e], 0);
                acc[x] += pu * vv;
            }
        }
    }
    for (int x = 0; x < D / 64; ++x) {
        const float o = acc[x] / l;
        if constexpr (OUT_BF16) reinterpret_cast<__bf16*>(ck.out)[at + x * 64 + lane] = (__bf16)o;
        else reinterpret_cast<float*>(ck.out)[at + x * 64 + lane] = o;
    }
}

template <int D, int KIND>
hipError_t launch_chunk_d(const Shape& s, const Pages& pg, const Chunk& ck, hipStream_t st) {
    constexpr int RPP = kThreads / (D / 8);
    const int units = s.B * s.L;
    const long long rows = (long long)ck.chunk * s.Hkv;
    const int parts = (int)std::min<long long>((rows + RPP - 1) / RPP, 256);
    hipLaunchKernelGGL((append_kernel<D, KIND>), dim3(units, parts), dim3(kThreads), 0, st, s, pg, ck);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)(((long long)units * ck.chunk * s.H + 3) / 4));
    if (ck.out_bf16) hipLaunchKernelGGL((chunk_kernel<D, KIND, true>), grid, dim3(kThreads), 0, st, s, pg, ck);
    else hipLaunchKernelGGL((chunk_kernel<D, KIND, false>), grid, dim3(kThreads), 0, st, s, pg, ck);
    return hipGetLastError();
}

}  // namespace

size_t chunk_workspace(const Shape&, int32_t) { return 0; }

hipError_t launch_chunk(const Shape& s, const Pages& pg, const Chunk& ck, hipStream_t st) {
    if ((long long)s.B * s.L == 0) return hipSuccess;
    if (s.D == 128) {
        if (pg.kind == kCacheBf16) return launch_chunk_d<128, kCacheBf16>(s, pg, ck, st);
        if (pg.kind == kCacheFp8) return launch_chunk_d<128, kCacheFp8>(s, pg, ck, st);
        return launch_chunk_d<128, kCacheInt8>(s, pg, ck, st);
    }
    if (pg.kind == kCacheBf16) return launch_chunk_d<64, kCacheBf16>(s, pg, ck, st);
    if (pg.kind == kCacheFp8) return launch_chunk_d<64, kCacheFp8>(s, pg, ck, st);
    return launch_chunk_d<64, kCacheInt8>(s, pg, ck, st);
}

}  // namespace tgvkv
