// Attention of new tokens over pages or packed rows on the fp32 matrix instructions: fp32 tensors, and bf16 ones with a head size
// that the bf16 kernels do not have.  Any head_dim <= 256 that is a multiple of 4.
//
// A wave owns 16 rows and goes through its keys alone, 16 or 32 at a time: S^T = K Q^T (16x16x4: a lane then holds one query and
// four keys of every 16), one running (max, sum) per row, O^T += V^T P^T.  The contraction index of an MFMA is the lane group
// g = lane / 16; which dims or keys that stands for is free as long as both operands agree, and is chosen so that no operand is
// ever moved between lanes: dims 16s + 4g + c of step (s, c) for the first product (a lane reads K and Q four dims at a time),
// key 4g + i of step i for the second (where register i of S^T already is).  K and V come straight from memory into registers:
// a row is read in runs of 64 bytes (K) and 256 (V), the four waves of a workgroup find each other's rows in L1.
// With few rows the four waves share one block of 16 rows and deal the keys among themselves; they merge through LDS.
//
// What bounds it: the matrix pipe (32 cycles per 16x16x4; two products of 2 * 16 * keys * d), and for small prompts the start: prompts
// of 1 to 641 tokens, 8 heads on 4 of 64, take 16.8 us, about ten of them lookups, first trips to memory and the last row block's walk.
#include "attend.h"

namespace dyspec {

typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kF32Waves = 4;

template <typename T, int DP, bool Paged>
__global__ __launch_bounds__(64 * kF32Waves, DP <= 128 || (DP == 192 && sizeof(T) == 2) ? 2 : 1) void attend_f32_kernel(AttendArgs, int row_waves)
{
    const AttendArgs& a = attend_args_here();
    typedef typename Four<T>::raw raw;
    constexpr int NS = DP / 16, NB = DP / 64;
    constexpr int KB = DP <= 128 ? 32 : 16, N16 = KB / 16, RUNS = KB / 8;      // keys of a step; runs of eight keys lie each within a page
    constexpr int kAhead = 64 / RUNS;                                          // steps whose page numbers the lanes hold
    __shared__ float merge_area[kF32Waves - 1][64 * (16 * NB + 2)];
    __shared__ int flag;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;
    const int R = 16 * row_waves, key_waves = kF32Waves / row_waves;
    const int wq = wave & (row_waves - 1), wk = row_waves == 1 ? wave : 0;
    const AttendItem it = attend_item(a, blockIdx.x);
    const AttendSeq& s = it.s;
    const int d = a.d, rows = a.G * s.N, r0 = it.block * R;
    const int r = r0 + 16 * wq + n, rc = min(r, rows - 1);
    const int j = div_G(a, rc), h = it.kvh * a.G + (rc - j * a.G);
    const int end = s.C + div_G(a, min(r0 + R, rows) - 1) + 1;     // keys that some row of the block may see
    const int n_parts = s.parts > 1 ? (end + s.share - 1) / s.share : 1;
    if (it.part >= n_parts) return;
    const int k_begin = s.parts > 1 ? it.part * s.share : 0, k_end = s.parts > 1 ? min(end, k_begin + s.share) : end;
    const int last = k_end - 1;
    const int full = a.mask ? s.C : s.C + div_G(a, min(r0 + 16 * wq, rows - 1)) + 1;       // keys before this one are every row's of the wave
    const int size = (int)sizeof(T);
    const long long k_stride = a.k_stride, v_stride = a.v_stride, page_bytes = a.page_bytes;
    const char* const kp = a.k + (long long)it.kvh * d * size;
    const char* const vp = a.v + (long long)it.kvh * d * size;
    const float c2 = a.c2;

    // Q: dims 16s + 4g .. of query n; a piece past head_dim is zero here and in K
    float4 q[NS];
    const char* const qrow = a.q + (long long)(s.row0 + j) * a.q_stride + (long long)h * d * size;
#pragma unroll
    for (int x = 0; x < NS; ++x) {
        const int dim = 16 * x + 4 * g;
        q[x] = dim < d ? Four<T>::wide(*reinterpret_cast<const raw*>(qrow + dim * size)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    floatx4 acc[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[b][c] = floatx4{ 0.0f, 0.0f, 0.0f, 0.0f };
    float m = kLowest, l = 0.0f;

    // page numbers of this wave's steps i0 .. i0 + kAhead - 1: lane RUNS (i - i0) + u has run u's
    const int first_key = k_begin + KB * wk, key_step = KB * key_waves;
    const int page_shift = a.page_shift, page_mask = (1 << page_shift) - 1;
    auto fetch_pages = [=, &a](int i0) __attribute__((always_inline)) -> uint32_t {
        const int key = min(first_key + key_step * (i0 + lane / RUNS) + 8 * (lane % RUNS), last);
        return min((uint32_t)a.table[(long long)s.id * a.table_stride + (key >> page_shift)], (uint32_t)a.n_pages - 1u);
    };
    uint32_t pages = 0u;
    if constexpr (Paged) pages = fetch_pages(0);
    // Row of key key0 + off (of run u_lo where low, else of the next one) of step i; keys past the last one repeat it.
    auto row_of = [=](const char* base, long long stride, uint32_t window, int i, int key0, int off, int u_lo, bool low) __attribute__((always_inline)) -> const char* {
        const int key = min(key0 + off, last);
        if constexpr (Paged) {
            const uint32_t p0 = (uint32_t)__builtin_amdgcn_readlane((int)window, RUNS * (i & (kAhead - 1)) + u_lo);
            const uint32_t p1 = (uint32_t)__builtin_amdgcn_readlane((int)window, RUNS * (i & (kAhead - 1)) + u_lo + 1);
            const long long b0 = (long long)p0 * page_bytes, b1 = (long long)p1 * page_bytes;
            return base + (low ? b0 : b1) + (key & page_mask) * stride;
        } else {
            return base + (s.row0 + key) * stride;
        }
    };
    auto load_k = [=](raw (&kr)[N16][NS], uint32_t window, int i, int key0) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < N16; ++b) {
            const char* const row = row_of(kp, k_stride, window, i, key0, 16 * b + n, 2 * b, n < 8);
#pragma unroll
            for (int x = 0; x < NS; ++x) {
                const int dim = 16 * x + 4 * g;
                kr[b][x] = *reinterpret_cast<const raw*>(row + (dim < d ? dim : 0) * size);
            }
        }
    };
    raw kr[N16][NS];
    int key0 = first_key;
    if (key0 < k_end) load_k(kr, pages, 0, key0);
    for (int i = 0; key0 < k_end; ++i, key0 += key_step) {
        // V: dims 64b + 4n .. of keys 4g + x
        raw vr[N16][4][NB];
#pragma unroll
        for (int b = 0; b < N16; ++b)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const char* const row = row_of(vp, v_stride, pages, i, key0, 16 * b + 4 * g + x, 2 * b, g < 2);
#pragma unroll
                for (int y = 0; y < NB; ++y) {
                    const int dim = 64 * y + 4 * n;
                    vr[b][x][y] = *reinterpret_cast<const raw*>(row + (dim < d ? dim : 0) * size);
                }
            }
        floatx4 S[N16];                                            // (the blocks' chains in turn: a dependent MFMA waits for its accumulator)
#pragma unroll
        for (int b = 0; b < N16; ++b) S[b] = floatx4{ 0.0f, 0.0f, 0.0f, 0.0f };
#pragma unroll
        for (int x = 0; x < NS; ++x) {
            float4 k[N16];
#pragma unroll
            for (int b = 0; b < N16; ++b) {
                k[b] = Four<T>::wide(kr[b][x]);
                if (16 * x + 16 > d && 16 * x + 4 * g >= d) k[b] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
#pragma unroll
            for (int b = 0; b < N16; ++b) S[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[b].x, q[x].x, S[b], 0, 0, 0);
#pragma unroll
            for (int b = 0; b < N16; ++b) S[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[b].y, q[x].y, S[b], 0, 0, 0);
#pragma unroll
            for (int b = 0; b < N16; ++b) S[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[b].z, q[x].z, S[b], 0, 0, 0);
#pragma unroll
            for (int b = 0; b < N16; ++b) S[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[b].w, q[x].w, S[b], 0, 0, 0);
        }
        if (key0 + key_step < k_end) {
            if constexpr (Paged)
                if (((i + 1) & (kAhead - 1)) == 0) pages = fetch_pages(i + 1);
            load_k(kr, pages, i + 1, key0 + key_step);
        }
        // scores of keys a row does not see: -inf, whatever K holds there
        if (key0 + KB > full || key0 + KB > k_end) {
            uint32_t seen = seen_bits(a, s, j, key0);
            if (k_end - key0 < KB) seen &= (1u << (k_end - key0)) - 1u;
#pragma unroll
            for (int b = 0; b < N16; ++b)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (!((seen >> (16 * b + 4 * g + x)) & 1u)) S[b][x] = -INFINITY;
        }
        float up = m;
#pragma unroll
        for (int b = 0; b < N16; ++b) up = fmaxf(fmaxf(fmaxf(S[b][0], S[b][1]), fmaxf(S[b][2], S[b][3])), up);
        up = fmaxf(up, __shfl_xor(up, 16, kWave));
        up = fmaxf(up, __shfl_xor(up, 32, kWave));
        if (__any(up != m)) {
            const float f = __builtin_amdgcn_exp2f((m - up) * c2);
            m = up;
            l *= f;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[b][c] *= f;
        }
#pragma unroll
        for (int b = 0; b < N16; ++b)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float p = S[b][x] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((S[b][x] - m) * c2);
                l += p;
#pragma unroll
                for (int y = 0; y < NB; ++y) {
                    const float4 v = Four<T>::wide(vr[b][x][y]);
                    acc[y][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.x, p, acc[y][0], 0, 0, 0);
                    acc[y][1] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.y, p, acc[y][1], 0, 0, 0);
                    acc[y][2] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.z, p, acc[y][2], 0, 0, 0);
                    acc[y][3] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.w, p, acc[y][3], 0, 0, 0);
                }
            }
    }
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);

    // ---- waves that shared a block of rows
    if (key_waves > 1) {
        if (wk > 0) {
            float* const dst = merge_area[wk - 1] + lane;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) dst[64 * (16 * b + 4 * c + i)] = acc[b][c][i];
            dst[64 * 16 * NB] = m;
            dst[64 * (16 * NB + 1)] = l;
        }
        __syncthreads();
        if (wk == 0) {
            for (int w = 1; w < key_waves; ++w) {
                const float* const src = merge_area[w - 1] + lane;
                const float m1 = src[64 * 16 * NB], up = fmaxf(m, m1);
                const float f0 = exp2f((m - up) * a.c2), f1 = exp2f((m1 - up) * a.c2);
                m = up;
                l = l * f0 + src[64 * (16 * NB + 1)] * f1;
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[b][c][i] = acc[b][c][i] * f0 + src[64 * (16 * b + 4 * c + i)] * f1;
            }
        }
    }
    // ---- the rows leave: acc[b][c][i] is dim 64b + 16g + 4i + c
    float* const slot = part_slot(a, it, R);
    if (wk == 0) {
        bool nan = l != l;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (64 * b + 16 * g + 4 * i < a.d) nan |= acc[b][c][i] != acc[b][c][i];
        const uint64_t lanes = __builtin_amdgcn_ballot_w64(nan && r < rows);
        const uint32_t bad = (uint32_t)((lanes | lanes >> 16 | lanes >> 32 | lanes >> 48) & 0xffffu);
        const bool leave = r < rows;
        if (n_parts > 1) {
            if (g == 0 && leave) store_pair(slot_max_sum(a, slot, R, 16 * wq + n), m, l);
            if (leave) {
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int dim = 64 * b + 16 * g + 4 * i;
                        if (dim < a.d)
                            store_four(slot + slot_place<kSlotF32>(a.d, 16 * wq + n, dim / 4), acc[b][0][i], acc[b][1][i], acc[b][2][i], acc[b][3][i]);
                    }
            }
        } else if (leave) {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            char* const dst = out_row(a, s, j, h, size);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int dim = 64 * b + 16 * g + 4 * i;
                    if (dim < a.d)
                        Four<T>::store(dst + dim * size, make_float4(acc[b][0][i] * inv, acc[b][1][i] * inv, acc[b][2][i] * inv, acc[b][3][i] * inv));
                }
        }
        if (__builtin_expect(bad != 0u, 0))
            look_again<T, kSlotF32, DP>(bad, 16 * wq, 0, a.d, R, [=](int row) { return __shfl(m, row & 15, kWave); });
    }
    if (n_parts > 1 && arrive_last(a, it, n_parts, &flag)) merge_parts<T, kSlotF32, 0>(a, it, n_parts, R, 64 * kF32Waves);
}

template <typename T, bool Paged>
static void launch_f32(const AttendArgs& a, int row_waves, int blocks, hipStream_t stream)
{
    if (a.d <= 64) attend_f32_kernel<T, 64, Paged><<<blocks, 64 * kF32Waves, 0, stream>>>(a, row_waves);
    else if (a.d <= 128) attend_f32_kernel<T, 128, Paged><<<blocks, 64 * kF32Waves, 0, stream>>>(a, row_waves);
    else if (a.d <= 192) attend_f32_kernel<T, 192, Paged><<<blocks, 64 * kF32Waves, 0, stream>>>(a, row_waves);
    else attend_f32_kernel<T, 256, Paged><<<blocks, 64 * kF32Waves, 0, stream>>>(a, row_waves);
}

hipError_t launch_attend_f32(const AttendArgs& a, int dtype, int row_waves, int items, hipStream_t stream)
{
    const int blocks = items * a.Hkv;
    if (dtype == DYSPEC_F32) {
        if (a.table) launch_f32<float, true>(a, row_waves, blocks, stream); else launch_f32<float, false>(a, row_waves, blocks, stream);
    } else {
        if (a.table) launch_f32<__bf16, true>(a, row_waves, blocks, stream); else launch_f32<__bf16, false>(a, row_waves, blocks, stream);
    }
    return hipGetLastError();
}

hipError_t prepare_attend_f32()                                    // (asking loads the code)
{
    hipFuncAttributes at;
    return hipFuncGetAttributes(&at, reinterpret_cast<const void*>(&attend_f32_kernel<float, 64, true>));
}

}  // namespace dyspec
