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
// What bounds it: the matrix pipe (32 cycles per 16x16x4; two products of 2 * 16 * keys * d).
#include "attend.h"

namespace dyspec {

typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kF32Waves = 4;

template <typename T, int DP>
__global__ __launch_bounds__(64 * kF32Waves) void attend_f32_kernel(AttendArgs, int row_waves)
{
    const AttendArgs& a = attend_args_here();
    typedef typename Four<T>::raw raw;
    constexpr int NS = DP / 16, NB = DP / 64;
    constexpr int KB = DP <= 128 ? 32 : 16, N16 = KB / 16;         // keys of a step
    __shared__ float merge_area[kF32Waves - 1][64 * (16 * NB + 2)];
    __shared__ int flag;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;
    const int R = 16 * row_waves, key_waves = kF32Waves / row_waves;
    const int wq = wave % row_waves, wk = wave / row_waves;
    const AttendItem it = attend_item(a, blockIdx.x, R);
    const AttendSeq& s = it.s;
    const int rows = a.G * s.N, r0 = it.block * R;
    const int r = r0 + 16 * wq + n, rc = min(r, rows - 1);
    const int j = div_G(a, rc), h = it.kvh * a.G + (rc - j * a.G);
    const int end = s.C + div_G(a, min(r0 + R, rows) - 1) + 1;     // keys that some row of the block may see
    const int n_parts = s.parts > 1 ? (end + s.share - 1) / s.share : 1;
    if (it.part >= n_parts) return;
    const int k_begin = s.parts > 1 ? it.part * s.share : 0, k_end = s.parts > 1 ? min(end, k_begin + s.share) : end;
    const int last = k_end - 1;
    const int size = (int)sizeof(T);
    const char* const kp = a.k + (long long)it.kvh * a.d * size;
    const char* const vp = a.v + (long long)it.kvh * a.d * size;

    // Q: dims 16s + 4g .. of query n; a piece past head_dim is zero here and in K
    float4 q[NS];
    const char* const qrow = a.q + (long long)(s.row0 + j) * a.q_stride + (long long)h * a.d * size;
#pragma unroll
    for (int x = 0; x < NS; ++x) {
        const int dim = 16 * x + 4 * g;
        q[x] = dim < a.d ? Four<T>::wide(*reinterpret_cast<const raw*>(qrow + dim * size)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    floatx4 acc[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[b][c] = floatx4{ 0.0f, 0.0f, 0.0f, 0.0f };
    float m = kLowest, l = 0.0f;

    // 16 keys from key16 on are two runs of eight rows, each within a page; rows past the last key repeat it
    auto runs = [&](int key16, long long stride, int (&first)[2], long long (&off)[2]) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            first[u] = min(key16 + 8 * u, last) & ~7;
            off[u] = key_offset(a, s, first[u], stride);
        }
    };
    auto load_k = [&](int key0, raw (&kr)[N16][NS]) {
#pragma unroll
        for (int b = 0; b < N16; ++b) {
            int first[2];
            long long off[2];
            runs(key0 + 16 * b, a.k_stride, first, off);
            const int key = min(key0 + 16 * b + n, last);
            const char* const row = kp + (n < 8 ? off[0] + (key - first[0]) * a.k_stride : off[1] + (key - first[1]) * a.k_stride);
#pragma unroll
            for (int x = 0; x < NS; ++x) {
                const int dim = 16 * x + 4 * g;
                kr[b][x] = *reinterpret_cast<const raw*>(row + (dim < a.d ? dim : 0) * size);
            }
        }
    };
    raw kr[N16][NS];
    int key0 = k_begin + KB * wk;
    if (key0 < k_end) load_k(key0, kr);
    for (; key0 < k_end; key0 += KB * key_waves) {
        // V: dims 64b + 4n .. of keys 4g + i
        raw vr[N16][4][NB];
#pragma unroll
        for (int b = 0; b < N16; ++b) {
            int first[2];
            long long off[2];
            runs(key0 + 16 * b, a.v_stride, first, off);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = min(key0 + 16 * b + 4 * g + i, last);
                const char* const row = vp + (g < 2 ? off[0] + (key - first[0]) * a.v_stride : off[1] + (key - first[1]) * a.v_stride);
#pragma unroll
                for (int x = 0; x < NB; ++x) {
                    const int dim = 64 * x + 4 * n;
                    vr[b][i][x] = *reinterpret_cast<const raw*>(row + (dim < a.d ? dim : 0) * size);
                }
            }
        }
        floatx4 S[N16];
#pragma unroll
        for (int b = 0; b < N16; ++b) {
            S[b] = floatx4{ 0.0f, 0.0f, 0.0f, 0.0f };
#pragma unroll
            for (int x = 0; x < NS; ++x) {
                float4 k = Four<T>::wide(kr[b][x]);
                if (DP > a.d && 16 * x + 4 * g >= a.d) k = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                S[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x, q[x].x, S[b], 0, 0, 0);
                S[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.y, q[x].y, S[b], 0, 0, 0);
                S[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.z, q[x].z, S[b], 0, 0, 0);
                S[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.w, q[x].w, S[b], 0, 0, 0);
            }
        }
        const int next = key0 + KB * key_waves;
        if (next < k_end) load_k(next, kr);
        // scores of keys a row does not see: -inf, whatever K holds there
        uint32_t seen = seen_bits(a, s, j, key0);
        if (k_end - key0 < KB) seen &= (1u << (k_end - key0)) - 1u;
        float up = m;
#pragma unroll
        for (int b = 0; b < N16; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!((seen >> (16 * b + 4 * g + i)) & 1u)) S[b][i] = -INFINITY;
                up = fmaxf(up, S[b][i]);
            }
        up = fmaxf(up, __shfl_xor(up, 16, kWave));
        up = fmaxf(up, __shfl_xor(up, 32, kWave));
        const float f = exp2f((m - up) * a.c2);
        m = up;
        l *= f;
        if (__any(f != 1.0f)) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[b][c] *= f;
        }
#pragma unroll
        for (int b = 0; b < N16; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = S[b][i] == -INFINITY ? 0.0f : exp2f((S[b][i] - m) * a.c2);
                l += p;
#pragma unroll
                for (int x = 0; x < NB; ++x) {
                    const float4 v = Four<T>::wide(vr[b][i][x]);
                    acc[x][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.x, p, acc[x][0], 0, 0, 0);
                    acc[x][1] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.y, p, acc[x][1], 0, 0, 0);
                    acc[x][2] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.z, p, acc[x][2], 0, 0, 0);
                    acc[x][3] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.w, p, acc[x][3], 0, 0, 0);
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
        uint64_t lanes = __builtin_amdgcn_ballot_w64(nan && r < rows);
        uint32_t bad = (uint32_t)((lanes | lanes >> 16 | lanes >> 32 | lanes >> 48) & 0xffffu);
        const bool leave = r < rows && !((bad >> n) & 1u);
        if (n_parts > 1) {
            if (g == 0 && r < rows) store_pair(slot_max_sum(a, slot, R, 16 * wq + n), m, l);
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
        leave_exact_rows<T, kSlotF32>(a, it, bad, 16 * wq, 0, a.d, R, k_begin, k_end, n_parts, slot,
                                   [=](int row) { return __shfl(m, row - 16 * wq, kWave); });
    }
    if (n_parts > 1 && arrive_last(a, it, n_parts, &flag)) merge_parts<T, kSlotF32, 0>(a, it, n_parts, R, 64 * kF32Waves);
}

template <typename T>
static void launch_f32(const AttendArgs& a, int row_waves, int blocks, hipStream_t stream)
{
    if (a.d <= 64) attend_f32_kernel<T, 64><<<blocks, 64 * kF32Waves, 0, stream>>>(a, row_waves);
    else if (a.d <= 128) attend_f32_kernel<T, 128><<<blocks, 64 * kF32Waves, 0, stream>>>(a, row_waves);
    else if (a.d <= 192) attend_f32_kernel<T, 192><<<blocks, 64 * kF32Waves, 0, stream>>>(a, row_waves);
    else attend_f32_kernel<T, 256><<<blocks, 64 * kF32Waves, 0, stream>>>(a, row_waves);
}

hipError_t launch_attend_f32(const AttendArgs& a, int dtype, int row_waves, int items, hipStream_t stream)
{
    if (dtype == DYSPEC_F32) launch_f32<float>(a, row_waves, items * a.Hkv, stream);
    else launch_f32<__bf16>(a, row_waves, items * a.Hkv, stream);
    return hipGetLastError();
}

}  // namespace dyspec
