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
__global__ __launch_bounds__(64 * kF32Waves) void attend_f32_kernel(AttendArgs a, int row_waves)
{
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
    const int index = blockIdx.x;
    const AttendItem it = attend_item(a, index, R);
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
    float* const slot = part_slot(a, index, R);
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
            if (leave) {
                float* const dst = slot + (16 * wq + n) * a.d;
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int dim = 64 * b + 16 * g + 4 * i;
                        if (dim < a.d) {
                            store_pair(dst + dim, acc[b][0][i], acc[b][1][i]);
                            store_pair(dst + dim + 2, acc[b][2][i], acc[b][3][i]);
                        }
                    }
                if (g == 0) store_pair(slot + R * a.d + 2 * (16 * wq + n), m, l);
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
        while (bad) {
            const int row = 16 * wq + __builtin_ctz(bad);
            bad &= bad - 1u;
            float4 o;
            float em, el;
            exact_row<T>(a, s, it.kvh, r0 + row, k_begin, k_end, o, em, el);
            if (n_parts > 1) {
                if (4 * lane < a.d) {
                    store_pair(slot + row * a.d + 4 * lane, o.x, o.y);
                    store_pair(slot + row * a.d + 4 * lane + 2, o.z, o.w);
                }
                if (lane == 0) store_pair(slot + R * a.d + 2 * row, em, el);
            } else if (4 * lane < a.d) {
                const float inv = el == 0.0f ? 0.0f : 1.0f / el;
                const int bj = div_G(a, r0 + row);
                Four<T>::store(out_row(a, s, bj, it.kvh * a.G + (r0 + row - bj * a.G), size) + 4 * lane * size, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
            }
        }
    }
    if (n_parts > 1 && arrive_last(a, it, n_parts, &flag)) merge_parts<T>(a, it, index, n_parts, R, 64 * kF32Waves);
}

// ---- how a batch is cut
//
// A row block is one workgroup's as long as the blocks fill the chip; otherwise the walks are cut into shares of one length until
// there are about two workgroups per CU, no share below 128 keys (four steps of a wave).
constexpr int kF32Items = 512, kF32Share = 128;

struct F32Cut { int row_waves, items, groups; bool split; };

static F32Cut cut_f32(const AttendBatch& b, AttendArgs& a)
{
    F32Cut c;
    int most = 0;
    for (int s = 0; s < b.n_seq; ++s) most = max(most, b.row0[s + 1] - b.row0[s]);
    c.row_waves = (long long)most * a.G <= 16 ? 1 : kF32Waves;
    const int R = 16 * c.row_waves;
    long long blocks = 0, keys = 0;
    for (int s = 0; s < b.n_seq; ++s) {
        const long long nb = ((long long)(b.row0[s + 1] - b.row0[s]) * a.G + R - 1) / R;
        blocks += nb;
        keys += nb * (b.context[s] + b.row0[s + 1] - b.row0[s]);
    }
    c.split = blocks * a.Hkv < kF32Items / 2 && blocks * a.Hkv * (long long)sizeof(unsigned) <= DYSPEC_PAGED_COUNTER_BYTES;
    long long share = max(keys * a.Hkv / kF32Items, (long long)kF32Share);
    share = (share + kF32Share - 1) / kF32Share * kF32Share;
    a.n_seq = 0;
    c.items = c.groups = 0;
    // longest first
    int order[DYSPEC_MAX_SEQ], n = 0;
    for (int s = 0; s < b.n_seq; ++s)
        if (b.row0[s + 1] > b.row0[s]) {
            int at = n++;
            for (; at > 0 && b.context[order[at - 1]] < b.context[s]; --at) order[at] = order[at - 1];
            order[at] = s;
        }
    for (int x = 0; x < n; ++x) {
        const int s = order[x];
        AttendSeq& q = a.seq[a.n_seq++];
        q.id = s; q.row0 = b.row0[s]; q.N = b.row0[s + 1] - b.row0[s]; q.C = b.context[s];
        q.item0 = c.items; q.group0 = c.groups;
        const int nb = (int)(((long long)q.N * a.G + R - 1) / R);
        q.parts = c.split ? (int)((q.C + q.N + share - 1) / share) : 1;
        q.share = (int)share;
        c.items += nb * q.parts;
        c.groups += nb;
    }
    c.split = c.items > c.groups;
    return c;
}

template <typename T>
static void launch_f32(const AttendArgs& a, const F32Cut& c, hipStream_t stream)
{
    const int blocks = c.items * a.Hkv;
    if (a.d <= 64) attend_f32_kernel<T, 64><<<blocks, 64 * kF32Waves, 0, stream>>>(a, c.row_waves);
    else if (a.d <= 128) attend_f32_kernel<T, 128><<<blocks, 64 * kF32Waves, 0, stream>>>(a, c.row_waves);
    else if (a.d <= 192) attend_f32_kernel<T, 192><<<blocks, 64 * kF32Waves, 0, stream>>>(a, c.row_waves);
    else attend_f32_kernel<T, 256><<<blocks, 64 * kF32Waves, 0, stream>>>(a, c.row_waves);
}

static size_t part_bytes(const AttendArgs& a, const F32Cut& c)
{
    return c.split ? DYSPEC_PAGED_COUNTER_BYTES + (size_t)c.items * a.Hkv * 16 * c.row_waves * (a.d + 2) * sizeof(float) : 0;
}

size_t attend_workspace_bytes(const AttendBatch& b, int, int Hq, int Hkv, int d)
{
    AttendArgs a;
    a.Hq = Hq; a.Hkv = Hkv; a.G = Hq / Hkv; a.d = d;
    return part_bytes(a, cut_f32(b, a));
}

hipError_t launch_attend(AttendArgs a, const AttendBatch& b, int dtype, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    F32Cut c = cut_f32(b, a);
    if (c.split && (!workspace || workspace_bytes < part_bytes(a, c))) {      // no room: one workgroup walks it all
        c.items = 0;
        for (int s = 0; s < a.n_seq; ++s) {
            AttendSeq& q = a.seq[s];
            q.parts = 1; q.item0 = c.items;
            c.items += (int)(((long long)q.N * a.G + 16 * c.row_waves - 1) / (16 * c.row_waves));
        }
        c.split = false;
    }
    if (c.items == 0) return hipSuccess;
    a.counters = static_cast<unsigned*>(workspace);
    a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + DYSPEC_PAGED_COUNTER_BYTES);
    if (dtype == DYSPEC_F32) launch_f32<float>(a, c, stream);
    else launch_f32<__bf16>(a, c, stream);
    return hipGetLastError();
}

hipError_t prepare_attend() { return hipSuccess; }

}  // namespace dyspec
