// What the kernels of dyspec_paged_attn and dyspec_prompt_attn share: their arguments, which rows and keys a workgroup has, where
// a key lies, which keys a row sees, the merge of the parts of a long walk, the exact form of a row that met a NaN.
//
// Rows.  All G = Hq/Hkv query heads of a KV head are folded into the row dimension (row = token*G + head), so a block of rows
// streams K and V of its KV head once.  Keys are numbered from the start of the sequence: the context's, then the new tokens'.
//
// Row j of the new tokens sees every key of the context and, of the new ones, key i if i <= j and, under an ancestor mask, bit i
// of its mask row is set.
#pragma once
#include "dyspec_device.h"

namespace dyspec {

constexpr float kLowest = -3.402823466e38f;      // running maximum before the first key

// One sequence of a launch.  Its row blocks (of the kernel's R rows) times `parts` are consecutive items; a workgroup takes one
// item of one KV head.  Blocks come last row first: under a causal mask the long walks start first.
struct AttendSeq {
    int item0;        // first item
    int group0;       // first row block, counted over the launch
    int id;           // row of the page table
    int row0;         // first token in q, k, v, out, mask
    int N, C;         // new tokens, tokens before them
    int parts;        // items per row block
    int share;        // keys per part, a multiple of the kernel's step
};

struct AttendArgs {
    const char *q, *k, *v;
    char* out;
    const int* table;              // nullptr: k and v are rows of tokens like q
    const uint32_t* mask;          // nullptr: causal
    float* part;                   // [items * Hkv][R * (d + 2)]: rows times their weight, then (max, sum) per row
    unsigned* counters;            // [row blocks * Hkv], zero between launches
    long long q_stride, out_stride, k_stride, v_stride;      // bytes between tokens (in a page: between its rows)
    long long page_bytes;          // between pages
    int table_stride, page_shift, n_pages;
    int mask_words;                // 32-bit words per mask row
    int Hq, Hkv, G, d;
    uint32_t g_magic;              // r / G = hi(r * g_magic), G = 1: r
    float c2;                      // softmax scale * log2(e): weights are exp2(c2 * score)
    int n_seq;
    AttendSeq seq[DYSPEC_MAX_SEQ];
};

// A workgroup's place: block of rows, part of the walk.
struct AttendItem { AttendSeq s; int kvh, block, part; };

typedef __attribute__((address_space(4))) const int* scalar_ints;

__device__ __forceinline__ AttendItem attend_item(const AttendArgs& a, int index, int rows_per_block)
{
    AttendItem it;
    const int item = index / a.Hkv;
    it.kvh = index - item * a.Hkv;
    it.s = a.seq[0];
    if (a.n_seq > 1) {                                     // sequences that start at or before this item
        const int lane = threadIdx.x & 63;
        const int at = lane < a.n_seq ? a.seq[lane].item0 : 0x7fffffff;
        it.s = a.seq[__builtin_popcountll(__builtin_amdgcn_ballot_w64(item >= at)) - 1];
    }
    const int local = item - it.s.item0;
    const int blocks = (a.G * it.s.N + rows_per_block - 1) / rows_per_block;
    const int lb = it.s.parts > 1 ? local / it.s.parts : local;
    it.part = local - lb * it.s.parts;
    it.block = blocks - 1 - lb;
    return it;
}

__device__ __forceinline__ int div_G(const AttendArgs& a, int r) { return a.g_magic ? (int)__umulhi((uint32_t)r, a.g_magic) : r; }

// Byte offset of key `key` (uniform over the wave) from the pool's or the packed rows' start.  A page number outside the pool
// reads its last page: a wrong result, but no access outside the cache.
__device__ __forceinline__ long long key_offset(const AttendArgs& a, const AttendSeq& s, int key, long long stride)
{
    if (a.table) {
        const unsigned p = (unsigned)((scalar_ints)(a.table + (long long)s.id * a.table_stride))[key >> a.page_shift];
        return (long long)min(p, (unsigned)a.n_pages - 1u) * a.page_bytes + (long long)(key & ((1 << a.page_shift) - 1)) * stride;
    }
    return (long long)(s.row0 + key) * stride;
}

// Bit b: row j of the new tokens sees key k0 + b.
__device__ __forceinline__ uint32_t seen_bits(const AttendArgs& a, const AttendSeq& s, int j, int k0)
{
    const int upto = s.C + j + 1 - k0;                     // keys up to the row's own
    uint32_t w = upto >= 32 ? ~0u : upto <= 0 ? 0u : (1u << upto) - 1u;
    const int i0 = k0 - s.C;                               // key k0 + b is new token i0 + b
    if (a.mask && i0 > -32) {
        const uint32_t* const row = a.mask + (long long)(s.row0 + j) * a.mask_words;
        uint32_t m;
        if (i0 < 0) {
            m = (row[0] << -i0) | ((1u << -i0) - 1u);
        } else {
            const int q = i0 >> 5, r = i0 & 31;
            const uint32_t lo = q < a.mask_words ? row[q] : 0u, hi = q + 1 < a.mask_words ? row[q + 1] : 0u;
            m = __builtin_amdgcn_alignbit(hi, lo, r);
        }
        w &= m;
    }
    return w;
}

template <typename T> struct Four;
template <> struct Four<float> {
    typedef float4 raw;
    static __device__ __forceinline__ float4 wide(raw v) { return v; }
    static __device__ __forceinline__ void store(char* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
};
template <> struct Four<__bf16> {
    typedef uint2 raw;
    static __device__ __forceinline__ float4 wide(raw w)
    {
        return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
    }
    static __device__ __forceinline__ void store(char* p, float4 v)
    {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        const f2 lo = { v.x, v.y }, hi = { v.z, v.w };
        uint2 w;
        w.x = __builtin_bit_cast(uint32_t, __builtin_convertvector(lo, b2));
        w.y = __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, b2));
        *reinterpret_cast<uint2*>(p) = w;
    }
};

__device__ __forceinline__ char* out_row(const AttendArgs& a, const AttendSeq& s, int j, int h, int size)
{
    return a.out + (long long)(s.row0 + j) * a.out_stride + (long long)h * a.d * size;
}

// ---- a row that met a NaN
//
// A weight of a key that a row does not see is zero, but zero times an infinity or a NaN of that key's V row is a NaN in the
// matrix product.  Such keys may hold anything (a later token that overflowed), so a row that comes out with a NaN is done again
// by this: keys one at a time, those the row does not see left out.  One wave, lane i holds dims 4i..; a NaN of the row's own
// keys comes out as one again.
template <typename T>
__device__ __forceinline__ void exact_row(const AttendArgs& a, const AttendSeq& s, int kvh, int r, int k_begin, int k_end, float4& o, float& m, float& l)
{
    typedef typename Four<T>::raw raw;
    const int lane = threadIdx.x & 63;
    const bool mine = 4 * lane < a.d;
    const int piece = mine ? lane : 0;
    const int j = div_G(a, r), h = kvh * a.G + (r - j * a.G);
    const float zero = 0.0f;
    float4 q = Four<T>::wide(*reinterpret_cast<const raw*>(a.q + (long long)(s.row0 + j) * a.q_stride + ((long long)h * a.d + 4 * piece) * (int)sizeof(T)));
    o = make_float4(zero, zero, zero, zero);
    m = kLowest; l = 0.0f;
    const long long head = (long long)kvh * a.d * (int)sizeof(T);
#pragma unroll 1
    for (int key = k_begin; key < k_end; ++key) {
        if (!(__builtin_amdgcn_readfirstlane((int)seen_bits(a, s, j, key)) & 1)) continue;
        const float4 k = Four<T>::wide(*reinterpret_cast<const raw*>(a.k + key_offset(a, s, key, a.k_stride) + head + 4 * piece * (int)sizeof(T)));
        const float4 v = Four<T>::wide(*reinterpret_cast<const raw*>(a.v + key_offset(a, s, key, a.v_stride) + head + 4 * piece * (int)sizeof(T)));
        const float dot = wave_sum(mine ? (q.x * k.x + q.y * k.y) + (q.z * k.z + q.w * k.w) : 0.0f);
        const float up = fmaxf(m, dot);
        const float f = exp2f((m - up) * a.c2), p = exp2f((dot - up) * a.c2);
        m = up;
        l = l * f + p;
        o.x = o.x * f + p * v.x; o.y = o.y * f + p * v.y; o.z = o.z * f + p * v.z; o.w = o.w * f + p * v.w;
    }
}

// ---- parts
//
// A walk cut into parts: every workgroup leaves its rows (times their weight, fp32: nothing is rounded twice) with their (max,
// sum) in its slot and arrives at its row block's counter; the one that arrives last sums the slots in the order of the keys
// and writes the rows.  The counter wraps to zero with the last arrival.  Slots go through device-scope accesses: they reach the
// level of memory that all XCDs share without a write-back of whole caches.
__device__ __forceinline__ void store_pair(float* p, float x, float y)
{
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), ((unsigned long long)__float_as_uint(y) << 32) | __float_as_uint(x),
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_pair(const float* p)
{
    const unsigned long long w = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32)));
}
// The workgroup's slot; part z of the same row block has its own z - part places further.
__device__ __forceinline__ float* part_slot(const AttendArgs& a, int index, int rows_per_block)
{
    return a.part + (long long)index * rows_per_block * (a.d + 2);
}
// Called by all threads after their stores to the slot.  True in the workgroup that arrives last.
__device__ __forceinline__ bool arrive_last(const AttendArgs& a, const AttendItem& it, int n_parts, int* flag)
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");     // every store of the thread has been acknowledged
    __syncthreads();
    if (threadIdx.x == 0) {
        const unsigned before = __builtin_amdgcn_atomic_inc32(a.counters + (long long)(it.s.group0 + it.block) * a.Hkv + it.kvh, (unsigned)n_parts - 1u,
                                                              __ATOMIC_RELAXED, "agent");
        *flag = before == (unsigned)n_parts - 1u;
    }
    __syncthreads();
    return *flag != 0;
}
template <typename T>
__device__ __forceinline__ void merge_parts(const AttendArgs& a, const AttendItem& it, int index, int n_parts, int rows_per_block, int n_threads)
{
    const int r0 = it.block * rows_per_block, rows = min(rows_per_block, a.G * it.s.N - r0);
    const int pieces = a.d / 4;
    const float* const first = part_slot(a, index - it.part * a.Hkv, rows_per_block);
    const long long step = (long long)a.Hkv * rows_per_block * (a.d + 2);
    constexpr int kBatch = 4;                              // parts per trip to memory
    for (int x = threadIdx.x; x < rows * pieces; x += n_threads) {
        const int row = x / pieces, piece = x - row * pieces;
        float M = kLowest, L = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int z0 = 0; z0 < n_parts; z0 += kBatch) {
            float2 ml[kBatch], lo[kBatch], hi[kBatch];
#pragma unroll
            for (int z = 0; z < kBatch; ++z) {
                const float* const slot = first + min(z0 + z, n_parts - 1) * step;
                ml[z] = load_pair(slot + (long long)rows_per_block * a.d + 2 * row);
                lo[z] = load_pair(slot + (long long)row * a.d + 4 * piece);
                hi[z] = load_pair(slot + (long long)row * a.d + 4 * piece + 2);
            }
            float up = M;
#pragma unroll
            for (int z = 0; z < kBatch; ++z) up = fmaxf(up, ml[z].x);
            const float f = exp2f((M - up) * a.c2);
            M = up;
            L *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
#pragma unroll
            for (int z = 0; z < kBatch; ++z) {
                if (z0 + z >= n_parts || ml[z].y == 0.0f) continue;      // no key seen there
                const float w = exp2f((ml[z].x - M) * a.c2);
                L += w * ml[z].y;
                o.x += w * lo[z].x; o.y += w * lo[z].y; o.z += w * hi[z].x; o.w += w * hi[z].y;
            }
        }
        const float inv = L == 0.0f ? 0.0f : 1.0f / L;
        const int j = div_G(a, r0 + row), h = it.kvh * a.G + (r0 + row - j * a.G);
        Four<T>::store(out_row(a, it.s, j, h, sizeof(T)) + 4 * piece * (int)sizeof(T), make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    }
}

// ---- launches (one per source file); `a` without its sequences: those are picked and cut by the launcher's rule
struct AttendBatch { int n_seq; int row0[DYSPEC_MAX_SEQ + 1]; int context[DYSPEC_MAX_SEQ]; };
size_t attend_workspace_bytes(const AttendBatch& b, int dtype, int Hq, int Hkv, int d);
hipError_t launch_attend(AttendArgs a, const AttendBatch& b, int dtype, void* workspace, size_t workspace_bytes, hipStream_t stream);
hipError_t prepare_attend();

}  // namespace dyspec
