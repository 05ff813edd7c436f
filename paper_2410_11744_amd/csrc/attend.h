// What the kernels of dyspec_paged_attn and dyspec_prompt_attn share: their arguments, which rows and keys a workgroup has, where
// a key lies, which keys a row sees, the merge of the parts of a long walk, the second look at rows that met a NaN.
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

// One sequence of a launch, or some row blocks of one.  Its row blocks (of the kernel's R rows) times `parts` are consecutive items;
// a workgroup takes one item of one KV head.  Blocks come last row first: under a causal mask the long walks start first.
struct AttendSeq {
    int item0;        // first item
    int end_block;    // the first item's row block is the one before this
    int group0;       // the sequence's first row block, counted over the launch
    int id;           // row of the page table
    int row0;         // first token in q, k, v, out, mask
    int N, C;         // new tokens, tokens before them
    int parts;        // items per row block
    int share;        // keys per part, a multiple of the kernel's step
    int slot0;        // parts > 1: first item's place among the slots
};

struct AttendArgs {
    const char *q, *k, *v;
    char* out;
    const int* table;              // nullptr: k and v are rows of tokens like q
    const uint32_t* mask;          // nullptr: causal
    float* part;                   // [slots * Hkv][R * (d + 2)]: rows times their weight, then (max, sum) per row
    unsigned* counters;            // [row blocks * Hkv], zero between launches
    long long q_stride, out_stride, k_stride, v_stride;      // bytes between tokens (in a page: between its rows)
    long long page_bytes;          // between pages
    int table_stride, page_shift, n_pages;
    int mask_words;                // 32-bit words per mask row
    int Hq, Hkv, G, d;
    uint32_t g_magic;              // r / G = hi(r * g_magic), G = 1: r
    float c2;                      // softmax scale * log2(e): weights are exp2(c2 * score)
    int n_seq;                     // entries of the table
    AttendSeq seq[DYSPEC_MAX_SEQ];
};

// The arguments where they are: read from the kernel's argument segment, whose first parameter they have to be.  (Taken as a
// by-value parameter, the table of sequences, indexed at run time, would be copied to scratch memory by every lane.)
__device__ __forceinline__ const AttendArgs& attend_args_here()
{
    return *(const AttendArgs*)(__attribute__((address_space(4))) const AttendArgs*)__builtin_amdgcn_kernarg_segment_ptr();
}

// A workgroup's place: block of rows, part of the walk.
struct AttendItem { AttendSeq s; int kvh, block, part, local; };      // local: the item's number in its entry

typedef __attribute__((address_space(4))) const int* scalar_ints;

__device__ __forceinline__ AttendItem attend_item(const AttendArgs& a, int index)
{
    AttendItem it;
    const int item = index / a.Hkv;
    it.kvh = index - item * a.Hkv;
    it.s = a.seq[0];
    if (a.n_seq > 1) {                                     // entries that start at or before this item
        const int lane = threadIdx.x & 63;
        const int at = lane < a.n_seq ? a.seq[lane].item0 : 0x7fffffff;
        it.s = a.seq[__builtin_popcountll(__builtin_amdgcn_ballot_w64(item >= at)) - 1];
    }
    const int local = item - it.s.item0;
    it.local = local;
    const int lb = it.s.parts > 1 ? local / it.s.parts : local;
    it.part = local - lb * it.s.parts;
    it.block = it.s.end_block - 1 - lb;
    return it;
}

__device__ __forceinline__ int div_G(const AttendArgs& a, int r) { return a.g_magic ? (int)__umulhi((uint32_t)r, a.g_magic) : r; }

// Byte offset of key `key` (uniform over the wave) from the pool's or the packed rows' start.  A page number outside the pool
// reads its last page: a wrong result, but no access outside the cache.
template <bool Paged>
__device__ __forceinline__ long long key_offset(const AttendArgs& a, const AttendSeq& s, int key, long long stride)
{
    if constexpr (Paged) {
        const unsigned p = (unsigned)((scalar_ints)(a.table + (long long)s.id * a.table_stride))[key >> a.page_shift];
        return (long long)min(p, (unsigned)a.n_pages - 1u) * a.page_bytes + (long long)(key & ((1 << a.page_shift) - 1)) * stride;
    }
    return (long long)(s.row0 + key) * stride;
}
__device__ __forceinline__ long long key_offset(const AttendArgs& a, const AttendSeq& s, int key, long long stride)
{
    return a.table ? key_offset<true>(a, s, key, stride) : key_offset<false>(a, s, key, stride);
}

// 32-bit word q of row j's mask, numbered from the first new token; words before it are the context's, which every row sees.
__device__ __forceinline__ uint32_t mask_word(const AttendArgs& a, const AttendSeq& s, int j, int q)
{
    return q < 0 ? ~0u : q < a.mask_words ? a.mask[(long long)(s.row0 + j) * a.mask_words + q] : 0u;
}
// Bit b: key k0 + b is not behind row j's own.
__device__ __forceinline__ uint32_t causal_bits(const AttendSeq& s, int j, int k0)
{
    const int upto = s.C + j + 1 - k0;
    return upto >= 32 ? ~0u : upto <= 0 ? 0u : (1u << upto) - 1u;
}
// Bit b: row j of the new tokens sees key k0 + b.
__device__ __forceinline__ uint32_t seen_bits(const AttendArgs& a, const AttendSeq& s, int j, int k0)
{
    uint32_t w = causal_bits(s, j, k0);
    if (a.mask) {
        const int i0 = k0 - s.C;                           // key k0 + b is new token i0 + b
        w &= __builtin_amdgcn_alignbit(mask_word(a, s, j, (i0 >> 5) + 1), mask_word(a, s, j, i0 >> 5), (uint32_t)i0 & 31u);
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

// ---- parts
//
// A walk cut into parts: every workgroup leaves its rows (times their weight, fp32: nothing is rounded twice) with their (max,
// sum) in its slot and arrives at its row block's counter; the one that arrives last sums the slots in the order of the keys
// and writes the rows.  The counter wraps to zero with the last arrival.  Slots go through device-scope accesses: they reach the
// level of memory that all XCDs share without a write-back of whole caches.  A slot holds the rows in the order in which the
// kernel's lanes have them, four dims to a lane, so that each store of a wave is one run of a kilobyte.
__device__ __forceinline__ void store_four(float* p, float x, float y, float z, float w)
{
    typedef float f4 __attribute__((ext_vector_type(4)));
    const f4 v = { x, y, z, w };
    // (arrive_last waits for it; the wait states keep the next instruction from overwriting the data while they are read)
    asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 3" :: "v"(p), "v"(v) : "memory");
}
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
// Lane orders: blocks of 32 rows as O^T lies in 32x32 accumulators (attend_mfma.hip); row after row, eight dims to a lane
// (attend_short.hip); blocks of 16 rows as in 16x16 accumulators, head_dim padded to 64s (attend_f32.hip).
enum SlotOrder { kSlotMany, kSlotFew, kSlotF32 };
constexpr __host__ __device__ int slot_dims(int d) { return (d + 63) / 64 * 64; }
constexpr __host__ __device__ int slot_floats(int d, int rows_per_block) { return rows_per_block * (slot_dims(d) + 2); }
// floats from the slot's start to dims 4 * piece .. of row `row`
template <SlotOrder O> __device__ __forceinline__ int slot_place(int d, int row, int piece)
{
    if constexpr (O == kSlotMany) return ((row >> 5) * (d / 8) + (piece >> 1)) * 256 + 4 * ((row & 31) + 32 * (piece & 1));
    if constexpr (O == kSlotFew) { const int t = row * (d / 8) + (piece >> 1); return (t >> 6) * 512 + (piece & 1) * 256 + 4 * (t & 63); }
    return ((row >> 4) * (slot_dims(d) / 16) + (piece >> 4) * 4 + (piece & 3)) * 256 + 4 * ((row & 15) + 16 * ((piece >> 2) & 3));
}
// ... and back: what lies at floats 4 * x ..
template <SlotOrder O> __device__ __forceinline__ void slot_piece(int d, int x, int& row, int& piece)
{
    const int lane = x & 63, y = x >> 6;
    if constexpr (O == kSlotMany) { const int b = y / (d / 8); row = 32 * b + (lane & 31); piece = 2 * (y - b * (d / 8)) + (lane >> 5); }
    else if constexpr (O == kSlotFew) { const int t = (y >> 1) * 64 + lane; row = t / (d / 8); piece = 2 * (t - row * (d / 8)) + (y & 1); }
    else { const int nb = slot_dims(d) / 64, b = (y >> 2) / nb; row = 16 * b + (lane & 15); piece = 16 * ((y >> 2) - b * nb) + 4 * (lane >> 4) + (y & 3); }
}
__device__ __forceinline__ float* slot_max_sum(const AttendArgs& a, float* slot, int rows_per_block, int row)
{
    return slot + rows_per_block * slot_dims(a.d) + 2 * row;
}
// The workgroup's slot; part z of the same row block has its own Hkv * (z - part) places further.
__device__ __forceinline__ float* part_slot(const AttendArgs& a, const AttendItem& it, int rows_per_block)
{
    return a.part + ((long long)(it.s.slot0 + it.local) * a.Hkv + it.kvh) * slot_floats(a.d, rows_per_block);
}
// Called by all threads after their stores to the slot.  True in the workgroup that arrives last.
__device__ __forceinline__ bool arrive_last(const AttendArgs& a, const AttendItem& it, int n_parts, int* flag)
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // every store of the wave has been acknowledged
    __syncthreads();
    if (threadIdx.x == 0) {
        const unsigned before = __builtin_amdgcn_atomic_inc32(a.counters + (long long)(it.s.group0 + it.block) * a.Hkv + it.kvh, (unsigned)n_parts - 1u,
                                                              __ATOMIC_RELAXED, "agent");
        *flag = before == (unsigned)n_parts - 1u;
    }
    __syncthreads();
    return *flag != 0;
}
// (D: head_dim where the kernel knows it, or 0)
template <typename T, SlotOrder O, int D>
__device__ __forceinline__ void merge_parts(const AttendArgs& a, const AttendItem& it, int n_parts, int rows_per_block, int n_threads)
{
    const int d = D ? D : a.d;
    const int r0 = it.block * rows_per_block, rows = min(rows_per_block, a.G * it.s.N - r0);
    const long long step = (long long)a.Hkv * slot_floats(d, rows_per_block);
    float* const first = part_slot(a, it, rows_per_block) - it.part * step;
    constexpr int kBatch = 4;                              // parts per trip to memory
    for (int x = threadIdx.x; x < rows_per_block * slot_dims(d) / 4; x += n_threads) {
        int row, piece;
        slot_piece<O>(d, x, row, piece);
        if (row >= rows || 4 * piece >= d) continue;
        const float* const at = first + 4 * x;
        const float* const ml_at = slot_max_sum(a, first, rows_per_block, row);
        float M = kLowest, L = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int z0 = 0; z0 < n_parts; z0 += kBatch) {
            float2 ml[kBatch], lo[kBatch], hi[kBatch];
#pragma unroll
            for (int z = 0; z < kBatch; ++z) {
                const long long off = min(z0 + z, n_parts - 1) * step;
                ml[z] = load_pair(ml_at + off);
                lo[z] = load_pair(at + off);
                hi[z] = load_pair(at + off + 2);
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

// ---- a row that met a NaN
//
// A weight of a key that a row does not see is zero, but zero times an infinity or a NaN of that key's V row is a NaN in the
// matrix product.  Such keys may hold anything (a later token that overflowed), so rows that come out with a NaN are looked at
// again: if what their block took at a weight of zero was all finite, the NaN is the row's own and stays.

// Whether V of the walk's keys that meet a weight of zero is finite: of those that some row of the block may not see, and of the last
// one, if it may be repeated to fill a block of (up to 64) keys.  One wave, lane i reads dims 4i..
template <typename T>
__device__ __forceinline__ bool hidden_are_finite(const AttendArgs& a, const AttendSeq& s, int kvh, int r0, int k_begin, int k_end)
{
    typedef typename Four<T>::raw raw;
    const int size = (int)sizeof(T), lane = threadIdx.x & 63, piece = 4 * lane < a.d ? lane : 0;
    float4 z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);            // stays zero unless something is infinite or a NaN
    auto add = [&](float4 x) { z.x = fmaf(x.x, 0.0f, z.x); z.y = fmaf(x.y, 0.0f, z.y); z.z = fmaf(x.z, 0.0f, z.z); z.w = fmaf(x.w, 0.0f, z.w); };
    const long long head = (long long)kvh * a.d * size + 4 * piece * size;
    const int hidden = max(k_begin, a.mask ? s.C : s.C + div_G(a, r0) + 1), repeated = (k_end - k_begin) % 64 ? k_end - 1 : k_end;
#pragma unroll 4
    for (int key = min(hidden, repeated); key < k_end; ++key)
        add(Four<T>::wide(*reinterpret_cast<const raw*>(a.v + key_offset(a, s, key, a.v_stride) + head)));
    return !__any((z.x + z.y) + (z.z + z.w) != 0.0f);          // (a NaN is not equal)
}

// The rows `bad` (bit b: row row0 + b of the block) came out with a NaN, and have left, into their slot or finished: where that may be
// another row's matter, their dims dim0 .. dim1 - 1 are done again, 16 rows at a time, without what they do not see, and leave again.
// m_of(row): the reference that the row's (max, sum) go by.  One wave.
//
// The fp32 matrix instructions from registers alone, as in attend_f32.hip (where the layouts are explained): a lane has one query and
// four keys of every 16 of the scores, dims 64y + 16g + 4i + c of one query of the sums.  The second product takes zeros in place of V's
// infinities and NaN; a key that has some is added by itself, to the rows that see it.  So a hidden token that overflowed costs one
// such walk of the rows beside it: a prompt of 8192 tokens, 64 heads on 8, with a NaN in one value takes up to 2.9 ms in place of 1.0,
// a tree of 512 rows over 4096 tokens 2.0 in place of 0.09 (row by row and key by key it was 98, and 60).
template <typename T, SlotOrder O, int DP, typename F>
__device__ __forceinline__ void look_again(uint32_t bad, int row0, int dim0, int dim1, int rows_per_block, F m_of)
{
    // all of the call is looked up anew: nothing is held for this through the walk
    auto args = (__attribute__((address_space(4))) const AttendArgs*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    const AttendArgs& a = *(const AttendArgs*)args;
    const AttendItem it = attend_item(a, blockIdx.x);
    const int block_end = min((it.block + 1) * rows_per_block, a.G * it.s.N), end = it.s.C + div_G(a, block_end - 1) + 1;
    const int n_parts = it.s.parts > 1 ? (end + it.s.share - 1) / it.s.share : 1;
    const int k_begin = n_parts > 1 ? it.part * it.s.share : 0, k_end = n_parts > 1 ? min(end, k_begin + it.s.share) : end;
    if (hidden_are_finite<T>(a, it.s, it.kvh, it.block * rows_per_block, k_begin, k_end)) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");               // (the rows as they were have left before they leave again)
    float* const slot = part_slot(a, it, rows_per_block);
    typedef typename Four<T>::raw raw;
    typedef float f4 __attribute__((ext_vector_type(4)));
    constexpr int size = (int)sizeof(T), NS = DP / 16, NB = DP / 64;
    const AttendSeq& s = it.s;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int d = a.d, r0 = it.block * rows_per_block, last = k_end - 1;
    const char* const kp = a.k + (long long)it.kvh * d * size;
    const char* const vp = a.v + (long long)it.kvh * d * size;
#pragma unroll 1
    for (int first = 0; first < 32; first += 16) {
        const uint32_t some = (bad >> first) & 0xffffu;
        if (some == 0u) continue;
        const int row = min(row0 + first + n, rows_per_block - 1), r = min(r0 + row, a.G * s.N - 1);
        const int j = div_G(a, r), h = it.kvh * a.G + (r - j * a.G);
        const bool wanted = (some >> n) & 1u;
        const float m = m_of(row);
        raw q[NS];                                                 // (a piece past head_dim meets zeros of K)
        const char* const qrow = a.q + (long long)(s.row0 + j) * a.q_stride + (long long)h * d * size;
#pragma unroll
        for (int x = 0; x < NS; ++x) {
            const int dim = 16 * x + 4 * g;
            q[x] = dim < d ? *reinterpret_cast<const raw*>(qrow + dim * size) : raw{};
        }
        f4 acc[NB][4];
#pragma unroll
        for (int y = 0; y < NB; ++y)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[y][c] = f4{ 0.0f, 0.0f, 0.0f, 0.0f };
        float l = 0.0f;
        bool done = false;                                         // every row is a NaN in all its dims: nothing else comes of it
#pragma unroll 1
        for (int key0 = k_begin; key0 < k_end && !done; key0 += 16) {
            // the step's two runs of eight keys, each within a page; keys past the last repeat it
            const int at0 = min(key0, last), at1 = min(key0 + 8, last) & ~7;
            auto row_of = [&](const char* base, long long stride, int off, bool low) __attribute__((always_inline)) -> const char* {
                const long long b0 = key_offset(a, s, at0, stride), b1 = key_offset(a, s, at1, stride);
                return base + (low ? b0 : b1) + (min(key0 + off, last) - (low ? at0 : at1)) * stride;
            };
            const char* const krow = row_of(kp, a.k_stride, n, n < 8);
            raw k[NS], v[4][NB];                                   // V: dims 64y + 4n .. of key 4g + x
#pragma unroll
            for (int x = 0; x < NS; ++x) {
                const int dim = 16 * x + 4 * g;
                k[x] = *reinterpret_cast<const raw*>(krow + (dim < d ? dim : 0) * size);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const char* const at = row_of(vp, a.v_stride, 4 * g + x, g < 2);
#pragma unroll
                for (int y = 0; y < NB; ++y) {
                    const int dim = 64 * y + 4 * n;
                    v[x][y] = *reinterpret_cast<const raw*>(at + (dim < d ? dim : 0) * size);
                }
            }
            uint32_t seen = seen_bits(a, s, j, key0) & 0xffffu;
            if (k_end - key0 < 16) seen &= (1u << (k_end - key0)) - 1u;
            f4 S = { 0.0f, 0.0f, 0.0f, 0.0f };
#pragma unroll
            for (int x = 0; x < NS; ++x) {
                float4 w = Four<T>::wide(k[x]);
                const float4 u = Four<T>::wide(q[x]);
                if (16 * x + 16 > d && 16 * x + 4 * g >= d) w = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                S = __builtin_amdgcn_mfma_f32_16x16x4f32(w.x, u.x, S, 0, 0, 0);
                S = __builtin_amdgcn_mfma_f32_16x16x4f32(w.y, u.y, S, 0, 0, 0);
                S = __builtin_amdgcn_mfma_f32_16x16x4f32(w.z, u.z, S, 0, 0, 0);
                S = __builtin_amdgcn_mfma_f32_16x16x4f32(w.w, u.w, S, 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            f4 p;
            uint32_t odd = 0u;                                     // bit x: V of the lane's key x has something infinite or a NaN
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                p[x] = (seen >> (4 * g + x)) & 1u ? exp2f((S[x] - m) * a.c2) : 0.0f;
                l += p[x];
#pragma unroll
                for (int y = 0; y < NB; ++y) {
                    float4 w = Four<T>::wide(v[x][y]);
                    auto finite = [&](float& e) __attribute__((always_inline)) {
                        const bool fine = e * 0.0f == 0.0f;
                        if (!fine) odd |= 1u << x;
                        e = fine ? e : 0.0f;
                    };
                    finite(w.x); finite(w.y); finite(w.z); finite(w.w);
                    acc[y][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(w.x, p[x], acc[y][0], 0, 0, 0);
                    acc[y][1] = __builtin_amdgcn_mfma_f32_16x16x4f32(w.y, p[x], acc[y][1], 0, 0, 0);
                    acc[y][2] = __builtin_amdgcn_mfma_f32_16x16x4f32(w.z, p[x], acc[y][2], 0, 0, 0);
                    acc[y][3] = __builtin_amdgcn_mfma_f32_16x16x4f32(w.w, p[x], acc[y][3], 0, 0, 0);
                }
            }
            if (!__any(odd != 0u)) continue;
#pragma unroll 1
            for (int off = 0; off < 16 && key0 + off < k_end; ++off) {         // key 4 (off / 4) + off % 4
                const uint64_t lanes = __builtin_amdgcn_ballot_w64((odd >> (off & 3)) & 1u);
                if (!((lanes >> (16 * (off >> 2))) & 0xffffull)) continue;
                const float mine = (off & 2) ? (off & 1 ? p[3] : p[2]) : (off & 1 ? p[1] : p[0]);
                const float w0 = __shfl(mine, n + 16 * (off >> 2), kWave);     // the query's weight of it
                if (!((seen >> off) & 1u)) continue;
                const char* const at = vp + key_offset(a, s, key0 + off, a.v_stride);
#pragma unroll
                for (int y = 0; y < NB; ++y)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int dim = 64 * y + 16 * g + 4 * i;
                        const float4 w = Four<T>::wide(*reinterpret_cast<const raw*>(at + (dim < d ? dim : 0) * size));
                        acc[y][0][i] += w.x * 0.0f == 0.0f ? 0.0f : w0 * w.x;
                        acc[y][1][i] += w.y * 0.0f == 0.0f ? 0.0f : w0 * w.y;
                        acc[y][2][i] += w.z * 0.0f == 0.0f ? 0.0f : w0 * w.z;
                        acc[y][3][i] += w.w * 0.0f == 0.0f ? 0.0f : w0 * w.w;
                        __builtin_amdgcn_sched_barrier(0);         // (rare: not worth registers)
                    }
            }
            bool all = true;
#pragma unroll
            for (int y = 0; y < NB; ++y)
#pragma unroll
                for (int i = 0; i < 16; ++i) all &= acc[y][i / 4][i % 4] != acc[y][i / 4][i % 4];
            done = __all(all || !wanted);
        }
        l += __shfl_xor(l, 16, kWave);
        l += __shfl_xor(l, 32, kWave);
        if (!wanted) continue;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int y = 0; y < NB; ++y)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int dim = 64 * y + 16 * g + 4 * i;
                if (dim < dim0 || dim >= dim1) continue;
                if (n_parts > 1) store_four(slot + slot_place<O>(d, row, dim / 4), acc[y][0][i], acc[y][1][i], acc[y][2][i], acc[y][3][i]);
                else Four<T>::store(out_row(a, s, j, h, size) + dim * size, make_float4(acc[y][0][i] * inv, acc[y][1][i] * inv, acc[y][2][i] * inv, acc[y][3][i] * inv));
            }
    }
}

// ---- launches
struct AttendBatch { int n_seq; int row0[DYSPEC_MAX_SEQ + 1]; int context[DYSPEC_MAX_SEQ]; };
size_t attend_workspace_bytes(const AttendBatch& b, int dtype, int Hq, int Hkv, int d);
// `a` without its sequences, which are dealt to the kernels and cut into items (attend.hip), or, with a form (tests), all given to
// one kernel (0 .. 5: few rows, 8 and 4 waves; many rows, 8 and 4 waves; fp32, blocks of 16 and 64 rows), walks cut into shares of
// that many keys (0: not) but for those of the first `whole` row blocks; hipErrorInvalidValue where there is no such form
struct AttendForm { int kernel, share, whole; };
hipError_t launch_attend(AttendArgs a, const AttendBatch& b, int dtype, const AttendForm* form, void* workspace, size_t workspace_bytes, hipStream_t stream);
hipError_t prepare_attend();

// the kernels, on `items` items of a's sequences
constexpr int kManyRows = 128, kFewRows = 32;                      // rows of a block: attend_mfma.hip, attend_short.hip
hipError_t launch_attend_f32(const AttendArgs& a, int dtype, int row_waves, int items, hipStream_t stream);      // blocks of 16 * row_waves rows
hipError_t launch_attend_mfma(const AttendArgs& a, int waves, int items, hipStream_t stream);
hipError_t launch_attend_short(const AttendArgs& a, int waves, int most_new, int items, hipStream_t stream);
hipError_t prepare_attend_mfma();
hipError_t prepare_attend_short();
hipError_t prepare_attend_f32();

}  // namespace dyspec
