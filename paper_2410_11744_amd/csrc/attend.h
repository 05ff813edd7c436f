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

// ---- a row that met a NaN
//
// A weight of a key that a row does not see is zero, but zero times an infinity or a NaN of that key's V row is a NaN in the
// matrix product.  Such keys may hold anything (a later token that overflowed), so rows that come out with a NaN are looked at
// again: if what their block took at a weight of zero was all finite, the NaN is the row's own and stays.
// (Otherwise a NaN at the start of a long context would send every row through the walk below, a thousand times slower.)

// Whether the block's query rows (which lie where a V tile would be, at weights of zero, when a walk starts) and V of the walk's keys
// that meet a weight of zero are finite: those that some row of the block may not see, and the last one, which is repeated behind the
// end of a block of keys.  One wave, lane i reads dims 4i..
template <typename T>
__device__ __forceinline__ bool hidden_are_finite(const AttendArgs& a, const AttendSeq& s, int kvh, int r0, int r1, int k_begin, int k_end)
{
    typedef typename Four<T>::raw raw;
    const int size = (int)sizeof(T), lane = threadIdx.x & 63, piece = 4 * lane < a.d ? lane : 0;
    float4 z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);            // stays zero unless something is infinite or a NaN
    auto add = [&](float4 x) { z.x = fmaf(x.x, 0.0f, z.x); z.y = fmaf(x.y, 0.0f, z.y); z.z = fmaf(x.z, 0.0f, z.z); z.w = fmaf(x.w, 0.0f, z.w); };
#pragma unroll 4
    for (int r = r0; r < r1; ++r) {
        const int j = div_G(a, r), h = kvh * a.G + (r - j * a.G);
        add(Four<T>::wide(*reinterpret_cast<const raw*>(a.q + (long long)(s.row0 + j) * a.q_stride + ((long long)h * a.d + 4 * piece) * size)));
    }
    const long long head = (long long)kvh * a.d * size + 4 * piece * size;
#pragma unroll 4
    for (int key = max(k_begin, min(a.mask ? s.C : s.C + div_G(a, r0) + 1, k_end - 1)); key < k_end; ++key)
        add(Four<T>::wide(*reinterpret_cast<const raw*>(a.v + key_offset(a, s, key, a.v_stride) + head)));
    return !__any((z.x + z.y) + (z.z + z.w) != 0.0f);          // (a NaN is not equal)
}

// The row again: keys one at a time, those it does not see left out, weights against the reference m that the row has.  One wave,
// lane i holds dims 4i..; a NaN of the row's own keys comes out as one again (and ends the walk where it is in all dims).
template <typename T>
__device__ __forceinline__ void exact_row(const AttendArgs& a, const AttendSeq& s, int kvh, int r, int k_begin, int k_end, float m, float4& o, float& l)
{
    typedef typename Four<T>::raw raw;
    const int lane = threadIdx.x & 63;
    const bool mine = 4 * lane < a.d;
    const int piece = mine ? lane : 0;
    const int j = div_G(a, r), h = kvh * a.G + (r - j * a.G);
    const float4 q = Four<T>::wide(*reinterpret_cast<const raw*>(a.q + (long long)(s.row0 + j) * a.q_stride + ((long long)h * a.d + 4 * piece) * (int)sizeof(T)));
    o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    l = 0.0f;
    const long long head = (long long)kvh * a.d * (int)sizeof(T) + 4 * piece * (int)sizeof(T);
    constexpr int kBatch = 4;                                  // keys per trip to memory
#pragma unroll 1
    for (int key = k_begin; key < k_end; key += kBatch) {
        const uint32_t seen = (uint32_t)__builtin_amdgcn_readfirstlane((int)seen_bits(a, s, j, key));
        float4 k[kBatch], v[kBatch];
#pragma unroll
        for (int x = 0; x < kBatch; ++x) {
            const int at = min(key + x, k_end - 1);
            k[x] = Four<T>::wide(*reinterpret_cast<const raw*>(a.k + key_offset(a, s, at, a.k_stride) + head));
            v[x] = Four<T>::wide(*reinterpret_cast<const raw*>(a.v + key_offset(a, s, at, a.v_stride) + head));
        }
#pragma unroll
        for (int x = 0; x < kBatch; ++x) {
            if (key + x >= k_end || !((seen >> x) & 1u)) continue;
            const float dot = wave_sum(mine ? (q.x * k[x].x + q.y * k[x].y) + (q.z * k[x].z + q.w * k[x].w) : 0.0f);
            const float p = exp2f((dot - m) * a.c2);
            l += p;
            o.x += p * v[x].x; o.y += p * v[x].y; o.z += p * v[x].z; o.w += p * v[x].w;
        }
        if (__all(o.x != o.x && o.y != o.y && o.z != o.z && o.w != o.w)) return;      // nothing else comes of it
    }
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

// The rows `bad` (bit b: row row0 + b of the block), dims dim0 .. dim1 - 1 of them, leave as exact_row has them: into the slot, or
// finished.  m_of(row): the reference that the row's (max, sum) go by.
template <typename T, SlotOrder O, typename F>
__device__ __forceinline__ void leave_exact_rows(const AttendArgs& a, const AttendItem& it, uint32_t bad, int row0, int dim0, int dim1, int rows_per_block, int k_begin,
                                                 int k_end, int n_parts, float* slot, F m_of)
{
    const int lane = threadIdx.x & 63, r0 = it.block * rows_per_block;
    const bool mine = 4 * lane >= dim0 && 4 * lane < dim1;
    while (bad) {
        const int row = row0 + __builtin_ctz(bad);
        bad &= bad - 1u;
        float4 o;
        float l;
        exact_row<T>(a, it.s, it.kvh, r0 + row, k_begin, k_end, m_of(row), o, l);
        if (!mine) continue;
        if (n_parts > 1) {
            store_four(slot + slot_place<O>(a.d, row, lane), o.x, o.y, o.z, o.w);
        } else {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const int j = div_G(a, r0 + row);
            Four<T>::store(out_row(a, it.s, j, it.kvh * a.G + (r0 + row - j * a.G), sizeof(T)) + 4 * lane * (int)sizeof(T),
                           make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
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
