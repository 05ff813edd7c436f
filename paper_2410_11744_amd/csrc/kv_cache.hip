// The paged cache's own calls: dyspec_kv_append (new tokens' keys, rotated, and values into the pages, their queries beside) and
// dyspec_kv_keep (the accepted path's rows move up behind the root's).  Both move bytes: what bounds them is memory, and for a
// decode step's few hundred KB the trips to it.
#include "kv_cache.h"

#include "launch.h"

namespace dyspec {

template <typename Args> __device__ __forceinline__ const Args& args_here()      // (read where they are: a copy would go to scratch memory)
{
    return *(const Args*)(__attribute__((address_space(4))) const Args*)__builtin_amdgcn_kernarg_segment_ptr();
}
template <int S> static void fill(Sequences<S>& to, const Sequences<DYSPEC_MAX_SEQ>& from, int n_seq)
{
    for (int s = 0; s < n_seq; ++s) { to.row0[s] = from.row0[s]; to.context[s] = from.context[s]; }
    to.row0[n_seq] = from.row0[n_seq];
}

// ---- append
//
// Pair i of a head is turned by the angle pos * inv_freq[i].  The product of a position and an fp32 frequency is exact in 64
// bits, and so is kept in turns to 2^-53 of its size; the fraction of a turn, in [-1/2, 1/2], is what goes to 32 bits, so far
// positions lose nothing.
//
// A unit is VEC pairs: two pieces of VEC elements, which one thread reads, turns and writes, so that a tensor may be rotated in
// place.  Units past the rotated dims, and those of V, are copied.  A workgroup has one token (with few tokens a share of one's
// units).  A thread asks for its first unit before it looks anything up, so that the trips to memory for the page, the
// frequencies and the rows overlap; the sines are computed once a workgroup, for all heads, into LDS.
//
// What bounds it: memory with many tokens (4322 tokens of 40 heads of 128, bf16, 266 MB: 52 us, 5.05 TB/s; a copy of 1 GiB
// reaches 5.24), the trips one after the other with few (64 tokens of 64 + 8 heads: 3.6 us).  Four tokens a workgroup, or four units
// of a thread in flight, were slower (70 us).
constexpr int kAppendThreads = 256, kAppendBatch = 2;
static_assert(kAppendThreads >= 128, "a thread per pair of a head");

template <typename T, int VEC> struct alignas(VEC * sizeof(T)) Piece { T e[VEC]; };

template <typename T, int VEC, int S>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(AppendArgs<S>)
{
    const AppendArgs<S>& a = args_here<AppendArgs<S>>();
    __shared__ float2 turn[128];                           // cos, sin
    typedef Piece<T, VEC> piece;
    const int token = blockIdx.x, tid = threadIdx.x;
    const int half = a.half, d = a.d, Hq = a.Hq, Hkv = a.Hkv;
    const bool apart = !a.interleaved;
    struct Unit { int head, at0, at1; piece p0, p1; };
    auto fetch = [&](Unit& w, uint32_t x) __attribute__((always_inline)) {
        w.head = a.per_head_magic ? (int)__umulhi(x, a.per_head_magic) : (int)x;
        const int u = (int)x - w.head * a.per_head, h = w.head;
        const bool turns = h < Hq + Hkv && u * VEC < half;
        w.at0 = turns && apart ? u * VEC : 2 * u * VEC;
        w.at1 = turns && apart ? half + u * VEC : w.at0 + VEC;
        const T* const src = (h < Hq ? static_cast<const T*>(a.q) + token * a.q_stride + (long long)h * d
                              : h < Hq + Hkv ? static_cast<const T*>(a.k) + token * a.k_stride + (long long)(h - Hq) * d
                                             : static_cast<const T*>(a.v) + token * a.v_stride + (long long)(h - Hq - Hkv) * d);
        w.p0 = *reinterpret_cast<const piece*>(src + w.at0);
        if (w.at1 < d) w.p1 = *reinterpret_cast<const piece*>(src + w.at1);
    };
    long long row = -1;                                    // element offset of the token's row in the pool, -1: no page
    auto finish = [&](Unit& w) __attribute__((always_inline)) {
        const bool is_q = w.head < Hq, is_v = w.head >= Hq + Hkv;
        if (!is_v && w.at0 < (apart ? half : 2 * half)) {
            const float2* const cs = turn + (apart ? w.at0 : w.at0 / 2);
            if (apart) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float x = (float)w.p0.e[e], y = (float)w.p1.e[e];
                    w.p0.e[e] = (T)(x * cs[e].x - y * cs[e].y);
                    w.p1.e[e] = (T)(x * cs[e].y + y * cs[e].x);
                }
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {            // pair e: elements 2e and 2e + 1 of both pieces end to end
                    T& lo = 2 * e < VEC ? w.p0.e[(2 * e) % VEC] : w.p1.e[(2 * e) % VEC];
                    T& hi = 2 * e + 1 < VEC ? w.p0.e[(2 * e + 1) % VEC] : w.p1.e[(2 * e + 1) % VEC];
                    const float x = (float)lo, y = (float)hi;
                    lo = (T)(x * cs[e].x - y * cs[e].y);
                    hi = (T)(x * cs[e].y + y * cs[e].x);
                }
            }
        }
        auto leave = [&](T* dst) __attribute__((always_inline)) {
            *reinterpret_cast<piece*>(dst + w.at0) = w.p0;
            if (w.at1 < d) *reinterpret_cast<piece*>(dst + w.at1) = w.p1;
        };
        if (is_q) {
            leave(static_cast<T*>(a.q_out) + ((long long)token * Hq + w.head) * d);
        } else {
            const int h = is_v ? w.head - Hq - Hkv : w.head - Hq;
            if (row >= 0) leave(static_cast<T*>(is_v ? a.v_pages : a.k_pages) + row + (long long)h * d);
            if (!is_v && a.k_out) leave(static_cast<T*>(a.k_out) + ((long long)token * Hkv + h) * d);
        }
    };
    const uint32_t end = min((uint32_t)a.units, (blockIdx.y + 1) * a.share);
    uint32_t x = blockIdx.y * a.share + tid;
    Unit first;
    const bool some = x < end;
    if (some) fetch(first, x);
    // ---- the token's sequence (lanes ask one each), its place, its angles
    const int lane = tid & 63;
    const int s = __builtin_popcountll(__builtin_amdgcn_ballot_w64(token >= (lane < a.n_seq ? a.seq.row0[lane] : 0x7fffffff))) - 1;
    const int C = a.seq.context[s], local = token - a.seq.row0[s], at = C + local;
    const unsigned page = (unsigned)a.table[(long long)s * a.table_stride + (at >> a.page_shift)];
    if (tid < half) {
        const long long pos = (long long)C + (a.rel_pos ? a.rel_pos[token] : local);
        const double turns = (double)pos * (double)a.inv_freq[tid] * 0.15915494309189533577;      // 1 / 2 pi
        float sn, cs;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
        turn[tid] = make_float2(cs, sn);
    }
    if (page < (unsigned)a.n_pages) row = (long long)page * a.page_stride + (long long)(at & ((1 << a.page_shift) - 1)) * Hkv * d;
    __syncthreads();
    if (some) finish(first);
    for (x += kAppendThreads; x < end; x += kAppendBatch * kAppendThreads) {
        Unit w[kAppendBatch];
#pragma unroll
        for (int y = 0; y < kAppendBatch; ++y)
            if (x + y * kAppendThreads < end) fetch(w[y], x + y * kAppendThreads);
#pragma unroll
        for (int y = 0; y < kAppendBatch; ++y)
            if (x + y * kAppendThreads < end) finish(w[y]);
    }
}

template <typename T, int VEC, int S>
static hipError_t launch_append(const AppendHead& head, const Sequences<DYSPEC_MAX_SEQ>& seq, hipStream_t stream)
{
    static Kernel kernel(reinterpret_cast<const void*>(&kv_append_kernel<T, VEC, S>));
    AppendArgs<S> a;
    static_cast<AppendHead&>(a) = head;
    fill(a.seq, seq, head.n_seq);
    const uint32_t total = (uint32_t)seq.row0[head.n_seq];
    a.per_head = (a.d + 2 * VEC - 1) / (2 * VEC);
    a.units = a.per_head * (a.Hq + 2 * a.Hkv);
    // few tokens: up to a workgroup per 256 units, so that about two workgroups a CU share the work
    const uint32_t cuts = max(1u, min(512u / total, (uint32_t)(a.units + kAppendThreads - 1) / kAppendThreads));
    a.share = ((a.units + cuts - 1) / cuts + kAppendThreads - 1) / kAppendThreads * kAppendThreads;
    // x / n as hi(x * magic), exact while x * n < 2^32: at most 24576 heads of 128 units
    a.per_head_magic = a.per_head == 1 ? 0u : (uint32_t)((1ull << 32) / a.per_head + 1);
    return kernel.launch(dim3(total, (a.units + a.share - 1) / a.share), kAppendThreads, 0, stream, a);
}
template <typename T, int VEC>
static hipError_t launch_append(const AppendHead& head, const Sequences<DYSPEC_MAX_SEQ>& seq, hipStream_t stream)
{
    return head.n_seq <= kFewSeq ? launch_append<T, VEC, kFewSeq>(head, seq, stream) : launch_append<T, VEC, DYSPEC_MAX_SEQ>(head, seq, stream);
}

hipError_t launch_kv_append(const AppendHead& a, const Sequences<DYSPEC_MAX_SEQ>& seq, int dtype, bool wide, hipStream_t stream)
{
    if (seq.row0[a.n_seq] == 0) return hipSuccess;
    if (dtype == DYSPEC_F32) return wide ? launch_append<float, 4>(a, seq, stream) : launch_append<float, 1>(a, seq, stream);
    return wide ? launch_append<__bf16, 8>(a, seq, stream) : launch_append<__bf16, 1>(a, seq, stream);
}

// ---- keep
//
// Row C + 1 + i of a sequence takes row C + accepted[i].  A path's rows ascend and the root is row 0, so accepted[i] > i: a row
// is only ever read from its own place or from behind every place written before, and a thread that moves its 16-byte column
// eight rows at a time (all eight read before the first is written) needs no copy of the rows and no other thread.
// Lane l of a wave looks up the l-th move of the eight, so that the list, the page numbers and the rows are three trips to memory.
// Those bound it: 9 rows of 80 layers of 8 heads of 128, bf16 (5.9 MB, which memory could move in 1.1 us), take 4.7 us.
constexpr int kKeepThreads = 128, kKeepBatch = 8;

typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef uint32_t words2 __attribute__((ext_vector_type(2)));

template <typename V, int S>
__global__ __launch_bounds__(kKeepThreads) void kv_keep_kernel(KeepArgs<S>)
{
    const KeepArgs<S>& a = args_here<KeepArgs<S>>();
    const int s = blockIdx.y, first = a.seq.row0[s], N = a.seq.row0[s + 1] - first, C = a.seq.context[s];
    if (N < 2) return;
    const int lane = threadIdx.x & 63, col = blockIdx.x * kKeepThreads + threadIdx.x;
    const bool mine = col < a.row_pieces;
    char* const pool = (blockIdx.z & 1 ? a.v_pages : a.k_pages) + (blockIdx.z >> 1) * a.layer_bytes + (long long)col * (int)sizeof(V);
    const int* const table = a.table + (long long)s * a.table_stride;
    const int page_mask = (1 << a.page_shift) - 1;
    auto listed = [&](int i0) { return a.accepted[first + min(i0 + (lane & (kKeepBatch - 1)), N - 2)]; };
    int from = listed(0);                                          // (with the count: it does not wait for that)
    const int n = min(a.n_accepted[s], N - 1);
    for (int i0 = 0; i0 < n; i0 += kKeepBatch) {
        const int i = i0 + (lane & (kKeepBatch - 1));
        long long src = -1, dst = -1;                              // byte offsets of this lane's move
        if (i < n && from > i + 1 && from < N) {                   // (from == i + 1: in place already)
            const unsigned p = (unsigned)table[(C + from) >> a.page_shift], q = (unsigned)table[(C + 1 + i) >> a.page_shift];
            if (p < (unsigned)a.n_pages && q < (unsigned)a.n_pages) {
                src = p * a.page_bytes + ((C + from) & page_mask) * a.row_bytes;
                dst = q * a.page_bytes + ((C + 1 + i) & page_mask) * a.row_bytes;
            }
        }
        if (i0 + kKeepBatch < n) from = listed(i0 + kKeepBatch);
        auto of_lane = [](long long x, int l) {
            return (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32) | (unsigned)__builtin_amdgcn_readlane((int)x, l));
        };
        V v[kKeepBatch];
        long long to[kKeepBatch];
#pragma unroll
        for (int x = 0; x < kKeepBatch; ++x) {
            const long long at = of_lane(src, x);
            to[x] = of_lane(dst, x);
            if (at >= 0 && mine) v[x] = *reinterpret_cast<const V*>(pool + at);
        }
#pragma unroll
        for (int x = 0; x < kKeepBatch; ++x)
            if (to[x] >= 0 && mine) *reinterpret_cast<V*>(pool + to[x]) = v[x];
    }
}

template <typename V, int S>
static hipError_t launch_keep(const KeepHead& head, const Sequences<DYSPEC_MAX_SEQ>& seq, int n_layers, hipStream_t stream)
{
    static Kernel kernel(reinterpret_cast<const void*>(&kv_keep_kernel<V, S>));
    KeepArgs<S> a;
    static_cast<KeepHead&>(a) = head;
    fill(a.seq, seq, head.n_seq);
    return kernel.launch(dim3((a.row_pieces + kKeepThreads - 1) / kKeepThreads, a.n_seq, 2 * n_layers), kKeepThreads, 0, stream, a);
}
template <typename V>
static hipError_t launch_keep(const KeepHead& head, const Sequences<DYSPEC_MAX_SEQ>& seq, int n_layers, hipStream_t stream)
{
    return head.n_seq <= kFewSeq ? launch_keep<V, kFewSeq>(head, seq, n_layers, stream) : launch_keep<V, DYSPEC_MAX_SEQ>(head, seq, n_layers, stream);
}

hipError_t launch_kv_keep(const KeepHead& a, const Sequences<DYSPEC_MAX_SEQ>& seq, int n_layers, hipStream_t stream)
{
    if (seq.row0[a.n_seq] == 0) return hipSuccess;
    return a.piece_bytes == 16 ? launch_keep<words4>(a, seq, n_layers, stream) : launch_keep<words2>(a, seq, n_layers, stream);
}

hipError_t prepare_kv_cache()                                      // (asking loads the code)
{
    hipFunction_t f;
    return Kernel(reinterpret_cast<const void*>(&kv_keep_kernel<words4, kFewSeq>)).find(&f);
}

}  // namespace dyspec
