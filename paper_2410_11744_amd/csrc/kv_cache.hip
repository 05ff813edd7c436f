// The paged cache's own calls: dyspec_kv_append (new tokens' keys, rotated, and values into the pages, their queries beside) and
// dyspec_kv_keep (the accepted path's rows move up behind the root's).  Both move bytes: what bounds them is memory, and for a
// decode step's few hundred KB the trips to it.
#include "kv_cache.h"

namespace dyspec {

// ---- append
//
// Pair i of a head is turned by the angle pos * inv_freq[i].  The product of a position and an fp32 frequency is exact in 64
// bits, and so is kept in turns to 2^-53 of its size; the fraction of a turn, in [-1/2, 1/2], is what goes to 32 bits, so far
// positions lose nothing.  A workgroup computes the sines of its tokens once, for all heads, into LDS.
//
// A unit is VEC pairs: two pieces of VEC elements, which one thread reads, turns and writes, so that a tensor may be rotated in
// place.  Units past the rotated dims, and those of V, are copied.
constexpr int kAppendThreads = 256;

template <typename T, int VEC> struct alignas(VEC * sizeof(T)) Piece { T e[VEC]; };

template <typename T, int VEC>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(AppendArgs a)
{
    extern __shared__ float2 turn[];                       // [tokens][half]: cos, sin
    __shared__ long long place[kAppendTokens];             // element offset of a token's row in the pool, -1: no page
    const int t0 = blockIdx.x * a.tokens, count = min(a.tokens, a.total - t0);
    for (int x = threadIdx.x; x < count * max(a.half, 1); x += kAppendThreads) {
        const int t = a.half > 0 ? x / a.half : x, i = x - t * a.half;
        const int row = t0 + t;
        int s = 0;
        while (s + 1 < a.n_seq && row >= a.row0[s + 1]) ++s;
        const int local = row - a.row0[s];
        if (a.half > 0) {
            const long long pos = (long long)a.context[s] + (a.rel_pos ? a.rel_pos[row] : local);
            const double turns = (double)pos * (double)a.inv_freq[i] * 0.15915494309189533577;    // 1 / 2 pi
            float sn, cs;
            sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
            turn[x] = make_float2(cs, sn);
        }
        if (i == 0) {
            const int at = a.context[s] + local;
            const unsigned page = (unsigned)a.table[(long long)s * a.table_stride + (at >> a.page_shift)];
            place[t] = page < (unsigned)a.n_pages ? (long long)page * a.page_stride + (long long)(at & ((1 << a.page_shift) - 1)) * a.Hkv * a.d : -1;
        }
    }
    __syncthreads();
    typedef Piece<T, VEC> piece;
    const int heads = a.Hq + 2 * a.Hkv, per_head = (a.d + 2 * VEC - 1) / (2 * VEC), turned = a.half / VEC;
    for (int x = threadIdx.x; x < count * heads * per_head; x += kAppendThreads) {
        const int u = x % per_head, y = x / per_head;
        const int head = y % heads, t = y / heads;
        const bool is_q = head < a.Hq, is_v = head >= a.Hq + a.Hkv;
        const int hh = is_q ? head : is_v ? head - a.Hq - a.Hkv : head - a.Hq;
        const T* const src = (is_q ? static_cast<const T*>(a.q) + (t0 + t) * a.q_stride
                                   : is_v ? static_cast<const T*>(a.v) + (t0 + t) * a.v_stride
                                          : static_cast<const T*>(a.k) + (t0 + t) * a.k_stride) + (long long)hh * a.d;
        const bool turns = !is_v && u < turned;
        const int at0 = turns && !a.interleaved ? u * VEC : 2 * u * VEC;
        const int at1 = turns && !a.interleaved ? a.half + u * VEC : at0 + VEC;
        piece p0 = *reinterpret_cast<const piece*>(src + at0), p1;
        if (at1 < a.d) p1 = *reinterpret_cast<const piece*>(src + at1);
        if (turns) {
            const float2* const cs = turn + t * a.half + u * VEC;
            if (a.interleaved) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {            // pair e: elements 2e and 2e + 1 of both pieces end to end
                    T* const lo = 2 * e < VEC ? &p0.e[2 * e] : &p1.e[2 * e - VEC];
                    T* const hi = 2 * e + 1 < VEC ? &p0.e[2 * e + 1] : &p1.e[2 * e + 1 - VEC];
                    const float u0 = (float)*lo, u1 = (float)*hi;
                    *lo = (T)(u0 * cs[e].x - u1 * cs[e].y);
                    *hi = (T)(u0 * cs[e].y + u1 * cs[e].x);
                }
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float u0 = (float)p0.e[e], u1 = (float)p1.e[e];
                    p0.e[e] = (T)(u0 * cs[e].x - u1 * cs[e].y);
                    p1.e[e] = (T)(u0 * cs[e].y + u1 * cs[e].x);
                }
            }
        }
        auto leave = [&](T* dst) {
            *reinterpret_cast<piece*>(dst + at0) = p0;
            if (at1 < a.d) *reinterpret_cast<piece*>(dst + at1) = p1;
        };
        if (is_q) {
            leave(static_cast<T*>(a.q_out) + ((long long)(t0 + t) * a.Hq + hh) * a.d);
        } else {
            if (place[t] >= 0) leave(static_cast<T*>(is_v ? a.v_pages : a.k_pages) + place[t] + (long long)hh * a.d);
            if (!is_v && a.k_out) leave(static_cast<T*>(a.k_out) + ((long long)(t0 + t) * a.Hkv + hh) * a.d);
        }
    }
}

template <typename T>
static void launch_append(const AppendArgs& a, bool wide, int blocks, hipStream_t stream)
{
    const size_t lds = (size_t)a.tokens * a.half * sizeof(float2);
    if (wide) kv_append_kernel<T, 16 / (int)sizeof(T)><<<blocks, kAppendThreads, lds, stream>>>(a);
    else kv_append_kernel<T, 1><<<blocks, kAppendThreads, lds, stream>>>(a);
}

hipError_t launch_kv_append(AppendArgs a, int dtype, bool wide, hipStream_t stream)
{
    if (a.total == 0) return hipSuccess;
    a.tokens = a.total <= 1024 ? 1 : kAppendTokens;
    const int blocks = (a.total + a.tokens - 1) / a.tokens;
    if (dtype == DYSPEC_F32) launch_append<float>(a, wide, blocks, stream);
    else launch_append<__bf16>(a, wide, blocks, stream);
    return hipGetLastError();
}

// ---- keep
//
// Row C + 1 + i of a sequence takes row C + accepted[i].  A path's rows ascend and the root is row 0, so accepted[i] > i: a row
// is only ever read from its own place or from behind every place written before, and a thread that moves its 16-byte column
// eight rows at a time (all eight read before the first is written) needs no copy of the rows and no other thread.
constexpr int kKeepThreads = 128, kKeepBatch = 8;

typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef uint32_t words2 __attribute__((ext_vector_type(2)));

template <typename V>
__global__ __launch_bounds__(kKeepThreads) void kv_keep_kernel(KeepArgs a)
{
    const int s = blockIdx.y, N = a.row0[s + 1] - a.row0[s], C = a.context[s];
    const int n = min(a.n_accepted[s], N - 1);
    const int col = blockIdx.x * kKeepThreads + threadIdx.x;
    if (col >= a.row_pieces || n <= 0) return;
    const int layer = blockIdx.z >> 1;
    char* const pool = (blockIdx.z & 1 ? a.v_pages : a.k_pages) + layer * a.layer_bytes + (long long)col * (int)sizeof(V);
    const int* const table = a.table + (long long)s * a.table_stride;
    auto offset = [&](int at) -> long long {
        const unsigned page = (unsigned)table[at >> a.page_shift];
        return page < (unsigned)a.n_pages ? (long long)page * a.page_bytes + (long long)(at & ((1 << a.page_shift) - 1)) * a.row_bytes : -1;
    };
    for (int i0 = 0; i0 < n; i0 += kKeepBatch) {
        V v[kKeepBatch];
        long long to[kKeepBatch];
#pragma unroll
        for (int x = 0; x < kKeepBatch; ++x) {
            const int i = min(i0 + x, n - 1);
            const int from = a.accepted[a.row0[s] + i];
            to[x] = -1;
            if (i0 + x < n && from > i + 1 && from < N) {          // from == i + 1: in place already
                const long long src = offset(C + from);
                if (src >= 0) {
                    to[x] = offset(C + 1 + i);
                    v[x] = *reinterpret_cast<const V*>(pool + src);
                }
            }
        }
#pragma unroll
        for (int x = 0; x < kKeepBatch; ++x)
            if (to[x] >= 0) *reinterpret_cast<V*>(pool + to[x]) = v[x];
    }
}

hipError_t launch_kv_keep(const KeepArgs& a, int n_layers, hipStream_t stream)
{
    if (a.row0[a.n_seq] == 0) return hipSuccess;
    const dim3 grid((a.row_pieces + kKeepThreads - 1) / kKeepThreads, a.n_seq, 2 * n_layers);
    if (a.piece_bytes == 16) kv_keep_kernel<words4><<<grid, kKeepThreads, 0, stream>>>(a);
    else kv_keep_kernel<words2><<<grid, kKeepThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace dyspec
