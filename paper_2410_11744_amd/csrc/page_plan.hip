// dyspec_page_plan: page tables and slot maps follow the requests' lengths.
//
// Sequence s holds A = ceil(held / page) pages and is to hold B = ceil(wanted / page).  The free pages are a ring: `count` of them
// from `head` on, round the end.  With sums over the sequences before s (wave scans, a lane a sequence, done by every wave for
// itself), the page of column c is known at once:
//   B > A   table[c] = ring[head + sum of (B - A) + c - A]             if the sum up to and with s is at most `count`
//   B < A   ring[head + count + sum of (A - B) + c - B] = table[c],    table[c] = -1
// Pages are taken from one end and given back behind the other, so no place of the ring is read and written in one call.
//
// What bounds it: trips to memory one after the other (the lengths and the ring's state, then the pages; with several workgroups the
// arrival), not the bytes: a token each of 64 sequences 3.9 us, of which an empty kernel takes 2; 64 sequences of which 16 end and 16 come
// with prompts of 500 to 8000 tokens 6.1 us for 0.7 MB.
#include "page_plan.h"

#include "launch.h"

namespace dyspec {

constexpr int kPlanFew = 256, kPlanMany = 1024;   // threads of a workgroup
constexpr int kPlanBatch = 4;                    // slots of a thread that are looked up together
constexpr int kPlanMost = 2;                     // workgroups of a sequence

// Sum over the lanes up to and with this one.
__device__ __forceinline__ long long upto_lane(long long v, int lane)
{
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const long long up = __shfl_up(v, o, kWave);
        if (lane >= o) v += up;
    }
    return v;
}
// x of lane s, which is the same for the whole wave.
__device__ __forceinline__ long long of_lane(long long x, int s)
{
    return (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), s) << 32) | (unsigned)__builtin_amdgcn_readlane((int)x, s));
}

__global__ __launch_bounds__(kPlanMany) void page_plan_kernel(PlanArgs a)
{
    const int s = blockIdx.x, lane = threadIdx.x & 63;
    const unsigned n_pages = (unsigned)a.n_pages;
    // ---- every sequence's lengths, a lane each
    const bool there = lane < a.n_seq;
    const int x = there ? a.held[lane] : 0, y = there ? a.wanted[lane] : 0;
    const int since = a.slots_from ? (there ? a.slots_from[lane] : 0) : x;
    const unsigned head = (unsigned)a.state[0] % n_pages;
    const long long count = min(max(a.state[1], 0), a.n_pages);
    const int page = 1 << a.page_shift;
    const bool sized = x >= 0 && y >= 0 && x <= DYSPEC_MAX_CONTEXT && y <= DYSPEC_MAX_CONTEXT;
    const int A = sized ? (x + page - 1) >> a.page_shift : 0, B = sized ? (y + page - 1) >> a.page_shift : 0;
    const bool right = sized && A <= a.max_pages && B <= a.max_pages;
    // first token that gets a slot: no further on than the last one's end, so that places (in 32 bits) stay below 2^30 and a few thousand
    const int z = right ? min(max(since, 0), y) : 0;
    const long long need = right ? max(B - A, 0) : 0, back = right ? max(A - B, 0) : 0, marked = right ? y - z : 0;
    const long long need_upto = upto_lane(need, lane), back_upto = upto_lane(back, lane), marked_upto = upto_lane(marked, lane);
    const bool fits = need_upto <= count;
    // what is taken in all: demands come in order, so it is the last sum that fits
    const unsigned long long fitting = __builtin_amdgcn_ballot_w64(fits);
    const long long taken = fitting ? of_lane(need_upto, 63 - __builtin_clzll(fitting)) : 0;
    const long long room = min(of_lane(back_upto, 63), (long long)a.n_pages - count);     // (more can only be pages given back twice)
    // ---- this workgroup's sequence
    const int held = __builtin_amdgcn_readlane(x, s), wanted = __builtin_amdgcn_readlane(y, s);
    const int before = __builtin_amdgcn_readlane(A, s), after = __builtin_amdgcn_readlane(B, s);
    const bool ok = (__builtin_amdgcn_ballot_w64(right) >> s) & 1ull;
    const bool granted = before >= after || ((fitting >> s) & 1ull);
    int* const table = a.table + (long long)s * a.table_stride;
    const int first = blockIdx.y * blockDim.x + threadIdx.x, step = gridDim.y * blockDim.x;
    // (`off` places on from `at`, both below n_pages: round the end once)
    auto on = [=](unsigned at, unsigned off) { const unsigned x = at + off; return x >= n_pages ? x - n_pages : x; };
    const unsigned next = on(head, (unsigned)(granted ? min(of_lane(need_upto - need, s), (long long)n_pages - 1) : 0));       // column `before`
    auto fresh = [&](int column) { return a.ring[on(next, (unsigned)(column - before))]; };
    if (ok && granted)
        for (int c = before + first; c < after; c += step) table[c] = fresh(c);
    if (ok && before > after) {
        const long long given = of_lane(back_upto - back, s);
        for (int c = after + first; c < before; c += step) {
            const long long i = given + (c - after);
            const int p = table[c];
            if (i < room) a.ring[on(head, (unsigned)(count + i))] = p;
            table[c] = -1;
        }
    }
    if (a.slots && ok) {
        const long long at = of_lane(marked_upto - marked, s);
        const int from = __builtin_amdgcn_readlane(z, s), upto = (int)min((long long)wanted, from + max(a.n_slots - at, 0LL));
        for (int p0 = from + first; p0 < upto; p0 += kPlanBatch * step) {
            int page_of[kPlanBatch];
#pragma unroll
            for (int y = 0; y < kPlanBatch; ++y) {
                const int column = (int)min((long long)p0 + (long long)y * step, (long long)upto - 1) >> a.page_shift;
                page_of[y] = !granted ? -1 : column < before ? table[column] : fresh(column);
            }
#pragma unroll
            for (int y = 0; y < kPlanBatch; ++y) {
                const int place = p0 + y * step;
                if (place < upto) a.slots[at + (place - from)] = page_of[y] < 0 ? -1 : ((long long)page_of[y] << a.page_shift) + (place & (page - 1));
            }
        }
    }
    __syncthreads();                                       // (every wave that goes by the ring's state has it)
    if (threadIdx.x != 0) return;
    if (blockIdx.y == 0) a.granted[s] = !ok ? -1 : granted ? wanted : held;
    // ---- the ring's state changes when every workgroup has read it
    const unsigned last = gridDim.x * gridDim.y - 1u;
    if (last == 0u || __builtin_amdgcn_atomic_inc32(reinterpret_cast<unsigned*>(a.state) + 2, last, __ATOMIC_RELAXED, "agent") == last) {
        a.state[0] = (int)on(head, taken < (long long)n_pages ? (unsigned)taken : 0u);
        a.state[1] = (int)(count - taken + room);
    }
}

static Kernel plan_kernel(reinterpret_cast<const void*>(&page_plan_kernel));

hipError_t launch_page_plan(const PlanArgs& a, hipStream_t stream)
{
    // Few large workgroups: each arrives at the ring's state by an atomic of its own, and those take turns (64 sequences, 66000 slots:
    // 8.9 us with eight workgroups of 256 threads a sequence, 6.1 with up to two of 1024).
    const long long most = a.slots ? max((long long)a.max_pages, a.n_slots) : a.max_pages;
    const int threads = most <= kPlanBatch * kPlanFew ? kPlanFew : kPlanMany;
    const unsigned cuts = most <= kPlanBatch * kPlanMany ? 1 : kPlanMost;
    return plan_kernel.launch(dim3(a.n_seq, cuts), threads, 0, stream, a);
}

hipError_t prepare_page_plan()                   // (asking loads the code)
{
    hipFunction_t f;
    return plan_kernel.find(&f);
}

}  // namespace dyspec
