// dyspec_sample and dyspec_filter_logits: what top-k, top-p and min-p leave of a row of logits, and a token drawn from it.
//
// The tokens of a row are ordered by falling logit, equal ones by rising index.  Every filter keeps the first so many of that
// order, so together they keep the tokens up to a cut (a logit and, among the tokens that have it, an index), and a row takes:
// its maximum; the cut of top-k, then of top-p, then of min-p; the sum of what is kept and the place in it where the draw falls.
//
// Weights exp((x - max) / T) are computed in 64 bits to 4e-14 and held as whole numbers of 2^-45, so that their sums (of up to 2^18
// of them) are exact, the same in every order: histograms are filled by atomics, and a call gives the same bits every time.
// A token below 2^-46 of the row's largest weighs nothing: it can be kept, but is not drawn.
//
// A cut by sums (of weights, or of ones for top-k) is found in three steps: a histogram over 2048 even steps of the distance to the
// maximum (a few tokens a bin; by the bits of the logits most tokens would meet in a few bins), the bin where the sum reaches what
// is kept, and the tokens of that bin one by one: each adds up those before it.  A bin with more than kListed tokens (equal logits,
// or masks of the type's lowest value) is gone through by the bits of its logits instead, and equal ones by index.
//
// A workgroup has one row, held in registers up to 32768 tokens, else read again for every pass; each of its 16 waves has a run of
// the vocabulary, so that sums over waves, and then over the threads of one run, find a place in the order of the indices.
#include "sample.h"

#include "launch.h"
#include "vocab_common.h"

namespace dyspec {

typedef unsigned long long u64;

constexpr int kRowThreads = 1024, kRowWaves = kRowThreads / kWave;
constexpr int kBins = 2048, kListed = 1024;
constexpr int kHeldTokens = 32;                  // of a thread whose row is held
constexpr int kWeightBits = 45;                  // the largest weight is 2^kWeightBits: 2^18 of them stay below 2^63
static_assert(DYSPEC_MAX_SAMPLE_VOCAB <= 1 << (63 - kWeightBits), "sums fit");

struct Listed { float x; int i; u64 amount; };

struct SampleLds {
    u64 hist[kBins];
    Listed list[kListed];
    u64 sums[kRowWaves];
    float hi[kRowWaves], lo[kRowWaves];
    int odd[kRowWaves];
    int counts[kRowWaves];
    u64 before;                                  // of a bin, of a token: the sum up to it
    u64 amount;
    int found, n_listed;
    float cut_x;
    int cut_i;
};

template <typename T> struct RowPiece;           // 16 bytes of a row
template <> struct RowPiece<float> {
    static constexpr int kTokens = 4;
    static __device__ __forceinline__ float value(const uint4& r, int e) { return __uint_as_float((&r.x)[e]); }
    static __device__ __forceinline__ uint32_t bits(float x) { return __float_as_uint(x); }
};
template <> struct RowPiece<__bf16> {
    static constexpr int kTokens = 8;
    static __device__ __forceinline__ float value(const uint4& r, int e) { const uint32_t w = (&r.x)[e / 2]; return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16); }
};

// exp2(z) in whole numbers of 2^-kWeightBits, z <= 0.  The fraction's power by a polynomial through Chebyshev's nodes, to 3.7e-14.
__device__ __forceinline__ u64 weight_of(double z)
{
    constexpr double kShift = 6755399441055744.0;              // 1.5 * 2^52: the sum's low bits are the nearest whole number
    z = fmax(z, -100.0);
    const double t = z + kShift, f = z - (t - kShift);
    const int n = (int)__double2loint(t);
    double p = 1.0203121063391729e-07;
    p = fma(p, f, 1.3255224878668817e-06);
    p = fma(p, f, 1.525268684626772e-05);
    p = fma(p, f, 0.00015403455852453838);
    p = fma(p, f, 0.0013333558179043112);
    p = fma(p, f, 0.009618129159402558);
    p = fma(p, f, 0.055504108664760424);
    p = fma(p, f, 0.2402265069581299);
    p = fma(p, f, 0.6931471805599453);
    p = fma(p, f, 1.0);
    const double w = ldexp(p, n + kWeightBits) + 4503599627370496.0;      // + 2^52: rounded to a whole number in the low bits
    return (u64)__double_as_longlong(w) & 0xfffffffffffffull;
}

// Ascending with x; -0 and 0 alike.
__device__ __forceinline__ uint32_t ordered_bits(float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}

// A row as a thread has it.  Wave w has tokens w * span .. of the row, lane l of it the kTokens from w * span + (64 p + l) * kTokens
// on, p < pieces.  Places past the row's end hold a NaN, which no comparison keeps.
template <typename T, bool Held> struct Row {
    static constexpr int VEC = RowPiece<T>::kTokens, NP = Held ? kHeldTokens / VEC : 1;
    const T* at;
    int V, pieces, first;                        // first: of this thread
    uint4 held[NP];

    __device__ __forceinline__ int span() const { return pieces * kWave * VEC; }
    __device__ __forceinline__ int index(int p) const { return first + p * kWave * VEC; }
    __device__ __forceinline__ uint4 fetch(int p) const
    {
        typedef typename Unaligned<T>::Piece raw;
        const int i = index(p);
        if (V >= VEC) {                          // (the same for all)
            const raw r = *reinterpret_cast<const raw*>(at + (i + VEC <= V ? i : 0));
            return make_uint4(r.x, r.y, r.z, r.w);
        }
        return make_uint4(~0u, ~0u, ~0u, ~0u);
    }
    __device__ __forceinline__ uint4 mended(uint4 r, int p) const
    {
        const int i = index(p);
        if (i + VEC <= V) return r;
        r = make_uint4(~0u, ~0u, ~0u, ~0u);
        for (int e = 0; e < VEC && i + e < V; ++e) {
            if constexpr (sizeof(T) == 4) (&r.x)[e] = __float_as_uint(at[i + e]);
            else (&r.x)[e / 2] = (e & 1) ? ((&r.x)[e / 2] & 0xffffu) | bits_of(at[i + e]) << 16 : ((&r.x)[e / 2] & 0xffff0000u) | bits_of(at[i + e]);
        }
        return r;
    }
    __device__ __forceinline__ void load()
    {
        if constexpr (Held) {
#pragma unroll
            for (int p = 0; p < NP; ++p)
                if (p < pieces) held[p] = fetch(p);
#pragma unroll
            for (int p = 0; p < NP; ++p) held[p] = p < pieces ? mended(held[p], p) : make_uint4(~0u, ~0u, ~0u, ~0u);
        }
    }
    // f(piece, index of its first token)
    template <typename F> __device__ __forceinline__ void each_piece(F&& f) const
    {
        if constexpr (Held) {
#pragma unroll
            for (int p = 0; p < NP; ++p)
                if (p < pieces) f(held[p], index(p));
        } else {
            constexpr int kAhead = 4;
            for (int p0 = 0; p0 < pieces; p0 += kAhead) {
                uint4 r[kAhead];
#pragma unroll
                for (int y = 0; y < kAhead; ++y) r[y] = fetch(min(p0 + y, pieces - 1));
#pragma unroll
                for (int y = 0; y < kAhead; ++y)
                    if (p0 + y < pieces) f(mended(r[y], p0 + y), index(p0 + y));
            }
        }
    }
    // f(logit, index)
    template <typename F> __device__ __forceinline__ void each(F&& f) const
    {
        each_piece([&](const uint4& r, int i) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f(RowPiece<T>::value(r, e), i + e);
        });
    }
};

// Which tokens are kept: those with a logit above x, and of those with x the ones up to index i.
struct Cut {
    float x;
    int i;
    __device__ __forceinline__ bool keeps(float y, int j) const { return y > x || (y == x && j <= i); }
};

__device__ __forceinline__ u64 wave_upto(u64 v, int lane)
{
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const u64 up = __shfl_up(v, o, kWave);
        if (lane >= o) v += up;
    }
    return v;
}

// The token at which the sum of amount(logit, index), in order of the indices, first exceeds target_of(total); there is one.  Its sum
// is left in lds.amount and the total returned.  By all threads; lds.sums and what follows it is free before and after.
template <typename T, bool Held, typename A, typename G>
__device__ __forceinline__ int locate(const Row<T, Held>& row, SampleLds& lds, A&& amount, G&& target_of, u64* total_out)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    u64 s = 0;
    row.each([&](float x, int i) __attribute__((always_inline)) { s += amount(x, i); });
    s = wave_sum(s);
    if (lane == 0) lds.sums[wave] = s;
    __syncthreads();
    u64 total = 0;
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) total += lds.sums[w];
    const u64 target = target_of(total);
    u64 before = 0;
    int owner = 0;
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) {
        const bool past = before + lds.sums[w] <= target && owner == w;      // (all runs up to this one, and not yet there)
        if (past) { before += lds.sums[w]; owner = w + 1; }
    }
    owner = min(owner, kRowWaves - 1);
    __syncthreads();
    // that run once more, shared out among all threads
    const int each = (row.span() + kRowThreads - 1) / kRowThreads;
    const int begin = owner * row.span() + tid * each, end = min(min(begin + each, (owner + 1) * row.span()), row.V);
    u64 mine = 0;
    for (int i = begin; i < end; ++i) mine += amount(logit_to_float(row.at[i]), i);
    const u64 upto = wave_upto(mine, lane);
    if (lane == kWave - 1) lds.sums[wave] = upto;
    __syncthreads();
    u64 base = before;
    for (int w = 0; w < wave; ++w) base += lds.sums[w];
    u64 at = base + upto - mine;
    if (at <= target && target < base + upto) {
        for (int i = begin; i < end; ++i) {
            const u64 a = amount(logit_to_float(row.at[i]), i);
            if (target < at + a) { lds.found = i; lds.amount = a; break; }
            at += a;
        }
    }
    __syncthreads();
    *total_out = total;
    return lds.found;
}

// The histogram's bin, from bin 0 on, with which the sum first reaches what target_of(total) says.  lds.before: the sum before it.
template <typename G>
__device__ __forceinline__ int reach(SampleLds& lds, G&& target_of, u64* target_out)
{
    constexpr int PER = kBins / kRowThreads;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    u64 h[PER], s = 0;
#pragma unroll
    for (int y = 0; y < PER; ++y) s += h[y] = lds.hist[PER * tid + y];
    const u64 upto = wave_upto(s, lane);
    if (lane == kWave - 1) lds.sums[wave] = upto;
    __syncthreads();
    u64 base = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) {
        if (w == wave) base = total;
        total += lds.sums[w];
    }
    const u64 target = target_of(total);
    u64 at = base + upto - s;
    if (at < target && target <= base + upto) {
#pragma unroll
        for (int y = 0; y < PER; ++y) {
            if (at < target && target <= at + h[y]) { lds.found = PER * tid + y; lds.before = at; }
            at += h[y];
        }
    }
    __syncthreads();
    *target_out = target;
    return lds.found;
}

__device__ __forceinline__ void clear_bins(SampleLds& lds)
{
#pragma unroll
    for (int y = 0; y < kBins / kRowThreads; ++y) lds.hist[y * kRowThreads + threadIdx.x] = 0;
    if (threadIdx.x == 0) lds.n_listed = 0;
    __syncthreads();
}

// The cut within `cut` at which the sum of amount(logit), taken in the tokens' order, first reaches target_of(total).  `range`: distance
// to the maximum that the bins share out.
template <typename T, bool Held, typename A, typename G>
__device__ __forceinline__ Cut select(const Row<T, Held>& row, SampleLds& lds, Cut cut, float top, float range, A&& amount, G&& target_of)
{
    const int tid = threadIdx.x;
    const float scale = range > 1e-30f ? (float)(kBins - 1) / range : 0.0f;
    // (roundings keep the order, so bins are in it; a distance of infinity times a scale of zero is a NaN, which fminf passes over)
    auto bin_of = [=](float x) __attribute__((always_inline)) -> int { return (int)fminf((top - x) * scale, (float)(kBins - 1)); };
    clear_bins(lds);
    row.each([&](float x, int i) __attribute__((always_inline)) {
        if (cut.keeps(x, i)) atomicAdd(&lds.hist[bin_of(x)], amount(x));
    });
    __syncthreads();
    u64 target;
    const int bin = reach(lds, target_of, &target);
    u64 before = lds.before;
    row.each([&](float x, int i) __attribute__((always_inline)) {
        if (cut.keeps(x, i) && bin_of(x) == bin) {
            const int n = atomicAdd(&lds.n_listed, 1);
            if (n < kListed) lds.list[n] = Listed{ x, i, amount(x) };
        }
    });
    __syncthreads();
    const int n = lds.n_listed;
    if (n <= kListed) {
        if (tid < n) {
            const Listed me = lds.list[tid];
            u64 at = before;
            for (int y = 0; y < n; ++y) {
                const Listed l = lds.list[y];
                if (l.x > me.x || (l.x == me.x && l.i < me.i)) at += l.amount;
            }
            if (at < target && target <= at + me.amount) { lds.cut_x = me.x; lds.cut_i = me.i; }
        }
        __syncthreads();
        return Cut{ lds.cut_x, lds.cut_i };
    }
    // too many: by the bits of the logits, eleven at a time, from the highest value down
    __syncthreads();                                               // (all have seen n)
    uint32_t known = 0u;                                           // the bits so far
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t digits = pass == 2 ? 1023u : 2047u, high = pass == 0 ? 0u : pass == 1 ? 0xffe00000u : 0xfffffc00u;
        clear_bins(lds);
        row.each([&](float x, int i) __attribute__((always_inline)) {
            const uint32_t key = ordered_bits(x);
            if (cut.keeps(x, i) && bin_of(x) == bin && (key & high) == known) atomicAdd(&lds.hist[digits - ((key >> shift) & digits)], amount(x));
        });
        __syncthreads();
        u64 unused;
        const u64 rest = target - before;
        const int digit = reach(lds, [=](u64) { return rest; }, &unused);
        known |= (digits - (uint32_t)digit) << shift;
        before += lds.before;
        __syncthreads();
    }
    const float x_cut = __uint_as_float(known & 0x80000000u ? known ^ 0x80000000u : ~known);
    const u64 each = amount(x_cut), last = (target - before + each - 1) / each - 1;      // so many equal ones are before the last that is kept
    u64 unused;
    const int i_cut = locate(row, lds, [=](float x, int i) -> u64 { return x == x_cut && cut.keeps(x, i); }, [=](u64) { return last; }, &unused);
    return Cut{ x_cut, i_cut };
}

template <typename T, bool Held, int S>
__global__ __launch_bounds__(kRowThreads) void sample_kernel(SampleArgs<S>)
{
    const SampleArgs<S>& a = *(const SampleArgs<S>*)(__attribute__((address_space(4))) const SampleArgs<S>*)__builtin_amdgcn_kernarg_segment_ptr();
    __shared__ SampleLds lds;
    constexpr int VEC = RowPiece<T>::kTokens;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = blockIdx.x;
    Row<T, Held> row;
    row.at = static_cast<const T*>(a.logits) + r * a.stride;
    row.V = a.V;
    row.pieces = (a.V + kRowThreads * VEC - 1) / (kRowThreads * VEC);
    row.first = wave * row.span() + lane * VEC;
    row.load();
    const int seq = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < a.n_seq && r >= a.row0[lane < a.n_seq ? lane : 0])) - 1;
    const Filter filter = a.filter[seq];
    // ---- the largest logit, the smallest finite one; a row with a NaN or +inf, or without a finite logit, has no distribution
    float hi = -INFINITY, lo = INFINITY;
    int odd = 0;
    row.each([&](float x, int i) __attribute__((always_inline)) {
        odd |= !(x < INFINITY) && i < a.V;
        hi = fmaxf(hi, x);
        lo = fminf(lo, x > -INFINITY ? x : INFINITY);
    });
    hi = wave_max(hi);
    lo = -wave_max(-lo);
    odd = __any(odd);
    if (lane == 0) { lds.hi[wave] = hi; lds.lo[wave] = lo; lds.odd[wave] = odd; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) { hi = fmaxf(hi, lds.hi[w]); lo = fminf(lo, lds.lo[w]); odd |= lds.odd[w]; }
    const float top = hi;
    const bool none = odd || !(top > -INFINITY);
    Cut cut{ -INFINITY, a.V };
    const double per_nat = 1.4426950408889634074 / (double)filter.temperature;
    auto weight = [=](float x) __attribute__((always_inline)) -> u64 { return weight_of(((double)x - (double)top) * per_nat); };
    if (none) {
        cut = Cut{ INFINITY, -1 };
    } else if (filter.temperature == 0.0f) {
        u64 unused;
        cut = Cut{ top, locate(row, lds, [=](float x, int) -> u64 { return x == top; }, [](u64) -> u64 { return 0; }, &unused) };
    } else {
        if (filter.top_k > 0 && filter.top_k < a.V) {
            const u64 k = (u64)filter.top_k;
            cut = select(row, lds, cut, top, fminf(top - lo, 64.0f), [](float) -> u64 { return 1; }, [=](u64) { return k; });
        }
        if (filter.top_p < 1.0f) {
            const double p = (double)filter.top_p;
            // (kept: what has less than p of the sum before it)
            cut = select(row, lds, cut, top, fminf(top - lo, 32.0f * filter.temperature), weight,
                         [=](u64 total) -> u64 { return max((u64)1, (u64)ceil(p * (double)total)); });
        }
        if (filter.min_p > 0.0f) {
            // the smallest logit whose weight, as a number of 64 bits, is min_p or more (those within 2^-54 of 1 are 1)
            const double least = log2((double)filter.min_p) - 0x1p-54;
            const float near = (float)((double)top + least / per_nat);
            uint32_t key = max(ordered_bits(near), ordered_bits(-3.402823466e38f) + 2u) - 2u;
            float x;
            for (;; ++key) {
                x = __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
                if (((double)x - (double)top) * per_nat >= least || x >= top) break;
            }
            if (x > cut.x) cut = Cut{ x, a.V };
        }
    }
    if (a.out) {
        T* const out = static_cast<T*>(a.out) + r * a.out_stride;
        constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : 0xff80u;      // -inf
        __syncthreads();                                           // (in place: every thread has read what it wants of others)
        row.each_piece([&](const uint4& in, int i) __attribute__((always_inline)) {
            uint4 w = in;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const bool keep = cut.keeps(RowPiece<T>::value(in, e), i + e);
                if constexpr (sizeof(T) == 4) (&w.x)[e] = keep ? (&w.x)[e] : kNone;
                else if (!keep) (&w.x)[e / 2] = (e & 1) ? ((&w.x)[e / 2] & 0xffffu) | kNone << 16 : ((&w.x)[e / 2] & 0xffff0000u) | kNone;
            }
            if (i + VEC <= a.V) {
                typedef typename Unaligned<T>::Piece raw;
                *reinterpret_cast<raw*>(out + i) = raw{ w.x, w.y, w.z, w.w };
            } else {
                for (int e = 0; e < VEC && i + e < a.V; ++e) {
                    if constexpr (sizeof(T) == 4) out[i + e] = __uint_as_float((&w.x)[e]);
                    else out[i + e] = __builtin_bit_cast(__bf16, (unsigned short)((&w.x)[e / 2] >> (16 * (e & 1))));
                }
            }
        });
        return;
    }
    // ---- the draw
    if (none) {
        if (tid == 0) { a.token[r] = -1; a.prob[r] = 0.0f; a.n_kept[r] = 0; }
        return;
    }
    int kept = 0;
    row.each([&](float x, int i) __attribute__((always_inline)) { kept += __builtin_popcountll(__builtin_amdgcn_ballot_w64(cut.keeps(x, i))); });
    if (lane == 0) lds.counts[wave] = kept;
    int token;
    u64 total, mine;
    if (filter.temperature == 0.0f) {
        __syncthreads();
        token = cut.i;
        total = mine = 1;
    } else {
        const double u = (double)fminf(fmaxf(a.uniform[r], 0.0f), 1.0f - 0x1p-24f);
        token = locate(row, lds, [=](float x, int i) __attribute__((always_inline)) -> u64 { return cut.keeps(x, i) ? weight(x) : 0; },
                       [=](u64 total) -> u64 { return (u64)(u * (double)total); }, &total);
        mine = lds.amount;
    }
    if (tid == 0) {
        int n = 0;
        for (int w = 0; w < kRowWaves; ++w) n += lds.counts[w];
        a.token[r] = token;
        a.prob[r] = (float)((double)mine / (double)total);
        a.n_kept[r] = n;
    }
}

template <typename T, bool Held, int S>
static hipError_t launch_rows(const SampleHead& head, const int* row0, const Filter* filter, hipStream_t stream)
{
    static Kernel kernel(reinterpret_cast<const void*>(&sample_kernel<T, Held, S>));
    SampleArgs<S> a;
    static_cast<SampleHead&>(a) = head;
    for (int s = 0; s < head.n_seq; ++s) { a.row0[s] = row0[s]; a.filter[s] = filter[s]; }
    return kernel.launch(dim3(head.rows), kRowThreads, 0, stream, a);
}
template <typename T, bool Held>
static hipError_t launch_rows(const SampleHead& head, const int* row0, const Filter* filter, hipStream_t stream)
{
    return head.n_seq <= 8 ? launch_rows<T, Held, 8>(head, row0, filter, stream) : launch_rows<T, Held, DYSPEC_MAX_SEQ>(head, row0, filter, stream);
}
template <typename T>
static hipError_t launch_rows(const SampleHead& head, const int* row0, const Filter* filter, bool held, hipStream_t stream)
{
    return held ? launch_rows<T, true>(head, row0, filter, stream) : launch_rows<T, false>(head, row0, filter, stream);
}

hipError_t launch_sample(const SampleHead& a, const int* row0, const Filter* filter, int dtype, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    const bool held = a.V <= kHeldTokens * kRowThreads;
    return dtype == DYSPEC_F32 ? launch_rows<float>(a, row0, filter, held, stream) : launch_rows<__bf16>(a, row0, filter, held, stream);
}

hipError_t prepare_sample()                      // (asking loads the code)
{
    hipFunction_t f;
    return Kernel(reinterpret_cast<const void*>(&sample_kernel<float, true, 8>)).find(&f);
}

}  // namespace dyspec
