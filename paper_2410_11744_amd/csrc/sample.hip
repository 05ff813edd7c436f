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
// is kept, and the tokens of that bin one by one: each adds up those before it.  A bin with more than kRanked tokens (equal logits,
// or masks of the type's lowest value) is gone through by the bits of its logits instead, and equal ones by index.
//
// Passes over the whole row cost most (a compute unit has 32000 tokens of it), so a draw makes a list of the tokens that can be kept, in
// order of their indices, once the first cut's bin is known: what follows goes over the list if that has up to kListMost tokens.
//
// A workgroup has one row, held in registers up to 32768 tokens, else read again for every pass; each of its 16 waves has a run of
// the vocabulary, so that sums over waves, and then over the threads of one run, find a place in the order of the indices.
//
// What bounds it: the CU that has the row, and its passes one after the other.  A weight takes 24 instructions, most of 64 bits, a pass over
// 32000 of them 6 us, one that counts or compares 1 to 2; eleven barriers a draw.  2517 rows of bf16 with eight sequences' settings 125 to 129 us
// (vector unit issuing 68 % of the cycles).  512 rows of 32000 fp32 through top-p 40.8 us (131 MB, 3.2 TB/s of the 5.2 that a copy reaches; the
// vector unit 45 %): two rows a CU that start together, so that loads, weights and stores come in turn.  One token 12.9 us, 64 tokens of
// mixed settings 18.2.  Rows above 32768 tokens are read again for every pass: one row of 131072 fp32 through top-p 64 us, drawn from 109.
#include "sample.h"

#include "lane_ops.h"
#include "launch.h"
#include "min_p_cut.h"
#include "vocab_common.h"

namespace dyspec {

constexpr int kMostWaves = 16;
constexpr int kHeldTokens = 32768;               // rows up to that are held in registers
constexpr int kBins = 2048, kRanked = 1024;      // kRanked: tokens of a bin that are looked at one by one
constexpr int kListMost = 4096;
constexpr int kRankAll = 128;                    // of a list that short every token is, without a histogram
constexpr int kWeightBits = 45;                  // the largest weight is 2^kWeightBits: 2^18 of them stay below 2^63
static_assert(DYSPEC_MAX_SAMPLE_VOCAB <= 1 << (63 - kWeightBits), "sums fit");
static_assert(kMostWaves == 16, "what the waves leave is gone through by a row of 16 lanes");

struct Token { float x; int i; };
struct Ranked { float x; int i; u64 amount; };

struct SampleLds {
    u64 hist[kBins];
    Ranked ranked[kRanked];
    u64 in_front[kRanked];                       // of a token in `ranked`: the amounts of those in front of it
    u64 sums[kMostWaves];                        // (what a smaller workgroup has no wave for stays zero)
    float hi[kMostWaves], lo[kMostWaves];
    int odd[kMostWaves], counts[kMostWaves], kept[kMostWaves];
    u64 before;                                  // of a bin: the sum up to it
    u64 amount;                                  // of a token
    int found, n_ranked;
    Token cut;
    Token list[kListMost];
};

template <typename T> struct RowPiece;           // 16 bytes of a row
template <> struct RowPiece<float> {
    static constexpr int kTokens = 4;
    static __device__ __forceinline__ float value(const uint4& r, int e) { return __uint_as_float((&r.x)[e]); }
};
template <> struct RowPiece<__bf16> {
    static constexpr int kTokens = 8;
    static __device__ __forceinline__ float value(const uint4& r, int e) { const uint32_t w = (&r.x)[e / 2]; return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16); }
};

// (without the moves that fmaxf and fminf make to quiet NaN)
__device__ __forceinline__ float max3(float x, float y, float z) { asm("v_max3_f32 %0, %0, %1, %2" : "+v"(x) : "v"(y), "v"(z)); return x; }
__device__ __forceinline__ float min3(float x, float y, float z) { asm("v_min3_f32 %0, %0, %1, %2" : "+v"(x) : "v"(y), "v"(z)); return x; }

// (of 64 bits, as an operand that takes no vector registers)
__device__ __forceinline__ double constant(double c) { asm("" : "+s"(c)); return c; }

// exp2(z) in whole numbers of 2^-kWeightBits, z <= 0.  The fraction's power by a polynomial through Chebyshev's nodes, to 3.7e-14.
__device__ __forceinline__ u64 weight_of(double z)
{
    const double shift = constant(6755399441055744.0);         // 1.5 * 2^52: the sum's low bits are the nearest whole number
    z = fmax(z, -100.0);
    const double t = z + shift, f = z - (t - shift);
    const int n = (int)__double2loint(t);
    double p = constant(1.0203121063391729e-07);
    p = fma(p, f, constant(1.3255224878668817e-06));
    p = fma(p, f, constant(1.525268684626772e-05));
    p = fma(p, f, constant(0.00015403455852453838));
    p = fma(p, f, constant(0.0013333558179043112));
    p = fma(p, f, constant(0.009618129159402558));
    p = fma(p, f, constant(0.055504108664760424));
    p = fma(p, f, constant(0.2402265069581299));
    p = fma(p, f, constant(0.6931471805599453));
    p = fma(p, f, 1.0);
    // times 2^(n + kWeightBits) by the exponent's bits; + 2^52: rounded to a whole number in the low bits
    const double w = __hiloint2double(__double2hiint(p) + ((n + kWeightBits) << 20), __double2loint(p)) + constant(4503599627370496.0);
    return (u64)__double_as_longlong(w) & 0xfffffffffffffull;
}

// A row as a thread has it.  Wave w has tokens w * span .. of the row, lane l of it the kTokens from w * span + (64 p + l) * kTokens
// on, p < pieces.  Places past the row's end hold a NaN, which no comparison keeps.
template <typename T, bool Held, int NT> struct Row {
    static constexpr int VEC = RowPiece<T>::kTokens, NP = Held ? kHeldTokens / NT / VEC : 1;
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
            for (int p = 0; p < NP; ++p) {
                int i = index(p);
                asm volatile("" : "+v"(i));
                if (p < pieces) f(held[p], i);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            constexpr int kAhead = 4;
#pragma unroll 1
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
    // f(logit, index).  (What a pass makes of a logit is made anew by the next: kept from one to the other it would not fit the registers.)
    template <typename F> __device__ __forceinline__ void each(F&& f) const
    {
        each_piece([&](const uint4& r, int i) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float x = RowPiece<T>::value(r, e);
                asm volatile("" : "+v"(x));
                f(x, i + e);
                if (e & 1) __builtin_amdgcn_sched_barrier(0);      // (two at a time: more chains of weights side by side would not fit either)
            }
        });
    }
};

// The list, of which a thread has a token or a few, one after the other.
struct List {
    const Token* at;
    int n, each_n;                               // tokens of the list, of a thread

    // f(logit, index); NaN where a thread has none
    template <typename F> __device__ __forceinline__ void each(F&& f) const
    {
#pragma unroll 1
        for (int y = 0; y < each_n; ++y) {
            const int to = (int)threadIdx.x * each_n + y;
            const Token k = at[min(to, kListMost - 1)];
            f(to < n ? k.x : __uint_as_float(~0u), k.i);
        }
    }
};

// Which tokens are kept: those with a logit above x, and of those with x the ones up to index i.
struct Cut {
    float x;
    int i;
    __device__ __forceinline__ bool keeps(float y, int j) const { return (y > x) | ((y == x) & (j <= i)); }
};

// Even steps of the distance to the maximum.  Roundings keep the order, so the bins are in it; a distance of infinity times a scale of
// zero is a NaN, which fminf passes over, and so is what stands where there is no token: the last bin, at a weight of zero.
struct Bins {
    float top, scale;
    __device__ __forceinline__ Bins(float top, float range) : top(top), scale(uniform(range > 1e-30f ? (float)(kBins - 1) / range : 0.0f)) {}
    __device__ __forceinline__ int of(float x) const { return (int)fminf((top - x) * scale, (float)(kBins - 1)); }
    // no token of the bins up to this one is below, none of it above (a few of the bins beside it may lie between)
    __device__ __forceinline__ float least(int bin) const
    {
        if (bin == kBins - 1 || scale == 0.0f) return -INFINITY;
        return uniform(top - (float)(bin + 1) / scale * (1.0f + 0x1p-20f) - fabsf(top) * 0x1p-22f);
    }
    __device__ __forceinline__ float most(int bin) const
    {
        return bin == 0 ? top : uniform(top - (float)bin / scale * (1.0f - 0x1p-20f) + fabsf(top) * 0x1p-22f);
    }
};

template <int CTRL, int ROW_MASK = 0xf> __device__ __forceinline__ u64 dpp_or_zero(u64 x)
{
    return (u64)(uint32_t)dpp_or_zero<CTRL, ROW_MASK>((int)(x >> 32)) << 32 | (uint32_t)dpp_or_zero<CTRL, ROW_MASK>((int)x);
}
// The sum over the lanes of a row of 16 up to this one; of the wave.
template <typename N> __device__ __forceinline__ N row_upto(N x)
{
    x += dpp_or_zero<0x111>(x);
    x += dpp_or_zero<0x112>(x);
    x += dpp_or_zero<0x114>(x);
    x += dpp_or_zero<0x118>(x);
    return x;
}
__device__ __forceinline__ u64 wave_upto(u64 x)
{
    x = row_upto(x);
    x += dpp_or_zero<kDppBcast15, 0xa>(x);
    x += dpp_or_zero<kDppBcast31, 0xc>(x);
    return x;
}
__device__ __forceinline__ int of_lane(int x, int l) { return __builtin_amdgcn_readlane(x, l); }
__device__ __forceinline__ u64 of_lane(u64 x, int l) { return (u64)(uint32_t)of_lane((int)(x >> 32), l) << 32 | (uint32_t)of_lane((int)x, l); }
__device__ __forceinline__ float dpp_max(float x)              // of the row of 16
{
    auto with = [](float y, auto ctrl) { return fmaxf(y, __int_as_float(dpp_or_zero<decltype(ctrl)::value>(__float_as_int(y)))); };
    x = with(x, std::integral_constant<int, kDppXor1>{});
    x = with(x, std::integral_constant<int, kDppXor2>{});
    x = with(x, std::integral_constant<int, kDppHalfMirror>{});
    return with(x, std::integral_constant<int, kDppMirror>{});
}
__device__ __forceinline__ float wave_max_dpp(float x)
{
    x = dpp_max(x);
    return fmaxf(fmaxf(readlane_f32(x, 0), readlane_f32(x, 16)), fmaxf(readlane_f32(x, 32), readlane_f32(x, 48)));
}

// Of what the 16 waves left: the sum before this wave's, and of all.
template <typename N> __device__ __forceinline__ N before_wave(const N* left, int wave, N* total)
{
    const N upto = row_upto(left[threadIdx.x & 15]);
    *total = of_lane(upto, 15);
    return wave == 0 ? 0 : of_lane(upto, wave - 1);
}
// The sum of the threads' own up to and with this one's, and of all.  One barrier; lds.sums is free before.
__device__ __forceinline__ u64 block_upto(SampleLds& lds, u64 mine, u64* total)
{
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const u64 upto = wave_upto(mine);
    if (lane == kWave - 1) lds.sums[wave] = upto;
    __syncthreads();
    return before_wave(lds.sums, wave, total) + upto;
}

// The token at which the sum of amount(logit, index), in order of the indices, first exceeds target_of(total); there is one.  Its amount
// is left in lds.amount.  By all threads; lds.sums is free before and after.
template <typename T, bool Held, int NT, typename A, typename G>
__device__ __forceinline__ int locate(const Row<T, Held, NT>& row, SampleLds& lds, A&& amount, G&& target_of, u64* total)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    u64 s = 0;
    row.each([&](float x, int i) __attribute__((always_inline)) { s += amount(x, i); });
    s = wave_upto(s);
    if (lane == kWave - 1) lds.sums[wave] = s;
    __syncthreads();
    const u64 upto = row_upto(lds.sums[lane & 15]);
    *total = of_lane(upto, 15);
    const u64 target = target_of(*total);
    const int owner = min(__builtin_popcountll(ballot(upto <= target) & 0xffffull), NT / kWave - 1);      // the first run that goes past the target
    const u64 before = owner == 0 ? 0 : of_lane(upto, owner - 1);
    __syncthreads();
    // that run once more, shared out among all threads
    const int each = (row.span() + NT - 1) / NT;
    const int begin = owner * row.span() + tid * each, end = min(min(begin + each, (owner + 1) * row.span()), row.V);
    u64 mine = 0;
    for (int i = begin; i < end; ++i) mine += amount(logit_to_float(row.at[i]), i);
    u64 unused, at = before + block_upto(lds, mine, &unused) - mine;
    if (at <= target && target < at + mine) {
        for (int i = begin; i < end; ++i) {
            const u64 a = amount(logit_to_float(row.at[i]), i);
            if (target < at + a) { lds.found = i; lds.amount = a; break; }
            at += a;
        }
    }
    __syncthreads();
    return uniform(lds.found);
}
// The same of the list.
template <typename A, typename G>
__device__ __forceinline__ int locate(const List& list, SampleLds& lds, A&& amount, G&& target_of, u64* total)
{
    u64 mine = 0;
    list.each([&](float x, int i) __attribute__((always_inline)) { mine += amount(x, i); });
    u64 at = block_upto(lds, mine, total) - mine;
    const u64 target = target_of(*total);
    if (at <= target && target < at + mine)
        list.each([&](float x, int i) __attribute__((always_inline)) {
            const u64 a = amount(x, i);
            if (at <= target && target < at + a) { lds.found = i; lds.amount = a; }
            at += a;
        });
    __syncthreads();
    return uniform(lds.found);
}

// The histogram's bin, from bin 0 on, with which the sum first reaches what target_of(total) says (the last one, where that is not
// reached).  lds.before: the sum before it.
template <int NT, typename G>
__device__ __forceinline__ int reach(SampleLds& lds, G&& target_of, u64* target)
{
    constexpr int PER = kBins / NT;
    u64 h[PER], s = 0;
#pragma unroll
    for (int y = 0; y < PER; ++y) s += h[y] = lds.hist[PER * threadIdx.x + y];
    u64 total, at = block_upto(lds, s, &total) - s;
    *target = target_of(total);
    if (at < *target && *target <= at + s) {
#pragma unroll
        for (int y = 0; y < PER; ++y) {
            if (at < *target && *target <= at + h[y]) { lds.found = PER * threadIdx.x + y; lds.before = at; }
            at += h[y];
        }
    }
    if (total < *target && threadIdx.x == NT - 1) { lds.found = kBins - 1; lds.before = total - h[PER - 1]; }      // (the last bin is not filled whole)
    __syncthreads();
    return uniform(lds.found);
}
template <int NT> __device__ __forceinline__ void clear_bins(SampleLds& lds)     // (a barrier follows)
{
#pragma unroll
    for (int y = 0; y < kBins / NT; ++y) lds.hist[y * NT + threadIdx.x] = 0;
    if (threadIdx.x == 0) lds.n_ranked = 0;
}

// Of the n tokens in lds.ranked, their amounts to be filled in: the one with which `before` and the amounts of those in front of it first
// reach the target.  A lane has a token, the waves share out those that it is compared with.
template <int NT, typename A>
__device__ __forceinline__ Cut rank(SampleLds& lds, int n, u64 before, u64 target, A&& amount)
{
    constexpr int NW = NT / kWave;
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    for (int y = threadIdx.x; y < n; y += NT) {
        lds.ranked[y].amount = amount(lds.ranked[y].x, lds.ranked[y].i);
        lds.in_front[y] = 0;
    }
    __syncthreads();
    const int share = (n + NW - 1) / NW, from = wave * share, to = min(from + share, n);
#pragma unroll 1
    for (int c = 0; c < n; c += kWave) {
        const Ranked me = lds.ranked[min(c + lane, n - 1)];
        u64 front = 0;
        constexpr int kAhead = 4;                                  // (a read of LDS takes longer than looking at what came)
#pragma unroll 1
        for (int y0 = from; y0 < to; y0 += kAhead) {
            Ranked l[kAhead];
#pragma unroll
            for (int y = 0; y < kAhead; ++y) l[y] = lds.ranked[min(y0 + y, n - 1)];
#pragma unroll
            for (int y = 0; y < kAhead; ++y)
                front += (y0 + y < to) & ((l[y].x > me.x) | ((l[y].x == me.x) & (l[y].i < me.i))) ? l[y].amount : 0;
        }
        if (front != 0 && c + lane < n) atomicAdd(&lds.in_front[c + lane], front);
    }
    __syncthreads();
    for (int y = threadIdx.x; y < n; y += NT) {
        const u64 at = before + lds.in_front[y];
        if (at < target && target <= at + lds.ranked[y].amount) lds.cut = Token{ lds.ranked[y].x, lds.ranked[y].i };
    }
    __syncthreads();
    return Cut{ uniform(lds.cut.x), uniform(lds.cut.i) };
}

// The cut inside a bin: where, with `before` before the bin, the sum of the amounts of its tokens first reaches the target.  src: the row
// or the list, of which `cut` says what counts.
template <typename T, bool Held, int NT, typename Src, typename A>
__device__ __forceinline__ Cut resolve(const Row<T, Held, NT>& row, const Src& src, SampleLds& lds, const Cut& cut, const Bins& bins, int bin, u64 before, u64 target, A&& amount)
{
    const float least = bins.least(bin), most = bins.most(bin);
    src.each([&](float x, int i) __attribute__((always_inline)) {
        if ((x >= least) & (x <= most)) {
            if (cut.keeps(x, i) & (bins.of(x) == bin)) {
                const int n = atomicAdd(&lds.n_ranked, 1);
                if (n < kRanked) { lds.ranked[n].x = x; lds.ranked[n].i = i; }
            }
        }
    });
    __syncthreads();
    const int n = uniform(lds.n_ranked);
    if (n <= kRanked) return rank<NT>(lds, n, before, target, [=](float x, int) { return amount(x); });
    // too many: by the bits of the logits, eleven at a time, from the highest value down
    __syncthreads();                                               // (all have seen n)
    uint32_t known = 0u;                                           // the bits so far
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t digits = pass == 2 ? 1023u : 2047u, high = pass == 0 ? 0u : pass == 1 ? 0xffe00000u : 0xfffffc00u;
        clear_bins<NT>(lds);
        __syncthreads();
        src.each([&](float x, int i) __attribute__((always_inline)) {
            const uint32_t key = ordered_bits(x);
            if (cut.keeps(x, i) & (bins.of(x) == bin) & ((key & high) == known)) atomicAdd(&lds.hist[digits - ((key >> shift) & digits)], amount(x));
        });
        __syncthreads();
        u64 unused;
        const u64 rest = target - before;
        const int digit = reach<NT>(lds, [=](u64) { return rest; }, &unused);
        known |= (digits - (uint32_t)digit) << shift;
        before += uniform(lds.before);
        __syncthreads();
    }
    const float x_cut = of_ordered_bits(known);
    const u64 each = amount(x_cut), last = (target - before + each - 1) / each - 1;      // so many equal ones are before the last that is kept
    u64 unused;
    const Cut within = cut;
    return Cut{ x_cut, locate(row, lds, [=](float x, int i) -> u64 { return (x == x_cut) & within.keeps(x, i); }, [=](u64) { return last; }, &unused) };
}

// The tokens with a logit of `least` or more, in order of their indices, if they are kListMost or fewer.
template <typename T, bool Held, int NT>
__device__ __forceinline__ bool make_list(const Row<T, Held, NT>& row, SampleLds& lds, float least, List& list)
{
    constexpr int VEC = RowPiece<T>::kTokens;
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    int mine = 0;
    row.each([&](float x, int) __attribute__((always_inline)) { mine += __builtin_popcountll(ballot(x >= least)); });
    if (lane == 0) lds.counts[wave] = mine;
    __syncthreads();
    int at = before_wave(lds.counts, wave, &list.n);
    __syncthreads();
    list.at = lds.list;
    list.each_n = (list.n + NT - 1) / NT;
    if (list.n > kListMost) return false;
    row.each_piece([&](const uint4& r, int i) __attribute__((always_inline)) {
        // (before this piece's tokens of this lane: those of earlier pieces, those of lower lanes)
        int place = at;
        u64 any = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            float x = RowPiece<T>::value(r, e);
            asm volatile("" : "+v"(x));
            const u64 there = ballot(x >= least);
            any |= there;
            place = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(there >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)there, (uint32_t)place));
            at += __builtin_popcountll(there);
        }
        if (any != 0) {                                            // (the same for the wave)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float x = RowPiece<T>::value(r, e);
                asm volatile("" : "+v"(x));
                if (x >= least) lds.list[place++] = Token{ x, i + e };
            }
        }
    });
    __syncthreads();
    return true;
}

// Drawn: a token is drawn; else the filtered logits are written.  WAVES: of a SIMD, for which registers are left.
template <typename T, bool Held, bool Drawn, int NT, int WAVES, int S>
__global__ __launch_bounds__(NT, WAVES) void sample_kernel(SampleArgs<S>)
{
    const SampleArgs<S>& a = *(const SampleArgs<S>*)(__attribute__((address_space(4))) const SampleArgs<S>*)__builtin_amdgcn_kernarg_segment_ptr();
    __shared__ SampleLds lds;
    constexpr int VEC = RowPiece<T>::kTokens;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int r = blockIdx.x;
    Row<T, Held, NT> row;
    row.at = static_cast<const T*>(a.logits) + r * a.stride;
    row.V = a.V;
    row.pieces = (a.V + NT * VEC - 1) / (NT * VEC);
    row.first = wave * row.span() + lane * VEC;
    row.load();
    const int seq = __builtin_popcountll(ballot(lane < a.n_seq && r >= a.row0[lane < a.n_seq ? lane : 0])) - 1;
    const Filter filter = a.filter[seq];
    clear_bins<NT>(lds);
    if (NT / kWave < kMostWaves && tid >= NT / kWave && tid < kMostWaves) {      // what is left for waves that are not there
        lds.sums[tid] = 0;
        lds.counts[tid] = lds.kept[tid] = lds.odd[tid] = 0;
        lds.hi[tid] = -INFINITY; lds.lo[tid] = INFINITY;
    }
    // ---- the largest logit and the smallest; a row with a NaN or +inf, or without a finite logit, has no distribution
    float hi = -INFINITY, lo = INFINITY;
    bool odd = false;
    row.each_piece([&](const uint4& p, int i) __attribute__((always_inline)) {
        bool nan = false;
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
            const float x = RowPiece<T>::value(p, e), y = RowPiece<T>::value(p, e + 1);
            nan |= (x != x) | (y != y);
            hi = max3(hi, x, y);
            lo = min3(lo, x, y);
        }
        if (i + VEC <= a.V) odd |= nan;
        else
            for (int e = 0; e < VEC && i + e < a.V; ++e) {
                const float x = logit_to_float(row.at[i + e]);
                odd |= x != x;
            }
    });
    const float mine_hi = hi;                                      // of this thread's tokens
    hi = wave_max_dpp(hi);
    lo = -wave_max_dpp(-lo);
    const bool any_odd = ballot(odd) != 0;
    if (lane == 0) { lds.hi[wave] = hi; lds.lo[wave] = lo; lds.odd[wave] = any_odd; }
    __syncthreads();
    const float top = uniform(dpp_max(lds.hi[lane & 15]));
    lo = uniform(-dpp_max(-lds.lo[lane & 15]));
    const bool none = ballot(lds.odd[lane & 15] != 0) != 0 || !(fabsf(top) < INFINITY);
    const bool greedy = filter.temperature == 0.0f;
    Cut cut{ -INFINITY, a.V };
    List list;
    list.n = 0;
    bool listed = false;                                           // the list holds every token that is kept
    const double per_nat = filter.per_nat, top64 = uniform((double)top);
    auto weight = [=](float x) __attribute__((always_inline)) -> u64 { return weight_of(((double)x - top64) * per_nat); };
    if (none) {
        cut = Cut{ INFINITY, -1 };
    } else if (greedy) {
        int first = 0x7fffffff;
        row.each([&](float x, int i) __attribute__((always_inline)) { first = min(first, x == top ? i : 0x7fffffff); });
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) first = min(first, __shfl_xor(first, o, kWave));
        if (lane == 0) lds.counts[wave] = first;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NT / kWave; ++w) first = min(first, lds.counts[w]);
        cut = Cut{ top, uniform(first) };
    } else {
        bool cleared = true;
#pragma unroll 1
        for (int by_weight = 0; by_weight < 2; ++by_weight) {      // top-k's cut by ones, top-p's by weights
            if (by_weight ? !(filter.top_p < 1.0f) : filter.top_k == 0 || filter.top_k >= a.V) continue;
            auto amount = [=](float x) __attribute__((always_inline)) -> u64 { return by_weight ? weight(x) : 1; };
            // (top-p keeps what has less than its share of the sum before it)
            auto target_of = [=](u64 total) -> u64 { return by_weight ? max((u64)1, (u64)ceil((double)filter.top_p * (double)total)) : (u64)filter.top_k; };
            const Bins bins(top, fminf(top - lo, by_weight ? 32.0f * filter.temperature : 64.0f));
            if (!by_weight && filter.top_k <= NT) {
                // As many threads as tokens are wanted have a token that is as large as the top_k-th of the threads' largest: the
                // wanted ones are among the tokens that are that large.
                if (mine_hi > -INFINITY) atomicAdd(&lds.hist[bins.of(mine_hi)], (u64)1);
                __syncthreads();
                u64 target;
                const int bin = reach<NT>(lds, target_of, &target);
                listed = make_list(row, lds, bins.least(bin), list);
                clear_bins<NT>(lds);
                __syncthreads();
            }
            if (listed && list.n <= kRankAll) {                    // (a token a thread)
                const Token k = list.at[min(tid, kListMost - 1)];
                const u64 mine = tid < list.n && cut.keeps(k.x, k.i) ? amount(k.x) : 0;
                u64 total;
                block_upto(lds, mine, &total);
                if (tid < list.n) { lds.ranked[tid].x = k.x; lds.ranked[tid].i = k.i; }
                __syncthreads();
                cut = rank<NT>(lds, list.n, 0, target_of(total), [=](float x, int i) -> u64 { return cut.keeps(x, i) ? amount(x) : 0; });
                continue;
            }
            const bool whole = !listed && cut.x == -INFINITY && cut.i >= a.V;
            if (!cleared) {
                clear_bins<NT>(lds);
                __syncthreads();
            }
            cleared = false;
            // (what weighs nothing, or is masked, is most of some rows and would meet in the last bin: it is added to a bin of the thread's)
            auto add = [&](float x, u64 n) __attribute__((always_inline)) { atomicAdd(&lds.hist[n != 0 ? bins.of(x) : tid], n); };
            if (listed) list.each([&](float x, int i) __attribute__((always_inline)) { add(x, cut.keeps(x, i) ? amount(x) : 0); });
            else if (!whole) row.each([&](float x, int i) __attribute__((always_inline)) { add(x, cut.keeps(x, i) ? weight(x) : 0); });      // (top-k was first)
            else if (by_weight) row.each([&](float x, int) __attribute__((always_inline)) { add(x, weight(x)); });
            else row.each([&](float x, int) __attribute__((always_inline)) { add(x, top - x < 65.0f); });
            __syncthreads();
            u64 target;
            const int bin = reach<NT>(lds, target_of, &target);
            const u64 before = uniform(lds.before);
            if (Drawn && whole) listed = make_list(row, lds, bins.least(bin), list);
            if (listed) cut = resolve(row, list, lds, cut, bins, bin, before, target, amount);
            else cut = resolve(row, row, lds, cut, bins, bin, before, target, amount);
        }
        if (filter.min_p > 0.0f) {
            const float x = uniform(min_p_cut(top, filter.temperature, per_nat, filter.least, [] {}));
            if (x > cut.x) cut = Cut{ x, a.V };
        }
    }
    if constexpr (!Drawn) {
        T* const out = static_cast<T*>(a.out) + r * a.out_stride;
        constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : 0xff80u;      // -inf
        __syncthreads();                                           // (in place: every thread has read what it wants of others)
        auto leave = [&](const uint4& in, int i, auto ties_c) __attribute__((always_inline)) {
            constexpr bool ties = decltype(ties_c)::value;         // some of the equal ones at the cut go
            uint4 w = in;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float x = RowPiece<T>::value(in, e);
                const bool keep = ties ? cut.keeps(x, i + e) : x >= cut.x;
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
        };
        if (cut.i >= a.V) row.each_piece([&](const uint4& in, int i) __attribute__((always_inline)) { leave(in, i, std::false_type{}); });
        else row.each_piece([&](const uint4& in, int i) __attribute__((always_inline)) { leave(in, i, std::true_type{}); });
    } else {
        if (none || greedy) {
            if (tid == 0) { a.token[r] = none ? -1 : cut.i; a.prob[r] = none ? 0.0f : 1.0f; a.n_kept[r] = none ? 0 : 1; }
            return;
        }
        const bool whole = cut.x == -INFINITY && cut.i >= a.V;     // every token is kept
        if (!listed && cut.x > -INFINITY) listed = make_list(row, lds, cut.x, list);
        const double u = (double)fminf(fmaxf(a.uniform[r], 0.0f), 1.0f - 0x1p-24f);
        auto kept_weight = [=](float x, int i) __attribute__((always_inline)) -> u64 { return cut.keeps(x, i) ? weight(x) : 0; };
        auto target_of = [=](u64 total) -> u64 { return (u64)(u * (double)total); };
        int kept = 0;
        auto count = [&](float x, int i) __attribute__((always_inline)) { kept += __builtin_popcountll(ballot(cut.keeps(x, i))); };
        if (listed) list.each(count);
        else if (!whole) row.each(count);
        if (lane == 0) lds.kept[wave] = kept;
        u64 total;
        int token;
        if (listed) token = locate(list, lds, kept_weight, target_of, &total);
        else if (!whole) token = locate(row, lds, kept_weight, target_of, &total);
        else token = locate(row, lds, [=](float x, int) __attribute__((always_inline)) -> u64 { return weight(x); }, target_of, &total);
        int n;
        before_wave(lds.kept, 0, &n);
        if (tid == 0) {
            a.token[r] = token;
            a.prob[r] = (float)((double)lds.amount / (double)total);
            a.n_kept[r] = whole ? a.V : n;
        }
    }
}

template <typename T, bool Held, bool Drawn, int NT, int WAVES, int S>
static hipError_t launch_rows(const SampleHead& head, const int* row0, const Filter* filter, hipStream_t stream)
{
    static Kernel kernel(reinterpret_cast<const void*>(&sample_kernel<T, Held, Drawn, NT, WAVES, S>));
    SampleArgs<S> a;
    static_cast<SampleHead&>(a) = head;
    for (int s = 0; s < head.n_seq; ++s) { a.row0[s] = row0[s]; a.filter[s] = filter[s]; }
    return kernel.launch(dim3(head.rows), NT, 0, stream, a);
}
template <typename T, bool Held, bool Drawn, int NT, int WAVES>
static hipError_t launch_rows(const SampleHead& head, const int* row0, const Filter* filter, hipStream_t stream)
{
    return head.n_seq <= 8 ? launch_rows<T, Held, Drawn, NT, WAVES, 8>(head, row0, filter, stream) : launch_rows<T, Held, Drawn, NT, WAVES, DYSPEC_MAX_SEQ>(head, row0, filter, stream);
}
// A row's passes take turns with its waits, so where there are more rows than CUs two rows share one: of fp32 by workgroups of 512
// threads (512 rows of 32000 through top-p: 46.5 us with 1024 threads, 40.7 with 512), of bf16, held in half the registers, by the
// ones of 1024 with 64 registers a thread (2517 rows: 151 us with a CU each, 126; 134 with 512 threads).  One row alone is faster
// with 1024 threads and as many registers as they want (a draw of one token: 12.9 us, 14.7 with 64 registers, 14.6 with 512 threads).
// Draws have a CU a row however many there are; above 256 rows they would gain as well (32000 tokens through top-p, one and two rows a
// CU: fp32 300 rows 40.7 and 36.9 us, 754 65.5 and 57.8, 2048 164 and 127; bf16 512 rows 40.2 and 38.9, 2048 154 and 121), which is open.
constexpr int kCus = 256;
template <typename T, bool Held, bool Drawn>
static hipError_t launch_rows(const SampleHead& head, const int* row0, const Filter* filter, hipStream_t stream)
{
    if constexpr (Held && !Drawn)
        if (head.rows > kCus)
            return launch_rows<T, Held, Drawn, sizeof(T) == 4 ? 512 : 1024, sizeof(T) == 4 ? 4 : 8>(head, row0, filter, stream);
    return launch_rows<T, Held, Drawn, 1024, 4>(head, row0, filter, stream);
}
template <typename T>
static hipError_t launch_rows(const SampleHead& head, const int* row0, const Filter* filter, hipStream_t stream)
{
    const bool drawn = head.out == nullptr;
    if (head.V <= kHeldTokens)
        return drawn ? launch_rows<T, true, true>(head, row0, filter, stream) : launch_rows<T, true, false>(head, row0, filter, stream);
    return drawn ? launch_rows<T, false, true>(head, row0, filter, stream) : launch_rows<T, false, false>(head, row0, filter, stream);
}

hipError_t launch_sample(const SampleHead& a, const int* row0, const Filter* filter, int dtype, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    return dtype == DYSPEC_F32 ? launch_rows<float>(a, row0, filter, stream) : launch_rows<__bf16>(a, row0, filter, stream);
}

hipError_t prepare_sample()                      // (asking loads the code)
{
    hipFunction_t f;
    return Kernel(reinterpret_cast<const void*>(&sample_kernel<float, true, true, 1024, 4, 8>)).find(&f);
}

}  // namespace dyspec
