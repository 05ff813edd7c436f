// Attention of new tokens over pages or packed rows: which kernel takes which sequence, and how the walks are cut into items.
//
// bf16 with head_dim 64 or 128 goes to the bf16 matrix cores: attend_short.hip (blocks of 32 rows, the waves share out the keys)
// and attend_mfma.hip (blocks of 128 rows).  Everything else goes to attend_f32.hip.
#include "attend.h"

namespace dyspec {

// A kernel as the choice sees it: a launch, then items (workgroups).  One that has a CU to itself takes `once` and `step` per
// `keys` keys, more by the share `alone` over its sequence's row blocks (the first to read a key reads it from memory); of a CU
// that is full, with `per_cu` items, each takes up `busy_once` and `busy_step`.  Microseconds.  The bf16 kernels' are fitted to
// measurements, those of the fp32 kernel are estimates, the same for all head sizes above 64.  They are the costs of plain scores, by which
// capped ones (whose steps take up to a fifth longer) are dealt out as well.  How far the choice is from the best of
// all kernels, each whole and in 2 to 32 parts (1 to 64 sequences, 1 to 4096 new tokens, 0 to 16384 tokens of context, 1 to 32 KV heads, 1 to
// 8 query heads each; geometric mean, nine in ten, worst):
//   bf16, 128   pages (153 shapes) 1.3 %, 7 %, 35 %: 256 tokens over 16384, 8 heads on 1, 47.0 us against 34.8 by attend_short.hip in 4 parts
//               prompts (44) 1.5 %, 3.5 %, 23 %: six of 1500 to 20, 8 heads, 28.0 against 22.8 by attend_short.hip
//   bf16, 64    pages (153) 3.2 %, 10 %, 22 %; prompts (44) 1.4 %, 5 %, 9 %
//   fp32, 64    pages (95) 5.4 %, 18 %, 24 %; prompts (24) 1.1 %, 1.4 %, 18 %
//   fp32, 128   pages (95) 7.4 %, 25 %, 30 %: one token over 300 stays whole, 16.5 against 12.7 in 3 parts; prompts (24) 1.4 %, 1.7 %, 30 %
//   bf16, 80    pages (95) 6.2 %, 25 %, 29 %; prompts (24) 1.5 %, 1.6 %, 31 %
//   bf16, 256   pages (95) 7.3 %, 26 %, 47 %: 64 tokens over 1500, 32 heads on 8, 96.0 against 65.3 with 16 rows a block in 2 parts;
//               prompts (24) 2.3 %, 1.6 %, 35 %
enum AttendKind { kFew8, kFew4, kMany8, kMany4, kF32Few, kF32Many, kKinds };
struct KindCost { int rows, keys, per_cu; float launch, once, step, alone, busy_once, busy_step; };
constexpr KindCost kCosts[2][kKinds] = {
    // head_dim 128
    { { kFewRows, 32, 1, 3.5f, 3.0f, 0.26f, 0.4f, 4.0f, 0.20f }, { kFewRows, 32, 2, 3.8f, 3.0f, 0.36f, 0.1f, 2.7f, 0.21f },
      { kManyRows, 64, 1, 4.0f, 5.0f, 0.87f, 0.05f, 6.0f, 0.87f }, { kManyRows, 64, 2, 4.0f, 4.5f, 0.98f, 0.05f, 3.8f, 0.80f },
      { 16, 128, 2, 4.0f, 3.0f, 2.0f, 0.0f, 2.0f, 1.0f }, { 64, 32, 2, 4.0f, 3.0f, 1.7f, 0.0f, 2.0f, 0.85f } },
    // head_dim 64
    { { kFewRows, 32, 2, 3.5f, 2.5f, 0.155f, 0.5f, 2.2f, 0.115f }, { kFewRows, 32, 4, 3.3f, 1.9f, 0.25f, 0.1f, 1.2f, 0.12f },
      { kManyRows, 64, 1, 3.5f, 4.2f, 0.52f, 0.3f, 5.0f, 0.53f }, { kManyRows, 64, 3, 3.5f, 4.0f, 0.60f, 0.3f, 2.4f, 0.48f },
      { 16, 128, 3, 4.0f, 3.0f, 1.0f, 0.0f, 1.5f, 0.5f }, { 64, 32, 3, 4.0f, 3.0f, 0.85f, 0.0f, 1.5f, 0.43f } },
};
constexpr int kCus = 256;
constexpr float kBytesPerUs = 5.5e6f;          // K and V from memory
constexpr float kPartBytesPerUs = 2.5e6f;      // parts to memory and back
constexpr float kPartOnce = 3.0f;              // the arrival, and the last workgroup's trip
constexpr float kTail = 0.6f;                  // of the rounds of what is cut beside whole walks: it fills up the CUs that those leave
constexpr int kUnit = 128;                     // a share is a multiple of this many keys

static const KindCost& cost_of(const AttendArgs& a, AttendKind k) { return kCosts[a.d <= 64][k]; }

// A set of sequences (indices, longest walks first) for one kernel.  Walks are cut into shares of at most `share` keys, but for
// those of the first `whole` row blocks in the order of the launch, which leave no parts: the blocks of long prompts beside single
// tokens with long contexts (pieces of prompts of 700 and 331 tokens beside five that decode: 110 -> 87 us), or the first rounds
// of workgroups, where what is left after them is shared out (40 row blocks of 8 heads over 4700 tokens: 115 -> 109 us).
struct Set { AttendKind kind; int n, share, whole; int seq[DYSPEC_MAX_SEQ]; };

static int new_of(const AttendBatch& b, int s) { return b.row0[s + 1] - b.row0[s]; }
// Keys that the longest walk of a sequence's tokens before `to` has, in blocks of `rows` rows: with a window, those of a block's first row,
// what its other rows (with positions given: any row) have behind that, and the 63 before that it may begin with.
static int walk_of(const AttendArgs& a, const AttendBatch& b, int s, int to, int rows)
{
    if (a.window >= kNoWindow) return b.context[s] + to;
    return (int)min((long long)b.context[s] + to, (long long)a.window + (a.rel ? to : (rows - 1) / a.G + 1) + 63);
}
static int keys_of(const AttendArgs& a, const AttendBatch& b, int s) { return walk_of(a, b, s, new_of(b, s), kManyRows); }
static int blocks_of(const AttendArgs& a, const AttendBatch& b, int s, int rows) { return (int)(((long long)new_of(b, s) * a.G + rows - 1) / rows); }
static int parts_of(int keys, int share) { return share >= keys ? 1 : (keys + share - 1) / share; }

// Row blocks end - blocks .. end - 1 of a sequence: new tokens `from` .. `to` - 1.
struct Piece { int s, end, blocks, parts, from, to; };

// The set's pieces in the order of the launch: a sequence each, or two where `whole` ends inside one.
template <typename F> static void each_piece(const AttendArgs& a, const AttendBatch& b, const Set& set, F f)
{
    const int rows = cost_of(a, set.kind).rows;
    long long left = set.whole;
    for (int x = 0; x < set.n; ++x) {
        const int s = set.seq[x], N = new_of(b, s), blocks = blocks_of(a, b, s, rows), uncut = (int)min(left, (long long)blocks), cut = blocks - uncut;
        left -= uncut;
        const int border = cut ? min(N, (int)(((long long)cut * rows + a.G - 1) / a.G)) : 0;      // tokens of the blocks that are cut
        if (uncut) f(Piece{ s, blocks, uncut, 1, border, N });
        if (cut) f(Piece{ s, cut, cut, parts_of(walk_of(a, b, s, border, rows), set.share), 0, border });
    }
}

// Time of a set.  It ends no sooner than its longest item does, than a CU with the most items does, than the keys and values
// come from memory.  *floor: what no way of cutting can go below.
static float time_of(const AttendArgs& a, const AttendBatch& b, const Set& set, int elt, float* floor = nullptr)
{
    const KindCost& c = cost_of(a, set.kind);
    float longest = 0.0f, worst = 0.0f, bytes = 0.0f, slot_bytes = 0.0f;
    double busy = 0.0, head = 0.0;                 // a CU's share of the items, of those before `whole`
    long long before = 0, blocks_before = 0;
    each_piece(a, b, set, [&](const Piece& p) {
        if (blocks_before == set.whole) { head = busy; before = 0; worst = 0.0f; }
        blocks_before += p.blocks;
        const int keys = walk_of(a, b, p.s, p.to, c.rows);
        const long long items = (long long)p.blocks * p.parts * a.Hkv;
        const float near = 1.0f + c.alone / (float)p.blocks, unit = 1.0f / (float)c.keys;
        const float whole = (float)keys / (float)p.parts * unit + 0.5f;
        const float mean = (float)walk_of(a, b, p.s, (p.from + p.to + 1) / 2, c.rows) / (float)p.parts * unit + 0.5f;
        const float item = c.once + c.step * near * whole, usual = c.once + c.step * near * mean, full = c.busy_once + c.busy_step * mean;
        before += items;
        busy += (double)items * full / kCus;
        // items of a CU so far, if all were as long as this one
        const long long q = (before + kCus - 1) / kCus, rest = q % c.per_cu;
        const float cu = (float)(q - rest) * full + (rest ? fmaxf(usual, (float)rest * full) : 0.0f);
        longest = fmaxf(longest, item);
        worst = fmaxf(worst, fmaxf(item, cu));
        if (p.to == new_of(b, p.s)) bytes += (float)min((long long)b.context[p.s] + p.to, (long long)a.window + p.to) * (float)a.Hkv * (float)(a.d * 2 * elt);
        if (p.parts > 1) slot_bytes += (float)items * (float)(min((long long)c.rows, (long long)p.to * a.G) * a.d * 4);
    });
    const float shared = (float)busy, memory = bytes / kBytesPerUs;
    if (floor) *floor = c.launch + fmaxf(shared, memory);
    if (set.n == 0) return 0.0f;
    const float work = fmaxf(longest, (float)head + fmaxf(head > 0.0 ? kTail * worst : worst, (float)(busy - head)));
    float t = c.launch + cbrtf(work * work * work + memory * memory * memory);          // (where both are near, neither is reached)
    if (slot_bytes > 0.0f) t += kPartOnce + 2.0f * slot_bytes / kPartBytesPerUs;
    return t;
}

static long long counters_of(const AttendArgs& a, const AttendBatch& b, const Set& set)
{
    long long n = 0;
    for (int x = 0; x < set.n; ++x) n += blocks_of(a, b, set.seq[x], cost_of(a, set.kind).rows);
    return n * a.Hkv;
}

// The share that takes least time (its own, if counters and a workspace allow parts).
static float cut(const AttendArgs& a, const AttendBatch& b, Set& set, int elt, bool parts)
{
    set.share = DYSPEC_MAX_CONTEXT;
    set.whole = 0;
    float floor, best = time_of(a, b, set, elt, &floor);
    if (!parts || set.n == 0 || counters_of(a, b, set) * (long long)sizeof(unsigned) > DYSPEC_PAGED_COUNTER_BYTES / 2) return best;
    if (best < 1.15f * floor) return best;
    Set found = set;
    auto tries = [&](int longest, long long whole) {
        constexpr int kTries[] = { 2, 3, 4, 6, 8, 12, 16, 24, 32 };
        for (int p : kTries) {
            set.share = ((longest + p - 1) / p + kUnit - 1) / kUnit * kUnit;
            set.whole = (int)whole;
            const float t = time_of(a, b, set, elt);
            if (t < 0.97f * best) { best = t; found = set; }
            else if (t > 1.3f * best) break;
            if (set.share == kUnit) break;
        }
    };
    tries(keys_of(a, b, set.seq[0]), 0);
    if (cost_of(a, set.kind).rows != kManyRows) { set = found; return best; }
    // long walks of single blocks beside sequences of many: those whole and first, these cut
    const int rows = cost_of(a, set.kind).rows;
    const Set before = set;
    long long whole = 0;
    int n = 0, longest_single = 0;
    for (int single = 0; single < 2; ++single) {
        for (int x = 0; x < before.n; ++x) {
            const int blocks = blocks_of(a, b, before.seq[x], rows);
            if ((blocks == 1) != (single == 1)) continue;
            set.seq[n++] = before.seq[x];
            if (!single) whole += blocks;
        }
        if (!single && (n == 0 || n == before.n)) break;
        if (!single) longest_single = n;
    }
    if (longest_single) tries(keys_of(a, b, set.seq[longest_single]), whole);
    // what is left after some rounds of a workgroup a CU cut
    set = before;
    const long long rounds = counters_of(a, b, set) / kCus;
    for (long long r = rounds; r >= 1 && r > rounds - 3 && set.n < DYSPEC_MAX_SEQ; --r) {      // (a table entry more)
        whole = r * kCus / a.Hkv;
        int x = 0;                                         // the sequence in which they end, its longest walk after them
        long long upto = blocks_of(a, b, set.seq[0], rows);
        while (x < set.n - 1 && upto <= whole) upto += blocks_of(a, b, set.seq[++x], rows);
        if (upto > whole) tries(walk_of(a, b, set.seq[x], (int)min((long long)new_of(b, set.seq[x]), ((upto - whole) * rows + a.G - 1) / a.G), rows), whole);
    }
    set = found;
    return best;
}

struct Plan { int n; Set set[2]; };

static bool on_bf16_cores(const AttendArgs& a, int dtype)
{
    auto pieces = [](const void* p, long long stride) { return reinterpret_cast<size_t>(p) % 16 == 0 && stride % 16 == 0; };
    return dtype == DYSPEC_BF16 && a.cap <= kMostBf16Cap && (a.d == 64 || a.d == 128) && pieces(a.q, a.q_stride) && pieces(a.k, a.k_stride) && pieces(a.v, a.v_stride) &&
           pieces(a.out, a.out_stride);
}

// The plan of a form that was asked for: all sequences with one kernel.
static bool plan_given(const AttendArgs& a, const AttendBatch& b, int dtype, const AttendForm& form, Plan& plan)
{
    if (form.kernel < 0 || form.kernel >= kKinds || form.share < 0 || form.share % kUnit || form.whole < 0) return false;
    if (form.kernel < kF32Few && !on_bf16_cores(a, dtype)) return false;
    plan.n = 1;
    Set& set = plan.set[0];
    set.kind = (AttendKind)form.kernel;
    set.share = form.share ? form.share : DYSPEC_MAX_CONTEXT;
    set.whole = form.whole;
    set.n = 0;
    for (int s = 0; s < b.n_seq; ++s)
        if (new_of(b, s) > 0) set.seq[set.n++] = s;
    if (form.whole && set.n == DYSPEC_MAX_SEQ) return false;
    return form.share == 0 || counters_of(a, b, set) * (long long)sizeof(unsigned) <= DYSPEC_PAGED_COUNTER_BYTES;
}

static void plan_of(const AttendArgs& a, const AttendBatch& b, int dtype, bool parts, Plan& plan)
{
    int order[DYSPEC_MAX_SEQ], n = 0;
    for (int s = 0; s < b.n_seq; ++s) {
        if (new_of(b, s) == 0) continue;
        int at = n++;
        for (; at > 0 && keys_of(a, b, order[at - 1]) < keys_of(a, b, s); --at) order[at] = order[at - 1];
        order[at] = s;
    }
    const bool bf16 = on_bf16_cores(a, dtype);
    const int elt = dtype == DYSPEC_BF16 ? 2 : 4;
    // sequences of at most `rows` rows to `few`, the others to `many`; kept if that is the fastest so far
    float best = 0.0f;
    plan.n = 0;
    auto consider = [&](long long rows, AttendKind few, AttendKind many) {
        Plan p;
        p.n = 2;
        p.set[0].kind = many; p.set[1].kind = few;
        p.set[0].n = p.set[1].n = 0;
        for (int x = 0; x < n; ++x) {
            Set& set = p.set[(long long)new_of(b, order[x]) * a.G <= rows];
            set.seq[set.n++] = order[x];
        }
        const float t = cut(a, b, p.set[0], elt, parts) + cut(a, b, p.set[1], elt, parts);
        if (plan.n == 0 || t < best) { plan = p; best = t; }
    };
    constexpr long long kAll = 1LL << 62;
    if (!bf16) {
        consider(16, kF32Few, kF32Many);
        consider(kAll, kF32Few, kF32Many);
    } else {
        long long most = 0, blocks = 0;
        for (int x = 0; x < n; ++x) {
            most = max(most, (long long)new_of(b, order[x]) * a.G);
            blocks += blocks_of(a, b, order[x], kFewRows);
        }
        const bool crowded = blocks * a.Hkv > kCus;                // otherwise fewer waves a workgroup gain nothing
        consider(kAll, kFew8, kMany8);
        if (crowded) consider(kAll, kFew4, kMany8);
        if (most > kFewRows) {
            consider(0, kFew8, kMany8);
            if (n > 1) consider(2 * kFewRows, kFew8, kMany8);
            if (crowded) {
                consider(0, kFew8, kMany4);
                if (n > 1) consider(2 * kFewRows, kFew4, kMany4);
            }
        }
    }
}

static size_t slot_bytes(const AttendArgs& a, AttendKind k) { return (size_t)a.Hkv * slot_floats(a.d, cost_of(a, k).rows) * sizeof(float); }

// The set's pieces in a's table; returns items, and the row blocks and slots they take.
static int fill(AttendArgs& a, const AttendBatch& b, const Set& set, int* groups, long long* slots, int* most_new)
{
    int items = 0, n = 0;
    *groups = 0; *slots = 0; *most_new = 0;
    each_piece(a, b, set, [&](const Piece& p) {
        const int s = p.s, keys = walk_of(a, b, s, p.to, cost_of(a, set.kind).rows);
        AttendSeq& q = a.seq[n];
        q.id = s; q.row0 = b.row0[s]; q.N = new_of(b, s); q.C = b.context[s];
        q.item0 = items; q.end_block = p.end; q.slot0 = (int)*slots;
        q.share = p.parts == 1 ? keys : ((keys + p.parts - 1) / p.parts + kUnit - 1) / kUnit * kUnit;
        q.parts = parts_of(keys, q.share);
        items += p.blocks * q.parts;
        q.group0 = *groups - (p.end - p.blocks);
        *groups += p.blocks;
        if (q.parts > 1) *slots += (long long)p.blocks * q.parts;
        *most_new = max(*most_new, q.N);
        ++n;
    });
    a.n_seq = n;
    return items;
}

static void set_scores(AttendArgs& a, const AttendScores& x)
{
    a.window = x.window; a.rel = x.window < kNoWindow ? x.rel : nullptr;
    a.cap = x.cap;
    a.cap_in = 0.0f; a.c2 = x.scale * 1.4426950408889634f;
}
// What a kernel multiplies scores by (capped_score).
static void set_cap(AttendArgs& a, const AttendScores& x, bool exact)
{
    if (x.cap == 0.0f) return;
    a.c2 = (exact ? 1.0f : 2.0f) * x.cap * 1.4426950408889634f;
    a.cap_in = exact ? x.scale / x.cap : 2.0f * 1.4426950408889634f * (x.scale / x.cap);
}

size_t attend_workspace_bytes(const AttendBatch& b, const AttendScores& scores, int dtype, int Hq, int Hkv, int d)
{
    AttendArgs a;
    set_scores(a, scores);
    a.Hq = Hq; a.Hkv = Hkv; a.G = Hq / Hkv; a.d = d;
    a.q = a.k = a.v = a.out = nullptr;
    a.q_stride = a.out_stride = a.k_stride = a.v_stride = 16;
    Plan plan;
    plan_of(a, b, dtype, true, plan);
    size_t bytes = 0;
    for (int x = 0; x < plan.n; ++x) {
        int groups, most;
        long long slots;
        fill(a, b, plan.set[x], &groups, &slots, &most);
        bytes += (size_t)slots * slot_bytes(a, plan.set[x].kind);
    }
    return bytes ? DYSPEC_PAGED_COUNTER_BYTES + bytes : 0;
}

hipError_t launch_attend(AttendArgs a, const AttendBatch& b, const AttendScores& scores, int dtype, const AttendForm* form, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    set_scores(a, scores);
    Plan plan;
    for (int parts = workspace != nullptr; parts >= 0; --parts) {
        if (form && !plan_given(a, b, dtype, *form, plan)) return hipErrorInvalidValue;
        if (!form) plan_of(a, b, dtype, parts != 0, plan);
        size_t need = DYSPEC_PAGED_COUNTER_BYTES;
        for (int x = 0; x < plan.n && (parts || form); ++x) {
            int groups, most;
            long long slots;
            fill(a, b, plan.set[x], &groups, &slots, &most);
            need += (size_t)slots * slot_bytes(a, plan.set[x].kind);
        }
        if (form && need > DYSPEC_PAGED_COUNTER_BYTES && (!workspace || need > workspace_bytes)) return hipErrorInvalidValue;
        if (!parts || form || need <= workspace_bytes || need == DYSPEC_PAGED_COUNTER_BYTES) break;      // no room: every walk in one piece
    }
    char* slots_at = static_cast<char*>(workspace) + DYSPEC_PAGED_COUNTER_BYTES;
    unsigned* counters = static_cast<unsigned*>(workspace);
    for (int x = 0; x < plan.n; ++x) {
        const Set& set = plan.set[x];
        int groups, most;
        long long slots;
        const int items = fill(a, b, set, &groups, &slots, &most);
        if (items == 0) continue;
        a.part = reinterpret_cast<float*>(slots_at);
        a.counters = counters;
        if (slots) {
            slots_at += (size_t)slots * slot_bytes(a, set.kind);
            counters += groups * a.Hkv;
        }
        set_cap(a, scores, set.kind >= kF32Few);
        hipError_t e = hipSuccess;
        switch (set.kind) {
            case kMany8: e = launch_attend_mfma(a, 8, items, stream); break;
            case kMany4: e = launch_attend_mfma(a, 4, items, stream); break;
            case kFew8: e = launch_attend_short(a, 8, most, items, stream); break;
            case kFew4: e = launch_attend_short(a, 4, most, items, stream); break;
            case kF32Many: e = launch_attend_f32(a, dtype, 4, items, stream); break;
            default: e = launch_attend_f32(a, dtype, 1, items, stream); break;
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t prepare_attend()
{
    hipError_t e = prepare_attend_mfma();
    if (e == hipSuccess) e = prepare_attend_short();
    return e == hipSuccess ? prepare_attend_f32() : e;
}

}  // namespace dyspec
