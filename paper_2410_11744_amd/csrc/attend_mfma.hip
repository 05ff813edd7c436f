// Attention of new tokens over pages or packed rows on the bf16 matrix cores, many rows: head_dim 64 or 128, fp32 accumulation.
//
// Workgroup = NW waves on 128 rows of one KV head (attend.h); wave w owns the 32-row block w & 3.  With eight waves (one workgroup a
// CU) the two waves of a row block take 64-key tiles in turn, even and odd, and merge (max, sum, rows) through LDS at the end: a
// lone workgroup goes through its keys sooner.  With four (two workgroups a CU) a wave takes every tile: more row blocks than CUs
// are dealt more evenly, and one workgroup computes while the other starts or ends (packed prompts of 1 to 1300 tokens, 32 heads:
// 78 us with eight, 58 with four; one tree of 512 rows over 4096 tokens, as many row blocks as CUs: 74 with eight, 85 with four).
// Per 32-key half tile a wave computes S^T = K Q^T (a lane then holds one query and 16 keys), the weights, and O^T += V^T P^T,
// whose B operand is already where the weights are.
//
// The loop is skewed by half tiles, as vector and matrix work overlap only when they are finely mixed: a half step does the
// exponentials of half h between the MFMAs of the second product of half h - 1 and of the first product of half h + 1.  Weights
// are taken against a running reference that is not the maximum but at most ten bits below it; only when a lane's sum of a half
// leaves that range is the half done again with its true maximum.  Weights are rounded to bf16 once, for the product (half a step,
// 2^-8 of each, as the output's own rounding); their sum is of the unrounded ones in fp32.
//
// K and V go from memory to LDS by direct loads, two slots per matrix.  A wave brings 32 rows of one matrix per step, as four runs
// of eight rows that lie each within a page: their addresses are uniform over the wave and are made by the scalar unit from page
// numbers which 64 lanes hold for 16 steps ahead.  So pages cost the vector and matrix units nothing.
//
// What bounds it: over a prompt of 8192 tokens, 64 query heads on 8, the power the card may draw: the matrix cores are busy 70 % of the
// cycles, LDS 36 %, and the clock goes down to 1.5 GHz; reading operands earlier, other wave priorities or orders of the loop's
// instructions change nothing (0.92 to 1.04 ms, 1.06 to 1.19 PFLOP/s by the clock that a card holds; a matrix product of 8192 cubed, by the
// library: 1.34).  A tree of 512 rows over 4096 tokens in pages of 16, one row block a CU (70 to 80 us, 0.86 to 0.98 PFLOP/s), is another
// matter: the matrix cores are busy 46 % of the cycles at 2.0 GHz.  17 us go without any context (launch, start, the tree's own tiles,
// end), 14 to 15 with every 1024 tokens of it (1.2 PFLOP/s).
#include <atomic>

#include "attend.h"
#include "attn_mfma.h"

namespace dyspec {

constexpr int kRows = kManyRows, kTile = 64;
constexpr float kSumLimit = 1024.0f;             // a lane's sum of a half above this raises the reference
constexpr int kLead = 2;                         // fragment slots between an LDS read and its MFMA

template <int D, int NW> struct ManyGeo {
    static constexpr int kTiles = NW / 4;                        // tiles of a step: one for every four waves
    static constexpr int kRowBytes = 2 * D;
    static constexpr int kChunks = D / 8;                        // 16-byte chunks per row
    static constexpr int kRowsPerLoad = 1024 / kRowBytes;        // rows one wave-wide direct load covers
    static constexpr int kMatBytes = kTile * kRowBytes;          // one K or V tile
    static constexpr int kSlotBytes = kTiles * kMatBytes;        // a slot holds a step's tiles
    static constexpr int kVBase = 2 * kSlotBytes;                // K slots 0 and 1, then V slots 0 and 1
    static constexpr int kLdsBytes = 4 * kSlotBytes + (kTiles == 1 ? kMatBytes : 0);      // (two workgroups of the latter fill a CU's 160 KB)
    static constexpr int kLoads = 32 / kRowsPerLoad;             // direct loads of a wave per step
};

template <int D, bool Paged, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attend_mfma_kernel(AttendArgs)
{
    const AttendArgs& a = attend_args_here();
    using L = ManyGeo<D, NW>;
    constexpr int TP = L::kTiles, KK = D / 16, DB = D / 32;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, g = lane >> 5;
    const int wq = wave & 3, wk = wave >> 2;

    // ---- which rows, which keys
    const AttendItem it = attend_item(a, blockIdx.x);
    const AttendSeq& s = it.s;
    const int rows = a.G * s.N, r0 = it.block * kRows;
    const int j_first = div_G(a, r0);
    const int end = s.C + div_G(a, min(r0 + kRows, rows) - 1) + 1;           // keys that some row of the block may see
    const int n_parts = s.parts > 1 ? (end + s.share - 1) / s.share : 1;
    if (it.part >= n_parts) return;
    const int k_begin = s.parts > 1 ? it.part * s.share : 0;
    const int k_end = s.parts > 1 ? min(end, k_begin + s.share) : end;
    const int last = k_end - 1;
    const int nT = (k_end - k_begin + kTile - 1) / kTile;                    // tiles; one from there on stands for "no tile"
    const int nWhole = (k_end - k_begin) / kTile;
    const int rc = min(r0 + 32 * wq + n, rows - 1);
    const int row_j = div_G(a, rc);

    // Bytes from the block's first token's first head (of this KV head) to row x of the block.  All factors are below 2^24.
    const int row_first = r0 - j_first * a.G;
    auto row_offset = [=](int x, uint32_t stride) __attribute__((always_inline)) -> uint32_t {
        const int y = row_first + x, j = div_G(a, y);
        return __umul24((uint32_t)j, stride) + (uint32_t)(y - (int)__umul24((uint32_t)j, (uint32_t)a.G)) * (D * 2);
    };

    // ---- this wave's loads of a step: 32 rows (half ld_half) of K or V of one of its tiles
    const int ld_mm = wave >> 1, ld_half = wave & 1;
    const bool ld_is_v = ld_mm >= TP;
    const int ld_par = ld_mm % TP;
    const int lrow = lane / L::kChunks, cpos = lane % L::kChunks;            // row and chunk position in a direct load
    const uint32_t k_stride = (uint32_t)a.k_stride, v_stride = (uint32_t)a.v_stride;
    const uint32_t st_stride = ld_is_v ? v_stride : k_stride;
    const char* const k_head = a.k + (long long)it.kvh * (D * 2);
    const char* const v_head = a.v + (long long)it.kvh * (D * 2);
    const char* const st_head = ld_is_v ? v_head : k_head;
    const uint32_t lds0 = lds_address(lds);
    // lane offsets within a load; chunk position p of a row holds chunk p ^ swz(row), which repeats after four loads
    auto lane_offset = [=](bool is_v, int x, uint32_t stride) __attribute__((always_inline)) -> uint32_t {
        const int row = L::kRowsPerLoad * (x & 3) + lrow;
        return (uint32_t)lrow * stride + 16u * (uint32_t)(cpos ^ (is_v ? swz_v<D>(row) : swz_k<D>(row)));
    };
    uint32_t st_voff[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) st_voff[x] = lane_offset(ld_is_v, x, st_stride);
    // four runs of eight rows from key0 on, at the bases of their runs; rows behind the last key repeat it
    auto issue_ragged = [=](const char* const (&base)[4], bool is_v, uint32_t stride, int key0, uint32_t dst) __attribute__((always_inline)) {
        static_for<L::kLoads>([&](auto xc) {
            constexpr int x = decltype(xc)::value, u = x * L::kRowsPerLoad / 8;
            const int run = min(key0 + 8 * u, last) & ~7;                    // where base[u] points
            const int key = min(key0 + L::kRowsPerLoad * x + lrow, last);
            const int row = L::kRowsPerLoad * (x & 3) + lrow;
            const uint32_t c = 16u * (uint32_t)(cpos ^ (is_v ? swz_v<D>(row) : swz_k<D>(row)));
            direct_load_16(base[u], (uint32_t)(key - run) * stride + c, dst + x * 1024);
        });
    };
    // 32 rows from key0 on, addresses looked up now (the prologue's loads)
    auto issue_now = [=](const char* head, bool is_v, uint32_t stride, int tile, int half, uint32_t dst) __attribute__((always_inline)) {
        if (tile >= nT) return;
        const int key0 = k_begin + kTile * tile + 32 * half;
        const char* base[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) base[u] = head + key_offset<Paged>(a, s, min(key0 + 8 * u, last) & ~7, stride);
        issue_ragged(base, is_v, stride, key0, dst);
    };
    // steady state: in step i this wave brings its half of tile tile_in(i)
    const int ld_first = (ld_is_v ? TP : 2 * TP) + ld_par;
    auto tile_in = [=](int i) __attribute__((always_inline)) -> int { return TP * i + ld_first; };
    // page numbers of steps i0 .. i0 + 15: lane 4 (i - i0) + u has run u's.  They are fetched 16 steps before they are due.
    auto fetch_pages = [=](int i0) __attribute__((always_inline)) -> uint32_t {
        const int t = tile_in(i0 + (lane >> 2));
        const int key = min(k_begin + (t < nT ? kTile * t : 0) + 32 * ld_half + 8 * (lane & 3), last);
        return (uint32_t)a.table[(long long)s.id * a.table_stride + (key >> a.page_shift)];
    };
    const uint32_t last_page = (uint32_t)a.n_pages - 1u;
    const int page_mask = (1 << a.page_shift) - 1;
    const long long page_bytes = a.page_bytes;
    uint32_t pages = 0u, pages_next = 0u;
    if constexpr (Paged) { pages = min(fetch_pages(0), last_page); pages_next = fetch_pages(16); }
    // base of run u of step i; a tile that does not exist stands for the first one (whole, where this is used for it)
    auto run_base = [&](int i, int u) __attribute__((always_inline)) -> const char* {
        const int t = tile_in(i);
        const int key = min(k_begin + (t < nT ? kTile * t : 0) + 32 * ld_half + 8 * u, last) & ~7;
        if constexpr (Paged) {
            const uint32_t p = (uint32_t)__builtin_amdgcn_readlane((int)pages, 4 * (i & 15) + u);
            return st_head + (long long)p * page_bytes + (long long)(uint32_t)(key & page_mask) * st_stride;
        } else {
            return st_head + (long long)(s.row0 + key) * st_stride;
        }
    };
    const uint32_t st_dst = lds0 + (ld_is_v ? L::kVBase : 0) + ld_par * L::kMatBytes + ld_half * (32 * L::kRowBytes);
    auto slot_of = [=](int i) __attribute__((always_inline)) -> uint32_t { return (uint32_t)(((ld_is_v ? i + 1 : i) & 1) * L::kSlotBytes); };

    // ---- prologue: the query rows (into V slot 1, of one tile a slot also into the place behind it, laid out like K: no V tile
    //      comes to slot 1 before the middle of step 0), K of the first two steps, V of the first.
    const uint32_t q_lds = lds0 + L::kVBase + L::kSlotBytes;
    {
        constexpr int QL = kRows / L::kRowsPerLoad / NW;
        const char* const q_seq = a.q + (long long)(s.row0 + j_first) * a.q_stride + (long long)it.kvh * a.G * (D * 2);
#pragma unroll
        for (int x = 0; x < QL; ++x) {
            const int X = wave * QL + x;
            const int R = X * L::kRowsPerLoad + lrow;
            direct_load_16(q_seq, row_offset(min(R, rows - 1 - r0), (uint32_t)a.q_stride) + 16u * (uint32_t)(cpos ^ swz_k<D>(R)), q_lds + X * 1024);
        }
    }
    auto issue_first_k = [=]() __attribute__((always_inline)) {
        issue_now(k_head, false, k_stride, ld_mm, ld_half, lds0 + ld_mm * L::kMatBytes + ld_half * (32 * L::kRowBytes));
    };
    auto issue_first_v = [=]() __attribute__((always_inline)) {
        if (ld_is_v) issue_now(v_head, true, v_stride, ld_par, ld_half, st_dst);
    };
    if (!ld_is_v) issue_first_k();               // what the first product needs
    // a V tile of slot 0 that does not exist is cleared: weights of zero meet it, and zero times what LDS held may be a NaN
    if (TP == 2 && nT < 2) {
        const uint4 z = { 0u, 0u, 0u, 0u };
        for (int x = tid; x < L::kMatBytes / 16; x += 64 * NW) reinterpret_cast<uint4*>(lds + L::kVBase + L::kMatBytes)[x] = z;
    }
    floatx16 acc[DB];                            // O^T
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[db][i] = 0.0f;
    floatx16 S[2];                               // scores of a half: half e in buffer e
    uint32_t pw[2][2][4];                        // weights as bf16 pairs [buffer][16-key step][word]
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int ts = 0; ts < 2; ++ts)
#pragma unroll
            for (int w = 0; w < 4; ++w) pw[e][ts][w] = 0u;
    float m_run = -INFINITY, l_run = 0.0f, ls_half = 0.0f;         // (so that the first half a wave sees is done again, whatever the scale)
    const float c2 = a.c2;
    __syncthreads();                             // (the later loads queue up behind the urgent ones)
    if (ld_is_v) issue_first_k();
    issue_first_v();
    // the others wait for their query rows only: K of the second step and V are needed from the middle of step 0 on
    if (ld_is_v && ld_mm < nT && ld_par < nT) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(2 * L::kLoads) : "memory");
    else wait_direct_loads();
    __syncthreads();
    bf16x8 qf[KK];                               // B operand: lane holds query n, dims 16 kk + 8 g ..
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        const int R = 32 * wq + n;
        qf[kk] = *(lds_bf16x8)(uint32_t)(q_lds + R * L::kRowBytes + (((2 * kk + g) ^ swz_k<D>(R)) << 4));
    }
    // ---- LDS read addresses of this lane
    int k_off[KK];                               // K fragment of step kk, key row n of a half
    {
        const int h = g ^ swz_k<D>(n);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) k_off[kk] = (int)lds0 + wk * L::kMatBytes + n * L::kRowBytes + (((2 * kk) ^ h) << 4);
    }
    // V^T fragments by the transposing read: lanes 4 j + r of a group of 16 point at key row j, columns 4 r .. of a 16-column slab,
    // lane i receives column i of the four keys: four consecutive k-slots of an A operand whose row is dim i
    int v_off[DB];
    {
        const int sl = lane & 15, grp = (lane >> 4) & 1;
        const int row = (sl >> 2) + 4 * g;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const int chunk = 4 * db + 2 * grp + ((sl & 3) >> 1);
            v_off[db] = (int)lds0 + L::kVBase + wk * L::kMatBytes + row * L::kRowBytes + ((chunk ^ swz_v<D>(row)) << 4) + 8 * (sl & 1);
        }
    }

    // ---- which of a tile's 64 keys the lane's row sees.  The mask's words are fetched a step ahead and put together when they are due.
    struct Words { uint32_t w[3]; };
    auto fetch_words = [=](int t) __attribute__((always_inline)) -> Words {
        Words x = { { ~0u, ~0u, ~0u } };
        if (a.mask && t < nT) {
            const int q = (k_begin + kTile * t - s.C) >> 5;
            if (q + 2 >= 0) {
#pragma unroll
                for (int e = 0; e < 3; ++e) x.w[e] = mask_word(a, s, row_j, q + e);
            }
        }
        return x;
    };
    auto seen_in = [=](int t, const Words& x) __attribute__((always_inline)) -> uint64_t {
        if (t >= nT) return 0ull;
        const int k0 = k_begin + kTile * t;
        const uint32_t r = (uint32_t)(k0 - s.C) & 31u;
        const uint32_t lo = causal_bits(s, row_j, k0) & __builtin_amdgcn_alignbit(x.w[1], x.w[0], r);
        const uint32_t hi = causal_bits(s, row_j, k0 + 32) & __builtin_amdgcn_alignbit(x.w[2], x.w[1], r);
        return ((uint64_t)hi << 32) | lo;
    };

    // ---- one half step, for the half e of this wave's tile of step i (SP = i & 1: its LDS slot).  HS: weights of this half from S[e] into pw[e];
    //      HP: second product of the previous half (pw[e^1]); HQ: first product of the next half into S[e^1]; MK: this half is
    //      masked (seen: its 32 bits >> 4 g).  The lower half step finds the bases of the step's loads (PB: step ld_step), the upper
    //      one issues them (LD), one per two slots.
    const floatx16 zero16 = { 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0 };
    const char* ld_base[4] = { st_head, st_head, st_head, st_head };
    auto half_step = [&](auto hp_c, auto hq_c, auto hs_c, auto mk_c, auto pb_c, auto ld_c, auto sp_c, auto e_c, uint32_t seen, int ld_step, uint32_t ld_dst) __attribute__((always_inline)) {
        constexpr bool PB = decltype(pb_c)::value, LD = decltype(ld_c)::value, HP = decltype(hp_c)::value, HQ = decltype(hq_c)::value;
        constexpr bool HS = decltype(hs_c)::value, MK = decltype(mk_c)::value;
        constexpr int SP = decltype(sp_c)::value, E = decltype(e_c)::value, O = E ^ 1;
        constexpr int NP = 2 * DB, NQ = KK;                        // fragments of the second and first product
        static_assert(NP == NQ, "the interleave alternates the two products");
        constexpr int NS = (HP ? NP : 0) + (HQ ? NQ : 0);
        // the previous half is the upper one of step i - 1 (slot SP^1) or the lower one of i; the next is the upper one of i or the
        // lower one of i + 1 (slot SP^1)
        constexpr int kVsrc = (E == 0 ? (SP ^ 1) : SP) * L::kSlotBytes + 32 * O * L::kRowBytes;
        constexpr int kKsrc = (E == 0 ? SP : (SP ^ 1)) * L::kSlotBytes + 32 * O * L::kRowBytes;
        const float mc = m_run * c2;
        float ls = 0.0f;
        // Register i of S is key 8 (i / 4) + 4 g + i % 4 of the half.  Vector work on pair k (scores 2k, 2k + 1): F the exponents,
        // X the exponentials, M the mask, C the rounding, D the sum.  A dependent instruction waits for its operand, so the stages
        // of a pair sit in different items: item h holds X(k) and D(k-1) when even, M(k), F(k+1) and C(k) when odd.
        float ft[8][2], pt[8][2];
        auto stage_f = [&](auto kc) __attribute__((always_inline)) {
            constexpr int k = decltype(kc)::value;
            ft[k][0] = fmaf(S[E][2 * k], c2, -mc);
            ft[k][1] = fmaf(S[E][2 * k + 1], c2, -mc);
        };
        auto stage_d = [&](auto kc) __attribute__((always_inline)) {
            constexpr int k = decltype(kc)::value;
            ls += pt[k][0];
            ls += pt[k][1];
        };
        auto item = [&](auto hc) __attribute__((always_inline)) {
            constexpr int h = decltype(hc)::value, k = h / 2, i = 2 * k;
            if constexpr (h % 2 == 0) {
                pt[k][0] = fast_exp2(ft[k][0]);
                pt[k][1] = fast_exp2(ft[k][1]);
                if constexpr (k > 0) stage_d(std::integral_constant<int, k - 1>{});
            } else {
                float p0 = pt[k][0], p1 = pt[k][1];
                if constexpr (MK) {
                    p0 = and_bits(p0, __builtin_amdgcn_sbfe((int)seen, 8 * (i / 4) + (i % 4), 1));
                    p1 = and_bits(p1, __builtin_amdgcn_sbfe((int)seen, 8 * (i / 4) + (i % 4) + 1, 1));
                }
                if constexpr (k + 1 < 8) stage_f(std::integral_constant<int, k + 1>{});
                floatx2 pp = { p0, p1 };
                uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector(pp, bf16x2));
                asm volatile("" : "+v"(w));                        // the conversion stays in this scheduling group
                if constexpr (MK) { pt[k][0] = p0; pt[k][1] = p1; }
                pw[E][k / 4][k % 4] = w;
            }
        };
        if constexpr (HS) stage_f(std::integral_constant<int, 0>{});
        // with both products, even slots belong to the first and odd slots to the second
        bf16x8 fr[NS];
        auto read_slot = [&](auto sc) __attribute__((always_inline)) {
            constexpr int x = decltype(sc)::value, idx = (HP && HQ) ? x / 2 : x;
            if constexpr (HP && (!HQ || x % 2 == 1)) {
                constexpr int ts = idx / DB, db = idx % DB;        // k-slot (g, e) of step ts is key 8 (2 ts + e / 4) + 4 g + e % 4
                union { short4v h[2]; bf16x8 v; } f;
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    f.h[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4)(uint32_t)(kVsrc + 8 * (2 * ts + half) * L::kRowBytes + v_off[db]));
                fr[x] = f.v;
            } else {
                fr[x] = *(lds_bf16x8)(uint32_t)(kKsrc + k_off[idx]);
            }
        };
        auto mfma_slot = [&](auto sc) __attribute__((always_inline)) {
            constexpr int x = decltype(sc)::value, idx = (HP && HQ) ? x / 2 : x;
            if constexpr (HP && (!HQ || x % 2 == 1)) {
                constexpr int ts = idx / DB, db = idx % DB;
                union { uint32_t w[4]; bf16x8 v; } b;
#pragma unroll
                for (int w = 0; w < 4; ++w) b.w[w] = pw[O][ts][w];
                acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[x], b.v, acc[db], 0, 0, 0);
            } else {
                S[O] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[x], qf[idx], idx == 0 ? zero16 : S[O], 0, 0, 0);
            }
        };
        constexpr int IPS = 16 / NS, LEVERY = 2 * L::kLoads <= NS ? 2 : 1;
        static_assert(!LD || LEVERY * L::kLoads <= NS, "the loads of a step fit its upper half step");
        static_for<(kLead < NS ? kLead : NS)>([&](auto sc) { read_slot(sc); });
        static_for<NS>([&](auto sc) {
            constexpr int x = decltype(sc)::value;
            if constexpr (x + kLead < NS) read_slot(std::integral_constant<int, x + kLead>{});
            mfma_slot(sc);
            if constexpr (PB && x % 2 == 0 && x < 8) ld_base[x / 2] = run_base(ld_step, x / 2);
            if constexpr (LD && x % LEVERY == 0 && x / LEVERY < L::kLoads) {
                constexpr int y = x / LEVERY;
                direct_load_16(ld_base[y * L::kRowsPerLoad / 8] + (y * L::kRowsPerLoad % 8) * st_stride, st_voff[y & 3], ld_dst + y * 1024);
            }
            if constexpr (HS) static_for<IPS>([&](auto hc) { item(std::integral_constant<int, x * IPS + decltype(hc)::value>{}); });
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (HS) {
            stage_d(std::integral_constant<int, 7>{});
            ls_half = ls;
        }
    };
    // Rare (and the first half a wave sees): a score is far above the reference.  The reference goes up to the true maximum, what has
    // been summed is rescaled (the second product of the previous half is complete here), the half's weights are done again.
    auto redo_half = [&](auto e_c, bool mk, uint32_t seen) __attribute__((always_inline)) {
        constexpr int E = decltype(e_c)::value;
        float sm[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) sm[i] = (mk && !((seen >> (8 * (i / 4) + (i % 4))) & 1u)) ? -INFINITY : S[E][i];
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; i += 2) mx = max3(mx, sm[i], sm[i + 1]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
        const float m_new = max3(m_run, mx, kLowest);
        const float alpha = fast_exp2((m_run - m_new) * c2);
        // A row without a sum so far starts at zero whatever acc holds: the first half's second product takes what lies in V's slot then,
        // query rows, at weights of zero, and a row's NaN is nothing to other rows.
        const bool fresh = m_run <= kLowest;
        m_run = m_new;
        l_run *= alpha;
        if (__all(fresh)) {
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = zero16;
        } else if (__any(alpha != 1.0f)) {                         // (fresh rows' is 0, or they stay fresh)
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[db][i] = fresh ? 0.0f : acc[db][i] * alpha;
        }
        const float mc = fmaxf(m_run * c2, kLowest);
        float ls = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float p0 = fast_exp2(fmaf(sm[i], c2, -mc)), p1 = fast_exp2(fmaf(sm[i + 1], c2, -mc));
            floatx2 pp = { p0, p1 };
            ls += p0;
            ls += p1;
            pw[E][i / 8][(i / 2) % 4] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pp, bf16x2));
        }
        ls_half = ls;
    };
    const std::true_type yes{};
    const std::false_type no{};
    const std::integral_constant<int, 0> even{};
    const std::integral_constant<int, 1> odd{};
    auto run_half = [&](auto mk_c, auto pb_c, auto ld_c, auto sp_c, auto e_c, uint32_t seen, int ld_step, uint32_t ld_dst) __attribute__((always_inline)) {
        half_step(yes, yes, yes, mk_c, pb_c, ld_c, sp_c, e_c, seen, ld_step, ld_dst);
        if (__any(!(ls_half <= kSumLimit))) redo_half(e_c, decltype(mk_c)::value, seen);
        l_run += ls_half;
    };

    // first product of the lower half of step 0
    half_step(no, yes, no, no, no, no, odd, odd, 0u, 0, 0u);

    // ---- a step's middle: the loads of the step before have landed everywhere
    auto turn_pages = [&](int ii) __attribute__((always_inline)) {
        if constexpr (Paged)
            if ((ii & 15) == 0 && ii > 0) { pages = min(pages_next, last_page); pages_next = fetch_pages(ii + 16); }
    };
    auto middle = [&]() __attribute__((always_inline)) {
        wait_direct_loads();
        __syncthreads();
    };
    // ---- plain steps: the step's tiles are seen whole by every row, what it loads (tiles up to TP (i + 3) - 1) is whole or does not
    //      exist
    const int full = max(min(a.mask ? s.C : s.C + j_first + 1, k_end) - k_begin, 0) / kTile;
    const int nPlain = min(full / TP, nWhole < nT ? max(nWhole - 2 * TP, 0) / TP : full);
    auto plain_step = [&](auto sp_c, int ii) __attribute__((always_inline)) {
        if constexpr (decltype(sp_c)::value == 0) turn_pages(ii);
        run_half(no, yes, no, sp_c, even, 0u, ii, 0u);
        middle();
        run_half(no, no, yes, sp_c, odd, 0u, ii, st_dst + slot_of(ii));
    };
    int i = 0;
    for (; i + 1 < nPlain; i += 2) {
        plain_step(even, i);
        plain_step(odd, i + 1);
    }
    if (i < nPlain) plain_step(even, i++);
    // ---- masked steps.  A half step is run only if the wave's rows see a key of the half or of a neighbour, whose product it
    //      carries; otherwise its weights are cleared.
    const int nIt = (nT + TP - 1) / TP;
    uint64_t visC, visN;
    {
        const int tc = TP * i + wk, tn = TP * (i + 1) + wk;
        const Words xc = fetch_words(tc), xn = fetch_words(tn);
        visC = seen_in(tc, xc);
        visN = seen_in(tn, xn);
    }
    auto masked_half = [&](auto sp_c, auto e_c, bool act, uint32_t seen) __attribute__((always_inline)) {
        if (act) {
            run_half(yes, no, no, sp_c, e_c, seen, 0, 0u);
        } else {
#pragma unroll
            for (int ts = 0; ts < 2; ++ts)
#pragma unroll
                for (int w = 0; w < 4; ++w) pw[decltype(e_c)::value][ts][w] = 0u;
        }
    };
    bool aP1 = i > 0;                                              // the upper half of the step before
    auto masked_step = [&](auto sp_c, int ii) __attribute__((always_inline)) {
        const int t2 = TP * (ii + 2) + wk;
        Words x2 = fetch_words(t2);
        const bool aC0 = __any((uint32_t)visC != 0u), aC1 = __any((uint32_t)(visC >> 32) != 0u), aN0 = __any((uint32_t)visN != 0u);
        masked_half(sp_c, even, aP1 || aC0 || aC1, (uint32_t)visC >> (4 * g));
        turn_pages(ii);
        middle();
        if (const int t = tile_in(ii); t < nT) {
#pragma unroll
            for (int u = 0; u < 4; ++u) ld_base[u] = run_base(ii, u);
            issue_ragged(ld_base, ld_is_v, st_stride, k_begin + kTile * t + 32 * ld_half, st_dst + slot_of(ii));
        }
        masked_half(sp_c, odd, aC0 || aC1 || aN0, (uint32_t)(visC >> 32) >> (4 * g));
        aP1 = aC1;
        visC = visN;
        visN = seen_in(t2, x2);
    };
    if ((i & 1) && i < nIt) masked_step(odd, i++);
    for (; i < nIt; i += 2) {
        masked_step(even, i);
        if (i + 1 < nIt) masked_step(odd, i + 1);
    }
    // ---- the second product of the last upper half
    if (aP1) {
        if (nIt & 1) half_step(yes, no, no, no, no, no, odd, even, 0u, 0, 0u);
        else half_step(yes, no, no, no, no, no, even, even, 0u, 0, 0u);
    }
    wait_direct_loads();
    __syncthreads();                                               // every read of LDS is done, and nothing is under way to it

    // ---- the rows leave.  With two tiles a step the two waves of a row block merge first: each finishes half of the dims, leaves
    //      the other half with its (max, sum) in LDS and takes its own of the other wave.
    l_run += __shfl_xor(l_run, 32, kWave);
    if (__any(m_run <= kLowest)) {                                 // rows that saw no key here: zeros, as above
        const bool none = m_run <= kLowest;
        m_run = fmaxf(m_run, kLowest);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[db][i] = none ? 0.0f : acc[db][i];
    }
    constexpr int HB = DB / TP, kArea = TP == 2 ? HB * 4 * 1024 : 0;         // 32-dim blocks a wave finishes, bytes it leaves
    constexpr int kMl = TP == 2 ? 512 : 0;
    typedef float floatx4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) floatx4* lds_floatx4;
    typedef __attribute__((address_space(3))) floatx2* lds_floatx2;
    auto each_half = [&](auto f) __attribute__((always_inline)) {  // (registers are named at compile time)
        if (TP == 1 || wk == 0) f(std::integral_constant<int, 0>{}); else f(std::integral_constant<int, DB - HB>{});
    };
    const uint32_t area1 = lds0 + (uint32_t)(wave ^ 4) * kArea, ml_at1 = lds0 + NW * kArea + (uint32_t)(wave ^ 4) * kMl;
    float m = m_run, l = l_run, f0 = 1.0f, f1 = 0.0f;
    if constexpr (TP == 2) {
        const uint32_t area = lds0 + (uint32_t)wave * kArea, ml_at = lds0 + NW * kArea + (uint32_t)wave * kMl;
        each_half([&](auto mine_c) __attribute__((always_inline)) {
            constexpr int other = decltype(mine_c)::value == 0 ? HB : 0;
#pragma unroll
            for (int b = 0; b < HB; ++b)
#pragma unroll
                for (int ib = 0; ib < 4; ++ib)
                    *(lds_floatx4)(uint32_t)(area + (4 * b + ib) * 1024 + 16 * lane) =
                        floatx4{ acc[other + b][4 * ib], acc[other + b][4 * ib + 1], acc[other + b][4 * ib + 2], acc[other + b][4 * ib + 3] };
        });
        *(lds_floatx2)(uint32_t)(ml_at + 8 * lane) = floatx2{ m_run, l_run };
        __syncthreads();
        const floatx2 ml1 = *(lds_floatx2)(uint32_t)(ml_at1 + 8 * lane);
        m = fmaxf(m_run, ml1.x);
        f0 = fast_exp2((m_run - m) * c2);
        f1 = fast_exp2((ml1.x - m) * c2);
        l = l_run * f0 + ml1.y * f1;
    }
    float* const slot = part_slot(a, it, kRows);
    const float inv = n_parts > 1 ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;      // a part leaves unnormalised
    const float w0 = f0 * inv, w1 = f1 * inv;
    const int left = rows - (r0 + 32 * wq);                        // rows of this row block that exist
    if (n_parts > 1 && wk == 0 && g == 0 && n < left) store_pair(slot_max_sum(a, slot, kRows, 32 * wq + n), m, l);
    each_half([&](auto mine_c) __attribute__((always_inline)) {
        constexpr int mine = decltype(mine_c)::value;
        float zero[4] = { l * 0.0f, 0.0f, 0.0f, 0.0f };            // stay zero unless something is infinite or a NaN
#pragma unroll
        for (int b = 0; b < HB; ++b)
#pragma unroll
            for (int ib = 0; ib < 4; ++ib) {
                floatx4 x = { 0.0f, 0.0f, 0.0f, 0.0f };
                if constexpr (TP == 2) x = *(lds_floatx4)(uint32_t)(area1 + (4 * b + ib) * 1024 + 16 * lane);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float o = TP == 2 ? acc[mine + b][4 * ib + e] * w0 + x[e] * w1 : acc[mine + b][4 * ib + e] * w0;
                    acc[mine + b][4 * ib + e] = o;
                    zero[e] = fmaf(o, 0.0f, zero[e]);
                }
            }
        const uint64_t lanes = __builtin_amdgcn_ballot_w64((zero[0] + zero[1]) + (zero[2] + zero[3]) != 0.0f);      // (a NaN is not equal)
        uint32_t bad = (uint32_t)(lanes | lanes >> 32);
        if (left < 32) bad &= left > 0 ? (1u << left) - 1u : 0u;
        if (n_parts > 1) {
            if (n < left) {
#pragma unroll
                for (int b = 0; b < HB; ++b)
#pragma unroll
                    for (int ib = 0; ib < 4; ++ib) {
                        const int piece = 8 * (mine + b) + 2 * ib + g;
                        store_four(slot + slot_place<kSlotMany>(D, 32 * wq + n, piece), acc[mine + b][4 * ib], acc[mine + b][4 * ib + 1], acc[mine + b][4 * ib + 2],
                                   acc[mine + b][4 * ib + 3]);
                    }
            }
        } else {
            // the rows (or halves of rows) go through LDS and leave 16 bytes a lane, in runs of 64 * HB bytes
            constexpr int kPitch = 64 * HB + 16, CPR = 4 * HB;
            const uint32_t stage = lds0 + NW * (kArea + kMl) + (uint32_t)wave * (32 * kPitch);
            static_assert(NW * (kArea + kMl) + NW * 32 * kPitch <= L::kLdsBytes, "areas and stages fit");
            char* const out_first = a.out + (long long)(s.row0 + j_first) * a.out_stride + (long long)it.kvh * a.G * (D * 2);
            const uint32_t out_stride = (uint32_t)a.out_stride;
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
            for (int b = 0; b < HB; ++b)
#pragma unroll
                for (int ib = 0; ib < 4; ++ib) {
                    const floatx2 lo = { acc[mine + b][4 * ib], acc[mine + b][4 * ib + 1] }, hi = { acc[mine + b][4 * ib + 2], acc[mine + b][4 * ib + 3] };
                    *(__attribute__((address_space(3))) u32x2*)(uint32_t)(stage + n * kPitch + (32 * b + 8 * ib + 4 * g) * 2) =
                        u32x2{ __builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)), __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2)) };
                }
#pragma unroll
            for (int t = 0; t < 32 * CPR / kWave; ++t) {
                const int c = lane + kWave * t, rn = c / CPR, cc = c % CPR;
                if (rn >= left) continue;
                const u32x4 v = *(__attribute__((address_space(3))) u32x4*)(uint32_t)(stage + rn * kPitch + cc * 16);
                __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(out_first + (row_offset(32 * wq + rn, out_stride) + 64 * mine + cc * 16)));
            }
        }
        if (__builtin_expect(bad != 0u, 0))
            look_again<__bf16, kSlotMany, D>(bad, 32 * wq, 32 * mine, 32 * (mine + HB), kRows, [=](int row) { return __shfl(m, row & 31, kWave); });
    });
    if (n_parts > 1 && arrive_last(a, it, n_parts, reinterpret_cast<int*>(lds))) merge_parts<__bf16, kSlotMany, D>(a, it, n_parts, kRows, 64 * NW);
}

template <int D, bool Paged, int NW>
static hipError_t launch_many(const AttendArgs* a, int blocks, hipStream_t stream)
{
    static std::atomic<unsigned long long> done{0};
    constexpr int lds = ManyGeo<D, NW>::kLdsBytes;
    const hipError_t e = raise_dynamic_lds_once(reinterpret_cast<const void*>(&attend_mfma_kernel<D, Paged, NW>), lds, done);
    if (e != hipSuccess || !a) return e;
    attend_mfma_kernel<D, Paged, NW><<<blocks, 64 * NW, lds, stream>>>(*a);
    return hipGetLastError();
}
template <int D, bool Paged>
static hipError_t launch_many(const AttendArgs* a, int waves, int blocks, hipStream_t stream)
{
    return waves == 8 ? launch_many<D, Paged, 8>(a, blocks, stream) : launch_many<D, Paged, 4>(a, blocks, stream);
}
static hipError_t launch_many(const AttendArgs* a, int d, bool paged, int waves, int blocks, hipStream_t stream)
{
    if (d == 128) return paged ? launch_many<128, true>(a, waves, blocks, stream) : launch_many<128, false>(a, waves, blocks, stream);
    return paged ? launch_many<64, true>(a, waves, blocks, stream) : launch_many<64, false>(a, waves, blocks, stream);
}

hipError_t prepare_attend_mfma()
{
    for (int x = 0; x < 8; ++x) {
        const hipError_t e = launch_many(nullptr, x & 1 ? 128 : 64, x & 2, x & 4 ? 8 : 4, 0, nullptr);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_attend_mfma(const AttendArgs& a, int waves, int items, hipStream_t stream)
{
    return launch_many(&a, a.d, a.table != nullptr, waves, items * a.Hkv, stream);
}

}  // namespace dyspec
