// Attention of new tokens over pages or packed rows on the bf16 matrix cores, few rows (single tokens, narrow trees, short chunks):
// head_dim 64 or 128, fp32 accumulation.
//
// Workgroup = NW waves on one block of 32 rows of one KV head (attend.h).  The waves share out the keys: wave w takes blocks w,
// w + NW, ... of 32 keys.  Each brings its keys into LDS of its own (direct loads, 32 rows of K and of V) and waits for nobody;
// page numbers are held by its lanes for 16 blocks ahead, so a block's addresses come from the scalar unit.  The waves meet at the
// end, where (max, sum, rows) of all are merged through LDS in fp32 and every wave finishes 32 / NW rows.
// As in attend_mfma.hip weights are taken against a lagging reference and rounded to bf16 once, their sum is of the unrounded ones.
//
// What bounds it: for one token of many sequences memory (64 sequences of 500 to 8000 tokens, 8 KV heads of 128: 222 us, 5.6 TB/s,
// what a kernel that only reads reaches); for one sequence the trips to memory one after the other (one token over 1024, 32 heads,
// 17 MB: 10.8 us, of which memory could do with 3).  Eight waves a workgroup where the row blocks do not fill the chip, four where they do.
#include <atomic>

#include "attend.h"
#include "attn_mfma.h"

namespace dyspec {

constexpr int kKeys = 32;                        // keys of a block
constexpr float kFewSumLimit = 1024.0f;          // a lane's sum of a block above this raises the reference

template <int D> struct FewGeo {
    static constexpr int kRowBytes = 2 * D;
    static constexpr int kChunks = D / 8;                        // 16-byte chunks per row
    static constexpr int kRowsPerLoad = 1024 / kRowBytes;        // rows one wave-wide direct load covers
    static constexpr int kMatBytes = 32 * kRowBytes;             // 32 rows
    static constexpr int kLoads = 32 / kRowsPerLoad;             // direct loads per 32 rows
};
// LDS: a K and a V slot per wave, the query rows, the waves' (max, sum) per row, a mask's bits of the new tokens' blocks
template <int D, int NW> constexpr int few_lds_bytes(int seen_blocks)
{
    return (2 * NW + 1) * FewGeo<D>::kMatBytes + 8 * kFewRows * NW + 4 * kFewRows * seen_blocks;
}

template <int N> __device__ __forceinline__ void wait_loads_but() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

template <int D, int NW>
__global__ __launch_bounds__(64 * NW) void attend_short_kernel(AttendArgs)
{
    const AttendArgs& a = attend_args_here();
    using L = FewGeo<D>;
    constexpr int KK = D / 16, DB = D / 32;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    __shared__ int flag;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = lane & 31, g = lane >> 5;

    // ---- which rows, which keys
    const AttendItem it = attend_item(a, blockIdx.x);
    const AttendSeq& s = it.s;
    const int rows = a.G * s.N, r0 = it.block * kFewRows;
    const int j_first = div_G(a, r0);
    const int end = s.C + div_G(a, min(r0 + kFewRows, rows) - 1) + 1;        // keys that some row of the block may see
    const int n_parts = s.parts > 1 ? (end + s.share - 1) / s.share : 1;
    if (it.part >= n_parts) return;
    const int k_begin = s.parts > 1 ? it.part * s.share : 0;
    const int k_end = s.parts > 1 ? min(end, k_begin + s.share) : end;
    const int last = k_end - 1;
    const int n_blocks = (k_end - k_begin + kKeys - 1) / kKeys;
    const int row_j = div_G(a, min(r0 + n, rows - 1));

    // page numbers of this wave's blocks i0 .. i0 + 15: lane 4 (i - i0) + u has that of rows 8 u .. of block i
    const bool paged = a.table != nullptr;
    const int page_mask = (1 << a.page_shift) - 1;
    auto fetch_pages = [=](int i0) __attribute__((always_inline)) -> uint32_t {
        const int b = wave + NW * (i0 + (lane >> 2));
        const int key = min(k_begin + kKeys * min(b, n_blocks) + 8 * (lane & 3), last);
        return min((uint32_t)a.table[(long long)s.id * a.table_stride + (key >> a.page_shift)], (uint32_t)a.n_pages - 1u);
    };
    uint32_t pages = paged ? fetch_pages(0) : 0u;

    const uint32_t lds0 = lds_address(lds);
    const uint32_t slot = lds0 + wave * 2 * L::kMatBytes;                    // this wave's K rows, then its V rows
    const uint32_t q_lds = lds0 + 2 * NW * L::kMatBytes;
    const uint32_t ml_lds = q_lds + L::kMatBytes;
    const uint32_t seen_lds = ml_lds + 8 * kFewRows * NW;                    // [block from the first one with a new token][row]
    const int lrow = lane / L::kChunks, cpos = lane % L::kChunks;            // row and chunk position in a direct load

    // ---- the query rows (a row past the end repeats the last one), the mask's bits
    {
        const char* const q_seq = a.q + (long long)(s.row0 + j_first) * a.q_stride + (long long)it.kvh * a.G * (D * 2);
#pragma unroll
        for (int xx = 0; xx < (L::kLoads + NW - 1) / NW; ++xx) {
            const int x = xx * NW + wave;
            if (x < L::kLoads) {
                const int R = x * L::kRowsPerLoad + lrow;
                const int r = min(r0 + R, rows - 1), j = div_G(a, r);
                direct_load_16(q_seq, (uint32_t)(j - j_first) * (uint32_t)a.q_stride + (uint32_t)(r - j * a.G) * (D * 2) + 16u * (uint32_t)(cpos ^ swz_k<D>(R)),
                               q_lds + x * 1024);
            }
        }
    }
    const int seen0 = max(s.C - k_begin, 0) / kKeys;                         // first block with a new token
    if (a.mask) {
        typedef __attribute__((address_space(3))) uint32_t* lds_u32;
        for (int x = threadIdx.x; x < (n_blocks - seen0) * kFewRows; x += 64 * NW)
            *(lds_u32)(uint32_t)(seen_lds + 4 * x) = seen_bits(a, s, div_G(a, min(r0 + (x & 31), rows - 1)), k_begin + kKeys * (seen0 + (x >> 5)));
    }
    // ---- direct loads of a block: load x brings rows kRowsPerLoad * x ..; rows past the last key repeat it
    const uint32_t k_stride = (uint32_t)a.k_stride, v_stride = (uint32_t)a.v_stride;
    const char* const k_head = a.k + (long long)it.kvh * (D * 2);
    const char* const v_head = a.v + (long long)it.kvh * (D * 2);
    uint32_t voff_k[4], voff_v[4];                                           // the swizzles repeat after four loads
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int row = L::kRowsPerLoad * x + lrow;
        voff_k[x] = (uint32_t)lrow * k_stride + 16u * (uint32_t)(cpos ^ swz_k<D>(row));
        voff_v[x] = (uint32_t)lrow * v_stride + 16u * (uint32_t)(cpos ^ swz_v<D>(row));
    }
    auto issue = [=](auto v_c, int i, int key0, uint32_t window) __attribute__((always_inline)) {
        constexpr bool is_v = decltype(v_c)::value;
        const char* const head = is_v ? v_head : k_head;
        const uint32_t stride = is_v ? v_stride : k_stride;
        const uint32_t dst = slot + (is_v ? L::kMatBytes : 0);
        const char* base[4];
        static_for<4>([&](auto uc) {
            constexpr int u = decltype(uc)::value;
            const int key = min(key0 + 8 * u, last) & ~7;
            if (paged) {
                const uint32_t p = (uint32_t)__builtin_amdgcn_readlane((int)window, 4 * (i & 15) + u);
                base[u] = head + (long long)p * a.page_bytes + (long long)(uint32_t)(key & page_mask) * stride;
            } else {
                base[u] = head + (long long)(s.row0 + key) * stride;
            }
        });
        if (key0 + kKeys <= k_end) {
            static_for<L::kLoads>([&](auto xc) {
                constexpr int x = decltype(xc)::value;
                direct_load_16(base[x * L::kRowsPerLoad / 8] + (x * L::kRowsPerLoad % 8) * stride, (is_v ? voff_v : voff_k)[x & 3], dst + x * 1024);
            });
        } else {
            static_for<L::kLoads>([&](auto xc) {
                constexpr int x = decltype(xc)::value, u = x * L::kRowsPerLoad / 8;
                const int run = min(key0 + 8 * u, last) & ~7;                // where base[u] points
                const int key = min(key0 + L::kRowsPerLoad * x + lrow, last);
                const int row = L::kRowsPerLoad * x + lrow;
                direct_load_16(base[u], (uint32_t)(key - run) * stride + 16u * (uint32_t)(cpos ^ (is_v ? swz_v<D>(row) : swz_k<D>(row))), dst + x * 1024);
            });
        }
    };
    int i = 0, b = wave;                                                     // this wave's i-th block, its place among all
    bool have = b < n_blocks;
    if (have) {
        issue(std::false_type{}, 0, k_begin + kKeys * b, pages);
        issue(std::true_type{}, 0, k_begin + kKeys * b, pages);
        wait_loads_but<2 * L::kLoads>();                                     // the query rows have landed
    } else {
        wait_direct_loads();
    }
    __syncthreads();
    bf16x8 qf[KK];                                                           // B operand: lane holds query n, dims 16 kk + 8 g ..
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = *(lds_bf16x8)(uint32_t)(q_lds + n * L::kRowBytes + (((2 * kk + g) ^ swz_k<D>(n)) << 4));

    // ---- LDS read addresses
    int k_off[KK];                               // K fragment of step kk, key row n
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) k_off[kk] = (int)slot + n * L::kRowBytes + (((2 * kk + g) ^ swz_k<D>(n)) << 4);
    int v_off[DB];                               // V^T fragments by the transposing read (attend_mfma.hip)
    {
        const int sl = lane & 15, grp = (lane >> 4) & 1;
        const int row = (sl >> 2) + 4 * g;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const int chunk = 4 * db + 2 * grp + ((sl & 3) >> 1);
            v_off[db] = (int)slot + L::kMatBytes + row * L::kRowBytes + ((chunk ^ swz_v<D>(row)) << 4) + 8 * (sl & 1);
        }
    }
    const floatx16 zero16 = { 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0 };
    floatx16 acc[DB];                            // O^T: dim 32 db + 8 (x / 4) + 4 g + x % 4 of query n in register x
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = zero16;
    float m_run = kLowest, l_run = 0.0f;
    const float c2 = a.c2;
    const int full = a.mask ? s.C : s.C + j_first + 1;                       // keys before this one are every row's

    while (have) {
        const int key0 = k_begin + kKeys * b, next = b + NW;
        const bool more = next < n_blocks;
        if (paged && ((i + 1) & 15) == 0 && more) {                          // (waits for the fetch: once in 16 blocks)
            pages = fetch_pages(i + 1);
            asm volatile("" : "+v"(pages));
        }
        // ---- S^T = K Q^T; the next block's K follows as soon as this one's is in registers
        wait_loads_but<L::kLoads>();             // (all but this block's V)
        bf16x8 fr[KK];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) fr[kk] = *(lds_bf16x8)(uint32_t)k_off[kk];
        const bool masked = key0 + kKeys > full || key0 + kKeys > k_end;
        uint32_t seen = ~0u;                     // bit 8 (x / 4) + x % 4: the lane's key of register x
        if (masked) {
            if (a.mask && b >= seen0) seen = *(__attribute__((address_space(3))) const uint32_t*)(uint32_t)(seen_lds + 4 * (kFewRows * (b - seen0) + n));
            else seen = causal_bits(s, row_j, key0);
            if (k_end - key0 < kKeys) seen &= (1u << (k_end - key0)) - 1u;
            seen >>= 4 * g;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        if (more) issue(std::false_type{}, i + 1, k_begin + kKeys * next, pages);
        floatx16 S = zero16;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[kk], qf[kk], S, 0, 0, 0);
        // ---- weights against the reference as it stands; if a lane's sum says that is too low (the first block's always does)
        //      it is raised to the true maximum and they are taken again
        float p[16], ls = 0.0f;
        {
            const float mc = m_run * c2;
#pragma unroll
            for (int x = 0; x < 16; ++x) p[x] = fast_exp2(fmaf(S[x], c2, -mc));
            if (masked) {
#pragma unroll
                for (int x = 0; x < 16; ++x) p[x] = and_bits(p[x], __builtin_amdgcn_sbfe((int)seen, 8 * (x / 4) + (x % 4), 1));
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) ls += p[x];
        }
        if (__any(!(ls <= kFewSumLimit))) {
            float sm[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) sm[x] = (masked && !((seen >> (8 * (x / 4) + (x % 4))) & 1u)) ? -INFINITY : S[x];
            float mx = -INFINITY;
#pragma unroll
            for (int x = 0; x < 16; x += 2) mx = max3(mx, sm[x], sm[x + 1]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
            const float m_new = fmaxf(m_run, mx);
            const float alpha = fast_exp2((m_run - m_new) * c2);
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int x = 0; x < 16; ++x) acc[db][x] *= alpha;
            m_run = m_new;
            const float mc = fmaxf(m_run * c2, kLowest);
            ls = 0.0f;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                p[x] = fast_exp2(fmaf(sm[x], c2, -mc));
                ls += p[x];
            }
        }
        l_run += ls;
        union { uint32_t w[8]; bf16x8 v[2]; } pb;
#pragma unroll
        for (int x = 0; x < 16; x += 2) {
            const floatx2 pp = { p[x], p[x + 1] };
            pb.w[x / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pp, bf16x2));
        }
        // ---- O^T += V^T P^T; then the next block's V
        if (more) wait_loads_but<L::kLoads>(); else wait_direct_loads();
        bf16x8 vf[2][DB];
#pragma unroll
        for (int ts = 0; ts < 2; ++ts)
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                union { short4v h[2]; bf16x8 v; } f;
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    f.h[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4)(uint32_t)(8 * (2 * ts + half) * L::kRowBytes + v_off[db]));
                vf[ts][db] = f.v;
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        if (more) issue(std::true_type{}, i + 1, k_begin + kKeys * next, pages);
#pragma unroll
        for (int ts = 0; ts < 2; ++ts)
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ts][db], pb.v[ts], acc[db], 0, 0, 0);
        ++i;
        b = next;
        have = more;
    }

    // ---- merge.  Every wave leaves its rows in its own slots: piece 2 k + e (four dims) of row n at 16-byte place
    //      32 (2 k + e) + (n ^ (k + 16 e)), so that a wave's writes (one piece of all rows) and its reads (a row's even or odd
    //      pieces) both spread over all banks; maxima and sums beside.
    l_run += __shfl_xor(l_run, 32, kWave);
    typedef float floatx4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) floatx4* lds_floatx4;
    typedef __attribute__((address_space(3))) floatx2* lds_floatx2;
    if (r0 + n < rows)
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int ib = 0; ib < 4; ++ib) {
            const int k = 4 * db + ib;
            *(lds_floatx4)(uint32_t)(slot + 16 * (32 * (2 * k + g) + (n ^ (k + 16 * g)))) =
                floatx4{ acc[db][4 * ib], acc[db][4 * ib + 1], acc[db][4 * ib + 2], acc[db][4 * ib + 3] };
        }
    if (g == 0) *(lds_floatx2)(uint32_t)(ml_lds + 8 * (32 * wave + n)) = floatx2{ m_run, l_run };
    __syncthreads();
    // A lane finishes eight dims of a row at a time (16 bytes of output), wave w rows 32 / NW * w ..
    constexpr int DP = D / 8, RW = kFewRows / NW, IT = (RW * DP + 63) / 64;
    float* const part = part_slot(a, it, kFewRows);
    uint32_t bad = 0u;                                                       // rows with a NaN, from the wave's first on
#pragma unroll
    for (int t = 0; t < IT; ++t) {
        const int idx = 64 * t + lane, dp = idx % DP, sub = idx / DP, row = wave * RW + sub;
        const bool there = idx < RW * DP && r0 + row < rows;
        float M = kLowest, l = 0.0f, o[8] = { 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f };
        if (there) {
            floatx2 ml[NW];
#pragma unroll
            for (int z = 0; z < NW; ++z) {
                ml[z] = *(lds_floatx2)(uint32_t)(ml_lds + 8 * (32 * z + row));
                M = fmaxf(M, ml[z].x);
            }
#pragma unroll
            for (int z = 0; z < NW; ++z) {
                const float f = fast_exp2((ml[z].x - M) * c2);
                l = fmaf(ml[z].y, f, l);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const floatx4 x = *(lds_floatx4)(uint32_t)(lds0 + z * 2 * L::kMatBytes + 16 * (32 * (2 * dp + e) + (row ^ (dp + 16 * e))));
#pragma unroll
                    for (int y = 0; y < 4; ++y) o[4 * e + y] = fmaf(x[y], f, o[4 * e + y]);
                }
            }
        }
        bool nan = l != l;
#pragma unroll
        for (int e = 0; e < 8; ++e) nan |= o[e] != o[e];
        const uint64_t lanes = __builtin_amdgcn_ballot_w64(nan);
        uint32_t here = 0u;                                                  // of this trip's rows
#pragma unroll
        for (int x = 0; x < 64 / DP; ++x)
            if ((lanes >> (x * DP)) & ((1ull << DP) - 1ull)) here |= 1u << x;
        bad |= here << (t * (64 / DP));
        if (there && n_parts > 1 && dp == 0) store_pair(slot_max_sum(a, part, kFewRows, row), M, l);
        if (!there) continue;
        if (n_parts > 1) {
#pragma unroll
            for (int e = 0; e < 2; ++e) store_four(part + slot_place<kSlotFew>(D, row, 2 * dp + e), o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        } else {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const int r = r0 + row, j = div_G(a, r);
            char* const dst = out_row(a, s, j, it.kvh * a.G + (r - j * a.G), 2) + 16 * dp;
            uint4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const floatx2 v = { o[2 * e] * inv, o[2 * e + 1] * inv };
                (&w.x)[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
            }
            *reinterpret_cast<uint4*>(dst) = w;
        }
    }
    if (__builtin_expect(bad != 0u, 0))
        look_again<__bf16, kSlotFew, D>(bad, wave * RW, 0, D, kFewRows, [=](int row) {
            float M = kLowest;
#pragma unroll
            for (int z = 0; z < NW; ++z) M = fmaxf(M, (*(lds_floatx2)(uint32_t)(ml_lds + 8 * (32 * z + row))).x);
            return M;
        });
    if (n_parts > 1 && arrive_last(a, it, n_parts, &flag)) merge_parts<__bf16, kSlotFew, D>(a, it, n_parts, kFewRows, 64 * NW);
}

// the last blocks of a tree of N rows: it may begin and end inside a block
static int seen_blocks(const AttendArgs& a, int most_new) { return a.mask ? (most_new + kKeys - 1) / kKeys + 1 : 0; }

template <int D, int NW>
static hipError_t raise_lds()
{
    static std::atomic<unsigned long long> done{0};
    return raise_dynamic_lds_once(reinterpret_cast<const void*>(&attend_short_kernel<D, NW>), few_lds_bytes<D, NW>(DYSPEC_MAX_NODES / kKeys + 1), done);
}

hipError_t prepare_attend_short()
{
    hipError_t e = raise_lds<128, 8>();
    if (e == hipSuccess) e = raise_lds<128, 4>();
    if (e == hipSuccess) e = raise_lds<64, 8>();
    return e == hipSuccess ? raise_lds<64, 4>() : e;
}

template <int D, int NW>
static hipError_t launch_few(const AttendArgs& a, int most_new, int blocks, hipStream_t stream)
{
    const hipError_t e = raise_lds<D, NW>();
    if (e != hipSuccess) return e;
    attend_short_kernel<D, NW><<<blocks, 64 * NW, few_lds_bytes<D, NW>(seen_blocks(a, most_new)), stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_attend_short(const AttendArgs& a, int waves, int most_new, int items, hipStream_t stream)
{
    const int blocks = items * a.Hkv;
    if (a.d == 128) return waves == 8 ? launch_few<128, 8>(a, most_new, blocks, stream) : launch_few<128, 4>(a, most_new, blocks, stream);
    return waves == 8 ? launch_few<64, 8>(a, most_new, blocks, stream) : launch_few<64, 4>(a, most_new, blocks, stream);
}

}  // namespace dyspec
