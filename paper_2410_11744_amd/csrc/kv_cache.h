// Arguments and launchers of the paged cache's calls (kv_cache.hip).
#pragma once
#include "dyspec_device.h"

namespace dyspec {

// The sequences of a batch as a kernel gets them, with room for S: what a launch costs the host grows with its arguments (160 bytes
// 2.5 us, 700 bytes 3.5), so small batches pass few.
constexpr int kFewSeq = 8;
template <int S> struct Sequences { int row0[S + 1], context[S]; };

struct AppendHead {
    const void *q, *k, *v;
    void *q_out, *k_out, *k_pages, *v_pages;     // k_out: nullptr or the rotated keys as dense rows
    const int *table, *rel_pos;
    const float* inv_freq;
    long long q_stride, k_stride, v_stride, page_stride;         // elements
    int table_stride, page_shift, n_pages;
    int Hq, Hkv, d, half, interleaved;           // Hq 0: no queries
    int per_head, units;                         // units of a head, of a token; of a workgroup (the launcher's)
    uint32_t share, per_head_magic;              // x / per_head = hi(x * magic), per_head 1: x
    int n_seq;
};
template <int S> struct AppendArgs : AppendHead { Sequences<S> seq; };

struct KeepHead {
    char *k_pages, *v_pages;
    const int *table, *accepted, *n_accepted;
    long long layer_bytes, page_bytes, row_bytes;
    int row_pieces, piece_bytes;                 // a row in pieces of 16 or 8 bytes
    int table_stride, page_shift, n_pages;
    int n_seq;
};
template <int S> struct KeepArgs : KeepHead { Sequences<S> seq; };

// `wide`: rows, strides and dims allow 16-byte pieces
hipError_t launch_kv_append(const AppendHead& a, const Sequences<DYSPEC_MAX_SEQ>& seq, int dtype, bool wide, hipStream_t stream);
hipError_t launch_kv_keep(const KeepHead& a, const Sequences<DYSPEC_MAX_SEQ>& seq, int n_layers, hipStream_t stream);
hipError_t prepare_kv_cache();

}  // namespace dyspec
