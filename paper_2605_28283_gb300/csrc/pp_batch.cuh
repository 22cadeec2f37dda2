// Device view of a step's sequences (pp_batch): lengths checked on the
// device, page lookup, and the search for a token's sequence.
#pragma once

#include "pp_attn.h"
#include "pp_common.cuh"

namespace pp {

struct Seq {
    int q0;    // first new token
    int n;     // new tokens (0 for a sequence that is skipped)
    int ctx;   // cached tokens before them
    bool bad;  // lengths that no cache can hold: nothing is read or written for the sequence
};

PP_DEVINL Seq load_seq(const BatchArgs& B, int b) {
    const int q0 = B.q_start[b], q1 = B.q_start[b + 1], ctx = B.ctx_len[b];
    Seq s{q0, 0, ctx, true};
    if (q0 < 0 || q1 < q0 || q1 > B.n_tokens || ctx < 0) return s;
    // 64-bit: max_pages * page_size may pass 2^31
    const long long cap = (long long)B.max_pages * B.page_size;
    const long long need = (long long)ctx + (q1 - q0);
    if (need > cap || need > 0x7fffff00ll) return s;  // entry numbers, rounded up to a key tile, stay in 32 bits
    s.n = q1 - q0;
    s.bad = false;
    return s;
}

// Page of entry j of sequence b (0 <= j < max_pages * page_size), or -1 when
// the table names none.
PP_DEVINL int entry_page(const BatchArgs& B, int b, int j) {
    const int p = B.pages[(size_t)b * B.max_pages + (unsigned)j / (unsigned)B.page_size];
    return p >= 0 && p < B.n_pages ? p : -1;
}

PP_DEVINL long long entry_offset(const BatchArgs& B, const PageArgs& C, int page, int j) {
    return (long long)page * C.page_stride + (long long)((unsigned)j % (unsigned)B.page_size) * C.token_stride;
}

// Sequence of token t: the last b with q_start[b] <= t.  One warp; 32 probes
// a step, so up to 1024 sequences take two dependent loads.
PP_DEVINL int find_seq(const BatchArgs& B, int t, int lane) {
    int lo = 0, hi = B.n_seqs;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const int at = lo + lane * step;
        const unsigned le = __ballot_sync(kFull, at < hi && B.q_start[at < hi ? at : lo] <= t);
        const int c = __popc(le);
        if (c == 0) break;
        lo += (c - 1) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

}  // namespace pp
