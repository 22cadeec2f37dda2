// Division of an attention call over the CTAs of one launch.
//
// An item is a tile of up to ROWS query rows of one (sequence, key head): the
// rows are the (new token, query head of the group) pairs, token-major.  Its
// work is the key tiles of TOK tokens that any of its rows may see.  All
// items' tiles form one line, ordered by sequence, key head and row tile, and
// CTA c of C takes the c-th of C equal stretches of it, so that every SM
// streams the same number of keys however ragged the batch is, without the
// host knowing a length.  A stretch covers whole items and at most one part
// of an item at each end.  A part that is not its whole item leaves its
// unnormalised sum, maximum and weight sum in the workspace; the CTA that
// arrives last, or a second kernel, adds an item's parts up in stretch order
// (so the result does not depend on who does it).
#pragma once

#include "pp_batch.cuh"

namespace pp {

constexpr int kLongStretch = 16;  // tiles of a stretch from which items are padded

// Quotient of two non-negative numbers, in 32 bits where they fit (a 64-bit
// division is a call of a hundred instructions).
PP_DEVINL long long quotient(long long a, long long b) {
    if ((unsigned long long)(a | b) >> 32 == 0) return (long long)((unsigned)a / (unsigned)b);
    return a / b;
}

// Tiles of the key line: the schedule is recomputed by whoever walks it, from
// the lengths alone.  GROUPED: 1 << shift CTAs side by side take as many key
// heads side by side, the same stretch of a line that has one such group of heads
// for a head, so that what lies together in memory is read at the same time; and
// where stretches are long, an item counts `pad` tiles more than it has (ahead of
// its own), for what starting and finishing it costs, so that CTAs with many
// short items get fewer tiles.
template <int ROWS, int TOK, bool GROUPED = false>
struct Sched {
    const AttnArgs* a;
    long long total;  // key tiles of the line
    int ctas;         // CTAs (groups of them) with work
    int pad_, shift_;
    PP_DEVINL int pad() const { return GROUPED ? pad_ : 0; }
    PP_DEVINL int shift() const { return GROUPED ? shift_ : 0; }
    PP_DEVINL int heads() const { return a->n_kv_heads >> shift(); }

    // Sequence b, without its tokens where another launch takes it.
    PP_DEVINL Seq sequence(int b) const {
        Seq s = load_seq(a->batch, b);
        const unsigned rows = (unsigned)s.n * (unsigned)a->group;
        if (rows < a->min_rows || rows > a->max_rows) s.n = 0;
        return s;
    }

    PP_DEVINL int row_tiles(const Seq& s) const { return (int)(((unsigned)s.n * (unsigned)a->group + ROWS - 1) / ROWS); }

    // Entries that row tile j's rows may see (all of a masked tree's).
    PP_DEVINL int key_end(const Seq& s, int j) const {
        if (a->mask) return s.ctx + s.n;
        const unsigned last = ((unsigned)(j + 1) * ROWS - 1u) / (unsigned)a->group;  // rows stay below 2^31
        return s.ctx + min(s.n, (int)last + 1);
    }
    PP_DEVINL int key_tiles(const Seq& s, int j) const { return max(1, (key_end(s, j) + TOK - 1) / TOK); }

    // An item's length on the line.
    PP_DEVINL int length(const Seq& s, int j) const { return key_tiles(s, j) + pad(); }

    // Length of one key head of a sequence on the line.
    PP_DEVINL long long head_tiles(const Seq& s) const {
        const int m = row_tiles(s);
        if (a->mask || m <= 1) return m ? (long long)m * length(s, m - 1) : 0;
        long long sum = 0;
        for (int j = 0; j < m; j++) sum += length(s, j);
        return sum;
    }

    // Stretches: the first `longer` ones of `each` + 1 tiles, the others of `each`.
    long long each;
    int longer;
    // Short stretches: as few CTAs as finish with the longest of them, and
    // `least` tiles each, since every part of a split item costs.  Long ones:
    // all CTAs.  "Short" as up to 1 / 4 / 16 tiles, bf16: one token over 2048
    // entries of 32 key heads 16.2 / 13.5 / 13.5 us, two trees of 32 tokens over
    // 4000 (8 key heads) 21.0 / 18.6 / 18.5, 8 trees of 32 over 500 to 6000 35.1 /
    // 35.3 / 37.5; fp32: one token over 1024 22.8 / 16.3 / 16.3, over 2048 35.4 /
    // 40.8 / 40.5, over 4096 56.4 / 57.1 / 61.2.
    PP_DEVINL void deal(long long total_, int grid, int least) {
        total = total_;
        const long long longest = max(quotient(total + grid - 1, grid), (long long)least);
        ctas = longest > 4 ? grid : (int)quotient(total + longest - 1, longest);
        if (ctas == 0) return;
        each = quotient(total, ctas);
        longer = (int)(total - each * ctas);
    }
    PP_DEVINL long long begin_of(int c) const { return each * c + min(c, longer); }
    // CTA whose stretch holds tile u
    PP_DEVINL int cta_of(long long u) const {
        const long long head = (each + 1) * longer;
        return u < head ? (int)quotient(u, each + 1) : longer + (int)quotient(u - head, each);
    }
};

// One CTA's share of an item.
struct Part {
    int b, h, j;       // sequence, key head, row tile
    Seq seq;
    int key_end;       // entries any row of the tile may see
    int t0, t1;        // key tiles of the part
    int tiles;         // key tiles of the item
    long long first;   // the item's first tile on the line
    PP_DEVINL bool whole() const { return t0 == 0 && t1 == tiles; }
};

// Walks the parts of one CTA's stretch.
template <int ROWS, int TOK, bool GROUPED = false>
struct Walk {
    Sched<ROWS, TOK, GROUPED> sched;
    long long at, end;  // the rest of the stretch
    long long base;     // line position of sequence b
    int b, h, j;
    long long head_base;  // line position of the current item
    Seq seq;
    int m;

    PP_DEVINL void enter(int b_, long long base_) {
        b = b_;
        base = base_;
        seq = sched.sequence(b);
        m = sched.row_tiles(seq);
        h = 0;
        j = 0;
        head_base = base;
        const long long per = sched.head_tiles(seq);
        if (per > 0) {
            h = (int)quotient(at - base, per);
            head_base = base + (long long)h * per;
        }
        while (m > 0 && j + 1 < m && head_base + sched.length(seq, j) <= at) {
            head_base += sched.length(seq, j);
            j++;
        }
    }

    // The next part; false at the end of the stretch.
    PP_DEVINL bool next(Part& p) {
        do {
            if (at >= end) return false;
            while (m == 0 || h >= sched.heads()) enter(b + 1, m == 0 ? base : head_base);
            const int pad = sched.pad();
            p.b = b;
            p.h = h << sched.shift() | ((int)blockIdx.x & ((1 << sched.shift()) - 1));
            p.j = j;
            p.seq = seq;
            p.key_end = sched.key_end(seq, j);
            p.tiles = sched.key_tiles(seq, j);
            p.first = head_base;
            const int len = p.tiles + pad, u1 = (int)min((long long)len, end - head_base);
            p.t0 = max((int)(at - head_base) - pad, 0);
            p.t1 = max(u1 - pad, 0);
            at = head_base + u1;
            if (u1 == len) {
                head_base += len;
                if (++j == m) {
                    j = 0;
                    h++;
                }
            }
        } while (GROUPED && p.t1 == 0);  // the stretch ends ahead of the item's first tile
        return true;
    }
};

// The line's length and this CTA's first sequence, by one whole warp: a lane
// counts a run of sequences, a scan over the lanes gives the total, and the
// lane whose run holds this CTA's first tile looks for its sequence.  Short
// code on purpose: it runs once, from a cold instruction cache.
template <int ROWS, int TOK, bool GROUPED = false>
PP_DEVINL Walk<ROWS, TOK, GROUPED> start_walk(const AttnArgs* a, int lane, bool report, int least, int pad = 0, int shift = 0) {
    Walk<ROWS, TOK, GROUPED> w;
    w.sched.a = a;
    w.sched.pad_ = 0;
    w.sched.shift_ = shift;
    const int grid = (int)gridDim.x >> w.sched.shift(), me = (int)blockIdx.x >> w.sched.shift();
    const int B = a->batch.n_seqs, run = (B + 31) / 32;
    const int b0 = min(lane * run, B), b1 = min(b0 + run, B);
    long long mine = 0, items = 0;
#pragma unroll 2
    for (int b = b0; b < b1; b++) {
        const Seq q = w.sched.sequence(b);
        if (report && q.bad) record_status(a->status, PP_ERR_INVALID_ARG);
        mine += w.sched.head_tiles(q);
        if (GROUPED) items += w.sched.row_tiles(q);
    }
    mine *= w.sched.heads();
    if (GROUPED) {
        // stretches of at least kLongStretch tiles
        long long all = mine;
#pragma unroll 1
        for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(kFull, all, o);
        if (all >= (long long)kLongStretch * grid) w.sched.pad_ = pad;
        mine += items * w.sched.heads() * w.sched.pad_;
    }
    long long sum = mine;
#pragma unroll 1
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(kFull, sum, o);
        if (lane >= o) sum += u;
    }
    w.sched.deal(__shfl_sync(kFull, sum, 31), grid, least);
    w.at = w.end = 0;
    w.m = 0;
    if (me >= w.sched.ctas) return w;
    w.at = w.sched.begin_of(me);
    w.end = w.sched.begin_of(me + 1);
    long long base = sum - mine;
    int b = b0;
    const bool here = base <= w.at && w.at < sum;
    if (here) {
#pragma unroll 1
        for (; b + 1 < b1; b++) {
            const long long t = w.sched.head_tiles(w.sched.sequence(b)) * w.sched.heads();
            if (base + t > w.at) break;
            base += t;
        }
    }
    const int owner = __ffs(__ballot_sync(kFull, here)) - 1;
    w.b = __shfl_sync(kFull, b, owner) - 1;  // next() enters the sequence
    w.base = __shfl_sync(kFull, base, owner);
    return w;
}

// ------------------------------------------------------------ split items
// Partial results: CTA c has two places, for the item its stretch begins in
// (2 c) and for the one it ends in (2 c + 1); a place holds the sums
// [ROWS][D], then the maxima and the weight sums [ROWS] each.
template <int ROWS>
PP_DEVINL float* part_place(const AttnArgs& a, int c, bool tail) {
    return a.part + (size_t)(2 * c + (tail ? 1 : 0)) * ROWS * (a.head_dim + 2);
}

// Range of CTAs that hold a split item's parts.
template <int ROWS, int TOK>
struct Split {
    int c0, c1;      // (groups of) CTAs
    int step, lane;  // of a group: its CTAs, and this item's among them
    bool c0_tail;  // the first part lies in c0's second place
    Split() = default;
    template <bool GROUPED>
    PP_DEVINL Split(const Sched<ROWS, TOK, GROUPED>& s, const Part& p) {
        c0 = s.cta_of(p.first + s.pad());
        c1 = s.cta_of(p.first + s.pad() + p.tiles - 1);
        c0_tail = s.begin_of(c0) < p.first;
        step = 1 << s.shift();
        lane = (int)blockIdx.x & (step - 1);
    }
    PP_DEVINL int cta(int c) const { return c * step + lane; }
    PP_DEVINL float* place(const AttnArgs& a, int c) const { return part_place<ROWS>(a, cta(c), c == c0 && c0_tail); }
};

// Arrival of one part's CTA at its item, after a barrier behind the stores of
// the part; true for the last one, which then sees every part.  (The barrier
// orders the other threads' stores before this thread's release.)
PP_DEVINL bool arrive_last(unsigned* counter, unsigned parts) {
    unsigned old;
    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(old) : "l"(counter) : "memory");
    if (old + 1 != parts) return false;
    *counter = 0;  // at rest again; the next launch on the workspace is ordered behind this one
    return true;
}

// Address of row r of an item in out (or q, with its own stride).
PP_DEVINL long long row_offset(const AttnArgs& a, const Part& p, int row, long long stride, int esz) {
    const int tok = row / a.group, g = row - tok * a.group;
    return (long long)(p.seq.q0 + tok) * stride + ((long long)p.h * a.group + g) * a.head_dim * esz;
}

template <typename T>
PP_DEVINL void store4(char* dst, const float4& o, float f) {
    if (sizeof(T) == 4)
        *reinterpret_cast<float4*>(dst) = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
    else
        *reinterpret_cast<uint2*>(dst) = make_uint2(Elem<__nv_bfloat16>::pair(o.x * f, o.y * f),
                                                    Elem<__nv_bfloat16>::pair(o.z * f, o.w * f));
}

// Place of 4 sums, elements 4 d4.. of row r.  Many rows (by_row): a thread
// has a row, and the rows of a warp lie side by side; few: a row's elements do.
template <int ROWS>
PP_DEVINL size_t part_at(bool by_row, int D, int r, int d4) {
    return by_row ? ((size_t)d4 * ROWS + r) * 4 : (size_t)r * D + d4 * 4;
}

// Adds up the parts of an item for 4 N elements (from 4 d0 on) of row r (of
// the row tile) and writes them.  The parts are visible to the caller (arrival
// counter, or a launch of its own).  Bound by the latency of its loads: U parts
// are read at once, without a branch between the loads.  One token over 1024
// entries, joined inside the kernel: U = 1 12.9 us, 2 11.9, 4 11.3; 8 drafted
// trees: 44.2, 44.2, 42.3; in the fp32 kernel, longer code only costs
// (3 drafted trees: 18.7, 22.1, 21.2).
template <typename T, int ROWS, int TOK, int N, int U, bool BY_ROW>
PP_DEVINL void merge_row(const AttnArgs& a, const Part& p, const Split<ROWS, TOK>& sp, int r, int d0) {
    const int D = a.head_dim, d4s = D / 4;
    float m = -INFINITY, l = 0.f;
    float4 o[N];
#pragma unroll
    for (int i = 0; i < N; i++) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int c = sp.c0; c <= sp.c1; c += U) {
        float mc[U], lc[U];
        float4 v[U][N];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const float* pl = sp.place(a, min(c + u, sp.c1));
            mc[u] = __ldcg(pl + (size_t)ROWS * D + r);
            lc[u] = __ldcg(pl + (size_t)ROWS * (D + 1) + r);
#pragma unroll
            for (int i = 0; i < N; i++)
                v[u][i] = __ldcg(reinterpret_cast<const float4*>(pl + part_at<ROWS>(BY_ROW, D, r, min(d0 + i, d4s - 1))));
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (c + u > sp.c1) mc[u] = -INFINITY;
            top = fmaxf(top, mc[u]);
        }
        const float base = top == -INFINITY ? 0.f : top;  // nothing seen (or NaN scores only: the sums stay NaN)
        const float f = exp2f(m - base);
        m = top;
        l *= f;
#pragma unroll
        for (int i = 0; i < N; i++) {
            o[i].x *= f;
            o[i].y *= f;
            o[i].z *= f;
            o[i].w *= f;
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (c + u > sp.c1) continue;  // a repeated part (0 * NaN is NaN)
            const float w = exp2f(mc[u] - base);
            l += w * lc[u];
#pragma unroll
            for (int i = 0; i < N; i++) {
                o[i].x += w * v[u][i].x;
                o[i].y += w * v[u][i].y;
                o[i].z += w * v[u][i].z;
                o[i].w += w * v[u][i].w;
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    char* dst = a.out + row_offset(a, p, p.j * ROWS + r, a.out_stride, (int)sizeof(T));
#pragma unroll
    for (int i = 0; i < N; i++)
        if (d0 + i < d4s) store4<T>(dst + (d0 + i) * 4 * (int)sizeof(T), o[i], inv);
}

// All `rows` rows of an item of few, four elements a thread.
template <typename T, int ROWS, int TOK, int U>
PP_DEVINL void merge_few(const AttnArgs& a, const Part& p, const Split<ROWS, TOK>& sp, int rows, int tid, int nthr) {
    const int d4s = a.head_dim / 4;
#pragma unroll 1
    for (int e = tid; e < rows * d4s; e += nthr) merge_row<T, ROWS, TOK, 1, U, false>(a, p, sp, e / d4s, e % d4s);
}

}  // namespace pp
