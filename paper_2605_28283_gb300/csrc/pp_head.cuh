// A head's row of D elements over the lanes of a group: norm and rotation.
//
// A row is cut into vectors of V elements (16 bytes, or 2 elements where the
// rotated part does not split into whole vectors) and into units of two
// vectors, so that both elements of a rotated pair lie in one lane: vectors
// (u, u + rv) of half-split pairs, (2 u, 2 u + 1) of interleaved ones and of
// the elements that are not rotated.  A group of G lanes (a power of two)
// holds the row, UPL units a lane; only the sum of squares crosses lanes.
// Pair p of the rotated ones belongs to unit p / V in both layouts.
#pragma once

#include "pp_attn.h"
#include "pp_tc_attn.cuh"
#include "pp_vec.cuh"

namespace pp {

// Units of a row (host).
template <int V>
int head_units(const HeadArgs& h) {
    return (h.head_dim / V + 1) / 2;
}

// Per-token factors of the rotated pairs in shared memory: pairs p and p + 1 of
// a unit side by side as (cos, cos, sin, sin), 16 bytes, and the units' side by
// side for each such two, so that the 16-byte reads of neighbouring lanes do not
// meet in a bank.
PP_DEVINL void put_pair(float* cs, int p, int V, int pitch, float2 v) {
    float* at = cs + (p % V / 2 * pitch + p / V) * 4 + (p & 1);
    at[0] = v.x;
    at[2] = v.y;
}

// Factors of one token by `n` threads.
PP_DEVINL void fill_pairs(float* cs, const HeadArgs& h, int V, int pos, int tid, int n) {
    const int pitch = (h.rot_dim / 2 + V - 1) / V;
    for (int p = tid; p < h.rot_dim / 2; p += n) {
        const float2 v = cos_sin(pos, h.inv_freq[p]);
        put_pair(cs, p, V, pitch, make_float2(v.x * h.scale, v.y * h.scale));
    }
}

using F2 = unsigned long long;  // two fp32 values, for the instructions that take two at once

template <typename T, int V, bool HALF, int UPL>
struct HeadLane {
    static constexpr int kBytes = V * (int)sizeof(T), V2 = V / 2;
    int va[UPL], vb[UPL];           // vectors of the lane's units, or -1
    bool turn_a[UPL], turn_b[UPL];  // rotated
    int unit[UPL];

    PP_DEVINL HeadLane(const HeadArgs& h, int lane) {  // lane in its group
        const int nvec = h.head_dim / V, rv = HALF ? h.rot_dim / 2 / V : 0;
#pragma unroll
        for (int k = 0; k < UPL; k++) {
            const int u = lane + k * h.group;
            unit[k] = u;
            va[k] = HALF && u < rv ? u : 2 * u;
            vb[k] = HALF && u < rv ? u + rv : 2 * u + 1;
            turn_a[k] = HALF ? u < rv : va[k] * V < h.rot_dim;
            turn_b[k] = HALF ? u < rv : vb[k] * V < h.rot_dim;
            if (va[k] >= nvec) va[k] = -1;
            if (vb[k] >= nvec) vb[k] = -1;
        }
    }
    // cosines and sines of the lane's pairs, from a token's table
    struct Factors {
        float c[UPL][V], s[UPL][V];
    };
    PP_DEVINL void factors(const float* cs, const HeadArgs& h, Factors& f) const {
        const int pitch = (h.rot_dim / 2 + V - 1) / V;
#pragma unroll
        for (int k = 0; k < UPL; k++) {
            if (!turn_a[k]) continue;
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                if (!HALF && i * 2 >= V && !turn_b[k]) continue;
                const float4 v = *reinterpret_cast<const float4*>(cs + (i / 2 * pitch + unit[k]) * 4);
                f.c[k][i] = v.x;
                f.c[k][i + 1] = v.y;
                f.s[k][i] = v.z;
                f.s[k][i + 1] = v.w;
            }
        }
    }
    // the lane's vectors of a row (zeros where it holds nothing)
    PP_DEVINL void load(const char* row, Vec<T, V> (&x)[UPL][2]) const {
#pragma unroll
        for (int k = 0; k < UPL; k++) {
            x[k][0].raw = x[k][1].raw = typename Raw<kBytes>::type{};
            if (va[k] >= 0) x[k][0].load(row + va[k] * kBytes);
            if (vb[k] >= 0) x[k][1].load(row + vb[k] * kBytes);
        }
    }
    // ... from a thread's places in shared memory, `step` bytes apart
    PP_DEVINL void load_own(const unsigned char* from, int step, bool in, Vec<T, V> (&x)[UPL][2]) const {
#pragma unroll
        for (int k = 0; k < UPL; k++) {
            x[k][0].raw = x[k][1].raw = typename Raw<kBytes>::type{};
            if (in && va[k] >= 0) x[k][0].raw = *reinterpret_cast<const typename Raw<kBytes>::type*>(from + 2 * k * step);
            if (in && vb[k] >= 0) x[k][1].raw = *reinterpret_cast<const typename Raw<kBytes>::type*>(from + (2 * k + 1) * step);
        }
    }
    PP_DEVINL void store(char* row, const Vec<T, V> (&x)[UPL][2]) const {
#pragma unroll
        for (int k = 0; k < UPL; k++) {
            if (va[k] >= 0) x[k][0].store(row + va[k] * kBytes);
            if (vb[k] >= 0) x[k][1].store(row + vb[k] * kBytes);
        }
    }
    PP_DEVINL static void widen(const Vec<T, V> (&x)[UPL][2], F2 (&f)[UPL][2][V2]) {
#pragma unroll
        for (int k = 0; k < UPL; k++)
#pragma unroll
            for (int v = 0; v < 2; v++)
#pragma unroll
                for (int i = 0; i < V2; i++) f[k][v][i] = pair2(x[k][v].get(2 * i), x[k][v].get(2 * i + 1));
    }
    PP_DEVINL static void narrow(const F2 (&f)[UPL][2][V2], Vec<T, V> (&x)[UPL][2]) {
#pragma unroll
        for (int k = 0; k < UPL; k++)
#pragma unroll
            for (int v = 0; v < 2; v++)
#pragma unroll
                for (int i = 0; i < V2; i++) {
                    float a, b;
                    unpair2(f[k][v][i], a, b);
                    x[k][v].set2(2 * i, a, b);
                }
    }
    // weights of a norm (of elements, in T); ones without
    PP_DEVINL void weights(const char* gamma, F2 (&g)[UPL][2][V2]) const {
#pragma unroll
        for (int k = 0; k < UPL; k++)
#pragma unroll
            for (int s = 0; s < 2; s++) {
                const int v = s ? vb[k] : va[k];
                Vec<T, V> x;
                x.raw = typename Raw<kBytes>::type{};
                if (gamma && v >= 0) x.raw = *reinterpret_cast<const typename Raw<kBytes>::type*>(gamma + v * kBytes);
#pragma unroll
                for (int i = 0; i < V2; i++) g[k][s][i] = gamma ? pair2(x.get(2 * i), x.get(2 * i + 1)) : pair2(1.f, 1.f);
            }
    }
    // the group's sum of a value a lane
    PP_DEVINL static float group_sum(float v, int group) {
        for (int o = group >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
        return v;
    }
    PP_DEVINL static float dot(const F2 (&a)[UPL][2][V2], const F2 (&b)[UPL][2][V2]) {
        F2 s[2] = {0ull, 0ull};
#pragma unroll
        for (int k = 0; k < UPL; k++)
#pragma unroll
            for (int i = 0; i < V2; i++) {
                s[0] = fma2(a[k][0][i], b[k][0][i], s[0]);
                s[1] = fma2(a[k][1][i], b[k][1][i], s[1]);
            }
        float x, y;
        unpair2(add2(s[0], s[1]), x, y);
        return x + y;
    }
    // BACK: rotated by the negative angle
    template <bool BACK = false>
    PP_DEVINL void rotate(F2 (&f)[UPL][2][V2], const Factors& w) const {
#pragma unroll
        for (int k = 0; k < UPL; k++) {
            if (HALF) {
                if (!turn_a[k]) continue;
#pragma unroll
                for (int i = 0; i < V2; i++) {
                    const F2 c = pair2(w.c[k][2 * i], w.c[k][2 * i + 1]), s = pair2(w.s[k][2 * i], w.s[k][2 * i + 1]),
                             n = pair2(-w.s[k][2 * i], -w.s[k][2 * i + 1]);
                    const F2 a = f[k][0][i], b = f[k][1][i];
                    f[k][0][i] = fma2(a, c, mul2(b, BACK ? s : n));
                    f[k][1][i] = fma2(b, c, mul2(a, BACK ? n : s));
                }
            } else {
#pragma unroll
                for (int v = 0; v < 2; v++) {
                    if (!(v ? turn_b[k] : turn_a[k])) continue;
#pragma unroll
                    for (int i = 0; i < V2; i++) {
                        const float c = w.c[k][v * V2 + i], s = BACK ? -w.s[k][v * V2 + i] : w.s[k][v * V2 + i];
                        float a, b;
                        unpair2(f[k][v][i], a, b);
                        f[k][v][i] = fma2(f[k][v][i], pair2(c, c), mul2(pair2(b, a), pair2(-s, s)));
                    }
                }
            }
        }
    }
    PP_DEVINL static void scale_by(F2 (&f)[UPL][2][V2], float r, const F2 (&g)[UPL][2][V2]) {
        const F2 r2 = pair2(r, r);
#pragma unroll
        for (int k = 0; k < UPL; k++)
#pragma unroll
            for (int s = 0; s < 2; s++)
#pragma unroll
                for (int i = 0; i < V2; i++) f[k][s][i] = mul2(mul2(f[k][s][i], r2), g[k][s][i]);
    }
};

// 1 / root mean square of a row whose squares sum to ss.
// (rsqrtf is good to 2 ulp; 1 / D is rounded on the host.)
PP_DEVINL float inverse_rms(float ss, const HeadArgs& h) { return rsqrtf(fmaf(ss, h.inv_dim, h.eps)); }

}  // namespace pp
