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
#include "pp_vec.cuh"

namespace pp {

// Units of a row (host).
template <int V>
int head_units(const HeadArgs& h) {
    return (h.head_dim / V + 1) / 2;
}

// Per-token factors (cos, sin) in shared memory, laid out so that the 16-byte
// reads of neighbouring units lie side by side: two pairs of unit u at
// 16 (i / 2 * pitch + u).
PP_DEVINL int pair_slot(int p, int V, int pitch) { return (p % V / 2 * pitch + p / V) * 2 + (p & 1); }

// Factors of one token by `n` threads.
PP_DEVINL void fill_pairs(float2* cs, const HeadArgs& h, int V, int pos, bool inverse, int tid, int n) {
    const int pitch = (h.rot_dim / 2 + V - 1) / V;
    for (int p = tid; p < h.rot_dim / 2; p += n) {
        const float2 v = cos_sin(pos, h.inv_freq[p]);
        cs[pair_slot(p, V, pitch)] = make_float2(v.x * h.scale, (inverse ? -v.y : v.y) * h.scale);
    }
}

template <typename T, int V, bool HALF, int UPL>
struct HeadLane {
    static constexpr int kBytes = V * (int)sizeof(T);
    int va[UPL], vb[UPL];          // vectors of the lane's units, or -1
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
    // (cos, sin) of the lane's pairs, from a token's table
    PP_DEVINL void factors(const float2* cs, const HeadArgs& h, float2 (&f)[UPL][V]) const {
        const int pitch = (h.rot_dim / 2 + V - 1) / V;
#pragma unroll
        for (int k = 0; k < UPL; k++) {
            if (!turn_a[k]) continue;
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                if (!HALF && i * 2 >= V && !turn_b[k]) continue;
                const float4 v = *reinterpret_cast<const float4*>(cs + (i / 2 * pitch + unit[k]) * 2);
                f[k][i] = make_float2(v.x, v.y);
                f[k][i + 1] = make_float2(v.z, v.w);
            }
        }
    }
    PP_DEVINL void load(const char* row, Vec<T, V> (&x)[UPL][2]) const {
#pragma unroll
        for (int k = 0; k < UPL; k++) {
            if (va[k] >= 0) x[k][0].load(row + va[k] * kBytes);
            if (vb[k] >= 0) x[k][1].load(row + vb[k] * kBytes);
        }
    }
    PP_DEVINL void store(char* row, const Vec<T, V> (&x)[UPL][2]) const {
#pragma unroll
        for (int k = 0; k < UPL; k++) {
            if (va[k] >= 0) x[k][0].store(row + va[k] * kBytes);
            if (vb[k] >= 0) x[k][1].store(row + vb[k] * kBytes);
        }
    }
    // fp32 values (zeros where the lane holds nothing)
    PP_DEVINL void widen(const Vec<T, V> (&x)[UPL][2], float (&f)[UPL][2][V]) const {
#pragma unroll
        for (int k = 0; k < UPL; k++)
#pragma unroll
            for (int i = 0; i < V; i++) {
                f[k][0][i] = va[k] >= 0 ? x[k][0].get(i) : 0.f;
                f[k][1][i] = vb[k] >= 0 ? x[k][1].get(i) : 0.f;
            }
    }
    PP_DEVINL void narrow(const float (&f)[UPL][2][V], Vec<T, V> (&x)[UPL][2]) const {
#pragma unroll
        for (int k = 0; k < UPL; k++)
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                x[k][0].set2(i, f[k][0][i], f[k][0][i + 1]);
                x[k][1].set2(i, f[k][1][i], f[k][1][i + 1]);
            }
    }
    // weights of a norm (of elements, in T); ones without
    PP_DEVINL void weights(const char* gamma, float (&g)[UPL][2][V]) const {
#pragma unroll
        for (int k = 0; k < UPL; k++)
#pragma unroll
            for (int s = 0; s < 2; s++) {
                const int v = s ? vb[k] : va[k];
                typename Raw<kBytes>::type w{};
                if (gamma && v >= 0) w = *reinterpret_cast<const typename Raw<kBytes>::type*>(gamma + v * kBytes);
                Vec<T, V> x;
                x.raw = w;
#pragma unroll
                for (int i = 0; i < V; i++) g[k][s][i] = gamma ? x.get(i) : 1.f;
            }
    }
    // the group's sum of a value a lane
    PP_DEVINL static float group_sum(float v, int group) {
        for (int o = group >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
        return v;
    }
    PP_DEVINL static float dot(const float (&a)[UPL][2][V], const float (&b)[UPL][2][V]) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < UPL; k++)
#pragma unroll
            for (int i = 0; i < V; i++) {
                s[0] = fmaf(a[k][0][i], b[k][0][i], s[0]);
                s[1] = fmaf(a[k][1][i], b[k][1][i], s[1]);
            }
        return s[0] + s[1];
    }
    PP_DEVINL void rotate(float (&f)[UPL][2][V], const float2 (&c)[UPL][V]) const {
#pragma unroll
        for (int k = 0; k < UPL; k++) {
            if (HALF) {
                if (!turn_a[k]) continue;
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const float a = f[k][0][i], b = f[k][1][i];
                    f[k][0][i] = a * c[k][i].x - b * c[k][i].y;
                    f[k][1][i] = b * c[k][i].x + a * c[k][i].y;
                }
            } else {
#pragma unroll
                for (int s = 0; s < 2; s++) {
                    if (!(s ? turn_b[k] : turn_a[k])) continue;
#pragma unroll
                    for (int i = 0; i < V; i += 2) {
                        const float2 w = c[k][(s * V + i) / 2];
                        const float a = f[k][s][i], b = f[k][s][i + 1];
                        f[k][s][i] = a * w.x - b * w.y;
                        f[k][s][i + 1] = b * w.x + a * w.y;
                    }
                }
            }
        }
    }
    PP_DEVINL static void scale_by(float (&f)[UPL][2][V], float r, const float (&g)[UPL][2][V]) {
#pragma unroll
        for (int k = 0; k < UPL; k++)
#pragma unroll
            for (int s = 0; s < 2; s++)
#pragma unroll
                for (int i = 0; i < V; i++) f[k][s][i] = f[k][s][i] * r * g[k][s][i];
    }
};

// 1 / root mean square of a row whose squares sum to ss.
PP_DEVINL float inverse_rms(float ss, const HeadArgs& h) { return 1.0f / sqrtf(ss / (float)h.head_dim + h.eps); }

}  // namespace pp
