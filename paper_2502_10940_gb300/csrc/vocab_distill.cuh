// vocab_distill.cuh -- the distillation loss against a teacher's most likely tokens, and its gradient.
#pragma once
#include "vocab_rows.cuh"

namespace cola {

// ------------------------------------------------------------- distillation
// r + exp(-r) - 1 >= 0.  Where q and p both sum to 1, KL(q || p) is the sum of
// q excess(log q / p): a sum of nonnegative terms, exact to a few ulp where
// that of q log(q / p) cancels.  (From r = -1 down nothing does, while q may be too
// small a number to hold its digits and exp(-r) too large a one: there an entry's
// term is p + q (r - 1).)
__device__ __forceinline__ float excess(float r)
{
    if (fabsf(r) < 0.3f)
        return __fmul_rn(r * r, fmaf(-r, fmaf(-r, fmaf(-r, fmaf(-r, fmaf(r, -1.f / 5040, 1.f / 720), 1.f / 120), 1.f / 24),
                                              1.f / 6), 0.5f));
    return r + expm1f(-r);
}

// A teacher's list, taken in by every CTA of the row: entry i by thread i mod GT.
template <int GT>
struct ListShared {
    int id[VOCAB_MAX_K];                    // -1: no token
    float u[VOCAB_MAX_K], x[VOCAB_MAX_K];   // the teacher's exponent, the student's logit
    float2 student[Group<GT>::W], teacher[Group<GT>::W];   // maximum and sum, per warp
    float sum[Group<GT>::W];
    unsigned int edges;                     // bits of the row's edge elements that are on the list
};

template <class T>
using Bits = typename Elem<T>::Bits;        // a bit per element of a tile that a thread holds

// PASS: the forward, forward and backward, or the backward from saved statistics.
// The listed tokens' sums are apart from the rest's from the start: they are
// struck from the registers (one word of bits per thread and tile) before the
// row's maximum and sum, so that the rest's probability is its own sum, down to
// any size, and not 1 - sum p.  The first half of the time of a short row goes by
// on the list's way: ids, then the student's logits at them, both under way
// while the row is read.  A step of 16384 x 32000 with lists of 64 takes 331 us,
// 6.3 TB/s, of 17,500 instructions a row where the cross entropy's 13,200 leave
// HBM the bound; a forward of 4096 x 200000 with lists of 128, 246 us (6.7 TB/s);
// a backward of 8192 x 65536 with lists of 32, 308 us (7.0 TB/s).
// (A warp's row and its gradient need more registers than eight CTAs' 64: 160 us on six
// against 164 us for a step of 65536 x 2000 with lists of 64; the forward 135 us on eight, 153 us on six.)
template <class T, int PASS, int GT, bool APART>
__global__ void __launch_bounds__(Group<GT>::THREADS, GT == 32 && PASS != VOCAB_FWD ? 6 : Group<GT>::CTAS)
    topk_distill_kernel(const VocabParams P)
{
    constexpr int E = Elem<T>::E;
    using G = Group<GT>;
    extern __shared__ unsigned long long listed_raw[];   // forward: a word of bits per thread and tile
    __shared__ float4 slots[GT == 32 || PASS == VOCAB_BWD ? 1 : CLUSTER_MAX * G::W];
    __shared__ ListShared<GT> lists[G::ROWS];
    const G g;
    if (GT == 32 && g.row >= P.n) return;
    const bool cluster = g.parts > 1;
    if (cluster) cluster_arrive();
    const Row<T> row(static_cast<const T*>(P.logits) + g.row * P.ld, P.vocab);
    const Part<T, GT> part(row, g, P.each);
    ListShared<GT>& list = lists[g.slot];
    // the list's loads are under way before the row's
    const float shift = P.rest && P.t_lse ? P.t_lse[g.row] : 0.f;
    const long long t0 = g.tid < P.k ? P.t_ids[g.row * P.k + g.tid] : -1;
    const float u0 = g.tid < P.k ? P.t_vals[g.row * P.k + g.tid] : 0.f;
    uint4 d[NV];
    part.load(row, g, 0, d);
    if (PASS == VOCAB_STEP) part.prefetch(row, g);
    if (g.warp == 0 && g.row + P.ahead < P.n) {   // a later row's list
        const long long at = (g.row + P.ahead) * P.k;
        if (g.lane * 16 < P.k) prefetch_l2(P.t_ids + at + g.lane * 16);
        if (g.lane * 32 < P.k) prefetch_l2(P.t_vals + at + g.lane * 32);
    }
    const bool edge = g.has_edges() && g.lane < row.edges();
    const int edge_id = edge ? row.edge(g.lane) : -1;
    float xe = edge ? Elem<T>::get(row.p + edge_id) : NEG_INF;
    const float w = PASS != VOCAB_FWD ? P.dloss[g.row] : 0.f;
    float m = 0.f, logs = 0.f, mr = 0.f, logr = 0.f, s, sr;
    if (PASS == VOCAB_BWD) {
        const float4 st = reinterpret_cast<const float4*>(P.stats)[g.row];
        m = st.x, logs = st.y, mr = st.z, logr = st.w;
        s = expf(logs), sr = expf(logr);
    }
    Bits<T>* listed = reinterpret_cast<Bits<T>*>(listed_raw) + g.slot * GT;
    if (PASS != VOCAB_BWD) {
        for (int t = 0; t < part.tiles; ++t) listed[t * GT + g.tid] = 0;
        if (g.tid == 0) list.edges = 0;
        G::sync();
    }
    const bool lister = g.warp * 32 < P.k;   // the warp has entries
    float x0 = NEG_INF;                      // the thread's first entry's, under way until after the barrier
    if (lister) {
        float um = NEG_INF, us = 0.f;
        for (int i = g.tid; i < P.k; i += GT) {
            const long long t = i == g.tid ? t0 : P.t_ids[g.row * P.k + i];
            const bool there = t >= 0 && t < P.vocab;
            const int id = there ? static_cast<int>(t) : -1;
            if (there) {
                if (i == g.tid) x0 = Elem<T>::get(row.p + id);
                if (PASS != VOCAB_BWD) {
                    const int at = id - row.head, v = at / E - part.begin, tile = v / G::TILE;
                    if (at < 0 || at >= row.full * E)
                        atomicOr(&list.edges, 1u << (at < 0 ? id : row.head + at - row.full * E));
                    else if (v >= 0 && part.begin + v < part.end)
                        atomicOr(listed + tile * GT + v % GT, static_cast<Bits<T>>(1) << (v % G::TILE / GT * E + at % E));
                }
            }
            const float u = there ? fmaf(i == g.tid ? u0 : P.t_vals[g.row * P.k + i], P.t_c, -shift) : NEG_INF;
            list.id[i] = id;
            list.u[i] = u;
            um = max_nan(um, u);
        }
        um = P.rest ? 0.f : max_nan_warp(um);
        for (int i = g.tid; i < P.k; i += GT)
            if (list.id[i] >= 0 && um != NEG_INF) us += expf(list.u[i] - um);
        us = sum_warp(us);
        if (g.lane == 0) list.teacher[g.warp] = make_float2(um, us);
    }
    if (PASS != VOCAB_BWD) {
        G::sync();
        if (edge && list.edges >> g.lane & 1) xe = NEG_INF;
    }
    // the student's statistics on the list, a share per warp (the gathers were issued before the barrier)
    const auto gather = [&]() {
        if (!lister) return;
        float xm = NEG_INF, xs = 0.f;
        for (int i = g.tid; i < P.k; i += GT) {
            const int id = list.id[i];
            const float x = i == g.tid ? x0 : id >= 0 ? Elem<T>::get(row.p + id) : NEG_INF;
            list.x[i] = x;
            xm = max_nan(xm, x);
        }
        xm = max_nan_warp(xm);
        for (int i = g.tid; i < P.k; i += GT)
            if (list.id[i] >= 0 && xm != NEG_INF) xs += ex2((list.x[i] - xm) * P.c2);
        xs = sum_warp(xs);
        if (g.lane == 0) list.student[g.warp] = make_float2(xm, xs);
    };
    Acc r = acc_none();
    if (PASS == VOCAB_BWD) {
        gather();
        // in place: the list's logits are read before any CTA of the row stores
        if (cluster) {
            cluster_wait();
            cluster_sync();
        } else {
            G::sync();
        }
    } else {
        Acc a = acc_none();
        for (int t = 0; t < part.tiles; ++t) {
            if (t > 0) part.load(row, g, t, d);
            const Bits<T> mine = listed[t * GT + g.tid];
            if (mine) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const uint32_t b = static_cast<uint32_t>(mine >> (j * E)) & ((1u << E) - 1);
                    if (b) Elem<T>::ban(d[j], b);
                }
            }
            const Acc b = acc_tile<T, false>(d, part.used(t), Elem<T>::max_of(d), P.c2);
            a = t > 0 ? acc_merge<false>(a, b, P.c2) : b;
        }
        if (g.has_edges() && row.edges() > 0) a = acc_merge<false>(a, acc_one(xe), P.c2);
        gather();
        r = acc_warp<false>(a, P.c2);
        if (GT == 32) {
            G::sync();
        } else {
            exchange(r, 0.f, g, slots);
            if (PASS == VOCAB_FWD && (g.rank != 0 || !lister)) {
                if (g.rank == 0) __syncthreads();
                return;
            }
            r = acc_slots<GT, false>(slots, G::W * g.parts, g, P.c2);
        }
        mr = r.m, sr = r.s;
    }
    // the list's statistics over its warps: the student's, the teacher's
    Acc l = acc_none();
    float um = NEG_INF, us = 0.f;
    if (g.lane < G::W && g.lane * 32 < P.k) {
        const float2 o = list.student[g.lane], q = list.teacher[g.lane];
        l = Acc{o.x, o.y, 0.f};
        um = q.x, us = q.y;
    }
    l = acc_warp<false>(l, P.c2);
    if (P.rest) {
        us = sum_warp(us);
    } else {
        const float uml = max_nan_warp(um);
        us = sum_warp(us == 0.f ? 0.f : us * expf(um - uml));
        um = uml;
    }
    if (PASS != VOCAB_BWD) {
        m = max_nan(l.m, r.m);
        s = acc_to<false>(l, m, P.c2).s + acc_to<false>(r, m, P.c2).s;
    }
    const float m0 = m == NEG_INF ? 0.f : m;
    // teacher: q_k = exp(u_k - um) / us, or exp(u_k) = q_k where the rest counts; Q = sum q;
    // the rest is an entry of its own where q_R > 0
    const float Q = P.rest ? us : us == 0.f ? 0.f : us - us + 1.f;
    const float qr = P.rest && mr != NEG_INF ? fmaxf(1.f - Q, 0.f) : 0.f;
    const bool entry = qr > 0.f;
    const float wt = w * P.temperature;
    const bool live = w != 0.f && m != NEG_INF;
    float logpr = 0.f;
    // loss, and the list's gradients (stored over the row's below)
    float kl = 0.f;
    if (lister) {
        if (PASS != VOCAB_BWD) {
            logs = m == NEG_INF ? 0.f : logf(s);
            logr = mr == NEG_INF ? 0.f : logf(sr);
        }
        logpr = __fadd_rn(fmaf(mr - m0, P.c, logr), -logs);
        const float u_top = P.rest || us == 0.f ? 0.f : um, log_us = P.rest || us == 0.f ? 0.f : logf(us);
        for (int i = g.tid; i < P.k; i += GT) {
            if (list.id[i] < 0) continue;
            const float logq = (list.u[i] - u_top) - log_us, q = us == 0.f ? 0.f : expf(logq);
            // (roundings written out: the same loss from passes that share a row alike)
            const float logp = fmaf(list.x[i] - m0, P.c, -logs), p = expf(logp);
            if (PASS != VOCAB_BWD) {
                const float r = __fadd_rn(logq, -logp);
                float term;
                if (!entry) term = q > 0.f ? __fmul_rn(q, r) : 0.f * q;
                else if (!(q > 0.f)) term = p;
                else if (r > -1.f) term = __fmul_rn(q, excess(r));
                else term = fmaf(q, __fadd_rn(r, -1.f), p);
                kl = __fadd_rn(kl, term);
            }
            if (PASS != VOCAB_FWD) list.u[i] = wt * ((entry ? 1.f : Q) * p - q);
        }
        if (PASS != VOCAB_BWD) {
            kl = sum_warp(kl);
            if (g.lane == 0) list.sum[g.warp] = kl;
        }
    }
    if constexpr (PASS != VOCAB_FWD) {
        T* out = static_cast<T*>(P.dlogits) + g.row * P.ld_d;
        uint4* vout = reinterpret_cast<uint4*>(out + row.head);
        const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15u) == 0;
        const bool near = fabsf(mr * P.c2) < NEAR;
        const Base base(mr, P.c2);
        // rate of exp(c (x - mr)): with the rest (Q - sum p) / sr, else Q p_R / sr
        const float rate = mr == NEG_INF ? 0.f
                           : entry       ? wt * (Q - acc_to<false>(l, m, P.c2).s * rcp(s)) * rcp(sr)
                                         : wt * Q * ex2((mr - m) * P.c2) * rcp(s);
        const float A = rate * ex2(-base.delta);
        const auto one = [&](float x) -> float {
            if (!live || mr == NEG_INF) return 0.f;
            return rate * ex2((x - mr) * P.c2);
        };
        if (!APART && live && near && same) {
            const Pair cc = pair(P.c2, P.c2), nb = pair(-base.b, -base.b), A2 = pair(A, A);
            for (int t = part.tiles - 1; t >= 0; --t) {
                const int first = part.at(g, t), left = part.left(g, t);
                if (t < part.tiles - 1 || (PASS == VOCAB_BWD && t > 0)) part.template load<true>(row, g, t, d);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    if (j % 2 == 0 && j >= part.used(t)) break;
                    float x[E];
                    Elem<T>::unpack(d[j], x);
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        float y0, y1;
                        split(fma2(pair(x[e], x[e + 1]), cc, nb), y0, y1);
                        split(mul2(pair(ex2(y0), ex2(y1)), A2), x[e], x[e + 1]);
                    }
                    if (left > j * GT) __stcs(vout + first + j * GT, Elem<T>::pack(x));
                }
            }
        } else {
            for (int t = 0; t < part.tiles; ++t) {
                const int first = part.at(g, t);
                emit_again<T, GT, APART>(row.vec() + first, out + row.head + first * E, part.left(g, t), min(part.used(t), NV),
                                         mr, P.c2, rate, 0.f, live && mr != NEG_INF);
            }
        }
        if (edge) Elem<T>::put(out + edge_id, one(xe));
        G::sync();
        for (int i = g.tid; live && i < P.k; i += GT) {
            const int id = list.id[i];
            if (id < 0) continue;
            const int at = id - row.head, v = at / E;
            const bool vector = at >= 0 && v < row.full;
            if (vector ? v >= part.begin && v < part.end : g.rank == 0) Elem<T>::put(out + id, list.u[i]);
        }
    } else {
        G::sync();
    }
    if (PASS != VOCAB_BWD && g.rank == 0 && g.tid == 0) {
        kl = 0.f;
        for (int i = 0; i < G::W && i * 32 < P.k; ++i) kl += list.sum[i];
        if (entry) kl = __fadd_rn(kl, __fmul_rn(qr, excess(__fadd_rn(log1pf(-Q), -logpr))));
        P.loss[g.row] = P.temperature * P.temperature * kl;
        if (PASS == VOCAB_FWD && P.stats) reinterpret_cast<float4*>(P.stats)[g.row] = make_float4(m, logs, mr, logr);
    }
}

}  // namespace cola
