// vocab_logprob.cuh -- log probabilities of given tokens with the row's entropy, and their gradient.
#pragma once
#include "vocab_rows.cuh"

namespace cola {

// ------------------------------------------------- token log probabilities
// Bound by HBM: a row is read once (a step's second read hits L2), a gradient
// written once.  Per element the forward takes 3.5 instructions (half a packed
// maximum, an unpacking, half a packed fused product and sum each, an exponential)
// and the gradient as many; an SM has about 11 for each bf16 logit that HBM gives
// it.  bf16 logits, 32000 a row: forward of 8192 rows 77 us (6.8 TB/s), step of
// 32768 rows 598 us (7.0 TB/s); fp32 backward with entropy of 4096 x 65537, rows
// unaligned, 312 us (6.9 TB/s).
//
// The gradient of one CTA's share of a row.  H: with the entropy's term,
//   c p (-g - h (logp + H)) = 2^y (A + B y),   y = c2 x - base.b.
template <class T, int PASS, int GT, bool ENT, bool APART>
__device__ __forceinline__ void emit_logprob(const VocabParams& P, const Row<T>& row, const Part<T, GT>& part, const Group<GT>& g,
                                             float m, float inv_s, float logs, float H, float up_g, float up_h, int y, float xe,
                                             uint4 (&d)[NV])
{
    constexpr int E = Elem<T>::E;
    T* out = static_cast<T*>(P.dlogits) + g.row * P.ld_d;
    uint4* vout = reinterpret_cast<uint4*>(out + row.head);
    const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15u) == 0;
    const bool live = (up_g != 0.f || up_h != 0.f) && m != NEG_INF, near = fabsf(m * P.c2) < NEAR;
    const Base base(m, P.c2);
    const float scale = -P.c * inv_s * ex2(-base.delta);
    const float A = scale * (up_g + (ENT ? up_h * (H - logs - LN2 * base.delta) : 0.f)), B = ENT ? scale * up_h * LN2 : 0.f;
    const auto one = [&](float x) -> float {   // without the target's own term
        if (!live) return 0.f;
        const float l = (x - m) * P.c2, p = inv_s * ex2(l);
        return -P.c * p * (up_g + (ENT ? up_h * (LN2 * fmaxf(l, FLOOR) - logs + H) : 0.f));
    };
    if (!APART && live && near && same) {
        const Pair cc = pair(P.c2, P.c2), nb = pair(-base.b, -base.b), A2 = pair(A, A), B2 = pair(B, B);
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
                    const Pair w = pair(ex2(y0), ex2(y1));
                    split(mul2(w, ENT ? fma2(pair(fmaxf(y0, FLOOR), fmaxf(y1, FLOOR)), B2, A2) : A2), x[e], x[e + 1]);
                }
                if (left > j * GT) __stcs(vout + first + j * GT, Elem<T>::pack(x));
            }
        }
    } else {
        for (int t = 0; t < part.tiles; ++t) {
            const int first = part.at(g, t);
            emit_again<T, GT, APART>(row.vec() + first, out + row.head + first * E, part.left(g, t), min(part.used(t), NV), m,
                                     P.c2, -P.c * inv_s * (up_g + (ENT ? up_h * (H - logs) : 0.f)),
                                     ENT ? -P.c * inv_s * up_h * LN2 : 0.f, live);
        }
    }
    if (g.has_edges() && g.lane < row.edges()) {
        const int id = row.edge(g.lane);
        Elem<T>::put(out + id, one(xe) + (live && id == y ? P.c * up_g : 0.f));
    }
}

template <class T, int PASS, int GT, bool ENT, bool APART>
__global__ void __launch_bounds__(Group<GT>::THREADS, Group<GT>::CTAS) token_logprob_kernel(const VocabParams P)
{
    constexpr int E = Elem<T>::E;
    using G = Group<GT>;
    __shared__ float4 slots[PASS == VOCAB_BWD || GT == 32 ? 1 : CLUSTER_MAX * G::W];
    const G g;
    if (GT == 32 && g.row >= P.n) return;
    if (PASS != VOCAB_BWD && g.parts > 1) cluster_arrive();
    const Row<T> row(static_cast<const T*>(P.logits) + g.row * P.ld, P.vocab);
    const Part<T, GT> part(row, g, P.each);
    uint4 d[NV];
    part.load(row, g, 0, d);
    if (PASS == VOCAB_STEP) part.prefetch(row, g);
    const long long target = P.targets ? P.targets[g.row] : -1;
    const bool there = target >= 0 && target < P.vocab;
    const int y = there ? static_cast<int>(target) : -1;
    // the target's logit: for its log probability, and its own gradient (the
    // thread that holds its vector)
    const int vy = y >= row.head && y < row.head + row.full * E ? (y - row.head) / E : -1;
    const bool owner = PASS != VOCAB_FWD && part.owns(g, vy);
    float xy = 0.f, xe = NEG_INF, up_g = 0.f, up_h = 0.f;
    if (there && (owner || (PASS != VOCAB_BWD && g.rank == 0 && g.tid == 0))) xy = Elem<T>::get(row.p + y);
    if (g.has_edges() && g.lane < row.edges()) xe = Elem<T>::get(row.p + row.edge(g.lane));
    if (PASS != VOCAB_FWD) {
        up_g = there && P.dlogp ? P.dlogp[g.row] : 0.f;
        up_h = ENT && P.dentropy ? P.dentropy[g.row] : 0.f;
    }
    float m, s, logs = 0.f, H = 0.f;
    if (PASS == VOCAB_BWD) {
        const float4 st = reinterpret_cast<const float4*>(P.stats)[g.row];
        m = st.x, logs = st.y, H = st.z, s = expf(logs);
    } else {
        Acc a = acc_none();
        for (int t = 0; t < part.tiles; ++t) {
            if (t > 0) part.load(row, g, t, d);
            const Acc b = acc_tile<T, ENT>(d, part.used(t), Elem<T>::max_of(d), P.c2);
            a = t > 0 ? acc_merge<ENT>(a, b, P.c2) : b;
        }
        if (g.has_edges() && row.edges() > 0) a = acc_merge<ENT>(a, acc_one(xe), P.c2);
        a = acc_warp<ENT>(a, P.c2);
        if (GT != 32) {
            exchange(a, 0.f, g, slots);
            if (PASS == VOCAB_FWD && (g.rank != 0 || g.warp != 0)) return;
            a = acc_slots<GT, ENT>(slots, G::W * g.parts, g, P.c2);
        }
        m = a.m, s = a.s;
        if (ENT || (g.rank == 0 && g.warp == 0)) {
            logs = m == NEG_INF ? 0.f : logf(s);
            H = ENT && m != NEG_INF ? logs - LN2 * (a.t / s) : 0.f;
        }
    }
    if (PASS != VOCAB_BWD && g.rank == 0 && g.tid == 0) {
        if (P.logp) P.logp[g.row] = there ? (xy - (m == NEG_INF ? 0.f : m)) * P.c - logs : 0.f;
        if (ENT && P.entropy) P.entropy[g.row] = H;
        if (PASS == VOCAB_FWD && P.stats) reinterpret_cast<float4*>(P.stats)[g.row] = make_float4(m, logs, H, 0.f);
    }
    if constexpr (PASS != VOCAB_FWD) {
        const float inv_s = rcp(s);
        if (!ENT || up_h == 0.f) emit_logprob<T, PASS, GT, false, APART>(P, row, part, g, m, inv_s, logs, H, up_g, 0.f, y, xe, d);
        else emit_logprob<T, PASS, GT, true, APART>(P, row, part, g, m, inv_s, logs, H, up_g, up_h, y, xe, d);
        if (APART) __syncwarp();   // (the neighbouring lane may have stored that element)
        if (owner && m != NEG_INF && (up_g != 0.f || up_h != 0.f)) {   // over its own store of that vector
            const float l = (xy - m) * P.c2, p = inv_s * ex2(l);
            const float r = P.c * (up_g - p * (up_g + up_h * (LN2 * fmaxf(l, FLOOR) - logs + H)));
            Elem<T>::put(static_cast<T*>(P.dlogits) + g.row * P.ld_d + y, r);
        }
    }
}

}  // namespace cola
