// Distillation of a draft model from the top logits of the target: loss and gradient.
//
// A row has the target's k listed tokens y_j with logits v_j, and the draft's logits z over the vocabulary.
//   q_v = exp(z_v/T) / sum_u exp(z_u/T)
//   p_j = exp(v_j/T - lse), R = max(0, 1 - sum p)      with the target's log-sum-exp: what the list leaves out is one
//                                                      more outcome, of draft probability Q = sum of q outside the list
//   p_j = exp(v_j/T) / sum_i exp(v_i/T), R = 0         without: the list is renormalised
//   loss = sum_j p_j (log p_j - log q_{y_j}) + R (log R - log Q)
//   d loss / d z_v = (mass q_v - p_v) / T              v in the list, mass = sum p + R
//                  = q_v (mass - R/Q) / T              v outside
// Only the k listed tokens differ from a multiple of q, so the gradient is one pass over the row and k corrections.
//
// Q is summed from the terms outside the list, not taken as 1 - sum of the listed q: the draft has most of its mass in
// the list, and the difference would keep few digits.  A bitmap of the CTA's part of the row tells list from rest.
// sum p, R and the loss are in 64 bits for the same reason; they are a few values per listed token.
//
// A row is spread over a cluster of up to 8 CTAs, a warp holding 256 16-byte vectors (4 KB) of it in registers: its terms
// are summed, the sums of all warps meet through distributed shared memory, and the gradient is formed from the same
// registers: one read and one write of the row.  Rows that are longer than the cluster's registers are walked in chunks and
// read a second time.  A listed token belongs to the CTA that has its logit, which adds its part to the sums and corrects
// its gradient.
#include <algorithm>

#include "rows.cuh"

namespace {

using namespace rw;

constexpr int PER_SM = 4;

// What a warp adds to the row's sums.
struct Record {
    double e, f, g;                                 // of its listed tokens: sum e, sum e L (see below), sum e (z - z_ref)
    float s_out, s_in, m;                           // terms outside and inside the list, against m
    float z_ref;
    int flags;                                      // 1: a token that is none, or listed twice; 2: the list has an entry
};

struct DistillShared {
    uint4 chunk[NW][CHUNK];
    Record record[NW];
    float wmax[NW];
    // of the row, once the records have met
    float m, scale;
    double mass, s, e;
    int zero;
};

__device__ __forceinline__ uint32_t store_pair(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t store_pair(float a, float b, __half) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void store_one(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_one(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store_one(__half* p, float v) { *p = __float2half_rn(v); }

// Elements [j*N - shift, ... + N) of the gradient row; one 16-byte store where they lie inside the row and `wide` says
// that the gradient row has the alignment of the logit row.
template <typename T>
__device__ __forceinline__ void store_vec(T* row, int shift, int V, int j, bool wide, const float (&g)[Row<T>::N]) {
    constexpr int N = Row<T>::N;
    const int e0 = j * N - shift;
    if (wide && e0 >= 0 && e0 + N <= V) {
        uint4 w;
        if constexpr (N == 4) w = make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
        else w = make_uint4(store_pair(g[0], g[1], T()), store_pair(g[2], g[3], T()), store_pair(g[4], g[5], T()), store_pair(g[6], g[7], T()));
        *reinterpret_cast<uint4*>(row + e0) = w;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e0 + e >= 0 && e0 + e < V) store_one(row + e0 + e, g[e]);
    }
}

// Bits of the bitmap that belong to vector j of the slice.
template <typename T>
__device__ __forceinline__ unsigned listed_bits(const uint32_t* bitmap, int j) {
    const int bit = j * Row<T>::N;
    return (bitmap[bit >> 5] >> (bit & 31)) & ((1u << Row<T>::N) - 1u);
}

// The same for logits so large that only those equal to the largest count; from memory, rarely.
template <typename T>
__device__ __noinline__ void huge_terms(const Slice<T>& S, const uint32_t* bitmap, int j0, float top, int lane, float& s_out, float& s_in) {
#pragma unroll 1
    for (int i = 0; i < S.depth; ++i)
        for (int e = 0; e < Row<T>::N; ++e) {
            const int j = j0 + i * 32 + lane, v = j * Row<T>::N - S.shift + e;
            if (j >= S.v1 || v < 0 || v >= S.V) continue;
            const float t = top == INFINITY ? NAN : huge_term(Row<T>::wide(S.row[v]), top);
            if (listed_bits<T>(bitmap, j - S.v0) >> e & 1u) s_in += t; else s_out += t;
        }
}

template <typename T, DistillMode MODE>
__global__ void __launch_bounds__(NT, PER_SM) distill_kernel(const __grid_constant__ DistillParams P) {
    constexpr int N = Row<T>::N;
    constexpr bool STATS = MODE != DistillMode::Gradient, GRAD = MODE != DistillMode::Loss;
    extern __shared__ __align__(16) unsigned char raw[];
    DistillShared& sh = *reinterpret_cast<DistillShared*>(raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, k = P.k, C = P.cluster;
    // one entry per listed token of this CTA, at the token's place in the list; an entry is its thread's alone
    double* prob = reinterpret_cast<double*>(raw + sizeof(DistillShared));       // [k] e, then p
    int* ids = reinterpret_cast<int*>(prob + k);                                 // [k] -1: not of this CTA
    float* zs = reinterpret_cast<float*>(ids + k);                               // [k]
    uint32_t* bitmap = reinterpret_cast<uint32_t*>(zs + k);                      // [slice_words] listed tokens of this CTA
    const int row_id = blockIdx.x / C;
    const uint32_t rank = blockIdx.x - row_id * C;
    const Slice<T> S(static_cast<const T*>(P.z) + row_id * P.z_stride, P.V, C, rank);
    const int own_steps = S.chunks_of(warp), stride = 32 * S.depth, j_first = S.start(S.first_chunk(warp));
    const float weight = GRAD ? P.weight[row_id] : 1.f;

    bool zero = GRAD && weight == 0.f;              // the row takes no part
    float m = 0.f;
    double s = 1.0, mass = 0.0;
    float scale = 0.f;                              // of q's term, outside the list
    if (MODE == DistillMode::Gradient) {
        const float4 sv = *reinterpret_cast<const float4*>(P.saved + (size_t)row_id * 4);
        m = sv.x;
        s = sv.y;
        mass = sv.w;
        zero |= sv.w < 0.f;
        scale = (float)((double)weight / P.T * (double)sv.z / s);
    }
    if (!zero && own_steps > 0) S.fetch(j_first, lane, sh.chunk[warp]);        // on its way while the list is read

    // ---- the list: e = exp(L), L = v/T - lse, or (v - the largest v)/T to be divided by the sum
    double e_sum = 0.0, f_sum = 0.0;
    int flags = 0;
    if (!zero) {
        if (STATS)
            for (int i = tid; i < P.slice_words; i += NT) bitmap[i] = 0;
        double norm;
        if (P.lse) {
            norm = (double)P.lse[row_id];
            if (STATS) __syncthreads();             // the bitmap is empty
        } else {
            float v_max = -INFINITY;
            for (int i = tid; i < k; i += NT)
                if ((unsigned)P.tokens[(size_t)row_id * k + i] < (unsigned)P.V) v_max = fmaxf(v_max, P.values[(size_t)row_id * k + i]);
            v_max = warp_max(v_max);
            if (lane == 0) sh.wmax[warp] = v_max;
            __syncthreads();
            for (int w = 0; w < NW; ++w) v_max = fmaxf(v_max, sh.wmax[w]);
            norm = (double)v_max / P.T;
        }
        for (int i = tid; i < k; i += NT) {
            const int id = P.tokens[(size_t)row_id * k + i];
            const bool in = id >= 0 && id < P.V;
            const int at = (id + S.shift) / N;      // its vector
            const bool own = in && at >= S.v0 && at < S.v1;
            flags |= (in ? 2 : 0) | (id >= P.V || id < -1 ? 1 : 0);
            ids[i] = own ? id : -1;
            // a renormalised gradient needs the whole list's sum, and has no other CTA to ask
            if (!own && !(MODE == DistillMode::Gradient && !P.lse && in)) continue;
            const float v = P.values[(size_t)row_id * k + i];
            const double L = (double)v / P.T - norm, e = v == -INFINITY ? 0.0 : exp(L);
            e_sum += e;
            if (e != 0.0) f_sum += e * L;           // not 0 * -inf
            if (!own) continue;
            prob[i] = e;
            if (STATS) {
                const int bit = id + S.shift - S.v0 * N;
                flags |= (atomicOr(&bitmap[bit >> 5], 1u << (bit & 31)) >> (bit & 31)) & 1u;       // listed twice
            }
        }
    }
    uint4 r[NV];
    chunk_wait();
    __syncthreads();                                // the bitmap is complete, and every warp's chunk is there
#pragma unroll
    for (int i = 0; i < NV; ++i) r[i] = sh.chunk[warp][i * 32 + lane];
    if (!zero)
        for (int i = tid; i < k; i += NT)
            if (const int id = ids[i]; id >= 0) {
                const int e = id + S.shift - S.v0 * N;
                zs[i] = Row<T>::wide(S.steps() == 1 ? reinterpret_cast<const T*>(sh.chunk)[e / (stride * N) * (CHUNK * N) + e % (stride * N)] : S.row[id]);
            }

    if (MODE == DistillMode::Gradient && S.steps() > 1) __syncthreads();       // the gradient may lie on the logits
    if (STATS && !zero) {
        // ---- the draft's terms
        float s_out = 0.f, s_in = 0.f, top = -INFINITY;
        int j0 = j_first;
        for (int step = 0; step < own_steps; ++step, j0 += stride) {
            if (step > 0) {
                S.fetch(j0, lane, sh.chunk[warp]);
                chunk_wait();
#pragma unroll
                for (int i = 0; i < NV; ++i) r[i] = sh.chunk[warp][i * 32 + lane];
            }
            Max<T> mx{r[0]};
#pragma unroll
            for (int i = 1; i < NV; ++i) mx = Max<T>{mx, Max<T>{r[i]}};
            const float own = mx.value(), wm = warp_max(own == own ? own : -INFINITY);    // NaN is met in the sums
            if (wm > top) {
                const float f = move_terms(top, wm, P.c);            // the sums are 0 so far where top is -inf
                s_out *= f;
                s_in *= f;
                top = wm;
            }
            if (ordinary(top) || top == -INFINITY) {
                const float u = reference(top) * P.c;
                const f2 neg = sd::pack2(-u, -u), c2 = sd::pack2(P.c, P.c);
                f2 acc = sd::pack2(0.f, 0.f);
                float in = 0.f;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    f2 x[N / 2];
                    pairs(r[i], x, T());
                    const unsigned bits = i < S.depth ? listed_bits<T>(bitmap, min(j0 + i * 32 + lane, S.v1 - 1) - S.v0) : 0u;
                    if (bits == 0u) {
                        acc = sd::add2(acc, terms<N / 2>(x, c2, neg));
                    } else {
#pragma unroll
                        for (int q = 0; q < N / 2; ++q) {
                            float a, b;
                            sd::unpack2(term2(x[q], c2, neg), a, b);
                            const bool la = bits >> (2 * q) & 1u, lb = bits >> (2 * q + 1) & 1u;
                            in += (la ? a : 0.f) + (lb ? b : 0.f);
                            acc = sd::add2(acc, sd::pack2(la ? 0.f : a, lb ? 0.f : b));
                        }
                    }
                }
                s_out += fold2(acc);
                s_in += in;
            } else {
                huge_terms(S, bitmap, j0, top, lane, s_out, s_in);
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s_out += __shfl_xor_sync(0xffffffffu, s_out, o);
            s_in += __shfl_xor_sync(0xffffffffu, s_in, o);
        }
        // ---- this warp's record.  Differences of logits are formed first, whatever the logits' size
        double g_sum = 0.0;
        float z_ref = -INFINITY;
        if (warp * 32 < k) {
            for (int i = tid; i < k; i += NT)
                if (ids[i] >= 0 && prob[i] != 0.0) z_ref = fmaxf(z_ref, zs[i]);
            z_ref = reference(warp_max(z_ref));
            for (int i = tid; i < k; i += NT)
                if (ids[i] >= 0 && prob[i] != 0.0) g_sum += prob[i] * ((double)zs[i] - (double)z_ref);
            e_sum = warp_sum(e_sum);
            f_sum = warp_sum(f_sum);
            g_sum = warp_sum(g_sum);
            flags = __reduce_or_sync(0xffffffffu, flags);
        }
        if (lane == 0) sh.record[warp] = Record{e_sum, f_sum, g_sum, s_out, s_in, top, z_ref, flags};
        if (C > 1) sd::cl_sync(); else __syncthreads();
        double plogp = 0.0, pz = 0.0, S_out = 0.0, R = 0.0;
        if (warp == 0) {
            // ---- the row's sums, by every CTA for itself; two records a lane
            Record rec[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int q = h * 32 + lane;
                rec[h] = Record{0.0, 0.0, 0.0, 0.f, 0.f, -INFINITY, 0.f, 0};
                if (q < C * NW) {
                    const Record* from = &sh.record[q % NW];
                    const uint32_t at = q / NW;
                    rec[h].s_out = cl_ld_f32(&from->s_out, at);
                    rec[h].s_in = cl_ld_f32(&from->s_in, at);
                    rec[h].m = cl_ld_f32(&from->m, at);
                    if (q % NW * 32 < k) {
                        rec[h].e = cl_ld_f64(&from->e, at);
                        rec[h].f = cl_ld_f64(&from->f, at);
                        rec[h].g = cl_ld_f64(&from->g, at);
                        rec[h].z_ref = cl_ld_f32(&from->z_ref, at);
                        rec[h].flags = cl_ld_s32(&from->flags, at);
                    }
                }
            }
            const float all = warp_max(fmaxf(rec[0].m, rec[1].m));
            m = reference(all);
            double out = 0.0, in = 0.0, e = 0.0, f = 0.0, g = 0.0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float to = move_terms(rec[h].m, all, P.c);
                out += (double)(rec[h].s_out * to);
                in += (double)(rec[h].s_in * to);
                e += rec[h].e;
                f += rec[h].f;
                g += rec[h].g + (rec[h].e != 0.0 ? rec[h].e * ((double)rec[h].z_ref - (double)m) : 0.0);
            }
            const double exact = unround(m, P.c);
            S_out = warp_sum(out) * exact;
            s = S_out + warp_sum(in) * exact;
            e = warp_sum(e);
            plogp = warp_sum(f);
            pz = warp_sum(g);
            flags = __reduce_or_sync(0xffffffffu, rec[0].flags | rec[1].flags);
            if (!P.lse) {                           // p = e / sum e
                plogp = e > 0.0 ? plogp / e - log(e) : e;
                pz = e > 0.0 ? pz / e : e;
            }
            const double p = P.lse ? e : e > 0.0 ? 1.0 : e;         // sum p; NaN stays NaN
            R = P.lse && S_out > 0.0 ? fmax(0.0, 1.0 - p) : 0.0;     // a draft with nothing outside the list has no rest
            mass = p + R;
            const double out_factor = mass - (R > 0.0 ? R * s / S_out : 0.0);
            zero = flags != 2 || s == 0.0;          // a bad list, an empty one, or no logit above -inf
            if (lane == 0) {
                sh.m = m;
                sh.s = s;
                sh.mass = mass;
                sh.e = P.lse || e == 0.0 ? 1.0 : e;         // what e is divided by; a list without mass stays one
                sh.scale = (float)((double)weight / P.T * out_factor / (s / exact));       // of a term against the rounded m*c
                sh.zero = zero;
                if (rank == 0) {
                    float loss;
                    if (flags & 1) loss = NAN;
                    else if (flags == 0) loss = 0.f;
                    else if (s == 0.0) loss = p > 0.0 ? INFINITY : 0.f;
                    else {
                        double l = plogp;
                        if (p > 0.0) l += p * log(s) - pz / P.T;
                        if (R > 0.0) l += R * (log(R) - log(S_out / s));
                        loss = s == s ? (float)l : NAN;
                    }
                    P.loss[row_id] = loss;
                    if (flags & 1) atomicOr(P.status, SPECDEC_DATA_BAD_TOKEN);
                    if (MODE == DistillMode::Loss)
                        *reinterpret_cast<float4*>(P.saved + (size_t)row_id * 4) = make_float4(m, (float)(s / exact), (float)out_factor, zero ? -1.f : (float)mass);
                }
            }
        }
        if (C > 1) sd::cl_sync(); else __syncthreads();      // nobody leaves, or writes over logits, while others still read
        if (!GRAD) return;
        m = sh.m;
        s = sh.s;
        mass = sh.mass;
        scale = sh.scale;
        zero = sh.zero;
        e_sum = sh.e;
    } else if (STATS && rank == 0 && tid == 0) {    // a step of weight 0
        P.loss[row_id] = 0.f;
    }
    if constexpr (GRAD) {
        const float u = m * P.c;
        if (MODE == DistillMode::Gradient && !zero) {
            s *= unround(m, P.c);                   // against m itself
            if (!P.lse) {                           // the list's sum
                e_sum = warp_sum(e_sum);
                if (lane == 0) sh.record[warp].e = e_sum;
                __syncthreads();
                e_sum = 0.0;
                for (int w = 0; w < NW; ++w) e_sum += sh.record[w].e;
                if (e_sum == 0.0) e_sum = 1.0;
            } else {
                e_sum = 1.0;
            }
        }
        // ---- the gradient, from the chunk that the registers hold: the last one, or the first
        T* grad = static_cast<T*>(P.grad) + row_id * P.g_stride;
        const bool wide = row_shift(grad) == S.shift;
        const f2 c2 = sd::pack2(P.c, P.c), neg = sd::pack2(-u, -u), scale2 = sd::pack2(scale, scale);
        const bool normal = ordinary(m);
        for (int n = 0; n < own_steps; ++n) {
            const int j0 = j_first + (STATS ? own_steps - 1 - n : n) * stride;
            if (!zero && n > 0) {
                S.fetch(j0, lane, sh.chunk[warp]);
                chunk_wait();
#pragma unroll
                for (int i = 0; i < NV; ++i) r[i] = sh.chunk[warp][i * 32 + lane];
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int j = j0 + i * 32 + lane;
                if (i >= S.depth || j >= S.v1) continue;
                float g[N];
                f2 x[N / 2];
                pairs(r[i], x, T());
#pragma unroll
                for (int q = 0; q < N / 2; ++q) sd::unpack2(sd::mul2(term2(x[q], c2, neg), scale2), g[2 * q], g[2 * q + 1]);
                if (!normal || zero) {
                    widen<T>(r[i], g);
#pragma unroll
                    for (int e = 0; e < N; ++e) g[e] = zero ? 0.f : huge_term(g[e], m) * scale;
                }
                store_vec<T>(grad, S.shift, S.V, j, wide, g);
            }
        }
        if (zero) return;
        __syncthreads();                            // the CTA's part is written: the listed tokens are written over
        const double wt = (double)weight / P.T;
        for (int i = tid; i < k; i += NT)
            if (const int id = ids[i]; id >= 0) {
                const double q = exp(((double)zs[i] - (double)m) / P.T) / s;
                store_one(grad + id, (float)(wt * (mass * q - prob[i] / e_sum)));
            }
    }
}

template <typename T>
cudaError_t launch_as(const DistillParams& p, DistillMode mode, int rows, size_t smem, cudaStream_t s) {
    switch (mode) {
        case DistillMode::Loss: return rw::launch(distill_kernel<T, DistillMode::Loss>, p, rows, p.cluster, smem, s);
        case DistillMode::Gradient: return rw::launch(distill_kernel<T, DistillMode::Gradient>, p, rows, p.cluster, smem, s);
        default: return rw::launch(distill_kernel<T, DistillMode::Step>, p, rows, p.cluster, smem, s);
    }
}

}  // namespace

cudaError_t launch_distill(DistillParams p, specdec_dtype dtype, DistillMode mode, int rows, int sm_count, cudaStream_t s) {
    const int n = dtype == SPECDEC_F32 ? 4 : 8;
    const int most = (p.V + 2 * n - 2) / n;        // vectors of a row at its worst alignment
    const int hold = NW * CHUNK;                   // vectors that a CTA's registers hold
    p.cluster = rw::cluster_size(rows, most, sm_count, std::min(MAX_CLUSTER, (most + hold - 1) / hold));
    p.slice_words = ((most + p.cluster - 1) / p.cluster * n + 31) / 32;
    const size_t smem = sizeof(DistillShared) + (size_t)p.slice_words * 4 + (size_t)p.k * 16;
    if (dtype == SPECDEC_F32) return launch_as<float>(p, mode, rows, smem, s);
    if (dtype == SPECDEC_BF16) return launch_as<__nv_bfloat16>(p, mode, rows, smem, s);
    return launch_as<__half>(p, mode, rows, smem, s);
}
