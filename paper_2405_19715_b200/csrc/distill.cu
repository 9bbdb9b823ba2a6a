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
// A CTA holds up to 4096 16-byte vectors of the row in registers, a cluster of up to 8 CTAs a row; sums meet through
// distributed shared memory.  The step then forms the gradient from the registers: one read and one write of the row.
// Longer rows are walked in tiles and read a second time.
#include "rows.cuh"

namespace {

using namespace rw;

struct DistillShared {
    double wsum[WARPS], wsum2[WARPS];
    float wmax[WARPS];
    double s_out, s_in;                             // this CTA's sums outside and inside the list, against m
    float m;
    int bad;
};

// Sum over the CTA of one double per thread, the same in every thread.  Two barriers: `slot` may be reused at once.
__device__ __forceinline__ double block_sum(double v, double (&slot)[WARPS], int lane, int warp) {
    v = warp_sum(v);
    if (lane == 0) slot[warp] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += slot[w];
    __syncthreads();
    return s;
}
__device__ __forceinline__ float block_max(float v, float (&slot)[WARPS], int lane, int warp) {
    v = warp_max(v);
    if (lane == 0) slot[warp] = v;
    __syncthreads();
    float m = slot[0];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) m = fmaxf(m, slot[w]);
    __syncthreads();
    return m;
}

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

template <typename T, DistillMode MODE>
__global__ void __launch_bounds__(THREADS, 2) distill_kernel(const __grid_constant__ DistillParams P) {
    constexpr int N = Row<T>::N;
    constexpr bool STATS = MODE != DistillMode::Gradient, GRAD = MODE != DistillMode::Loss;
    __shared__ DistillShared sh;
    extern __shared__ double dyn[];
    double* prob = dyn;                             // [k] p; entry i is its thread's alone, here and below
    int* ids = reinterpret_cast<int*>(prob + P.k);
    float* zs = reinterpret_cast<float*>(ids + P.k);            // the draft's logits of the listed tokens that this CTA needs
    uint32_t* bitmap = reinterpret_cast<uint32_t*>(zs + P.k);   // [slice_words] tokens of the list in this CTA's part of the row
    const int C = P.cluster, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row_id = blockIdx.x / C;
    const uint32_t rank = blockIdx.x - row_id * C;
    const T* row = static_cast<const T*>(P.z) + row_id * P.z_stride;
    const int V = P.V, k = P.k, shift = row_shift(row), nvec = row_vectors<T>(shift, V);
    const int per = (nvec + C - 1) / C, v0 = min(nvec, (int)rank * per), v1 = min(nvec, v0 + per);
    T* grad = GRAD ? static_cast<T*>(P.grad) + row_id * P.g_stride : nullptr;
    const bool wide = GRAD && row_shift(grad) == shift;
    const float weight = GRAD ? P.weight[row_id] : 1.f;

    bool zero = GRAD && weight == 0.f;              // the row takes no part
    float saved_m = 0.f, saved_s = 1.f, saved_out = 0.f, saved_mass = 0.f;
    if (MODE == DistillMode::Gradient) {
        const float* sv = P.saved + (size_t)row_id * 4;
        saved_m = sv[0];
        saved_s = sv[1];
        saved_out = sv[2];
        saved_mass = sv[3];
        zero |= saved_mass < 0.f;
    }
    uint4 r[NV];
    if (!zero) load_tile<T>(row, shift, V, v0, v1, tid, r);     // on its way while the list is read

    // ---- the list
    bool any = false;
    int bad = 0;
    double mass_p = 0.0, plogp = 0.0;               // sum p, sum p log p
    if (!zero) {
        if (STATS)
            for (int i = tid; i < P.slice_words; i += THREADS) bitmap[i] = 0;
        float vmax = -INFINITY;
        for (int i = tid; i < k; i += THREADS) {
            const int id = P.tokens[(size_t)row_id * k + i];
            const bool in = id >= 0 && id < V;
            bad |= id >= V || id < -1;
            any |= in;
            ids[i] = in ? id : -1;
            if (in) vmax = fmaxf(vmax, P.values[(size_t)row_id * k + i]);
        }
        any = __syncthreads_or(any);                // the bitmap is empty, too
        double norm;
        if (P.lse) {
            norm = (double)P.lse[row_id];
        } else {
            const float top = block_max(vmax, sh.wmax, lane, warp);
            double e = 0.0;
            for (int i = tid; i < k; i += THREADS) {
                const float v = P.values[(size_t)row_id * k + i];
                if (ids[i] >= 0 && v != -INFINITY) e += exp(((double)v - (double)top) / P.T);
            }
            norm = (double)top / P.T + log(block_sum(e, sh.wsum, lane, warp));
        }
        for (int i = tid; i < k; i += THREADS) {
            const int id = ids[i];
            if (id < 0) continue;
            const int at = (id + shift) / N;
            const bool own = at >= v0 && at < v1;
            if (STATS && own) {
                const int bit = id + shift - v0 * N;
                bad |= (atomicOr(&bitmap[bit >> 5], 1u << (bit & 31)) >> (bit & 31)) & 1u;   // a token listed twice
            }
            const float v = P.values[(size_t)row_id * k + i];
            const double log_p = (double)v / P.T - norm, p = v == -INFINITY ? 0.0 : exp(log_p);
            prob[i] = p;
            if (own || (STATS && rank == 0)) zs[i] = Row<T>::wide(row[id]);
            if (p != 0.0) {
                mass_p += p;
                plogp += p * log_p;
            }
        }
    }

    // ---- the draft's sums
    double S = 1.0, f_out = 0.0, mass = 0.0;
    float M = 0.f;
    if (STATS && !zero) {
        const f2 hi2 = sd::pack2(P.c.hi, P.c.hi), lo2 = sd::pack2(P.c.lo, P.c.lo);
        double s_out = 0.0, s_in = 0.0;             // of this thread, against run_m
        float run_m = -INFINITY;
        for (int t0 = v0; t0 < v1; t0 += TILE) {
            if (t0 != v0) load_tile<T>(row, shift, V, t0, v1, tid, r);
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < NV; ++i) m = fmaxf(m, vec_max(r[i], T()));        // NaN is skipped here, and met in the sum
            const float tm = block_max(m, sh.wmax, lane, warp);                   // the bitmap is complete, too
            const float ref = reference(tm);
            const f2 neg = sd::pack2(-ref, -ref);
            f2 acc = sd::pack2(0.f, 0.f);
            float in = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                f2 x[N / 2];
                pairs(r[i], x, T());
                const int j = t0 + i * THREADS + tid;
                const unsigned bits = j < v1 ? listed_bits<T>(bitmap, j - v0) : 0u;
                if (bits == 0u) {
                    acc = sd::add2(acc, terms<N / 2>(x, neg, hi2, lo2));
                } else {
                    float out = 0.f;
#pragma unroll
                    for (int q = 0; q < N / 2; ++q) {
                        float a, b;
                        sd::unpack2(term2(x[q], neg, hi2, lo2), a, b);
                        if (bits >> (2 * q) & 1u) in += a; else out += a;
                        if (bits >> (2 * q + 1) & 1u) in += b; else out += b;
                    }
                    acc = sd::add2(acc, sd::pack2(out, 0.f));
                }
            }
            const float to = fmaxf(run_m, tm);
            const double f0 = rescale(run_m, to, P.log2e_t), f1 = rescale(tm, to, P.log2e_t);
            s_out = s_out * f0 + (double)fold2(acc) * f1;
            s_in = s_in * f0 + (double)in * f1;
            run_m = to;
        }
        s_out = block_sum(s_out, sh.wsum, lane, warp);
        s_in = block_sum(s_in, sh.wsum, lane, warp);
        bad = __syncthreads_or(bad);
        M = run_m;
        if (C > 1) {
            if (tid == 0) {
                sh.s_out = s_out;
                sh.s_in = s_in;
                sh.m = run_m;
                sh.bad = bad;
            }
            sd::cl_sync();
            for (int q = 0; q < C; ++q) M = fmaxf(M, cl_ld_f32(&sh.m, q));
            s_out = s_in = 0.0;
            for (int q = 0; q < C; ++q) {
                const double f = rescale(cl_ld_f32(&sh.m, q), M, P.log2e_t);
                s_out += cl_ld_f64(&sh.s_out, q) * f;
                s_in += cl_ld_f64(&sh.s_in, q) * f;
                bad |= cl_ld_s32(&sh.bad, q);
            }
            sd::cl_sync();                          // nobody leaves, or overwrites logits, while others may still read
        }
        S = s_out + s_in;
        mass_p = block_sum(mass_p, sh.wsum, lane, warp);
        const double R0 = P.lse ? fmax(0.0, 1.0 - mass_p) : 0.0;
        const double R = s_out > 0.0 ? R0 : 0.0;    // a draft with nothing outside the list has no such outcome
        mass = mass_p + R;
        const double share = R > 0.0 ? R * S / s_out : 0.0;
        f_out = mass - share;
        const bool empty = S == 0.0;                // no logit above -inf
        if (rank == 0) {
            double pz = 0.0;                        // sum p (z - m): differences first, whatever the logits' size
            for (int i = tid; i < k; i += THREADS)
                if (ids[i] >= 0 && prob[i] != 0.0) pz += prob[i] * ((double)zs[i] - (double)reference(M));
            plogp = block_sum(plogp, sh.wsum, lane, warp);
            pz = block_sum(pz, sh.wsum, lane, warp);
            if (tid == 0) {
                float loss;
                if (bad) loss = NAN;
                else if (!any) loss = 0.f;
                else if (empty) loss = mass_p > 0.0 ? INFINITY : 0.f;
                else {
                    double l = plogp;
                    if (mass_p > 0.0) l += mass_p * log(S) - pz / P.T;
                    if (R > 0.0) l += R * (log(R) - log(s_out / S));
                    loss = (float)(S != S ? (double)NAN : l);
                }
                P.loss[row_id] = loss;
                if (bad) atomicOr(P.status, SPECDEC_DATA_BAD_TOKEN);
                if (MODE == DistillMode::Loss) {
                    float* sv = P.saved + (size_t)row_id * 4;
                    sv[0] = reference(M);
                    sv[1] = (float)S;
                    sv[2] = (float)f_out;
                    sv[3] = !any || bad || empty ? -1.f : (float)mass;
                }
            }
        }
        M = reference(M);
        zero = !any || bad || empty;
    } else if (MODE == DistillMode::Gradient) {
        M = saved_m;
        S = saved_s;
        f_out = saved_out;
        mass = saved_mass;
        __syncthreads();                            // the listed logits are in shared memory: the gradient may lie on the logits
    } else if (STATS && rank == 0 && tid == 0) {    // Step with weight 0
        P.loss[row_id] = 0.f;
    }
    if constexpr (!GRAD) return;

    // ---- the gradient
    const double wt = (double)weight / P.T;
    const float scale = zero ? 0.f : (float)(wt * f_out / S);
    const f2 hi2 = sd::pack2(P.c.hi, P.c.hi), lo2 = sd::pack2(P.c.lo, P.c.lo), neg = sd::pack2(-M, -M), scale2 = sd::pack2(scale, scale);
    const int tiles = (v1 - v0 + TILE - 1) / TILE;
    for (int n = 0; n < tiles; ++n) {               // from the tile that the registers hold: the last one, or the first
        const int t0 = v0 + (STATS ? tiles - 1 - n : n) * TILE;
        if (!zero && n > 0) load_tile<T>(row, shift, V, t0, v1, tid, r);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = t0 + i * THREADS + tid;
            if (j >= v1) continue;
            float g[N];
            if (zero) {
#pragma unroll
                for (int e = 0; e < N; ++e) g[e] = 0.f;
            } else {
                f2 x[N / 2];
                pairs(r[i], x, T());
#pragma unroll
                for (int q = 0; q < N / 2; ++q) sd::unpack2(sd::mul2(term2(x[q], neg, hi2, lo2), scale2), g[2 * q], g[2 * q + 1]);
            }
            store_vec<T>(grad, shift, V, j, wide, g);
        }
    }
    if (zero) return;
    __syncthreads();                                // the CTA's part is written: the listed tokens are written over
    for (int i = tid; i < k; i += THREADS) {
        const int id = ids[i];
        const int at = (id + shift) / N;
        if (id < 0 || at < v0 || at >= v1) continue;
        const double q = exp(((double)zs[i] - (double)M) / P.T) / S;
        store_one(grad + id, (float)(wt * (mass * q - prob[i])));
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
    p.cluster = rw::cluster_size(rows, (p.V + n - 1) / n, sm_count);
    p.slice_words = ((most + p.cluster - 1) / p.cluster * n + 31) / 32;
    const size_t smem = (size_t)p.slice_words * 4 + (size_t)p.k * 16;
    if (dtype == SPECDEC_F32) return launch_as<float>(p, mode, rows, smem, s);
    if (dtype == SPECDEC_BF16) return launch_as<__nv_bfloat16>(p, mode, rows, smem, s);
    return launch_as<__half>(p, mode, rows, smem, s);
}
