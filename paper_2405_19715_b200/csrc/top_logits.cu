// The k largest logits of a row in order, and the row's log-sum-exp: what a draft model's training keeps of a target
// row, and what beam selection starts from.
//
// The row passes through registers once.  A CTA holds a tile of 4096 16-byte vectors (8 per thread); rows of more
// are spread over a thread-block cluster, longer ones still walked tile by tile.  Per tile:
//   1. thread maxima; per warp the r-th largest of them, r = ceil(k / 16): the least of these over the 16 warps is a
//      lower bound on the tile's k-th largest (k threads hold an element at or above it), and a close one because
//      few of the k largest share a thread;
//   2. the softmax terms are summed against the tile's maximum, and the elements at or above the bound, k and some
//      tens, go into a buffer in shared memory;
//   3. each of them finds its rank by counting the larger ones.  Keys carry the token, so no two are equal, ranks
//      are unique and the result does not depend on the order of arrival.
// Where the bound lets too many through (masked rows, ties, values that grow along the row), the k-th largest value
// is found by counting over the registers, and ties with it are taken in token order.
// The CTAs of a cluster then read one another's lists and each places its own entries.
#include "rows.cuh"

namespace {

using namespace rw;

constexpr int CAP = 2048;                  // candidates in shared memory: MAX_CLUSTER lists of MAX_TOP entries, too
constexpr int MAX_TOP = SPECDEC_TOP_LOGITS_MAX;
static_assert(CAP >= MAX_CLUSTER * MAX_TOP && MAX_TOP <= THREADS, "the lists of a cluster fit the buffer");

struct TopShared {
    unsigned long long buf[CAP];
    unsigned long long list[2][MAX_TOP];
    double wsum[WARPS];
    float wmax[WARPS], wrth[WARPS];
    int wcount[2][WARPS];
    int count, n_list;
    Part part;
};

// r-th largest of the lane values; -inf when fewer than r are above -inf.
__device__ __forceinline__ float warp_rth_largest(float v, int r, int lane) {
    float cur = -INFINITY;
    for (int it = 0; it < r; ++it) {
        cur = warp_max(v);
        if (cur == -INFINITY) break;
        const unsigned who = __ballot_sync(0xffffffffu, v == cur);
        if (lane == __ffs(who) - 1) v = -INFINITY;
    }
    return cur;
}

// Sum of one int per thread over the CTA; `buf` alternates between two sets so that one barrier is enough.
__device__ __forceinline__ int block_count(int v, int (&slot)[WARPS], int lane, int warp) {
    v = __reduce_add_sync(0xffffffffu, v);
    if (lane == 0) slot[warp] = v;
    __syncthreads();
    int n = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) n += slot[w];
    return n;
}

template <typename T, typename F>
__device__ __forceinline__ int count_if(const uint4 (&r)[NV], F f) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float x[Row<T>::N];
        widen<T>(r[i], x);
#pragma unroll
        for (int e = 0; e < Row<T>::N; ++e) n += f(x[e]) ? 1 : 0;
    }
    return n;
}

// The `need` largest of the tile (it has that many elements), appended to the buffer.  By counting: the value of the
// need-th largest is built from its key's leading bits, elements above it are all taken, those equal to it in token
// order.  Called by the whole CTA, rarely.
template <typename T>
__device__ __noinline__ void exact_select(const uint4 (&r)[NV], int shift, int V, int t0, int v1, int need, TopShared& sh, int tid) {
    constexpr int N = Row<T>::N;
    const int lane = tid & 31, warp = tid >> 5;
    int turn = 0;
    // level: lo <= x < hi are the elements equal to the need-th largest, hi <= x those above it; `nans`: the level
    // is NaN, which ranks below everything
    float lo = -INFINITY, hi = -3.402823466e38f;
    bool nans = false;
    int above = block_count(count_if<T>(r, [&](float x) { return x >= hi; }), sh.wcount[turn ^= 1], lane, warp);
    if (above >= need) {
        uint32_t prefix = 0;
        for (int bit = 31; bit >= 32 - Row<T>::KEY_BITS; --bit) {
            const uint32_t trial = prefix | (1u << bit);
            const float f = key_value(trial);        // a NaN where the trial lies beyond +inf: nothing is counted
            if (block_count(count_if<T>(r, [&](float x) { return x >= f; }), sh.wcount[turn ^= 1], lane, warp) >= need) prefix = trial;
        }
        lo = key_value(prefix);
        hi = key_value(prefix + (1u << (32 - Row<T>::KEY_BITS)));
        above = block_count(count_if<T>(r, [&](float x) { return x >= hi; }), sh.wcount[turn ^= 1], lane, warp);
    } else {
        // fewer than `need` above -inf: the elements past the row's ends, held as -inf, must not count
        int real = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = t0 + i * THREADS + tid;
            float x[N];
            widen<T>(r[i], x);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int v = j * N - shift + e;
                real += (x[e] == -INFINITY && j < v1 && v >= 0 && v < V) ? 1 : 0;
            }
        }
        const int with_inf = above + block_count(real, sh.wcount[turn ^= 1], lane, warp);
        if (with_inf < need) {
            nans = true;
            above = with_inf;
        }
    }
    int taken = above;                               // ties still wanted: need - taken
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = t0 + i * THREADS + tid;
        float x[N];
        widen<T>(r[i], x);
        unsigned ties = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int v = j * N - shift + e;
            const bool real = j < v1 && v >= 0 && v < V;
            const bool gt = nans ? x[e] == x[e] : x[e] >= hi;
            const bool eq = nans ? x[e] != x[e] : x[e] >= lo && !(x[e] >= hi);
            if (real && gt) sh.buf[atomicAdd(&sh.count, 1)] = full_key(x[e], v);
            if (real && eq) ties |= 1u << e;
        }
        // ties of vectors before this thread's: tokens grow with i, then with the thread, then with e
        const int mine = __popc(ties);
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        int* slot = sh.wcount[turn ^= 1];
        if (lane == 31) slot[warp] = incl;
        __syncthreads();
        int before = incl - mine, all = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            if (w < warp) before += slot[w];
            all += slot[w];
        }
#pragma unroll
        for (int e = 0; e < N; ++e)
            if ((ties >> e) & 1u) {
                if (taken + before < need) sh.buf[atomicAdd(&sh.count, 1)] = full_key(x[e], j * N - shift + e);
                ++before;
            }
        taken = min(need, taken + all);
    }
}

template <typename T>
__global__ void __launch_bounds__(THREADS, 2) top_logits_kernel(const __grid_constant__ TopParams P) {
    constexpr int N = Row<T>::N;
    __shared__ TopShared sh;
    const int C = P.cluster, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row_id = blockIdx.x / C;
    const uint32_t rank = blockIdx.x - row_id * C;
    const int outer = row_id / P.inner, in = row_id - outer * P.inner;
    if (P.scores) {                                 // beam selection: beams that offer nothing of their row
        const float s = P.scores[row_id];
        if (!(s > -INFINITY && s < INFINITY) || (P.finished && P.finished[row_id])) return;      // the whole cluster
    }
    const T* row = static_cast<const T*>(P.x) + outer * P.outer_stride + in * P.row_stride;
    const int V = P.V, k = P.k, shift = row_shift(row), nvec = row_vectors<T>(shift, V);
    const int per = (nvec + C - 1) / C, v0 = min(nvec, (int)rank * per), v1 = min(nvec, v0 + per);
    const f2 hi2 = sd::pack2(P.c.hi, P.c.hi), lo2 = sd::pack2(P.c.lo, P.c.lo);

    Part run{0.0, -INFINITY};                       // the same in every thread
    int n_list = 0, cur = 0;
    for (int t0 = v0; t0 < v1; t0 += TILE) {
        uint4 r[NV];
        load_tile<T>(row, shift, V, t0, v1, tid, r);
        float m = vec_max(r[0], T());
#pragma unroll
        for (int i = 1; i < NV; ++i) m = max_nan(m, vec_max(r[i], T()));
        const float m_num = m == m ? m : -INFINITY;
        const int active = min(WARPS, (v1 - t0 + 31) / 32), rth = (k + active - 1) / active;   // warps that hold a part of the tile
        const float wm = warp_max(m_num), wr = warp_rth_largest(m_num, rth, lane);
        if (lane == 0) { sh.wmax[warp] = wm; sh.wrth[warp] = wr; }
        if (tid < n_list) sh.buf[tid] = sh.list[cur][tid];
        if (tid == 0) sh.count = n_list;
        __syncthreads();
        float bound = sh.wrth[0], tm = sh.wmax[0];
        for (int w = 1; w < active; ++w) { bound = fminf(bound, sh.wrth[w]); tm = fmaxf(tm, sh.wmax[w]); }
        if (n_list == k) {                          // a full list from earlier tiles bounds this one as well
            const uint32_t least = (uint32_t)(sh.list[cur][k - 1] >> 32);
            if (least) bound = fmaxf(bound, key_value(least));
        }
        const float ref = reference(tm);
        f2 acc = sd::pack2(0.f, 0.f);
        const f2 neg = sd::pack2(-ref, -ref);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            f2 x[N / 2];
            pairs(r[i], x, T());
            acc = sd::add2(acc, terms<N / 2>(x, neg, hi2, lo2));
        }
        const double ws = warp_sum((double)fold2(acc));
        if (lane == 0) sh.wsum[warp] = ws;
        if (!(m < bound)) {                         // NaN always passes: its key ranks it last
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (vec_max(r[i], T()) < bound) continue;
                const int j = t0 + i * THREADS + tid;
                float x[N];
                widen<T>(r[i], x);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const int v = j * N - shift + e;
                    if (!(x[e] < bound) && j < v1 && v >= 0 && v < V) {
                        const int pos = atomicAdd(&sh.count, 1);
                        if (pos < CAP) sh.buf[pos] = full_key(x[e], v);
                    }
                }
            }
        }
        __syncthreads();
        int n = sh.count;
        if (n > CAP) {
            const int t1 = min(v1, t0 + TILE);
            const int real = min(V, t1 * N - shift) - max(0, t0 * N - shift);
            __syncthreads();                        // everyone has read the count
            if (tid == 0) sh.count = n_list;
            __syncthreads();
            exact_select<T>(r, shift, V, t0, v1, min(k, real), sh, tid);
            __syncthreads();
            n = sh.count;
        }
        for (int i = tid; i < n; i += THREADS) {
            const unsigned long long key = sh.buf[i];
            int place = 0;
            for (int q = 0; q < n; ++q) place += sh.buf[q] > key;
            if (place < k) sh.list[cur ^ 1][place] = key;
        }
        double s = 0.0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) s += sh.wsum[w];
        const float to = fmaxf(run.m, tm);
        run.s = run.s * rescale(run.m, to, P.log2e_t) + s * rescale(tm, to, P.log2e_t);
        run.m = to;
        n_list = min(k, n);
        cur ^= 1;
        __syncthreads();
    }

    if (C > 1) {
        if (tid == 0) {
            // the other CTAs find the finished list in list[0]
            sh.n_list = n_list;
            sh.part = run;
        }
        if (cur == 1 && tid < n_list) sh.list[0][tid] = sh.list[1][tid];
        sd::cl_sync();
        for (int q = tid; q < C * MAX_TOP; q += THREADS) {
            const uint32_t from = q / MAX_TOP;
            const int i = q - from * MAX_TOP;
            if (from != rank && i < cl_ld_s32(&sh.n_list, from)) sh.buf[q] = cl_ld_u64(&sh.list[0][i], from);
        }
        if (rank == 0 && tid == 0) {
            float to = run.m;
            for (int q = 1; q < C; ++q) to = fmaxf(to, cl_ld_f32(&sh.part.m, q));
            double s = run.s * rescale(run.m, to, P.log2e_t);
            for (int q = 1; q < C; ++q) s += cl_ld_f64(&sh.part.s, q) * rescale(cl_ld_f32(&sh.part.m, q), to, P.log2e_t);
            run.s = s;
            run.m = to;
        }
        if (tid < C) sh.wcount[0][tid] = cl_ld_s32(&sh.n_list, tid);
        sd::cl_sync();                              // nobody leaves while its list may still be read
        cur = 0;
    }
    if (rank == 0 && tid == 0) {
        if (P.lse) P.lse[row_id] = (float)((double)reference(run.m) / P.T + log(run.s));
        if (P.parts) P.parts[row_id] = run;
    }
    if (tid < n_list) {
        const unsigned long long key = sh.list[cur][tid];
        int place = tid;
        for (int q = 0; q < C; ++q) {
            if (q == (int)rank) continue;
            int a = 0, b = sh.wcount[0][q];         // entries of list q above this one: keys fall along it
            while (a < b) {
                const int mid = (a + b) >> 1;
                if (sh.buf[q * MAX_TOP + mid] > key) a = mid + 1; else b = mid;
            }
            place += a;
        }
        if (place < k) {
            const size_t o = (size_t)row_id * k + place;
            const uint32_t vk = (uint32_t)(key >> 32);
            P.values[o] = vk ? key_value(vk) : __int_as_float(0x7fffffff);
            P.tokens[o] = key_token(key);
        }
    }
}

}  // namespace

cudaError_t launch_top_logits(TopParams p, specdec_dtype dtype, int rows, int sm_count, cudaStream_t s) {
    const int n = dtype == SPECDEC_F32 ? 4 : 8;
    p.cluster = rw::cluster_size(rows, (p.V + n - 1) / n, sm_count);
    if (dtype == SPECDEC_F32) return rw::launch(top_logits_kernel<float>, p, rows, p.cluster, 0, s);
    if (dtype == SPECDEC_BF16) return rw::launch(top_logits_kernel<__nv_bfloat16>, p, rows, p.cluster, 0, s);
    return rw::launch(top_logits_kernel<__half>, p, rows, p.cluster, 0, s);
}
