// Rotary positions with several axes (height and width of an image; time, height and width of a video) on queries and keys.
//
// A head's 2R leading elements are R pairs.  Pair p belongs to one axis a and turns by angle pos[t, a] w_p, w_p = theta^(-i / n_a)
// for the i-th of the axis' n_a pairs (or theta^(-p / R)):
//   y_lo = x_lo cos - x_hi sin,  y_hi = x_lo sin + x_hi cos;  backward is the same by the opposite angle.
//
// Bound by HBM: queries and keys are read once and written once, wherever the rows of a packed projection hold them.  A
// workgroup takes a few tokens, forms the tokens' R cosines and sines once, in LDS, and turns all their heads with
// them.  Angles are reduced in 64 bits, as turns, whose whole part falls away exactly: in fp32 position 10^5 would be off by
// 2^-24 10^5 = 6e-3 turns' radians and more.
//
// Measured (three sets of inputs in turn): 12844 tokens of 32 heads x 128 fp32 76.0 us, 5.5 TB/s; 8192 tokens of 40 heads x 64 bf16 in packed rows 18.2 us, 4.6 TB/s.  From cold inputs
// into cold results 77.4 and 22.0, the latter for 84 MB (copies of 63 and 105 MB: 14.0 and 22.3).  Axes that no access but a single element's divides take twice that: 8192 tokens of 40 x 64
// bf16, cold, 16 + 16 pairs in halves 21.2, 13 + 18 40.1, the same as neighbours (accesses of two) 32.3; fp32 34.1 and 46.3.
#include "common.hpp"

#include <math.h>
#include <string.h>

namespace sd {

constexpr int ROPE_AXES = SD_ROPE_MAX_AXES, ROPE_MAX_D = 256, ROPE_THREADS = 256;
constexpr int ROPE_MAX_TOKENS = 32;        // of a workgroup

struct RopeArgs {
    const float* pos;
    int64_t pos_stride, rows;
    const void *q, *k;
    void *yq, *yk;
    int64_t ldq, ldk, ldyq, ldyk;          // elements between tokens
    int32_t T, n_axes, tokens;             // tokens of a workgroup
    int32_t heads_q, heads, D, R;
    int32_t units, rot_units;              // of a head; the first of them turn
    uint32_t by_token, by_head;            // 2^32 / (units of a token), / (units of a head), rounded up (divisors of 1 aside); the first 0 for one token a workgroup
    int32_t axis_halves;
    int32_t first[ROPE_AXES + 1];          // first pair of each axis, then R
    float sign;
    double log2_step[ROPE_AXES];           // log2 of the ratio of two neighbouring frequencies
    int32_t whole;
};

template <class T, int V>
struct RopeVec { typedef T type __attribute__((ext_vector_type(V))); };
template <class T>
struct RopeVec<T, 1> { typedef T type; };
template <class T, int V>
__device__ __forceinline__ T& elem(typename RopeVec<T, V>::type& v, int i) { return reinterpret_cast<T*>(&v)[i]; }

// A unit is what a thread moves at a time: V neighbouring elements (INTER: pairs are neighbours), or V of them and the V
// that they are paired with.
template <class T, int V, bool INTER>
__global__ __launch_bounds__(ROPE_THREADS) void rope_kernel(const RopeArgs a) {
    typedef typename RopeVec<T, V>::type vec;
    extern __shared__ float2 table[];
    const int64_t row0 = (int64_t)blockIdx.x * a.tokens;
    const int tokens = (int)min((int64_t)a.tokens, a.rows - row0);
    // ---- cosines and sines of the tokens' angles
    const int64_t b0 = row0 / a.T;
    const int t0 = (int)(row0 - b0 * a.T);
    for (int i = threadIdx.x; i < tokens * a.R; i += ROPE_THREADS) {
        const int tok = i / a.R, p = i - tok * a.R;
        int ax = 0;
#pragma unroll
        for (int j = 1; j < ROPE_AXES; ++j) ax += p >= a.first[j] ? 1 : 0;
        int64_t b = b0;
        int t = t0 + tok;
        while (t >= a.T) {
            t -= a.T;
            ++b;
        }
        const double w = exp2(-(double)(a.whole ? p : p - a.first[ax]) * a.log2_step[ax]) * 0.15915494309189533577;   // turns per unit of position
        const double turns = (double)a.pos[b * a.pos_stride + (int64_t)t * a.n_axes + ax] * w;
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        table[i] = make_float2(c, a.sign * s);
    }
    __syncthreads();
    // ---- the heads: a thread's units are 256 apart, BATCH of them in flight together
    const int per = a.heads * a.units, n = tokens * per;
    constexpr int BATCH = 4, PIECES = INTER ? 1 : 2;
    for (int i0 = threadIdx.x; i0 < n; i0 += ROPE_THREADS * BATCH) {
        vec v[BATCH][PIECES];
        T* out[BATCH];
        int lo[BATCH], hi[BATCH], at[BATCH];          // of the pieces; of the unit's first cosine, or -1
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int i = min(i0 + k * ROPE_THREADS, n - 1);
            const int tok = per == 1 ? i : (int)__umulhi((uint32_t)i, a.by_token), rem = i - tok * per;
            const int head = a.units == 1 ? rem : (int)__umulhi((uint32_t)rem, a.by_head), u = rem - head * a.units;
            const bool isq = head < a.heads_q;
            const int64_t row = row0 + tok;
            const int h = (isq ? head : head - a.heads_q) * a.D;
            const T* const x = static_cast<const T*>(isq ? a.q : a.k) + row * (isq ? a.ldq : a.ldk) + h;
            out[k] = static_cast<T*>(isq ? a.yq : a.yk) + row * (isq ? a.ldyq : a.ldyk) + h;
            const bool turn = u < a.rot_units;
            if constexpr (INTER) {
                lo[k] = u * V;
                hi[k] = 0;
                at[k] = turn ? tok * a.R + u * (V / 2) : -1;
                v[k][0] = *reinterpret_cast<const vec*>(x + lo[k]);
            } else {
                const int p = u * V;
                lo[k] = p;
                hi[k] = p + a.R;
                if (!turn) {
                    lo[k] = 2 * a.R + (u - a.rot_units) * 2 * V;
                    hi[k] = lo[k] + V;
                } else if (a.axis_halves) {
                    int first = 0, end = a.first[1];
#pragma unroll
                    for (int j = 1; j < ROPE_AXES; ++j)
                        if (p >= a.first[j]) first = a.first[j], end = a.first[j + 1];
                    lo[k] = first + p;
                    hi[k] = lo[k] + end - first;
                }
                at[k] = turn ? tok * a.R + p : -1;
                v[k][0] = *reinterpret_cast<const vec*>(x + lo[k]);
                v[k][PIECES - 1] = *reinterpret_cast<const vec*>(x + hi[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            if (i0 + k * ROPE_THREADS >= n) break;
            vec &l = v[k][0], &r = v[k][PIECES - 1];
            if (at[k] >= 0) {
                const float2* const cs = table + at[k];
                if constexpr (INTER) {
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const float2 f = cs[e / 2];
                        const float c = (float)elem<T, V>(l, e), d = (float)elem<T, V>(l, e + 1);
                        elem<T, V>(l, e) = (T)(c * f.x - d * f.y);
                        elem<T, V>(l, e + 1) = (T)(c * f.y + d * f.x);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float2 f = cs[e];
                        const float c = (float)elem<T, V>(l, e), d = (float)elem<T, V>(r, e);
                        elem<T, V>(l, e) = (T)(c * f.x - d * f.y);
                        elem<T, V>(r, e) = (T)(c * f.y + d * f.x);
                    }
                }
            }
            *reinterpret_cast<vec*>(out[k] + lo[k]) = l;
            if constexpr (!INTER) *reinterpret_cast<vec*>(out[k] + hi[k]) = r;
        }
    }
}

template <class T, int V, bool INTER>
static int launch_rope(RopeArgs& a, hipStream_t stream) {
    a.units = INTER ? a.D / V : a.D / (2 * V);
    a.rot_units = INTER ? 2 * a.R / V : a.R / V;
    const int per = a.heads * a.units;
    // So many tokens that a thread has up to four units, but no fewer workgroups than four a CU while there are tokens.  (us, cold inputs and results, at 4 / 8 units: 12844 tokens of 32 heads x 128 fp32 79.7 /
    // 83.4, 8192 of 40 x 64 bf16 22.8 / 23.0; as few workgroups as eight units take / four a CU: 40 tokens of 4 x 88 6.0 / 2.9, 54 of 24 x 32 5.7 / 3.5)
    const int64_t most = (a.rows + 1023) / 1024;
    int tokens = 4 * ROPE_THREADS / per;
    tokens = tokens > ROPE_MAX_TOKENS ? ROPE_MAX_TOKENS : tokens;
    tokens = tokens > most ? (int)most : tokens < 1 ? 1 : tokens;
    static_assert(ROPE_MAX_TOKENS * (ROPE_MAX_D / 2) * sizeof(float2) <= 32768, "the table");
    const int64_t groups = (a.rows - 1) / tokens + 1;
    SD_REQUIRE(groups < (1 << 24), SD_EUNSUPPORTED, "rope: %lld tokens of %d heads", (long long)a.rows, a.heads);      // (threads of a launch stay below 2^32)
    a.tokens = tokens;
    // (exact: a unit's number times the divisor stays below 2^32)
    a.by_token = tokens == 1 ? 0 : (uint32_t)((1ull << 32) / per + 1);
    a.by_head = (uint32_t)((1ull << 32) / a.units + 1);
    if (SD_DRY_RUN("rope %s%d; ", INTER ? "neighbours " : "halves ", V)) return SD_OK;
    hipLaunchKernelGGL((rope_kernel<T, V, INTER>), dim3((unsigned)groups), dim3(ROPE_THREADS), tokens * a.R * sizeof(float2), stream, a);
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}

// Elements of an access: as many as 16 bytes hold, fewer where an axis or what a head keeps unturned ends inside.
template <class T>
static int launch_rope_as(RopeArgs& a, bool inter, hipStream_t stream) {
    constexpr int MAXV = 16 / (int)sizeof(T);
    int v = MAXV;
    for (; v > 1; v /= 2) {
        if (inter) {
            if (2 * a.R % v == 0) break;
            continue;
        }
        bool ok = a.R % v == 0 && (a.D - 2 * a.R) % (2 * v) == 0;
        for (int j = 1; ok && a.axis_halves && j < a.n_axes; ++j) ok = a.first[j] % v == 0;
        if (ok) break;
    }
    if (inter) {
        if constexpr (MAXV == 8)
            if (v == 8) return launch_rope<T, 8, true>(a, stream);
        if (v == 4) return launch_rope<T, 4, true>(a, stream);
        return launch_rope<T, 2, true>(a, stream);
    }
    if constexpr (MAXV == 8)
        if (v == 8) return launch_rope<T, 8, false>(a, stream);
    if (v == 4) return launch_rope<T, 4, false>(a, stream);
    if (v == 2) return launch_rope<T, 2, false>(a, stream);
    return launch_rope<T, 1, false>(a, stream);
}

static int rope(const char* who, float sign, const sd_rope* r, const float* pos, int64_t pos_stride, const void* q, int64_t ldq, int heads_q, void* yq, int64_t ldyq,
                const void* k, int64_t ldk, int heads_k, void* yk, int64_t ldyk, int dtype, int Bn, int T, hipStream_t stream) {
    SD_REQUIRE(r, SD_EINVAL, "%s: no description", who);
    SD_REQUIRE(r->head_dim > 0 && r->head_dim <= ROPE_MAX_D && r->head_dim % 8 == 0, SD_EUNSUPPORTED, "%s: head dim %d (a multiple of 8, at most %d)", who, r->head_dim, ROPE_MAX_D);
    SD_REQUIRE(r->n_axes >= 1 && r->n_axes <= ROPE_AXES, SD_EINVAL, "%s: %d axes (1 to %d)", who, r->n_axes, ROPE_AXES);
    SD_REQUIRE(r->layout == SD_ROPE_INTERLEAVED || r->layout == SD_ROPE_HALVES || r->layout == SD_ROPE_AXIS_HALVES, SD_EINVAL, "%s: layout %d", who, r->layout);
    SD_REQUIRE(r->theta > 0 && r->theta < 1e300, SD_EINVAL, "%s: theta %g", who, r->theta);
    SD_REQUIRE(dtype == SD_BF16 || dtype == SD_F32, SD_EINVAL, "%s: type %d", who, dtype);
    RopeArgs a;
    memset(&a, 0, sizeof(a));
    int64_t R = 0;
    for (int j = 0; j < r->n_axes; ++j) {
        SD_REQUIRE(r->pairs[j] >= 1, SD_EINVAL, "%s: axis %d has %d pairs", who, j, r->pairs[j]);
        a.first[j] = (int32_t)R;
        R += r->pairs[j];
        SD_REQUIRE(2 * R <= r->head_dim, SD_EINVAL, "%s: more pairs than half of the head dim %d", who, r->head_dim);
    }
    for (int j = r->n_axes; j <= ROPE_AXES; ++j) a.first[j] = (int32_t)R;
    for (int j = 0; j < r->n_axes; ++j) a.log2_step[j] = log2(r->theta) / (double)(r->whole ? R : r->pairs[j]);
    SD_REQUIRE(Bn >= 0 && T >= 0 && heads_q >= 0 && heads_k >= 0 && heads_q <= SD_ROPE_MAX_HEADS && heads_k <= SD_ROPE_MAX_HEADS, SD_EINVAL,
               "%s: Bn=%d T=%d heads %d, %d (at most %d)", who, Bn, T, heads_q, heads_k, SD_ROPE_MAX_HEADS);
    if (Bn == 0 || T == 0 || heads_q + heads_k == 0) return SD_OK;
    SD_REQUIRE(pos && (reinterpret_cast<uintptr_t>(pos) & 3u) == 0 && (pos_stride == 0 || pos_stride >= (int64_t)T * r->n_axes), SD_EINVAL, "%s: positions %p, %lld apart", who, (const void*)pos,
               (long long)pos_stride);
    const int64_t wq = (int64_t)heads_q * r->head_dim, wk = (int64_t)heads_k * r->head_dim;
    SD_REQUIRE(heads_q == 0 || (q && yq && aligned16(q) && aligned16(yq) && ldq >= wq && ldyq >= wq && ldq % 8 == 0 && ldyq % 8 == 0), SD_EINVAL,
               "%s: queries need 16-byte aligned pointers and rows of a multiple of 8 elements, %lld at least", who, (long long)wq);
    SD_REQUIRE(heads_k == 0 || (k && yk && aligned16(k) && aligned16(yk) && ldk >= wk && ldyk >= wk && ldk % 8 == 0 && ldyk % 8 == 0), SD_EINVAL,
               "%s: keys need 16-byte aligned pointers and rows of a multiple of 8 elements, %lld at least", who, (long long)wk);
    SD_REQUIRE(heads_q == 0 || heads_k == 0 || (yq != yk && yq != k && yk != q), SD_EINVAL, "%s: a result in the other's place", who);
    a.rows = (int64_t)Bn * T;
    // (workgroups take their tokens in any order: at another distance a token would be written over one that is still to be read)
    SD_REQUIRE(a.rows == 1 || ((heads_q == 0 || yq != q || ldyq == ldq) && (heads_k == 0 || yk != k || ldyk == ldk)), SD_EINVAL, "%s: in place with rows at another distance", who);
    SD_REQUIRE(a.rows <= 0x7fffffff, SD_EUNSUPPORTED, "%s: %lld tokens", who, (long long)a.rows);
    a.pos = pos; a.pos_stride = pos_stride; a.q = q; a.k = k; a.yq = yq; a.yk = yk;
    a.ldq = ldq; a.ldk = ldk; a.ldyq = ldyq; a.ldyk = ldyk;
    a.T = T; a.n_axes = r->n_axes; a.heads_q = heads_q; a.heads = heads_q + heads_k; a.D = r->head_dim; a.R = (int32_t)R;
    a.axis_halves = r->layout == SD_ROPE_AXIS_HALVES;
    a.sign = sign;
    a.whole = r->whole != 0;
    const bool inter = r->layout == SD_ROPE_INTERLEAVED;
    return dtype == SD_F32 ? launch_rope_as<float>(a, inter, stream) : launch_rope_as<__bf16>(a, inter, stream);
}

}  // namespace sd

extern "C" int sd_rope_fwd(const sd_rope* r, const float* pos, int64_t pos_stride, const void* q, int64_t ldq, int32_t heads_q, void* yq, int64_t ldyq,
                           const void* k, int64_t ldk, int32_t heads_k, void* yk, int64_t ldyk, int32_t dtype, int32_t Bn, int32_t T, void* stream) {
    return sd::rope("rope_fwd", 1.f, r, pos, pos_stride, q, ldq, heads_q, yq, ldyq, k, ldk, heads_k, yk, ldyk, dtype, Bn, T, static_cast<hipStream_t>(stream));
}
extern "C" int sd_rope_bwd(const sd_rope* r, const float* pos, int64_t pos_stride, const void* dq, int64_t ldq, int32_t heads_q, void* dxq, int64_t ldyq,
                           const void* dk, int64_t ldk, int32_t heads_k, void* dxk, int64_t ldyk, int32_t dtype, int32_t Bn, int32_t T, void* stream) {
    return sd::rope("rope_bwd", -1.f, r, pos, pos_stride, dq, ldq, heads_q, dxq, ldyq, dk, ldk, heads_k, dxk, ldyk, dtype, Bn, T, static_cast<hipStream_t>(stream));
}
