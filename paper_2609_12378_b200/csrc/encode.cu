// Encode: slot values -> plaintext limbs.
//
//   E1  Z[e_j] = z_j,  e_j = ((5^j mod 2N) - 1) / 4
//   E2  b_k = sum_e Z[e] omega^(-e k)   (size n, unnormalised), radix-2 decimation in time:
//       bit-reversed input, stages m = 2, 4, .., n, butterfly (u, v) -> (u + w v, u - w v) with
//       w = conj(omega^(j n / m)); every product and every sum rounded on its own (no FMA)
//   E3  a_k = b_k conj(zeta^k)
//   E4  m_k = rint(Re a_k * scale/n), m_{k+n} = rint(Im a_k * scale/n), ties to even
//   E5  residues of m_k modulo every prime, E6 NTT per limb.
//
// The transform of size n is split like the NTT: the stages with span <= CH run on
// contiguous chunks of CH points in shared memory, the remaining ones on strips of
// 16 columns of the [n/CH][CH] view.  Each radix-2 butterfly is performed exactly once
// with the operands the definition gives it, so the result does not depend on the split.
#include "common.cuh"

namespace {

constexpr uint32_t THREADS = 256;
constexpr uint32_t CH = 1024;   // points per chunk in the first pass
constexpr uint32_t COLS = 16;   // columns per CTA in the second pass

__device__ __forceinline__ double2 cmul_conj_w(double2 w, double2 v) {   // conj(w) * v, four products, two sums
    const double wr = w.x, wi = -w.y;
    const double p0 = __dmul_rn(wr, v.x), p1 = __dmul_rn(wi, v.y), p2 = __dmul_rn(wr, v.y), p3 = __dmul_rn(wi, v.x);
    return make_double2(__dsub_rn(p0, p1), __dadd_rn(p2, p3));
}

// ---- what a slot holds: an array's value, or one formed here (a launch and a trip through memory less) ---------------------
struct SlotArray { const double *re, *im; };
__device__ __forceinline__ double2 slot_value(const SlotArray &a, uint32_t b, uint32_t j, uint32_t n) {
    return make_double2(a.re[(size_t)b * n + j], a.im ? a.im[(size_t)b * n + j] : 0.0);
}
__device__ __forceinline__ double2 slot_value(const SlotPositions &a, uint32_t b, uint32_t j, uint32_t) {
    const uint32_t kind = b % a.kinds, set = b / a.kinds, t = j & ((1u << a.inner) - 1), d = j >> (a.inner + a.heads) & ((1u << a.dim) - 1), half = a.rot >> 1;
    if (t < a.begin[set] || t >= a.end[set]) return make_double2(0.0, 0.0);
    if (kind > a.nrot) return make_double2(1.0, 0.0);
    if (d >= a.rot) return make_double2(kind ? 0.0 : 1.0, 0.0);
    const bool second = a.interleaved ? d & 1 : d >= half;
    const uint32_t pair = a.interleaved ? d >> 1 : second ? d - half : d;
    const size_t at = ((size_t)a.row[set] + (size_t)(t - a.begin[set]) * a.step) * half + pair;
    if (!kind) return make_double2(a.cos[at], 0.0);
    // one rotation serves both channels of a pair; of two, the first (to the left) serves the first channel, the other the second
    if (a.nrot == 2 && second != (kind == 2)) return make_double2(0.0, 0.0);
    return make_double2(second ? a.sin[at] : -a.sin[at], 0.0);
}
__device__ __forceinline__ double2 slot_value(const SlotTokens &a, uint32_t b, uint32_t j, uint32_t) {
    const uint32_t t = j & ((1u << a.inner) - 1);
    return make_double2(t >= a.begin[b] && t < a.end[b] ? 1.0 : 0.0, 0.0);
}
__device__ __forceinline__ double2 slot_value(const SlotScores &a, uint32_t b, uint32_t j, uint32_t) {
    const uint32_t x = j >> a.copies, pos = x >> (a.inner + a.heads), per = a.tokens - a.inner, tokens = 1u << a.tokens;
    const uint32_t e = pos >> per, i = ((pos & ((1u << per) - 1)) << a.inner) + (x & ((1u << a.inner) - 1));
    // the key operand holds token (i + e) mod tokens in block e; group g is its rotation by g blocks' tokens over (e, i)
    uint32_t f = i + (a.g0 + b) * a.block, fe = e;
    if (f >= tokens) { f -= tokens; fe = e + 1 == a.block ? 0 : e + 1; }
    const uint32_t key = (f + fe) & (tokens - 1);
    const long long at = (long long)i + a.offset;
    const bool live = key >= a.key_begin && key < a.key_end && (!a.causal || (long long)key <= at) && (!a.window || (long long)key > at - (long long)a.window);
    return make_double2(live ? 1.0 : 0.0, 0.0);
}
__device__ __forceinline__ double2 slot_value(const SlotHeads &a, uint32_t, uint32_t j, uint32_t) {
    return make_double2(-a.weights[j >> (a.copies + a.inner) & ((1u << a.heads) - 1)], 0.0);
}

// Pass 1: gather (E1 + bit reversal), stages m = 2 .. min(n, CH) on chunks of CH points.  The stages' twiddles come from
// a copy in shared memory (stage by stage, so that a warp reads consecutive entries): fetched from the full table they
// were 5120 scattered 16-byte loads per CTA and the kernel was bound by the traffic between L2 and L1.
template <class Src>
__global__ void __launch_bounds__(THREADS) fft_chunks(DevTables c, const __grid_constant__ Src src, double2 *buf, uint32_t n, uint32_t ch) {
    __shared__ double2 sm[CH];
    __shared__ double2 tw[CH];
    const uint32_t b = blockIdx.y, base = blockIdx.x * ch;
    grid_dep_sync();
    for (uint32_t x = threadIdx.x; x < ch; x += THREADS) {
        const uint32_t j = c.enc_src[base + x];
        sm[x] = slot_value(src, b, j, n);
        tw[x] = c.enc_omega_st[x];
    }
    __syncthreads();
    // two stages per pass over shared memory: a thread takes the four points j, j + h, j + 2h, j + 3h of a block of 4h and does
    // the two butterflies of span h and the two of span 2h on registers (the same butterflies with the same operands as one
    // stage at a time; the kernel is bound by shared-memory traffic, which this halves)
    uint32_t m = 2;
    for (; 2 * m <= ch; m <<= 2) {
        const uint32_t h = m >> 1;
        for (uint32_t x = threadIdx.x; x < ch / 4; x += THREADS) {
            const uint32_t j = x & (h - 1), i0 = ((x - j) << 2) + j;
            double2 a0 = sm[i0], a1 = sm[i0 + h], a2 = sm[i0 + 2 * h], a3 = sm[i0 + 3 * h];
            const double2 w1 = tw[h + j];
            double2 t = cmul_conj_w(w1, a1);
            a1 = make_double2(__dsub_rn(a0.x, t.x), __dsub_rn(a0.y, t.y));
            a0 = make_double2(__dadd_rn(a0.x, t.x), __dadd_rn(a0.y, t.y));
            t = cmul_conj_w(w1, a3);
            a3 = make_double2(__dsub_rn(a2.x, t.x), __dsub_rn(a2.y, t.y));
            a2 = make_double2(__dadd_rn(a2.x, t.x), __dadd_rn(a2.y, t.y));
            t = cmul_conj_w(tw[2 * h + j], a2);
            a2 = make_double2(__dsub_rn(a0.x, t.x), __dsub_rn(a0.y, t.y));
            a0 = make_double2(__dadd_rn(a0.x, t.x), __dadd_rn(a0.y, t.y));
            t = cmul_conj_w(tw[2 * h + j + h], a3);
            a3 = make_double2(__dsub_rn(a1.x, t.x), __dsub_rn(a1.y, t.y));
            a1 = make_double2(__dadd_rn(a1.x, t.x), __dadd_rn(a1.y, t.y));
            sm[i0] = a0; sm[i0 + h] = a1; sm[i0 + 2 * h] = a2; sm[i0 + 3 * h] = a3;
        }
        __syncthreads();
    }
    for (; m <= ch; m <<= 1) {             // a last single stage when the number of stages is odd
        const uint32_t half = m >> 1;
        for (uint32_t x = threadIdx.x; x < ch / 2; x += THREADS) {
            const uint32_t j = x & (half - 1), i1 = ((x - j) << 1) + j;
            const double2 t = cmul_conj_w(tw[half + j], sm[i1 + half]);
            const double2 u = sm[i1];
            sm[i1] = make_double2(__dadd_rn(u.x, t.x), __dadd_rn(u.y, t.y));
            sm[i1 + half] = make_double2(__dsub_rn(u.x, t.x), __dsub_rn(u.y, t.y));
        }
        __syncthreads();
    }
    for (uint32_t x = threadIdx.x; x < ch; x += THREADS) buf[(size_t)b * n + base + x] = sm[x];
}

// Pass 2: stages m = 2 CH .. n on strips of COLS columns (rows = n/ch), then E3, E4 -> int64 coefficients.
__global__ void __launch_bounds__(THREADS) fft_strips_round(DevTables c, const double2 *buf, long long *coef, uint32_t n, uint32_t ch, double s) {
    extern __shared__ double2 sm2[];
    const uint32_t b = blockIdx.y, rows = n / ch, col0 = blockIdx.x * COLS;
    double2 *tw = sm2 + rows * COLS;          // the strip's twiddles, entry (hr + jr) * COLS + column (row 0 unused)
    grid_dep_sync();
    for (uint32_t x = threadIdx.x; x < rows * COLS; x += THREADS) {
        sm2[x] = buf[(size_t)b * n + (size_t)(x / COLS) * ch + col0 + x % COLS];
        tw[x] = c.enc_omega_st2[(size_t)(x / COLS) * ch + col0 + x % COLS];
    }
    __syncthreads();
    for (uint32_t m = 2 * ch; m <= n; m <<= 1) {
        const uint32_t half = m >> 1, hr = half / ch;      // hr = distance in rows
        for (uint32_t x = threadIdx.x; x < (rows / 2) * COLS; x += THREADS) {
            const uint32_t cc = x % COLS, y = x / COLS, jr = y & (hr - 1), r1 = ((y - jr) << 1) + jr;
            // twiddle omega^(j n / m) of position j = jr ch + col0 + cc inside the half block
            const double2 t = cmul_conj_w(tw[(hr + jr) * COLS + cc], sm2[(r1 + hr) * COLS + cc]);
            const double2 u = sm2[r1 * COLS + cc];
            sm2[r1 * COLS + cc] = make_double2(__dadd_rn(u.x, t.x), __dadd_rn(u.y, t.y));
            sm2[(r1 + hr) * COLS + cc] = make_double2(__dsub_rn(u.x, t.x), __dsub_rn(u.y, t.y));
        }
        __syncthreads();
    }
    for (uint32_t x = threadIdx.x; x < rows * COLS; x += THREADS) {
        const uint32_t k = (x / COLS) * ch + col0 + x % COLS;
        const double2 a = cmul_conj_w(c.enc_zeta[k], sm2[x]);
        double xr = __dmul_rn(a.x, s), xi = __dmul_rn(a.y, s);
        if (!(fabs(xr) < 4611686018427387904.0) || !(fabs(xi) < 4611686018427387904.0)) { *c.range_flag = 1; xr = xi = 0.0; }
        coef[(size_t)b * 2 * n + k] = __double2ll_rn(xr);
        coef[(size_t)b * 2 * n + n + k] = __double2ll_rn(xi);
    }
}

// slots[kk][r*T + t] = d'_k[r],  k = k0 + kk,  d'_k[r] = d_k[(r - (k - k mod B)) mod F],
// d_k[r'] = W^T[out0 + r' mod m_out, in0 + (r' + k) mod m_in]
__global__ void __launch_bounds__(THREADS) extract_diagonals(const double *W, uint32_t d_out_total, uint32_t in0, uint32_t m_in,
                                                             uint32_t out0, uint32_t m_out, uint32_t F, uint32_t T, uint32_t k0,
                                                             uint32_t B, double *slots, uint32_t n) {
    const uint32_t x = blockIdx.x * THREADS + threadIdx.x;
    grid_dep_sync();
    if (x >= n) return;
    const uint32_t r = x / T, k = k0 + blockIdx.y;
    const uint32_t rp = (r + F - (k - k % B) % F) % F;
    const uint32_t ro = rp % m_out, ci = (rp + k) % m_in;
    slots[(size_t)blockIdx.y * n + x] = W[(size_t)(in0 + ci) * d_out_total + out0 + ro];
}

}  // namespace

size_t encode_workspace_bytes(const ckks_ctx *c, uint32_t batch) {
    return (size_t)batch * ((size_t)c->n * sizeof(double2) + (size_t)c->N * sizeof(long long));
}

void launch_encode(const ckks_ctx *c, const double *re, const double *im, uint32_t batch, double scale, uint32_t level,
                   u64 *out, void *ws, cudaStream_t s, TiledOut tiled, u64 *tiled_out) {
    const uint32_t n = c->n, N = c->N, ch = n < CH ? n : CH;
    double2 *buf = (double2 *)ws;
    long long *coef = (long long *)(buf + (size_t)batch * n);
    const double sc = scale / (double)n;
    for (uint32_t b0 = 0; b0 < batch; b0 += 32768) {
        const uint32_t nb = batch - b0 < 32768 ? batch - b0 : 32768;
        launch(fft_chunks<SlotArray>, dim3(n / ch, nb), THREADS, 0, s, c->dev, SlotArray{re + (size_t)b0 * n, im ? im + (size_t)b0 * n : nullptr}, buf + (size_t)b0 * n, n, ch);
        launch(fft_strips_round, dim3(ch / COLS, nb), THREADS, (size_t)2 * (n / ch) * COLS * sizeof(double2), s, c->dev, buf + (size_t)b0 * n, coef + (size_t)b0 * N, n, ch, sc);
    }
    // the first NTT pass reduces the signed coefficients itself; the last one can write the tiled layout
    const NttPrologue pro{(const u64 *)coef, false, 0};
    NttEpilogue ep{};
    ep.mode = 2; ep.out.base = tiled_out; ep.level = level; ep.tl = tiled;
    launch_ntt(c, out, batch * level, plain_map(0, level), false, s, tiled.R ? &ep : nullptr, &pro);
}

template <class Slots>
void launch_encode_slots(const ckks_ctx *c, const Slots &slots, uint32_t batch, double scale, void *ws, cudaStream_t s) {
    const uint32_t n = c->n, ch = n < CH ? n : CH;
    double2 *buf = (double2 *)ws;
    long long *coef = (long long *)(buf + (size_t)batch * n);
    launch(fft_chunks<Slots>, dim3(n / ch, batch), THREADS, 0, s, c->dev, slots, buf, n, ch);
    launch(fft_strips_round, dim3(ch / COLS, batch), THREADS, (size_t)2 * (n / ch) * COLS * sizeof(double2), s, c->dev, buf, coef, n, ch, scale / (double)n);
}
template void launch_encode_slots(const ckks_ctx *, const SlotPositions &, uint32_t, double, void *, cudaStream_t);
template void launch_encode_slots(const ckks_ctx *, const SlotTokens &, uint32_t, double, void *, cudaStream_t);
template void launch_encode_slots(const ckks_ctx *, const SlotScores &, uint32_t, double, void *, cudaStream_t);
template void launch_encode_slots(const ckks_ctx *, const SlotHeads &, uint32_t, double, void *, cudaStream_t);

void launch_encode_coefs(const ckks_ctx *c, const void *ws, uint32_t batch, uint32_t limbs, const LimbMap &map, u64 *out, cudaStream_t s, bool sets) {
    const long long *coef = (const long long *)((const double2 *)ws + (size_t)batch * c->n);
    NttPrologue pro{(const u64 *)coef, false, 0};
    pro.sets = sets;
    launch_ntt(c, out, limbs, map, false, s, nullptr, &pro);
}

void launch_extract_diagonals(const ckks_ctx *c, const double *W, uint32_t d_out_total, uint32_t in0, uint32_t m_in,
                              uint32_t out0, uint32_t m_out, uint32_t F, uint32_t T, uint32_t k0, uint32_t count,
                              uint32_t B, double *slots, cudaStream_t s) {
    launch(extract_diagonals, dim3((c->n + THREADS - 1) / THREADS, count), THREADS, 0, s, W, d_out_total, in0, m_in, out0, m_out, F, T, k0, B, slots, c->n);
}
