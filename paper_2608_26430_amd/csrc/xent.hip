// Cross entropy of a head's logits, forward and gradient, without keeping the logits.
//
// With H (T x n) the activations, W (V x n) the head, z = H W^T:
//   lse_t = log sum_v exp z_tv,   loss_t = lse_t - z_t,target
//   P_tv  = (exp(z_tv - lse_t) - [v = target_t]) dloss_t,   dH = scale P W,   dW = scale P^T H
// Tokens whose target is no vocabulary entry have loss 0 and P = 0.
//
// The products run on MFMA (xent_gemm.h).  Only P, in the activations' type, passes through memory, a bounded
// piece of it at a time:
//   loss alone      logits product whose epilogue leaves (maximum, sum of exponentials) per token and wave's columns
//                   and the target's logit; nothing of the logits is written.
//   loss + gradient the same product also writes e = exp(z - maximum of the wave's other columns); when the statistics
//                   of a token are joined, e becomes P in place: 2 products (3 with dW) instead of the 3 (4) of a
//                   backward that computes the logits again.
//   backward alone  logits product whose epilogue writes P from the saved lse.
// P is kept in the activations' type: each of its values carries one rounding (up to 2^-8 relative in bf16), as do the
// factors W and H; e, stored first, is in fp16 (2^-11 down to 2^-29 of the columns' maximum).  Maxima and sums leave the
// target out: its own value of P, exp(z - lse) - 1, is then minus the others' share, the loss of a token whose target
// has the largest logit is log(1 + others), and the others' exponentials are in fp16's range however far the target is
// above them, so that all keep their digits when the target's probability is near one.
// scale is applied to the products' fp32 results: P of a token whose target is unlikely then holds minus nearly one, whose
// rounding is at most 2^-9, where nearly 1 / T of many tokens would all be rounded alike by up to twice that (3289 tokens,
// 1920 wide, 41,071 entries: dH's error 0.0025 -> 0.0019).
// With few tokens (kPairTokens) a handful of those roundings would decide the result (one token's dH would be off by its
// target's, up to 2^-8), so P is kept as a sum of two bf16 matrices there, the second one what rounding left of the
// first, as further tokens of dH's product and further k of dW's; the products are bound by reading W and writing dW.
// Long calls are cut into pieces of tokens (P of a piece at most kPieceBytes), whose dH are complete.  With dW a cut
// by tokens would have to add up V x n sums in fp32, so there the pieces are of the vocabulary (dW rows complete,
// dH summed in fp32), and the forward runs by itself first.
#include <cmath>

#include "xent_gemm.h"
#include "xent_plan.h"

namespace ff {
namespace xent {

hipError_t launch_gemm_0_0(int tile, const GemmArgs& a, hipStream_t s);
hipError_t launch_gemm_0_1(int tile, const GemmArgs& a, hipStream_t s);
hipError_t launch_gemm_1_0(int tile, const GemmArgs& a, hipStream_t s);
hipError_t launch_gemm_1_1(int tile, const GemmArgs& a, hipStream_t s);
hipError_t launch_gemm_2_0(int tile, const GemmArgs& a, hipStream_t s);
hipError_t launch_gemm_2_1(int tile, const GemmArgs& a, hipStream_t s);

hipError_t launch_gemm(int layout, int bf16, int tile, const GemmArgs& a, hipStream_t s) {
  switch (layout * 2 + bf16) {
    case 0: return launch_gemm_0_0(tile, a, s);
    case 1: return launch_gemm_0_1(tile, a, s);
    case 2: return launch_gemm_1_0(tile, a, s);
    case 3: return launch_gemm_1_1(tile, a, s);
    case 4: return launch_gemm_2_0(tile, a, s);
    default: return launch_gemm_2_1(tile, a, s);
  }
}

namespace {

// Joins the statistics of a token's columns, (maximum, sum of exponentials), both without the target: a workgroup takes TK
// tokens, its 256 / TK shares of the entries are joined through LDS.  The result is that of threads with part 0.
template <int TK>
__device__ __forceinline__ float2 join_stats(const float2* stats, int nstat, int N, int t, int part, int tk,
                                             float2 (&sh)[256 / TK][TK]) {
  constexpr int kShares = 256 / TK;
  float top = -INFINITY, sum = 0.f;
  auto join = [&](float2 s) {
    const float m = fmaxf(top, s.x);
    // columns of -inf have sum 0, a NaN logit makes the sum NaN
    const float ref = m == -INFINITY ? 0.f : m;
    sum = sum * expf(top - ref) + s.y * expf(s.x - ref);
    top = m;
  };
  if (t < N) {
    int i = part;
    for (; i + 7 * kShares < nstat; i += 8 * kShares) {      // eight loads in flight
      float2 s[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] = stats[(int64_t)(i + k * kShares) * N + t];
#pragma unroll
      for (int k = 0; k < 8; ++k) join(s[k]);
    }
    for (; i < nstat; i += kShares) join(stats[(int64_t)i * N + t]);
  }
  sh[part][tk] = make_float2(top, sum);
  for (int h = kShares / 2; h; h >>= 1) {
    __syncthreads();
    if (part < h) {
      join(sh[part + h][tk]);
      sh[part][tk] = make_float2(top, sum);
    }
  }
  return make_float2(top, sum);
}

// A token's loss and lse, and the target's value of P before its weight.
struct Token {
  float lse, loss, own;
};
__device__ __forceinline__ Token token_of(float2 joined, int64_t target, int64_t vocab, float z) {
  const float m = joined.x, others = joined.y;
  if (target < 0 || target >= vocab) return Token{m + logf(others), 0.f, 0.f};
  if (z >= m) {
    const float rest = others * expf(m - z), ls = log1pf(rest) + (z - z);     // (an infinite z: NaN)
    return Token{z + ls, ls, -rest / (1.f + rest)};
  }
  const float total = others + expf(z - m), ls = logf(total);
  return Token{m + ls, (m - z) + ls, -others / total};
}

template <int TK>
__global__ void __launch_bounds__(256) combine_kernel(const float2* stats, int nstat, int N, const int64_t* target,
                                                      int64_t vocab, float* zt, float* loss, float* lse) {
  __shared__ float2 sh[256 / TK][TK];
  const int tk = threadIdx.x % TK, part = threadIdx.x / TK;
  const int t = blockIdx.x * TK + tk;
  const float2 joined = join_stats<TK>(stats, nstat, N, t, part, tk, sh);
  if (part || t >= N) return;
  const Token k = token_of(joined, target[t], vocab, zt[t]);
  lse[t] = k.lse;
  loss[t] = k.loss;
  zt[t] = k.own;
}

template <class E>
struct Piece16;   // a 16-byte piece as floats
template <>
struct Piece16<__bf16> {
  static constexpr int kN = 8;
  // exponentials, stored in fp16
  static __device__ __forceinline__ void get_exp(const __bf16* p, float* v) {
    typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
    const f16x8 w = *reinterpret_cast<const f16x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)w[i] * (1.f / (1 << kExpShift));
  }
  static __device__ __forceinline__ void put(__bf16* p, const float* v) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (unsigned)bf16_bits(v[2 * i]) | (unsigned)bf16_bits(v[2 * i + 1]) << 16;
    *reinterpret_cast<u32x4*>(p) = w;
  }
};
template <>
struct Piece16<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void get_exp(const float* p, float* v) {
    const f32x4 w = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = w[i];
  }
  static __device__ __forceinline__ void put(float* p, const float* v) {
    const f32x4 w = {v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4*>(p) = w;
  }
};

// e = exp(z - maximum of its columns but the target) -> P, in place; rest: elements from a row to the one that takes what rounding left
// (0: none).  Bound by memory: P is read and written once (4096 x 32,000 in bf16: 74 us, 7 TB/s out of the last-level cache).
// JOIN: zt still holds the target's logit, and every workgroup of a token joins its statistics for itself, the first one
// writing loss and lse: a launch less than with combine_kernel, whose sums these are, where that reads little (12
// tokens, 1847 entries: 5.3 us for 4.6 + 3.5; 40 of 32,000, 160,000 statistics read: 8.7 for 6.0 + 5.0; 64 of 128,000 in
// fp32, 8 million: 44 for 11.5 + 10.6).
constexpr int kRescaleRow = 4;   // pieces per thread
template <class E, bool JOIN>
__global__ void __launch_bounds__(256) rescale_kernel(E* P, int64_t ldp, int64_t rest, int N, int V, const float2* stats, int cols,
                                                      const int64_t* target, const float* zt, float* loss, float* lse,
                                                      const float* dloss) {
  constexpr int kN = Piece16<E>::kN;
  const int t = blockIdx.y;
  const int64_t tg = target[t];
  const bool counted = tg >= 0 && tg < V;
  const float w = counted ? (dloss ? dloss[t] : 1.f) : 0.f;
  float ls, own = 0.f;
  if constexpr (JOIN) {
    __shared__ float2 sh[256][1];
    __shared__ Token joined;
    const float2 s = join_stats<1>(stats, (V + cols - 1) / cols, N, t, threadIdx.x, 0, sh);
    if (threadIdx.x == 0) {
      joined = token_of(s, tg, V, counted ? zt[t] : 0.f);
      if (blockIdx.x == 0) lse[t] = joined.lse, loss[t] = joined.loss;
    }
    __syncthreads();
    ls = joined.lse, own = joined.own;
  } else {
    ls = lse[t];
    if (counted) own = zt[t];
  }
  E* row = P + (int64_t)t * ldp;
#pragma unroll
  for (int q = 0; q < kRescaleRow; ++q) {
    const int c = ((blockIdx.x * kRescaleRow + q) * 256 + threadIdx.x) * kN;
    if (c >= ldp) return;
    float v[kN];
    if (counted) {
      Piece16<E>::get_exp(row + c, v);
      // columns past V hold zeros; their entry may be one past the statistics' last
      const float f = c < V ? expf(stats[(int64_t)(c / cols) * N + t].x - ls) * w : 0.f;
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] *= f;
      if (tg >= c && tg < c + kN) {
        const float p = own * w;
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] = tg == c + i ? p : v[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] = 0.f;
    }
    Piece16<E>::put(row + c, v);
    if (sizeof(E) == 2 && rest) {
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] -= (float)(E)v[i];
      Piece16<E>::put(row + rest + c, v);
    }
  }
}

// out = beta out + sum over the splits of part: N x M, M a multiple of four, from group `first` of four results on.  SH threads share the splits of four results;
// their sums are joined in a fixed order.  Few results of many splits are bound by the latency of one load after the
// other: 8 tokens, 176 wide, 128 sums 33 us with one thread, 3.9 with 16.
template <class E, int SH>
__global__ void __launch_bounds__(256) sum_kernel(const float* part, int splits, int64_t N, int M, float beta,
                                                  E* out, int64_t ldo, int64_t first) {
  constexpr int kWide = 256 / SH;
  __shared__ f32x4 sh[SH][kWide];
  const int lane = threadIdx.x % kWide, share = threadIdx.x / kWide;
  const int64_t per = M / 4, id = first + (int64_t)blockIdx.x * kWide + lane;
  const int64_t row = id / per;
  const int c = (int)(id - row * per) * 4;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (row < N) {
#pragma unroll 4
    for (int s = share; s < splits; s += SH) v += load4(part + ((int64_t)s * N + row) * M + c);
  }
  if constexpr (SH > 1) {
    sh[share][lane] = v;
    __syncthreads();
    if (share) return;
#pragma unroll
    for (int i = 1; i < SH; ++i) v += sh[i][lane];
  }
  if (row >= N) return;
  E* p = out + row * ldo + c;
  if (beta != 0.f) v += beta * load4(p);
  store4(p, v);
}

// Rows of H with a target; zeros elsewhere, so that nothing a skipped token holds (NaN, infinities) reaches dW, where
// its zero of P would be multiplied by it.  From piece `first` on.
template <class E>
__global__ void __launch_bounds__(256) live_rows_kernel(const E* H, int64_t ldh, int64_t T, int n, const int64_t* target,
                                                        int64_t vocab, int copies, E* out, int64_t first) {
  constexpr int kN = Piece16<E>::kN;
  const int64_t per = n / kN, id = first + (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= T * per) return;
  const int64_t t = id / per;
  const int c = (int)(id - t * per) * kN;
  const int64_t tg = target[t];
  u32x4 v = {0u, 0u, 0u, 0u};
  if (tg >= 0 && tg < vocab) v = *reinterpret_cast<const u32x4*>(H + t * ldh + c);
  for (int k = 0; k < copies; ++k) *reinterpret_cast<u32x4*>(out + (k * T + t) * n + c) = v;
}

// ------------------------------------------------------------------------------------------- a call's launches

struct Tensors {
  const char* H;
  int64_t ldh;
  const char* W;
  int64_t ldw;
  const int64_t* target;
  const float* dloss;
  float scale;
  float* loss;
  float* lse;
  float beta_dh, beta_dw;
  char* dH;
  int64_t lddh;
  char* dW;
  int64_t lddw;
  char* ws;
  hipStream_t s;
};

constexpr int64_t kLaunchItems = (int64_t)1 << 28;   // threads of one launch of sums or copies: it must have fewer than 2^32

#define XENT_TRY(call)                   \
  do {                                   \
    const hipError_t e_ = (call);        \
    if (e_ != hipSuccess) return e_;     \
  } while (0)

// tokens t0 .. t0 + N - 1, vocabulary entries v0 .. v0 + M - 1
hipError_t run_logits(const Call& c, const Tensors& x, int64_t t0, int64_t N, int64_t v0, int64_t M, int mode,
                      int* stat) {
  const Product p = logits_product(c, N, M);
  GemmArgs a{};
  a.A = x.W + v0 * x.ldw * c.esz, a.lda = x.ldw;
  a.B = x.H + t0 * x.ldh * c.esz, a.ldb = x.ldh;
  a.M = (int)M, a.N = (int)N, a.K = (int)c.n;
  a.tm = (int)(up(M, tile_m(p.tile)) / tile_m(p.tile)), a.tn = (int)(up(N, tile_n(p.tile)) / tile_n(p.tile));
  a.kt = a.kt_split = p.kt_split, a.splits = 1, a.mode = mode;
  a.out = x.ws + c.off_p, a.ldo = up(M, 64), a.ocols = (int)up(M, 64);
  a.rest = c.terms == 2 ? N * a.ldo : 0;
  a.stats = reinterpret_cast<float2*>(x.ws + c.off_stats);
  a.target = x.target + t0, a.v0 = v0, a.vocab = c.V;
  a.zt = reinterpret_cast<float*>(x.ws + c.off_zt);
  a.lse = x.lse + t0, a.loss = x.loss ? x.loss + t0 : nullptr, a.dloss = x.dloss ? x.dloss + t0 : nullptr;
  *stat = stat_cols(p.tile);
  return launch_gemm(0, c.bf16, p.tile, a, x.s);
}

hipError_t run_combine(const Call& c, const Tensors& x, int64_t t0, int64_t N, int stat) {
  const float2* stats = reinterpret_cast<const float2*>(x.ws + c.off_stats);
  float* zt = reinterpret_cast<float*>(x.ws + c.off_zt);
  const int nstat = (int)(up(c.V, stat) / stat);
  // few tokens: all threads on one (a token's entries lie N apart, so that many tokens are read side by side)
  if (N <= kFewTokens)
    hipLaunchKernelGGL(combine_kernel<1>, dim3((unsigned)N), dim3(256), 0, x.s, stats, nstat, (int)N, x.target + t0, c.V, zt,
                       x.loss + t0, x.lse + t0);
  else
    hipLaunchKernelGGL(combine_kernel<8>, dim3((unsigned)((N + 7) / 8)), dim3(256), 0, x.s, stats, nstat, (int)N,
                       x.target + t0, c.V, zt, x.loss + t0, x.lse + t0);
  return hipGetLastError();
}

template <class E, bool JOIN>
void rescale(const Call& c, const Tensors& x, int64_t t0, int64_t N, int stat) {
  const int64_t ldp = up(c.V, 64), seg = 256 * kRescaleRow * Piece16<E>::kN;
  // rows in groups that fit the grid's second dimension
  for (int64_t r = 0; r < N; r += 32768) {
    const int64_t rows = N - r < 32768 ? N - r : 32768;
    hipLaunchKernelGGL((rescale_kernel<E, JOIN>), dim3((unsigned)((ldp + seg - 1) / seg), (unsigned)rows), dim3(256), 0, x.s,
                       reinterpret_cast<E*>(x.ws + c.off_p) + r * ldp, ldp, c.terms == 2 ? N * ldp : 0, (int)N, (int)c.V,
                       reinterpret_cast<const float2*>(x.ws + c.off_stats) + r, stat, x.target + t0 + r,
                       reinterpret_cast<const float*>(x.ws + c.off_zt) + r, x.loss + t0 + r, x.lse + t0 + r,
                       x.dloss ? x.dloss + t0 + r : nullptr);
  }
}

hipError_t run_sum(const Call& c, const Tensors& x, int splits, int64_t N, int64_t M, float beta, void* out, int64_t ldo) {
  const int64_t threads = N * (M / 4);
  const float* part = reinterpret_cast<const float*>(x.ws + c.off_part);
  const int shares = splits >= 16 && threads <= 65536 ? 16 : 1;
  for (int64_t first = 0; first < threads; first += kLaunchItems) {
    const int64_t items = threads - first < kLaunchItems ? threads - first : kLaunchItems;
    const dim3 grid((unsigned)((items * shares + 255) / 256)), block(256);
    if (c.bf16) {
      __bf16* o = static_cast<__bf16*>(out);
      if (shares > 1) hipLaunchKernelGGL((sum_kernel<__bf16, 16>), grid, block, 0, x.s, part, splits, N, (int)M, beta, o, ldo, first);
      else hipLaunchKernelGGL((sum_kernel<__bf16, 1>), grid, block, 0, x.s, part, splits, N, (int)M, beta, o, ldo, first);
    } else {
      float* o = static_cast<float*>(out);
      if (shares > 1) hipLaunchKernelGGL((sum_kernel<float, 16>), grid, block, 0, x.s, part, splits, N, (int)M, beta, o, ldo, first);
      else hipLaunchKernelGGL((sum_kernel<float, 1>), grid, block, 0, x.s, part, splits, N, (int)M, beta, o, ldo, first);
    }
    XENT_TRY(hipGetLastError());
  }
  return hipSuccess;
}

// dH of tokens t0 .. from P of vocabulary entries v0 ..; first / last piece of the vocabulary
hipError_t run_dh(const Call& c, const Tensors& x, int64_t t0, int64_t N, int64_t v0, int64_t M, bool first, bool last) {
  const int64_t rows = c.terms * N;
  const Product p = dh_product(c, rows, c.Vp);     // the same split for every piece of the vocabulary
  GemmArgs a{};
  a.A = x.W + v0 * x.ldw * c.esz, a.lda = x.ldw;
  a.B = x.ws + c.off_p, a.ldb = up(M, 64);
  a.M = (int)c.n, a.N = (int)rows, a.K = (int)M;
  a.tm = (int)(up(c.n, tile_m(p.tile)) / tile_m(p.tile)), a.tn = (int)(up(rows, tile_n(p.tile)) / tile_n(p.tile));
  a.kt = (int)(up(M, c.kk) / c.kk), a.kt_split = p.kt_split, a.splits = p.splits;
  const bool direct = p.splits * c.terms == 1 && first && last;
  void* out = x.dH + t0 * x.lddh * c.esz;
  a.mode = direct ? kOut : kPart;
  a.out = out, a.ldo = x.lddh, a.alpha = x.scale, a.beta = x.beta_dh;
  a.part = reinterpret_cast<float*>(x.ws + c.off_part), a.part_add = !first;
  XENT_TRY(launch_gemm(1, c.bf16, p.tile, a, x.s));
  return direct || !last ? hipSuccess : run_sum(c, x, p.splits * c.terms, N, c.n, x.beta_dh, out, x.lddh);
}

// rows v0 .. v0 + M - 1 of dW from P of all tokens
hipError_t run_dw(const Call& c, const Tensors& x, int64_t v0, int64_t M) {
  const int64_t K = c.terms * c.T;
  Product p = dw_product(c, M, K);
  if (c.by_vocab) p.splits = 1, p.kt_split = (int)(up(K, c.kk) / c.kk);   // the partial sums' place holds dH's
  GemmArgs a{};
  a.A = x.ws + c.off_live, a.lda = c.n;
  a.B = x.ws + c.off_p, a.ldb = up(M, 64);
  a.M = (int)c.n, a.N = (int)M, a.K = (int)K;
  a.tm = (int)(up(c.n, tile_m(p.tile)) / tile_m(p.tile)), a.tn = (int)(up(M, tile_n(p.tile)) / tile_n(p.tile));
  a.kt = (int)(up(K, c.kk) / c.kk), a.kt_split = p.kt_split, a.splits = p.splits;
  void* out = x.dW + v0 * x.lddw * c.esz;
  a.mode = p.splits == 1 ? kOut : kPart;
  a.out = out, a.ldo = x.lddw, a.alpha = x.scale, a.beta = x.beta_dw;
  a.part = reinterpret_cast<float*>(x.ws + c.off_part);
  XENT_TRY(launch_gemm(2, c.bf16, p.tile, a, x.s));
  return p.splits == 1 ? hipSuccess : run_sum(c, x, p.splits, M, c.n, x.beta_dw, out, x.lddw);
}

hipError_t run_live_rows(const Call& c, const Tensors& x) {
  const int64_t threads = c.T * (c.n * c.esz / 16);
  for (int64_t first = 0; first < threads; first += kLaunchItems) {
    const int64_t items = threads - first < kLaunchItems ? threads - first : kLaunchItems;
    const dim3 grid((unsigned)((items + 255) / 256));
    if (c.bf16)
      hipLaunchKernelGGL(live_rows_kernel<__bf16>, grid, dim3(256), 0, x.s, reinterpret_cast<const __bf16*>(x.H), x.ldh,
                         c.T, (int)c.n, x.target, c.V, c.terms, reinterpret_cast<__bf16*>(x.ws + c.off_live), first);
    else
      hipLaunchKernelGGL(live_rows_kernel<float>, grid, dim3(256), 0, x.s, reinterpret_cast<const float*>(x.H), x.ldh, c.T,
                         (int)c.n, x.target, c.V, c.terms, reinterpret_cast<float*>(x.ws + c.off_live), first);
    XENT_TRY(hipGetLastError());
  }
  return hipSuccess;
}

hipError_t run_fwd(const Call& c, const Tensors& x) {
  for (int64_t t0 = 0; t0 < c.T; t0 += c.Tf) {
    const int64_t N = c.T - t0 < c.Tf ? c.T - t0 : c.Tf;
    int stat = 0;
    XENT_TRY(run_logits(c, x, t0, N, 0, c.V, kStats, &stat));
    XENT_TRY(run_combine(c, x, t0, N, stat));
  }
  return hipSuccess;
}

// step: with the forward (loss and lse written); otherwise from the saved lse
hipError_t run_bwd(const Call& c, const Tensors& x, bool step) {
  if (c.T == 0) return c.dw ? run_sum(c, x, 0, c.V, c.n, x.beta_dw, x.dW, x.lddw) : hipSuccess;
  if (c.dw) XENT_TRY(run_live_rows(c, x));
  int stat = 0;
  if (c.by_vocab) {
    if (step) XENT_TRY(run_fwd(c, x));
    for (int64_t v0 = 0; v0 < c.V; v0 += c.Vp) {
      const int64_t M = c.V - v0 < c.Vp ? c.V - v0 : c.Vp;
      XENT_TRY(run_logits(c, x, 0, c.T, v0, M, kGrad, &stat));
      if (c.dh) XENT_TRY(run_dh(c, x, 0, c.T, v0, M, v0 == 0, v0 + M == c.V));
      XENT_TRY(run_dw(c, x, v0, M));
    }
    return hipSuccess;
  }
  for (int64_t t0 = 0; t0 < c.T; t0 += c.Tp) {
    const int64_t N = c.T - t0 < c.Tp ? c.T - t0 : c.Tp;
    XENT_TRY(run_logits(c, x, t0, N, 0, c.V, step ? kExp : kGrad, &stat));
    if (step) {
      const int64_t seg = 256 * kRescaleRow * (16 / c.esz);     // of a workgroup's columns
      if (N <= kFewTokens && N * (up(c.V, stat) / stat) * (up(c.V, seg) / seg) <= kJoinReads) {
        if (c.bf16) rescale<__bf16, true>(c, x, t0, N, stat);
        else rescale<float, true>(c, x, t0, N, stat);
      } else {
        XENT_TRY(run_combine(c, x, t0, N, stat));
        if (c.bf16) rescale<__bf16, false>(c, x, t0, N, stat);
        else rescale<float, false>(c, x, t0, N, stat);
      }
      XENT_TRY(hipGetLastError());
    }
    if (c.dh) XENT_TRY(run_dh(c, x, t0, N, 0, c.V, true, true));
    if (c.dw) XENT_TRY(run_dw(c, x, 0, c.V));
  }
  return hipSuccess;
}

// ------------------------------------------------------------------------------------------- argument checks

ff_status check_sizes(int64_t T, int64_t n, int64_t V, int act, bool grad) {
  if (act != FF_F32 && act != FF_BF16) return fail(FF_EINVAL, "unknown activation dtype %d", act);
  const int64_t mult = act == FF_BF16 ? 8 : 4;
  if (T < 0 || T > ((int64_t)1 << 28)) return fail(FF_EINVAL, "T=%lld out of range", (long long)T);
  if (V < 1 || V > (grad ? kMaxGradVocab : (int64_t)1 << 24)) return fail(FF_EINVAL, "V=%lld out of range", (long long)V);
  if (n < mult || n > ((int64_t)1 << 18) || n % mult)
    return fail(FF_EINVAL, "n=%lld must be a multiple of %lld, at most 262144", (long long)n, (long long)mult);
  return FF_OK;
}

ff_status check_rows(const char* name, const void* p, int64_t ld, int64_t n, int act) {
  const int64_t mult = act == FF_BF16 ? 8 : 4;
  if (!p) return fail(FF_EINVAL, "%s is NULL", name);
  if (ld < n || ld > kMaxLd || ld % mult)
    return fail(FF_EINVAL, "leading dimension of %s (%lld) must be a multiple of %lld, from %lld to 1048576", name,
                (long long)ld, (long long)mult, (long long)n);
  if ((uintptr_t)p % 16) return fail(FF_EINVAL, "%s is not 16-byte aligned", name);
  return FF_OK;
}

ff_status check_vector(const char* name, const void* p, int align) {
  if (!p) return fail(FF_EINVAL, "%s is NULL", name);
  if ((uintptr_t)p % align) return fail(FF_EINVAL, "%s is not %d-byte aligned", name, align);
  return FF_OK;
}

ff_status check_workspace(const Call& c, const void* ws, int64_t bytes) {
  if (!ws || (uintptr_t)ws % 256) return fail(FF_EINVAL, "the workspace is NULL or not 256-byte aligned");
  if (bytes < (int64_t)c.bytes)
    return fail(FF_EINVAL, "the workspace holds %lld bytes, the call needs %lld", (long long)bytes, (long long)c.bytes);
  return FF_OK;
}

ff_status done(hipError_t e, const char* what) {
  return e == hipSuccess ? FF_OK : fail(FF_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

#define XENT_CHECK(call)                 \
  do {                                   \
    const ff_status st_ = (call);        \
    if (st_ != FF_OK) return st_;        \
  } while (0)

ff_status check_grad(const Call& c, const Tensors& x, int act, int64_t ws_bytes) {
  if (c.T > 0) {
    XENT_CHECK(check_rows("H", x.H, x.ldh, c.n, act));
    XENT_CHECK(check_rows("W", x.W, x.ldw, c.n, act));
    XENT_CHECK(check_vector("target", x.target, 8));
    XENT_CHECK(check_vector("lse", x.lse, 4));
    if (x.loss) XENT_CHECK(check_vector("loss", x.loss, 4));
    if (x.dloss) XENT_CHECK(check_vector("dloss", x.dloss, 4));
    if (c.dh) XENT_CHECK(check_rows("dH", x.dH, x.lddh, c.n, act));
    XENT_CHECK(check_workspace(c, x.ws, ws_bytes));
  }
  if (c.dw) XENT_CHECK(check_rows("dW", x.dW, x.lddw, c.n, act));
  return FF_OK;
}

}  // namespace
}  // namespace xent
}  // namespace ff

using ff::xent::Call;
using ff::xent::Tensors;

extern "C" {

ff_status ff_xent_workspace(int64_t T, int64_t n, int64_t V, int act, int want, int64_t* bytes) {
  ff::clear_error();
  XENT_CHECK(ff::xent::check_sizes(T, n, V, act, want != 0));
  if (want < 0 || want > (FF_XENT_DH | FF_XENT_DW)) return ff::fail(FF_EINVAL, "unknown outputs %d", want);
  if (!bytes) return ff::fail(FF_EINVAL, "bytes is NULL");
  *bytes = (int64_t)ff::xent::plan(T, n, V, act, want & FF_XENT_DH, want & FF_XENT_DW).bytes;
  return FF_OK;
}

ff_status ff_xent_fwd(int64_t T, int64_t n, int64_t V, int act, const void* H, int64_t ldh, const void* W, int64_t ldw,
                      const int64_t* target, float* loss, float* lse, void* workspace, int64_t workspace_bytes,
                      void* stream) {
  ff::clear_error();
  XENT_CHECK(ff::xent::check_sizes(T, n, V, act, false));
  if (T == 0) return FF_OK;
  const Call c = ff::xent::plan(T, n, V, act, false, false);
  XENT_CHECK(ff::xent::check_rows("H", H, ldh, n, act));
  XENT_CHECK(ff::xent::check_rows("W", W, ldw, n, act));
  XENT_CHECK(ff::xent::check_vector("target", target, 8));
  XENT_CHECK(ff::xent::check_vector("loss", loss, 4));
  XENT_CHECK(ff::xent::check_vector("lse", lse, 4));
  XENT_CHECK(ff::xent::check_workspace(c, workspace, workspace_bytes));
  Tensors x{};
  x.H = (const char*)H, x.ldh = ldh, x.W = (const char*)W, x.ldw = ldw, x.target = target, x.loss = loss, x.lse = lse;
  x.ws = (char*)workspace, x.s = (hipStream_t)stream;
  return ff::xent::done(ff::xent::run_fwd(c, x), "loss forward");
}

ff_status ff_xent_bwd(int64_t T, int64_t n, int64_t V, int act, const void* H, int64_t ldh, const void* W, int64_t ldw,
                      const int64_t* target, const float* lse, const float* loss, const float* dloss, float scale,
                      float beta_dh, void* dH, int64_t lddh, float beta_dw, void* dW, int64_t lddw, void* workspace,
                      int64_t workspace_bytes, void* stream) {
  ff::clear_error();
  XENT_CHECK(ff::xent::check_sizes(T, n, V, act, true));
  if (!dH && !dW) return FF_OK;
  const Call c = ff::xent::plan(T, n, V, act, dH != nullptr, dW != nullptr);
  Tensors x{(const char*)H, ldh, (const char*)W, ldw, target, dloss, scale, const_cast<float*>(loss), const_cast<float*>(lse), beta_dh,
            beta_dw, (char*)dH, lddh, (char*)dW, lddw, (char*)workspace, (hipStream_t)stream};
  XENT_CHECK(ff::xent::check_grad(c, x, act, workspace_bytes));
  return ff::xent::done(ff::xent::run_bwd(c, x, false), "loss backward");
}

ff_status ff_xent_step(int64_t T, int64_t n, int64_t V, int act, const void* H, int64_t ldh, const void* W, int64_t ldw,
                       const int64_t* target, const float* dloss, float scale, float* loss, float* lse, float beta_dh,
                       void* dH, int64_t lddh, float beta_dw, void* dW, int64_t lddw, void* workspace,
                       int64_t workspace_bytes, void* stream) {
  ff::clear_error();
  XENT_CHECK(ff::xent::check_sizes(T, n, V, act, dH || dW));
  const Call c = ff::xent::plan(T, n, V, act, dH != nullptr, dW != nullptr);
  Tensors x{(const char*)H, ldh, (const char*)W, ldw, target, dloss, scale, loss, lse, beta_dh, beta_dw, (char*)dH, lddh,
            (char*)dW, lddw, (char*)workspace, (hipStream_t)stream};
  if (T > 0) XENT_CHECK(ff::xent::check_vector("loss", loss, 4));
  XENT_CHECK(ff::xent::check_grad(c, x, act, workspace_bytes));
  if (!dH && !dW) return T == 0 ? FF_OK : ff::xent::done(ff::xent::run_fwd(c, x), "loss forward");
  return ff::xent::done(ff::xent::run_bwd(c, x, true), "loss step");
}

}  // extern "C"
