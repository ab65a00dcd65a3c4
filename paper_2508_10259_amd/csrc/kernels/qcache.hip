// The 8-bit K/V cache: append, attention and the selection of pages (kernels.h, QCache).
//
// Layout.  A page holds 64 positions of every head of one layer.  Keys are rows [64][D] of
// e4m3; values are stored four positions to a dword, [16][D][4].  With keys as the A operand
// of S^T = K Q^T and values as the A operand of O^T = V^T P^T a lane's fragments are whole
// 16-byte words of either page, and the probabilities leave the first product in the registers
// the second one reads: nothing is transposed.
//   16x16x32 product, lane l = 16 g + i:  A row i, B column i, k slots 8 g .. 8 g + 7,
//   C column i, rows 4 g .. 4 g + 3.
//   S^T tile t of a 32-position step: A row i = position 16 t + i, k slots of step s = channels
//     g D/4 + 8 s .. + 7 (both operands agree on that order); the lane gets the scores of query i
//     at positions 16 t + 4 g + r.
//   O^T tile j: A row i = channel 64 (j / 4) + 4 i + j % 4, k slots of group g = positions 4 g ..
//     4 g + 3 of tile 0, then of tile 1: one dword of the value page each, and the lane's own scores.
// A scale is a power of two: e4m3 keeps its three mantissa bits at any exponent, so a finer scale
// would not round better, and moving a page to a larger scale is exact but for subnormals.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace ams {

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int PG = KV_PAGE;
constexpr float QC_LOG2E = 1.4426950408889634f;

// A segment of the call's tokens: n tokens from t0 on, at positions p0 .. of row `row`.  Everything
// read from the device is brought into range here, so no value of it can lead outside a buffer.
struct Seg {
  int row, t0, n, p0, len;
};
template <bool UNIFORM = true>  // whether s is the same for the whole wave
__device__ __forceinline__ Seg seg_of(const QSegs& sg, int s, int rows, int cap) {
  auto at = [](const int32_t* p, int k) { return UNIFORM ? ld_const_uniform(p, k) : p[k]; };
  Seg x;
  x.row = sg.row ? at(sg.row, s) : s;
  x.t0 = sg.off ? at(sg.off, s) : s;
  const int t1 = sg.off ? at(sg.off, s + 1) : s + 1;
  x.t0 = min(max(x.t0, 0), sg.n_tok);
  x.n = min(min(max(t1, x.t0), sg.n_tok) - x.t0, sg.max_new);
  if (sg.pos) {
    x.p0 = at(sg.pos, s);
    x.len = min(max(x.p0, -sg.n_tok) + x.n, cap);
  } else {
    x.len = min(max(at(sg.len, s), 0) + sg.len_add, cap);
  }
  x.p0 = x.len - x.n;
  if (x.row < 0 || x.row >= rows) x.n = 0;
  return x;
}

// The pool page of a row's page `lp` (lp < ppr), -1 for one outside the pool.
__device__ __forceinline__ int page_of(const QCache& c, int row, int lp) {
  const int p = ld_const_uniform(c.pt, (size_t)row * c.ppr + lp);
  return (unsigned)p < (unsigned)c.n_pages ? p : -1;
}

// Eight consecutive elements of type dt (DType) as fp32; al: their address is 16-byte aligned.
__device__ __forceinline__ void load8(const void* p, int64_t at, int dt, bool al, float* x) {
  if (dt == DT_F32) {
    const float* f = (const float*)p + at;
    if (al) {
      *(float4*)x = *(const float4*)f;
      *(float4*)(x + 4) = *(const float4*)(f + 4);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = f[e];
    }
    return;
  }
  uint32_t w[4];
  const uint16_t* h = (const uint16_t*)p + at;
  if (al) {
    *(uint4*)w = *(const uint4*)h;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (uint32_t)h[2 * e] | (uint32_t)h[2 * e + 1] << 16;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (dt == DT_BF16) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    } else {
      const half2v v = __builtin_bit_cast(half2v, w[e]);
      x[2 * e] = (float)v[0];
      x[2 * e + 1] = (float)v[1];
    }
  }
}

// bf16 nearest even, NaN kept (the sums of an attention may be NaN).
__device__ __forceinline__ uint32_t to_bf16(float f) { return f != f ? 0x7FC0u : f2bf(f); }
__device__ __forceinline__ uint32_t to_f16(float f) {
  const float c = f != f ? f : fminf(fmaxf(f, -F16_MAX), F16_MAX);
  return __builtin_bit_cast(uint16_t, (f16)c);
}

// N (4 or 8) consecutive outputs of type dt; lo: also the rounding errors of an fp16 output.
template <int N>
__device__ __forceinline__ void store_row(void* p, int64_t at, int dt, bool al, const float* x, f16* lo) {
  if (dt == DT_F32) {
    float* f = (float*)p + at;
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      if (al) *(float4*)(f + e) = float4{x[e], x[e + 1], x[e + 2], x[e + 3]};
      else
#pragma unroll
        for (int k = 0; k < 4; ++k) f[e + k] = x[e + k];
    }
    return;
  }
  uint32_t w[N / 2];
#pragma unroll
  for (int e = 0; e < N / 2; ++e)
    w[e] = dt == DT_BF16 ? to_bf16(x[2 * e]) | to_bf16(x[2 * e + 1]) << 16
                         : to_f16(x[2 * e]) | to_f16(x[2 * e + 1]) << 16;
  uint16_t* h = (uint16_t*)p + at;
  if (al) {
    if (N == 8) *(uint4*)h = uint4{w[0], w[1], w[N / 2 - 2], w[N / 2 - 1]};
    else *(uint2*)h = uint2{w[0], w[1]};
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) h[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
  }
  if (lo) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const f16 hi = __builtin_bit_cast(f16, (uint16_t)(w[e / 2] >> (16 * (e & 1))));
      lo[at + e] = sat16(x[e] - (float)hi);
    }
  }
}

// Eight e4m3 codes as fp16 times `scale` (a power of two).
__device__ __forceinline__ half8 codes_f16(uint32_t a, uint32_t b, float scale) {
  const half2v x0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, scale, false);
  const half2v x1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, scale, true);
  const half2v x2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, scale, false);
  const half2v x3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, scale, true);
  return half8{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
}

__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ void unpack_codes(uint32_t w, float* x) {
  x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
  x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
  x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
  x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
}
// Four codes rounded again after a multiplication by 2^de.
__device__ __forceinline__ uint32_t rescale_codes(uint32_t w, int de) {
  float x[4];
  unpack_codes(w, x);
  return pack_codes(ldexpf(x[0], de), ldexpf(x[1], de), ldexpf(x[2], de), ldexpf(x[3], de));
}

// ---------------------------------------------------------------------------
// Append.  One workgroup per (page, head): it alone writes that page's codes, scales and bounds.
// D/8 lanes take a quad of slots, 8 channels each: a lane's four values of a channel are one dword of the value page,
// its four keys 8 bytes of their rows.  With few tokens they take one slot, and a value is a byte of that dword.  The
// tokens stay in registers from the maximum, which sets the scale, to the rounding.
// Measured: 64 prefixes of 200 to 400 tokens, 32 heads of 128, bf16 with rotation: 136 us for 0.48 GB, 3.5 TB/s (a
// large copy: 4.85); the chain load, maximum, round, store bounds it, four waves a SIMD deep.  One token for each of 64
// rows: 7 us, a launch and four dependent round trips.

// The least e >= -32 with a <= 448 2^e (448 = 0.875 * 2^9).
__device__ __forceinline__ int scale_exponent(float a) {
  int x;
  const float m = frexpf(a, &x);
  const int e = x - 9 + (m > 0.875f ? 1 : 0);
  return a > 0.f ? min(max(e, -32), 8) : -32;
}
__device__ __forceinline__ int exponent_of(float scale) {
  int x;
  frexpf(scale, &x);
  return x - 1;
}

struct AppendArgs {
  QCache c;
  QSegs sg;
  const void *k, *v;
  int64_t ldk, ldv;
  int dt, alk, alv, chunks;
  const float2* rope;
};

template <int D, int NT, int PER>  // PER: slots of a lane
__global__ __launch_bounds__(NT) void k_qcache_append(AppendArgs a) {
  constexpr int LPT = D / 8, NW = NT / 64;
  const QCache& c = a.c;
  const int h = blockIdx.x % c.H, rest = blockIdx.x / c.H, chunk = rest % a.chunks, s = rest / a.chunks;
  const Seg sg = seg_of(a.sg, s, c.rows, c.ppr * PG);
  const int first = max(sg.p0, 0);  // tokens at positions below 0 have no place
  if (sg.n <= 0 || sg.len <= first) return;
  const int lp = first / PG + chunk;
  if (lp * PG >= sg.len) return;
  const int page = page_of(c, sg.row, lp);  // (looked at after the tokens' loads, which do not wait for it)
  const int s0 = max(first - lp * PG, 0), s1 = min(sg.len - lp * PG, PG);
  const int tok = sg.t0 + (lp * PG - sg.p0);  // token at slot 0 (slots s0 .. s1 - 1 are this call's)
  const int tid = threadIdx.x, sub = tid % LPT, grp = tid / LPT, lane = tid & 63, wave = tid >> 6;
  const int slot0 = PER == 4 ? grp * 4 : s0 + grp;
  __shared__ float red[2][NW];
  __shared__ float bred[2][NW][D];

  float k[PER][8], v[PER][8];
  uint32_t fresh = 0u;  // a byte for each of the lane's slots that this call writes
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int slot = slot0 + p;
    if (slot >= s0 && slot < s1) {
      load8(a.k, (int64_t)(tok + slot) * a.ldk + (int64_t)h * D + sub * 8, a.dt, a.alk, k[p]);
      load8(a.v, (int64_t)(tok + slot) * a.ldv + (int64_t)h * D + sub * 8, a.dt, a.alv, v[p]);
      fresh |= 0xFFu << (8 * p);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) k[p][e] = v[p][e] = 0.f;
    }
  }
  if (page < 0) return;
  const size_t ph = (size_t)page * c.H + h;
  // The scales of the page's older positions.  Every wave asks for them before the workgroup's barrier: the first
  // thread overwrites them at the end, when other waves may only just have left that barrier.
  float ks_old = 0.f, vs_old = 0.f;
  if (s0 > 0) {
    ks_old = c.ks[ph];
    vs_old = c.vs[ph];
  }
  // each channel's largest and smallest key (rounding keeps their order, so their codes are the codes' bounds), and
  // the largest |value|
  float hi[8], lo[8], va = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    hi[e] = -INFINITY;
    lo[e] = INFINITY;
  }
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    if (a.rope) {  // pair (i, i + D/2): the partner's channels sit D/16 lanes away
      const float2* tab =
          a.rope + (size_t)min(lp * PG + slot0 + p, c.ppr * PG - 1) * (D / 2) + (sub % (LPT / 2)) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float other = __shfl_xor(k[p][e], LPT / 2, 64);
        const float2 cs = tab[e];
        float x, y;
        const bool low = sub < LPT / 2;
        rope_pair(low ? k[p][e] : other, low ? other : k[p][e], cs.x, cs.y, x, y);
        k[p][e] = low ? x : y;
      }
    }
    bool nan = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) nan |= __builtin_isunordered(k[p][e], v[p][e]);
    const uint64_t nans = __ballot(nan);
    if (nans) {
      // a NaN anywhere in the token's key or value: its key gets one, its value none, so that the
      // queries which see the token read NaN and no other query does (0 * NaN would reach those)
      const bool mine = nans >> (lane - lane % LPT) & ((1ull << LPT) - 1ull);
      if (mine && sub == 0) k[p][0] = __uint_as_float(0x7FC00000u);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (k[p][e] == k[p][e]) k[p][e] = fminf(fmaxf(k[p][e], -F16_MAX), F16_MAX);
        v[p][e] = v[p][e] == v[p][e] ? fminf(fmaxf(v[p][e], -F16_MAX), F16_MAX) : 0.f;
      }
    } else {  // one instruction each
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        k[p][e] = __builtin_amdgcn_fmed3f(k[p][e], -F16_MAX, F16_MAX);
        v[p][e] = __builtin_amdgcn_fmed3f(v[p][e], -F16_MAX, F16_MAX);
      }
    }
    if (fresh >> (8 * p) & 1u) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {  // (a NaN counts in none)
        hi[e] = fmaxf(hi[e], k[p][e]);
        lo[e] = fminf(lo[e], k[p][e]);
        va = fmaxf(va, fabsf(v[p][e]));
      }
    }
  }
  float ka = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) ka = fmaxf(ka, fmaxf(hi[e], -lo[e]));
  ka = wave_max(ka);
  va = wave_max(va);
  // the channels' bounds over the wave's tokens, then over the workgroup's
#pragma unroll
  for (int o = LPT; o < 64; o <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi[e] = fmaxf(hi[e], __shfl_xor(hi[e], o, 64));
      lo[e] = fminf(lo[e], __shfl_xor(lo[e], o, 64));
    }
  if (NW > 1) {
    if (lane == 0) {
      red[0][wave] = ka;
      red[1][wave] = va;
    }
    if (lane < LPT)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        bred[0][wave][sub * 8 + e] = hi[e];
        bred[1][wave][sub * 8 + e] = lo[e];
      }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      ka = fmaxf(ka, red[0][w]);
      va = fmaxf(va, red[1][w]);
    }
  }
  int ke = scale_exponent(ka), ve = scale_exponent(va), kd = 0, vd = 0;  // kd, vd: older codes' shift (<= 0)
  if (s0 > 0) {
    const int ko = exponent_of(ks_old), vo = exponent_of(vs_old);
    ke = max(ke, ko);
    ve = max(ve, vo);
    kd = ko - ke;
    vd = vo - ve;
  }

  uint8_t* kpage = c.k + ph * (PG * D);
  uint8_t* vpage = c.v + ph * (PG * D);
  if (kd < 0)
    for (int i = tid; i < s0 * (D / 8); i += NT) {
      uint2* w = (uint2*)kpage + i;
      const uint2 x = *w;
      *w = uint2{rescale_codes(x.x, kd), rescale_codes(x.y, kd)};
    }
  if (vd < 0) {
    // (PER 4: the quad that holds older and new slots is left to its lanes)
    const int quads = PER == 4 ? s0 / 4 : (s0 + 3) / 4;
    for (int i = tid; i < quads * D; i += NT) {
      uint32_t* w = (uint32_t*)vpage + i;
      const int n = s0 - i / D * 4;
      const uint32_t older = n >= 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u;
      *w = (rescale_codes(*w, vd) & older) | (*w & ~older);
    }
    if (PER == 1) __syncthreads();
  }
  const float ki = ldexpf(1.f, -ke), vi = ldexpf(1.f, -ve);
#pragma unroll
  for (int p = 0; p < PER; ++p)
    if (fresh >> (8 * p) & 1u) {
      uint2 w;
      w.x = pack_codes(k[p][0] * ki, k[p][1] * ki, k[p][2] * ki, k[p][3] * ki);
      w.y = pack_codes(k[p][4] * ki, k[p][5] * ki, k[p][6] * ki, k[p][7] * ki);
      *(uint2*)(kpage + (slot0 + p) * D + sub * 8) = w;
    }
  uint8_t* vdst = vpage + ((slot0 >> 2) * D + sub * 8) * 4;  // eight channels of the quad: 32 bytes
  if (PER == 1 && fresh) {  // a byte of each dword
    const uint32_t w[2] = {pack_codes(v[0][0] * vi, v[0][1] * vi, v[0][2] * vi, v[0][3] * vi),
                           pack_codes(v[0][4] * vi, v[0][5] * vi, v[0][6] * vi, v[0][7] * vi)};
#pragma unroll
    for (int e = 0; e < 8; ++e) vdst[4 * e + (slot0 & 3)] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
  }
  if (PER == 4 && fresh) {
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      w[e] = pack_codes(v[0][e] * vi, v[PER > 1 ? 1 : 0][e] * vi, v[PER > 2 ? 2 : 0][e] * vi, v[PER > 3 ? 3 : 0][e] * vi);
    uint4* dst = (uint4*)vdst;
    if (fresh != 0xFFFFFFFFu) {  // slots that are not this call's keep their codes, older ones at the new scale
      uint32_t old[8];
      *(uint4*)old = dst[0];
      *(uint4*)(old + 4) = dst[1];
      const int n = min(max(s0 - slot0, 0), 4);  // older slots
      const uint32_t older = n ? 0xFFFFFFFFu >> (32 - 8 * n) : 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (vd < 0) old[e] = (rescale_codes(old[e], vd) & older) | (old[e] & ~older);
        w[e] = (w[e] & fresh) | (old[e] & ~fresh);
      }
    }
    dst[0] = uint4{w[0], w[1], w[2], w[3]};
    dst[1] = uint4{w[4], w[5], w[6], w[7]};
  }
  if (tid < LPT) {
    int8_t* b = c.kb + ph * (2 * D) + sub * 8;
    __align__(8) int8_t bh[8], bl[8];
    if (s0 > 0) {
      *(uint2*)bh = *(const uint2*)b;
      *(uint2*)bl = *(const uint2*)(b + D);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (NW > 1)
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          hi[e] = fmaxf(hi[e], bred[0][w][sub * 8 + e]);
          lo[e] = fminf(lo[e], bred[1][w][sub * 8 + e]);
        }
      const bool some = hi[e] >= lo[e];  // (a channel may hold NaN only)
      const uint32_t w = pack_codes(some ? hi[e] * ki : 0.f, some ? lo[e] * ki : 0.f, 0.f, 0.f);
      float nh = some ? ceilf(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * 0.25f) : -128.f;
      float nl = some ? floorf(__builtin_amdgcn_cvt_f32_fp8((int)w, 1) * 0.25f) : 127.f;
      if (s0 > 0 && bh[e] != -128) {  // (-128: NaN only so far, a bound that does not move with the scale)
        nh = fmaxf(nh, ceilf(ldexpf((float)bh[e], kd)));
        nl = fminf(nl, floorf(ldexpf((float)bl[e], kd)));
      }
      bh[e] = (int8_t)nh;
      bl[e] = (int8_t)nl;
    }
    *(uint2*)b = *(uint2*)bh;
    *(uint2*)(b + D) = *(uint2*)bl;
  }
  if (tid == 0) {
    c.ks[ph] = ldexpf(1.f, ke);
    c.vs[ph] = ldexpf(1.f, ve);
  }
}

// ---------------------------------------------------------------------------
// Attention.  A query's column c of a segment is head c % G of the KV head's group at token c / G.
// A wave keeps its columns' running maximum and sum in the lanes that hold them and walks 32-position steps.  With few
// columns (k_qcache_attend: QT tiles of 16) the four waves share them and deal the steps among themselves, so the cache
// streams once; with many (k_qcache_attend_wide) each wave has its own and all walk the same steps, whose K/V come from
// the L1 for three waves of four.  PAIR (fp32 queries): queries and probabilities as fp16 pairs, about 22 bits.  fp16 and
// bf16 queries enter as they are, and their probabilities are rounded to fp16: fp16 outputs are off by 2.3e-4 to 2.9e-4 of
// their norm (2.0e-4 by their own rounding), bf16 ones by 1.7e-3 with or without.  Pairs would cost a build half as much
// again (eight prefixes of 2,048 tokens, 8 x 4 heads: 374 us, 564 with them) and a decode 1 to 3% (64 rows: 52.0, 53.4).
// Measured: few columns are bound by memory (4 rows of 70,000 to 131,000 positions, 8 x 4 heads of 128: 152 us for 0.82
// GB, 5.4 TB/s; 64 rows of 200 to 768 positions, 32 heads: 51 us for 0.25 GB), many by the vector unit and the products
// of the same waves taking turns (eight prefixes of 1,500 to 2,048 tokens, 8 x 4 heads: 293 us, 0.71 PFLOP/s).

struct AttendArgs {
  QCache c;
  QSegs sg;
  const void* q;
  int64_t ldq;
  void* o;
  int64_t ldo;
  f16* olo;
  int dt, odt, alq, alo, G;
  float scale;
  const float2* rope;
  const int32_t* sel;  // [n_tok][H][n_sel] pages of a token's row (SEL)
  int n_sel, tiles, splits, per, by_xcd;  // per: 32-position steps of a split
  bool even;  // the segments' lengths set it instead (even_steps)
  float* part;
};

template <int D> struct Step {  // a lane's K and V bytes of 32 positions
  i32x4 k[D / 32];
  uint4 v[2][D / 64];
};

// The 32-position steps a wave takes: `from`, from + inc, ... below `end` of its row, or of the pages in `list`, that
// begin below vmax and whose page lies in the pool.  Lane j holds page, position and scales of the j-th of 64 steps (a
// bit of `todo` each), so that no step waits for the page table: one round trip for 64 steps.
template <bool SEL> struct Walk {
  const QCache& c;
  const int32_t* list;
  int row, h, lane, from, inc, end, vmax;
  int lane_page, lane_pos;
  float lane_ks, lane_vs;
  uint64_t todo;
  // the step that find() found, lane j's
  int j;
  size_t ph;  // page * heads + head
  int pos;
  float ks, vs;
  bool ok;

  __device__ __forceinline__ void fill() {
    const int st = from + lane * inc;
    bool there = st < end;
    if (there) {
      int lp = st >> 1;
      if (SEL) lp = list[lp];
      lane_pos = lp * PG + 32 * (st & 1);
      // (a position at or behind vmax: the last page's second half)
      there = (unsigned)lp < (unsigned)c.ppr && lane_pos < vmax;
      if (there) {
        lane_page = c.pt[(size_t)row * c.ppr + lp];
        there = (unsigned)lane_page < (unsigned)c.n_pages;
        if (there) {
          lane_ks = c.ks[(size_t)lane_page * c.H + h];
          lane_vs = c.vs[(size_t)lane_page * c.H + h];
        }
      }
    }
    todo = __ballot(there);
  }
  // Waits for fill's scales.  Left to their first use, which may or may not follow a fill, the wait would be for every
  // load in flight, the next step's K and V among them, in every step.  (This and `step` without conditions around its
  // loads: eight prefixes of 1,500 to 2,048 tokens, 8 x 4 heads of 128, 320 -> 291 us.)
  __device__ __forceinline__ void settle() { asm volatile("" : "+v"(lane_ks), "+v"(lane_vs)); }
  __device__ __forceinline__ void find() {
    while (todo == 0) {
      from += 64 * inc;
      if (from >= end) {
        ok = false;
        return;
      }
      fill();
      settle();
    }
    j = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)todo) - 1);
    todo &= todo - 1;
    ph = (size_t)__builtin_amdgcn_readlane(lane_page, j) * c.H + h;
    pos = __builtin_amdgcn_readlane(lane_pos, j);
    ok = true;
  }
  __device__ __forceinline__ void scales() {
    ks = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(lane_ks), j));
    vs = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(lane_vs), j));
  }
  __device__ __forceinline__ void next() {
    find();
    if (ok) scales();
  }
};

// (Plain loads: non-temporal ones cost 4% over 64 ragged rows and 36% where tokens select the same pages.)
template <int D>
__device__ __forceinline__ void load_k(const QCache& c, size_t ph, int half, int lane, i32x4 (&k)[D / 32]) {
  const uint8_t* p = c.k + (ph * (PG * D) + half * (32 * D));
  const uint32_t at = lane * 16u;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) k[e] = *(const i32x4*)(p + at + e * 1024);
}
// A product wants a key to a lane, and 16-byte loads whose neighbouring lanes are in different rows pass the L1 at a
// quarter of its rate (measured: 15.7 bytes a cycle and CU, 59 with neighbours side by side).  So a wave loads its 32
// keys as they lie in memory, and turns them in LDS of its own: the 16-byte pieces of a row are permuted so that eight
// lanes meet all banks, in the writes (one row, or two of 64) and in the reads (eight rows' pieces).  4 x 48 new tokens
// over 32 selected pages each, 8 x 4 heads of 128, where pages come from the L2: 84 us without, 68 with.
template <int D>
__device__ __forceinline__ int k_slot(int row, int piece) {
  return row * D + (piece ^ (D == 128 ? row & 7 : (row >> 1) & 3)) * 16;
}
template <int D>
__device__ __forceinline__ void turn_k(const i32x4 (&k)[D / 32], char* lds, int lane) {
  constexpr int PR = D / 16;  // pieces of a row
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (lanes read what others wrote)
#pragma unroll
  for (int e = 0; e < D / 32; ++e) *(i32x4*)(lds + k_slot<D>(e * (64 / PR) + lane / PR, lane % PR)) = k[e];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
template <int D>
__device__ __forceinline__ void load_v(const QCache& c, size_t ph, int half, int lane, uint4 (&v)[2][D / 64]) {
  const uint8_t* p = c.v + (ph * (PG * D) + half * (32 * D));
  const uint32_t at = (lane >> 4) * (4u * D) + (lane & 15) * 16u;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int e = 0; e < D / 64; ++e) v[t][e] = *(const uint4*)(p + at + t * 16 * D + e * 256);
}

// The 32-position steps that segment s's last token sees.
__device__ __forceinline__ int steps_of(const AttendArgs& a, int s) {
  if (s >= a.sg.n_seg) return 0;
  const Seg x = seg_of<false>(a.sg, s, a.c.rows, a.c.ppr * PG);
  return x.n > 0 ? (max(x.len, 0) + 31) / 32 : 0;
}
// Steps per split that cut all segments into equal pieces, `splits` of them and one more for each segment at most: the
// launch has as many workgroups as run at once, and ragged rows keep them all equally long.
__device__ __forceinline__ int even_steps(const AttendArgs& a, int lane) {
  int total = 0;
  for (int r = lane; r < a.sg.n_seg; r += 64) total += steps_of(a, r);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o, 64);
  return __builtin_amdgcn_readfirstlane(max((total + a.splits - 1) / a.splits, QCACHE_LEAST_STEPS));
}

// Probabilities are 2^(score - m), where the reference m is `lift` below a running maximum that moves only when a score
// exceeds it by more than `slack`: at most 2^14 in fp16.  Those of the largest score and down to 2^-18 of it (2^-28 once the
// slack is used up) have 11 bits; smaller ones are subnormal, off by 2^-25 at most, that is 2^-29 of the largest.  Pairs keep their
// second halves above the subnormals by a larger lift.
// (Eight prefixes of 1,500 to 2,048 tokens, 8 x 4 heads of 128: 361 us with no slack when 333 with it.)
constexpr float slack_of(bool pair) { return pair ? 0.f : 10.f; }
constexpr float lift_of(bool pair) { return pair ? 12.f : 4.f; }
// A score is rounded to fp32 before the reference is subtracted: left to a fused operation, scores of 2^26 and more exceed
// their own maximum, or fall short of it, by half an fp32 step, which no fp16 probability holds.
__device__ __forceinline__ float mul_rounded(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}
// The reference for a largest score; where fp32 steps are larger than the lift, no more than 15 below it.
template <bool PAIR> __device__ __forceinline__ float reference_of(float top) {
  const float m = top - lift_of(PAIR);
  return top - m > 15.f ? top : m;
}
// fp16 probabilities are summed as they enter the product, rounded, so that their weights add up to one: a query that
// one position dominates gets that position's value exactly.
__device__ __forceinline__ float sum_of(half8 p, float l) {
  const half2v one = {(f16)1.f, (f16)1.f};
#pragma unroll
  for (int e = 0; e < 8; e += 2) l = __builtin_amdgcn_fdot2(half2v{p[e], p[e + 1]}, one, l, false);
  return l;
}

template <int D, int QT, bool PAIR, bool SEL>
__global__ __launch_bounds__(256, QT == 1 ? (PAIR ? 3 : 4) : 2) void k_qcache_attend(AttendArgs a) {
  constexpr int NS = D / 32, NJ = D / 16, CT = 16 * QT;
  constexpr float SLACK = slack_of(PAIR), LIFT = lift_of(PAIR);
  const QCache& c = a.c;
  // block -> (split, column tile, head, segment[, token])
  int id = blockIdx.x;
  int split, tile, h, s, tokn = 0, per = a.per;
  if (!SEL && a.even) {
    const int lane = threadIdx.x & 63;
    per = even_steps(a, lane);
    h = id % c.H; id /= c.H;
    tile = a.tiles - 1 - id % a.tiles; id /= a.tiles;
    // piece `id` of the segments' pieces one after another
    s = -1;
    for (int r = 0, base = 0; r < a.sg.n_seg; r += 64) {
      const int n = (steps_of(a, r + lane) + per - 1) / per;
      int upto = n;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(upto, o, 64);
        if (lane >= o) upto += y;
      }
      const uint64_t mine = __ballot(id - base < upto && id - base >= upto - n);
      if (mine) {
        const int j = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)mine) - 1);
        s = r + j;
        split = id - base - __builtin_amdgcn_readlane(upto - n, j);
        break;
      }
      base += __builtin_amdgcn_readlane(upto, 63);
    }
    if (s < 0) return;
  } else if (a.by_xcd) {
    // Blocks go to the 8 XCDs in turn; those of one (segment, head) pair follow each other on one XCD and
    // read the same pages through its L2.  The tiles with the most positions go first.
    const int x = id & 7;
    id >>= 3;
    split = id % a.splits; id /= a.splits;
    tile = a.tiles - 1 - id % a.tiles; id /= a.tiles;
    if (SEL) { tokn = id % a.sg.max_new; id /= a.sg.max_new; }
    const int pair = id * 8 + x;
    if (pair >= a.sg.n_seg * c.H) return;
    h = pair % c.H;
    s = pair / c.H;
  } else {
    // splits fastest, each (head, tile, ...) starting at another one: a short row's last splits have no work, and
    // every XCD gets its share of those
    split = id % a.splits; id /= a.splits;
    split = (split + id) % a.splits;
    h = id % c.H; id /= c.H;
    if (SEL) { tokn = id % a.sg.max_new; id /= a.sg.max_new; }
    tile = a.tiles - 1 - id % a.tiles; id /= a.tiles;
    s = id;
  }
  Seg sg = seg_of(a.sg, s, c.rows, c.ppr * PG);
  if (SEL) {  // one token of the segment
    if (tokn >= sg.n) return;
    sg.t0 += tokn;
    sg.p0 += tokn;
    sg.n = 1;
  }
  const int G = a.G, ncols = sg.n * G;
  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col0 = tile * CT;
  if (col0 >= ncols) return;

  // what the first and the last column see
  const int vmin = max(sg.p0 + col0 / G + 1, 0);
  const int vmax = max(sg.p0 + (min(col0 + CT, ncols) - 1) / G + 1, 0);

  // 32-position steps of this split, dealt to the waves (with `per` from an estimate of the length the last split
  // takes what a row has beyond it)
  const int steps = SEL ? 2 * a.n_sel : (vmax + 31) / 32;
  const int begin = split * per, end = split == a.splits - 1 && !a.even ? steps : min(steps, begin + per);
  Walk<SEL> at{c, SEL ? a.sel + ((size_t)sg.t0 * c.H + h) * a.n_sel : nullptr, sg.row, h, lane, begin + wave, 4, end, vmax};

  f32x4 o[QT][NJ];
  float m[QT], l[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // o is in units of 2^vref: a value page's scale relative to it goes into the conversion of its codes
  int vref = 0;
  bool first = true;

  constexpr int LD = D + 4;
  // the four waves' sums meet in LDS, after each wave's keys of a step
  // (32 columns: in two rounds, since four waves' sums take more than 64 KB)
  constexpr int SLOTS = QT == 1 ? 4 : 2;
  __shared__ __align__(16) float so[SLOTS * CT * LD];
  __shared__ float sm[4][CT], sl[4][CT];
  char* keys = (char*)so + wave * (32 * D);
  static_assert(4 * 32 * D <= sizeof(so));

  Step<D> x;
  at.fill();
  at.find();
  if (at.ok) {
    load_k<D>(c, at.ph, (at.pos >> 5) & 1, lane, x.k);
    load_v<D>(c, at.ph, (at.pos >> 5) & 1, lane, x.v);
  }
  at.settle();
  at.scales();
  // (the first positions are on their way)
  // queries: scaled by a power of two so that a column's largest element is in [2^10, 2^11).  An infinite one makes every
  // score infinite or NaN, so every output NaN; said at once, since a score of -infinity stands for a masked one here.
  half8 qh[QT][NS], ql[PAIR ? QT : 1][NS];
  float cq[QT];
  int vis[QT], tokc[QT], headc[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int col = col0 + 16 * t + i;
    const bool ok = col < ncols;
    tokc[t] = ok ? col / G : 0;
    headc[t] = h * G + (ok ? col % G : 0);
    vis[t] = ok ? sg.p0 + tokc[t] + 1 : 0;
    tokc[t] = ok ? sg.t0 + tokc[t] : -1;
    float x[NS][8], m = 0.f;
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      if (ok) load8(a.q, (int64_t)tokc[t] * a.ldq + (int64_t)headc[t] * D + g * (D / 4) + k * 8, a.dt, a.alq, x[k]);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) x[k][e] = 0.f;
    }
    if (a.rope) {
      const float2* tab = a.rope + (size_t)min(max(vis[t] - 1, 0), c.ppr * PG - 1) * (D / 2) + (g & 1) * (D / 4);
#pragma unroll
      for (int k = 0; k < NS; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float other = __shfl_xor(x[k][e], 32, 64);
          const float2 cs = tab[k * 8 + e];
          float lo, hi;
          rope_pair(g < 2 ? x[k][e] : other, g < 2 ? other : x[k][e], cs.x, cs.y, lo, hi);
          x[k][e] = g < 2 ? lo : hi;
        }
    }
#pragma unroll
    for (int k = 0; k < NS; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[k][e]));
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    int ex;
    frexpf(m, &ex);
    if (!(m > 0.f)) ex = 0;
    cq[t] = ldexpf(a.scale * QC_LOG2E, ex - 11);
#pragma unroll
    for (int k = 0; k < NS; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = ldexpf(x[k][e], 11 - ex);
        qh[t][k][e] = (f16)y;
        if (PAIR) ql[t][k][e] = (f16)(y - (float)qh[t][k][e]);
      }
    if (m == INFINITY) qh[t][0][0] = (f16)NAN;
  }
  // One step; EDGE: some of its positions are masked for a column, or lie behind the row's last one.  MORE: the next
  // one's loads go out as its registers get free, without a condition, so that each wait is for what it needs alone.
  int p0 = 0;
  float ks = 0.f, vs = 0.f;
  auto advance = [&] {
    p0 = at.pos;
    ks = at.ks;
    vs = at.vs;
    at.next();
  };
  auto step = [&](auto edge_tag, auto more_tag) {
    constexpr bool EDGE = decltype(edge_tag)::value, MORE = decltype(more_tag)::value;
    turn_k<D>(x.k, keys, lane);
    if (MORE) load_k<D>(c, at.ph, (at.pos >> 5) & 1, lane, x.k);
    // S^T = K Q^T
    f32x4 sc[QT][2];
#pragma unroll
    for (int t = 0; t < QT; ++t) sc[t][0] = sc[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        const i32x4 w = *(const i32x4*)(keys + k_slot<D>(16 * n + i, g * (D / 64) + k / 2));
        const half8 A = k & 1 ? codes_f16(w[2], w[3], 1.f) : codes_f16(w[0], w[1], 1.f);
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          sc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, qh[t][k], sc[t][n], 0, 0, 0);
          if (PAIR) sc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, ql[t][k], sc[t][n], 0, 0, 0);
        }
      }
    // softmax of the 32 positions
    int ve = exponent_of(vs);
    if (first) vref = ve;
    first = false;
    float fall = 1.f;  // o to another unit where the page's scale is far from it
    if (ve - vref > 4 || ve - vref < -6) {
      fall = ldexpf(1.f, vref - ve);
      vref = ve;
    }
    const float vr = ldexpf(1.f, ve - vref);
    half8 ph8[QT], pl8[PAIR ? QT : 1];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float cs = cq[t] * ks;
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          sc[t][n][r] = mul_rounded(sc[t][n][r], cs);
          if (EDGE && p0 + 16 * n + 4 * g + r >= vis[t]) sc[t][n][r] = -INFINITY;
          top = fmaxf(top, sc[t][n][r]);
        }
      // most steps leave the reference and o alone
      if (__any(top - m[t] > SLACK + LIFT) || fall != 1.f) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float nm = top - m[t] > SLACK + LIFT ? reference_of<PAIR>(top) : m[t];
        const float al = nm == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[t] - nm);
        l[t] *= al;
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[t][j] *= al * fall;
        m[t] = nm;
      }
      const float base = m[t] == -INFINITY ? 0.f : m[t];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = __builtin_amdgcn_exp2f(sc[t][n][r] - base);
          ph8[t][4 * n + r] = (f16)p;
          if (PAIR) {
            pl8[t][4 * n + r] = (f16)(p - (float)ph8[t][4 * n + r]);
            l[t] += p;
          }
        }
      if (!PAIR) l[t] = sum_of(ph8[t], l[t]);
    }
    // O^T += V^T P^T; codes behind the row's last position may be anything
    if (EDGE) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int left = min(max(sg.len - (p0 + 16 * n + 4 * g), 0), 4);
        const uint32_t keep = left == 4 ? 0xFFFFFFFFu : (1u << (8 * left)) - 1u;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) {
          x.v[n][e].x &= keep;
          x.v[n][e].y &= keep;
          x.v[n][e].z &= keep;
          x.v[n][e].w &= keep;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const uint4 w0 = x.v[0][j / 4], w1 = x.v[1][j / 4];
      const uint32_t d0 = j % 4 == 0 ? w0.x : j % 4 == 1 ? w0.y : j % 4 == 2 ? w0.z : w0.w;
      const uint32_t d1 = j % 4 == 0 ? w1.x : j % 4 == 1 ? w1.y : j % 4 == 2 ? w1.z : w1.w;
      const half8 A = codes_f16(d0, d1, vr);
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        o[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, ph8[t], o[t][j], 0, 0, 0);
        if (PAIR) o[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, pl8[t], o[t][j], 0, 0, 0);
      }
    }
    if (MORE) load_v<D>(c, at.ph, (at.pos >> 5) & 1, lane, x.v);
  };
  // (positions increase, so the steps at the edge are the last ones; vmin <= len)
  if (at.ok) {
    for (advance(); at.ok && p0 + 32 <= vmin; advance()) step(std::false_type{}, std::true_type{});
    for (; at.ok; advance()) step(std::true_type{}, std::true_type{});
    step(std::true_type{}, std::false_type{});
  }
  const float unit = ldexpf(1.f, vref);
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l[t] += __shfl_xor(l[t], 16, 64);
    l[t] += __shfl_xor(l[t], 32, 64);
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[t][j] *= unit;
  }

  const int live = min(ncols - col0, CT);
  if (g == 0)
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      sm[wave][16 * t + i] = m[t];
      sl[wave][16 * t + i] = l[t];
    }
  __syncthreads();
  auto put = [&](int slot) {
#pragma unroll
    for (int t = 0; t < QT; ++t)
      if (16 * t + i < live)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < NJ; j += 4)
            *(f32x4*)&so[(slot * CT + 16 * t + i) * LD + j * 16 + (4 * g + r) * 4] =
                f32x4{o[t][j][r], o[t][j + 1][r], o[t][j + 2][r], o[t][j + 3][r]};
  };
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, sm[w][16 * t + i]);
    const float f = m[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[t] - M);
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[t][j] *= f;
  }
  if (SLOTS == 4) {
    put(wave);
  } else {
    if (wave >= 2) put(wave - 2);
    __syncthreads();
    if (wave < 2)
#pragma unroll
      for (int t = 0; t < QT; ++t)
        if (16 * t + i < live)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < NJ; ++j) o[t][j][r] += so[(wave * CT + 16 * t + i) * LD + j / 4 * 64 + (4 * g + r) * 4 + j % 4];
    // each of the two waves writes where it alone has read
    if (wave < 2) put(wave);
  }
  __syncthreads();
  for (int k = tid; k < live * (D / 4); k += 256) {
    const int cc = k / (D / 4), ch = k % (D / 4) * 4;
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, sm[w][cc]);
#pragma unroll
    for (int w = 0; w < 4; ++w) L += sm[w][cc] == -INFINITY ? 0.f : sl[w][cc] * __builtin_amdgcn_exp2f(sm[w][cc] - M);
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < SLOTS; ++w) y += *(const f32x4*)&so[(w * CT + cc) * LD + ch];
    const int col = col0 + cc, tok = sg.t0 + col / G, head = h * G + col % G;
    if (a.splits == 1) {
      const float inv = L == 0.f ? 0.f : 1.f / L;
      const float z[4] = {y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
      store_row<4>(a.o, (int64_t)tok * a.ldo + (int64_t)head * D + ch, a.odt, a.alo, z, a.olo);
    } else {
      float* p = a.part + (((size_t)tok * (c.H * G) + head) * a.splits + split) * LD;
      *(f32x4*)(p + ch) = y;
      if (ch == 0) {
        p[D] = M;
        p[D + 1] = L;
      }
    }
  }
}

// Many columns: each of the workgroup's four waves has 32 of its own, and all walk the same steps.  One 32x32x16
// product takes 32 positions (or channels) by 32 columns:
//   lane l = 32 f + i:  A row i, B column i, k slots 8 f .. 8 f + 7,  C column i, rows 8 (r / 4) + 4 f + r % 4
//   S^T: A row i = position i, k slots of step s = channels f D/2 + 8 s ..
//   O^T tile j: A row i = channel i D/32 + j; of half u of the positions, k slots = positions 16 u + 4 f .. + 3 and
//     16 u + 8 + 4 f .. + 3: two dwords of the value page, and scores 8 u .. 8 u + 7 of the lane
// so a lane has one column, and half the instructions around the products of the 16-column kernel.
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int D, bool PAIR>
__global__ __launch_bounds__(256, 2) void k_qcache_attend_wide(AttendArgs a) {
  constexpr int NS = D / 16, NJ = D / 32, LD = D + 4;
  constexpr float SLACK = slack_of(PAIR), LIFT = lift_of(PAIR);
  const QCache& c = a.c;
  int id = blockIdx.x, pair;
  const int x = id & 7;
  if (a.by_xcd) id >>= 3;
  const int split = id % a.splits;
  id /= a.splits;
  if (a.by_xcd) {
    // Blocks go to the 8 XCDs in turn; those of one (segment, head) pair follow each other on one XCD and
    // read the same pages through its L2.  The tiles with the most positions go first.
    pair = id / a.tiles * 8 + x;
    id %= a.tiles;
  } else {
    pair = id % (a.sg.n_seg * c.H);
    id /= a.sg.n_seg * c.H;
  }
  if (pair >= a.sg.n_seg * c.H) return;
  const int h = pair % c.H, tile = a.tiles - 1 - id;
  const Seg sg = seg_of(a.sg, pair / c.H, c.rows, c.ppr * PG);
  const int G = a.G, ncols = sg.n * G;
  const int lane = threadIdx.x & 63, i = lane & 31, f = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col0 = tile * 128 + wave * 32;
  if (col0 >= ncols) return;
  const int vmin = max(sg.p0 + col0 / G + 1, 0);
  const int vmax = max(sg.p0 + (min(col0 + 32, ncols) - 1) / G + 1, 0);
  const int steps = (vmax + 31) / 32, begin = split * a.per;
  Walk<false> at{c, nullptr, sg.row, h, lane, begin, 1, split == a.splits - 1 ? steps : min(steps, begin + a.per), vmax};

  i32x4 kb[D / 32];
  uint32_t vb[4][NJ];  // of quads f, 2 + f, 4 + f and 6 + f
  __shared__ __align__(16) char turn[4 * 32 * D];
  char* keys = turn + wave * (32 * D);
  auto load_keys = [&] { load_k<D>(c, at.ph, (at.pos >> 5) & 1, lane, kb); };
  auto load_values = [&] {
    const uint8_t* p = c.v + (at.ph * (PG * D) + ((at.pos >> 5) & 1) * (32 * D));
    const uint32_t first = f * (4u * D) + i * (4u * NJ);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (NJ == 4) *(uint4*)vb[e] = *(const uint4*)(p + first + e * 8 * D);
      else *(uint2*)vb[e] = *(const uint2*)(p + first + e * 8 * D);
    }
  };
  at.fill();
  at.find();
  if (at.ok) {
    load_keys();
    load_values();
  }
  at.settle();
  at.scales();

  // the query, scaled by a power of two so that its largest element is in [2^10, 2^11)
  const int col = col0 + i;
  const bool live = col < ncols;
  const int tok = sg.t0 + (live ? col / G : 0), head = h * G + (live ? col % G : 0);
  const int vis = live ? sg.p0 + col / G + 1 : 0;
  half8 qh[NS], ql[PAIR ? NS : 1];
  float cq;
  {
    float y[NS][8], top = 0.f;
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      if (live) load8(a.q, (int64_t)tok * a.ldq + (int64_t)head * D + f * (D / 2) + k * 8, a.dt, a.alq, y[k]);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) y[k][e] = 0.f;
    }
    if (a.rope) {
      const float2* tab = a.rope + (size_t)min(max(vis - 1, 0), c.ppr * PG - 1) * (D / 2);
#pragma unroll
      for (int k = 0; k < NS; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float other = __shfl_xor(y[k][e], 32, 64);
          const float2 cs = tab[k * 8 + e];
          float lo, hi;
          rope_pair(f ? other : y[k][e], f ? y[k][e] : other, cs.x, cs.y, lo, hi);
          y[k][e] = f ? hi : lo;
        }
    }
#pragma unroll
    for (int k = 0; k < NS; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(y[k][e]));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    int ex;
    frexpf(top, &ex);
    if (!(top > 0.f)) ex = 0;
    cq = ldexpf(a.scale * QC_LOG2E, ex - 11);
#pragma unroll
    for (int k = 0; k < NS; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float z = ldexpf(y[k][e], 11 - ex);
        qh[k][e] = (f16)z;
        if (PAIR) ql[k][e] = (f16)(z - (float)qh[k][e]);
      }
    if (top == INFINITY) qh[0][0] = (f16)NAN;
  }

  f32x16 o[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[j][r] = 0.f;
  float m = -INFINITY, l = 0.f;
  bool far = false;  // a column's reference is beyond +-2^18
  int vref = 0;  // o is in units of 2^vref
  bool first = true;
  int p0 = 0;
  float ks = 0.f, vs = 0.f;
  auto advance = [&] {
    p0 = at.pos;
    ks = at.ks;
    vs = at.vs;
    at.next();
  };
  auto step = [&](auto edge_tag, auto more_tag) {  // as above
    constexpr bool EDGE = decltype(edge_tag)::value, MORE = decltype(more_tag)::value;
    const float cs = fmaxf(cq * ks, 1e-37f);  // (not 0: -inf stays -inf)
    const int ve = exponent_of(vs);
    turn_k<D>(kb, keys, lane);
    if (MORE) load_keys();
    f32x16 sc;
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      const i32x4 w = *(const i32x4*)(keys + k_slot<D>(i, f * (D / 32) + k / 2));
      const half8 A = k & 1 ? codes_f16(w[2], w[3], 1.f) : codes_f16(w[0], w[1], 1.f);
      sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(A, qh[k], sc, 0, 0, 0);
      if (PAIR) sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(A, ql[k], sc, 0, 0, 0);
    }
    if (first) vref = ve;
    first = false;
    float fall = 1.f;  // o to another unit where the page's scale is far from it
    if (ve - vref > 4 || ve - vref < -6) {
      fall = ldexpf(1.f, vref - ve);
      vref = ve;
    }
    const float vr = ldexpf(1.f, ve - vref);
    float top = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if (EDGE && p0 + 8 * (r / 4) + 4 * f + r % 4 >= vis) sc[r] = -INFINITY;
      top = fmaxf(top, sc[r]);
    }
    top *= cs;
    if (__any(top - m > SLACK + LIFT) || fall != 1.f) {
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float nm = top - m > SLACK + LIFT ? reference_of<PAIR>(top) : m;
      const float al = nm == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - nm);
      l *= al;
#pragma unroll
      for (int j = 0; j < NJ; ++j) o[j] *= al * fall;
      m = nm;
      far = __any(m > -INFINITY && fabsf(m) > 0x1p18f);
    }
    const float base = m == -INFINITY ? 0.f : m;
    // (the product rounded by itself only where it matters: 300 us in every step, 293 with the fused form, for eight
    // prefixes of 1,500 to 2,048 tokens, 8 x 4 heads of 128)
    if (far) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = mul_rounded(sc[r], cs);
    }
    const float slope = far ? 1.f : cs;
    half8 ph8[2], pl8[PAIR ? 2 : 1];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float p = __builtin_amdgcn_exp2f(fmaf(sc[r], slope, -base));
      ph8[r / 8][r % 8] = (f16)p;
      if (PAIR) {
        pl8[r / 8][r % 8] = (f16)(p - (float)ph8[r / 8][r % 8]);
        l += p;
      }
    }
    if (!PAIR) l = sum_of(ph8[1], sum_of(ph8[0], l));
    if (EDGE) {  // codes behind the row's last position may be anything
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int left = min(max(sg.len - (p0 + 8 * e + 4 * f), 0), 4);
        const uint32_t keep = left == 4 ? 0xFFFFFFFFu : (1u << (8 * left)) - 1u;
#pragma unroll
        for (int j = 0; j < NJ; ++j) vb[e][j] &= keep;
      }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const half8 A = codes_f16(vb[2 * u][j], vb[2 * u + 1][j], vr);
        o[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(A, ph8[u], o[j], 0, 0, 0);
        if (PAIR) o[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(A, pl8[u], o[j], 0, 0, 0);
      }
    if (MORE) load_values();
  };
  if (at.ok) {
    for (advance(); at.ok && p0 + 32 <= vmin; advance()) step(std::false_type{}, std::true_type{});
    for (; at.ok; advance()) step(std::true_type{}, std::true_type{});
    step(std::true_type{}, std::false_type{});
  }
  l += __shfl_xor(l, 32, 64);
  if (!live) return;
  const float out = a.splits > 1 ? ldexpf(1.f, vref) : l == 0.f ? 0.f : ldexpf(1.f, vref) / l;
  float* part = a.part + (((size_t)tok * (c.H * G) + head) * a.splits + split) * LD;
#pragma unroll
  for (int r = 0; r < 16; r += 2) {  // two rows' channels follow each other
    const int ch = (8 * (r / 4) + 4 * f + r % 4) * NJ;
    float z[2 * NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      z[j] = o[j][r] * out;
      z[NJ + j] = o[j][r + 1] * out;
    }
    if (a.splits == 1) {
      store_row<2 * NJ>(a.o, (int64_t)tok * a.ldo + (int64_t)head * D + ch, a.odt, a.alo, z, a.olo);
    } else {
#pragma unroll
      for (int e = 0; e < 2 * NJ; e += 4) *(f32x4*)(part + ch + e) = f32x4{z[e], z[e + 1], z[e + 2], z[e + 3]};
    }
  }
  if (a.splits > 1 && f == 0) {
    part[D] = m;
    part[D + 1] = l;
  }
}

// Joins the splits of each (token, head): a wave each, in split order.  (4 rows of 32 heads in about 16 splits: 7 us,
// all launch and round trips.)
template <int D>
__global__ __launch_bounds__(256) void k_qcache_join(AttendArgs a) {
  constexpr int LD = D + 4, E = D / 64;
  const int heads = a.c.H * a.G, lane = threadIdx.x & 63;
  const int item = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int head = item % heads, rest = item / heads, tokn = rest % a.sg.max_new, s = rest / a.sg.max_new;
  if (s >= a.sg.n_seg) return;
  const Seg sg = seg_of(a.sg, __builtin_amdgcn_readfirstlane(s), a.c.rows, a.c.ppr * PG);
  if (tokn >= sg.n) return;
  const int tok = sg.t0 + tokn;
  const float* p = a.part + ((size_t)tok * heads + head) * a.splits * LD;
  int splits = a.splits;
  if (a.even) {
    const int per = even_steps(a, lane);
    splits = (steps_of(a, s) + per - 1) / per;
  }
  // The first splits' sums are on their way before their factors are known: a launch of this size is all
  // latency.  Lane k holds the factor of split k0 + k.
  constexpr int PRE = 16;
  float pre[PRE][E];
#pragma unroll
  for (int k = 0; k < PRE; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) pre[k][e] = p[(size_t)max(min(k, splits - 1), 0) * LD + lane * E + e];
  float M = -INFINITY, L = 0.f, y[E];
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = 0.f;
  for (int k = lane; k < splits; k += 64) M = fmaxf(M, p[(size_t)k * LD + D]);
  M = wave_max(M);
  auto factor = [](float f, int k) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), k)); };
  for (int k0 = 0; k0 < splits; k0 += 64) {
    float f = 0.f, l = 0.f;
    if (k0 + lane < splits) {
      const float* q = p + (size_t)(k0 + lane) * LD + D;
      f = q[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(q[0] - M);
      l = q[0] == -INFINITY ? 0.f : q[1] * f;
    }
    L += wave_sum(l);
    const int n = min(splits - k0, 64);
    const float* q = p + (size_t)k0 * LD + lane * E;
    if (k0 == 0)
#pragma unroll
      for (int k = 0; k < PRE; ++k)  // (the factor of a split that is not there is 0, its sums are another's)
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] += k < n ? pre[k][e] * factor(f, k) : 0.f;
#pragma unroll 8
    for (int k = k0 == 0 ? PRE : 0; k < n; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = fmaf(q[(size_t)k * LD + e], factor(f, k), y[e]);
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int64_t at = (int64_t)tok * a.ldo + (int64_t)head * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float z = y[e] * inv;
    if (a.odt == DT_F32) ((float*)a.o)[at + e] = z;
    else if (a.odt == DT_BF16) ((uint16_t*)a.o)[at + e] = (uint16_t)to_bf16(z);
    else {
      const uint16_t w = (uint16_t)to_f16(z);
      ((uint16_t*)a.o)[at + e] = w;
      if (a.olo) a.olo[at + e] = sat16(z - (float)__builtin_bit_cast(f16, w));
    }
  }
}

// ---------------------------------------------------------------------------
// Selection.  A workgroup per KV head and token, or 16 / G of a row's tokens (they read the same bounds).  The score of
// a page is an upper bound of q . k over its keys, from each channel's largest and smallest key, in whole numbers
// (|q^| <= 127 times bounds of at most 112, 128 channels: below 2^21), so it has the same bits in any order of
// summation:
//   2^ke max over heads of sum_d max(q^_d, 0) hi_d + min(q^_d, 0) lo_d
// as one 8-bit product of [q^+ | q^-] (a head per row) with the bounds [hi | lo] (a page per column).
// Then the n_sel best, ties to the lower page: a wave finds the key of rank n_sel bit by bit; 257 to 1,024 pages of a
// single token by eight waves, three bits a round; more than 1,024 by four 8-bit digits.
// Measured (8 KV heads of 128): 8 tokens over 470 to 1,024 pages 19 us, 192 tokens over 125 to 256 pages 13 us, one
// over 63 pages 6.8 us: page table, bounds and ranking wait for each other, on as many CUs as there are tokens and
// heads (of the 19: 12 for the scores, 0.25 MB a workgroup, and 3 for the ranking).

struct SelectArgs {
  QCache c;
  QSegs sg;
  const void* q;
  int64_t ldq;
  int dt, alq, G, n_sel, toks;  // toks: tokens of a row that a workgroup takes
  const float2* rope;
  int32_t* sel;
};

constexpr int SEL_OUT = 0;  // the key of a page that cannot be chosen; every other key is larger

// Writes the indexes of the keys above T in order, with the first of those equal to it that make them n_sel.
template <int N>
__device__ __forceinline__ void take_above(const uint32_t (&k)[N], uint32_t T, int n_sel, int lane, int32_t* out) {
  int count = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) count += (int)__popcll(__ballot(k[j] > T));
  int need = T == (uint32_t)SEL_OUT ? 0 : n_sel - count, at = 0;  // how many of T itself
  const uint64_t below = (1ull << lane) - 1ull;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const uint64_t same = __ballot(k[j] == T);
    const bool take = k[j] > T || (k[j] == T && (int)__popcll(same & below) < need);
    const uint64_t taken = __ballot(take);
    if (take) out[at + (int)__popcll(taken & below)] = j * 64 + lane;
    at += (int)__popcll(taken);
    need -= min(need, (int)__popcll(same));
  }
  for (int p = at + lane; p < n_sel; p += 64) out[p] = -1;
}

// The n_sel best of np <= 64 N keys by one wave, N keys to a lane: the key of rank n_sel bit by bit, counts in the
// scalar unit.
template <int N>
__device__ __forceinline__ void select_wave(const uint32_t* key, int np, int n_sel, int lane, int32_t* out) {
  uint32_t k[N], T = 0u;
#pragma unroll
  for (int j = 0; j < N; ++j) k[j] = j * 64 + lane < np ? key[j * 64 + lane] : 0u;
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t t = T | 1u << bit;
    int n = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) n += (int)__popcll(__ballot(k[j] >= t));
    if (n >= n_sel) T = t;
    if (n == n_sel) break;
  }
  take_above<N>(k, T, n_sel, lane, out);
}

// Every page in view of a token that sees n_sel or fewer: the ones in the pool, in order.
__device__ __forceinline__ void select_all(const QCache& c, int row, int np, int n_sel, int lane, int32_t* out) {
  int at = 0;
  for (int p0 = 0; p0 < np; p0 += 64) {
    const int p = p0 + lane;
    const bool ok = p < np && (unsigned)c.pt[(size_t)row * c.ppr + p] < (unsigned)c.n_pages;
    const uint64_t b = __ballot(ok);
    if (ok) out[at + (int)__popcll(b & ((1ull << lane) - 1ull))] = p;
    at += (int)__popcll(b);
  }
  for (int p = at + lane; p < n_sel; p += 64) out[p] = -1;
}

template <int D, int NT>
__global__ __launch_bounds__(NT) void k_qcache_select(SelectArgs a) {
  // U groups of 16 pages at a time: a wave waits twice (page table, bounds) for all of them
  constexpr int NW = NT / 64, NB = 2 * D / 64, U = 4;
  extern __shared__ uint32_t key[];  // [tokens][ppr]
  __shared__ uint32_t hist[256];
  __shared__ uint32_t pick[2];
  __shared__ uint32_t wsum[2][NW];
  __shared__ i32x4 turn[NW][NB * 64];
  const QCache& c = a.c;
  int id = blockIdx.x;
  const int h = id % c.H;
  id /= c.H;
  const int per_row = (a.sg.max_new + a.toks - 1) / a.toks;
  const int tok0 = id % per_row * a.toks, s = id / per_row;
  const Seg sg = seg_of(a.sg, s, c.rows, c.ppr * PG);
  if (tok0 >= sg.n) return;
  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // nt tokens; token t sees `vis_of(t)` positions on `pages_of(t)` pages, the last one the most
  const int nt = min(a.toks, sg.n - tok0), G = a.G;
  auto vis_of = [&](int t) { return max(sg.p0 + tok0 + t + 1, 0); };
  auto pages_of = [&](int t) { return (vis_of(t) + PG - 1) / PG; };
  auto out_of = [&](int t) { return a.sel + ((size_t)(sg.t0 + tok0 + t) * c.H + h) * a.n_sel; };
  const int np = pages_of(nt - 1);

  if (np > a.n_sel) {
    constexpr int PC = D / 8;  // 16-byte pieces of a page's bounds
    int page[U];
    float ks[U];
    i32x4 bound[U][NB];
    auto fetch = [&](int p0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        page[u] = c.pt[(size_t)sg.row * c.ppr + min(p0 + u * NW * 16 + i, np - 1)];
        page[u] = (unsigned)page[u] < (unsigned)c.n_pages ? page[u] : -1;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        ks[u] = c.ks[(size_t)max(page[u], 0) * c.H + h];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const size_t ph = (size_t)max(__shfl(page[u], n * (64 / PC) + lane / PC, 64), 0) * c.H + h;
          bound[u][n] = *((const i32x4*)(c.kb + ph * (2 * D)) + lane % PC);
        }
      }
    };
    // 16 pages' bounds were loaded as they lie, and are turned in LDS to a page to a lane, as the attention's keys are
    // (8 tokens over 470 to 1,024 pages, the whole call: 43.2 -> 41.1 us)
    auto turned = [&](int u) {
      i32x4* t = turn[wave];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int row = n * (64 / PC) + lane / PC;
        t[row * PC + (lane % PC ^ (row & 7))] = bound[u][n];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int n = 0; n < NB; ++n) bound[u][n] = t[i * PC + ((4 * n + g) ^ (i & 7))];
    };
    fetch(wave * 16);  // (on their way while the queries are)
    // Row i of the products: one token's head c0 + i, or, of several tokens, head i % G of token i / G.  Lane (i, g)
    // reads its channels 64 b + 16 g .. of each block b of 64 (all waves the same).
    const int rt = a.toks == 1 ? 0 : i / G;
    const bool live = rt < nt;
    const int vis = live ? vis_of(rt) : 0;
    auto load16 = [&](int col, int b, float* x) {
      const int64_t at = (int64_t)(sg.t0 + tok0 + rt) * a.ldq + (int64_t)(h * G + col) * D + (64 * b + 16 * g) % D;
      load8(a.q, at, a.dt, a.alq, x);
      load8(a.q, at + 8, a.dt, a.alq, x + 8);
      if (a.rope) {
        const int d0 = (64 * b + 16 * g) % D;
        const bool low = d0 < D / 2;
        float y[16];
        load8(a.q, at + (low ? D / 2 : -D / 2), a.dt, a.alq, y);
        load8(a.q, at + (low ? D / 2 : -D / 2) + 8, a.dt, a.alq, y + 8);
        const float2* tab = a.rope + (size_t)min(max(vis - 1, 0), c.ppr * PG - 1) * (D / 2) + d0 % (D / 2);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float lo, hi;
          rope_pair(low ? x[e] : y[e], low ? y[e] : x[e], tab[e].x, tab[e].y, lo, hi);
          x[e] = low ? lo : hi;
        }
      }
    };
    const int first_col = a.toks == 1 ? i : i % G;
    // the largest |q| of the group's heads
    float m = 0.f;
    if (live)
      for (int col = first_col; col < G; col += 16)
#pragma unroll
        for (int b = 0; b < D / 64; ++b) {
          float x[16];
          load16(col, b, x);
#pragma unroll
          for (int e = 0; e < 16; ++e) m = fmaxf(m, fabsf(x[e]));
        }
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    for (int o = 1; o < (a.toks == 1 ? 16 : G); o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    int ex;
    frexpf(m, &ex);
    const bool flat = !(m > 0.f) || m == INFINITY;  // nothing to rank by: every score 0
    for (int c0 = 0; c0 < G; c0 += 16) {
      const int col = c0 + first_col;
      i32x4 A[NB];
#pragma unroll
      for (int b = 0; b < D / 64; ++b) {
        float x[16];
        if (live && col < G && !flat) load16(col, b, x);
        else
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] = 0.f;
        i32x4 up = {0, 0, 0, 0}, dn = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float f = x[e] == x[e] ? rintf(ldexpf(x[e], 7 - ex)) : 0.f;
          const int v = (int)fminf(fmaxf(f, -127.f), 127.f);
          up[e / 4] |= (max(v, 0) & 255) << (8 * (e % 4));
          dn[e / 4] |= (min(v, 0) & 255) << (8 * (e % 4));
        }
        A[b] = up;
        A[b + D / 64] = dn;
      }
      for (int p0 = wave * 16; p0 < np; p0 += NW * 16 * U) {
        if (c0 > 0 || p0 != wave * 16) fetch(p0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          turned(u);
          i32x4 acc = {0, 0, 0, 0};
#pragma unroll
          for (int n = 0; n < NB; ++n) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(A[n], bound[u][n], acc, 0, 0, 0);
          const int lp = p0 + u * NW * 16 + i;  // the lane's page; its rows are 4 g + r
          auto put = [&](int t, int v) {
            if (t >= nt || lp >= np) return;
            uint32_t k = __float_as_uint((float)v * ks[u]);
            k = k & 0x80000000u ? ~k : k | 0x80000000u;
            if (lp == pages_of(t) - 1) k = 0xFFFFFFFFu;
            if (page[u] < 0) k = SEL_OUT;
            uint32_t* at = key + (size_t)t * c.ppr + lp;
            *at = c0 ? max(*at, k) : k;
          };
          if (a.toks == 1) {
            int v = INT_MIN;
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (c0 + 4 * g + r < G) v = max(v, acc[r]);
            v = max(v, __shfl_xor(v, 16, 64));
            v = max(v, __shfl_xor(v, 32, 64));
            if (g == 0) put(0, v);
          } else if (G == 1) {
#pragma unroll
            for (int r = 0; r < 4; ++r) put(4 * g + r, acc[r]);
          } else if (G == 2) {
            put(2 * g, max(acc[0], acc[1]));
            put(2 * g + 1, max(acc[2], acc[3]));
          } else {
            int v = max(max(acc[0], acc[1]), max(acc[2], acc[3]));
            if (G == 8) v = max(v, __shfl_xor(v, 16, 64));
            if (G == 4 || (g & 1) == 0) put(4 * g / G, v);
          }
        }
      }
    }
    __syncthreads();
    if (NW == 8 && nt == 1 && np > 256 && np <= 1024) {
      // A workgroup with one token: all keys in every wave, 16 to a lane, and each wave counts for a threshold of its
      // own, three bits a round instead of one (64 of 1,024 pages, the whole call: 45.2 -> 43.0 us).
      uint32_t k[16], T = 0u;
#pragma unroll
      for (int j = 0; j < 16; ++j) k[j] = j * 64 + lane < np ? key[j * 64 + lane] : 0u;
      for (int shift = 30; shift >= 0; shift -= 3) {
        const uint32_t t = T + ((uint32_t)(wave + 1) << shift);
        int n = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) n += (int)__popcll(__ballot(k[j] >= t));
        const bool over = wave == 7 || (shift == 30 && wave >= 3);  // no such digit (the first round has two bits)
        if (lane == 0) hist[(shift & 1) * 8 + wave] = over ? 0u : (uint32_t)n;
        __syncthreads();
        const uint32_t cnt = hist[(shift & 1) * 8 + (lane & 7)];
        const int digit = (int)__popcll(__ballot(lane < 8 && cnt >= (uint32_t)a.n_sel));
        T += (uint32_t)digit << shift;
        if (__ballot(lane < 8 && lane == digit - 1 && cnt == (uint32_t)a.n_sel)) break;
      }
      if (wave == 0) take_above<16>(k, T, a.n_sel, lane, out_of(0));
      return;
    }
    if (c.ppr <= 1024) {
      for (int t = wave; t < nt; t += NW) {
        const int n = pages_of(t);
        const uint32_t* k = key + (size_t)t * c.ppr;
        if (n <= a.n_sel) select_all(c, sg.row, n, a.n_sel, lane, out_of(t));
        else if (n <= 64) select_wave<1>(k, n, a.n_sel, lane, out_of(t));
        else if (n <= 256) select_wave<4>(k, n, a.n_sel, lane, out_of(t));
        else select_wave<16>(k, n, a.n_sel, lane, out_of(t));
      }
      return;
    }
    int32_t* out = out_of(0);  // (one token)
    // the key of rank n_sel: digit by digit, `need` of the keys with the digits so far are wanted
    uint32_t prefix = 0u, need = a.n_sel;
    for (int d = 24; d >= 0; d -= 8) {
      for (int b = tid; b < 256; b += NT) hist[b] = 0u;
      __syncthreads();
      for (int p = tid; p < np; p += NT) {
        const uint32_t u = key[p];
        if (d == 24 || (u >> (d + 8)) == (prefix >> (d + 8))) atomicAdd(&hist[(u >> d) & 255u], 1u);
      }
      __syncthreads();
      if (wave == 0) {  // lane l: digits 255 - 4 l .. 252 - 4 l; the sums from the top down
        uint32_t n[4], t = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          n[e] = hist[255 - 4 * lane - e];
          t += n[e];
        }
        uint32_t above = t;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const uint32_t y = __shfl_up(above, o, 64);
          if (lane >= o) above += y;
        }
        above -= t;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (above < need && need <= above + n[e]) {
            pick[0] = prefix | (uint32_t)(255 - 4 * lane - e) << d;
            pick[1] = need - above;
          }
          above += n[e];
        }
      }
      __syncthreads();
      prefix = pick[0];
      need = pick[1];
    }
    // a thread takes consecutive pages: counts of larger and of equal keys, then their places in order
    const int each = (np + NT - 1) / NT, b0 = min(tid * each, np), b1 = min(b0 + each, np);
    uint32_t more = 0u, same = 0u;
    for (int p = b0; p < b1; ++p) {
      more += key[p] > prefix;
      same += key[p] == prefix;
    }
    uint32_t im = more, is = same;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(im, o, 64), z = __shfl_up(is, o, 64);
      if (lane >= o) {
        im += y;
        is += z;
      }
    }
    if (lane == 63) {
      wsum[0][wave] = im;
      wsum[1][wave] = is;
    }
    __syncthreads();
    uint32_t pm = im - more, ps = is - same;
    for (int w = 0; w < wave; ++w) {
      pm += wsum[0][w];
      ps += wsum[1][w];
    }
    const bool real = prefix != SEL_OUT;  // fewer pages than n_sel can be chosen otherwise
    for (int p = b0; p < b1; ++p) {
      const uint32_t u = key[p];
      const bool eq = u == prefix;
      if (u > prefix || (eq && real && ps < need)) out[pm + (real ? min(ps, need) : 0u)] = p;
      pm += u > prefix;
      ps += eq;
    }
    if (!real) {
      uint32_t total = 0u;
      for (int w = 0; w < NW; ++w) total += wsum[0][w];
      for (int p = (int)total + tid; p < a.n_sel; p += NT) out[p] = -1;
    }
    return;
  }
  for (int t = wave; t < nt; t += NW) select_all(c, sg.row, pages_of(t), a.n_sel, lane, out_of(t));
}

bool aligned16(const void* p, int64_t ld, int es) { return ((uintptr_t)p & 15) == 0 && (ld * es) % 16 == 0; }
int type_bytes(int dt) { return dt == DT_F32 ? 4 : 2; }

}  // namespace

hipError_t qcache_append(const QCache& c, const QSegs& sg, const void* k, int64_t ldk, const void* v,
                         int64_t ldv, int dt, const float2* rope, hipStream_t s) {
  AppendArgs a{c, sg, k, v, ldk, ldv, dt, aligned16(k, ldk, type_bytes(dt)), aligned16(v, ldv, type_bytes(dt)), 0, rope};
  const int max_new = sg.max_new;
  // n tokens touch at most (n + 62) / 64 + 1 pages
  a.chunks = (max_new + 62) / PG + 1;
  const unsigned grid = (unsigned)a.chunks * c.H * sg.n_seg;
  // A wave holds 512 / D tokens, one to a group of lanes; a page of 64 takes a quad to a group of lanes.
  const bool few = max_new <= 512 / c.dh;
  if (c.dh == 128) {
    if (few) k_qcache_append<128, 64, 1><<<grid, 64, 0, s>>>(a);
    else k_qcache_append<128, 256, 4><<<grid, 256, 0, s>>>(a);
  } else {
    if (few) k_qcache_append<64, 64, 1><<<grid, 64, 0, s>>>(a);
    else k_qcache_append<64, 128, 4><<<grid, 128, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <int D, bool PAIR>
static hipError_t attend_launch(const QAttendPlan& p, AttendArgs& a, hipStream_t s) {
  const unsigned pairs = (unsigned)a.sg.n_seg * a.c.H;
  const unsigned grid = p.even ? a.c.H * p.tiles * (p.splits + a.sg.n_seg)
                               : (a.by_xcd ? (pairs + 7) / 8 * 8 : pairs) * p.tiles * p.splits * (a.sel ? a.sg.max_new : 1);
  if (a.sel) k_qcache_attend<D, 1, PAIR, true><<<grid, 256, 0, s>>>(a);
  else if (!p.keys) k_qcache_attend_wide<D, PAIR><<<grid, 256, 0, s>>>(a);
  else if (p.qt == 1) k_qcache_attend<D, 1, PAIR, false><<<grid, 256, 0, s>>>(a);
  else k_qcache_attend<D, 2, PAIR, false><<<grid, 256, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const size_t items = (size_t)a.sg.n_seg * a.sg.max_new * a.c.H * a.G;
  k_qcache_join<D><<<(unsigned)((items + 3) / 4), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t qcache_attend(const QCache& c, const QSegs& sg, const QAttendPlan& p, int n_heads,
                         const void* q, int64_t ldq, int dt, bool pair, float scale, const float2* rope,
                         const int32_t* sel, int n_sel, void* o, int64_t ldo, int odt, void* olo, float* part,
                         hipStream_t s) {
  // Several workgroups that read the same pages share an L2 where that leaves no XCD idle: with a multiple of 8
  // pairs, or many.
  const int pairs = sg.n_seg * c.H;
  const bool shared = p.tiles > 1 || (sel && sg.max_new > 1);
  const int by_xcd = shared && (pairs % 8 == 0 || pairs >= 64);
  AttendArgs a{c, sg, q, ldq, o, ldo, (f16*)olo, dt, odt, aligned16(q, ldq, type_bytes(dt)),
               aligned16(o, ldo, type_bytes(odt)), n_heads / c.H, scale, rope, sel, n_sel, p.tiles, p.splits, p.per, by_xcd, p.even, part};
  if (c.dh == 128) return pair ? attend_launch<128, true>(p, a, s) : attend_launch<128, false>(p, a, s);
  return pair ? attend_launch<64, true>(p, a, s) : attend_launch<64, false>(p, a, s);
}

template <int D, int NT>
static hipError_t select_launch(const SelectArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)a.sg.n_seg * a.c.H * ((a.sg.max_new + a.toks - 1) / a.toks);
  const size_t lds = (size_t)a.toks * a.c.ppr * 4;
  // Above 64 KB with the kernel's own.  The limit is the widest table's in every call, so that none lowers another thread's.
  if (lds > 28 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)k_qcache_select<D, NT>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                       16384 * 4);
    if (e != hipSuccess) return e;
  }
  k_qcache_select<D, NT><<<grid, NT, lds, s>>>(a);
  return hipGetLastError();
}

hipError_t qcache_select(const QCache& c, const QSegs& sg, int n_heads, const void* q, int64_t ldq,
                         int dt, const float2* rope, int n_sel, int32_t* sel, hipStream_t s) {
  SelectArgs a{c, sg, q, ldq, dt, aligned16(q, ldq, type_bytes(dt)), n_heads / c.H, n_sel, 1, rope, sel};
  // the rows of one product hold the heads of several tokens where they divide it; their keys fit 48 KB of LDS
  if (a.G == 1 || a.G == 2 || a.G == 4 || a.G == 8)
    if (c.ppr <= 1024) a.toks = std::max(1, std::min({16 / a.G, 12288 / c.ppr, sg.max_new}));
  if (c.ppr <= 256) return c.dh == 128 ? select_launch<128, 256>(a, s) : select_launch<64, 256>(a, s);
  return c.dh == 128 ? select_launch<128, 512>(a, s) : select_launch<64, 512>(a, s);
}

}  // namespace ams
