// kv_rotate.cu -- queries, keys and values of new tokens on their way into the paged key-value cache
// (p2p_kv_write_rotated): norms of each head, rotary positions and the write, in one pass.
//
// For a head's row x of a token at position p: y = x * w / sqrt(mean x^2 + eps) where there are weights; then pair j of
// the rotated values, (y[j], y[j + rot / 2]) or (y[2 j], y[2 j + 1]), becomes amplitude * (a cos - b sin, a sin + b
// cos) of the angle p * f_j.  Everything in 32 bits, rounded once.
//
// The angle is held in turns: f_j comes as a fraction of a turn a position, in 64 bits after the point, and the product
// with p drops whole turns by overflowing: what is left is exact to p * 2^-64 of a turn, so a position of 2^31 - 1 is
// rotated as precisely as one of 1.  (In 32-bit floats an angle of 10^5 radians is off by 2^-8.)
//
// Bound by the bytes read and written, and nearly as much by issue slots: 61 prompts of 71,000 tokens with 64 / 8 heads
// of 128, normed, into 8 bits are 2.8 GB in 621 us on one GB300 (67% of the copy bandwidth, 56% of the issue slots; with
// the kinds of rows in one loop, and no rows on their way ahead, 1,052).  33 single tokens: 5.4 us, a launch and a chain
// of five loads.  A lane has two 16-byte pieces of a row, those that hold each other's partners, so that a row is four
// to sixteen lanes and no value crosses lanes but for the norm; a token's sines are the lane's for all its heads.
#include "kv_values.cuh"

namespace p2p {
namespace {

constexpr int kTurnThreads = 256, kTurnWarps = kTurnThreads / 32;
constexpr int kTurnTokens = 32;  // of a CTA at most: a warp finds their places

// A half-turn's fraction in [-1, 1) of a position's angle.
__device__ __forceinline__ float half_turns(uint64_t turns, int32_t pos) {
  const uint64_t x = turns * (uint32_t)pos + 0x80000000u;  // (rounded where it is cut)
  return (float)(int32_t)(x >> 32) * 0x1p-31f;
}
template <int KIND>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if (KIND == P2P_KV_BF16) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *(const uint32_t*)&x;
  }
  const __half2 x = __floats2half2_rn(a, b);
  return *(const uint32_t*)&x;
}
__device__ __forceinline__ float scale_of(const KvView& c, int32_t layer, int32_t head, bool value) {
  return (value ? c.v_scale : c.k_scale)[layer * c.heads + head];
}
// Row r of a token: queries first, then keys, then values.
struct TurnRow {
  int32_t kind, head;  // kind 0, 1, 2
};
__device__ __forceinline__ TurnRow turn_row(const KvView& c, const KvTurn& a, int32_t r) {
  if (r < a.heads) return {0, r};
  r -= a.heads;
  return r < c.heads ? TurnRow{1, r} : TurnRow{2, r - c.heads};
}

// x / scale rounded to 32 bits, and where that is a tie of 8 bits and the quotient is not, to its side of it (see
// divide_extreme); inverse: 1 / scale, positive and of an ordinary size.  (The product with the inverse, corrected once by
// its exact remainder: Markstein, Computation of Elementary Functions on the IBM RISC System/6000 Processor, 1990.)
__device__ __forceinline__ float divide(float x, float scale, float inverse) {
  const float z0 = x * inverse;
  float z = fmaf(fmaf(-z0, scale, x), inverse, z0);
  if (!(fabsf(z) < INFINITY)) z = z0;  // (infinities and NaN)
  int32_t b = __float_as_int(z);
  if ((b & 0x7ffff) == 0) {
    const float r = fmaf(-z, scale, x);
    if (r < 0.f || r > 0.f) b += (r < 0.f) == (x < 0.f) ? 1 : -1;
  }
  return __int_as_float(b);
}

// IN: the type of q, k and v; EIGHT: the cache holds 8 bits, else IN; NORMED: there are weights; PAIRS: interleaved.
// Rows lie on 16-byte boundaries and the rotated halves are whole pieces; log_lanes: of a row.  Queries, then keys,
// then values: what a kind's rows need stays in registers, and a batch of rows is read while the one before it is
// worked on.
template <int IN, bool EIGHT, bool NORMED, bool PAIRS>
__global__ void __launch_bounds__(kTurnThreads, 2)
    turn_kernel(KvView c, KvScratch s, KvTurn a, int32_t layer, int32_t n, const int32_t* seq, const int64_t* offsets,
                int64_t n_tokens, int32_t tokens, int32_t log_lanes, int32_t share) {
  constexpr int BATCH = 2;
  __shared__ int64_t place[kTurnTokens];
  __shared__ int32_t position[kTurnTokens];
  begin_kernel();
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x == 0 && blockIdx.y == 0) check_offsets(offsets, n, n_tokens, s.err);
  if (warp == 0) {
    int32_t pos;
    const int64_t at = place_of(c, s, n, seq, offsets, n_tokens, t0, *s.halt, pos);
    place[lane] = at, position[lane] = pos;
  }
  __syncthreads();
  // The lane's pieces, each eight values; -1: none.
  const int u = lane & ((1 << log_lanes) - 1), pieces = c.dim / 8, turned = a.rot / 16;
  int first = 2 * u, second = 2 * u + 1;
  if (!PAIRS && u < turned) first = u, second = u + turned;
  if (first >= pieces) first = -1;
  if (second >= pieces) second = -1;
  // pairs of the lane that are rotated
  const int mine = first < 0 || (!PAIRS && u >= turned) ? 0 : min(8, a.rot / 2 - 8 * u);
  const int step = 32 >> log_lanes, of_warp = lane >> log_lanes;
  const int32_t rows = a.heads + 2 * c.heads, begin = blockIdx.y * share, end = min(rows, begin + share);
  const float per_value = 1.f / c.dim;
#pragma unroll 1
  for (int32_t i = warp; i < tokens && t0 + i < n_tokens; i += kTurnWarps) {
    const int64_t at = place[i], t = t0 + i;
    if (at < 0) continue;
    float cs[8], sn[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      cs[j] = 1.f, sn[j] = 0.f;
      if (j < mine) {
        sincospif(half_turns(a.turns[8 * u + j], position[i]), &sn[j], &cs[j]);
        cs[j] *= a.amplitude, sn[j] *= a.amplitude;
      }
    }
#pragma unroll 1
    for (int kind = 0; kind < 3; ++kind) {
      const int32_t r_first = kind == 0 ? 0 : a.heads + (kind - 1) * c.heads, heads = kind == 0 ? a.heads : c.heads;
      const int32_t h0 = max(begin - r_first, 0), h1 = min(end - r_first, heads);
      if (h0 >= h1) continue;
      const uint16_t* const from = kind == 0 ? (const uint16_t*)a.q + t * a.q_token
          : (const uint16_t*)(kind == 1 ? a.k : a.v) + t * a.token;
      const int64_t apart = kind == 0 ? a.q_head : a.head;
      const float* const weight = !NORMED ? nullptr : kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr;
      float of_value[NORMED ? 16 : 1];
      if (NORMED && weight) {
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int piece = y < 2 ? first : second;
          const float4 f = piece >= 0 ? *(const float4*)(weight + piece * 8 + (y & 1) * 4)
              : make_float4(0.f, 0.f, 0.f, 0.f);
          of_value[4 * y] = f.x, of_value[4 * y + 1] = f.y, of_value[4 * y + 2] = f.z, of_value[4 * y + 3] = f.w;
        }
      }
      uint4 raw[BATCH][2];
      const auto read = [&](int32_t h) {
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
          const uint16_t* const p = from + (h + k * step + of_warp) * apart;
          const bool there = h + k * step + of_warp < h1;
          raw[k][0] = there && first >= 0 ? __ldcs((const uint4*)(p + first * 8)) : make_uint4(0, 0, 0, 0);
          raw[k][1] = there && second >= 0 ? __ldcs((const uint4*)(p + second * 8)) : make_uint4(0, 0, 0, 0);
        }
      };
      read(h0);
#pragma unroll 1
      for (int32_t h = h0; h < h1; h += BATCH * step) {
        uint4 now[BATCH][2];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) now[k][0] = raw[k][0], now[k][1] = raw[k][1];
        if (h + BATCH * step < h1) read(h + BATCH * step);
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
          const int32_t head = h + k * step + of_warp;
          const uint32_t in[8] = {now[k][0].x, now[k][0].y, now[k][0].z, now[k][0].w,
                                  now[k][1].x, now[k][1].y, now[k][1].z, now[k][1].w};
          float x[16];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 f = two_values<IN == P2P_KV_BF16>(in[j]);
            x[2 * j] = f.x, x[2 * j + 1] = f.y;
          }
          if (NORMED && weight) {
            float sum = 0.f, sum2 = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(x[j], x[j], sum), sum2 = fmaf(x[8 + j], x[8 + j], sum2);
            sum += sum2;
            for (int d = 1 << log_lanes >> 1; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
            const float by = rsqrtf(fmaf(sum, per_value, a.eps));
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] *= by * of_value[j];
          }
          if (head >= h1) continue;
          if (kind != 2 && mine > 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              // (what is not rotated is left as it is: 0 times an infinity would not be)
              if (j < mine) {
                constexpr int kStep = PAIRS ? 2 : 1, kApart = PAIRS ? 1 : 8;
                const float p = x[kStep * j], q = x[kStep * j + kApart];
                x[kStep * j] = p * cs[j] - q * sn[j];
                x[kStep * j + kApart] = p * sn[j] + q * cs[j];
              }
            }
          }
          if (EIGHT && kind != 0) {
            char* const to = (kind == 2 ? c.v : c.k) + (int64_t)layer * c.layer_stride + head * c.head_stride + at;
            const float scale = scale_of(c, layer, head, kind == 2), inverse = __frcp_rn(scale);
            const bool usual = scale > 0x1p-60f && scale < 0x1p60f;
            uint2 b[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              float z[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) z[j] = usual ? divide(x[8 * y + j], scale, inverse)
                  : divide_extreme(x[8 * y + j], scale);
              b[y].x = narrow(make_float2(z[0], z[1])) | narrow(make_float2(z[2], z[3])) << 16;
              b[y].y = narrow(make_float2(z[4], z[5])) | narrow(make_float2(z[6], z[7])) << 16;
            }
            if (first >= 0) __stcs((uint2*)(to + first * 8), b[0]);
            if (second >= 0) __stcs((uint2*)(to + second * 8), b[1]);
            continue;
          }
          uint4 v[2] = {now[k][0], now[k][1]};  // (values of 16 bits are stored as they are)
          if (kind != 2) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
              v[y] = make_uint4(pack16<IN>(x[8 * y], x[8 * y + 1]), pack16<IN>(x[8 * y + 2], x[8 * y + 3]),
                                pack16<IN>(x[8 * y + 4], x[8 * y + 5]), pack16<IN>(x[8 * y + 6], x[8 * y + 7]));
          }
          uint16_t* const to = kind == 0 ? (uint16_t*)a.out + t * a.out_token + head * a.out_head
                                         : (uint16_t*)((kind == 2 ? c.v : c.k) + (int64_t)layer * c.layer_stride +
                                             head * c.head_stride + at);
          if (first >= 0) __stcs((uint4*)(to + first * 8), v[0]);
          if (second >= 0) __stcs((uint4*)(to + second * 8), v[1]);
        }
      }
    }
  }
}

// The same for rows anywhere and any rotated values: a warp a row, a lane every 32nd pair.
template <int IN, bool EIGHT>
__global__ void __launch_bounds__(kTurnThreads)
    turn_any_kernel(KvView c, KvScratch s, KvTurn a, int32_t layer, int32_t n, const int32_t* seq,
                    const int64_t* offsets, int64_t n_tokens, int32_t tokens, int32_t share) {
  __shared__ int64_t place[kTurnTokens];
  __shared__ int32_t position[kTurnTokens];
  begin_kernel();
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x == 0 && blockIdx.y == 0) check_offsets(offsets, n, n_tokens, s.err);
  if (warp == 0) {
    int32_t pos;
    const int64_t at = place_of(c, s, n, seq, offsets, n_tokens, t0, *s.halt, pos);
    place[lane] = at, position[lane] = pos;
  }
  __syncthreads();
  const auto number = [](uint16_t b) {
    return IN == P2P_KV_BF16 ? __uint_as_float((uint32_t)b << 16) : __half2float(__ushort_as_half(b));
  };
  constexpr int kMost = 4;  // pairs of a lane: head_dim is at most 256
  const int32_t rows = a.heads + 2 * c.heads, r1 = min(rows, (int32_t)(blockIdx.y + 1) * share), half = a.rot / 2;
  for (int32_t i = warp; i < tokens && t0 + i < n_tokens; i += kTurnWarps) {
    const int64_t at = place[i], t = t0 + i;
    if (at < 0) continue;
    float cs[kMost], sn[kMost];
    int where[kMost][2];  // a pair's values
#pragma unroll
    for (int m = 0; m < kMost; ++m) {
      const int j = lane + 32 * m;
      const bool turned = j < half;
      where[m][0] = turned && !a.pairs ? j : 2 * j;
      where[m][1] = turned && !a.pairs ? j + half : 2 * j + 1;
      if (2 * j >= c.dim) where[m][0] = -1;
      cs[m] = 1.f, sn[m] = 0.f;
      if (turned) {
        sincospif(half_turns(a.turns[j], position[i]), &sn[m], &cs[m]);
        cs[m] *= a.amplitude, sn[m] *= a.amplitude;
      }
    }
    for (int32_t r = blockIdx.y * share; r < r1; ++r) {
      const TurnRow w = turn_row(c, a, r);
      const uint16_t* from = w.kind == 0 ? (const uint16_t*)a.q + t * a.q_token + w.head * a.q_head
                                         : (const uint16_t*)(w.kind == 1 ? a.k : a.v) + t * a.token + w.head * a.head;
      float x[kMost][2], sum = 0.f;
      uint16_t raw[kMost][2];
#pragma unroll
      for (int m = 0; m < kMost; ++m)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          raw[m][y] = where[m][0] >= 0 ? from[where[m][y]] : 0;
          x[m][y] = number(raw[m][y]);
          sum = fmaf(x[m][y], x[m][y], sum);
        }
#pragma unroll
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
      const float* weight = w.kind == 0 ? a.q_weight : w.kind == 1 ? a.k_weight : nullptr;
      const float by = weight ? rsqrtf(sum / c.dim + a.eps) : 1.f;
      char* to = (w.kind == 2 ? c.v : c.k) + (int64_t)layer * c.layer_stride + w.head * c.head_stride + at;
      uint16_t* out = w.kind == 0 ? (uint16_t*)a.out + t * a.out_token + w.head * a.out_head : (uint16_t*)to;
#pragma unroll
      for (int m = 0; m < kMost; ++m) {
        if (where[m][0] < 0) continue;
        float p = x[m][0], q = x[m][1];
        if (weight) p *= by * weight[where[m][0]], q *= by * weight[where[m][1]];
        if (w.kind != 2 && lane + 32 * m < half) {
          const float p1 = p * cs[m] - q * sn[m];
          q = p * sn[m] + q * cs[m];
          p = p1;
        }
        if (EIGHT && w.kind != 0) {
          const float scale = scale_of(c, layer, w.head, w.kind == 2);
          const uint32_t b = narrow(make_float2(divide_extreme(p, scale), divide_extreme(q, scale)));
          to[where[m][0]] = (char)b, to[where[m][1]] = (char)(b >> 8);
        } else {
          const uint32_t b = w.kind == 2 ? raw[m][0] | (uint32_t)raw[m][1] << 16 : pack16<IN>(p, q);
          out[where[m][0]] = (uint16_t)b, out[where[m][1]] = (uint16_t)(b >> 16);
        }
      }
    }
  }
}

template <int IN, bool EIGHT>
cudaError_t launch(const KvView& c, const KvScratch& s, const KvTurn& a, int32_t layer, int32_t n, const int32_t* seq,
                   const int64_t* offsets, int64_t n_tokens, bool wide, int num_sms, cudaStream_t st) {
  constexpr int kBatch = 2;  // (as in turn_kernel)
  int log_lanes = 0;
  while ((16 << log_lanes) < c.dim) ++log_lanes;
  const int32_t step = wide ? kBatch * (32 >> log_lanes) : 1;  // rows that a warp takes at a time
  const int32_t rows = a.heads + 2 * c.heads, steps = (rows + step - 1) / step;
  // A token's rows are one warp's where there are tokens enough for 16 warps an SM, else as many warps' as that takes.
  const int64_t want = 16LL * num_sms;
  const int32_t tokens = n_tokens >= 4 * want ? kTurnTokens : kTurnWarps;
  const int32_t parts = (int32_t)std::min<int64_t>(steps, std::max<int64_t>(1, want / n_tokens));
  const int32_t share = (steps + parts - 1) / parts * step;
  const dim3 grid((unsigned)((n_tokens + tokens - 1) / tokens), (unsigned)((rows + share - 1) / share));
  const bool normed = a.q_weight || a.k_weight;
  if (wide)
    return launch_early(a.pairs ? (normed ? turn_kernel<IN, EIGHT, true, true> : turn_kernel<IN, EIGHT, false, true>)
                                : (normed ? turn_kernel<IN, EIGHT, true, false> : turn_kernel<IN, EIGHT, false, false>),
                        grid, kTurnThreads, 0, st, c, s, a, layer, n, seq, offsets, n_tokens, tokens, log_lanes, share);
  return launch_early(turn_any_kernel<IN, EIGHT>, grid, kTurnThreads, 0, st, c, s, a, layer, n, seq, offsets, n_tokens,
                      tokens, share);
}

}  // namespace

cudaError_t launch_kv_turn(const KvView& c, const KvScratch& s, const KvTurn& a, int32_t layer, int32_t n,
                           const int32_t* seq, const int64_t* offsets, int64_t n_tokens, int num_sms, cudaStream_t st) {
  const auto on16 = [](const void* p, int64_t x, int64_t y) {
    return (uintptr_t)p % 16 == 0 && x % 8 == 0 && y % 8 == 0;
  };
  const bool wide = on16(a.q, a.q_token, a.q_head) && on16(a.out, a.out_token, a.out_head) &&
                    on16(a.k, a.token, a.head) && on16(a.v, a.token, a.head) &&
                    (!a.q_weight || (uintptr_t)a.q_weight % 16 == 0) &&
                        (!a.k_weight || (uintptr_t)a.k_weight % 16 == 0) &&
                    (a.pairs || a.rot % 16 == 0);
  const auto f = a.type == P2P_KV_BF16 ? (c.type == P2P_KV_E4M3 ? launch<P2P_KV_BF16, true> : launch<P2P_KV_BF16,
      false>)
                                       : (c.type == P2P_KV_E4M3 ? launch<P2P_KV_F16, true> : launch<P2P_KV_F16, false>);
  return f(c, s, a, layer, n, seq, offsets, n_tokens, wide, num_sms, st);
}

}  // namespace p2p
