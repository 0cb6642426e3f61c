// The paged cache written and read back (pkv_cache_append, pkv_cache_read), and
// the entry points of the serving calls.
//
// Both kernels move rows (one token, one head, K and V): a workgroup takes up to
// 128 consecutive tokens of the call's buffers and all heads.  It finds the
// tokens' places in the cache (sequence, position, page), one thread per
// token, and leaves them in LDS, the first rows already on their way; then groups
// of D/8 lanes (rounded up to a power of two) take one row each, 8 channels
// per lane, with neighbouring groups on neighbouring tokens of one head, so that the
// codes they store or load are one run of the head's tile.
//
// A row of 128 channels is 256 bytes in 16 bits against 68 in 4, read once and
// written once.  Reading back is bound by memory: 99485 rows of 8 heads of 128 from 4 bits
// take 106 us, 4.9 TB/s (a plain copy of 512 MiB: 5.2).  Appending is bound by the vector
// units, which are busy 79% of the time with ranges, roundings and packing: 87541
// rows of 8 heads into 4 bits take 126 us, 3.6 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pkv.h"
#include "pkv_internal.h"
#include "serve.h"

namespace pkv {
namespace {

constexpr int kThreads = 256;
constexpr int kMostTokens = 128;   // of a workgroup (rows of 16 channels: two lanes each)
constexpr int kStartsInLds = 1024; // sequences whose starts are searched in LDS

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float f16_float(uint32_t bits) {
  return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits)));
}
__device__ __forceinline__ uint32_t f16_bits(float f) {
  return __builtin_bit_cast(uint16_t, static_cast<_Float16>(f));
}

// Element e of 8 16-bit cache values.
template <bool BF16>
__device__ __forceinline__ float value(const u32x4& w, int e) {
  const uint32_t word = w[e >> 1];
  if constexpr (BF16) return __uint_as_float(e & 1 ? word & 0xFFFF0000u : word << 16);
  return f16_float(e & 1 ? word >> 16 : word);
}

template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  if constexpr (BF16) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
  } else {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
  }
}

// Where row i of the call lies: its slot in the cache (page * P + slot in the
// page), -1 where there is none, -2 for a row of no sequence.  `starts` is token_start, in LDS if it fits there.
__device__ __forceinline__ int64_t place_of(const ServeArgs& a, const int32_t* starts, int32_t i) {
  int32_t s = 0;
  for (int32_t end = a.num_seqs; end - s > 1;) {
    const int32_t mid = s + (end - s) / 2;
    if (starts[mid] <= i) s = mid; else end = mid;
  }
  const int32_t end = starts[s + 1] < a.num_tokens ? starts[s + 1] : a.num_tokens;
  if (i < starts[s] || i >= end) return -2;
  int64_t pos;
  if (a.positions) {
    pos = a.positions[i];
  } else {
    const int32_t len = a.kv_lens[s];
    pos = int64_t(len < a.max_kv ? len : a.max_kv) - (end - i);
  }
  const int64_t page_at = pos >> a.log2P;
  if (pos < 0 || page_at >= a.pages_per_seq) return -1;
  const int64_t page = a.page_table[int64_t(s) * a.pages_per_seq + page_at];
  if (page < 0 || page >= a.pool_pages) return -1;
  return (page << a.log2P) | (pos & ((int64_t(1) << a.log2P) - 1));
}

// Where a token's rows of head 0 lie: bytes from the layer's first key (code) and value (code), words from its first scale; k < 0
// as place_of.
struct Place {
  int64_t k, v, scale;
};

// The places of tokens [i0, i0 + n) into `place`, by the whole workgroup.
template <int KB, int VB>
__device__ __forceinline__ void find_places(const ServeArgs& a, int32_t i0, int32_t n, int32_t* starts, Place* place) {
  const int tid = threadIdx.x;
  const bool in_lds = a.num_seqs < kStartsInLds;
  if (in_lds)
    for (int32_t j = tid; j <= a.num_seqs; j += kThreads) starts[j] = a.token_start[j];
  __syncthreads();
  if (tid < n) {
    const int64_t at = in_lds ? place_of(a, starts, i0 + tid) : place_of(a, a.token_start, i0 + tid);
    Place p{at, at, at};
    if (at >= 0) {
      const int64_t page = at >> a.log2P, slot = at & ((int64_t(1) << a.log2P) - 1);
      if constexpr (KB == 16) {
        p.k = p.v = 2 * (page * a.page_stride + slot * a.H * a.D);
      } else {
        p.k = page * a.page_stride + slot * (a.D * KB / 8);
        p.v = page * a.page_stride + a.v_offset + slot * (a.D * VB / 8);
        p.scale = page * a.scale_stride + slot;
      }
    }
    place[tid] = p;
  }
  __syncthreads();
}

template <bool BF16>
__device__ __forceinline__ void piece_range(const u32x4& w, float& mn, float& mx) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = value<BF16>(w, e);
    mn = __builtin_fminf(mn, x);
    mx = __builtin_fmaxf(mx, x);
  }
}

// The plain instructions: rows are finite (the quantiser's contract), and fminf's care for signalling NaN takes two more.
__device__ __forceinline__ float least(float a, float b) {
  asm("v_min_f32 %0, %1, %2" : "=v"(a) : "v"(a), "v"(b));
  return a;
}
__device__ __forceinline__ float most(float a, float b) {
  asm("v_max_f32 %0, %1, %2" : "=v"(a) : "v"(a), "v"(b));
  return a;
}

// Minimum and maximum over the 2, 4, .. 64 lanes of a row, which lie next to each other: exchanges within quads, halves of
// 16 and 16 lanes by the operand path of the minimum itself, beyond by lane swaps.
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}
// (of K and of V)
template <int CTRL>
__device__ __forceinline__ void range_step(float (&mn)[2], float (&mx)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    mn[i] = least(mn[i], moved<CTRL>(mn[i]));
    mx[i] = most(mx[i], moved<CTRL>(mx[i]));
  }
}
__device__ __forceinline__ void row_range(float (&mn)[2], float (&mx)[2], int32_t lanes) {
  range_step<0xB1>(mn, mx);                  // quad_perm [1, 0, 3, 2]
  if (lanes > 2) range_step<0x4E>(mn, mx);   // quad_perm [2, 3, 0, 1]
  if (lanes > 4) range_step<0x141>(mn, mx);  // row_half_mirror
  if (lanes > 8) range_step<0x140>(mn, mx);  // row_mirror
  for (int off = 16; off < lanes; off <<= 1) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      mn[i] = least(mn[i], __shfl_xor(mn[i], off));
      mx[i] = most(mx[i], __shfl_xor(mx[i], off));
    }
  }
}

// Zero and scale of a row from its range.  The zero is exact in single precision.  The scale is the least binary16 s with s *
// (2^bits - 1) + zero >= max: the binary16 number at or next above the quotient, taken a little (2^-20) too
// small so that it is never past s, and the one after it if the condition does not hold yet.  The condition is decided
// exactly: the product has at most 19 bits, and its sum with zero is a pair of numbers, the rounded sum and its error.
struct RowQuant {
  float zero, inv, scale;
  uint32_t word;  // scale, then zero
};

// The sign of x - (a + b), exactly.
__device__ __forceinline__ int compare_sum(float x, float a, float b) {
  const float sum = a + b, back = sum - a, error = (a - (sum - back)) + (b - back);
  const float over = x - sum;  // (its sign is exact)
  return over > 0.0f ? 1 : over < 0.0f ? -1 : error < 0.0f ? 1 : error > 0.0f ? -1 : 0;
}

template <int BITS>
__device__ __forceinline__ RowQuant row_quant(float mn, float mx) {
  constexpr float kMost = float((1 << BITS) - 1);
  RowQuant q;
  mn += 0.0f;  // -0 counts as +0
  uint32_t z = f16_bits(mn);
  if (f16_float(z) > mn) z = z & 0x8000 ? z + 1 : z == 0 ? 0x8001u : z - 1;
  q.zero = f16_float(z);
  const float low = (mx - q.zero) * ((1.0f - 0x1p-20f) / kMost);
  uint32_t s = low > 0.0f ? f16_bits(low) : 0;
  if (f16_float(s) < low) ++s;
  if (compare_sum(mx, f16_float(s) * kMost, q.zero) > 0) ++s;
  q.scale = f16_float(s);
  q.inv = s ? __builtin_amdgcn_rcpf(q.scale) : 0.0f;
  q.word = s | (z << 16);
  return q;
}

// Codes of N values (8 of 4 bits or 4 of 8 bits) in one word.  t = (x - zero) * (1 / scale) is off the quotient by at most
// 2.4e-7 of it (roundings of 2^-24, 2^-23 and 2^-24), is rounded half to even by adding 1.5 * 2^23, in whose low bits
// the code then lies, and `far` keeps the largest distance of a t from its code: past 1/2 - kNear the rounding is in doubt.
constexpr float kRound = 12582912.0f;
template <int BITS>
constexpr float kNear = BITS == 4 ? 5e-6f : 8e-5f;

template <bool BF16, int BITS>
__device__ __forceinline__ uint32_t row_codes(const u32x4& w, int first, const RowQuant& q, float& far) {
  constexpr int N = 32 / BITS;
  uint32_t r[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float t = (value<BF16>(w, first + e) - q.zero) * q.inv, up = t + kRound;
    far = __builtin_fmaxf(far, __builtin_fabsf(t - (up - kRound)));
    r[e] = __float_as_uint(up);
  }
  // Low bytes together; of 4-bit codes the even channels' and the odd ones', which go between.
  auto bytes = [](uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u),
                                 0x05040100u);
  };
  if constexpr (BITS == 8) return bytes(r[0], r[1], r[2], r[3]);
  else return bytes(r[0], r[2], r[4], r[6]) | (bytes(r[1], r[3], r[5], r[7]) << 4);
}

// The same codes with the rounding decided exactly: with b = floor(t), the code is b or b + 1 as x is below or above zero +
// (b + 1/2) scale, and the even one where they are equal.  (b + 1/2) scale is exact in single precision (at most 20 bits).
template <bool BF16, int BITS>
__device__ __forceinline__ uint32_t row_codes_exact(const u32x4& w, int first, const RowQuant& q) {
  constexpr int N = 32 / BITS;
  uint32_t packed = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float x = value<BF16>(w, first + e), b = __builtin_floorf((x - q.zero) * q.inv);
    const int side = compare_sum(x, (b + 0.5f) * q.scale, q.zero);
    const int32_t low = static_cast<int32_t>(b);
    packed |= static_cast<uint32_t>(low + (side > 0 || (side == 0 && (low & 1)) ? 1 : 0)) << (BITS * e);
  }
  return packed;
}

// A row's pieces (8 channels of K and of V) as codes.
template <bool BF16, int BITS>
__device__ __forceinline__ void piece_codes(const u32x4& w, const RowQuant& q, uint32_t (&codes)[BITS / 4]) {
  float far = 0.0f;
#pragma unroll
  for (int i = 0; i < BITS / 4; ++i) codes[i] = row_codes<BF16, BITS>(w, 4 * i, q, far);
  if (far > 0.5f - kNear<BITS>) {
#pragma unroll
    for (int i = 0; i < BITS / 4; ++i) codes[i] = row_codes_exact<BF16, BITS>(w, 4 * i, q);
  }
}

// A row piece from the cache, as 8 16-bit values.
template <bool BF16, int BITS>
__device__ __forceinline__ u32x4 get(const uint8_t* row, uint32_t sz, int32_t piece) {
  const float s = f16_float(sz), z = f16_float(sz >> 16);
  float x[8];
  if constexpr (BITS == 8) {
    const u32x2 c = *reinterpret_cast<const u32x2*>(row + 8 * piece);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(static_cast<float>((c[e >> 2] >> (8 * (e & 3))) & 0xFF), s, z);
  } else {
    const uint32_t c = *reinterpret_cast<const uint32_t*>(row + 4 * piece);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(static_cast<float>((c >> (4 * e)) & 0xF), s, z);
  }
  return u32x4{pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]), pack2<BF16>(x[4], x[5]), pack2<BF16>(x[6], x[7])};
}

struct RowWork {
  int32_t log2_tokens;  // of a workgroup
  int32_t log2_lanes;   // of a row
};

template <bool BF16, int KB, int VB, bool WRITE>
__global__ __launch_bounds__(kThreads) void rows_kernel(ServeArgs a, RowArgs r, RowWork w) {
  __shared__ int32_t starts[kStartsInLds];
  __shared__ Place place[kMostTokens];
  constexpr bool kCodes = KB != 16;
  const int32_t tokens = 1 << w.log2_tokens, lanes = 1 << w.log2_lanes;
  const int32_t i0 = int32_t(blockIdx.x) << w.log2_tokens;
  const int32_t n = tokens < a.num_tokens - i0 ? tokens : a.num_tokens - i0;
  // A pass takes all of the workgroup's tokens and as many heads as there are groups of lanes for; a thread stays
  // with its token.
  const int32_t piece = threadIdx.x & (lanes - 1), group = threadIdx.x >> w.log2_lanes;
  const int32_t t = group & (tokens - 1), head0 = group >> w.log2_tokens;
  const int32_t heads = (kThreads >> w.log2_lanes) >> w.log2_tokens;
  const bool mine = 8 * piece < a.D && t < n;
  int64_t off = int64_t(i0 + t) * r.token_stride + head0 * r.head_stride + 8 * piece;
  u32x4 k{}, v{};
  if (WRITE && mine && head0 < a.H) {  // on their way while the places are found
    k = *reinterpret_cast<const u32x4*>(r.k + off);
    v = *reinterpret_cast<const u32x4*>(r.v + off);
  }
  find_places<KB, VB>(a, i0, n, starts, place);
  const Place at = place[t < n ? t : 0];
  const bool on = mine && at.k >= 0;
  uint8_t* codes = a.codes + head0 * a.head_stride;
  uint32_t* scales = a.scales + at.scale + ((int64_t(head0) * 2) << a.log2P);
  char* k16 = reinterpret_cast<char*>(a.k_cache) + at.k + 2 * (head0 * a.D + 8 * piece);
  char* v16 = reinterpret_cast<char*>(a.v_cache) + at.v + 2 * (head0 * a.D + 8 * piece);
  // Every lane of a row's group runs the same passes, so the exchanges are between live lanes.
  for (int32_t head = head0; head < a.H; head += heads) {
    const int64_t next = off + heads * r.head_stride;
    if constexpr (WRITE) {
      const u32x4 k_now = k, v_now = v;
      if (mine && head + heads < a.H) {
        k = *reinterpret_cast<const u32x4*>(r.k + next);
        v = *reinterpret_cast<const u32x4*>(r.v + next);
      }
      if constexpr (kCodes) {
        float mn[2] = {__builtin_inff(), __builtin_inff()}, mx[2] = {-__builtin_inff(), -__builtin_inff()};
        if (8 * piece < a.D) {
          piece_range<BF16>(k_now, mn[0], mx[0]);
          piece_range<BF16>(v_now, mn[1], mx[1]);
        }
        row_range(mn, mx, lanes);
        const RowQuant kq = row_quant<KB>(mn[0], mx[0]), vq = row_quant<VB>(mn[1], mx[1]);
        uint32_t kc[KB / 4], vc[VB / 4];
        piece_codes<BF16, KB>(k_now, kq, kc);
        piece_codes<BF16, VB>(v_now, vq, vc);
        if (on) {
          if constexpr (KB == 8)
            *reinterpret_cast<u32x2*>(codes + at.k + 8 * piece) = u32x2{kc[0], kc[KB / 4 - 1]};
          else
            *reinterpret_cast<uint32_t*>(codes + at.k + 4 * piece) = kc[0];
          if constexpr (VB == 8)
            *reinterpret_cast<u32x2*>(codes + at.v + 8 * piece) = u32x2{vc[0], vc[VB / 4 - 1]};
          else
            *reinterpret_cast<uint32_t*>(codes + at.v + 4 * piece) = vc[0];
          if (piece < 2) scales[int64_t(piece) << a.log2P] = piece ? vq.word : kq.word;
        }
      } else if (on) {
        *reinterpret_cast<u32x4*>(k16) = k_now;
        *reinterpret_cast<u32x4*>(v16) = v_now;
      }
    } else if (mine && at.k != -2) {
      k = v = u32x4{};
      if (on) {
        if constexpr (kCodes) {
          const uint32_t ks = scales[0], vs = scales[int64_t(1) << a.log2P];
          k = get<BF16, KB>(codes + at.k, ks, piece);
          v = get<BF16, VB>(codes + at.v, vs, piece);
        } else {
          k = *reinterpret_cast<const u32x4*>(k16);
          v = *reinterpret_cast<const u32x4*>(v16);
        }
      }
      *reinterpret_cast<u32x4*>(r.k + off) = k;
      *reinterpret_cast<u32x4*>(r.v + off) = v;
    }
    off = next;
    codes += heads * a.head_stride;
    scales += (int64_t(heads) * 2) << a.log2P;
    k16 += 2 * heads * a.D;
    v16 += 2 * heads * a.D;
  }
}

template <bool WRITE>
pkv_status_t launch_rows(const ServeArgs& s, const RowArgs& r, hipStream_t stream) {
  RowWork w{0, 0};
  while ((8 << w.log2_lanes) < s.D) ++w.log2_lanes;
  // Enough tokens for one pass of a workgroup; up to a pass of one head while that leaves eight workgroups to a compute
  // unit (a prompt of 8192 tokens, append and read back: 15.2 + 9.2 us; with four 18.1 + 10.2, with sixteen 15.9 + 9.4).
  const int32_t pass = kThreads >> w.log2_lanes;
  while ((1 << w.log2_tokens) < pass &&
         ((s.H << w.log2_tokens) < pass || (s.num_tokens >> w.log2_tokens) >= 2048))
    ++w.log2_tokens;
  const dim3 grid((uint32_t(s.num_tokens) + (1u << w.log2_tokens) - 1) >> w.log2_tokens);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, s, r, w); };
  const int which = s.tag * 2 + (s.bf16 ? 1 : 0);
  switch (which) {
    case 0:  // 16-bit rows are copied as they are
    case 1: go(rows_kernel<false, 16, 16, WRITE>); break;
    case 2: go(rows_kernel<false, 8, 8, WRITE>); break;
    case 3: go(rows_kernel<true, 8, 8, WRITE>); break;
    case 4: go(rows_kernel<false, 8, 4, WRITE>); break;
    case 5: go(rows_kernel<true, 8, 4, WRITE>); break;
    case 6: go(rows_kernel<false, 4, 4, WRITE>); break;
    default: go(rows_kernel<true, 4, 4, WRITE>); break;
  }
  return hipGetLastError() == hipSuccess ? PKV_OK : PKV_ERR_DEVICE;
}

// Whether every buffer of a call is memory of the current device.
struct OnDevice {
  int dev = -1;
  bool ok = false;
  OnDevice() { ok = hipGetDevice(&dev) == hipSuccess; }
  bool has(const void* p) const {
    if (!p) return true;
    hipPointerAttribute_t a;
    if (hipPointerGetAttributes(&a, p) != hipSuccess) {
      (void)hipGetLastError();
      return false;
    }
    return (a.type == hipMemoryTypeDevice || a.type == hipMemoryTypeManaged) && a.device == dev;
  }
  bool has(const ServeArgs& s) const {
    return has(s.token_start) && has(s.kv_lens) && has(s.positions) && has(s.page_table) && has(s.k_cache) &&
           has(s.v_cache) && has(s.codes) && has(s.scales);
  }
};

template <bool WRITE>
pkv_status_t rows_call(const pkv_model_t* model, const pkv_paged_cache_t* cache, const pkv_batch_t* batch, const void* k,
                       const void* v, int64_t token_stride, int64_t head_stride, void* hip_stream) {
  ServeArgs s;
  RowArgs r;
  pkv_status_t st = serve_args(model, cache, batch, true, &s);
  if (st == PKV_OK) st = row_args(s, k, v, token_stride, head_stride, &r);
  if (st != PKV_OK || s.num_seqs == 0 || s.num_tokens == 0) return st;
  const OnDevice here;
  if (!here.ok) return PKV_ERR_DEVICE;
  if (!here.has(s) || !here.has(r.k) || !here.has(r.v)) return PKV_ERR_INVALID_ARGUMENT;
  return launch_rows<WRITE>(s, r, static_cast<hipStream_t>(hip_stream));
}

}  // namespace

// One per head_dim, in objects of their own (attend.hip).
pkv_status_t launch_attend_64(const ServeArgs& s, const AttendArgs& a, int64_t groups, hipStream_t stream);
pkv_status_t launch_attend_128(const ServeArgs& s, const AttendArgs& a, int64_t groups, hipStream_t stream);
pkv_status_t launch_attend_256(const ServeArgs& s, const AttendArgs& a, int64_t groups, hipStream_t stream);

}  // namespace pkv

extern "C" {

pkv_status_t pkv_cache_append(const pkv_model_t* model, const pkv_paged_cache_t* cache, const pkv_batch_t* batch,
                              const void* k, const void* v, int64_t token_stride, int64_t head_stride,
                              void* hip_stream) {
  return pkv::rows_call<true>(model, cache, batch, k, v, token_stride, head_stride, hip_stream);
}

pkv_status_t pkv_cache_read(const pkv_model_t* model, const pkv_paged_cache_t* cache, const pkv_batch_t* batch, void* k,
                            void* v, int64_t token_stride, int64_t head_stride, void* hip_stream) {
  return pkv::rows_call<false>(model, cache, batch, k, v, token_stride, head_stride, hip_stream);
}

pkv_status_t pkv_attention(const pkv_model_t* model, const pkv_paged_cache_t* cache, const pkv_batch_t* batch,
                           const pkv_attention_t* attention, void* hip_stream) {
  pkv::ServeArgs s;
  pkv::AttendArgs a;
  pkv_status_t st = pkv::serve_args(model, cache, batch, true, &s);
  if (st == PKV_OK) st = pkv::attend_args(s, attention, true, &a);
  if (st != PKV_OK || s.num_seqs == 0 || s.num_tokens == 0) return st;
  const pkv::AttendLaunch l = pkv::attend_launch(s, a);
  const pkv::OnDevice here;
  if (!here.ok) return PKV_ERR_DEVICE;
  if (!here.has(s) || !here.has(a.q) || !here.has(a.out) || !here.has(a.lse) || !here.has(a.part))
    return PKV_ERR_INVALID_ARGUMENT;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (s.D == 64) return pkv::launch_attend_64(s, a, l.groups, stream);
  if (s.D == 128) return pkv::launch_attend_128(s, a, l.groups, stream);
  return pkv::launch_attend_256(s, a, l.groups, stream);
}

}  // extern "C"
