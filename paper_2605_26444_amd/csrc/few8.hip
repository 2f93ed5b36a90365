// The 8-bit head for up to 16 hidden rows: the hidden rows are rounded to 8 bits in the kernel and stay in registers, the list streams past
// them.
//
// A call on few rows is one launch: a launch of its own for the hidden rows would cost as much as it has to read (2.5 us; 3000
// rows of 4096 bytes are 2 us at the rate of a large read).  Every workgroup rounds all hidden rows -- M d numbers, from its die's
// L2, while its first rows of W are on their way -- into LDS and takes its operands from there.
//
// What bounds it: on short lists one round trip after the other -- arguments, row count with ids and hidden rows, W, sums, logits -- and the rounding (3000 x 4096 in a graph: M = 1
// 5.3 us, M = 8 6.8, without any rounding 5.4); on the whole matrix HBM (128256 x 4096, M = 8 88 us, 6.0 TB/s); on batches the bytes beyond a die's L2 (64 sequences of 2300 x
// 4096, M = 8 56 us, 287 MB for 193 MB of distinct rows).  The bf16 kernels: 7.4, 172 and 103 us.
#include "common.h"

namespace nanospec {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// sum over the four lanes of a quad, in every lane of it (DPP quad_perm: neighbours 1 apart, then 2 apart)
__device__ __forceinline__ int quad_sum(int x) { return dpp_add_int<0x4E, 0xf>(dpp_add_int<0xB1, 0xf>(x)); }

// Wavefront w: group rg = w % ng of the list rows (ng a power of two), slice ks = w / ng of the columns (256 KS bytes).  Operand layout: the 16
// operand rows are 4 list rows x 4 column parts against 4 hidden rows x the same parts (MT tiles of them), so that a load covers 4 rows x 256
// contiguous bytes; of a product's 16 x 16 results the 4 x 4 with equal parts count.  A step is such a quad of rows for every group -- a block
// of 4 ng rows for the workgroup --, KS loads a wavefront; D steps are in flight.
// Grid: 8 dies x sequences x parts, np = 8 parts pieces (a power of two) of every list.  One sequence: piece p takes blocks p, p + np, ..., so that the ids
// of its first steps can be asked for together with the row count.  Several: piece p = die * parts + part takes a stretch of the list: consecutive
// workgroups go to the dies in turn, so that a die works on the same eighth of every sequence's list and finds the rows that sequences share in its L2.
// The sums of at most seg steps (a multiple of D) meet in LDS, where the slices are added and the scales applied.
// ROUND: hidden rows from H, else from Hq and H_scale.  LISTED: rows from ids (cap of them, n_dev live), else rows 0 .. cap - 1.
template <int MT, int KS, int D, bool ROUND, bool LISTED>
__global__ __launch_bounds__(512, 2) void head_few_i8_kernel(const int8_t* __restrict__ W, const float* __restrict__ W_scale, const uint16_t* __restrict__ H,
                                                             const int8_t* __restrict__ Hq, const float* __restrict__ H_scale, const int32_t* __restrict__ ids,
                                                             const int32_t* __restrict__ n_dev, int cap, int V, int M, int d, int64_t ld,
                                                             float* __restrict__ logits, int log_np, int nk, int log_ng, int seg) {
  constexpr int MH = 4 * MT, HP = 8;                                      // HP: pieces of 16 bytes of a hidden row that a lane holds: all of 4096 numbers
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int log_rows = 2 + log_ng, seg_rows = seg << log_rows, segp = seg_rows + 4;
  float* hscale = reinterpret_cast<float*>(smem);                         // [MH]
  float* wscale = hscale + 16;                                            // [seg_rows]
  int* red = reinterpret_cast<int*>(wscale + seg_rows);                   // [slice][hidden row][row of the segment]
  char* hq = reinterpret_cast<char*>(red);                                // the hidden rows in 8 bits, before the first sums
  const int hstride = d + 16;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
  const int rg = w & ((1 << log_ng) - 1), ks = w >> log_ng;
  const int orow = (lane & 15) >> 2, part = lane & 3, q = lane >> 4;
  const int b = blockIdx.y, p = blockIdx.x * gridDim.z + blockIdx.z;      // blockIdx.x: the die
  const bool strided = gridDim.y == 1;
  const int stride = strided ? 1 << log_np : 1;
  int base = p;                                                           // blocks of this piece: base + t * stride

  // the row count, hidden row w and -- for one sequence -- the ids of the first steps are on their way together
  int n_lane = cap;
  if (LISTED) {
    int at = b;
    asm("" : "+v"(at));                                                   // a vector load: the wait for a scalar one would be one for all of them
    n_lane = n_dev[at];
    ids += (int64_t)b * ld;
  }
  const uint16_t* Hb = H + (int64_t)b * M * d;
  u32x4 hx[HP];
  auto load_hidden = [&](int m) {
#pragma unroll
    for (int i = 0; i < HP; ++i) {
      const int c = (i * 64 + lane) * 8;
      hx[i] = *reinterpret_cast<const u32x4*>(Hb + (int64_t)m * d + (c < d ? c : 0));
    }
  };
  if (ROUND && w < M) load_hidden(w);
  // the id at a place of the list; places past its room are its last, those past its live rows hold anything: neither row is stored
  auto id_at = [&](int r) {
    r = r < cap ? r : cap - 1;
    return LISTED ? ids[r] : r;
  };
  auto id_of = [&](int t) { return id_at((((base + t * stride) << log_ng) + rg) * 4 + orow); };     // this lane's row of step t
  // list row behind local row j of the segment that begins with step t0
  auto place = [&](int t0, int j) { return ((base + (t0 + (j >> log_rows)) * stride) << log_rows) + (j & ((1 << log_rows) - 1)); };
  int idn[D], id2[D], sr[2];
  auto ask = [&] {
#pragma unroll
    for (int i = 0; i < D; ++i) idn[i] = id_of(i);
#pragma unroll
    for (int i = 0; i < 2; ++i) sr[i] = id_at(place(0, tid + i * (int)blockDim.x));
#pragma unroll
    for (int i = 0; i < D; ++i) id2[i] = id_of(D + i);
  };
  if (strided) ask();
  const int n = __builtin_amdgcn_readfirstlane(n_lane), blocks = (((n + 3) >> 2) + (1 << log_ng) - 1) >> log_ng;
  int steps;                                                              // blocks of this piece
  if (strided) {
    steps = (blocks - p + stride - 1) >> log_np;
  } else {
    const int each = blocks >> log_np, more = blocks - (each << log_np);
    base = p * each + (p < more ? p : more);
    steps = each + (p < more ? 1 : 0);
  }
  if (steps <= 0) return;
  if (!strided) ask();
  logits += (int64_t)b * M * ld;

  const int col = ks * (256 * KS) + q * 64 + part * 16;                   // + t * 256
  uint32_t coff[KS];                                                      // this lane's pieces of a row; those past its end are its first, against zeros
#pragma unroll
  for (int t = 0; t < KS; ++t) coff[t] = col + t * 256 < d ? col + t * 256 : 0;
  int pm[4];                                                              // masks of this lane's part: no branches around the sums over lanes
#pragma unroll
  for (int i = 0; i < 4; ++i) pm[i] = part == i ? -1 : 0;
  auto clamped = [&](int id) { return id < 0 ? 0 : (id >= V ? V - 1 : id); };
  auto fetch = [&](u32x4(&v)[KS], int id, int t) {
    const uint32_t row = (uint32_t)clamped(id) * (uint32_t)d, in = t < steps ? 0xffffffffu : 0u;    // a step past the end: all lanes at one address
#pragma unroll
    for (int i = 0; i < KS; ++i) v[i] = *reinterpret_cast<const u32x4*>(W + (row + (coff[i] & in)));
  };
  float sc[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) sc[i] = W_scale[clamped(sr[i])];
  u32x4 wv[D][KS], hv[MT][KS];
#pragma unroll
  for (int i = 0; i < D; ++i) {
    fetch(wv[i], idn[i], i);
    idn[i] = id2[i];
  }
  __builtin_amdgcn_sched_barrier(0);

  if (ROUND) {
    auto round_hidden = [&](int m) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < HP; ++i)                                        // a piece past the end is a copy of the row's first
#pragma unroll
        for (int e = 0; e < 4; ++e) top = bf16_tops(top, hx[i][e]);
      const I8Row k = i8_row(wave_top(top));
      char* to = hq + m * hstride;
      auto put = [&](auto tiny) {
        auto one = [&](int c, const u32x4 y) {
          constexpr bool T = decltype(tiny)::value;
          *reinterpret_cast<u32x2*>(to + c) = u32x2{i8_round4<T>(k, y[0], y[1]), i8_round4<T>(k, y[2], y[3])};
        };
#pragma unroll
        for (int i = 0; i < HP; ++i) {
          const int c = (i * 64 + lane) * 8;
          if (c < d) one(c, hx[i]);
        }
      };
      if (k.p == 1.f) put(Flag<false>());
      else put(Flag<true>());
      if (lane == 0) hscale[m] = k.scale;
    };
    // the first row on its own: as a loop's first its registers might hold later loads, and the wait for it would be one for W
    if (w < M) round_hidden(w);
    for (int m = w + nw; m < M; m += nw) {
      load_hidden(m);
      round_hidden(m);
    }
    __syncthreads();
  } else if (tid < M) {
    hscale[tid] = H_scale[b * M + tid];
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int m = mt * 4 + orow < M ? mt * 4 + orow : M - 1;              // a row past M is a copy, never stored
    const char* hp = ROUND ? hq + m * hstride : reinterpret_cast<const char*>(Hq) + ((int64_t)b * M + m) * d;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(hp + coff[t]);
      hv[mt][t] = col + t * 256 < d ? v : u32x4{0u, 0u, 0u, 0u};
    }
  }
  if (ROUND) __syncthreads();                                             // the hidden rows' place is the sums' from here on

  for (int t0 = 0; t0 < steps; t0 += seg) {
    const int tn = steps - t0 < seg ? steps - t0 : seg;
    if (t0) {
#pragma unroll
      for (int i = 0; i < 2; ++i) sc[i] = W_scale[clamped(id_at(place(t0, tid + i * (int)blockDim.x)))];
    }
    for (int i0 = 0; i0 < tn; i0 += D) {
#pragma unroll
      for (int u = 0; u < D; ++u) {
        const int i = i0 + u, id = idn[u];
        idn[u] = id_of(t0 + i + 2 * D);
        if (i < tn) {
          i32x4 acc[MT];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) acc[mt] = i32x4{0, 0, 0, 0};
#pragma unroll
          for (int t = 0; t < KS; ++t)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
              acc[mt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, wv[u][t]), __builtin_bit_cast(i32x4, hv[mt][t]), acc[mt], 0, 0, 0);
          // result lane l holds product rows 4 * (l / 16) + v, column l % 16; the diagonal block entry is v == l % 4.  After the sum over the
          // parts all four lanes of a quad hold the sum of (list row q, hidden row 4 mt + orow): lane `part` keeps tile mt == part
          int y = 0;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const i32x4 a = acc[mt];
            y |= quad_sum((a[0] & pm[0]) | (a[1] & pm[1]) | (a[2] & pm[2]) | (a[3] & pm[3])) & pm[mt];
          }
          if (part < MT) red[(ks * MH + part * 4 + orow) * segp + ((i << log_ng) + rg) * 4 + q] = y;
        }
        fetch(wv[u], id, t0 + i + D);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = tid + i * (int)blockDim.x;
      if (j < seg_rows) wscale[j] = sc[i];
    }
    __syncthreads();
    for (int m = w; m < M; m += nw) {
      const float hs = hscale[m];
      for (int j = lane; j < tn << log_rows; j += 64) {
        int s = red[m * segp + j];
        for (int k = 1; k < nk; ++k) s += red[(k * MH + m) * segp + j];
        const int r = place(t0, j);
        if (r < n) logits[(int64_t)m * ld + r] = i8_logit(s, wscale[j], hs);
      }
    }
    if (t0 + seg < steps) __syncthreads();
  }
}

template <int MT, int KS, int D, bool ROUND, typename... A>
static hipError_t run_few_i8(const FewPlan& f, bool listed, int batch, hipStream_t s, A... a) {
  const dim3 grid(8, (unsigned)batch, 1u << f.log_parts);
  if (listed) head_few_i8_kernel<MT, KS, D, ROUND, true><<<grid, 64 * f.waves, f.lds, s>>>(a..., f.log_parts + 3, f.slices, f.log_groups, f.seg);
  else head_few_i8_kernel<MT, KS, D, ROUND, false><<<grid, 64 * f.waves, f.lds, s>>>(a..., f.log_parts + 3, f.slices, f.log_groups, f.seg);
  return hipGetLastError();
}

template <bool ROUND, typename... A>
static hipError_t run_few_i8_shape(int M, const FewPlan& f, A... a) {
  if (f.KS == 2) return M <= 4 ? run_few_i8<1, 2, 4, ROUND>(f, a...) : M <= 8 ? run_few_i8<2, 2, 4, ROUND>(f, a...) : run_few_i8<4, 2, 4, ROUND>(f, a...);
  if (f.KS == 4) return M <= 4 ? run_few_i8<1, 4, 4, ROUND>(f, a...) : M <= 8 ? run_few_i8<2, 4, 4, ROUND>(f, a...) : run_few_i8<4, 4, 4, ROUND>(f, a...);
  return M <= 4 ? run_few_i8<1, 8, 2, ROUND>(f, a...) : run_few_i8<2, 8, 2, ROUND>(f, a...);
}

// H: bf16, rounded in the kernel; or null, and Hq with H_scale: rounded before
hipError_t launch_head_few_i8(const int8_t* W, const float* W_scale, const void* H, const int8_t* Hq, const float* H_scale, const int32_t* ids, const int32_t* n_dev,
                              int32_t cap_rows, int32_t V, int32_t batch, int32_t M, int32_t d, int64_t ld, float* logits, hipStream_t s) {
  const FewPlan f = few_plan(M, d, batch, cap_rows, H != nullptr);
  const uint16_t* h = static_cast<const uint16_t*>(H);
  if (h) return run_few_i8_shape<true>(M, f, ids != nullptr, batch, s, W, W_scale, h, Hq, H_scale, ids, n_dev, cap_rows, V, M, d, ld, logits);
  return run_few_i8_shape<false>(M, f, ids != nullptr, batch, s, W, W_scale, h, Hq, H_scale, ids, n_dev, cap_rows, V, M, d, ld, logits);
}

template <int MT, int KS, int D>
static hipError_t configure_few() {
  const void* fns[] = {reinterpret_cast<const void*>(head_few_i8_kernel<MT, KS, D, false, false>), reinterpret_cast<const void*>(head_few_i8_kernel<MT, KS, D, false, true>),
                       reinterpret_cast<const void*>(head_few_i8_kernel<MT, KS, D, true, false>), reinterpret_cast<const void*>(head_few_i8_kernel<MT, KS, D, true, true>)};
  for (const void* f : fns) {
    hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t few_configure_device() {
  hipError_t e = configure_few<1, 2, 4>();
  if (e == hipSuccess) e = configure_few<2, 2, 4>();
  if (e == hipSuccess) e = configure_few<4, 2, 4>();
  if (e == hipSuccess) e = configure_few<1, 4, 4>();
  if (e == hipSuccess) e = configure_few<2, 4, 4>();
  if (e == hipSuccess) e = configure_few<4, 4, 4>();
  if (e == hipSuccess) e = configure_few<1, 8, 2>();
  if (e == hipSuccess) e = configure_few<2, 8, 2>();
  return e;
}

}  // namespace nanospec
