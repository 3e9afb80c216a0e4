// aspd_norm_rope_append: the step between the metadata and the attention call for models that norm their query and key
// heads, turn them by positions on several axes, or bias their scores by distance.  Per new token: every query and key head
// x <- x / sqrt(mean(x^2) + eps) * (offset + w), pair (i, i + D/2) turned by p(axis(i)) * theta^(-2i/D); the query to its
// row of q_out, the key and the value to the paged cache, the token's position to its slot's entry of slot_pos.
//
// Many rows: bound by the bytes, every element read and written once.  Few rows: by the way from the launch over the
// position and its angles to the stores.  One workgroup per row, as in aspd_rope_append, a lane with the same 16-byte chunks
// of either half in every head it takes: its cosines, sines and weights are its own in all of them, and the sum of a head's
// squares goes over as many neighbouring lanes as hold the head.  Units, weights and the slot's entry are on their way before
// the angles are worked out.  32/8 heads of 128 in bf16 out of one projection, norms of both, in graph replay: 98 997 rows
// 412 us, 5.9 TB/s (a copy of 2 GiB: 5.0); 7 994 rows on three axes 40 us; 391 rows 4.7 us; three rows of fp32 2.5 us
// (aspd_rope_append 2.1).  With weights loaded as they are needed, sums by shuffles and the angle's sine in fp64: 445, 41, 4.6 and
// 2.7.  With half the threads, two units each: 427, 40, 4.6, 3.0; the slot's entry written last: 416, 41, 5.0, 2.9.
#include <algorithm>
#include <cmath>

#include "aspd_common.h"

namespace {

constexpr int NR_THREADS = 256;  // at most

template <typename T>
struct NormRopeArgs {
  KvView         kv;
  const int32_t* position_ids;
  const int64_t* slot_mapping;
  const int32_t* q_seq;         // with pos_offset or slot_pos
  const int32_t* logical_slot;  // with slot_pos
  const int32_t* axis_pos;
  long           axis_stride;
  const int32_t* pos_offset;
  int32_t*       slot_pos;
  int            B, owner_stride;
  const T*       q;
  const T*       k;
  const T*       v;
  T*             q_out;
  long           q_stride, k_stride, v_stride, out_stride;
  const T*       q_weight;
  const T*       k_weight;
  float          eps, offset;
  double         log2_theta;    // 0: nothing turns
  uint32_t       axes[4];       // axis of pair i in bits 2 (i % 16) .. of word i / 16
};

// Sum over N consecutive lanes (N a power of two); all of them get it.  Within a row of 16 lanes by data-parallel moves, a
// shuffle through LDS takes a hundred cycles each.
template <int CTRL>
__device__ __forceinline__ float plus_moved(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
template <int N>
__device__ __forceinline__ float sum_lanes(float v) {
  if (N > 1) v = plus_moved<0xb1>(v);    // one further
  if (N > 2) v = plus_moved<0x4e>(v);    // two further
  if (N > 4) v = plus_moved<0x141>(v);   // mirrored in the half row
  if (N > 8) v = plus_moved<0x140>(v);   // mirrored in the row
#pragma unroll
  for (int off = 16; off < N; off *= 2) v += __shfl_xor(v, off);
  return v;
}

// Cosine and sine of p * freq turns.  The product and the distance to the next quarter turn in fp64 (a float product would be
// 1e-3 rad off at positions of a few ten thousand), the rest, an eighth of a turn at most either way, in fp32: off by 2^-23.
__device__ __forceinline__ void turn(double p, double freq, float* c, float* s) {
  const double t = 4.0 * (p * freq - rint(p * freq));
  const double q = rint(t);
  float sine, cosine;
  sincospif(0.5f * (float)(t - q), &sine, &cosine);
  const int quarter = (int)q & 3;
  const float a = quarter & 1 ? sine : cosine, b = quarter & 1 ? cosine : sine;
  *c = quarter == 1 || quarter == 2 ? -a : a;
  *s = quarter >= 2 ? -b : b;
}

// VEC pairs per unit: 16 bytes of T from either half of a head, or 1 where a pointer or stride is not a multiple of 16 bytes.
template <typename T, int D, int VEC>
__global__ __launch_bounds__(NR_THREADS) void norm_rope_append_kernel(NormRopeArgs<T> a) {
  constexpr int HALF = D / 2;
  constexpr int UPH = HALF / VEC;  // units per head: as many lanes side by side hold a head
  constexpr int U = 2;             // units a thread keeps in flight
  static_assert(64 % UPH == 0, "a thread has the same pairs in every head");
  typedef T vec __attribute__((ext_vector_type(VEC)));
  __shared__ __attribute__((aligned(16))) float cs[HALF], sn[HALF];
  const int tid = threadIdx.x, threads = blockDim.x;
  const long row = blockIdx.x;
  const int uq = a.kv.num_q_heads * UPH, uk = a.kv.num_kv_heads * UPH, units = uq + 2 * uk;
  const T* qrow = a.q + row * a.q_stride;
  const T* krow = a.k + row * a.k_stride;
  const T* vrow = a.v + row * a.v_stride;
  T* orow = a.q_out + row * a.out_stride;
  const long slot = a.slot_mapping[row];
  const int pos = a.position_ids[row];
  const int ch = tid % UPH * VEC;  // the thread's pairs in every head

  vec x[U], y[U];
  auto issue = [&](int u0) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = u0 + i * threads;
      if (u >= units) continue;
      const T* src = u < uq ? qrow + u / UPH * D : (u < uq + uk ? krow + (u - uq) / UPH * D : vrow + (u - uq - uk) / UPH * D);
      x[i] = *(const vec*)(src + ch);
      y[i] = *(const vec*)(src + ch + HALF);
    }
  };
  issue(tid);
  vec wq[2] = {}, wk[2] = {};  // the thread's weights
  if (a.q_weight) {
    wq[0] = *(const vec*)(a.q_weight + ch);
    wq[1] = *(const vec*)(a.q_weight + ch + HALF);
  }
  if (a.k_weight) {
    wk[0] = *(const vec*)(a.k_weight + ch);
    wk[1] = *(const vec*)(a.k_weight + ch + HALF);
  }
  asm volatile("" ::: "memory");  // these loads leave before the angles are worked out
  if (tid < HALF) {
    float s = 0.f, c = 1.f;
    if (a.log2_theta != 0.0) {
      int p = pos;
      if (a.axis_pos) p = a.axis_pos[(long)((a.axes[tid >> 4] >> (2 * (tid & 15))) & 3) * a.axis_stride + row];
      else if (a.pos_offset) p += a.pos_offset[min(max(a.q_seq[row], 0), a.B - 1)];
      turn((double)p, exp2(-(2.0 * tid / D) * a.log2_theta) * 0.15915494309189535 /* 1 / 2 pi */, &c, &s);
    }
    cs[tid] = c;
    sn[tid] = s;
  }
  if (a.slot_pos && tid == threads - 1) {
    const int s = a.q_seq[row], j = a.logical_slot[row];
    if (s >= 0 && s < a.B && j >= 0 && j < a.owner_stride) a.slot_pos[(long)s * a.owner_stride + j] = pos;
  }
  __syncthreads();
  const bool placed = slot >= 0 && slot < (long)a.kv.num_blocks * ASPD_BLOCK;  // never write outside the pools
  const long place = placed ? ((slot / ASPD_BLOCK) * a.kv.num_kv_heads * ASPD_BLOCK + slot % ASPD_BLOCK) * D : 0;
  for (int u0 = tid;;) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = u0 + i * threads;
      if (u >= units || (u >= uq && !placed)) continue;  // (the lanes of a head go the same way)
      const bool is_q = u < uq, is_v = u >= uq + uk;
      T* dst = is_q ? orow + u / UPH * D
                    : (T*)(is_v ? a.kv.v : a.kv.k) + place + (long)((u - uq - (is_v ? uk : 0)) / UPH) * ASPD_BLOCK * D;
      vec oa = x[i], ob = y[i];
      if (!is_v) {
        float fa[VEC], fb[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          fa[e] = (float)x[i][e];
          fb[e] = (float)y[i][e];
        }
        if (is_q ? a.q_weight : a.k_weight) {
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < VEC; ++e) sum += fa[e] * fa[e] + fb[e] * fb[e];
          const float r = rsqrtf(sum_lanes<UPH>(sum) * (1.f / D) + a.eps);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            fa[e] *= r * (a.offset + (float)(is_q ? wq[0][e] : wk[0][e]));
            fb[e] *= r * (a.offset + (float)(is_q ? wq[1][e] : wk[1][e]));
          }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float c = cs[ch + e], s = sn[ch + e];
          oa[e] = (T)(fa[e] * c - fb[e] * s);
          ob[e] = (T)(fb[e] * c + fa[e] * s);
        }
      }
      *(vec*)(dst + ch) = oa;
      *(vec*)(dst + ch + HALF) = ob;
    }
    u0 += U * threads;
    if (u0 >= units) break;
    issue(u0);
  }
}

template <typename T, int D>
void norm_rope_launch(const NormRopeArgs<T>& a, int rows, bool wide, hipStream_t hs) {
  // a thread per unit of a row, up to four waves
  const int vec = wide ? 16 / (int)sizeof(T) : 1, units = (a.kv.num_q_heads + 2 * a.kv.num_kv_heads) * (D / 2 / vec);
  const int threads = std::min(NR_THREADS, (units + 63) / 64 * 64);
  if (wide) hipLaunchKernelGGL((norm_rope_append_kernel<T, D, 16 / sizeof(T)>), dim3(rows), dim3(threads), 0, hs, a);
  else hipLaunchKernelGGL((norm_rope_append_kernel<T, D, 1>), dim3(rows), dim3(threads), 0, hs, a);
}

template <typename T>
int norm_rope_append(const aspd_kv* kv, const aspd_state* state, const aspd_step* step, const aspd_rotary* how, void* q,
                     long q_stride, const void* k, long k_stride, const void* v, long v_stride, void* q_out, int32_t* slot_pos,
                     hipStream_t hs) {
  NormRopeArgs<T> a;
  const int D = kv->head_dim;
  const long q_row = (long)kv->num_q_heads * D, kv_row = (long)kv->num_kv_heads * D;
  a.kv = make_view(kv);
  a.position_ids = step->position_ids_d;
  a.slot_mapping = step->slot_mapping_d;
  a.q_seq = step->q_seq_d;
  a.logical_slot = step->logical_slot_d;
  a.axis_pos = how->axis_pos_d;
  a.axis_stride = how->axis_stride;
  a.pos_offset = how->pos_offset_d;
  a.slot_pos = slot_pos;
  a.B = state ? state->B : 0;
  a.owner_stride = state ? state->owner_stride : 0;
  a.q = (const T*)q;
  a.k = (const T*)k;
  a.v = (const T*)v;
  a.q_stride = q_stride ? q_stride : q_row;
  a.k_stride = k_stride ? k_stride : kv_row;
  a.v_stride = v_stride ? v_stride : kv_row;
  a.q_out = q_out ? (T*)q_out : (T*)q;
  a.out_stride = q_out ? q_row : a.q_stride;
  a.q_weight = (const T*)how->q_weight_d;
  a.k_weight = (const T*)how->k_weight_d;
  a.eps = how->norm_eps;
  a.offset = how->weight_offset;
  a.log2_theta = how->rope_theta == 0.f ? 0.0 : log2((double)how->rope_theta);
  for (int w = 0; w < 4; ++w) a.axes[w] = 0;
  if (how->axis_pos_d && how->axis_of_pair)
    for (int i = 0; i < D / 2; ++i) a.axes[i >> 4] |= (uint32_t)how->axis_of_pair[i] << (2 * (i & 15));
  // units of 16 bytes where everything they are read from and written to lies on 16 bytes
  const uintptr_t at = (uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)a.q_out | (uintptr_t)a.kv.k | (uintptr_t)a.kv.v |
                       (uintptr_t)how->q_weight_d | (uintptr_t)how->k_weight_d | (uintptr_t)((a.q_stride | a.k_stride | a.v_stride) * (long)sizeof(T));
  const bool wide = (at & 15) == 0;
  if (D == 128) norm_rope_launch<T, 128>(a, step->NQ, wide, hs);
  else norm_rope_launch<T, 64>(a, step->NQ, wide, hs);
  ASPD_HIP_CHECK(hipGetLastError());
  return ASPD_OK;
}

}  // namespace

extern "C" int aspd_norm_rope_append(const aspd_kv* kv, const aspd_state* state, const aspd_step* step,
                                     const aspd_rotary* how, void* q_d, int64_t q_stride, const void* k_new_d,
                                     int64_t k_stride, const void* v_new_d, int64_t v_stride, void* q_out_d,
                                     int32_t* slot_pos_d, void* stream) {
  int rc = aspd_check_kv(kv);
  if (rc != ASPD_OK) return rc;
  if (!step || step->NQ < 0 || !how) return ASPD_ERR_INVALID_ARG;
  if (how->rope_theta != 0.f && !(how->rope_theta > 1.f && std::isfinite(how->rope_theta))) return ASPD_ERR_INVALID_ARG;
  if ((how->q_weight_d || how->k_weight_d) &&
      !(how->norm_eps > 0.f && std::isfinite(how->norm_eps) && std::isfinite(how->weight_offset)))
    return ASPD_ERR_INVALID_ARG;
  if (how->axis_pos_d) {
    if (how->num_axes < 1 || how->axis_stride < step->NQ || how->pos_offset_d) return ASPD_ERR_INVALID_ARG;
    if (how->num_axes > ASPD_MAX_AXES) return ASPD_ERR_UNSUPPORTED;
    if (how->axis_of_pair)
      for (int i = 0; i < kv->head_dim / 2; ++i)
        if (how->axis_of_pair[i] >= how->num_axes) return ASPD_ERR_INVALID_ARG;
  }
  if ((how->pos_offset_d || slot_pos_d) && (!state || state->B <= 0)) return ASPD_ERR_INVALID_ARG;
  if (slot_pos_d && state->owner_stride <= 0) return ASPD_ERR_INVALID_ARG;
  const int64_t q_row = (int64_t)kv->num_q_heads * kv->head_dim, kv_row = (int64_t)kv->num_kv_heads * kv->head_dim;
  if ((q_stride != 0 && q_stride < q_row) || (k_stride != 0 && k_stride < kv_row) || (v_stride != 0 && v_stride < kv_row))
    return ASPD_ERR_INVALID_ARG;
  if (step->NQ == 0) return ASPD_OK;
  if (!step->position_ids_d || !step->slot_mapping_d || !q_d || !k_new_d || !v_new_d) return ASPD_ERR_INVALID_ARG;
  if ((how->pos_offset_d || slot_pos_d) && !step->q_seq_d) return ASPD_ERR_INVALID_ARG;
  if (slot_pos_d && !step->logical_slot_d) return ASPD_ERR_INVALID_ARG;
  if (q_out_d == q_d && q_stride != 0 && q_stride != q_row) return ASPD_ERR_INVALID_ARG;  // (rows would land on others)
  hipStream_t hs = (hipStream_t)stream;
  if (kv->dtype == ASPD_BF16)
    return norm_rope_append<__bf16>(kv, state, step, how, q_d, q_stride, k_new_d, k_stride, v_new_d, v_stride, q_out_d, slot_pos_d, hs);
  return norm_rope_append<float>(kv, state, step, how, q_d, q_stride, k_new_d, k_stride, v_new_d, v_stride, q_out_d, slot_pos_d, hs);
}
