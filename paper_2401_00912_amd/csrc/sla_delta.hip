// The gated delta rule in chunk form, forward (sla_delta.h has the mathematics).  Two launches:
// k_delta_prep makes T and P of every chunk, k_delta_walk goes through every window's chunks.
#include "sla_delta_chunk.h"

namespace sla {
namespace {

using namespace delta;

template <typename T, int DK>
hipError_t forward_impl(const Args& a, int dtype, const void* q, const void* k, const void* v, const float* g,
                        const float* beta, const float* state_in, void* o, float* state_out, void* workspace,
                        hipStream_t stream) {
  const Space sp = space_of(a.n, a.W, dtype, a.Hk, a.H, a.dk, kRecord);
  char* ws = static_cast<char*>(workspace);
  _Float16* images = reinterpret_cast<_Float16*>(ws + sp.images);
  _Float16* records = reinterpret_cast<_Float16*>(ws + sp.records);
  if (a.n > 0)
    k_delta_prep<T, DK, false><<<dim3(a.slots, a.Hk), 256, 0, stream>>>(
        a, static_cast<const T*>(q), static_cast<const T*>(k), g, beta, images, records);
  float* ends = reinterpret_cast<float*>(ws + align_up(sp.total, 256));
  _Float16* maps = reinterpret_cast<_Float16*>(ends) + (a.part ? ends_halfs(a, DK) : 0);
  if (a.n > 0) launch_ends<T, DK>(a, static_cast<const T*>(v), state_in, images, records, kRecord, ends, maps, stream);
  with_walk<T, DK>(a, [&](auto nw, auto ahead, dim3 grid) {
    constexpr int NW = decltype(nw)::value;
    k_delta_walk<T, DK, kOut, NW, decltype(ahead)::value><<<grid, 64 * NW, 0, stream>>>(
        a, static_cast<const T*>(v), state_in, images, records, kRecord, ends, maps, static_cast<T*>(o), nullptr,
        WalkOut{state_out, nullptr, nullptr, nullptr, nullptr});
  });
  return hipGetLastError();
}

template <typename T>
hipError_t forward_dk(const Args& a, int dtype, const void* q, const void* k, const void* v, const float* g,
                      const float* beta, const float* state_in, void* o, float* state_out, void* workspace,
                      hipStream_t stream) {
  switch (pad_dk(a.dk)) {
    case 32: return forward_impl<T, 32>(a, dtype, q, k, v, g, beta, state_in, o, state_out, workspace, stream);
    case 64: return forward_impl<T, 64>(a, dtype, q, k, v, g, beta, state_in, o, state_out, workspace, stream);
    default: return forward_impl<T, 128>(a, dtype, q, k, v, g, beta, state_in, o, state_out, workspace, stream);
  }
}

}  // namespace

size_t delta_workspace_bytes(int64_t n, int32_t W, int dtype, int32_t Hk, int32_t H, int32_t dk, int32_t dv) {
  const Args a = args_of(nullptr, n, W, nullptr, Hk, H, dk, dv, 1.f);
  return space_of(n, W, dtype, Hk, H, dk, kRecord).total + parts_bytes(a);
}

hipError_t launch_forward_delta(const int32_t* offsets, int32_t n, int32_t W, const int32_t* order, int dtype,
                                int32_t Hk, int32_t H, int32_t dk, int32_t dv, float scale, const void* q,
                                const void* k, const void* v, const float* g, const float* beta,
                                const float* state_in, void* o, float* state_out, void* workspace,
                                hipStream_t stream) {
  const Args a = args_of(offsets, n, W, order, Hk, H, dk, dv, scale);
  if (dtype == 0)
    return forward_dk<float>(a, dtype, q, k, v, g, beta, state_in, o, state_out, workspace, stream);
  if (dtype == 1)
    return forward_dk<_Float16>(a, dtype, q, k, v, g, beta, state_in, o, state_out, workspace, stream);
  return forward_dk<bf16_t>(a, dtype, q, k, v, g, beta, state_in, o, state_out, workspace, stream);
}

}  // namespace sla
