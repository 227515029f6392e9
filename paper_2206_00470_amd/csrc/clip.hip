// Entry points of the global gradient norm and of clipping.
#include "clip.hpp"

#include <algorithm>
#include <cstring>
#include <new>
#include <vector>

#include "internal.hpp"
#include "rules.hpp"

using namespace adapm;

namespace {

constexpr int64_t NUMEL_MAX = int64_t(1) << 38;   // the chunks of CLIP_TENSORS tensors stay below 2^32

// The launches of a call carry CLIP_TENSORS tensors each.
int64_t list_count(int32_t count) { return std::max<int64_t>(1, div_up(count, CLIP_TENSORS)); }

struct Span {
  uintptr_t lo, hi;
};

bool overlap(std::vector<Span>& v) {
  std::sort(v.begin(), v.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
  for (size_t i = 1; i < v.size(); ++i)
    if (v[i].lo < v[i - 1].hi) return true;
  return false;
}

ps_status check_tensors(int32_t count, const void* const* grads, void* const* outs, const int64_t* numel,
                        const int32_t* types) {
  if (count < 0) return raise(PS_ERR_INVALID, "negative size %d", count);
  if (count > 0 && (!grads || !numel || !types)) return raise(PS_ERR_INVALID, "grads, numel or types is NULL");
  for (int32_t k = 0; k < count; ++k) {
    if (numel[k] < 0) return raise(PS_ERR_INVALID, "tensor %d: negative size %lld", k, (long long)numel[k]);
    if (numel[k] > NUMEL_MAX) return raise(PS_ERR_UNSUPPORTED, "tensor %d: %lld elements", k, (long long)numel[k]);
    if (types[k] != PS_F32 && types[k] != PS_BF16 && types[k] != PS_F16)
      return raise(PS_ERR_INVALID, "tensor %d: unknown element type %d", k, types[k]);
    if (numel[k] == 0) continue;
    const size_t b = types[k] == PS_F32 ? 4 : 2;
    if (!grads[k] || (outs && !outs[k])) return raise(PS_ERR_INVALID, "tensor %d: NULL address", k);
    if (!on_bytes(grads[k], b) || (outs && !on_bytes(outs[k], b)))
      return raise(PS_ERR_INVALID, "tensor %d is not aligned to its elements", k);
  }
  if (!outs) return PS_OK;
  // what one tensor writes no other reads or writes: outputs lie apart from
  // each other and from every input but their own, which they may equal
  std::vector<Span> all, in;
  for (int32_t k = 0; k < count; ++k) {
    if (numel[k] == 0) continue;
    const uintptr_t b = static_cast<uintptr_t>(numel[k]) * (types[k] == PS_F32 ? 4 : 2);
    const uintptr_t i = reinterpret_cast<uintptr_t>(grads[k]), o = reinterpret_cast<uintptr_t>(outs[k]);
    all.push_back(Span{o, o + b});
    if (i != o) in.push_back(Span{i, i + b});
  }
  std::sort(in.begin(), in.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
  // inputs that are only read may overlap each other: one span a stretch
  std::vector<Span> read;
  for (const Span& x : in) {
    if (!read.empty() && x.lo < read.back().hi) read.back().hi = std::max(read.back().hi, x.hi);
    else read.push_back(x);
  }
  all.insert(all.end(), read.begin(), read.end());
  if (overlap(all)) return raise(PS_ERR_INVALID, "an output overlaps another tensor");
  return PS_OK;
}

ps_status check_call(bool scaling, double max_norm, double* norm, void* ws, size_t ws_bytes, size_t need) {
  if (!norm) return raise(PS_ERR_INVALID, "norm is NULL");
  if (!on_bytes(norm, 8)) return raise(PS_ERR_INVALID, "norm is not aligned to its elements");
  if (scaling && !(max_norm > 0.0)) return raise(PS_ERR_INVALID, "need max_norm > 0");
  if (!ws) return raise(PS_ERR_INVALID, "workspace pointer is NULL");
  if (ws_bytes < need) return raise(PS_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
  if (!on_bytes(ws, 8)) return raise(PS_ERR_INVALID, "the workspace must be 8-byte aligned");
  return PS_OK;
}

// Outputs of so many bytes, apart from what is read, are written past the caches.
bool streams(int64_t apart) { return apart > LLC_BYTES / 2; }

ps_status total(const double* part, int64_t parts, double* norm, hipStream_t st) {
  hipLaunchKernelGGL(k_norm_total, dim3(1), dim3(BLOCK), 0, st, part, parts, norm);
  RAISE_HIP(hipGetLastError());
  return PS_OK;
}

ps_status clip(int32_t count, const void* const* grads, void* const* outs, const int64_t* numel, const int32_t* types,
               double max_norm, double* norm, void* ws, size_t ws_bytes, hipStream_t st) {
  if (ps_status r = check_tensors(count, grads, outs, numel, types)) return r;
  if (ps_status r = check_call(outs, max_norm, norm, ws, ws_bytes, ps_clip_workspace_bytes(count))) return r;
  double* part = static_cast<double*>(ws);
  std::vector<TensorList> lists;
  int32_t k = 0;
  while (k < count) {
    TensorList t{};
    int64_t chunks = 0;
    for (; k < count && t.count < CLIP_TENSORS; ++k) {
      if (numel[k] == 0) continue;
      t.in[t.count] = grads[k];
      t.out[t.count] = outs ? outs[k] : nullptr;
      t.numel[t.count] = numel[k];
      t.type[t.count] = (uint8_t)types[k];
      t.first[t.count] = (uint32_t)chunks;
      chunks += div_up(numel[k], CLIP_CHUNK);
      t.first[++t.count] = (uint32_t)chunks;
    }
    if (t.count) lists.push_back(t);
  }
  auto grid = [](const TensorList& t) { return std::min<int64_t>(t.first[t.count], CLIP_GRID); };
  int64_t parts = 0;
  for (const TensorList& t : lists) {
    hipLaunchKernelGGL(k_norm_part<TensorList>, dim3(grid(t)), dim3(BLOCK), 0, st, t, part + parts);
    RAISE_HIP(hipGetLastError());
    parts += grid(t);
  }
  if (!outs || lists.empty()) return total(part, parts, norm, st);
  int64_t apart = 0;
  for (int32_t i = 0; i < count; ++i)
    if (grads[i] != outs[i]) apart += numel[i] * type_bytes(types[i]);
  auto kernel = streams(apart) ? k_clip_scale<true, TensorList> : k_clip_scale<false, TensorList>;
  for (size_t i = lists.size(); i-- > 0;) {
    hipLaunchKernelGGL(kernel, dim3(grid(lists[i])), dim3(BLOCK), 0, st, lists[i], part, parts, max_norm,
                       i == 0 ? norm : nullptr);
    RAISE_HIP(hipGetLastError());
  }
  return PS_OK;
}

}  // namespace

extern "C" {

size_t ps_clip_workspace_bytes(int32_t count) {
  if (count < 0) return 0;
  return size_t(list_count(count)) * CLIP_GRID * sizeof(double);
}

ps_status ps_grad_norm(int32_t count, const void* const* grads, const int64_t* numel, const int32_t* types,
                       double* norm, void* ws, size_t ws_bytes, void* stream) {
  try {
    return clip(count, grads, nullptr, numel, types, 0.0, norm, ws, ws_bytes, static_cast<hipStream_t>(stream));
  } catch (const std::bad_alloc&) {
    return raise(PS_ERR_DEVICE, "out of host memory");
  }
}

ps_status ps_clip_grads(int32_t count, const void* const* grads, void* const* outs, const int64_t* numel,
                        const int32_t* types, double max_norm, double* norm, void* ws, size_t ws_bytes, void* stream) {
  if (!outs && count > 0) return raise(PS_ERR_INVALID, "outs is NULL");
  try {
    static void* const none[1] = {nullptr};
    return clip(count, grads, outs ? outs : none, numel, types, max_norm, norm, ws, ws_bytes,
                static_cast<hipStream_t>(stream));
  } catch (const std::bad_alloc&) {
    return raise(PS_ERR_DEVICE, "out of host memory");
  }
}

size_t ps_clip_plan_bytes(int32_t count, const int64_t* numel) {
  if (count < 0 || (count > 0 && !numel)) return 0;
  int64_t chunks = 0;
  for (int32_t k = 0; k < count; ++k) {
    if (numel[k] < 0 || numel[k] > NUMEL_MAX) return 0;
    chunks += div_up(numel[k], CLIP_CHUNK);
  }
  return size_t(chunks) * sizeof(ClipChunk);
}

ps_status ps_clip_plan(int32_t count, const void* const* grads, void* const* outs, const int64_t* numel,
                       const int32_t* types, void* plan, size_t plan_bytes, int64_t* apart) {
  if (count > 0 && !outs) return raise(PS_ERR_INVALID, "outs is NULL");
  if (!apart) return raise(PS_ERR_INVALID, "apart is NULL");
  try {
    if (ps_status r = check_tensors(count, grads, outs, numel, types)) return r;
    if (plan_bytes != ps_clip_plan_bytes(count, numel))
      return raise(PS_ERR_INVALID, "the plan has %zu bytes, not %zu", plan_bytes, ps_clip_plan_bytes(count, numel));
    if (plan_bytes / sizeof(ClipChunk) > UINT32_MAX / 2) return raise(PS_ERR_UNSUPPORTED, "%zu bytes of chunks", plan_bytes);
    if (plan_bytes > 0 && !plan) return raise(PS_ERR_INVALID, "plan is NULL");
    char* to = static_cast<char*>(plan);
    *apart = 0;
    for (int32_t k = 0; k < count; ++k) {
      const int64_t b = type_bytes(types[k]);
      if (grads[k] != outs[k]) *apart += numel[k] * b;
      for (int64_t i = 0; i < numel[k]; i += CLIP_CHUNK, to += sizeof(ClipChunk)) {
        const ClipChunk c{static_cast<const char*>(grads[k]) + i * b, static_cast<char*>(outs[k]) + i * b,
                          (uint32_t)std::min(numel[k] - i, CLIP_CHUNK), (uint32_t)types[k]};
        std::memcpy(to, &c, sizeof c);
      }
    }
    return PS_OK;
  } catch (const std::bad_alloc&) {
    return raise(PS_ERR_DEVICE, "out of host memory");
  }
}

ps_status ps_clip_run(const void* plan, size_t plan_bytes, int64_t apart, int32_t scaling, double max_norm,
                      double* norm, void* ws, size_t ws_bytes, void* stream) {
  if (plan_bytes % sizeof(ClipChunk) || plan_bytes / sizeof(ClipChunk) > UINT32_MAX / 2)
    return raise(PS_ERR_INVALID, "%zu bytes are no plan", plan_bytes);
  if (plan_bytes > 0 && (!plan || !on_bytes(plan, alignof(ClipChunk))))
    return raise(PS_ERR_INVALID, "plan is NULL or not 8-byte aligned");
  if (ps_status r = check_call(scaling, max_norm, norm, ws, ws_bytes, ps_clip_workspace_bytes(1))) return r;
  hipStream_t st = static_cast<hipStream_t>(stream);
  double* part = static_cast<double*>(ws);
  const ChunkList t{static_cast<const ClipChunk*>(plan), (uint32_t)(plan_bytes / sizeof(ClipChunk))};
  const uint32_t grid = std::min<uint32_t>(t.n, CLIP_GRID);
  if (grid > 0) {
    hipLaunchKernelGGL(k_norm_part<ChunkList>, dim3(grid), dim3(BLOCK), 0, st, t, part);
    RAISE_HIP(hipGetLastError());
  }
  if (!scaling || grid == 0) return total(part, grid, norm, st);
  auto kernel = streams(apart) ? k_clip_scale<true, ChunkList> : k_clip_scale<false, ChunkList>;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(BLOCK), 0, st, t, part, int64_t(grid), max_norm, norm);
  RAISE_HIP(hipGetLastError());
  return PS_OK;
}

}  // extern "C"
