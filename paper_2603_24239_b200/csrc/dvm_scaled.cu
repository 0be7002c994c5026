// Scaled matmul meta-kernel, host half of its launch; and dvm_launch's entry for the codes of a layer of experts.
#include <atomic>

#include "dvm_describe.h"
#include "dvm_experts_launch.h"
#include "dvm_scaled.cuh"

static thread_local int t_last_tile = -1;

namespace {
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// A tensor map of `rank` dims, columns first; a box is 128 bytes of `rows` rows, 128-byte swizzle.  What a box reaches beyond the
// tensor is filled with zeros when loaded, and left out when stored.
int encode_map(CUtensorMap* map, CUtensorMapDataType type, int width, const void* ptr, int rank, const cuuint64_t* dims, const cuuint64_t* strides, int rows) {
  static std::atomic<EncodeTiledFn> cached{nullptr};
  EncodeTiledFn fn = cached.load();
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found);
    if (e != cudaSuccess || found != cudaDriverEntryPointSuccess || !p) {
      dvm_note_cuda_error(e != cudaSuccess ? (int)e : (int)cudaErrorNotSupported);
      (void)cudaGetLastError();
      return DVM_ERR_CUDA;
    }
    fn = (EncodeTiledFn)p;
    cached.store(fn);
  }
  const cuuint32_t box[3] = {(cuuint32_t)(128 / width), (cuuint32_t)rows, 1}, one[3] = {1, 1, 1};
  if (fn(map, type, rank, const_cast<void*>(ptr), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
    dvm_note_cuda_error((int)cudaErrorInvalidValue);
    return DVM_ERR_CUDA;
  }
  return DVM_OK;
}
// (the stride of a dim of size 1 is never walked: any legal one)
inline cuuint64_t map_stride(int64_t size, int64_t stride) { return size > 1 ? (cuuint64_t)stride : 16; }
}  // namespace

extern "C" int dvm_last_scaled_matmul_tile(int* rows) {
  if (!rows || t_last_tile < 0) return DVM_ERR_INVALID_ARG;
  *rows = t_last_tile;
  return DVM_OK;
}

int dvm_launch_scaled_matmul(const dvm_scaled_matmul_desc& d, void* const* t, cudaStream_t stream) {
  using namespace dvm::scaled;
  const ScaledSlots s = dvm_slots(d);
  DvmDeviceInfo dev;
  int st = dvm_device_state(&dev);
  if (st != DVM_OK) return st;
  Args a = {};
  a.xs = (const float*)t[s.xs]; a.ws = (const float*)t[s.ws];
  a.starts = s.starts >= 0 ? (const int*)t[s.starts] : nullptr;
  a.out = t[s.out]; a.work = (uint8_t*)t[s.work]; a.status = dev.scratch;
  a.xs_stride = d.x_scales_stride; a.out_stride = d.out_stride;
  a.rows = (int)d.rows; a.n = (int)d.n; a.groups = (int)d.groups;
  a.k_blocks = (int)dvm_up(d.k, DVM_SCALE_BLOCK); a.n_blocks = (int)dvm_up(d.n, DVM_SCALE_BLOCK);
  a.out_bf16 = d.out_dtype == DVM_BF16;
  const int tile = dvm_scaled_tile(d), es = a.out_bf16 ? 2 : 4;
  const bool many = tile == DVM_SCALED_MANY;
  a.out_tma = (uintptr_t)a.out % 16 == 0 && (d.rows <= 1 || (d.out_stride * es % 16 == 0 && d.out_stride * es < (1ll << 40)));
  CUtensorMap x, w, out = {};
  const cuuint64_t xd[2] = {(cuuint64_t)d.k, (cuuint64_t)d.rows}, xt[1] = {map_stride(d.rows, d.x_stride)};
  const cuuint64_t wd[3] = {(cuuint64_t)d.k, (cuuint64_t)d.n, (cuuint64_t)d.groups}, wt[2] = {map_stride(d.n, d.w_stride[1]), map_stride(d.groups, d.w_stride[0])};
  const cuuint64_t od[2] = {(cuuint64_t)d.n, (cuuint64_t)d.rows}, ot[1] = {map_stride(d.rows, d.out_stride * es)};
  st = encode_map(&x, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, t[s.x], 2, xd, xt, many ? 128 : 16);
  if (st == DVM_OK) st = encode_map(&w, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, t[s.w], 3, wd, wt, many ? 256 : 128);
  if (st == DVM_OK && many && a.out_tma) st = encode_map(&out, a.out_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, es, a.out, 2, od, ot, 32);
  if (st == DVM_OK) st = many ? dvm_launch_scaled_many(x, w, out, a, dev.sm_count, dev.device, stream) : dvm_launch_scaled_few(x, w, a, tile, dev.device, stream);
  if (st == DVM_OK) t_last_tile = tile;
  return st;
}

int dvm_launch_experts(const uint32_t* w, void* const* tensors, int n_tensors, cudaStream_t stream) {
  const int nt = w[DVM_H_COUNTS] & 0xff;
  if (n_tensors != nt) return DVM_ERR_INVALID_ARG;
  if (w[DVM_H_N_TILES] == 0) return DVM_OK;
  int64_t need[DVM_MAX_TENSORS];
  dvm_extents_experts(w, need);
  for (int i = 0; i < nt; ++i)
    if (need[i] > 0 && !tensors[i]) return DVM_ERR_INVALID_ARG;
  const uint32_t type = w[DVM_H_KERNEL_TYPE];
  int may[2] = {-1, -1};   // an output that may be this input
  if (type == DVM_KERNEL_COMBINE) {
    dvm_combine_desc d;
    dvm_descriptor(w, &d);
    const CombineSlots s = dvm_slots(d);
    if (d.based && (d.tokens <= 1 || d.base_stride == d.out_stride)) { may[0] = s.base; may[1] = s.out; }
  }
  for (int i = (w[DVM_H_COUNTS] >> 8) & 0xff; i < nt; ++i)
    for (int j = 0; j < nt; ++j)
      if (i != j && need[i] > 0 && need[j] > 0 && tensors[i] == tensors[j] && !(j == may[0] && i == may[1])) return DVM_ERR_INVALID_ARG;
  auto aligned = [&](int slot, int bytes) { return slot < 0 || need[slot] <= 0 || ((uintptr_t)tensors[slot] & (bytes - 1)) == 0; };
  auto es = [](int dtype) { return dtype == DVM_BF16 ? 2 : 4; };
  if (type == DVM_KERNEL_ROUTING) {
    dvm_routing_desc d;
    dvm_descriptor(w, &d);
    const RoutingSlots s = dvm_slots(d);
    if (!aligned(s.logits, es(d.dtype)) || !aligned(s.bias, 4) || !aligned(s.positions, 4) || !aligned(s.ids, 4) || !aligned(s.weights, 4) || !aligned(s.places, 4) ||
        !aligned(s.starts, 4) || !aligned(s.ws, 16))
      return DVM_ERR_INVALID_ARG;
    return dvm_launch_routing(d, tensors, stream);
  }
  if (type == DVM_KERNEL_QUANTIZE) {
    dvm_quantize_desc d;
    dvm_descriptor(w, &d);
    const QuantizeSlots s = dvm_slots(d);
    if (!aligned(s.x, es(d.dtype)) || !aligned(s.places, 4) || !aligned(s.codes, 16) || !aligned(s.scales, 4)) return DVM_ERR_INVALID_ARG;
    return dvm_launch_quantize(d, tensors, stream);
  }
  if (type == DVM_KERNEL_SCALED_MATMUL) {
    dvm_scaled_matmul_desc d;
    dvm_descriptor(w, &d);
    const ScaledSlots s = dvm_slots(d);
    if (!aligned(s.x, 16) || !aligned(s.xs, 4) || !aligned(s.w, 16) || !aligned(s.ws, 4) || !aligned(s.starts, 4) || !aligned(s.out, es(d.out_dtype)) || !aligned(s.work, 16))
      return DVM_ERR_INVALID_ARG;
    return dvm_launch_scaled_matmul(d, tensors, stream);
  }
  dvm_combine_desc d;
  dvm_descriptor(w, &d);
  const CombineSlots s = dvm_slots(d);
  if (!aligned(s.y, es(d.dtype)) || !aligned(s.places, 4) || !aligned(s.weights, 4) || !aligned(s.base, es(d.dtype)) || !aligned(s.out, es(d.dtype)))
    return DVM_ERR_INVALID_ARG;
  return dvm_launch_combine(d, tensors, stream);
}
