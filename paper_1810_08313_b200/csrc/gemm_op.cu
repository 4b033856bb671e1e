// Host side of the tensor-core product of gemm_op.cuh that does not depend on its template arguments.
#include "gemm_op.cuh"

namespace ls {
namespace gop {
namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult qr;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qr) != cudaSuccess ||
        qr != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

__device__ int g_op_error;               // zero when the library is loaded
int* g_error_addr[64] = {nullptr};       // its address on every device, looked up once

}  // namespace

int* device_error_word() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  if (g_error_addr[dev] == nullptr) {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_op_error) != cudaSuccess) return nullptr;
    g_error_addr[dev] = static_cast<int*>(p);
  }
  return g_error_addr[dev];
}

static int make_map(CUtensorMap* out, const void* base, MapType type, int64_t rows, int64_t cols, int64_t planes, int64_t ld,
                    int64_t plane, int row_bytes, int box_rows, bool swizzled) {
  EncodeTiledFn fn = encode_fn();
  if (fn == nullptr) return cudaErrorNotSupported;
  const int64_t eb = type == MAP_F32 ? 4 : 2;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)(ld * eb), (cuuint64_t)(plane * eb)};
  cuuint32_t box[3] = {(cuuint32_t)(row_bytes / eb), (cuuint32_t)box_rows, 1};
  cuuint32_t es[3] = {1, 1, 1};
  const CUtensorMapDataType dt = type == MAP_F32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                 : type == MAP_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                   : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  const CUtensorMapSwizzle sw = !swizzled          ? CU_TENSOR_MAP_SWIZZLE_NONE
                                : row_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B
                                                   : CU_TENSOR_MAP_SWIZZLE_64B;
  CUresult r = fn(out, dt, 3, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, sw,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}
int make_operand_map(CUtensorMap* out, const void* base, MapType type, int64_t rows, int64_t cols, int64_t planes, int64_t ld,
                     int64_t plane, int box_rows) {
  return make_map(out, base, type, rows, cols, planes, ld, plane, 128, box_rows, true);
}
int make_output_map(CUtensorMap* out, void* base, MapType type, int64_t rows, int64_t cols, int64_t planes, int64_t ld,
                    int64_t plane, int row_bytes, bool transposed) {
  return make_map(out, base, type, rows, cols, planes, ld, plane, row_bytes, 32, !transposed);
}

}  // namespace gop
}  // namespace ls

extern "C" int ls_device_status(void* cuda_stream) {
  int* word = ls::gop::device_error_word();
  if (word == nullptr) return LS_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  int code = 0;
  if (cudaMemcpyAsync(&code, word, sizeof(int), cudaMemcpyDeviceToHost, st) != cudaSuccess) return LS_ERR_CUDA;
  if (cudaStreamSynchronize(st) != cudaSuccess) return LS_ERR_CUDA;
  if (code == 0) return LS_OK;
  if (cudaMemsetAsync(word, 0, sizeof(int), st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
    return LS_ERR_CUDA;
  return LS_ERR_DEVICE_TIMEOUT;
}
