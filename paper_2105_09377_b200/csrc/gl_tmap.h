// Host side of the TMA unit, shared by the kernel files: driver entry points, cached tensor maps, device facts.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <mutex>
#include <string>
#include <unordered_map>

namespace gl {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
typedef CUresult (*EncodeIm2colFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const int*, const int*, cuuint32_t, cuuint32_t,
                                   const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct DriverApi {
  EncodeTiledFn tiled = nullptr;
  EncodeIm2colFn im2col = nullptr;
  bool ok = false;
};

inline const DriverApi& driver_api() {
  static DriverApi api;
  static std::once_flag once;
  std::call_once(once, [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || !f) return;
    api.tiled = reinterpret_cast<EncodeTiledFn>(f);
    f = nullptr;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeIm2col", &f, cudaEnableDefault, &q) != cudaSuccess || !f) return;
    api.im2col = reinterpret_cast<EncodeIm2colFn>(f);
    api.ok = true;
  });
  return api;
}

// Encoded tensor maps, kept per argument list (base address, extents, strides, box, modes).  A program that
// calls the library on the same buffers again - every layer of a network on every step - skips the driver's
// encoding, which costs more host time than the rest of a call.  The map depends on nothing but its arguments,
// so a recycled address with the same geometry yields the same, still valid, map.
class TensorMapCache {
 public:
  template <typename Encode>
  bool get(const std::string& key, CUtensorMap* out, Encode&& encode) {
    {
      std::lock_guard<std::mutex> lock(mu_);
      auto it = maps_.find(key);
      if (it != maps_.end()) { *out = it->second; return true; }
    }
    if (!encode(out)) return false;
    std::lock_guard<std::mutex> lock(mu_);
    if (maps_.size() >= kMaxEntries) maps_.clear();
    maps_.emplace(key, *out);
    return true;
  }

 private:
  static constexpr size_t kMaxEntries = 4096;
  std::mutex mu_;
  std::unordered_map<std::string, CUtensorMap> maps_;
};

inline TensorMapCache& map_cache() {
  static TensorMapCache cache;
  return cache;
}

template <typename T>
inline void key_add(std::string* key, const T* v, size_t n) { key->append(reinterpret_cast<const char*>(v), n * sizeof(T)); }

inline bool encode_tiled_cached(CUtensorMap* m, CUtensorMapDataType dt, cuuint32_t rank, const void* base, const cuuint64_t* dims,
                         const cuuint64_t* strides, const cuuint32_t* box, const cuuint32_t* estr, CUtensorMapSwizzle swz,
                         CUtensorMapL2promotion l2) {
  std::string key;
  key.reserve(160);
  const uint32_t head[4] = {0u, static_cast<uint32_t>(dt), rank, static_cast<uint32_t>(swz) | (static_cast<uint32_t>(l2) << 8)};
  key_add(&key, head, 4);
  key_add(&key, &base, 1);
  key_add(&key, dims, rank);
  key_add(&key, strides, rank - 1);
  key_add(&key, box, rank);
  key_add(&key, estr, rank);
  return map_cache().get(key, m, [&](CUtensorMap* out) {
    return driver_api().tiled(out, dt, rank, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swz,
                              l2, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  });
}

inline bool encode_im2col_cached(CUtensorMap* m, const void* base, const cuuint64_t* dims, const cuuint64_t* strides, const int* lower,
                          const int* upper, cuuint32_t channels, cuuint32_t pixels, const cuuint32_t* estr,
                          CUtensorMapSwizzle swz) {
  std::string key;
  key.reserve(160);
  const uint32_t head[4] = {1u, channels, pixels, static_cast<uint32_t>(swz)};
  key_add(&key, head, 4);
  key_add(&key, &base, 1);
  key_add(&key, dims, 4);
  key_add(&key, strides, 3);
  key_add(&key, lower, 2);
  key_add(&key, upper, 2);
  key_add(&key, estr, 4);
  return map_cache().get(key, m, [&](CUtensorMap* out) {
    return driver_api().im2col(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, lower, upper,
                               channels, pixels, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swz, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  });
}

inline int num_sms() {
  static int sms[64] = {0};   // per device
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  if (!sms[dev]) cudaDeviceGetAttribute(&sms[dev], cudaDevAttrMultiProcessorCount, dev);
  return sms[dev] > 0 ? sms[dev] : 148;
}

}  // namespace gl
