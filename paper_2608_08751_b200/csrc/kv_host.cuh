// What the translation units of the library share on the host: the error text, the device's context, the launch counter and
// the tensor map of a cache.  Defined beside the entry points of ivf_api.cu.
#pragma once
#include <cuda.h>
#include <stdint.h>

#include "kv_common.cuh"

namespace ivf {

#define IVF_INTERNAL __attribute__((visibility("hidden")))

struct KvHostCtx {
    int index;  // of the current device
    int num_sms;
    int* status;
    uint64_t limit_ns;  // of a device-side wait
};

IVF_INTERNAL int kv_host_fail(int code, const char* text);
IVF_INTERNAL int kv_host_ctx(KvHostCtx* out);
IVF_INTERNAL void kv_host_launched();
// A page of one head (64 tokens of it at most), 64 columns wide, with the 128-byte swizzle.  False where the cache's layout has no map.
IVF_INTERNAL bool kv_host_map(CUtensorMap* map, const KvPlane& c, int dim, int page, int n_kv_heads, int64_t num_pages, bool bf16);

}  // namespace ivf
