// launch_recorder.hip with what the losses' kernels are given besides a product.
#include <hip/hip_runtime.h>

#define hipLaunchKernel launch_without_losses
#include "launch_recorder.hip"
#undef hipLaunchKernel

#include "loss_common.h"

SHOWN hipError_t hipLaunchKernel(const void* host, dim3 grid, dim3 block, void** args, size_t lds, hipStream_t stream) {
  launch_without_losses(host, grid, block, args, lds, stream);
  const std::string name = names()[host];
  auto is = [&](const char* part) { return name.find(part) != std::string::npos; };
  auto arg = [&](int i) { return *static_cast<const void* const*>(args[i]); };
  auto whole = [&](int i) { return (int64_t)*static_cast<const int*>(args[i]); };
  text.resize(text.size() - 2);                    // "}\n"
  if (is("loss_ring_kernel") || is("loss_wide_kernel")) {
    const linear::LossProduct& p = *static_cast<const linear::LossProduct*>(args[0]);
    put("row0", p.row0), put("sums", p.sums), put("at", p.at), put("lse", p.lse), put("w", p.w), put("dZ", p.dZ);
    put("lddz", p.lddz), put("db", p.db), put("k", (int64_t)p.y.k), put("bins", (int64_t)p.y.bins), put("bin", p.y.bin);
    put("index", p.y.index), put("weight", p.y.weight), put("counts", p.y.count), put("add", (int64_t)p.add);
  }
  if (is("join_loss_kernel")) put("parts", whole(0)), put("N", whole(1)), put("sums", arg(3)), put("at", arg(4));
  if (is("list_kernel")) {
    put("k", whole(1)), put("size", whole(2)), put("bins", whole(9)), put("sorted", arg(10)), put("weight", arg(11));
    put("bin", arg(12)), put("counts", arg(13));
  }
  if (is("column_kernel")) put("t", whole(0)), put("w", arg(6)), put("back", arg(7));
  if (is("input_kernel")) put("t", *static_cast<const int64_t*>(args[1])), put("w", arg(4)), put("to", arg(5)), put("ldto", *static_cast<const int64_t*>(args[6]));
  if (is("row_sum_kernel")) put("M", whole(0)), put("parts", whole(1)), put("part", arg(2));
  if (is("shared_loss_kernel") || is("shared_dz_kernel")) {
    const linear::LossProduct& p = *static_cast<const linear::LossProduct*>(args[0]);
    put("M", p.M), put("N", p.N), put("row0", p.row0), put("shares", p.shares), put("w", p.w), put("dZ", p.dZ), put("lddz", p.lddz);
    put("db", p.db), put("splits", whole(1));
  }
  if (is("ring_kernel") || is("wide_kernel")) put("adds", (int64_t)static_cast<const linear::Product*>(args[0])->add);
  text += "}\n";
  return hipSuccess;
}
