// register_check.h -- whether a kernel whose warps hand registers on with
// setmaxnreg was compiled with as many as they will hold: an increase beyond a
// block's own would wait for ever.  Host code without a CUDA call of its own.
#pragma once

#include <atomic>

#include <cuda_runtime_api.h>

namespace puro {

class RegisterCheck {
  public:
    // cudaSuccess where `warps` warps of the registers a thread that query(int *)
    // reports hold at least `need` (the sum over the warps), else
    // cudaErrorLaunchOutOfResources.  A device is asked until a query has
    // succeeded, whose error is returned otherwise.
    template <class Query>
    cudaError_t enough(int device, int warps, int need, Query query) {
        const bool keep = device >= 0 && device < kDevices;
        int regs = keep ? regs_[device].load(std::memory_order_relaxed) : 0;
        if (regs == 0) {
            const cudaError_t e = query(&regs);
            if (e != cudaSuccess) return e;
            if (keep) regs_[device].store(regs, std::memory_order_relaxed);
        }
        return regs * warps >= need ? cudaSuccess : cudaErrorLaunchOutOfResources;
    }

  private:
    static constexpr int kDevices = 64;
    std::atomic<int> regs_[kDevices] = {};  // registers a thread, 0: not known yet
};

}  // namespace puro
