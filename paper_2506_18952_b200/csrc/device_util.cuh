// device_util.cuh - what the kernels of both translation units need (inside their anonymous namespaces).

// Programmatic dependent launch: the grid may have been started while the kernel before it in the stream was still
// running.  grid_dependency_wait returns once that kernel has completed and its writes are visible; it must precede
// every global-memory access of the calling thread that could touch what that kernel reads or writes.
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_dependency_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

__device__ __forceinline__ float max3_nan(float a, float b, float c) {     // NaN where one of them is
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

__device__ __forceinline__ float warp_max_f32(float x) {       // (of numbers; -inf among them)
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));       // (volatile: whole warps, stays where it is)
  return r;
}
