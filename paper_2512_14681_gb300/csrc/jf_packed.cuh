// What the kernels of packed attention and its backward pass share (jf_ops.h: jf_packed).
#pragma once
#include "../../include/jf_ops.h"
#include "jf_device.cuh"
#include "jf_internal.h"

namespace jf {

constexpr int kPackedMaxSeqs = 1024, kPackedMaxGroup = 128;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

// A call's arguments. Rows of q, k, v, d_out, dq, dk, dv lie ld_* elements apart, those of out and lse side by side.
struct PackedParams {
  jf_packed t;
  const void *q, *k, *v;
  long long ld_q, ld_k, ld_v;
  int Hq, Hkv;
  float scale;
  void* out;         // forward: written, backward: read
  float* lse;        // (forward: may be null)
  const void* d_out;
  void *dq, *dk, *dv;
  long long ld_do, ld_dq, ld_dk, ld_dv;
  float* delta;      // [n_rows][Hq]: sum of d_out * out
  int* cuts;         // where CTAs' runs begin (null: no unit is shared by several)
  float* states;     // partial results of units that several CTAs share
  int* err;
};

// 2^x by the MUFU ex2 instruction (flushes results below 2^-126 to zero; 2^-inf = 0).
JF_DEV float packed_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Whether the texts lie one behind the other within the rows, none longer than max_rows. One that does not leaves the
// whole call undone: its rows could be another's.
JF_DEV bool packed_text_ok(const jf_packed& t, int b) {
  const int s0 = t.row_start[b], s1 = t.row_start[b + 1];
  return s0 >= 0 && s1 >= s0 && s1 <= t.n_rows && s1 - s0 <= t.max_rows;
}

// The tensor-core form (jf_packed_tc.cu): whether its copies can read a call's rows, its workspace, its launches.
bool packed_tc_rows(const void* p, long long ld);
jf_status packed_tc_workspace(const jf_packed& t, int Hq, int Hkv, int hd, bool backward, size_t* out_bytes);
jf_status packed_tc_forward(const PackedParams& a, int hd, void* workspace, cudaStream_t st);
jf_status packed_tc_backward(const PackedParams& a, int hd, void* workspace, cudaStream_t st);

// cluster: CTAs of one, along x.
template <typename K, typename... Args>
cudaError_t packed_launch_clusters(K kernel, int cluster, dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)cluster, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <typename K, typename... Args>
cudaError_t packed_launch(K kernel, dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
  return packed_launch_clusters(kernel, 1, grid, block, smem, st, args...);
}

}  // namespace jf
