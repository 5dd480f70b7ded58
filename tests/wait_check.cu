// A wait that runs out, for test_gpu_waits.py: one block whose second barrier nobody arrives on.
#include "../paper_2608_15762_gb300/csrc/gmgop_ptx.cuh"

using namespace gop;

// out: [0, 64) each thread's answer of its first wait (a lane of warp 0 waits on either barrier by
// turns, those of warp 1 on the completed one), [64, 128) whether a wait has given up, [128, 192)
// the answer of a second wait on the barrier that nobody arrives on, [192] and [193] lanes elected
// in the warps after it, [194] and [195] milliseconds of warp 0's waits.
__global__ void wait_kernel(int* out) {
  __shared__ uint64_t bars[2];
  __shared__ uint32_t failed_word;
  volatile uint32_t* failed = &failed_word;
  const int t = threadIdx.x, lane = t & 31;
  const uint32_t some = smem_addr(bars), none = some + 8;
  if (t == 0) {
    bar_init(some, 1), bar_init(none, 1);
    failed_word = 0;
    fence_bar_init();
  }
  __syncthreads();
  if (t == 0) bar_arrive(some);
  __syncthreads();
  uint64_t t0, t1, t2;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
  out[t] = bar_wait(t < 32 && lane % 2 ? none : some, 0, failed);
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t1));
  __syncthreads();
  out[64 + t] = gave_up(failed);
  out[128 + t] = t < 32 ? bar_wait(none, 0, failed) : bar_wait_both(some, 0, none, 0, failed);
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t2));
  if (elect_one()) atomicAdd(&out[192 + t / 32], 1);
  if (t == 0) out[194] = int((t1 - t0) / 1000000), out[195] = int((t2 - t1) / 1000000);
}

// Four warps that meet: out[0] counts words of another warp's that were not seen behind a meeting; then
// a meeting of five that a fifth never comes to: [1] gave up, [2] and [3] milliseconds of it and of
// 100 meetings after it.
__global__ void meet_kernel(int* out) {
  __shared__ uint64_t bars[2];
  __shared__ uint32_t failed_word;
  __shared__ int word[128];
  volatile uint32_t* failed = &failed_word;
  const int t = threadIdx.x;
  const uint32_t four = smem_addr(bars), five = four + 8;
  if (t == 0) {
    bar_init(four, 4), bar_init(five, 5);
    failed_word = 0;
    fence_bar_init();
  }
  __syncthreads();
  uint32_t phase = 0;
  for (int i = 1; i <= 1000; ++i) {
    word[t] = i * 128 + t;
    bar_meet(four, &phase, failed);
    const int other = (t * 37 + i) & 127;
    if (word[other] != i * 128 + other) atomicAdd(&out[0], 1);
    bar_meet(four, &phase, failed);
  }
  if (gave_up(failed)) atomicAdd(&out[0], 1);
  uint64_t t0, t1, t2;
  phase = 0;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
  bar_meet(five, &phase, failed);
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t1));
  for (int i = 0; i < 100; ++i) bar_meet(five, &phase, failed);
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t2));
  const bool gone = gave_up(failed);
  if (t == 0) out[1] = gone, out[2] = int((t1 - t0) / 1000000), out[3] = int((t2 - t1) / 1000000);
}

extern "C" int wait_check(int which, int* host) {
  int* out;
  if (cudaMalloc(&out, 196 * sizeof(int)) != cudaSuccess) return -1;
  cudaMemset(out, 0, 196 * sizeof(int));
  if (which == 0) wait_kernel<<<1, 64>>>(out);
  else meet_kernel<<<1, 128>>>(out);
  const cudaError_t e = cudaMemcpy(host, out, 196 * sizeof(int), cudaMemcpyDeviceToHost);
  cudaFree(out);
  return e == cudaSuccess ? 0 : -2;
}
