// Stand-in for the library's loads into LDS on the host CPU: each lane's part is there when the lane goes on, and everybody's when a wait is over.
#ifndef CKV_DMA_H_
#define CKV_DMA_H_

#include <hip/hip_runtime.h>

namespace ckv {

template <bool STREAM>
inline void dma_16(const char *from, char *lds) { memcpy(lds + 16 * emu::lane(), from, 16); }
inline void dma_4(const void *from, void *lds) { memcpy(static_cast<char *>(lds) + 4 * emu::lane(), from, 4); }
template <int N>
inline void wait_vm_at_most() {
  const char nothing = 0;
  emu::exchange(&nothing, 1);
}
inline void wait_lds_reads() { wait_vm_at_most<0>(); }

}  // namespace ckv
#endif
