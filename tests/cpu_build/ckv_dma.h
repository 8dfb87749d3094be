// Stand-in for the library's loads into LDS on the host CPU: what they overwrite is gone when they are issued, what they bring is there when
// they have been waited for, and no lane ends before.
#ifndef CKV_DMA_H_
#define CKV_DMA_H_

#include <hip/hip_runtime.h>

namespace ckv {

template <bool STREAM>
inline void dma_16(const char *from, char *lds) { emu::load_later(lds + 16 * emu::lane(), from, 16); }
inline void dma_4(const void *from, void *lds) { emu::load_later(static_cast<char *>(lds) + 4 * emu::lane(), from, 4); }
template <int N>
inline void wait_vm_at_most() { emu::loads_at_most(N); }
inline void wait_lds_reads() {
  const char nothing = 0;
  emu::exchange(&nothing, 1);
}

}  // namespace ckv
#endif
