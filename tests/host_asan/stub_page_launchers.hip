// Stand-ins for the launchers that sa_pages_api.hip calls: each counts a launch.
#include "../../paper_2608_15522_amd/csrc/sa_device.h"
#include "../../paper_2608_15522_amd/csrc/sa_internal.h"

int sa_stub_page_launches = 0;

namespace sa {
void launch_pages_reserve(int32_t*, int32_t*, int32_t*, const int32_t*, int, int, int, int,
                          int32_t*, hipStream_t) {
  ++sa_stub_page_launches;
}
void launch_pages_fork(int32_t*, int32_t*, int32_t*, const int32_t*, const int32_t*, int, int, int,
                       int, int, int32_t*, int32_t*, int32_t*, hipStream_t) {
  ++sa_stub_page_launches;
}
void launch_pages_free(int32_t*, int32_t*, int32_t*, const int32_t*, int, int, int, int, int,
                       hipStream_t) {
  ++sa_stub_page_launches;
}
void launch_pages_compact(int32_t*, int32_t*, int, int, int, int32_t*, int32_t*, int32_t*,
                          hipStream_t) {
  ++sa_stub_page_launches;
}
void launch_pages_copy(void*, int, int, size_t, const int32_t*, const int32_t*, int, hipStream_t) {
  ++sa_stub_page_launches;
}
void launch_pages_write(const void*, const void*, void*, void*, const int32_t*, const int32_t*,
                        const int32_t*, const int32_t*, int, int, int, int, int, int, int,
                        hipStream_t) {
  ++sa_stub_page_launches;
}
void launch_prefix_attention(const PrefixCall&, int, int, char*, hipStream_t) {
  ++sa_stub_page_launches;
}
}  // namespace sa
