// Host helpers shared by the translation units of the C ABI (defined in solo_api.cu).
#pragma once

namespace solo {

int sm_count(int device);      // multiprocessors of a device (cached)
void count_launch();           // one more kernel launch for solo_launch_count

}  // namespace solo
