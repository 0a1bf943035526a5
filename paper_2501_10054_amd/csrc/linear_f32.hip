// linear_kernel for x, W and b in fp32
#include "linear_tile.h"

tardis_status_t td_linear_init_f32() {
    static td_once once;
    return once.run([]() { return linear_init<float>(); });
}
void td_linear_launch_f32(const LinearArgs& p, bool grouped, bool direct, int shape, int blocks, hipStream_t s) {
    linear_launch<float>(p, grouped, direct, shape, blocks, s);
}
