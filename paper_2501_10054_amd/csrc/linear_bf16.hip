// linear_kernel for x, W and b in bf16
#include "linear_tile.h"

tardis_status_t td_linear_init_bf16() {
    static td_once once;
    return once.run([]() { return linear_init<bf16_t>(); });
}
void td_linear_launch_bf16(const LinearArgs& p, bool grouped, bool direct, int shape, int blocks, hipStream_t s) {
    linear_launch<bf16_t>(p, grouped, direct, shape, blocks, s);
}
