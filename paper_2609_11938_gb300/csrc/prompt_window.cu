// prompt_window.cu -- the kernels of prompt.cuh through a window.
#include "prompt.cuh"

namespace opattr {

opattr_status prompt_window(Ctx &c, Serve &s, PromptArgs &p, const Maps<true> &m) {
    return p.a.dtype == OPATTR_BF16 ? prompt_of<__nv_bfloat16, true>(c, s, p, m) : prompt_of<__half, true>(c, s, p, m);
}

}  // namespace opattr
