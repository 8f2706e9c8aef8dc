// token_window.cu -- the kernel of token.cuh for pages of 16 bits, through a window.
#include "token.cuh"

namespace opattr {

opattr_status token_window(Ctx &c, Serve &s, TokenArgs &p, int dtype) {
    return dtype == OPATTR_BF16 ? token_of<__nv_bfloat16, false, true>(c, s, p) : token_of<__half, false, true>(c, s, p);
}

}  // namespace opattr
