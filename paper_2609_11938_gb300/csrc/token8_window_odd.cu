// token8_window_odd.cu -- the kernel of token.cuh for the same pages, through a window.
#include "token.cuh"

namespace opattr {

opattr_status token8_window_odd(Ctx &c, Serve &s, TokenArgs &p, int dtype) {
    return token_of<true, true, false>(c, s, p, dtype);
}

}  // namespace opattr
