// token8_window.cu -- the kernel of token.cuh for pages of 8 bits, through a window.
#include "token.cuh"

namespace opattr {

opattr_status token8_window(Ctx &c, Serve &s, TokenArgs &p, int dtype) {
    return token_of<true, true, true>(c, s, p, dtype);
}

}  // namespace opattr
