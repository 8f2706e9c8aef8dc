// token8.cu -- the kernel of token.cuh for pages of 8 bits.
#include "token.cuh"

namespace opattr {

opattr_status token8_plain(Ctx &c, Serve &s, TokenArgs &p, int dtype) {
    return token_of<true, false, true>(c, s, p, dtype);
}

}  // namespace opattr
