// token8_odd.cu -- the kernel of token.cuh for pages of 8 bits whose heads are neither 64 nor 128 wide.
#include "token.cuh"

namespace opattr {

opattr_status token8_plain_odd(Ctx &c, Serve &s, TokenArgs &p, int dtype) {
    return token_of<true, false, false>(c, s, p, dtype);
}

}  // namespace opattr
