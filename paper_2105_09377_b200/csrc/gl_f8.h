// Declarations of the 8-bit operators that other translation units use.
#pragma once

namespace gl {
// Device status word of gl_f8.cu: reads and clears, GL_ERR_TIMEOUT when one was raised.
int take_status_f8();
}  // namespace gl
