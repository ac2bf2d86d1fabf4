// Message of the last failed call, on this thread, of an entry point that takes no context.
#pragma once

namespace pt {
const char* ops_last_error();
}
